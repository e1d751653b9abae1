"""Sizes and arguments of the calls over a paged cache, on the host."""
import pytest
import torch

from paper_2506_19645_amd import binding as B


@pytest.mark.parametrize("T,heads,kv", [(8, 32, 32), (8, 64, 8), (4, 32, 8), (1, 40, 1), (1, 8, 8), (2, 6, 2)])
def test_one_workspace_serves_smaller_batches(T, heads, kv):
    """Sized for the most new tokens, whatever the rows, the sequences and the table: no call with fewer of any is refused."""
    last = 0
    for max_new in (1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 500, 2048, 8192):
        sizes = {B.paged_attn_workspace_bytes(B.paged_desc(T=T, batch=batch, n_heads=heads, n_kv_heads=kv, rows=rows, max_new=max_new,
                                                           page_size=16, n_pages=1 << 20, max_pages=columns, cache_type=cache))
                 for batch in (1, 3, 64, 1000) for rows in (1, 8, 100, 1536, 4096, 20000) for columns in (1, 64, 8192)
                 for cache in (B.CACHE_BF16, B.CACHE_E4M3)}
        assert len(sizes) == 1
        size = sizes.pop()
        assert size >= last and size > 0
        last = size


class Tensor:
    """What the binding looks at of a device tensor."""
    is_cuda = True
    def __init__(self, itemsize=2, floating=True, shape=(2, 3, 128), strides=None, at=0x1000):
        self.itemsize, self.floating, self.shape, self.strides, self.at = itemsize, floating, shape, strides, at
        self.dtype = {1: torch.uint8, 2: torch.bfloat16 if floating else torch.int16, 4: torch.float32 if floating else torch.int32,
                      8: torch.float64 if floating else torch.int64}[itemsize]
    def element_size(self): return self.itemsize
    def is_floating_point(self): return self.floating
    def is_contiguous(self): return self.strides is None
    def dim(self): return len(self.shape)
    def stride(self): return self.strides
    def data_ptr(self): return self.at
    def numel(self): return 1 << 40


INT, FP32 = Tensor(4, False), Tensor(4)
GOOD = dict(q=Tensor(), out=Tensor(), row_start=INT, lens=INT, table=INT, k=Tensor(), v=Tensor(), ks=None, vs=None)
POOL, STRIDES = (2, 7, 4, 16, 128), (7 * 2 * 8192, 2 * 8192, 2048, 128)     # keys and values of a page one after the other


def calls(desc, **kw):
    """The three entry points with a descriptor that the library refuses: EINVAL says that the binding let the tensors through."""
    a = dict(GOOD, **kw)
    lists, ws = (a["row_start"], a["lens"], a["table"], a["k"], a["v"]), Tensor(1)
    yield lambda: B.paged_append(desc, a["q"], a["out"], *lists, a["ks"], a["vs"], stream=0, check=False)
    yield lambda: B.paged_attn(desc, a["q"], a["out"], *lists, ws, a["ks"], a["vs"], stream=0, check=False)
    yield lambda: B.paged_layer_fwd(B.caat_desc(kind=B.ATTN_DECODE), desc, [Tensor()] * 6, Tensor(), Tensor(), *lists, ws, a["ks"], a["vs"],
                                    stream=0, check=False)


def _refusing(e4m3=False, **kw):
    return B.paged_desc(**dict(dict(T=2, batch=0, n_heads=8, n_kv_heads=8, rows=3, page_size=16, n_pages=7, max_pages=1, strides=STRIDES,
                                    cache_type=B.CACHE_E4M3 if e4m3 else B.CACHE_BF16), **kw))


@pytest.mark.parametrize("e4m3", [False, True])
def test_views_of_a_pool_are_taken(e4m3):
    """Keys and values interleaved in one allocation, and queries inside wider rows, are what the descriptor's strides are for."""
    k, v = (Tensor(1 if e4m3 else 2, shape=POOL, strides=STRIDES + (1,)) for _ in range(2))
    for call in calls(_refusing(e4m3), k=k, v=v, ks=FP32 if e4m3 else None, row_start=None):
        assert call() == B.EINVAL
    q = Tensor(shape=(2, 3, 512), strides=(3 * 1536, 1536, 1))
    append, attend, _ = calls(_refusing(ld_q=1536, ld_qkv=1536), q=q)
    assert append() == B.EINVAL and attend() == B.EINVAL


@pytest.mark.parametrize("name,bad", [
    ("row_start", Tensor(8, False)), ("lens", Tensor(8, False)), ("table", Tensor(8, False)), ("lens", FP32), ("table", Tensor(2, False)),
    ("table", Tensor(4, False, (2, 3), (7, 1))), ("ks", Tensor(2)), ("vs", Tensor(8)), ("ks", INT), ("k", Tensor(4)), ("v", Tensor(1)),
    ("k", Tensor(shape=POOL, strides=STRIDES + (2,))), ("v", Tensor(shape=POOL, strides=STRIDES[:3] + (256, 1))),
    ("v", Tensor(shape=POOL[1:], strides=STRIDES[1:] + (1,)))])
def test_tensors_of_the_wrong_kind_are_refused(name, bad):
    for call in calls(_refusing(), **{name: bad}):
        with pytest.raises(ValueError):
            call()


def test_a_cache_of_the_other_type_is_refused():
    """Codes where the descriptor says bf16 would be read past their end."""
    for e4m3, cache in ((False, Tensor(1)), (True, Tensor(2))):
        for name in "kv":
            for call in calls(_refusing(e4m3), **dict({"k": Tensor(1 if e4m3 else 2), "v": Tensor(1 if e4m3 else 2)}, **{name: cache})):
                with pytest.raises(ValueError):
                    call()


@pytest.mark.parametrize("bad", [Tensor(4), Tensor(shape=(2, 3, 512), strides=(3 * 1536, 1536, 2)),
                                 Tensor(shape=(2, 3, 512), strides=(3 * 1024, 1024, 1)), Tensor(shape=(3, 2, 512), strides=(1536, 3 * 1536, 1))])
def test_rows_that_the_descriptor_does_not_describe_are_refused(bad):
    append, attend, _ = calls(_refusing(ld_q=1536, ld_qkv=1536), q=bad)
    for call in (append, attend):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("there", [False, True])
def test_the_current_stream_with_and_without_torchs_shortcut(monkeypatch, there):
    """The shortcut to the stream's handle is no public name of torch: without it the public one serves."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: type("Stream", (), {"cuda_stream": 77}))
    if there:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 50 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert B._stream(None) == (53 if there else 77) and B._stream(5) == 5


@pytest.mark.parametrize("T,heads,kv", [(2, 8, 8), (8, 64, 8)])
def test_one_workspace_serves_smaller_batches_of_the_layer(T, heads, kv):
    """The layer's size never falls when rows or new tokens grow."""
    from paper_2506_19645_amd import inputs as I
    for max_new in (1, 5, 300):
        last = 0
        for rows in (1, 2, 7, 64, 65, 100, 512, 1536, 4096, 20000):
            cfg = I.BlockConfig("dec", I.KIND_DECODE, I.NORM_RMSNORM, h=1024, T=T, p=0.5, batch=rows, seq=1, ffn=1024, n_heads=heads,
                                head_dim=128, n_kv_heads=kv)
            pages = B.paged_desc(T=T, batch=3, n_heads=heads, n_kv_heads=kv, rows=rows, max_new=max_new, page_size=16, n_pages=99,
                                 max_pages=50)
            size = B.paged_layer_workspace_bytes(B.make_desc(cfg), pages)
            assert size >= last and size > 0
            last = size
