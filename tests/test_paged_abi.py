"""What the calls over a paged cache refuse, on the host, before anything is launched."""
import pytest

from paper_2506_19645_amd import binding as B

FAKE = 0x1000


def _desc(**kw):
    base = dict(T=2, batch=3, n_heads=8, n_kv_heads=4, rows=10, max_new=4, page_size=16, n_pages=7, max_pages=5)
    base.update(kw)
    return B.paged_desc(**base)


class Workspace:      # stands in for a device buffer: the call ends before anything is read
    is_cuda = True
    def __init__(self, n, at=FAKE): self.n, self.at = n, at
    def numel(self): return self.n
    def element_size(self): return 1
    def is_contiguous(self): return True
    def data_ptr(self): return self.at


def append(d, qkv=FAKE, q=2 * FAKE, row_start=FAKE, lens=FAKE, table=FAKE, k=FAKE, v=FAKE, ks=None, vs=None):
    return B.paged_append(d, qkv, q, row_start, lens, table, k, v, ks, vs, stream=0, check=False)


def attend(d, q=FAKE, out=FAKE, row_start=FAKE, lens=FAKE, table=FAKE, k=FAKE, v=FAKE, ks=None, vs=None, ws=Workspace(1 << 40)):
    return B.paged_attn(d, q, out, row_start, lens, table, k, v, ws, ks, vs, stream=0, check=False)


@pytest.mark.parametrize("field,value,status", [
    ("T", 0, B.EINVAL), ("batch", 0, B.EINVAL), ("rows", -1, B.EINVAL), ("n_pages", -1, B.EINVAL), ("max_new", 0, B.EINVAL),
    ("cache_type", 2, B.EINVAL), ("cache_type", -1, B.EINVAL), ("n_heads", 0, B.EINVAL), ("n_kv_heads", -1, B.EINVAL),
    ("max_pages", 0, B.EINVAL), ("page_size", 0, B.EINVAL), ("head_dim", 0, B.EINVAL),
    ("T", 3, B.ESHAPE), ("n_kv_heads", 3, B.ESHAPE), ("n_kv_heads", 1, B.ESHAPE), ("head_dim", 64, B.EUNSUPPORTED),
    ("page_size", 8, B.ESHAPE), ("page_size", 24, B.ESHAPE), ("n_pages", 1 << 31, B.ESHAPE), ("rows", 1 << 31, B.ESHAPE), ("rows", (1 << 23) + 1, B.ESHAPE), ("batch", 1 << 21, B.ESHAPE),
    ("max_pages", 1 << 28, B.ESHAPE), ("n_heads", 1 << 20, B.ESHAPE),
    ("ld_q", 4 * 128 - 8, B.ESHAPE), ("ld_q", 4 * 128 + 4, B.ESHAPE), ("ld_qkv", 4 * 128, B.ESHAPE), ("ld_qkv", 8 * 128 + 1, B.ESHAPE),
    ("strides", (1 << 20, 1 << 12, 2048, 120), B.ESHAPE), ("strides", (1 << 20, 1 << 12, 2048, 64), B.ESHAPE),
    ("strides", (1 << 20, 1 << 12, 2047, 128), B.ESHAPE), ("strides", (1 << 20, -4096, 2048, 128), B.ESHAPE),
    ("strides", (1 << 40, 1 << 12, 1 << 35, 1 << 27), B.ESHAPE),
])
def test_descriptors_that_are_refused(field, value, status):
    d = _desc(**{field: value})
    assert append(d) == status and attend(d) == status
    assert B.paged_attn_workspace_bytes(d) == 0


def test_arguments_that_are_refused():
    d, e = _desc(), _desc(cache_type=B.CACHE_E4M3)
    for call, names in ((append, ("qkv", "q", "lens", "table", "k", "v")), (attend, ("q", "out", "lens", "table", "k", "v"))):
        for n in names:
            assert call(d, **{n: None}) == B.EINVAL
            assert call(d, **{n: 2 * FAKE + (2 if n in ("lens", "table") else 8)}) == B.EALIGN
        assert call(d, row_start=FAKE + 2) == B.EALIGN
        assert call(d, ks=FAKE) == B.EINVAL and call(d, vs=FAKE) == B.EINVAL        # a bf16 cache has no scales
        assert call(e, ks=FAKE + 2) == B.EALIGN and call(e, vs=FAKE + 1) == B.EALIGN
        assert call(_desc(rows=2), row_start=None) == B.ESHAPE                      # a row for every sequence
    for base in (0.0, -1.0, float("nan")):
        assert append(_desc(rope_base=base)) == B.EINVAL
    assert append(d, qkv=FAKE, q=FAKE) == B.ESHAPE                                  # in place only with the same row stride
    assert B.paged_append(d, FAKE, FAKE * 2, None, None, None, FAKE, FAKE, stream=0, check=False) in (B.EINVAL, B.ESHAPE)
    with pytest.raises(B.CaatError):
        B.paged_append(_desc(T=0), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, stream=0)
    with pytest.raises(B.CaatError):
        B.paged_attn(_desc(T=0), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, stream=0)


def test_layer_arguments_that_are_refused():
    from paper_2506_19645_amd import inputs as I
    cfg = I.BlockConfig("dec", I.KIND_DECODE, I.NORM_RMSNORM, h=1024, T=2, p=0.5, batch=10, seq=1, ffn=512, n_heads=8, head_dim=128,
                        n_kv_heads=4)
    call = lambda d, pg, ws=Workspace(1 << 40), w=[FAKE] * 6, r=FAKE, lens=FAKE, k=FAKE, ks=None: B.paged_layer_fwd(
        d, pg, w, r, FAKE, FAKE, lens, FAKE, k, FAKE, ws, ks, None, stream=0, check=False)
    good = B.make_desc(cfg)
    size = B.paged_layer_workspace_bytes(good, _desc())
    assert size >= B.workspace_bytes(good) + B.paged_attn_workspace_bytes(_desc())
    assert call(good, _desc(), ws=Workspace(size - 1)) == B.EWORKSPACE and call(good, _desc(), ws=None) == B.EINVAL
    for field, value, status in (("T", 1, B.ESHAPE), ("n_heads", 16, B.ESHAPE), ("n_kv_heads", 8, B.ESHAPE), ("rows", 11, B.ESHAPE),
                                 ("ld_q", 1024, B.ESHAPE), ("ld_qkv", 2048, B.ESHAPE), ("rope_base", 500.0, B.EINVAL),
                                 ("page_size", 8, B.ESHAPE), ("cache_type", 3, B.EINVAL)):
        assert call(good, _desc(**{field: value})) == status
    prefill = B.make_desc(cfg.with_(kind=I.KIND_PREFILL, batch=2, seq=5))
    assert call(prefill, _desc()) == B.EINVAL and B.paged_layer_workspace_bytes(prefill, _desc()) == 0
    assert B.paged_layer_workspace_bytes(good, _desc(T=0)) == 0
    assert call(good, _desc(), lens=None) == B.EINVAL and call(good, _desc(), r=None) == B.EINVAL
    assert call(good, _desc(), k=None) == B.EINVAL and call(good, _desc(), k=FAKE + 8) == B.EALIGN
    assert call(good, _desc(), ks=FAKE) == B.EINVAL and call(good, _desc(), w=[FAKE] * 5 + [None]) == B.EINVAL
    norm = B.make_desc(cfg)
    norm.norm = B.LAYERNORM
    assert call(norm, _desc()) == B.EUNSUPPORTED
    with pytest.raises(B.CaatError):
        B.paged_layer_fwd(prefill, _desc(), [FAKE] * 6, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, stream=0)
