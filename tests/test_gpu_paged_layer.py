"""Append and attention over a paged cache as they are used: in the decoder layer, in captured graphs, on other streams, in pools
of more than 4 GiB."""
import numpy as np
import pytest

from oracle import caat_oracle as O
from paper_2506_19645_amd import binding as B
from paper_2506_19645_amd import inputs as I
from tests import paged_util as P
from tests.util import assert_close, bits_to_f64, hs_of, make_inputs

pytestmark = pytest.mark.gpu


def _layer_weights(d):
    return [B.to_device(d["gamma_attn"]), B.to_device(d["Wqkv"]), B.to_device(d["Wo"]), B.to_device(d["gamma"]),
            B.to_device(np.concatenate([d["Wg"], d["Wu"]], axis=1)), B.to_device(d["B"])]


def _descs(cfg, c, **kw):
    desc = B.make_desc(cfg.with_(kind=I.KIND_DECODE, batch=c.rows, seq=1, kv_len=0), **kw)
    return desc, c.desc


@pytest.mark.parametrize("T,heads,kv,ffn,page,p,e4m3,steps", [
    (2, 4, 4, 2 * 256, 16, 0.5, False, [[37, 20, 0], [1, 1, 50], [1, 1, 1], [0, 3, 1]]),
    (2, 8, 2, 2 * 344, 32, 0.3, False, [[5, 130, 1], [1, 1, 1], [70, 2, 0]]),
    (4, 8, 8, 4 * 128, 48, 1.0, False, [[1, 1, 1], [1, 1, 1], [1, 1, 1]]),
    (8, 16, 8, 8 * 128, 16, 0.5, True, [[33, 20, 4], [1, 1, 2]]),
])
def test_layer_over_pages_step_by_step(T, heads, kv, ffn, page, p, e4m3, steps):
    """Prompts, chunks, drafts and single tokens of three sequences through caat_paged_layer_fwd, against the layer of the oracle
    over each sequence's whole history.  With e4m3 codes in the cache the heads' output is held to the attention over the codes."""
    total = [sum(s[b] for s in steps) for b in range(3)]
    cfg = I.BlockConfig("layer", I.KIND_PREFILL, I.NORM_RMSNORM, h=heads * 128, T=T, p=p, batch=1, seq=sum(total), ffn=ffn,
                        n_heads=heads, head_dim=128, n_kv_heads=kv)
    data = make_inputs(cfg, seed=41, weight_std=0.05)
    w = {k: O.widen_bf16(v) for k, v in data.items()}
    at = np.concatenate([[0], np.cumsum(total)])
    ref = [O.prefill_layer_fwd(w["R"][:, at[b]:at[b + 1]], w, batch=1, seq=total[b], heads_per_rank=heads // T, head_dim=128, hs=hs_of(cfg),
                               kv_heads_per_rank=kv // T) for b in range(3)]
    weights = _layer_weights(data)
    whole = P.make(42, T, heads, kv, total, total, page, e4m3, scales=False)
    k, v, lens = whole.k, whole.v, [0, 0, 0]
    for i, news in enumerate(steps):
        begun = list(lens)
        lens = [x + n for x, n in zip(lens, news)]
        c = P.make(50 + i, T, heads, kv, lens, news, page, e4m3, spare=0, columns=whole.table.shape[1])
        scale = 0.01 if e4m3 else 1.0
        c.n_pages, c.table, c.k, c.v, c.ks, c.vs = whole.n_pages, whole.table.copy(), k, v, whole.ks * scale, whole.vs * scale
        c.desc.n_pages, c.desc.stride_rank, c.desc.stride_page = whole.n_pages, whole.desc.stride_rank, whole.desc.stride_page
        d = P.on_gpu(c)
        desc, pages = _descs(cfg, c)
        rows = np.concatenate([np.arange(at[b] + begun[b], at[b] + lens[b]) for b in range(3)])
        r = B.to_device(np.ascontiguousarray(data["R"][:, rows]))
        r_out = r.clone()
        import torch
        ws = torch.full((B.paged_layer_workspace_bytes(desc, pages),), 255, dtype=torch.uint8, device="cuda")
        B.paged_layer_fwd(desc, pages, weights, r, r_out, d.row_start, d.lens, d.table, d.k, d.v, ws, d.ks, d.vs)
        k, v = P.bits(d.k).copy(), P.bits(d.v).copy()
        L = B.workspace_layout(desc)
        read = lambda off, size: ws[off:off + size].cpu().numpy().view(np.uint16).reshape(T, len(rows), -1)
        c.ld_q, c.k, c.v = (heads // T + 2 * kv // T) * 128, k, v
        P.check_attn(c, read(L.off_H, L.bytes_H), *P.ref_attn(c, q=read(L.off_Q, L.bytes_Q)), P.slack(c))
        if not e4m3:
            want = np.concatenate([ref[b]["R2"][:, begun[b]:lens[b]] for b in range(3)], axis=1)
            assert_close(bits_to_f64(B.to_host_bits(r_out)), want, "R2 of step %d" % i)
            for b in range(3):
                for t in range(begun[b], lens[b]):
                    pg, off = whole.table[b, t // page], t % page
                    assert_close(P.widen(P.view(c, k)[:, pg, :, off]), ref[b]["K"].reshape(T, kv // T, total[b], 128)[:, :, t], "K")


def test_layer_over_pages_is_the_layer_over_a_cache():
    """One new token for sequences of one length: caat_block_fwd over its contiguous caches and the layer over pages."""
    import torch
    T, heads, b, L = 2, 8, 5, 211
    cfg = I.BlockConfig("dec", I.KIND_DECODE, I.NORM_RMSNORM, h=heads * 128, T=T, p=0.5, batch=b, seq=1, ffn=2 * 256, n_heads=heads,
                        head_dim=128, kv_len=L, n_kv_heads=4)
    data = make_inputs(cfg, seed=43, weight_std=0.05)
    weights = _layer_weights(data)
    desc = B.make_desc(cfg)
    r = B.to_device(data["R"])
    kc, vc, out = B.to_device(data["Kc"]), B.to_device(data["Vc"]), torch.empty_like(r)
    ws = torch.empty(B.workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    B.block_fwd(desc, weights, None, r, out, None, ws, kv_k=kc, kv_v=vc)
    c = P.make(44, T, heads, 4, [L + 1] * b, [1] * b, 16)
    for name, x in (("Kc", P.view(c, c.k)), ("Vc", P.view(c, c.v))):
        for s in range(b):
            for t in range(L):
                x[:, c.table[s, t // 16], :, t % 16] = data[name][:, s, :, t]
    d = P.on_gpu(c)
    got = torch.empty_like(r)
    wp = torch.empty(B.paged_layer_workspace_bytes(desc, c.desc), dtype=torch.uint8, device="cuda")
    B.paged_layer_fwd(desc, c.desc, weights, r, got, None, d.lens, d.table, d.k, d.v, wp)
    # two roundings of a bf16 value that fall apart, through the layer: half of what is allowed against the oracle
    assert_close(bits_to_f64(B.to_host_bits(got)), bits_to_f64(B.to_host_bits(out)), "R2", tol=1e-2)
    v = P.widen(P.view(c, P.bits(d.v)))
    new = np.stack([v[:, c.table[s, L // 16], :, L % 16] for s in range(b)], axis=1)
    assert np.array_equal(new, bits_to_f64(B.to_host_bits(vc))[:, :, :, L])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [1, 3, 80])
def test_graphs_follow_lengths_rows_and_tables(e4m3, new):
    """Two captured graphs that share a workspace: replayed in turns with lists that change in between and the program's own work
    between the replays; every replay is the eager call's bits."""
    import torch
    T, heads, kv, page = 2, 8, 2, 16
    lens = [new + 200, new + 3, new + 90, new + 415]
    batches = [P.make(60 + i, T, heads, kv, lens[i:] + lens[:i], [max(1, new - j) for j in range(4)], page, e4m3, pad_rows=20, columns=40)
               for i in range(3)]
    n_pages = max(c.n_pages for c in batches)
    state = P.on_gpu(max(batches, key=lambda c: c.n_pages))
    base = max(batches, key=lambda c: c.n_pages)
    rows = max(c.rows for c in batches)
    desc = base.desc
    desc.rows, desc.max_new = rows, new
    state.qkv = torch.zeros((T, rows, base.ld_qkv), dtype=torch.int16, device="cuda")
    state.q_out = torch.zeros((T, rows, base.ld_q), dtype=torch.bfloat16, device="cuda")
    state.out = torch.zeros((T, rows, base.hpr * 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.paged_attn_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")

    def load(c):
        state.qkv[:, :c.rows] = torch.from_numpy(c.qkv.view(np.int16)).cuda()
        state.row_start.copy_(torch.from_numpy(c.row_start))
        state.lens.copy_(torch.from_numpy(c.lens))
        state.table.copy_(torch.from_numpy(c.table))

    def step():
        B.paged_append(desc, state.qkv, state.q_out, state.row_start, state.lens, state.table, state.k, state.v, state.ks, state.vs)
        B.paged_attn(desc, state.q_out, state.out, state.row_start, state.lens, state.table, state.k, state.v, ws, state.ks, state.vs)

    def step_again():
        B.paged_attn(desc, state.q_out, state.out, state.row_start, state.lens, state.table, state.k, state.v, ws, state.ks, state.vs)

    load(batches[0])
    step()
    torch.cuda.synchronize()
    graphs = []
    for body in (step, step_again):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            body()
        graphs.append(g)
    k0, v0 = state.k.clone(), state.v.clone()
    for turn in range(2):
        for c in batches:
            load(c)
            state.k.copy_(k0)
            state.v.copy_(v0)
            state.out.zero_()
            step()
            want = [P.bits(x).copy() for x in (state.out, state.q_out, state.k, state.v)]
            for which in (0, 1, 0):
                state.out.zero_()
                if which == 0:
                    state.k.copy_(k0)
                    state.v.copy_(v0)
                graphs[which].replay()
                got = [P.bits(x) for x in (state.out, state.q_out, state.k, state.v)]
                assert all(np.array_equal(a, b) for a, b in zip(got, want))
                ws.fill_(turn * 77)                    # nothing in it is kept


def test_on_a_stream_of_the_caller():
    """The stream that is handed over, and the current one where none is: each waits for its own inputs."""
    import torch
    c = P.make(70, 2, 8, 4, [300, 41, 77], [1, 1, 1], 16)
    ref = P.on_gpu(c)
    P.append(c, ref)
    P.attend(c, ref, q=ref.q_out)
    want = P.bits(ref.out).copy()
    side = torch.cuda.Stream()
    for how in ("argument", "current"):
        d = P.on_gpu(c)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            big = torch.ones(1 << 26, device="cuda")
            for _ in range(20):
                big = big * 1.0001
            qkv = d.qkv + (big[:1] * 0).to(torch.int16)      # ready only when the stream gets there
            d.qkv = qkv
            if how == "current":
                P.append(c, d)
                P.attend(c, d, q=d.q_out)
        if how == "argument":
            P.append(c, d, stream=side)
            P.attend(c, d, q=d.q_out, stream=side)
        side.synchronize()
        assert np.array_equal(P.bits(d.out), want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [1, 100])
def test_pools_of_more_than_four_gib(e4m3, new):
    """Pages at the end of a pool whose offsets pass 32 bits, in elements and in bytes."""
    import torch
    c = P.make(80, 1, 4, 1, [new + 300, new + 1000], [new, new], 64, e4m3)
    small = c.n_pages
    n_pages = (5 << 30) // (64 * 128 * (1 if e4m3 else 2)) + small
    d = P.on_gpu(c)
    first = n_pages - small
    want, want_k = P.on_gpu(c), None
    P.append(c, want)
    P.attend(c, want, q=want.q_out)
    want_out, want_k = P.bits(want.out).copy(), P.bits(want.k).copy()
    big = {}
    for name in "kv":
        x = getattr(d, name)
        big[name] = torch.empty((1, n_pages) + tuple(x.shape[2:]), dtype=x.dtype, device="cuda")
        big[name][:, first:] = x
    d.k, d.v, d.table = big["k"], big["v"], torch.where(d.table >= 0, d.table + first, d.table)
    c.desc.n_pages, c.desc.stride_rank = n_pages, n_pages * c.desc.stride_page
    P.append(c, d)
    P.attend(c, d, q=d.q_out)
    assert np.array_equal(P.bits(d.out), want_out)
    assert np.array_equal(P.bits(d.k[:, first:].contiguous()), want_k)
