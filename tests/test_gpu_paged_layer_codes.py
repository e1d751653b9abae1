"""The decoder layer over a paged cache, piece by piece: what it appends is held to the projections of its own inputs, its heads'
output to the attention over what the caches hold, its output to the rest of the layer over the heads' output.  None of the three
needs a tolerance for the codes' quantisation, so an 8-bit cache is checked as closely as a bf16 one."""
import numpy as np
import pytest

from oracle import caat_oracle as O
from paper_2506_19645_amd import binding as B
from paper_2506_19645_amd import inputs as I
from tests import paged_util as P
from tests.test_gpu_paged_layer import _descs, _layer_weights
from tests.util import assert_close, bits_to_f64, hs_of, make_inputs

pytestmark = pytest.mark.gpu


def _rest_of_the_layer(R, H, w, hs):
    """o_proj, the partial channel-reduce and the residual, RMSNorm, the SwiGLU MLP and its reduce over the heads' output."""
    T = R.shape[0]
    R1 = R + O.partial_channel_reduce(np.stack([H[m] @ w["Wo"][m].T for m in range(T)]), hs)
    X2 = O.norm_fwd(R1, w["gamma"], None, O.RMSNORM, 1e-5)[0]
    Y = [O.silu(X2[m] @ w["Wg"][m].T) * (X2[m] @ w["Wu"][m].T) for m in range(T)]
    return R1 + O.partial_channel_reduce(np.stack([Y[m] @ w["B"][m].T for m in range(T)]), hs)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("T,heads,kv,ffn,page,p,steps", [
    (2, 4, 4, 2 * 256, 16, 0.5, [[37, 20, 0], [1, 1, 50], [1, 1, 1], [0, 3, 1]]),
    (2, 8, 2, 2 * 344, 48, 0.3, [[300, 140, 1], [1, 250, 1], [130, 1, 90], [1, 1, 1]]),     # prompts beside single tokens
    (8, 16, 8, 8 * 128, 64, 0.5, [[600, 33, 4], [5, 700, 2], [1, 1, 1]]),
])
def test_layer_over_pages_piece_by_piece(T, heads, kv, ffn, page, p, steps, e4m3):
    import torch
    total = [sum(s[b] for s in steps) for b in range(3)]
    cfg = I.BlockConfig("layer", I.KIND_PREFILL, I.NORM_RMSNORM, h=heads * 128, T=T, p=p, batch=1, seq=sum(total), ffn=ffn,
                        n_heads=heads, head_dim=128, n_kv_heads=kv)
    data = make_inputs(cfg, seed=95, weight_std=0.05)
    w = {k: O.widen_bf16(v) for k, v in data.items()}
    at = np.concatenate([[0], np.cumsum(total)])
    weights = _layer_weights(data)
    whole = P.make(96, T, heads, kv, total, total, page, e4m3, scales=False)
    k, v, lens = whole.k, whole.v, [0, 0, 0]
    hpr, kvpr = heads // T, kv // T
    for i, news in enumerate(steps):
        begun = list(lens)
        lens = [x + n for x, n in zip(lens, news)]
        c = P.make(97 + i, T, heads, kv, lens, news, page, e4m3, spare=0, columns=whole.table.shape[1])
        c.n_pages, c.table, c.k, c.v = whole.n_pages, whole.table.copy(), k, v
        if e4m3:
            c.ks, c.vs = whole.ks * np.float32(0.011), whole.vs * np.float32(0.013)
        c.desc.n_pages, c.desc.stride_rank, c.desc.stride_page = whole.n_pages, whole.desc.stride_rank, whole.desc.stride_page
        d = P.on_gpu(c)
        desc, pages = _descs(cfg, c)
        rows = np.concatenate([np.arange(at[b] + begun[b], at[b] + lens[b]) for b in range(3)])
        r = B.to_device(np.ascontiguousarray(data["R"][:, rows]))
        r_out = torch.empty_like(r)
        ws = torch.full((B.paged_layer_workspace_bytes(desc, pages),), 255, dtype=torch.uint8, device="cuda")
        B.paged_layer_fwd(desc, pages, weights, r, r_out, d.row_start, d.lens, d.table, d.k, d.v, ws, d.ks, d.vs)
        L = B.workspace_layout(desc)
        read = lambda off, size: ws[off:off + size].cpu().numpy().view(np.uint16).reshape(T, len(rows), -1)
        QKV, H = read(L.off_Q, L.bytes_Q), read(L.off_H, L.bytes_H)

        # the projections of this step's rows: q rotated, k and v as they come
        R = w["R"][:, rows]
        X1 = O.norm_fwd(R, w["gamma_attn"], None, O.RMSNORM, 1e-5)[0]
        raw = np.stack([X1[m] @ w["Wqkv"][m].T for m in range(T)]).reshape(T, len(rows), hpr + 2 * kvpr, 128)
        pos = np.concatenate([np.arange(begun[b], lens[b]) for b in range(3)])
        rot = raw.copy()
        angle = pos[:, None] * 10000.0 ** (-np.arange(0, 128, 2) / 128)
        cs, sn = np.cos(angle)[:, None], np.sin(angle)[:, None]
        rot[..., :64], rot[..., 64:] = raw[..., :64] * cs - raw[..., 64:] * sn, raw[..., 64:] * cs + raw[..., :64] * sn
        got = P.widen(QKV).reshape(raw.shape)
        assert_close(got[:, :, :hpr], rot[:, :, :hpr], "q of step %d" % i)
        assert_close(got[:, :, hpr:], raw[:, :, hpr:], "k and v of step %d" % i)

        # what was appended of them, to their places and no others
        c.qkv = QKV
        _, _, places, want_k, want_v, size = P.ref_append(c)
        assert len(places) == len(rows)
        for now, was, want, slack in ((P.bits(d.k).copy(), k, want_k, size), (P.bits(d.v).copy(), v, want_v, 0 * want_v)):
            new = np.zeros(P.view(c, was).shape, dtype=bool)
            vals = P.decode(P.view(c, now), e4m3)
            for row, (pg, off) in places.items():
                new[:, pg, :, off] = True
                x = np.clip(want[:, row], -448, 448) if e4m3 else want[:, row]
                # half a step of the type, the quotient's rounding, and of k the angle, sine and cosine (5e-6) and the products
                tol = (2.0 ** -4 + 2.0 ** -23) * np.abs(x) + 2.0 ** -10 if e4m3 else 2.0 ** -8 * np.abs(x)
                assert np.all(np.abs(vals[:, pg, :, off] - x) <= tol + 6e-6 * slack[:, row])
            assert np.array_equal(P.view(c, now)[~new], P.view(c, was)[~new])
        k, v = P.bits(d.k).copy(), P.bits(d.v).copy()

        # the heads' output over what the caches hold, and the layer's over the heads'
        c.ld_q, c.k, c.v = (hpr + 2 * kvpr) * 128, k, v
        P.check_attn(c, H, *P.ref_attn(c, q=QKV), P.slack(c))
        assert_close(bits_to_f64(B.to_host_bits(r_out)), _rest_of_the_layer(R, P.widen(H), w, hs_of(cfg)), "r_out of step %d" % i)
