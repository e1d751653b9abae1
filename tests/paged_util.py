"""A ragged batch over a paged key / value cache: its inputs, and the append and the attention written out in 64 bits."""
import math
from types import SimpleNamespace

import numpy as np

from paper_2506_19645_amd import binding as B

D = 128


def bf16(x):
    """Values rounded to bf16, as uint16 bit patterns."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)).astype(np.uint16)


def widen(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


_CODES = np.array([(-1.0) ** (c >> 7) * (np.nan if c & 0x7F == 0x7F else (c & 7) * 2.0 ** -9 if (c >> 3) & 15 == 0 else
                                          (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7)) for c in range(256)])


def decode(raw, e4m3):
    """Cache contents (uint8 e4m3 codes or uint16 bf16 bits) as values."""
    return _CODES[raw] if e4m3 else widen(raw)


def make(seed, T, heads, kv_heads, lens, news, page, e4m3=False, order="phrd", spare=3, pad_rows=0, ld_q=0, ld_qkv=0, scales=True,
         std=1.0, columns=None):
    """order: how a rank's cache runs through pages (p), heads (h), rows of a page (r) and channels (d), outermost first."""
    rng = np.random.default_rng(seed)
    kvpr, hpr = kv_heads // T, heads // T
    need = [-(-max(x, 0) // page) for x in lens]
    n_pages, columns = sum(need) + spare, columns or max(1, max(need))
    free = rng.permutation(n_pages)
    table = np.full((len(lens), columns), -1, dtype=np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = free[at:at + k]
        at += k
    rows = sum(news) + pad_rows
    hd, qw = hpr * D, (hpr + 2 * kvpr) * D
    size = {"p": n_pages, "h": kvpr, "r": page, "d": D}
    shape = (T,) + tuple(size[x] for x in order)
    stride, run = {}, 1
    for x in reversed(order):
        stride[x] = run
        run *= size[x]
    c = SimpleNamespace(T=T, heads=heads, kv_heads=kv_heads, kvpr=kvpr, hpr=hpr, lens=np.array(lens, np.int32), page=page, e4m3=e4m3,
                        row_start=np.concatenate([[0], np.cumsum(news)]).astype(np.int32), news=list(news), table=table, rows=rows,
                        n_pages=n_pages, order=order, ld_q=ld_q or hd, ld_qkv=ld_qkv or qw, ks=np.ones((T, kvpr)), vs=np.ones((T, kvpr)))
    c.desc = B.paged_desc(T=T, batch=len(lens), n_heads=heads, n_kv_heads=kv_heads, rows=rows, page_size=page, n_pages=n_pages,
                          max_pages=columns, max_new=max(list(news) + [1]), cache_type=B.CACHE_E4M3 if e4m3 else B.CACHE_BF16,
                          ld_q=ld_q, ld_qkv=ld_qkv, strides=(run, stride["p"], stride["h"], stride["r"]))
    c.qkv, c.q = bf16(rng.standard_normal((T, rows, c.ld_qkv)) * std), bf16(rng.standard_normal((T, rows, c.ld_q)) * std)
    if e4m3:
        if scales:
            c.ks, c.vs = (np.float32(rng.uniform(0.008, 0.02, (T, kvpr))).astype(np.float64) for _ in range(2))
        codes = np.clip(rng.integers(0, 256, (2,) + shape), 0, 255).astype(np.uint8)
        codes[(codes & 0x7F) > 0x78] = 0x31          # no NaN, and none of the largest codes
        c.k, c.v = codes
    else:
        c.k, c.v = bf16(rng.standard_normal(shape)), bf16(rng.standard_normal(shape))
    return c


def view(c, x):
    """A cache array as [T, page, head, row, channel], whatever its order in memory."""
    return np.moveaxis(x, [1 + c.order.index(a) for a in "phrd"], [1, 2, 3, 4])


def _tokens(c):
    for b, n in enumerate(c.news):
        for i in range(n):
            yield b, int(c.row_start[b]) + i, max(int(c.lens[b]), 0) - n + i


def _page(c, b, pos):
    col = pos // c.page
    page = int(c.table[b, col]) if 0 <= pos and col < c.table.shape[1] else -1
    return page if 0 <= page < c.n_pages else -1


def ref_append(c, base=10000.0):
    """(q, its slack [T, rows, ld_q]) and {(b, row, pos): (page, offset)}, k and v values [T, rows, kvpr, D] over their scales, slack of k."""
    x = widen(c.qkv)[:, :, :(c.hpr + 2 * c.kvpr) * D].reshape(c.T, c.rows, -1, D)
    q = np.full((c.T, c.rows, c.ld_q), np.nan)
    qs, places = np.zeros_like(q), {}
    k, v, ks = (np.zeros((c.T, c.rows, c.kvpr, D)) for _ in range(3))
    freq = base ** (-np.arange(0, D, 2) / D)
    for b, row, pos in _tokens(c):
        cs, sn = np.cos(pos * freq), np.sin(pos * freq)
        a, z = x[:, row, :c.hpr + c.kvpr, :64], x[:, row, :c.hpr + c.kvpr, 64:]
        rot = np.concatenate([a * cs - z * sn, z * cs + a * sn], axis=-1)
        size = np.concatenate([np.abs(a) + np.abs(z)] * 2, axis=-1)
        q[:, row, :c.hpr * D] = rot[:, :c.hpr].reshape(c.T, -1)
        qs[:, row, :c.hpr * D] = size[:, :c.hpr].reshape(c.T, -1)
        k[:, row], ks[:, row] = rot[:, c.hpr:] / c.ks[:, :, None], size[:, c.hpr:] / c.ks[:, :, None]
        v[:, row] = x[:, row, c.hpr + c.kvpr:] / c.vs[:, :, None]
        if _page(c, b, pos) >= 0:
            places[row] = (_page(c, b, pos), pos % c.page)
    return q, qs, places, k, v, ks


def ref_attn(c, q=None, k=None, v=None):
    """out [T, rows, hd] and sum_t p_t |v_t|, NaN in rows of no sequence."""
    q = widen(c.q if q is None else q)
    k, v = (decode(view(c, x), c.e4m3) for x in (c.k if k is None else k, c.v if v is None else v))
    out = np.full((c.T, c.rows, c.hpr * D), np.nan)
    size = np.zeros_like(out)
    grp = c.hpr // c.kvpr
    owned = {}
    for b, row, pos in _tokens(c):
        owned.setdefault(b, []).append((row, pos))
    for b, here in owned.items():
        last = min(here[-1][1] + 1, c.table.shape[1] * c.page)
        spots = [(t, _page(c, b, t)) for t in range(last)]
        spots = [(t, g) for t, g in spots if g >= 0]
        t = np.array([s[0] for s in spots], dtype=int)
        g = np.array([s[1] for s in spots], dtype=int)
        rows, pos = [r for r, _ in here], np.array([p for _, p in here])
        out[:, rows] = 0.0
        if not len(t):
            continue
        see = t[None] <= pos[:, None]
        for m in range(c.T):
            for h in range(c.hpr):
                kh = h // grp
                kk, vv = k[m, g, kh, t % c.page] * c.ks[m, kh], v[m, g, kh, t % c.page] * c.vs[m, kh]
                with np.errstate(invalid="ignore"):
                    s = np.where(see, q[m, rows, h * D:(h + 1) * D] @ np.where(np.isfinite(kk), kk, 0.0).T / math.sqrt(D), -np.inf)
                top = s.max(axis=1, keepdims=True)
                p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
                den = p.sum(axis=1, keepdims=True)
                p = p / np.where(den == 0, 1.0, den)
                out[m, rows, h * D:(h + 1) * D] = p @ vv
                size[m, rows, h * D:(h + 1) * D] = p @ np.abs(vv)
    return out, size


def on_gpu(c):
    """The device tensors of a case."""
    import torch
    def dev(x):
        x = np.ascontiguousarray(x)
        return torch.from_numpy(x.view({2: np.int16, 1: np.uint8, 4: np.int32}[x.itemsize]) if x.dtype != np.float32 else x).cuda()
    d = SimpleNamespace(qkv=dev(c.qkv), q=dev(c.q), k=dev(c.k), v=dev(c.v), row_start=dev(c.row_start), lens=dev(c.lens), table=dev(c.table))
    d.ks, d.vs = (dev(np.float32(x)) if c.e4m3 else None for x in (c.ks, c.vs))
    d.out = torch.full((c.T, max(c.rows, 1), c.hpr * D), -7.0, dtype=torch.bfloat16, device="cuda")
    d.q_out = torch.full((c.T, max(c.rows, 1), c.ld_q), -7.0, dtype=torch.bfloat16, device="cuda")
    d.ws = torch.full((B.paged_attn_workspace_bytes(c.desc),), 255, dtype=torch.uint8, device="cuda")
    return d


def append(c, d, **kw):
    return B.paged_append(c.desc, d.qkv, d.q_out, d.row_start, d.lens, d.table, d.k, d.v, d.ks, d.vs, **kw)


def attend(c, d, q=None, **kw):
    return B.paged_attn(c.desc, d.q if q is None else q, d.out, d.row_start, d.lens, d.table, d.k, d.v, d.ws, d.ks, d.vs, **kw)


def bits(t):
    """A device tensor's bit patterns."""
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy() if t.element_size() == 1 else t.view(torch.int16).cpu().numpy().view(np.uint16)


# What a result may be off.  A bf16 rounding is half a step, 2^-8 of the value.  In front of it: scores of 128 fp32 products,
# 128 * 2^-24 * sum |q k| / sqrt(128) (about 7 for N(0, 1) values), so 6e-5 of a probability, twice with the normalisation: 2^-13
# of sum p |v|.  Probabilities rounded to bf16 (prompts) add 2^-8, twice with the normalisation.
FEW, MANY = 2.0 ** -13, 2.0 ** -7 + 2.0 ** -13


def slack(c):
    """Up to 32 (token, head of the group) rows of a sequence keep 16 bits of a probability, more of them 8."""
    return FEW if c.desc.max_new * (c.hpr // c.kvpr) <= 32 else MANY


def check_attn(c, got_bits, ref, size, slack):
    got = widen(got_bits)[:, :c.rows]
    own = ~np.isnan(ref)
    assert np.all(got[~own] == -7.0), "a row of no sequence was written"
    err = np.abs(got - ref)[own] - (2.0 ** -8 * np.abs(ref) + slack * size)[own]
    assert np.all(np.isfinite(got[own])), "not finite"
    assert err.size == 0 or err.max() <= 1e-30, "off by %.3g more than allowed" % err.max()


def check_append(c, d_q, d_k, d_v, k0, v0):
    q, qs, places, k, v, ks = ref_append(c)
    got = widen(d_q)[:, :c.rows]
    own = ~np.isnan(q)
    assert np.all(got[~own] == -7.0), "a row or column of no sequence was written"
    # the angle is 1e-6 off at most, sine and cosine 4e-6 more, products and sum 2^-23 of their size
    assert np.all((np.abs(got - q) <= 2.0 ** -8 * np.abs(q) + 6e-6 * qs)[own])
    for got, was, want, size in ((d_k, k0, k, ks), (d_v, v0, v, 0 * v)):
        new = np.zeros(view(c, was).shape, dtype=bool)
        vals = decode(view(c, got), c.e4m3)
        for row, (page, off) in places.items():
            new[:, page, :, off] = True
            w = want[:, row]
            if c.e4m3:
                w = np.clip(w, -448, 448)
                tol = 2.0 ** -4 * np.abs(w) + 2.0 ** -10 + 6e-6 * size[:, row] + 2.0 ** -23 * np.abs(w)
            else:
                tol = 2.0 ** -8 * np.abs(w) + 6e-6 * size[:, row]
            assert np.all(np.abs(vals[:, page, :, off] - w) <= tol)
        assert np.array_equal(view(c, got)[~new], view(c, was)[~new]), "a place of no new token was written"
