"""Attention over and append to a paged cache at the edges of what the calls promise: how exact the probabilities are, scores and
scales far from 1, rows whose scores are all minus infinity, batches of unlike sequences."""
import numpy as np
import pytest

from paper_2506_19645_amd import binding as B
from tests import paged_util as P

pytestmark = pytest.mark.gpu


def _codes(x, e4m3):
    """Values that the cache type holds exactly, as its codes."""
    if not e4m3:
        return P.bf16(x)
    near = np.abs(P._CODES[None, :] - np.asarray(x, dtype=np.float64).reshape(-1, 1))
    near[:, np.isnan(P._CODES)] = np.inf
    assert np.all(near.min(axis=1) == 0)
    return near.argmin(axis=1).astype(np.uint8).reshape(np.shape(x))


def _fill(c, b, head, k, v):
    """Keys and values [positions, 128] of sequence b to its pages, on every rank."""
    for t in range(len(k)):
        page, off = c.table[b, t // c.page], t % c.page
        P.view(c, c.k)[:, page, head, off], P.view(c, c.v)[:, page, head, off] = _codes(k[t], c.e4m3), _codes(v[t], c.e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads", [1, 16, 20])
@pytest.mark.parametrize("repeat", [1, 20, 300])
def test_probabilities_are_whole(e4m3, heads, repeat):
    """Keys of two scores whose weighted values nearly cancel, so that what is left shows the probabilities' own error: less than
    2^-20 of sum p |v|.  The scores are exact (one product); times 1.44 / sqrt(128), twice rounded, they are 2^-23 * 0.7 off, so
    their exponentials 2^-23.5 and the instruction's ulp, 2^-23; the sums run near zero, where a key's rounding is at most 2^-22 of
    it.  Probabilities of 16 bits are 2^-17.8 off here."""
    c1, c2, a, b, n1, n2 = -1.625, -5.0, 11.0, 14.0, 17, 18
    block = [(0.0, 0.0)]
    while n1 + n2:                                       # in turn, so that the sums stay small
        if n2 >= n1 and n2:
            block.append((c2, -b)); n2 -= 1
        else:
            block.append((c1, a)); n1 -= 1
    keys = np.zeros((36 * repeat, 2))
    keys[:] = block * repeat
    c = P.make(90, 1, heads, 1, [len(keys)], [1], 16, e4m3, scales=False)
    k, v = np.zeros((len(keys), 128)), np.zeros((len(keys), 128))
    k[:, 0] = keys[:, 0]
    v[:, ::2], v[:, 1::2] = keys[:, 1:], -keys[:, 1:] / 2
    _fill(c, 0, 0, k, v)
    q = np.zeros((1, 1, heads, 128))
    q[..., 0] = 1.0
    c.q = P.bf16(q.reshape(1, 1, -1))
    d = P.on_gpu(c)
    P.attend(c, d)
    ref, size = P.ref_attn(c)
    got = P.widen(P.bits(d.out))
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * size), np.max(np.abs(got - ref) / size) * 2 ** 20


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,grp", [(1, 1), (1, 20), (3, 4), (9, 4), (150, 1)])
@pytest.mark.parametrize("long", [0, 70, 1500])
def test_scores_of_minus_infinity_alone_make_zeros(e4m3, new, grp, long):
    """Every score of a row is minus infinity: zeros, also where the values are infinite or NaN."""
    c = P.make(91, 1, 2 * grp, 2, [long + new, new + 20], [new, new], 16, e4m3)
    q = c.q.reshape(1, 2 * new, 2 * grp, 128)
    q[0, :new, :grp, 3] = 0xFF80
    k, v = P.view(c, c.k), P.view(c, c.v)
    pages = c.table[0][c.table[0] >= 0]
    one, nan, inf = (0x38, 0x7F, 0xFF) if e4m3 else (0x3F80, 0x7FC0, 0x7F80)
    k[0, pages, 0, :, 3] = one
    was = v[0, pages, 0].copy()
    v[0, pages, 0] = 0
    ref, size = P.ref_attn(c)
    v[0, pages, 0] = was
    v[0, pages, 0, :, 5], v[0, pages, 0, ::3, 77] = nan, inf
    d = P.on_gpu(c)
    P.attend(c, d)
    got = P.bits(d.out)
    assert np.all(ref.reshape(1, 2 * new, 2 * grp, 128)[:, :new, :grp] == 0)
    P.check_attn(c, got, ref, size, P.slack(c))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,grp", [(1, 1), (3, 4), (9, 4), (40, 1), (150, 2)])
@pytest.mark.parametrize("long", [0, 70, 1500])
@pytest.mark.parametrize("power", [13, 15, 18, 30])
def test_scores_far_from_one(e4m3, new, grp, long, power):
    """Queries and keys of 2^13 to 2^30: scores whose last place is more than an exponential's range.  The two largest scores of a row
    are at least 1.6e-5 of the largest apart for these inputs, the fp32 sums 1e-6: one key's value each."""
    c = P.make(92, 1, 2 * grp, 2, [long + new, new + 33], [new, new], 16, e4m3)
    c.q = P.bf16(P.widen(c.q) * 2.0 ** power)
    if e4m3:
        c.ks = c.ks * 2.0 ** power
    else:
        c.k = P.bf16(P.widen(c.k) * 2.0 ** power)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


def _nearest_codes(x):
    """e4m3 values nearest to x, halves to the even code, saturating."""
    x = np.clip(np.asarray(x, dtype=np.float64), -448, 448)
    grid = P._CODES[:0x7F]                               # the non-negative codes run upwards
    at = np.searchsorted(grid, np.abs(x)).clip(1, len(grid) - 1)
    lo, hi = grid[at - 1], grid[at]
    up = (np.abs(x) - lo > hi - np.abs(x)) | ((np.abs(x) - lo == hi - np.abs(x)) & (at % 2 == 0))
    return np.copysign(np.where(up, hi, lo), x)


@pytest.mark.parametrize("scale", [7.0, 7.0 / 512, 3.0, 25.0 / 1024, 2.0 ** -130, 3 * 2.0 ** -149, 2.0 ** 100])
def test_codes_are_of_the_quotient(scale):
    """Values in the middle of two codes times scales that are no power of two, and scales whose reciprocal is none of fp32's: the
    code is that of value / scale.  Position 0, so that keys are stored as they come."""
    c = P.make(93, 1, 1, 1, [1], [1], 16, True, scales=False)
    x = np.zeros(128)
    m = np.array([17, 19, 21, 23, 25, 27, 29, 31, 16, 18, 3, 5, 448, 449, 464, 480], dtype=np.float64)
    for i in range(8):
        x[i * 16:(i + 1) * 16] = m * 2.0 ** (i - 6) * (-1) ** i
    x[15::16] = 0.0
    want = P.bf16(x * scale)                             # rounded to bf16 where the product has more bits
    c.qkv[0, 0, 128:256], c.qkv[0, 0, 256:] = want, want
    c.ks[:], c.vs[:] = scale, scale
    d = P.on_gpu(c)
    P.append(c, d)
    codes = _nearest_codes(np.float32(P.widen(want) / scale))
    for got in (d.k, d.v):
        assert np.array_equal(P.decode(P.view(c, P.bits(got))[0, c.table[0, 0], 0, 0], True), codes)


@pytest.mark.parametrize("new,grp", [(1, 1), (3, 4), (9, 4), (40, 1), (150, 2)])
@pytest.mark.parametrize("long", [0, 70, 1500])
@pytest.mark.parametrize("scale", [2.0 ** -149, 2.0 ** -126, 2.0 ** -60, 2.0 ** 100])
def test_scales_of_keys_far_from_one(new, grp, long, scale):
    """Any positive scale.  With the small ones all keys that are seen weigh the same; with 2^100 one key takes all, by a gap of 1.4e-5
    of the largest score for these inputs."""
    c = P.make(94, 1, 2 * grp, 2, [long + new, new + 33], [new, new], 16, True)
    c.ks[:] = scale
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


# Relative 2-norm of the outputs' error over N(0, 1) queries, keys and values: a probability's rounding to bf16 and the output's own are
# at most half a step each, spread evenly over it, 2^-8 / sqrt(3); of independent values their squares add up to (2^-8)^2 * 2 / 3.
WHOLE = 2.0 ** -8


def check_norm(c, got_bits, ref):
    own = ~np.isnan(ref)
    err = P.widen(got_bits)[:, :c.rows][own] - ref[own]
    assert np.linalg.norm(err) <= WHOLE * np.linalg.norm(ref[own]), np.linalg.norm(err) / np.linalg.norm(ref[own])


@pytest.mark.parametrize("T,heads,kv,lens,news,page,e4m3", [
    (8, 32, 32, [2500, 33], [1600, 1], 16, False),           # 416 full tiles and more: each its own workgroup
    (8, 32, 32, [2500, 33], [1600, 1], 64, True),
    (8, 64, 8, [1900, 400, 1500, 1], [700, 90, 1, 1], 48, False),    # 404
    (8, 64, 8, [900, 1, 30, 2900], [820, 1, 2, 1], 16, True),        # the longest sequence last, one new token
])
def test_prompts_without_a_line(T, heads, kv, lens, news, page, e4m3):
    """More full tiles than share a line, over more than a thousand keys, single tokens and drafts among the prompts."""
    c = P.make(98, T, heads, kv, lens, news, page, e4m3, pad_rows=3)
    d = P.on_gpu(c)
    P.attend(c, d)
    ref, size = P.ref_attn(c)
    P.check_attn(c, P.bits(d.out), ref, size, P.slack(c))
    check_norm(c, P.bits(d.out), ref)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("T,heads,kv", [(2, 8, 2), (4, 8, 8)])
def test_single_tokens_and_prompts_in_two_calls(T, heads, kv, e4m3):
    """The sequences of a batch whose first have single tokens and whose last have prompts, in a call each over the same buffers: the
    rows of the other call's sequences are nobody's and stay, and the single tokens have whole probabilities."""
    lens, news = [3000, 1, 77, 0, 640, 300, 210], [1, 1, 1, 0, 2, 150, 210]
    c = P.make(99, T, heads, kv, lens, news, 32, e4m3, pad_rows=2)
    few = 5
    def part(b0, b1):
        return B.paged_desc(T=T, batch=b1 - b0, n_heads=heads, n_kv_heads=kv, rows=c.rows, page_size=32, n_pages=c.n_pages,
                            max_pages=c.table.shape[1], max_new=max(news[b0:b1]), cache_type=c.desc.cache_type)
    d, e = P.on_gpu(c), P.on_gpu(c)
    P.append(c, e)
    ref, size = P.ref_attn(c)
    for b0, b1 in ((0, few), (few, 7)):
        d.out.fill_(-7.0)
        pg = part(b0, b1)
        lists = (d.row_start[b0:b1 + 1].clone(), d.lens[b0:b1].clone(), d.table[b0:b1].clone())
        B.paged_append(pg, d.qkv, d.q_out, *lists, d.k, d.v, d.ks, d.vs)
        c2 = P.on_gpu(c)                                     # the caches as they were: what ref_attn looks at
        B.paged_attn(pg, c2.q, d.out, *lists, c2.k, c2.v, c2.ws, c2.ks, c2.vs)
        r0, r1 = int(c.row_start[b0]), int(c.row_start[b1])
        mine = np.full(ref.shape, np.nan)
        mine[:, r0:r1] = ref[:, r0:r1]
        P.check_attn(c, P.bits(d.out), mine, size, P.FEW if b0 == 0 else P.MANY)
        check_norm(c, P.bits(d.out), mine)
    for x in ("q_out", "k", "v"):                            # both appends together: the one call's
        assert np.array_equal(P.bits(getattr(d, x)), P.bits(getattr(e, x)))


@pytest.mark.parametrize("e4m3", [False, True])
def test_views_of_one_allocation(e4m3):
    """Keys and values of a page one after the other in one pool, q inside qkv's rows: the bits of tensors of their own."""
    import torch
    c = P.make(100, 2, 8, 4, [100, 33, 7], [30, 1, 7], 48, e4m3)
    d, e = P.on_gpu(c), P.on_gpu(c)
    P.append(c, d)
    P.attend(c, d, q=d.q_out)
    T, pages, kvpr, page = e.k.shape[:4]
    pool = torch.stack((e.k, e.v), dim=2)                    # [T][pages][2][heads][page][128]
    k, v = pool[:, :, 0], pool[:, :, 1]
    qw = (c.hpr + 2 * c.kvpr) * 128
    desc = B.paged_desc(T=2, batch=3, n_heads=8, n_kv_heads=4, rows=c.rows, page_size=48, n_pages=c.n_pages, max_pages=c.table.shape[1],
                        max_new=30, cache_type=c.desc.cache_type, ld_q=qw, strides=k.stride()[:4])
    q = e.qkv[:, :, :c.hpr * 128]
    B.paged_append(desc, e.qkv, e.qkv, e.row_start, e.lens, e.table, k, v, e.ks, e.vs)
    B.paged_attn(desc, q, e.out, e.row_start, e.lens, e.table, k, v, e.ws, e.ks, e.vs)
    for got, want in ((e.out, d.out), (q.contiguous(), d.q_out), (k.contiguous(), d.k), (v.contiguous(), d.v)):
        assert np.array_equal(P.bits(got), P.bits(want))
