"""Append to and attention over a paged key / value cache, against the definition in 64 bits, through the C ABI."""
import numpy as np
import pytest

from paper_2506_19645_amd import binding as B
from tests import paged_util as P

pytestmark = pytest.mark.gpu

# T, heads, kv_heads, lens, news, page, e4m3, order
FEW_TOKENS = [
    (1, 1, 1, [1], [1], 16, False, "phrd"),
    (2, 4, 4, [37], [1], 16, False, "phrd"),
    (1, 4, 1, [15, 16, 17, 31, 32, 33, 0, 1], [1, 1, 1, 1, 1, 1, 0, 1], 16, False, "phrd"),
    (2, 16, 4, [300, 1, 511, 64], [1, 1, 1, 1], 64, False, "prhd"),          # [page][position][head]
    (1, 40, 2, [77, 129], [1, 1], 48, False, "hprd"),                        # groups of 20 heads: more than one tile of rows
    (2, 2, 2, [2000, 3, 700], [1, 1, 1], 80, False, "phrd"),
    (1, 8, 2, [100, 9, 0, 260], [5, 9, 0, 4], 16, False, "phrd"),            # drafts; 9 new of 9
    (1, 2, 2, [64, 200], [17, 3], 32, False, "phrd"),                        # 17 rows
    (1, 3, 1, [50, 4], [5, 4], 16, False, "phrd"),                           # 15 and 12 rows
    (1, 16, 2, [300, 77, 50], [5, 6, 3], 16, False, "phrd"),                 # 40, 48 and 24 rows
    (1, 8, 1, [1500, 30, 9], [8, 7, 1], 16, False, "phrd"),                  # 64 and 56 rows
    (1, 6, 1, [3001], [7], 64, False, "phrd"),                               # 42 rows, many workgroups inside one unit
    (1, 8, 1, [2222, 40], [4, 3], 32, True, "phrd"),                         # 32 and 24 rows
    (2, 4, 2, [(17 * i) % 311 for i in range(70)], [int(i % 9 != 0) for i in range(70)], 32, False, "phrd"),   # more than 64 sequences
    (1, 8, 4, [(29 * i) % 801 + 1 for i in range(150)], [i % 3 for i in range(150)], 16, True, "phrd"),
    (1, 2, 1, [5 + 40 * (i == 131) for i in range(200)], [1] * 200, 16, False, "phrd"),   # short sequences around one
    (1, 2, 2, [1000, 200], [1, 1], 512, True, "phrd"),                       # a workgroup per unit
    (8, 8, 8, [500], [1], 16, False, "phrd"),
    (1, 1, 1, [1], [1], 16, True, "phrd"),
    (2, 8, 2, [15, 16, 17, 31, 32, 33, 0, 1], [1, 1, 1, 1, 1, 1, 0, 1], 16, True, "phrd"),
    (1, 8, 1, [300, 1, 511, 64], [1, 2, 3, 2], 48, True, "prhd"),
    (2, 2, 2, [2000, 3, 700], [1, 1, 1], 32, True, "phrd"),
    (4, 64, 8, [1500], [1], 256, True, "hprd"),
]
PROMPTS = [
    (1, 2, 2, [128], [128], 16, False, "phrd"),
    (2, 4, 2, [63, 64, 65], [63, 64, 65], 16, False, "phrd"),
    (1, 2, 1, [129, 1, 0, 300], [129, 1, 0, 40], 64, False, "prhd"),
    (1, 6, 2, [500, 333], [257, 91], 48, False, "hprd"),                     # groups of 3 heads: tokens across tiles
    (1, 1, 1, [700], [33], 80, False, "phrd"),
    (2, 8, 2, [200, 77], [200, 50], 16, True, "phrd"),
    (1, 3, 1, [500, 2, 90], [257, 2, 90], 48, True, "prhd"),
    (1, 2, 2, [1000], [130], 128, True, "phrd"),
    (1, 2, 1, [3001, 500, 0, 33], [70, 40, 0, 33], 16, False, "phrd"),       # the keys of a tile dealt to many workgroups,
    (2, 4, 2, [2500, 90], [90, 90], 48, True, "phrd"),                       # of a short sequence to some that have none
    (1, 8, 1, [5000], [300], 256, False, "prhd"),
]


@pytest.mark.parametrize("T,heads,kv,lens,news,page,e4m3,order", FEW_TOKENS + PROMPTS)
def test_append(T, heads, kv, lens, news, page, e4m3, order):
    c = P.make(11, T, heads, kv, lens, news, page, e4m3, order, pad_rows=2)
    d = P.on_gpu(c)
    k0, v0 = c.k.copy(), c.v.copy()
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), k0, v0)


@pytest.mark.parametrize("T,heads,kv,lens,news,page,e4m3,order", FEW_TOKENS)
def test_attention_of_few_tokens(T, heads, kv, lens, news, page, e4m3, order):
    c = P.make(12, T, heads, kv, lens, news, page, e4m3, order, pad_rows=2)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("T,heads,kv,lens,news,page,e4m3,order", PROMPTS)
def test_attention_of_prompts(T, heads, kv, lens, news, page, e4m3, order):
    c = P.make(13, T, heads, kv, lens, news, page, e4m3, order, pad_rows=2)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("T,heads,kv,e4m3", [(8, 64, 8, True), (8, 32, 32, False), (4, 16, 8, False), (8, 64, 8, False)])
def test_the_same_bits_every_time(T, heads, kv, e4m3):
    """Workgroups that go through several units, waves that go through several, many joins: the same call gives the same bits, and
    the definition's values on some rows."""
    lens = [399, 4001, 17, 0, 1, 803, 250, 1500, 64, 333, 2048, 90, 411, 700, 37, 128, 999, 555, 16, 1201] * 3
    c = P.make(23, T, heads, kv, lens, [int(x > 0) for x in lens], 32, e4m3)
    d = P.on_gpu(c)
    P.attend(c, d)
    first = P.bits(d.out).copy()
    for _ in range(20):
        d.out.fill_(-7.0)
        P.attend(c, d)
        assert np.array_equal(P.bits(d.out), first)
    P.check_attn(c, first, *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("T,heads,kv,e4m3,keys", [(8, 32, 32, False, 700), (8, 32, 32, True, 1500), (8, 32, 32, False, 60), (4, 64, 32, True, 90)])
def test_more_units_than_waves(T, heads, kv, e4m3, keys):
    """More (sequence, head) pairs than the waves of a launch, with long and with short caches."""
    lens = [keys - (37 * i) % (keys // 2) for i in range(90)]
    c = P.make(24, T, heads, kv, lens, [1] * 90, 32, e4m3)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("batch", [65, 300, 4300])
@pytest.mark.parametrize("e4m3", [False, True])
def test_many_sequences(batch, e4m3):
    """More sequences than a wave looks at together, and than it keeps sums of; free slots among them."""
    lens = [(7 * i) % 61 for i in range(batch)]
    lens[batch - 2] = 500
    c = P.make(26, 1, 2, 1, lens, [int(x > 0 and i % 7 != 3) for i, x in enumerate(lens)], 16, e4m3)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), c.k, c.v)


@pytest.mark.parametrize("batch", [5, 90])
def test_rows_in_another_order_than_the_sequences(batch):
    """Sequence 0 owns the last rows, sequence 2 the first ones; nobody owns any other way."""
    news = [30, 0, 50] + [0] * (batch - 3)
    c = P.make(27, 1, 4, 2, [77, 5, 50] + [9] * (batch - 3), news, 16)
    c.row_start = np.array([50, 80, 0] + [50] * (batch - 2), dtype=np.int32)
    d = P.on_gpu(c)
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), c.k, c.v)
    P.attend(c, d, q=d.q_out)
    c.k, c.v = P.bits(d.k), P.bits(d.v)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c, q=P.bits(d.q_out)), P.slack(c))


def test_the_caches_own_order_without_strides():
    """Strides of 0: [rank][page][head][position][channel], the same bits as with the strides spelled out."""
    c = P.make(28, 2, 8, 4, [100, 33], [1, 1], 48)
    d, e = P.on_gpu(c), P.on_gpu(c)
    P.append(c, d)
    P.attend(c, d, q=d.q_out)
    c.desc.stride_rank = c.desc.stride_page = c.desc.stride_head = c.desc.stride_row = 0
    P.append(c, e)
    P.attend(c, e, q=e.q_out)
    assert all(np.array_equal(P.bits(getattr(d, x)), P.bits(getattr(e, x))) for x in ("q_out", "k", "v", "out"))


@pytest.mark.parametrize("hint", [1, 2, 5, 30, 400])
@pytest.mark.parametrize("e4m3", [False, True])
def test_any_number_of_new_tokens_whatever_max_new_says(hint, e4m3):
    """max_new chooses the kernel alone."""
    c = P.make(25, 1, 8, 2, [700, 40, 333, 0, 5], [90, 1, 33, 0, 5], 16, e4m3)
    c.desc.max_new = hint
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


def test_append_far_positions_and_wide_rows():
    """Positions up to 2^24 - 1 (the angle is carried beyond fp32), rows of qkv and q wider than their heads, other base."""
    far = [2 ** 24 - 16, 1000003, 131071]
    c = P.make(14, 1, 4, 2, [3, 2, 1], [3, 2, 1], 16, ld_q=4 * 128 + 40, ld_qkv=8 * 128 + 8)
    c.lens[:] = far                                      # behind every column of the table: rotated, and stored nowhere
    d = P.on_gpu(c)
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), c.k, c.v)
    c.desc.rope_base = 500000.0
    d = P.on_gpu(c)
    P.append(c, d)
    q, qs = P.ref_append(c, 500000.0)[:2]
    got, own = P.widen(P.bits(d.q_out)), ~np.isnan(q)
    assert np.all((np.abs(got - q) <= 2.0 ** -8 * np.abs(q) + 6e-6 * qs)[own])


def test_append_in_place():
    """q rotated where it lies: the same bits as into a buffer of its own, k and v of the rows as they were."""
    c = P.make(15, 2, 8, 2, [40, 9], [7, 3], 16)
    d, e = P.on_gpu(c), P.on_gpu(c)
    P.append(c, d)
    c.desc.ld_q = c.ld_qkv
    B.paged_append(c.desc, e.qkv, e.qkv, e.row_start, e.lens, e.table, e.k, e.v)
    got = P.bits(e.qkv)
    assert np.array_equal(got[:, :, :c.hpr * 128], P.bits(d.q_out)) and np.array_equal(got[:, :, c.hpr * 128:], c.qkv[:, :, c.hpr * 128:])
    assert np.array_equal(P.bits(e.k), P.bits(d.k)) and np.array_equal(P.bits(e.v), P.bits(d.v))


def test_append_e4m3_ends_of_the_range():
    """Beyond +-448 the largest code, NaN stays NaN, halves go to even, the smallest codes are there; scale 1 where none is given."""
    c = P.make(16, 1, 1, 1, [1], [1], 16, True, scales=False)
    vals = np.zeros(128, dtype=np.float32)
    vals[:12] = [1000.0, -1e30, np.inf, -np.inf, np.nan, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 448.0, 464.0]
    c.qkv[0, 0, 256:] = P.bf16(vals)
    c.qkv[0, 0, 260] = 0x7FC0
    d = P.on_gpu(c)
    d.ks = d.vs = None
    P.append(c, d)
    got = P.decode(P.view(c, P.bits(d.v))[0, c.table[0, 0], 0, 0], True)
    want = np.zeros(128)
    want[:12] = [448, -448, 448, -448, np.nan, 16, 20, 2.0 ** -9, 0, 2 * 2.0 ** -9, 448, 448]
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_what_no_query_sees_does_not_matter(e4m3, new):
    """NaN and infinities behind a sequence's length, in pages of nobody and in pages that are masked; lengths that end inside
    a page."""
    lens = [new + 5, new + 27, new + 48]
    c = P.make(17, 1, 4, 2, lens, [new] * 3, 32, e4m3)
    used = np.zeros((c.n_pages, c.page), dtype=bool)
    for b, x in enumerate(lens):
        for t in range(x):
            used[c.table[b, t // c.page], t % c.page] = True
    for x in (c.k, c.v):
        w = P.view(c, x)
        bad = [0x7F, 0xFF] if e4m3 else [0x7FC0, 0xFF80, 0x7F80, 0xFFFF]
        fill = np.resize(np.array(bad, dtype=x.dtype), w.shape)
        w[:, ~used.any(axis=1)] = fill[:, ~used.any(axis=1)]
        for page, off in zip(*np.where(~used)):
            w[:, page, :, off] = fill[:, page, :, off]
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("new", [1, 3, 6, 90])
@pytest.mark.parametrize("long", [70, 1200])
def test_infinities_that_are_seen(new, long):
    """An infinite value gives infinities of its sign in its channel (NaN where both signs meet) and leaves the other channels
    alone; an infinite key makes NaN of the rows that see it."""
    c = P.make(22, 1, 16, 2, [long + new, new + 33], [new, new], 16)
    w, k = P.view(c, c.v), P.view(c, c.k)
    at = lambda b, t: (c.table[b, t // 16], t % 16)
    (p0, o0), (p1, o1), (p2, o2) = at(0, 20), at(0, 37), at(1, 9)
    w[0, p0, 0, o0, 5], w[0, p1, 0, o1, 6], w[0, p0, 0, o0, 7], w[0, p1, 0, o1, 7] = 0x7F80, 0xFF80, 0x7F80, 0xFF80
    k[0, p2, 1, o2, 3] = 0x7F80
    d = P.on_gpu(c)
    P.attend(c, d)
    got = P.widen(P.bits(d.out)).reshape(1, -1, 16, 128)
    with np.errstate(invalid="ignore"):
        ref, size = (x.reshape(1, -1, 16, 128) for x in P.ref_attn(c))
    assert np.all(got[0, :new, :8, 5] == np.inf) and np.all(got[0, :new, :8, 6] == -np.inf) and np.all(np.isnan(got[0, :new, :8, 7]))
    with np.errstate(invalid="ignore"):
        q = P.widen(c.q)[0, new:].reshape(-1, 16, 128)[:, 8:, 3]
    assert np.all(np.isnan(got[0, new:, 8:]) | (q < 0)[:, :, None])          # + infinity: NaN; - infinity: a probability of 0
    fine = np.ones(got.shape, dtype=bool)
    fine[0, :new, :8, 5:8] = False
    fine[0, new:, 8:] = False
    got, ref, size = got[fine], ref[fine], size[fine]
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + P.slack(c) * size)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [1, 2, 90])
def test_lists_that_are_wrong(e4m3, new):
    """Entries that are no page, lengths below the number of new tokens, negative or behind the table, rows outside the packed
    ones: nothing outside is read or written, and what is left is computed."""
    lens = [new + 100, new + 40, new + 33, new + 64, new + 20, new + 7]
    c = P.make(18, 2, 4, 2, lens, [new] * 6, 16, e4m3, pad_rows=1)
    c.table[0, 2], c.table[0, 4] = -1, c.n_pages         # holes in the middle
    c.table[1, :] = 2 ** 31 - 1                          # no page at all
    c.lens[2] = new - 1                                  # its first token sits in front of position 0
    c.lens[3] = -5
    c.lens[4] = c.table.shape[1] * c.page + 3            # behind the last column
    c.table[4, :] = c.table[5, 0]
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))
    c.table[4, :] = -1                                   # (two tokens must not be appended to one place)
    d = P.on_gpu(c)
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), c.k, c.v)
    for wrong in ([-1, new, 2 * new, 3 * new, 4 * new, 5 * new, 6 * new], [0, new, new - 1, 2 ** 31 - 1, 4 * new, 4 * new, 6 * new + 2],
                  [0, 6 * new, 0, 6 * new, 0, 6 * new, 0], [0] + [6 * new] * 6):
        d = P.on_gpu(c)
        import torch
        d.row_start = torch.tensor(wrong, dtype=torch.int32, device="cuda")
        P.append(c, d)
        P.attend(c, d)
        got = P.widen(P.bits(d.out))
        owned = np.zeros(c.rows, dtype=bool)
        for r0, r1 in zip(wrong[:-1], wrong[1:]):
            if 0 <= r0 < r1 <= c.rows:
                owned[r0:r1] = True
        assert np.all(got[:, ~owned] == -7.0) and np.all(np.isfinite(got))


def test_without_a_list_of_rows():
    """row_start NULL: sequence b owns row b, the rows behind the last sequence nobody's."""
    c = P.make(19, 2, 8, 4, [33, 0, 200, 16], [1, 1, 1, 1], 16, pad_rows=3)
    ref, size = P.ref_attn(c)
    d = P.on_gpu(c)
    d.row_start = None
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), ref, size, P.slack(c))
    P.append(c, d)
    P.check_append(c, P.bits(d.q_out), P.bits(d.k), P.bits(d.v), c.k, c.v)


def test_no_rows():
    c = P.make(20, 1, 2, 2, [40, 3], [0, 0], 16)
    d = P.on_gpu(c)
    P.append(c, d)
    P.attend(c, d)
    assert np.all(P.widen(P.bits(d.out)) == -7.0) and np.array_equal(P.bits(d.k), c.k)


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_batch_that_grows_step_by_step(e4m3):
    """Prompts are appended and attended, then tokens one by one and two by two, pages handed out on the way: every output is
    that of the definition over what the caches hold, and what they hold is what the definition appends."""
    import torch
    T, heads, kv, page = 2, 8, 2, 16
    steps = [[70, 1, 33], [1, 1, 1], [1, 2, 1], [0, 14, 1], [2, 0, 2]]
    total = [sum(s[b] for s in steps) for b in range(3)]
    whole = P.make(21, T, heads, kv, total, total, page, e4m3)
    k, v, ws = None, None, None
    lens = [0, 0, 0]
    for i, news in enumerate(steps):
        lens = [x + n for x, n in zip(lens, news)]
        c = P.make(30 + i, T, heads, kv, lens, news, page, e4m3, spare=0, columns=whole.table.shape[1])
        c.n_pages, c.table, c.ks, c.vs = whole.n_pages, whole.table.copy(), whole.ks, whole.vs
        for b, x in enumerate(lens):
            c.table[b, -(-x // page):] = -1
        c.desc.n_pages = whole.n_pages
        c.desc.stride_rank, c.desc.stride_page = whole.desc.stride_rank, whole.desc.stride_page
        c.k, c.v = (whole.k, whole.v) if k is None else (k, v)
        d = P.on_gpu(c)
        P.append(c, d)
        P.attend(c, d, q=d.q_out)
        k, v = P.bits(d.k).copy(), P.bits(d.v).copy()
        P.check_append(c, P.bits(d.q_out), k, v, c.k, c.v)
        c.k, c.v = k, v
        P.check_attn(c, P.bits(d.out), *P.ref_attn(c, q=P.bits(d.q_out)), P.slack(c))


# 33 to 64 rows of a key / value head: two waves share 32 rows
DRAFTS = [
    (1, 8, 1, [500, 40, 0, 7], [8, 5, 0, 7], 16, False, "phrd"),             # 64, 40 and 56 rows
    (2, 16, 2, [700, 33, 64, 65, 1], [5, 1, 5, 5, 1], 48, False, "prhd"),
    (1, 1, 1, [32, 33, 64, 96, 97, 129], [32, 33, 64, 40, 50, 64], 16, False, "phrd"),   # blocks of which one half has no keys
    (2, 4, 4, [4100, 55], [50, 55], 80, False, "hprd"),                      # the keys of a tile dealt to many workgroups
    (1, 8, 1, [3001, 500, 8], [8, 6, 1], 32, True, "phrd"),
    (2, 6, 2, [200, 77, 20], [20, 21, 20], 16, True, "prhd"),                # 60 and 63 rows, groups of 3 heads
    (8, 64, 8, [(97 * i) % 613 for i in range(50)], [min((97 * i) % 613, 6) for i in range(50)], 16, False, "phrd"),   # 400 tiles
    (8, 64, 8, [(97 * i) % 613 for i in range(50)], [min((97 * i) % 613, 5) for i in range(50)], 32, True, "phrd"),
    (1, 2, 1, [2000 * (i % 2) + 25 for i in range(70)], [25 - i % 7 for i in range(70)], 64, False, "phrd"),
]


@pytest.mark.parametrize("T,heads,kv,lens,news,page,e4m3,order", DRAFTS)
def test_attention_of_drafts(T, heads, kv, lens, news, page, e4m3, order):
    c = P.make(40, T, heads, kv, lens, news, page, e4m3, order, pad_rows=2)
    d = P.on_gpu(c)
    P.attend(c, d)
    first = P.bits(d.out).copy()
    P.check_attn(c, first, *P.ref_attn(c), P.slack(c))
    for _ in range(3):
        d.out.fill_(-7.0)
        P.attend(c, d)
        assert np.array_equal(P.bits(d.out), first)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hint", [9, 16])
def test_more_new_tokens_than_max_new_says(hint, e4m3):
    """Tiles of 64 rows, several of a sequence."""
    c = P.make(41, 1, 8, 2, [3000, 40, 333, 0, 5], [190, 1, 33, 0, 5], 16, e4m3)
    c.desc.max_new = hint
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("e4m3", [False, True])
def test_what_no_query_of_a_draft_sees_does_not_matter(e4m3):
    """NaN and infinities behind a sequence's length, in pages of nobody and in both halves of a block; a page that is none in either."""
    lens, new = [6 + 20, 6 + 33, 6 + 90, 2100], 6
    c = P.make(42, 1, 8, 1, lens, [new] * 4, 16, e4m3)
    c.table[1, 0], c.table[2, 3], c.table[2, 4], c.table[3, 100] = -1, -1, c.n_pages, 2 ** 31 - 1
    used = np.zeros((c.n_pages, c.page), dtype=bool)
    for b, x in enumerate(lens):
        for t in range(x):
            if 0 <= c.table[b, t // c.page] < c.n_pages:
                used[c.table[b, t // c.page], t % c.page] = True
    for x in (c.k, c.v):
        w = P.view(c, x)
        bad = [0x7F, 0xFF] if e4m3 else [0x7FC0, 0xFF80, 0x7F80, 0xFFFF]
        fill = np.resize(np.array(bad, dtype=x.dtype), w.shape)
        for page, off in zip(*np.where(~used)):
            w[:, page, :, off] = fill[:, page, :, off]
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))


@pytest.mark.parametrize("new", [1, 16, 30, 90])
def test_rows_that_everybody_claims(new):
    """A list that gives all rows to 3000 sequences of 2^24 positions: more work than 31 bits count.  Nothing is written outside
    the packed rows, and nothing done at length."""
    import torch
    c = P.make(43, 1, 2, 1, [new] * 2, [new] * 2, 16, pad_rows=1)
    batch, columns = 6000, 1 << 10
    d = P.on_gpu(c)
    desc = B.paged_desc(T=1, batch=batch, n_heads=2, n_kv_heads=1, rows=c.rows, page_size=1 << 14, n_pages=c.n_pages,
                        max_pages=columns, max_new=new)
    rows = torch.tensor([0, c.rows - 1] * (batch // 2) + [0], dtype=torch.int32, device="cuda")
    lens = torch.full((batch,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    table = torch.full((batch, columns), -1, dtype=torch.int32, device="cuda")
    ws = torch.full((max(B.paged_attn_workspace_bytes(desc), 1),), 0x7B, dtype=torch.uint8, device="cuda")
    B.paged_attn(desc, d.q, d.out, rows, lens, table, d.k, d.v, ws)
    got = P.widen(P.bits(d.out))
    assert np.all(got[:, -1] == -7.0) and np.all((got == 0.0) | (got == -7.0))


@pytest.mark.parametrize("new,grp", [(2, 4), (4, 4), (3, 8), (8, 8), (33, 1), (40, 3), (150, 2)])
@pytest.mark.parametrize("long", [0, 70, 1500])
@pytest.mark.parametrize("e4m3", [False, True])
def test_what_later_tokens_hold_does_not_matter(new, grp, long, e4m3):
    """Values and keys of new tokens that are not finite: only the tokens from there on see them."""
    c = P.make(44, 1, 2 * grp, 2, [long + new, new + 33], [new, new], 16, e4m3)
    k, v = P.view(c, c.k), P.view(c, c.v)
    mid, last = new // 2, new - 1
    nan, inf = (0x7F, 0xFF) if e4m3 else (0x7FC0, 0xFF80)
    odd = np.zeros((2 * new, 2 * grp, 128), dtype=bool)
    poison = []
    for b in range(2):
        at = lambda i: (c.table[b, (c.lens[b] - new + i) // 16], (c.lens[b] - new + i) % 16)
        (p0, o0), (p1, o1) = at(mid), at(last)
        poison += [(p0, 0, o0, 5, nan), (p0, 0, o0, 77, inf), (p0, 1, o0, 100, inf)] + [(p1, 0, o1, x, nan) for x in range(128)]
        odd[b * new + mid:(b + 1) * new, :grp, [5, 77]] = True
        odd[b * new + mid:(b + 1) * new, grp:, 100] = True
        odd[b * new + last, :grp] = True
        k[0, p1, 1, o1, 3] = nan
        odd[b * new + last, grp:] = True
    for p, h, o, x, _ in poison:
        v[0, p, h, o, x] = 0
    ref, size = (x.reshape(2 * new, 2 * grp, 128)[~odd] for x in P.ref_attn(c))
    for p, h, o, x, code in poison:
        v[0, p, h, o, x] = code
    d = P.on_gpu(c)
    P.attend(c, d)
    first = P.bits(d.out).copy()
    got = P.widen(first).reshape(2 * new, 2 * grp, 128)
    assert not np.any(np.isfinite(got[odd]))
    assert np.all(np.abs(got[~odd] - ref) <= 2.0 ** -8 * np.abs(ref) + P.slack(c) * size)
    d.out.fill_(-7.0)
    P.attend(c, d)
    assert np.array_equal(P.bits(d.out), first)


@pytest.mark.parametrize("T,heads,kv,new,e4m3", [(8, 64, 8, 5, False), (8, 64, 8, 5, True), (4, 16, 16, 40, False), (8, 64, 8, 9, True), (1, 8, 8, 80, False)])
def test_a_long_line_of_tiles(T, heads, kv, new, e4m3):
    """More tiles than workgroups, of many sequences with lengths far apart, free slots among them."""
    lens = [(397 * i) % 1700 + 1 if i % 7 else 0 for i in range(70)]
    lens[33] = 3500
    news = [min(x, 1 + (i * 5) % new) if i % 3 else min(x, new) for i, x in enumerate(lens)]
    c = P.make(45, T, heads, kv, lens, news, 32, e4m3, pad_rows=1)
    d = P.on_gpu(c)
    P.attend(c, d)
    first = P.bits(d.out).copy()
    P.check_attn(c, first, *P.ref_attn(c), P.slack(c))
    d.out.fill_(-7.0)
    P.attend(c, d)
    assert np.array_equal(P.bits(d.out), first)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("batch,keys,new", [(70, 60, 3), (70, 300, 4), (5, 300, 4), (5, 30, 4), (9, 900, 3)])
def test_drafts_over_short_tables(batch, keys, new, e4m3):
    """17 to 32 rows of a key / value head, in more and in fewer units than a launch has workgroups."""
    lens = [keys - (11 * i) % (keys - new) for i in range(batch)]
    c = P.make(46, 8, 64, 8, lens, [new - i % 2 for i in range(batch)], 16, e4m3, pad_rows=1)
    d = P.on_gpu(c)
    P.attend(c, d)
    P.check_attn(c, P.bits(d.out), *P.ref_attn(c), P.slack(c))
