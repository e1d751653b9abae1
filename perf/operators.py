"""The operators over a paged key / value cache, as cases that can be timed and compared.

  append   caat_paged_append: the new tokens' q and k are rotated to their positions, k and v stored to their pages
  attend   caat_paged_attn: causal attention of every sequence's new tokens over its pages (its own tokens among them)

A cache is a pool of pages per tensor-parallel rank, [T][pages][key / value heads of a rank][page size][128], in bfloat16 or
in e4m3 with one fp32 scale per rank and head.  The ranks share the page table [batch][columns].  The new tokens of all
sequences are packed into rows: sequence b has rows row_start[b] .. row_start[b + 1] - 1, and lens[b] cached positions
with them.  Queries, keys and values are N(0, 1), as in the other cases of the library; head dimension 128.
"""
import math
import random

import torch

own = False   # True: the library's kernels, False: plain torch in 32 bits

D = 128
BASE = 10000.0


def _case(name, op, T, heads, kv_heads, batch, ctx, new, page, cache="bf16", ragged=False):
    """ctx: cached positions of the longest sequence, the new ones among them; new: new tokens of the sequence that has
    most; ragged: the others have fewer of both, one has none."""
    return dict(name=name, op=op, T=T, heads=heads, kv_heads=kv_heads, batch=batch, ctx=ctx, new=new, page=page, cache=cache,
                ragged=ragged)


def listed():
    return [
        # Interactive serving: the one new token of one sequence.
        _case("append_one", "append", 8, 32, 32, 1, 777, 1, 16),
        # A decode step of a full server into an 8-bit cache, 70B-shape heads.
        _case("append_step_e4m3", "append", 8, 64, 8, 128, 4096, 1, 64, "e4m3", True),
        # Prompts of different lengths that arrive together.
        _case("append_prompts", "append", 8, 32, 32, 9, 2048, 2048, 16, "bf16", True),
        # Interactive serving, short cache: latency.
        _case("attend_one", "attend", 8, 32, 32, 1, 300, 1, 16),
        # 64 sequences of 2048, 7B heads: the benchmark's decode step over pages.
        _case("attend_7b_b64", "attend", 8, 32, 32, 64, 2048, 1, 64),
        # A server's mix: short and long conversations, grouped-query heads, small pages.
        _case("attend_70b_ragged", "attend", 8, 64, 8, 48, 16384, 1, 16, "bf16", True),
        # One very long document.
        _case("attend_long_one", "attend", 4, 32, 8, 1, 131072, 1, 256),
        # The mix over an 8-bit cache.
        _case("attend_e4m3_ragged", "attend", 8, 64, 8, 64, 8191, 1, 32, "e4m3", True),
        # Drafted tokens checked in one step: up to 5 per sequence.
        _case("attend_drafts", "attend", 8, 64, 8, 24, 6000, 5, 16, "bf16", True),
        # Prompts of 2048, 7B heads: time to first token.
        _case("attend_prompts_7b", "attend", 8, 32, 32, 4, 2048, 2048, 64),
        # Chunks of prompts of odd lengths behind what is cached already, pages that no tile is a multiple of.
        _case("attend_chunks_ragged", "attend", 4, 16, 8, 6, 5003, 701, 48, "bf16", True),
        # A chunk of a long prompt, 8-bit cache.
        _case("attend_chunk_e4m3", "attend", 8, 64, 8, 1, 16384, 512, 128, "e4m3"),
    ]


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend"])
    T = rng.choice([1, 2, 4, 8])
    heads = rng.choice([8, 16, 24, 32, 64])
    kv_heads = rng.choice([k for k in (heads, heads // 2, heads // 4, heads // 8) if k >= T and k % T == 0])
    batch, ctx = _log(rng, 1, 128), _log(rng, 1, 65536)
    new = min(ctx, rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 2048)]))
    return _case("", op, T, heads, kv_heads, batch, ctx, new, rng.choice([16, 32, 48, 64, 80, 128, 256]),
                 rng.choice(["bf16", "bf16", "e4m3"]), rng.random() < 0.7)


def _cost(case):
    w = work(case)
    return w["flops"] / 2.5e15 + w["bytes"] / 8e12


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        n, L = _lengths(c)
        pool = sum(-(-x // c["page"]) for x in L) * c["page"] * c["kv_heads"] * D
        wide = c["batch"] * c["ctx"] * (c["kv_heads"] * D + c["heads"] * c["new"])   # what the plain form pads to
        if _cost(c) <= most and pool <= 1 << 30 and wide <= 1 << 31 and sum(n) <= 32768:
            del c["name"]
            return c


# ---------------------------------------------------------------- state
def _lengths(c):
    """New tokens and cached positions of every sequence: a property of the case, whatever the seed."""
    b, most, ctx = c["batch"], c["new"], c["ctx"]
    n, L = [most] * b, [ctx] * b
    if c["ragged"]:
        rng = random.Random(1000003 * ctx + 1009 * most + b)
        for i in range(1, b):
            n[i] = rng.randint(1, most)
            L[i] = max(n[i], _log(rng, max(1, ctx // 64), ctx))
        if b >= 4:
            n[2] = L[2] = 0              # a slot of the batch that is free
            n[3], L[3] = 1, 1            # a sequence that begins
    return n, L


def _plan(c):
    """What a program keeps for calls of these sizes."""
    from paper_2506_19645_amd import binding as B
    n, L = _lengths(c)
    desc = B.paged_desc(T=c["T"], batch=c["batch"], n_heads=c["heads"], n_kv_heads=c["kv_heads"], rows=_rows(n), max_new=c["new"],
                        page_size=c["page"], n_pages=_pages(c, L), max_pages=_columns(c),
                        cache_type=B.CACHE_E4M3 if c["cache"] == "e4m3" else B.CACHE_BF16, rope_base=BASE)
    ws = torch.empty(B.paged_attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda") if c["op"] == "attend" else None
    return B, desc, ws


def _rows(n):
    return -(-sum(n) // 8) * 8 if len(n) > 1 else sum(n)      # a batch is padded, its last rows belong to nobody


def _pages(c, L):
    return sum(-(-x // c["page"]) for x in L) + 3


def _columns(c):
    return -(-c["ctx"] // c["page"])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    n, L = _lengths(c)
    T, page, rows, pages = c["T"], c["page"], _rows(n), _pages(c, L)
    kvpr, hd = c["kv_heads"] // T, c["heads"] // T * D
    # the pages of the pool in the order in which they were handed out
    free = torch.randperm(pages, generator=gen, device="cuda").tolist()
    table = [[free.pop() if k * page < x else -1 for k in range(_columns(c))] for x in L]
    starts = [sum(n[:i]) for i in range(len(n) + 1)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    s = {"case": c, "row_start": ints(starts), "lens": ints(L), "table": ints(table), "k_scale": None, "v_scale": None,
         "k": normal(T, pages, kvpr, page, D), "v": normal(T, pages, kvpr, page, D)}
    if c["cache"] == "e4m3":
        for x in "kv":
            # the largest of N(0, 1) values lies near 4.5 and e4m3 ends at 448
            scale = 0.01 + 0.004 * torch.rand((T, kvpr), generator=gen, device="cuda")
            s[x + "_scale"] = scale
            s[x] = (s[x] / scale[:, None, :, None, None].bfloat16()).clamp(-448, 448).to(torch.float8_e4m3fn)
    if c["op"] == "append":
        s["qkv"] = normal(T, rows, hd + 2 * kvpr * D)
        s["q"] = torch.zeros((T, rows, hd), dtype=torch.bfloat16, device="cuda")
    else:
        s["q"] = normal(T, rows, hd)
        s["out"] = torch.zeros((T, rows, hd), dtype=torch.bfloat16, device="cuda")
    if own:
        s["plan"] = _plan(c)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    s = state
    if own:
        B, desc, ws = s["plan"]
        if s["case"]["op"] == "append":
            B.paged_append(desc, s["qkv"], s["q"], s["row_start"], s["lens"], s["table"], s["k"], s["v"], s["k_scale"], s["v_scale"])
        else:
            B.paged_attn(desc, s["q"], s["out"], s["row_start"], s["lens"], s["table"], s["k"], s["v"], ws, s["k_scale"], s["v_scale"])
    elif s["case"]["op"] == "append":
        _append(s)
    else:
        _attend(s)
    return {"q": s["q"], "k": s["k"], "v": s["v"]} if s["case"]["op"] == "append" else s["out"]


def _row_map(s, rows):
    """Sequence, index inside its new tokens, position and validity of every packed row."""
    r = torch.arange(rows, device="cuda")
    start = s["row_start"].long()
    b = torch.searchsorted(start[1:].contiguous(), r, right=True).clamp(max=start.numel() - 2)
    j = r - start[b]
    pos = s["lens"].long()[b] - (start[b + 1] - start[b]) + j
    return b, j, pos, r < start[-1]


def _append(s):
    c = s["case"]
    T, page = c["T"], c["page"]
    kvpr, hpr = c["kv_heads"] // T, c["heads"] // T
    rows = s["qkv"].shape[1]
    b, _, pos, ok = _row_map(s, rows)
    freq = BASE ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    angle = pos.double()[:, None] * freq
    cs, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]          # [rows, 1, 64]
    x = s["qkv"].float().view(T, rows, hpr + 2 * kvpr, D)
    lo, hi = x[:, :, :hpr + kvpr, :D // 2], x[:, :, :hpr + kvpr, D // 2:]
    rot = torch.cat((lo * cs - hi * sn, hi * cs + lo * sn), dim=-1)
    q = rot[:, :, :hpr].reshape(T, rows, hpr * D).bfloat16()
    s["q"].copy_(torch.where(ok[None, :, None], q, s["q"]))
    where = s["table"].long()[b, (pos // page).clamp(min=0)]
    # rows that belong to nobody write the first row's values to the first row's place once more
    where, off, row = (torch.where(ok, t, t[0]) for t in (where, pos % page, torch.arange(rows, device="cuda")))
    for name, new in (("k", rot[:, :, hpr:]), ("v", x[:, :, hpr + kvpr:])):
        if s[name + "_scale"] is not None:
            new = (new / s[name + "_scale"][:, None, :, None]).clamp(-448, 448)
        new = new[:, row].to(s[name].dtype)                                       # [T, rows, kvpr, D]
        if new.dtype == torch.float8_e4m3fn:
            s[name].view(torch.uint8)[:, where, :, off] = new.view(torch.uint8).transpose(0, 1)
        else:
            s[name][:, where, :, off] = new.transpose(0, 1)


def _attend(s):
    c = s["case"]
    T, page, batch, most = c["T"], c["page"], c["batch"], c["new"]
    kvpr, grp = c["kv_heads"] // T, c["heads"] // c["kv_heads"]
    rows = s["q"].shape[1]
    start, lens = s["row_start"].long(), s["lens"].long()
    n = start[1:] - start[:-1]
    j = torch.arange(most, device="cuda")
    token = (start[:-1, None] + j).clamp(max=rows - 1)                            # [batch, most]
    q = s["q"].view(T, rows, kvpr, grp, D)[:, token].float()                      # [T, batch, most, kvpr, grp, D]
    q = q.permute(0, 1, 3, 2, 4, 5).reshape(T, batch, kvpr, most * grp, D)
    idx = s["table"].long().clamp(min=0)

    def rows_of(x, scale):
        if x.dtype == torch.float8_e4m3fn:
            x = x.view(torch.uint8)[:, idx].view(torch.float8_e4m3fn)
        else:
            x = x[:, idx]
        x = x.float().permute(0, 1, 3, 2, 4, 5).reshape(T, batch, kvpr, -1, D)    # from [T, batch, columns, kvpr, page, D]
        return x if scale is None else x * scale[:, None, :, None, None]

    score = torch.matmul(q, rows_of(s["k"], s["k_scale"]).transpose(-1, -2)) / math.sqrt(D)
    key = torch.arange(score.shape[-1], device="cuda")
    see = (key <= ((lens - n)[:, None] + j)[:, :, None]) & (j < n[:, None])[:, :, None]      # [batch, most, keys]
    see = see[:, :, None].expand(-1, -1, grp, -1).reshape(batch, 1, most * grp, -1)
    score = score.masked_fill(~see, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    den = p.sum(-1, keepdim=True)
    o = torch.matmul(p, rows_of(s["v"], s["v_scale"])) / torch.where(den == 0, 1.0, den)
    o = o.view(T, batch, kvpr, most, grp, D)
    b, i, _, ok = _row_map(s, rows)
    o = o.permute(1, 3, 0, 2, 4, 5)[b, i.clamp(max=most - 1)]                     # [rows, T, kvpr, grp, D]
    o = o.transpose(0, 1).reshape(T, rows, -1).bfloat16()
    s["out"].copy_(torch.where(ok[None, :, None], o, s["out"]))


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """append: every row read, q and the pages' rows written.  attend: q and the cached rows of every sequence read, the
    heads written; two products per query head and key that it sees."""
    c = case
    n, L = _lengths(c)
    elt = 1 if c["cache"] == "e4m3" else 2
    hd, kvd, tokens = c["heads"] * D, c["kv_heads"] * D, sum(n)
    if c["op"] == "append":
        return {"bytes": tokens * (4 * hd + 4 * kvd + 2 * kvd * elt), "flops": tokens * 6 * (hd + kvd)}
    pairs = sum(m * (x - m) + m * (m + 1) // 2 for m, x in zip(n, L))
    return {"bytes": tokens * 4 * hd + sum(L) * 2 * kvd * elt, "flops": 4 * hd * pairs}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    n, L = _lengths(c)
    T, page = c["T"], c["page"]
    kvpr, hpr = c["kv_heads"] // T, c["heads"] // T
    grp = hpr // kvpr
    table = s["table"].tolist()
    one = torch.ones((T, kvpr), dtype=torch.float64, device="cuda")
    ks, vs = (one if s[x] is None else s[x].double() for x in ("k_scale", "v_scale"))
    first = 0
    if c["op"] == "append":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        freq = torch.tensor([BASE ** (-2.0 * i / D) for i in range(D // 2)], dtype=torch.float64, device="cuda")
        limit = 448.0 if c["cache"] == "e4m3" else math.inf
        for b, (m, x) in enumerate(zip(n, L)):
            if m == 0:
                continue
            pos = torch.arange(x - m, x, device="cuda")
            turn = torch.polar(torch.ones_like(freq).expand(m, -1), pos.double()[:, None] * freq)      # e^(i angle), [m, 64]
            rows = s["qkv"][:, first:first + m].double()
            z = rows.view(T, m, hpr + 2 * kvpr, 2, D // 2)
            z = torch.complex(z[:, :, :, 0].contiguous(), z[:, :, :, 1].contiguous())
            w = z * turn[:, None]
            w = torch.cat((w.real, w.imag), dim=-1)                              # [T, m, heads, 128]
            q[:, first:first + m] = w[:, :, :hpr].reshape(T, m, hpr * D)
            at = torch.tensor([table[b][p // page] for p in range(x - m, x)], device="cuda")
            for h in range(kvpr):
                for t in range(T):
                    k[t, at, h, pos % page] = (w[t, :, hpr + h] / ks[t, h]).clamp(-limit, limit)
                    v[t, at, h, pos % page] = (rows[t, :, (hpr + kvpr + h) * D:(hpr + kvpr + h + 1) * D] / vs[t, h]).clamp(-limit, limit)
            first += m
        return {"q": q, "k": k, "v": v}
    out = s["out"].double()
    for b, (m, x) in enumerate(zip(n, L)):
        if m == 0:
            continue
        pages = torch.tensor(table[b][:-(-x // page)], device="cuda")
        hidden = torch.arange(x, device="cuda") > torch.arange(x - m, x, device="cuda")[:, None]
        for t in range(T):
            for h in range(kvpr):
                k = s["k"][t, :, h].view(torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16)[pages].view(s["k"].dtype)
                v = s["v"][t, :, h].view(torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16)[pages].view(s["v"].dtype)
                k = k.double().reshape(-1, D)[:x] * ks[t, h]
                v = v.double().reshape(-1, D)[:x] * vs[t, h]
                q = s["q"][t, first:first + m].double().view(m, hpr, D)[:, h * grp:(h + 1) * grp]
                a = torch.einsum("mgd,xd->gmx", q, k) * D ** -0.5
                a = torch.softmax(a.masked_fill(hidden, -math.inf), dim=-1)
                o = torch.matmul(a, v).transpose(0, 1)                          # [m, grp, D]
                out[t, first:first + m, h * grp * D:(h + 1) * grp * D] = o.reshape(m, grp * D)
        first += m
    return out
