"""Performance cases of the operators that serve from a committed cache of 8 bits.

A case is a dict of plain values.  Its "kind" names the calls of one pass:

  pages    page tables and slot maps from request lengths: the lengths of one
           scheduling step are taken back and set again (two calls of
           ``carryover_assign_pages``), then every new row's position and slot
           (``carryover_slot_map``)
  store    rows of keys and values written to their slots of the 8-bit cache
           (``carryover_store_kv8``)
  attend   block attention over [C;U], C in the 8-bit cache, with or without
           the block's own rows (``drafter_block_attention_kv8``)

A page of the cache holds 16 tokens of one layer and KV head: keys [16][hd] and
values [hd][16] as e4m3 codes, with one scale byte b each, code * 2^(b - 127).
Without ``own``, ``run`` computes the same in elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 16
BIAS = 127                         # of the scale bytes
LARGEST = 1.75                     # of e4m3, over 2^8
SMALLEST = -126                    # exponent of the smallest scale
F8 = torch.float8_e4m3fn


# ------------------------------------------------------------------ the cases

def _heads(L, Hq, Hkv, hd, theta):
    return dict(L=L, Hq=Hq, Hkv=Hkv, hd=hd, theta=theta)


def _attend(name, S, B, lo, hi, reject, heads, own_rows=False):
    return dict(name=name, kind="attend", S=S, B=B, ctx_lo=lo, ctx_hi=hi, reject=reject,
                own_rows=own_rows, **heads)


def listed():
    large = _heads(1, 32, 8, 128, 1e6)
    return [
        # one request of a short prompt enters an idle server: launches and latency
        dict(name="pages_one", kind="pages", S=1, lo=37, hi=37, most=37, turn=1.0, reserve=0),
        # a decoding batch: every sequence commits up to a block, room for the next one is kept
        dict(name="pages_decode32", kind="pages", S=32, lo=512, hi=8192, most=16, turn=0.0,
             reserve=16),
        # a busy server: half of 256 requests end, the others' prompts enter
        dict(name="pages_turn256", kind="pages", S=256, lo=1, hi=8192, most=8192, turn=1.0,
             reserve=16),
        # one token of a small drafter, in the middle of a page: latency
        dict(name="store_token", kind="store", rows="window", S=1, B=1, ctx_lo=21, ctx_hi=21,
             reject=0.0, **_heads(1, 4, 2, 64, 1e4)),
        # a round's committed rows of 32 sequences, all layers of a large drafter
        dict(name="store_round32_5layer", kind="store", rows="window", S=32, B=16, ctx_lo=512,
             ctx_hi=8192, reject=0.25, **_heads(5, 32, 8, 128, 1e6)),
        # ragged prompts of a large drafter, packed row behind row: memory traffic
        dict(name="store_prompts", kind="store", rows="packed", S=13, B=1, ctx_lo=1, ctx_hi=2500,
             reject=0.0, **_heads(5, 32, 8, 128, 1e6)),
        # one token of one short stream: the smallest call
        _attend("attend_token", 1, 1, 300, 300, 1.0, _heads(1, 4, 2, 64, 1e4)),
        # one interactive stream's block
        _attend("attend_block_batch1", 1, 16, 2048, 2048, 0.25, large),
        # single tokens of a large serving batch
        _attend("attend_tokens_batch64", 64, 1, 100, 4000, 1.0, large),
        # the serving batch: 32 ragged contexts, 16 rows each
        _attend("attend_block_batch32", 32, 16, 512, 8192, 0.25, large),
        # long contexts and five drafter layers: the most memory traffic
        _attend("attend_long_5layer", 16, 16, 16384, 32768, 0.3, _heads(5, 32, 8, 128, 1e6)),
        # odd sizes: 7 rows with their own keys, three query heads per KV head,
        # contexts from none at all
        _attend("attend_odd_own_rows", 11, 7, 0, 1500, 0.2, _heads(2, 12, 4, 128, 1e6), True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng, B):
    Hkv = rng.choice((1, 2, 3, 4, 8))
    G = rng.choice([g for g in (1, 2, 3, 4, 6, 8) if B * g <= 64])
    return _heads(rng.choice((1, 1, 2, 3, 5)), G * Hkv, Hkv, rng.choice((64, 128)),
                  rng.choice((1e4, 1e6)))


def draw(rng):
    kind = rng.choice(("pages", "store", "store", "attend", "attend", "attend"))
    if kind == "pages":
        S = _log(rng, 1, 1024)
        hi = _log(rng, 16, max(16, min(16384, 2 ** 21 // S)))
        return dict(kind=kind, S=S, lo=rng.randint(1, hi), hi=hi, most=_log(rng, 1, hi),
                    turn=rng.choice((0.0, 0.1, 0.5, 1.0)), reserve=rng.choice((0, 16, 7)))
    B = rng.choice((1, 16, 16, 8, rng.randint(1, 32)))
    heads = _draw_heads(rng, B)
    S = _log(rng, 1, 64)
    if kind == "store":
        rows = rng.choice(("window", "packed"))
        most = 16384 * 5 * 8 * 128 // (heads["L"] * heads["Hkv"] * heads["hd"]) // S
        hi = _log(rng, 16, max(16, min(8192, most)))
        return dict(kind=kind, rows=rows, S=S, B=B if rows == "window" else 1,
                    ctx_lo=rng.randint(1, hi), ctx_hi=hi, reject=round(rng.uniform(0.05, 0.5), 2),
                    **heads)
    cap = int(1.5e9 / (2 * heads["L"] * heads["Hkv"] * heads["hd"] * S))
    hi = _log(rng, 16, max(16, min(65536, cap)))
    return dict(kind=kind, S=S, B=B, ctx_lo=rng.randint(0, hi), ctx_hi=hi,
                reject=round(rng.uniform(0.05, 0.5), 2), own_rows=rng.random() < 0.3, **heads)


# ------------------------------------------------------------- common pieces

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lengths(c, seed):
    """Committed lengths: spread evenly over the case's range, in a seeded order."""
    S, lo, hi = c["S"], c["ctx_lo"], c["ctx_hi"]
    n = [hi if S == 1 else lo + (hi - lo) * i // (S - 1) for i in range(S)]
    random.Random(seed).shuffle(n)
    return n


def _accepted(c, seed):
    """Accepted prefix lengths: every position rejected with probability ``reject``."""
    r = random.Random(seed + 1)
    return [next((j for j in range(c["B"]) if r.random() < c["reject"]), c["B"])
            for _ in range(c["S"])]


def _page_rows(pages, max_pages, seed):
    """Rows of distinct page ids in a random order; unused entries 0."""
    ids = list(range(sum(pages)))
    random.Random(seed + 2).shuffle(ids)
    rows, at = [], 0
    for n in pages:
        rows.append(ids[at:at + n] + [0] * (max_pages - n))
        at += n
    return rows, max(1, len(ids))


def _exponent(a):
    """Exponent of the smallest power of two 2^k with a <= 448 * 2^k, from SMALLEST on."""
    m, e = torch.frexp(a)                                   # a = m * 2^e, m in [0.5, 1)
    k = e - 9 + (2 * m > LARGEST)
    return torch.where(a > 0, k, SMALLEST).clamp_min(SMALLEST)


def _power(k):
    """2^k in 32 bits, exactly (the exponent's bits)."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _code(x, k):
    """e4m3 codes of x * 2^-k, as bytes."""
    return (x * _power(-k)).to(F8).view(torch.uint8)


def _value(codes, b):
    """The 32-bit values that codes with scale bytes b stand for."""
    return codes.view(F8).float() * _power(b.int() - BIAS)


def _filled(c, pages, g):
    """Keys and values of earlier tokens in every page: codes and scales.  Heads differ
    in magnitude by up to a factor of four, as heads do."""
    L, H, hd = c["L"], c["Hkv"], c["hd"]
    cache = dict(k_pages=torch.empty((L, pages, H, PAGE, hd), dtype=torch.uint8, device="cuda"),
                 v_pages=torch.empty((L, pages, H, hd, PAGE), dtype=torch.uint8, device="cuda"),
                 k_scale=torch.empty((L, pages, H), dtype=torch.uint8, device="cuda"),
                 v_scale=torch.empty((L, pages, H), dtype=torch.uint8, device="cuda"))
    for layer in range(L):
        for x in ("k", "v"):
            to = cache[x + "_pages"][layer]
            size = torch.exp2(2 * torch.rand((1, H, 1, 1), generator=g, device="cuda") - 1)
            rows = size * torch.randn(to.shape, generator=g, device="cuda")
            k = _exponent(rows.abs().amax((2, 3)))
            to.copy_(_code(rows, k[..., None, None]))
            cache[x + "_scale"][layer] = (k + BIAS).to(torch.uint8)
    return cache


def _rotate(x, pos, theta):
    """Rotate-half pairs (i, i + hd/2) of x [..., hd] at pos, in 64 bits."""
    half = x.shape[-1] // 2
    inv = theta ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    ang = pos.double()[..., None] * inv
    cs, sn = torch.cos(ang), torch.sin(ang)
    lo, hi = x[..., :half].double(), x[..., half:].double()
    return torch.cat((lo * cs - hi * sn, hi * cs + lo * sn), -1)


# ----------------------------------------------------------------- prepare

def prepare(case, seed):
    return {"pages": _prepare_pages, "store": _prepare_store,
            "attend": _prepare_attend}[case["kind"]](case, seed)


def _prepare_pages(c, seed):
    """Lengths before and after one step, and the tables as the step left them."""
    r, S = random.Random(seed), c["S"]
    n = [c["hi"] if S == 1 else c["lo"] + (c["hi"] - c["lo"]) * i // (S - 1) for i in range(S)]
    step, change = [], random.Random(c["hi"])           # the same lengths for every seed
    change.shuffle(n)
    for i, x in enumerate(n):
        if change.random() < c["turn"]:                 # one enters, the next one ends
            step.append((0, min(x, c["most"])) if i % 2 == 0 else (x, 0))
        else:
            step.append((x, x + change.randint(1, c["most"])))
    r.shuffle(step)
    before, after = [x for x, _ in step], [x for _, x in step]
    width = lambda x: -(-(x + c["reserve"]) // PAGE) if x else 0  # noqa: E731
    held = [width(x) for x in before]
    max_pages = max(1, max(width(x) for x in before + after)) + 1
    rows, _ = _page_rows(held, max_pages, seed)
    rows = [row[:h] + [-1] * (max_pages - h) for row, h in zip(rows, held)]
    spare = 64 + max(0, sum(width(x) for x in after) - sum(held))
    pages = sum(held) + spare
    free = list(range(sum(held), pages))
    r.shuffle(free)
    new = [max(0, a - b) for a, b in zip(after, before)]
    start = [0]
    for x in new:
        start.append(start[-1] + x)
    s = dict(case=c, max_pages=max_pages, num_pages=pages, num_rows=start[-1], before=_int(before),
             after=_int(after), row_start=_int(start),
             pool=dict(page_table=_int(rows), held=_int(held),
                       free_pages=_int(free + [-1] * sum(held)), free_count=_int([len(free)])),
             row_pos=torch.zeros(start[-1], dtype=torch.int32, device="cuda"),
             row_dst=torch.zeros(start[-1], dtype=torch.int32, device="cuda"), status=_int([0]))
    _plain_assign(s["pool"], s["after"], c["reserve"])
    return s


def _prepare_store(c, seed):
    g, S, B = _gen(seed), c["S"], c["B"]
    n = _lengths(c, seed)
    if c["rows"] == "packed":                           # whole prompts, from position 0 on
        pages = [-(-x // PAGE) for x in n]
        pos = [(s, t) for s, x in enumerate(n) for t in range(x)]
    else:                                               # each window's accepted rows
        pages = [(x + B) // PAGE + 1 for x in n]
        pos = [(s, n[s] + j if j < m else None) for s, m in enumerate(_accepted(c, seed))
               for j in range(B)]
    table, total = _page_rows(pages, max(pages), seed)
    first = next((t for t in pos if t[1] is not None), None)
    if first is None:                                   # at least one row is accepted
        pos[0] = (0, n[0])
    dst = [-2 ** 31 if t is None else table[s][t // PAGE] * PAGE + t % PAGE for s, t in pos]
    shape = (c["L"], len(pos), c["Hkv"], c["hd"])
    row = lambda: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    return dict(case=c, num_pages=total, max_pages=max(pages), num_rows=len(pos), k_rows=row(),
                v_rows=row(), row_dst=_int(dst), cache=_filled(c, total, g), status=_int([0]))


def _prepare_attend(c, seed):
    g, S, B, L, H, hd = _gen(seed), c["S"], c["B"], c["L"], c["Hkv"], c["hd"]
    n = _lengths(c, seed)
    pages = [-(-x // PAGE) + 1 for x in n]
    max_pages = -(-c["ctx_hi"] // PAGE) + 4
    table, total = _page_rows(pages, max_pages, seed)
    CP = -(-B // PAGE)
    norm = lambda *shape: (torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
                           .normal_(generator=g))
    return dict(case=c, num_pages=total, max_pages=max_pages, ctx_len=_int(n),
                carry_len=_int([B - m for m in _accepted(c, seed)]), page_table=_int(table),
                cache=_filled(c, total, g), k_carry=norm(L, S, CP, H, PAGE, hd),
                v_carry=norm(L, S, CP, H, hd, PAGE), q=norm(L, S, B, c["Hq"], hd),
                k_self=norm(L, S, B, H, hd) if c["own_rows"] else None,
                v_self=norm(L, S, B, H, hd) if c["own_rows"] else None, status=_int([0]))


# --------------------------------------------------------------------- run

def run(state):
    if own:
        return {"pages": _own_pages, "store": _own_store,
                "attend": _own_attend}[state["case"]["kind"]](state)
    return {"pages": _plain_pages, "store": _plain_store,
            "attend": _plain_attend}[state["case"]["kind"]](state)


def _pages_out(s):
    return dict(s["pool"], row_pos=s["row_pos"], row_dst=s["row_dst"], status=s["status"])


def _store_out(s):
    """The cache: codes as the values they stand for under their scales."""
    c = s["cache"]
    return dict(k=c["k_pages"].view(F8), v=c["v_pages"].view(F8), k_scale=c["k_scale"],
                v_scale=c["v_scale"], status=s["status"])


# ------------------------------------------------- the framework's own calls

def _handle(s, B, rows_of):
    """Dims, workspace and buffers that a program keeps over its calls."""
    import paper_2609_14717_amd as co
    if "dims" not in s:
        c = s["case"]
        h = c if "hd" in c else _heads(1, 1, 1, 64, 1e4)
        d = co.make_dims(c["S"], B, 64, 64, h["L"], h["Hq"], h["Hkv"], h["hd"], s["max_pages"],
                         s["num_pages"], "bf16", h["theta"])
        size = co.workspace_bytes(d, rows_of(co)) if rows_of else 0
        s["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")
        if "q" in s:
            s["out"] = torch.empty_like(s["q"])
            s["state"] = dict(ctx_len=s["ctx_len"], carry_len=s["carry_len"],
                              page_table=s["page_table"], k_cache=None, v_cache=None,
                              k_carry=s["k_carry"], v_carry=s["v_carry"], status=s["status"])
        s["dims"] = d
    return co


def _own_pages(s):
    co = _handle(s, 1, lambda co: co.CO_WS_ASSIGN_PAGES)
    keep = s["case"]["reserve"]
    co.carryover_assign_pages(s["dims"], s["before"], keep, s["pool"], s["status"], s["ws"])
    co.carryover_assign_pages(s["dims"], s["after"], keep, s["pool"], s["status"], s["ws"])
    co.carryover_slot_map(s["dims"], s["num_rows"], s["row_start"], s["before"],
                          s["pool"]["page_table"], s["row_pos"], s["row_dst"], s["status"])
    return _pages_out(s)


def _own_store(s):
    co = _handle(s, s["case"]["B"], None)
    co.carryover_store_kv8(s["dims"], s["num_rows"], s["k_rows"], s["v_rows"], s["row_dst"],
                           s["cache"], s["status"])
    return _store_out(s)


def _own_attend(s):
    co = _handle(s, s["case"]["B"], lambda co: co.CO_WS_ATTENTION_KV8)
    co.drafter_block_attention_kv8(s["dims"], 0, s["case"]["L"], s["q"], s["k_self"], s["v_self"],
                                   s["state"], s["cache"], s["out"], None, None, 0, s["ws"])
    return dict(out=s["out"], status=s["status"])


# ------------------------------------------------------------ the plain forms

def _plain_assign(pool, want, reserve):
    """Pages of lengths ``want``: every place that is needed takes the released page of
    its number, or from the end of the free list; released pages beyond go there."""
    table, held, free, count = (pool[k] for k in ("page_table", "held", "free_pages",
                                                  "free_count"))
    n, last = free.numel(), held.long()
    need = torch.where(want > 0, (want.long() + reserve + PAGE - 1) // PAGE, 0)
    grow, back = (need - last).clamp_min(0), (last - need).clamp_min(0)
    have = count.long() + back.sum()
    fits = grow.cumsum(0) <= have
    grow = torch.where(fits, grow, 0)
    taken, returned = grow.sum(), back.sum()
    j = torch.arange(table.shape[1], device="cuda")[None]
    lo, hi = need[:, None], last[:, None]
    out = (j >= lo) & (j < hi)                              # released places
    into = (j >= hi) & (j < hi + grow[:, None])             # taken places
    i_out = (back.cumsum(0) - back)[:, None] + j - lo
    i_in = (grow.cumsum(0) - grow)[:, None] + j - hi
    spare = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    listed_ = torch.empty(n + 1, dtype=torch.int32, device="cuda")
    listed_[torch.where(out, i_out, n)] = table             # released pages in their order
    place = have - 1 - i_in                                 # of the free list
    ids = torch.where(i_in < returned, listed_[i_in.clamp(0, n)], free[place.clamp(0, n - 1)])
    to = torch.where(out & (i_out >= taken), have - 1 - i_out, n)
    longer = torch.cat((free, spare))
    longer[to] = torch.where(out, table, -1)
    free.copy_(longer[:n])
    table.copy_(torch.where(into, ids, torch.where(out, -1, table)))
    held.copy_(torch.where(back > 0, need, last + grow))
    count.copy_(have - taken)


def _plain_pages(s):
    _plain_assign(s["pool"], s["before"], s["case"]["reserve"])
    _plain_assign(s["pool"], s["after"], s["case"]["reserve"])
    r = torch.arange(s["num_rows"], device="cuda")
    i = torch.searchsorted(s["row_start"].long(), r, right=True) - 1
    pos = s["before"].long()[i] + r - s["row_start"].long()[i]
    s["row_pos"].copy_(pos)
    s["row_dst"].copy_(s["pool"]["page_table"][i, pos // PAGE].long() * PAGE + pos % PAGE)
    return _pages_out(s)


def _plain_store_one(pages, scale, page, at, slot, given, rows):
    """Rows [L][r][Hkv][hd] into slots ``slot`` of the pages ``page``[``at``], whose
    contents are laid out [L][pages][Hkv][16][hd]; ``given`` [pages][16]: the slots
    that rows go to."""
    old = scale[:, page].int()
    held = _value(pages[:, page], old[..., None, None])
    new = torch.zeros_like(held)
    new.permute(1, 3, 0, 2, 4)[at, slot] = rows.float().transpose(0, 1)
    size = torch.where(torch.isfinite(new), new.abs(), 0).amax((3, 4))
    fresh = given[:, 0][None, :, None]
    k = _exponent(size)
    k = torch.where(fresh, k, torch.maximum(k, old - BIAS))
    held = torch.where(fresh[..., None, None], 0, held)
    x = torch.where(given[None, :, None, :, None], new, held)
    return _code(x, k[..., None, None]), (k + BIAS).to(torch.uint8)


def _plain_store(s):
    c, dst = s["cache"], s["row_dst"].long()
    rows = (dst >= 0).nonzero()[:, 0]
    page, at = torch.unique_consecutive(dst[rows] // PAGE, return_inverse=True)
    slot = dst[rows] % PAGE
    given = torch.zeros((page.numel(), PAGE), dtype=torch.bool, device="cuda")
    given[at, slot] = True
    codes, b = _plain_store_one(c["k_pages"], c["k_scale"], page, at, slot, given,
                                s["k_rows"][:, rows])
    c["k_pages"][:, page] = codes
    c["k_scale"][:, page] = b
    codes, b = _plain_store_one(c["v_pages"].transpose(3, 4), c["v_scale"], page, at, slot, given,
                                s["v_rows"][:, rows])
    c["v_pages"][:, page] = codes.transpose(3, 4)
    c["v_scale"][:, page] = b
    return _store_out(s)


def _keys(s):
    """Values of the committed pages [L][S][Hkv][tokens][hd]: keys and values."""
    c, at = s["cache"], s["page_table"].long()
    L, (S, P), H, hd = c["k_pages"].shape[0], at.shape, c["k_pages"].shape[2], c["k_pages"].shape[4]
    k = _value(c["k_pages"][:, at], c["k_scale"][:, at][..., None, None])
    v = _value(c["v_pages"][:, at], c["v_scale"][:, at][..., None, None])
    return (k.permute(0, 1, 3, 2, 4, 5).reshape(L, S, H, P * PAGE, hd),
            v.permute(0, 1, 3, 2, 5, 4).reshape(L, S, H, P * PAGE, hd))


def _plain_attend(s):
    c, ctx, q = s["case"], s["ctx_len"].long(), s["q"]
    L, S, B, Hq, hd = q.shape
    H, G = c["Hkv"], Hq // c["Hkv"]
    k, v = _keys(s)
    T, CP = k.shape[3], s["k_carry"].shape[2]
    kc = s["k_carry"].float().permute(0, 1, 3, 2, 4, 5).reshape(L, S, H, CP * PAGE, hd)
    vc = s["v_carry"].float().permute(0, 1, 3, 2, 5, 4).reshape(L, S, H, CP * PAGE, hd)
    arange = lambda n: torch.arange(n, device="cuda")[None]  # noqa: E731
    pos = ctx[:, None] + arange(B)                          # of the block's rows
    seen = torch.cat((arange(T) < ctx[:, None], arange(CP * PAGE) < s["carry_len"][:, None]), 1)
    ks, vs = [k, kc], [v, vc]
    if s["k_self"] is not None:
        ks.append(_rotate(s["k_self"], pos[..., None], c["theta"]).float().transpose(2, 3))
        vs.append(s["v_self"].float().transpose(2, 3))
        seen = torch.cat((seen, torch.ones((S, B), dtype=torch.bool, device="cuda")), 1)
    k, v = torch.cat(ks, 3), torch.cat(vs, 3)
    qr = (_rotate(q, pos[..., None], c["theta"]) / math.sqrt(hd)).float()
    qr = qr.view(L, S, B, H, G, hd).permute(0, 1, 3, 2, 4, 5).reshape(L, S, H, B * G, hd)
    x = torch.matmul(qr, k.transpose(3, 4))
    x.masked_fill_(~seen[None, :, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp_(x.sub_(torch.where(top == -math.inf, 0, top)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1)
    o = o.view(L, S, H, B, G, hd).permute(0, 1, 3, 2, 4, 5).reshape(q.shape)
    return dict(out=o.to(q.dtype), status=s["status"])


# -------------------------------------------------------------------- work

def work(c):
    if c["kind"] == "pages":
        # both calls: the lengths and holdings; of the pages that change hands the
        # old entry and the new one; then 8 bytes a row, and its page's entry
        S, most = c["S"], c["most"]
        mean = (c["lo"] + c["hi"]) / 2 if S > 1 else c["hi"]
        new = c["turn"] * min(mean, most) / (1 if S == 1 else 2) + (1 - c["turn"]) * (1 + most) / 2
        moved = S * (c["turn"] * mean + (1 - c["turn"]) * (1 + most) / 2) / PAGE
        return {"bytes": 2 * (S * 12 + moved * 12) + S * new * 8.25, "flops": 0.0}
    L, H, hd, S, B = c["L"], c["Hkv"], c["hd"], c["S"], c["B"]
    mean = (c["ctx_lo"] + c["ctx_hi"]) / 2 if S > 1 else c["ctx_hi"]
    m = sum((1 - c["reject"]) ** j for j in range(1, B + 1))        # accepted rows of a window
    if c["kind"] == "store":
        rows = S * (mean if c["rows"] == "packed" else max(m, 1 / S))
        # each row in, its codes out; the scales of its pages
        return {"bytes": rows * (2 * L * H * (hd * 3 + 0.25) + 4), "flops": 0.0}
    extra = (B - m) + (B if c["own_rows"] else 0)                   # bf16 keys of a sequence
    kv = S * L * H * (mean * (2 * hd + 2 / PAGE) + extra * 4 * hd)
    return {"bytes": kv + 4 * L * S * B * c["Hq"] * hd,
            "flops": 4.0 * S * (mean + extra) * L * B * c["Hq"] * hd}


# ------------------------------------------------- the same results in 64 bits

def exact(case, seed):
    if case["kind"] == "pages":
        return None                                                 # whole numbers only
    s = prepare(case, seed)
    return _exact_store(s) if case["kind"] == "store" else _exact_attend(s)


def _e4m3(x):
    """x to the nearest value 1.mmm * 2^e, e >= -6 (below, multiples of 2^-9), ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp_min(-6)
    unit = torch.exp2(e - 3)
    return torch.round(x / unit) * unit


def _exact_store(s):
    """Page after page: one scale for all of its rows, or the larger one of two."""
    c, dst = s["cache"], s["row_dst"].tolist()
    K, V = c["k_pages"].view(F8).double(), c["v_pages"].view(F8).double()
    runs = []
    for r, d in enumerate(dst):
        if d < 0:
            continue
        if runs and runs[-1][0] == d // PAGE and runs[-1][1] + runs[-1][3] == r:
            runs[-1][3] += 1
        else:
            runs.append([d // PAGE, r, d % PAGE, 1])
    for all_, scale, x, dim in ((K, c["k_scale"], s["k_rows"], 2), (V, c["v_scale"], s["v_rows"], 3)):
        for page, r, t, n in runs:
            x64 = x[:, r:r + n].double().transpose(1, 2)            # [L][Hkv][n][hd]
            top = x64.abs().amax((2, 3)) / (LARGEST * 256)
            b = torch.ceil(torch.log2(top.clamp_min(2.0 ** SMALLEST))) + BIAS
            part = all_[:, page] if dim == 2 else all_[:, page].transpose(2, 3)
            if t == 0:
                part.zero_()
            else:
                now = torch.maximum(b, scale[:, page].double())
                part.copy_(_e4m3(part * torch.exp2(scale[:, page].double() - now)[..., None, None]))
                b = now
            part[:, :, t:t + n] = _e4m3(x64 * torch.exp2(BIAS - b)[..., None, None])
    return dict(k=K, v=V, k_scale=None, v_scale=None, status=None)


def _exact_attend(s):
    c, q, cache = s["case"], s["q"], s["cache"]
    L, S, B, Hq, hd = q.shape
    H, G = c["Hkv"], Hq // c["Hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for i in range(S):
        n, u = int(s["ctx_len"][i]), int(s["carry_len"][i])
        at = s["page_table"][i, :-(-n // PAGE)].long()
        pos = n + torch.arange(B, device="cuda")
        for layer in range(L):
            unit = lambda b: torch.exp2(b[layer][at].double() - BIAS)[..., None, None]  # noqa: E731
            k = cache["k_pages"][layer][at].view(F8).double() * unit(cache["k_scale"])
            v = cache["v_pages"][layer][at].view(F8).double() * unit(cache["v_scale"])
            k = k.transpose(0, 1).reshape(H, -1, hd)[:, :n]
            v = v.permute(1, 0, 3, 2).reshape(H, -1, hd)[:, :n]
            kc = s["k_carry"][layer, i].double().transpose(0, 1).reshape(H, -1, hd)[:, :u]
            vc = s["v_carry"][layer, i].double().permute(1, 0, 3, 2).reshape(H, -1, hd)[:, :u]
            k, v = torch.cat((k, kc), 1), torch.cat((v, vc), 1)
            if s["k_self"] is not None:
                ks = _rotate(s["k_self"][layer, i], pos[:, None], c["theta"])
                k = torch.cat((k, ks.transpose(0, 1)), 1)
                v = torch.cat((v, s["v_self"][layer, i].double().transpose(0, 1)), 1)
            if k.shape[1] == 0:
                continue
            x = _rotate(q[layer, i], pos[:, None], c["theta"]) / math.sqrt(hd)
            x = x.view(B, H, G, hd).transpose(0, 1).reshape(H, B * G, hd)
            o = torch.softmax(x @ k.transpose(1, 2), -1) @ v
            out[layer, i] = o.view(H, B, G, hd).transpose(0, 1).reshape(B, Hq, hd)
    return dict(out=out, status=None)
