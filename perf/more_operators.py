"""Performance cases of 8-bit integer products and of the way from logits to a verifier's
probabilities.

A case is a dict of plain values.  Its "kind" names the calls of one pass:

  product  rows of features to 8-bit codes with a scale for each row, then their product with
           8-bit weights that have a scale for each output (``carryover_quantize_i8``,
           ``carryover_matmul_i8``)
  project  a window's rows through F and the K/V weights in 8 bits, rotated and stored
           (``carryover_project_kv_i8``)
  history  the token history of entering requests: their prompts, then one round's accepted
           proposals and its corrections (three calls of ``carryover_count_tokens``)
  rules    penalties, biases and grammar masks on the logits of a window
           (``carryover_logit_rules``)
  probs    the same rules, then the probabilities that a verification takes
           (``carryover_probabilities``)

Codes: a row's scale is its largest magnitude a over 127, the code of an entry x the nearest
integer of 127 x / a (ties to even).  A history word has 16 bits: the highest says that the token
is in the prompt, the others count how often it was generated.  Without ``own``, ``run`` computes
the same in elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
SKIP = -2 ** 31
MOST_COUNT = 32767                       # of a history word
LEAST = 127.0 * 2.0 ** -126              # magnitude below which a row's scale no longer shrinks
RMS_EPS = 1e-6


# ------------------------------------------------------------------ the cases

def _product(name, m, n, k, src="bf16", out="bf16", bias=False):
    return dict(name=name, kind="product", m=m, n=n, k=k, src=src, out=out, bias=bias)


def _project(name, S, B, Dcat, d, L, Hkv, hd, theta, reject, norms=False):
    return dict(name=name, kind="project", S=S, B=B, Dcat=Dcat, d=d, L=L, Hkv=Hkv, hd=hd,
                theta=theta, reject=reject, norms=norms)


def _rows(name, kind, S, B, rows, V, dtype, window=False, penalties=True, bias=0, masked=0.0):
    return dict(name=name, kind=kind, S=S, B=B, rows=rows, V=V, dtype=dtype, window=window,
                penalties=penalties, bias=bias, masked=masked)


def listed():
    return [
        # one row through F of the small drafter: launches and latency
        _product("product_row", 1, 256, 768),
        # one stream's window (16 proposals and the bonus) through the target's output head:
        # reading the head's weights
        _product("product_head17", 17, 128000, 4096),
        # the windows of a serving batch of 32 through the head: arithmetic
        _product("product_head544", 544, 128000, 4096),
        # odd sizes, a bias, 32-bit features and logits
        _product("product_odd", 77, 32001, 832, "f32", "f32", True),
        # an interactive round of a large drafter: reading F's weights
        _project("project_batch1", 1, 16, 20480, 4096, 1, 8, 128, 1e6, 0.25),
        # a serving round of 32 sequences, five drafter layers
        _project("project_batch32_5layer", 32, 16, 20480, 4096, 5, 8, 128, 1e6, 0.25),
        # one request with a short prompt enters
        dict(name="history_one", kind="history", S=1, B=16, V=1000, lo=37, hi=37),
        # a batch of 64 requests over a large vocabulary, long prompts
        dict(name="history_batch64", kind="history", S=64, B=16, V=128000, lo=16, hi=8192),
        # single tokens of a large batch, 32-bit logits, every rule
        _rows("rules_tokens64", "rules", 64, 1, 1, 128000, "f32", False, True, 300, 0.25),
        # odd sizes: seven proposals and the bonus, an odd vocabulary, every row masked
        _rows("rules_window11", "rules", 11, 7, 8, 32001, "bf16", True, True, 20, 1.0),
        # one stream's window over a small vocabulary: launches and latency
        _rows("probs_window1", "probs", 1, 16, 17, 1000, "f32", True, True, 0, 0.0),
        # the verification of a serving batch of 32 over a large vocabulary: memory traffic
        _rows("probs_batch32", "probs", 32, 16, 17, 128000, "bf16", True, True, 100, 0.25),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("product", "product", "product", "project", "history", "rules", "probs",
                       "probs"))
    if kind == "product":
        k = 64 * _log(rng, 1, 320)
        n = _log(rng, 16, max(16, min(131072, 128000 * 4096 // k)))
        m = _log(rng, 1, max(1, min(4096, 544 * 128000 * 4096 // (n * k), 544 * 128000 // n)))
        return dict(kind=kind, m=m, n=n, k=k, src=rng.choice(("bf16", "bf16", "f32")),
                    out=rng.choice(("bf16", "f32")), bias=rng.random() < 0.3)
    if kind == "project":
        B = rng.choice((1, 16, 16, 8, rng.randint(1, 32)))
        return dict(kind=kind, S=_log(rng, 1, 32 * 16 // B), B=B, Dcat=64 * _log(rng, 1, 320),
                    d=64 * _log(rng, 1, 64), L=rng.choice((1, 1, 2, 5)),
                    Hkv=rng.choice((1, 2, 3, 8)), hd=rng.choice((64, 128)),
                    theta=rng.choice((1e4, 1e6)), reject=round(rng.uniform(0.05, 0.5), 2),
                    norms=rng.random() < 0.3)
    V = _log(rng, 50, 131072)
    if kind == "history":
        S = _log(rng, 1, max(1, min(256, 64 * 128000 // V)))
        hi = _log(rng, 1, 8192)
        return dict(kind=kind, S=S, B=rng.choice((1, 16, 7)), V=V, lo=rng.randint(1, hi), hi=hi)
    B = rng.choice((1, 16, 16, 8, rng.randint(1, 32)))
    rows = rng.choice((1, B, B + 1, B + 1))
    S = _log(rng, 1, max(1, min(128, 32 * 17 * 128000 // (rows * V))))
    return dict(kind=kind, S=S, B=B, rows=rows, V=V, dtype=rng.choice(("bf16", "f32")),
                window=rows > 1 and rng.random() < 0.7, penalties=rng.random() < 0.8,
                bias=rng.choice((0, 0, 5, 300)), masked=rng.choice((0.0, 0.0, 0.25, 1.0)))


# ------------------------------------------------------------- common pieces

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _normal(g, shape, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return x if scale == 1.0 else x.mul_(scale)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _whole(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _spread(lo, hi, S):
    return [hi if S == 1 else lo + (hi - lo) * i // (S - 1) for i in range(S)]


def _codes(x):
    """Codes and scales of the rows of x: the nearest whole numbers (in 64 bits, for entries
    of 16 bits lie in the middle of two of them)."""
    x = x.float()
    top = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    a = torch.where(fine, top, 0).clamp_min(LEAST)
    codes = torch.round(x.double() * 127 / a.double()[..., None])
    return (torch.where(fine[..., None], codes, 0).to(torch.int8),
            torch.where(fine, a / torch.full_like(a, 127.0), math.nan))


def _weights(g, n, k):
    """8-bit weights [n][k] as a quantiser leaves them: normal rows whose largest code is 127."""
    codes = torch.empty((n, k), dtype=torch.int8, device="cuda")
    for at in range(0, n, 16384):
        x = _normal(g, (min(16384, n - at), k), torch.float32)
        codes[at:at + 16384] = torch.round(x * (127 / x.abs().amax(-1, keepdim=True)))
    return codes, 0.02 * (3 + _uniform(g, n)) / 127


def _tokens(g, V, *shape):
    """Token ids, a few of them frequent."""
    return (V * _uniform(g, *shape) ** 3).int().clamp_max(V - 1)


def _accepted(g, c):
    """Accepted prefix lengths: every position rejected with probability ``reject``."""
    gone = _uniform(g, c["S"], c["B"]) < c.get("reject", 0.25)
    return (gone.int().cumsum(1) == 0).sum(1).int()


# ----------------------------------------------------------------- prepare

def prepare(case, seed):
    return {"product": _prepare_product, "project": _prepare_project,
            "history": _prepare_history, "rules": _prepare_rows,
            "probs": _prepare_rows}[case["kind"]](case, seed)


def _prepare_product(c, seed):
    g = _gen(seed)
    w, w_scale = _weights(g, c["n"], c["k"])
    return dict(case=c, x=_normal(g, (c["m"], c["k"]), _type(c["src"])), w=w, w_scale=w_scale,
                bias=_normal(g, (c["n"],), torch.float32) if c["bias"] else None)


def _prepare_project(c, seed):
    g, S, B, L, H, hd = _gen(seed), c["S"], c["B"], c["L"], c["Hkv"], c["hd"]
    nkv = 2 * L * H * hd
    w_f, w_f_scale = _weights(g, c["d"], c["Dcat"])
    w_kv, w_kv_scale = _weights(g, nkv, c["d"])
    m = _accepted(g, c)
    j = torch.arange(B, device="cuda", dtype=torch.int32)[None]
    # every sequence's window starts somewhere in a page of a long context; two or more pages
    # of its own take the accepted rows
    first = _whole(g, 0, PAGE, S)[:, None]
    pages = (B + 2 * PAGE - 2) // PAGE
    table = torch.randperm(S * pages, generator=g, device="cuda").view(S, pages).int()
    at = first + j
    slot = table.gather(1, (at // PAGE).long()) * PAGE + at % PAGE
    CP = -(-B // PAGE)
    new = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    sigma = 0.02 * math.sqrt(c["Dcat"])
    return dict(case=c, num_pages=S * pages, hidden=_normal(g, (S * B, c["Dcat"]), torch.bfloat16),
                w_f=w_f, w_f_scale=w_f_scale, w_kv=w_kv, w_kv_scale=w_kv_scale,
                f_e=_normal(g, (c["d"],), torch.float32, 0.1 * sigma),
                z_norm=1 + 0.1 * _normal(g, (c["d"],), torch.float32) if c["norms"] else None,
                k_norm=1 + 0.1 * _normal(g, (L, hd), torch.float32) if c["norms"] else None,
                accept_len=m, row_pos=_whole(g, 0, 512, S)[:, None] * PAGE + at,
                row_dst=torch.where(j < m[:, None], slot, m[:, None] - 1 - j),
                k_cache=new(L, S * pages, H, PAGE, hd), v_cache=new(L, S * pages, H, hd, PAGE),
                k_carry=new(L, S, CP, H, PAGE, hd), v_carry=new(L, S, CP, H, hd, PAGE),
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_history(c, seed):
    g, S = _gen(seed), c["S"]
    length = torch.tensor(_spread(c["lo"], c["hi"], S), dtype=torch.int32, device="cuda")
    length = length[torch.randperm(S, generator=g, device="cuda")]
    prompt = _tokens(g, c["V"], S, c["hi"])
    past = torch.arange(c["hi"], device="cuda")[None] >= length[:, None]
    return dict(case=c, prompt=torch.where(past, -1, prompt), length=length,
                draft=_tokens(g, c["V"], S, c["B"]), accept_len=_accepted(g, c),
                next_tok=_tokens(g, c["V"], S),
                seen=torch.zeros((S, c["V"]), dtype=torch.int16, device="cuda"),
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_rows(c, seed):
    g, S, B, R, V = _gen(seed), c["S"], c["B"], c["rows"], c["V"]
    s = dict(case=c, logits=_normal(g, (S, R, V), _type(c["dtype"]), 3.0),
             draft=_tokens(g, V, S, B) if c["window"] else None, seen=None, bias_start=None,
             bias_tok=None, bias_val=None, mask_row=None, mask_bits=None,
             status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    pick = lambda *values: torch.tensor(values, device="cuda")[_whole(g, 0, len(values), S).long()]  # noqa: E731
    if c["penalties"]:                  # requests of many turns: hundreds of distinct tokens
        seen = torch.zeros((S, V), dtype=torch.int16, device="cuda")
        text = _tokens(g, V, S, min(V, 2000))
        seen.scatter_(1, text[:, ::2].long(), -2 ** 15)
        made = torch.zeros_like(seen)
        made.scatter_add_(1, text[:, 1::2].long(), torch.ones_like(text[:, 1::2], dtype=torch.int16))
        s.update(seen=seen + made, repetition=pick(1.0, 1.1, 1.3), presence=pick(0.0, 0.5, -0.2),
                 frequency=pick(0.0, 0.3, 0.05))
    if c["bias"]:                       # lists of up to so many entries, some requests without
        n = _whole(g, 0, c["bias"] + 1, S)
        start = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
        start[1:] = n.cumsum(0)
        s.update(bias_start=start, bias_tok=_whole(g, 0, V, S * c["bias"]),
                 bias_val=_normal(g, (S * c["bias"],), torch.float32, 2.0))
    if c["masked"]:                     # grammars leave a few tokens or most of them
        rows = torch.where((_uniform(g, S) < c["masked"])[:, None], _whole(g, 0, S * R, S, R), -1)
        share = 0.01 + 0.98 * _uniform(g, S * R, 1)
        words = -(-V // 32)
        bits = torch.zeros((S * R, words), dtype=torch.int64, device="cuda")
        for b in range(32):
            bits += (_uniform(g, S * R, words) < share).long() << b
        s.update(mask_row=rows, mask_bits=torch.where(bits < 2 ** 31, bits, bits - 2 ** 32).int())
    if c["kind"] == "probs":            # some requests are greedy
        s.update(temperature=pick(1.0, 1.0, 0.7, 0.0),
                 probs=torch.empty((S, R, V), dtype=torch.float32, device="cuda"),
                 top=torch.empty((S, R), dtype=torch.int32, device="cuda"))
    else:
        s["out"] = torch.empty_like(s["logits"])
    return s


# --------------------------------------------------------------------- run

def run(state):
    if own:
        return {"product": _own_product, "project": _own_project, "history": _own_history,
                "rules": _own_rules, "probs": _own_probs}[state["case"]["kind"]](state)
    return {"product": _plain_product, "project": _plain_project, "history": _plain_history,
            "rules": _plain_rules, "probs": _plain_probs}[state["case"]["kind"]](state)


def _project_out(s):
    return {k: s[k] for k in ("k_cache", "v_cache", "k_carry", "v_carry", "status")}


# ------------------------------------------------- the framework's own calls

def _own_product(s):
    import paper_2609_14717_amd as co
    c = s["case"]
    m, n, k = c["m"], c["n"], c["k"]
    if "codes" not in s:                # buffers that a program keeps over its calls
        s["codes"] = torch.empty((m, k), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(m, dtype=torch.float32, device="cuda")
        s["out"] = torch.empty((m, n), dtype=_type(c["out"]), device="cuda")
        s["ws"] = torch.empty(max(256, co.matmul_i8_workspace_bytes(m, n, k)), dtype=torch.uint8,
                              device="cuda")
    co.carryover_quantize_i8(m, k, c["src"], s["x"], s["codes"], s["scale"])
    co.carryover_matmul_i8(m, n, k, s["codes"], s["scale"], s["w"], s["w_scale"], s["bias"],
                           c["out"], s["out"], s["ws"])
    return s["out"]


def _own_project(s):
    import paper_2609_14717_amd as co
    if "dims" not in s:
        c = s["case"]
        s["dims"] = co.make_dims(c["S"], c["B"], c["Dcat"], c["d"], c["L"], c["Hkv"], c["Hkv"],
                                 c["hd"], 1, s["num_pages"], "bf16", c["theta"])
        s["weights"] = co.weights_i8(s["w_f"], s["w_f_scale"], s["w_kv"], s["w_kv_scale"],
                                     s["f_e"], s["z_norm"], s["k_norm"])
        s["ws"] = torch.empty(co.workspace_bytes(s["dims"], co.CO_WS_PROJECT_I8),
                              dtype=torch.uint8, device="cuda")
        s["route"] = dict(accept_len=s["accept_len"], row_pos=s["row_pos"], row_dst=s["row_dst"])
        s["state"] = dict(ctx_len=s["accept_len"], carry_len=s["accept_len"],
                          page_table=s["row_dst"], k_cache=s["k_cache"], v_cache=s["v_cache"],
                          k_carry=s["k_carry"], v_carry=s["v_carry"], status=s["status"])
    co.carryover_project_kv_i8(s["dims"], s["weights"], s["hidden"], s["route"], s["state"],
                               s["ws"])
    return _project_out(s)


def _dims(s):
    import paper_2609_14717_amd as co
    if "dims" not in s:
        c = s["case"]
        s["dims"] = co.make_dims(c["S"], c["B"], 64, 64, 1, 1, 1, 64, 1, 1, "bf16", 1e4)
        if c["kind"] != "history":
            s["rules"] = co.logit_rules(
                seen=s["seen"], repetition=s.get("repetition"), presence=s.get("presence"),
                frequency=s.get("frequency"), bias_start=s["bias_start"], bias_tok=s["bias_tok"],
                bias_val=s["bias_val"], mask_row=s["mask_row"], mask_bits=s["mask_bits"])
        if c["kind"] == "probs":
            size = co.probabilities_workspace_bytes(s["dims"], c["V"], c["rows"])
            s["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")
    return co


def _own_history(s):
    co, c = _dims(s), s["case"]
    co.carryover_count_tokens(s["dims"], c["V"], c["hi"], s["prompt"], s["length"],
                              co.CO_COUNT_PROMPT | co.CO_COUNT_FRESH, s["seen"], s["status"])
    co.carryover_count_tokens(s["dims"], c["V"], c["B"], s["draft"], s["accept_len"], 0,
                              s["seen"], s["status"])
    co.carryover_count_tokens(s["dims"], c["V"], 1, s["next_tok"], None, 0, s["seen"],
                              s["status"])
    return dict(seen=s["seen"], status=s["status"])


def _own_rules(s):
    co, c = _dims(s), s["case"]
    co.carryover_logit_rules(s["dims"], c["V"], c["rows"], c["dtype"], s["logits"], s["draft"],
                             s["rules"], s["out"], s["status"])
    return dict(logits=s["out"], status=s["status"])


def _own_probs(s):
    co, c = _dims(s), s["case"]
    co.carryover_probabilities(s["dims"], c["V"], c["rows"], c["dtype"], s["logits"], s["draft"],
                               s["rules"], s["temperature"], s["probs"], s["top"], s["status"],
                               s["ws"])
    return dict(probs=s["probs"], top=s["top"], status=s["status"])


# ------------------------------------------------------------ the plain forms

def _plain_product(s):
    codes, scale = _codes(s["x"])
    y = torch.matmul(codes.float(), s["w"].float().t()) * (scale[:, None] * s["w_scale"])
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(_type(s["case"]["out"]))


def _plain_project(s):
    c, dst = s["case"], s["row_dst"].reshape(-1).long()
    S, B, L, H, hd = c["S"], c["B"], c["L"], c["Hkv"], c["hd"]
    codes, scale = _codes(s["hidden"])
    z = torch.matmul(codes.float(), s["w_f"].float().t()) * (scale[:, None] * s["w_f_scale"])
    z = torch.where(((dst < 0) & (dst != SKIP))[:, None], z + s["f_e"], z)
    if s["z_norm"] is not None:
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + RMS_EPS) * s["z_norm"]
    codes, scale = _codes(z)
    y = torch.matmul(codes.float(), s["w_kv"].float().t()) * (scale[:, None] * s["w_kv_scale"])
    y = y.view(S * B, L, 2, H, hd)
    k, v = y[:, :, 0], y[:, :, 1]
    if s["k_norm"] is not None:
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + RMS_EPS) * s["k_norm"][:, None]
    half = hd // 2
    inv = c["theta"] ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = s["row_pos"].reshape(-1).double()[:, None] * inv
    cs, sn = torch.cos(angle).float()[:, None, None], torch.sin(angle).float()[:, None, None]
    lo, hi = k[..., :half], k[..., half:]
    k = torch.cat((lo * cs - hi * sn, hi * cs + lo * sn), -1).bfloat16()
    v = v.bfloat16()
    r = torch.arange(S * B, device="cuda")
    kept, left = (dst >= 0).nonzero()[:, 0], ((dst < 0) & (dst != SKIP)).nonzero()[:, 0]
    page, t = dst[kept] // PAGE, dst[kept] % PAGE
    s["k_cache"].permute(1, 3, 0, 2, 4)[page, t] = k[kept]
    s["v_cache"].permute(1, 4, 0, 2, 3)[page, t] = v[kept]
    row = -1 - dst[left]
    s["k_carry"].permute(1, 2, 4, 0, 3, 5)[r[left] // B, row // PAGE, row % PAGE] = k[left]
    s["v_carry"].permute(1, 2, 5, 0, 3, 4)[r[left] // B, row // PAGE, row % PAGE] = v[left]
    return _project_out(s)


def _plain_history(s):
    V = s["case"]["V"]
    here = torch.arange(s["prompt"].shape[1], device="cuda")[None] < s["length"][:, None]
    word = torch.zeros((s["seen"].shape[0], V + 1), dtype=torch.int32, device="cuda")
    word.scatter_(1, torch.where(here, s["prompt"], V).long(), 1)
    count = torch.zeros_like(word)
    kept = torch.arange(s["draft"].shape[1], device="cuda")[None] < s["accept_len"][:, None]
    made = torch.cat((torch.where(kept, s["draft"], V), s["next_tok"][:, None]), 1).long()
    count.scatter_add_(1, made, torch.ones_like(made, dtype=torch.int32))
    s["seen"].copy_((count.clamp_max(MOST_COUNT) - 2 ** 15 * word)[:, :V])
    return dict(seen=s["seen"], status=s["status"])


def _ruled(s, dtype=torch.float32):
    """The logits after the rules, in ``dtype``."""
    c, x = s["case"], s["logits"].to(dtype)
    S, R, V = x.shape
    rule = lambda name: s[name].to(dtype)[:, None, None]  # noqa: E731
    if s["seen"] is not None:
        word = s["seen"].int()[:, None]
        count, prompt = word & MOST_COUNT, word < 0
        if s["draft"] is not None:      # row j comes after the proposals before it
            more = torch.zeros((S, R, V), dtype=torch.int32, device="cuda")
            before = s["draft"][:, :R - 1].long()[..., None]
            more[:, 1:].scatter_(2, before, 1)
            count = count + more.cumsum(1, dtype=torch.int32)
        r = rule("repetition")
        x = torch.where(prompt | (count > 0), torch.where(x > 0, x / r, x * r), x)
        x = x - rule("frequency") * count.to(dtype)
        x = x - rule("presence") * (count > 0).to(dtype)
    if s["bias_start"] is not None:     # a token's last entry counts
        start = s["bias_start"].long()
        i = torch.arange(s["bias_tok"].numel(), device="cuda")
        i = i[:, None].expand(-1, S)
        inside = (i >= start[:-1]) & (i < start[1:])
        last = torch.full((S, V + 1), -1, dtype=torch.int64, device="cuda")
        to = torch.where(inside, s["bias_tok"].long()[:, None], V).t()
        last.scatter_reduce_(1, to, torch.where(inside, i, -1).t(), "amax")
        last = last[:, None, :V]
        x = torch.where(last >= 0, x + s["bias_val"].to(dtype)[last.clamp_min(0)], x)
    if s["mask_row"] is not None:
        v = torch.arange(V, device="cuda")
        bits = s["mask_bits"][s["mask_row"].clamp_min(0).long()]
        allowed = ((bits[..., v // 32] >> (v % 32).int()) & 1) != 0
        x = torch.where(allowed | (s["mask_row"] < 0)[..., None], x, -math.inf)
    return x


def _plain_rules(s):
    return dict(logits=_ruled(s).to(s["logits"].dtype), status=s["status"])


def _plain_probs(s):
    x, t = _ruled(s), s["temperature"][:, None, None]
    V = x.shape[-1]
    top = x.amax(-1, keepdim=True)
    v = torch.arange(V, device="cuda")
    first = torch.where(x == top, v, V).amin(-1, keepdim=True)
    some = top > -math.inf
    x = torch.where(some, x - top, -math.inf)
    w = torch.exp(x / torch.where(t > 0, t, 1))
    w = torch.where(t > 0, w, ((v == first) & some).float())
    total = w.sum(-1, keepdim=True, dtype=torch.float64)
    p = w / torch.where(total > 0, total, 1).float()
    return dict(probs=p, top=torch.where(some, first, -1)[..., 0].int(), status=s["status"])


# -------------------------------------------------------------------- work

def work(c):
    es = {"bf16": 2, "f32": 4}
    if c["kind"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * k * es[c["src"]] + n * k + 4 * n * (2 if c["bias"] else 1) +
                m * n * es[c["out"]], "flops": 2.0 * m * n * k}
    if c["kind"] == "project":
        M, nkv = c["S"] * c["B"], 2 * c["L"] * c["Hkv"] * c["hd"]
        return {"bytes": 2 * M * c["Dcat"] + c["d"] * c["Dcat"] + nkv * c["d"] + 8 * c["d"] +
                4 * nkv + 2 * M * nkv + 8 * M, "flops": 2.0 * M * c["d"] * (c["Dcat"] + nkv)}
    if c["kind"] == "history":
        mean = (c["lo"] + c["hi"]) / 2 if c["S"] > 1 else c["hi"]
        return {"bytes": c["S"] * (2 * c["V"] + 4 * mean + 4 * c["B"] + 12), "flops": 0.0}
    rows, V = c["S"] * c["rows"], c["V"]
    size = es[c["dtype"]]
    extra = 2 * c["S"] * V * c["penalties"] + 4 * c["S"] * c["bias"] + rows * c["masked"] * V / 8
    return {"bytes": rows * V * (size + (4 if c["kind"] == "probs" else size)) + extra,
            "flops": 0.0}


# ------------------------------------------------- the same results in 64 bits

def exact(case, seed):
    if case["kind"] == "history":
        return None                                             # whole numbers only
    s = prepare(case, seed)
    if case["kind"] == "product":
        q, a = _steps(s["x"].double())
        y = (q @ s["w"].double().t()) * a * s["w_scale"].double()
        return y if s["bias"] is None else y + s["bias"].double()
    return {"project": _exact_project, "rules": _exact_rules,
            "probs": _exact_probs}[case["kind"]](s)


def _steps(x):
    """Whole multiples of a 127th of each row's largest magnitude, and that 127th."""
    largest = x.abs().amax(1, keepdim=True).clamp_min(LEAST)
    return torch.round(127 * x / largest), largest / 127


def _exact_project(s):
    c = s["case"]
    B, L, H, hd = c["B"], c["L"], c["Hkv"], c["hd"]
    q, a = _steps(s["hidden"].double())
    z = (q @ s["w_f"].double().t()) * a * s["w_f_scale"].double()
    out = {k: s[k].double() for k in ("k_cache", "v_cache", "k_carry", "v_carry")}
    where = s["row_dst"].reshape(-1).tolist()
    for r, d in enumerate(where):
        if d < 0:
            z[r] += s["f_e"].double()
    if s["z_norm"] is not None:
        z = z / torch.sqrt((z ** 2).mean(1, keepdim=True) + RMS_EPS) * s["z_norm"].double()
    q, a = _steps(z)
    y = (q @ s["w_kv"].double().t()) * a * s["w_kv_scale"].double()
    pair = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
    turn = torch.exp(-math.log(c["theta"]) * 2 * pair / hd)
    turn = torch.exp(1j * s["row_pos"].reshape(-1, 1).double() * turn)
    for r, d in enumerate(where):
        row = y[r].view(L, 2, H, hd)
        k, v = row[:, 0], row[:, 1]
        if s["k_norm"] is not None:
            k = k / torch.sqrt((k ** 2).mean(2, keepdim=True) + RMS_EPS) * s["k_norm"].double()[:, None]
        k = torch.complex(k[..., :hd // 2].contiguous(), k[..., hd // 2:].contiguous()) * turn[r]
        k = torch.cat((k.real, k.imag), 2)
        if d >= 0:
            out["k_cache"][:, d // PAGE, :, d % PAGE] = k
            out["v_cache"][:, d // PAGE, :, :, d % PAGE] = v
        else:
            u = -1 - d
            out["k_carry"][:, r // B, u // PAGE, :, u % PAGE] = k
            out["v_carry"][:, r // B, u // PAGE, :, :, u % PAGE] = v
    return dict(out, status=None)


def _exact_row(s, i, j, counts, biases):
    """Row j of sequence i after the rules; counts: how often each token was generated."""
    x = s["logits"][i, j].double()
    if s["seen"] is not None:
        r = float(s["repetition"][i])
        known = (counts > 0) | (s["seen"][i] < 0)
        x = torch.where(known, torch.where(x > 0, x / r, x * r), x)
        x = x - float(s["frequency"][i]) * counts
        x = torch.where(counts > 0, x - float(s["presence"][i]), x)
    if biases:
        at = torch.tensor(list(biases), device="cuda")
        x[at] += torch.tensor(list(biases.values()), dtype=torch.float64, device="cuda")
    if s["mask_row"] is not None and int(s["mask_row"][i, j]) >= 0:
        words = s["mask_bits"][int(s["mask_row"][i, j])]
        bit = torch.ones(32, dtype=torch.int32, device="cuda") << torch.arange(32, device="cuda").int()
        allowed = ((words[:, None] & bit) != 0).reshape(-1)[:x.numel()]
        x[~allowed] = -math.inf
    return x


def _exact_rows(s):
    """(sequence, row, logits after the rules) of every row."""
    S, R, _ = s["logits"].shape
    for i in range(S):
        counts, biases = None, {}
        if s["seen"] is not None:
            counts = torch.bitwise_and(s["seen"][i].long(), MOST_COUNT)
        if s["bias_start"] is not None:
            lo, hi = int(s["bias_start"][i]), int(s["bias_start"][i + 1])
            biases = dict(zip(s["bias_tok"][lo:hi].tolist(), s["bias_val"][lo:hi].tolist()))
        for j in range(R):
            if j and counts is not None and s["draft"] is not None:
                counts[int(s["draft"][i, j - 1])] += 1
            yield i, j, _exact_row(s, i, j, counts, biases)


def _exact_rules(s):
    out = torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda")
    for i, j, x in _exact_rows(s):
        out[i, j] = x
    return dict(logits=out, status=None)


def _exact_probs(s):
    out = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
    for i, j, x in _exact_rows(s):
        t = float(s["temperature"][i])
        if not bool(torch.isfinite(x).any()):
            continue
        if t > 0:
            out[i, j] = torch.softmax(x / t, 0)
        else:
            out[i, j, int((x == x.max()).nonzero()[0])] = 1.0
    return dict(probs=out, top=None, status=None)
