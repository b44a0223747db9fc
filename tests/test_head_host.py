"""8-bit products, logit rules and probabilities without a GPU: the oracle's pins and the
host checks of the entry points (refusals return before anything is enqueued; no compute
call runs here)."""
import os
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle
import paper_2609_14717_amd as co
from oracle import head

needs_lib = pytest.mark.skipif(not os.path.exists(co.LIB_PATH), reason="library not built")
FAKE = 1 << 20      # an aligned, non-null address that is never dereferenced here


# ------------------------------------------------------------------ the oracle

def test_codes_are_the_nearest_integers_of_the_exact_quotient():
    rng = np.random.default_rng(7)
    x = rng.standard_normal((6, 64)).astype(np.float32)
    x[1] = torch.tensor(x[1]).bfloat16().float().numpy()
    x[2] = np.arange(64) * 0.5                  # many middles: 127 x / 31.5 = 4.03.. x
    x[3] = (np.arange(64) - 32) / 254.0 * 127   # 127 x / a with a = 16: exact quarters
    x[3, 0] = 63.5                              # a = 63.5: 127 x / a = 2 x, exact halves
    x[4] = 0.0
    codes, scale = head.quantize(x)
    for i in range(len(x)):
        a = max(Fraction(float(np.abs(x[i]).max())), Fraction(127, 2 ** 126))
        for k in range(64):
            q = Fraction(127) * Fraction(float(x[i, k])) / a
            assert codes[i, k] == round(q)      # (of a fraction: ties to even)
        assert scale[i] == pytest.approx(float(a) / 127, rel=1e-15)
    codes, scale = head.quantize([[1.0] * 63 + [np.inf], [np.nan] * 64, [-2.0] + [0.0] * 63])
    assert not codes[:2].any() and np.isnan(scale[:2]).all()
    assert codes[2, 0] == -127 and scale[2] == 2 / 127


def test_product_of_codes_is_the_scaled_integer_sum():
    a = np.array([[1, -2, 3], [127, 127, 127]])
    w = np.array([[4, 5, -6], [-128, -128, -128]])
    y, _ = head.matmul_i8(a, [0.5, 1.0], w, [2.0, 1.0], [10.0, 0.0])
    np.testing.assert_array_equal(y, [[-24 * 1.0 + 10, -256 * 0.5], [381 * 2.0 + 10, -48768.0]])


def test_projection_with_exact_codes_is_the_plain_projection():
    """Integer rows whose largest entry is 127 are their own codes at the first product; with
    F = 127 e_k selections z keeps them, so that both products are exact."""
    rng = np.random.default_rng(3)
    M, D, L, Hkv, hd = 4, 128, 1, 1, 64
    H = rng.integers(-127, 128, (M, D)).astype(np.float64)
    H[:, 5] = 127
    perm = rng.permutation(D)
    wf = np.zeros((D, D), np.int64)
    wf[np.arange(D), perm] = 1
    wkv = rng.integers(-127, 128, (2 * hd, D))
    sf, skv = np.ones(D), np.full(2 * hd, 0.01)
    pos = np.array([0, 3, 70, 5000])
    k, v, *_ = head.project_i8(H, wf, sf, wkv, skv, None, np.zeros(M), pos, L, Hkv, hd, 1e4)
    K, V = oracle.project(H, np.zeros(D), np.zeros(M, bool), wf.astype(float), wkv * skv[:, None],
                          pos, L, Hkv, hd, 1e4)
    np.testing.assert_allclose(k.reshape(-1), np.asarray(K).reshape(k.shape).reshape(-1), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(v.reshape(-1), np.asarray(V).reshape(v.shape).reshape(-1), rtol=1e-12, atol=1e-12)


def test_history_words():
    seen = np.zeros((3, 5), np.uint16)
    seen[1] = 9
    seen[2, 4] = 32766
    tok = np.array([[1, 1, -1, 4], [0, 2, 2, 2], [4, 4, 4, 0]])
    w, st = head.count_tokens(seen, tok, [3, 0, 3], prompt=False, fresh=False)
    np.testing.assert_array_equal(w, [[0, 2, 0, 0, 0], [9] * 5, [0, 0, 0, 0, 32767]])
    assert st == oracle.OK
    w, st = head.count_tokens(w, tok, [4, 0, 4], prompt=True, fresh=True)
    np.testing.assert_array_equal(w, [[0, 0x8000, 0, 0, 0x8000], [9] * 5, [0x8000, 0, 0, 0, 0x8000]])
    _, st = head.count_tokens(w, tok + 1, [4, 5, 0], prompt=True, fresh=False)
    assert st == oracle.ERR_LENGTH
    _, st = head.count_tokens(w, tok + 1, [4, 0, 0], prompt=True, fresh=False)
    assert st == oracle.ERR_TOKEN


def test_rules_by_hand():
    x = [2.0, -2.0, 2.0, 2.0, 0.5, np.nan]
    word = [0x8000, 0x8000 | 1, 0, 3, 0, 0]
    y, err = head.rules_row(x, word, window=[2, 2, 0, 99, -1], repetition=2.0, presence=0.25,
                            frequency=0.5, biases=[(4, 7.0), (3, -1.0), (4, 1.0), (77, 3.0)],
                            allowed=[1, 1, 1, 1, 1, 0])
    np.testing.assert_array_equal(y, [1 - 0.5 - 0.25, -4 - 0.5 - 0.25, 1 - 1.0 - 0.25,
                                      1 - 1.5 - 0.25 - 1, 1.5, -np.inf])
    assert err[4] == 1.5 * 2.0 ** -24 and err[5] == 0 and (err[:4] > 0).all()


def test_probabilities_by_hand():
    p, tol, top = head.probabilities_row(np.array([0.0, np.log(3.0), -np.inf]), np.zeros(3))
    np.testing.assert_allclose(p, [0.25, 0.75, 0.0], rtol=1e-15)
    assert top == 1 and tol[0] < 1e-4
    p, _, top = head.probabilities_row(np.array([1.0, 5.0, 5.0]), np.zeros(3), temperature=0.0)
    np.testing.assert_array_equal(p, [0, 1, 0])
    assert top == 1
    p, _, top = head.probabilities_row(np.array([-np.inf, np.nan]), np.zeros(2))
    assert top == -1 and not p.any()
    p, _, top = head.probabilities_row(np.array([np.inf, 3.0, np.inf]), np.zeros(3))
    np.testing.assert_array_equal(p, [0.5, 0, 0.5])
    assert top == 0


# ------------------------------------------------------------------ refusals

def _rc(fn):
    try:
        fn()
    except co.CarryoverError as e:
        return e.code
    return co.CO_OK


def dims(S=2, B=16, **kw):
    base = dict(Dcat=768, d=256, L=1, Hq=4, Hkv=2, hd=64, max_pages_per_seq=8, num_pages=16,
                dtype="bf16", theta=1e4)
    base.update(kw)
    return co.make_dims(S, B, **base)


@needs_lib
@pytest.mark.parametrize("rows,cols,dtype,kw,code", [
    (-1, 64, "bf16", {}, co.CO_ERR_INVALID_ARG),
    (1, 0, "bf16", {}, co.CO_ERR_INVALID_ARG),
    (1, 65, "bf16", {}, co.CO_ERR_UNSUPPORTED),
    (1 << 22, 64, "bf16", {}, co.CO_ERR_UNSUPPORTED),
    (1, 64, 7, {}, co.CO_ERR_UNSUPPORTED),
    (1, 64, "f32", dict(x=0), co.CO_ERR_INVALID_ARG),
    (1, 64, "f32", dict(x=FAKE + 4), co.CO_ERR_INVALID_ARG),
    (1, 64, "f32", dict(codes=FAKE + 8), co.CO_ERR_INVALID_ARG),
    (1, 64, "f32", dict(scale=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (1, 64, "f32", dict(scale=0), co.CO_ERR_INVALID_ARG),
])
def test_quantize_refusals(rows, cols, dtype, kw, code):
    p = dict(x=FAKE, codes=FAKE, scale=FAKE, **{})
    p.update(kw)
    assert _rc(lambda: co.carryover_quantize_i8(rows, cols, dtype, p["x"], p["codes"], p["scale"],
                                                stream=0)) == code


@needs_lib
@pytest.mark.parametrize("m,n,k,kw,code", [
    (-1, 64, 64, {}, co.CO_ERR_INVALID_ARG),
    (1, -1, 64, {}, co.CO_ERR_INVALID_ARG),
    (1, 64, 0, {}, co.CO_ERR_UNSUPPORTED),
    (1, 64, 32, {}, co.CO_ERR_UNSUPPORTED),
    (1, 64, 131072, {}, co.CO_ERR_UNSUPPORTED),
    (1 << 24, 1, 64, {}, co.CO_ERR_UNSUPPORTED),
    (1, 1 << 24, 64, {}, co.CO_ERR_UNSUPPORTED),
    ((1 << 24) - 1, (1 << 24) - 1, 64, {}, co.CO_ERR_UNSUPPORTED),
    (1, 64, 64, dict(dtype=2), co.CO_ERR_UNSUPPORTED),
    (1, 64, 64, dict(a=0), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(a=FAKE + 8), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(w=FAKE + 1), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(a_scale=0), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(w_scale=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(bias=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(out=0), co.CO_ERR_INVALID_ARG),
    (1, 64, 64, dict(out=FAKE + 4), co.CO_ERR_INVALID_ARG),
])
def test_matmul_refusals(m, n, k, kw, code):
    p = dict(a=FAKE, a_scale=FAKE, w=FAKE, w_scale=FAKE, bias=None, dtype="bf16", out=FAKE)
    p.update(kw)
    assert _rc(lambda: co.carryover_matmul_i8(m, n, k, p["a"], p["a_scale"], p["w"], p["w_scale"],
                                              p["bias"], p["dtype"], p["out"], FAKE, stream=0,
                                              ws_bytes=1 << 40)) == code
    if not kw:
        assert co.matmul_i8_workspace_bytes(m, n, k) == 0


@needs_lib
@pytest.mark.parametrize("m,n,k", [(1, 256, 768), (16, 4096, 20480), (17, 128000, 4096)])
def test_matmul_workspace_is_checked(m, n, k):
    need = co.matmul_i8_workspace_bytes(m, n, k)
    call = lambda ws, nb: _rc(lambda: co.carryover_matmul_i8(  # noqa: E731
        m, n, k, FAKE, FAKE, FAKE, FAKE, None, "bf16", FAKE, ws, stream=0, ws_bytes=nb))
    if need:
        assert call(FAKE, need - 1) == co.CO_ERR_WORKSPACE
        assert call(FAKE + 16, need) == co.CO_ERR_INVALID_ARG
        assert call(0, need) == co.CO_ERR_INVALID_ARG


@needs_lib
@pytest.mark.parametrize("m,n,k,parts", [(1, 256, 768, 0), (17, 128000, 4096, 0), (45, 3001, 4160, 6),
                                         (16, 4096, 20480, 8), (64, 130, 8256, 11)])
def test_products_in_parts_need_their_workspace(m, n, k, parts):
    """int32 results for every part of K, to whole lines of 256 bytes."""
    need = co.matmul_i8_workspace_bytes(m, n, k)
    assert need == -(-parts * m * n * 4 // 256) * 256
    call = lambda ws, nb: _rc(lambda: co.carryover_matmul_i8(  # noqa: E731
        m, n, k, FAKE, FAKE, FAKE, FAKE, None, "bf16", FAKE, ws, stream=0, ws_bytes=nb))
    if parts:
        assert call(FAKE, need - 1) == co.CO_ERR_WORKSPACE
        assert call(FAKE + 16, need) == co.CO_ERR_INVALID_ARG
        assert call(0, need) == co.CO_ERR_INVALID_ARG


def _weights_i8(**kw):
    p = dict(w_f=FAKE, w_f_scale=FAKE, w_kv=FAKE, w_kv_scale=FAKE)
    p.update(kw)
    return co.weights_i8(**p)


@needs_lib
@pytest.mark.parametrize("d,w,code", [
    (dict(dtype="f32"), {}, co.CO_ERR_UNSUPPORTED),
    (dict(Dcat=131072), {}, co.CO_ERR_UNSUPPORTED),
    (dict(d=131072), {}, co.CO_ERR_UNSUPPORTED),
    (dict(d=16448), dict(z_norm=FAKE), co.CO_ERR_UNSUPPORTED),
    (dict(S=1 << 18), {}, co.CO_ERR_UNSUPPORTED),
    (dict(S=1 << 16, d=4096), {}, co.CO_ERR_UNSUPPORTED),
    ({}, dict(w_f=0), co.CO_ERR_INVALID_ARG),
    ({}, dict(w_f_scale=0), co.CO_ERR_INVALID_ARG),
    ({}, dict(w_kv=FAKE + 8), co.CO_ERR_INVALID_ARG),
    ({}, dict(w_kv_scale=FAKE + 2), co.CO_ERR_INVALID_ARG),
    ({}, dict(f_e=FAKE + 4), co.CO_ERR_INVALID_ARG),
])
def test_project_refusals(d, w, code):
    d = dims(**d)
    st = {k: FAKE for k in ("ctx_len", "carry_len", "page_table", "k_cache", "v_cache", "k_carry",
                            "v_carry", "status")}
    rt = {k: FAKE for k in ("accept_len", "row_pos", "row_dst")}
    assert _rc(lambda: co.carryover_project_kv_i8(d, _weights_i8(**w), FAKE, rt, st, FAKE, stream=0,
                                                  ws_bytes=1 << 50)) == code


@needs_lib
def test_project_workspace_is_checked():
    d = dims()
    st = {k: FAKE for k in ("ctx_len", "carry_len", "page_table", "k_cache", "v_cache", "k_carry",
                            "v_carry", "status")}
    rt = {k: FAKE for k in ("accept_len", "row_pos", "row_dst")}
    need = co.workspace_bytes(d, co.CO_WS_PROJECT_I8)
    call = lambda ws, nb: _rc(lambda: co.carryover_project_kv_i8(  # noqa: E731
        d, _weights_i8(), FAKE, rt, st, ws, stream=0, ws_bytes=nb))
    assert need > 0 and call(FAKE, need - 1) == co.CO_ERR_WORKSPACE
    assert call(FAKE + 128, need) == co.CO_ERR_INVALID_ARG
    assert call(0, need) == co.CO_ERR_INVALID_ARG
    assert co.workspace_bytes(dims(dtype="f32"), co.CO_WS_PROJECT_I8) == 0
    st["status"] = 0
    assert call(FAKE, need) == co.CO_ERR_INVALID_ARG


@needs_lib
@pytest.mark.parametrize("kw,code", [
    (dict(vocab=0), co.CO_ERR_UNSUPPORTED),
    (dict(width=-1), co.CO_ERR_INVALID_ARG),
    (dict(tokens=0), co.CO_ERR_INVALID_ARG),
    (dict(lens=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (dict(flags=4), co.CO_ERR_INVALID_ARG),
    (dict(seen=0), co.CO_ERR_INVALID_ARG),
    (dict(seen=FAKE + 1), co.CO_ERR_INVALID_ARG),
    (dict(status=0), co.CO_ERR_INVALID_ARG),
    (dict(dims=dims(B=0)), co.CO_ERR_INVALID_ARG),
    (dict(dims=dims(S=1 << 20), vocab=1 << 20), co.CO_ERR_UNSUPPORTED),
    (dict(dims=dims(S=1), vocab=(1 << 30) + 1), co.CO_ERR_UNSUPPORTED),
])
def test_count_refusals(kw, code):
    p = dict(dims=dims(), vocab=1000, width=16, tokens=FAKE, lens=None, flags=0, seen=FAKE, status=FAKE)
    p.update(kw)
    assert _rc(lambda: co.carryover_count_tokens(*p.values(), stream=0)) == code


def _rules(**kw):
    return co.logit_rules(**{k: v for k, v in kw.items() if k not in ("num_bias", "num_masks")})


RULE_CASES = [
    (dict(repetition=FAKE), co.CO_ERR_INVALID_ARG),                      # penalties need a history
    (dict(frequency=FAKE), co.CO_ERR_INVALID_ARG),
    (dict(seen=FAKE + 1), co.CO_ERR_INVALID_ARG),
    (dict(seen=FAKE, presence=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (dict(bias_start=FAKE), co.CO_ERR_INVALID_ARG),                      # three or none
    (dict(mask_row=FAKE), co.CO_ERR_INVALID_ARG),                        # both or none
]


def _raw_rules(**kw):
    r = co.co_logit_rules()
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@needs_lib
@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(vocab=0), co.CO_ERR_UNSUPPORTED),
    (dict(rows=0), co.CO_ERR_INVALID_ARG),
    (dict(rows=18), co.CO_ERR_INVALID_ARG),                              # block + 1 at most
    (dict(dtype=3), co.CO_ERR_UNSUPPORTED),
    (dict(logits=0), co.CO_ERR_INVALID_ARG),
    (dict(logits=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (dict(draft=FAKE + 2), co.CO_ERR_INVALID_ARG),
    (dict(out=0), co.CO_ERR_INVALID_ARG),
    (dict(out=FAKE + 64), co.CO_ERR_INVALID_ARG),                        # overlaps the logits
    (dict(status=0), co.CO_ERR_INVALID_ARG),
    (dict(dims=dims(B=1025)), co.CO_ERR_UNSUPPORTED),
    (dict(dims=dims(S=1 << 20), vocab=1 << 20), co.CO_ERR_UNSUPPORTED),
    (dict(dims=dims(S=1), vocab=(1 << 30) + 1), co.CO_ERR_UNSUPPORTED),
] + [(dict(rules=_raw_rules(**r)), c) for r, c in RULE_CASES] + [
    (dict(rules=_raw_rules(num_bias=-1)), co.CO_ERR_INVALID_ARG),
    (dict(rules=_raw_rules(num_masks=-1)), co.CO_ERR_INVALID_ARG),
])
def test_logit_refusals(probs, kw, code):
    p = dict(dims=dims(), vocab=1000, rows=17, dtype="f32", logits=FAKE, draft=None, rules=_raw_rules(),
             out=1 << 30, status=FAKE)
    p.update(kw)
    if probs:
        call = lambda: co.carryover_probabilities(  # noqa: E731
            p["dims"], p["vocab"], p["rows"], p["dtype"], p["logits"], p["draft"], p["rules"], None,
            p["out"], None, p["status"], FAKE, stream=0, ws_bytes=1 << 50)
    else:
        call = lambda: co.carryover_logit_rules(*p.values(), stream=0)  # noqa: E731
    assert _rc(call) == code


@needs_lib
def test_probabilities_workspace_temperature_and_top():
    d = dims()
    need = co.probabilities_workspace_bytes(d, 1000, 17)
    assert need > 0 and co.probabilities_workspace_bytes(d, 0, 17) == 0
    assert co.probabilities_workspace_bytes(d, 1000, 18) == 0

    def call(ws=FAKE, nb=need, t=None, top=None, out=1 << 30):
        return _rc(lambda: co.carryover_probabilities(d, 1000, 17, "f32", FAKE, None, None, t, out, top,
                                                      FAKE, ws, stream=0, ws_bytes=nb))
    assert call(nb=need - 1) == co.CO_ERR_WORKSPACE
    assert call(ws=FAKE + 64) == co.CO_ERR_INVALID_ARG
    assert call(ws=0) == co.CO_ERR_INVALID_ARG
    assert call(t=FAKE + 1) == co.CO_ERR_INVALID_ARG
    assert call(top=FAKE + 1) == co.CO_ERR_INVALID_ARG
    assert call(out=FAKE) == co.CO_ERR_INVALID_ARG          # in place is the rules' call


@needs_lib
@pytest.mark.parametrize("vocab,rows,S,ok", [
    (2049, 1, 1 << 22, False), (2049, 4, (1 << 23) - 1, False), (4096, 5, 1 << 21, False),
    (4096, 4, (1 << 22) - 1, True), (2048, 4, 1 << 22, True), (4097, 4, (1 << 22) - 1, True)])
def test_probabilities_of_more_threads_than_a_launch_has_are_refused(vocab, rows, S, ok):
    """Whole rows of more than 2048 tokens have a workgroup of 1024 threads for up to four rows:
    2^22 workgroups are 2^32 threads.  The rules' call has 256 threads at any size."""
    d = dims(S=S, B=rows)
    assert (co.probabilities_workspace_bytes(d, vocab, rows) > 0) == ok
    if not ok:
        assert _rc(lambda: co.carryover_probabilities(d, vocab, rows, "bf16", FAKE, None, None, None, 1 << 45, None,
                                                      FAKE, FAKE, stream=0, ws_bytes=1 << 60)) == co.CO_ERR_UNSUPPORTED


@needs_lib
def test_rules_call_needs_rules():
    import ctypes
    d = dims()
    assert co.lib().carryover_logit_rules(ctypes.byref(d), 1000, 17, 0, FAKE, None, None, 1 << 30, FAKE,
                                          0) == co.CO_ERR_INVALID_ARG


@needs_lib
def test_calls_of_nothing_take_empty_tensors():
    """An empty tensor has no address."""
    i8, f = torch.empty(0, 64, dtype=torch.int8), torch.empty(0)
    w = torch.zeros(4, 64, dtype=torch.int8)
    co.carryover_quantize_i8(0, 64, "f32", torch.empty(0, 64), i8, f, stream=0)
    co.carryover_matmul_i8(0, 4, 64, i8, f, w, torch.zeros(4), None, "bf16", f, None, stream=0)
    co.carryover_matmul_i8(4, 0, 64, w, torch.zeros(4), i8, f, None, "bf16", f, None, stream=0)
    co.carryover_count_tokens(dims(S=2), 10, 0, torch.empty(2, 0, dtype=torch.int32), None, 0, FAKE, FAKE,
                              stream=0)
    with pytest.raises(co.CarryoverError):
        co.carryover_matmul_i8(0, 4, 65, i8, f, w, torch.zeros(4), None, "bf16", f, None, stream=0)


@needs_lib
def test_empty_batches_take_empty_tensors():
    """num_seqs 0: sizes, weights and rules are checked, then there is nothing to do."""
    d, i32 = dims(S=0), lambda *s: torch.empty(s, dtype=torch.int32)  # noqa: E731
    e = lambda *s, t=torch.float32: torch.empty(s, dtype=t)  # noqa: E731
    seen, status = e(0, 1000, t=torch.int16), torch.zeros(1, dtype=torch.int32)
    co.carryover_count_tokens(d, 1000, 16, i32(0, 16), i32(0), co.CO_COUNT_PROMPT, seen, status, stream=0)
    r = co.logit_rules(seen, e(0), e(0), e(0), torch.zeros(1, dtype=torch.int32), i32(0), e(0), i32(0, 17),
                       torch.zeros(3, 32, dtype=torch.int32))
    x = e(0, 17, 1000)
    co.carryover_logit_rules(d, 1000, 17, "f32", x, i32(0, 16), r, x, status, stream=0)
    assert co.probabilities_workspace_bytes(d, 1000, 17) == 0
    ws = e(0, t=torch.uint8)
    for rules in (r, None):
        co.carryover_probabilities(d, 1000, 17, "f32", x, i32(0, 16), rules, e(0), e(0, 17, 1000), i32(0, 17), status, ws,
                                   stream=0)
    st = dict(ctx_len=i32(0), carry_len=i32(0), page_table=i32(0, 8), k_cache=e(1, 16, 2, 16, 64), v_cache=e(1, 16, 2, 64, 16),
              k_carry=e(1, 0, 1, 2, 16, 64), v_carry=e(1, 0, 1, 2, 64, 16), status=status)
    rt = dict(accept_len=i32(0), row_pos=i32(0, 16), row_dst=i32(0, 16))
    project = lambda **w: _rc(lambda: co.carryover_project_kv_i8(  # noqa: E731
        d, _weights_i8(**w), e(0, 768, t=torch.bfloat16), rt, st, ws, stream=0))
    assert project() == co.CO_OK
    # what does not hang on the batch is refused as ever
    assert project(w_f=FAKE + 8) == co.CO_ERR_INVALID_ARG
    assert _rc(lambda: co.carryover_count_tokens(d, 1000, 16, 0, 0, 4, 0, 0, stream=0)) == co.CO_ERR_INVALID_ARG
    assert _rc(lambda: co.carryover_count_tokens(d, 0, 16, 0, 0, 0, 0, 0, stream=0)) == co.CO_ERR_UNSUPPORTED
    assert _rc(lambda: co.carryover_logit_rules(d, 1000, 18, "f32", x, None, r, x, status,
                                                stream=0)) == co.CO_ERR_INVALID_ARG


@needs_lib
def test_lists_too_long_to_walk_in_32_bits_are_refused():
    assert _rc(lambda: co.carryover_count_tokens(dims(), 1000, (1 << 30) + 1, FAKE, None, 0, FAKE, FAKE,
                                                 stream=0)) == co.CO_ERR_UNSUPPORTED
    r = _raw_rules(bias_start=FAKE, bias_tok=FAKE, bias_val=FAKE, num_bias=(1 << 30) + 1)
    assert _rc(lambda: co.carryover_logit_rules(dims(), 1000, 17, "f32", FAKE, None, r, 1 << 30, FAKE,
                                                stream=0)) == co.CO_ERR_INVALID_ARG


def test_empty_lists_of_rules_have_addresses():
    e = torch.empty(0)
    r = co.logit_rules(bias_start=torch.zeros(3), bias_tok=e, bias_val=e, mask_row=torch.zeros(2),
                       mask_bits=torch.empty(0, 4))
    assert r.bias_tok and r.bias_val and r.mask_bits and r.num_bias == r.num_masks == 0


def test_rules_and_weights_keep_their_tensors():
    import weakref
    t = torch.zeros(4)
    alive = weakref.ref(t)
    r, w = co.logit_rules(repetition=t), co.weights_i8(t, t, t, t)
    del t
    assert alive() is not None
    del r
    assert alive() is not None
    del w
    assert alive() is None


def test_strided_tensors_are_refused():
    x = torch.zeros(4, 128)[:, ::2]
    with pytest.raises(ValueError, match="x is not contiguous"):
        co._dense(x, "x")
    with pytest.raises(ValueError, match="seen is not contiguous"):
        co.logit_rules(seen=torch.zeros(4, 6, dtype=torch.int16).t())
    with pytest.raises(ValueError, match="w_f is not contiguous"):
        co.weights_i8(torch.zeros(64, 64, dtype=torch.int8).t(), None, None, None)


@needs_lib
def test_mask_status_has_a_message():
    assert "mask" in co.status_string(co.CO_ERR_MASK)
