"""GPU parity of 8-bit integer products, logit rules, token history and probabilities with the
fp64 oracle.

Tolerances count roundings, each off by at most half a step: 2^-24 of the value in fp32, 2^-8
for a bf16 result.  Codes, history words, sums of codes and truth values are equal.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import oracle  # noqa: E402
import paper_2609_14717_amd as co  # noqa: E402
from oracle import head  # noqa: E402

DEV = "cuda"
F32, BF16 = 2.0 ** -24, 2.0 ** -8


def np_(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def zero():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def typed(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def within(got, want, tol, what):
    """got within tol of want, equal where want is not finite."""
    got, want, tol = (np.asarray(x, np.float64) for x in (got, want, np.broadcast_to(tol, np.shape(want))))
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    assert not off.size or off.max() <= 0, f"{what}: {off.max():.3e} beyond the tolerance"


# ------------------------------------------------------------- quantisation

def quantize(x):
    rows, cols = x.shape
    codes = torch.full((rows, cols), 99, dtype=torch.int8, device=DEV)
    scale = torch.full((rows,), -1.0, device=DEV)
    co.carryover_quantize_i8(rows, cols, "bf16" if x.dtype == torch.bfloat16 else "f32", x, codes, scale)
    return codes, scale


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 64), (3, 768), (17, 4096), (5, 20480), (2, 131008), (2, 131136),
                                       (700, 192), (33, 8256)])
def test_codes_and_scales(rows, cols, dtype):
    print(f"[quantize] {rows} x {cols} {dtype}", flush=True)
    g = torch.Generator(device=DEV).manual_seed(rows * cols)
    x = (torch.randn(rows, cols, generator=g, device=DEV) * torch.exp2(
        20 * torch.rand(rows, 1, generator=g, device=DEV) - 10)).to(typed(dtype))
    codes, scale = quantize(x)
    want, s = head.quantize(np_(x))
    np.testing.assert_array_equal(np_(codes), want)
    within(np_(scale), s, F32 * s, "scale")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_special_rows(dtype):
    """Middles of two codes, zeros, tiny and huge rows, infinities and NaNs."""
    n = 256
    x = torch.zeros(12, n)
    x[0] = torch.arange(n) * 0.25 - 31.75          # 127 x / 31.75 = 4 x: whole numbers
    x[1] = torch.arange(n) * 0.5 - 63.5            # 2 x
    x[2] = (torch.arange(n) - 128) * 0.5
    x[2, 0] = 127.0                                # codes are x: middles at every other entry
    x[4] = torch.randn(n, generator=torch.Generator().manual_seed(1)) * 2.0 ** -133
    x[5, 3] = 2.0 ** -126
    x[6] = torch.linspace(-3e38, 3e38, n)
    x[7] = 1.0
    x[7, 9] = float("inf")
    x[8, 200] = float("nan")
    x[9] = -1.0
    x[10, 255] = -5.0
    x[11] = 127 * 2.0 ** -126
    x = x.to(typed(dtype)).to(DEV)
    codes, scale = quantize(x)
    want, s = head.quantize(np_(x))
    np.testing.assert_array_equal(np_(codes), want)
    within(np.nan_to_num(np_(scale), nan=-7), np.nan_to_num(s, nan=-7), F32 * np.nan_to_num(s), "scale")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_the_longest_row(dtype):
    """2^31 - 64 columns: the column behind a thread's last one passes 31 bits.  A few entries in
    all of it, the largest at the end; what lies behind the row stays as it was."""
    cols, guard = 2 ** 31 - 64, 1 << 20
    print(f"[quantize] 1 x {cols} {dtype}", flush=True)
    x = torch.zeros(cols + guard, dtype=typed(dtype), device=DEV)
    x[cols:] = 1000.0                                   # (a row that reads on has another scale)
    at = [0, 7, 8191, 8192, 10 ** 9 + 1, cols - 8193, cols - 8192, cols - 9, cols - 1]
    value = [1.0, -2.0, 3.0, -4.0, 5.0, -6.0, 7.0, -8.0, 127.0]
    for i, v in zip(at, value):
        x[i] = v
    codes = torch.full((cols + guard,), 99, dtype=torch.int8, device=DEV)
    scale = torch.full((2,), -1.0, device=DEV)
    co.carryover_quantize_i8(1, cols, dtype, x, codes, scale)
    assert scale.tolist() == [1.0, -1.0]
    assert [int(codes[i]) for i in at] == value
    assert (codes[cols:] == 99).all()
    parts = [codes[a:min(a + (1 << 28), cols)] for a in range(0, cols, 1 << 28)]
    assert sum(int(p.count_nonzero()) for p in parts) == len(at)


def test_quantize_of_no_rows_touches_nothing():
    s = torch.full((4,), 5.0, device=DEV)
    c = torch.full((4, 64), 7, dtype=torch.int8, device=DEV)
    co.carryover_quantize_i8(0, 64, "f32", torch.zeros(4, 64, device=DEV), c, s)
    assert (s == 5).all() and (c == 7).all()


# ------------------------------------------------------------------ product

def operands(m, n, k, seed, bias):
    g = torch.Generator(device=DEV).manual_seed(seed)
    a = torch.randint(-128, 128, (m, k), generator=g, device=DEV, dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    sa = 0.01 + torch.rand(m, generator=g, device=DEV)
    sw = 0.001 + 0.01 * torch.rand(n, generator=g, device=DEV)
    b = 100 * torch.randn(n, generator=g, device=DEV) if bias else None
    return a, sa, w, sw, b


def product(a, sa, w, sw, b, dtype, stream=None):
    (m, k), n = a.shape, w.shape[0]
    guard = 64                                          # past the end: left as it was
    out = torch.full((m * n + guard,), 3.0, dtype=typed(dtype), device=DEV)
    ws = torch.full((max(256, co.matmul_i8_workspace_bytes(m, n, k)),), 0xA5, dtype=torch.uint8, device=DEV)
    co.carryover_matmul_i8(m, n, k, a, sa, w, sw, b, dtype, out, ws, stream)
    assert (out[m * n:] == 3).all()
    return out[:m * n].view(m, n)


def check_product(a, sa, w, sw, b, dtype, got, what):
    acc = torch.matmul(a.double(), w.double().t()).cpu().numpy()      # whole numbers below 2^53
    y = acc * (np_(sa)[:, None] * np_(sw))
    want = y if b is None else y + np_(b)
    tol = 3.01 * F32 * np.abs(y) + F32 * np.abs(want)
    if dtype == "bf16":
        tol = tol + BF16 * (np.abs(want) + tol)
    within(np_(got), want, tol, what)


SIZES = [(1, 1, 64), (1, 256, 768), (2, 3, 131008), (16, 64, 64), (16, 4096, 1024), (17, 1000, 4096),
         (33, 33, 128), (64, 129, 448), (65, 2048, 192), (77, 321, 832), (128, 128, 6400), (130, 257, 192),
         (256, 512, 1024), (300, 5000, 256), (512, 300, 2048), (545, 1111, 320), (1025, 640, 576),
         (4, 40000, 128), (3000, 17, 512), (31, 96, 20480)]


@pytest.mark.parametrize("dtype,bias", [("bf16", False), ("f32", True)])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(m, n, k, dtype, bias):
    print(f"[product] {m} x {n} x {k} {dtype}", flush=True)
    ops = operands(m, n, k, m * n + k, bias)
    check_product(*ops, dtype, product(*ops, dtype), f"{m} x {n} x {k}")


@pytest.mark.parametrize("variant", range(10))
def test_product_variants(variant, tune):
    """Every tile at sizes that end inside it, with one stage of K, few and many, with and
    without a split of K."""
    tune("matmul_i8", variant)
    for m, n, k in ((1, 1, 64), (31, 255, 128), (70, 300, 256), (257, 129, 640), (193, 513, 4096), (20, 70, 8256),
                    (513, 260, 1088)):
        print(f"[product] variant {variant}: {m} x {n} x {k}", flush=True)
        ops = operands(m, n, k, m + n + k, True)
        check_product(*ops, "f32", product(*ops, "f32"), f"variant {variant}: {m} x {n} x {k}")


def test_product_of_the_largest_sums():
    """-128 times -128 at the longest rows: 131008 * 2^14, the sum that fits 32 bits."""
    m, n, k = 3, 5, 131008
    a = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    w = torch.full((n, k), -128, dtype=torch.int8, device=DEV)
    w[1] = 127
    one = torch.ones(5, device=DEV)
    got = product(a, one[:m], w, one, None, "f32")
    want = np.full((m, n), 131008.0 * 16384)
    want[:, 1] = -131008.0 * 128 * 127
    within(np_(got), want, F32 * np.abs(want), "largest sums")


def test_product_of_a_row_that_is_not_finite():
    x = torch.randn(4, 128, device=DEV)
    x[2, 5] = float("inf")
    a, sa = quantize(x)
    w, sw = quantize(torch.randn(70, 128, device=DEV))
    got = product(a, sa, w, sw, None, "bf16")
    assert torch.isnan(got[2]).all() and torch.isfinite(got[[0, 1, 3]]).all()


@pytest.mark.parametrize("m,n", [(0, 5), (5, 0)])
def test_product_without_rows(m, n):
    out = torch.full((16,), 2.0, device=DEV)
    a = torch.zeros(8, 64, dtype=torch.int8, device=DEV)
    s = torch.zeros(8, device=DEV)
    co.carryover_matmul_i8(m, n, 64, a, s, a, s, None, "f32", out, None)
    assert (out == 2).all()


@pytest.mark.parametrize("m", [3, 16, 19, 32])
def test_product_of_few_rows_with_many_columns(m):
    """Two column tiles a workgroup, the second of the last one partly and wholly outside."""
    for n, k in ((16389, 1088), (17010, 1024)):
        print(f"[product] {m} x {n} x {k}", flush=True)
        ops = operands(m, n, k, m + n, False)
        check_product(*ops, "bf16", product(*ops, "bf16"), f"{m} x {n} x {k}")


@pytest.mark.parametrize("dtype,bias", [("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("m,n,k,forced", [
    (33, 70, 8256, False), (45, 3001, 4160, False), (47, 255, 1088, False), (64, 130, 8256, False),   # split over K
    (33, 70, 64, True), (48, 65, 448, True), (64, 300, 960, True),                                    # in one part
    (16, 33000, 5184, False), (1, 70, 64, True), (5, 300, 448, True), (16, 64, 960, True),
    (17, 33, 448, True), (32, 300, 960, True), (16, 4096, 20480, False)])
def test_product_of_streamed_weights(m, n, k, forced, dtype, bias, tune):
    """The kernel for up to 64 rows with one, two and four row tiles, K whole and in parts."""
    print(f"[product] {m} x {n} x {k} {dtype} bias={bias} forced={forced}", flush=True)
    if forced:
        tune("matmul_i8", 9)
    parts = co.matmul_i8_workspace_bytes(m, n, k) > 0
    assert parts == (k >= 1024 and n != 33000)
    ops = operands(m, n, k, m + n + k, bias)
    check_product(*ops, dtype, product(*ops, dtype), f"{m} x {n} x {k}")


def test_product_repeats_bit_for_bit_on_another_stream():
    ops = operands(45, 3001, 4160, 5, True)
    first = product(*ops, "f32")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = product(*ops, "f32")
        third = product(*ops, "f32", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, second) and torch.equal(first, third)


# ------------------------------------------------- projection in 8 bits

def project_case(S, B, Dcat, d, L, Hkv, hd, theta, seed, norms, embed=True, skip=0.1):
    rng = np.random.default_rng(seed)
    M, nkv, CP = S * B, 2 * L * Hkv * hd, -(-B // 16)
    bf = lambda x: torch.tensor(x, dtype=torch.float32).bfloat16().to(DEV)  # noqa: E731
    f = lambda x: torch.tensor(x, dtype=torch.float32, device=DEV)  # noqa: E731
    hidden = bf(rng.standard_normal((M, Dcat)))
    wf, wfs = quantize(bf(0.02 * rng.standard_normal((d, Dcat))))
    wkv, wkvs = quantize(bf(0.02 * rng.standard_normal((nkv, d))))
    f_e = f(0.3 * rng.standard_normal(d)) if embed else None
    zn = f(1 + 0.1 * rng.standard_normal(d)) if norms else None
    kn = f(1 + 0.1 * rng.standard_normal((L, hd))) if norms else None
    pages = S * 3 + M // 16 + 2
    table = rng.permutation(pages)
    pos = np.zeros((S, B), np.int64)
    dst = np.full((S, B), oracle.SKIP, np.int64)
    at = 0
    for s in range(S):
        p0, m = int(rng.integers(0, 40000)), int(rng.integers(0, B + 1))
        for j in range(B):
            pos[s, j] = p0 + j
            if rng.random() < skip:
                continue
            if j < m:
                dst[s, j] = table[at // 16] * 16 + at % 16
                at += 1
            else:
                dst[s, j] = -1 - (j - m)
        at = -(-at // 16) * 16
    assert at // 16 <= pages
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    dims = co.make_dims(S, B, Dcat, d, L, Hkv, Hkv, hd, 4, pages, "bf16", theta)
    st = co.alloc_state(dims, np.zeros((S, 4)), DEV)
    for k in ("k_cache", "v_cache", "k_carry", "v_carry"):
        st[k].fill_(77.0)
    rt = dict(accept_len=i32(np.zeros(S)), row_pos=i32(pos), row_dst=i32(dst))
    W = co.weights_i8(wf, wfs, wkv, wkvs, f_e, zn, kn)
    return dict(dims=dims, W=W, keep=(wf, wfs, wkv, wkvs, f_e, zn, kn), hidden=hidden, st=st, rt=rt, pos=pos,
                dst=dst, shape=(S, B, L, Hkv, hd, CP), theta=theta)


def run_project(c, stream=None):
    ws = torch.full((co.workspace_bytes(c["dims"], co.CO_WS_PROJECT_I8),), 0xA5, dtype=torch.uint8, device=DEV)
    co.carryover_project_kv_i8(c["dims"], c["W"], c["hidden"], c["rt"], c["st"], ws, stream)


def check_project(c):
    S, B, L, Hkv, hd, CP = c["shape"]
    wf, wfs, wkv, wkvs, f_e, zn, kn = (None if x is None else np_(x) for x in c["keep"])
    dst, pos = c["dst"].reshape(-1), c["pos"].reshape(-1)
    carried = (dst < 0) & (dst != oracle.SKIP)
    k, v, k_off, v_off, size = head.project_i8(np_(c["hidden"]), wf, wfs, wkv, wkvs, f_e, carried, pos, L, Hkv,
                                               hd, c["theta"], zn, kn)
    want = {n: np.full(c["st"][n].shape, 77.0) for n in ("k_cache", "v_cache", "k_carry", "v_carry")}
    tol = {n: np.zeros(c["st"][n].shape) for n in want}
    # fp32 operations before the rounding to bf16 are some ten of 2^-24, the rotation's sine and
    # cosine good to 2^-16: all below a 2^-14 of the pair's entries
    kt = k_off + BF16 * (np.abs(k) + k_off) + 2.0 ** -14 * size
    vt = v_off + BF16 * (np.abs(v) + v_off) + 2.0 ** -18 * np.abs(v)
    for r, d in enumerate(dst):
        if d == oracle.SKIP:
            continue
        if d >= 0:
            at, to = (slice(None), d // 16), ("k_cache", "v_cache")
            t = d % 16
        else:
            at, to = (slice(None), r // B, (-1 - d) // 16), ("k_carry", "v_carry")
            t = (-1 - d) % 16
        want[to[0]][at][:, :, t], tol[to[0]][at][:, :, t] = k[r], kt[r]
        want[to[1]][at][:, :, :, t], tol[to[1]][at][:, :, :, t] = v[r], vt[r]
    assert int(c["st"]["status"]) == 0
    for n in want:
        within(np_(c["st"][n]), want[n], tol[n], n)


@pytest.mark.parametrize("S,B,Dcat,d,L,Hkv,hd,theta,norms", [
    (1, 1, 64, 64, 1, 1, 64, 1e4, False),
    (1, 16, 768, 256, 1, 2, 64, 1e4, False),
    (1, 16, 20480, 512, 1, 8, 128, 1e6, False),
    (3, 7, 320, 448, 2, 3, 128, 1e6, True),
    (32, 16, 768, 256, 1, 2, 64, 1e4, True),
    (20, 16, 1024, 1088, 5, 2, 128, 1e6, False),
    (40, 33, 192, 128, 1, 1, 64, 1e4, False),
])
def test_project(S, B, Dcat, d, L, Hkv, hd, theta, norms):
    print(f"[project i8] S={S} B={B} {Dcat}->{d} L={L} {Hkv}x{hd} norms={norms}", flush=True)
    c = project_case(S, B, Dcat, d, L, Hkv, hd, theta, S * B + d, norms)
    run_project(c)
    check_project(c)


@pytest.mark.parametrize("variant", range(10))
@pytest.mark.parametrize("S,B,Dcat,d,L,Hkv,hd", [(5, 16, 192, 128, 1, 1, 64), (9, 15, 320, 1088, 2, 3, 128),
                                                  (3, 100, 64, 64, 1, 5, 64), (2, 13, 256, 2112, 1, 1, 128)])
def test_project_variants(variant, S, B, Dcat, d, L, Hkv, hd, tune):
    """Every tile of both products, whose last one stores the rows itself, split and unsplit."""
    print(f"[project i8] variant {variant} S={S} B={B} {Dcat}->{d} L={L} {Hkv}x{hd}", flush=True)
    tune("matmul_i8", variant)
    c = project_case(S, B, Dcat, d, L, Hkv, hd, 1e4, variant + d, False)
    run_project(c)
    check_project(c)


@pytest.mark.parametrize("S,B,hd", [(1, 4, 128), (3, 7, 64), (1, 32, 128)])
def test_project_of_few_rows_into_many_heads(S, B, hd):
    """Two column tiles a workgroup, which are rotation pairs of a head."""
    c = project_case(S, B, 128, 1088, 5, 2048 // hd, hd, 1e4, S * B, False)
    run_project(c)
    check_project(c)


@pytest.mark.parametrize("S,B,Dcat,d,norms,force", [
    (1, 5, 64, 4160, True, None),              # F's results in fp32, z's rows in registers
    (5, 16, 128, 4160, False, None),
    (1, 16, 6400, 4160, True, None),           # F's parts added up by the reader
    (2, 3, 64, 16384, True, None),
    (1, 3, 1088, 16384, True, 9),
    (1, 5, 64, 16448, False, None),            # z's rows by way of memory, over F's results
    (5, 16, 64, 16448, False, None),
    (2, 7, 1088, 16448, False, 9),             # or beside its parts
    (1, 2, 64, 20480, False, None),
])
def test_project_of_wide_models(S, B, Dcat, d, norms, force, tune):
    print(f"[project i8] S={S} B={B} {Dcat}->{d} norms={norms} force={force}", flush=True)
    if force is not None:
        tune("matmul_i8", force)
    c = project_case(S, B, Dcat, d, 1, 1, 64, 1e4, S * B + d, norms)
    run_project(c)
    check_project(c)


@pytest.mark.parametrize("S,B,Dcat,d,L,Hkv,hd,norms", [
    (3, 16, 4160, 1088, 1, 2, 128, False), (3, 16, 4160, 1088, 1, 2, 128, True), (11, 3, 2112, 1088, 1, 1, 64, True),
    (4, 16, 8256, 2048, 2, 1, 64, False)])
def test_project_of_up_to_64_rows(S, B, Dcat, d, L, Hkv, hd, norms):
    """33 to 64 rows whose products are both split over K: z and the stores add the parts up."""
    print(f"[project i8] S={S} B={B} {Dcat}->{d} L={L} {Hkv}x{hd} norms={norms}", flush=True)
    c = project_case(S, B, Dcat, d, L, Hkv, hd, 1e6, S * B + d, norms)
    run_project(c)
    check_project(c)


def test_project_without_an_embedding():
    c = project_case(2, 8, 256, 256, 1, 2, 64, 1e4, 9, False, embed=False)
    run_project(c)
    check_project(c)


def test_project_reports_pages_that_are_not_there():
    c = project_case(2, 8, 128, 128, 1, 1, 64, 1e4, 4, False, skip=0.0)
    pages = c["dims"].num_pages
    c["dst"][0, 0] = pages * 16
    c["rt"]["row_dst"] = torch.tensor(c["dst"], dtype=torch.int32, device=DEV)
    run_project(c)
    assert int(c["st"]["status"]) == co.CO_ERR_PAGE_RANGE
    c["st"]["status"].zero_()
    c["dst"][0, 0] = oracle.SKIP
    check_project(c)


# ------------------------------------------------------------------ history

def history_dims(S, B=16):
    return co.make_dims(S, B, 64, 64, 1, 1, 1, 64, 1, 1, "bf16", 1e4)


def u16(x):
    return np_(x).astype(np.int64) & 0xFFFF


@pytest.mark.parametrize("S,V,width,flags", [
    (1, 1, 1, 0), (1, 50, 40, 3), (3, 1000, 16, 0), (5, 1000, 64, 1), (4, 1000, 65, 0), (2, 8192, 300, 2),
    (3, 8193, 5000, 3), (7, 32001, 700, 1), (2, 40000, 64, 3), (600, 77, 8, 0), (2, 131077, 3001, 3),
    (300, 70003, 90, 3), (3, 65537, 2000, 2), (150, 70001, 100, 1)])
@pytest.mark.parametrize("lens", [True, False])
def test_history(S, V, width, flags, lens):
    print(f"[history] S={S} V={V} width={width} flags={flags}", flush=True)
    rng = np.random.default_rng(S * V + width)
    seen = rng.integers(0, 3, (S, V)) * rng.integers(0, 2, (S, V)) + 0x8000 * rng.integers(0, 2, (S, V))
    seen[0, 0] = 32766
    tok = (V * rng.random((S, width)) ** 3).astype(np.int64)
    tok[rng.random((S, width)) < 0.1] = -1
    tok[0, :] = 0                                        # one token over and over
    n = rng.integers(0, width + 1, S) if lens else None
    dev = torch.full((S * V + 8,), 1234, dtype=torch.int16, device=DEV)
    dev[:S * V] = torch.tensor(seen.astype(np.uint16).view(np.int16).reshape(-1))
    st = zero()
    i32 = lambda x: torch.tensor(np.array(x), dtype=torch.int32, device=DEV)  # noqa: E731
    co.carryover_count_tokens(history_dims(S), V, width, i32(tok), None if n is None else i32(n), flags, dev, st)
    want, _ = head.count_tokens(seen, tok, n, bool(flags & 1), bool(flags & 2))
    np.testing.assert_array_equal(u16(dev[:S * V]).reshape(S, V), want.astype(np.int64))
    assert (dev[S * V:] == 1234).all() and int(st) == 0


@pytest.mark.parametrize("width", [4, 100])
def test_history_errors_leave_the_rest(width):
    S, V = 4, 300
    tok = torch.randint(0, V, (S, width), dtype=torch.int32, device=DEV)
    tok[1, 2] = V
    lens = torch.tensor([3, 3, -1, width + 1], dtype=torch.int32, device=DEV)
    for bad, code in ((lens, None), (torch.tensor([3, 3, 0, 0], dtype=torch.int32, device=DEV),
                                     co.CO_ERR_TOKEN)):
        seen, st = torch.zeros(S, V, dtype=torch.int16, device=DEV), zero()
        co.carryover_count_tokens(history_dims(S), V, width, tok, bad, 0, seen, st)
        want, _ = head.count_tokens(np.zeros((S, V)), np_(tok), np_(bad), False, False)
        np.testing.assert_array_equal(u16(seen), want)
        assert int(st) == (code or int(st)) and int(st) in (co.CO_ERR_TOKEN, co.CO_ERR_LENGTH)


def test_history_of_nothing():
    seen, st = torch.full((2, 10), 5, dtype=torch.int16, device=DEV), zero()
    tok = torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    co.carryover_count_tokens(history_dims(2), 10, 0, tok, None, co.CO_COUNT_FRESH, seen, st)
    co.carryover_count_tokens(history_dims(2), 10, 4, tok, torch.zeros(2, dtype=torch.int32, device=DEV),
                              co.CO_COUNT_FRESH, seen, st)
    assert (seen == 5).all() and int(st) == 0


# --------------------------------------------------------- rules, probabilities

@pytest.mark.parametrize("mask", [-1, 0])
def test_rules_of_empty_lists(mask):
    """A batch in which no request has a bias and there are no masks; a mask named all the
    same allows nothing."""
    S, V = 2, 300
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    r = co.logit_rules(bias_start=i32([0, 0, 0]), bias_tok=i32([]), bias_val=torch.empty(0, device=DEV),
                       mask_row=i32([[mask], [-1]]), mask_bits=torch.empty(0, 10, dtype=torch.int32, device=DEV))
    x, st = torch.randn(S, 1, V, device=DEV), zero()
    out = torch.empty_like(x)
    co.carryover_logit_rules(history_dims(S), V, 1, "f32", x, None, r, out, st)
    assert torch.equal(out[1], x[1])
    assert torch.isneginf(out[0]).all() if mask == 0 else torch.equal(out[0], x[0])
    assert int(st) == (co.CO_ERR_MASK if mask == 0 else 0)


class Logits:
    """Logits of a batch with rules, beside the oracle."""

    def __init__(self, S, B, R, V, dtype, seed, window=True, penalties=True, bias=0, masked=0.0, greedy=0.2,
                 spread=3.0):
        rng = self.rng = np.random.default_rng(seed)
        self.S, self.B, self.R, self.V, self.dtype = S, B, R, V, dtype
        self.x = torch.tensor(spread * rng.standard_normal((S, R, V)), dtype=torch.float32).to(typed(dtype)).to(DEV)
        self.draft = rng.integers(0, V, (S, B)) if window else None
        if window and B > 1:
            self.draft[:, 1] = self.draft[:, 0]          # the same token twice
        self.seen = self.pen = None
        if penalties:
            self.seen = np.where(rng.random((S, V)) < 0.2, rng.integers(0, 4, (S, V)), 0) + \
                0x8000 * (rng.random((S, V)) < 0.1)
            self.pen = [rng.choice([1.0, 1.3, 0.7], S), rng.choice([0.0, 0.5, -0.25], S),
                        rng.choice([0.0, 0.3], S)]
        self.start = self.tok = self.val = None
        if bias:
            n = rng.integers(0, bias + 1, S)
            self.start = np.concatenate([[0], np.cumsum(n)])
            self.tok = rng.integers(0, max(1, V // 2), self.start[-1] + 3)     # tokens come twice
            self.val = rng.standard_normal(len(self.tok))
            self.val[rng.random(len(self.tok)) < 0.1] = -np.inf                # a bias may forbid
        self.mask_row = self.bits = None
        if masked:
            self.mask_row = np.where(rng.random((S, R)) < masked, rng.integers(0, S * R, (S, R)), -1)
            self.allowed = rng.random((S * R, -(-V // 32) * 32)) < rng.random((S * R, 1))
            self.allowed[0, :V] = False
            self.mask_row[0, 0] = 0                                            # a row with nothing left
            self.bits = np.packbits(self.allowed, axis=1, bitorder="little").view(np.uint32)
        self.temp = rng.choice([1.0, 0.7, 2.5], S)
        self.temp[rng.random(S) < greedy] = 0.0
        self.status = zero()
        self.dims = history_dims(S, B)

    def rules(self):
        f = lambda x: None if x is None else torch.tensor(np.array(x), dtype=torch.float32, device=DEV)  # noqa: E731
        i = lambda x: None if x is None else torch.tensor(np.array(x), dtype=torch.int32, device=DEV)  # noqa: E731
        seen = None if self.seen is None else torch.tensor(
            self.seen.astype(np.uint16).view(np.int16), device=DEV)
        bits = None if self.bits is None else torch.tensor(self.bits.view(np.int32), device=DEV)
        p = self.pen or [None] * 3
        t = dict(seen=seen, repetition=f(p[0]), presence=f(p[1]), frequency=f(p[2]), bias_start=i(self.start),
                 bias_tok=i(self.tok), bias_val=f(self.val), mask_row=i(self.mask_row), mask_bits=bits)
        self.keep = t
        return co.logit_rules(**t)

    def device_draft(self):
        return None if self.draft is None else torch.tensor(self.draft, dtype=torch.int32, device=DEV)

    def apply(self, out=None, stream=None):
        r, d = self.rules(), self.device_draft()
        out = torch.full_like(self.x, 7.0) if out is None else out
        co.carryover_logit_rules(self.dims, self.V, self.R, self.dtype, self.x, d, r, out, self.status, stream)
        torch.cuda.synchronize()
        return out

    def probs(self, top=True, temperature=True, rules=True, stream=None):
        r, d = self.rules() if rules else None, self.device_draft()
        n = self.S * self.R * self.V
        p = torch.full((n + 64,), 7.0, device=DEV)
        t = torch.tensor(self.temp, dtype=torch.float32, device=DEV) if temperature else None
        first = torch.full((self.S, self.R), -9, dtype=torch.int32, device=DEV) if top else None
        ws = torch.full((max(256, co.probabilities_workspace_bytes(self.dims, self.V, self.R)),), 0xA5,
                        dtype=torch.uint8, device=DEV)
        co.carryover_probabilities(self.dims, self.V, self.R, self.dtype, self.x, d, r, t, p, first, self.status,
                                   ws, stream=stream)
        torch.cuda.synchronize()
        assert (p[n:] == 7).all()
        return p[:n].view(self.S, self.R, self.V), first

    def row(self, s, j, rules=True):
        if not rules:
            return head.rules_row(np_(self.x[s, j]))
        f32 = lambda v: float(np.float32(v))  # noqa: E731
        kw = {}
        if self.seen is not None:
            kw = dict(word=self.seen[s], repetition=f32(self.pen[0][s]), presence=f32(self.pen[1][s]),
                      frequency=f32(self.pen[2][s]), window=() if self.draft is None else self.draft[s, :j])
        if self.start is not None:
            a, b = self.start[s], self.start[s + 1]
            kw["biases"] = [(t, f32(v)) for t, v in zip(self.tok[a:b], self.val[a:b])]
        if self.mask_row is not None and self.mask_row[s, j] >= 0:
            kw["allowed"] = self.allowed[self.mask_row[s, j], :self.V]
        return head.rules_row(np_(self.x[s, j]), **kw)

    def check(self, out):
        for s in range(self.S):
            for j in range(self.R):
                want, err = self.row(s, j)
                if self.dtype == "bf16":
                    with np.errstate(invalid="ignore"):
                        err = np.where(np.isfinite(want), err + BF16 * (np.abs(want) + err), 0)
                within(np_(out[s, j]), want, np.where(np.isfinite(err), err, 0), f"row {s} {j}")

    def check_probs(self, p, top, rules=True, temperature=True):
        for s in range(self.S):
            for j in range(self.R):
                x, err = self.row(s, j, rules)
                t = float(np.float32(self.temp[s])) if temperature else 1.0
                want, tol, first = head.probabilities_row(x, err, t)
                got = np_(p[s, j])
                if top is not None:
                    f = int(top[s, j])
                    # a logit within its roundings of the largest may stand for it
                    assert f == first or (first >= 0 and x[f] + err[f] + err[first] >= x[first]), f"top of row {s} {j}"
                    if first >= 0 and not t > 0:
                        want = np.zeros(self.V)
                        want[f] = 1.0
                within(got, want, tol, f"row {s} {j}")


CASES = [
    # S, B, R, V, dtype, window, penalties, bias, masked
    (1, 1, 1, 1, "f32", True, True, 0, 0.0),
    (1, 16, 17, 1000, "f32", True, True, 0, 0.0),
    (2, 16, 17, 1000, "bf16", True, True, 9, 0.5),
    (5, 7, 8, 2047, "bf16", True, True, 20, 1.0),
    (3, 7, 7, 2048, "f32", False, True, 300, 0.3),
    (4, 1, 1, 2049, "bf16", False, False, 5, 0.0),
    (3, 16, 16, 4100, "f32", True, False, 0, 1.0),
    (64, 1, 1, 777, "f32", False, True, 30, 0.25),
    (2, 3, 4, 32001, "bf16", True, True, 50, 0.5),
    (9, 4, 5, 9001, "f32", True, True, 50, 0.5),
    (1, 40, 41, 130, "bf16", True, True, 4, 0.2),
    (1, 100, 101, 40, "f32", True, True, 4, 0.2),          # more proposals than lanes
    (2, 100, 101, 17000, "bf16", True, True, 0, 0.0),
    (2, 3, 4, 600, "f32", True, True, 1500, 0.3),          # more biases of a tile than are held
    (1, 1, 2, 20000, "bf16", False, True, 9000, 0.0),
    (3, 2, 3, 7, "f32", True, True, 3, 0.5),               # less than a vector
    (1, 2, 3, 131072, "bf16", True, True, 100, 0.3),
    (300, 2, 3, 33, "f32", True, True, 3, 0.3),
    (200, 3, 4, 8195, "bf16", True, True, 3, 0.3),
]


@pytest.mark.parametrize("c", CASES, ids=str)
def test_rules(c):
    print(f"[rules] {c}", flush=True)
    S, B, R, V, dtype, window, penalties, bias, masked = c
    a = Logits(S, B, R, V, dtype, S * V + R, window, penalties, bias, masked)
    before = a.x.clone()
    out = a.apply()
    assert torch.equal(before, a.x) and int(a.status) == 0
    a.check(out)
    same = a.x                                             # in place, the same bits
    a.apply(out=same)
    assert torch.equal(same, out)


@pytest.mark.parametrize("c", CASES, ids=str)
def test_probabilities(c):
    print(f"[probabilities] {c}", flush=True)
    S, B, R, V, dtype, window, penalties, bias, masked = c
    a = Logits(S, B, R, V, dtype, S * V + R + 1, window, penalties, bias, masked)
    before = a.x.clone()
    p, top = a.probs()
    assert torch.equal(before, a.x) and int(a.status) == 0
    a.check_probs(p, top)


@pytest.mark.parametrize("S,R,V,bias", [(2, 3, 300, 3000), (2, 5, 4099, 9000), (1, 3, 9000, 9000), (2, 2, 16001, 60000),
                                        (1, 6, 20011, 50000)])
def test_long_lists_of_biases(S, R, V, bias):
    """Tokens many times over, more distinct ones in a tile than it can look up, and lists of
    which a tile holds few."""
    print(f"[biases] {S} x {R} x {V}, up to {bias}", flush=True)
    a = Logits(S, 7, R, V, "f32", V, bias=bias, masked=0.3)
    a.check(a.apply())
    a.check_probs(*a.probs())


@pytest.mark.parametrize("S,B,R,V,dtype,window,bias,masked,crowded", [
    (2, 8, 9, 32001, "bf16", True, 30, 0.5, False), (2, 8, 9, 32001, "f32", True, 30, 0.5, False),
    (3, 16, 17, 20011, "bf16", True, 0, 0.0, False), (1, 16, 17, 128000, "bf16", True, 100, 0.25, False),
    (1, 4, 3, 128000, "f32", False, 0, 0.0, False), (40, 2, 3, 16385, "f32", True, 5, 0.3, False),
    (2, 8, 9, 32001, "bf16", True, 30, 0.5, True), (5, 1, 1, 50003, "f32", False, 20, 1.0, True)])
def test_sparse_histories_of_large_vocabularies(S, B, R, V, dtype, window, bias, masked, crowded):
    """Few special tokens in most tiles, as a text of hundreds of tokens leaves them: the second
    pass finds their marks and logits in the workspace.  crowded: every token of one block of 512
    was seen, so that its tile has more than the workspace holds, beside tiles that have few."""
    print(f"[sparse] {S} x {R} x {V} {dtype} crowded={crowded}", flush=True)
    a = Logits(S, B, R, V, dtype, S * V + R, window, True, bias, masked)
    rng = a.rng
    a.seen = np.where(rng.random((S, V)) < 0.01, rng.integers(1, 4, (S, V)), 0) + 0x8000 * (rng.random((S, V)) < 0.01)
    a.seen[:, V - 1] = 0x8001                           # behind the last whole vector, or its last
    if crowded:
        a.seen[0, 512:1024] = 0x8000
    a.x[0, 0, 3:5] = float("nan")
    a.x[0, -1, V - 1] = 40.0                            # the largest is special
    p, top = a.probs()
    assert int(a.status) == 0
    a.check_probs(p, top)
    a.check(a.apply())


def test_probabilities_without_rules_or_temperature():
    a = Logits(3, 4, 5, 3001, "bf16", 11, window=False, penalties=False)
    p, top = a.probs(rules=False, temperature=False)
    a.check_probs(p, top, rules=False, temperature=False)
    q, none = a.probs(rules=False, temperature=False, top=False)
    assert none is None and torch.equal(p, q)


def test_results_repeat_bit_for_bit():
    a = Logits(5, 7, 8, 20011, "bf16", 77, bias=40, masked=0.5)
    p, top = a.probs()
    out = a.apply()
    for _ in range(3):
        q, t = a.probs()
        assert torch.equal(p, q) and torch.equal(top, t) and torch.equal(out, a.apply())


def test_counts_stop_at_their_largest():
    """A word that is full stays full in a window, and its prompt bit stays clear."""
    a = Logits(1, 4, 5, 64, "f32", 3, penalties=True)
    a.seen[:] = 0
    a.seen[0, 5], a.seen[0, 6] = 32767, 0x8000 | 32766
    a.draft[:] = [[5, 6, 6, 5]]
    a.pen = [np.array([1.5]), np.array([0.25]), np.array([2.0 ** -10])]
    out = a.apply()
    a.check(out)
    assert float(out[0, 4, 5]) == float(np.float32(a.row(0, 4)[0][5]))


def test_equal_logits_have_equal_probabilities_and_the_lowest_token_wins():
    a = Logits(2, 3, 4, 6000, "bf16", 5, penalties=False, window=False)
    a.x[:] = 1.0
    a.x[:, :, 4000] = 3.0
    a.x[:, :, 5999] = 3.0
    a.x[:, :, 17] = 3.0
    a.temp[:] = [0.0, 1.0]
    p, top = a.probs()
    assert (top == 17).all()
    assert (p[0, :, 17] == 1).all() and (p[0].sum(-1) == 1).all()
    assert (p[1, :, 17] == p[1, :, 4000]).all() and (p[1, :, 17] == p[1, :, 5999]).all()
    assert (p[1, :, 0] == p[1, :, 5998]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 5000])
def test_infinities_and_nans(dtype, V):
    """NaNs are left out; infinite logits share their row; a row of minus infinity or NaNs has
    nothing; masked NaNs and infinities do not count."""
    inf, nan = float("inf"), float("nan")
    a = Logits(2, 6, 7, V, dtype, 3, window=False, penalties=False, masked=0.0)
    a.x[:, 0, 3] = nan
    a.x[:, 1, :] = -inf
    a.x[:, 2, :] = nan
    a.x[:, 3, [5, V - 1]] = inf
    a.x[:, 4, :] = -inf
    a.x[:, 4, V - 2] = -1e30
    a.x[:, 5, [0, 1]] = torch.tensor([inf, nan], device=DEV).to(a.x.dtype)
    a.temp[:] = [1.0, 0.0]
    a.mask_row = np.full((2, 7), -1)
    a.mask_row[:, 5] = 0
    a.allowed = np.ones((1, -(-V // 32) * 32), bool)
    a.allowed[0, [0, 1]] = False
    a.bits = np.packbits(a.allowed, axis=1, bitorder="little").view(np.uint32)
    p, top = a.probs()
    assert int(a.status) == 0
    assert not p[:, 1:3].any() and (top[:, 1:3] == -1).all()
    assert (p[0, 3, [5, V - 1]] == 0.5).all() and p[0, 3].sum() == 1 and (top[:, 3] == 5).all()
    assert p[1, 3, 5] == 1 and p[1, 3].sum() == 1
    assert (p[:, 4, V - 2] == 1).all() and (p[:, 4].sum(-1) == 1).all()
    for s in range(2):
        for j in (0, 5, 6):
            x, err = a.row(s, j)
            want, tol, first = head.probabilities_row(x, err, a.temp[s])
            within(np_(p[s, j]), want, tol, f"{s} {j}")
            assert int(top[s, j]) == first


@pytest.mark.parametrize("t", [1e-30, 1e-45, 1e30, float("inf"), float("nan"), -1.0, -0.0])
def test_temperatures_at_the_ends(t):
    a = Logits(1, 1, 2, 3000, "f32", 8, window=False, penalties=False)
    a.x[0, 1, 1000:] = -float("inf")
    a.temp[:] = t
    p, top = a.probs()
    p = np_(p)
    assert np.isfinite(p).all() and not p[0, 1, 1000:].any()
    if t > 1:                                          # all alike
        within(p[0, 0], np.full(3000, 1 / 3000), 1e-6, "uniform")
        within(p[0, 1, :1000], np.full(1000, 1e-3), 1e-6, "uniform")
    else:                                              # the largest alone
        for j in range(2):
            assert p[0, j, int(top[0, j])] == 1 and p[0, j].sum() == 1


def test_data_errors_are_reported_and_the_rest_is_right():
    def fresh():
        return Logits(3, 4, 5, 700, "f32", 21, bias=6, masked=0.5)
    a = fresh()
    a.draft[1, 2] = 700                                # (out of the vocabulary: not counted)
    a.draft[2, 0] = -1
    out = a.apply()
    assert int(a.status) == co.CO_ERR_TOKEN
    a.check(out)
    a = fresh()
    a.tok[a.start[1]] = -5
    p, top = a.probs()
    assert int(a.status) == (co.CO_ERR_TOKEN if a.start[2] > a.start[1] else 0)
    a.check_probs(p, top)
    for bad in ([0, 5, 2, 6], [-1, 0, 0, 0], [0, 0, 0, 10 ** 6]):
        a = fresh()
        a.tok, a.val = a.rng.integers(0, 700, 9), a.rng.standard_normal(9)
        a.start = np.array(bad)
        out = a.apply()
        assert int(a.status) == co.CO_ERR_LENGTH
        a.start = np.array([0, 0, 0, 0])
        if bad[1] == 5:                                # sequence 0 has its list, 2 has entries 2 .. 5
            a.tok, a.val = (np.concatenate([x[:5], x[2:6]]) for x in (a.tok, a.val))
            a.start = np.array([0, 5, 5, 9])
        a.check(out)
    a = fresh()
    a.mask_row[1, 3] = 15
    out = a.apply()
    assert int(a.status) == co.CO_ERR_MASK and (out[1, 3] == -float("inf")).all()
    a.mask_row[1, 3] = -1
    keep = out[1, 3].clone()
    a.allowed = np.concatenate([a.allowed, np.zeros_like(a.allowed[:1])])
    a.mask_row[1, 3] = 15
    a.check(out)
    assert torch.equal(keep, out[1, 3])


def test_rules_and_probabilities_of_no_sequences():
    a = Logits(1, 1, 1, 40, "f32", 2)
    a.dims = history_dims(0, 1)
    assert (a.apply() == 7).all()


def test_rows_that_start_at_odd_addresses():
    """Buffers that are aligned to one element only, of an odd vocabulary."""
    for dtype in ("bf16", "f32"):
        a = Logits(3, 3, 4, 1001, dtype, 31, bias=4, masked=0.5)
        big = torch.empty(a.x.numel() + 1, dtype=a.x.dtype, device=DEV)
        big[1:] = a.x.reshape(-1)
        a.x = big[1:].view(a.x.shape)
        out = torch.full_like(big, 7.0)
        got = a.apply(out=out[1:].view(a.x.shape))
        assert out[0] == 7
        a.check(got)
        p, top = a.probs()
        a.check_probs(p, top)


def test_rows_past_32_bits():
    """Offsets beyond 2^31 elements: the last rows of a long buffer."""
    S, R, V = 17, 17, 131072 * 64
    dims = history_dims(S, 16)
    x = torch.zeros(S * R * V, dtype=torch.bfloat16, device=DEV).view(S, R, V)
    x[-1, -1, -3] = 30.0
    x[-1, 0, 5] = 30.0
    r = co.logit_rules(bias_start=torch.tensor([0] * S + [1], dtype=torch.int32, device=DEV),
                       bias_tok=torch.tensor([V - 1], dtype=torch.int32, device=DEV),
                       bias_val=torch.tensor([2.0], device=DEV))
    st = zero()
    co.carryover_logit_rules(dims, V, R, "bf16", x, None, r, x, st)
    assert x[-1, -1, -1] == 2 and x[-1, -1, -3] == 30 and x[-1, -2, -1] == 2 and x[-2, -1, -1] == 0
    assert int(st) == 0 and int(torch.count_nonzero(x)) == R + 2
    p = torch.empty(S * R * V, dtype=torch.float32, device=DEV).view(S, R, V)
    top = torch.empty(S, R, dtype=torch.int32, device=DEV)
    ws = torch.empty(co.probabilities_workspace_bytes(dims, V, R), dtype=torch.uint8, device=DEV)
    co.carryover_probabilities(dims, V, R, "bf16", x, None, None, None, p, top, st, ws)
    assert int(top[-1, -1]) == V - 3 and int(top[-1, 0]) == 5 and int(top[0, 0]) == 0
    want = np.exp(30.0) / (np.exp(30.0) + V - 2 + np.exp(2.0))
    assert abs(float(p[-1, -1, -3]) - want) < 1e-4 * want
    assert abs(float(p[0, 0, V - 1]) * V - 1) < 1e-3


# -------------------------------------------- the calls together, and in graphs

def test_a_served_step():
    """Hidden rows to the verifier's answer, as a server runs it: output head in 8 bits, rules and
    probabilities of target and drafter, verification, the accepted tokens into the history, the
    carried and committed rows through the projection in 8 bits.  Every step against the oracle on
    what the step before left on the device; then the same captured and replayed."""
    S, B, V, d, seed = 6, 8, 1003, 256, 77
    R = B + 1
    g = torch.Generator(device=DEV).manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    head_w, head_s = quantize((0.3 * rn(V, d)).bfloat16())
    rows_t, rows_q = rn(S * R, d).bfloat16(), rn(S * B, d).bfloat16()
    rows_q.view(S, B, d).copy_(rows_t.view(S, R, d)[:, :B] + 0.1 * rn(S, B, d).bfloat16())
    dims = history_dims(S, B)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    seen = torch.zeros(S, V, dtype=torch.int16, device=DEV)
    prompt = torch.randint(0, V, (S, 100), generator=g, device=DEV, dtype=torch.int32)
    status = zero()
    co.carryover_count_tokens(dims, V, 100, prompt, None, co.CO_COUNT_PROMPT | co.CO_COUNT_FRESH, seen, status)
    pen = [torch.full((S,), v, device=DEV) for v in (1.2, 0.1, 0.2)]
    temp = torch.tensor([1.0, 0.8, 0.0, 1.0, 1.5, 1.0], device=DEV)
    bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, -(-V // 32)), generator=g, device=DEV).int()
    mask_row = i32(S, R) - 1
    mask_row[1] = 0
    mask_row[4, 2:] = 1
    rules_t = co.logit_rules(seen, *pen, mask_row=mask_row, mask_bits=bits)
    mask_q = mask_row[:, :B].contiguous()
    rules_q = co.logit_rules(seen, *pen, mask_row=mask_q, mask_bits=bits)
    draft = i32(S, B)
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (S, R), generator=g, device=DEV).int()
    buf = {}
    for name, rows in (("t", R), ("q", B)):
        m = S * rows
        buf[name] = dict(codes=torch.zeros(m, d, dtype=torch.int8, device=DEV), scale=torch.zeros(m, device=DEV),
                         logits=torch.zeros(S, rows, V, dtype=torch.bfloat16, device=DEV),
                         probs=torch.zeros(S, rows, V, device=DEV), top=i32(S, rows),
                         mws=torch.zeros(max(256, co.matmul_i8_workspace_bytes(m, V, d)), dtype=torch.uint8, device=DEV),
                         pws=torch.zeros(max(256, co.probabilities_workspace_bytes(dims, V, rows)), dtype=torch.uint8,
                                         device=DEV))
    bits_out, acc, nxt = i32(S, B), i32(S), i32(S)
    c = project_case(S, B, 128, 128, 2, 2, 64, 1e4, 5, False)
    pws = torch.zeros(co.workspace_bytes(c["dims"], co.CO_WS_PROJECT_I8), dtype=torch.uint8, device=DEV)

    def head_of(name, rows, x, draft_tok, rules):
        b, m = buf[name], S * rows
        co.carryover_quantize_i8(m, d, "bf16", x, b["codes"], b["scale"])
        co.carryover_matmul_i8(m, V, d, b["codes"], b["scale"], head_w, head_s, None, "bf16", b["logits"], b["mws"])
        co.carryover_probabilities(dims, V, rows, "bf16", b["logits"], draft_tok, rules, temp, b["probs"], b["top"],
                                   status, b["pws"])

    def step():
        head_of("q", B, rows_q, None, rules_q)
        draft.copy_(buf["q"]["top"])                     # proposals: the drafter's first choices
        head_of("t", R, rows_t, draft, rules_t)
        co.carryover_verify_sample(dims, V, draft, buf["t"]["probs"], buf["q"]["probs"], words, bits_out, acc, nxt,
                                   status)
        co.carryover_count_tokens(dims, V, B, draft, acc, 0, seen, status)
        co.carryover_count_tokens(dims, V, 1, nxt, None, 0, seen, status)
        co.carryover_project_kv_i8(c["dims"], c["W"], c["hidden"], c["rt"], c["st"], pws)

    seen0 = seen.clone()
    step()
    torch.cuda.synchronize()
    assert int(status) == 0
    word = u16(seen0)
    for name, rows in (("q", B), ("t", R)):
        b = buf[name]
        x = rows_q if name == "q" else rows_t
        q, s = head.quantize(np_(x))
        np.testing.assert_array_equal(np_(b["codes"]), q)
        check_product(b["codes"], b["scale"], head_w, head_s, None, "bf16", b["logits"].view(S * rows, V), name)
        for i in range(S):
            for j in range(rows):
                ok = None
                if int(mask_row[i, j]) >= 0:
                    w = np_(bits[int(mask_row[i, j])]).view(np.uint32)
                    ok = np.unpackbits(w.view(np.uint8), bitorder="little")[:V]
                lg, err = head.rules_row(np_(b["logits"][i, j]), word[i],
                                         np_(draft[i, :j]) if name == "t" else (), *(float(np.float32(p)) for p in
                                                                                     (1.2, 0.1, 0.2)), allowed=ok)
                want, tol, first = head.probabilities_row(lg, err, float(temp[i]))
                within(np_(b["probs"][i, j]), want, tol, f"{name} {i} {j}")
                assert int(b["top"][i, j]) == first
    new = word
    for i in range(S):
        m, t, st = oracle.verify_sample(np_(draft[i]), buf["t"]["probs"][i].cpu().numpy(),
                                        buf["q"]["probs"][i].cpu().numpy(), np_(words[i]).view(np.uint32))
        assert (m, t, st) == (int(acc[i]), int(nxt[i]), 0)
        for v in list(np_(draft[i, :m])) + [t]:
            if v >= 0:
                new[i, v] += 1
    np.testing.assert_array_equal(u16(seen), new)
    assert int(acc.max()) > 0 and int(acc.min()) < B
    check_project(c)

    # captured: replays with the program's own work between them give the eager results
    results = [(t, t.clone()) for t in (buf["t"]["probs"], buf["q"]["probs"], draft, acc, nxt, seen,
                                        c["st"]["k_cache"], c["st"]["v_carry"])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    seen.copy_(seen0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(4):
        seen.copy_(seen0)
        for t, _w in results:
            if t is not seen:
                t.zero_()
        c["st"]["k_cache"].fill_(77.0)
        c["st"]["v_carry"].fill_(77.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (t, w) in enumerate(results):
            assert torch.equal(t, w), f"result {i} of a replay"
    assert int(status) == 0


def test_two_streams_at_once():
    """Two batches with buffers of their own, on two streams in turn."""
    jobs = []
    for seed in (1, 2):
        a = Logits(4, 7, 8, 5001, "bf16", seed, bias=9, masked=0.4)
        jobs.append((a, a.rules(), a.device_draft(), torch.tensor(a.temp, dtype=torch.float32, device=DEV),
                     torch.zeros(4, 8, 5001, device=DEV), torch.zeros(4, 8, dtype=torch.int32, device=DEV),
                     torch.zeros(co.probabilities_workspace_bytes(a.dims, 5001, 8), dtype=torch.uint8, device=DEV),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for a, r, d, t, p, top, ws, stream in jobs:
            co.carryover_probabilities(a.dims, a.V, a.R, a.dtype, a.x, d, r, t, p, top, a.status, ws, stream=stream)
    torch.cuda.synchronize()
    for a, r, d, t, p, top, ws, stream in jobs:
        a.check_probs(p, top)
