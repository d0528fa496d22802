"""Products with microscaled 4-bit matrices on the GPU.

Exact cases: operands whose products and partial sums, in any order, are multiples of one power of two below 2^24 of it, so that float32 has
no rounding and every element must be the float64 result rounded once.  Others: N products summed in float32 in any order are off by at most
N steps of 2^-23 (a step that truncates) of the sum of magnitudes, and the result's own rounding by half a step of its type."""
import numpy as np
import pytest

import mx4_reference as R
from test_gpu_mx4 import dev, dtype, floats, mat, nz  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 17, 33), (1, 4096, 4096), (2, 64, 64), (3, 5, 7), (15, 100, 31), (16, 128, 128), (17, 33, 65), (31, 260, 520), (33, 128, 1000),
         (64, 64, 64), (65, 130, 257), (100, 96, 2050), (128, 256, 512), (129, 257, 513), (200, 1030, 96), (257, 300, 771), (300, 515, 4100),
         (512, 512, 512), (520, 776, 1544), (48, 300, 7000), (150, 7000, 300), (31, 100, 6900), (260, 390, 6400), (1, 2, 5000), (5, 2500, 64), (1000, 40, 130), (1031, 1290, 320), (1, 8205, 260), (4, 9000, 2300),
         (6, 8200, 1100), (20, 8200, 140)]


def check(nz, kind, left, b, m, n, k, out, want, ld_pad=0, exact=True, slack=None):
    """Runs the product into a buffer with a frame around it and compares.  left: Mx4, or a float tensor with its own row length."""
    import torch
    inner, outer = (n, k) if kind == nz.MX4_GRAD else (k, n)
    ldc = outer + ld_pad
    y = torch.full((m + 2, ldc), 7.0, dtype=dtype(out), device="cuda:0")
    c = y[1:m + 1] if ldc * y.element_size() % 16 == 0 else y[:m]
    wsb = nz.nz_mx4_workspace_bytes(kind, None if kind == nz.MX4_PRODUCT else left.dtype, m, n, k)
    ws = torch.full((max(wsb, 16),), 0xFF, dtype=torch.uint8, device="cuda:0")
    if kind == nz.MX4_PRODUCT:
        rc = nz.nz_mx4_product(left, b, m, n, k, c, ldc, ws, wsb)
    else:
        call = nz.nz_mx4_linear if kind == nz.MX4_LINEAR else nz.nz_mx4_grad
        rc = call(left, left.shape[1], b, m, n, k, c, ldc, ws, wsb)
    assert rc == 0
    got = c[:, :outer].cpu()
    if exact:
        w = torch.from_numpy(want).float()
        assert np.array_equal(w.double().numpy(), want, equal_nan=True)  # (the case is what it is meant to be)
        w = w.to(dtype(out))
        bad = torch.nonzero(~((got == w) | (got.isnan() & w.isnan())))
        assert bad.numel() == 0, (bad[:4], got[tuple(bad[0])], w[tuple(bad[0])])
    else:
        tol = slack + torch.finfo(dtype(out)).eps / 2 * (np.abs(want) + slack) + torch.finfo(dtype(out)).tiny
        err = np.abs(got.double().numpy() - want)
        assert (err <= tol).all(), (np.argwhere(err > tol)[:4], (err / tol).max())
    assert (c[:, outer:] == 7).all()
    rest = torch.ones(m + 2, dtype=torch.bool)
    at = (c.data_ptr() - y.data_ptr()) // (ldc * y.element_size())
    rest[at:at + m] = False
    assert (y[rest.to(y.device)] == 7).all()
    return y


def exact_floats(rng, rows, cols):
    return rng.integers(-8, 9, (rows, cols)) / 4.0


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_product_exact(nz, size):
    """Multiples of 1/16 (codes of 1/2, scales of 1/2 to 2), at most 144 each: 144 * 7000 * 16 < 2^24."""
    m, n, k = size
    rng = np.random.default_rng(m * 31 + n * 7 + k)
    a, b = R.random_matrix(rng, m, k, 126, 129), R.random_matrix(rng, n, k, 126, 129)
    want = R.values(*a, k) @ R.values(*b, k).T
    for i, out in enumerate(("f32", "bf16", "f16")):
        am, bm = mat(nz, *R.place(*a, k, 4 * i)), mat(nz, *R.place(*b, k, 4 * (i == 1)))
        check(nz, nz.MX4_PRODUCT, am, bm, m, n, k, out, want, ld_pad=3 * i)


@pytest.mark.parametrize("left", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_and_grad_exact(nz, size, left):
    """Floats of 1/4 up to 2 against multiples of 1/4 up to 12: 24 * 7000 * 16 < 2^24."""
    m, n, k = size
    rng = np.random.default_rng(m * 31 + n * 7 + k + 1)
    b = R.random_matrix(rng, n, k, 126, 129)
    w = R.values(*b, k)
    x, g = exact_floats(rng, m, k), exact_floats(rng, m, n)
    for i, out in enumerate(("f32", "bf16", "f16")):
        bm = mat(nz, *R.place(*b, k, 4 * (i == 2)))
        pad = (0, 8, 1)[i]                                               # rows of floats at 16 bytes or not, NaN behind them
        check(nz, nz.MX4_LINEAR, floats(nz, x, left, k + pad)[0], bm, m, n, k, out, x @ w.T, ld_pad=pad)
        check(nz, nz.MX4_GRAD, floats(nz, g, left, n + pad)[0], bm, m, n, k, out, g @ w, ld_pad=pad)


@pytest.mark.parametrize("size", [(1, 40, 20000), (3, 40, 20000), (20, 24, 20011), (40, 24, 20000), (1, 20000, 300), (16, 20001, 40), (33, 20000, 264)],
                         ids=str)
def test_long_sums(nz, size):
    """Scales of 1: multiples of 1/4 up to 36 and of 1/8 up to 12, so 36 * 20011 * 4 and 12 * 20011 * 8 are below 2^24."""
    m, n, k = size
    rng = np.random.default_rng(m + k)
    a, b = R.random_matrix(rng, m, k, 127, 128), R.random_matrix(rng, n, k, 127, 128)
    w = R.values(*b, k)
    bm = mat(nz, *R.place(*b, k))
    check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), bm, m, n, k, "f32", R.values(*a, k) @ w.T)
    for left in ("bf16", "f16", "f32"):
        x, g = exact_floats(rng, m, k), exact_floats(rng, m, n)
        check(nz, nz.MX4_LINEAR, floats(nz, x, left)[0], bm, m, n, k, "f32", x @ w.T)
        check(nz, nz.MX4_GRAD, floats(nz, g, left)[0], bm, m, n, k, "f32", g @ w)


@pytest.mark.parametrize("size", [(3588, 3850, 300), (3841, 4100, 1056)], ids=str)
def test_sizes_that_fill_the_chip(nz, size):
    """Large tiles, ragged in every direction, against float64 on the GPU."""
    import torch
    m, n, k = size
    rng = np.random.default_rng(m)
    a, b = R.random_matrix(rng, m, k, 126, 129), R.random_matrix(rng, n, k, 126, 129)
    av, w = dev(R.values(*a, k)), dev(R.values(*b, k))
    bm = mat(nz, *R.place(*b, k))
    check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), bm, m, n, k, "f32", (av @ w.t()).cpu().numpy(), ld_pad=1)
    for left in ("bf16", "f16"):
        x, g = exact_floats(rng, m, k), exact_floats(rng, m, n)
        check(nz, nz.MX4_LINEAR, floats(nz, x, left, k + 4)[0], bm, m, n, k, "bf16", (dev(x) @ w.t()).cpu().numpy())
        check(nz, nz.MX4_GRAD, floats(nz, g, left, n + 2)[0], bm, m, n, k, "f16", (dev(g) @ w).cpu().numpy())
    # and the widest of the gradient: as many columns of B as make large tiles there
    n, k = k, n
    b = R.random_matrix(rng, n, k, 126, 129)
    g = exact_floats(rng, m, n)
    check(nz, nz.MX4_GRAD, floats(nz, g, "bf16", (n + 7) // 8 * 8)[0], mat(nz, *R.place(*b, k)), m, n, k, "f32", (dev(g) @ dev(R.values(*b, k))).cpu().numpy())


@pytest.mark.parametrize("left", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [(1, 300, 2000), (7, 513, 900), (40, 200, 1500), (130, 700, 260), (600, 300, 515)], ids=str)
def test_linear_and_grad_of_full_mantissas(nz, size, left):
    m, n, k = size
    rng = np.random.default_rng(m + n + k)
    b = R.random_matrix(rng, n, k, 100, 150)
    w = R.values(*b, k)
    bm = mat(nz, *R.place(*b, k))
    x, x64 = floats(nz, rng.standard_normal((m, k)) * 2.0 ** rng.integers(-3, 4, (m, k)), left)
    g, g64 = floats(nz, rng.standard_normal((m, n)) * 2.0 ** rng.integers(-3, 4, (m, n)), left)
    terms = {"bf16": 1, "f16": 2, "f32": 3}[left]                        # a float may count as so many addends
    check(nz, nz.MX4_LINEAR, x, bm, m, n, k, "f32", x64 @ w.T, exact=False, slack=terms * k * 2.0 ** -23 * (np.abs(x64) @ np.abs(w).T))
    check(nz, nz.MX4_GRAD, g, bm, m, n, k, "f32", g64 @ w, exact=False, slack=terms * n * 2.0 ** -23 * (np.abs(g64) @ np.abs(w)))
    a = R.random_matrix(rng, m, k, 100, 150)
    av = R.values(*a, k)
    check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), bm, m, n, k, "f32", av @ w.T, exact=False, slack=k * 2.0 ** -23 * (np.abs(av) @ np.abs(w).T))


@pytest.mark.parametrize("m", [1, 20, 150, 300])
def test_a_float_keeps_all_its_bits(nz, m):
    """One nonzero weight of 1 (or 0.5 in a block of another scale): the result is the float itself, every mantissa bit, zeros beside it."""
    n, k = 96, 256
    rng = np.random.default_rng(m)
    codes, scales = np.zeros((n, k // 2), np.uint8), np.full((n, k // 32), 127, np.uint8)
    pick = rng.permutation(k)[:n]
    for j, i in enumerate(pick):
        codes[j, i // 2] = 2 << (4 * (i % 2))
    bm = mat(nz, *R.place(codes, scales, k))
    for left in ("f32", "bf16", "f16"):
        lo, hi = (-14, 15) if left == "f16" else (-60, 60)
        v = rng.standard_normal((m, k)) * 2.0 ** rng.integers(lo, hi, (m, k))
        x, x64 = floats(nz, v, left)
        check(nz, nz.MX4_LINEAR, x, bm, m, n, k, "f32", x64[:, pick])
        g, g64 = floats(nz, v[:, :n], left)
        want = np.zeros((m, k))
        want[:, pick] = g64
        check(nz, nz.MX4_GRAD, g, bm, m, n, k, "f32", want)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_nan_and_infinity_stay_where_they_belong(nz, m):
    n, k = 200, 420
    rng = np.random.default_rng(4)
    b = R.random_matrix(rng, n, k, 126, 129)
    b[1][7, 3] = 255                                                     # row 7 of B, columns 96 .. 127
    w = R.values(*b, k)
    bm = mat(nz, *R.place(*b, k))
    a = R.random_matrix(rng, m, k, 126, 129)
    a[1][m // 2, 13] = 255                                               # the ragged last block of a row of A
    with np.errstate(invalid="ignore"):
        check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), bm, m, n, k, "f32", R.values(*a, k) @ w.T)
        for left in ("bf16", "f16", "f32"):
            x = exact_floats(rng, m, k)
            x[m - 1, k - 1] = np.inf
            x[0, 5] = np.nan
            t, x64 = floats(nz, x, left, k + 1)
            check(nz, nz.MX4_LINEAR, t, bm, m, n, k, "f32", x64 @ w.T)
            g = exact_floats(rng, m, n)
            g[m - 1, n - 1] = -np.inf
            t, g64 = floats(nz, g, left, n + 1)
            check(nz, nz.MX4_GRAD, t, bm, m, n, k, "f32", g64 @ w)


def test_large_floats_do_not_become_infinite(nz):
    """The largest float32 (whose leading bits round up past the type) times 0.5, and sums that cancel."""
    big = np.float32(3.4028235e38)
    k = 64
    codes, scales = np.zeros((2, 32), np.uint8), np.full((2, 2), 127, np.uint8)
    codes[0, 0] = 0x01                                                   # 0.5 * x0
    codes[1, 0] = 0x91                                                   # 0.5 * x0 - 0.5 * x1
    x = np.zeros((3, k), np.float32)
    x[:, 0] = x[:, 1] = big
    bm = mat(nz, *R.place(codes, scales, k))
    t, x64 = floats(nz, x, "f32")
    check(nz, nz.MX4_LINEAR, t, bm, 3, 2, k, "f32", x64 @ R.values(codes, scales, k).T)


def test_extreme_scales(nz):
    """Scales at both ends that meet in the middle, for the product of two matrices and for floats."""
    n, m, k = 40, 33, 160
    rng = np.random.default_rng(6)
    for lo_a, lo_b in ((0, 250), (250, 0), (1, 200), (254, 1)):
        a, b = R.random_matrix(rng, m, k, lo_a, lo_a + 1), R.random_matrix(rng, n, k, lo_b, lo_b + 1)
        check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), mat(nz, *R.place(*b, k)), m, n, k, "f32", R.values(*a, k) @ R.values(*b, k).T)


@pytest.mark.parametrize("m", [1, 20, 40, 300])
def test_small_floats(nz, m):
    """Multiples of 2^-133 (floats without their leading bit) against large weights, 2^100 against the smallest weights, and results that
    are small: no product or sum is flushed.  Multiples of a power of two as in the exact cases.  Bits of float32 below 2^-133 are cut off."""
    n, k = 136, 264
    rng = np.random.default_rng(m)
    for e, s in ((-131, 240), (100, 0), (-60, 62), (-64, 62)):
        b = R.random_matrix(rng, n, k, s, s + 3)
        w = R.values(*b, k)
        bm = mat(nz, *R.place(*b, k))
        x, g = exact_floats(rng, m, k) * 2.0 ** e, exact_floats(rng, m, n) * 2.0 ** e
        for left in ("bf16", "f32"):
            low_x, low_g = (np.copysign(rng.integers(0, 2 ** 16, v.shape) * 2.0 ** -149, v) if left == "f32" and e == -131 else 0 for v in (x, g))
            check(nz, nz.MX4_LINEAR, floats(nz, x + low_x, left)[0], bm, m, n, k, "f32", x @ w.T)
            check(nz, nz.MX4_GRAD, floats(nz, g + low_g, left)[0], bm, m, n, k, "f32", g @ w)


def test_weights_past_the_range_of_float32(nz):
    n, k = 48, 64
    b = nz.Mx4.empty(n, k, "cuda:0")
    b.codes.fill_(0x66)                                                  # 4
    b.scales.fill_(254)                                                  # times 2^127
    import torch
    for m in (1, 20, 40):
        for left in ("bf16", "f16", "f32"):
            for call, kind, inner, outer in ((nz.nz_mx4_linear, nz.MX4_LINEAR, k, n), (nz.nz_mx4_grad, nz.MX4_GRAD, n, k)):
                x = torch.full((m, inner), 1.5, dtype=dtype(left), device="cuda:0")
                y = torch.zeros(m, outer, device="cuda:0")
                wsb = nz.nz_mx4_workspace_bytes(kind, x.dtype, m, n, k)
                ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda:0")
                assert call(x, inner, b, m, n, k, y, outer, ws, wsb) == 0
                assert not y.isfinite().any()


def test_grad_against_differences(nz):
    """C is linear in X, so a difference of C along any direction is the gradient's product with it, to the roundings of both."""
    import torch
    m, n, k = 21, 130, 300
    rng = np.random.default_rng(9)
    b = R.random_matrix(rng, n, k, 126, 129)
    bm = mat(nz, *R.place(*b, k))
    x, d, g = exact_floats(rng, m, k), exact_floats(rng, m, k), exact_floats(rng, m, n)
    ys = []
    for v in (x + d, x - d):
        y = torch.empty(m, n, device="cuda:0")
        t = floats(nz, v, "f32")[0]
        wsb = nz.nz_mx4_workspace_bytes(nz.MX4_LINEAR, t.dtype, m, n, k)
        assert nz.nz_mx4_linear(t, k, bm, m, n, k, y, n, torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda:0"), wsb) == 0
        ys.append(y.double().cpu().numpy())
    y = check(nz, nz.MX4_GRAD, floats(nz, g, "f32")[0], bm, m, n, k, "f32", g @ R.values(*b, k))
    at = 1 if k * 4 % 16 == 0 else 0
    grad = y[at:at + m, :k].double().cpu().numpy()
    assert ((ys[0] - ys[1]) / 2 * g).sum() == (grad * d).sum()


def test_gradient_of_both_sides_of_a_product(nz):
    """C = A B^T: the gradient for A, and for B from the transposed gradient with A in B's place."""
    m, n, k = 140, 96, 352
    rng = np.random.default_rng(10)
    a, b = R.random_matrix(rng, m, k, 126, 129), R.random_matrix(rng, n, k, 126, 129)
    g = exact_floats(rng, m, n)
    check(nz, nz.MX4_GRAD, floats(nz, g, "bf16")[0], mat(nz, *R.place(*b, k)), m, n, k, "f32", g @ R.values(*b, k))
    check(nz, nz.MX4_GRAD, floats(nz, g.T, "bf16")[0], mat(nz, *R.place(*a, k)), n, m, k, "f32", g.T @ R.values(*a, k))


def test_results_repeat_bit_for_bit(nz):
    import torch
    rng = np.random.default_rng(12)
    for m, n, k in ((1, 4096, 4096), (24, 512, 8192), (96, 640, 4096), (700, 520, 1100)):
        b = mat(nz, *R.place(*R.random_matrix(rng, n, k, 100, 150), k))
        a = mat(nz, *R.place(*R.random_matrix(rng, m, k, 100, 150), k))
        x, g = torch.randn(m, k, device="cuda:0").bfloat16(), torch.randn(m, n, device="cuda:0").bfloat16()
        seen = []
        for _ in range(3):
            ys = []
            for kind, left, outer in ((nz.MX4_PRODUCT, a, n), (nz.MX4_LINEAR, x, n), (nz.MX4_GRAD, g, k)):
                y = torch.empty(m, outer, device="cuda:0")
                wsb = nz.nz_mx4_workspace_bytes(kind, None if left is a else left.dtype, m, n, k)
                ws = torch.randint(0, 256, (max(wsb, 16),), dtype=torch.uint8, device="cuda:0")
                rc = (nz.nz_mx4_product(a, b, m, n, k, y, outer, ws, wsb) if left is a else
                      (nz.nz_mx4_linear if left is x else nz.nz_mx4_grad)(left, left.shape[1], b, m, n, k, y, outer, ws, wsb))
                assert rc == 0
                ys.append(y)
            seen.append(ys)
        for ys in seen[1:]:
            assert all(torch.equal(p, q) for p, q in zip(seen[0], ys))


def test_codes_past_32_bits(nz):
    """8.6 GB of codes: one token and a hundred against 2^18 rows of 2^16 columns; columns of the result at both ends are looked at."""
    import torch
    n, k = 1 << 18, 1 << 16
    codes = torch.randint(0, 256, (1024, k // 2), dtype=torch.uint8, device="cuda:0").repeat(n // 1024, 1)
    scales = torch.randint(126, 129, (1024, k // 32), dtype=torch.uint8, device="cuda:0").repeat(n // 1024, 1)
    codes[-1], scales[-1] = codes[5], scales[5]
    b = nz.Mx4(codes, scales)
    look = [0, 1, 1023, 131071, 131072, 131073, n - 2, n - 1]
    w = R.values(codes[look].cpu().numpy(), scales[look].cpu().numpy(), k)
    rng = np.random.default_rng(2)
    for m in (1, 100):
        x, x64 = floats(nz, rng.standard_normal((m, k)), "bf16")
        y = torch.empty(m, n, device="cuda:0")
        wsb = nz.nz_mx4_workspace_bytes(nz.MX4_LINEAR, x.dtype, m, n, k)
        ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda:0")
        assert nz.nz_mx4_linear(x, k, b, m, n, k, y, n, ws, wsb) == 0
        assert (np.abs(y[:, look].double().cpu().numpy() - x64 @ w.T) <= k * 2.0 ** -23 * (np.abs(x64) @ np.abs(w).T)).all()
        rows = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda:0")
        rows[:, n - 1] = 1
        y = torch.empty(m, k, device="cuda:0")
        wsb = nz.nz_mx4_workspace_bytes(nz.MX4_GRAD, rows.dtype, m, n, k)
        ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda:0")
        assert nz.nz_mx4_grad(rows, n, b, m, n, k, y, k, ws, wsb) == 0
        assert (y.cpu().numpy() == w[-1]).all()


def test_a_very_tall_left_side(nz):
    """More rows than one launch has threads for along x, where their floats are laid out anew (rows of two bytes): 69 GB of workspace."""
    import torch
    m = (1 << 29) + 5
    b = nz.Mx4.empty(1, 1, "cuda:0")
    b.codes.zero_()
    b.codes[0, 0] = 5                                                    # 3
    b.scales.fill_(128)                                                  # times 2
    x = (torch.arange(m, device="cuda:0", dtype=torch.int32) % 251 - 100).bfloat16()
    for call, kind in ((nz.nz_mx4_linear, nz.MX4_LINEAR), (nz.nz_mx4_grad, nz.MX4_GRAD)):
        wsb = nz.nz_mx4_workspace_bytes(kind, x.dtype, m, 1, 1)
        y, ws = torch.full((m + 8,), 9.0, dtype=torch.bfloat16, device="cuda:0"), torch.empty(wsb, dtype=torch.uint8, device="cuda:0")
        assert call(x, 1, b, m, 1, 1, y, 1, ws, wsb) == 0
        for at in range(0, m, 1 << 27):                                  # (6 times eight bits, rounded once)
            assert torch.equal(y[at:min(at + (1 << 27), m)], (x[at:at + (1 << 27)].float() * 6).bfloat16())
        assert (y[m:] == 9).all()
        del y, ws
    torch.cuda.empty_cache()


def test_a_sharded_training_step(nz):
    """As it is used: each of four ranks sends its weight shard in four bits, the gathered weights are multiplied as they landed, the gradient
    goes back through them, and the ranks' weight gradients are rounded without bias, summed into the shard's floats, and handed on."""
    import torch
    ranks, m, n, k = 4, 96, 256, 320
    rng = np.random.default_rng(13)
    weights = rng.standard_normal((n, k)) * 0.05
    gathered = nz.Mx4.empty(n, k)
    shard = n // ranks
    for r in range(ranks):
        w = floats(nz, weights[r * shard:(r + 1) * shard], "f32")[0]
        part = nz.Mx4(gathered.codes[r * shard:(r + 1) * shard], gathered.scales[r * shard:(r + 1) * shard])
        assert nz.nz_mx4_quantize(w, shard, k, k, nz.MX4_NEAREST, 0, part) == 0
    ref = R.place(*R.quantize(weights.astype(np.float32)), k)
    assert (gathered.codes.cpu().numpy()[:, :160] == ref[0][:, :160]).all()
    w64 = R.values(ref[0], ref[1], k)
    sent = []
    total = None
    for r in range(ranks):
        x, x64 = floats(nz, rng.standard_normal((m, k)), "bf16")
        y = check(nz, nz.MX4_LINEAR, x, gathered, m, n, k, "f32", x64 @ w64.T, exact=False, slack=k * 2.0 ** -23 * (np.abs(x64) @ np.abs(w64).T))
        g = y[1:m + 1, :n].bfloat16().contiguous()                       # (a loss of half the square: the gradient is C)
        g64 = g.double().cpu().numpy()
        check(nz, nz.MX4_GRAD, g, gathered, m, n, k, "bf16", g64 @ w64, exact=False, slack=n * 2.0 ** -23 * (np.abs(g64) @ np.abs(w64)))
        dw = g.float().t().contiguous() @ x.float()
        msg = nz.Mx4.empty(1, n * k)
        assert nz.nz_mx4_quantize(dw, 1, n * k, n * k, nz.MX4_STOCHASTIC, 100 + r, msg) == 0
        rc, rs = R.quantize(dw.reshape(1, -1).double().cpu().numpy(), True, 100 + r)
        assert (msg.codes.cpu().numpy() == rc).all() and (msg.scales.cpu().numpy() == rs).all()
        sent.append(msg)
        v = R.values(rc, rs, n * k)
        total = v.astype(np.float32) if total is None else total + v.astype(np.float32)
    mine = torch.empty(1, n * k, device="cuda:0")
    assert nz.nz_mx4_sum_k(sent, None, 0, 1, n * k, mine, n * k) == 0
    assert (mine.cpu().numpy() == total).all()
    out = nz.Mx4.empty(1, n * k)
    assert nz.nz_mx4_reduce_k(sent[1:], mine, n * k, 1, n * k, nz.MX4_NEAREST, 0, out) == 0


def test_products_in_a_graph(nz):
    """All three recorded on a stream of their own, with a workspace each, replayed between eager calls on new data."""
    import torch
    for m, n, k in ((1, 300, 520), (30, 520, 4096), (200, 260, 1100)):
        x, g = (torch.empty(m, c, dtype=torch.float16, device="cuda:0") for c in (k, n))
        a, b = nz.Mx4.empty(m, k), nz.Mx4.empty(n, k)
        w = torch.empty(n, k, device="cuda:0")
        wsb = [nz.nz_mx4_workspace_bytes(kind, x.dtype, m, n, k) for kind in range(3)]

        def step(ws, ys):
            assert nz.nz_mx4_quantize(w, n, k, k, 0, 0, b) == 0
            assert nz.nz_mx4_quantize(x, m, k, k, 0, 0, a) == 0
            assert nz.nz_mx4_product(a, b, m, n, k, ys[0], n, ws[0], wsb[0]) == 0
            assert nz.nz_mx4_linear(x, k, b, m, n, k, ys[1], n, ws[1], wsb[1]) == 0
            assert nz.nz_mx4_grad(g, n, b, m, n, k, ys[2], k, ws[2], wsb[2]) == 0

        def buffers():
            return ([torch.empty(max(v, 16), dtype=torch.uint8, device="cuda:0") for v in wsb],
                    [torch.zeros(m, c, device="cuda:0") for c in (n, n, k)])

        gw, gy = buffers()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(gw, gy)
        for seed in range(3):
            gen = torch.Generator().manual_seed(seed)
            for t in (x, g, w):
                t.copy_(torch.randn(t.shape, generator=gen))
            graph.replay()
            torch.cuda.synchronize()
            got = [y.clone() for y in gy]
            ew, ey = buffers()
            step(ew, ey)
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) and p.abs().sum() > 0 for p, q in zip(got, ey))


@pytest.mark.parametrize("m", [1, 20, 40])
@pytest.mark.parametrize("s,code,value", [(253, 5, 3.0), (253, 6, 4.0), (253, 7, 6.0), (254, 3, 1.5), (254, 4, 2.0), (254, 5, 3.0), (254, 7, 6.0)])
def test_the_border_of_float32s_range(nz, s, code, value, m):
    """The last weights that float32 holds and the first that it does not: 2^128 is the border.  One element of each row of the left is
    2^-20, the rest 0, so that what is finite is exact."""
    import torch
    n, k = 48, 96
    codes, scales = np.full((n, k // 2), code * 17, np.uint8), np.full((n, k // 32), s, np.uint8)
    weight = value * 2.0 ** (s - 127)
    finite = weight < 2.0 ** 128
    bm = mat(nz, *R.place(codes, scales, k))
    y = torch.zeros(n, k, device="cuda:0")
    assert nz.nz_mx4_dequantize(bm, n, k, y, k) == 0
    assert (y == (weight if finite else float("inf"))).all()
    a = np.zeros((m, k // 2), np.uint8), np.full((m, k // 32), 107, np.uint8)        # 2^-20
    a[0][:, 3] = 2
    check(nz, nz.MX4_PRODUCT, mat(nz, *R.place(*a, k)), bm, m, n, k, "f32", np.full((m, n), weight * 2.0 ** -20))
    for left in ("bf16", "f16", "f32"):
        for kind, call, inner, outer in ((nz.MX4_LINEAR, nz.nz_mx4_linear, k, n), (nz.MX4_GRAD, nz.nz_mx4_grad, n, k)):
            x = np.zeros((m, inner))
            x[:, 5] = 2.0 ** -20
            t = floats(nz, x, left)[0]
            if finite:
                check(nz, kind, t, bm, m, n, k, "f32", np.full((m, outer), weight * 2.0 ** -20))
            else:
                c = torch.zeros(m, outer, device="cuda:0")
                wsb = nz.nz_mx4_workspace_bytes(kind, t.dtype, m, n, k)
                ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda:0")
                assert call(t, inner, bm, m, n, k, c, outer, ws, wsb) == 0
                assert not c.isfinite().any()


def test_the_sum_that_a_rank_hands_on(nz):
    """The last hop of the sharded step: three peers' gradients, rounded without bias, and the rank's own float32 sum, last, go on in four bits."""
    import torch
    rng = np.random.default_rng(14)
    n = 256 * 320
    sent, values = [], []
    for r in range(3):
        g = floats(nz, rng.standard_normal((1, n)) * 0.01, "f32")[0]
        msg = nz.Mx4.empty(1, n)
        assert nz.nz_mx4_quantize(g, 1, n, n, nz.MX4_STOCHASTIC, 100 + r, msg) == 0
        sent.append(msg)
        values.append(R.values(msg.codes.cpu().numpy(), msg.scales.cpu().numpy(), n).astype(np.float32))
    mine, mine64 = floats(nz, rng.standard_normal((1, n)) * 0.02, "f32")
    total = values[0]
    for v in values[1:] + [mine64.astype(np.float32)]:
        total = total + v
    for rounding in (nz.MX4_NEAREST, nz.MX4_STOCHASTIC):
        out = nz.Mx4(torch.full_like(sent[0].codes, 0xA5), torch.full_like(sent[0].scales, 0xA5))
        assert nz.nz_mx4_reduce_k(sent, mine, n, 1, n, rounding, 9, out) == 0
        rc, rs = R.quantize(total.astype(np.float64), bool(rounding), 9)
        assert (out.codes.cpu().numpy() == rc).all() and (out.scales.cpu().numpy() == rs).all()
