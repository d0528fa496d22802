"""Microscaled 4-bit operators without a GPU: worked values of the tests' own reference, sizing, and every refusal of the C entry points (which
return before anything is launched)."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

import mx4_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def nz():
    from paper_2605_12396_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_12396_amd import build
        build.build()
    binding.lib()
    return binding


def _codes(x, **kw):
    codes, scales = R.quantize(np.array([x], np.float32), **kw)
    b = codes[0]
    return [int(v) for v in np.stack([b & 15, b >> 4], 1).reshape(-1)[:len(x)]], [int(s) for s in scales[0]]


def test_reference_worked_values():
    # peak 6: scale 2^(2 - 2) = 1; ties 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    assert _codes([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, -0.0]) == ([7, 0, 2, 2, 4, 4, 6, 6, 14, 8], [127])
    assert _codes([7.9, 0, 1]) == ([7, 0, 2], [127])                    # above the largest code: held at it
    assert _codes([8, 0, 1]) == ([6, 0, 1], [128])
    assert _codes([0, 0]) == ([0, 0], [0])
    assert _codes([1, float("nan")]) == ([0, 0], [255]) and _codes([1, float("-inf")]) == ([0, 0], [255])
    assert _codes([2.0 ** -140]) == ([0], [0]) and _codes([2.0 ** -128]) == ([1], [0])
    # stochastic: 7.9 > 6, so the scale is 2 and 3.95 lies between 3 (code 5) and 4 (code 6)
    seen = {tuple(_codes([7.9, 2, 1], stochastic=True, seed=s)[0]) for s in range(40)}
    assert seen == {(5, 2, 1), (6, 2, 1)} and _codes([7.9], stochastic=True)[1] == [128]
    assert _codes([6, 3], stochastic=True, seed=5) == ([7, 5], [127])
    assert list(R.values(np.array([[0x21, 0xF9] + [0] * 14], np.uint8), np.array([[128]], np.uint8), 4)[0]) == [1, 2, -1, -12]


def test_reference_draws_without_bias():
    """0.3 of the way from 2 to 3: over N draws the mean is within 4 sigma (sqrt(0.21 / N)) plus 2^-17 of 2.3."""
    n = 200000
    codes, scales = R.quantize(np.concatenate([np.full((1, n), 2.3), np.full((1, 32), 6.0)], 1).astype(np.float64), True, 11)
    v = R.values(codes, scales, n)[0]
    v = v.reshape(-1, 32)
    peak2 = v[v.max(1) <= 3]                            # blocks of 2.3 alone have scale 1/2
    assert set(np.unique(peak2)) == {2.0, 3.0} or set(np.unique(peak2)) == {2.0, 2.5, 3.0}
    step = 1.0 if 2.5 not in peak2 else 0.5
    p = (2.3 - 2.0) / step
    assert abs(peak2.mean() - 2.3) <= step * (4 * np.sqrt(p * (1 - p) / peak2.size) + 2.0 ** -17)


def test_header_is_c99_and_exports_exist(nz, tmp_path):
    inc = os.path.join(ROOT, "include")
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(inc, "nz_mx4.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(nz_mx4_\w+)\s*\(", hdr))
    assert names == {"nz_mx4_pitch", "nz_mx4_quantize", "nz_mx4_dequantize", "nz_mx4_reduce_k", "nz_mx4_sum_k", "nz_mx4_workspace_bytes",
                     "nz_mx4_product", "nz_mx4_linear", "nz_mx4_grad"}
    for n in names:
        assert hasattr(nz.lib(), n), n
    src = tmp_path / "h.c"
    src.write_text('#include "nz_mx4.h"\n#include <stdio.h>\nint main(void) { printf("%zu %d %d %d", sizeof(nz_mx4_matrix), NZ_F16, '
                   'NZ_MX4_STOCHASTIC, NZ_MX4_GRAD); return 0; }\n')
    exe = tmp_path / "h"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", inc, "-o", str(exe), str(src)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    assert out == "%d %d %d %d" % (C.sizeof(nz.Mx4Matrix), nz.F16, nz.MX4_STOCHASTIC, nz.MX4_GRAD)


def test_sizes(nz):
    for cols in (0, 1, 31, 32, 33, 127, 128, 129, 4096, 1 << 40):
        assert nz.nz_mx4_pitch(cols) == (R.pitch(cols) if cols else 0)
    import torch
    for kind, left in ((nz.MX4_PRODUCT, None), (nz.MX4_LINEAR, torch.bfloat16), (nz.MX4_GRAD, torch.float32)):
        assert nz.nz_mx4_workspace_bytes(kind, left, 1, 1, 1) >= 0
        for m, n, k in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 30, 1, 1), (1, 1 << 30, 1), (1, 1, 1 << 30), (1 << 20, 1 << 20, 1)):
            with pytest.raises(ValueError):
                nz.nz_mx4_workspace_bytes(kind, left, m, n, k)
    with pytest.raises(ValueError):
        nz.nz_mx4_workspace_bytes(3, torch.float32, 1, 1, 1)
    with pytest.raises(ValueError):
        nz.nz_mx4_workspace_bytes(nz.MX4_LINEAR, torch.float64, 1, 1, 1)


# Addresses that are never read: every call below is refused on the host.
P, Q, S = 1 << 20, 1 << 21, 1 << 22


def _mat(nz, codes=Q, scales=S, pitch=4):
    return C.byref(nz.Mx4Matrix(codes, scales, pitch))


def _bad_mats(nz, pitch):
    return [None, _mat(nz, codes=None, pitch=pitch), _mat(nz, scales=None, pitch=pitch), _mat(nz, codes=Q + 8, pitch=pitch),
            _mat(nz, scales=S + 1, pitch=pitch), _mat(nz, pitch=pitch - 4), _mat(nz, pitch=pitch + 2)]


def test_conversions_refuse(nz):
    L, bad = nz.lib(), []
    good = dict(d=P, t=0, rows=3, cols=200, ld=200, rnd=0, m=_mat(nz, pitch=8))
    for kw in ([dict(d=None), dict(d=P + 4), dict(t=3), dict(t=-1), dict(rows=0), dict(cols=0), dict(ld=199), dict(rows=1 << 31),
                dict(cols=1 << 31, ld=1 << 31, m=_mat(nz, pitch=1 << 26)), dict(rows=1 << 30, cols=256, ld=256)]
               + [dict(m=m) for m in _bad_mats(nz, 8)]):
        a = dict(good, **kw)
        bad.append(L.nz_mx4_quantize(a["d"], a["t"], a["rows"], a["cols"], a["ld"], a["rnd"], 0, a["m"], None))
        bad.append(L.nz_mx4_dequantize(a["m"], a["rows"], a["cols"], a["d"], a["t"], a["ld"], None))
        bad.append(L.nz_mx4_sum_k(a["m"], 1, None, 0, a["rows"], a["cols"], a["d"], a["t"], a["ld"], None))
    for rnd in (-1, 2):
        bad.append(L.nz_mx4_quantize(P, 0, 3, 200, 200, rnd, 0, good["m"], None))
        bad.append(L.nz_mx4_reduce_k(good["m"], 1, None, 0, 3, 200, rnd, 0, good["m"], None))
    for k in (0, 65):
        bad.append(L.nz_mx4_reduce_k(good["m"], k, None, 0, 3, 200, 0, 0, good["m"], None))
        bad.append(L.nz_mx4_sum_k(good["m"], k, None, 0, 3, 200, P, 0, 200, None))
    for m in _bad_mats(nz, 8):
        bad.append(L.nz_mx4_reduce_k(good["m"], 1, None, 0, 3, 200, 0, 0, m, None))
        bad.append(L.nz_mx4_reduce_k(m, 1, None, 0, 3, 200, 0, 0, good["m"], None))
    for local, ld in ((P + 4, 200), (P, 199)):
        bad.append(L.nz_mx4_reduce_k(good["m"], 1, local, ld, 3, 200, 0, 0, good["m"], None))
        bad.append(L.nz_mx4_sum_k(good["m"], 1, local, ld, 3, 200, P, 0, 200, None))
    two = (nz.Mx4Matrix * 2)(nz.Mx4Matrix(Q, S, 8), nz.Mx4Matrix(Q, S, 4))
    bad.append(L.nz_mx4_reduce_k(two, 2, None, 0, 3, 200, 0, 0, good["m"], None))
    assert set(bad) == {nz.ERR_INVALID}


def test_products_refuse(nz):
    L, bad = nz.lib(), []
    W, big = 1 << 23, 1 << 40

    def call(a=None, b=None, x=P, xt=1, ldx=None, m=5, n=40, k=200, c=P, ct=0, ldc=None, ws=W, wsb=big, only=None):
        p = 8 if k == 200 else nz.nz_mx4_pitch(k)
        a, b = a if a is not None else _mat(nz, pitch=p), b if b is not None else _mat(nz, pitch=p)
        a, b = None if a == "null" else a, None if b == "null" else b
        if only in (None, 0):
            bad.append(L.nz_mx4_product(a, b, m, n, k, c, ct, n if ldc is None else ldc, ws, wsb, None))
        if only in (None, 1):
            bad.append(L.nz_mx4_linear(x, xt, k if ldx is None else ldx, b, m, n, k, c, ct, n if ldc is None else ldc, ws, wsb, None))
        if only in (None, 2):
            bad.append(L.nz_mx4_grad(x, xt, n if ldx is None else ldx, b, m, n, k, c, ct, k if ldc is None else ldc, ws, wsb, None))

    for kw in (dict(m=0), dict(n=0), dict(k=0), dict(m=1 << 30), dict(n=1 << 30, ldc=1 << 30), dict(k=1 << 30), dict(c=None), dict(c=P + 2),
               dict(ct=3), dict(ct=-1), dict(ldc=39)):
        call(**kw)
    for b in _bad_mats(nz, 8):
        call(b=b if b is not None else "null")
        call(a=b if b is not None else "null", only=0)
    for kw in (dict(x=None), dict(x=P + 4), dict(xt=5), dict(ldx=39)):
        call(only=1, **kw)
        call(only=2, **kw)
    call(k=1 << 24)                                      # a row of codes past 4 MiB
    call(ldx=1 << 22, only=1)                            # a row of floats past 4 MiB
    call(ldc=1 << 21)
    for kind, only in ((nz.MX4_PRODUCT, 0), (nz.MX4_LINEAR, 1), (nz.MX4_GRAD, 2)):
        need = L.nz_mx4_workspace_bytes(kind, 1, 5, 40, 200)
        if need:
            for kw in (dict(ws=None), dict(ws=W + 8), dict(wsb=need - 1)):
                call(only=only, **kw)
    assert set(bad) == {nz.ERR_INVALID}


def test_binding_refuses_host_tensors(nz):
    import torch
    x = torch.zeros(64)
    m = nz.Mx4(torch.zeros(1, 64, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.uint8))
    assert nz.nz_mx4_quantize(x, 1, 64, 64, 0, 0, m) == nz.ERR_INVALID
    assert nz.nz_mx4_dequantize(m, 1, 64, x, 64) == nz.ERR_INVALID
    assert nz.nz_mx4_reduce_k([m], None, 0, 1, 64, 0, 0, m) == nz.ERR_INVALID
    assert nz.nz_mx4_sum_k([m], x, 64, 1, 64, x, 64) == nz.ERR_INVALID
    assert nz.nz_mx4_product(m, m, 1, 1, 64, x, 1) == nz.ERR_INVALID
    assert nz.nz_mx4_linear(x, 64, m, 1, 1, 64, x, 1) == nz.ERR_INVALID
    assert nz.nz_mx4_grad(x, 1, m, 1, 1, 64, x, 64) == nz.ERR_INVALID
    assert nz.nz_mx4_product(m, m, 2, 1, 64, x, 1) == nz.ERR_INVALID                # more rows than the matrix has
    for codes, scales in ((torch.zeros(1, 63, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.uint8)),
                          (torch.zeros(2, 64, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.uint8)),
                          (torch.zeros(1, 64), torch.zeros(1, 4, dtype=torch.uint8)),
                          (torch.zeros(64, 4, dtype=torch.uint8).t(), torch.zeros(4, 4, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            nz.Mx4(codes, scales)


def test_a_length_is_not_parted_more_than_it_can_be(nz):
    """Floats on the left: their terms of bfloat16, in rows of whole steps of 64 elements, and float32 sums for every part of the length.  A part
    is made of pairs of such steps, so that there are no more sums than pairs (a workgroup without steps would write sums of zeros)."""
    import torch
    rng = np.random.default_rng(0)
    for left, terms in ((torch.bfloat16, 1), (torch.float16, 2), (torch.float32, 3)):
        for m, n, k in [(58, 1674, 226), (40, 128, 65), (33, 64, 64)] + [tuple(int(v) for v in np.exp(rng.uniform(np.log(33), np.log(4096), 3))) for _ in range(500)]:
            chunks = -(-k // 64)
            pairs = -(-chunks // 2)
            most = chunks * 128 * terms * m + (pairs * m * -(-n // 4) * 4 * 4 if pairs > 1 else 0)
            assert nz.nz_mx4_workspace_bytes(nz.MX4_LINEAR, left, m, n, k) <= most, (left, m, n, k)


def test_products_refuse_a_single_row_that_is_too_long(nz):
    """The row length of a matrix of one row is held to the same limit, and its bytes do not pass 64 bits unseen."""
    L, W = nz.lib(), 1 << 23
    for pitch in ((1 << 18) + 4, 1 << 60, (1 << 60) + 8, (1 << 64) - 4):
        long_, short = _mat(nz, pitch=pitch), _mat(nz, pitch=8)
        assert L.nz_mx4_product(long_, short, 1, 40, 200, P, 0, 40, W, 1 << 40, None) == nz.ERR_INVALID, pitch
        assert L.nz_mx4_product(short, long_, 5, 1, 200, P, 0, 1, W, 1 << 40, None) == nz.ERR_INVALID, pitch
        assert L.nz_mx4_linear(P, 1, 200, long_, 5, 1, 200, P, 0, 1, W, 1 << 40, None) == nz.ERR_INVALID, pitch
        assert L.nz_mx4_grad(P, 1, 1, long_, 5, 1, 200, P, 0, 200, W, 1 << 40, None) == nz.ERR_INVALID, pitch


def test_products_refuse_matrices_of_2_to_the_38_elements(nz):
    """The limit of a matrix holds for those of the products as well (sides and rows within theirs)."""
    import torch
    L, W = nz.lib(), 1 << 23
    n, k = 1 << 18, 1 << 20                                # rows of 512 KB of codes
    wide = _mat(nz, pitch=k // 32)
    assert L.nz_mx4_product(wide, wide, 5, n, k, P, 0, n, W, 1 << 50, None) == nz.ERR_INVALID
    assert L.nz_mx4_product(wide, wide, n, 5, k, P, 0, 5, W, 1 << 50, None) == nz.ERR_INVALID
    assert L.nz_mx4_linear(P, 1, k, wide, 5, n, k, P, 0, n, W, 1 << 50, None) == nz.ERR_INVALID
    assert L.nz_mx4_grad(P, 1, n, wide, 5, n, k, P, 0, k, W, 1 << 50, None) == nz.ERR_INVALID
    for kind, left in ((nz.MX4_PRODUCT, None), (nz.MX4_LINEAR, torch.bfloat16), (nz.MX4_GRAD, torch.bfloat16)):
        with pytest.raises(ValueError):
            nz.nz_mx4_workspace_bytes(kind, left, 5, n, k)
        assert nz.nz_mx4_workspace_bytes(kind, left, 5, n - 1, k) >= 0
    with pytest.raises(ValueError):
        nz.nz_mx4_workspace_bytes(nz.MX4_PRODUCT, None, n, 5, k)
    assert nz.nz_mx4_workspace_bytes(nz.MX4_LINEAR, torch.bfloat16, n, 5, k) >= 0        # (floats: below 2^40)
