"""Microscaled 4-bit conversions and sums on the GPU against the plain float64 implementation: every byte equal."""
import numpy as np
import pytest

import mx4_reference as R

pytestmark = pytest.mark.gpu

NP = {"f32": np.float32, "f16": np.float16}


@pytest.fixture(scope="module")
def nz(gpu_device):
    from paper_2605_12396_amd import binding
    binding.lib()
    return binding


def dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def mat(nz, codes, scales):
    return nz.Mx4(dev(codes), dev(scales))


def floats(nz, x, name, ld=None, fill=float("nan")):
    """A device tensor [rows, ld] of the type, x in its first columns, `fill` behind; and what x became, in float64."""
    import torch
    x = np.atleast_2d(x)
    t = torch.full((x.shape[0], ld or x.shape[1]), fill, dtype=torch.float32)
    t[:, :x.shape[1]] = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    t = t.to(dtype(name)).to("cuda:0")
    return t, t[:, :x.shape[1]].double().cpu().numpy()


def check_quantize(nz, x, name="f32", stochastic=False, seed=0, ld=None, extra=0):
    d, x64 = floats(nz, x, name, ld)
    rows, cols = x64.shape
    ref_c, ref_s = R.quantize(x64, stochastic, seed)
    want_c, want_s = R.place(ref_c, ref_s, cols, extra, 0xA5)
    m = mat(nz, np.full_like(want_c, 0xA5), np.full_like(want_s, 0xA5))
    assert nz.nz_mx4_quantize(d, rows, cols, d.shape[1], int(stochastic), seed, m) == 0
    got_c, got_s = m.codes.cpu().numpy(), m.scales.cpu().numpy()
    assert (got_s == want_s).all(), np.argwhere(got_s != want_s)[:4]
    assert (got_c == want_c).all(), (np.argwhere(got_c != want_c)[:4], got_c[got_c != want_c][:4], want_c[got_c != want_c][:4])


def spread(rng, rows, cols):
    """Values over many octaves, block by block."""
    return rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-12, 12, (rows, 1)) * np.where(rng.random((rows, cols)) < 0.02, 30, 1)


SHAPES = [(1, 1, None, 0), (1, 31, None, 0), (1, 32, None, 0), (1, 33, None, 4), (1, 16384, None, 0), (1, 300007, None, 0), (3, 129, 131, 0),
          (5, 4095, None, 0), (7, 128, None, 0), (64, 256, None, 0), (64, 256, 264, 0), (64, 256, None, 4), (700, 40, 41, 8), (257, 1000, 1000, 0),
          (2, 8, 8, 0), (4097, 33, None, 0)]


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_quantize(nz, shape, name, stochastic):
    rows, cols, ld, extra = shape
    rng = np.random.default_rng(rows * 7919 + cols)
    check_quantize(nz, spread(rng, rows, cols), name, stochastic, 1234567 + cols, ld, extra)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_quantize_borders(nz, name, stochastic):
    """Every tie and its neighbours at many scales, the smallest and largest floats, zeros, infinities and NaN, alone in a block or not."""
    one = np.float32(1)
    ties = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7, 7.75], np.float32)
    near = np.concatenate([ties, np.nextafter(ties, 8 * one), np.nextafter(ties, -one)])
    rows = []
    scales = [2.0 ** e for e in ((-149, -140, -130, -127, -126, -100, -14, -1, 0, 1, 12, 100, 124, 125) if name != "f16" else (-24, -20, -14, -3, 0, 1, 12))]
    for s in scales:
        for sign in (1, -1):
            v = np.zeros(64, np.float64)
            v[:near.size] = near.astype(np.float64) * s * sign
            v[31] = v[63] = 4 * s                                  # the scale that makes the ties ties
            rows.append(v)
    special = [0.0, -0.0, 1e-45, -1e-40, 3.4e38, -3.4e38, float("inf"), -float("inf"), float("nan")]
    for a in special:
        for b in (0.0, 1.0, 1e-30):
            v = np.full(64, b)
            v[5], v[40] = a, a
            rows.append(v)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    check_quantize(nz, x, name, stochastic, 99)


def test_stochastic_share_to_the_last_bit(nz):
    """Shares that equal a draw's border, and the floats on either side of it, in both ranges of spacing."""
    n = 4096
    u = R.draws(0, n, 21).astype(np.float64)
    border = (u + 0.5) / 65536
    for base, gap in ((0.0, 0.5), (0.5, 0.5), (1.0, 0.5), (2.0, 1.0), (4.0, 2.0)):
        x = (base + gap * border).astype(np.float32)
        for y in (x, np.nextafter(x, np.float32(8)), np.nextafter(x, np.float32(-1))):
            y = y.reshape(-1, 32).copy()
            y[:, 0] = 6.0
            check_quantize(nz, y.reshape(1, -1), "f32", True, 21)


def test_draws_change_with_the_seed_and_not_with_the_layout(nz):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 256)).astype(np.float32)
    d, _ = floats(nz, x, "f32")
    a, b, c = (nz.Mx4.empty(6, 256) for _ in range(3))
    wide = nz.Mx4(dev(np.zeros((6, 12 * 16), np.uint8)), dev(np.zeros((6, 12), np.uint8)))
    for m, seed in ((a, 5), (b, 5), (c, 6), (wide, 5)):
        assert nz.nz_mx4_quantize(d, 6, 256, 256, nz.MX4_STOCHASTIC, seed, m) == 0
    assert (a.codes == b.codes).all() and not (a.codes == c.codes).all()
    assert (a.codes == wide.codes[:, :128]).all() and (a.scales == wide.scales[:, :8]).all()


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_dequantize_every_code_under_every_scale(nz, name):
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(1, 16, 16), (256, 1, 1)).reshape(256, 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    for cols, ld in ((512, 512), (511, 513), (509, 520)):
        y = torch.full((256, ld), 77.0, dtype=dtype(name), device="cuda:0")
        assert nz.nz_mx4_dequantize(mat(nz, codes, scales), 256, cols, y, ld) == 0
        want = torch.from_numpy(R.values(codes, scales, cols)).to(dtype(name))
        assert torch.equal(y[:, :cols].cpu().nan_to_num(nan=-1.0), want.nan_to_num(nan=-1.0))
        assert torch.equal(y[:, :cols].cpu().isnan(), want.isnan())
        assert (y[:, cols:] == 77).all()


def sum64(parts, local):
    """The fold in float32 (numpy), as float64."""
    with np.errstate(all="ignore"):
        acc = parts[0].astype(np.float32)
        for p in parts[1:]:
            acc = acc + p.astype(np.float32)
        return (acc + local.astype(np.float32) if local is not None else acc).astype(np.float64)


@pytest.mark.parametrize("k", [1, 2, 3, 7, 8, 9, 16, 64])
@pytest.mark.parametrize("shape", [(1, 5000, 0, None), (3, 257, 4, 259), (33, 256, 0, None), (1, 1, 0, None), (40, 96, 0, 96)], ids=str)
def test_sums(nz, shape, k):
    import torch
    rows, cols, extra, ld_local = shape
    rng = np.random.default_rng(k * 100 + cols)
    raw = [R.random_matrix(rng, rows, cols, 110, 140) for _ in range(k)]
    parts = [R.values(c, s, cols) for c, s in raw]
    ms = [mat(nz, *R.place(c, s, cols, extra if i % 2 else 0)) for i, (c, s) in enumerate(raw)]
    local = rng.standard_normal((rows, cols)).astype(np.float32) * 100
    for own in (None, local):
        ld = cols if own is None else (ld_local or cols)
        d = None if own is None else floats(nz, own, "f32", ld)[0]
        want = sum64(parts, own)
        for name in ("f32", "bf16", "f16"):
            y = torch.full((rows, cols + 3), 5.0, dtype=dtype(name), device="cuda:0")
            assert nz.nz_mx4_sum_k(ms, d, ld, rows, cols, y, cols + 3) == 0
            assert torch.equal(y[:, :cols].cpu(), torch.from_numpy(want).float().to(dtype(name))) and (y[:, cols:] == 5).all()
        for stochastic in (0, 1):
            wc, ws = R.place(*R.quantize(want, bool(stochastic), 4321), cols, extra, 0x5A)
            out = mat(nz, np.full_like(wc, 0x5A), np.full_like(ws, 0x5A))
            assert nz.nz_mx4_reduce_k(ms, d, ld, rows, cols, stochastic, 4321, out) == 0
            assert (out.scales.cpu().numpy() == ws).all() and (out.codes.cpu().numpy() == wc).all()


def test_sum_of_many_orders_its_roundings(nz):
    """Operands of very different size: the float32 fold is not the exact sum, and it is the fold in the order given."""
    import torch
    rng = np.random.default_rng(8)
    raw = [R.random_matrix(rng, 4, 320, lo, lo + 3) for lo in (150, 110, 120, 100, 149)]
    parts = [R.values(c, s, 320) for c, s in raw]
    want = sum64(parts, None)
    assert (want != sum(parts)).any() and (want != sum64(parts[::-1], None)).any()
    y = torch.empty(4, 320, device="cuda:0")
    assert nz.nz_mx4_sum_k([mat(nz, *R.place(c, s, 320)) for c, s in raw], None, 0, 4, 320, y, 320) == 0
    assert (y.cpu().numpy() == want).all()


def test_sums_pass_nan_infinity_and_overflow_on(nz):
    import torch
    c, s = R.random_matrix(np.random.default_rng(1), 3, 96, 126, 129)
    c[:] = 0x77                                                   # 6 everywhere
    s1, s2 = s.copy(), s.copy()
    s1[0, 1] = 255                                                # NaN block
    s1[1, 0] = s2[1, 0] = 254                                     # 6 * 2^127 is infinite as float32, and so is the sum
    want = sum64([R.values(c, s1, 96), R.values(c, s2, 96)], None)
    ms = [mat(nz, *R.place(c, t, 96)) for t in (s1, s2)]
    y = torch.empty(3, 96, device="cuda:0")
    assert nz.nz_mx4_sum_k(ms, None, 0, 3, 96, y, 96) == 0
    assert np.array_equal(y.cpu().numpy().astype(np.float64), want, equal_nan=True) and np.isinf(want).any() and np.isnan(want).any()
    out = nz.Mx4.empty(3, 96)
    assert nz.nz_mx4_reduce_k(ms, None, 0, 3, 96, 0, 0, out) == 0
    got = out.scales.cpu().numpy()
    assert got[0, 1] == 255 and got[1, 0] == 255 and (out.codes.cpu().numpy()[0, 16:32] == 0).all() and (got[2, :3] != 255).all()


def test_reduce_onto_an_operand(nz):
    rng = np.random.default_rng(5)
    for rows, cols in ((1, 70001), (50, 200)):
        raw = [R.random_matrix(rng, rows, cols) for _ in range(3)]
        want = R.place(*R.quantize(sum64([R.values(c, s, cols) for c, s in raw], None)), cols)
        for i in range(3):
            ms = [mat(nz, *R.place(c, s, cols)) for c, s in raw]
            assert nz.nz_mx4_reduce_k(ms, None, 0, rows, cols, 0, 0, ms[i]) == 0
            assert (ms[i].codes.cpu().numpy() == want[0]).all() and (ms[i].scales.cpu().numpy() == want[1]).all()


def test_capture_and_streams(nz):
    """Conversions and sums recorded into a graph on a stream of their own, replayed between eager calls on new data."""
    import torch
    rows, cols = 37, 515
    x = torch.empty(rows, cols, device="cuda:0")
    a, b, o = (nz.Mx4.empty(rows, cols) for _ in range(3))
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0")

    def step(stream, y):
        assert nz.nz_mx4_quantize(x, rows, cols, cols, 1, 3, a, stream) == 0
        assert nz.nz_mx4_quantize(x, rows, cols, cols, 0, 0, b, stream) == 0
        assert nz.nz_mx4_reduce_k([a, b], x, cols, rows, cols, 1, 4, o, stream) == 0
        assert nz.nz_mx4_dequantize(o, rows, cols, y, cols, stream) == 0

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step(None, y)
    for seed in range(4):
        x.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        eager = torch.empty_like(y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        step(side, eager)
        side.synchronize()
        assert torch.equal(got, eager) and got.abs().sum() > 0


@pytest.mark.parametrize("name", ["f32", "f16"])
def test_large_floats_equal_small_ones(nz, name):
    """Floats of more than 128 MB take another way to memory; the same rows, one call each, do not."""
    import torch
    rows, cols, ld = 3, 23000001 if name == "f16" else 12000001, 23000008
    pitch = 718752                                                       # (rows of scales, and of floats, at multiples of 16 bytes)
    m = nz.Mx4(torch.randint(0, 256, (rows, 16 * pitch), dtype=torch.uint8, device="cuda:0"),
               torch.randint(110, 140, (rows, pitch), dtype=torch.uint8, device="cuda:0"))
    whole, single = (torch.full((rows, ld), 3.0, dtype=dtype(name), device="cuda:0") for _ in range(2))
    assert nz.nz_mx4_sum_k([m, m], None, 0, rows, cols, whole, ld) == 0
    for r in range(rows):
        one = nz.Mx4(m.codes[r:r + 1], m.scales[r:r + 1])
        assert nz.nz_mx4_sum_k([one, one], None, 0, 1, cols, single[r], ld) == 0
    assert torch.equal(whole, single) and (whole[:, cols:] == 3).all() and whole[:, :cols].abs().max() > 4


def test_offsets_past_32_bits(nz):
    """9.2e9 elements: 18 GB of bf16 and 4.9 GB of codes, whole rows and ragged ones; rows at both ends and around 2^32 bytes are looked at."""
    import torch
    rows, cols = 70001, 131072
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    base = torch.randn(1001, cols, device="cuda:0").to(torch.bfloat16)
    for r in range(0, rows, 1001):
        x[r:r + 1001] = base[:min(1001, rows - r)]
    look = [0, 1, 4095, 32767, 32768, 65535, 65536, 70000]
    for c in (cols, cols - 5):
        m = nz.Mx4.empty(rows, c)
        assert nz.nz_mx4_quantize(x, rows, c, cols, 1, 17, m) == 0
        codes, scales = (t[look].cpu().numpy() for t in (m.codes, m.scales))
        for i, r in enumerate(look):
            rc, rs = R.quantize(x[r:r + 1, :c].double().cpu().numpy(), True, 17, first=r * R.blocks(c) * 32)
            assert (scales[i, :rs.shape[1]] == rs[0]).all() and (codes[i, :rc.shape[1]] == rc[0]).all(), (c, r)
        y = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0")
        assert nz.nz_mx4_dequantize(m, rows, c, y, cols) == 0
        for i, r in enumerate(look):
            want = torch.from_numpy(R.values(codes[i:i + 1], scales[i:i + 1], c)).to(torch.bfloat16)
            assert torch.equal(y[r:r + 1, :c].cpu(), want), (c, r)
        del m, y


def test_more_rows_than_one_layer_of_the_grid(nz):
    """Rows are laid over the grid in groups of fewer than 2^29 blocks; past that a second group starts, whose draws, rows and shorter end are its
    own.  2^29 + 5 rows of one block: rows on either side of the border, and at both ends."""
    import torch
    rows, cols = (1 << 29) + 5, 2
    base = torch.randn(1 << 20, cols, device="cuda:0").bfloat16()
    x = base.repeat(-(-rows // base.shape[0]), 1)[:rows]
    m = nz.Mx4(torch.empty(rows, 64, dtype=torch.uint8, device="cuda:0"), torch.empty(rows, 4, dtype=torch.uint8, device="cuda:0"))
    y = torch.full((rows + 3, cols), 9.0, dtype=torch.bfloat16, device="cuda:0")
    border = (1 << 29) - 1                                               # rows of the first group
    parts = [(0, 3), (border - 3, border), (border, border + 3), (rows - 3, rows)]
    for stochastic in (0, 1):
        m.codes.fill_(0xA5)
        m.scales.fill_(0xA5)
        assert nz.nz_mx4_quantize(x, rows, cols, cols, stochastic, 23, m) == 0
        assert nz.nz_mx4_dequantize(m, rows, cols, y, cols) == 0
        for a, b in parts:
            rc, rs = R.quantize(x[a:b].double().cpu().numpy(), bool(stochastic), 23, first=a * 32)
            want_c, want_s = R.place(rc, rs, cols, 0, 0xA5)
            assert (m.codes[a:b].cpu().numpy() == want_c).all() and (m.scales[a:b].cpu().numpy() == want_s).all(), (a, stochastic)
            assert torch.equal(y[a:b].cpu(), torch.from_numpy(R.values(rc, rs, cols)).bfloat16()), (a, stochastic)
        assert (y[rows:] == 9).all()
    # four bits into four bits, with float32 data of its own
    local = torch.ones(rows, cols, device="cuda:0")
    out = nz.Mx4(torch.empty_like(m.codes), torch.empty_like(m.scales))
    assert nz.nz_mx4_reduce_k([m], local, cols, rows, cols, 1, 29, out) == 0
    for a, b in parts:
        want = sum64([R.values(m.codes[a:b].cpu().numpy(), m.scales[a:b].cpu().numpy(), cols)], np.ones((b - a, cols)))
        rc, rs = R.quantize(want, True, 29, first=a * 32)
        assert (out.codes[a:b, :16].cpu().numpy() == rc).all() and (out.scales[a:b, :1].cpu().numpy() == rs).all(), a
    del x, m, y, local, out
    torch.cuda.empty_cache()
