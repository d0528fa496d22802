"""What the microscaled 4-bit operators are measured on.

A matrix in this form (nz_mx4_*) holds each row in blocks of 32 elements: 16 bytes of codes, the low half of a byte first, and one byte s
that scales the block by 2^(s - 127).  A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Five operators deal with it:

  convert  a float matrix or message into that form and back out of it, as its sender and its receiver do;
  reduce   k such messages, and a rank's own float32 data, into one message or into floats;
  product  of two such matrices over their rows' common length, C = A B^T;
  linear   the same with floats for A: activations against weights that arrived in four bits;
  grad     the gradient of either product for its left operand, dA = G B.

Messages have the sizes of perf/cases.py; the products' sizes are ordinary widths of a layer, from one token to thousands.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SMALLEST, LARGEST = 16 << 10, 64 << 20      # elements of a message: 64 KB and 256 MB of float32
LARGEST_REDUCE = 32 << 20                   # elements of each of up to eight messages
LARGEST_SIDE = 8192                         # of a product


def _message(name, op, rows, cols, kind="f32", out="f32", sr=False, k=1, local=False):
    """kind: type of the floats that go in; out: of those that come out, "mx4" where a reduce hands on four bits; sr: stochastic rounding."""
    c = {"op": op, "rows": rows, "cols": cols, "kind": kind, "out": out, "sr": sr, "k": k, "local": local}
    return dict(c, name=name) if name else c


def _product(name, op, m, n, k, kind, out):
    """kind: type of the left operand ("mx4" for product)."""
    c = {"op": op, "m": m, "n": n, "k": k, "kind": kind, "out": out}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest message of the size sweep, sent and received: nothing but latency
        _message("convert-64KB", "convert", 1, 16384),
        # activations of a batch of ragged length in a width that is no multiple of a block
        _message("convert-2049x4095-bf16", "convert", 2049, 4095, "bf16", "bf16"),
        # the 256 MB gradient, rounded without bias
        _message("convert-256MB-stochastic", "convert", 1, 64 << 20, sr=True),
        # ring step on a bucket of gradients: the incoming message and the rank's own data, sent on in four bits
        _message("ring-step-1MB", "reduce", 1, 300007, out="mx4", local=True),
        # eight peers' chunks become the float shard that an optimizer reads
        _message("reduce-8x128MB", "reduce", 1, 32 << 20, k=8),
        # one token, weights and activations in four bits
        _product("product-1-token", "product", 1, 4096, 4096, "mx4", "bf16"),
        # a ragged batch in odd widths
        _product("product-777x4100x2050", "product", 777, 4100, 2050, "mx4", "f32"),
        # a large batch
        _product("product-8192", "product", 8192, 8192, 8192, "mx4", "bf16"),
        # one token against a layer's weights
        _product("linear-1-token", "linear", 1, 8192, 8192, "bf16", "bf16"),
        # a training batch against a layer's weights, and back
        _product("linear-4096-tokens", "linear", 4096, 8192, 4096, "bf16", "bf16"),
        _product("grad-4096-tokens", "grad", 4096, 8192, 4096, "bf16", "bf16"),
        # a small ragged batch of float32 gradients through odd widths
        _product("grad-509-tokens-f32", "grad", 509, 4096, 2050, "f32", "f32"),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("convert", "convert", "reduce", "reduce", "product", "product", "linear", "linear", "grad"))
    if op in ("convert", "reduce"):
        n = _spread(rng, SMALLEST, LARGEST if op == "convert" else LARGEST_REDUCE)
        rows = _spread(rng, 2, 2048) if rng.random() < 0.5 else 1
        cols = max(1, n // rows)
        if op == "convert":
            return _message(None, op, rows, cols, rng.choice(tuple(TYPES)), rng.choice(tuple(TYPES)), rng.random() < 0.5)
        return _message(None, op, rows, cols, "f32", rng.choice(("mx4", "mx4", "f32", "bf16", "f16")), rng.random() < 0.5, rng.randint(1, 8),
                        rng.random() < 0.5)
    n, k = _spread(rng, 64, LARGEST_SIDE), _spread(rng, 64, LARGEST_SIDE)
    m = _spread(rng, 1, LARGEST_SIDE if op == "product" else LARGEST_SIDE // 2)
    if op != "product":
        k = min(k, LARGEST_SIDE // 2)
    return _product(None, op, m, n, k, "mx4" if op == "product" else rng.choice(("bf16", "bf16", "f16", "f32")),
                    rng.choice(("bf16", "f16", "f32")))


# ---- the form, with elementary operations ----

def _row_blocks(cols):
    return (cols + 31) // 32


def _pitch(cols):
    return (_row_blocks(cols) + 3) // 4 * 4


def _power(s):
    """2^(s - 127) as float32 from its bits; 255 stands for NaN."""
    s = s.to(torch.int32)
    return torch.where(s == 0, 0x00400000, torch.where(s == 255, 0x7FC00000, s << 23)).to(torch.int32).view(torch.float32)


def _inverse(s):
    """2^(127 - s) as float32, for s up to 253."""
    return ((254 - s.clamp(max=253).to(torch.int32)) << 23).view(torch.float32)


def _times32(h, c):
    """h * c modulo 2^32, in int64 without overflow."""
    return ((h & 0xFFFF) * c + (((h >> 16) * c & 0xFFFF) << 16)) & 0xFFFFFFFF


def _fmix(h):
    """32-bit finalizer of MurmurHash3."""
    h = _times32(h ^ (h >> 16), 0x85EBCA6B)
    h = _times32(h ^ (h >> 13), 0xC2B2AE35)
    return h ^ (h >> 16)


def _draws(count, seed, device):
    """16 bits for each of `count` elements, 32 of a pair at a time, from a counter."""
    pair = torch.arange((count + 1) // 2, dtype=torch.int64, device=device)
    key = _fmix((seed + 0x9E3779B9 * (pair >> 32)) & 0xFFFFFFFF)
    h = _fmix((pair & 0xFFFFFFFF) ^ key)
    return torch.stack((h & 0xFFFF, h >> 16), 1).reshape(-1)[:count].to(torch.float32)


def _encode(x, sr, seed):
    """Codes [rows, blocks, 32] and scales [rows, blocks] of float32 x [rows, cols]."""
    rows, cols = x.shape
    nb = _row_blocks(cols)
    if cols != nb * 32:
        x = torch.nn.functional.pad(x, (0, nb * 32 - cols))
    x = x.reshape(rows, nb, 32)
    peak = (x.view(torch.int32) & 0x7FFFFFFF).amax(2)
    e = peak >> 23
    s = e - 2
    if sr:                                      # no element past 6: the rounding stays without bias
        s = s + ((peak & 0x7FFFFF) > 0x400000).to(torch.int32)
    s = s.clamp(0, 252)
    bad = e == 255
    a = x.abs() * _inverse(s)[..., None]
    if sr:
        c = sum((a >= g).to(torch.int8) for g in GRID[1:])
        grid = torch.tensor(GRID + (8.0,), device=x.device)
        low = grid[c.int()]
        frac = (a - low) / (grid[c.int() + 1] - low)
        u = _draws(rows * nb * 32, seed, x.device).reshape(rows, nb, 32)
        c = (c + ((u + 0.5) * 2.0 ** -16 < frac).to(torch.int8)).clamp(max=7)
    else:                                       # ties to the even code
        c = ((a > 0.25).to(torch.int8) + (a >= 0.75).to(torch.int8) + (a > 1.25).to(torch.int8) + (a >= 1.75).to(torch.int8)
             + (a > 2.5).to(torch.int8) + (a >= 3.5).to(torch.int8) + (a > 5.0).to(torch.int8))
    c = torch.where(bad[..., None], 0, c | ((x.view(torch.int32) < 0).to(torch.int8) << 3))
    return c.to(torch.uint8), torch.where(bad, 255, s).to(torch.uint8)


def _values(c, s, cols):
    """float32 [rows, cols] of codes and scales."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=c.device)
    v = grid[c.int()] * _power(s)[..., None]
    return v.reshape(c.shape[0], -1)[:, :cols]


def _pack(c, s, cols):
    """The bytes that the operators take: codes [rows, 16 pitch], scales [rows, pitch]."""
    rows, nb = s.shape
    codes = torch.zeros(rows, _pitch(cols) * 16, dtype=torch.uint8, device=c.device)
    scales = torch.zeros(rows, _pitch(cols), dtype=torch.uint8, device=c.device)
    c = c.reshape(rows, nb * 16, 2)
    codes[:, :nb * 16] = c[..., 0] | (c[..., 1] << 4)
    scales[:, :nb] = s
    return codes, scales


def _unpack(codes, scales, cols):
    rows, nb = codes.shape[0], _row_blocks(cols)
    b = codes[:, :nb * 16]
    return _values(torch.stack((b & 15, b >> 4), 2).reshape(rows, nb, 32), scales[:, :nb], cols)


# ---- inputs ----

def _gradient(rows, cols, g):
    """Heavy tails about nothing, and a few outliers."""
    u = torch.rand(rows, cols, generator=g, device="cuda") - 0.5
    x = -torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.4999999)) * 1e-3
    return torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 1e-4, x * 50, x)


def _activation(rows, cols, g):
    """Normal, with a few loud columns."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    loud = torch.rand(cols, generator=g, device="cuda") < 0.01
    return torch.where(loud, x * 20, x)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case, "seed": seed & 0xFFFFFFFF}
    if case["op"] in ("convert", "reduce"):
        rows, cols = case["rows"], case["cols"]
        shape = (rows, _pitch(cols))
        if case["op"] == "convert":
            make = _gradient if rows == 1 else _activation
            st["x"] = make(rows, cols, g).to(TYPES[case["kind"]])
        else:
            st["in"] = [_pack(*_encode(_gradient(rows, cols, g), False, 0), cols) for _ in range(case["k"])]
            st["local"] = _gradient(rows, cols, g) if case["local"] else None
        # the buffers that a rank keeps: the message it sends, and the floats it reads
        st["codes"] = torch.zeros(rows, shape[1] * 16, dtype=torch.uint8, device="cuda")
        st["scales"] = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        st["y"] = torch.empty(rows, cols, dtype=TYPES["f32" if case["out"] == "mx4" else case["out"]], device="cuda")
    else:
        m, n, k = case["m"], case["n"], case["k"]
        st["b"] = _pack(*_encode(torch.randn(n, k, generator=g, device="cuda") * 0.02, False, 0), k)
        if case["op"] == "product":
            st["a"] = _pack(*_encode(_activation(m, k, g), False, 0), k)
        elif case["op"] == "linear":
            st["x"] = _activation(m, k, g).to(TYPES[case["kind"]])
        else:
            st["x"] = torch.randn(m, n, generator=g, device="cuda").to(TYPES[case["kind"]])
        st["y"] = torch.empty(m, k if case["op"] == "grad" else n, dtype=TYPES[case["out"]], device="cuda")
    if own:
        from paper_2605_12396_amd import binding as nz
        st["nz"] = nz
        for name in ("a", "b"):
            if name in st:
                st["h" + name] = nz.Mx4(*st[name])
        if "in" in st:
            st["hin"] = [nz.Mx4(*t) for t in st["in"]]
        if "codes" in st:
            st["hout"] = nz.Mx4(st["codes"], st["scales"])
        if "b" in st:
            kind = {"product": nz.MX4_PRODUCT, "linear": nz.MX4_LINEAR, "grad": nz.MX4_GRAD}[case["op"]]
            st["ws_bytes"] = nz.nz_mx4_workspace_bytes(kind, st["x"].dtype if "x" in st else None, m, n, k)
            st["ws"] = torch.empty(max(st["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return st


# ---- one pass ----

def _run_own(st):
    nz, case = st["nz"], st["case"]
    y = st["y"]
    if case["op"] in ("convert", "reduce"):
        rows, cols = case["rows"], case["cols"]
        rounding = nz.MX4_STOCHASTIC if case["sr"] else nz.MX4_NEAREST
        if case["op"] == "convert":
            rc = nz.nz_mx4_quantize(st["x"], rows, cols, cols, rounding, st["seed"], st["hout"])
        elif case["out"] == "mx4":
            rc = nz.nz_mx4_reduce_k(st["hin"], st["local"], cols, rows, cols, rounding, st["seed"], st["hout"])
        else:
            rc = nz.nz_mx4_sum_k(st["hin"], st["local"], cols, rows, cols, y, cols)
        if rc == 0 and (case["op"] == "convert" or case["out"] == "mx4"):
            rc = nz.nz_mx4_dequantize(st["hout"], rows, cols, y, cols)
    else:
        m, n, k = case["m"], case["n"], case["k"]
        if case["op"] == "product":
            rc = nz.nz_mx4_product(st["ha"], st["hb"], m, n, k, y, n, st["ws"], st["ws_bytes"])
        elif case["op"] == "linear":
            rc = nz.nz_mx4_linear(st["x"], k, st["hb"], m, n, k, y, n, st["ws"], st["ws_bytes"])
        else:
            rc = nz.nz_mx4_grad(st["x"], n, st["hb"], m, n, k, y, k, st["ws"], st["ws_bytes"])
    if rc != 0:
        raise RuntimeError("status %d" % rc)
    return y


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    out = st["y"].dtype
    if case["op"] == "convert":
        return _values(*_encode(st["x"].float(), case["sr"], st["seed"]), case["cols"]).to(out)
    if case["op"] == "reduce":
        acc = None
        for codes, scales in st["in"]:
            v = _unpack(codes, scales, case["cols"])
            acc = v if acc is None else acc + v
        if st["local"] is not None:
            acc = acc + st["local"]
        if case["out"] == "mx4":
            acc = _values(*_encode(acc, case["sr"], st["seed"]), case["cols"])
        return acc.to(out)
    k = case["k"]
    b = _unpack(*st["b"], k)
    if case["op"] == "product":
        return (_unpack(*st["a"], k) @ b.t()).to(out)
    if case["op"] == "linear":
        return (st["x"].float() @ b.t()).to(out)
    return (st["x"].float() @ b).to(out)


def work(case):
    def held(rows, cols):
        return rows * (_row_blocks(cols) * 17)
    if case["op"] in ("convert", "reduce"):
        n = case["rows"] * case["cols"]
        four = held(case["rows"], case["cols"])
        floats = n * BYTES["f32" if case["out"] == "mx4" else case["out"]]
        if case["op"] == "convert":             # written by the sender, read by the receiver
            return {"bytes": n * BYTES[case["kind"]] + 2 * four + floats, "flops": 3 * n}
        again = 2 * four if case["out"] == "mx4" else 0
        local = 4 * n if case["local"] else 0
        return {"bytes": case["k"] * four + local + again + floats, "flops": (2 * case["k"] + 3) * n}
    m, n, k = case["m"], case["n"], case["k"]
    inner, outer = (n, k) if case["op"] == "grad" else (k, n)
    left = held(m, k) if case["op"] == "product" else m * inner * BYTES[case["kind"]]
    return {"bytes": left + held(n, k) + m * outer * BYTES[case["out"]], "flops": 2 * m * n * k}


# ---- the definition, in 64 bits ----

def _held64(codes, scales, cols):
    """Element j of block i of a row: (-1)^sign * magnitude * 2^(s - 127), magnitude from its exponent and mantissa bits."""
    rows, nb = codes.shape[0], _row_blocks(cols)
    c = codes[:, :nb * 16].reshape(rows, nb, 16, 1) >> torch.tensor([0, 4], dtype=torch.uint8, device=codes.device)
    c = (c & 15).reshape(rows, nb, 32).to(torch.float64)
    sign = 1 - 2 * torch.floor(c / 8)
    c = torch.remainder(c, 8)
    e, f = torch.floor(c / 2), torch.remainder(c, 2)
    mag = torch.where(e == 0, f / 2, (1 + f / 2) * torch.exp2(e - 1))
    s = scales[:, :nb].to(torch.float64)
    scale = torch.where(s == 255, float("nan"), torch.exp2(s - 127))
    return (sign * mag * scale[..., None]).reshape(rows, nb * 32)[:, :cols]


def _pairs64(count, seed):
    """The draws of `count` pairs of elements: MurmurHash3's finalizer of the pair's number and of the seed's."""
    def mix(h):
        h = h.astype(np.uint32)
        h ^= h >> np.uint32(16)
        h *= np.uint32(0x85EBCA6B)
        h ^= h >> np.uint32(13)
        h *= np.uint32(0xC2B2AE35)
        return h ^ (h >> np.uint32(16))
    i = np.arange(count, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    key = mix((np.uint64(seed) + np.uint64(0x9E3779B9) * (i >> np.uint64(32))) & low)
    return mix((i & low).astype(np.uint32) ^ key)


def _nearest64(x, sr, seed):
    """What a row of float64 x stands for once held in four bits, by the definition: the block's power of two from its peak, then the
    nearer of the two neighbours in the grid (ties to an even mantissa), or the one that the draw picks."""
    rows, cols = x.shape
    nb = _row_blocks(cols)
    full = torch.zeros(rows, nb * 32, dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    full = full.reshape(rows, nb, 32)
    peak = full.abs().amax(2)
    _, exponent = torch.frexp(torch.where(peak > 0, peak, 1.0))
    e = torch.where(peak > 0, exponent.to(torch.float64) - 1, -200.0) - 2       # 2^e lies two octaves under the peak
    if sr:
        e = torch.where(peak > 6 * torch.exp2(e), e + 1, e)
    e = e.clamp(-127, 125)
    unit = torch.exp2(e)[..., None]
    a = full.abs() / unit
    octave = torch.frexp(a.clamp(min=1.0, max=7.0))[1].to(torch.float64) - 1
    spacing = torch.exp2(octave) / 2                                            # 1/2 under 2, 1 under 4, 2 from there
    if sr:
        low = torch.floor(a / spacing)
        h = _pairs64(rows * nb * 16, seed)
        u = torch.from_numpy(np.stack((h & np.uint32(0xFFFF), h >> np.uint32(16)), 1).reshape(-1).astype(np.float64)).to(x.device)
        q = (low + ((u.reshape(rows, nb, 32) + 0.5) / 65536 < a / spacing - low).double()) * spacing
    else:
        q = torch.round(a / spacing) * spacing                                  # halves to even
    q = torch.where(full < 0, -q.clamp(max=6.0), q.clamp(max=6.0)) * unit
    return q.reshape(rows, nb * 32)[:, :cols]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "convert":
        return _nearest64(st["x"].double(), case["sr"], st["seed"])
    if case["op"] == "reduce":
        total = sum(_held64(*t, case["cols"]) for t in st["in"])
        if st["local"] is not None:
            total = total + st["local"].double()
        if case["out"] == "mx4":                # what a receiver adds is float32
            return _nearest64(total.float().double(), case["sr"], st["seed"])
        return total
    b = _held64(*st["b"], case["k"])
    if case["op"] == "product":
        return _held64(*st["a"], case["k"]) @ b.t()
    return st["x"].double() @ (b.t() if case["op"] == "linear" else b)
