"""Registers and shared memory of the microscaled products' kernels, from the metadata of the built library: what the choice of tiles and of
kernels for few rows counts on."""
import os
import re
import struct

import msgpack
import pytest

PRODUCT, LINEAR, GRAD = 0, 1, 2


@pytest.fixture(scope="module")
def kernels():
    from paper_2605_12396_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_12396_amd import build
        build.build()
    blob, found, at = open(binding.LIB_PATH, "rb").read(), {}, 0
    while (at := blob.find(b"AMDGPU\0\0", at + 1)) >= 0:         # ELF notes: name size, size, type, name, then a MessagePack map
        name_size, size, kind = struct.unpack_from("<III", blob, at - 12)
        if (name_size, kind) == (7, 32):
            for k in msgpack.unpackb(blob[at + 8:at + 8 + size])["amdhsa.kernels"]:
                m = re.match(r"_ZN2nz(?:12_GLOBAL__N_1)?\d+(k_mx_[a-z_]+?)(?:I((?:L[ibj]n?\d+E)+)E|E)", k[".name"])
                if m:
                    found[(m.group(1),) + tuple(int(x.replace("n", "-")) for x in re.findall(r"L[ibj](n?\d+)E", m.group(2) or ""))] = k
    return found


def resident(k):
    """Workgroups of a compute unit: 160 KB of shared memory, given out in pieces of 1280 bytes, and 512 registers a lane of a SIMD."""
    by_memory = (160 << 10) // max((k[".group_segment_fixed_size"] + 1279) // 1280 * 1280, 1)
    waves = -(-k[".max_flat_workgroup_size"] // 64 // 4)                # of a workgroup, on each SIMD
    return min(by_memory, 512 // ((k[".vgpr_count"] + 7) // 8 * 8) // waves)


@pytest.mark.parametrize("op", [PRODUCT, LINEAR, GRAD])
def test_tiles_of_a_compute_unit(kernels, op):
    """One tile of 256 x 256, two of 128 x 128: 256 and 512 on the chip."""
    tiles = {n[2]: k for n, k in kernels.items() if n[:2] == ("k_mx_tile", op)}
    assert set(tiles) == {128, 256}
    assert resident(tiles[256]) == 1 and resident(tiles[128]) == 2


def test_few_rows_of_a_compute_unit(kernels):
    """Kernels whose left comes through shared memory: two workgroups.  The others keep the next codes in registers instead and run alone."""
    few = {n: k for n, k in kernels.items() if n[0] == "k_mx_rows" and n[4] == 1}
    other = {n: k for n, k in kernels.items() if n[0] in ("k_mx_rows", "k_mx_grad_rows") and n not in few}
    assert len(few) == 8 and len(other) == 16 + 3
    assert all(resident(k) == 2 for k in few.values()) and all(resident(k) >= 1 for k in other.values())


def test_registers_spilled(kernels):
    """None but these: the gradient's tiles of 256 x 256, which have 512 registers a lane and save some after their loop, and one token
    of bfloat16 against many columns, which has 128 and saves two."""
    allowed = {("k_mx_tile", GRAD, 256, 256, 2, 2): 48, ("k_mx_rows", 1, 1, 2, 1): 2}
    assert len(kernels) > 40
    for n, k in kernels.items():
        assert k[".vgpr_spill_count"] <= allowed.get(n, 0), (n, k[".vgpr_spill_count"])
