"""Which kernel serves a product of e4m3 rows (0: the one for few rows, else rows per chunk of the tile kernel), and what the compiler made of the e4m3
and gate kernels.  No kernel is launched here."""
import re
import shutil
import subprocess

import pytest

from paper_2407_14417_amd import binding as mm
from tests.test_built_code import LIB, _code_objects

READELF = shutil.which("llvm-readelf", path="/opt/rocm/llvm/bin")
F16, F32 = False, True


def rows_per_chunk(P, inn, out, exact, E=1, T=None, gathered=False, up=False):
    return mm.lib().moemix_fp8_rows_per_chunk(E, T or P, P, out, inn, int(gathered), int(exact), int(up))


@pytest.mark.parametrize("P,inn,out,exact,E,tile", [
    # (both kernels measured, us: few and tile)
    (8, 4096, 14336, F16, 1, False),      # 16.7, 18.6
    (48, 4096, 14336, F16, 1, True),      # 25.0, 18.9
    (32, 4096, 14336, F32, 1, False),     # 21.3, 24.5
    (64, 14336, 4096, F32, 1, False),     # 37.4, 61
    (8, 14336, 4096, F32, 8, False),      # 83, 106
    (8, 1408, 2048, F32, 32, False),      # 6.3, 9.1
    # one row, a ragged handful, a prompt, a gradient, experts of a prompt and with a skewed load
    (1, 4096, 14336, F16, 1, False), (37, 1488, 1001, F32, 1, False), (4096, 4096, 14336, F16, 1, True), (1000, 14336, 4096, F32, 1, True),
    (4096, 4096, 14336, F16, 8, True), (1200, 2048, 1408, F32, 32, True),
])
def test_the_faster_kernel_of_the_two(P, inn, out, exact, E, tile):
    assert (rows_per_chunk(P, inn, out, exact, E) > 0) == tile


@pytest.mark.parametrize("inn,out,exact", [(4096, 14336, F16), (4096, 14336, F32), (14336, 4096, F16), (1024, 8192, F16), (2048, 2048, F32)])
def test_more_rows_end_in_the_tile_kernel(inn, out, exact):
    """One row has the kernel for few rows, thousands the tile kernel, in chunks of whole tiles that it has room for."""
    chunks = [rows_per_chunk(P, inn, out, exact) for P in (1, 4096)]
    assert chunks[0] == 0 and chunks[1] > 0
    for P in range(1, 4200, 67):
        per = rows_per_chunk(P, inn, out, exact)
        assert per % 16 == 0 and 0 <= per <= (160 if exact else 256)


def test_rows_past_32_bit_offsets_are_not_gathered_by_the_tile_kernel():
    for gathered, n, tile in ((True, (1 << 20) - 2, True), (True, 1 << 20, False), (False, 1 << 20, True)):
        assert (rows_per_chunk(4096, 4096, 4096, F16, 8, n, gathered) > 0) == tile
    assert rows_per_chunk(4096, 0, 4096, F16) == 0           # sums over no columns


@pytest.mark.skipif(READELF is None or not LIB.exists(), reason="needs llvm-readelf and the built library")
def test_registers_do_not_spill_to_memory(tmp_path):
    seen = {}
    for i, code in enumerate(_code_objects()):
        obj = tmp_path / f"{i}.co"
        obj.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
        for kernel in notes.split("- .agpr_count:")[1:]:
            name = re.search(r"\.symbol:\s+(\S+)", kernel).group(1)
            if re.search(r"fp8|balance_|gate_|route_kernel", name):
                seen[name] = [int(re.search(rf"\.{k}:\s+(\d+)", kernel).group(1)) for k in ("vgpr_spill_count", "private_segment_fixed_size")]
    assert sum("fp8_tile_kernel" in n for n in seen) == 4 and sum("gate_dx_dw_kernel" in n for n in seen) == 4
    assert all(v == [0, 0] for v in seen.values()), {n: v for n, v in seen.items() if v != [0, 0]}
