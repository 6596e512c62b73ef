"""The device code of the e4m3 products: transfers into LDS written as inline assembly keep the distance that a lane read of their base asks
for, M0 is written by scalar instructions only."""
import re
import subprocess

import pytest

from tests.test_built_code import LIB, OBJDUMP, _code_objects


@pytest.mark.skipif(OBJDUMP is None or not LIB.exists(), reason="needs llvm-objdump and the built library")
def test_transfers_into_lds_after_lane_reads(tmp_path):
    transfers = 0
    for i, code in enumerate(_code_objects()):
        if b"fp8_tile_kernel" not in code:
            continue
        obj = tmp_path / f"{i}.co"
        obj.write_bytes(code)
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(obj)], capture_output=True, text=True, check=True).stdout
        recent = []                                        # the last instructions: (scalars a lane read wrote, wait states)
        for line in asm.splitlines():
            ins = re.match(r"\s+([a-z]\w+)\s*(.*?)\s*(//.*)?$", line)
            if not ins:
                continue
            name, args = ins.group(1), ins.group(2)
            if name.startswith("global_load_lds"):
                transfers += 1
                lo, hi = map(int, re.search(r"s\[(\d+):(\d+)\]", args).groups())
                states = 0
                for wrote, wait in reversed(recent):
                    if states >= 5:
                        break
                    assert not wrote & {lo, hi}, line
                    states += wait
            dst = re.match(r"s(\d+)", args)
            lane = {int(dst.group(1))} if name in ("v_readlane_b32", "v_readfirstlane_b32") and dst else set()
            assert name.startswith("s_") or not args.startswith("m0,"), line
            recent = recent[-8:] + [(lane, 1 + int(args, 0) if name == "s_nop" else 1)]
    assert transfers > 50
