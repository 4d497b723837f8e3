"""Plans of the attention over the 8-bit cache, checked on the host (the plan header is plain C++),
and the register use of its kernels."""
import os
import random
import re
import shutil
import subprocess

import pytest

from paper_2606_18394_amd import build
import test_gpu_fp8_plans
from test_kernel_registers import READELF, code_objects

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18394_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("flags", [["-O1"], ["-O1", "-g", "-fsanitize=address,undefined",
                                             "-fno-sanitize-recover=undefined"]])
def test_plans(tmp_path, flags):
    """Over a grid of shapes, also under the host's sanitizers."""
    exe = tmp_path / "plan_fp8_check"
    made = subprocess.run(["g++", "-std=c++17", *flags, "-I", CSRC,
                           os.path.join(ROOT, "tests", "native", "plan_fp8_check.cpp"), "-o", str(exe)],
                          capture_output=True, text=True)
    if made.returncode != 0 and len(flags) > 1:
        pytest.skip("host sanitizer runtime not available: " + made.stderr[-200:])
    assert made.returncode == 0, made.stderr[-2000:]
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0 and "FAIL" not in res.stdout, res.stdout[-2000:] + res.stderr[-1000:]
    assert int(re.search(r"\d+", res.stdout).group()) > 10000


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_way_has_a_case(tmp_path):
    """All arrangements, unsplit and with either merge, that a draw of shapes takes are among the GPU
    parity cases."""
    exe = tmp_path / "plan_fp8_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC,
                    os.path.join(ROOT, "tests", "native", "plan_fp8_check.cpp"), "-o", str(exe)], check=True)

    def ways(shapes):
        res = subprocess.run([str(exe), "-"], input="".join("%d %d %d %d %d %d\n" % s for s in shapes),
                             capture_output=True, text=True, check=True)
        return set(res.stdout.splitlines())

    rng = random.Random(4)
    drawn = []
    for _ in range(40000):
        hq, hkv = rng.choice([(4, 2), (32, 8), (32, 4), (8, 8), (16, 8), (8, 1), (24, 8), (2, 1), (64, 8),
                              (1, 1), (16, 1)])
        drawn.append((rng.choice([1, 1, 2, 3, 5, 9, 20, 40]), rng.choice([1, 2, 17, 33, 64, 100, 150, 300, 512]),
                      hq, hkv, rng.choice([64, 128]), 32 * rng.choice([8, 20, 40, 64, 100, 128, 200, 300, 1000])))
    taken = ways(drawn)
    assert len(taken) >= 40 and taken <= ways(test_gpu_fp8_plans.CASES), taken - ways(test_gpu_fp8_plans.CASES)


@pytest.mark.skipif(not shutil.which(READELF), reason="needs llvm-readelf")
def test_kernels_do_not_spill(tmp_path):
    """Nor do the writers and page kernels.  The exception: waves of 32 rows with rings of their own
    at D = 128 put three values away ahead of the tile loop that are read behind it (holding V's
    codes for a shorter time instead does not change a call's time)."""
    if not os.path.exists(build.LIB):
        build.build()
    seen = {}
    for k, obj in enumerate(code_objects(build.LIB)):
        elf = tmp_path / f"{k}.o"
        elf.write_bytes(obj)
        notes = subprocess.run([READELF, "--notes", str(elf)], capture_output=True, text=True,
                               check=True).stdout
        for entry in re.split(r"\n\s*- \.agpr_count:", notes)[1:]:
            name = re.search(r"\n\s*\.name:\s*(\S+)", entry).group(1)
            if not re.search(r"(attn|combine)_fp8|write_|grow_|reserve_|fork_|free_|copy_|compact_", name):
                continue
            seen[name] = [int(re.search(rf"\n\s*\.{f}:\s*(\d+)\n", entry).group(1))
                          for f in ("vgpr_spill_count", "private_segment_fixed_size")]
    assert sum("attn_fp8" in n for n in seen) == 14 and len(seen) >= 26, sorted(seen)
    for name, (spills, scratch) in seen.items():
        kept = re.search(r"attn_fp8ILi128ELi1ELi[48]ELi2E", name)
        assert spills <= (3 if kept else 0) and scratch <= (16 if kept else 0), (name, spills, scratch)
