"""GPU parity of the attention over the 8-bit cache in every way that its plan runs it: waves of 16 and
32 rows, each arrangement of them, sequences whole or split evenly by their lengths, and the partials
merged by the last workgroup or by a second kernel; batches of very different lengths."""
import numpy as np
import pytest

from paper_2606_18394_amd import synth
from test_gpu_fp8_attention import fp8_cache, gpu, oracle_and_bound, trees

pytestmark = pytest.mark.gpu

# (B, N, Hq, Hkv, D, capacity): the smallest of many shapes that take each way
CASES = [
    (2, 1, 1, 1, 64, 256),
    (2, 1, 1, 1, 64, 2048),
    (40, 1, 8, 8, 64, 256),
    (2, 300, 1, 1, 64, 1280),
    (9, 512, 1, 1, 64, 256),
    (2, 17, 4, 2, 64, 32000),
    (9, 17, 4, 2, 64, 3200),
    (40, 17, 8, 8, 64, 256),
    (2, 150, 1, 1, 64, 32000),
    (2, 300, 2, 1, 64, 2048),
    (20, 17, 32, 4, 64, 256),
    (2, 33, 4, 2, 64, 16000),
    (9, 33, 2, 1, 64, 9600),
    (40, 33, 8, 8, 64, 256),
    (3, 33, 16, 1, 64, 16000),
    (9, 33, 8, 8, 64, 6400),
    (40, 33, 16, 8, 64, 256),
    (3, 100, 8, 1, 64, 16000),
    (20, 33, 24, 8, 64, 2048),
    (2, 1, 1, 1, 128, 256),
    (5, 1, 1, 1, 128, 32000),
    (2, 1, 1, 1, 128, 2048),
    (40, 1, 8, 8, 128, 256),
    (2, 1, 1, 1, 128, 16000),
    (3, 1, 1, 1, 128, 1280),
    (9, 512, 1, 1, 128, 256),
    (2, 33, 1, 1, 128, 32000),
    (9, 17, 4, 2, 128, 3200),
    (40, 17, 8, 8, 128, 256),
    (2, 33, 8, 1, 128, 9600),
    (2, 300, 2, 1, 128, 2048),
    (20, 17, 32, 4, 128, 256),
    (9, 33, 2, 1, 128, 6400),
    (9, 100, 2, 1, 128, 3200),
    (40, 33, 8, 8, 128, 256),
    (3, 33, 16, 1, 128, 16000),
    (9, 33, 16, 1, 128, 3200),
    (40, 33, 16, 8, 128, 256),
    (3, 100, 8, 1, 128, 16000),
    (20, 33, 24, 8, 128, 2048),
    (20, 1, 1, 1, 128, 2048),
    (2, 1, 8, 8, 128, 1280),
    (9, 1, 1, 1, 64, 6400),
    (5, 1, 1, 1, 64, 2048),
    (9, 100, 2, 1, 64, 3200),
]


def lengths(B, L):
    """One nearly full, one empty, one of half, the rest up to a quarter."""
    return ([L - 5, 0, L // 2 + 3] + [(41 * i * i + 7) % (L // 4 + 1) for i in range(B)])[:B]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_parity(case):
    B, N, Hq, Hkv, D, L = CASES[case]
    print(f"plan case {CASES[case]}", flush=True)
    rng = np.random.default_rng(7000 + case)
    bs = 64 if L % 64 == 0 else 32
    kvl = lengths(B, L)
    k, v, ke, ve, bt = fp8_cache(rng, B, Hkv, D, bs, L // bs, kvl)
    q = synth._normal_bf16(rng, (B, N, Hq, D))
    kt, vt = (synth._normal_bf16(rng, (B, N, Hkv, D)) for _ in range(2))
    args = (q, k, v, ke, ve, bt, kt, vt, trees(rng, B, N, "random" if N > 1 else "none"), np.array(kvl))
    out = gpu(*args)
    ref, tol = oracle_and_bound(*args)
    assert np.isfinite(out).all()
    err = np.abs(out - ref)
    assert (err <= tol).all(), (err / tol).max()
