"""lora_batched where a token's low-rank values differ widely in size.

Tolerance as in test_gpu_norm_lora: half a unit in the last place of fp16, and
2^-16 of |s| |B| (|A| |x|) for fp32 sums and low-rank values held to 22 bits
down to 2^-17 of a token's largest, to 19 bits down to 2^-20.
"""

import numpy as np
import pytest

from oracle import layer_ops as lo
from gpu_util import to_dev, to_np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
fasq = pytest.importorskip("paper_2605_04084_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fasq.lib()
    yield
    torch.cuda.synchronize()


# sums by a workgroup itself (up to 16 ranks, up to 64, more), and folded before
# (blocks of 64 and of 128 tokens)
SHAPES = [(20, 512, 96, 16, 3), (20, 512, 100, 40, 3), (40, 512, 72, 130, 4), (200, 512, 130, 40, 3), (200, 512, 136, 130, 2),
          (1030, 128, 22016, 40, 3)]


def _run(x, ids, A, B, scales, base):
    got, = fasq.lora_batched(to_dev(x), to_dev(ids), [to_dev(A)], [to_dev(B)], to_dev(scales), [None if base is None else to_dev(base)])
    return to_np(got).astype(np.float64)


@pytest.mark.parametrize("bits", [12, 16, 20])
@pytest.mark.parametrize("M,K,N,r,L", SHAPES)
def test_ranks_of_different_size(M, K, N, r, L, bits):
    """Every other rank is 2^bits smaller in A and as much larger in B, so that all count alike."""
    rng = np.random.default_rng(M + r + bits)
    small = np.arange(r) % 2 == 1
    size_a = np.where(small, 2.0 ** (8 - bits), 2.0 ** 8) * K ** -0.5
    size_b = np.where(small, 2.0 ** (bits - 12), 2.0 ** -12)
    x = rng.standard_normal((M, K)).astype(np.float16)
    A = (rng.standard_normal((L, r, K)) * size_a[:, None]).astype(np.float16)
    B = (rng.standard_normal((L, N, r)) * size_b).astype(np.float16)
    ids = rng.integers(-1, L, M).astype(np.int32)
    scales = rng.uniform(0.5, 2, L).astype(np.float32)
    ref, mass = lo.lora(x, ids, A, B, scales)
    got = _run(x, ids, A, B, scales, None)
    tol = np.abs(ref) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * 2.0 ** -16
    err = np.abs(got - ref)
    assert (err <= tol).all(), (int((err > tol).sum()), float((err - tol).max()), float(np.abs(ref).max()))
