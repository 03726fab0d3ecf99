"""lora_batched where a low-rank value is infinite: the outputs are what the
definition gives, infinite by that rank's sign or NaN, whatever the finite ranks
beside it are.
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


@pytest.mark.parametrize("M,N,r", [(20, 40, 8), (20, 40, 60), (33, 24, 200), (200, 72, 40), (200, 72, 200)])
def test_infinite_beside_large_ranks(M, N, r):
    rng = np.random.default_rng(M + r)
    K, L = 64, 2
    x = rng.standard_normal((M, K)).astype(np.float16)
    x[:, 0] = np.where(np.arange(M) % 3 == 0, 0, 1)  # every third token meets the infinity with a zero
    A = (rng.standard_normal((L, r, K)) * 1e4).astype(np.float16)  # other ranks beyond fp16's largest value
    A[:, :, 0] = 0
    A[0, 3, 0], A[1, r - 1, 0] = np.inf, -np.inf
    B = rng.standard_normal((L, N, r)).astype(np.float16)
    B[:, 5] = 0
    ids = rng.integers(-1, L, M).astype(np.int32)
    scales = np.array([1.5, -0.5], np.float32)
    with np.errstate(invalid="ignore"):
        ref, _ = lo.lora(x, ids, A, B, scales)
    got, = fasq.lora_batched(to_dev(x), to_dev(ids), [to_dev(A)], [to_dev(B)], to_dev(scales), [None])
    got = to_np(got).astype(np.float64)
    assert not np.isfinite(ref[ids >= 0]).any()
    assert np.isinf(ref).sum() > 100 and np.isnan(ref).sum() > 100 and np.isfinite(A).sum() == A.size - 2
    wrong = int((~((got == ref) | (np.isnan(got) & np.isnan(ref)))).sum())
    assert wrong == 0
