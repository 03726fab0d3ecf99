"""Biases of any steepness: that of the nearest key, which is zero, and what its score
adds to it keep all their bits, however much the far keys' biases are.  Tolerances:
test_gpu_attention_scores.py (a bias' roundings are relative to itself).
"""

import numpy as np
import pytest

from test_gpu_attention_scores import Scored

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


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (8, 4, 64), (8, 2, 80), (8, 2, 256)])
@pytest.mark.parametrize("reqs", [[(1, 200), (1, 33), (1, 1), (4, 4000)], [(40, 170), (300, 300), (1, 90)], [(150, 150)]])
@pytest.mark.parametrize("softcap", [0.0, 30.0])
def test_steep_slopes(Hq, Hkv, D, reqs, softcap):
    b = Scored(reqs, Hq, Hkv, D, 16, seed=D)
    slopes = np.array([0.3, 1.7, 9.1, 77.3, 801.7, 9001.3, 1e5 / 3, 1e7 / 3], dtype=np.float32)
    b.both(slopes=slopes, softcap=softcap)
    b.both(slopes=-slopes, softcap=softcap)
    b.both(slopes=slopes, softcap=softcap, causal=False)


@pytest.mark.parametrize("reqs", [[(3, 2000), (1, 500)], [(200, 2000)]])
def test_steep_slopes_of_far_runs(reqs):
    """The nearest key that a token may see is far, or in the middle of a block of keys."""
    b = Scored(reqs, 4, 2, 64, 16, seed=5)
    slopes = np.array([2.3, 41.7, 907.1, 70001.3], dtype=np.float32)
    spans = np.array([[10 + i % 5, 150 + 7 * i % 200] for n, _ in reqs for i in range(n)], dtype=np.int32)
    b.both(slopes=slopes, spans=spans)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 1, 128), (8, 4, 64), (8, 2, 256)])
@pytest.mark.parametrize("kv", [32, 64, 96, 256, 4000, 4096])
def test_steep_slopes_at_a_blocks_end(Hq, Hkv, D, kv):
    """A single token that is the last of 32 keys, and one that sees the end of such a block alone."""
    b = Scored([(1, kv), (1, kv)], Hq, Hkv, D, 32, seed=D)
    slopes = np.array([0.3, 1.7, 9.1, 77.3, 801.7, 9001.3, 1e5 / 3, 1e7 / 3], dtype=np.float32)
    b.both(slopes=slopes)
    spans = np.array([[kv - 1, kv], [kv - 32, kv]], dtype=np.int32)
    b.both(slopes=slopes, spans=spans)
    b.both(slopes=slopes, softcap=30.0)
