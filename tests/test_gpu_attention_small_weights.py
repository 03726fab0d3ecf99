"""paged_attention where most of a row's weight lies in many small weights.

Scores are exact: one key (the sink) stands a given number of powers of two
above all others, whose values alone are not zero.  The tolerance of a
logarithm of a sum is test_gpu_attention's: 2^-20 of the sum of |q| |k| and of
itself, a few fp32 roundings, whatever the number of keys.  Of an output: half
a unit in the last place; 2^-11 of the weighted sum of |v| for weights held in
fp16, and 2^-14 of it for fp32 scores and sums; and where weights lie among
fp16's subnormals a step of 2^-24 at a scale where the row's largest is 2^7 or
more: 2^-32 of the largest |v| per key.
"""

import math

import numpy as np
import pytest

from oracle import layer_ops as lo
from test_gpu_attention import Batch

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


def _sink(n, kv, Hq, D, at):
    b = Batch([(n, kv)], Hq, 1, D, 64, seed=kv)
    b.q[:] = 0
    b.q[..., 0] = 1
    j = np.arange(kv)
    k, v = np.zeros((kv, 1, D), np.float16), np.ones((kv, 1, D), np.float16)
    k[at, :, 0] = 1
    v[at] = 0
    v[:, :, 1] *= (j % 7)[:, None] / 8
    b.k[b.slot(0, j)], b.v[b.slot(0, j)] = k, v
    return b


CASES = pytest.mark.parametrize("n,kv,Hq,D,at,split", [
    (1, 131072, 2, 64, 0, False), (1, 131072, 2, 64, 70000, True), (1, 40000, 1, 256, 5, False),
    (100, 131072, 2, 64, 0, False), (100, 30000, 2, 128, 4, True), (70, 20000, 2, 256, 19000, False),
])
POWERS = pytest.mark.parametrize("powers", [16.0, 22.4, 24.6, 25.5, 28.0])


def _both(b, powers, split):
    scale = powers * math.log(2.0)
    kw = {} if split else {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda:0")}
    return b.run(scale=scale, **kw), lo.paged_attention(b.q, b.k, b.v, b.pages, b.q_start, b.kv_len, scale), scale


@POWERS
@CASES
def test_sum_of_many_weights_far_below_one(n, kv, Hq, D, at, split, powers):
    (_, lse), (_, want, _), scale = _both(_sink(n, kv, Hq, D, at), powers, split)
    assert (np.abs(lse - want) <= 2.0 ** -20 * (scale + np.abs(want) + 1)).all(), float(np.abs(lse - want).max())


@POWERS
@CASES
def test_output_of_many_weights_far_below_one(n, kv, Hq, D, at, split, powers):
    (out, _), (want, _, mass), _ = _both(_sink(n, kv, Hq, D, at), powers, split)
    tol = np.abs(want) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -14) + kv * 2.0 ** -32
    err = np.abs(out.astype(np.float64) - want)
    assert (err <= tol).all(), (float((err - tol).max()), float((err / np.maximum(want, 1e-30)).max()))


@pytest.mark.parametrize("n,split", [(1, True), (3, False), (100, True), (100, False)])
@pytest.mark.parametrize("top", [2.0 ** 23, 2.0 ** 25, 2.0 ** 27])
def test_scores_whose_rounding_passes_the_weights(n, split, top):
    """Equal scores so large that fp32 rounds them to whole powers of two and
    more: every key counts alike."""
    kv, D = 700, 64
    b = Batch([(n, kv)], 2, 1, D, 16, seed=n)
    b.q[:], b.k[:] = 1, np.where(np.isnan(b.k), b.k, 1)
    b.k[..., 1:] = np.where(np.isnan(b.k[..., 1:]), b.k[..., 1:], 0)
    scale = np.float32(top * math.log(2.0) * 1.1)
    kw = {} if split else {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda:0")}
    out, lse = b.run(scale=float(scale), **kw)
    want, want_lse, mass = lo.paged_attention(b.q, b.k, b.v, b.pages, b.q_start, b.kv_len, float(scale))
    tol = np.abs(want) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -14)
    assert (np.abs(out.astype(np.float64) - want) <= tol).all()
    assert (np.abs(lse - want_lse) <= 2.0 ** -20 * (scale + np.abs(want_lse) + 1)).all()
