"""process_logits where logits are finite and large: masks of -1e10 or -1e30 over
whole waves of a row (512 neighbouring logits, or two such runs), over all but one
of them and over all, and small temperatures over fp16's lowest value.

Without rules a value is the logit itself, so the choice is exact.  The logarithm:
2^-19 for the sum (see test_gpu_logits.py) and 2^-22 of itself for the roundings of
the largest value, the logarithm and their sum.  With a temperature a value takes two
roundings (the reciprocal and the product), 2^-23 of itself; one more is left to it
in the tolerance of a choice.
"""

import numpy as np
import pytest

from gpu_util import to_dev, to_np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
fasq = pytest.importorskip("paper_2605_04084_amd")

WAVE = 512


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fasq.lib()
    yield
    torch.cuda.synchronize()


def check(got, x, slack=0.0):
    """got: (rows, choice, lse) of the values x [R x V] in fp64, each off by at most ``slack`` of itself."""
    out, choice, lse = got
    top = x.max(1)
    total = top + np.log(np.exp(x - top[:, None]).sum(1))
    chosen = np.take_along_axis(x, to_np(choice)[:, None].astype(np.int64), 1)[:, 0]
    assert (chosen >= top - 2 * slack * np.abs(top)).all()
    if slack == 0:
        assert np.array_equal(to_np(choice), x.argmax(1))
    err = np.abs(to_np(lse).astype(np.float64) - total)
    assert (err <= 2.0 ** -19 + (2.0 ** -22 + slack) * np.abs(total)).all(), (err, total)
    if out is not None:
        y = to_np(out).astype(np.float64)
        assert (np.abs(y - x) <= slack * np.abs(x)).all()


def rows(V, count, mask, seed=0):
    """Rows that hold ``mask`` in one wave's logits, in those of all but one, everywhere, everywhere but in
    one place, in the last wave and in every third logit, again and again."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((count, V)) * 3).astype(np.float32)
    for r in range(count):
        kind, wave = r % 6, r // 6 % max(1, V // WAVE) * WAVE
        kept = x[r, wave:wave + WAVE].copy()
        if kind == 0:  # where a wave holds two runs, both
            x[r, wave:wave + WAVE] = mask
            x[r, wave + 8 * WAVE:wave + 9 * WAVE] = mask
        elif kind == 1:
            x[r] = mask
            x[r, wave:wave + WAVE] = kept
        elif kind == 2:
            x[r] = mask
        elif kind == 3:
            x[r] = mask
            x[r, V // 2] = kept[0]
        elif kind == 4:
            x[r, V // WAVE * WAVE:] = mask
        else:
            x[r, ::3] = mask
    return x


LARGE = [1e5, 1048575.0, 1048577.0, 1e8, 1e9, 2e9, 3e9, 5e9, 1e10, 1e12, 1e15, 1e20, 1e30, 9e37, 1.1e38, 3.4e38]


@pytest.mark.parametrize("V, count", [(700, 12), (9001, 24), (33001, 48)])  # the last one with two runs a wave
@pytest.mark.parametrize("mask", LARGE)
@pytest.mark.parametrize("sign", [-1, 1])
def test_large_logits(V, count, mask, sign):
    x = rows(V, count, np.float32(sign * mask))
    for write in (False, True):
        check(fasq.process_logits(to_dev(x), choose=True, write=write), x.astype(np.float64))


@pytest.mark.parametrize("mask", [-1e10, -1e30, 1e12])
@pytest.mark.parametrize("V, count", [(9001, 2), (33001, 34)])
def test_large_biases(V, count, mask):
    """A wave's logits made large by their biases: one rounding of the sum."""
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((count, V)) * 3).astype(np.float16)
    ids = np.tile(np.arange(2 * WAVE, 3 * WAVE), (count, 1)).astype(np.int32)
    values = np.full(ids.shape, mask, dtype=np.float32)
    got = fasq.process_logits(to_dev(x), bias_ids=to_dev(ids), bias_values=to_dev(values), choose=True, write=False)
    want = x.astype(np.float64)
    want[:, 2 * WAVE:3 * WAVE] += np.float64(np.float32(mask))
    check(got, want, 2.0 ** -24)


@pytest.mark.parametrize("tau", [1e-2, 1e-5, 1e-8, 1e-10, 1e-20, 1e-30])
@pytest.mark.parametrize("V, count", [(700, 12), (9001, 24), (33001, 48)])
def test_small_temperatures(V, count, tau):
    x = rows(V, count, np.float32(np.finfo(np.float16).min)).astype(np.float16)
    tau = np.full(count, tau, dtype=np.float32)
    out = torch.empty((count, V), dtype=torch.float32, device="cuda:0")
    got = fasq.process_logits(to_dev(x), temperature=to_dev(tau), choose=True, out=out)
    check(got, x.astype(np.float64) / tau.astype(np.float64)[:, None], 3 * 2.0 ** -24)


def test_not_a_number_beside_large_logits():
    """Only a logit that is NaN makes a row NaN, and it is the choice."""
    x = rows(9001, 12, np.float32(-1e10))
    x[3, 4711] = np.nan
    x[8, [17, 8000]] = np.nan
    _, choice, lse = fasq.process_logits(to_dev(x), choose=True)
    choice, lse = to_np(choice), to_np(lse)
    assert choice[3] == 4711 and choice[8] == 17
    assert np.array_equal(np.isnan(lse), np.isnan(x).any(1))
