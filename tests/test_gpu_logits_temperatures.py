"""process_logits at the ends of what a temperature may be."""

import numpy as np
import pytest

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


@pytest.mark.parametrize("V", [1, 7, 1000, 4095, 4096, 4100, 8191, 33001])
@pytest.mark.parametrize("count", [1, 40])
@pytest.mark.parametrize("rules", [False, True])
def test_infinite_temperatures(V, count, rules):
    """Every token is as likely as any other: the first one is chosen, the logarithm is that of their number
    (2^-19 for the sum, 2^-22 of itself)."""
    rng = np.random.default_rng(V)
    x = to_dev((rng.standard_normal((count, V)) * 3).astype(np.float16))
    kw = dict(temperature=torch.full((count,), float("inf"), device="cuda:0"))
    if rules:
        kw.update(tokens=to_dev(rng.integers(0, V, (count, 50)).astype(np.int32)), repetition=torch.full((count,), 1.5, device="cuda:0"),
                  token_count=torch.full((count,), 50, dtype=torch.int32, device="cuda:0"),
                  bias_ids=to_dev(rng.integers(0, V, (count, 3)).astype(np.int32)), bias_values=torch.ones((count, 3), device="cuda:0"))
    out, choice, lse = fasq.process_logits(x, choose=True, **kw)
    assert (to_np(out) == 0).all() and (to_np(choice) == 0).all()
    assert np.abs(to_np(lse) - np.log(V)).max() <= 2.0 ** -19 + 2.0 ** -22 * np.log(V)
    # of those that are allowed
    bits = rng.random((count, V)) < 0.4
    bits[0] = False
    words = np.zeros((count, -(-V // 32) * 32), dtype=np.uint8)
    words[:, :V] = bits
    _, choice, lse = fasq.process_logits(x, choose=True, allowed=to_dev(np.packbits(words, axis=1, bitorder="little").view(np.int32)), **kw)
    choice, lse = to_np(choice), to_np(lse)
    for r in range(count):
        if not bits[r].any():
            assert choice[r] == -1 and np.isneginf(lse[r])
        else:
            n = int(bits[r].sum())
            assert choice[r] == bits[r].argmax() and abs(lse[r] - np.log(n)) <= 2.0 ** -19 + 2.0 ** -22 * np.log(n)


@pytest.mark.parametrize("tau", [2.0 ** -127, 1e-39, 2.0 ** -149])
def test_temperatures_without_a_reciprocal(tau):
    """Below 2^-128 fp32 holds no reciprocal: a logit of zero stays zero, and all others are too large
    for fp16 (the smallest, 2^-24, becomes 2^103 at least)."""
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((3, 5000)) * 3).astype(np.float16)
    x[:, ::7] = 0
    x[0] = -np.abs(x[0])      # zeros are the largest
    x[1, 4321] = 2.0 ** -24
    x[1, :4321] = 0
    x[1, 4322:] = -1
    x[2] = np.where(x[2] > 0, -x[2], x[2])
    x[2, 4000:] = -3
    x[2, :4000] = np.where(x[2, :4000] == 0, -1, x[2, :4000])
    got = fasq.process_logits(to_dev(x), temperature=torch.full((3,), tau, dtype=torch.float32, device="cuda:0"), choose=True)
    out, choice, lse = (to_np(t) for t in got)
    with np.errstate(over="ignore", invalid="ignore"):
        assert np.array_equal(out, np.where(x == 0, 0, np.sign(x.astype(np.float32)) * np.inf).astype(np.float16))
    assert choice[0] == (x[0] == 0).argmax() and choice[1] == 4321
    assert abs(lse[0] - np.log((x[0] == 0).sum())) <= 2.0 ** -19 + 2.0 ** -22 * 9
    assert x[2, choice[2]] < 0 and not np.isnan(lse).any()
