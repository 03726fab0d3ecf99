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
