"""paged_attention where the keys that a tile's tokens see lie unusually:
windows without causality, whose later keys every token sees.  Tolerances are those of
test_gpu_attention.
"""

import numpy as np
import pytest

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


def _none():
    return torch.empty(0, dtype=torch.uint8, device="cuda:0")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("reqs,Hq,Hkv,window", [
    ([(150, 3100)], 4, 1, 100),                    # tiles of 128 rows
    ([(300, 300)], 4, 1, 16),                      # far more tokens than the window holds
    ([(64, 1000)], 1, 1, 64),                      # tiles of 32 rows
    ([(8, 500)], 8, 1, 1),
    ([(300, 300), (200, 900), (1, 50)], 4, 2, 16),
    ([(20, 700), (30, 31), (9, 4000), (0, 10)], 1, 1, 3),
    ([(130, 1300)] * 3, 3, 1, 33),                 # requests of one length
])
def test_windows_without_causality(reqs, Hq, Hkv, window, D):
    b = Batch(reqs, Hq, Hkv, D, 16, seed=window)
    b.check(b.run(causal=False, window=window), causal=False, window=window)
    b.check(b.run(causal=False, window=window, workspace=_none()), causal=False, window=window)


def test_windows_without_causality_and_more_tokens_than_keys():
    b = Batch([(400, 90), (90, 400), (33, 0)], 2, 1, 64, 20)
    b.check(b.run(causal=False, window=25), causal=False, window=25)


def test_no_requests():
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for pages in (i(0, 3), i(0, 0)):
        out, lse = fasq.paged_attention(h(0, 4, 64), h(3, 16, 2, 64), h(3, 16, 2, 64), pages, i(1), i(0), return_lse=True)
        assert tuple(out.shape) == (0, 4, 64) and tuple(lse.shape) == (0, 4)
    assert tuple(fasq.paged_attention(h(0, 4, 64), h(3, 16, 2, 64), h(3, 16, 2, 64), i(2, 0), i(3), i(2)).shape) == (0, 4, 64)
