"""paged_attention over a billion keys and more: page tables whose entries all
name the same few pages, so that the keys repeat.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
fasq = pytest.importorskip("paper_2605_04084_amd")

SIZE, D = 16, 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fasq.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _inputs(n, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    q, k, v = (torch.randn(s, generator=g, device="cuda:0").half() for s in ((n, 2, D), (2, SIZE, 1, D), (2, SIZE, 1, D)))
    return q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda:0")


def _len(kv):
    return torch.tensor([kv], dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("n", [1, 100])
def test_windows_of_more_than_2_to_the_30_keys(n):
    """The first keys, which lie before the window, are another page's and would take all the weight."""
    q, k, v, q_start = _inputs(n, 9)
    q[:] = 1
    k[1], v[1] = 1, 50
    k[0] *= 0.1
    window = 2 ** 30 + 5
    kv = window + n - 1 + 992  # 62 pages before the first token's window
    pages = torch.zeros((1, -(-kv // SIZE)), dtype=torch.int32, device="cuda:0")
    pages[0, :62] = 1
    out = fasq.paged_attention(q, k, v, pages, q_start, _len(kv), window=window, scale=1.0)
    s = k[0, :, 0].double().sum(1)
    want = torch.softmax(s, 0) @ v[0, :, 0].double()
    assert float((out.double() - want).abs().max()) <= 2.0 ** -9 * float(v[0].abs().max())
