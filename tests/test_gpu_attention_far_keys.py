"""paged_attention over a billion keys and more: page tables whose entries all
name the same few pages, so that the keys repeat.
"""

import math

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


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 20, 200])
def test_windows_at_the_largest_length(n, causal, split):
    """The last keys there can be, as a short cache has them."""
    q, k, v, q_start = _inputs(n, n)
    kw = dict(window=100, causal=causal, return_lse=True)
    if not split:
        kw["workspace"] = torch.empty(0, dtype=torch.uint8, device="cuda:0")
    kv = 2 ** 31 - 1024
    pages = torch.zeros((1, kv // SIZE), dtype=torch.int32, device="cuda:0")
    far = fasq.paged_attention(q, k, v, pages, q_start, _len(kv), **kw)
    near = fasq.paged_attention(q, k, v, pages[:, :100], q_start, _len(1600), **kw)
    assert all(torch.equal(a, b) for a, b in zip(far, near))


def test_all_keys_of_the_largest_length():
    q, k, v, q_start = _inputs(1, 5)
    kv = 2 ** 31 - 1024
    pages = torch.zeros((1, kv // SIZE), dtype=torch.int32, device="cuda:0")
    out, lse = fasq.paged_attention(q, k, v, pages, q_start, _len(kv), return_lse=True)
    near, near_lse = fasq.paged_attention(q, k, v, pages[:, :1], q_start, _len(SIZE), return_lse=True)
    # weights in fp16 (2^-11 of |v| on each side); 2^31 keys over 2^10 waves, 16 a
    # product: 2^17 additions in fp32 in turn, 2^-24 each
    assert float((out - near).abs().max()) <= (2.0 ** -7 + 2.0 ** -9) * float(v.abs().max())
    assert float((lse - near_lse - math.log(kv // SIZE)).abs().max()) <= 2.0 ** -10


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


@pytest.mark.parametrize("n", [1, 20, 200])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=3.0), dict(slopes=True)])
def test_runs_and_trees_at_the_largest_length(n, kw):
    """Runs of keys at the end of the longest cache, as a short cache has them; the
    keys may be split elsewhere, so up to a rounding of the weights and one of the result on each side."""
    q, k, v, q_start = _inputs(n, n)
    kw = dict(kw, slopes=torch.tensor([0.5, 0.01], device="cuda:0")) if kw.get("slopes") else dict(kw)
    far_kv, near_kv = 2 ** 31 - 1024, 1600
    pages = torch.zeros((1, far_kv // SIZE), dtype=torch.int32, device="cuda:0")
    i = torch.arange(n, device="cuda:0")
    if "slopes" not in kw:
        kw["tree"] = torch.randint(-2 ** 31, 2 ** 31, (n, 7), device="cuda:0").int()

    def run(kv):
        spans = torch.stack([kv - n + i - 300, kv - n + i + 1], 1).int()
        return fasq.paged_attention(q, k, v, pages[:, :kv // SIZE], q_start, _len(kv), spans=spans, return_lse=True, **kw)

    far, near = run(far_kv), run(near_kv)
    assert float((far[0] - near[0]).abs().max()) <= 4 * 2.0 ** -11 * float(v.abs().max())
    assert float((far[1] - near[1]).abs().max()) <= 2.0 ** -12


def test_a_tree_over_the_largest_length():
    """All keys before the tree are alike, so each node's result is theirs."""
    q, k, v, q_start = _inputs(3, 5)
    kv = 2 ** 31 - 1024
    pages = torch.zeros((1, kv // SIZE), dtype=torch.int32, device="cuda:0")
    tree = torch.tensor([[1], [3], [4]], dtype=torch.int32, device="cuda:0")
    out = fasq.paged_attention(q, k, v, pages, q_start, _len(kv), tree=tree)
    near = fasq.paged_attention(q, k, v, pages[:, :1], q_start, _len(SIZE), causal=False)
    assert float((out - near).abs().max()) <= (2.0 ** -7 + 2.0 ** -9) * float(v.abs().max())  # as above
