"""Workspaces that calls allocate while a launch list records: they are the
list's until nothing uses them, and one serves all of a list's calls.
"""

import numpy as np
import pytest

import pq_inputs as pi
from gpu_util import to_dev

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


def _matmul(M, K, N, d, C, per_subspace=False):
    rng = np.random.default_rng(M + N)
    S = K // d
    books = np.stack([pi.draw_codebook(rng, C, d) for _ in range(S if per_subspace else 1)])
    idx = pi.pack_indices(pi.draw_ids(rng, N, S, C), 8)
    return to_dev(pi.draw_x(rng, M, K)), to_dev(idx), to_dev(books if per_subspace else books[0])


def _gemv_ex():
    x, idx, books = _matmul(3, 4096, 1000, 2, 256, True)
    out = torch.zeros((3, 1000), dtype=torch.float16, device="cuda:0")
    return lambda: [fasq.pq_gemv_ex(x, idx, 8, 2, books, out=out)], fasq.gemv_ex_workspace_bytes(3, 4096, 1000, 8, 2, 256, 512)


def _gemm_ex():
    x, idx, book = _matmul(128, 4096, 4096, 4, 256)
    out = torch.zeros((128, 4096), dtype=torch.float16, device="cuda:0")
    return lambda: [fasq.pq_gemm_ex(x, idx, 8, 4, book, out=out)], fasq.gemm_ex_workspace_bytes(128, 4096, 4096, 8, 4, 256)


def _encode():
    rng = np.random.default_rng(5)
    w, first = pi.draw_weights(rng, 256, 512), pi.draw_codebook(rng, 256, 4)
    w, first = to_dev(w), to_dev(first)
    return lambda: list(fasq.pq_encode(w, 4, 8, first, 3)), fasq.encode_workspace_bytes(256, 512, 4, 256)


def _attention():
    q = torch.randn((300, 4, 128), device="cuda:0").half()
    k, v = (torch.randn((60, 16, 2, 128), device="cuda:0").half() for _ in range(2))
    pages = torch.arange(60, dtype=torch.int32, device="cuda:0").view(1, 60)
    lens = [torch.tensor(a, dtype=torch.int32, device="cuda:0") for a in ([0, 300], [900])]
    out = torch.zeros_like(q)
    return lambda: [fasq.paged_attention(q, k, v, pages, *lens, out=out)], fasq.paged_attention_workspace_bytes(300, 1, 4, 2, 128)


MAKE = {"gemv_ex": _gemv_ex, "gemm_ex": _gemm_ex, "encode": _encode, "attention": _attention}


def _record(name):
    """The list, its outputs, what they should be, the workspace's bytes, and what holds the inputs."""
    call, need = MAKE[name]()
    assert need > 0
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    lst = fasq.LaunchList()
    with lst:
        outs = call()
    for t in outs:
        t.zero_()
    return lst, outs, want, need, call


@pytest.mark.parametrize("name", MAKE)
def test_no_other_tensor_takes_its_place(name):
    lst, outs, want, need, inputs = _record(name)
    others = [torch.full((need,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(4)]
    for _ in range(2):
        lst.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert all(bool((t == 255).all()) for t in others)
    lst.close()


def test_closed_while_a_run_waits_on_the_null_stream():
    """Recorded on a side stream, run on the null stream, whose handle is 0."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lst, outs, want, need, inputs = _record("attention")
    torch.cuda.current_stream().wait_stream(side)
    big = torch.randn(8192, 8192, device="cuda:0")
    for _ in range(4):
        big = big @ big
    lst.run(0)
    lst.close()
    with torch.cuda.stream(side):
        others = [torch.full((need,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert all(bool((t == 255).all()) for t in others)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", MAKE)
def test_closed_while_a_run_waits_on_another_stream(name, raw):
    """The workspace is nobody else's before the runs that were queued are over."""
    lst, outs, want, need, inputs = _record(name)
    big = torch.randn(8192, 8192, device="cuda:0")
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        for _ in range(4):
            big = big @ big  # some milliseconds
    lst.run(other.cuda_stream if raw else other)
    lst.close()
    others = [torch.full((need,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert all(bool((t == 255).all()) for t in others)


def _requested():
    """Bytes of all tensors as they were asked for (the allocator hands out whole blocks)."""
    return torch.cuda.memory_stats()["requested_bytes.all.current"]


def test_one_workspace_serves_a_list():
    """Launches of a list run one after another, so its calls share the largest."""
    call, need = _attention()
    small, small_need = _gemv_ex()
    want, want_small = (f()[0].clone() for f in (call, small))
    torch.cuda.synchronize()
    before = _requested()
    lst = fasq.LaunchList()
    with lst:
        for _ in range(8):
            out, = small()
            big, = call()
    assert _requested() - before <= need + small_need + 8192
    out.zero_()
    big.zero_()
    lst.run()
    torch.cuda.synchronize()
    assert torch.equal(big, want) and torch.equal(out, want_small)
    lst.close()
    assert _requested() <= before
