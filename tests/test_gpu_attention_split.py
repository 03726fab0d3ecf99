"""paged_attention where keys are split over workgroups and joined: batches
whose shares begin and end at every kind of border.  Tolerances are those of
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


@pytest.mark.parametrize("size", [16, 20, 7])
@pytest.mark.parametrize("Hq,Hkv,D", [(2, 1, 256), (4, 1, 80), (8, 2, 128), (3, 3, 64)])
def test_chunk_over_a_long_cache(size, Hq, Hkv, D):
    b = Batch([(150, 3100), (1, 700), (65, 65)], Hq, Hkv, D, size, seed=size)
    b.check(b.run())
    b.check(b.run(window=900), window=900)


@pytest.mark.parametrize("D", [64, 128])
def test_more_requests_than_lanes(D):
    rng = np.random.default_rng(D)
    reqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 90))) for _ in range(70)]
    reqs[3], reqs[40], reqs[66] = (1, 6000), (1, 2500), (2, 3333)
    b = Batch(reqs, 4, 2, D, 16)
    b.check(b.run())


def test_more_requests_than_lanes_with_chunks():
    rng = np.random.default_rng(9)
    reqs = [(int(rng.integers(0, 4)), int(rng.integers(4, 60))) for _ in range(70)]
    reqs[10], reqs[69] = (1300, 1400), (1400, 4000)
    b = Batch(reqs, 2, 2, 64, 16)
    b.check(b.run())


@pytest.mark.parametrize("reqs", [[(1, 40)] * 3, [(2, 900), (2, 1200)], [(140, 2100)], [(300, 400), (5, 5)]])
def test_with_and_without_workspace(reqs):
    """Both forms, and a dirty workspace."""
    b = Batch(reqs, 8, 2, 64, 16)
    T, B = int(b.q_start[-1]), len(reqs)
    need = fasq.paged_attention_workspace_bytes(T, B, 8, 2, 64)
    first = b.run(workspace=torch.full((need,), 0xff, dtype=torch.uint8, device="cuda:0"))
    b.check(first)
    b.check(b.run(workspace=torch.empty(0, dtype=torch.uint8, device="cuda:0")))
    again = b.run(workspace=torch.full((need + 32,), 0x7b, dtype=torch.uint8, device="cuda:0"))
    assert np.array_equal(first[0].view(np.uint16), again[0].view(np.uint16)) and np.array_equal(first[1], again[1])


def test_lengths_that_end_on_a_share():
    """Every length around a multiple of the steps: shares end with tiles."""
    for kv in range(500, 1700, 37):
        b = Batch([(1, kv), (1, 512), (1, 1024 - kv % 256)], 4, 4, 64, 16, seed=kv)
        b.check(b.run())


@pytest.mark.parametrize("n,kv,Hq,Hkv,D", [(1024, 1024, 8, 8, 128), (1024, 1500, 16, 8, 64), (16, 4000, 8, 2, 128),
                                           (17, 4000, 8, 2, 128), (64, 700, 2, 2, 256), (65, 700, 2, 2, 256)])
def test_around_the_choices_of_tiles(n, kv, Hq, Hkv, D):
    """Whole tiles that just fill the chip or do not, and tiles of 32 and of 128 rows."""
    b = Batch([(n, kv)], Hq, Hkv, D, 16, seed=n)
    b.check(b.run())


@pytest.mark.parametrize("n,kv,B,window,D", [(300, 300, 1, 0, 128), (500, 2000, 1, 100, 64), (200, 900, 4, 33, 96),
                                             (150, 150, 1, 0, 256), (700, 1000, 1, 200, 256)])
def test_short_tiles_stay_whole(n, kv, B, window, D):
    b = Batch([(n, kv)] * B, 4, 2, D, 16, seed=n)
    b.check(b.run(window=window), window=window)
