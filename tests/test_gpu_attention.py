"""paged_attention against the fp64 definition.

Tolerance of an output value: half a unit in the last place of fp16 for the
result; 2^-11 of the weighted sum of |v| for weights held in fp16, and 2^-14
of it for fp32 scores (sums of at most 256 products) and sums; 2^-25 of the
largest |v| per key for weights among fp16's subnormals.  Of a logarithm of a
sum: 2^-20 of the largest sum of |q| |k| and of itself.
"""

import numpy as np
import pytest

from oracle import layer_ops as lo
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


def _half(rng, shape, std=1.0):
    return (rng.standard_normal(shape) * std).astype(np.float16)


class Batch:
    """Requests (new tokens, keys) over a cache whose unused slots hold NaN."""

    def __init__(self, reqs, Hq, Hkv, D, size, seed=0, q_std=2.0, tail_rows=0):
        rng = np.random.default_rng(seed + Hq * 31 + D + size)
        self.reqs, self.Hq, self.Hkv, self.D, self.size = reqs, Hq, Hkv, D, size
        need = [-(-kv // size) for _, kv in reqs]
        P = max(max(need), 1)
        order = rng.permutation(sum(need) + 3)
        self.pages = np.full((len(reqs), P), 2 ** 30, dtype=np.int32)  # entries that are not used
        shape = (sum(need) + 3, size, Hkv, D)
        self.k, self.v = np.full(shape, np.nan, np.float16), np.full(shape, np.nan, np.float16)
        at = 0
        for b, (n, kv) in enumerate(reqs):
            self.pages[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            j = np.arange(kv)
            self.k[self.pages[b][j // size], j % size] = _half(rng, (kv, Hkv, D))
            self.v[self.pages[b][j // size], j % size] = _half(rng, (kv, Hkv, D))
        self.q_start = np.cumsum([0] + [n for n, _ in reqs]).astype(np.int32)
        self.kv_len = np.array([kv for _, kv in reqs], dtype=np.int32)
        self.q = _half(rng, (int(self.q_start[-1]) + tail_rows, Hq, D), q_std)

    def slot(self, b, j):
        return self.pages[b][j // self.size], j % self.size

    def run(self, **kw):
        c = {k: to_dev(getattr(self, k)) for k in ("q", "k", "v", "pages", "q_start", "kv_len")}
        c.update(kw.pop("replace", {}))
        out, lse = fasq.paged_attention(c["q"], c["k"], c["v"], c["pages"], c["q_start"], c["kv_len"], return_lse=True, **kw)
        return to_np(out), to_np(lse)

    def check(self, got, scale=None, causal=True, window=0):
        scale = self.D ** -0.5 if scale is None else scale
        T = int(self.q_start[-1])
        ref, lse, mass = lo.paged_attention(self.q[:T], self.k, self.v, self.pages, self.q_start, self.kv_len, scale, causal, window)
        out, got_lse = got[0][:T].astype(np.float64), got[1][:T].astype(np.float64)
        assert np.array_equal(np.isnan(out), np.isnan(ref))
        fine = np.isfinite(ref)
        assert np.array_equal(out[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
        top_v = max([1.0] + [float(np.abs(t[np.isfinite(t)]).max()) for t in (self.v,) if np.isfinite(t).any()])
        keys = max([kv for _, kv in self.reqs] + [1])
        tol = np.abs(ref) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -14) + keys * 2.0 ** -25 * top_v
        err = np.abs(out - ref)
        bad = fine & ~(err <= tol)
        assert not bad.any(), (int(bad.sum()), float((err - tol)[fine].max()), np.argwhere(bad)[:4].tolist())
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse), empty) and (out[empty] == 0).all()
        top_k = float(np.abs(self.k[np.isfinite(self.k)]).max()) if np.isfinite(self.k).any() else 0.0
        tol = 2.0 ** -20 * (abs(scale) * np.abs(self.q[:T].astype(np.float64)).sum(2) * top_k + np.abs(np.where(empty, 0, lse)) + 1)
        fine = np.isfinite(lse)
        assert np.array_equal(np.isnan(got_lse), np.isnan(lse))
        assert (np.abs(got_lse - lse)[fine] <= tol[fine]).all()


HEADS = [(4, 1, 128), (8, 8, 64), (6, 2, 80), (7, 1, 128), (32, 1, 128), (3, 3, 96), (2, 1, 256), (4, 2, 192), (1, 1, 8), (5, 1, 72),
         (40, 1, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("size", [16, 20])
def test_decode(Hq, Hkv, D, size):
    b = Batch([(1, kv) for kv in (1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300)], Hq, Hkv, D, size)
    b.check(b.run())


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("n,kv", [(2, 2), (5, 5), (17, 40), (33, 33), (64, 100), (130, 131), (70, 333)])
def test_chunk(Hq, Hkv, D, n, kv):
    b = Batch([(n, kv)], Hq, Hkv, D, 16, seed=n)
    b.check(b.run())


@pytest.mark.parametrize("size", [1, 3, 16, 48, 64, 100, 128, 512])
@pytest.mark.parametrize("window", [0, 1, 30, 64, 150])
def test_pages_and_windows(size, window):
    b = Batch([(1, 200), (40, 170), (9, 9), (1, 64), (2, 129)], 4, 2, 64, size, seed=window)
    b.check(b.run(window=window), window=window)


@pytest.mark.parametrize("window", [0, 37])
def test_not_causal(window):
    b = Batch([(3, 100), (40, 70), (1, 1)], 4, 1, 128, 16)
    b.check(b.run(causal=False, window=window, scale=0.05), scale=0.05, causal=False, window=window)


def test_requests_without_tokens_or_keys():
    """No new tokens; no keys at all; more new tokens than keys (rows that see nothing)."""
    b = Batch([(0, 50), (1, 70), (0, 0), (3, 0), (20, 6), (0, 9), (2, 33), (0, 0)], 4, 2, 128, 16)
    got = b.run()
    b.check(got)
    assert (got[0][1:4] == 0).all() and np.isneginf(got[1][1:4]).all()
    assert (got[0][4:18] == 0).all() and np.isneginf(got[1][4:18]).all()
    got = b.run(causal=False, window=4)
    b.check(got, causal=False, window=4)


def test_tokens_of_no_request_are_left_alone():
    b = Batch([(2, 40), (1, 17)], 4, 2, 64, 16, tail_rows=5)
    out = torch.full((8, 4, 64), 7.0, dtype=torch.float16, device="cuda:0")
    got = b.run(out=out)
    b.check(got)
    assert (got[0][3:] == 7).all()


@pytest.mark.parametrize("kv", [1000, 4099, 20000])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (16, 1, 64), (2, 1, 256)])
def test_long_caches_with_few_tokens(kv, Hq, Hkv, D):
    """The keys of a row are split over workgroups and joined."""
    b = Batch([(1, kv), (3, 77), (2, kv // 3)], Hq, Hkv, D, 16, seed=kv)
    got = b.run()
    b.check(got)
    again = b.run()
    assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])
    # the same without the workspace, in one part
    b.check(b.run(workspace=torch.empty(0, dtype=torch.uint8, device="cuda:0")))


def test_long_chunk_with_split_keys():
    b = Batch([(60, 2500)], 4, 1, 128, 32)
    b.check(b.run())
    b.check(b.run(window=700), window=700)


def test_many_requests():
    rng = np.random.default_rng(4)
    reqs = [(int(rng.integers(0, 3)), int(rng.integers(0, 90))) for _ in range(300)]
    reqs[150] = (90, 400)
    b = Batch(reqs, 4, 2, 64, 16)
    b.check(b.run())


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf, 65504.0])
@pytest.mark.parametrize("n", [5, 150])
def test_what_a_token_does_not_see_does_not_reach_it(bad, n):
    """Keys and values of later tokens, and of tokens before the window."""
    kv, window = n + 100, 80
    b = Batch([(n, kv)], 4, 1, 128, 16, seed=9)
    whole = b.run(window=window)
    for j in (kv - 1, kv - n + 3, 0, 22):
        b.k[b.slot(0, j)] = bad
        b.v[b.slot(0, j)] = bad
    got = b.run(window=window)
    pos = kv - n + np.arange(n)
    clean = np.ones(n, bool)
    for j in (kv - 1, kv - n + 3, 0, 22):
        clean &= ~((j <= pos) & (j > pos - window))
    assert clean.any() and not clean.all()
    for a, c in zip(got, whole):
        assert np.array_equal(a[clean], c[clean])
    if not np.isfinite(bad):
        # where a seen value is not finite, neither is the output
        assert not np.isfinite(got[0][~clean]).any()


def test_values_that_are_not_finite_and_weighted():
    """An infinite value that a token sees makes that dimension infinite, for
    the tokens that see it only (they do not share a result)."""
    b = Batch([(70, 100)], 2, 1, 64, 16, seed=2)
    page, off = b.slot(0, 60)  # seen from token 30 on
    b.v[page, off, 0, 5] = np.inf
    b.v[page, off, 0, 9] = np.nan
    b.check(b.run())


def test_peaked_flat_and_large_scores():
    b = Batch([(1, 300), (40, 90)], 4, 2, 128, 16, q_std=60.0)  # one key takes nearly all
    b.check(b.run())
    b.check(b.run(scale=0.0), scale=0.0)  # all keys alike
    b.check(b.run(scale=-0.01), scale=-0.01)
    b.k[:] = np.where(np.isnan(b.k), b.k, 200)
    b.q[:] = 300  # scores of 7.7e6, all equal
    b.check(b.run(scale=1.0), scale=1.0)


def test_scores_rising_and_falling_along_the_cache():
    """The running maximum grows at every key, or is set by the first."""
    for sign in (1, -1):
        b = Batch([(1, 500), (20, 260)], 2, 1, 64, 16, seed=sign + 3)
        for r, (n, kv) in enumerate(b.reqs):
            j = np.arange(kv)
            b.k[b.slot(r, j)] = (sign * j / 8.0 % 128)[:, None, None].astype(np.float16)
        b.q[:] = 1
        b.check(b.run())


def test_strided_queries_outputs_and_caches():
    """q and out inside larger buffers (unaligned too), caches with the heads before the slots."""
    b = Batch([(3, 50), (1, 200), (30, 45)], 4, 2, 80, 16)
    T = len(b.q)
    ref = b.run()
    for pad in (8, 3, 1):
        q = torch.zeros((T, 6, 80 + pad), dtype=torch.float16, device="cuda:0")
        q[:, 1:5, pad:] = to_dev(b.q)
        out = torch.zeros((T, 5, 80 + pad), dtype=torch.float16, device="cuda:0")
        got = b.run(replace={"q": q[:, 1:5, pad:]}, out=out[:, :4, pad:])
        assert np.array_equal(got[0], ref[0]) and np.array_equal(got[1], ref[1])
        assert not out[:, 4].any() and not out[..., :pad].any()
    k, v = (to_dev(t).transpose(1, 2).contiguous().transpose(1, 2) for t in (b.k, b.v))
    got = b.run(replace={"k": k, "v": v})
    assert np.array_equal(got[0], ref[0])
    kv = torch.stack([to_dev(b.k), to_dev(b.v)], 1)  # [pages, 2, page_size, heads, D]
    got = b.run(replace={"k": kv[:, 0], "v": kv[:, 1]})
    assert np.array_equal(got[0], ref[0])
    wide = torch.zeros((len(b.reqs), 40), dtype=torch.int32, device="cuda:0")
    wide[:, 5:5 + b.pages.shape[1]] = to_dev(b.pages)
    got = b.run(replace={"pages": wide[:, 5:5 + b.pages.shape[1]]})
    assert np.array_equal(got[0], ref[0])


def test_pages_past_32_bits():
    H, size, D = 8, 16, 128
    b = Batch([(1, 100), (20, 40)], 8, H, D, size)
    pages = 2 ** 32 // (H * size * D) + 16
    k = torch.empty((pages, size, H, D), dtype=torch.float16, device="cuda:0")
    v = torch.empty_like(k)
    n = len(b.k)
    k[pages - n:], v[pages - n:] = to_dev(b.k), to_dev(b.v)
    ref = b.run()
    used = np.where(b.pages < n, b.pages + (pages - n), b.pages).astype(np.int32)
    got = b.run(replace={"k": k, "v": v, "pages": to_dev(used)})
    assert np.array_equal(got[0], ref[0]) and np.array_equal(got[1], ref[1])


def test_lengths_are_cut_at_the_table():
    b = Batch([(1, 64), (2, 20)], 4, 2, 64, 16)
    ref = b.run()
    b.kv_len[0] = 10 ** 6
    got = b.run()
    assert np.array_equal(got[0], ref[0])
    b.kv_len[0] = -5
    got = b.run()
    assert (got[0][0] == 0).all() and np.array_equal(got[0][1:], ref[0][1:])


def test_another_stream_and_a_graph():
    b = Batch([(1, 3000), (7, 90)], 8, 2, 128, 16)
    ref = b.run()
    c = {k: to_dev(getattr(b, k)) for k in ("q", "k", "v", "pages", "q_start", "kv_len")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = fasq.paged_attention(*c.values())
    side.synchronize()
    assert np.array_equal(to_np(out), ref[0])
    out = torch.empty_like(c["q"])
    need = fasq.paged_attention_workspace_bytes(len(b.q), 2, 8, 2, 128)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fasq.paged_attention(*c.values(), out=out, workspace=ws)
    for kv in (3000, 17, 2047):  # the lengths are read when the graph runs
        c["kv_len"][0] = kv
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.kv_len[0] = kv
        eager = fasq.paged_attention(*c.values())
        assert torch.equal(eager, out)
        b.check((to_np(out), b.run()[1]))


def test_binding_refuses():
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda:0")  # noqa: E731
    ok = dict(q=h(2, 4, 64), k_cache=h(3, 16, 2, 64), v_cache=h(3, 16, 2, 64), pages=i(2, 2), q_start=i(3), kv_len=i(2))
    for change, error in [(dict(q=h(2, 3, 64)), ValueError), (dict(q=h(2, 4, 32)), ValueError), (dict(q=h(2, 4, 64).float()), TypeError),
                          (dict(pages=i(3, 2)), ValueError), (dict(q_start=i(2)), ValueError), (dict(kv_len=i(2).long()), TypeError),
                          (dict(v_cache=h(3, 16, 1, 64)), ValueError), (dict(out=h(1, 4, 64)), ValueError), (dict(window=-1), fasq.FasqError),
                          (dict(scale=float("nan")), fasq.FasqError), (dict(kv_len=torch.zeros(2, dtype=torch.int32)), ValueError)]:
        with pytest.raises(error):
            fasq.paged_attention(**{**ok, **change})
    odd = dict(ok, q=h(2, 4, 60), k_cache=h(3, 16, 2, 60), v_cache=h(3, 16, 2, 60))
    with pytest.raises(fasq.FasqError, match="multiple of 8"):
        fasq.paged_attention(**odd)
    assert tuple(fasq.paged_attention(**dict(ok, q=h(0, 4, 64))).shape) == (0, 4, 64)
