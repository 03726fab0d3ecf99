"""paged_attention with capped scores, biases, runs of keys and trees of drafted
tokens against the fp64 definition.

Tolerance of an output value, besides that of the plain call (see
test_gpu_attention.py): a capped score is off by 2^-21 of the cap, which moves
weights and their sum by that much each, so 2^-20 c of the weighted sum of |v|; a
bias takes up to 16 roundings of 2^-24 (its parts, and the products added to it)
of itself, counted twice for the sum: 2^-19 of ``slack``.  Of the logarithm:
2^-21 c and 2^-20 of its own slack.
"""

import numpy as np
import pytest

from oracle import layer_ops as lo
from gpu_util import to_dev
from test_gpu_attention import Batch, _half

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


class Scored(Batch):
    def run(self, **kw):
        for name in ("slopes", "spans", "tree"):
            if isinstance(kw.get(name), np.ndarray):
                kw[name] = to_dev(kw[name])
        return super().run(**kw)

    def check(self, got, scale=None, softcap=0.0, **kw):
        scale = self.D ** -0.5 if scale is None else scale
        T = int(self.q_start[-1])
        with np.errstate(invalid="ignore"):
            ref, lse, mass, slack, lse_slack = lo.scored_attention(
                self.q[:T], self.k, self.v, self.pages, self.q_start, self.kv_len, scale, softcap=softcap, **kw)
        out, got_lse = got[0][:T].astype(np.float64), got[1][:T].astype(np.float64)
        assert np.array_equal(np.isnan(out), np.isnan(ref))
        fine = np.isfinite(ref)
        assert np.array_equal(out[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
        top_v = max([1.0] + [float(np.abs(t[np.isfinite(t)]).max()) for t in (self.v,) if np.isfinite(t).any()])
        keys = max([kv for _, kv in self.reqs] + [1])
        tol = (np.abs(ref) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -14 + 2.0 ** -20 * softcap)
               + keys * 2.0 ** -25 * top_v + slack * 2.0 ** -19)
        with np.errstate(invalid="ignore"):
            err = np.abs(out - ref)
        bad = fine & ~(err <= tol)
        assert not bad.any(), (int(bad.sum()), float((err - tol)[fine].max()), np.argwhere(bad)[:4].tolist())
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse), empty) and (out[empty] == 0).all()
        top_k = float(np.abs(self.k[np.isfinite(self.k)]).max()) if np.isfinite(self.k).any() else 0.0
        q_abs = np.abs(np.where(np.isfinite(self.q[:T]), self.q[:T], 0).astype(np.float64)).sum(2)
        tol = (2.0 ** -20 * (abs(scale) * q_abs * top_k + np.abs(np.where(empty, 0, lse)) + 1 + lse_slack) + 2.0 ** -21 * softcap)
        fine = np.isfinite(lse)
        assert np.array_equal(np.isnan(got_lse), np.isnan(lse))
        assert (np.abs(got_lse - lse)[fine] <= tol[fine]).all()

    def both(self, **kw):
        got = self.run(**kw)
        kw.pop("workspace", None)
        self.check(got, **kw)
        return got


MIXED = [(1, 200), (40, 170), (9, 9), (1, 64), (2, 129), (1, 1)]
HEADS = [(4, 1, 128), (8, 8, 64), (6, 2, 80), (7, 1, 128), (2, 1, 256), (4, 2, 192), (1, 1, 8)]


def slopes_of(Hq):
    return (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)


def random_tree(rng, n):
    parents = [-1] + [int(rng.integers(-1 if i % 7 == 0 else max(0, i - 5), i)) for i in range(1, n)]
    return parents


def trees_of(rng, reqs):
    tree, _ = fasq.draft_tree([random_tree(rng, n) for n, _ in reqs if n > 0], device="cpu")
    return tree.numpy()


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("kw", [dict(softcap=1.5), dict(softcap=50.0, window=37), dict(slopes=True), dict(slopes=True, softcap=20.0),
                                dict(softcap=1024.0, causal=False), dict(slopes=True, causal=False, window=60)])
def test_scores(Hq, Hkv, D, kw):
    b = Scored(MIXED, Hq, Hkv, D, 16 if D < 100 else 20, seed=D)
    kw = dict(kw, slopes=slopes_of(Hq)) if kw.get("slopes") else kw
    b.both(**kw)
    b.both(**kw, workspace=torch.empty(0, dtype=torch.uint8, device="cuda:0"))


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("n,kv", [(2, 2), (33, 33), (64, 100), (130, 131), (70, 333)])
@pytest.mark.parametrize("kw", [dict(softcap=3.0), dict(slopes=True), dict(slopes=True, softcap=8.0)])
def test_chunks(Hq, Hkv, D, n, kv, kw):
    b = Scored([(n, kv)], Hq, Hkv, D, 16, seed=n)
    b.both(**(dict(kw, slopes=slopes_of(Hq)) if kw.get("slopes") else kw))


@pytest.mark.parametrize("softcap", [0.0, 5.0])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_spans(Hq, Hkv, D, softcap):
    """Any runs: some empty, some past the keys or before them, some in another order than the tokens."""
    rng = np.random.default_rng(Hq + D)
    for reqs in (MIXED, [(150, 300)], [(5, 700), (3, 40)], [(1, 3000), (1, 90)]):
        b = Scored(reqs, Hq, Hkv, D, 16, seed=len(reqs))
        spans = np.zeros((int(b.q_start[-1]), 2), dtype=np.int32)
        for r, (n, kv) in enumerate(reqs):
            for t in range(int(b.q_start[r]), int(b.q_start[r + 1])):
                begin = int(rng.integers(-20, kv))
                spans[t] = begin, begin + int(rng.integers(-3, kv + 20))
        spans[0] = -2 ** 31, 2 ** 31 - 1
        b.both(spans=spans, softcap=softcap)
        if not softcap:
            b.both(spans=spans, slopes=slopes_of(Hq))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_documents_and_prefixes(D):
    n, G = 400, 4
    b = Scored([(n, n), (30, 90)], G, 1, D, 64, seed=3)
    spans = np.zeros((n + 30, 2), dtype=np.int32)
    for begin, end in ((0, 1), (1, 34), (34, 260), (260, 400)):
        for t in range(begin, end):
            spans[t] = begin, max(t + 1, min(begin + 20, end))
    for i in range(30):
        spans[n + i] = 5, 61 + i
    b.both(spans=spans)


def test_far_spans_keep_their_biases():
    """A token far from all keys it sees: only the differences of their biases count."""
    kv = 70000
    b = Scored([(1, kv), (40, kv)], 2, 1, 64, 64, seed=5)
    spans = np.zeros((41, 2), dtype=np.int32)
    spans[:, 0], spans[:, 1] = 100, 400 + np.arange(41)
    slopes = np.array([1.0, 0.03], dtype=np.float32)
    b.both(spans=spans, slopes=slopes)
    spans[:, 0], spans[:, 1] = kv - 1, kv  # one key, its neighbour or itself
    b.both(spans=spans, slopes=-slopes)


@pytest.mark.parametrize("softcap", [0.0, 4.0])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("reqs", [[(1, 1)], [(13, 200)], [(32, 32)], [(33, 40), (64, 500), (7, 7), (1, 90)], [(100, 1000)], [(64, 3)]])
def test_tree(Hq, Hkv, D, reqs, softcap):
    b = Scored(reqs, Hq, Hkv, D, 16, seed=len(reqs))
    b.both(tree=trees_of(np.random.default_rng(D), reqs), softcap=softcap)


def test_tree_of_long_caches():
    """The keys of a tile are split over workgroups."""
    reqs = [(50, 20011), (5, 4099), (3, 17)]
    b = Scored(reqs, 8, 2, 128, 16, seed=1)
    tree = trees_of(np.random.default_rng(1), reqs)
    got, again = b.both(tree=tree), b.run(tree=tree)
    assert np.array_equal(got[0], again[0]) and np.array_equal(got[1], again[1])
    b.both(tree=tree, workspace=torch.empty(0, dtype=torch.uint8, device="cuda:0"))


@pytest.mark.parametrize("reqs", [[(40, 40)], [(20, 20), (3, 90)], [(6, 200), (70, 75)]])
def test_words_of_any_kind(reqs):
    """Rows without a bit, bits past the last token, fewer words than tokens, runs beside the tree."""
    rng = np.random.default_rng(7)
    b = Scored(reqs, 4, 2, 64, 16, seed=2)
    T = int(b.q_start[-1])
    words = rng.integers(-2 ** 31, 2 ** 31, (T, 2)).astype(np.int32)
    words[0] = 0
    words[T // 2] = 0
    words[1] = -1
    b.both(tree=words)
    b.both(tree=words[:, :1].copy())
    spans = np.zeros((T, 2), dtype=np.int32)
    for r, (n, kv) in enumerate(reqs):
        for t in range(int(b.q_start[r]), int(b.q_start[r + 1])):
            spans[t] = rng.integers(0, kv), kv - rng.integers(0, 3)
    b.both(tree=words, spans=spans, softcap=6.0)
    wide = np.zeros((T, 5), dtype=np.int32)  # rows with a stride
    wide[:, 1:3] = words
    got = b.run(tree=to_dev(wide)[:, 1:3])
    assert all(np.array_equal(x, y) for x, y in zip(got, b.run(tree=words)))


@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("kw", [dict(softcap=7.0), dict(slopes=True), dict(), dict(slopes=True, softcap=9.0)])
def test_unseen_keys_and_values_do_not_matter(what, kw):
    """What other branches of a tree, other documents and later tokens hold."""
    rng = np.random.default_rng(11)
    reqs = [(36, 80), (5, 300)]
    kw = dict(kw, slopes=slopes_of(4)) if kw.get("slopes") else dict(kw)
    b = Scored(reqs, 4, 2, 64, 16, seed=4)
    T = int(b.q_start[-1])
    spans = np.zeros((T, 2), dtype=np.int32)
    for r, (n, kv) in enumerate(reqs):
        for i, t in enumerate(range(int(b.q_start[r]), int(b.q_start[r + 1]))):
            spans[t] = 3 * (i % 4), kv - n + i + 1
    if "slopes" not in kw:
        kw["tree"] = trees_of(rng, reqs)
    for r, j in ((0, 44 + 17), (0, 79), (1, 299), (0, 4), (1, 1), (1, 150)):
        page, at = b.slot(r, j)
        b.k[page, at] = what
        b.v[page, at] = -what
    b.both(spans=spans, **kw)
    # keys alone: a score of any size is a score of the cap's size
    b2 = Scored([(3, 50)], 4, 2, 64, 16, seed=4)
    page, at = b2.slot(0, 7)
    b2.k[page, at] = what
    b2.both(softcap=5.0)


def test_saturated_scores():
    """Products far past the cap, on both sides, and rows whose scores are all at its lower end."""
    b = Scored([(4, 60), (35, 90)], 4, 2, 64, 16, seed=6, q_std=300.0)
    b.both(softcap=2.0)
    b.both(softcap=200.0)
    b.k[...] = np.where(np.isfinite(b.k), np.abs(b.k), b.k)
    b.q[...] = -np.abs(b.q)
    b.both(softcap=700.0)
    b.both(softcap=700.0, scale=-0.125)


def test_plain_calls_through_the_extended_entry():
    """No field set: the bits of the plain entry point; a span or tree that says what causality says: its values."""
    reqs = [(3, 100), (40, 70), (1, 33)]
    b = Scored(reqs, 4, 2, 128, 16, seed=8)
    spans = np.array([[0, kv - n + i + 1] for n, kv in reqs for i in range(n)], dtype=np.int32)
    plain = b.run()
    for kw in (dict(spans=spans), dict(tree=np.array([[(1 << i + 1) - 1 & 0xFFFFFFFF, (1 << i + 1) - 1 >> 32] for n, _ in reqs
                                                      for i in range(n)], dtype=np.int64).astype(np.uint32).view(np.int32))):
        got = b.both(**kw)
        assert np.allclose(got[0].astype(np.float32), plain[0].astype(np.float32), atol=2e-3)


def test_rows_of_no_request_are_left_alone():
    b = Scored([(2, 40), (1, 17)], 4, 2, 64, 16, tail_rows=5)
    out = torch.full((8, 4, 64), 7.0, dtype=torch.float16, device="cuda:0")
    tree = np.full((8, 1), 3, dtype=np.int32)
    got = b.run(out=out, tree=tree, softcap=3.0)
    b.check(got, tree=tree, softcap=3.0)
    assert (got[0][3:] == 7).all()


def test_tensors_are_checked():
    b = Scored([(2, 40)], 4, 2, 64, 16)
    f32, i32 = dict(dtype=torch.float32, device="cuda:0"), dict(dtype=torch.int32, device="cuda:0")
    for kw in (dict(slopes=torch.zeros(3, **f32)), dict(slopes=torch.zeros(4, **i32)), dict(spans=torch.zeros((2, 3), **i32)),
               dict(spans=torch.zeros((3, 2), **i32)), dict(spans=torch.zeros((2, 2), dtype=torch.int64, device="cuda:0")),
               dict(tree=torch.zeros((2, 0), **i32)), dict(tree=torch.zeros((1, 1), **i32)), dict(tree=torch.zeros((2, 1), dtype=torch.int32)),
               dict(tree=torch.zeros((2, 4), **i32)[:, ::2])):
        with pytest.raises((TypeError, ValueError)):
            b.run(**kw)
    for kw in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=1e-5), dict(softcap=3000.0),
               dict(slopes=torch.zeros(4, **f32), tree=torch.zeros((2, 1), **i32)), dict(spans=torch.zeros((2, 2), **i32), window=3),
               dict(tree=torch.zeros((2, 1), **i32), window=3), dict(slopes=torch.zeros(4, **f32), scale=0.0)):
        with pytest.raises(fasq.FasqError):
            b.run(**kw)


@pytest.mark.parametrize("reqs", [[(64, 5000), (64, 3333)], [(40, 7000), (70, 2000), (33, 6001), (0, 50)], [(100, 9000)], [(50, 64), (200, 4100), (3, 20)]])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (4, 1, 64), (3, 1, 80)])
def test_trees_of_several_tiles_over_long_caches(reqs, Hq, Hkv, D):
    """One to seven tiles a request, their keys split over workgroups, even and odd numbers of them."""
    b = Scored(reqs, Hq, Hkv, D, 64, seed=9)
    b.both(tree=trees_of(np.random.default_rng(9), reqs))
    b.both(softcap=20.0)


@pytest.mark.parametrize("reqs", [[(20, 3000), (32, 2500), (9, 700)], [(200, 6000)], [(33, 4000), (64, 300)], [(1, 9000)], [(24, 30)]])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (5, 1, 64)])
def test_trees_in_windows(reqs, Hq, Hkv, D):
    """Each node sees a window before its own depth: short runs of long caches."""
    b = Scored(reqs, Hq, Hkv, D, 16, seed=21)
    rng = np.random.default_rng(21)
    tree, depth = fasq.draft_tree([random_tree(rng, n) for n, _ in reqs], device="cpu")
    start = np.repeat([kv - n for n, kv in reqs], [n for n, _ in reqs])
    spans = np.stack([np.maximum(0, start + depth.numpy() - 99), np.repeat([kv for _, kv in reqs], [n for n, _ in reqs])], 1).astype(np.int32)
    b.both(tree=tree.numpy(), spans=spans)
    b.both(tree=tree.numpy(), spans=spans, workspace=torch.empty(0, dtype=torch.uint8, device="cuda:0"))


@pytest.mark.parametrize("n", [63, 65, 300, 1000, 2030, 4096, 4097])
@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (3, 1, 80), (7, 1, 128)])
def test_one_request_of_many_runs(n, Hq, Hkv, D):
    """Shares by the longest run of a tile: documents, a long run among short ones at any place, runs of nothing."""
    rng = np.random.default_rng(n + Hq)
    b = Scored([(n, n)], Hq, Hkv, D, 20, seed=n)
    ends = np.unique(np.append(rng.integers(1, n, 7), n))
    spans = np.zeros((n, 2), dtype=np.int32)
    begin = 0
    for end in ends:
        spans[begin:end, 0] = begin
        spans[begin:end, 1] = np.maximum(np.arange(begin, end) + 1, min(begin + 9, end))
        begin = end
    b.both(spans=spans)
    short = np.stack([np.maximum(0, np.arange(n) - 5), np.arange(n) + 1], 1).astype(np.int32)
    for at in (0, n // 2, n - 1):
        spans = short.copy()
        spans[at] = 0, n
        b.both(spans=spans)
    spans[:] = 7, 7
    spans[n // 3] = n - 40, n
    b.both(spans=spans)
