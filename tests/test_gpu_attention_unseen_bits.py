"""What a token does not see does not reach its output: not a bit of it.

Two calls of the same shape differ in keys and values that some tokens do not see
and in the queries of the others; the results of the former must be equal bit by bit,
with caps too, whose formula depends on how large a score is.
"""

import numpy as np
import pytest

from gpu_util import to_dev
from test_gpu_attention_scores import Scored, slopes_of

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


def _same(got, want, rows):
    for x, y in zip(got, want):
        x, y = (np.ascontiguousarray(t[rows]).view(np.uint8) for t in (x, y))
        assert np.array_equal(x, y)


# Products of about a tenth of the cap, so that only what is put in passes its border of 0.6.
KINDS = [dict(softcap=20.0), dict(softcap=20.0, window=50), dict(softcap=20.0, slopes=True), dict(), dict(slopes=True)]
SHAPES = [(4, 1, 64, 20, 90), (4, 2, 128, 6, 300), (2, 1, 256, 30, 31), (4, 1, 64, 150, 300), (8, 2, 128, 70, 900), (4, 2, 192, 100, 100)]


@pytest.mark.parametrize("Hq,Hkv,D,n,kv", SHAPES)
@pytest.mark.parametrize("kw", KINDS)
@pytest.mark.parametrize("what", [900.0, -900.0, np.inf, np.nan])
def test_later_tokens(Hq, Hkv, D, n, kv, kw, what):
    b = Scored([(n, kv)], Hq, Hkv, D, 16, seed=n)
    kw = dict(kw, slopes=slopes_of(Hq) / 64) if kw.get("slopes") else kw
    want = b.run(**kw)
    m = n // 3  # tokens up to this one stay
    for j in range(kv - n + m + 1, kv):
        page, at = b.slot(0, j)
        b.k[page, at, :, 0] = what if j % 2 else -what
        b.v[page, at] = what
    b.q[m + 1:] *= 40
    _same(b.run(**kw), want, slice(0, m + 1))


@pytest.mark.parametrize("Hq,Hkv,D,n,kv", SHAPES)
@pytest.mark.parametrize("kw", KINDS)
def test_other_heads(Hq, Hkv, D, n, kv, kw):
    b = Scored([(n, kv)], Hq, Hkv, D, 16, seed=n + 1)
    kw = dict(kw, slopes=slopes_of(Hq) / 64) if kw.get("slopes") else kw
    want = b.run(**kw)
    b.q[:, 1::2] *= 60
    got = b.run(**kw)
    _same(got, want, (slice(None), slice(0, None, 2)))


@pytest.mark.parametrize("Hq,Hkv,D,n,kv", SHAPES)
@pytest.mark.parametrize("softcap", [20.0, 0.0])
@pytest.mark.parametrize("what", [900.0, np.nan])
def test_other_branches_and_runs(Hq, Hkv, D, n, kv, softcap, what):
    """Even nodes see the even ones before them, or the keys of their run."""
    b = Scored([(n, kv)], Hq, Hkv, D, 16, seed=n + 2)
    tree = np.zeros((n, -(-n // 32)), dtype=np.uint32)
    for i in range(n):
        for j in range(i % 2, i + 1, 2):
            tree[i, j // 32] |= np.uint32(1 << j % 32)
    spans = np.zeros((n, 2), dtype=np.int32)
    cut = kv // 2 + 5
    spans[0::2, 1], spans[1::2, 0], spans[1::2, 1] = cut, cut, kv
    for kw, hidden in ((dict(tree=tree.view(np.int32)), range(kv - n + 1, kv, 2)), (dict(spans=spans), range(cut, kv))):
        want = b.run(softcap=softcap, **kw)
        k, v, q = b.k.copy(), b.v.copy(), b.q.copy()
        for j in hidden:
            page, at = b.slot(0, j)
            b.k[page, at, :, 0] = what
            b.v[page, at] = what
        b.q[1::2] *= 40
        _same(b.run(softcap=softcap, **kw), want, slice(0, None, 2))
        b.k, b.v, b.q = k, v, q
