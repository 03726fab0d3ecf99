"""Scores of 2^28 powers of two and more, beside which fp32 rounds whole powers of two:
the largest one still counts, and equal ones alike, whichever way it is rounded.
Tolerances of equal scores: test_gpu_attention_small_weights.py.
"""

import math

import numpy as np
import pytest

from oracle import layer_ops as lo
from test_gpu_attention import Batch
from test_gpu_attention_scores import Scored

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


FACTORS = [1.0, 1.1, 1.27, 1.3, 1.45, 1.7, 1.9, 1.99]


@pytest.mark.parametrize("n,split", [(1, True), (3, False), (100, True), (100, False)])
@pytest.mark.parametrize("top", [28, 29, 31, 33, 40, 60])
def test_equal_scores(n, split, top):
    kv, D = 700, 64
    b = Batch([(n, kv)], 2, 1, D, 16, seed=n)
    b.q[:], b.k[:] = 1, np.where(np.isnan(b.k), b.k, 1)
    b.k[..., 1:] = np.where(np.isnan(b.k[..., 1:]), b.k[..., 1:], 0)
    kw = {} if split else {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda:0")}
    for factor in FACTORS:
        for sign in (1, -1):
            scale = float(np.float32(sign * 2.0 ** top * math.log(2.0) * factor))
            out, lse = b.run(scale=scale, **kw)
            want, want_lse, mass = lo.paged_attention(b.q, b.k, b.v, b.pages, b.q_start, b.kv_len, scale)
            tol = np.abs(want) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -14)
            assert (np.abs(out.astype(np.float64) - want) <= tol).all(), (factor, sign)
            assert (np.abs(lse - want_lse) <= 2.0 ** -20 * (abs(scale) + np.abs(want_lse) + 1)).all(), (factor, sign)


@pytest.mark.parametrize("reqs", [[(1, 300), (3, 40), (1, 1)], [(100, 500)], [(1, 9000)], [(40, 40), (150, 333)]])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (6, 2, 80), (2, 1, 256), (8, 2, 128)])
@pytest.mark.parametrize("kw", [dict(), dict(window=33), dict(spans=True)])
def test_the_largest_of_scores_far_apart(reqs, Hq, Hkv, D, kw):
    """All weight lies on one key: the output is its value.  fp32 forms a score with an error of at most
    D 2^-24 sum |q| |k|; rows whose two largest are nearer than four of that are left out.

    The weight w of that key is 2^7 only if fp32 holds its score exactly: the output is rn(rn(w) v / w), where
    each rn is fp16's, off by at most 2^-11 of its value (half a step), or 2^-25 below the smallest normal number;
    2^-20 of |v| is left to the fp32 operations between them."""
    b = Scored(reqs, Hq, Hkv, D, 16, seed=D)
    T = int(b.q_start[-1])
    spans = np.array([[i % 3, max(1, kv - n + i + 1)] for n, kv in reqs for i in range(n)], dtype=np.int32)
    seen_by = dict(kw, spans=spans) if kw.get("spans") else kw
    compared = 0
    for power in (30, 33, 37, 45, 60):
        out, lse = b.run(scale=2.0 ** power, **seen_by)
        assert not np.isnan(out).any() and not np.isnan(lse).any()
        for r, (n, kv) in enumerate(reqs):
            j = np.arange(kv)
            keys, values = (c[b.slot(r, j)].astype(np.float64) for c in (b.k, b.v))
            for i in range(n):
                t, pos = int(b.q_start[r]) + i, kv - n + i
                first = max(0, pos - 32) if "window" in kw else i % 3 if "spans" in kw else 0
                if first > pos:
                    continue
                for h in range(Hq):
                    g = h // (Hq // Hkv)
                    q = b.q[t, h].astype(np.float64)
                    s = keys[first:pos + 1, g] @ q
                    order = np.argsort(s)
                    best = order[-1]
                    near = 4 * D * 2.0 ** -24 * (np.abs(keys[first:pos + 1, g]) @ np.abs(q)).max()
                    if len(s) > 1 and s[best] - s[order[-2]] <= near:
                        continue
                    compared += 1
                    v = values[first + best, g]
                    assert (np.abs(out[t, h] - v) <= np.abs(v) * (2 * 2.0 ** -11 + 2.0 ** -20) + 2.0 ** -25).all(), (power, t, h)
                    assert abs(lse[t, h] - s[best] * 2.0 ** power) <= 2.0 ** power * near
    assert compared >= T * Hq * 4
