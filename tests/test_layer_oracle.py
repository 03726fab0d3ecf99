"""Pins of the fp64 definitions in ``oracle/layer_ops.py`` against closed forms,
pure-Python loops and invariants; and the rotary frequencies of the binding."""

import math

import numpy as np
import pytest

import paper_2605_04084_amd as fasq
from oracle import layer_ops as lo


def test_rope_turns_a_pair_by_its_angle():
    w = [1.0, 0.25]
    table = lo.rope_table(w, 8)
    x = np.array([[[1.0, 0.0, 0.0, 2.0]]])
    # half layout: pairs (0, 2) and (1, 3)
    y = lo.rope(x, table, [3], False)[0, 0]
    assert y == pytest.approx([math.cos(3), -2 * math.sin(0.75), math.sin(3), 2 * math.cos(0.75)], abs=1e-12)
    # interleaved: pairs (0, 1) and (2, 3)
    y = lo.rope(x, table, [3], True)[0, 0]
    assert y == pytest.approx([math.cos(3), math.sin(3), -2 * math.sin(0.75), 2 * math.cos(0.75)], abs=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_scores_depend_on_the_distance_only(interleaved):
    rng = np.random.default_rng(0)
    table = lo.rope_table([10000 ** (-2 * i / 12) for i in range(6)], 64)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    dot = lambda p, r: float((lo.rope(q, table, [p], interleaved) * lo.rope(k, table, [r], interleaved)).sum())  # noqa: E731
    assert dot(5, 2) == pytest.approx(dot(43, 40), rel=1e-12)
    assert dot(0, 0) == pytest.approx(float((q * k).sum()), rel=1e-12)
    assert dot(5, 2) != pytest.approx(dot(5, 3), rel=1e-6)


def test_rope_norm_and_tail_and_outside():
    x = np.array([[[3.0, 4.0, 5.0]]])
    y = lo.rope(x, lo.rope_table([1.0], 2), [0], False, norm=[1.0, 2.0, 0.5], eps=1e-6)
    r = math.sqrt(50 / 3 + 1e-6)
    assert y[0, 0] == pytest.approx([3 / r, 8 / r, 2.5 / r], rel=1e-12)
    assert np.isnan(lo.rope(x, lo.rope_table([1.0], 2), [2], False)).all()


def test_append_leaves_other_slots_and_skips_padding():
    cache = np.zeros((3, 2, 1, 1))
    out = lo.append(cache, np.array([[[7.0]], [[8.0]], [[9.0]]]), [5, -1, 6])
    assert out[2, 1, 0, 0] == 7.0 and np.count_nonzero(out) == 1


def _py_attention(q, keys, values, scale, begin, end):
    s = [scale * math.fsum(a * b for a, b in zip(q, k)) for k in keys[begin:end]]
    e = [math.exp(v) for v in s]
    out = [math.fsum(w * v[d] for w, v in zip(e, values[begin:end])) / math.fsum(e) for d in range(len(q))]
    return out, math.log(math.fsum(e))


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 2)])
def test_attention_against_python_loops(causal, window):
    rng = np.random.default_rng(1)
    Hq, Hkv, D, size = 4, 2, 3, 4
    k_cache, v_cache = rng.standard_normal((9, size, Hkv, D)), rng.standard_normal((9, size, Hkv, D))
    pages = np.array([[3, 1, 7], [8, 0, 2]])
    q_start, kv_len = [0, 3, 4], [9, 2]
    q = rng.standard_normal((4, Hq, D))
    out, lse, _ = lo.paged_attention(q, k_cache, v_cache, pages, q_start, kv_len, 0.7, causal, window)
    for b, (n, kv) in enumerate([(3, 9), (1, 2)]):
        for i in range(n):
            pos = kv - n + i
            begin = max(0, pos - window + 1) if window else 0
            end = pos + 1 if causal else kv
            for h in range(Hq):
                keys = [k_cache[pages[b][j // size], j % size, h // 2].tolist() for j in range(kv)]
                values = [v_cache[pages[b][j // size], j % size, h // 2].tolist() for j in range(kv)]
                o, z = _py_attention(q[q_start[b] + i, h].tolist(), keys, values, 0.7, begin, end)
                assert out[q_start[b] + i, h] == pytest.approx(o, rel=1e-12)
                assert lse[q_start[b] + i, h] == pytest.approx(z, rel=1e-12)


def test_attention_empty_rows_and_masked_nan():
    k = np.ones((2, 4, 1, 2))
    v = np.arange(16.0).reshape(2, 4, 1, 2)
    k[1, 2:], v[1, 2:] = np.nan, np.nan  # past the length
    v[1, 1] = np.nan                     # seen by the last token only
    q = np.ones((7, 1, 2))
    # 7 new tokens, 6 keys in all: the first token sees nothing
    out, lse, _ = lo.paged_attention(q, k, v, np.array([[0, 1]]), [0, 7], [6], 1.0)
    assert (out[0] == 0).all() and lse[0, 0] == -np.inf
    assert out[1, 0].tolist() == [0.0, 1.0] and out[3, 0].tolist() == [2.0, 3.0]
    assert np.isnan(out[6]).all() and np.isfinite(out[:6]).all()


def test_residual_norm_closed_form():
    x_new, h = lo.residual_norm([[1.0, 1.0]], [[3.0, 4.0]], [1.0, 2.0], 1e-9, post_weight=[1.0, 1.0], gate=[2.0, 0.0],
                                scale=0.5)
    a = 1 + 3 / math.sqrt(12.5)
    assert x_new[0] == pytest.approx([a, 1.0], rel=1e-8)
    r = math.sqrt((a * a + 1) / 2)
    assert h[0] == pytest.approx([a / r, 2 / r], rel=1e-8)
    x_new, h = lo.residual_norm([[2.0, 0.0]])
    assert h is None and x_new[0].tolist() == [2.0, 0.0]


def test_lora_is_a_dense_update_of_the_weights():
    rng = np.random.default_rng(2)
    x, W = rng.standard_normal((3, 5)), rng.standard_normal((4, 5))
    A, B = rng.standard_normal((2, 2, 5)), rng.standard_normal((2, 4, 2))
    y, _ = lo.lora(x, [1, -1, 0], A, B, [0.5, 3.0], x @ W.T)
    for m, (a, s) in enumerate([(1, 3.0), (0, 0.0), (0, 0.5)]):
        assert y[m] == pytest.approx((W + s * B[a] @ A[a]) @ x[m], rel=1e-12)
    y, _ = lo.lora(x, [2, 1, 0], A, B, [0.5, 3.0])
    assert (y[0] == 0).all()  # outside the pool, no base


# ---------------------------------------------------------------------------
# rope_frequencies
# ---------------------------------------------------------------------------

def test_frequencies_unscaled_and_linear():
    w, s = fasq.rope_frequencies(8, base=10000.0)
    assert w == pytest.approx([1.0, 0.1, 0.01, 0.001]) and s == 1.0
    w, s = fasq.rope_frequencies(8, base=10000.0, scaling="linear", factor=4.0)
    assert w == pytest.approx([0.25, 0.025, 0.0025, 0.00025]) and s == 1.0


def test_frequencies_ntk_slows_the_slowest_pair_by_the_factor():
    w0, _ = fasq.rope_frequencies(64)
    w, _ = fasq.rope_frequencies(64, scaling="ntk", factor=8.0)
    assert w[0] == w0[0] and w[-1] == pytest.approx(w0[-1] / 8)
    assert all(a > b for a, b in zip(w, w[1:]))


def test_frequencies_wavelength_keeps_fast_and_slows_slow_pairs():
    kw = dict(base=500000.0, scaling="wavelength", factor=8.0, original=8192, low=1.0, high=4.0)
    w0, _ = fasq.rope_frequencies(128, base=500000.0)
    w, s = fasq.rope_frequencies(128, **kw)
    assert s == 1.0
    for a, b in zip(w0, w):
        length = 2 * math.pi / a
        if length < 8192 / 4:
            assert b == a
        elif length > 8192:
            assert b == pytest.approx(a / 8)
        else:
            smooth = (8192 / length - 1) / 3
            assert b == pytest.approx((1 - smooth) * a / 8 + smooth * a)


def test_frequencies_yarn():
    w0, _ = fasq.rope_frequencies(128)
    w, s = fasq.rope_frequencies(128, scaling="yarn", factor=4.0, original=4096, low=1.0, high=32.0)
    assert s == pytest.approx(0.1 * math.log(4) + 1)
    assert w[0] == w0[0] and w[-1] == pytest.approx(w0[-1] / 4)
    ratio = [a / b for a, b in zip(w, w0)]
    assert all(a >= b - 1e-12 for a, b in zip(ratio, ratio[1:])) and 0.25 < ratio[32] < 1


@pytest.mark.parametrize("kw", [dict(rot=7), dict(rot=0), dict(rot=258), dict(rot=8, base=0.0), dict(rot=8, scaling="cubic"),
                                dict(rot=8, scaling="yarn"), dict(rot=8, scaling="wavelength", original=100, low=4, high=1),
                                dict(rot=8, scaling="linear", factor=0.0), dict(rot=2, scaling="ntk", factor=2.0)])
def test_frequencies_refuse(kw):
    with pytest.raises(ValueError):
        fasq.rope_frequencies(**kw)
