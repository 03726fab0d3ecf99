"""Scores and masks of attention, and the rules between logits and tokens,
without a GPU: refusals before anything touches one, pins of the fp64
definitions against closed forms, and the trees of the binding."""

import ctypes
import math

import numpy as np
import pytest

import paper_2605_04084_amd as fasq
from oracle import layer_ops as lo
from test_layer_abi_host import DUMMY, L, _cache, _refused  # noqa: F401


def _attention(L, scores, **kw):
    a = dict(q=DUMMY, qs=256, qh=64, T=3, Hq=4, cache=_cache(), Hkv=2, D=64, pages=DUMMY, prs=8, maxp=8, qst=DUMMY, kv=DUMMY,
             B=2, scale=0.125, causal=1, window=0, scores=scores, out=DUMMY + 64, os=256, oh=64, lse=0, ws=0, wb=0)
    a.update(kw)
    return L.fasq_paged_attention_ex(*a.values(), 0)


@pytest.mark.parametrize("scores,kw,why", [
    (dict(softcap=-1.0), {}, "softcap"), (dict(softcap=float("nan")), {}, "softcap"), (dict(softcap=1e-4), {}, "softcap"),
    (dict(softcap=5.0), dict(scale=float("inf")), "softcap needs"), (dict(softcap=5.0), dict(scale=-1e20), "softcap needs"),
    (dict(slopes=DUMMY), dict(scale=0.0), "slopes need"), (dict(slopes=DUMMY), dict(scale=1e20), "slopes need"),
    (dict(spans=DUMMY), dict(window=5), "window"), (dict(tree=DUMMY, tree_words=1, tree_stride=1), dict(window=5), "window"),
    (dict(tree=DUMMY), {}, "tree_words"), (dict(tree=DUMMY, tree_words=2 ** 25, tree_stride=1), {}, "tree_words"),
    (dict(tree=DUMMY, tree_words=2, tree_stride=-1), {}, "tree_stride"), (dict(tree=DUMMY + 2, tree_words=1, tree_stride=1), {}, "4-byte"),
    (dict(slopes=DUMMY + 1), {}, "4-byte"), (dict(spans=DUMMY + 2), {}, "4-byte"), (dict(), dict(T=-1), "T must"),
    (dict(softcap=5.0), dict(out=DUMMY), "out must not be q"),
])
def test_attention_refuses(L, scores, kw, why):  # noqa: F811
    _refused(_attention(L, fasq.AttentionScores(**scores), **kw), why)


@pytest.mark.parametrize("scores,why", [(dict(softcap=1025.0), "1024"), (dict(slopes=DUMMY, tree=DUMMY, tree_words=1, tree_stride=1), "slopes with tree")])
def test_attention_does_not_support(L, scores, why):  # noqa: F811
    _refused(_attention(L, fasq.AttentionScores(**scores)), why, fasq.FASQ_ERR_UNSUPPORTED)


def test_no_tokens_are_a_valid_call(L):  # noqa: F811
    assert _attention(L, fasq.AttentionScores(softcap=3.0), T=0, B=0, maxp=0, q=0, out=0) == fasq.FASQ_OK
    assert _attention(L, None, T=0, B=0, maxp=0, q=0, out=0) == fasq.FASQ_OK


def _logits(L, fields=None, **kw):
    a = dict(logits=DUMMY, wide=0, stride=100, R=3, V=100, rules=fasq.TokenRules(**{**dict(S=3), **(fields or {})}), out=DUMMY + 4096, out_wide=0,
             out_stride=100, choice=0, lse=0, ws=0, wb=0)
    a.update(kw)
    held = a["rules"]
    if held is not None:
        a["rules"] = ctypes.addressof(held)
    return L.fasq_process_logits(*a.values(), 0)


TREE = dict(draft_tokens=DUMMY, q_start=DUMMY, tree=DUMMY, tree_words=1, tree_stride=1)


@pytest.mark.parametrize("rules,kw,why", [
    ({}, dict(R=-1), "R must"), ({}, dict(V=0), "V must"), ({}, dict(V=2 ** 31), "V must"), ({}, dict(rules=None), "rules is NULL"),
    (dict(S=-1), {}, "S must"), (dict(S=4), {}, "S must be R"), ({}, dict(logits=0), "NULL"), ({}, dict(out=0), "nothing to write"),
    ({}, dict(logits=DUMMY + 1), "aligned"), ({}, dict(out=DUMMY + 2, out_wide=1), "aligned"), ({}, dict(stride=-1), "strides"),
    ({}, dict(out_stride=99), "overlap"), ({}, dict(out=DUMMY, out_wide=1), "out = logits"), ({}, dict(out=DUMMY, out_stride=104), "out = logits"),
    (dict(tokens=DUMMY, max_tokens=5), {}, "together"), (dict(token_count=DUMMY, max_tokens=5), {}, "together"),
    (dict(prompt_len=DUMMY), {}, "prompt_len"), (dict(tokens=DUMMY, token_count=DUMMY, max_tokens=-1), {}, "max_tokens"),
    (dict(bias_ids=DUMMY), {}, "together"), (dict(bias_values=DUMMY), {}, "together"),
    (dict(bias_ids=DUMMY, bias_values=DUMMY, max_bias=-1), {}, "max_bias"), (dict(allowed=DUMMY, allowed_stride=-4), {}, "strides"),
    (dict(draft_tokens=DUMMY), {}, "together"), ({**TREE, "q_start": 0}, {}, "together"), ({**TREE, "tree_words": 0}, {}, "tree_words"),
    ({**TREE, "tree_stride": -1}, {}, "tree_stride"), (dict(repetition=DUMMY), {}, "need tokens"), (dict(frequency=DUMMY), {}, "need tokens"),
    (dict(temperature=DUMMY + 2), {}, "4-byte"), ({}, dict(lse=DUMMY + 2), "4-byte"),
])
def test_logits_refuse(L, rules, kw, why):  # noqa: F811
    _refused(_logits(L, rules, **kw), why)


def test_no_rows_are_a_valid_call(L):  # noqa: F811
    assert _logits(L, dict(S=0), R=0, logits=0, out=0) == fasq.FASQ_OK
    assert L.fasq_process_logits_workspace_bytes(-1, 5) == -1 and L.fasq_process_logits_workspace_bytes(5, 0) == -1


# ---------------------------------------------------------------------------
# Pins of the definitions
# ---------------------------------------------------------------------------

def _keys(kv, scores, values):
    """A cache of one head of eight dimensions whose products with q = e_0 are ``scores``."""
    k, v = np.zeros((1, kv, 1, 8)), np.zeros((1, kv, 1, 8))
    k[0, :, 0, 0], v[0, :, 0, 0] = scores, values
    return k, v


def _one(scores, values, n=1, **kw):
    kv = len(scores)
    k, v = _keys(kv, scores, values)
    q = np.zeros((n, 1, 8))
    q[:, 0, 0] = 1
    out, lse = lo.scored_attention(q, k, v, np.array([[0]]), [0, n], [kv], 1.0, **kw)[:2]
    return out[:, 0, 0], lse[:, 0]


def test_a_cap_bounds_scores():
    out, lse = _one([1e9, -1e9], [1.0, 0.0], softcap=2.0)
    assert out[0] == pytest.approx(1 / (1 + math.exp(-4)), rel=1e-12)
    assert lse[0] == pytest.approx(math.log(math.exp(2) + math.exp(-2)), rel=1e-12)
    assert _one([0.5, -0.25], [1.0, 0.0], softcap=1e6)[0][0] == pytest.approx(_one([0.5, -0.25], [1.0, 0.0])[0][0], rel=1e-9)


def test_a_bias_is_a_geometric_weight():
    out, lse = _one([0.0] * 4, [8.0, 4.0, 2.0, 1.0], slopes=[math.log(2)])
    w = [1 / 8, 1 / 4, 1 / 2, 1]
    assert out[0] == pytest.approx(4 / sum(w), rel=1e-12) and lse[0] == pytest.approx(math.log(sum(w)), rel=1e-12)


def test_spans_and_trees_choose_keys():
    out, lse = _one([0.0] * 4, [1.0, 10.0, 100.0, 1000.0], n=2, spans=[[1, 3], [4, 9]])
    assert out[0] == pytest.approx(55.0) and out[1] == 0 and lse[1] == -math.inf
    tree, depth = fasq.draft_tree([[-1, 0, 0]], device="cpu")
    assert tree.tolist() == [[1], [3], [5]] and depth.tolist() == [0, 1, 1]
    out, _ = _one([0.0] * 4, [1.0, 10.0, 100.0, 1000.0], n=3, tree=tree.numpy())
    assert out == pytest.approx([5.5, 37.0, 337.0])


def test_a_chain_is_causal():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((3, 4, 1, 8)), rng.standard_normal((3, 4, 1, 8))
    pages = np.array([[2, 0, 1]])
    tree = fasq.draft_tree([[-1, 0, 1, 2, 3]], device="cpu")[0].numpy()
    want = lo.paged_attention(q, k, v, pages, [0, 5], [11], 0.3)
    for kw in (dict(), dict(tree=tree), dict(spans=[[0, 7 + i] for i in range(5)]), dict(slopes=[0.0, 0.0])):
        got = lo.scored_attention(q, k, v, pages, [0, 5], [11], 0.3, **kw)
        assert np.allclose(got[0], want[0], rtol=1e-12) and np.allclose(got[1], want[1], rtol=1e-12)


def test_draft_trees():
    parents = [[-1] + [i // 2 for i in range(1, 40)], [], [-1, -1, 1]]
    tree, depth = fasq.draft_tree(parents, device="cpu")
    assert tree.shape == (43, 2) and depth[:3].tolist() == [0, 1, 2]
    for i, p in enumerate(parents[0]):
        way = [i]
        while parents[0][way[-1]] >= 0:
            way.append(parents[0][way[-1]])
        assert np.nonzero(lo.tree_bits(tree.numpy(), i, 64))[0].tolist() == sorted(way) and depth[i] == len(way) - 1
    assert tree[40:].tolist() == [[1, 0], [2, 0], [6, 0]]
    full = fasq.draft_tree([[-1] + list(range(31))], device="cpu")[0]
    assert full[31].tolist() == [-1]  # all bits of a word
    for bad in ([[0]], [[-1, 1]], [[-2]]):
        with pytest.raises(ValueError):
            fasq.draft_tree(bad, device="cpu")
    assert fasq.draft_tree([], device="cpu")[0].shape == (0, 1)


def test_rules_of_logits():
    x, choice, lse = lo.process_logits([2.0, -2.0, 1.0, 0.5], True, tokens=[0, 1, 1, 1, 2, 9], prompt_len=1, repetition=2.0,
                                       presence=0.25, frequency=0.5, bias=[(3, 7.0), (3, 1.0), (-1, 5.0)], temperature=0.5)
    # token 0 occurs in the prompt alone, token 1 three times, token 2 once; the last bias counts
    assert x == pytest.approx([2.0, 2 * (-4 - 1.75), 2 * (0.5 - 0.75), 3.0])
    assert choice == 3 and lse == pytest.approx(math.log(sum(math.exp(v) for v in x)))
    x, choice, lse = lo.process_logits([1.0, 1.0, 5.0], True, allowed=[True, True, False])
    assert choice == 0 and x[2] == -np.inf and lse == pytest.approx(1 + math.log(2))
    assert lo.process_logits([1.0], True, allowed=[False])[1:] == (-1, -np.inf)
    assert lo.process_logits([1.0, np.nan], True)[1] == 1
