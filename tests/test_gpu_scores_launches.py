"""Attention with scores and masks of its own and process_logits in launch
lists, HIP graphs and on other streams, as in test_gpu_layer_launches.py; and a
step of drafted decoding: the new keys to the cache, attention over the trees,
the rules on every node, all in one graph.
"""

import numpy as np
import pytest

import test_gpu_layer_launches as base
from test_gpu_layer_launches import Attention, _direct, _half, _i32, _same
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


class Scored(Attention):
    """Runs of keys, or trees, or biases change between runs too."""

    def __init__(self, T, B, kv, what, **kw):
        super().__init__(T, B, kv, **kw)
        self.what, Hq = what, self.inputs[0].shape[1]
        rng = np.random.default_rng(T)
        self.inputs.append({"spans": lambda: _i32(np.tile([0, kv], (T, 1))), "tree": lambda: _i32(rng.integers(-2 ** 31, 2 ** 31, (T, 2))),
                            "slopes": lambda: to_dev(np.linspace(0.01, 1, Hq).astype(np.float32))}[what]())

    def call(self, outs):
        q, q_start, kv_len, more = self.inputs
        fasq.paged_attention(q, self.k, self.v, self.pages, q_start, kv_len, out=outs[0], workspace=self.ws, softcap=6.0,
                             **{self.what: more})

    def change(self, rng):
        super().change(rng)
        t = self.inputs[3]
        if self.what == "slopes":
            t.copy_(to_dev(rng.uniform(0, 1, t.shape).astype(np.float32)))
        elif self.what == "spans":
            t.copy_(_i32(np.sort(rng.integers(0, self.kv, t.shape), axis=1)))
        else:
            t.copy_(_i32(rng.integers(-2 ** 31, 2 ** 31, t.shape)))


class Logits:
    def __init__(self, S, n, V):
        rng = np.random.default_rng(S)
        R, self.V, self.L = S * n, V, 90
        f32 = lambda lo, hi: to_dev(rng.uniform(lo, hi, S).astype(np.float32))  # noqa: E731
        self.inputs = [_half(rng, R, V), _i32(rng.integers(0, V, (S, self.L))), _i32(rng.integers(0, self.L, S)), f32(1, 2), f32(0, 1), f32(0, 1),
                       f32(0.5, 1), _i32(rng.integers(-2 ** 31, 2 ** 31, (R, -(-V // 32)))), _i32(rng.integers(0, V, R)),
                       _i32(rng.integers(-2 ** 31, 2 ** 31, (R, 1)))]
        self.requests, self.q_start = _i32(np.repeat(np.arange(S), n)), _i32(np.arange(0, R + 1, n))
        dev = dict(device="cuda:0")
        self.outputs = [torch.zeros((R, V), dtype=torch.float32, **dev), torch.zeros(R, dtype=torch.int32, **dev), torch.zeros(R, **dev)]
        self.ws = torch.zeros(fasq.process_logits_workspace_bytes(R, V), dtype=torch.uint8, **dev)

    def call(self, outs):
        x, tokens, count, rho, presence, frequency, tau, allowed, drafts, tree = self.inputs
        fasq.process_logits(x, self.requests, tokens=tokens, token_count=count, repetition=rho, presence=presence, frequency=frequency,
                            temperature=tau, allowed=allowed, draft_tokens=drafts, tree=tree, q_start=self.q_start, out=outs[0],
                            choose=True, choice=outs[1], lse=outs[2], workspace=self.ws)

    def change(self, rng):
        self.inputs[0].copy_(_half(rng, *self.inputs[0].shape))
        self.inputs[1].copy_(_i32(rng.integers(0, self.V, self.inputs[1].shape)))
        self.inputs[2].copy_(_i32(rng.integers(0, self.L + 1, self.inputs[2].shape)))
        for i in (7, 9):
            self.inputs[i].copy_(_i32(rng.integers(-2 ** 31, 2 ** 31, self.inputs[i].shape)))


MAKE = {
    "tree-few": lambda: Scored(7, 2, 3000, "tree"), "tree-tile": lambda: Scored(100, 2, 2100, "tree", D=128, Hq=8),
    "spans-few": lambda: Scored(3, 3, 3000, "spans"), "spans-tile": lambda: Scored(300, 3, 900, "spans", D=128),
    "slopes-few": lambda: Scored(3, 3, 3000, "slopes"), "slopes-tile": lambda: Scored(300, 3, 900, "slopes", D=128),
    "logits": lambda: Logits(3, 1, 5003), "logits-trees": lambda: Logits(4, 9, 20000),
}


@pytest.fixture(autouse=True)
def _cases(monkeypatch):
    monkeypatch.setattr(base, "MAKE", MAKE)


@pytest.mark.parametrize("name", MAKE)
def test_launch_list(name):
    base.test_launch_list(name)


@pytest.mark.parametrize("name", MAKE)
def test_graph_replays(name):
    base.test_graph_replays(name)


@pytest.mark.parametrize("name", MAKE)
def test_another_stream(name):
    base.test_another_stream(name)


@pytest.mark.parametrize("name", MAKE)
def test_launch_list_keeps_its_workspaces(name):
    base.test_launch_list_keeps_its_workspaces(name)


class Step:
    """Drafted tokens of two requests: keys and values to the cache, attention over the trees, logits and their rules."""

    def __init__(self):
        rng = np.random.default_rng(0)
        n, Hq, Hkv, D, size, V = 6, 4, 2, 64, 16, 3001
        T = 2 * n
        self.k, self.v = _half(rng, 40, size, Hkv, D), _half(rng, 40, size, Hkv, D)
        self.kept = self.k.clone(), self.v.clone()
        self.pages = rng.permutation(40).reshape(2, 20)
        self.tree, self.depth = fasq.draft_tree([[-1, 0, 0, 1, 1, 2]] * 2)
        w, scale = fasq.rope_frequencies(D)
        self.table = fasq.rope_table(w, 400, scale)
        self.head = _half(rng, Hq * D, V)
        self.q_start, self.requests = _i32([0, n, T]), _i32([0] * n + [1] * n)
        self.device_pages = _i32(self.pages)
        self.n, self.size = n, size
        self.inputs = [_half(rng, T, Hq, D), _half(rng, T, Hkv, D), _half(rng, T, Hkv, D), _i32(np.zeros(T)), _i32(np.zeros(T)), _i32([0, 0]),
                       _i32(rng.integers(0, V, (2, 50))), _i32([50, 20]), _i32(rng.integers(0, V, T))]
        self.outputs = [torch.zeros((T, Hq, D), dtype=torch.float16, device="cuda:0"), torch.zeros(T, dtype=torch.int32, device="cuda:0"),
                        torch.zeros(T, device="cuda:0")]
        self.penalty = to_dev(np.full(2, 1.3, dtype=np.float32))
        self.lengths(rng)

    def lengths(self, rng):
        start = rng.integers(0, 300, 2)
        at = start.repeat(self.n) + np.tile(np.arange(self.n), 2)
        slot = self.pages[np.repeat([0, 1], self.n), at // self.size] * self.size + at % self.size
        self.inputs[3].copy_(_i32(start.repeat(self.n)) + self.depth)
        self.inputs[4].copy_(_i32(slot))
        self.inputs[5].copy_(_i32(start + self.n))

    def call(self, outs):
        q, k, v, positions, slots, kv_len, tokens, count, drafts = self.inputs
        q = fasq.rope_append(q, k, v, self.table, positions, slots, self.k, self.v)
        a = fasq.paged_attention(q, self.k, self.v, self.device_pages, self.q_start, kv_len, out=outs[0], tree=self.tree)
        fasq.process_logits(a.flatten(1) @ self.head, self.requests, tokens=tokens, token_count=count, repetition=self.penalty,
                            draft_tokens=drafts, tree=self.tree, q_start=self.q_start, write=False, choose=True, choice=outs[1], lse=outs[2])

    def change(self, rng):
        for t in self.inputs[:3]:
            t.copy_(_half(rng, *t.shape))
        self.lengths(rng)


def test_a_drafted_step_in_a_graph():
    case = Step()
    _direct(case)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.call(case.outputs)
    rng = np.random.default_rng(3)
    for _ in range(4):
        graph.replay()
        got = [t.clone() for t in case.outputs]
        for a, b in zip(got, _direct(case)):
            assert torch.equal(a, b)
        case.change(rng)


def test_nodes_are_the_tokens_of_their_branch():
    """Every node's result is that of its own branch alone, appended token by token."""
    case = Step()
    case.call(case.outputs)
    q, k, v, positions, slots, kv_len, *_ = case.inputs
    start = (kv_len - case.n).tolist()
    for node, way in ((0, [0]), (2, [0, 2]), (4, [0, 1, 4]), (5, [0, 2, 5]), (6 + 3, [6, 7, 9])):
        r = node // case.n
        ck, cv = (t.clone() for t in case.kept)
        at = start[r] + np.arange(len(way))
        s = _i32(case.pages[r, at // case.size] * case.size + at % case.size)
        pick = torch.tensor(way, device="cuda:0")
        qq = fasq.rope_append(q[pick], k[pick], v[pick], case.table, positions[pick].contiguous(), s, ck, cv)
        out = fasq.paged_attention(qq, ck, cv, case.device_pages[r:r + 1], _i32([0, len(way)]), _i32([start[r] + len(way)]))
        # each side: 2^-11 of values below one for its rounding, and as much for its weights
        assert torch.allclose(out[-1].float(), case.outputs[0][node].float(), rtol=0, atol=4 * 2.0 ** -11)
