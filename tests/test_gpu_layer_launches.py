"""The entry points between projections in launch lists, HIP graphs and on
other streams: bit for bit what a direct call writes, on inputs changed since
the recording, in every run.
"""

import numpy as np
import pytest

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


def _half(rng, *shape):
    return to_dev(rng.standard_normal(shape).astype(np.float16))


def _i32(a):
    return to_dev(np.asarray(a, dtype=np.int32))


class Rope:
    """Queries turned in place of another tensor, keys and values to mixed slots."""

    def __init__(self, T, Hq=4, Hkv=2, D=64, size=16):
        rng = np.random.default_rng(T)
        w, scale = fasq.rope_frequencies(D)
        self.table = fasq.rope_table(w, 400, scale)
        self.inputs = [_half(rng, T, Hq, D), _half(rng, T, Hkv, D), _half(rng, T, Hkv, D),
                       _i32(rng.integers(0, 400, T)), _i32(rng.permutation((T // size + 2) * size)[:T])]
        shape = (T // size + 2, size, Hkv, D)
        self.outputs = [torch.zeros(shape, dtype=torch.float16, device="cuda:0") for _ in range(2)] + \
            [torch.zeros((T, Hq, D), dtype=torch.float16, device="cuda:0")]

    def call(self, outs):
        q, k, v, pos, slots = self.inputs
        fasq.rope_append(q, k, v, self.table, pos, slots, outs[0], outs[1], out=outs[2])

    def change(self, rng):
        for t in self.inputs[:3]:
            t.copy_(_half(rng, *t.shape))
        self.inputs[3].copy_(_i32(rng.integers(0, 400, self.inputs[3].numel())))
        self.inputs[4].copy_(_i32(rng.permutation(self.outputs[0].shape[0] * self.outputs[0].shape[1])
                                  [:self.inputs[4].numel()]))


class Norm:
    def __init__(self, M, N):
        rng = np.random.default_rng(M)
        self.inputs = [_half(rng, M, N), _half(rng, M, N), _half(rng, N), _half(rng, N)]
        self.outputs = [torch.zeros((M, N), dtype=torch.float16, device="cuda:0") for _ in range(2)]

    def call(self, outs):
        x, y, w, post = self.inputs
        fasq.residual_norm(x, y, w, post_weight=post, scale=0.5, x_out=outs[0], out=outs[1])

    def change(self, rng):
        for t in self.inputs:
            t.copy_(_half(rng, *t.shape))


class Lora:
    def __init__(self, M, K=512, Ns=(256, 100), r=8, L=3):
        rng = np.random.default_rng(M)
        self.shape, self.L = (M, K), L
        self.As, self.Bs = [_half(rng, L, r, K) for _ in Ns], [_half(rng, L, n, r) for n in Ns]
        self.scales = to_dev(np.linspace(0.5, 1.5, L).astype(np.float32))
        self.inputs = [_half(rng, M, K), _i32(rng.integers(-1, L, M))] + [_half(rng, M, n) for n in Ns]
        self.outputs = [torch.zeros((M, n), dtype=torch.float16, device="cuda:0") for n in Ns]
        self.ws = torch.zeros(max(fasq.lora_workspace_bytes(M, K, r, len(Ns)), 1), dtype=torch.uint8, device="cuda:0")

    def call(self, outs):
        x, ids, *bases = self.inputs
        fasq.lora_batched(x, ids, self.As, self.Bs, self.scales, bases, outs=outs, workspace=self.ws)

    def change(self, rng):
        for t in [self.inputs[0]] + self.inputs[2:]:
            t.copy_(_half(rng, *t.shape))
        self.inputs[1].copy_(_i32(rng.integers(-1, self.L, self.shape[0])))


class Attention:
    """Lengths change between runs, so other shares of the split keys do too."""

    def __init__(self, T, B, kv, Hq=4, Hkv=2, D=64, size=16):
        rng = np.random.default_rng(T)
        P = -(-kv // size)
        self.T, self.B, self.kv = T, B, kv
        self.k, self.v = _half(rng, B * P, size, Hkv, D), _half(rng, B * P, size, Hkv, D)
        self.pages = _i32(rng.permutation(B * P).reshape(B, P))
        self.inputs = [_half(rng, T, Hq, D), _i32(np.linspace(0, T, B + 1)), _i32([kv] * B)]
        self.outputs = [torch.zeros((T, Hq, D), dtype=torch.float16, device="cuda:0")]
        need = fasq.paged_attention_workspace_bytes(T, B, Hq, Hkv, D)
        self.ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda:0")

    def call(self, outs):
        q, q_start, kv_len = self.inputs
        fasq.paged_attention(q, self.k, self.v, self.pages, q_start, kv_len, out=outs[0], workspace=self.ws)

    def change(self, rng):
        self.inputs[0].copy_(_half(rng, *self.inputs[0].shape))
        cuts = np.sort(rng.integers(0, self.T + 1, self.B - 1))
        self.inputs[1].copy_(_i32(np.concatenate([[0], cuts, [self.T]])))
        self.inputs[2].copy_(_i32(rng.integers(0, self.kv + 1, self.B)))


MAKE = {
    "rope": lambda: Rope(37), "rope-one": lambda: Rope(1, D=50),
    "norm": lambda: Norm(3, 1000), "norm-wide": lambda: Norm(2, 8192),
    "lora-few": lambda: Lora(5), "lora-many": lambda: Lora(300),
    "attention-few": lambda: Attention(3, 3, 3000), "attention-tile": lambda: Attention(300, 3, 900, D=128),
}


def _direct(case):
    outs = [torch.zeros_like(t) for t in case.outputs]
    case.call(outs)
    torch.cuda.synchronize()
    return outs


def _same(case, want):
    torch.cuda.synchronize()
    for a, b in zip(case.outputs, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", MAKE)
def test_launch_list(name):
    case = MAKE[name]()
    lst = fasq.LaunchList()
    with lst:
        case.call(case.outputs)
    torch.cuda.synchronize()
    assert len(lst) >= 1 and not any(t.any() for t in case.outputs)  # recorded, not run
    rng = np.random.default_rng(1)
    for i in range(4):
        want = _direct(case)
        for t in case.outputs:
            t.zero_()
        if i % 2:
            other = torch.cuda.Stream()
            other.wait_stream(torch.cuda.current_stream())
            lst.run(other)
            torch.cuda.current_stream().wait_stream(other)
        else:
            lst.run()
        _same(case, want)
        case.change(rng)
    lst.close()


@pytest.mark.parametrize("name", MAKE)
def test_graph_replays(name):
    case = MAKE[name]()
    _direct(case)  # kernels are loaded before a capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.call(case.outputs)
    rng = np.random.default_rng(2)
    for _ in range(5):
        for t in case.outputs:
            t.zero_()
        graph.replay()
        got = [t.clone() for t in case.outputs]
        want = _direct(case)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        case.change(rng)


@pytest.mark.parametrize("name", MAKE)
def test_another_stream(name):
    """The call goes to torch's current stream: it waits for what that stream
    still does to its inputs."""
    case = MAKE[name]()
    want = _direct(case)
    kept = [t.clone() for t in case.inputs]
    for t in case.inputs:
        t.zero_()
    busy = torch.randn(4096, 4096, device="cuda:0")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(3):
            busy = busy * 1.0001
        for t, k in zip(case.inputs, kept):
            t.copy_(k)
        case.call(case.outputs)
    torch.cuda.current_stream().wait_stream(stream)
    _same(case, want)


@pytest.mark.parametrize("name", ["lora-few", "lora-many", "attention-few", "attention-tile"])
def test_launch_list_keeps_its_workspaces(name):
    """A workspace that a recorded call allocated is no other tensor's memory
    while the list may run."""
    case = MAKE[name]()
    want = _direct(case)
    size = case.ws.numel()
    case.ws = None  # the calls allocate their own
    torch.cuda.synchronize()
    lst = fasq.LaunchList()
    with lst:
        case.call(case.outputs)
    # tensors that would take its place
    others = [torch.full((size,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(3)]
    for _ in range(2):
        lst.run()
        _same(case, want)
    for t in others:
        assert bool((t == 255).all())
    lst.close()
