"""process_logits against the fp64 definition of its rules.

A value takes at most eight roundings of fp32 (two reciprocals, their products, the
penalty's product, sum and difference, the bias): 8 * 2^-24 of the largest
magnitude on its way, then one of the output's type.  The choice is exact where
values can be held exactly, else one of those within that tolerance.  The logarithm:
2^-19 (sums of positive weights off by 2^-21 each, exponents of up to 2^5 by
2^-24) and the values' tolerance.
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


def words_of(bits):
    """int32 words of rows of truth values."""
    R, V = bits.shape
    pad = np.zeros((R, -(-V // 32) * 32), dtype=np.uint8)
    pad[:, :V] = bits
    return np.packbits(pad, axis=1, bitorder="little").view(np.int32)


class Rows:
    """S requests of n rows each over V logits, with every rule there is."""

    def __init__(self, S, n, V, L=40, E=6, wide=False, seed=0):
        rng = np.random.default_rng(seed + V)
        self.S, self.n, self.V, self.wide = S, n, V, wide
        self.logits = (rng.standard_normal((S * n, V)) * 3).astype(np.float32 if wide else np.float16)
        self.requests = np.repeat(np.arange(S), n).astype(np.int32)
        self.tokens = rng.integers(-3, min(V + 3, 60), (S, L)).astype(np.int32)
        self.token_count = rng.integers(0, L + 1, S).astype(np.int32)
        self.prompt_len = (self.token_count // 2).astype(np.int32)
        self.repetition = rng.uniform(0.8, 1.5, S).astype(np.float32)
        self.presence = rng.uniform(-0.5, 1, S).astype(np.float32)
        self.frequency = rng.uniform(-0.2, 0.5, S).astype(np.float32)
        self.temperature = rng.uniform(0.3, 2, S).astype(np.float32)
        self.bias_ids = rng.integers(-2, V + 2, (S, E)).astype(np.int32)
        if E > 3:
            self.bias_ids[:, 3] = self.bias_ids[:, 0]  # the same token twice
        self.bias_values = (rng.standard_normal((S, E)) * 4).astype(np.float32)
        self.bits = rng.random((S * n, V)) < 0.7
        self.allowed = words_of(self.bits)
        parents = [[-1] + [int(rng.integers(0, i)) for i in range(1, n)] for _ in range(S)]
        self.tree = fasq.draft_tree(parents, device="cpu")[0].numpy()
        self.draft_tokens = rng.integers(-1, min(V, 40), S * n).astype(np.int32)
        self.q_start = np.arange(0, S * n + 1, n).astype(np.int32)

    ALL = ("tokens", "token_count", "prompt_len", "repetition", "presence", "frequency", "temperature", "bias_ids", "bias_values",
           "allowed", "draft_tokens", "tree", "q_start")

    def run(self, names=ALL, **kw):
        args = {k: to_dev(getattr(self, k)) for k in names}
        args["requests"] = to_dev(self.requests)
        args.update(kw)
        logits = args.pop("logits", None)
        got = fasq.process_logits(to_dev(self.logits) if logits is None else logits, choose=True, requests_count=self.S, **args)
        return tuple(None if t is None else to_np(t) for t in got)

    def row(self, r, names):
        s = int(self.requests[r])
        if not 0 <= s < self.S:
            return None, 0.0
        kw, size = {}, np.abs(np.where(np.isfinite(self.logits[r]), self.logits[r], 0)).astype(np.float64)
        if "tokens" in names:
            kw["tokens"] = self.tokens[s][:max(0, int(self.token_count[s]))]
            kw["prompt_len"] = int(self.prompt_len[s]) if "prompt_len" in names else 0
        if "tree" in names:
            first, last = int(self.q_start[s]), int(self.q_start[s + 1])
            see = lo.tree_bits(self.tree, r, last - first)
            kw["drafted"] = self.draft_tokens[first:last][see]
        grow = 1.0
        for k in ("repetition", "presence", "frequency", "temperature"):
            if k in names:
                kw[k] = float(getattr(self, k)[s])
        if "repetition" in names:
            grow = max(kw["repetition"], 1 / kw["repetition"])
        times = len(kw.get("tokens", ())) + len(kw.get("drafted", ()))
        size = size * grow + abs(kw.get("frequency", 0)) * times + abs(kw.get("presence", 0))
        if "bias_ids" in names:
            kw["bias"] = list(zip(self.bias_ids[s].tolist(), self.bias_values[s].astype(np.float64).tolist()))
            size = size + max([abs(v) for _, v in kw["bias"]] + [0])
        if kw.get("temperature", 0) > 0:
            size = size / kw["temperature"]
        if "allowed" in names:
            kw["allowed"] = self.bits[r]
        return lo.process_logits(self.logits[r], True, **kw), 8 * 2.0 ** -24 * size

    def check(self, got, names=ALL):
        out, choice, lse = got
        for r in range(len(self.requests)):
            ref, tol = self.row(r, names)
            if ref is None:
                continue
            x, best, total = ref
            if out is not None:
                step = 2.0 ** -11 if out.dtype == np.float16 else 2.0 ** -24
                y = out[r].astype(np.float64)
                assert np.array_equal(np.isnan(y), np.isnan(x)) and np.array_equal(np.isneginf(y), np.isneginf(x))
                fine = np.isfinite(x) & (np.abs(x) < 65000)
                assert (np.abs(y - x)[fine] <= (tol + step * (np.abs(x) + tol) + (2.0 ** -25 if step > 1e-5 else 0))[fine]).all(), r
            if best < 0 or np.isnan(total):
                assert choice[r] == best
            else:
                assert x[choice[r]] + tol[choice[r]] >= x[best] - tol[best], (r, choice[r], best)
            if not np.isfinite(total):
                assert np.array_equal(lse[r], np.float32(total), equal_nan=True)
            else:
                assert abs(float(lse[r]) - total) <= 2.0 ** -19 + tol[np.isfinite(x)].max() + 2.0 ** -22 * abs(total), (r, lse[r], total)

    def both(self, names=ALL, **kw):
        got = self.run(names, **kw)
        self.check(got, names)
        return got


SIZES = [1, 2, 7, 8, 31, 33, 1000, 2047, 2048, 2049, 4096, 4103, 20011]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("wide", [False, True])
def test_all_rules(V, wide):
    Rows(3, 1, V, wide=wide).both()
    Rows(2, 5, V, wide=wide, seed=1).both()


RULES = [(), ("temperature",), ("bias_ids", "bias_values"), ("allowed",), ("tokens", "token_count", "repetition"),
         ("tokens", "token_count", "prompt_len", "frequency"), ("tokens", "token_count", "prompt_len", "presence", "repetition"),
         ("draft_tokens", "tree", "q_start", "frequency"), ("tokens", "token_count", "prompt_len")]


@pytest.mark.parametrize("names", RULES)
@pytest.mark.parametrize("out", [None, torch.float16, torch.float32])
def test_some_rules_and_outputs(names, out):
    b = Rows(3, 4, 5003, seed=2)
    kw = dict(write=False) if out is None else dict(out=torch.full((12, 5003), 9.0, dtype=out, device="cuda:0"))
    b.both(names, **kw)


def test_nothing_to_do_copies():
    b = Rows(4, 1, 3001, seed=3)
    out, choice, _ = b.both(())
    assert np.array_equal(out, b.logits)
    assert np.array_equal(choice, b.logits.astype(np.float64).argmax(1))


def test_the_lowest_of_equal_tokens():
    b = Rows(2, 1, 9000, seed=4)
    b.logits[:] = np.minimum(b.logits, 1)
    first = (b.logits == 1).argmax(1)
    assert np.array_equal(b.run(())[1], first)
    b.logits[:] = -0.0
    b.logits[1, 5:] = 0.0  # the zeros are equal
    assert b.run(())[1].tolist() == [0, 0]


def test_in_place_views_and_other_rows():
    """out = logits, rows with strides at odd addresses, rows that belong to no request."""
    b = Rows(3, 2, 2999, seed=5)
    plain = b.both()
    buffer = torch.full((6, 3011), 5.0, dtype=torch.float16, device="cuda:0")
    view = buffer[:, 7:7 + 2999]
    view.copy_(to_dev(b.logits))
    got = b.run(logits=view, out=view)
    for x, y in zip(got, plain):
        assert np.array_equal(x, y)
    assert (to_np(buffer[:, :7]) == 5).all() and (to_np(buffer[:, 7 + 2999:]) == 5).all()
    b.requests[[1, 4]] = [-1, 3]
    out = torch.full((6, 2999), 9.0, dtype=torch.float32, device="cuda:0")
    got = b.both(out=out)
    assert (got[0][[1, 4]] == 9).all() and (got[0][[0, 2, 3, 5]] != 9).any(1).all()


def test_masked_infinities_and_rows_without_tokens():
    b = Rows(5, 1, 4100, seed=6)
    b.logits[0, 17] = np.nan
    b.bits[0, 17] = False          # not allowed: does not matter
    b.logits[1, 4000] = np.nan
    b.bits[1, 4000] = True
    b.bits[2] = False              # nothing is allowed
    b.logits[3, 9] = np.inf
    b.bits[3, 9] = True
    b.logits[4] = -np.inf
    b.allowed = words_of(b.bits)
    names = ("allowed", "temperature")
    got = b.both(names)
    assert got[1][[1, 2, 4]].tolist() == [4000, -1, -1] and got[1][3] == 9
    assert np.isneginf(got[2][[2, 4]]).all() and np.isposinf(got[2][3]) and np.isnan(got[2][1])


def test_masks_of_the_lowest_value():
    """fp32 and fp16 logits whose masked tokens hold their type's lowest value, and rows of nothing else."""
    for wide, low in ((True, np.finfo(np.float32).min), (False, np.finfo(np.float16).min)):
        b = Rows(3, 1, 5000, wide=wide, seed=13)
        b.logits[0, 40:] = low
        b.logits[1] = low
        b.logits[2, ::3] = low
        got = b.both(())
        assert got[1][1] == 0 and got[1][0] == b.logits[0, :40].argmax()
        assert abs(float(got[2][1]) - float(low)) <= 2.0 ** -22 * abs(float(low)) + 9


def test_counts_of_any_length():
    """Lengths of nothing, of all there is, beyond it and below zero; a token thousands of times."""
    b = Rows(5, 1, 3000, L=5000, seed=7)
    b.tokens[:, ::2] = 11
    b.token_count[:] = [0, 5000, 70000, -4, 4999]
    b.prompt_len[:] = [0, 0, 2500, 3, -1]
    b.frequency[:] = 0.001
    names = ("tokens", "token_count", "prompt_len", "repetition", "presence", "frequency")
    got = b.run(names)
    b.token_count[:] = [0, 5000, 5000, 0, 4999]
    b.prompt_len[:] = [0, 0, 2500, 0, 0]
    b.check(got, names)


def test_temperature_of_zero_divides_nothing():
    b = Rows(3, 1, 500, seed=8)
    b.temperature[:] = [0, -1, 0.5]
    b.both(("temperature",))


def test_infinite_penalties_spare_the_prompt():
    logits = torch.arange(1, 21, dtype=torch.float32).reshape(1, 20).cuda()
    got, choice, lse = fasq.process_logits(
        logits, tokens=to_dev(np.array([[19, 18, 17, 18]], dtype=np.int32)), token_count=to_dev(np.array([4], dtype=np.int32)),
        prompt_len=to_dev(np.array([2], dtype=np.int32)), repetition=to_dev(np.array([2], dtype=np.float32)),
        frequency=to_dev(np.array([np.inf], dtype=np.float32)), choose=True)
    want, best, _ = lo.process_logits(to_np(logits)[0], True, [19, 18, 17, 18], 2, repetition=2.0, frequency=np.inf)
    assert (to_np(got)[0] == want).all()  # halves and infinities are exact
    assert int(choice) == best == 16 and np.isfinite(float(lse))


def test_trees_at_the_ends():
    """Fewer words than nodes, more nodes than threads, rows of no bit, starts past the rows."""
    b = Rows(1, 300, 70, seed=9)
    b.both()
    b.tree = np.ascontiguousarray(b.tree[:, :2])
    b.tree[5] = 0
    b.both()
    b.q_start = np.array([0, 2 ** 30], dtype=np.int32)
    got = b.run()
    b.q_start = np.array([0, 300], dtype=np.int32)
    b.check(got)


def test_same_bits_again_and_other_rows_do_not_matter():
    b = Rows(6, 3, 6007, seed=10)
    got = b.run()
    for x, y in zip(got, b.run()):
        assert np.array_equal(x, y)
    one = Rows(6, 3, 6007, seed=10)
    one.logits[3:] = 0
    for x, y in zip(got, one.run()):
        assert np.array_equal(x[:3], y[:3])


@pytest.mark.parametrize("names", [Rows.ALL[:10], ("bias_ids", "bias_values"), ("tokens", "token_count", "presence", "repetition"), ("temperature",)])
def test_requests_in_any_order(names):
    """Rows of many requests mixed, several to a request, and rows of none between them."""
    b = Rows(3, 11, 9001, seed=14)
    rng = np.random.default_rng(14)
    b.requests = rng.integers(-1, 4, 33).astype(np.int32)
    b.requests[7:15] = 1
    out = torch.full((33, 9001), 9.0, dtype=torch.float16, device="cuda:0")
    choice = torch.full((33,), -7, dtype=torch.int32, device="cuda:0")
    lse = torch.full((33,), 7.0, dtype=torch.float32, device="cuda:0")
    got = b.both(names, out=out, choice=choice, lse=lse)
    none = (b.requests < 0) | (b.requests > 2)
    assert none.any() and (got[0][none] == 9).all() and (got[1][none] == -7).all() and (got[2][none] == 7).all()


def test_broadcast_rules():
    """One text, one grammar and one tree for all, as expanded tensors."""
    b = Rows(4, 1, 3003, seed=15)
    b.tokens[:], b.allowed[:], b.bits[:], b.tree[:], b.logits[:] = b.tokens[0], b.allowed[0], b.bits[0], b.tree[0], b.logits[0]
    want = b.both()
    wide = {k: to_dev(getattr(b, k)[:1]).expand(4, -1) for k in ("tokens", "allowed", "tree", "logits")}
    for x, y in zip(b.run(**wide), want):
        assert np.array_equal(x, y)


def test_large_vocabulary_of_few_rows():
    b = Rows(2, 1, 128256, L=3000, E=300, seed=11)
    b.both()
    b.both(write=False)


def test_no_rows_and_no_tokens():
    empty = fasq.process_logits(torch.empty((0, 10), dtype=torch.float16, device="cuda:0"), choose=True)
    assert [t.shape for t in empty] == [(0, 10), (0,), (0,)]
    b = Rows(2, 1, 50, L=0, E=0, seed=12)
    b.both()


def test_tensors_are_checked():
    b = Rows(2, 3, 40)
    f32, i32 = dict(dtype=torch.float32, device="cuda:0"), dict(dtype=torch.int32, device="cuda:0")
    for kw in (dict(temperature=torch.zeros(3, **f32)), dict(repetition=torch.zeros(2, **i32)), dict(allowed=torch.zeros((6, 3), **i32)),
               dict(allowed=torch.zeros((2, 2), **i32)), dict(tree=torch.zeros((2, 1), **i32)), dict(bias_values=torch.zeros((2, 3), **f32)),
               dict(q_start=torch.zeros(2, **i32)), dict(draft_tokens=torch.zeros(5, **i32)), dict(requests=torch.zeros(5, **i32)),
               dict(out=torch.zeros((6, 41), dtype=torch.float16, device="cuda:0")), dict(out=torch.zeros((6, 40), **i32)),
               dict(logits=torch.zeros((6, 40), dtype=torch.bfloat16, device="cuda:0")), dict(logits=torch.zeros((6, 40))),
               dict(token_count=torch.zeros(2, dtype=torch.int64, device="cuda:0"))):
        with pytest.raises((TypeError, ValueError)):
            b.run(**kw)
    for kw in (dict(tokens=None), dict(choice=torch.zeros(5, **i32)), dict(lse=torch.zeros(6, **i32))):
        with pytest.raises((TypeError, ValueError)):
            b.run(**kw)
    with pytest.raises(ValueError):
        fasq.process_logits(to_dev(b.logits), lse=torch.zeros(6, **f32))
    for kw in (dict(tokens=None, token_count=None), dict(q_start=None), dict(bias_ids=None, bias_values=torch.zeros((2, 0), **f32)),
               dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda:0"), logits=torch.zeros((6, 9000), **f32), allowed=None)):
        with pytest.raises((fasq.FasqError, ValueError)):
            b.run(**kw)


@pytest.mark.parametrize("V, n, wide", [(131, 33, False), (131, 12, True), (517, 33, False), (517, 33, True)])
def test_many_rows_of_a_request(V, n, wide):
    """More rows than the chip holds at once: several follow each other in a workgroup."""
    b = Rows(130, n, V, wide=wide, seed=20)
    b.both()
    rng = np.random.default_rng(21)
    b.requests = np.repeat(rng.integers(-1, 131, -(-130 * n // 3)), 3)[:130 * n].astype(np.int32)
    logits = to_dev(b.logits)
    names = Rows.ALL[:10]
    got = b.both(names, logits=logits, out=logits)  # in place
    none = (b.requests < 0) | (b.requests > 129)
    assert none.any() and np.array_equal(got[0][none], b.logits[none])
    # a few of them alone, one to a workgroup
    few = slice(0, 40)
    args = {k: to_dev(getattr(b, k)) for k in names if k != "allowed"}
    alone = fasq.process_logits(to_dev(b.logits[few]), to_dev(b.requests[few]), requests_count=130, choose=True,
                                allowed=to_dev(b.allowed[few]), **args)
    assert np.array_equal(to_np(alone[0])[~none[few]], got[0][few][~none[few]])
    assert np.array_equal(to_np(alone[1])[~none[few]], got[1][few][~none[few]])
