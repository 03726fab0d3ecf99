"""residual_norm and lora_batched against the fp64 definitions.

Tolerances.  Each output is rounded to fp16 once: half a unit in the last
place (2^-11 of it; 2^-25 among the subnormals).  Norms: 2^-17 of |x| +
|scale gate u| for fp32 sums over a row of up to 32768 values (256 threads and
more: sums of at most 128 terms in turn) and for x_new's cancellation.
Adapters: 2^-16 of |s| |B| (|A| |x|), for sums of at most 256 terms in turn
and low-rank values held to 22 bits.
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


def _close(got, ref, slack):
    got = got.astype(np.float64)
    tol = np.abs(ref) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + slack
    err = np.abs(got - ref)
    assert (err <= tol).all(), (int((err > tol).sum()), float((err - tol).max()))


# ---------------------------------------------------------------------------
# residual_norm
# ---------------------------------------------------------------------------

def _norm_case(M, N, post, gate, scale, seed=0, eps=1e-5):
    rng = np.random.default_rng(seed + N)
    x, y = _half(rng, (M, N), 2.0), _half(rng, (M, N))
    w = _half(rng, (N,))
    p = _half(rng, (N,)) if post else None
    g = _half(rng, {"channel": (N,), "token": (M, N)}[gate]) if gate else None
    d = lambda t: None if t is None else to_dev(t)  # noqa: E731
    args = (d(x), d(y), d(w), eps)
    kw = dict(post_weight=d(p), gate=d(g), scale=scale)
    ref_x, ref_h = lo.residual_norm(x, y, w, eps, p, g, scale)
    mag = np.abs(x).astype(np.float64) + np.abs(ref_x - x)
    rms = np.sqrt(np.mean(ref_x ** 2, axis=1, keepdims=True) + eps)
    return args, kw, ref_x, ref_h, mag * 2.0 ** -17, mag / rms * np.abs(w).astype(np.float64) * 2.0 ** -17


@pytest.mark.parametrize("N", [1, 7, 8, 63, 64, 100, 512, 513, 1003, 2048, 2056, 4096, 5120, 8192, 8193, 14336, 16392, 32767, 32768])
@pytest.mark.parametrize("M,post,gate,scale", [(1, False, None, 1.0), (5, True, "channel", 0.3), (3, True, "token", -2.0),
                                               (2, False, "channel", 1.0)])
def test_residual_norm(N, M, post, gate, scale):
    args, kw, ref_x, ref_h, sx, sh = _norm_case(M, N, post, gate, scale)
    x_new, h = fasq.residual_norm(*args, **kw)
    _close(to_np(x_new), ref_x, sx)
    _close(to_np(h), ref_h, sh)
    # in place: the stream over x, the norm over y
    x, y, w, eps = args
    a, b = fasq.residual_norm(x, y, w, eps, x_out=x, out=y, **kw)
    assert a is x and b is y and torch.equal(a, x_new) and torch.equal(b, h)


def test_norm_alone_and_sum_alone():
    (x, y, w, eps), kw, ref_x, _, sx, _ = _norm_case(4, 640, False, None, 0.5)
    none, h = fasq.residual_norm(x, weight=w)
    assert none is None
    xs = to_np(x).astype(np.float64)
    _close(to_np(h), lo.rms_norm(xs, to_np(w), 1e-5), np.abs(lo.rms_norm(xs, to_np(w), 1e-5)) * 2.0 ** -17)
    x_new, none = fasq.residual_norm(x, y, scale=0.5)
    assert none is None
    _close(to_np(x_new), ref_x, sx)
    a, b = fasq.residual_norm(x[:0], y[:0], w)
    assert tuple(a.shape) == (0, 640) and tuple(b.shape) == (0, 640)


def test_norm_rows_do_not_mix_and_infinities_stay_in_their_row():
    (x, y, w, eps), kw, *_ = _norm_case(6, 1000, True, "channel", 1.0)
    whole = fasq.residual_norm(x, y, w, eps, **kw)
    x2 = x.clone()
    x2[2, 5], x2[4, 7] = float("inf"), float("nan")
    got = fasq.residual_norm(x2, y, w, eps, **kw)
    keep = [0, 1, 3, 5]
    for a, b in zip(whole, got):
        assert torch.equal(a[keep], b[keep])
    assert torch.isinf(got[0][2, 5]) and torch.isnan(got[1][2, 5]) and (got[1][2, :5] == 0).all()
    assert torch.isnan(got[1][4]).all()


def test_norm_unaligned_rows():
    rng = np.random.default_rng(3)
    buf, w = to_dev(_half(rng, (1 + 4 * 256,))), to_dev(_half(rng, (256,)))
    x = buf[1:].view(4, 256)
    _, h = fasq.residual_norm(x, weight=w)
    ref = lo.rms_norm(to_np(x), to_np(w), 1e-5)
    _close(to_np(h), ref, np.abs(ref) * 2.0 ** -17)


def test_norm_binding_refuses():
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    x = h(2, 8)
    for kw, error in [(dict(y=h(2, 9)), ValueError), (dict(weight=h(9)), ValueError), (dict(y=x, weight=h(8), gate=h(3, 8)), ValueError),
                      (dict(y=h(8, 2).t()), ValueError), (dict(weight=h(8).float()), TypeError), (dict(weight=h(8), out=h(3, 8)), ValueError),
                      (dict(), fasq.FasqError), (dict(weight=h(8), gate=h(8)), fasq.FasqError), (dict(weight=h(8), eps=0.0), fasq.FasqError)]:
        with pytest.raises(error):
            fasq.residual_norm(x, **kw)


# ---------------------------------------------------------------------------
# lora_batched
# ---------------------------------------------------------------------------

def _lora_case(M, K, Ns, r, L, ids, seed=0, a_std=None):
    rng = np.random.default_rng(seed + M * 7 + K)
    x = _half(rng, (M, K))
    if ids == "random":
        ids = rng.integers(-1, L + 1, M)  # both ends lie outside the pool
    elif ids == "blocks":
        ids = np.repeat(rng.integers(0, L, 4), -(-M // 4))[:M]
    elif ids == "none":
        ids = np.full(M, -1)
    ids = np.asarray(ids, dtype=np.int32)
    As = [_half(rng, (L, r, K), a_std or K ** -0.5) for _ in Ns]
    Bs = [_half(rng, (L, N, r), 0.3) for N in Ns]
    scales = rng.uniform(-2, 2, L).astype(np.float32)
    bases = [_half(rng, (M, N)) for N in Ns]
    return x, ids, As, Bs, scales, bases


def _run_lora(x, ids, As, Bs, scales, bases):
    got = fasq.lora_batched(to_dev(x), to_dev(ids), [to_dev(a) for a in As], [to_dev(b) for b in Bs], to_dev(scales),
                            [None if b is None else to_dev(b) for b in bases])
    return [to_np(g) for g in got]


def _check_lora(case, got):
    x, ids, As, Bs, scales, bases = case
    for g, A, B, base in zip(got, As, Bs, bases):
        ref, mass = lo.lora(x, ids, A, B, scales, base)
        _close(g, ref, mass * 2.0 ** -16)


LORA = [
    # M, K, Ns, r, L, ids
    (1, 512, (256,), 16, 3, [2]),
    (1, 4096, (1024, 256, 256), 16, 4, [1]),
    (1, 1, (1,), 1, 1, [0]),
    (3, 64, (64,), 8, 3, [-1, 3, -1]),           # no token has an adapter
    (16, 1024, (512, 128), 16, 16, "random"),
    (16, 1024, (512,), 64, 40, "random"),
    (17, 1000, (96, 40, 8), 16, 5, "random"),
    (37, 1516, (1003,), 10, 5, "random"),
    (37, 333, (77, 5), 3, 2, "random"),
    (64, 256, (144,), 32, 1, "random"),
    (65, 520, (200,), 20, 7, "blocks"),
    (100, 768, (264,), 100, 3, "random"),
    (130, 640, (1000, 72), 16, 9, "blocks"),
    (200, 512, (272,), 256, 2, "blocks"),
    (300, 1024, (528,), 64, 5, "random"),
    (513, 320, (130,), 8, 600, "random"),        # more adapters than tokens
    (33, 4100, (24,), 33, 4, "random"),
    (20, 264, (64, 48, 40, 32, 24, 16, 8, 1), 8, 3, "random"),
]


@pytest.mark.parametrize("M,K,Ns,r,L,ids", LORA)
def test_lora(M, K, Ns, r, L, ids):
    case = _lora_case(M, K, Ns, r, L, ids)
    got = _run_lora(*case)
    _check_lora(case, got)
    again = _run_lora(*case)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))


def test_lora_without_base_and_in_place():
    x, ids, As, Bs, scales, bases = _lora_case(21, 320, (136, 64), 16, 4, "random")
    case = (x, ids, As, Bs, scales, [None, bases[1]])
    _check_lora(case, _run_lora(*case))
    ys = [to_dev(b) for b in bases]
    got = fasq.lora_batched(to_dev(x), to_dev(ids), [to_dev(a) for a in As], [to_dev(b) for b in Bs], to_dev(scales), ys, outs=ys)
    assert all(g is y for g, y in zip(got, ys))
    _check_lora((x, ids, As, Bs, scales, bases), [to_np(y) for y in ys])
    assert all(np.array_equal(to_np(y)[m], b[m]) for y, b in zip(ys, bases) for m in range(21) if not 0 <= ids[m] < 4)


def test_lora_tokens_do_not_mix():
    """Infinite and NaN activations, adapters and bases stay with their own token."""
    x, ids, As, Bs, scales, bases = _lora_case(40, 264, (72,), 16, 6, "random")
    ids[:] = np.arange(40) % 6
    whole = _run_lora(x, ids, As, Bs, scales, bases)[0]
    x[3, 5], x[10, 0] = np.inf, np.nan  # adapters 3 and 4
    As[0][2, 3, 7], Bs[0][5, 11, 2], scales[1] = np.nan, np.inf, np.inf
    got = _run_lora(x, ids, As, Bs, scales, bases)[0]
    for m in range(40):
        if m in (3, 10) or ids[m] in (1, 2):
            assert not np.isfinite(got[m]).any()
        elif ids[m] == 5:
            assert np.array_equal(np.delete(got[m], 11), np.delete(whole[m], 11)) and not np.isfinite(got[m, 11])
        else:
            assert np.array_equal(got[m], whole[m])


@pytest.mark.parametrize("a_std,b_std", [(600.0, 0.002), (2e-5, 30.0)])
def test_lora_low_rank_values_outside_fp16(a_std, b_std):
    """A x beyond fp16's largest value, and far below its smallest normal one."""
    x, ids, As, Bs, scales, bases = _lora_case(19, 4096, (64,), 16, 3, "random", a_std=a_std)
    Bs = [(b.astype(np.float32) / 0.3 * b_std).astype(np.float16) for b in Bs]
    if a_std < 1:
        x = (x.astype(np.float32) * 2.0 ** -8).astype(np.float16)
    case = (x, ids, As, Bs, scales, [None])
    got = _run_lora(*case)
    ref = lo.lora(x, ids, As[0], Bs[0], scales)[0]
    assert np.isfinite(got[0]).all() and np.abs(ref).max() > 1e-3
    _check_lora(case, got)


def test_lora_unaligned_rows():
    x, ids, As, Bs, scales, bases = _lora_case(18, 256, (64,), 16, 3, "random")
    buf = to_dev(np.concatenate([[np.float16(0)], x.ravel()]))
    got = fasq.lora_batched(buf[1:].view(18, 256), to_dev(ids), [to_dev(As[0])], [to_dev(Bs[0])], to_dev(scales), [to_dev(bases[0])])
    _check_lora((x, ids, As, Bs, scales, bases), [to_np(got[0])])


def test_lora_binding_refuses():
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    ids, scales = torch.zeros(2, dtype=torch.int32, device="cuda:0"), torch.zeros(3, device="cuda:0")
    ok = dict(x=h(2, 16), adapters=ids, As=[h(3, 4, 16)], Bs=[h(3, 8, 4)], scales=scales, bases=[h(2, 8)])
    small = torch.zeros(4, dtype=torch.uint8, device="cuda:0")
    for change, error in [(dict(As=[]), ValueError), (dict(As=[h(3, 4, 15)]), ValueError), (dict(Bs=[h(3, 8, 5)]), ValueError),
                          (dict(Bs=[h(2, 8, 4)]), ValueError), (dict(bases=[h(2, 7)]), ValueError), (dict(adapters=ids.long()), TypeError),
                          (dict(adapters=ids[:1]), ValueError), (dict(scales=scales.half()), TypeError), (dict(outs=[h(1, 8)]), ValueError),
                          (dict(workspace=small), fasq.FasqError)]:
        with pytest.raises(error):
            fasq.lora_batched(**{**ok, **change})
    assert tuple(fasq.lora_batched(h(0, 16), ids[:0], ok["As"], ok["Bs"], scales, [h(0, 8)])[0].shape) == (0, 8)


@pytest.mark.parametrize("M,K,Ns,r,L,ids", [
    # blocks of 128 tokens (many features), of 64 and of 16, each beyond 128 tokens
    (1030, 128, (22016,), 40, 3, "blocks"),
    (1025, 136, (11011, 11003), 33, 4, "random"),
    (1030, 72, (22016,), 130, 3, "random"),
    (1000, 256, (520, 64), 17, 6, "random"),
    (193, 1000, (1531,), 20, 3, "random"),
    (320, 200, (136,), 129, 2, "blocks"),
    (1000, 333, (264, 5), 16, 5, "random"),
    (2051, 64, (72,), 1, 9, "blocks"),
])
def test_lora_blocks(M, K, Ns, r, L, ids):
    case = _lora_case(M, K, Ns, r, L, ids)
    got = _run_lora(*case)
    _check_lora(case, got)
    again = _run_lora(*case)
    assert all(np.array_equal(a.view(np.uint16), b.view(np.uint16)) for a, b in zip(got, again))
