"""rope_table and rope_append against the fp64 definitions.

Tolerance: the result is formed in fp32 and rounded to fp16 once: half a unit
in the last place of the value (2^-11 of it, 2^-25 among the subnormals), and
2^-20 of the two values of its pair for the fp32 arithmetic (products, the sum
of squares of up to 256 values, one root and one division).
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


def _check(got, ref, pair):
    got = got.astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    tol = np.abs(ref) * 2.0 ** -11 * 1.001 + 2.0 ** -25 + 2.0 ** -20 * pair
    err = np.abs(got - ref)
    bad = ~(err <= tol) & ~np.isnan(ref)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(err - tol)))


def _pair(x, norm, eps, rot, interleaved):
    """|x_a| + |x_b| of each value's pair (the value's own size behind them)."""
    y = np.abs(lo.rms_norm(x, norm, eps) if norm is not None else x.astype(np.float64))
    p = y.copy()
    half = rot // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        p[..., a] = p[..., b] = y[..., a] + y[..., b]
    return p


@pytest.mark.parametrize("positions,half,base,scale", [(1, 1, 100.0, 1.0), (131072, 8, 500000.0, 1.0), (777, 128, 1e4, 1.25)])
def test_table(positions, half, base, scale):
    w = [base ** (-i / half) for i in range(half)]
    got = to_np(fasq.rope_table(w, positions, scale)).astype(np.float64)
    ref = lo.rope_table(w, positions, scale)
    # one rounding to fp32, and 1e-15 per radian for the 64-bit angle
    assert (np.abs(got - ref) <= 2.0 ** -24 * 1.001 * np.abs(ref) + scale * (positions * 3e-16 + 2.0 ** -60)).all()


CASES = [
    # T, Hq, Hkv, D, rot, interleaved, norm, page_size
    (1, 32, 8, 128, 128, False, False, 16),
    (1, 1, 1, 128, 128, True, True, 1),
    (7, 4, 2, 64, 64, False, True, 16),
    (5, 6, 2, 64, 64, True, False, 20),
    (33, 3, 1, 80, 80, False, False, 16),
    (9, 2, 2, 80, 32, False, True, 5),
    (9, 2, 2, 96, 24, True, True, 7),
    (3, 8, 8, 256, 256, False, True, 64),
    (3, 7, 1, 256, 128, True, False, 64),
    (4, 3, 1, 72, 40, False, True, 16),   # pairs not in chunks of 8: one value a lane
    (4, 3, 1, 50, 50, True, False, 16),   # D not a multiple of 8
    (2, 2, 1, 5, 2, False, True, 3),
    (6, 2, 2, 200, 6, True, True, 9),
    (300, 5, 1, 128, 64, False, True, 32),
]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,interleaved,norm,size", CASES)
@pytest.mark.parametrize("fused", [False, True])
def test_append(T, Hq, Hkv, D, rot, interleaved, norm, size, fused):
    rng = np.random.default_rng(T * 1000 + D + rot)
    qkv = _half(rng, (T, Hq + 2 * Hkv, D))
    positions = rng.integers(0, 4000, T).astype(np.int32)
    pages = -(-T // size) + 2
    slots = rng.permutation(pages * size)[:T].astype(np.int32)
    table = lo.rope_table([1e4 ** (-2 * i / rot) for i in range(rot // 2)], 4000).astype(np.float32)
    kc, vc = _half(rng, (pages, size, Hkv, D)), _half(rng, (pages, size, Hkv, D))
    wq, wk = (_half(rng, (D,)), _half(rng, (D,))) if norm else (None, None)
    dev = to_dev(qkv)
    parts = [dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]]
    if not fused:
        parts = [p.contiguous() for p in parts]
    kd, vd = to_dev(kc), to_dev(vc)
    out = fasq.rope_append(*parts, to_dev(table), to_dev(positions), to_dev(slots), kd, vd, interleaved,
                           to_dev(wq) if norm else None, to_dev(wk) if norm else None, 1e-5)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    _check(to_np(out), lo.rope(q, table, positions, interleaved, wq, 1e-5), _pair(q, wq, 1e-5, rot, interleaved))
    ref = lo.append(kc, lo.rope(k, table, positions, interleaved, wk, 1e-5), slots)
    pair = lo.append(np.zeros(kc.shape), _pair(k, wk, 1e-5, rot, interleaved), slots)
    _check(to_np(kd), ref, pair)
    assert np.array_equal(to_np(vd), lo.append(vc, v, slots).astype(np.float16))
    if fused:  # in place over the projections' buffer
        got = fasq.rope_append(*parts, to_dev(table), to_dev(positions), to_dev(slots), kd, vd, interleaved,
                               to_dev(wq) if norm else None, to_dev(wk) if norm else None, 1e-5, out=parts[0])
        assert got is parts[0] and torch.equal(got, out)
        assert np.array_equal(to_np(dev[:, Hq:]), qkv[:, Hq:])


@pytest.mark.parametrize("D", [128, 50])
def test_padding_slots_and_positions_outside(D):
    rng = np.random.default_rng(5)
    T, H, size, pages = 6, 2, 4, 3
    q, k, v = _half(rng, (T, H, D)), _half(rng, (T, H, D)), _half(rng, (T, H, D))
    positions = np.array([0, -1, 64, 63, 5, 2 ** 31 - 1], dtype=np.int32)
    slots = np.array([0, 1, 2, -1, pages * size, 11], dtype=np.int32)
    rot = D // 16 * 16
    table = lo.rope_table([1e4 ** (-2 * i / rot) for i in range(rot // 2)], 64).astype(np.float32)
    kc = np.zeros((pages, size, H, D), np.float16)
    kd, vd = to_dev(kc), to_dev(kc)
    out = fasq.rope_append(to_dev(q), to_dev(k), to_dev(v), to_dev(table), to_dev(positions), to_dev(slots), kd, vd)
    ref = lo.rope(q, table, positions, False)
    _check(to_np(out), ref, _pair(q, None, 0, rot, False))
    assert np.isnan(to_np(out)[[1, 2, 5]]).all()
    _check(to_np(kd), lo.append(kc, lo.rope(k, table, positions, False), slots),
           lo.append(np.zeros(kc.shape), _pair(k, None, 0, rot, False), slots))
    assert np.array_equal(to_np(vd), lo.append(kc, v, slots).astype(np.float16))


def test_parts_alone_and_no_rotation():
    rng = np.random.default_rng(6)
    T, H, D, size = 5, 3, 64, 8
    q, k, v = (to_dev(_half(rng, (T, H, D))) for _ in range(3))
    table = to_dev(lo.rope_table([1e4 ** (-2 * i / D) for i in range(D // 2)], 64).astype(np.float32))
    positions, slots = to_dev(np.arange(T, dtype=np.int32)), to_dev(np.arange(T, dtype=np.int32))
    caches = [torch.zeros((2, size, H, D), dtype=torch.float16, device="cuda:0") for _ in range(4)]
    both = fasq.rope_append(q, k, v, table, positions, slots, caches[0], caches[1])
    assert torch.equal(fasq.rope_append(q, None, None, table, positions, None, None, None), both)
    assert fasq.rope_append(None, k, v, table, positions, slots, caches[2], caches[3]) is None
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    assert torch.equal(fasq.rope_append(q, k, v, None, None, slots, caches[0], caches[1]), q)
    assert torch.equal(caches[0].view(-1, H, D)[:T], k)
    empty = fasq.rope_append(q[:0], k[:0], v[:0], table, positions[:0], slots[:0], caches[0], caches[1])
    assert tuple(empty.shape) == (0, H, D)


def test_cache_with_heads_before_slots_and_far_pages():
    """[pages x heads x page_size x D] through a view, in pages past 2^32 elements."""
    rng = np.random.default_rng(7)
    T, H, D, size = 4, 8, 128, 16
    pages = 2 ** 32 // (H * size * D) + 8
    kc = torch.empty((pages, H, size, D), dtype=torch.float16, device="cuda:0")
    vc = torch.empty_like(kc)
    last = [pages - 1, 3, pages - 2, 0]
    for p in last:
        kc[p] = 0
        vc[p] = 0
    k, v = _half(rng, (T, H, D)), _half(rng, (T, H, D))
    slots = np.array([p * size + i for i, p in enumerate(last)], dtype=np.int32)
    fasq.rope_append(None, to_dev(k), to_dev(v), None, None, to_dev(slots), kc.transpose(1, 2), vc.transpose(1, 2))
    for i, p in enumerate(last):
        assert np.array_equal(to_np(kc[p, :, i]), k[i]) and np.array_equal(to_np(vc[p, :, i]), v[i])
        assert int(torch.count_nonzero(kc[p])) == np.count_nonzero(k[i])


def test_binding_refuses():
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda:0")  # noqa: E731
    q, k, c = h(3, 4, 64), h(3, 2, 64), h(2, 8, 2, 64)
    table = torch.zeros((9, 32, 2), device="cuda:0")
    ok = dict(q=q, k=k, v=k, table=table, positions=i(3), slots=i(3), k_cache=c, v_cache=c)
    for change, error in [(dict(q=None, k=None, v=None), ValueError), (dict(v=None), ValueError), (dict(v=h(3, 1, 64)), ValueError),
                          (dict(slots=i(2)), ValueError), (dict(slots=i(3).long()), TypeError), (dict(positions=i(4)), ValueError),
                          (dict(table=torch.zeros((9, 33, 2), device="cuda:0")), ValueError), (dict(table=table.half()), TypeError),
                          (dict(k_cache=h(2, 8, 1, 64)), ValueError), (dict(v_cache=h(2, 8, 64, 2).transpose(2, 3)), ValueError),
                          (dict(q=q.float()), TypeError), (dict(q=h(3, 64, 4).transpose(1, 2)), ValueError),
                          (dict(q_norm=h(32)), ValueError), (dict(out=h(3, 4, 32)), ValueError)]:
        with pytest.raises(error):
            fasq.rope_append(**{**ok, **change})
