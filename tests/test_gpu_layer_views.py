"""Strides at their edges in the entry points between projections: caches with
dimensions of one, whose strides mean nothing, and broadcast inputs.
"""

import pytest

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


def _i32(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda:0")


def _rand(*s):
    return torch.randn(s, device="cuda:0").half()


def _restride(t, strides):
    """The same values with other strides, in a buffer of their own."""
    room = 1 + sum((n - 1) * s for n, s in zip(t.shape, strides))
    out = torch.zeros(room, dtype=t.dtype, device=t.device).as_strided(t.shape, strides)
    return out.copy_(t)


@pytest.mark.parametrize("shape", [(3, 1, 2, 64), (1, 16, 2, 64), (3, 16, 1, 64), (1, 1, 1, 64), (1, 20, 1, 64)])
def test_dimensions_of_one(shape):
    """Both caches hold the same layout; the strides of their single pages,
    slots or heads differ, and are no multiples of 8."""
    pages, size, H, D = shape
    n = pages * size
    k, v, q = _rand(*shape), _rand(*shape), _rand(1, 2 * H, D)
    table = torch.arange(pages, dtype=torch.int32, device="cuda:0")[None]
    args = (table, _i32(0, 1), _i32(n))
    new = _rand(1, H, D), _rand(1, H, D), _i32(n - 1)
    fasq.rope_append(None, *new[:2], None, None, new[2], k, v)
    want = fasq.paged_attention(q, k, v, *args)
    for odd_k, odd_v in ((13, 7), (0, 5)):
        strides = [[s if m > 1 else odd for m, s in zip(shape[:3], k.stride())] + [1] for odd in (odd_k, odd_v)]
        k2, v2 = _restride(k, strides[0]), _restride(v, strides[1])
        assert torch.equal(fasq.paged_attention(q, k2, v2, *args), want)
        fasq.rope_append(None, new[1], new[0], None, None, new[2], k2, v2)
        assert torch.equal(k2.flatten(0, 1)[n - 1], new[1][0]) and torch.equal(v2.flatten(0, 1)[n - 1], new[0][0])
        assert torch.equal(k2.flatten(0, 1)[:n - 1], k.flatten(0, 1)[:n - 1])


def test_caches_of_different_layout_are_refused():
    k = _rand(3, 16, 2, 64)
    v = _rand(3, 2, 16, 64).transpose(1, 2)
    with pytest.raises(ValueError, match="strides"):
        fasq.paged_attention(_rand(1, 4, 64), k, v, _i32(0, 1, 2)[None], _i32(0, 1), _i32(40))


def test_broadcast_inputs_and_outputs():
    """Inputs may be expanded; what is written may not."""
    k, v, q = _rand(3, 16, 2, 64), _rand(3, 16, 2, 64), _rand(1, 1, 64)
    args = (_i32(0, 1, 2)[None], _i32(0, 5), _i32(48))
    wide = q.expand(5, 4, 64)
    want = fasq.paged_attention(wide.contiguous(), k, v, *args)
    assert torch.equal(fasq.paged_attention(wide, k, v, *args), want)
    one = _rand(1, 1, 1, 64).expand(3, 16, 2, 64)
    same = fasq.paged_attention(wide, one, one, *args)
    assert torch.equal(same, fasq.paged_attention(wide, one.contiguous(), one.contiguous(), *args))
    slots = torch.arange(5, dtype=torch.int32, device="cuda:0")
    out = fasq.rope_append(wide, wide[:, :2], wide[:, :2], None, None, slots, k, v)
    assert torch.equal(out, wide) and torch.equal(k.view(-1, 2, 64)[:5], wide[:, :2])
    with pytest.raises(fasq.FasqError, match="overlap"):
        fasq.paged_attention(wide, k, v, *args, out=torch.zeros((1, 4, 64), dtype=torch.float16, device="cuda:0").expand(5, 4, 64))
    with pytest.raises(fasq.FasqError, match="overlap"):
        fasq.rope_append(wide, wide[:, :2], wide[:, :2], None, None, slots, one, one)
