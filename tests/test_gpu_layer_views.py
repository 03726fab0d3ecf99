"""Strides at their edges in the entry points between projections: broadcast
inputs, and outputs that may not be.
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
