"""Refusals of the entry points between the projections: bad arguments return
a status and a text before anything touches the GPU."""

import ctypes
import os

import pytest

import paper_2605_04084_amd as fasq

DUMMY = 0x1000  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fasq.LIB_PATH):
        from paper_2605_04084_amd import _build

        _build.build()
    return fasq.lib()


def _cache(**kw):
    a = dict(k=DUMMY, v=DUMMY, num_pages=4, page_size=16, page_stride=16 * 2 * 64, slot_stride=2 * 64, head_stride=64)
    a.update(kw)
    return fasq.KvCache(*[a[f] for f, _ in fasq.KvCache._fields_])


def _refused(status, why, code=fasq.FASQ_ERR_INVALID_ARG):
    assert status == code, fasq.last_error()
    assert why in fasq.last_error()


@pytest.mark.parametrize("args,why", [
    (dict(half=0), "half"), (dict(half=129), "half"), (dict(positions=0), "positions"), (dict(table=0), "NULL"),
    (dict(table=DUMMY + 4), "8-byte"),
])
def test_rope_table_refuses(L, args, why):
    a = dict(half=4, positions=8, table=DUMMY)
    a.update(args)
    w = (ctypes.c_double * 129)()
    _refused(L.fasq_rope_table(w, a["half"], a["positions"], 1.0, a["table"], 0), why)
    _refused(L.fasq_rope_table(None, 4, 8, 1.0, DUMMY, 0), "NULL")


def _rope(L, **kw):
    a = dict(q=DUMMY, qs=256, qh=64, Hq=4, qo=DUMMY, qos=256, qoh=64, k=DUMMY, ks=128, kh=64, v=DUMMY, vs=128, vh=64,
             Hkv=2, T=3, D=64, table=DUMMY, rows=100, rot=64, inter=0, pos=DUMMY, slots=DUMMY, qn=0, kn=0, eps=1e-6,
             cache=_cache())
    a.update(kw)
    return L.fasq_rope_append(*a.values(), 0)


@pytest.mark.parametrize("args,why", [
    (dict(T=-1), "T must"), (dict(D=0), "D must"), (dict(D=257), "D must"), (dict(rot=63), "rot must"),
    (dict(rot=66), "rot must"), (dict(qo=0), "together"), (dict(k=0), "together"),
    (dict(q=0, qo=0, k=0, v=0), "nothing to do"), (dict(Hq=0), "Hq"), (dict(Hkv=0), "Hkv"), (dict(table=0), "NULL"),
    (dict(pos=0), "NULL"), (dict(slots=0), "NULL"), (dict(rows=0), "table_positions"), (dict(table=DUMMY + 4), "8-byte"),
    (dict(q=DUMMY + 1, qo=DUMMY + 1), "2-byte"), (dict(qos=512), "strides of q"), (dict(ks=-1), "strides"),
    (dict(qn=DUMMY, eps=0.0), "eps"), (dict(kn=DUMMY, eps=float("nan")), "eps"), (dict(cache=None), "cache is NULL"),
    (dict(cache=_cache(k=None)), "cache pointer"), (dict(cache=_cache(num_pages=0)), "num_pages"),
    (dict(cache=_cache(num_pages=1 << 30)), "31 bits"), (dict(cache=_cache(head_stride=-64)), "strides"),
])
def test_rope_append_refuses(L, args, why):
    _refused(_rope(L, **args), why)


def test_no_tokens_launch_nothing(L):
    """Zero tokens are valid, also where there is no device."""
    assert _rope(L, T=0) == fasq.FASQ_OK
    assert _attend(L, T=0) == fasq.FASQ_OK
    assert _norm(L, M=0) == fasq.FASQ_OK
    assert _lora(L, M=0) == fasq.FASQ_OK
    assert L.fasq_paged_attention_workspace_bytes(0, 1, 4, 2, 64) == 0
    assert L.fasq_lora_workspace_bytes(0, 64, 8, 1) == 0


def _attend(L, **kw):
    a = dict(q=DUMMY, qs=256, qh=64, T=3, Hq=4, cache=_cache(), Hkv=2, D=64, pages=DUMMY, stride=4, max_pages=4,
             q_start=DUMMY, kv_len=DUMMY, B=1, scale=0.125, causal=1, window=0, out=DUMMY, os=256, oh=64, lse=0, ws=0,
             ws_bytes=0)
    a.update(kw)
    return L.fasq_paged_attention(*a.values(), 0)


@pytest.mark.parametrize("args,why", [
    (dict(T=-1), "T must"), (dict(B=0), "B must"), (dict(Hq=5), "multiple of Hkv"), (dict(Hkv=0), "multiple of Hkv"),
    (dict(D=0), "D must"), (dict(max_pages=0), "max_pages"), (dict(stride=-1), "stride"), (dict(window=-1), "window"),
    (dict(scale=float("nan")), "scale"), (dict(ws_bytes=-1), "workspace_bytes"), (dict(ws=DUMMY + 8), "16-byte"),
    (dict(q=0), "NULL"), (dict(out=0), "NULL"), (dict(pages=0), "NULL"), (dict(q_start=0), "NULL"),
    (dict(kv_len=0), "NULL"), (dict(cache=None), "cache is NULL"), (dict(max_pages=1 << 28), "31 bits"),
    (dict(cache=_cache(k=DUMMY + 8)), "16-byte"), (dict(cache=_cache(slot_stride=100)), "multiples of 8"),
    (dict(out=DUMMY + 1), "2-byte"), (dict(qs=-1), "strides"), (dict(T=1 << 24, Hq=256), "2^30"),
])
def test_attention_refuses(L, args, why):
    _refused(_attend(L, **args), why)


@pytest.mark.parametrize("D", [4, 60, 264])
def test_attention_head_sizes_without_a_kernel(L, D):
    _refused(_attend(L, D=D), "multiple of 8", fasq.FASQ_ERR_UNSUPPORTED)
    assert L.fasq_paged_attention_workspace_bytes(1, 1, 4, 2, D) == -1


def test_attention_workspace_refuses(L):
    for a in [(-1, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 4, 3, 64), (1, 1, 0, 1, 64)]:
        assert L.fasq_paged_attention_workspace_bytes(*a) == -1


def _norm(L, **kw):
    a = dict(x=DUMMY, y=DUMMY, M=2, N=64, post=0, gate=0, stride=0, scale=1.0, w=DUMMY, eps=1e-5, x_out=DUMMY,
             h=DUMMY + 4096)
    a.update(kw)
    return L.fasq_residual_norm(*a.values(), 0)


@pytest.mark.parametrize("args,why", [
    (dict(M=-1), "M must"), (dict(N=0), "N must"), (dict(eps=0.0), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(x=0), "NULL"), (dict(y=0, post=DUMMY), "need y"), (dict(y=0, gate=DUMMY), "need y"), (dict(w=0), "together"),
    (dict(h=0), "together"), (dict(w=0, h=0, x_out=0), "nothing to write"), (dict(h=DUMMY), "must differ"),
    (dict(gate=DUMMY, stride=32), "gate_stride"), (dict(x=DUMMY + 1), "2-byte"),
])
def test_residual_norm_refuses(L, args, why):
    _refused(_norm(L, **args), why)


def test_residual_norm_long_rows_have_no_kernel(L):
    _refused(_norm(L, N=32769), "32768", fasq.FASQ_ERR_UNSUPPORTED)


def _lora(L, **kw):
    a = dict(x=DUMMY, M=2, K=64, ids=DUMMY, pool=3, r=8, scales=DUMMY, count=2, N=(32, 16), A=(DUMMY, DUMMY),
             B=(DUMMY, DUMMY), base=(0, DUMMY), y=(DUMMY, DUMMY), ws=0, ws_bytes=0)
    a.update(kw)
    i64, vp = ctypes.c_int64 * 2, ctypes.c_void_p * 2
    for f, t in (("N", i64), ("A", vp), ("B", vp), ("base", vp), ("y", vp)):
        a[f] = None if a[f] is None else t(*a[f])
    return L.fasq_lora_batched(*a.values(), 0)


@pytest.mark.parametrize("args,why", [
    (dict(M=-1), "M must"), (dict(K=0), "K, r and L"), (dict(r=0), "K, r and L"), (dict(pool=0), "K, r and L"),
    (dict(count=0), "count"), (dict(count=9), "count"), (dict(A=None), "array is NULL"), (dict(base=None), "array is NULL"),
    (dict(x=0), "NULL"), (dict(ids=0), "NULL"), (dict(scales=0), "NULL"), (dict(N=(32, 0)), "projection 1: N"),
    (dict(A=(DUMMY, 0)), "projection 1: a buffer"), (dict(y=(0, DUMMY)), "projection 0: a buffer"),
    (dict(B=(DUMMY + 1, DUMMY)), "projection 0: fp16"), (dict(K=1 << 40), "too large"),
])
def test_lora_refuses(L, args, why):
    _refused(_lora(L, **args), why)


def test_lora_rank_without_a_kernel(L):
    _refused(_lora(L, r=257), "rank", fasq.FASQ_ERR_UNSUPPORTED)
    assert L.fasq_lora_workspace_bytes(1, 64, 257, 1) == -1


def test_binding_refuses_host_tensors(L):
    torch = pytest.importorskip("torch")
    h = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="device"):
        fasq.rope_append(h(1, 2, 8), h(1, 1, 8), h(1, 1, 8), None, None, i(1), h(1, 4, 1, 8), h(1, 4, 1, 8))
    with pytest.raises(ValueError, match="device"):
        fasq.paged_attention(h(1, 2, 8), h(1, 4, 1, 8), h(1, 4, 1, 8), i(1, 1), i(2), i(1))
    with pytest.raises(ValueError, match="device"):
        fasq.residual_norm(h(1, 8), h(1, 8), h(8))
    with pytest.raises(ValueError, match="device"):
        fasq.lora_batched(h(1, 8), i(1), [h(1, 2, 8)], [h(1, 4, 2)], torch.zeros(1), [None])
    with pytest.raises(ValueError, match="device"):
        fasq.rope_table([1.0], 4, device="cpu")
