"""Calls of more rows than one launch holds (2^32 threads in a grid): the
sizes that the entry points accept are computed whole.
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
    torch.cuda.empty_cache()


def _pattern(n, period=257):
    """[n x 1] fp16 values that differ from row to row."""
    return ((torch.arange(n, device="cuda:0") % period).half() / 64 - 1)[:, None]


def test_rope_of_many_small_heads():
    """2^26 heads and some, a wave each; and keys and values alone."""
    T, H, D = 2 ** 21 + 5, 32, 2
    q = _pattern(T).expand(T, H * D).reshape(T, H, D).contiguous()
    table = torch.tensor([[[0.0, 1.0]]], device="cuda:0")  # a quarter turn
    positions = torch.zeros(T, dtype=torch.int32, device="cuda:0")
    out = fasq.rope_append(q, None, None, table, positions, None, None, None)
    assert torch.equal(out[..., 0], -q[..., 1]) and torch.equal(out[..., 1], q[..., 0])
    slots = torch.arange(T, dtype=torch.int32, device="cuda:0")
    k, v = (torch.zeros((T, 1, H // 2, D), dtype=torch.float16, device="cuda:0") for _ in range(2))
    part = q[:, :H // 2].contiguous()
    fasq.rope_append(None, part, part, None, None, slots, k, v)
    assert torch.equal(k.view_as(part), part) and torch.equal(v.view_as(part), part)


def test_norm_of_many_rows():
    """2^24 rows by 256 threads each; 2^22 by 1024."""
    for M, N in ((2 ** 24, 520), (2 ** 22 + 3, 4104)):
        x = _pattern(M).expand(M, N).contiguous()
        w = torch.ones(N, dtype=torch.float16, device="cuda:0")
        small = x[:1000].clone()
        _, h = fasq.residual_norm(x, weight=w, out=x)
        _, want = fasq.residual_norm(small, weight=w)
        assert h is x and torch.equal(h[:514], want[:514])
        for m0 in (2 ** 20, M // 2, M - 600):  # the rows repeat
            m0 = m0 // 257 * 257
            n = min(257, M - m0)
            assert torch.equal(h[m0:m0 + n], want[:n])
        del x, h


def test_adapters_of_many_tokens():
    """The low-rank values of 2^26 (token, projection) pairs and more, folded by a wave each."""
    M, K, r, count = 2 ** 23 + 2, 1, 17, 8
    x = _pattern(M)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda:0")
    A = torch.ones((1, r, K), dtype=torch.float16, device="cuda:0")
    B = torch.full((1, 1, r), 1 / 16, dtype=torch.float16, device="cuda:0")
    ys = fasq.lora_batched(x, ids, [A] * count, [B] * count, torch.ones(1, device="cuda:0"), [None] * count)
    want = (x.float() * (r / 16)).half()
    assert all(torch.equal(y, want) for y in ys)


def test_attention_of_many_whole_tiles():
    """2^24 tiles of 128 tokens and some; every token sees the same 16 keys."""
    T, H, D = 2 ** 20 + 9, 2049, 8
    q = torch.zeros((T, H, D), dtype=torch.float16, device="cuda:0")
    k, v = (torch.randn((1, 16, H, D), device="cuda:0").half() for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda:0")
    pages, kv_len = torch.zeros((1, 1), **i32), torch.tensor([16], **i32)

    def run(q):
        return fasq.paged_attention(q, k, v, pages, torch.tensor([0, q.shape[0]], **i32), kv_len, causal=False, out=torch.full_like(q, 7))

    want = run(q[:200])[:1].clone()
    assert torch.allclose(want[0].float(), v[0].float().mean(0), atol=2e-3)
    out = run(q)
    for part in out.split(2 ** 16):
        assert bool((part == want).all())


@pytest.mark.parametrize("split", [True, False])
def test_attention_of_the_most_requests(split):
    """2^16 requests of a token and a key each: the key's value."""
    B, H, D = 2 ** 16, 2, 8
    q, k = (torch.randn(s, device="cuda:0").half() for s in ((B, 2 * H, D), (B, 1, H, D)))
    v = torch.randn((B, 1, H, D), device="cuda:0").half()
    i32 = dict(dtype=torch.int32, device="cuda:0")
    pages = torch.randperm(B, **i32)[:, None]
    kw = {} if split else {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda:0")}
    out = fasq.paged_attention(q, k, v, pages, torch.arange(B + 1, **i32), torch.ones(B, **i32), **kw)
    want = v[pages[:, 0].long(), 0].repeat_interleave(2, dim=1)
    assert torch.equal(out, want)


@pytest.mark.parametrize("N", [2 ** 28 + 5, 2 ** 31 - 2 ** 17])
def test_adapters_of_the_widest_projections(N):
    """As many features as a projection may have: blocks of them beyond 65535 in y."""
    x = torch.full((1, 1), 2.0, dtype=torch.float16, device="cuda:0")
    ids = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    A = torch.ones((1, 1, 1), dtype=torch.float16, device="cuda:0")
    B = torch.empty((1, N, 1), dtype=torch.float16, device="cuda:0")
    B.view(-1)[:] = torch.arange(257, device="cuda:0").half().repeat(-(-N // 257))[:N]
    y, = fasq.lora_batched(x, ids, [A], [B], torch.ones(1, device="cuda:0"), [None])
    assert torch.equal(y[0], B.view(-1) * 2)
