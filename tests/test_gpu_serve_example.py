"""The serving example against a plain decoder in 64 bits.

Prompts read in steps that end inside prompts and pages, then tokens taken one
a step through a replayed graph; every output row is compared with the layers'
formulas over the whole sequence at once.

Tolerance of a row's relative L2 error: along a layer's longest chain 14
results are rounded to fp16 (norm, projection, adapter, turned head, weights,
attention, projection, sum, norm, gate and up, silu, product, projection, sum),
each by at most 2^-11 of itself, and the last norm once: 29 * 2^-11 = 1.4e-2
for two layers if all errors added up.  Scores of normed heads are about one
here, so the softmax does not enlarge them.  2e-2 covers that; a wrong
adapter, position or page changes rows by a third or more.
"""

import os
import sys

import numpy as np
import pytest

from oracle import layer_ops as ops
from oracle import pq_oracle as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
fasq = pytest.importorskip("paper_2605_04084_amd")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_decoder as ex  # noqa: E402

TOL = 2e-2


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fasq.lib()
    yield
    torch.cuda.synchronize()


def plain(cfg, w, tokens, adapter):
    """Output rows of one request's tokens, in 64 bits."""
    T = len(tokens)
    dense = {}

    def project(x, m):
        key = id(m[0])
        if key not in dense:
            ids = orc.unpack_indices(m[0], x.shape[1] // cfg.d, cfg.bits, cfg.codewords)
            dense[key] = m[1].astype(np.float64)[ids].reshape(ids.shape[0], -1)
        return x @ dense[key].T

    freq = 10000.0 ** (-2.0 * np.arange(cfg.head_dim // 2) / cfg.head_dim)
    table = ops.rope_table(freq, T)
    ad = np.full(T, adapter)
    x = w["embed"].astype(np.float64)[tokens]
    for L in w["layers"]:
        h = ops.rms_norm(x, L["norm"], cfg.eps)
        q, k, v = (ops.lora(h, ad, L["A"][i], L["B"][i], w["scales"], project(h, L["qkv"][i]))[0] for i in range(3))
        q = ops.rope(q.reshape(T, cfg.heads, -1), table, np.arange(T), False, L["q_norm"], cfg.eps)
        k = ops.rope(k.reshape(T, cfg.kv_heads, -1), table, np.arange(T), False, L["k_norm"], cfg.eps)
        v = v.reshape(T, cfg.kv_heads, -1)
        a, _, _ = ops.paged_attention(q, k[None], v[None], np.array([[0]]), [0, T], [T], cfg.head_dim ** -0.5,
                                      window=cfg.window)
        x = x + project(a.reshape(T, -1), L["o"][0])
        h = ops.rms_norm(x, L["mlp_norm"], cfg.eps)
        gate, up = project(h, L["gate_up"][0]), project(h, L["gate_up"][1])
        x = x + project(gate / (1 + np.exp(-gate)) * up, L["down"][0])
    return ops.rms_norm(x, w["norm"], cfg.eps)


def errors(got, want):
    return np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)


@pytest.mark.parametrize("change,chunk", [
    (dict(), 48),
    (dict(window=20, page_size=12, head_dim=80, heads=6, kv_heads=3), 33),
    (dict(kv_heads=8, page_size=64, rank=5), 500),
])
def test_example_matches_plain_decoder(change, chunk):
    cfg = ex.Config(hidden=256, inter=384, vocab=300, max_len=160, **change)
    lengths, count = [61, 1, 97, 16, 33], 8
    adapters = [0, -1, 2, 1, 0]
    w = ex.draw_weights(cfg, seed=3)
    dec = ex.Decoder(cfg, w, len(lengths))
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, cfg.vocab, n) for n in lengths]
    rows = ex.read_prompts(dec, prompts, adapters, chunk)
    first = dec.next_tokens(torch.stack([r[-1] for r in rows]))
    tokens, after = ex.answer(dec, lengths, first, adapters, count)
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        said = tokens[b].cpu().numpy()
        got = np.concatenate([rows[b].cpu().numpy(), after[b].cpu().numpy()]).astype(np.float64)
        seq = np.concatenate([prompts[b], said])
        want = plain(cfg, w, seq, adapters[b])
        e = errors(got, want)
        assert e.max() < TOL, (b, int(e.argmax()), e.max())
        # the comparison notices another adapter
        other = errors(got, plain(cfg, w, seq, (adapters[b] + 2) % cfg.adapters))
        assert other.max() > 5 * TOL
