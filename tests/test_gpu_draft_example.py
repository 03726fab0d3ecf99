"""Drafted decoding of the serving example against a plain decoder in 64 bits:
the rows of the branches that stand (read through trees, then moved in the cache),
and the tokens that follow them.  Tolerance of the rows: test_gpu_serve_example.py.
A token is the likeliest of its row's logits, or as likely within what the row's
error (that tolerance of its length, along the largest codeword rows) and fp16 leave.
"""

import numpy as np
import pytest

from oracle import pq_oracle as orc
from test_gpu_serve_example import TOL, errors, ex, plain

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


@pytest.mark.parametrize("change", [dict(), dict(window=20, page_size=12, head_dim=80, heads=6, kv_heads=3), dict(repetition=1.3, kv_heads=8)])
def test_drafted_answers(change):
    cfg = ex.Config(hidden=256, inter=384, vocab=300, max_len=200, **change)
    lengths, count, adapters = [61, 1, 97, 30], 12, [0, -1, 2, 1]
    w = ex.draw_weights(cfg, seed=3)
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, cfg.vocab, n) for n in lengths]

    def run(draft):
        dec = ex.Decoder(cfg, w, len(lengths))
        rows = ex.read_prompts(dec, prompts, adapters, 48)
        first = dec.next_tokens(torch.stack([r[-1] for r in rows]))
        return ex.answer_drafted(dec, prompts, first.tolist(), adapters, count, draft)

    alone, _, steps = run(lambda text: ([text[-1]], [-1]))
    assert steps == count

    def oracle(text):
        """Wrong guesses beside the right ones, on every level."""
        b = [i for i, p in enumerate(prompts) if len(text) > len(p) and text[:len(p)] == p.tolist()][0]
        after = alone[b][len(text) - len(prompts[b]):][:3]
        tokens, parents, node = [text[-1]], [-1], 0
        for t in after:
            tokens += [(t + 1) % cfg.vocab, t]
            parents += [node, node]
            node = len(tokens) - 1
        return tokens, parents

    said, after, steps = run(oracle)
    assert steps <= count // 2  # up to four tokens a step
    head = w["head"][0]
    dense = head[1].astype(np.float64)[orc.unpack_indices(head[0], cfg.hidden // cfg.d, cfg.bits, cfg.codewords)].reshape(cfg.vocab, -1)
    longest = np.linalg.norm(dense, axis=1).max()
    for b, p in enumerate(prompts):
        seq = np.concatenate([p, said[b]]).astype(int)
        got = after[b].cpu().numpy().astype(np.float64)
        want = plain(cfg, w, seq, adapters[b])[len(p):]
        assert len(said[b]) >= count and len(got) == len(want)
        e = errors(got, want)
        assert e.max() < TOL, (b, int(e.argmax()), e.max())
        for i in range(len(said[b]) - 1):
            x = dense @ want[i]
            if cfg.repetition != 1.0:
                met = np.unique(seq[:len(p) + i + 1])
                x[met] = np.where(x[met] > 0, x[met] / cfg.repetition, x[met] * cfg.repetition)
            slack = 2 * cfg.repetition * (TOL * np.linalg.norm(want[i]) * longest + 2.0 ** -11 * np.abs(x).max())
            assert x[said[b][i + 1]] >= x.max() - slack, (b, i)


def test_guesses():
    assert ex.guess([5, 7, 9, 5]) == ([5, 7, 9, 5], [-1, 0, 1, 2])
    assert ex.guess([1, 2]) == ([2], [-1])
    assert ex.guess([3, 1, 3, 2, 3], branches=2, depth=1) == ([3, 2, 1], [-1, 0, 0])


def test_answers_that_do_not_fit():
    cfg = ex.Config(hidden=256, inter=384, vocab=300, max_len=40, window=2, page_size=12)
    dec = ex.Decoder(cfg, ex.draw_weights(cfg, seed=3), 1)
    prompts = [np.arange(30)]
    first = dec.next_tokens(ex.read_prompts(dec, prompts, [-1], 48)[0][-1:]).tolist()
    alone = lambda text: ([text[-1]], [-1])
    with pytest.raises(ValueError, match="at most 40"):
        ex.answer_drafted(dec, prompts, first, [-1], 11, alone)
    with pytest.raises(ValueError, match="window"):
        ex.answer_drafted(dec, prompts, first, [-1], 10, lambda text: ([text[-1], 1, 2], [-1, 0, 1]))
    said, _, steps = ex.answer_drafted(dec, prompts, first, [-1], 10, alone)  # the longest there can be
    assert steps == 10 and len(said[0]) == 10
