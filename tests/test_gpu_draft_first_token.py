"""The serving example's first drafted token: the penalty for tokens that occur holds
from the first one on, over the prompt.

The logits are formed in 64 bits from the rows that the example itself has read.  A logit of
the example is off by 2^-11 of itself (fp16) and by at most 2^-14 of its products' sum (fp32
sums of 512 products), penalised ones by as much times the penalty: two of them are told apart
beyond twice that.
"""

import sys

import numpy as np
import pytest

from oracle import pq_oracle as orc
from test_gpu_serve_example import ex

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


@pytest.mark.parametrize("penalty", [1.0, 3.0])
def test_first_token(monkeypatch, penalty):
    seen = {}
    read, say = ex.read_prompts, ex.answer_drafted

    def read_prompts(*args):
        seen["rows"] = read(*args)
        return seen["rows"]

    def answer_drafted(dec, prompts, first, *args):
        seen.update(prompts=prompts, first=[int(t) for t in first])
        return say(dec, prompts, first, *args)

    monkeypatch.setattr(ex, "read_prompts", read_prompts)
    monkeypatch.setattr(ex, "answer_drafted", answer_drafted)
    lengths = [200, 7, 133, 1, 90]
    monkeypatch.setattr(sys, "argv", ["serve_decoder.py", "--draft", "--repetition", str(penalty), "--vocab", "100", "--answer", "5",
                                      "--prompts", ",".join(map(str, lengths))])
    ex.main()
    cfg = ex.Config(vocab=100)
    ids, book = ex.draw_weights(cfg)["head"][0]
    dense = book.astype(np.float64)[orc.unpack_indices(ids, cfg.hidden // cfg.d, cfg.bits, cfg.codewords)].reshape(cfg.vocab, -1)
    moved = 0
    for prompt, rows, first in zip(seen["prompts"], seen["rows"], seen["first"]):
        row = rows[-1].cpu().numpy().astype(np.float64)
        x = dense @ row
        slack = 2 * penalty * (2.0 ** -11 * np.abs(x) + 2.0 ** -14 * (np.abs(dense) @ np.abs(row))).max()
        likeliest = int(x.argmax())
        met = np.unique(prompt)
        x[met] = np.where(x[met] > 0, x[met] / penalty, x[met] * penalty)
        assert x[first] >= x.max() - slack
        moved += x[likeliest] < x.max() - slack
    assert moved >= 2 or penalty == 1
