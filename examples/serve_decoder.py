"""Serve a few requests with a small decoder whose weights are product-quantised.

    python examples/serve_decoder.py [--hidden 4096 --heads 32 --kv-heads 8 ...]

One decoder layer is, over the residual stream x of all tokens of a step,

    residual_norm              x + the last block's output, and its norm h
    pq_gemv_batched / pq_gemm  q, k, v of h
    lora_batched               + each token's own adapter
    rope_append                heads normed and turned, k and v to the paged cache
    paged_attention            over each request's pages
    pq_gemv / pq_gemm          output projection
    residual_norm              as above
    pq_gemv_batched / pq_gemm  gate and up;  silu(gate) * up;  down

Prompts are read in steps of at most ``chunk`` tokens that may end inside a
prompt and hold several requests.  The answers' tokens are then taken one a
step: the layers are captured into a HIP graph whose inputs (the tokens' rows,
positions, cache slots and lengths) stay on the device and are updated there.
Or several a step (--draft): a tree of guesses follows the last token, attention
lets each see its own branch, process_logits chooses a token after every one of
them, and the guesses that are what was chosen stand.
Weights are random, so the answers mean nothing.
"""

import argparse
import os
import sys
import time
from dataclasses import dataclass

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_04084_amd as fasq  # noqa: E402
import pq_inputs as pi  # noqa: E402


@dataclass
class Config:
    hidden: int = 512
    heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    inter: int = 1024
    layers: int = 2
    vocab: int = 1000
    adapters: int = 3
    rank: int = 8
    page_size: int = 16
    max_len: int = 512
    window: int = 0
    repetition: float = 1.0
    eps: float = 1e-5
    d: int = 2
    codewords: int = 256
    bits: int = 8


def draw_weights(cfg: Config, seed: int = 0) -> dict:
    """NumPy weights; a projection is (packed ids, codebook)."""
    rng = np.random.default_rng(seed)

    def pq(n, k):
        book = pi.draw_codebook(rng, cfg.codewords, cfg.d, std=k ** -0.5)
        return pi.pack_indices(pi.draw_ids(rng, n, k // cfg.d, cfg.codewords), cfg.bits), book

    def dense(*shape, std):
        return (rng.standard_normal(shape) * std).astype(np.float16)

    def norm(n):
        return (1 + 0.1 * rng.standard_normal(n)).astype(np.float16)

    q, kv, h = cfg.heads * cfg.head_dim, cfg.kv_heads * cfg.head_dim, cfg.hidden
    layers = []
    for _ in range(cfg.layers):
        layers.append(dict(
            qkv=[pq(q, h), pq(kv, h), pq(kv, h)], o=[pq(h, q)], gate_up=[pq(cfg.inter, h), pq(cfg.inter, h)],
            down=[pq(h, cfg.inter)], norm=norm(h), mlp_norm=norm(h), q_norm=norm(cfg.head_dim),
            k_norm=norm(cfg.head_dim), A=[dense(cfg.adapters, cfg.rank, h, std=h ** -0.5) for _ in range(3)],
            B=[dense(cfg.adapters, n, cfg.rank, std=cfg.rank ** -0.5) for n in (q, kv, kv)]))
    scales = np.linspace(0.25, 0.75, cfg.adapters).astype(np.float32)
    return dict(layers=layers, norm=norm(h), head=[pq(cfg.vocab, h)], embed=dense(cfg.vocab, h, std=1.0), scales=scales)


def to_device(w, device):
    if isinstance(w, dict):
        return {k: to_device(v, device) for k, v in w.items()}
    if isinstance(w, (list, tuple)):
        return type(w)(to_device(v, device) for v in w)
    return torch.from_numpy(w).to(device)


@dataclass
class Batch:
    """The requests' tokens of one step, on the device."""
    positions: torch.Tensor  # int32 [T]
    slots: torch.Tensor      # int32 [T]
    adapters: torch.Tensor   # int32 [T], -1: none
    q_start: torch.Tensor    # int32 [B + 1]
    kv_len: torch.Tensor     # int32 [B], with this step's tokens
    tree: torch.Tensor = None   # of drafted tokens: which of them each one sees,
    spans: torch.Tensor = None  # and its window


class Decoder:
    """Weights, paged caches (one pair a layer, the same pages in all) and the step."""

    def __init__(self, cfg: Config, weights: dict, requests: int, device="cuda"):
        self.cfg, self.device = cfg, torch.device(device)
        self.w = to_device(weights, device)
        freq, scale = fasq.rope_frequencies(cfg.head_dim, 10000.0)
        self.table = fasq.rope_table(freq, cfg.max_len, scale, device=device)
        self.per_request = -(-cfg.max_len // cfg.page_size)
        count = requests * self.per_request
        shape = (cfg.layers, count, cfg.page_size, cfg.kv_heads, cfg.head_dim)
        self.k = torch.zeros(shape, dtype=torch.float16, device=device)
        self.v = torch.zeros(shape, dtype=torch.float16, device=device)
        self.free = list(range(count))[::-1]
        # pages are handed out in the order in which requests need them, so
        # that they lie mixed in the cache
        self.pages = np.zeros((requests, self.per_request), dtype=np.int32)
        self.held = [0] * requests
        self.device_pages = torch.zeros((requests, self.per_request), dtype=torch.int32, device=device)

    def reserve(self, request: int, length: int) -> None:
        """Pages for the request's first ``length`` tokens."""
        if length > self.cfg.max_len:
            raise ValueError(f"a request holds at most {self.cfg.max_len} tokens")
        while self.held[request] * self.cfg.page_size < length:
            self.pages[request, self.held[request]] = self.free.pop()
            self.held[request] += 1

    def publish_pages(self) -> None:
        self.device_pages.copy_(torch.from_numpy(self.pages))

    def project(self, x, matrices):
        ids, books = [m[0] for m in matrices], [m[1] for m in matrices]
        cfg = self.cfg
        if x.shape[0] <= 16:
            return fasq.pq_gemv_batched(x, ids, cfg.bits, cfg.d, books)
        return [fasq.pq_gemm(x, i, cfg.bits, cfg.d, b) for i, b in zip(ids, books)]

    def layers(self, x, batch: Batch):
        """The normed output rows of the embedded tokens ``x`` [T x hidden]."""
        cfg, T, y = self.cfg, x.shape[0], None
        for i, w in enumerate(self.w["layers"]):
            new, h = fasq.residual_norm(x, y, w["norm"], cfg.eps)
            x = x if new is None else new
            qkv = self.project(h, w["qkv"])
            q, k, v = fasq.lora_batched(h, batch.adapters, w["A"], w["B"], self.w["scales"], qkv, outs=qkv)
            q = q.view(T, cfg.heads, cfg.head_dim)
            k, v = (t.view(T, cfg.kv_heads, cfg.head_dim) for t in (k, v))
            fasq.rope_append(q, k, v, self.table, batch.positions, batch.slots, self.k[i], self.v[i],
                             q_norm=w["q_norm"], k_norm=w["k_norm"], eps=cfg.eps, out=q)
            a = fasq.paged_attention(q, self.k[i], self.v[i], self.device_pages, batch.q_start, batch.kv_len,
                                     window=cfg.window if batch.tree is None else 0, spans=batch.spans, tree=batch.tree)
            y, = self.project(a.view(T, -1), w["o"])
            x, h = fasq.residual_norm(x, y, w["mlp_norm"], cfg.eps)
            gate, up = self.project(h, w["gate_up"])
            y, = self.project(torch.nn.functional.silu(gate).mul_(up), w["down"])
        return fasq.residual_norm(x, y, self.w["norm"], cfg.eps)[1]

    def next_tokens(self, rows, requests=None, **rules):
        """The likeliest tokens after these output rows, under these rules (see process_logits)."""
        logits, = self.project(rows, self.w["head"])
        return fasq.process_logits(logits, requests, write=False, choose=True, **rules)[1].long()

    def embed(self, tokens):
        return self.w["embed"].index_select(0, tokens)


def read_prompts(dec: Decoder, prompts, adapters, chunk: int):
    """Reads all prompts; returns the output rows of every prompt's tokens."""
    cfg, B = dec.cfg, len(prompts)
    done, rows = [0] * B, [[] for _ in range(B)]
    while any(done[b] < len(prompts[b]) for b in range(B)):
        left, counts = chunk, []
        for b in range(B):
            n = min(left, len(prompts[b]) - done[b])
            counts.append(n)
            left -= n
            dec.reserve(b, done[b] + n)
        dec.publish_pages()
        pos = np.concatenate([np.arange(done[b], done[b] + counts[b]) for b in range(B)])
        req = np.repeat(np.arange(B), counts)
        slots = dec.pages[req, pos // cfg.page_size] * cfg.page_size + pos % cfg.page_size

        def i32(a):
            return torch.from_numpy(np.asarray(a, dtype=np.int32)).to(dec.device)

        batch = Batch(i32(pos), i32(slots), i32(np.asarray(adapters)[req]), i32(np.cumsum([0] + counts)),
                      i32([done[b] + counts[b] for b in range(B)]))
        tokens = np.concatenate([prompts[b][done[b] : done[b] + counts[b]] for b in range(B)])
        out = dec.layers(dec.embed(torch.from_numpy(tokens.astype(np.int64)).to(dec.device)), batch)
        for b, part in enumerate(out.split(counts)):
            rows[b].append(part)
            done[b] += counts[b]
    return [torch.cat(r) for r in rows]


def answer(dec: Decoder, lengths, first, adapters, count: int):
    """``count`` tokens of every request after prompts of these lengths, one a
    step, from the tokens ``first`` on.  Returns the tokens [B x count] and the
    output rows of each [B x count x hidden]."""
    cfg, B = dec.cfg, len(lengths)
    for b, n in enumerate(lengths):
        dec.reserve(b, n + count)
    dec.publish_pages()
    request = torch.arange(B, device=dec.device)
    pos = torch.tensor(lengths, dtype=torch.int64, device=dec.device)

    def slots_of(p):
        page = dec.device_pages[request, p // cfg.page_size]
        return (page * cfg.page_size + p % cfg.page_size).to(torch.int32)

    batch = Batch(pos.to(torch.int32), slots_of(pos), torch.tensor(adapters, dtype=torch.int32, device=dec.device),
                  torch.arange(B + 1, dtype=torch.int32, device=dec.device), (pos + 1).to(torch.int32))
    x = dec.embed(first).clone()
    side = torch.cuda.Stream()  # a first run outside the capture; it writes what the first step writes again
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dec.layers(x, batch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = dec.layers(x, batch)
    tokens, rows, token = [], [], first
    for _ in range(count):
        x.copy_(dec.embed(token))
        batch.positions.copy_(pos)
        batch.slots.copy_(slots_of(pos))
        batch.kv_len.copy_(pos + 1)
        graph.replay()
        tokens.append(token)
        rows.append(out.clone())
        token = dec.next_tokens(out)
        pos = pos + 1
    return torch.stack(tokens, 1), torch.stack(rows, 1)


def guess(text, branches: int = 2, depth: int = 4):
    """A tree that may follow a text: what followed its last token before, the
    latest places first.  Tokens and the node that each follows; node 0 is the last token."""
    tokens, parents = [text[-1]], [-1]
    for at in [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]][:branches]:
        node = 0
        for t in text[at + 1:at + 1 + depth]:
            tokens.append(t)
            parents.append(node)
            node = len(tokens) - 1
    return tokens, parents


def first_tokens(dec: Decoder, prompts, rows):
    """The likeliest token after each prompt, whose output rows these are, with the penalty for the prompt's own tokens."""
    rules = {}
    if dec.cfg.repetition != 1.0:
        held = np.zeros((len(prompts), max(map(len, prompts))), dtype=np.int32)
        for b, p in enumerate(prompts):
            held[b, :len(p)] = p
        count = np.array([len(p) for p in prompts], dtype=np.int32)
        rules = dict(tokens=torch.from_numpy(held).to(dec.device), token_count=torch.from_numpy(count).to(dec.device),
                     repetition=torch.full((len(prompts),), dec.cfg.repetition, device=dec.device))
    return dec.next_tokens(torch.stack([r[-1] for r in rows]), **rules)


def answer_drafted(dec: Decoder, prompts, first, adapters, count: int, draft=guess):
    """At least ``count`` tokens of every request after its prompt, from the
    tokens ``first`` on, several a step where ``draft`` guesses them.  Returns the
    tokens, the output row of each (lists, one entry a request) and the number of steps."""
    cfg, B = dec.cfg, len(prompts)
    text = [list(map(int, p)) + [int(t)] for p, t in zip(prompts, first)]
    rows, steps = [[] for _ in range(B)], 0
    ends = [len(t) + count for t in text]
    if max(ends) - 1 > cfg.max_len:  # the last token is not cached
        raise ValueError(f"a request holds at most {cfg.max_len} tokens")
    held = torch.zeros((B, cfg.max_len), dtype=torch.int32)
    for b, t in enumerate(text):
        held[b, :len(t)] = torch.tensor(t)
    held = held.to(dec.device)

    def i32(a):
        return torch.from_numpy(np.asarray(a, dtype=np.int32)).to(dec.device)

    while any(len(t) < e for t, e in zip(text, ends)):
        steps += 1
        trees = [draft(t) if len(t) < e else ([], []) for t, e in zip(text, ends)]
        start = [len(t) - 1 for t in text]  # cached tokens
        trees = [(t[:cfg.max_len - s], p[:cfg.max_len - s]) for (t, p), s in zip(trees, start)]
        n = [len(t) for t, _ in trees]
        for b in range(B):
            dec.reserve(b, start[b] + n[b])
        dec.publish_pages()
        tree, depth = fasq.draft_tree([p for _, p in trees], device=dec.device)
        req, first_row = np.repeat(np.arange(B), n), np.cumsum([0] + n)
        at = np.array(start)[req] + np.arange(len(req)) - first_row[req]
        slots = dec.pages[req, at // cfg.page_size] * cfg.page_size + at % cfg.page_size
        positions, kv_len = i32(np.array(start)[req]) + depth, i32([s + m for s, m in zip(start, n)])
        spans = None
        if cfg.window:
            if int(depth.max()) >= cfg.window:  # a span cannot tell a branch's first nodes from its siblings
                raise ValueError("guesses deeper than the window")
            spans = torch.stack([(positions - cfg.window + 1).clamp_(min=0), kv_len[i32(req).long()]], 1)
        drafted = i32(np.concatenate([t for t, _ in trees]))
        batch = Batch(positions, i32(slots), i32(np.asarray(adapters)[req]), i32(first_row), kv_len, tree, spans)
        out = dec.layers(dec.embed(drafted), batch)
        rules = {}
        if cfg.repetition != 1.0:
            rules = dict(tokens=held, token_count=i32(start), repetition=torch.full((B,), cfg.repetition, device=dec.device),
                         draft_tokens=drafted, tree=tree, q_start=batch.q_start)
        chosen = dec.next_tokens(out, i32(req), requests_count=B, **rules).tolist()
        moved = [[], []]
        for b, (tokens, parents) in enumerate(trees):
            if not tokens:
                continue
            way, base = [0], int(first_row[b])
            while True:
                token = chosen[base + way[-1]]
                after = [j for j in range(len(tokens)) if parents[j] == way[-1] and tokens[j] == token]
                if not after:
                    break
                way.append(after[0])
            # the branch that stands moves up in the cache, to where its tokens belong
            for i, node in enumerate(way):
                to = start[b] + i
                moved[0].append(int(slots[base + node]))
                moved[1].append(int(dec.pages[b, to // cfg.page_size] * cfg.page_size + to % cfg.page_size))
            rows[b].append(out[base:base + len(tokens)][way])
            text[b] += [tokens[j] for j in way[1:]] + [token]
            held[b, :len(text[b])] = i32(text[b][:cfg.max_len])
        source, target = (torch.tensor(m, device=dec.device) for m in moved)
        for cache in (dec.k, dec.v):
            flat = cache.flatten(1, 2)
            flat[:, target] = flat[:, source]
    said = [t[len(p):-1] for t, p in zip(text, prompts)]
    return said, [torch.cat(r) for r in rows], steps


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name in ("hidden", "heads", "kv_heads", "head_dim", "inter", "layers", "vocab", "adapters", "rank",
                 "page_size", "max_len", "window"):
        p.add_argument("--" + name.replace("_", "-"), type=int, default=getattr(Config, name))
    p.add_argument("--prompts", default="200,7,133,1", help="prompt lengths, one request each (at most 16)")
    p.add_argument("--chunk", type=int, default=128, help="tokens of a prompt step")
    p.add_argument("--answer", type=int, default=32, help="tokens of every answer")
    p.add_argument("--draft", action="store_true", help="several tokens a step where the text so far lets them be guessed")
    p.add_argument("--repetition", type=float, default=Config.repetition, help="penalty for tokens that occurred (with --draft)")
    args = vars(p.parse_args())
    drafted = args.pop("draft")
    lengths, chunk, count = [int(n) for n in args.pop("prompts").split(",")], args.pop("chunk"), args.pop("answer")
    if not 1 <= len(lengths) <= 16 or min(lengths) < 1 or chunk < 1 or count < 1:
        p.error("1 to 16 prompts, lengths, chunk and answer of at least 1")
    cfg = Config(**args)
    dec = Decoder(cfg, draw_weights(cfg), len(lengths))
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, cfg.vocab, n) for n in lengths]
    adapters = [b % (cfg.adapters + 1) - 1 for b in range(len(lengths))]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    rows = read_prompts(dec, prompts, adapters, chunk)
    first = first_tokens(dec, prompts, rows) if drafted else dec.next_tokens(torch.stack([r[-1] for r in rows]))
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    steps = count
    if drafted:
        said, _, steps = answer_drafted(dec, prompts, first, adapters, count)
    else:
        said = answer(dec, lengths, first, adapters, count)[0].tolist()
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    for b, n in enumerate(lengths):
        print(f"request {b}: prompt of {n}, adapter {adapters[b]}: {said[b][:12]} ...")
    print(f"{sum(lengths)} prompt tokens in {(t1 - t0) * 1e3:.1f} ms (first calls included), "
          f"{sum(map(len, said))} tokens in {steps} steps in {(t2 - t1) * 1e3:.1f} ms (capture included)")


if __name__ == "__main__":
    main()
