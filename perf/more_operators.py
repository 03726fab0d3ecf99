"""What serving with capped or biased scores, packed prompts, drafted tokens and token rules adds to a decoder's step.

Three kinds of case:

* ``scores``: attention over the paged cache whose scores are capped by a tanh
  (``softcap``), get a bias that grows with the distance (``slopes``, one a
  head), or whose tokens see a run of keys of their own (``spans``: documents
  packed into one prompt, prefixes that are read in both directions);
* ``tree``: the same for a tree of drafted tokens, each of which sees what is
  cached and its own ancestors (``tree``: one bit a pair);
* ``logits``: what stands between the last projection and the choice of a
  token: penalties for repeated tokens, biases of single tokens, a grammar's
  set of allowed tokens, the temperature, the likeliest token and the
  logarithm of the softmax sum (``process_logits``), for one row a request or
  for every node of a drafted tree.

Queries, keys, values and logits are fp16, sums and statistics fp32.
"""

import math
import random

import torch

own = False  # True: run() calls the library; False: the same in plain torch


def listed():
    heads = {"Hq": 32, "Hkv": 8, "D": 128, "page": 16, "window": 0, "cap": 0.0, "slopes": False, "docs": 0, "prefix": 0}
    logits = {"kind": "logits", "V": 128256, "wide": False, "penalties": True, "bias": 16, "grammar": False,
              "temperature": True, "write": "half"}
    return [
        # a decode batch of conversations of all lengths, scores capped at 50
        {"name": "cap_decode_64", "kind": "scores", **heads, "cap": 50.0, "shape": "decode", "B": 64, "kv_lo": 300, "kv_hi": 8192},
        # the second chunk of a long prompt, capped scores
        {"name": "cap_chunk_2048", "kind": "scores", **heads, "page": 64, "cap": 30.0, "shape": "chunk", "B": 1, "n": 2048, "kv_lo": 4096, "kv_hi": 4096},
        # one user's token where positions enter as a bias: latency of a call
        {"name": "slopes_decode_one", "kind": "scores", **heads, "slopes": True, "shape": "decode", "B": 1, "kv_lo": 1531, "kv_hi": 1531},
        # a step that mixes a prompt's chunk, a short prompt and decoding requests; odd heads and pages
        {"name": "slopes_mixed_ragged", "kind": "scores", **heads, "Hq": 12, "Hkv": 4, "D": 80, "page": 20, "slopes": True, "shape": "mixed", "B": 24, "n": 509,
         "kv_lo": 77, "kv_hi": 3001},
        # eleven documents packed into one prompt, the first tokens of each read in both directions
        {"name": "documents_4096", "kind": "scores", **heads, "page": 64, "docs": 11, "prefix": 50, "shape": "chunk", "B": 1, "n": 4096, "kv_lo": 4096, "kv_hi": 4096},
        # one user's drafted tree: latency of a call
        {"name": "tree_one", "kind": "tree", **heads, "shape": "chunk", "B": 1, "n": 13, "kv_lo": 1531, "kv_hi": 1531},
        # sixteen requests, each with a tree of 32 drafted tokens
        {"name": "tree_batch_16", "kind": "tree", **heads, "shape": "chunk", "B": 16, "n": 32, "kv_lo": 300, "kv_hi": 8192},
        # large trees over two long documents
        {"name": "tree_long", "kind": "tree", **heads, "page": 64, "shape": "chunk", "B": 2, "n": 64, "kv_lo": 65536, "kv_hi": 131072},
        # one user's next token (the vocabulary of Llama-3-8B)
        {"name": "logits_one", **logits, "S": 1, "n": 1, "len_lo": 1531, "len_hi": 1531},
        # a decode batch with all rules, its logits kept in fp32 for a sampler
        {"name": "logits_batch_64", **logits, "grammar": True, "write": "float", "S": 64, "n": 1, "len_lo": 300, "len_hi": 8192},
        # every node of sixteen drafted trees, for the tokens alone
        {"name": "logits_trees_16", **logits, "grammar": True, "bias": 0, "write": "none", "S": 16, "n": 16, "len_lo": 300, "len_hi": 8192},
        # an odd vocabulary, fp32 logits, long documents
        {"name": "logits_long_5", **logits, "V": 32003, "wide": True, "bias": 300, "S": 5, "n": 1, "len_lo": 20000, "len_hi": 100000},
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer multiple of ``step`` in [lo, hi], uniform over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)), -(-lo // step)), hi // step) * step


def draw(rng):
    kind = rng.choice(["scores", "scores", "scores", "tree", "tree", "logits", "logits"])
    if kind == "logits":
        V = _log_int(rng, 1000, 152000)
        n = rng.choice([1, 1, _log_int(rng, 2, 64)])
        S = _log_int(rng, 1, max(2, min(128, 32000000 // (V * n))))
        hi = _log_int(rng, 8, max(9, min(131072, 500000 // S)))
        return {"kind": kind, "V": V, "wide": rng.choice([False, False, True]), "penalties": rng.choice([True, True, False]), "bias": rng.choice([0, 5, 300]),
                "grammar": rng.choice([False, True]), "temperature": rng.choice([True, True, False]), "write": rng.choice(["half", "float", "none"]),
                "S": S, "n": n, "len_lo": max(1, hi // rng.choice([1, 2, 20])), "len_hi": hi}
    Hkv, G = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 3, 4, 4, 7, 8])
    D = rng.choice([128, 128, 64, 80, 96, 256])
    case = {"kind": kind, "Hq": Hkv * G, "Hkv": Hkv, "D": D, "page": rng.choice([16, 16, 20, 32, 64, 128]),
            "window": rng.choice([0, 0, _log_int(rng, 100, 4096)]), "cap": rng.choice([0.0, 15.0, 50.0]), "slopes": False, "docs": 0, "prefix": 0}
    if kind == "tree":
        n = _log_int(rng, 2, 128)
        B = _log_int(rng, 1, max(2, min(32, 512 // n)))
        hi = _log_int(rng, n, max(n + 1, min(131072, int(2e10 / (B * n * Hkv * G * D)), int(1.9e8 / (B * Hkv * D)))))
        return {**case, "shape": "chunk", "B": B, "n": n, "kv_lo": max(n, hi // rng.choice([1, 2, 8])), "kv_hi": hi}
    what = rng.choice(["cap", "slopes", "both", "documents", "documents"])
    case.update(slopes=what in ("slopes", "both"), cap=0.0 if what == "slopes" else 15.0 if what == "both" else case["cap"])
    if what == "cap" and not case["cap"]:
        case["cap"] = 30.0
    shape = "chunk" if what == "documents" else rng.choice(["decode", "chunk", "mixed"])
    if shape == "decode":
        B = _log_int(rng, 1, 128)
        hi = _log_int(rng, 32, max(33, min(131072, int(1.9e8 / (B * Hkv * D)))))
        return {**case, "shape": shape, "B": B, "kv_lo": max(1, hi // rng.choice([1, 2, 8])), "kv_hi": hi}
    n = _log_int(rng, 2, 2048)
    hi = _log_int(rng, n, max(n + 1, min(8192, int(2.5e10 / (n * Hkv * G * D)))))
    if what == "documents":  # whole prompts
        case.update(window=0, docs=_log_int(rng, 1, 24), prefix=rng.choice([0, _log_int(rng, 2, 200)]))
        return {**case, "shape": shape, "B": rng.choice([1, 2, 5]) if n < 500 else 1, "n": n, "kv_lo": n, "kv_hi": n}
    if shape == "chunk":
        return {**case, "shape": shape, "B": 1, "n": n, "kv_lo": max(n, hi // 2), "kv_hi": hi}
    return {**case, "shape": shape, "B": _log_int(rng, 3, 32), "n": n, "kv_lo": max(2, hi // 8), "kv_hi": hi}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float16).mul_(std)


def _spread(B, lo, hi):
    """B lengths, even over the logarithm, in an order that is not sorted."""
    return [int(round(hi * (lo / hi) ** ((i * 7919 % B) / max(1, B - 1)))) for i in range(B)]


def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of each request."""
    B = case["B"]
    kv = _spread(B, case["kv_lo"], case["kv_hi"])
    if case["shape"] == "decode":
        return [1] * B, kv
    if case["shape"] == "chunk":
        return [case["n"]] * B, kv
    # the longest request runs a chunk, another is a short prompt from its first token, the rest decode
    n = [1] * B
    first = kv.index(max(kv))
    n[first] = case["n"]
    other = (first + B // 2) % B
    n[other] = kv[other] = min(kv[other], 4 * case["page"] - 3)
    return n, kv


def _parents(n):
    """A tree of n drafted tokens as they are drafted: the last token of the answer
    first, then candidates that follow it or one another (-1: no parent)."""
    rng = random.Random(n)
    return [-1] + [rng.choice([max(0, i - 1), i // 2, i // 3]) for i in range(1, n)]


def _ancestors(parents):
    """The nodes on the way to each node, itself among them."""
    ways = []
    for i, p in enumerate(parents):
        ways.append((ways[p] if p >= 0 else []) + [i])
    return ways


def _tree_words(parents):
    """int32 [n, ceil(n / 32)]: bit j of row i says whether j is i or an ancestor of it."""
    n = len(parents)
    bits = torch.zeros((n, -(-n // 32) * 32), dtype=torch.int64)
    for i, way in enumerate(_ancestors(parents)):
        bits[i, way] = 1
    words = (bits.view(n, -1, 32) << torch.arange(32)).sum(2)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _document_spans(case):
    """int64 [n, 2]: the keys that each token of a packed prompt sees.  Every document's first
    ``prefix`` tokens are read in both directions."""
    n, docs = case["n"], min(case["docs"], case["n"])
    weights = [1 + i * 7 % docs for i in range(docs)]
    ends = [max(i + 1, n * sum(weights[:i + 1]) // sum(weights)) for i in range(docs)]
    spans = torch.empty((n, 2), dtype=torch.int64)
    begin = 0
    for end in ends:
        at = torch.arange(begin, end)
        spans[begin:end, 0] = begin
        spans[begin:end, 1] = torch.clamp(at + 1, min=min(begin + case["prefix"], end))
        begin = end
    return spans


def _tree_spans(case, kv):
    """int64 [n, 2]: a window over a drafted tree's positions."""
    depth = torch.tensor([len(w) - 1 for w in _ancestors(_parents(case["n"]))])
    first = torch.clamp(kv - case["n"] + depth - case["window"] + 1, min=0)
    return torch.stack([first, torch.full_like(first, kv)], 1)


def _prepare_attention(case, seed):
    g = _gen(seed)
    n, kv = _lengths(case)
    B, ps, Hkv, D = case["B"], case["page"], case["Hkv"], case["D"]
    need = [-(-k // ps) for k in kv]
    spare = 3  # pages of other requests
    order = torch.randperm(sum(need) + spare, generator=g, device="cuda", dtype=torch.int32)
    pages = torch.zeros((B, max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        pages[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    shape = (sum(need) + spare, ps, Hkv, D)
    starts = [sum(n[:b]) for b in range(B + 1)]
    cuda = {"device": "cuda", "dtype": torch.int32}
    state = {"kind": case["kind"], "q": _normal(g, (starts[-1], case["Hq"], D), 2.0), "k": _normal(g, shape), "v": _normal(g, shape),
             "pages": pages, "q_start": torch.tensor(starts, **cuda), "kv_len": torch.tensor(kv, **cuda), "window": case["window"], "cap": case["cap"],
             "slopes": None, "spans": None, "tree": None}
    if case["slopes"]:  # a geometric sequence over the heads
        state["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["Hq"] + 1, device="cuda", dtype=torch.float32) / case["Hq"])
    if case["docs"]:
        state["spans"] = _document_spans(case).repeat(B, 1).to(**cuda)
    if case["kind"] == "tree":
        state["tree"] = _tree_words(_parents(case["n"])).repeat(B, 1).cuda()
        if case["window"]:
            state["spans"], state["window"] = torch.cat([_tree_spans(case, k) for k in kv]).to(**cuda), 0
    # the requests by the length of their chunk, for the plain form
    by = {}
    for b in range(B):
        by.setdefault(n[b], []).append(b)
    rows = torch.cat([torch.arange(starts[b], starts[b + 1]) for m in by for b in by[m]])
    state["groups"] = [(m, max(kv[b] for b in by[m]), torch.tensor(by[m], device="cuda")) for m in by]
    state["order"] = torch.argsort(rows).cuda() if len(by) > 1 else None
    return state


def _prepare_logits(case, seed):
    g = _gen(seed)
    S, n, V = case["S"], case["n"], case["V"]
    count = _spread(S, case["len_lo"], case["len_hi"])
    L = max(count) + 3
    cuda = {"device": "cuda", "dtype": torch.int32}
    logits = torch.randn((S * n, V), generator=g, device="cuda") * 3

    def words(shape):  # tokens as texts have them: few of them most of the time
        return (V ** torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)).to(torch.int32).clamp_(max=V) - 1

    def uniform(lo, hi):
        return torch.rand((S,), generator=g, device="cuda") * (hi - lo) + lo

    state = {"kind": "logits", "logits": logits if case["wide"] else logits.half(), "write": case["write"], "out": None,
             "requests": torch.arange(S, **cuda).repeat_interleave(n).contiguous(), "tokens": None, "prompt_len": None, "count": None, "repetition": None,
             "presence": None, "frequency": None, "bias_ids": None, "bias": None, "allowed": None, "temperature": None, "drafts": None, "tree": None,
             "q_start": None}
    if case["write"] != "none":
        state["out"] = torch.empty((S * n, V), device="cuda", dtype=torch.float16 if case["write"] == "half" else torch.float32)
    if case["penalties"]:
        state["tokens"], state["count"] = words((S, L)), torch.tensor(count, **cuda)
        state["prompt_len"] = torch.tensor([c * 3 // 4 for c in count], **cuda)
        state["repetition"], state["presence"], state["frequency"] = uniform(1.0, 1.3), uniform(0.0, 1.0), uniform(-0.1, 0.5)
        if n > 1:
            state["drafts"], state["tree"] = words((S * n,)), _tree_words(_parents(n)).repeat(S, 1).cuda()
            state["q_start"] = torch.arange(0, S * n + 1, n, **cuda)
    if case["bias"]:
        ids = torch.randint(0, V, (S, case["bias"]), generator=g, **cuda)
        ids[:, case["bias"] // 2 + 1:][1::3] = -1  # some requests have fewer
        state["bias_ids"], state["bias"] = ids, torch.randn((S, case["bias"]), generator=g, device="cuda") * 5
    if case["grammar"]:
        state["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (S * n, -(-V // 32)), generator=g, **cuda)
    if case["temperature"]:
        state["temperature"] = uniform(0.5, 1.5)
    return state


def prepare(case, seed):
    return (_prepare_logits if case["kind"] == "logits" else _prepare_attention)(case, seed)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    s = state
    if not own:
        return _plain_logits(s) if s["kind"] == "logits" else _plain_attention(s)
    import paper_2605_04084_amd as fasq

    if s["kind"] == "logits":
        return fasq.process_logits(s["logits"], s["requests"], tokens=s["tokens"], prompt_len=s["prompt_len"], token_count=s["count"],
                                   repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], bias_ids=s["bias_ids"],
                                   bias_values=s["bias"], allowed=s["allowed"], temperature=s["temperature"], draft_tokens=s["drafts"], tree=s["tree"],
                                   q_start=s["q_start"], out=s["out"], write=s["write"] != "none", choose=True)
    return fasq.paged_attention(s["q"], s["k"], s["v"], s["pages"], s["q_start"], s["kv_len"], window=s["window"], return_lse=True,
                                softcap=s["cap"], slopes=s["slopes"], spans=s["spans"], tree=s["tree"])


def _bits(words, count):
    """bool [.., count] of int32 words."""
    j = torch.arange(count, device="cuda")
    return (words[..., j // 32] >> (j % 32)) & 1 != 0


def _attend(s, n, kv, b):
    """The requests ``b``, all with ``n`` new tokens and at most ``kv`` cached ones."""
    ps, Hkv, D = s["k"].shape[1:]
    Hq = s["q"].shape[1]
    table = s["pages"][b, :-(-kv // ps)].long()
    k, v = (c[table].flatten(1, 2)[:, :kv].float() for c in (s["k"], s["v"]))  # [b, kv, Hkv, D]
    i = torch.arange(n, device="cuda")
    rows = s["q_start"][b].long()[:, None] + i
    q = s["q"][rows].float().view(-1, n, Hkv, Hq // Hkv, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(-1, Hq // Hkv * n, D)
    scores = (torch.bmm(q, k.permute(0, 2, 3, 1).reshape(-1, D, kv)) * D ** -0.5).view(-1, Hkv, Hq // Hkv, n, kv)
    j = torch.arange(kv, device="cuda")
    length = s["kv_len"][b].long()[:, None, None]
    at = length - n + i[:, None]  # the position of each token
    if s["slopes"] is not None:
        scores -= s["slopes"].view(Hkv, Hq // Hkv, 1, 1) * (at - j).abs().float()[:, None, None]
    if s["cap"]:
        scores = s["cap"] * torch.tanh(scores / s["cap"])
    if s["spans"] is not None:
        span = s["spans"][rows].long()
        seen = (j >= span[..., :1]) & (j < span[..., 1:]) & (j < length)
    elif s["tree"] is not None:
        seen = (j < length).expand(-1, n, -1)
    else:
        seen = j <= at
        if s["window"]:
            seen &= j > at - s["window"]
    if s["tree"] is not None:
        new = j - (length - n)  # which new token each key is
        drafted = _bits(s["tree"][rows], n).gather(2, new.clamp(0, n - 1).expand(-1, n, -1))
        seen = seen & ((new < 0) | drafted)
    scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(-1, Hq // Hkv * n, kv), v.permute(0, 2, 1, 3).reshape(-1, kv, D)).view(-1, Hkv, Hq // Hkv, n, D) / total
    lse = (top + torch.log(total)).squeeze(-1)
    return out.permute(0, 3, 1, 2, 4).reshape(-1, Hq, D).half(), lse.permute(0, 3, 1, 2).reshape(-1, Hq)


def _plain_attention(s):
    parts = [_attend(s, *group) for group in s["groups"]]
    if len(parts) == 1:
        return parts[0]
    return tuple(torch.cat(t)[s["order"]] for t in zip(*parts))


def _plain_logits(s):
    """A token's logit divided (if positive) or multiplied by the repetition penalty where the token has occurred, less its
    penalties, plus its bias, over the temperature; -inf where it is not allowed."""
    x = s["logits"].float()
    V, r = x.shape[1], s["requests"].long()
    if s["tokens"] is not None:
        i = torch.arange(s["tokens"].shape[1], device="cuda")
        held, answered = i < s["count"][:, None], i >= s["prompt_len"][:, None]
        where = torch.where(held, s["tokens"], V).long()  # column V: no token
        seen = torch.zeros((len(held), V + 1), dtype=torch.int32, device="cuda").scatter_add_(1, where, held.int())[r, :V]
        where = torch.where(held & answered, s["tokens"], V).long()
        times = torch.zeros((len(held), V + 1), dtype=torch.int32, device="cuda").scatter_add_(1, where, held.int())[r]
        if s["tree"] is not None:
            n = s["tree"].shape[0] // len(held)  # every request has as many nodes
            way = _bits(s["tree"], n)
            where = torch.where(way, s["drafts"].view(-1, n)[r], V).long()
            times.scatter_add_(1, where, way.int())
        times = times[:, :V]
        # reciprocals rounded once, then products
        rho = s["repetition"][r, None]
        x = torch.where((seen > 0) | (times > 0), torch.where(x > 0, x * (1 / rho), x * rho), x)
        x = x - (s["frequency"][r, None] * times + s["presence"][r, None] * (times > 0))
    if s["bias_ids"] is not None:
        where = torch.where(s["bias_ids"] >= 0, s["bias_ids"], V).long()
        entry = torch.arange(where.shape[1], device="cuda").expand_as(where)
        last = torch.full((len(where), V + 1), -1, device="cuda").scatter_reduce_(1, where, entry, "amax")[:, :V]
        x = x + torch.where(last >= 0, s["bias"].gather(1, last.clamp(min=0)), 0.0)[r]
    if s["temperature"] is not None:
        x = x * (1 / s["temperature"])[r, None]
    if s["allowed"] is not None:
        x = torch.where(_bits(s["allowed"], V), x, -math.inf)
    top = x.amax(1, keepdim=True)
    choice = torch.where(x == top, torch.arange(V, device="cuda", dtype=torch.int32), V).amin(1)
    lse = (top + torch.log(torch.exp(x - top).sum(1, keepdim=True))).squeeze(1)
    return x.to(s["out"].dtype) if s["out"] is not None else None, choice, lse


# ---------------------------------------------------------------------------
# What the path cannot do without
# ---------------------------------------------------------------------------

def _work_attention(case):
    n, kv = _lengths(case)
    Hq, Hkv, D, w = case["Hq"], case["Hkv"], case["D"], case["window"]
    pairs = read = more = 0  # visible (query, key) pairs of one head; keys that some query of the request sees; bytes of masks
    if case["docs"]:
        spans = _document_spans(case)
        pairs, read, more = case["B"] * int((spans[:, 1] - spans[:, 0]).sum()), sum(kv), 8 * sum(n)
    elif case["kind"] == "tree":
        m = case["n"]
        ways = _ancestors(_parents(m))
        for k in kv:
            first = _tree_spans(case, k)[:, 0].tolist() if w else [0] * m
            pairs += sum(max(0, k - m - f) + sum(k - m + j >= f for j in way) for f, way in zip(first, ways))
            read += k - min(first)
        more = 4 * sum(n) * -(-m // 32) + (8 * sum(n) if w else 0)
    else:
        for m, k in zip(n, kv):
            lo = k - m  # keys before the chunk
            pairs += sum(min(lo + i + 1, w) for i in range(m)) if w else m * lo + m * (m + 1) // 2
            read += min(k, w + m - 1) if w else k
    return {"bytes": 4 * read * Hkv * D + 4 * sum(n) * Hq * D + 4 * sum(n) * Hq + more, "flops": 4 * pairs * Hq * D}


def work(case):
    if case["kind"] != "logits":
        return _work_attention(case)
    S, V = case["S"], case["V"]
    R = S * case["n"]
    counts = _spread(S, case["len_lo"], case["len_hi"])
    write = {"half": 2, "float": 4, "none": 0}[case["write"]]
    return {"bytes": R * V * ((4 if case["wide"] else 2) + write) + (R * -(-V // 32) * 4 if case["grammar"] else 0) + 8 * S * case["bias"] + 12 * R
            + (4 * sum(counts) + 20 * S if case["penalties"] else 0) + (R * (4 + 4 * -(-case["n"] // 32)) if case["penalties"] and case["n"] > 1 else 0),
            "flops": R * V * (4 + (1 if case["temperature"] else 0))}


# ---------------------------------------------------------------------------
# The same results in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_attention(case, seed):
    s = _prepare_attention(case, seed)
    n, kv = _lengths(case)
    Hq, Hkv, D, ps, w = case["Hq"], case["Hkv"], case["D"], case["page"], case["window"]
    outs, lses, at = [], [], 0
    for b in range(case["B"]):
        place = torch.arange(kv[b], device="cuda")
        page = s["pages"][b][place // ps].long()
        keys, values = (c[page, place % ps].double() for c in (s["k"], s["v"]))
        chunk = s["q"][at:at + n[b]].double()
        at += n[b]
        token = torch.arange(kv[b] - n[b], kv[b], device="cuda")[:, None]
        if case["docs"]:
            first, last = _document_spans(case).cuda().split(1, 1)
            visible = ~((place < first) | (place >= last))
        elif case["kind"] == "tree":
            visible = torch.zeros((n[b], kv[b]), dtype=torch.bool)
            for i, way in enumerate(_ancestors(_parents(n[b]))):
                visible[i, :kv[b] - n[b]] = True
                visible[i, [kv[b] - n[b] + a for a in way]] = True
                if w:
                    visible[i, :max(0, kv[b] - n[b] + len(way) - w)] = False
            visible = visible.cuda()
        else:
            visible = ~((place > token) | (token - place >= w if w else place < 0))
        out = torch.empty((n[b], Hq, D), dtype=torch.float64, device="cuda")
        lse = torch.empty((n[b], Hq), dtype=torch.float64, device="cuda")
        for h in range(Hkv):
            kt, vv = keys[:, h].t().contiguous(), values[:, h].contiguous()
            for e in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z = (chunk[:, e].contiguous() @ kt) / math.sqrt(D)
                if s["slopes"] is not None:
                    z = z - float(s["slopes"][e]) * (place - token).abs()
                if case["cap"]:
                    z = torch.tanh(z / case["cap"]) * case["cap"]
                z = torch.where(visible, z, -math.inf)
                lse[:, e] = torch.logsumexp(z, 1)
                out[:, e] = torch.exp(z - lse[:, e, None]) @ vv
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)


def _exact_logits(case, seed):
    s = _prepare_logits(case, seed)
    S, n, V = case["S"], case["n"], case["V"]
    ways = _ancestors(_parents(n))
    value = {k: s[k].double().tolist() for k in ("repetition", "presence", "frequency", "temperature") if s[k] is not None}
    rows, sums = [], []
    for m in range(S * n):
        b = m // n
        z = s["logits"][m].double()
        if case["penalties"]:
            length, prompt = int(s["count"][b]), int(s["prompt_len"][b])
            text = s["tokens"][b, :length].long()
            answer = text[prompt:]
            if n > 1:
                answer = torch.cat([answer, s["drafts"][[b * n + a for a in ways[m % n]]].long()])
            times = torch.bincount(answer, minlength=V).double()
            met = times + torch.bincount(text[:prompt], minlength=V)
            scaled = torch.where(z > 0, z / value["repetition"][b], z * value["repetition"][b])
            z = torch.where(met > 0, scaled, z) - value["frequency"][b] * times - value["presence"][b] * times.clamp(max=1)
        if case["bias"]:
            extra = dict(zip(s["bias_ids"][b].tolist(), s["bias"][b].double().tolist()))  # a token's last entry counts
            extra.pop(-1, None)
            z[list(extra)] += torch.tensor(list(extra.values()), device="cuda", dtype=torch.float64)
        if case["temperature"]:
            z = z / value["temperature"][b]
        if case["grammar"]:
            word = s["allowed"][m].view(-1, 1).expand(-1, 32).bitwise_right_shift(torch.arange(32, device="cuda", dtype=torch.int32))
            z = z.masked_fill((word.flatten()[:V] & 1) == 0, -math.inf)
        sums.append(torch.logsumexp(z, 0))
        if case["write"] != "none":
            rows.append(z)
    return torch.stack(rows) if rows else None, None, torch.stack(sums)


def exact(case, seed):
    return (_exact_logits if case["kind"] == "logits" else _exact_attention)(case, seed)
