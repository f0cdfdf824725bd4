"""Measured operators around the paged 8-bit key/value cache (paper_2608_07971_amd.kv):
what an offline-inference job does before and after its attention.

Norms of queries and keys for each head with the position rotation in the same
pass, and their gradient; beam search's selection over beams and vocabulary,
and the cache's reordering by it; the attention weight that cached tokens get,
and eviction of those that got least.  Layouts: keys [page][layer][head]
[token][dim], values [page][layer][head][dim][token] in e4m3, scales
[page][layer][key, value][head] in float32, table [sequence][slot] with -1 for
none, accumulated weights [layer][sequence][head][token] in float32.

Every operator has a plain form in elementary torch operations and, where
`own` is set, the call a user makes of the framework's kernels.
"""
import math
import random
import types

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6                                              # of the norms


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # one decode step of 256 sequences: queries and keys normed and turned
        dict(name="norm step", op="norm", tokens=256, q_heads=32, k_heads=8, dim=128, rotary=128, interleaved=False,
             backward=False, reach=131072, type="bf16", weights="same"),
        # a step of training on packed sequences: forward and backward, master weights in float32
        dict(name="norm train", op="norm", tokens=16383, q_heads=32, k_heads=8, dim=128, rotary=128, interleaved=False,
             backward=True, reach=32768, type="bf16", weights="fp32"),
        # a prompt of a model of narrow heads, half of each turned
        dict(name="norm narrow", op="norm", tokens=4099, q_heads=16, k_heads=16, dim=64, rotary=32, interleaved=True,
             backward=True, reach=8192, type="fp16", weights="same"),
        # a single request of four beams, a step after the first: latency
        dict(name="select one", op="select", groups=1, beams=4, vocab=32000, width=4, banned=0.0, ended=0.0, first=False, type="bf16"),
        # 64 requests of eight beams over a large vocabulary
        dict(name="select batch", op="select", groups=64, beams=8, vocab=131072, width=8, banned=0.0, ended=0.0, first=False, type="bf16"),
        # constrained decoding: banned tokens, beams that have ended, twice as many candidates as beams, an odd vocabulary
        dict(name="select banned", op="select", groups=9, beams=5, vocab=50261, width=10, banned=0.4, ended=0.2, first=False, type="fp32"),
        # the cache follows the selection: 32 requests of eight beams that share their prompt
        dict(name="reorder batch", op="reorder", groups=32, beams=8, prompt=2000, grown=500, heads=8, dim=128, page=16, layers=2),
        # the same for a single request
        dict(name="reorder one", op="reorder", groups=1, beams=4, prompt=700, grown=77, heads=8, dim=128, page=16, layers=1),
        # a decode step's attention weights, sequences of unequal lengths
        dict(name="weigh step", op="weigh", rows=64, new=1, longest=8192, spread=1.0, heads=8, group=4, dim=128, page=16,
             window=0, decay=1.0, type="bf16"),
        # the weights that a prompt's tokens give each other and what is cached
        dict(name="weigh prompt", op="weigh", rows=3, new=2048, longest=12000, spread=0.5, heads=8, group=4, dim=128, page=32,
             window=0, decay=0.9, type="bf16"),
        # 32 sequences cut to half of the longest, pairs of them sharing a prefix, in four layers
        dict(name="evict batch", op="evict", rows=32, longest=4096, keep=2048, recent=64, shared=2, heads=8, dim=128, page=16, layers=4),
        # one sequence loses a third: latency
        dict(name="evict one", op="evict", rows=1, longest=1500, keep=1000, recent=32, shared=0, heads=8, dim=64, page=16, layers=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "select", "select", "reorder", "weigh", "weigh", "evict"])
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64])
    if op == "norm":
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        return dict(op=op, tokens=_log(rng, 1, 16384 * 128 // max(dim, 128)), q_heads=rng.randint(1, 32), k_heads=rng.randint(1, 8), dim=dim,
                    rotary=rng.choice([dim, dim // 2, 32]), interleaved=rng.random() < 0.5, backward=rng.random() < 0.6,
                    reach=_log(rng, 2000, 131072), type=rng.choice(["bf16", "fp16", "fp32"]) if dim < 128 else rng.choice(["bf16", "fp16"]),
                    weights=rng.choice(["same", "fp32"]))
    if op == "select":
        beams, vocab = rng.randint(1, 16), _log(rng, 500, 262144)
        groups = _log(rng, 1, max(1, min(64, (1 << 25) // (beams * vocab))))
        return dict(op=op, groups=groups, beams=beams, vocab=vocab, width=rng.choice([beams, beams, 2 * beams]),
                    banned=rng.choice([0.0, 0.0, rng.uniform(0.1, 0.9)]), ended=rng.choice([0.0, 0.3]), first=rng.random() < 0.2,
                    type=rng.choice(["bf16", "fp16", "fp32"]))
    if op == "reorder":
        beams = rng.randint(2, 8)
        return dict(op=op, groups=_log(rng, 1, 32), beams=beams, prompt=_log(rng, 4, 2000), grown=_log(rng, 1, 500),
                    heads=rng.choice([1, 4, 8]), dim=dim, page=page, layers=rng.randint(1, 2) if page < 64 else 1)
    if op == "evict":
        rows, longest = _log(rng, 1, 32), _log(rng, 40, 4096)
        keep = rng.randint(1, longest - 1)
        return dict(op=op, rows=rows, longest=longest, keep=keep, recent=rng.randint(0, keep), shared=rng.randint(0, 3),
                    heads=rng.choice([1, 2, 4, 8]), dim=dim, page=page, layers=rng.randint(1, 4))
    heads, group = rng.choice([(1, 8), (2, 4), (4, 4), (8, 1), (8, 4), (4, 6), (16, 1), (3, 5)])
    if rng.random() < 0.6:
        rows = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.7 else rng.randint(2, 6)
        longest = _log(rng, 1, min(65536, (1 << 29) // (rows * heads * dim)))
    else:
        rows = rng.randint(1, 3)
        new = _log(rng, 8, 2048)
        longest = new + _log(rng, 1, 12000 - new)
    return dict(op=op, rows=rows, new=new, longest=longest, spread=rng.choice([0.0, 0.3, 1.0]), heads=heads, group=group, dim=dim,
                page=page, window=rng.choice([0, 0, 0, rng.randint(1, longest)]), decay=rng.choice([1.0, 1.0, 0.9]),
                type=rng.choice(["bf16", "fp16"]))


def _rows(case):
    """(new tokens, length) of each sequence of a weighing: fixed by the case, so that work() knows them too."""
    r = random.Random("%d %d %d" % (case["rows"], case["new"], case["longest"]))
    new, length = [], []
    for b in range(case["rows"]):
        n = case["new"] if b == 0 or case["new"] < 8 else r.randint(1, case["new"])
        low = 1.0 - case["spread"]
        m = case["longest"] if b == 0 else int(case["longest"] * (low + (1 - low) * r.random() ** 2))
        if b % 16 == 15 and case["spread"] == 1.0:
            m = 0                                       # a place of the batch that holds no sequence
        elif case["new"] >= 8:
            m = max(m, n)
        new.append(n)
        length.append(m)
    return new, length


def _evict_lengths(case):
    r = random.Random("%d %d %d" % (case["rows"], case["longest"], case["keep"]))
    return [case["longest"] if b == 0 else r.randint(max(1, case["longest"] // 4), case["longest"]) for b in range(case["rows"])]


def _reorder_lengths(case):
    """(prompt, length) of each request."""
    r = random.Random("%d %d %d" % (case["groups"], case["prompt"], case["grown"]))
    out = [(case["prompt"], case["prompt"] + case["grown"])]
    for _ in range(case["groups"] - 1):
        p = r.randint(max(1, case["prompt"] // 2), case["prompt"])
        out.append((p, p + r.randint(1, case["grown"])))
    return out


def _pairs(new, length, window):
    """Visible (query, token) pairs and the tokens some query sees."""
    pairs = seen = 0
    for n, m in zip(new, length):
        first = max(0, m - n)
        if window:
            pairs += sum(min(p + 1, window) for p in range(first, m))
            seen += m - max(0, first - window + 1) if m else 0
        else:
            pairs += (first + 1 + m) * (m - first) // 2
            seen += m
    return pairs, seen


def _size(case):
    return 4 if case.get("type") == "fp32" else 2


def work(case):
    c = case
    if c["op"] == "norm":
        n = c["tokens"] * (c["q_heads"] + c["k_heads"])
        return {"bytes": (5 if c["backward"] else 2) * n * c["dim"] * _size(c), "flops": (20 if c["backward"] else 8) * n * c["dim"]}
    if c["op"] == "select":
        n = c["groups"] * c["beams"] * c["vocab"]
        return {"bytes": int(n * (1 - c["ended"])) * _size(c) + 12 * c["groups"] * c["width"], "flops": 3 * n}
    if c["op"] == "reorder":
        page_bytes = 2 * c["layers"] * c["heads"] * (c["page"] * c["dim"] + 4)
        lens = _reorder_lengths(c)
        moved = sum(m % c["page"] > 0 for _, m in lens) * c["beams"] // 2
        return {"bytes": moved * 2 * page_bytes + c["beams"] * 16 * sum(-(-m // c["page"]) for _, m in lens), "flops": 0}
    if c["op"] == "evict":
        lens = _evict_lengths(c)
        kept = sum(min(m, c["keep"]) for m in lens)
        moved = sum(c["keep"] for m in lens if m > c["keep"])
        per = c["layers"] * c["heads"]
        weights = sum(m for m in lens if m > c["keep"]) * 4 + moved * 4
        return {"bytes": per * (moved * 4 * c["dim"] + weights + kept * c["dim"] * 2 * 3), "flops": per * (moved * 4 + kept * 2) * c["dim"]}
    new, length = _rows(c)
    pairs, seen = _pairs(new, length, c["window"])
    heads = c["heads"] * c["group"]
    return {"bytes": seen * c["heads"] * (c["dim"] + 8) + sum(new) * heads * (2 * c["dim"] + 4), "flops": 2 * c["dim"] * heads * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _frequencies(rotary):
    """Radians a position of each pair, in 64 bits."""
    return 10000.0 ** (-2.0 * torch.arange(rotary // 2, dtype=torch.float64, device=DEV) / rotary)


def _table(counts, order):
    """Page tables of sequences with `counts` pages each, taken from `order` in turn."""
    counts = torch.tensor(counts, device=DEV, dtype=torch.int64)
    width = max(1, int(counts.max()))
    slot = torch.arange(width, device=DEV)
    at = (counts.cumsum(0) - counts)[:, None] + slot
    return torch.where(slot < counts[:, None], order[at.clamp(max=len(order) - 1)], -1).to(torch.int32)


def _pool(pages, layers, heads, page, dim, g):
    """Codes as quantised keys and values have them, a power of two as each block's scale."""
    def codes(*shape):
        out = torch.empty(shape, dtype=torch.uint8, device=DEV)
        flat = out.view(-1)
        for at in range(0, flat.numel(), 1 << 28):       # bounds the float32 copy
            n = min(1 << 28, flat.numel() - at)
            x = torch.randn(n, device=DEV, generator=g).mul_(100.0).clamp_(-448.0, 448.0)
            flat[at:at + n] = x.to(F8).view(torch.uint8)
        return out
    k, v = codes(pages, layers, heads, page, dim), codes(pages, layers, heads, dim, page)
    scale = torch.exp2(torch.randint(-8, -5, (pages, layers, 2, heads), device=DEV, generator=g).float())
    return k, v, scale


def _cache(k, v, scale, table, lengths):
    """The cache as a program holds it."""
    lengths = torch.tensor(lengths, device=DEV, dtype=torch.int32)
    refs = torch.bincount(table[table >= 0].long(), minlength=k.shape[0]).to(torch.int32)
    if not own:
        return types.SimpleNamespace(k=k.view(F8), v=v.view(F8), scale=scale, table=table, lengths=lengths, refs=refs)
    from paper_2608_07971_amd import kv
    return kv.PagedCache.adopt(k.view(F8), v.view(F8), scale, table, lengths, refs)


def _offsets(counts):
    return torch.tensor([0] + counts, device=DEV, dtype=torch.int32).cumsum(0).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    s = types.SimpleNamespace(case=case)
    {"norm": _prepare_norm, "select": _prepare_select, "reorder": _prepare_reorder, "weigh": _prepare_weigh,
     "evict": _prepare_evict}[case["op"]](s, case, g)
    return s


def _prepare_norm(s, case, g):
    dt, D, T = TYPES[case["type"]], case["dim"], case["tokens"]
    wt = torch.float32 if case["weights"] == "fp32" else dt
    s.positions = torch.randint(0, case["reach"], (T,), device=DEV, generator=g, dtype=torch.int32)
    s.q, s.k = ((torch.randn(T, h, D, device=DEV, generator=g) * 3.0).to(dt) for h in (case["q_heads"], case["k_heads"]))
    s.qw, s.kw = ((1.0 + 0.2 * torch.randn(D, device=DEV, generator=g)).to(wt) for _ in range(2))
    if case["backward"]:
        s.dq, s.dk = (torch.randn(x.shape, device=DEV, generator=g).to(dt) for x in (s.q, s.k))
        for x in (s.q, s.k, s.qw, s.kw):
            x.requires_grad_(True)
    if own:
        from paper_2608_07971_amd import kv
        s.rope = kv.Rope(D, rotary_dim=case["rotary"], interleaved=case["interleaved"])
    else:
        s.frequencies = _frequencies(case["rotary"])


def _prepare_select(s, case, g):
    dt, G, B, V = TYPES[case["type"]], case["groups"], case["beams"], case["vocab"]
    x = torch.randn(G, B, V, device=DEV, generator=g) * 2.5
    if case["banned"]:                                   # the same tokens for every beam of a request
        x.masked_fill_((torch.rand(G, 1, V, device=DEV, generator=g) < case["banned"]), -math.inf)
    s.logits = x.to(dt)
    s.scores = -5.0 - 60.0 * torch.rand(G, B, device=DEV, generator=g) * torch.rand(G, 1, device=DEV, generator=g)
    if case["first"]:                                    # the first step: only one beam of each request counts
        s.scores = torch.full((G, B), -math.inf, device=DEV)
        s.scores[:, 0] = 0.0
    s.ended = (torch.rand(G, B, device=DEV, generator=g) < case["ended"]) if case["ended"] else None


def _prepare_reorder(s, case, g):
    B, T = case["beams"], case["page"]
    lens = _reorder_lengths(case)
    shared = [p // T for p, _ in lens]                   # full pages of the prompt, which the beams share
    counts = [-(-m // T) - n for (_, m), n in zip(lens, shared) for _ in range(B)]
    P = sum(shared) + sum(counts) + B * len(lens) + 8
    order = torch.randperm(P, device=DEV, generator=g).to(torch.int32)
    front, back = _table(shared, order), _table(counts, order[sum(shared):])
    width = max(-(-m // T) for _, m in lens)
    table = torch.full((len(counts), width), -1, device=DEV, dtype=torch.int32)
    for i, n in enumerate(shared):
        rows = slice(i * B, i * B + B)
        table[rows, :n] = front[i, :n]
        table[rows, n:n + counts[i * B]] = back[rows, :counts[i * B]]
    k, v, scale = _pool(P, case["layers"], case["heads"], T, case["dim"], g)
    s.cache = _cache(k, v, scale, table, [m for _, m in lens for _ in range(B)])
    pick = torch.randint(0, B, (len(lens), B), device=DEV, generator=g, dtype=torch.int32)
    pick[:, 0] = torch.where(pick[:, 0] < B // 2, 0, pick[:, 0])                 # the best often goes on
    s.parents = (pick + torch.arange(len(lens), device=DEV, dtype=torch.int32)[:, None] * B).view(-1)
    if len(lens) >= 4:
        s.parents[-B:] = -1                              # a request that is done


def _prepare_weigh(s, case, g):
    H, G, D, T = case["heads"], case["group"], case["dim"], case["page"]
    s.new, s.length = _rows(case)
    counts = [-(-m // T) for m in s.length]
    P, tokens = sum(counts) + 8, sum(s.new)
    table = _table(counts, torch.randperm(P, device=DEV, generator=g).to(torch.int32))
    k, v, scale = _pool(P, 1, H, T, D, g)
    s.cache = _cache(k, v, scale, table, s.length)
    s.offsets = _offsets(s.new)
    s.q = (torch.randn(tokens, H * G, D, device=DEV, generator=g) * 1.4).to(TYPES[case["type"]])
    s.mass = torch.rand(1, case["rows"], H, table.shape[1] * T, device=DEV, generator=g) ** 4
    score, row, i = _scores(s)                           # the statistics that the attention before left
    top = score.amax(-1, keepdim=True)
    lse = (top + torch.log(torch.exp(score - torch.where(top == -math.inf, 0.0, top)).sum(-1, keepdim=True)))[..., 0]
    s.lse = lse.permute(0, 3, 1, 2)[row, i].reshape(tokens, H * G).contiguous()


def _prepare_evict(s, case, g):
    T, L, H, R = case["page"], case["layers"], case["heads"], case["rows"]
    s.length = _evict_lengths(case)
    counts = [-(-m // T) for m in s.length]
    P = sum(counts) + 2 * case["shared"] * R + 8
    table = _table(counts, torch.randperm(P, device=DEV, generator=g).to(torch.int32))
    for b in range(1, R, 2):                             # pairs of sequences share the pages of a prefix
        n = min(case["shared"], s.length[b] // T, s.length[b - 1] // T)
        table[b, :n] = table[b - 1, :n]
    k, v, scale = _pool(P, L, H, T, case["dim"], g)
    s.cache = _cache(k, v, scale, table, s.length)
    s.full = s.cache.lengths.clone()
    s.keep = torch.full((R,), case["keep"], device=DEV, dtype=torch.int32)
    # a few tokens get most of the weight, some get none
    x = torch.exp(3.0 * torch.randn(L, R, H, table.shape[1] * T, device=DEV, generator=g))
    s.mass = x.masked_fill_(torch.rand(x.shape, device=DEV, generator=g) < 0.05, 0.0)
    kept = [min(m, case["keep"]) for m in s.length]
    s.kept, s.total = _offsets(kept), sum(kept)
    s.starts = torch.zeros(R, device=DEV, dtype=torch.int32)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)[s.case["op"]](s)


def _pool_of(c):
    return {"k": c.k.view(torch.uint8), "v": c.v.view(torch.uint8), "scale": c.scale}


def _own_norm(s):
    from paper_2608_07971_amd import kv
    q, k = kv.norm_rotate(s.rope, s.q, s.k, s.qw, s.kw, s.positions, eps=EPS)
    if not s.case["backward"]:
        return {"q": q, "k": k}
    dq, dk, dqw, dkw = torch.autograd.grad((q, k), (s.q, s.k, s.qw, s.kw), (s.dq, s.dk))
    return {"q": q.detach(), "k": k.detach(), "dq": dq, "dk": dk, "dqw": dqw, "dkw": dkw}


def _own_select(s):
    from paper_2608_07971_amd import kv
    scores, parents, tokens = kv.select_beams(s.logits, s.scores, s.case["width"], ended=s.ended, pad=0)
    return {"scores": scores, "parents": parents, "tokens": tokens}


def _own_reorder(s):
    s.cache.reorder(s.parents)
    return dict(table=s.cache.table, lengths=s.cache.lengths, refs=s.cache.refs, **_pool_of(s.cache))


def _own_weigh(s):
    s.cache.weigh(0, s.q, s.lse, s.offsets, s.mass, window=s.case["window"], decay=s.case["decay"], max_new=s.case["new"],
                  max_length=s.case["longest"])
    return {"mass": s.mass}


def _own_evict(s):
    s.cache.resize(s.full)                               # later passes: the sequences have grown again
    s.cache.evict(s.keep, s.mass, recent=s.case["recent"])
    k, v = zip(*(s.cache.gather(layer, s.starts, s.kept, s.total) for layer in range(s.case["layers"])))
    return dict(table=s.cache.table, lengths=s.cache.lengths, refs=s.cache.refs, mass=s.mass, k=list(k), v=list(v))


_run_own = {"norm": _own_norm, "select": _own_select, "reorder": _own_reorder, "weigh": _own_weigh, "evict": _own_evict}


# Plain forms: elementary operations in 32 bits, rounded once at the end.

def _turn(x, cos, sin, case):
    """The rotary part of x [tokens][heads][dim] turned by angles [tokens][1][pairs]."""
    rot = case["rotary"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((y, z), -1).flatten(-2) if case["interleaved"] else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_norm(s):
    case, D = s.case, s.case["dim"]
    angle = s.positions.double()[:, None, None] * s.frequencies
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {}
    with torch.no_grad():
        for name, x, w in (("q", s.q, s.qw), ("k", s.k, s.kw)):
            f, weight = x.float(), w.float()
            r = torch.rsqrt((f * f).sum(-1, keepdim=True) / D + EPS)
            n = f * r
            out[name] = _turn(n * weight, cos, sin, case).to(x.dtype)
            if case["backward"]:
                g = _turn((s.dq if name == "q" else s.dk).float(), cos, -sin, case)
                out["d" + name + "w"] = (g * n).sum((0, 1)).to(w.dtype)
                g = g * weight
                out["d" + name] = (r * (g - n * ((g * n).sum(-1, keepdim=True) / D))).to(x.dtype)
    return out


def _plain_select(s):
    case = s.case
    B, V, W = case["beams"], case["vocab"], case["width"]
    x = s.logits.double()                                # neighbours at the border lie closer than 32 bits tell
    top = x.amax(-1, keepdim=True)
    # a row's sum is taken in the same order wherever the row lies
    e = torch.nn.functional.pad(torch.exp(x - torch.where(top == -math.inf, 0.0, top)), (0, -V % 64))
    lse = top + torch.log(e.sum(-1, keepdim=True))
    score = s.scores.double()[..., None] + (x - lse)
    if s.ended is not None:
        score = torch.where(s.ended[..., None], -math.inf, score)
        score[..., 0] = torch.where(s.ended, s.scores.double(), score[..., 0])
    score = torch.where(score == score, score, -math.inf).view(case["groups"], B * V)
    best, at = torch.topk(score, min(8 * W + 64, B * V), -1)                          # ties among these go to the lowest index
    at, order = torch.sort(at, -1)
    best, again = torch.sort(best.gather(-1, order), dim=-1, descending=True, stable=True)
    best, at = best[:, :W], at.gather(-1, again)[:, :W]
    there = best > -math.inf
    group = torch.arange(case["groups"], device=DEV)[:, None] * B
    return {"scores": best.float(), "parents": torch.where(there, at // V + group, -1).to(torch.int32),
            "tokens": torch.where(there, at % V, -1).to(torch.int32)}


def _copy_pages(c, source, to):
    for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.scale):
        t[to] = t[source]


def _plain_reorder(s):
    c, T, parents = s.cache, s.case["page"], s.parents.long()
    n = parents.shape[0]
    own_row = torch.arange(n, device=DEV)
    there = parents >= 0
    rows = torch.where(there[:, None], c.table[parents.clamp(min=0)], -1)
    length = torch.where(there, c.lengths[parents.clamp(min=0)], 0)
    # the child that goes on with its parent's partly filled page: the parent itself, or the first
    first = torch.full((n,), n, device=DEV).scatter_reduce(0, parents.clamp(min=0), torch.where(there, own_row, n), "amin")
    stays = parents.clamp(min=0)[parents.clamp(min=0)] == parents.clamp(min=0)
    keeper = torch.where(stays & there, parents, first[parents.clamp(min=0)])
    slot = torch.arange(rows.shape[1], device=DEV)
    copied = (slot == (length // T)[:, None]) & (length % T > 0)[:, None] & (keeper != own_row)[:, None] & there[:, None]
    shared = rows[(rows >= 0) & ~copied]
    refs = torch.zeros_like(c.refs).index_add_(0, shared.long(), torch.ones_like(shared))
    source = rows[copied]
    to = torch.nonzero(refs == 0)[:source.shape[0], 0].to(torch.int32)
    rows[copied] = to
    refs[to.long()] = 1
    _copy_pages(c, source.long(), to.long())
    c.table.copy_(rows)
    c.lengths.copy_(length)
    c.refs.copy_(refs)
    return dict(table=c.table, lengths=c.lengths, refs=c.refs, **_pool_of(c))


def _token_rows(offsets, tokens):
    """The sequence of each token and its number within it."""
    at = torch.arange(tokens, device=DEV)
    row = torch.searchsorted(offsets[1:].long(), at, right=True)
    return row, at - offsets.long()[row]


def _scores(s):
    """Scores [sequence][head][query head of it][new token][token] in 32 bits, -inf where a token is not seen, and the
    sequence and number of each new token."""
    c, case = s.cache, s.case
    H, G, D = case["heads"], case["group"], case["dim"]
    B, tokens, most = case["rows"], s.q.shape[0], max(s.new)
    pages = c.table.clamp(min=0).long()
    k = c.k.view(torch.uint8)[pages, 0].view(F8).float() * c.scale[pages, 0][..., 0, :, None, None]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    row, i = _token_rows(s.offsets, tokens)
    q = torch.zeros(B, most, H, G, D, device=DEV)
    q[row, i] = s.q.float().view(tokens, H, G, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(B, H, G * most, D)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(D)
    score = score.view(B, H, G, most, -1)
    new = (s.offsets[1:] - s.offsets[:-1]).long()
    p = (c.lengths.long() - new)[:, None] + torch.arange(most, device=DEV)
    t = torch.arange(k.shape[2], device=DEV)
    seen = (t <= p[..., None]) & (t < c.lengths.long()[:, None, None])
    if case["window"]:
        seen &= t > p[..., None] - case["window"]
    return score.masked_fill_(~seen[:, None, None], -math.inf), row, i


def _plain_weigh(s):
    c, case = s.cache, s.case
    H, G = case["heads"], case["group"]
    score, row, i = _scores(s)
    B, most = score.shape[0], score.shape[3]
    lse = torch.full((B, most, H, G), math.inf, device=DEV)
    lse[row, i] = s.lse.view(-1, H, G)
    lse = lse.permute(0, 2, 3, 1)[..., None]
    weight = torch.exp(score - torch.where(lse == -math.inf, math.inf, lse)).sum((2, 3))
    new = (s.offsets[1:] - s.offsets[:-1]).long()
    t, length = torch.arange(weight.shape[-1], device=DEV), c.lengths.long()
    old = (t < (length - new)[:, None])[:, None]
    now = torch.where(old, s.mass[0] * case["decay"], 0.0) + weight
    s.mass[0] = torch.where((t < length[:, None])[:, None], now, s.mass[0])
    return {"mass": s.mass}


def _plain_grow(c, T, length):
    """Sequences get the pages that their new lengths need: the free ones of lowest number, by sequence and slot."""
    slot = torch.arange(c.table.shape[1], device=DEV)
    need = (slot < (-(-length // T))[:, None]) & (c.table < 0)
    to = torch.nonzero(c.refs == 0)[:int(need.sum()), 0].to(torch.int32)
    c.refs[to.long()] = 1
    c.table[need] = to
    c.lengths.copy_(length)


def _plain_evict(s):
    c, case, T = s.cache, s.case, s.case["page"]
    L, H, keep = case["layers"], case["heads"], case["keep"]
    _plain_grow(c, T, s.full)
    length = c.lengths.long()
    cut = torch.nonzero(length > keep)[:, 0]
    n = cut.shape[0]
    t = torch.arange(s.mass.shape[-1], device=DEV)
    # the tokens that stay: the last `recent`, then by weight, then the lower index
    rank = torch.where(t < length[cut, None, None], s.mass[:, cut], -math.inf)
    recent = min(case["recent"], keep)
    rank = torch.where((t >= length[cut, None, None] - recent) & (t < length[cut, None, None]), math.inf, rank)
    kept = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :keep].sort(-1)[0]      # [L][n][H][keep]
    # private pages for them: a page that others name is replaced by a free one
    slots = -(-keep // T)
    old = c.table[cut]
    to = old[:, :slots].clone()
    others = c.refs[to.long()] > 1
    free = torch.nonzero(c.refs == 0)[:int(others.sum()), 0].to(torch.int32)
    to[others] = free
    gone = torch.cat((old[:, :slots][others], old[:, slots:][old[:, slots:] >= 0])).long()
    c.refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    c.refs[free.long()] = 1
    # codes and scales of the kept tokens, then the largest scale of each new page
    layer = torch.arange(L, device=DEV)[:, None, None, None]
    head = torch.arange(H, device=DEV)[:, None]
    page = old[torch.arange(n, device=DEV)[None, :, None, None], kept // T].long()
    pad = slots * T - keep
    moved = []
    for which, codes in ((0, c.k.view(torch.uint8)[page, layer, head, kept % T]),
                         (1, c.v.view(torch.uint8)[page, layer, head, :, kept % T])):
        was = c.scale[page, layer, which, head]
        now = torch.nn.functional.pad(was, (0, pad)).view(L, n, H, slots, T).amax(-1)
        by = was / now.repeat_interleave(T, -1)[..., :keep]
        x = (codes.view(F8).float() * by[..., None]).to(F8).view(torch.uint8)
        moved.append((which, x, now))
    place = to[:, torch.arange(keep, device=DEV) // T].long()[None, :, None]                  # [1][n][1][keep]
    at = (torch.arange(keep, device=DEV) % T)[None, None, None]
    for which, x, now in moved:
        if which == 0:
            c.k.view(torch.uint8)[place, layer, head, at] = x
        else:
            c.v.view(torch.uint8)[place, layer, head, :, at] = x
        c.scale[to.long()[None, :, None], layer, which, head] = now
    s.mass[:, cut, :, :keep] = s.mass[:, cut].gather(-1, kept)
    rows = torch.full_like(old, -1)
    rows[:, :slots] = to
    c.table[cut] = rows
    c.lengths[cut] = keep
    # what the cache holds now, token after token
    row, i = _token_rows(s.kept, s.total)
    page, at = c.table[row, i // T].long(), i % T
    k, v = [], []
    for layer in range(L):
        kk = c.k.view(torch.uint8)[page, layer, :, at].view(F8).float() * c.scale[page, layer, 0][..., None]
        vv = c.v.view(torch.uint8)[page, layer, :, :, at].view(F8).float() * c.scale[page, layer, 1][..., None]
        k.append(kk.to(torch.bfloat16))
        v.append(vv.to(torch.bfloat16))
    return dict(table=c.table, lengths=c.lengths, refs=c.refs, mass=s.mass, k=k, v=v)


_run_plain = {"norm": _plain_norm, "select": _plain_select, "reorder": _plain_reorder, "weigh": _plain_weigh, "evict": _plain_evict}


# ---------------------------------------------------------------------------
# The same from the definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "select": _exact_select, "reorder": lambda s: None, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["op"]](s)


def _exact_norm(s):
    case, rot = s.case, s.case["rotary"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s.positions.double()[:, None, None] * _frequencies(rot))

    def forward(x, w):
        y = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
        if case["interleaved"]:
            z = torch.view_as_real(torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
        else:
            z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
            z = torch.cat((z.real, z.imag), -1)
        return torch.cat((z, y[..., rot:]), -1)

    out = {}
    for name, x, w in (("q", s.q, s.qw), ("k", s.k, s.kw)):
        x, w = (t.detach().double().requires_grad_(case["backward"]) for t in (x, w))
        y = forward(x, w)
        out[name] = y.detach()
        if case["backward"]:
            out["d" + name], out["d" + name + "w"] = torch.autograd.grad(y, (x, w), (s.dq if name == "q" else s.dk).double())
    return out


def _exact_select(s):
    case = s.case
    rows = []
    for g in range(case["groups"]):
        best = []
        for b in range(case["beams"]):
            score = s.scores[g, b].double()
            if not bool(torch.isfinite(score)):
                continue
            if s.ended is not None and bool(s.ended[g, b]):
                best.append(score.view(1))
                continue
            x = s.logits[g, b].double()
            x = torch.sort(x[x > -math.inf], descending=True)[0]
            best.append(x[:case["width"]] - torch.logsumexp(x, 0) + score)
        best = torch.sort(torch.cat(best), descending=True)[0][:case["width"]] if best else torch.empty(0, dtype=torch.float64, device=DEV)
        rows.append(torch.nn.functional.pad(best, (0, case["width"] - best.shape[0]), value=-math.inf))
    return {"scores": torch.stack(rows), "parents": None, "tokens": None}


def _exact_weigh(s):
    c, case = s.cache, s.case
    T, H, G, D = case["page"], case["heads"], case["group"], case["dim"]
    mass, at = s.mass.double(), 0
    for b, (n, m) in enumerate(zip(s.new, s.length)):
        pages = c.table[b, :-(-m // T)].long()
        k = c.k.view(torch.uint8)[pages, 0].view(F8).double() * c.scale[pages, 0, 0].double()[..., None, None]
        k = k.permute(1, 0, 2, 3).reshape(H, -1, D)[:, :m]
        p, t = torch.arange(m - n, m, device=DEV)[:, None], torch.arange(m, device=DEV)
        hidden = (t > p) | ((t <= p - case["window"]) if case["window"] else False)
        q, lse = s.q[at:at + n].double().view(n, H, G, D), s.lse[at:at + n].double().view(n, H, G)
        for h in range(H if m else 0):
            total = torch.zeros(m, dtype=torch.float64, device=DEV)
            for e in range(G):
                w = torch.exp(q[:, h, e] @ k[h].T / math.sqrt(D) - lse[:, h, e, None])
                total += torch.where(hidden, 0.0, w).sum(0)
            mass[0, b, h, :max(0, m - n)] *= case["decay"]
            mass[0, b, h, max(0, m - n):m] = 0.0
            mass[0, b, h, :m] += total
        at += n
    return {"mass": mass}


def _exact_evict(s):
    """The numbers that the cache stands for, before a smaller block's codes are rounded to a larger one's scale."""
    c, case = s.cache, s.case
    T, H, keep = case["page"], case["heads"], case["keep"]
    out = {"table": None, "lengths": None, "refs": None, "mass": None, "k": [], "v": []}
    for layer in range(case["layers"]):
        ks, vs = [], []
        for b, m in enumerate(s.length):
            pages = c.table[b, :-(-m // T)].long()
            scale = c.scale[pages, layer].double()
            k = (c.k.view(torch.uint8)[pages, layer].view(F8).double() * scale[:, 0, :, None, None]).permute(1, 0, 2, 3).reshape(H, -1, case["dim"])
            v = (c.v.view(torch.uint8)[pages, layer].view(F8).double() * scale[:, 1, :, None, None]).permute(1, 0, 3, 2).reshape(H, -1, case["dim"])
            if m > keep:
                recent = min(case["recent"], keep)
                older = s.mass[layer, b, :, :m - recent]
                best = torch.argsort(-older, dim=-1, stable=True)[:, :keep - recent].sort(-1)[0]
                stay = torch.cat((best, torch.arange(m - recent, m, device=DEV).expand(H, -1)), -1)[..., None].expand(-1, -1, case["dim"])
                k, v = k.gather(1, stay), v.gather(1, stay)
            else:
                k, v = k[:, :m], v[:, :m]
            ks.append(k.transpose(0, 1))
            vs.append(v.transpose(0, 1))
        out["k"].append(torch.cat(ks))
        out["v"].append(torch.cat(vs))
    return out
