"""Answering with drafted tokens: cases to be timed, their plain forms and their values in 64 bits.

Four operators that belong together.  A small model drafts a tree of tokens for every sequence; the large one looks at all of them in one pass, in which their keys,
turned to their positions, go into the paged cache in 4 bits ("rotate") and every token attends to the sequence and to its own ancestors ("tree"); given random numbers
decide which of them stand ("verify"), and the cache keeps those and no others ("keep").  `run` computes them in elementary torch operations (`own` false) or through the
public functions of `paper_2012_01114_b200.binding` (`own` true).

A tree is given by `parents`: the parent of a token among its sequence's tokens of this pass, an earlier one, or -1.  Token 0, the root, is the last one of the answer so far.

The cache.  A page holds `page` tokens (a multiple of 16) of all key/value heads of a layer as [kv_heads][page / 16] blocks of
20 d bytes, a block being 16 tokens of one head:
    K codes  [16 tokens][4 t][d/32 groups] words of 32 bits: bits 4j .. 4j+3 hold channel 32 w + 8 t + 2 j, bits 16 + 4j .. the next one
    K scales [16 tokens][d/32 groups] pairs (S, M) of fp16
    V codes  [8 pairs of tokens][8 g][d/32 groups] words: bits 4j .. hold channel 32 w + 4 g + j of the even token, bits 16 + 4j .. of the odd one
    V scales [8 pairs of tokens][d/32 groups] (S even, S odd, M even, M odd) of fp16
A code c of a group of 32 channels stands for M + S (1 + c / 16).
"""
import math
import random

import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HELD_MAX = 20000.0          # numbers beyond this are held as this


# ---------------------------------------------------------------- cases
def _rotate(name, seqs, longest, held, heads, kv_heads, d, rot, interleaved, page, dtype, lengths, depth=0):
    """`longest`: most tokens of a sequence in this pass; `held`: most that it holds before; `depth`: of their tree (0: one after another); `rot`: channels that turn."""
    return dict(name=name, op="rotate", seqs=seqs, longest=longest, held=held, heads=heads, kv_heads=kv_heads, d=d, rot=rot, interleaved=interleaved, page=page, dtype=dtype, lengths=lengths,
                depth=depth)


def _tree(name, seqs, longest, tree, depth, heads, kv_heads, d, page, dtype, lengths):
    """`longest`: most tokens held, those of the tree among them; `tree`: most tokens of a tree, `depth`: its levels below the root."""
    return dict(name=name, op="tree", seqs=seqs, longest=longest, tree=tree, depth=depth, heads=heads, kv_heads=kv_heads, d=d, page=page, dtype=dtype, lengths=lengths)


def _verify(name, seqs, tree, depth, branch, vocab, drafts, temperature, dtype, lengths):
    """`branch`: most children of a token; `drafts`: whether the drafts were drawn from probabilities that are given too, or are the likeliest tokens; `temperature` 0: the likeliest token stands."""
    return dict(name=name, op="verify", seqs=seqs, tree=tree, depth=depth, branch=branch, vocab=vocab, drafts=drafts, temperature=temperature, dtype=dtype, lengths=lengths)


def _keep(name, seqs, longest, tree, depth, kv_heads, d, page, layers, lengths):
    return dict(name=name, op="keep", seqs=seqs, longest=longest, tree=tree, depth=depth, kv_heads=kv_heads, d=d, page=page, layers=layers, lengths=lengths)


def listed():
    return [
        # one token of a small model: latency and nothing else
        _rotate("rotate one", 1, 1, 300, 8, 2, 64, 64, False, 16, "bf16", 1),
        # a tree of drafted tokens for each sequence of a full batch
        _rotate("rotate drafts", 64, 16, 4000, 32, 8, 128, 128, False, 64, "bf16", 2, 5),
        # a packed batch of prompts, half of every head turning, neighbours together
        _rotate("rotate prompts", 16, 2500, 0, 32, 8, 128, 64, True, 64, "f16", 3),
        # one answer being written by a small model with a few drafted tokens: latency
        _tree("tree one", 1, 301, 6, 3, 8, 2, 64, 16, "bf16", 4),
        # a step of a full batch of answers of different lengths
        _tree("tree batch", 32, 8000, 12, 4, 32, 8, 128, 64, "bf16", 5),
        # two very long contexts: the long axis has to be split
        _tree("tree long", 2, 131072, 26, 6, 32, 8, 128, 128, "bf16", 6),
        # large trees for a few sequences, many query heads on few key heads: the products rule
        _tree("tree wide", 8, 6001, 64, 8, 32, 4, 128, 32, "f16", 7),
        # four tokens drafted in a row for one answer, the likeliest token stands: latency
        _verify("verify greedy", 1, 5, 4, 1, 32000, False, 0.0, "bf16", 8),
        # a full batch of drafted rows with the small model's probabilities
        _verify("verify rows", 64, 6, 5, 1, 128000, True, 0.8, "bf16", 9),
        # trees of drafted tokens, several to choose from at each, in 32 bits and with an odd number of words
        _verify("verify trees", 16, 33, 6, 4, 50001, True, 1.0, "f32", 10),
        # what stands of one tree moves together in a small model's layers: latency
        _keep("keep one", 1, 301, 8, 4, 2, 64, 16, 4, 11),
        # the same for a full batch and a larger model
        _keep("keep batch", 64, 2000, 24, 6, 8, 128, 64, 16, 12),
    ]


def _log(rng, low, high):
    v = max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))
    return v


def draw(rng):
    op = rng.choice(["rotate", "tree", "verify", "keep"])
    kv_heads, group, d = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 6, 7, 8]), rng.choice([64, 96, 128])
    dtype, lengths, page = rng.choice(["bf16", "bf16", "f16"]), rng.randrange(1 << 20), rng.choice([16, 32, 64, 128])
    depth = rng.randint(1, 8)
    if op == "rotate":
        drafts = rng.random() < 0.6
        longest = rng.choice([1, _log(rng, 1, 64)]) if drafts else _log(rng, 1, 2500)
        seqs = _log(rng, 1, min(128, max(1, 20000 // longest)))
        case = _rotate("", seqs, longest, _log(rng, 1, 4000), kv_heads * group, kv_heads, d, 8 * rng.randint(1, d // 8), rng.random() < 0.5, page, dtype, lengths, depth if drafts else 0)
    elif op == "tree":
        longest = _log(rng, 8, 131072)
        seqs = _log(rng, 1, min(64, 262144 // longest))
        tree = min(longest, _log(rng, 1, 64))
        while tree > 4 and seqs * longest * tree * kv_heads * group > 3 << 28:
            tree //= 2
        case = _tree("", seqs, longest, tree, depth, kv_heads * group, kv_heads, d, page, dtype, lengths)
    elif op == "verify":
        vocab = _log(rng, 1000, 150000)
        tree = _log(rng, 1, 48)
        seqs = _log(rng, 1, max(1, min(64, (40 << 20) // (vocab * tree))))
        case = _verify("", seqs, tree, depth, rng.choice([1, 2, 3, 4]), vocab, rng.random() < 0.6, rng.choice([0.0, 0.6, 0.8, 1.0, 1.3]), rng.choice(["bf16", "f16", "f32"]), lengths)
    else:
        case = _keep("", _log(rng, 1, 96), _log(rng, 20, 2000), _log(rng, 2, 64), depth, kv_heads, d, page, rng.choice([1, 2, 4, 8]), lengths)
    return {k: v for k, v in case.items() if k != "name"}


def _lengths(case, salt, low, high):
    """As many numbers as the case has sequences, spread over the logarithm, the first one the largest."""
    r = random.Random(case["lengths"] * 16 + salt)
    return [high] + [_log(r, max(low, 1), max(high, 1)) if high else 0 for _ in range(case["seqs"] - 1)]


def _trees(case, sizes):
    """Trees of these many tokens as lists of parents, at most case["depth"] levels below the root and case["branch"] children a token; where that leaves no room, fewer tokens."""
    r, trees = random.Random(case["lengths"] * 16 + 9), []
    depth, branch = max(case["depth"], 1), case.get("branch", 4)
    for n in sizes:
        parents, level, children = [-1], [0], [0]
        for i in range(1, n):
            room = [k for k in range(i) if level[k] < depth and children[k] < branch]
            if not room:
                break
            p = r.choice(room[-8:])
            parents.append(p)
            level.append(level[p] + 1)
            children[p] += 1
            children.append(0)
        trees.append((parents, level))
    return trees


def _sizes(case):
    """Tokens of each sequence's tree, at most those that it holds."""
    held = _lengths(case, 1, 1, case["longest"]) if "longest" in case else [case["tree"]] * case["seqs"]
    low = (case["tree"] + 1) // 2
    n = [case["tree"]] + [random.Random(case["lengths"] * 16 + 20 + i).randint(low, case["tree"]) for i in range(1, case["seqs"])]
    trees = _trees(case, [min(a, b) for a, b in zip(n, held)])
    return trees, held


def _path(case, trees):
    """For "keep": what stands of each tree, a path from the root that ends by chance."""
    r, paths = random.Random(case["lengths"] * 16 + 11), []
    for parents, _ in trees:
        at, path = 0, [0]
        while True:
            below = [i for i, p in enumerate(parents) if p == at]
            if not below or r.random() < 0.15:
                break
            at = r.choice(below)
            path.append(at)
        paths.append(path)
    return paths


def _new_and_old(case):
    new = _lengths(case, 1, 1, case["longest"])
    trees = _trees(case, new) if case["depth"] else None
    if trees:
        new = [len(p) for p, _ in trees]
    return new, _lengths(case, 2, 0, case["held"]), trees


def work(case):
    if case["op"] == "rotate":
        rows = sum(_new_and_old(case)[0])
        n = rows * case["kv_heads"] * case["d"] * 2
        q = rows * case["heads"] * case["d"]
        return {"bytes": 4 * q + 2 * n + 2 * n + 5 * n // 8, "flops": 6 * n + 3 * rows * case["rot"] * (case["heads"] + case["kv_heads"])}
    if case["op"] == "tree":
        trees, held = _sizes(case)
        numbers = sum(held) * case["kv_heads"] * case["d"] * 2
        rows = sum(len(p) for p, _ in trees)
        weights = sum((h - len(p)) * len(p) + sum(level) + len(p) for (p, level), h in zip(trees, held)) * case["heads"]
        return {"bytes": 5 * numbers // 8 + 4 * rows * case["heads"] * (case["d"] + 1) + 4 * sum(-(-h // case["page"]) for h in held), "flops": 4 * weights * case["d"]}
    if case["op"] == "verify":     # the rows on the path: as drafts go, seven in ten levels stand
        rows = sum(sum(0.7 ** i for i in range(max(level) + 1)) for _, level in _sizes(case)[0])
        both = 2 if case["drafts"] and case["temperature"] else 1
        return {"bytes": int(rows * case["vocab"] * both * (4 if case["dtype"] == "f32" else 2)), "flops": int(4 * rows * case["vocab"] * both)}
    moved = sum(sum(i != p for i, p in enumerate(path)) for path in _path(case, _sizes(case)[0]))
    return {"bytes": 2 * moved * case["layers"] * case["kv_heads"] * case["d"] * 5 // 4 + 8 * case["seqs"] * (case["tree"] + 2), "flops": 0}


# ---------------------------------------------------------------- inputs
def _normal(gen, shape, dtype):
    return torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return _ints(at)


def _tables(held, page, pages, gen):
    """Pages for sequences of these lengths, in the order of chance; entries behind a sequence's last page are -1."""
    need = torch.tensor([-(-h // page) for h in held], device="cuda")
    width = max(1, int(need.max()))
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int64).int()
    col = torch.arange(width, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    return torch.where(col < need[:, None], order[at.clamp(max=pages - 1)], -1).int().contiguous()


def _cache(s, held, page, gen):
    pages = sum(-(-h // page) for h in held) + 3
    s["tables"], s["lens"], s["seqs"] = _tables(held, page, pages, gen), _ints(held), torch.arange(len(held), dtype=torch.int32, device="cuda")
    return pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "rotate":
        new, old, trees = _new_and_old(case)
        rows, H, Hkv, d, dtype = sum(new), case["heads"], case["kv_heads"], case["d"], DTYPES[case["dtype"]]
        qkv = _normal(gen, (rows, H + 2 * Hkv, d), dtype)      # one matrix product gives all three: they lie side by side
        offset = torch.empty((1, Hkv, d), device="cuda").normal_(generator=gen)     # keys have channels that are large in every token
        qkv[:, H:H + Hkv] += (2 * offset).to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        pages = _cache(s, [a + b for a, b in zip(new, old)], case["page"], gen)
        s["starts"] = _starts(new)
        s["depths"] = _ints([x for _, level in trees for x in level]) if trees else None
        s["freqs"] = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"])
        s["pool"] = torch.zeros((pages, Hkv * case["page"] * d * 5 // 4), dtype=torch.uint8, device="cuda")
        s["q_out"], s["k_held"], s["v_held"] = (torch.empty((rows, h, d), dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))
    elif case["op"] == "tree":
        trees, held = _sizes(case)
        H, Hkv, d, page, n = case["heads"], case["kv_heads"], case["d"], case["page"], [len(p) for p, _ in trees]
        s["parents"], s["starts"], s["max_q"] = _ints([x for p, _ in trees for x in p]), _starts(n), max(n)
        s["q"] = _normal(gen, (sum(n), H, d), DTYPES[case["dtype"]])
        pages = _cache(s, held, page, gen)
        s["pool"] = torch.empty((pages, Hkv * page * d * 5 // 4), dtype=torch.uint8, device="cuda")
        offset = torch.empty((Hkv, 1, d), device="cuda").normal_(generator=gen)
        step = max(1, (1 << 25) // (Hkv * page * d))
        for at in range(0, pages, step):       # (in parts: the pool is large)
            m = min(step, pages - at)
            k, v = (torch.empty((m, Hkv, page, d), device="cuda").normal_(generator=gen) for _ in range(2))
            s["pool"][at:at + m] = _pack(*(_quantise(x) for x in (k + offset, v)), page)
    elif case["op"] == "verify":
        trees, _ = _sizes(case)
        n = [len(p) for p, _ in trees]
        rows, V, dtype = sum(n), case["vocab"], DTYPES[case["dtype"]]
        s["starts"], s["parents"] = _starts(n), _ints([x for p, _ in trees for x in p])
        logits = torch.empty((rows, V), device="cuda").normal_(generator=gen).mul_(3)
        drafts = logits + torch.empty((rows, V), device="cuda").normal_(generator=gen).mul_(0.5)
        s["logits"], s["drafts"] = logits.to(dtype), drafts.to(dtype) if case["drafts"] else None
        chance = torch.empty((rows, V), device="cuda").exponential_(generator=gen).log_() if case["drafts"] else 0
        best = (drafts / max(case["temperature"], 0.1) - chance).topk(case["branch"]).indices      # drawn without replacement, or the likeliest
        base = [0]
        for p, _ in trees:
            base.append(base[-1] + len(p))
        row, nth = [], []
        for b, (p, _) in enumerate(trees):
            for i, x in enumerate(p):
                row.append(base[b] + max(x, 0))
                nth.append(sum(y == x for y in p[:i]))
        s["tokens"] = best[torch.tensor(row, device="cuda"), torch.tensor(nth, device="cuda")].int()
        s["uniform"] = torch.empty(rows, device="cuda").uniform_(generator=gen)
        s["temperatures"] = torch.full((case["seqs"],), case["temperature"], device="cuda")
        s["path"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        s["accepted"], s["next"] = (torch.empty(case["seqs"], dtype=torch.int32, device="cuda") for _ in range(2))
        s["levels"], s["branch"], s["most"] = max(max(level) for _, level in trees) + 1, max(max(p.count(x) for x in p) for p, _ in trees), max(n)
    else:
        trees, held = _sizes(case)
        n, paths = [len(p) for p, _ in trees], _path(case, trees)
        pages = _cache(s, held, case["page"], gen)
        s["starts"], s["new_lens"] = _starts(n), s["lens"].clone()
        s["path"] = _ints([x for m, p in zip(n, paths) for x in p + [-1] * (m - len(p))])
        s["accepted"] = _ints([len(p) - 1 for p in paths])
        s["pool"] = torch.randint(0, 256, (case["layers"], pages, case["kv_heads"] * case["page"] * case["d"] * 5 // 4), dtype=torch.uint8, device="cuda", generator=gen)
    return s


# ---------------------------------------------------------------- the cache's numbers and bytes
def _quantise(x):
    """[..., d] in 32 bits -> codes [..., d/32, 32], S and M [..., d/32] in fp16."""
    x = x.unflatten(-1, (-1, 32)).clamp(-HELD_MAX, HELD_MAX)
    low, high = x.amin(-1), x.amax(-1)
    S = ((high - low) * (16.0 / 15.0)).half()
    M = (low - S.float()).half()
    step = torch.where(S > 0, 16.0 / S.float(), torch.zeros_like(low))
    code = ((x - (M.float() + S.float())[..., None]) * step[..., None]).round().clamp(0, 15)
    return code.int(), S, M


def _held(code, S, M):
    return (M.float()[..., None] + S.float()[..., None] * (1 + code.float() / 16)).flatten(-2)


def _bytes(x):
    return x.reshape(-1).view(torch.uint8)


def _pack(k, v, page):
    """k, v: what _quantise gives for [n, Hkv, page, d] -> [n, Hkv * page * d * 5 / 4] bytes."""
    (kc, kS, kM), (vc, vS, vM) = k, v
    n, H, _, G, _ = kc.shape
    B = page // 16
    even = 16 ** torch.arange(4, device=kc.device)
    place = torch.stack([even, even << 16], -1)                                     # [j, channel parity]
    words = (kc.view(n, H, B, 16, G, 4, 4, 2).long() * place).sum((-1, -2))         # [.., 16, G, t]
    kw = _bytes(words.transpose(-1, -2).to(torch.int32)).reshape(n, H, B, -1)
    ks = _bytes(torch.stack([kS, kM], -1).view(n, H, B, 16 * G * 2)).reshape(n, H, B, -1)
    pairs = (vc.view(n, H, B, 8, 2, G, 8, 4).long() * even).sum(-1)                 # [.., 8, 2, G, g]
    pairs = pairs[..., 0, :, :] + (pairs[..., 1, :, :] << 16)
    vw = _bytes(pairs.transpose(-1, -2).to(torch.int32)).reshape(n, H, B, -1)
    vs = torch.stack([vS.view(n, H, B, 8, 2, G), vM.view(n, H, B, 8, 2, G)], -3)    # [.., 8, S or M, 2, G]
    vs = _bytes(vs.permute(0, 1, 2, 3, 6, 4, 5)).reshape(n, H, B, -1)
    return torch.cat([kw, ks, vw, vs], -1).view(n, -1)


def _unpack(pages, kv_heads, d):
    """[..., page bytes] -> K and V [..., kv_heads, page, d] in 32 bits."""
    lead, G = pages.shape[:-1], d // 32
    b = pages.view(*lead, kv_heads, -1, 20 * d)
    shift = 4 * torch.arange(4, device=b.device, dtype=torch.int32)
    shift = torch.stack([shift, shift + 16], -1)                                    # [j, half]
    kw = b[..., :8 * d].contiguous().view(torch.int32).view(*b.shape[:-1], 16, 4, G, 1, 1)
    kc = ((kw >> shift) & 15).transpose(-4, -3).flatten(-3)                         # [.., 16, G, 32]
    ks = b[..., 8 * d:10 * d].contiguous().view(torch.float16).view(*b.shape[:-1], 16, G, 2)
    k = _held(kc, ks[..., 0], ks[..., 1])
    vw = b[..., 10 * d:18 * d].contiguous().view(torch.int32).view(*b.shape[:-1], 8, 8, G, 1, 1)
    vc = ((vw >> shift) & 15).permute(*range(vw.dim() - 5), -5, -1, -3, -4, -2).flatten(-2)
    vs = b[..., 18 * d:].contiguous().view(torch.float16).view(*b.shape[:-1], 8, G, 2, 2)
    vS, vM = vs[..., 0, :].transpose(-1, -2), vs[..., 1, :].transpose(-1, -2)       # [.., 8, half, G]
    v = _held(vc, vS, vM)
    return k.flatten(-3, -2), v.flatten(-4, -2)


def _places(at, in_page, Hkv, d, page):
    """Where, in numbers of 16 bits from the pool's beginning, the parts of tokens lie: page `at`, token `in_page` of it -> four index tensors [tokens, Hkv, n], K codes, K scales, V codes, V scales."""
    G, block, tok = d // 32, in_page // 16, in_page % 16
    head = torch.arange(Hkv, device=at.device)[None, :, None] * (page // 16 * 10 * d) + (at * (Hkv * page // 16 * 10 * d) + block * 10 * d)[:, None, None]
    tok = tok[:, None, None]
    i, w = torch.arange(4 * d // 16, device=at.device), torch.arange(2 * G, device=at.device)
    return head + tok * (d // 4) + i, head + 4 * d + tok * 2 * G + w, head + 5 * d + tok // 2 * (d // 2) + 2 * i + tok % 2, head + 9 * d + tok // 2 * 4 * G + 2 * w + tok % 2


# ---------------------------------------------------------------- plain forms
def _padded(x, starts, most):
    at = (starts[:-1, None].long() + torch.arange(most, device=x.device)).clamp(max=x.shape[0] - 1)
    return x[at]


def _packed(x, starts, rows):
    r = torch.arange(rows, device=x.device)
    b = torch.searchsorted(starts[1:].long(), r, right=True)
    return x[b, r - starts[b].long()]


def _turned(x, cos, sin, interleaved):
    """x [rows, heads, d] in 32 bits, cos, sin [rows, rot / 2]."""
    rot, cos, sin = 2 * cos.shape[1], cos[:, None], sin[:, None]
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :rot // 2], head[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def _plain_rotate(s):
    case, starts = s["case"], s["starts"].long()
    page, d, Hkv, dtype, rows = case["page"], case["d"], case["kv_heads"], s["k"].dtype, s["k"].shape[0]
    G = d // 32
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(starts[1:], r, right=True)
    seq = s["seqs"][b].long()
    base = s["lens"][seq].long() - (starts[b + 1] - starts[b])
    pos = base + r - starts[b]
    angle = (pos if s["depths"] is None else base + s["depths"])[:, None].double() * s["freqs"]      # (in 64 bits: far positions)
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turned(s["q"].float(), cos, sin, case["interleaved"]).to(dtype)
    k = _turned(s["k"].float(), cos, sin, case["interleaved"]).to(dtype)                               # (the cache is given what a turned tensor would hold)
    kq, vq = _quantise(k.float()), _quantise(s["v"].float())
    even = 16 ** torch.arange(4, device="cuda")
    halves = (kq[0].view(rows, Hkv, G, 4, 4, 2).long() * even[:, None]).sum(-2)                       # [rows, Hkv, G, t, half]
    k_codes = halves.transpose(2, 3).to(torch.int16)                                                  # [rows, Hkv, t, G, half]
    v_codes = (vq[0].view(rows, Hkv, G, 8, 4).long() * even).sum(-1).transpose(2, 3).to(torch.int16)  # [rows, Hkv, g, G]
    parts = (k_codes, torch.stack([kq[1], kq[2]], -1).view(torch.int16), v_codes, torch.stack([vq[1], vq[2]], -1).view(torch.int16))
    at = torch.cat([x.reshape(-1) for x in _places(s["tables"][seq, pos // page].long(), pos % page, Hkv, d, page)])
    s["pool"].view(torch.int16).view(-1)[at] = torch.cat([x.reshape(-1) for x in parts])
    return {"q": q, "k": _held(*kq).to(dtype), "v": _held(*vq).to(dtype)}


def _ancestors(parents, starts, most):
    """[sequences, most, most]: whether token j is token i or one of its ancestors."""
    p = _padded(parents, starts, most).long()
    a = torch.eye(most, device=p.device)[None] + (p[:, :, None] == torch.arange(most, device=p.device)).float()
    for _ in range(max(1, (most - 1).bit_length())):
        a = ((a @ a) > 0).float()
    return a > 0


def _plain_tree(s):
    case, seq, starts = s["case"], s["seqs"].long(), s["starts"]
    most, rows, H, Hkv, d = s["max_q"], s["q"].shape[0], case["heads"], case["kv_heads"], case["d"]
    k, v = _unpack(s["pool"][s["tables"][seq].long().clamp(min=0)], Hkv, d)      # [B, pages, Hkv, page, d]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))                     # [B, Hkv, K, d]
    q = _padded(s["q"], starts, most).float()
    B, Q, G, K = q.shape[0], most, H // Hkv, k.shape[2]
    w = (q.view(B, Q, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, d) @ k.transpose(-1, -2)).mul_(d ** -0.5).view(B, Hkv, G, Q, K)
    lens, n = s["lens"][seq].long(), starts.diff().long()
    j = torch.arange(K, device="cuda") - (lens - n)[:, None]                     # the place among the tree's tokens
    seen = _ancestors(s["parents"], starts, most).gather(2, j.clamp(0, most - 1)[:, None].expand(B, Q, K))
    seen = torch.where(j[:, None] < 0, torch.ones_like(seen), seen & (j < n[:, None])[:, None])
    w = w.masked_fill_(~seen[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, Q, H)
    out = ((w.view(B, Hkv, G * Q, K) @ v).view(B, Hkv, G, Q, d) / total).permute(0, 3, 1, 2, 4).reshape(B, Q, H, d)
    return {"out": _packed(out, starts, rows).to(s["q"].dtype).reshape(rows, -1), "lse": _packed(lse, starts, rows)}


def _plain_verify(s):
    """All sequences at once, level by level and sibling by sibling, in 64 bits: a number next to a border decides about a token."""
    starts, parents, tokens, u = s["starts"].long(), s["parents"].long(), s["tokens"].long(), s["uniform"].double()
    B, n, rows, most = starts.numel() - 1, starts.diff(), s["logits"].shape[0], s["most"]
    T = s["temperatures"].double()
    greedy = T == 0
    scale = torch.where(greedy, 1.0, 1 / torch.where(greedy, 1.0, T))[:, None]
    p_of = lambda at: torch.softmax(s["logits"][at].double() * scale, -1)  # noqa: E731
    q_of = lambda at: torch.softmax(s["drafts"][at].double() * scale, -1)  # noqa: E731
    place = torch.arange(most, device="cuda")
    mine = torch.where(place < n[:, None], _padded(parents, starts, most), -2)         # [B, most] parents of the sequence's tokens
    path = torch.full((B, most), -1, dtype=torch.int64, device="cuda")
    path[:, 0] = 0
    node, done, accepted = (torch.zeros(B, dtype=t, device="cuda") for t in (torch.int64, torch.bool, torch.int64))
    final = torch.zeros((B, s["logits"].shape[1]), dtype=torch.float64, device="cuda")
    for level in range(s["levels"]):
        p = p_of(starts[:-1] + node)
        likeliest = s["logits"][starts[:-1] + node].argmax(-1)
        w, q = p, q_of(starts[:-1] + node) if s["drafts"] is not None else None
        below = (mine == node[:, None]).int()
        child = torch.where(below.bool(), place, most).sort(-1).values                 # children first, in ascending order
        taken = torch.full((B,), -1, dtype=torch.int64, device="cuda")
        for k in range(min(s["branch"], most)):
            c = child[:, k]
            there = (c < most) & (taken < 0) & ~done
            at = starts[:-1] + c.clamp(max=most - 1)
            at = at.clamp(max=rows - 1)
            x = tokens[at][:, None]
            qx = torch.ones_like(u[at]) if q is None else q.gather(1, x)[:, 0]
            yes = torch.where(greedy, x[:, 0] == likeliest, u[at] * qx * w.sum(-1) < w.gather(1, x)[:, 0])
            taken = torch.where(there & yes, c, taken)
            no = (there & ~yes & ~greedy)[:, None]
            one = torch.zeros_like(w).scatter_(1, x, 1.0)
            less = (w / w.sum(-1, keepdim=True) - (one if q is None else q)).clamp(min=0)
            w = torch.where(no, less, w)
            if q is not None:                                                          # siblings are drawn without replacement
                q = torch.where(no & (one > 0), 0.0, q)
                q = torch.where(no, q / q.sum(-1, keepdim=True), q)
        ends = (taken < 0) & ~done
        final = torch.where((ends & ~greedy)[:, None], w, final)
        final = torch.where((ends & greedy)[:, None], torch.zeros_like(w).scatter_(1, likeliest[:, None], 1.0), final)
        done = done | ends
        accepted = accepted + (taken >= 0)
        path.scatter_(1, torch.where(taken >= 0, accepted, 0)[:, None], torch.where(taken >= 0, taken, 0)[:, None])
        node = torch.where(taken >= 0, taken, node)
    sums = final.cumsum(-1)
    next_token = (sums > u[starts[:-1]][:, None] * sums[:, -1:]).int().argmax(-1)
    return {"path": _packed(path, s["starts"], rows).int(), "accepted": accepted.int(), "next": next_token.int()}


def _plain_keep(s):
    case, starts, page = s["case"], s["starts"].long(), s["case"]["page"]
    rows, Hkv, d = s["path"].shape[0], case["kv_heads"], case["d"]
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(starts[1:], r, right=True)
    seq, i = s["seqs"][b].long(), r - starts[b]
    base = s["lens"][seq].long() - (starts[b + 1] - starts[b])
    i_from = torch.where(i <= s["accepted"][b], s["path"].long(), i)                   # (a token that does not stand is written where it is)
    src, dst = base + i_from, base + i
    pool = s["pool"].view(torch.int16).view(case["layers"], -1)
    where = lambda pos: torch.cat([x.reshape(rows, -1) for x in _places(s["tables"][seq, pos // page].long(), pos % page, Hkv, d, page)], 1).reshape(-1)  # noqa: E731
    pool[:, where(dst)] = pool[:, where(src)]
    s["new_lens"][s["seqs"].long()] = (s["lens"][s["seqs"].long()] - starts.diff() + 1 + s["accepted"]).int()
    return {"pool": s["pool"], "lens": s["new_lens"]}


def run(s):
    case = s["case"]
    if not own:
        return {"rotate": _plain_rotate, "tree": _plain_tree, "verify": _plain_verify, "keep": _plain_keep}[case["op"]](s)
    from paper_2012_01114_b200 import binding as psa
    if case["op"] == "rotate":
        psa.psa_cache_append_rotary(s["k"], s["v"], s["pool"], s["tables"], s["lens"], s["seqs"], s["starts"], case["page"], s["freqs"], Q=s["q"], depths=s["depths"],
                                    interleaved=case["interleaved"], q_out=s["q_out"], k_held=s["k_held"], v_held=s["v_held"])
        return {"q": s["q_out"], "k": s["k_held"], "v": s["v_held"]}
    if case["op"] == "tree":
        lse = torch.empty((s["q"].shape[0], case["heads"]), device="cuda")
        return {"out": psa.psa_tree_attention(s["q"], s["pool"], s["tables"], s["lens"], s["seqs"], s["starts"], s["parents"], case["kv_heads"], case["page"], s["max_q"], lse=lse), "lse": lse}
    if case["op"] == "verify":
        psa.psa_verify_drafts(s["logits"], s["tokens"], s["parents"], s["starts"], s["uniform"], s["path"], s["accepted"], s["next"], drafts=s["drafts"], temperatures=s["temperatures"])
        return {"path": s["path"], "accepted": s["accepted"], "next": s["next"]}
    psa.psa_cache_keep(s["pool"], s["tables"], s["lens"], s["seqs"], s["starts"], s["path"], s["accepted"], case["kv_heads"], case["page"], new_lens=s["new_lens"])
    return {"pool": s["pool"], "lens": s["new_lens"]}


# ---------------------------------------------------------------- the definitions in 64 bits
def _grid(x):
    """What a group of 32 numbers is held as, in 64 bits but for the two numbers that the cache holds in fp16."""
    x = x.double().clamp(-HELD_MAX, HELD_MAX).reshape(*x.shape[:-1], -1, 32)
    low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    S = ((high - low) * 16 / 15).half().double()
    M = (low - S).half().double()
    c = torch.round((x - M - S) / torch.where(S > 0, S / 16, torch.ones_like(S))).clamp(0, 15)
    return (M + S + torch.where(S > 0, S, 0 * S) / 16 * c).reshape(*x.shape[:-2], -1)


def _look(pool, page, block, tok, d):
    """K and V of single tokens, looked up by their definition: page, block (of the page), tok index tensors of one shape -> [.., d] each."""
    b = pool.view(pool.shape[0], -1, 20 * d)
    base = page * b.shape[1] + block
    flat = b.reshape(-1, 20 * d)
    c = torch.arange(d, device=pool.device)
    w, r, G = c // 32, c % 32, d // 32

    def nibble(byte0, bit):
        at = byte0 + bit // 8
        return (flat[base[..., None], at].long() >> (bit % 8)) & 15

    def half(byte0):
        return (flat[base[..., None], byte0].long() + 256 * flat[base[..., None], byte0 + 1].long()).to(torch.int16).view(torch.float16).double()

    t = tok[..., None]
    kc = nibble(t * (d // 2) + ((r // 8) * G + w) * 4, 4 * (r % 8 // 2) + 16 * (r % 2))
    ks = 8 * d + (t * G + w) * 4
    vc = nibble(10 * d + t // 2 * d + ((r // 4) * G + w) * 4, 4 * (r % 4) + 16 * (t % 2))
    vs = 18 * d + (t // 2 * G + w) * 8 + t % 2 * 2
    return half(ks + 2) + half(ks) * (1 + kc.double() / 16), half(vs + 4) + half(vs) * (1 + vc.double() / 16)


def exact(case, seed):
    if case["op"] in ("verify", "keep"):          # whole numbers only
        return None
    s = prepare(case, seed)
    starts = s["starts"].tolist()
    if case["op"] == "rotate":
        place, depths = [], None if s["depths"] is None else s["depths"].tolist()
        for b, n in enumerate(s["lens"].tolist()):
            m = starts[b + 1] - starts[b]
            place += [n - m + (i if depths is None else depths[starts[b] + i]) for i in range(m)]
        place = torch.tensor(place, dtype=torch.float64, device="cuda")
        rot = case["rot"]
        c = torch.arange(rot, device="cuda")
        pair = c // 2 if case["interleaved"] else c % (rot // 2)
        other = c ^ 1 if case["interleaved"] else (c + rot // 2) % rot
        first = (c % 2 == 0) if case["interleaved"] else c < rot // 2
        angle = place[:, None, None] * s["freqs"][pair]

        def turn(x):
            y = x.double()
            y[..., :rot] = y[..., :rot] * angle.cos() + torch.where(first, -1.0, 1.0) * y[..., :rot][..., other] * angle.sin()
            return y

        return {"q": turn(s["q"]), "k": _grid(turn(s["k"]).to(s["k"].dtype)), "v": _grid(s["v"])}
    rows, H, d = s["q"].shape
    out, lse = torch.zeros((rows, H, d), dtype=torch.float64, device="cuda"), torch.zeros((rows, H), dtype=torch.float64, device="cuda")
    parents, G, page = s["parents"].tolist(), H // case["kv_heads"], case["page"]
    for b, n in enumerate(s["lens"].tolist()):
        q0, m = starts[b], starts[b + 1] - starts[b]
        hidden = torch.ones((m, m), dtype=torch.bool)
        for i in range(m):
            at = i
            while at >= 0:
                hidden[i, at] = False
                at = parents[q0 + at]
        hidden = hidden.cuda()
        p = torch.arange(n, device="cuda")
        for h in range(case["kv_heads"]):
            k, v = _look(s["pool"], s["tables"][b].long()[p // page], h * (page // 16) + p % page // 16, p % 16, d)
            x = torch.einsum("mgd,nd->gmn", s["q"][q0:q0 + m, h * G:(h + 1) * G].double(), k) / math.sqrt(d)
            x[:, :, n - m:].masked_fill_(hidden, -math.inf)
            total = torch.logsumexp(x, -1)
            lse[q0:q0 + m, h * G:(h + 1) * G] = total.T
            out[q0:q0 + m, h * G:(h + 1) * G] = torch.einsum("gmn,nd->mgd", torch.exp(x - total[..., None]), v)
    return {"out": out.reshape(rows, -1), "lse": lse}
