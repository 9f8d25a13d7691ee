"""The serving operators as a user's program calls them: cases to be timed, their plain forms and their values in 64 bits.

Four operators that belong together: attention over packed prompts, appending to a paged cache held in 4 bits, attention
over that cache, and the pages' own bookkeeping.  `run` computes them in elementary torch operations (`own` false) or through
the public functions of `paper_2012_01114_b200.binding` (`own` true).

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
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
HELD_MAX = 20000.0          # numbers beyond this are held as this


# ---------------------------------------------------------------- cases
def _prompt(name, seqs, longest, prefix, heads, kv_heads, d, dtype, lengths):
    """`longest`: of the prompts; `prefix`: most keys ahead of a prompt's own (0: keys and queries are the same tokens)."""
    return dict(name=name, op="prompt", seqs=seqs, longest=longest, prefix=prefix, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, lengths=lengths)


def _append(name, seqs, longest, held, kv_heads, d, page, dtype, lengths):
    """`longest`: most tokens appended to a sequence; `held`: most tokens that one holds before."""
    return dict(name=name, op="append", seqs=seqs, longest=longest, held=held, kv_heads=kv_heads, d=d, page=page, dtype=dtype, lengths=lengths)


def _cache(name, seqs, longest, queries, heads, kv_heads, d, page, dtype, lengths):
    """`longest`: most tokens held; `queries`: most query tokens of a sequence, the last ones that it holds."""
    return dict(name=name, op="cache", seqs=seqs, longest=longest, queries=queries, heads=heads, kv_heads=kv_heads, d=d, page=page, dtype=dtype, lengths=lengths)


def _pages(name, kind, seqs, longest, tokens, kv_heads, d, page, layers, lengths):
    """kind "branch": drop the old branches, fork new ones, reserve up to `tokens` tokens for each; kind "compact": live pages to the front."""
    return dict(name=name, op="pages", kind=kind, seqs=seqs, longest=longest, tokens=tokens, kv_heads=kv_heads, d=d, page=page, layers=layers, lengths=lengths)


def listed():
    return [
        # one short question to a small model: latency and nothing else
        _prompt("prompt one short", 1, 37, 0, 4, 1, 64, "bf16", 1),
        # a batch of requests of very different lengths, one after another without padding
        _prompt("prompt packed", 24, 700, 0, 12, 4, 64, "bf16", 2),
        # pieces of prompts whose beginnings are known already (shared prefixes, prompts worked off in pieces)
        _prompt("prompt pieces", 6, 512, 4000, 32, 8, 128, "f16", 3),
        # two long documents: what a prompt pass costs when the product of the lengths rules
        _prompt("prompt long", 2, 8192, 0, 32, 8, 128, "bf16", 4),
        # one token each for a batch that is being answered
        _append("append step", 64, 1, 4000, 8, 128, 64, "bf16", 5),
        # the keys and values of a packed batch of prompts
        _append("append prompts", 16, 2500, 0, 8, 128, 64, "bf16", 6),
        # one answer being written by a small model: latency
        _cache("cache one", 1, 301, 1, 8, 2, 64, 16, "bf16", 7),
        # a step of a full batch of answers of different lengths
        _cache("cache batch", 64, 8000, 1, 32, 8, 128, 64, "bf16", 8),
        # two very long contexts, few rows: the long axis has to be split
        _cache("cache long", 2, 131072, 1, 32, 8, 128, 128, "bf16", 9),
        # a few guessed tokens for each sequence checked in one go
        _cache("cache drafts", 16, 4001, 5, 16, 2, 128, 32, "f16", 10),
        # branches of a batch dropped and drawn anew (beams, guesses, several answers to one question)
        _pages("pages branch", "branch", 64, 1500, 5, 8, 128, 64, 4, 11),
        # a pool with holes after many answers have ended
        _pages("pages compact", "compact", 400, 2000, 0, 8, 128, 64, 1, 12),
    ]


def _log(rng, low, high):
    v = max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["prompt", "append", "cache", "pages"])
    kv_heads, group, d = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 6, 7, 8]), rng.choice([64, 96, 128])
    dtype, lengths, page = rng.choice(["bf16", "bf16", "f16"]), rng.randrange(1 << 20), rng.choice([16, 32, 64, 128])
    if op == "prompt":
        longest = _log(rng, 1, 6000)
        prefix = rng.choice([0, _log(rng, 1, 6000)])
        while kv_heads * group * longest * (longest + prefix) > 1 << 30:
            longest, prefix = longest // 2, prefix // 2
        seqs = _log(rng, 1, min(64, (1 << 30) // (kv_heads * group * longest * (longest + prefix))))
        return {k: v for k, v in _prompt("", seqs, longest, prefix, kv_heads * group, kv_heads, d, dtype, lengths).items() if k != "name"}
    if op == "append":
        longest = rng.choice([1, _log(rng, 1, 2500)])
        seqs = _log(rng, 1, min(128, 40000 // longest))
        return {k: v for k, v in _append("", seqs, longest, _log(rng, 1, 4000), kv_heads, d, page, dtype, lengths).items() if k != "name"}
    if op == "cache":
        longest = _log(rng, 1, 131072)
        seqs = _log(rng, 1, min(128, 262144 // longest))
        return {k: v for k, v in _cache("", seqs, longest, min(longest, rng.choice([1, 1, 1, 2, 5, 9])), kv_heads * group, kv_heads, d, page, dtype, lengths).items() if k != "name"}
    kind, longest = rng.choice(["branch", "compact"]), _log(rng, 20, 2000)
    return {k: v for k, v in _pages("", kind, _log(rng, 2, 256), longest, _log(rng, 1, 100) if kind == "branch" else 0, kv_heads, d, page, rng.choice([1, 2, 4]), lengths).items() if k != "name"}


def _lengths(case, salt, low, high):
    """As many numbers as the case has sequences, spread over the logarithm, the first one the largest."""
    r = random.Random(case["lengths"] * 16 + salt)
    return [high] + [_log(r, max(low, 1), max(high, 1)) if high else 0 for _ in range(case["seqs"] - 1)]


def _queries(case):
    """Query tokens of each sequence and the tokens that it holds (those among them)."""
    held = _lengths(case, 1, 1, case["longest"])
    q = [case["queries"]] + [random.Random(case["lengths"] * 16 + 2 + i).randint(1, case["queries"]) for i in range(1, case["seqs"])]
    return [min(a, b) for a, b in zip(q, held)], held


def _prompt_lengths(case):
    q = _lengths(case, 1, 1, case["longest"])
    return q, [a + b for a, b in zip(q, _lengths(case, 2, 1, case["prefix"]))]


def work(case):
    if case["op"] == "prompt":
        q, k = _prompt_lengths(case)
        weights = sum(a * b - a * (a - 1) // 2 for a, b in zip(q, k))
        numbers = 2 * sum(q) * case["heads"] * case["d"] + 2 * sum(k) * case["kv_heads"] * case["d"]
        return {"bytes": 2 * numbers + 4 * sum(q) * case["heads"], "flops": 4 * weights * case["heads"] * case["d"]}
    if case["op"] == "append":
        n = sum(_lengths(case, 1, 1, case["longest"])) * case["kv_heads"] * case["d"] * 2
        return {"bytes": 2 * n + 2 * n + 5 * n // 8, "flops": 6 * n}
    if case["op"] == "cache":
        q, held = _queries(case)
        numbers = sum(held) * case["kv_heads"] * case["d"] * 2
        weights = sum(a * b - a * (a - 1) // 2 for a, b in zip(q, held)) * case["heads"]
        return {"bytes": 5 * numbers // 8 + 4 * sum(q) * case["heads"] * (case["d"] + 1) + 4 * sum(-(-h // case["page"]) for h in held),
                "flops": 4 * weights * case["d"]}
    page_bytes = case["kv_heads"] * case["page"] * case["d"] * 5 // 4 * case["layers"]
    if case["kind"] == "branch":     # the page that a branch writes to is copied; tables and counts
        held, pages, _ = _branch(case)
        return {"bytes": 2 * page_bytes * sum(1 for h in held if h % case["page"]) + 4 * (2 * pages + 4 * sum(-(-h // case["page"]) for h in held)), "flops": 0}
    held, pages, width = _fragments(case)
    live = sum(-(-h // case["page"]) for h in held)
    return {"bytes": 2 * page_bytes * live + 8 * (pages + live), "flops": 0}


# ---------------------------------------------------------------- inputs
def _normal(gen, shape, dtype):
    return torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _tables(held, page, pages, gen):
    """Pages for sequences of these lengths, in the order of chance; entries behind a sequence's last page are -1."""
    need = torch.tensor([-(-h // page) for h in held], device="cuda")
    width = max(1, int(need.max()))
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int64).int()
    col = torch.arange(width, device="cuda")
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    return torch.where(col < need[:, None], order[at.clamp(max=pages - 1)], -1).int().contiguous()


def _branch(case):
    """Tokens of the parents, pages of the pool, width of the tables."""
    held = _lengths(case, 1, 1, case["longest"])
    used = sum(-(-h // case["page"]) for h in held)
    extra = case["seqs"] * (2 + -(-case["tokens"] // case["page"]))
    return held, 2 * used + extra, -(-(case["longest"] + case["tokens"]) // case["page"]) + 1


def _fragments(case):
    held = _lengths(case, 1, 1, case["longest"])
    width = max(-(-h // case["page"]) for h in held)
    return held, sum(-(-h // case["page"]) for h in held) * 5 // 3 + 1, width


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "prompt":
        q, k = _prompt_lengths(case)
        dtype, H, Hkv, d = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["d"]
        s["q_starts"], s["max_q"], s["max_k"] = _starts(q), max(q), max(k)
        if case["prefix"]:
            s["q"], s["k"], s["v"] = (_normal(gen, (sum(n), h, d), dtype) for n, h in ((q, H), (k, Hkv), (k, Hkv)))
            s["k_starts"] = _starts(k)
        else:       # one matrix product gives all three: they lie side by side
            rows = _normal(gen, (sum(q), H + 2 * Hkv, d), dtype)
            s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:]
            s["k_starts"] = s["q_starts"]
    elif case["op"] == "append":
        new, old = _lengths(case, 1, 1, case["longest"]), _lengths(case, 2, 0, case["held"])
        rows, Hkv, d, page = sum(new), case["kv_heads"], case["d"], case["page"]
        qkv = _normal(gen, (rows, 6 * Hkv, d), DTYPES[case["dtype"]])
        offset = torch.empty((1, Hkv, d), device="cuda").normal_(generator=gen)     # keys have channels that are large in every token
        s["k"], s["v"] = (qkv[:, 4 * Hkv:5 * Hkv] + 2 * offset).to(qkv.dtype), qkv[:, 5 * Hkv:]
        held = [a + b for a, b in zip(new, old)]
        pages = sum(-(-h // page) for h in held) + 3
        s["tables"], s["lens"] = _tables(held, page, pages, gen), torch.tensor(held, dtype=torch.int32, device="cuda")
        s["seqs"], s["starts"] = torch.arange(case["seqs"], dtype=torch.int32, device="cuda"), _starts(new)
        s["pool"] = torch.zeros((pages, Hkv * page * d * 5 // 4), dtype=torch.uint8, device="cuda")
        s["k_held"], s["v_held"] = (torch.empty((rows, Hkv, d), dtype=qkv.dtype, device="cuda") for _ in range(2))
    elif case["op"] == "cache":
        q, held = _queries(case)
        H, Hkv, d, page = case["heads"], case["kv_heads"], case["d"], case["page"]
        pages = sum(-(-h // page) for h in held) + 3
        s["q"] = _normal(gen, (sum(q), H, d), DTYPES[case["dtype"]])
        s["q_starts"], s["max_q"] = _starts(q), max(q)
        s["tables"], s["lens"] = _tables(held, page, pages, gen), torch.tensor(held, dtype=torch.int32, device="cuda")
        s["seqs"] = torch.arange(case["seqs"], dtype=torch.int32, device="cuda")
        s["pool"] = torch.empty((pages, Hkv * page * d * 5 // 4), dtype=torch.uint8, device="cuda")
        offset = torch.empty((Hkv, 1, d), device="cuda").normal_(generator=gen)
        step = max(1, (1 << 25) // (Hkv * page * d))
        for at in range(0, pages, step):       # (in parts: the pool is large)
            n = min(step, pages - at)
            k, v = (torch.empty((n, Hkv, page, d), device="cuda").normal_(generator=gen) for _ in range(2))
            s["pool"][at:at + n] = _pack(*(_quantise(x) for x in (k + offset, v)), page)
    elif case["kind"] == "branch":
        held, pages, width = _branch(case)
        n = case["seqs"]
        used = _tables(held, case["page"], pages, gen)
        tables = torch.full((2 * n, width), -1, dtype=torch.int32, device="cuda")
        tables[:n, :used.shape[1]] = used
        s["lens"] = torch.tensor(held + [0] * n, dtype=torch.int32, device="cuda")
        s["refs"] = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, torch.where(tables >= 0, tables, pages).reshape(-1), torch.ones(2 * n * width, dtype=torch.int32, device="cuda"))[:pages].contiguous()
        s["tables"] = tables
        s["parents"] = torch.arange(n, dtype=torch.int32, device="cuda")
        s["children"] = torch.randperm(n, generator=gen, device="cuda").int() + n
        s["add"] = torch.tensor(_lengths(case, 3, 1, case["tokens"]), dtype=torch.int32, device="cuda")
        s["short"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        s["pool"] = torch.randint(0, 256, (case["layers"], pages, case["kv_heads"] * case["page"] * case["d"] * 5 // 4), dtype=torch.uint8, device="cuda", generator=gen)
    else:
        held, pages, width = _fragments(case)
        s["tables"] = _tables(held, case["page"], pages, gen)
        s["lens"] = torch.tensor(held, dtype=torch.int32, device="cuda")
        s["refs"] = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, torch.where(s["tables"] >= 0, s["tables"], pages).reshape(-1), torch.ones(s["tables"].numel(), dtype=torch.int32, device="cuda"))[:pages].contiguous()
        s["pool"] = torch.randint(0, 256, (case["layers"], pages, case["kv_heads"] * case["page"] * case["d"] * 5 // 4), dtype=torch.uint8, device="cuda", generator=gen)
        s["new_tables"], s["new_refs"], s["new_pool"] = torch.empty_like(s["tables"]), torch.empty_like(s["refs"]), torch.zeros_like(s["pool"])
        s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms
def _attend(q, k, v, lq, lk):
    """q [B, Q, H, d], k, v [B, K, Hkv, d] in 32 bits, padded; lq, lk: lengths.  Query i sees the keys up to i + lk - lq."""
    B, Q, H, d = q.shape
    Hkv, G = k.shape[2], H // k.shape[2]
    w = q.view(B, Q, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, d) @ k.permute(0, 2, 3, 1)
    w = w.mul_(d ** -0.5).view(B, Hkv, G, Q, -1)
    i, j = torch.arange(Q, device=q.device)[:, None], torch.arange(k.shape[1], device=q.device)
    seen = (j <= i + (lk - lq)[:, None, None]) & (j < lk[:, None, None])
    w = w.masked_fill_(~seen[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)[..., 0]
    out = (w.view(B, Hkv, G * Q, -1) @ v.permute(0, 2, 1, 3)).view(B, Hkv, G, Q, d) / torch.where(total > 0, total, torch.ones_like(total))
    return out.permute(0, 3, 1, 2, 4).reshape(B, Q, H, d), lse.permute(0, 3, 1, 2).reshape(B, Q, H)


def _padded(x, starts, most):
    at = (starts[:-1, None].long() + torch.arange(most, device=x.device)).clamp(max=x.shape[0] - 1)
    return x[at].float()


def _packed(x, starts, rows):
    r = torch.arange(rows, device=x.device)
    b = torch.searchsorted(starts[1:].long(), r, right=True)
    return x[b, r - starts[b].long()]


def _plain_prompt(s):
    q, k, v = _padded(s["q"], s["q_starts"], s["max_q"]), _padded(s["k"], s["k_starts"], s["max_k"]), _padded(s["v"], s["k_starts"], s["max_k"])
    out, lse = _attend(q, k, v, s["q_starts"].diff(), s["k_starts"].diff())
    rows = s["q"].shape[0]
    return {"out": _packed(out, s["q_starts"], rows).to(s["q"].dtype).reshape(rows, -1), "lse": _packed(lse, s["q_starts"], rows)}


def _quantise(x):
    """[..., d] in 32 bits -> codes [..., d/32, 32], S and M [..., d/32] in fp16."""
    x = x.unflatten(-1, (-1, 32))
    x = x.clamp(-HELD_MAX, HELD_MAX)
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


def _plain_append(s):
    case, starts = s["case"], s["starts"].long()
    page, G, Hkv = case["page"], case["d"] // 32, case["kv_heads"]
    rows = s["k"].shape[0]
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(starts[1:], r, right=True)
    seq = s["seqs"][b].long()
    pos = s["lens"][seq].long() - (starts[b + 1] - r)
    at = s["tables"][seq, pos // page].long()
    kq, vq = _quantise(s["k"].float()), _quantise(s["v"].float())
    # every token written into an empty page image of its own: the bytes that it owns there are the ones to be stored
    d, block, tok = case["d"], pos % page // 16, pos % 16
    even = 16 ** torch.arange(4, device="cuda")
    halves = (kq[0].view(rows, Hkv, G, 4, 4, 2).long() * even[:, None]).sum(-2)                       # [rows, Hkv, G, t, half]
    k_codes = halves.transpose(2, 3).to(torch.int16)                                                  # [rows, Hkv, t, G, half]
    v_codes = (vq[0].view(rows, Hkv, G, 8, 4).long() * even).sum(-1).transpose(2, 3).to(torch.int16)  # [rows, Hkv, g, G]
    pool = s["pool"].view(torch.int16)
    head = torch.arange(Hkv, device="cuda")[None, :, None] * (page // 16 * 10 * d) + (at * pool.shape[1] + block * 10 * d)[:, None, None]
    tok = tok[:, None, None]

    def store(place, x):
        pool.view(-1)[(head + place).reshape(-1)] = x.reshape(-1)

    i = torch.arange(4 * d // 16, device="cuda")
    store(tok * (d // 4) + i, k_codes.reshape(rows, Hkv, -1))
    store(4 * d + tok * 2 * G + torch.arange(2 * G, device="cuda"), torch.stack([kq[1], kq[2]], -1).reshape(rows, Hkv, -1).view(torch.int16))
    store(5 * d + tok // 2 * (d // 2) + 2 * i + tok % 2, v_codes.reshape(rows, Hkv, -1))
    w = torch.arange(2 * G, device="cuda")
    store(9 * d + tok // 2 * 4 * G + 2 * w + tok % 2, torch.stack([vq[1], vq[2]], -1).reshape(rows, Hkv, -1).view(torch.int16))
    return {"k": _held(*kq).to(s["k"].dtype), "v": _held(*vq).to(s["v"].dtype), "pool": s["pool"]}


def _plain_cache(s):
    case = s["case"]
    seq = s["seqs"].long()
    k, v = _unpack(s["pool"][s["tables"][seq].long().clamp(min=0)], case["kv_heads"], case["d"])      # [B, pages, Hkv, page, d]
    k, v = (x.transpose(1, 2).flatten(2, 3).transpose(1, 2) for x in (k, v))
    out, lse = _attend(_padded(s["q"], s["q_starts"], s["max_q"]), k, v, s["q_starts"].diff(), s["lens"][seq])
    rows = s["q"].shape[0]
    return {"out": _packed(out, s["q_starts"], rows).to(s["q"].dtype).reshape(rows, -1), "lse": _packed(lse, s["q_starts"], rows)}


def _plain_branch(s):
    tables, lens, refs, pool, page = s["tables"], s["lens"], s["refs"], s["pool"], s["case"]["page"]
    parents, children, pages, width = s["parents"].long(), s["children"].long(), refs.numel(), tables.shape[1]
    col = torch.arange(width, device="cuda")

    def count(rows, by):       # (-1 at places that hold no page: counted behind the last page and dropped)
        used = tables[rows]
        more = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
        more.index_add_(0, torch.where(used >= 0, used, pages).reshape(-1).long(), torch.full((used.numel(),), by, dtype=torch.int32, device="cuda"))
        refs.add_(more[:pages])

    count(children, -1)                        # the old branches end
    tables[children], lens[children] = -1, 0
    tables[children], lens[children] = tables[parents], lens[parents]     # the new ones share all pages
    count(children, 1)
    # room for `add` more tokens each: a shared page that is to be written to is copied
    held, have = lens[children], -(-lens[children].long() // page)
    want = -(-(held + s["add"]).long() // page)
    last = tables[children, (have - 1).clamp(min=0)].long()
    part = (held % page != 0) & (s["add"] > 0)
    before = ((last[None, :] == last[:, None]) & part[None, :] & part[:, None]).tril(-1).sum(1)
    copy = part & (refs[last.clamp(min=0)] - before > 1)
    need = want - have + copy
    free = torch.argsort((refs != 0).int(), stable=True)
    enough = need.sum() <= (refs == 0).sum()
    s["short"].copy_(torch.where(enough, 0, need.sum() - (refs == 0).sum()))
    first = torch.cumsum(need, 0) - need
    new_last = torch.where(copy & enough, free[first.clamp(max=pages - 1)], last)
    pool[:, new_last] = pool[:, last]
    grown = (col >= have[:, None]) & (col < want[:, None])
    given = free[((first + copy)[:, None] + col - have[:, None]).clamp(0, pages - 1)]
    mine = torch.where(grown & enough, given.int(), tables[children])
    mine = torch.where((col == (have - 1)[:, None]) & copy[:, None], new_last.int()[:, None], mine)
    tables[children] = mine
    gone = torch.zeros(pages, dtype=torch.int32, device="cuda").index_add_(0, last, -(copy & enough).int())
    taken = torch.zeros(pages, dtype=torch.int32, device="cuda").index_add_(0, free, (torch.arange(pages, device="cuda") < torch.where(enough, need.sum(), 0)).int())
    refs.add_(gone + taken)
    lens[children] = torch.where(enough, held + s["add"], held)
    return {"tables": tables, "lens": lens, "refs": refs, "short": s["short"], "pool": pool}


def _plain_compact(s):
    refs, pages = s["refs"], s["refs"].numel()
    live, at = refs > 0, torch.arange(pages, device="cuda")
    n = live.sum()
    moves, holes = live & (at >= n), ~live & (at < n)
    hole = torch.argsort((~holes).int(), stable=True)
    to = torch.where(moves, hole[(torch.cumsum(moves, 0) - 1).clamp(min=0)], at)
    s["new_tables"].copy_(torch.where(s["tables"] >= 0, to[s["tables"].long().clamp(min=0)].int(), s["tables"]))
    source = at.clone().scatter_(0, torch.where(live, to, pages - 1 + 0 * at), torch.where(live, at, at[-1]))
    source = torch.where(at < n, source, at)
    s["new_refs"].copy_(torch.where(at < n, refs[source], torch.zeros_like(refs)))
    s["new_pool"].copy_(torch.where((at < n)[:, None], s["pool"][:, source], s["new_pool"]))
    s["live"].copy_(n)
    return {"tables": s["new_tables"], "refs": s["new_refs"], "pool": s["new_pool"], "live": s["live"]}


def run(s):
    case = s["case"]
    if not own:
        plain = {"prompt": _plain_prompt, "append": _plain_append, "cache": _plain_cache}
        return plain[case["op"]](s) if case["op"] in plain else _plain_branch(s) if case["kind"] == "branch" else _plain_compact(s)
    from paper_2012_01114_b200 import binding as psa
    if case["op"] == "prompt":
        lse = torch.empty((s["q"].shape[0], case["heads"]), device="cuda")
        return {"out": psa.psa_prompt_attention(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], lse=lse), "lse": lse}
    if case["op"] == "append":
        psa.psa_cache_append(s["k"], s["v"], s["pool"], s["tables"], s["lens"], s["seqs"], s["starts"], case["page"], k_held=s["k_held"], v_held=s["v_held"])
        return {"k": s["k_held"], "v": s["v_held"], "pool": s["pool"]}
    if case["op"] == "cache":
        lse = torch.empty((s["q"].shape[0], case["heads"]), device="cuda")
        return {"out": psa.psa_cache_attention(s["q"], s["pool"], s["tables"], s["lens"], s["seqs"], s["q_starts"], case["kv_heads"], case["page"], s["max_q"], lse=lse), "lse": lse}
    if case["kind"] == "branch":
        psa.psa_pages_free(s["tables"], s["lens"], s["refs"], s["children"], case["page"])
        psa.psa_pages_fork(s["tables"], s["lens"], s["refs"], s["parents"], s["children"], case["page"])
        psa.psa_pages_reserve(s["tables"], s["lens"], s["refs"], s["pool"], s["children"], s["add"], case["page"], s["short"])
        return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"], "short": s["short"], "pool": s["pool"]}
    psa.psa_pages_compact(s["tables"], s["refs"], s["pool"], s["new_tables"], s["new_refs"], s["new_pool"], s["live"])
    return {"tables": s["new_tables"], "refs": s["new_refs"], "pool": s["new_pool"], "live": s["live"]}


# ---------------------------------------------------------------- the definitions in 64 bits
def _rows(q, k, v, out, lse):
    """One sequence, head by head: q [Q, H, d], k, v [K, Hkv, d]."""
    (Q, H, d), K, G = q.shape, k.shape[0], q.shape[1] // k.shape[1]
    for h in range(H):
        for at in range(0, Q, 4096):
            x = (q[at:at + 4096, h].double() @ k[:, h // G].double().T) / math.sqrt(d)
            last = torch.arange(at, at + x.shape[0], device=x.device) + K - Q
            x[torch.arange(K, device=x.device)[None] > last[:, None]] = -math.inf
            total = torch.logsumexp(x, -1)
            lse[at:at + 4096, h] = total
            out[at:at + 4096, h] = torch.exp(x - torch.where(total > -math.inf, total, 0.0)[:, None]) @ v[:, h // G].double()


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
    if case["op"] == "pages":          # whole numbers only
        return None
    s = prepare(case, seed)
    if case["op"] == "append":
        return {"k": _grid(s["k"]), "v": _grid(s["v"]), "pool": None}
    rows, H, d = s["q"].shape
    out, lse = torch.zeros((rows, H, d), dtype=torch.float64, device="cuda"), torch.full((rows, H), -math.inf, dtype=torch.float64, device="cuda")
    starts = s["q_starts"].tolist()
    for b in range(case["seqs"]):
        q0, q1 = starts[b], starts[b + 1]
        if case["op"] == "prompt":
            k0, k1 = s["k_starts"][b:b + 2].tolist()
            k, v = s["k"][k0:k1], s["v"][k0:k1]
            _rows(s["q"][q0:q1], k, v, out[q0:q1], lse[q0:q1])
        else:
            n, page, blocks = int(s["lens"][b]), case["page"], case["page"] // 16
            for h in range(case["kv_heads"]):
                p = torch.arange(n, device="cuda")
                at = s["tables"][b].long()[p // page]
                k, v = _look(s["pool"], at, h * blocks + p % page // 16, p % 16, d)
                g = slice(h * (H // case["kv_heads"]), (h + 1) * (H // case["kv_heads"]))
                _rows(s["q"][q0:q1, g], k[:, None], v[:, None], out[q0:q1, g], lse[q0:q1, g])
    return {"out": out.reshape(rows, -1), "lse": lse}
