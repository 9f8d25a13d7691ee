"""The serving operators' definitions in 64 bits, row by row, for the tests: attention over the keys that a row sees and no others, the 4-bit grid of the cache
with its layout byte by byte, and the pages' bookkeeping one sequence after another."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, k, v, scale):
    """q [nq, H, d], k, v [nk, Hkv, d] (any type, any device) -> out, size, lse in fp64 on the CPU.  size[i] = sum_j w_ij |v_j|, what the errors of an
    output are measured by.  Row i sees keys up to i + nk - nq."""
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    (nq, H, d), nk, G = q.shape, k.shape[0], q.shape[1] // max(k.shape[1], 1)
    out, size, lse = torch.zeros(nq, H, d, dtype=torch.float64), torch.zeros(nq, H, d, dtype=torch.float64), torch.full((nq, H), -math.inf, dtype=torch.float64)
    for i in range(nq):
        n = min(i + nk - nq + 1, nk)
        if n <= 0:
            continue
        for h in range(k.shape[1]):
            s = scale * (q[i, h * G:(h + 1) * G] @ k[:n, h].T)
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            total = w.sum(-1, keepdim=True)
            out[i, h * G:(h + 1) * G] = w @ v[:n, h] / total
            size[i, h * G:(h + 1) * G] = w @ v[:n, h].abs() / total
            lse[i, h * G:(h + 1) * G] = (top + total.log())[:, 0]
    return out, size, lse


def close(out, lse, ref, dtype, keys, roundings, v_max=4.0):
    """`roundings`: sum of the unit roundoffs that an output goes through (weights, held values, result).  1e-4: sums and exponentials in 32 bits.  keys 2^-25: weights
    in fp16 that fall below its normal numbers, against a largest weight of at least 1."""
    r, size, r_lse = ref
    got = out.detach().cpu().double().view(r.shape)
    tol = (roundings + 1e-4) * size + keys * 2.0 ** -25 * v_max + 2.0 ** -24
    assert torch.isfinite(got).all()
    assert ((got - r).abs() <= tol).all(), float(((got - r).abs() / tol).max())
    if lse is not None:
        l = lse.detach().cpu().double()
        seen = r_lse > -math.inf
        assert torch.equal(seen, l > -math.inf)
        assert ((l - r_lse).abs()[seen] <= 5e-5 * (1 + r_lse.abs()[seen])).all()


def starts(lengths, device="cuda"):
    return torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), dtype=torch.int32, device=device)


# ---------------------------------------------------------------- the cache in 4 bits
def quantise(x):
    """[..., d] fp32 -> codes [..., G, 32] int, S, M [..., G] fp16, every operation in fp32 by itself."""
    x = x.float().unflatten(-1, (-1, 32)).clamp(-20000, 20000)
    lo, hi = x.amin(-1), x.amax(-1)
    S = ((hi - lo) * torch.tensor(16.0 / 15.0, dtype=torch.float32)).half()
    M = (lo - S.float()).half()
    step = torch.where(S > 0, torch.tensor(16.0) / S.float(), torch.tensor(0.0))
    c = ((x - (M.float() + S.float())[..., None]) * step[..., None]).round().clamp(0, 15)
    return torch.nan_to_num(c).int(), S, M


def held(c, S, M):
    """What the codes stand for, in fp64."""
    return (M.double()[..., None] + S.double()[..., None] * (1 + c.double() / 16)).flatten(-2)


def put(page, head, page_size, d, tok, kq, vq):
    """Writes one token of one head into a page (uint8 [page bytes], on the CPU) by the layout's definition."""
    G, base, t = d // 32, (head * (page_size // 16) + tok // 16) * 20 * d, tok % 16
    half = lambda h: h.reshape(1).view(torch.uint8).tolist()  # noqa: E731

    def nibble(at, bit, c):
        at += bit // 8
        page[at] = (int(page[at]) & ~(15 << bit % 8)) | (int(c) << bit % 8)

    for w in range(G):
        for r in range(32):
            nibble(base + t * (d // 2) + ((r // 8) * G + w) * 4, 4 * (r % 8 // 2) + 16 * (r % 2), kq[0][w, r])
            nibble(base + 10 * d + t // 2 * d + ((r // 4) * G + w) * 4, 4 * (r % 4) + 16 * (t % 2), vq[0][w, r])
        for i, (k, v) in enumerate(zip(kq[1:], vq[1:])):
            at = base + 8 * d + (t * G + w) * 4 + 2 * i
            page[at], page[at + 1] = half(k[w])
            at = base + 18 * d + (t // 2 * G + w) * 8 + 4 * i + 2 * (t % 2)
            page[at], page[at + 1] = half(v[w])


def block_images(kq, vq, n):
    """Codes of `n` (a multiple of 16) tokens of one head -> [n / 16, 20 d] bytes, the same layout for whole blocks at once.  kq, vq: codes [n, G, 32], S, M [n, G]."""
    G = kq[0].shape[1]
    d, B = 32 * G, n // 16
    img = torch.zeros(B, 20 * d, dtype=torch.uint8)
    kc, vc = kq[0].view(B, 16, G, 32), vq[0].view(B, 16, G, 32)
    b, t, w, r = (x.reshape(-1) for x in torch.meshgrid(torch.arange(B), torch.arange(16), torch.arange(G), torch.arange(32), indexing="ij"))

    def nibbles(at, bit, c):
        at, shift = at + bit // 8, bit % 8
        acc = torch.zeros(B * 20 * d, dtype=torch.int32)
        acc.index_add_(0, b * 20 * d + at, (c.reshape(-1) << shift).int())
        return acc.view(B, -1).to(torch.uint8)

    img |= nibbles(t * (d // 2) + ((r // 8) * G + w) * 4, 4 * (r % 8 // 2) + 16 * (r % 2), kc)
    img |= nibbles(10 * d + t // 2 * d + ((r // 4) * G + w) * 4, 4 * (r % 4) + 16 * (t % 2), vc)
    ks = torch.stack([kq[1], kq[2]], -1).view(B, 16 * G * 2).view(torch.uint8)
    img[:, 8 * d:10 * d] = ks.reshape(B, -1)
    vs = torch.stack([vq[1].view(B, 8, 2, G), vq[2].view(B, 8, 2, G)], 2)            # [B, pair, S or M, token, G]
    img[:, 18 * d:] = vs.permute(0, 1, 4, 2, 3).contiguous().view(B, -1).view(torch.uint8)
    return img


# ---------------------------------------------------------------- pages
class Book:
    """Tables, lengths and counts as lists, changed one sequence at a time."""

    def __init__(self, slots, width, pages, page_size, pool):
        self.t, self.l, self.r = [[-1] * width for _ in range(slots)], [0] * slots, [0] * pages
        self.size, self.pool = page_size, pool

    def free(self, seqs):
        for s in seqs:
            for p in self.t[s]:
                if p >= 0:
                    self.r[p] -= 1
            self.t[s], self.l[s] = [-1] * len(self.t[s]), 0

    def fork(self, parents, children):
        for a, b in zip(parents, children):
            self.t[b], self.l[b] = list(self.t[a]), self.l[a]
            for p in self.t[b]:
                if p >= 0:
                    self.r[p] += 1

    def reserve(self, seqs, add):
        """Pages missing; 0: done."""
        t, l, r, copies = [list(x) for x in self.t], list(self.l), list(self.r), []
        free = [i for i, x in enumerate(r) if x == 0]
        need = 0
        for s, a in zip(seqs, add):
            have, want = -(-l[s] // self.size), -(-(l[s] + a) // self.size)
            cols = list(range(have, want))
            if l[s] % self.size and a > 0 and r[t[s][have - 1]] > 1:
                r[t[s][have - 1]] -= 1
                if need < len(free):
                    copies.append((t[s][have - 1], free[need]))
                cols = [have - 1] + cols
            for c in cols:
                if need < len(free):
                    t[s][c] = free[need]
                    r[free[need]] = 1
                need += 1
            l[s] += a
        if need > len(free):
            return need - len(free)
        self.t, self.l, self.r = t, l, r
        for a, b in copies:
            self.pool[:, b] = self.pool[:, a]
        return 0

    def compact(self):
        live = [i for i, x in enumerate(self.r) if x > 0]
        n = len(live)
        to = dict(zip([i for i in live if i >= n], [i for i in range(n) if self.r[i] <= 0]))
        for a, b in to.items():
            self.pool[:, b] = self.pool[:, a]
            self.r[b], self.r[a] = self.r[a], 0
        self.t = [[to.get(p, p) for p in row] for row in self.t]
        return n
