"""Plain definitions of the paged 8-bit cache for its tests: page tables step by step on the host, the store's codes by
the formula, attention in 64 bits.  All on the CPU, shared with nothing of the library."""
import math

import numpy as np
import torch

QMAX = {"int8": 127.0, "e4m3": 448.0}
ELEM = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # torch.finfo(t).eps / 2, relative


def key_at(t, ch, D):
    return t // 16 * (16 * D) + ch // 64 * 1024 + ch % 64 // 16 * 256 + t % 16 * 16 + ch % 16


def value_at(t, ch, D):
    return t // 16 * (16 * D) + ch // 64 * 1024 + t % 16 // 4 * 256 + ch % 16 * 16 + ch % 64 // 16 * 4 + t % 4


def order(P, D):
    """[2, P, D]: place of (side, token, channel) in a block's numbers."""
    t, ch = np.arange(P)[:, None], np.arange(D)[None]
    return torch.from_numpy(np.stack([key_at(t, ch, D), value_at(t, ch, D)]).astype(np.int64))


class Tables:
    """The page tables by the rules, one sequence after the other."""

    def __init__(self, n_seqs, page, n_pages, max_pages, free):
        self.P, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.lens = [0] * n_seqs
        self.tables = [[-1] * max_pages for _ in range(n_seqs)]
        self.free = list(free)          # the whole array
        self.count = len(self.free)

    def step(self, add, max_new):
        P = self.P
        for b, a in enumerate(add):
            if a < 0:
                for j in range(-(-self.lens[b] // P)):
                    self.free[self.count] = self.tables[b][j]
                    self.count += 1
                self.lens[b] = 0
        avail, top, needed, row = self.count, self.count, 0, 0
        start, cu, tok = [], [0], []
        for b, a in enumerate(add):
            T, n = max(a, 0), self.lens[b]
            ok = n + T <= P * self.max_pages and row + T <= max_new
            if ok:
                need = -(-(n + T) // P) - -(-n // P)
                needed += need
                ok = need == 0 or needed <= avail
            if ok:
                for j in range(need):
                    self.count -= 1
                    self.tables[b][-(-n // P) + j] = self.free[self.count]
                self.lens[b] = n + T
            start.append(n if ok else -1)
            for i in range(T):
                if row + i < max_new:
                    tok.append((b, n + i, self.tables[b][(n + i) // P] * P + (n + i) % P) if ok else (b, -1, -1))
            row += T
            cu.append(min(row, max_new))
        return start, cu, tok


def code_block(x, code):
    """x: [H, P, D] of one side -> (codes as the 8 bits, scale [H])."""
    x = x.float()
    amax = x.abs().amax((1, 2))
    scale = torch.maximum(amax / torch.tensor(QMAX[code]), torch.tensor(2.0 ** -64))
    y = (x * (1.0 / scale)[:, None, None]).clamp(-QMAX[code], QMAX[code])
    c = y.round().to(torch.int8) if code == "int8" else y.to(torch.float8_e4m3fn)
    return c.view(torch.uint8), scale


class Cache:
    """One layer's kv, scale and open arrays, kept by the rules."""

    def __init__(self, n_seqs, hkv, page, n_pages, D, elem, code, kv, scale, open_):
        self.P, self.D, self.hkv, self.code, self.n_pages = page, D, hkv, code, n_pages
        self.kv, self.scale, self.open = kv.clone(), scale.clone(), open_.clone()
        self.rows = [torch.zeros(0, 2, hkv, D, dtype=ELEM[elem]) for _ in range(n_seqs)]      # everything that was stored
        self.at = order(page, D)

    def store(self, start, cu, k, v, tables):
        P, H = self.P, self.hkv
        x = torch.stack((k, v), 1)
        for b, s in enumerate(start):
            if s < 0 or cu[b + 1] == cu[b]:
                continue
            self.rows[b] = torch.cat((self.rows[b][:s], x[cu[b]:cu[b + 1]]))
            end = s + cu[b + 1] - cu[b]
            for blk in range(s // P, end // P):
                page = tables[b][blk]
                if not 0 <= page < self.n_pages:
                    continue
                for side in range(2):
                    c, sc = code_block(self.rows[b][blk * P:(blk + 1) * P, side].transpose(0, 1), self.code)
                    self.kv[page, :, side, self.at[side].reshape(-1)] = c.reshape(H, -1)
                    self.scale[page, :, side] = sc
            for p in range(max(s, end // P * P), end):
                for side in range(2):
                    self.open[b, :, side, self.at[side][p % P]] = self.rows[b][p, side]

    def read(self, b, n, tables):
        """(keys, values, seen) of sequence b in 64 bits: [2, H, n, D] and which tokens are on a page that exists."""
        P, H, D = self.P, self.hkv, self.D
        out = torch.zeros(2, H, n, D, dtype=torch.float64)
        there = torch.ones(n, dtype=torch.bool)
        t8 = torch.int8 if self.code == "int8" else torch.float8_e4m3fn
        for blk in range(-(-n // P)):
            lo, hi = blk * P, min(n, blk * P + P)
            if hi == lo + P:
                page = tables[b][blk]
                if not 0 <= page < self.n_pages:
                    there[lo:hi] = False
                    continue
                for side in range(2):
                    c = self.kv[page, :, side][:, self.at[side].reshape(-1)].view(t8).double().reshape(H, P, D)
                    out[side, :, lo:hi] = c * self.scale[page, :, side].double()[:, None, None]
            else:
                for side in range(2):
                    out[side, :, lo:hi] = self.open[b, :, side][:, self.at[side][:hi - lo].reshape(-1)].double().reshape(H, hi - lo, D)
        return out[0], out[1], there


def attend(q, k, v, there, sm, causal, G):
    """q [m, hq, D], k, v [H, n, D] in 64 bits -> y, lse, sum p |v|, and the largest sum |q k| * sm of a row."""
    m, hq, D = q.shape
    n = k.shape[1]
    q = q.double()
    i = torch.arange(m)[:, None]
    hidden = ~there[None].expand(m, n) | ((torch.arange(n)[None] > n - m + i) if causal else torch.zeros(m, n, dtype=torch.bool))
    y = torch.zeros(m, hq, D, dtype=torch.float64)
    # mass: sum p |v|, and the share of it that tolerances() gives to weights far below the largest
    mass = torch.zeros_like(y)
    lse = torch.full((m, hq), -math.inf, dtype=torch.float64)
    big = torch.zeros(m, hq, dtype=torch.float64)
    if n == 0 or m == 0:
        return y, lse, mass, big
    for h in range(hq):
        z = (q[:, h] @ k[h // G].T * sm).masked_fill(hidden, -math.inf)
        top = z.amax(1, keepdim=True).clamp_min(-1e300)
        p = (z - top).exp()
        l = p.sum(1, keepdim=True)
        lse[:, h] = (top + l.log())[:, 0]
        p = p / torch.where(l > 0, l, 1.0)
        y[:, h] = p @ v[h // G]
        mass[:, h] = p @ v[h // G].abs()
        big[:, h] = (q[:, h].abs() @ k[h // G].abs().T * sm).amax(1)
    return y, lse, mass + ABSOLUTE * n * v.abs().amax((1, 2)).repeat_interleave(G)[None, :, None], big


# Weights are held in halves, p times the scale of the token's page relative to the largest such product, which stands
# at 2^12 or above; halves below 2^-14 are 2^-24 apart, so a weight is off by at most 2^-25 / 2^12 of the largest, whatever its own
# size.  A token adds that times its code, and the largest scale times the largest code is the largest |v| of the
# head (m steps of the scale; an open block is scaled to the same range): 2^-37 n max|v| in all, taken twice.  The
# bound on y multiplies its mass by rel >= 2^-11, so it is added there as 2^-36 / 2^-11.
ABSOLUTE = 2.0 ** -25


def tolerances(y, lse, mass, big, n, D, elem):
    """Bounds on the error of y and lse, by the arithmetic's roundings:
    a score is a sum of D exact products in 32 bits, then two multiplications and an addition: ds <= (D + 4) 2^-24 big;
    a weight carries exp(2 ds) of that, 2^-22 of the power's own error, and its rounding to 16 bits, 2^-11;
    sums of n weights in 32 bits: n 2^-24 (the worst order); small weights: see ABSOLUTE;
    the result is rounded to its type once."""
    ds = (D + 4) * 2.0 ** -24 * big
    rel = 2 * ds + 2.0 ** -11 + 2.0 ** -21 + n * 2.0 ** -23
    tiny = 2.0 ** -25 if elem == "f16" else 0.0                     # halves below 2^-14 are that far apart
    return HALF_STEP[elem] * (y.abs() + rel[..., None] * mass) + rel[..., None] * mass + tiny, \
        2 * ds + n * 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -22 * lse.abs().nan_to_num(0.0, 0.0, 0.0)
