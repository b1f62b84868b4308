"""Plain forms of the paged step's operators for their tests: 4-bit rows and pools from their definition, heads normalised
and rotated in extended precision, pages handed out and taken back sequence by sequence."""
import math

import numpy as np
import torch

from serving_reference import Pool, attention_rows

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                    dtype=torch.float64)


def e2m1_rows(x):
    """Rows x [..., dh] float64 -> (codes [..., dh], exponent bytes [..., dh / 32]), from the definition: the least scale of 32
    dimensions that reaches their largest magnitude, the nearest value, ties to the even code, and 3 * 2^126 where that would be
    2^128."""
    x = x.unflatten(-1, (-1, 32))
    fin = torch.isfinite(x).all(-1)
    a = torch.where(fin, x.abs().nan_to_num(0, 0, 0).amax(-1), torch.zeros(()).double())
    e = torch.ones(a.shape, dtype=torch.int64)
    for b in range(1, 255):
        e = torch.where(a > 6.0 * 2.0 ** (b - 127), torch.full_like(e, b + 1), e)
    top = (x.abs() >= 3.5 * 2.0 ** 126) & torch.isfinite(x)
    x = torch.where(top, torch.copysign(torch.full_like(x, 3 * 2.0 ** 126), x), x)
    y = x / torch.exp2((e - 127).double())[..., None]
    dist = (y.abs().nan_to_num(0, 0, 0)[..., None] - E2M1[:8]).abs()
    best = dist.amin(-1, keepdim=True)
    code = torch.where(dist == best, torch.tensor([0, 8, 1, 9, 2, 10, 3, 11]), 99).argmin(-1)   # even codes before odd ones
    code = code + 8 * torch.signbit(x)
    code = torch.where(fin[..., None], code, torch.zeros_like(code))
    return code.flatten(-2), torch.where(fin, e, torch.full_like(e, 255))


def scale_of(e):
    return torch.where(e == 255, torch.full(e.shape, math.nan, dtype=torch.float64), torch.exp2(e.double() - 127))


def key_bytes(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)


def value_bytes(code):
    c = code.unflatten(-1, (-1, 2, 16))
    return (c[..., 0, :] | c[..., 1, :] << 4).flatten(-2).to(torch.uint8)


def key_codes(byte):
    return torch.stack([byte & 15, byte >> 4], -1).flatten(-2).long()


def value_codes(byte):
    c = byte.unflatten(-1, (-1, 16))
    return torch.stack([c & 15, c >> 4], -2).flatten(-3).long()


class Pool4(Pool):
    """A random pool of 4 bits with its tables on the CPU, and the same on the device."""

    def __init__(self, dcl, lens, page, hkv, dh, seed=0, spare=2, width=None, fill=None):
        super().__init__(dcl, lens, page, hkv, dh, False, seed, spare, width)
        g = torch.Generator().manual_seed(seed + 1000)
        n, ng = self.n_pages, dh // 32
        self.k = torch.randint(0, 256, (n, hkv, page, dh // 2), generator=g, dtype=torch.uint8)
        self.v = torch.randint(0, 256, (n, hkv, dh // 2, page), generator=g, dtype=torch.uint8)
        self.ks = torch.randint(123, 127, (n, hkv, ng, page), generator=g, dtype=torch.uint8)
        self.vs = torch.randint(123, 128, (n, hkv, ng, page), generator=g, dtype=torch.uint8)
        if fill is not None:
            self.spoil4(fill)

    def spoil4(self, byte):
        """What lies behind every sequence's end: any codes, scales that make them NaN."""
        idle = torch.ones(self.n_pages, self.page, dtype=torch.bool)
        for b in range(len(self.lens)):
            if self.lens[b]:
                idle[self.places(b)] = False
        for x, y in ((self.k.permute(0, 2, 1, 3), byte), (self.v.permute(0, 3, 1, 2), byte),
                     (self.ks.permute(0, 3, 1, 2), 255), (self.vs.permute(0, 3, 1, 2), 255)):
            x[idle] = y

    def rows(self, b, n=None):
        pg, off = self.places(b, n)
        k, v = self.k.permute(0, 2, 1, 3)[pg, off], self.v.permute(0, 3, 1, 2)[pg, off]
        ks, vs = (scale_of(s.permute(0, 3, 1, 2)[pg, off]).repeat_interleave(32, -1) for s in (self.ks, self.vs))
        return E2M1[key_codes(k)] * ks, E2M1[value_codes(v)] * vs

    def device(self):
        d = self.dcl
        return d.KVPages(self.n_pages, self.page, self.hkv, self.dh, d.DCL_DTYPE_E2M1, k=self.k.cuda(), v=self.v.cuda(),
                         k_scale=self.ks.cuda(), v_scale=self.vs.cuda())


def norm_rope(x, pos, gain, eps, base, rot):
    """x [T, H, dh] float64, pos [T]. Returns y and the error that a float32 evaluation with a bfloat16 result may have:
    half a step of bfloat16, the sums' and products' roundings, sines and cosines to 2^-21 (an angle's fraction of a turn kept to
    2^-26, the functions to 2^-22), and what 52 bits of the turns leave of the angle at far positions."""
    T, H, dh = x.shape
    half = rot // 2
    y = x.clone()
    rel = 0.0
    if gain is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * gain.double()
        rel = (dh + 12) * 2.0 ** -24
    mag = y.abs()
    err = mag * rel
    if rot:
        p = pos.numpy().astype(np.longdouble)
        turns = p[:, None] * np.longdouble(base) ** (-2 * np.arange(half, dtype=np.longdouble) / rot) / (2 * np.longdouble(np.pi) +
                                                                                                         np.longdouble(2.4492935982947064e-16))
        angle = torch.from_numpy(((turns - np.round(turns)) * 2 * np.longdouble(np.pi)).astype(np.float64))[:, None]
        far = torch.from_numpy((np.abs(turns) * 2.0 ** -51).astype(np.float64))[:, None] * 2 * math.pi
        c, s = torch.cos(angle), torch.sin(angle)
        a, b = y[..., :half], y[..., half:rot]
        y = torch.cat([a * c - b * s, b * c + a * s, y[..., rot:]], -1)
        both = mag[..., :half] + mag[..., half:rot]
        e = both * (2.0 ** -21 + rel + 2.0 ** -22 + far)
        err = torch.cat([e, e, err[..., rot:]], -1)
    return y, err * (1 + 2.0 ** -8) + y.abs() * 2.0 ** -8 + 2.0 ** -133


class Turn:
    """Table, lengths and free list as Python lists; extend and shrink by their rules, one sequence after the other."""

    def __init__(self, table, length, free, n_free, page, n_pages):
        self.table, self.len, self.free, self.n_free = [list(r) for r in table], list(length), list(free), n_free
        self.page, self.n_pages, self.width = page, n_pages, len(table[0])

    def pages(self, n):
        return -(-n // self.page)

    def listed(self):
        return max(0, min(self.n_free, self.n_pages))

    def extend(self, count, T):
        B = len(self.len)
        count = [1] * B if count is None else count
        left, asked, wanted, at = self.listed(), 0, 0, 0
        have = left
        cu, pos, slot = [0], [-1] * T, [-1] * T
        for b in range(B):
            n, c = self.len[b], count[b]
            ok = 0 <= n and 0 <= c and n + c <= self.width * self.page
            if ok:
                asked += c
                ok = asked <= T
            if ok:
                need = self.pages(n + c) - self.pages(n)
                wanted += need
                ok = need == 0 or wanted <= have
            if ok:
                for x in range(n, n + c):
                    if x % self.page == 0:
                        left -= 1
                        self.table[b][x // self.page] = self.free[left]
                    pos[at] = x
                    pg = self.table[b][x // self.page]
                    slot[at] = pg * self.page + x % self.page if 0 <= pg < self.n_pages else -1
                    at += 1
                self.len[b] = n + c
            cu.append(at)
        self.n_free = left
        return cu, pos, slot

    def shrink(self, keep):
        back = []
        for b in range(len(self.len)):
            n, k = self.len[b], keep[b]
            if not (0 <= k < n and n <= self.width * self.page):
                continue
            for j in range(self.pages(k), self.pages(n)):
                if 0 <= self.table[b][j] < self.n_pages:
                    back.append(self.table[b][j])
                self.table[b][j] = -1
            self.len[b] = k
        self.n_free = self.listed()
        for pg in reversed(back):
            if self.n_free < self.n_pages:
                self.free[self.n_free] = pg
                self.n_free += 1


def attention_rows4(q, k, v, scale, sees):
    """attention_rows with what 4-bit pages add to its bounds.

    Values may be exactly 0, so that an output may consist of the least probabilities alone: a probability below 2^-126 of the
    reference point (which some key of the row has reached, so that they sum to 1 at least) may be flushed to 0, and with it
    2^-126 of its value.

    Heads of 128: the query is held as two e4m3 parts with scales s and s / 16 for every 32 dimensions, the largest of which is in (224 s,
    448 s]. The first part leaves at most half of its step, 16 s at most; the second is e4m3 of that over s / 16, at most
    256, to half a step: exact where eight significant bits of the element end above 2^-9 s / 16, otherwise within half of
    that step, 2^-14 s, below 2^-21 of the largest. A score moves by that times the sum of the group's |k|, a
    probability by twice the largest move of a score relative to itself, the lse by once."""
    o, lse, eo, el = attention_rows(q, k, v, scale, sees)
    for i in range(len(sees)):
        j = sees[i].nonzero()[:, 0]
        if len(j) == 0:
            continue
        eo[i] += v[j].abs().nan_to_num(0, 0, 0).sum(0) * 2.0 ** -126
        if q.shape[1] == 128:
            top = q[i].abs().nan_to_num(0, 0, 0).unflatten(0, (4, 32)).amax(-1)
            move = (k[j].abs().nan_to_num(0, 0, 0).unflatten(1, (4, 32)).sum(-1) @ top) * abs(scale) * 2.0 ** -21
            p = torch.exp((k[j] @ q[i]) * scale - lse[i])
            eo[i] += (p @ v[j].abs()).nan_to_num(0, 0, 0) * 2 * float(move.max())
            el[i] += float(move.max())
    return o, lse, eo, el


def check4(pool, out, lse, q, cu, counts, heads, causal, scale, max_new=None, seen=None):
    """Every row and head of an attention over a pool of 4 bits."""
    g = heads // pool.hkv
    for b, n in enumerate(counts):
        L = pool.lens[b]
        have = min(L, pool.width * pool.page)
        k, v = pool.rows(b, have)
        sees = torch.ones(n, have, dtype=torch.bool)
        if causal:
            sees &= torch.arange(have)[None, :] <= (L - n + torch.arange(n))[:, None]
        if seen is not None:
            sees &= seen(b, have)[None, :]
        for i in range(n if max_new is None else min(n, max_new)):
            t = int(cu[b]) + i
            for h in range(heads):
                o, s, eo, es = attention_rows4(q[t, h].double()[None], k[:, h // g], v[:, h // g], scale, sees[i:i + 1])
                got, want = out[t, h], o[0]
                assert torch.equal(torch.isnan(got), torch.isnan(want)), (b, i, h)
                ok = ~torch.isnan(want)
                err = (got - want).abs()
                assert bool((err[ok] <= eo[0][ok]).all()), (b, i, h, float((err / eo[0].clamp(min=1e-300))[ok].max()))
                if math.isfinite(float(s[0])):
                    assert abs(float(lse[t, h] - s[0])) <= float(es[0]), (b, i, h)
                else:
                    assert float(lse[t, h]) == float(s[0]) or math.isnan(float(s[0])), (b, i, h)
