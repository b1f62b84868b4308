"""Plain float64 forms of the serving operators (packed prompts, paged cache, sampling) for their tests, with the error
that a float32 evaluation with bfloat16 probabilities and outputs may have, from the operands alone."""
import math

import numpy as np
import torch

U32 = 2.0 ** -23          # a float32 operation, truncating accumulators included
BF16 = 2.0 ** -8          # half a bfloat16 step, relative
LN2 = math.log(2.0)


def attention_rows(q, k, v, scale, sees):
    """q [n, dh], k / v [m, dh] (float64 tensors), sees [n, m] bool. Returns o, lse and the bounds on their errors.
    A row that sees nothing: zeros, -inf. Keys that a row does not see play no part, whatever they hold."""
    n, m = sees.shape
    dh = q.shape[1]
    o, lse = torch.zeros(n, dh, dtype=torch.float64), torch.full((n,), -math.inf, dtype=torch.float64)
    eo, el = torch.zeros(n, dh, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        j = sees[i].nonzero()[:, 0]
        if len(j) == 0:
            continue
        x = (k[j] @ q[i]) * scale
        # the product's dh roundings and those of its scaling, absolute, in the exponent
        d = float(((k[j].abs() @ q[i].abs()) * abs(scale)).nan_to_num(0, 0, 0).max()) * (dh + 4) * U32
        # the exponent is taken in log2 units: exp2's argument carries |x - max| roundings of its own
        top = x.max()
        d += float((x - top).abs().nan_to_num(0, 0, 0).clamp(max=200).max()) * 4 * U32
        lse[i] = torch.logsumexp(x, 0)
        p = torch.exp(x - lse[i])
        o[i] = p @ v[j]
        mag = p @ v[j].abs()
        rel = 2 * d + (len(j) + 16) * U32                      # sums of len(j) terms, exp2, the quotient
        eo[i] = mag * (BF16 + rel) * (1 + BF16) + o[i].abs() * BF16 + 2.0 ** -133
        el[i] = d + rel + abs(float(lse[i])) * 2 * U32 if math.isfinite(float(lse[i])) else 0.0
    return o, lse, eo, el


def e4m3_value(byte):
    e, f, s = (byte >> 3) & 15, byte & 7, -1.0 if byte >> 7 else 1.0
    if e == 15 and f == 7:
        return math.nan
    return s * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))


E4M3 = torch.tensor([e4m3_value(b) for b in range(256)], dtype=torch.float64)


def e4m3_rows(x):
    """Rows x [..., dh] float64 -> (values of the stored bytes before the scale, exponent bytes), from the definition."""
    fin = torch.isfinite(x)
    a = torch.where(fin, x.abs(), torch.zeros_like(x)).amax(-1)
    e = torch.ones(a.shape, dtype=torch.int64)
    for b in range(1, 255):                                    # the least exponent whose scale reaches amax
        e = torch.where(a > 448.0 * 2.0 ** (b - 127), torch.full_like(e, b + 1), e)
    y = x / torch.exp2((e - 127).double())[..., None]
    pos = E4M3[:127]                                           # 0 .. 448, increasing
    mag = y.abs().nan_to_num(0, 0, 0)
    hi = torch.searchsorted(pos, mag).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, dn = pos[hi] - mag, mag - pos[lo]
    pick = torch.where((up < dn) | ((up == dn) & (hi % 2 == 0)), hi, lo)
    val = torch.copysign(pos[pick], x)
    return torch.where(fin, val, torch.full_like(val, math.nan)), e


class Pool:
    """A random pool with its tables on the CPU, and the same on the device."""

    def __init__(self, dcl, lens, page, hkv, dh, e4m3, seed=0, spare=2, width=None, fill=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.hkv, self.dh, self.e4m3 = list(lens), page, hkv, dh, e4m3
        need = [-(-n // page) for n in lens]
        self.n_pages, self.width = sum(need) + spare, max([1] + need) if width is None else width
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
        sk, sv = (self.n_pages, hkv, page, dh), (self.n_pages, hkv, dh, page)
        self.ks = self.vs = None
        if e4m3:
            def codes(shape):
                x = (torch.randn(shape, generator=g) * 48).to(torch.float8_e4m3fn).view(torch.uint8)
                return torch.where((x & 127) == 127, x - 1, x)
            self.k, self.v = codes(sk), codes(sv)
            self.ks = torch.randint(119, 124, sk[:3], generator=g, dtype=torch.uint8)
            self.vs = torch.randint(119, 124, sk[:3], generator=g, dtype=torch.uint8)
        else:
            self.k = torch.randn(sk, generator=g).to(torch.bfloat16)
            self.v = torch.randn(sv, generator=g).to(torch.bfloat16)
        if fill is not None:                                    # what lies behind every sequence's end
            self.spoil(fill)
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.dcl = dcl

    def places(self, b, n=None):
        """Page and offset of positions 0 .. n - 1 of sequence b."""
        x = torch.arange(self.lens[b] if n is None else n)
        return self.table[b].long()[x // self.page], x % self.page

    def spoil(self, byte):
        used = torch.zeros(self.n_pages, self.page, dtype=torch.bool)
        for b in range(len(self.lens)):
            if self.lens[b]:
                used[self.places(b)] = True
        idle = ~used
        if self.e4m3:
            self.k.permute(0, 2, 1, 3)[idle] = byte
            self.v.permute(0, 3, 1, 2)[idle] = byte
            self.ks.permute(0, 2, 1)[idle] = 255
            self.vs.permute(0, 2, 1)[idle] = 255
        else:
            bits = torch.tensor([byte << 8 | byte], dtype=torch.int32).to(torch.int16).view(torch.bfloat16)[0]
            self.k.permute(0, 2, 1, 3)[idle] = bits
            self.v.permute(0, 3, 1, 2)[idle] = bits

    def rows(self, b, n=None):
        """Keys and values [n, hkv, dh] of sequence b in float64."""
        pg, off = self.places(b, n)
        k, v = self.k.permute(0, 2, 1, 3)[pg, off], self.v.permute(0, 3, 1, 2)[pg, off]
        if not self.e4m3:
            return k.double(), v.double()
        ks, vs = (torch.exp2(s.permute(0, 2, 1)[pg, off].double() - 127)[..., None] for s in (self.ks, self.vs))
        return E4M3[k.long()] * ks, E4M3[v.long()] * vs

    def device(self):
        d = self.dcl
        t = {n: None if x is None else x.cuda() for n, x in (("k", self.k), ("v", self.v), ("k_scale", self.ks),
                                                             ("v_scale", self.vs))}
        return d.KVPages(self.n_pages, self.page, self.hkv, self.dh,
                         d.DCL_DTYPE_E4M3 if self.e4m3 else d.DCL_DTYPE_BF16, **t)


def starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)


def sample_row(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """Token, its share of the kept weight and the ids kept, in float64 from a sorted row. x: float64 numpy logits; the
    settings are the float32 values that the call takes."""
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    if x.max() == -np.inf:
        return -1, 0.0, 0
    greedy = not temperature > 0
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if greedy:
        return int(order[0]), 1.0, 1
    v = x[order]
    with np.errstate(all="ignore"):
        w = np.where(v == v[0], 1.0, np.nan_to_num(np.exp((v - v[0]) / temperature), nan=0.0))
    if top_k > 0:
        w = w[:top_k]
    keep = np.ones(len(w), bool)
    before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
    if top_p < 1:
        keep &= before < top_p * w.sum()
        keep[0] = True
    if min_p > 0:
        keep &= w >= min(min_p, 1.0)
    n = int(keep.sum())
    assert keep[:n].all()
    w = w[:n]
    upto = np.cumsum(w)
    u = 0.0 if not u > 0 else u
    at = min(int((upto <= u * upto[-1]).sum()), n - 1)
    if u >= 1:                                            # past the end: the last id with any weight
        at = int(np.nonzero(w > 2.0 ** -45)[0][-1])
    return int(order[at]), float(w[at] / upto[-1]), n
