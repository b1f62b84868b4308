"""The serving operators beside the denoising step, as cases that can be timed and checked.

A decode service keeps the keys and values of many sequences of different lengths in one pool of pages. A new
prompt is attended to as a whole (``dcl_prompt_attention``, prompts packed one behind the other), its keys and
values go into pages (``dcl_pages_write``, in bfloat16 or in 8 bits), every iteration attends from a few new tokens
to the pages (``dcl_pages_attention``), pages are read back when a sequence moves (``dcl_pages_read``), and the
head's logits become tokens (``dcl_sample_tokens``).

With ``own`` false ``run`` computes the same from elementary torch operations in float32 (float64 for the sampler's
sums, whose borders decide which id is drawn). ``exact`` evaluates the definitions in float64.

Lengths are part of a case: they come from its own numbers, not from the seed of its inputs.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # a handful of short prompts of the small model's heads, bidirectional: latency
        {"name": "prompt 6 short", "op": "prompt", "seqs": 6, "lo": 1, "hi": 48, "heads": 4, "kv_heads": 4, "dim": 64,
         "causal": False, "pad": 3, "lens": 1},
        # a batch of arriving prompts of ragged lengths, grouped heads
        {"name": "prompt ragged gqa", "op": "prompt", "seqs": 8, "lo": 65, "hi": 1531, "heads": 28, "kv_heads": 4,
         "dim": 128, "causal": True, "pad": 0, "lens": 2},
        # one long document
        {"name": "prompt 8192", "op": "prompt", "seqs": 1, "lo": 8192, "hi": 8192, "heads": 32, "kv_heads": 32,
         "dim": 128, "causal": True, "pad": 0, "lens": 3},
        # one token of four short sequences, bfloat16 pages: latency
        {"name": "pages 4x1 short", "op": "attend", "seqs": 4, "lo": 90, "hi": 700, "new": 1, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 32, "e4m3": False, "causal": True, "lens": 4},
        # one token of a large ragged batch, 8-bit pages, grouped heads
        {"name": "pages 64x1 e4m3", "op": "attend", "seqs": 64, "lo": 200, "hi": 8000, "new": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64, "e4m3": True, "causal": True, "lens": 5},
        # one token of two very long sequences
        {"name": "pages 2x1 long", "op": "attend", "seqs": 2, "lo": 90000, "hi": 131072, "new": 1, "heads": 28,
         "kv_heads": 4, "dim": 128, "page": 64, "e4m3": False, "causal": True, "lens": 6},
        # a denoising block: eight sequences' 64 tokens over 1216 cached ones, 8-bit pages, every token sees every other
        {"name": "pages 8x64 block", "op": "attend", "seqs": 8, "lo": 1280, "hi": 1280, "new": 64, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64, "e4m3": True, "causal": False, "lens": 7},
        # the new token of each sequence of a batch into 8-bit pages
        {"name": "write 64x1 e4m3", "op": "write", "seqs": 64, "lo": 100, "hi": 3000, "new": 1, "kv_heads": 8,
         "dim": 128, "page": 64, "e4m3": True, "lens": 8},
        # whole prompts into 8-bit pages
        {"name": "write prompts e4m3", "op": "write", "seqs": 9, "lo": 500, "hi": 7000, "new": 0, "kv_heads": 32,
         "dim": 128, "page": 64, "e4m3": True, "lens": 9},
        # whole sequences back into rows
        {"name": "read e4m3", "op": "read", "seqs": 7, "lo": 300, "hi": 5000, "new": 0, "kv_heads": 8, "dim": 128,
         "page": 32, "e4m3": True, "lens": 10},
        # the next token of four sequences: latency
        {"name": "sample 4", "op": "sample", "rows": 4, "vocab": 126464, "bf16": False, "sets": "filtered"},
        # a batch of masked positions, every request with its own settings
        {"name": "sample 512", "op": "sample", "rows": 512, "vocab": 152064, "bf16": True, "sets": "mixed"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "attend", "attend", "write", "read", "sample"])
    kv = rng.choice([1, 2, 4, 8, 32])
    heads = kv * rng.choice([1, 1, 2, 4, 7]) if kv < 32 else 32
    dim = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    lens = rng.randrange(1 << 30)
    if op == "prompt":
        hi = _log(rng, 8, 8192)
        causal = rng.random() < 0.6
        total = min(8192, math.isqrt((2 if causal else 1) * (1 << 30) // heads))
        hi = min(hi, total)
        seqs = max(1, min(_log(rng, 1, 24), total // hi))
        return {"op": op, "seqs": seqs, "lo": rng.choice([1, max(1, hi // 3)]), "hi": hi, "heads": heads,
                "kv_heads": kv, "dim": dim, "causal": causal, "pad": rng.choice([0, 0, 5]), "lens": lens}
    if op == "sample":
        vocab = _log(rng, 300, 152064)
        rows = _log(rng, 1, max(1, min(2000, (512 * 152064) // vocab)))
        return {"op": op, "rows": rows, "vocab": vocab, "bf16": rng.random() < 0.5,
                "sets": rng.choice(["mixed", "filtered", "plain"])}
    e4m3 = rng.random() < 0.6
    # tokens of all sequences together: a pool of half a GiB of bfloat16, where it is written or read half of that
    total = ((1 << 27) - (1 << 23) if op == "attend" else 1 << 26) // (kv * dim)
    hi = _log(rng, 20, 100000 if op == "attend" else 20000)
    hi = min(hi, total)
    seqs = max(1, min(_log(rng, 1, 128), total // hi))
    lo = max(1, hi // rng.choice([1, 3, 20]))
    c = {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "new": 0, "kv_heads": kv, "dim": dim, "page": page, "e4m3": e4m3,
         "lens": lens}
    if op == "attend":
        most = max(1, min(64, lo, (1 << 28) // (seqs * heads * hi)))
        c["new"] = rng.choice([1, 1, rng.randint(1, most)])
        c["heads"] = heads
        c["causal"] = rng.random() < 0.6
    elif op == "write":
        c["new"] = rng.choice([0, 1, min(lo, rng.randint(1, 300))])
    return c


def _lengths(case):
    """The sequences' lengths: log-uniform over [lo, hi], the first one hi."""
    r = random.Random(case["lens"])
    return [case["hi"]] + [_log(r, case["lo"], case["hi"]) for _ in range(case["seqs"] - 1)]


def _new(case):
    """How many tokens of each sequence the call takes: `new`, or with 0 the whole sequence."""
    return [min(case["new"], n) if case["new"] else n for n in _lengths(case)]


def work(case):
    op = case["op"]
    if op == "sample":
        return {"bytes": case["rows"] * case["vocab"] * (2 if case["bf16"] else 4), "flops": 0}
    n, d = _lengths(case), case["dim"]
    if op == "prompt":
        h, hkv, t = case["heads"], case["kv_heads"], sum(n)
        pairs = sum(x * (x + 1) // 2 if case["causal"] else x * x for x in n)
        return {"bytes": 4 * t * d * (h + hkv) + 4 * t * h, "flops": 4 * d * h * pairs}
    per = 2 * case["kv_heads"] * ((d + 1) if case["e4m3"] else 2 * d)     # one token in the pages
    if op == "attend":
        m, h = _new(case), case["heads"]
        pairs = sum(b * a - (b * (b - 1) // 2 if case["causal"] else 0) for a, b in zip(n, m))
        return {"bytes": per * sum(n) + 4 * sum(m) * h * d + 4 * sum(m) * h, "flops": 4 * d * h * pairs}
    t = sum(_new(case))
    return {"bytes": t * (per + 4 * case["kv_heads"] * d), "flops": 0}


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return (torch.randn(shape, device="cuda", generator=g) * std).to(torch.bfloat16)

    if case["op"] == "sample":
        return _prepare_sample(case, g)
    n, d = _lengths(case), case["dim"]
    s = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case["op"] == "prompt":
        t, h, hkv = sum(n) + case["pad"], case["heads"], case["kv_heads"]
        s.update(T=t, most=max(n), cu=_ints(_starts(n)), q=normal(t, h, d, std=1.5), k=normal(t, hkv, d),
                 v=normal(t, hkv, d), out=torch.zeros((t, h, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((t, h), device="cuda"))
        return s
    # a pool whose pages are handed out in no order, a few of them to nobody
    page, hkv, e4m3 = case["page"], case["kv_heads"], case["e4m3"]
    need = [-(-x // page) for x in n]
    pool, width = sum(need) + 3, max(need)
    order = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
    at = _starts(need)
    table = torch.full((len(n), width), -1, dtype=torch.int32, device="cuda")
    for b, c in enumerate(need):
        table[b, :c] = order[at[b]:at[b] + c]
    m = _new(case)
    t = sum(m)
    s.update(T=t, most=max(m), cu=_ints(_starts(m)), len=_ints(n), table=table, width=width, n_pages=pool)
    if e4m3:
        # any finite bit pattern is a value that a page may hold; scales near those of activations
        def codes(*shape):
            x = torch.randint(0, 256, shape, device="cuda", generator=g, dtype=torch.uint8)
            return torch.where((x & 0x7f) == 0x7f, x - 1, x)

        # values near 1: exponents of the stored bytes from 2^-6 to 2^1 times a scale of about one
        if case["op"] == "write":
            kp, vp = codes(pool, hkv, page, d), codes(pool, hkv, d, page)
        else:
            kp = normal(pool, hkv, page, d, std=64.0).to(torch.float8_e4m3fn).view(torch.uint8)
            vp = normal(pool, hkv, d, page, std=64.0).to(torch.float8_e4m3fn).view(torch.uint8)
        s.update(k_pages=kp, v_pages=vp,
                 k_scale=torch.randint(120, 123, (pool, hkv, page), device="cuda", generator=g, dtype=torch.uint8),
                 v_scale=torch.randint(120, 123, (pool, hkv, page), device="cuda", generator=g, dtype=torch.uint8))
    else:
        s.update(k_pages=normal(pool, hkv, page, d), v_pages=normal(pool, hkv, d, page), k_scale=None, v_scale=None)
    if case["op"] == "attend":
        h = case["heads"]
        s.update(q=normal(t, h, d, std=1.5), out=torch.zeros((t, h, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((t, h), device="cuda"))
    elif case["op"] == "write":
        # keys after the rotation have a few large dimensions; heads differ in size
        size = torch.exp(torch.randn((1, hkv, d), device="cuda", generator=g))
        s.update(k=(normal(t, hkv, d) * size).to(torch.bfloat16), v=normal(t, hkv, d))
    else:
        s.update(k=torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda"),
                 v=torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda"))
    s["handle"] = None
    return s


def _prepare_sample(case, g):
    n, vocab = case["rows"], case["vocab"]

    def uni(lo=0.0, hi=1.0, size=(n,)):
        return torch.rand(size, device="cuda", generator=g) * (hi - lo) + lo

    def pick(*values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (n,), device="cuda", generator=g)]

    # a head's logits: a broad floor and a few ids that stand out, by more or less
    x = torch.randn((n, vocab), device="cuda", generator=g) * uni(1.0, 2.5)[:, None]
    few = torch.randint(0, vocab, (n, 20), device="cuda", generator=g)
    x.scatter_add_(1, few, uni(4.0, 14.0)[:, None] * torch.rand((n, 20), device="cuda", generator=g))
    x[:, vocab - 1] = -math.inf                                   # the mask id, suppressed
    x = x.to(torch.bfloat16) if case["bf16"] else x
    s = {"case": case, "logits": x, "uniform": uni(), "temperature": None, "top_k": None, "top_p": None,
         "min_p": None}
    if case["sets"] == "filtered":                                # one setting for all requests
        s.update(temperature=torch.full((n,), 0.7, device="cuda"),
                 top_k=torch.full((n,), 50, dtype=torch.int32, device="cuda"),
                 top_p=torch.full((n,), 0.95, device="cuda"))
    elif case["sets"] == "mixed":                                 # every request its own, 0 or 1 where it has none
        s.update(temperature=pick(0.0, 0.2, 0.6, 1.0, 1.0, 1.3), top_k=pick(0, 0, 1, 20, 50, 1000).to(torch.int32),
                 top_p=pick(1.0, 1.0, 0.5, 0.9, 0.95), min_p=pick(0.0, 0.0, 0.0, 0.05))
    s.update(token=torch.zeros(n, dtype=torch.int32, device="cuda"), conf=torch.zeros(n, device="cuda"),
             kept=torch.zeros(n, dtype=torch.int32, device="cuda"))
    return s


def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


# ---------------------------------------------------------------- the framework's calls

def _handle(s):
    """The pool's description and the call's workspace, made at the first call and kept, as a program keeps them."""
    if s.get("handle") is None:
        import paper_2607_20467_amd as dcl
        c = s["case"]
        if c["op"] == "sample":
            need = dcl.dcl_sample_workspace_bytes(c["rows"], c["vocab"])
            s["handle"] = (dcl, None, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
        elif c["op"] == "prompt":
            s["handle"] = (dcl, None, None, 0)
        else:
            pool = dcl.KVPages(s["n_pages"], c["page"], c["kv_heads"], c["dim"],
                               dcl.DCL_DTYPE_E4M3 if c["e4m3"] else dcl.DCL_DTYPE_BF16, k=s["k_pages"],
                               v=s["v_pages"], k_scale=s["k_scale"], v_scale=s["v_scale"])
            ws, need = None, 0
            if c["op"] == "attend":
                need = dcl.dcl_pages_attention_workspace_bytes(pool, c["heads"], c["seqs"], s["T"], s["most"],
                                                               s["width"])
                ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            s["handle"] = (dcl, pool, ws, need)
    return s["handle"]


def _own_prompt(s):
    dcl, c = _handle(s)[0], s["case"]
    dcl.dcl_prompt_attention(s["q"], s["k"], s["v"], s["cu"], c["seqs"], s["T"], s["most"], c["heads"], c["kv_heads"],
                             c["dim"], s["scale"], c["causal"], s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_attend(s):
    (dcl, pool, ws, need), c = _handle(s), s["case"]
    dcl.dcl_pages_attention(pool, s["table"], s["len"], s["cu"], c["seqs"], s["T"], s["most"], s["q"], c["heads"],
                            s["scale"], c["causal"], s["out"], s["lse"], ws, need)
    return {"out": s["out"], "lse": s["lse"]}


def _pages_of(s):
    """The pool: 8-bit pages as the values of their bytes, with the scales' exponents."""
    if not s["case"]["e4m3"]:
        return {"k": s["k_pages"], "v": s["v_pages"]}
    return {"k": s["k_pages"].view(torch.float8_e4m3fn), "v": s["v_pages"].view(torch.float8_e4m3fn),
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _own_write(s):
    dcl, pool = _handle(s)[:2]
    dcl.dcl_pages_write(pool, s["table"], s["len"], s["cu"], s["case"]["seqs"], s["T"], s["most"], s["k"], s["v"])
    return _pages_of(s)


def _own_read(s):
    dcl, pool = _handle(s)[:2]
    dcl.dcl_pages_read(pool, s["table"], s["len"], s["cu"], s["case"]["seqs"], s["T"], s["most"], s["k"], s["v"])
    return {"k": s["k"], "v": s["v"]}


def _own_sample(s):
    (dcl, _, ws, need), c = _handle(s), s["case"]
    dcl.dcl_sample_tokens(s["logits"], c["rows"], c["vocab"], s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                          s["uniform"], s["token"], s["conf"], s["kept"], ws, need)
    return {"token": s["token"], "conf": s["conf"], "kept": s["kept"]}


_own = {"prompt": _own_prompt, "attend": _own_attend, "write": _own_write, "read": _own_read, "sample": _own_sample}


# ---------------------------------------------------------------- the plain forms

def _softmax_product(x, ok, v):
    """Rows of scores `x` (float32, overwritten) where `ok`, times `v`: the products, and log of the rows' sums of exp.
    A row without a key gives zeros and -inf."""
    x.masked_fill_(~ok, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total), lse


def _plain_prompt(s):
    c = s["case"]
    g, t = c["heads"] // c["kv_heads"], s["T"]
    q = s["q"].float().transpose(0, 1).contiguous() * s["scale"]
    k = s["k"].float().permute(1, 2, 0).repeat_interleave(g, 0)
    v = s["v"].float().transpose(0, 1).repeat_interleave(g, 0)
    at = torch.arange(t, dtype=torch.int32, device="cuda")
    seq = torch.bucketize(at, s["cu"][1:], right=True)
    ok = (seq[:, None] == seq[None, :]) & (seq[:, None] < c["seqs"])
    if c["causal"]:
        ok &= at[None, :] <= at[:, None]
    out, lse = _softmax_product(torch.matmul(q, k.contiguous()), ok, v)
    row = (seq < c["seqs"])[:, None]
    s["out"].copy_(torch.where(row[:, :, None], out.transpose(0, 1), s["out"].float()))
    s["lse"].copy_(torch.where(row, lse.transpose(0, 1), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _pow2(n):
    """2^n for whole numbers n in float64, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _rows_of_pages(s):
    """Keys and values [B, Hkv, width * page, dh] in float32, and which of them a page of the table holds."""
    c = s["case"]
    tab = s["table"].long().clamp(min=0)
    b, d, hkv, most = c["seqs"], c["dim"], c["kv_heads"], s["width"] * c["page"]
    k, v = s["k_pages"][tab], s["v_pages"][tab]                   # [B, width, Hkv, page, dh] and [.., dh, page]
    if c["e4m3"]:
        ks = _pow2(s["k_scale"][tab].long() - 127).float()
        vs = _pow2(s["v_scale"][tab].long() - 127).float()
        k = k.view(torch.float8_e4m3fn).float() * ks[..., None]
        v = v.view(torch.float8_e4m3fn).float() * vs[:, :, :, None, :]
    k = k.float().transpose(1, 2).reshape(b, hkv, most, d)
    v = v.float().permute(0, 2, 1, 4, 3).reshape(b, hkv, most, d)
    return k, v, (s["table"] >= 0).repeat_interleave(c["page"], 1)


def _new_rows(s):
    """For new token i of sequence b, [B, most]: its packed row (clamped), its position, and whether there is one."""
    i = torch.arange(s["most"], device="cuda")[None, :]
    count = (s["cu"][1:] - s["cu"][:-1])[:, None]
    row = (s["cu"][:-1][:, None] + i).clamp(max=s["T"] - 1)
    return row.long(), s["len"][:, None] - count + i, i < count


def _plain_attend(s):
    c = s["case"]
    b, h, hkv, d, most = c["seqs"], c["heads"], c["kv_heads"], c["dim"], s["most"]
    g = h // hkv
    k, v, held = _rows_of_pages(s)
    row, pos, is_new = _new_rows(s)
    q = s["q"].float()[row] * s["scale"]                          # [B, most, H, dh]
    q = q.view(b, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, most * g, d)
    j = torch.arange(k.shape[2], device="cuda")
    ok = (j[None, None, :] < s["len"][:, None, None]) & held[:, None, :]
    if c["causal"]:
        ok = ok & (j[None, None, :] <= pos[:, :, None])
    ok = ok.expand(b, most, -1).repeat_interleave(g, 1)[:, None]
    out, lse = _softmax_product(torch.matmul(q, k.transpose(2, 3).contiguous()), ok, v)
    out = out.view(b, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(b, most, h, d)
    lse = lse.view(b, hkv, most, g).permute(0, 2, 1, 3).reshape(b, most, h)
    s["out"][row[is_new]] = out[is_new].to(torch.bfloat16)
    s["lse"][row[is_new]] = lse[is_new]
    return {"out": s["out"], "lse": s["lse"]}


def _quantised(x):
    """Bytes and scale exponents of rows x [T, Hkv, dh]."""
    x = x.float()
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    frac, exp = torch.frexp(top)                                  # top = frac * 2^exp, frac in [0.5, 1); 448 = 0.875 * 2^9
    e = (exp - 9 + (frac > E4M3_MAX / 512.0).to(exp.dtype) + 127).clamp(1, 254)
    e = torch.where(top == 0, torch.ones_like(e), e)
    y = (x * _pow2(127 - e)[..., None]).float()
    return y.to(torch.float8_e4m3fn).view(torch.uint8), e.to(torch.uint8)


def _slots(s):
    """Page and offset of every row of the call."""
    c = s["case"]
    row, pos, is_new = _new_rows(s)
    page = s["table"].long().gather(1, (pos // c["page"]).clamp(min=0).long())
    return page[is_new], (pos % c["page"]).long()[is_new], row[is_new]


def _plain_write(s):
    page, off, row = _slots(s)
    k, v = s["k"][row], s["v"][row]
    if s["case"]["e4m3"]:
        k, ke = _quantised(k)
        v, ve = _quantised(v)
        s["k_scale"][page, :, off] = ke
        s["v_scale"][page, :, off] = ve
    s["k_pages"][page, :, off] = k
    s["v_pages"][page, :, :, off] = v
    return _pages_of(s)


def _plain_read(s):
    page, off, row = _slots(s)
    k, v = s["k_pages"][page, :, off], s["v_pages"][page, :, :, off]
    if s["case"]["e4m3"]:
        k = k.view(torch.float8_e4m3fn).float() * _pow2(s["k_scale"][page, :, off].long() - 127).float()[..., None]
        v = v.view(torch.float8_e4m3fn).float() * _pow2(s["v_scale"][page, :, off].long() - 127).float()[..., None]
    s["k"][row] = k.to(torch.bfloat16)
    s["v"][row] = v.to(torch.bfloat16)
    return {"k": s["k"], "v": s["v"]}


def _settings(s, n, vocab):
    """Temperature, top-k, top-p and min-p of every row [n, 1], those that are absent as values that change nothing."""
    one = torch.ones((n, 1), dtype=torch.float64, device="cuda")
    t = one if s["temperature"] is None else s["temperature"].double()[:, None]
    k = (one * 0).long() if s["top_k"] is None else s["top_k"].long()[:, None]
    p = one if s["top_p"] is None else s["top_p"].double()[:, None]
    m = one * 0 if s["min_p"] is None else s["min_p"].double()[:, None]
    greedy = ~(t > 0)
    return torch.where(greedy, one, t), torch.where(greedy, 1, torch.where(k > 0, k, vocab)), p, m.clamp(max=1.0)


def _plain_sample(s):
    x = s["logits"].float()
    n, vocab = x.shape
    t, k, p, m = _settings(s, n, vocab)
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    x, ids = torch.sort(x, dim=1, descending=True, stable=True)
    top = x[:, :1]
    w = torch.exp((x.double() - top.double()) / t)
    w = torch.where(x == top, torch.ones_like(w), w)
    rank = torch.arange(vocab, device="cuda")[None, :]
    keep = (x > -math.inf) & (rank < k)
    w = torch.where(keep, w, torch.zeros_like(w))
    upto = torch.cumsum(w, 1)
    before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], 1)
    keep &= ((before < p * upto[:, -1:]) | (rank == 0) | (p >= 1)) & (w >= m)
    w = torch.where(keep, w, torch.zeros_like(w))
    upto = torch.cumsum(w, 1)
    kept = keep.sum(1)
    at = (upto <= s["uniform"].double()[:, None] * upto[:, -1:]).sum(1)
    at = torch.minimum(at, kept - 1).clamp(min=0)[:, None]
    some = kept > 0
    s["token"].copy_(torch.where(some, ids.gather(1, at)[:, 0], -1))
    s["conf"].copy_(torch.where(some, (w.gather(1, at) / upto[:, -1:])[:, 0], 0.0))
    s["kept"].copy_(kept)
    return {"token": s["token"], "conf": s["conf"], "kept": s["kept"]}


_plain = {"prompt": _plain_prompt, "attend": _plain_attend, "write": _plain_write, "read": _plain_read,
          "sample": _plain_sample}


# ---------------------------------------------------------------- the definitions in float64

def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "attend": _exact_attend, "write": _exact_write, "read": _exact_read,
            "sample": _exact_sample}[case["op"]](s)


def _exact_attention(q, k, v, scale, limits):
    """Queries [n, dh] over keys [m, dh], query i over the first limits[i] of them: float64 output and lse."""
    x = (q.double() @ k.double().T) * scale
    dead = torch.arange(k.shape[0], device="cuda")[None, :] >= limits[:, None]
    lse = torch.logsumexp(x.masked_fill(dead, -math.inf), 1)
    p = torch.exp(x - lse[:, None]).masked_fill(dead, 0.0)
    return p @ v.double(), lse


def _exact_prompt(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    g, at = c["heads"] // c["kv_heads"], 0
    for n in _lengths(c):
        lim = torch.arange(1, n + 1, device="cuda") if c["causal"] else torch.full((n,), n, device="cuda")
        for h in range(c["heads"]):
            out[at:at + n, h], lse[at:at + n, h] = _exact_attention(
                s["q"][at:at + n, h], s["k"][at:at + n, h // g], s["v"][at:at + n, h // g], s["scale"], lim)
        at += n
    return {"out": out, "lse": lse}


def _e4m3_table():
    """The value of every byte: sign, four exponent bits of bias 7, three of the fraction."""
    val = []
    for byte in range(256):
        e, f = (byte >> 3) & 15, byte & 7
        x = f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7)
        val.append(math.nan if e == 15 and f == 7 else -x if byte >> 7 else x)
    return torch.tensor(val, dtype=torch.float64, device="cuda")


def _exact_rows(s, b, n):
    """Keys and values [Hkv, n, dh] of sequence b in float64."""
    c = s["case"]
    pages = s["table"][b, :-(-n // c["page"])].long()
    k, v = s["k_pages"][pages], s["v_pages"][pages].transpose(2, 3)
    if c["e4m3"]:
        val = _e4m3_table()
        k = val[k.long()] * _pow2(s["k_scale"][pages].long() - 127)[..., None]
        v = val[v.long()] * _pow2(s["v_scale"][pages].long() - 127)[..., None]
    return [x.double().transpose(0, 1).flatten(1, 2)[:, :n] for x in (k, v)]


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    g, at = c["heads"] // c["kv_heads"], 0
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        k, v = _exact_rows(s, b, n)
        lim = torch.arange(n - m + 1, n + 1, device="cuda") if c["causal"] else torch.full((m,), n, device="cuda")
        for h in range(c["heads"]):
            out[at:at + m, h], lse[at:at + m, h] = _exact_attention(s["q"][at:at + m, h], k[h // g], v[h // g],
                                                                    s["scale"], lim)
        at += m
    return {"out": out, "lse": lse}


def _exact_e4m3(x):
    """Rows x [T, Hkv, dh]: the nearest e4m3 values of x / scale, ties to even."""
    x = x.double()
    top = x.abs().amax(-1)
    e = torch.ceil(torch.log2(top / E4M3_MAX))                    # the least with top <= 448 * 2^e, but for rounding
    e = torch.where(top > E4M3_MAX * _pow2(e), e + 1, torch.where(top <= E4M3_MAX * _pow2(e - 1), e - 1, e))
    y = x / _pow2(e)[..., None]
    step = _pow2(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / step) * step


def _exact_write(s):
    c, at = s["case"], 0
    if not c["e4m3"]:
        k, v = s["k_pages"].double(), s["v_pages"].double()
    else:
        k, v = (s[x].view(torch.float8_e4m3fn).double() for x in ("k_pages", "v_pages"))
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        pos = torch.arange(n - m, n, device="cuda")
        page, off = s["table"][b].long()[pos // c["page"]], pos % c["page"]
        kr, vr = s["k"][at:at + m].double(), s["v"][at:at + m].double()
        if c["e4m3"]:
            kr, vr = _exact_e4m3(kr), _exact_e4m3(vr)
        k[page, :, off] = kr
        v[page, :, :, off] = vr
        at += m
    return {"k": k, "v": v, "k_scale": None, "v_scale": None} if c["e4m3"] else {"k": k, "v": v}


def _exact_read(s):
    c = s["case"]
    rows = [_exact_rows(s, b, n) for b, n in enumerate(_lengths(c))]
    k, v = (torch.cat([r[i].transpose(0, 1) for r in rows]) for i in (0, 1))
    return {"k": k, "v": v}


def _exact_sample(s):
    x = s["logits"].double()
    n, vocab = x.shape
    t, k, p, m = _settings(s, n, vocab)
    conf = torch.zeros(n, dtype=torch.float64, device="cuda")
    for r in range(n):
        y = x[r] / t[r]
        val, _ = torch.sort(y, descending=True)
        val = val[:int(min(int(k[r]), int((val > -math.inf).sum())))]
        prob = torch.exp(val - torch.logsumexp(val, 0))
        mass = torch.cumsum(prob, 0)
        count = vocab if p[r] >= 1 else int((mass < p[r]).sum()) + 1
        prob = prob[:count]
        prob = prob[prob >= prob[0] * m[r]]
        mass = torch.cumsum(prob, 0)
        at = min(int((mass <= s["uniform"][r].double() * mass[-1]).sum()), len(prob) - 1)
        conf[r] = prob[at] / mass[-1]
    return {"token": None, "conf": conf, "kept": None}
