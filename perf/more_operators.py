"""The step of a paged decode service between its projections, as cases that can be timed and checked.

A service that keeps many sequences in one pool of pages does the same things in every iteration: it hands pages to the
tokens that are about to be computed and says at which position and place each lies (``dcl_pages_extend``), takes pages
back when drafts are rejected or sequences end (``dcl_pages_shrink``), normalises each head of the new queries and keys
and rotates them by their positions (``dcl_heads_norm_rope``), keeps keys and values in 4 bits with a scale for every 32
dimensions (``dcl_pages_write``, ``dcl_pages_read`` over pages of that type), and attends from the new tokens to those
pages (``dcl_pages_attention``).

With ``own`` false ``run`` computes the same from elementary torch operations in float32 (angles in float64). ``exact``
evaluates the definitions in float64.

Lengths are part of a case: they come from its own numbers, not from the seed of its inputs.
"""
import math
import random

import torch

own = False

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)          # magnitudes of the 4-bit codes 0 .. 7; code + 8 is negative


def listed():
    return [
        # one more token of each of 64 sequences, taken back again: the bookkeeping of a decode iteration, latency
        {"name": "turn 64x1", "op": "turn", "seqs": 64, "lo": 50, "hi": 4000, "most": 1, "page": 64, "free": 1.0, "pad": 0,
         "lens": 1},
        # prompts of very different lengths arrive for thousands of sequences, with too few pages left for the last ones
        {"name": "turn 3000 prompts", "op": "turn", "seqs": 3000, "lo": 1, "hi": 2000, "most": 600, "page": 16, "free": 0.8,
         "pad": 100, "lens": 2},
        # the new token of four sequences, far into their contexts, grouped heads: latency
        {"name": "heads 4 rows", "op": "heads", "rows": 4, "heads": 28, "kv_heads": 4, "dim": 128, "rot": 128, "far": 131072,
         "run": 1, "pad": 0, "lens": 3},
        # drafts of a batch, small heads whose first half turns, rows of padding at the end
        {"name": "heads 1531 partial", "op": "heads", "rows": 1531, "heads": 12, "kv_heads": 12, "dim": 64, "rot": 32,
         "far": 5000, "run": 32, "pad": 7, "lens": 4},
        # whole prompts
        {"name": "heads 8192 rows", "op": "heads", "rows": 8192, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "far": 1, "run": 2048, "pad": 0, "lens": 5},
        # the new token of each sequence of a batch into 4-bit pages, and out again as attention will see it: latency
        {"name": "store 48x1", "op": "store", "seqs": 48, "lo": 100, "hi": 2500, "new": 1, "kv_heads": 8, "dim": 128,
         "page": 64, "lens": 6},
        # whole prompts into 4-bit pages, and out again
        {"name": "store prompts", "op": "store", "seqs": 10, "lo": 400, "hi": 6000, "new": 0, "kv_heads": 32, "dim": 128,
         "page": 64, "lens": 7},
        # whole sequences back into rows, as when a sequence moves
        {"name": "read sequences", "op": "read", "seqs": 9, "lo": 300, "hi": 5000, "new": 0, "kv_heads": 8, "dim": 128,
         "page": 32, "lens": 8},
        # one token of four short sequences: latency
        {"name": "attend 4x1 short", "op": "attend", "seqs": 4, "lo": 80, "hi": 720, "new": 1, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 32, "causal": True, "lens": 9},
        # one token of a large ragged batch, grouped heads
        {"name": "attend 80x1", "op": "attend", "seqs": 80, "lo": 250, "hi": 9000, "new": 1, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "causal": True, "lens": 10},
        # one token of two very long sequences
        {"name": "attend 2x1 long", "op": "attend", "seqs": 2, "lo": 100000, "hi": 131072, "new": 1, "heads": 28,
         "kv_heads": 4, "dim": 128, "page": 64, "causal": True, "lens": 11},
        # a denoising block: eight sequences' 64 tokens over about 1200 cached ones, every token sees every other
        {"name": "attend 8x64 block", "op": "attend", "seqs": 8, "lo": 1248, "hi": 1280, "new": 64, "heads": 32,
         "kv_heads": 32, "dim": 128, "page": 64, "causal": False, "lens": 12},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["turn", "heads", "heads", "store", "read", "attend", "attend", "attend"])
    lens = rng.randrange(1 << 30)
    if op == "turn":
        most = _log(rng, 1, 600)
        seqs = _log(rng, 1, 3000)
        return {"op": op, "seqs": seqs, "lo": 1, "hi": _log(rng, 1, 2000), "most": most,
                "page": rng.choice([16, 32, 64, 128]), "free": rng.choice([1.0, 1.0, 0.7]),
                "pad": rng.choice([0, 0, 9]), "lens": lens}
    kv = rng.choice([1, 2, 4, 8, 32])
    heads = kv * rng.choice([1, 1, 2, 4, 7]) if kv < 32 else 32
    dim = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if op == "heads":
        rows = _log(rng, 1, 8192 * 40 * 128 // ((heads + kv) * dim))
        return {"op": op, "rows": rows, "heads": heads, "kv_heads": kv, "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2, 16]), "far": _log(rng, 1, 200000), "run": _log(rng, 1, 2048),
                "pad": min(rng.choice([0, 0, 5]), rows // 2), "lens": lens}
    # tokens of all sequences together: at most those of the largest listed case
    total = ((1 << 27) - (1 << 23) if op == "attend" else (1 << 26) - (1 << 22)) // (kv * dim)
    hi = min(_log(rng, 20, 100000 if op == "attend" else 20000), total)
    seqs = max(1, min(_log(rng, 1, 128), total // hi))
    lo = max(1, hi // rng.choice([1, 3, 20]))
    c = {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "new": 0, "kv_heads": kv, "dim": dim, "page": page, "lens": lens}
    if op == "attend":
        most = max(1, min(64, lo, (1 << 24) // (seqs * heads * hi)))
        c["new"] = rng.choice([1, 1, rng.randint(1, most)])
        c["heads"] = heads
        c["causal"] = rng.random() < 0.6
    elif op == "store":
        c["new"] = rng.choice([0, 1, min(lo, rng.randint(1, 300))])
    return c


def _lengths(case):
    """The sequences' lengths: log-uniform over [lo, hi], the first one hi."""
    r = random.Random(case["lens"])
    return [case["hi"]] + [_log(r, case["lo"], case["hi"]) for _ in range(case["seqs"] - 1)]


def _new(case):
    """How many tokens of each sequence the call takes: `new`, or with 0 the whole sequence."""
    return [min(case["new"], n) if case["new"] else n for n in _lengths(case)]


def _counts(case):
    """How many tokens each sequence of a turn asks room for, 1 to `most`, here and there none."""
    r = random.Random(case["lens"] + 1)
    return [0 if case["most"] > 1 and r.random() < 0.05 else _log(r, 1, case["most"]) for _ in range(case["seqs"])]


def _grant(case):
    """For a turn: tokens granted to each sequence, from the lists themselves, and the pages they take."""
    page, left, got, took = case["page"], _free(case), [], 0
    short = False
    for n, c in zip(_lengths(case), _counts(case)):
        need = -(-(n + c) // page) - -(-n // page)
        short = short or need > left                      # whoever comes after one that does not fit gets no page either
        if need and short:
            got.append(0)
            continue
        got.append(c)
        left -= need
        took += need
    return got, took


def _free(case):
    page = case["page"]
    want = sum(-(-(n + c) // page) - -(-n // page) for n, c in zip(_lengths(case), _counts(case)))
    return int(want * case["free"])


def work(case):
    op = case["op"]
    if op == "turn":
        got, took = _grant(case)
        # lengths and counts in, borders and lengths out; a position and a place a row; a page from the list into the table;
        # and the pages back with the lengths to keep
        return {"bytes": 16 * case["seqs"] + 12 * (sum(_counts(case)) + case["pad"]) + 16 * took + 12 * case["seqs"],
                "flops": 0}
    d = case["dim"]
    if op == "heads":
        h = case["heads"] + case["kv_heads"]
        return {"bytes": case["rows"] * (4 * h * d + 4) + 8 * d, "flops": 8 * case["rows"] * h * d}
    n, m = _lengths(case), _new(case)
    per = 2 * case["kv_heads"] * (d // 2 + d // 32)                       # one token in the pages
    if op == "attend":
        h = case["heads"]
        pairs = sum(b * a - (b * (b - 1) // 2 if case["causal"] else 0) for a, b in zip(n, m))
        return {"bytes": per * sum(n) + 4 * sum(m) * h * d + 4 * sum(m) * h, "flops": 4 * d * h * pairs}
    rows = sum(m) * 4 * case["kv_heads"] * d
    return {"bytes": rows + per * sum(m) + (rows + per * sum(m) if op == "store" else 0), "flops": 0}


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"turn": _prepare_turn, "heads": _prepare_heads}.get(case["op"], _prepare_pages)(case, g)


def _deal(need, width, spare, g):
    """A table whose rows hold need[b] pages, handed out in no order, -1 behind them; and the pages that nobody has."""
    pool = sum(need) + spare
    order = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
    at = _starts(need)
    slot = torch.arange(width, device="cuda")[None, :]
    have, start = _ints(need)[:, None], _ints(at[:-1])[:, None]
    table = torch.where(slot < have, order[(start + slot).clamp(max=pool - 1).long()], -1).to(torch.int32)
    return table, order[at[-1]:], pool


def _prepare_turn(case, g):
    n, c, page = _lengths(case), _counts(case), case["page"]
    width = max(-(-(a + b) // page) for a, b in zip(n, c)) + 2
    free = _free(case)
    table, rest, pool = _deal([-(-x // page) for x in n], width, free + 5, g)
    t = sum(c) + case["pad"]
    stack = torch.full((pool,), -1, dtype=torch.int32, device="cuda")     # of the pages nobody has, `free` are on the list
    stack[:free] = rest[:free]
    return {"case": case, "T": t, "table": table, "width": width, "n_pages": pool, "len": _ints(n), "keep": _ints(n),
            "count": _ints(c), "free": stack, "n_free": _ints([free]), "cu": _ints([0] * (len(n) + 1)),
            "pos": torch.zeros(t, dtype=torch.int32, device="cuda"), "slot": torch.zeros(t, dtype=torch.int64, device="cuda"),
            "handle": None}


def _positions(case):
    """Runs of consecutive positions, each from a start of its own below `far`; -1 for the rows of padding."""
    r, out = random.Random(case["lens"]), []
    while len(out) < case["rows"] - case["pad"]:
        at = r.randrange(case["far"])
        out += range(at, at + r.randint(1, case["run"]))
    return out[:case["rows"] - case["pad"]] + [-1] * case["pad"]


def _prepare_heads(case, g):
    t, h, hkv, d = case["rows"], case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    # one projection's rows: queries, keys and values side by side; heads and a few dimensions of larger size
    row = normal(t, h + 2 * hkv, d) * torch.exp(0.7 * normal(1, h + 2 * hkv, 1)) * torch.exp(0.7 * normal(1, 1, d))
    row = row.to(torch.bfloat16)
    return {"case": case, "q": row[:, :h], "k": row[:, h:h + hkv], "pos": _ints(_positions(case)),
            "g_q": 1.0 + 0.3 * normal(d), "g_k": 1.0 + 0.3 * normal(d), "eps": 1e-6, "base": 1e6,
            "q_out": torch.zeros((t, h, d), dtype=torch.bfloat16, device="cuda"),
            "k_out": torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda"), "handle": None}


def _prepare_pages(case, g):
    def normal(*shape, std=1.0):
        return (torch.randn(shape, device="cuda", generator=g) * std).to(torch.bfloat16)

    def some(lo, hi, *shape):
        return torch.randint(lo, hi, shape, device="cuda", generator=g, dtype=torch.uint8)

    n, m, d, page, hkv = _lengths(case), _new(case), case["dim"], case["page"], case["kv_heads"]
    need = [-(-x // page) for x in n]
    table, _, pool = _deal(need, max(need), 3, g)
    t = sum(m)
    s = {"case": case, "scale": 1.0 / math.sqrt(d), "T": t, "most": max(m), "cu": _ints(_starts(m)), "len": _ints(n),
         "table": table, "width": max(need), "n_pages": pool, "handle": None}
    # any byte is two values that a page may hold; scales near those of activations
    s.update(k_pages=some(0, 256, pool, hkv, page, d // 2), v_pages=some(0, 256, pool, hkv, d // 2, page),
             k_scale=some(124, 127, pool, hkv, d // 32, page), v_scale=some(124, 127, pool, hkv, d // 32, page))
    if case["op"] == "attend":
        h = case["heads"]
        s.update(q=normal(t, h, d, std=1.5), out=torch.zeros((t, h, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((t, h), device="cuda"))
        return s
    if case["op"] == "store":
        # keys after the rotation have a few large dimensions; heads differ in size
        size = torch.exp(torch.randn((1, hkv, d), device="cuda", generator=g))
        s.update(k=(normal(t, hkv, d) * size).to(torch.bfloat16), v=normal(t, hkv, d))
    s.update(k_rows=torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda"),
             v_rows=torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda"))
    return s


def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


# ---------------------------------------------------------------- the framework's calls

def _handle(s):
    """The pool's description and the call's workspace, made at the first call and kept, as a program keeps them."""
    if s["handle"] is None:
        import paper_2607_20467_amd as dcl
        c, pool, need = s["case"], None, 0
        if c["op"] == "turn":
            pool = dcl.KVPages(s["n_pages"], c["page"], 1, 64, dcl.DCL_DTYPE_E2M1)
            need = dcl.dcl_pages_turn_workspace_bytes(c["seqs"])
        elif c["op"] != "heads":
            pool = dcl.KVPages(s["n_pages"], c["page"], c["kv_heads"], c["dim"], dcl.DCL_DTYPE_E2M1, k=s["k_pages"],
                               v=s["v_pages"], k_scale=s["k_scale"], v_scale=s["v_scale"])
            if c["op"] == "attend":
                need = dcl.dcl_pages_attention_workspace_bytes(pool, c["heads"], c["seqs"], s["T"], s["most"], s["width"])
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        s["handle"] = (dcl, pool, ws, need)
    return s["handle"]


def _turned(s):
    return {k: s[k] for k in ("table", "len", "cu", "pos", "slot", "free", "n_free")}


def _own_turn(s):
    (dcl, pool, ws, need), c = _handle(s), s["case"]
    dcl.dcl_pages_extend(pool, s["table"], s["len"], s["count"], c["seqs"], s["T"], s["free"], s["n_free"], s["cu"],
                         s["pos"], s["slot"], ws, need)
    dcl.dcl_pages_shrink(pool, s["table"], s["len"], s["keep"], c["seqs"], s["free"], s["n_free"], ws, need)
    return _turned(s)


def _own_heads(s):
    dcl, c = _handle(s)[0], s["case"]
    dcl.dcl_heads_norm_rope(s["q"], s["k"], s["pos"], c["rows"], c["heads"], c["kv_heads"], c["dim"], s["g_q"], s["g_k"],
                            s["eps"], s["base"], c["rot"], s["q_out"], s["k_out"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_store(s):
    (dcl, pool, _, _), c = _handle(s), s["case"]
    dcl.dcl_pages_write(pool, s["table"], s["len"], s["cu"], c["seqs"], s["T"], s["most"], s["k"], s["v"])
    dcl.dcl_pages_read(pool, s["table"], s["len"], s["cu"], c["seqs"], s["T"], s["most"], s["k_rows"], s["v_rows"])
    return {"k": s["k_rows"], "v": s["v_rows"]}


def _own_read(s):
    (dcl, pool, _, _), c = _handle(s), s["case"]
    dcl.dcl_pages_read(pool, s["table"], s["len"], s["cu"], c["seqs"], s["T"], s["most"], s["k_rows"], s["v_rows"])
    return {"k": s["k_rows"], "v": s["v_rows"]}


def _own_attend(s):
    (dcl, pool, ws, need), c = _handle(s), s["case"]
    dcl.dcl_pages_attention(pool, s["table"], s["len"], s["cu"], c["seqs"], s["T"], s["most"], s["q"], c["heads"],
                            s["scale"], c["causal"], s["out"], s["lse"], ws, need)
    return {"out": s["out"], "lse": s["lse"]}


_own = {"turn": _own_turn, "heads": _own_heads, "store": _own_store, "read": _own_read, "attend": _own_attend}


# ---------------------------------------------------------------- the plain forms

def _pages_of(n, page):
    return torch.div(n + page - 1, page, rounding_mode="floor")


def _plain_turn(s):
    _plain_extend(s)
    _plain_shrink(s)
    return _turned(s)


def _plain_extend(s):
    """Tokens in order of the sequences, each sequence's all or none: within its row of the table, within the T rows, and
    its new pages among those that are left."""
    page, t = s["case"]["page"], s["T"]
    n, c = s["len"].long(), s["count"].long()
    ok = (n >= 0) & (c >= 0) & (n + c <= s["width"] * page)
    ok &= torch.cumsum(torch.where(ok, c, 0), 0) <= t
    have = _pages_of(n, page)
    need = torch.where(ok, _pages_of(n + c, page) - have, 0)
    upto = torch.cumsum(need, 0)
    ok &= (need == 0) | (upto <= s["n_free"].long())
    c, need, before = torch.where(ok, c, 0), torch.where(ok, need, 0), upto - need
    s["cu"][1:] = torch.cumsum(c, 0)
    s["len"].add_(c.to(torch.int32))
    # rows: their sequence, position, page (of those just taken, or of before), place
    at = torch.arange(t, device="cuda")
    b = torch.bucketize(at, s["cu"][1:].long(), right=True)
    real = b < len(n)
    b = b.clamp(max=len(n) - 1)
    x = n[b] + at - s["cu"][b].long()
    j = torch.div(x, page, rounding_mode="floor").clamp(0, s["width"] - 1)
    new = real & (j >= have[b])
    taken = s["free"][(s["n_free"].long() - 1 - before[b] - (j - have[b])).clamp(0, s["n_pages"] - 1)]
    of = torch.where(new, taken, s["table"][b, j])
    s["pos"].copy_(torch.where(real, x, -1))
    s["slot"].copy_(torch.where(real & (of >= 0) & (of < s["n_pages"]), of.long() * page + x % page, -1))
    s["table"][b[new], j[new]] = of[new]
    s["n_free"].sub_(need.sum().to(torch.int32))


def _plain_shrink(s):
    """Pages behind the kept lengths go back on the list, the last one first."""
    page = s["case"]["page"]
    n, keep = s["len"].long(), s["keep"].long()
    cut = (keep >= 0) & (keep < n) & (n <= s["width"] * page)
    j = torch.arange(s["width"], device="cuda")[None, :]
    gone = cut[:, None] & (j >= _pages_of(keep, page)[:, None]) & (j < _pages_of(n, page)[:, None])
    back = s["table"][gone]
    back = back[(back >= 0) & (back < s["n_pages"])].flip(0)
    s["table"].masked_fill_(gone, -1)
    at = s["n_free"].long() + torch.arange(len(back), device="cuda")
    fits = at < s["n_pages"]
    s["free"][at[fits]] = back[fits]
    s["n_free"].add_(fits.sum().to(torch.int32))
    s["len"].copy_(torch.where(cut, keep, n))


def _plain_heads(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    angle = s["pos"].double()[:, None] * torch.exp(i * (-2.0 / rot * math.log(s["base"])))
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    real = (s["pos"] >= 0)[:, None, None]
    for x, gain, out in ((s["q"], s["g_q"], s["q_out"]), (s["k"], s["g_k"], s["k_out"])):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * gain
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1).to(torch.bfloat16)
        out.copy_(torch.where(real, y, out))
    return {"q": s["q_out"], "k": s["k_out"]}


def _pow2(n):
    """2^n for whole numbers n in float64, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _new_rows(s):
    """For new token i of sequence b, [B, most]: its packed row (clamped), its position, and whether there is one."""
    i = torch.arange(s["most"], device="cuda")[None, :]
    count = (s["cu"][1:] - s["cu"][:-1])[:, None]
    row = (s["cu"][:-1][:, None] + i).clamp(max=s["T"] - 1)
    return row.long(), s["len"][:, None] - count + i, i < count


def _slots(s):
    """Page and offset of every row of the call."""
    c = s["case"]
    row, pos, is_new = _new_rows(s)
    page = s["table"].long().gather(1, (pos // c["page"]).clamp(min=0).long())
    return page[is_new], (pos % c["page"]).long()[is_new], row[is_new]


def _codes(x):
    """Codes [T, Hkv, dh] (whole numbers 0 .. 15) and scale exponents [T, Hkv, dh / 32] of rows x [T, Hkv, dh]: the scale
    of 32 dimensions is the least power of two with the largest magnitude at most 6 times it; values to the nearest, ties to
    the even code."""
    x = x.float().unflatten(-1, (-1, 32))
    frac, exp = torch.frexp(x.abs().amax(-1))                     # frac in [0.5, 1); 6 = 0.75 * 2^3
    e = torch.where(frac == 0, 1, (exp - 3 + (frac > 0.75).to(exp.dtype) + 127).clamp(1, 254))
    y = (x * _pow2(127 - e)[..., None]).float().flatten(-2)
    m, code = y.abs(), torch.signbit(y).to(torch.uint8) << 3
    for mid, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (m >= mid) if up else (m > mid)
    return code, e.to(torch.uint8)


def _plain_write(s):
    page, off, row = _slots(s)
    (k, ke), (v, ve) = _codes(s["k"][row]), _codes(s["v"][row])
    v = v.unflatten(-1, (-1, 2, 16))                              # dimensions 16 apart share a byte
    s["k_pages"][page, :, off] = k[..., 0::2] | k[..., 1::2] << 4
    s["v_pages"][page, :, :, off] = (v[..., 0, :] | v[..., 1, :] << 4).flatten(-2)
    s["k_scale"][page, :, :, off] = ke
    s["v_scale"][page, :, :, off] = ve


def _values(byte, e):
    """Low and high codes' values of bytes under scale exponents e."""
    mag = torch.tensor(VALUES + tuple(-x for x in VALUES), device="cuda")
    f = _pow2(e.long() - 127).float()
    return mag[(byte & 15).int()] * f, mag[(byte >> 4).int()] * f


def _key_rows(byte, e):
    """Bytes [..., dh / 2] and exponents [..., dh / 32] to float32 [..., dh]."""
    lo, hi = _values(byte, e.repeat_interleave(16, -1))
    return torch.stack([lo, hi], -1).flatten(-2)


def _value_rows(byte, e):
    lo, hi = _values(byte, e.repeat_interleave(16, -1))
    return torch.stack([lo.unflatten(-1, (-1, 16)), hi.unflatten(-1, (-1, 16))], -2).flatten(-3)


def _plain_read(s):
    page, off, row = _slots(s)
    s["k_rows"][row] = _key_rows(s["k_pages"][page, :, off], s["k_scale"][page, :, :, off]).to(torch.bfloat16)
    s["v_rows"][row] = _value_rows(s["v_pages"][page, :, :, off], s["v_scale"][page, :, :, off]).to(torch.bfloat16)
    return {"k": s["k_rows"], "v": s["v_rows"]}


def _plain_store(s):
    _plain_write(s)
    return _plain_read(s)


def _plain_attend(s):
    c = s["case"]
    b, h, hkv, d, most = c["seqs"], c["heads"], c["kv_heads"], c["dim"], s["most"]
    g, page = h // hkv, c["page"]
    row, pos, is_new = _new_rows(s)
    q = s["q"].float()[row] * s["scale"]                          # [B, most, H, dh]
    q = q.view(b, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, most * g, d)
    out = torch.zeros((b, hkv, most * g, d), device="cuda")
    lse = torch.zeros((b, hkv, most * g), device="cuda")
    for i in range(b):                                            # a sequence at a time: its keys in float32 are eight times its pages
        held = s["table"][i] >= 0
        tab = s["table"][i].long().clamp(min=0)
        k = _key_rows(s["k_pages"][tab], s["k_scale"][tab].transpose(2, 3)).transpose(0, 1).reshape(hkv, -1, d)
        v = _value_rows(s["v_pages"][tab].transpose(2, 3), s["v_scale"][tab].transpose(2, 3)).transpose(0, 1).reshape(hkv, -1, d)
        j = torch.arange(k.shape[1], device="cuda")
        ok = (j < s["len"][i]) & held.repeat_interleave(page)
        ok = ok[None, :] & (j[None, :] <= pos[i][:, None]) if c["causal"] else ok[None, :].expand(most, -1)
        x = torch.matmul(q[i], k.transpose(1, 2).contiguous()).masked_fill_(~ok.repeat_interleave(g, 0)[None], -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        lse[i] = (top + torch.log(total)).squeeze(-1)
        out[i] = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(b, hkv, most, g, d).permute(0, 2, 1, 3, 4).reshape(b, most, h, d)
    lse = lse.view(b, hkv, most, g).permute(0, 2, 1, 3).reshape(b, most, h)
    s["out"][row[is_new]] = out[is_new].to(torch.bfloat16)
    s["lse"][row[is_new]] = lse[is_new]
    return {"out": s["out"], "lse": s["lse"]}


_plain = {"turn": _plain_turn, "heads": _plain_heads, "store": _plain_store, "read": _plain_read, "attend": _plain_attend}


# ---------------------------------------------------------------- the definitions in float64

def exact(case, seed):
    s = prepare(case, seed)
    return {"turn": _exact_turn, "heads": _exact_heads, "store": _exact_store, "read": _exact_read,
            "attend": _exact_attend}[case["op"]](s)


def _exact_turn(s):
    """Sequence by sequence, token by token."""
    c = s["case"]
    page, table, free = c["page"], s["table"].tolist(), s["free"].tolist()
    left = int(s["n_free"])
    cu, pos, slot = [0], [], []
    for b, (n, m) in enumerate(zip(_lengths(c), _grant(c)[0])):
        for x in range(n, n + m):
            if x % page == 0:
                left -= 1
                table[b][x // page] = free[left]
            pos.append(x)
            slot.append(table[b][x // page] * page + x % page)
        cu.append(len(pos))
    gap = [-1] * (s["T"] - len(pos))
    # what was taken goes back where it came from: table, lengths and list end as they began
    return {"table": s["table"], "len": s["len"], "cu": _ints(cu), "pos": _ints(pos + gap),
            "slot": torch.tensor(slot + gap, dtype=torch.int64, device="cuda"), "free": s["free"], "n_free": s["n_free"]}


def _exact_heads(s):
    c = s["case"]
    half, res = c["rot"] // 2, {}
    for name, gain in (("q", s["g_q"]), ("k", s["g_k"])):
        x = s[name].double()
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["dim"] + s["eps"]) * gain.double()
        y = x.clone()
        for i in range(half):
            a = s["pos"].double() / s["base"] ** (2 * i / c["rot"])
            co, si = torch.cos(a)[:, None], torch.sin(a)[:, None]
            y[:, :, i] = x[:, :, i] * co - x[:, :, i + half] * si
            y[:, :, i + half] = x[:, :, i] * si + x[:, :, i + half] * co
        res[name] = torch.where((s["pos"] >= 0)[:, None, None], y, 0.0)
    return res


def _exact_quantised(x):
    """Rows x [T, Hkv, dh] as the nearest values that 4 bits and their scales stand for, ties to even."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    e = torch.ceil(torch.log2(top / 6.0))                         # the least with top <= 6 * 2^e, but for rounding
    e = torch.where(top > 6.0 * _pow2(e), e + 1, torch.where(top <= 6.0 * _pow2(e - 1), e - 1, e))
    z = y / _pow2(e)[..., None]
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0)).double()
    return (torch.round(z / step) * step * _pow2(e)[..., None]).flatten(-2)


def _exact_store(s):
    return {"k": _exact_quantised(s["k"]), "v": _exact_quantised(s["v"])}


def _exact_rows(s, b, n):
    """Keys and values [Hkv, n, dh] of sequence b in float64, dimension by dimension."""
    c = s["case"]
    pages = s["table"][b, :-(-n // c["page"])].long()
    mag = torch.tensor([(-1) ** (x >> 3) * VALUES[x & 7] for x in range(16)], dtype=torch.float64, device="cuda")
    kb, vb = (s[x][pages].transpose(0, 1) for x in ("k_pages", "v_pages"))
    ks, vs = (_pow2(s[x][pages].transpose(0, 1).long() - 127) for x in ("k_scale", "v_scale"))
    k = torch.empty((c["kv_heads"], len(pages), c["page"], c["dim"]), dtype=torch.float64, device="cuda")
    v = torch.empty_like(k)
    for d in range(c["dim"]):
        k[..., d] = mag[((kb[..., d // 2] >> (4 * (d % 2))) & 15).long()] * ks[:, :, d // 32]
        v[..., d] = mag[((vb[:, :, d // 32 * 16 + d % 16] >> (d % 32 // 16 * 4)) & 15).long()] * vs[:, :, d // 32]
    return k.flatten(1, 2)[:, :n], v.flatten(1, 2)[:, :n]


def _exact_read(s):
    rows = [_exact_rows(s, b, n) for b, n in enumerate(_lengths(s["case"]))]
    k, v = (torch.cat([r[i].transpose(0, 1) for r in rows]) for i in (0, 1))
    return {"k": k, "v": v}


def _exact_attend(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    g, at = c["heads"] // c["kv_heads"], 0
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        k, v = _exact_rows(s, b, n)
        lim = torch.arange(n - m + 1, n + 1, device="cuda") if c["causal"] else torch.full((m,), n, device="cuda")
        dead = torch.arange(n, device="cuda")[None, :] >= lim[:, None]
        for h in range(c["heads"]):
            x = (s["q"][at:at + m, h].double() @ k[h // g].T) * s["scale"]
            total = torch.logsumexp(x.masked_fill(dead, -math.inf), 1)
            p = torch.exp(x - total[:, None]).masked_fill(dead, 0.0)
            out[at:at + m, h], lse[at:at + m, h] = p @ v[h // g], total
        at += m
    return {"out": out, "lse": lse}
