"""The serving operators together, as a decode loop uses them: prompts of different lengths attended to and written to
pages, blocks of new tokens over them, pages read back; the model's head drawn from, and the drawn tokens committed."""
import math

import numpy as np
import pytest
import torch

import synth

from helpers import runner_for, to_dev
from serving_reference import Pool, attention_rows, sample_row, starts
from test_gpu_step import CASES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dcl():
    import paper_2607_20467_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_then_blocks_over_pages(dcl, e4m3):
    heads, hkv, dh, page, scale = 8, 2, 64, 32, 0.125
    g = torch.Generator().manual_seed(3)
    prompts, blocks = [70, 5, 33], [[4, 4, 4], [1, 1, 1], [32, 1, 16]]
    final = [p + sum(b[i] for b in blocks) for i, p in enumerate(prompts)]
    pool = Pool(dcl, final, page, hkv, dh, e4m3, seed=4, fill=0x7F)
    dev, table = pool.device(), pool.table.cuda()
    K = [torch.randn(n, hkv, dh, generator=g).to(torch.bfloat16) for n in final]
    V = [torch.randn(n, hkv, dh, generator=g).to(torch.bfloat16) for n in final]
    Q = [torch.randn(n, heads, dh, generator=g).to(torch.bfloat16) for n in final]

    def packed(x, lo, n):
        return torch.cat([a[s:s + c] for a, s, c in zip(x, lo, n)]).cuda()
    done = [0, 0, 0]
    outs = [torch.zeros(n, heads, dh) for n in final]
    for step, new in enumerate([prompts] + blocks):
        T, most = sum(new), max(new)
        q, k, v, cu = packed(Q, done, new), packed(K, done, new), packed(V, done, new), starts(new).cuda()
        done = [a + b for a, b in zip(done, new)]
        ln = torch.tensor(done, dtype=torch.int32, device="cuda")
        out = torch.empty(T, heads, dh, dtype=torch.bfloat16, device="cuda")
        dcl.dcl_pages_write(dev, table, ln, cu, 3, T, most, k, v)
        if step == 0:
            dcl.dcl_prompt_attention(q, k, v, cu, 3, T, most, heads, hkv, dh, scale, True, out)
        else:
            need = dcl.dcl_pages_attention_workspace_bytes(dev, heads, 3, T, most, pool.width)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            dcl.dcl_pages_attention(dev, table, ln, cu, 3, T, most, q, heads, scale, True, out, None, ws, need)
        o, at = out.float().cpu(), 0
        for b, n in enumerate(new):
            outs[b][done[b] - n:done[b]] = o[at:at + n]
            at += n
    cu, T = starts(final).cuda(), sum(final)
    rk = torch.empty(T, hkv, dh, dtype=torch.bfloat16, device="cuda")
    rv = torch.empty_like(rk)
    dcl.dcl_pages_read(dev, table, torch.tensor(final, dtype=torch.int32, device="cuda"), cu, 3, T, max(final), rk, rv)
    rk, rv = rk.cpu().double(), rv.cpu().double()
    for b, n in enumerate(final):
        lo = int(cu[b])
        kd, vd = rk[lo:lo + n], rv[lo:lo + n]
        if not e4m3:
            assert torch.equal(kd, K[b].double()) and torch.equal(vd, V[b].double())
        else:                                            # four significant bits, and steps of 2^-9 of a scale
            amax = K[b].double().abs().amax(-1, keepdim=True)
            assert bool(((kd - K[b].double()).abs() <= K[b].double().abs() * 2.0 ** -4 + amax * 2.0 ** -17).all())
        sees = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(heads):
            # a prompt's rows saw its own rows, the later ones what the pages hold
            P = prompts[b]
            for rows, kk, vv in ((slice(0, P), K[b].double(), V[b].double()), (slice(P, n), kd, vd)):
                o, _, eo, _ = attention_rows(Q[b][rows, h].double(), kk[:, h // 4], vv[:, h // 4], scale, sees[rows])
                assert bool(((outs[b][rows, h].double() - o).abs() <= eo).all()), (b, h)


def test_one_block_is_the_same_over_pages_and_packed(dcl):
    """A whole sequence as the new tokens of its pages, against the packed call: both within their bounds of float64,
    so within the sum of them of each other; bidirectional and causal."""
    heads, hkv, dh = 4, 4, 128
    lens = [40, 64, 9]
    pool = Pool(dcl, lens, 16, hkv, dh, False, seed=6)
    g = torch.Generator().manual_seed(7)
    T = sum(lens)
    q = torch.randn(T, heads, dh, generator=g).to(torch.bfloat16).cuda()
    dev, cu = pool.device(), starts(lens).cuda()
    k, v = torch.empty(T, hkv, dh, dtype=torch.bfloat16, device="cuda"), torch.empty(T, hkv, dh, dtype=torch.bfloat16,
                                                                                     device="cuda")
    a = (dev, pool.table.cuda(), pool.len.cuda(), cu, 3, T, 64)
    dcl.dcl_pages_read(*a, k, v)
    for causal in (False, True):
        one, two = torch.empty_like(q), torch.empty_like(q)
        l1, l2 = torch.empty(T, heads, device="cuda"), torch.empty(T, heads, device="cuda")
        dcl.dcl_prompt_attention(q, k, v, cu, 3, T, 64, heads, hkv, dh, 0.09, causal, one, l1)
        need = dcl.dcl_pages_attention_workspace_bytes(dev, heads, 3, T, 64, pool.width)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        dcl.dcl_pages_attention(*a, q, heads, 0.09, causal, two, l2, ws, need)
        big = v.double().abs().max()
        assert float((one.double() - two.double()).abs().max()) <= 4 * 2.0 ** -8 * float(big)
        assert float((l1 - l2).abs().max()) <= 1e-4


def test_sampling_the_models_head_and_committing(dcl):
    """dcl_sample_hidden is the head's logits drawn from; its tokens and shares commit as a step's top-1 would."""
    w = CASES["c1s"]
    g = w.geom
    run = runner_for(w, synth.make_weights(g))
    tok_h, p_h = synth.initial_state(w)
    B, S = tok_h.shape
    tok, p = to_dev(tok_h), to_dev(p_h)
    st = run.step(tok, p, w.gen_end)
    scored = (st["top1"].view(-1) >= 0).nonzero()[:, 0].to(torch.int32)
    logits, hid = run.logits(tok, scored, with_hidden=True)
    n = scored.numel()
    gen = torch.Generator().manual_seed(1)
    u = torch.rand(n, generator=gen).cuda()
    temp, top_p = torch.full((n,), 0.8, device="cuda"), torch.full((n,), 0.9, device="cuda")
    r = run.sample_hidden(hid, u, temperature=temp, top_p=top_p)
    ws = torch.empty(dcl.dcl_sample_workspace_bytes(n, g.vocab), dtype=torch.uint8, device="cuda")
    token, conf = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    dcl.dcl_sample_tokens(logits, n, g.vocab, temp, None, top_p, None, u, token, conf, None, ws, ws.numel())
    assert torch.equal(r["token"], token) and torch.equal(r["conf"], conf)
    x, f = logits.double().cpu().numpy(), np.float32
    for i in range(0, n, 7):
        t, c, kept = sample_row(x[i], float(f(0.8)), 0, float(f(0.9)), 0.0, float(u[i]))
        assert (int(token[i]), int(r["kept"][i])) == (t, kept) and math.isclose(float(conf[i]), c, rel_tol=1e-6)
    best = run.sample_hidden(hid, u, temperature=torch.zeros(n, device="cuda"))
    assert torch.equal(best["token"], st["top1"].view(-1)[scored.long()])
    st["top1"].view(-1)[scored.long()] = token
    st["conf"].view(-1)[scored.long()] = conf
    k_eff = torch.zeros(B, dtype=torch.int32, device="cuda")
    dcl.dcl_select_contiguous(tok, B, S, p, w.gen_end, w.window, 0.2, 2.0, g.mask_id, st, None, k_eff)
    drawn = np.full(B * S, -1)
    drawn[scored.cpu().numpy()] = token.cpu().numpy()
    now, ke = tok.cpu().numpy(), k_eff.cpu().numpy()
    for b in range(B):
        lo = int(p_h[b])
        assert ke[b] >= 1 and (now[b, lo:lo + ke[b]] == drawn.reshape(B, S)[b, lo:lo + ke[b]]).all()
        assert int(p[b]) == lo + ke[b]


def test_a_captured_iteration_of_all_of_them(dcl):
    """Two graphs, each with its own workspaces, of write, attention and sampling; replayed in turn."""
    pool = Pool(dcl, [300, 40], 64, 2, 128, True, seed=8)
    dev, table, ln, cu = pool.device(), pool.table.cuda(), pool.len.cuda(), starts([1, 1]).cuda()
    g = torch.Generator().manual_seed(2)
    W = torch.randn(8 * 128, 500, generator=g).cuda() * 0.1
    state = []
    for _ in range(2):
        need = dcl.dcl_pages_attention_workspace_bytes(dev, 8, 2, 2, 1, pool.width)
        ns = dcl.dcl_sample_workspace_bytes(2, 500)
        state.append(dict(
            q=torch.randn(2, 8, 128, generator=g).to(torch.bfloat16).cuda(), u=torch.rand(2, generator=g).cuda(),
            k=torch.randn(2, 2, 128, generator=g).to(torch.bfloat16).cuda(), out=torch.empty(2, 8, 128, dtype=torch.bfloat16,
                                                                                             device="cuda"),
            x=torch.empty(2, 500, device="cuda"), tok=torch.empty(2, dtype=torch.int32, device="cuda"),
            conf=torch.empty(2, device="cuda"), ws=torch.empty(need, dtype=torch.uint8, device="cuda"), need=need,
            ws2=torch.empty(ns, dtype=torch.uint8, device="cuda"), ns=ns))

    def step(s):
        dcl.dcl_pages_write(dev, table, ln, cu, 2, 2, 1, s["k"], s["k"])
        dcl.dcl_pages_attention(dev, table, ln, cu, 2, 2, 1, s["q"], 8, 0.09, True, s["out"], None, s["ws"], s["need"])
        torch.mul(s["out"].float().view(2, -1)[:, :500], W[0], out=s["x"])
        dcl.dcl_sample_tokens(s["x"], 2, 500, None, None, None, None, s["u"], s["tok"], s["conf"], None, s["ws2"], s["ns"])
    want = []
    for s in state:
        step(s)
        torch.cuda.synchronize()
        want.append([s[n].clone() for n in ("out", "tok", "conf")])
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for s in state:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            step(s)
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1, 0):
        for n in ("out", "tok", "conf"):
            state[i][n].fill_(3)
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(state[i][n], w) for n, w in zip(("out", "tok", "conf"), want[i]))


def test_drawing_on_another_stream_than_the_current_one(dcl):
    """The call's buffers belong to its stream: what the current stream allocates and fills beside it touches none of them."""
    w = CASES["c1s"]
    g = w.geom
    run = runner_for(w, synth.make_weights(g))
    n, gen = 64, torch.Generator().manual_seed(5)
    hid = torch.randn(n, g.d_model, generator=gen).to(torch.bfloat16).cuda()
    u = torch.rand(n, generator=gen).cuda()
    want = run.sample_hidden(hid, u)
    scored = run.score_hidden(hid)
    need = dcl.dcl_sample_hidden_workspace_bytes(run.model, n)
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            for _ in range(20):
                torch.mm(busy, busy)                     # the call waits behind these
        got = run.sample_hidden(hid, u, stream=stream)
        again = run.score_hidden(hid, stream=stream)
        for size in (need, n * 4, n * 4, n * 4, dcl.dcl_score_workspace_bytes(run.model, n)):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)
        assert all(torch.equal(again[k], scored[k]) for k in scored)


def test_a_greedy_rows_conf_is_its_share_of_what_is_kept(dcl):
    """conf 1 passes every threshold below 1, so that a window of greedy rows commits as a whole; with the confidences that
    dcl_score_hidden gives for the same rows the drawn tokens commit as the step's own do."""
    w = CASES["c1s"]
    g = w.geom
    run = runner_for(w, synth.make_weights(g))
    tok_h, p_h = synth.initial_state(w)
    B, S = tok_h.shape
    st = run.step(to_dev(tok_h), to_dev(p_h), w.gen_end)
    scored = (st["top1"].view(-1) >= 0).nonzero()[:, 0].to(torch.int32)
    _, hid = run.logits(to_dev(tok_h), scored, with_hidden=True)
    n, at = scored.numel(), scored.long()
    u = torch.rand(n, generator=torch.Generator().manual_seed(3)).cuda()
    drawn = run.sample_hidden(hid, u, temperature=torch.zeros(n, device="cuda"))
    own = run.score_hidden(hid)
    # at least half of the rows of a window lie below the threshold, some above
    tau = float(own["conf"].median())

    def select(token, conf):
        tok, p, k = to_dev(tok_h), to_dev(p_h), torch.zeros(B, dtype=torch.int32, device="cuda")
        s = {name: a.clone() for name, a in st.items()}
        s["top1"].view(-1)[at], s["conf"].view(-1)[at] = token, conf
        dcl.dcl_select_contiguous(tok, B, S, p, w.gen_end, w.window, tau, 2.0, g.mask_id, s, None, k)
        return tok.cpu(), p.cpu(), k.cpu()
    share, model, step = select(drawn["token"], drawn["conf"]), select(drawn["token"], own["conf"]), \
        select(st["top1"].view(-1)[at], own["conf"])
    assert bool((drawn["conf"] == 1).all()) and bool((drawn["kept"] == 1).all())
    whole = torch.tensor([min(w.window, w.gen_end - int(x)) for x in p_h])
    assert torch.equal(share[2].long(), whole)
    assert all(torch.equal(a, b) for a, b in zip(model, step)) and bool((model[2].long() < whole).any())
