"""GPU tests of the 8-bit cache and of adjusted head outputs as the framework's own paths run them: one backbone layer
(vfm_layer_forward_q8) against the oracle's parts over the cache that the layer leaves, the continuous-batching loop with
such a cache against a 64-bit forward that keeps one, and penalties, biases and masks in the loop.

Tolerances.  The layer's attention reads codes, so its reference reads them too, and the windowed layer's tolerance holds
(2e-2 bf16, 1e-5 fp32, of a row's norm).  The codes themselves: a rounding to e4m3 is off by at most 2^-4 of an element (2^-10
of its scale below e4m3's normal numbers), and the rows that are rounded by that tolerance.  The loop's 64-bit forward
makes codes of its own: where its unrounded key differs by d of itself, a share of 2 d / 2^-4 of the codes may be the
neighbouring one, at most 2^-3 from it, which is 2^-3 sqrt(share) of a key's norm: 2.2e-3 in fp32 (d = 1e-5) and 3.1e-2 in
bf16 (d = 2^-9), beside the other roundings' 1e-5 and 2e-2."""
import numpy as np
import pytest
import torch

from oracle import vfm_oracle as O
from paper_2606_09643_amd import binding as B
from paper_2606_09643_amd import runner as R
from paper_2606_09643_amd import workloads as wl
from tests import decode_common as D
from tests import kv8_common as K
from tests.gpu_common import as_f32, expected_embed, log, set_rows, tol
from tests.helpers import np64, oracle_adapter, oracle_weights, spec_of
from tests.test_gpu_windowed import REQUESTS, SAMPLING, _decoder, _loop, _model

pytestmark = pytest.mark.gpu


class _Pool:
    """A layer's 8-bit pool with the pages that a step needs and no others; slots that no row sees and none is written to
    hold NaN codes, their runs' exponents 255."""

    def __init__(self, w, lens, ctx, page, window, sinks, seed):
        rng = np.random.default_rng(seed)
        self.page, self.H, self.dh = page, w.n_heads, w.head_dim
        wide = int((ctx + lens).max() - 1) // page + 1
        need = []
        for m, c in zip(lens, ctx):
            j = np.arange((int(c) + int(m) - 1) // page + 1)
            lo = max(0, int(c) - window + 1) // page if window else 0
            need.append(j[(j >= lo) | ((j * page < sinks) & (window > 0))])
        perm = rng.permutation(sum(map(len, need)) + 3).astype(np.int32)
        self.table = np.full((len(lens), wide), -1, np.int32)
        at = 0
        for i, j in enumerate(need):
            self.table[i, j] = perm[at:at + len(j)]
            at += len(j)
        slots = len(perm) * page
        codes = [np.full((self.H, slots, self.dh), 0x7F, np.uint8) for _ in range(2)]
        exps = np.full((slots // 16, self.H, 2), 255, np.uint8)
        for i, c in enumerate(ctx):
            pos = np.arange(int(c))
            see = (pos > int(c) - window) | (pos < sinks) if window else np.ones(len(pos), bool)
            see |= pos >= int(c) // 16 * 16                 # the run that the first new row joins
            s = self.slots(i, pos[see])
            exps[np.unique(s // 16)] = rng.integers(118, 122, (len(np.unique(s // 16)), self.H, 2))
            for x in codes:
                x[:, s] = K.to_codes(np.clip(rng.standard_normal((self.H, len(s), self.dh)) * 90, -448, 448))
        self.k, self.v, self.exps = (torch.from_numpy(x).cuda() for x in (*codes, exps))
        self.kv = B.PagedKVQ8(self.k, self.v, self.exps, page, self.table)

    def slots(self, i, pos):
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page

    def values(self, i, pos):
        """(k, v) at positions of request i as the pool holds them now, [positions, H * dh]."""
        s = self.slots(i, pos)
        e = self.exps.cpu().numpy()[s // 16]
        return [(K.VALUES[x[:, s].cpu().numpy()].transpose(1, 0, 2) * 2.0 ** (e[:, :, n] - 127.0)[..., None])
                .reshape(len(pos), -1) for n, x in enumerate((self.k, self.v))]


def _rows(spec, W, ad, x, pos):
    """The oracle's rotated queries and keys and its values of rows x."""
    h = O.norm(x, W["norm1_w"], W.get("norm1_b"), spec["norm"], spec["eps"])
    qkv = [O._proj(h, m, b, ad, n) for (m, b), n in zip(O._split_qkv(W), "qkv")]
    if spec["rope_theta"]:
        qkv[:2] = [O.rope(t, pos, spec["n_heads"], spec["head_dim"], spec["rope_theta"]) for t in qkv[:2]]
    return qkv


def _rest(spec, W, ad, x, a):
    """The oracle's layer behind the attention's rows a (of rows x)."""
    x = x + O._proj(a, W["w_o"], W.get("b_o"), ad, "o")
    h = O.norm(x, W["norm2_w"], W.get("norm2_b"), spec["norm"], spec["eps"])
    u = O.silu(O._proj(h, W["w_gate"], None, ad, "gate")) * O._proj(h, W["w_up"], None, ad, "up")
    return x + O._proj(u, W["w_down"], W.get("b_down"), ad, "down")


def _run_layer(w, lens, ctx, task, page, window, sinks, rope=True, rows=None):
    lens, ctx, task = (np.array(a, np.int32) for a in (lens, ctx, task))
    batch = wl.Batch(task, lens, ctx)
    model, inp = R.Model(w, n_layers=1, b_std=0.1), R.Inputs(w, batch)
    pool = _Pool(w, lens, ctx, page, window, sinks, seed=21)
    before = [t.clone() for t in (pool.k, pool.v)]
    cfg, spec = R.cfg_for(w), spec_of(w)
    cfg.attn = B.VFM_ATTN_MIXED
    if not rope:
        cfg.rope_theta = spec["rope_theta"] = 0.0
    pb = B.Batch(task, lens, w.n_tasks, ctx_len=ctx)
    pl = O.plan(task, lens, w.n_tasks, ctx=ctx)
    x_in = as_f32(expected_embed(w, batch, inp, pl))
    x = torch.empty(pb.T, w.d, dtype=torch.float32, device="cuda")
    set_rows(x, x_in)
    ws = torch.full((B.vfm_workspace_size_q8(cfg, pb.c, model.lora_c(0), window, sinks),), 255, dtype=torch.uint8, device="cuda")
    log(f"q8 layer {w.dtype} d {w.d} dh {w.head_dim} lens {list(lens)} ctx {list(ctx)} window {window} sinks {sinks}")
    B.vfm_layer_forward_q8(cfg, model.c_layers[0], model.lora_c(0), pb.c, x, pool.kv, window, sinks, ws)
    torch.cuda.synchronize()
    got, W = np64(x), oracle_weights(model.layers[0])
    assert np.isfinite(got).all()
    worst, coded = 0.0, 0.0
    written = np.zeros(pool.k.shape[1], bool)
    for p in range(len(lens)):
        i, r0 = int(pl["order"][p]), int(pl["cu_seqlens"][p])
        c, m, ad = int(ctx[i]), int(lens[i]), oracle_adapter(model.adapters[0], int(pl["task"][p]))
        q, k, v = _rows(spec, W, ad, x_in[r0:r0 + m], c + np.arange(m))
        new = pool.values(i, c + np.arange(m))
        coded = max(coded, *(O.row_rel_error(a, b) for a, b in zip(new, (k, v))))
        for j in range(m) if rows is None else sorted(set(np.linspace(0, m - 1, rows).astype(int).tolist())):
            pos = np.arange(c + j + 1)
            ka, va = pool.values(i, pos[D.visible(c + j, pos, window, sinks)])
            a = O.attention(q[j:j + 1], ka, va, w.n_heads, w.head_dim)
            worst = max(worst, O.row_rel_error(got[r0 + j][None], _rest(spec, W, ad, x_in[r0 + j:r0 + j + 1], a)))
        written[pool.slots(i, np.arange(c // 16 * 16, c + m))] = True
    log(f"  max rel err {worst:.3e}, of the codes' numbers {coded:.3e}")
    assert worst < tol(w) and coded < 2.0 ** -4 + tol(w)
    keep = torch.from_numpy(~written).cuda()
    for now, was in zip((pool.k, pool.v), before):
        assert torch.equal(now[:, keep], was[:, keep])
    return x


@pytest.mark.parametrize("dtype,hd,page,window,sinks,rope", [
    ("bf16", 128, 16, 20, 3, True), ("bf16", 64, 32, 64, 0, True), ("f32", 128, 16, 20, 3, True),
    ("f32", 64, 16, 1, 1, True), ("bf16", 64, 16, 33, 40, False), ("f32", 64, 32, 50, 2, False),
    ("bf16", 128, 16, 0, 5, True), ("f32", 128, 16, 0, 0, True)])
def test_layer_mixed_step(dtype, hd, page, window, sinks, rope):
    """Prompts, chunks after cached tokens and single rows in one step."""
    _run_layer(_decoder(dtype, hd), [1, 40, 7, 1, 70, 1], [90, 0, 33, 0, 150, 700], [2, 0, 1, 1, 0, 2], page, window,
               sinks, rope)


@pytest.mark.parametrize("hd", [64, 128])
def test_layer_large_batch(hd):
    """Above the small-batch threshold, where the products are other kernels; and an append of grouped rows."""
    lens, ctx = [300, 1, 1513, 260], [50, 1500, 0, 700]
    _run_layer(_decoder("bf16", hd, d=1024), lens, ctx, [1, 0, 2, 1], 64, 100, 4, rows=5)


class _Seq8:
    """A request's forward in 64 bits, a token at a time, every layer's keys and values kept in 8 bits."""

    def __init__(self, w, model, emb_np, task, window, sinks, room):
        self.spec, self.window, self.sinks, self.emb = spec_of(w), window, sinks, emb_np
        self.W = [oracle_weights(W) for W in model.layers]
        self.ad = [oracle_adapter(a, task) for a in model.adapters]
        self.head = (np64(model.heads.W[task]), np64(model.heads.b[task]))
        self.final = (np64(model.final["w"]), np64(model.final.get("b")))
        H, dh, runs = w.n_heads, w.head_dim, -(-room // 16)
        self.pool = [[(np.zeros((runs * 16, dh), np.uint8), np.zeros(runs, np.uint8)) for _ in range(2 * H)] for _ in model.layers]
        self.n = 0

    def feed(self, token):
        x, j, H, dh = self.emb[[token]], self.n, self.spec["n_heads"], self.spec["head_dim"]
        pos = np.arange(j + 1)
        see = pos[D.visible(j, pos, self.window, self.sinks)]
        for W, ad, pool in zip(self.W, self.ad, self.pool):
            q, k, v = _rows(self.spec, W, ad, x, np.array([j]))
            kv = []
            for rows, heads in ((k, pool[:H]), (v, pool[H:])):
                for h, (codes, exps) in enumerate(heads):
                    K.append(codes, exps, rows[:, h * dh:(h + 1) * dh], np.array([j]), j)
                kv.append(np.concatenate([K.VALUES[codes[see]] * 2.0 ** (exps[see // 16] - 127.0)[:, None]
                                          for codes, exps in heads], 1))
            x = _rest(self.spec, W, ad, x, O.attention(q, *kv, H, dh))
        self.n += 1
        return O.head(O.final(self.spec, *self.final, x)[-1], *self.head)


@pytest.mark.parametrize("dtype,window,sched", [("f32", 20, "fifo"), ("f32", None, "fifo"), ("bf16", 20, "bfq"),
                                                ("bf16", None, "whole-prompts")])
def test_loop(dtype, window, sched):
    """Sequences of up to 115 positions in 8 bits, under a window in rings of pages or without one; prompts in chunks (that
    end inside runs) or at once: every step's head outputs are the 64-bit forward's, whose tokens come one by one."""
    sinks = 18 if window else 0
    w = _decoder(dtype, 128)
    model, emb, prompts = _model(w)
    kw = dict(window=window, n_sink=sinks, kv8=True)
    if window is None:
        kw.update(max_pages=8, n_pages=24)
    if sched == "bfq":
        kw["bfq"] = B.BFQ([1.0, 2.0, 1.0], np.linspace(1.0, 2.0, 3), b_max=2)
    if sched == "whole-prompts":
        kw.update(chunk_prompts=False, max_step_tokens=96, max_pages=10)
    done, outs, cb = _loop(w, model, emb, prompts, **kw)
    emb_np, worst = np64(emb), 0.0
    for rid, (task, _, n_new) in enumerate(REQUESTS):
        seq = _Seq8(w, model, emb_np, task, window or 0, sinks, len(prompts[rid]) + n_new)
        for tok in prompts[rid]:
            ref = seq.feed(int(tok))
        for j in range(n_new):
            got = outs[rid][j]
            worst = max(worst, O.row_rel_error(got[None], ref[None]))
            assert done[rid][j] == int(np.argmax(got))
            ref = seq.feed(done[rid][j]) if j + 1 < n_new else None       # both go on with the loop's token
    log(f"  {sched} {dtype} window {window}: {cb.steps} steps, max rel err {worst:.3e}")
    d = 2.0 ** -9 if dtype == "bf16" else 1e-5
    assert worst < tol(w) + 2.0 ** -3 * (2 * d / 2.0 ** -4) ** 0.5


def _no_repeat(n):
    """A grammar: no token twice, and after 8 tokens only those from n // 2 on."""
    def allowed(answer):
        ok = np.ones(n, bool)
        ok[list(answer)] = False
        if len(answer) >= 8:
            ok[:n // 2] = False
        return ok
    return allowed


@pytest.mark.parametrize("kv8", [False, True])
def test_loop_adjusts_outputs(kv8):
    """Tokens are those of the head outputs after the 64-bit form of each request's own penalties, biases and mask,
    drawn or greedy, with requests beside them that have none; the loop without read-backs gives the same."""
    w = _decoder("bf16", 64)
    model, emb, prompts = _model(w)
    n = int(model.heads.n_out[0])
    static = np.arange(n) % 3 == 0
    adjust = [R.AdjustParams(1.5, 0.5, 0.2), R.AdjustParams(bias={7: 2.5, 3: -1e9, 11: -np.inf}, presence=1.0),
              R.AdjustParams(0.9, -0.3, 0.4, allowed=_no_repeat(n)), None, R.AdjustParams(allowed=static)]
    kw = dict(max_pages=9, n_pages=24, kv8=kv8, window=40 if kv8 else None)

    def run(record):
        cb = R.ContinuousBatcher(model, emb, **{**dict(page_size=16, max_seqs=3, max_step_tokens=48, record=record), **kw})
        for rid, ((task, _, n_new), pr) in enumerate(zip(REQUESTS, prompts)):
            cb.submit(rid, task, pr, n_new, sampling=SAMPLING[rid], adjust=adjust[rid])
        return cb.run(), cb
    done, cb = run(True)
    outs = {rid: [] for rid in done}
    for step in cb.trace:
        for rid, o in step:
            outs[rid].append(o)
    near = 0
    for rid, (a, sp) in enumerate(zip(adjust, SAMPLING)):
        rng = np.random.default_rng(sp.seed) if sp is not None else None
        assert len(done[rid]) == REQUESTS[rid][2]
        for j, (got, o) in enumerate(zip(done[rid], outs[rid])):
            l = o.astype(np.float64)
            if a is not None:
                f32 = [float(np.float32(x)) for x in (a.repetition, a.presence, a.frequency)]
                ok = a.allowed(done[rid][:j]) if callable(a.allowed) else a.allowed
                l = K.adjust(o, *f32, hist=list(prompts[rid]) + done[rid][:j], n_prompt=len(prompts[rid]),
                             bias=list(zip(a.bias_id.tolist(), a.bias.astype(np.float64).tolist())), allowed=ok)
                assert ok is None or ok[got]
            l = l.astype(np.float32)
            if sp is None or sp.temperature == 0:
                if sp is not None:
                    rng.random(dtype=np.float32)
                assert l[got] == l.max()
                continue
            u = rng.random(dtype=np.float32)
            f32 = [float(np.float32(t)) for t in (sp.temperature, sp.top_p, sp.min_p)]
            want, _, gap = D.sample(l, f32[0], sp.top_k, f32[1], f32[2], float(u))
            near += gap < 2.0 ** -22                       # an output's rounding to fp32, times 256
            assert got == want or gap < 2.0 ** -22, (rid, j)
    assert near <= 3
    assert len(set(done[2])) == len(done[2]) and min(done[2][8:]) >= n // 2
    assert run(False)[0] == done


def test_append_attend_adjust_sample_in_one_step():
    """The four calls as a step of a model of grouped heads, on one stream and replayed from one graph: new rows rotated
    into the 8-bit cache, attention over it, outputs adjusted in place, and a token drawn per request."""
    H, KH, dh, page, window, sinks, theta = 8, 2, 64, 16, 40, 3, 10000.0
    lens, ctx, task = np.array([1, 12, 1, 60], np.int32), np.array([130, 0, 55, 20], np.int32), np.zeros(4, np.int32)
    attn = B.make_attn(B.VFM_BF16, H, KH, dh, window=window, n_sink=sinks, rope_theta=theta)
    n_out = H * dh
    pb = B.Batch(task, lens, 1, ctx_len=ctx, n_out=np.array([n_out], np.int32))
    rng = np.random.default_rng(9)
    pages = [-(-int(c + m) // page) for c, m in zip(ctx, lens)]
    table = np.zeros((4, max(pages)), np.int32)
    perm, at = rng.permutation(sum(pages)).astype(np.int32), 0
    for i, k in enumerate(pages):
        table[i, :k] = perm[at:at + k]
        at += k
    slots = sum(pages) * page
    codes = [K.to_codes(np.clip(rng.standard_normal((KH, slots, dh)) * 90, -448, 448)) for _ in range(2)]
    exps = rng.integers(118, 122, (slots // 16, KH, 2)).astype(np.uint8)
    kp, vp, ep = (torch.from_numpy(x).cuda() for x in (*codes, exps))
    kv = B.PagedKVQ8(kp.clone(), vp.clone(), ep.clone(), page, table)
    host = torch.from_numpy(rng.standard_normal((pb.T, (H + 2 * KH) * dh))).to(torch.bfloat16)
    x, q = host.cuda(), torch.empty(pb.T, H * dh, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(max(1, B.vfm_attention_workspace_q8(attn, pb.c)), dtype=torch.uint8, device="cuda")
    last = torch.from_numpy(np.cumsum(lens) - 1).cuda()          # one task: plan order is the original one
    raw, logits = torch.empty(4 * n_out, device="cuda"), torch.empty(4 * n_out, device="cuda")
    temp, u = torch.tensor([1.0, 0.2, 0.0, 2.0], device="cuda"), torch.tensor([0.3, 0.9, 0.5, 0.1], device="cuda")
    params = B.Sampling(temperature=temp)
    hist = rng.integers(0, n_out, (4, 50)).astype(np.int32)
    allowed = rng.random(n_out) < 0.3
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    adj = B.OutputAdjust(repetition=dev(np.array([1.3, 1.0, 0.8, 1.0], np.float32)),
                         frequency=dev(np.array([0.0, 0.5, 0.1, 0.0], np.float32)), hist=dev(hist),
                         hist_begin=dev(np.arange(4) * 50), hist_len=dev(np.array([50, 20, 33, 0], np.int32)),
                         mask=dev(K.mask_words(allowed, n_out // 32)[None]), mask_row=dev(np.array([-1, 0, -1, 0], np.int32)))
    ids, logp = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")

    def step():
        B.vfm_kv_append_q8(attn, pb.c, x, q, kv)
        B.vfm_attention_paged_q8(attn, pb.c, q, kv, out, ws)
        raw.copy_(out[last].float().view(-1) * 30)
        logits.copy_(raw)
        B.vfm_adjust_outputs(pb.c, logits, adj)
        B.vfm_sample_tokens(pb.c, logits, params, u, ids, logp)

    log("append, attend, adjust, sample in 8 bits")
    step()
    torch.cuda.synchronize()
    # the cache that the forms make of it, and attention over that
    cu = np.concatenate([[0], np.cumsum(lens)])
    for i in range(4):
        c, m = int(ctx[i]), int(lens[i])
        _, k, v = K.rotated(np64(host)[cu[i]:cu[i + 1]].reshape(m, H + 2 * KH, dh), H, KH, np.arange(c, c + m), theta)
        runs = -(-(c + m) // 16)
        s = np.concatenate([table[i, j] * page + np.arange(page) for j in range(runs)])
        vals = []
        for n, rows in enumerate((k, v)):
            for h in range(KH):
                got, e = codes[n][h, s], exps[s[::16] // 16, h, n]
                K.append(got, e, rows[:, h], np.arange(c, c + m), c)
                codes[n][h, s], exps[s[::16] // 16, h, n] = got, e
            ev = exps[s // 16, :, n]
            vals.append((K.VALUES[codes[n][:, s]].transpose(1, 0, 2) * 2.0 ** (ev - 127.0)[..., None])[:c + m])
        q_got = np64(q)[cu[i]:cu[i + 1]].reshape(m, H, dh)
        ref, a, seen = D.attention(q_got, *vals, c, window, sinks, dh ** -0.5)
        dot = D.score_sizes(q_got, vals[0], dh ** -0.5)[:, :, None]
        lim = (2.0 ** -8 + (seen[:, None, None] + 16) * 2.0 ** -24) * (a + np.abs(ref)) \
            + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
        assert np.all(np.abs(np64(out)[cu[i]:cu[i + 1]].reshape(m, H, dh) - ref) <= lim)
        l = raw.cpu().numpy().reshape(4, n_out)[i]
        r, f, hl = [1.3, 1.0, 0.8, 1.0][i], [0.0, 0.5, 0.1, 0.0][i], [50, 20, 33, 0][i]
        want = K.adjust(l, float(np.float32(r)), 0.0, float(np.float32(f)), hist[i, :hl], 0,
                        allowed=allowed if i in (1, 3) else None).astype(np.float32)
        assert np.array_equal(logits.cpu().numpy().reshape(4, n_out)[i], want)
        tok, lp, gap = D.sample(want, float(temp[i]), 0, 1.0, 0.0, float(u[i]))
        assert gap > 2.0 ** -30 and int(ids[i]) == tok and abs(float(logp[i]) - lp) <= 2.0 ** -20 * (1 + abs(lp))
    assert np.array_equal(kv.k.cpu().numpy(), codes[0]) and np.array_equal(kv.v.cpu().numpy(), codes[1])
    assert np.array_equal(kv.exps.cpu().numpy(), exps)
    first = [t.clone() for t in (out, logits, ids, logp, kv.k, kv.v, kv.exps)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (out, logits, ids, logp, q):
            t.fill_(0)
        for t, was in ((kv.k, kp), (kv.v, vp), (kv.exps, ep)):
            t.copy_(was)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip((out, logits, ids, logp, kv.k, kv.v, kv.exps), first):
            assert torch.equal(t.nan_to_num(3.0) if t.is_floating_point() else t,
                               want.nan_to_num(3.0) if t.is_floating_point() else want)
