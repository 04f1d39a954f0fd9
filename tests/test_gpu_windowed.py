"""GPU tests of decoding over a bounded cache as the framework's own paths run
it: one backbone layer with the windowed attention (vfm_layer_forward_windowed)
against the oracle, row by row over the keys that the row sees; the
continuous-batching loop with a window, whose sequences keep a ring of pages;
and drawn tokens, in the loop and in a step put together from the calls."""
import numpy as np
import pytest
import torch

from oracle import vfm_oracle as O
from paper_2606_09643_amd import binding as B
from paper_2606_09643_amd import runner as R
from paper_2606_09643_amd import workloads as wl
from tests import decode_common as D
from tests.gpu_common import as_f32, expected_embed, log, set_rows, tol
from tests.helpers import np64, oracle_adapter, oracle_weights, spec_of

pytestmark = pytest.mark.gpu


def _decoder(dtype, hd, d=256, **kw):
    return wl.Workload(6, f"tiny-decoder-{dtype}", dtype, "decoder", 2, d, d // hd, hd, 2 * d, n_tasks=3, n_req=6, rank=8,
                       lora_targets=wl.PROJ, lora_scale=2.0, zipf_s=None, seq_len=(1, 40), mode="prefill", ctx=None,
                       inputs="tokens", pool="last", head="fixed:256", vocab=256).replace(**kw)


def _windowed_layer(spec, W, ad, x, kc, vc, window, sinks, rows):
    """The oracle's layer for `rows` of a request whose rows x follow the cached kc, vc: a row
    attends to the cached and earlier rows that it sees, and to itself.  ({row: y}, k, v of all rows)"""
    c, m = len(kc), len(x)
    pos = c + np.arange(m)
    _, k, v = O.layer(spec, W, ad, x, pos=pos)         # keys and values do not depend on the attention
    ka, va = np.concatenate([kc, k]), np.concatenate([vc, v])
    y = {}
    for i in rows:
        see = D.visible(c + i, np.arange(c + i), window, sinks)
        y[i] = O.layer(spec, W, ad, x[i:i + 1], pos=pos[i:i + 1], kv=(ka[:c + i][see], va[:c + i][see]))[0][0]
    return y, k, v


class _Cache:
    """A pool with the pages that a windowed step needs and no others: table entries between the
    sinks and the window are -1, slots that no row sees and none is written to hold NaN."""

    def __init__(self, w, lens, ctx, page, window, sinks, seed):
        rng = np.random.default_rng(seed)
        self.page = page
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
        shape = (w.n_heads, len(perm) * page, w.head_dim)
        k, v = np.full(shape, np.nan, np.float32), np.full(shape, np.nan, np.float32)
        self.rows = []
        for i, (m, c) in enumerate(zip(lens, ctx)):
            pos = np.arange(int(c))
            see = (pos > int(c) - window) | (pos < sinks) if window else np.ones(len(pos), bool)
            kc, vc = [torch.from_numpy(rng.standard_normal((int(c), w.d))).to(w.torch_dtype).double().numpy()
                      for _ in range(2)]
            s = self.slots(i, pos[see])
            k[:, s] = kc[see].reshape(-1, w.n_heads, w.head_dim).transpose(1, 0, 2)
            v[:, s] = vc[see].reshape(-1, w.n_heads, w.head_dim).transpose(1, 0, 2)
            self.rows.append((kc, vc))
        self.k, self.v = [torch.from_numpy(t).to(w.torch_dtype).cuda() for t in (k, v)]

    def slots(self, i, pos):
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page

    def new_rows(self, t, i, c, m):
        return np64(t[:, self.slots(i, np.arange(c, c + m))].permute(1, 0, 2).reshape(m, -1))


def _run_layer(w, lens, ctx, task, page, window, sinks, rope=True, rows=None, attn=B.VFM_ATTN_MIXED):
    """One windowed layer; returns (its output, the cache after it), both checked against the oracle."""
    lens, ctx, task = (np.array(a, np.int32) for a in (lens, ctx, task))
    batch = wl.Batch(task, lens, ctx)
    model = R.Model(w, n_layers=1, b_std=0.1)
    inp = R.Inputs(w, batch)
    cache = _Cache(w, lens, ctx, page, window, sinks, seed=21)
    k0, v0 = cache.k.clone(), cache.v.clone()
    cfg = R.cfg_for(w)
    cfg.attn = attn
    spec = spec_of(w)
    if not rope:
        cfg.rope_theta = spec["rope_theta"] = 0.0
    pb = B.Batch(task, lens, w.n_tasks, ctx_len=ctx)
    pl = O.plan(task, lens, w.n_tasks, ctx=ctx)
    x_in = as_f32(expected_embed(w, batch, inp, pl))
    x = torch.empty(pb.T, w.d, dtype=torch.float32, device="cuda")
    set_rows(x, x_in)
    ws = torch.full((B.vfm_workspace_size_windowed(cfg, pb.c, model.lora_c(0), window, sinks),), 255, dtype=torch.uint8,
                    device="cuda")
    log(f"windowed layer {w.dtype} d {w.d} dh {w.head_dim} lens {list(lens)} ctx {list(ctx)} window {window} sinks {sinks}")
    B.vfm_layer_forward_windowed(cfg, model.c_layers[0], model.lora_c(0), pb.c, x,
                                 B.PagedKV(cache.k, cache.v, page, cache.table), window, sinks, ws)
    torch.cuda.synchronize()
    got = np64(x)
    assert np.isfinite(got).all()
    W_np = oracle_weights(model.layers[0])
    cu, worst = pl["cu_seqlens"], 0.0
    written = np.zeros(cache.k.shape[1], bool)
    for p in range(len(lens)):
        i, t = int(pl["order"][p]), int(pl["task"][p])
        c, m, r0 = int(ctx[i]), int(lens[i]), int(cu[p])
        some = range(m) if rows is None else sorted(set(np.linspace(0, m - 1, rows).astype(int).tolist()))
        y, k, v = _windowed_layer(spec, W_np, oracle_adapter(model.adapters[0], t), x_in[r0:r0 + m], *cache.rows[i],
                                  window, sinks, some)
        for j in some:
            worst = max(worst, O.row_rel_error(got[r0 + j][None], y[j][None]))
        worst = max(worst, O.row_rel_error(cache.new_rows(cache.k, i, c, m), k),
                    O.row_rel_error(cache.new_rows(cache.v, i, c, m), v))
        written[cache.slots(i, np.arange(c, c + m))] = True
    log(f"  max rel err {worst:.3e}")
    assert worst < tol(w)
    keep = torch.from_numpy(~written).cuda()
    bits = torch.int16 if w.dtype == "bf16" else torch.int32
    for now, before in ((cache.k, k0), (cache.v, v0)):
        assert torch.equal(now[:, keep].view(bits), before[:, keep].view(bits))
    return x


@pytest.mark.parametrize("dtype,hd,page,window,sinks,rope", [
    ("bf16", 128, 16, 20, 3, True), ("bf16", 64, 32, 64, 0, True), ("f32", 128, 16, 20, 3, True),
    ("f32", 64, 16, 1, 1, True), ("bf16", 64, 16, 33, 40, False), ("f32", 64, 32, 50, 2, False),
    ("bf16", 128, 16, 0, 5, True), ("f32", 128, 16, 0, 0, True)])
def test_windowed_layer_mixed_step(dtype, hd, page, window, sinks, rope):
    """Prompts, chunks after cached tokens and single rows in one step."""
    _run_layer(_decoder(dtype, hd), [1, 40, 7, 1, 70, 1], [90, 0, 33, 0, 150, 700], [2, 0, 1, 1, 0, 2], page, window,
               sinks, rope)


@pytest.mark.parametrize("attn,lens,ctx", [("causal", [50, 1, 9], [0, 0, 0]), ("decode", [1, 1, 1], [400, 0, 17])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windowed_layer_prompts_and_decode(dtype, attn, lens, ctx):
    code = B.VFM_ATTN_CAUSAL if attn == "causal" else B.VFM_ATTN_DECODE
    _run_layer(_decoder(dtype, 64), lens, ctx, [1, 0, 2], 16, 24, 4, attn=code)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windowed_layer_far_positions(dtype):
    """At position 60000 an angle of 24 bits is off by up to 0.004, far more than the fp32 tolerance."""
    _run_layer(_decoder(dtype, 64), [1, 5], [60000, 59990], [0, 1], 64, 100, 2)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rope", [True, False])
def test_windowed_layer_large_batch(hd, rope):
    """Above the small-batch threshold the rotation is the QKV product's store pass; the cache is
    written by a pass of its own."""
    lens, ctx = [300, 1, 513, 260], [50, 1500, 0, 700]
    assert sum(lens) >= B.VFM_SMALL_BATCH_ROWS
    _run_layer(_decoder("bf16", hd, d=1024), lens, ctx, [1, 0, 2, 1], 64, 100, 4, rope, rows=7)


def test_windowed_layer_that_sees_everything():
    """A window of every position gives the bits of no window."""
    args = ([1, 40, 70], [90, 0, 150], [2, 0, 1], 16)
    w = _decoder("bf16", 64)
    assert torch.equal(_run_layer(w, *args, 0, 0), _run_layer(w, *args, 220, 3))


# ---- the continuous-batching loop ------------------------------------------
REQUESTS = [  # (task, prompt length, new tokens)
    (0, 5, 40), (2, 61, 30), (1, 1, 70), (0, 33, 4), (2, 90, 25)]


def _loop(w, model, emb, prompts, sampling=None, requests=REQUESTS, **kw):
    args = dict(page_size=16, n_pages=18, max_seqs=3, max_step_tokens=48, max_pages=7, record=True)
    args.update(kw)
    cb = R.ContinuousBatcher(model, emb, **args)
    for rid, ((task, _, n_new), pr) in enumerate(zip(requests, prompts)):
        cb.submit(rid, task, pr, n_new, sampling=sampling[rid] if sampling is not None else None)
    done = cb.run()
    assert sorted(done) == list(range(len(requests))) and [len(done[r]) for r in sorted(done)] == [n for _, _, n in requests]
    assert cb.alloc.count(0)[1] == args["n_pages"] and cb.committed == 0
    outs = {rid: [] for rid in done}
    for step in cb.trace:
        for rid, o in step:
            outs[rid].append(o)
    return done, outs, cb


def _model(w):
    model = R.Model(w, n_layers=2, b_std=0.1)
    _, emb = wl.token_inputs(w, wl.Batch(np.zeros(1, np.int32), np.ones(1, np.int32), None), "cuda")
    rng = np.random.default_rng(5)
    return model, emb, [rng.integers(0, w.vocab, size=L).astype(np.int32) for _, L, _ in REQUESTS]


class _OracleSeq:
    """A request's windowed forward in the oracle, a token at a time, every layer's keys kept."""

    def __init__(self, w, model, emb_np, task, window, sinks):
        self.spec, self.window, self.sinks, self.emb = spec_of(w), window, sinks, emb_np
        self.W = [oracle_weights(W) for W in model.layers]
        self.ad = [oracle_adapter(a, task) for a in model.adapters]
        self.head = (np64(model.heads.W[task]), np64(model.heads.b[task]))
        self.final = (np64(model.final["w"]), np64(model.final.get("b")))
        self.kv = [(np.zeros((0, w.d)), np.zeros((0, w.d))) for _ in model.layers]

    def feed(self, token):
        x, j = self.emb[[token]], len(self.kv[0][0])
        see = D.visible(j, np.arange(j), self.window, self.sinks)
        for li, (k, v) in enumerate(self.kv):
            x, kn, vn = O.layer(self.spec, self.W[li], self.ad[li], x, pos=np.array([j]), kv=(k[see], v[see]))
            self.kv[li] = (np.concatenate([k, kn]), np.concatenate([v, vn]))
        return O.head(O.final(self.spec, *self.final, x)[-1], *self.head)


@pytest.mark.parametrize("dtype,sched", [("bf16", "fifo"), ("f32", "fifo"), ("bf16", "bfq"), ("f32", "whole-prompts")])
def test_loop_with_a_window(dtype, sched):
    """Sequences of up to 115 positions under a window of 20 and 18 sinks, prompts in chunks of at most 20 rows: each
    holds at most 2 + 4 pages of 16, and every step's head outputs are the oracle's over the visible keys."""
    window, sinks = 20, 18
    w = _decoder(dtype, 128)
    model, emb, prompts = _model(w)
    kw = dict(window=window, n_sink=sinks)
    if sched == "bfq":
        kw["bfq"] = B.BFQ([1.0, 2.0, 1.0], np.linspace(1.0, 2.0, 3), b_max=2)
    if sched == "whole-prompts":                   # rings of window + prompt
        kw.update(chunk_prompts=False, max_step_tokens=96, max_pages=10, n_pages=24)
    done, outs, cb = _loop(w, model, emb, prompts, **kw)
    if sched != "whole-prompts":
        assert max(s.budget for s in cb.done.values()) == 2 + 4
    emb_np, worst, compared = np64(emb), 0.0, 0
    for rid, (task, _, n_new) in enumerate(REQUESTS):
        seq = _OracleSeq(w, model, emb_np, task, window, sinks)
        for tok in prompts[rid]:
            ref = seq.feed(int(tok))
        for j in range(n_new):
            got = outs[rid][j]
            worst = max(worst, O.row_rel_error(got[None], ref[None]))
            assert done[rid][j] == int(np.argmax(got))
            compared += 1
            ref = seq.feed(done[rid][j]) if j + 1 < n_new else None       # both go on with the loop's token
    log(f"  {sched} {dtype}: {cb.steps} steps, {compared} outputs, max rel err {worst:.3e}")
    assert worst < tol(w)


def test_loop_with_a_wide_window_keeps_the_picks():
    """A window that no sequence reaches: the outputs of the loop without one, to rounding."""
    w = _decoder("f32", 64)
    model, emb, prompts = _model(w)
    kw = dict(max_step_tokens=96, max_pages=9, n_pages=24, chunk_prompts=False)
    done, outs, _ = _loop(w, model, emb, prompts, **kw)
    done_w, outs_w, _ = _loop(w, model, emb, prompts, window=500, **kw)
    for rid in done:
        for a, b, x, y in zip(outs[rid], outs_w[rid], done[rid], done_w[rid]):
            assert O.row_rel_error(a[None], b[None].astype(np.float64)) < tol(w)
            if x != y:                             # from a near-tie on they decode different tokens
                break


SAMPLING = [R.SamplingParams(0.8, seed=1), R.SamplingParams(1.5, top_k=12, seed=2), None,
            R.SamplingParams(1.0, top_p=0.7, min_p=0.02, seed=4), R.SamplingParams(0.0, seed=5)]


@pytest.mark.parametrize("window", [None, 24])
def test_loop_draws_tokens(window):
    """Drawn tokens are the 64-bit form's of the step's outputs and the request's own numbers, whatever else is in the
    batch; a request without parameters stays greedy, and the loop without read-backs draws the same."""
    w = _decoder("bf16", 64)
    model, emb, prompts = _model(w)
    kw = dict(window=window, n_sink=2 if window else 0, max_pages=9, n_pages=24)
    done, outs, cb = _loop(w, model, emb, prompts, SAMPLING, **kw)
    near = 0
    for rid, sp in enumerate(SAMPLING):
        rng = np.random.default_rng(sp.seed) if sp is not None else None
        for got, o in zip(done[rid], outs[rid]):
            if sp is None:
                assert got == int(np.argmax(o))
                continue
            u = rng.random(dtype=np.float32)
            f32 = [float(np.float32(t)) for t in (sp.temperature, sp.top_p, sp.min_p)]
            want, _, gap = D.sample(o, f32[0], sp.top_k, f32[1], f32[2], float(u))
            if gap < 2.0 ** -36:                   # 256 weights of 44 bits: a border that rounding may cross
                near += 1
                continue
            assert got == want, rid
    assert near <= 1
    assert _loop(w, model, emb, prompts, SAMPLING, **dict(kw, record=False))[0] == done
    alone = _loop(w, model, emb, prompts[1:2], SAMPLING[1:2], requests=REQUESTS[1:2], **kw)
    for a, b, x, y in zip(alone[1][0], outs[1], alone[0][0], done[1]):
        if not np.array_equal(a, b):               # another batch may take other products: equal outputs, equal draws
            break
        assert x == y


def test_append_attend_sample_in_one_step():
    """The three calls as a step of a model of grouped heads, on one stream and replayed from one graph: new rows
    rotated into the cache, attention over it, and a token drawn per request from outputs of the attention's width."""
    H, KH, dh, page, window, sinks, theta = 8, 2, 64, 16, 40, 3, 10000.0
    lens, ctx, task = np.array([1, 12, 1, 60], np.int32), np.array([130, 0, 55, 20], np.int32), np.zeros(4, np.int32)
    attn = B.make_attn(B.VFM_BF16, H, KH, dh, window=window, n_sink=sinks, rope_theta=theta)
    n_out = H * dh
    pb = B.Batch(task, lens, 1, ctx_len=ctx, n_out=np.array([n_out], np.int32))
    rng = np.random.default_rng(9)
    pages = [-(-int(c + m) // page) for c, m in zip(ctx, lens)]
    table = np.zeros((4, max(pages)), np.int32)
    perm, at = rng.permutation(sum(pages)).astype(np.int32), 0
    for i, n in enumerate(pages):
        table[i, :n] = perm[at:at + n]
        at += n

    def draw(*shape):
        return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16)
    kp, vp, qkv = draw(KH, sum(pages) * page, dh), draw(KH, sum(pages) * page, dh), draw(pb.T, (H + 2 * KH) * dh)
    kv = B.PagedKV(kp.cuda(), vp.cuda(), page, table)
    x, q, out = qkv.cuda(), torch.empty(pb.T, H * dh, dtype=torch.bfloat16, device="cuda"), None
    out = torch.empty_like(q)
    ws = torch.empty(max(1, B.vfm_attention_workspace(attn, pb.c)), dtype=torch.uint8, device="cuda")
    last = torch.from_numpy(np.cumsum(lens) - 1).cuda()          # one task: plan order is the original one
    logits = torch.empty(4 * n_out, device="cuda")
    temp = torch.tensor([1.0, 0.2, 0.0, 2.0], device="cuda")
    top_k = torch.tensor([0, 20, 0, 100], dtype=torch.int32, device="cuda")
    u = torch.tensor([0.3, 0.9, 0.5, 0.1], device="cuda")
    ids, logp = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    params = B.Sampling(temperature=temp, top_k=top_k)

    def step():
        B.vfm_kv_append(attn, pb.c, x, q, kv)
        B.vfm_attention_paged(attn, pb.c, q, kv, out, ws)
        logits.copy_(out[last].float().view(-1) * 30)
        B.vfm_sample_tokens(pb.c, logits, params, u, ids, logp)

    def check():
        rows, o, lg = np64(qkv), np64(out), logits.cpu().numpy().reshape(4, n_out)
        cu = np.concatenate([[0], np.cumsum(lens)])
        eps = 2.0 ** -8
        for i in range(4):
            c, m = int(ctx[i]), int(lens[i])
            r = rows[cu[i]:cu[i + 1]].reshape(m, H + 2 * KH, dh)
            at = lambda t, p: np64(t[:, table[i, p // page].astype(np.int64) * page + p % page]).transpose(1, 0, 2)
            old, pos = np.arange(c), c + np.arange(m)
            qr, kr = D.rotate(r[:, :H], pos, theta), D.rotate(r[:, H:H + KH], pos, theta)
            # one rounding of the rotated values, whose terms are at most |a| + |b|
            assert np.all(np.abs(at(kv.k.cpu(), pos) - kr) <= eps * np.abs(kr) + 2.0 ** -22 * np.abs(r).max())
            assert np.array_equal(at(kv.v.cpu(), pos), r[:, H + KH:])
            q_got = np64(q)[cu[i]:cu[i + 1]].reshape(m, H, dh)
            assert np.all(np.abs(q_got - qr) <= eps * np.abs(qr) + 2.0 ** -22 * np.abs(r).max())
            # the attention's part from the rows that the append left: weights and outputs rounded once each
            ka = np.concatenate([at(kp, old), at(kv.k.cpu(), pos)])
            va = np.concatenate([at(vp, old), r[:, H + KH:]])
            ref, a, n = D.attention(q_got, ka, va, c, window, sinks, dh ** -0.5)
            dot = D.score_sizes(q_got, ka, dh ** -0.5)[:, :, None]
            lim = (eps + (n[:, None, None] + 16) * 2.0 ** -24) * (a + np.abs(ref)) \
                + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
            assert np.all(np.abs(o[cu[i]:cu[i + 1]].reshape(m, H, dh) - ref) <= lim)
            want, lp, gap = D.sample(lg[i], float(temp[i]), int(top_k[i]), 1.0, 0.0, float(u[i]))
            assert gap > 2.0 ** -30 and int(ids[i]) == want and abs(float(logp[i]) - lp) <= 2.0 ** -20 * (1 + abs(lp))

    log("append, attend, sample")
    step()
    torch.cuda.synchronize()
    check()
    first = [t.clone() for t in (out, ids, logp, kv.k, kv.v)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (out, ids, logp, q):
            t.fill_(0)
        kv.k.copy_(kp)
        kv.v.copy_(vp)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip((out, ids, logp, kv.k, kv.v), first):
            assert torch.equal(t, want)


def test_windowed_layer_replayed_from_a_graph():
    """A captured layer replays to the eager bits, with eager work on the same stream between the replays."""
    w = _decoder("bf16", 64)
    lens, ctx, task = np.array([1, 30, 1], np.int32), np.array([80, 10, 300], np.int32), np.array([0, 2, 1], np.int32)
    window, sinks, page = 40, 2, 16
    model = R.Model(w, n_layers=1, b_std=0.1)
    cache = _Cache(w, lens, ctx, page, window, sinks, seed=3)
    cfg = R.cfg_for(w)
    cfg.attn = B.VFM_ATTN_MIXED
    pb = B.Batch(task, lens, w.n_tasks, ctx_len=ctx)
    x0 = torch.from_numpy(np.random.default_rng(8).standard_normal((pb.T, w.d)).astype(np.float32)).cuda()
    ws = torch.empty(B.vfm_workspace_size_windowed(cfg, pb.c, model.lora_c(0), window, sinks), dtype=torch.uint8, device="cuda")
    kv = B.PagedKV(cache.k, cache.v, page, cache.table)
    x = x0.clone()

    def layer():
        B.vfm_layer_forward_windowed(cfg, model.c_layers[0], model.lora_c(0), pb.c, x, kv, window, sinks, ws)
    log("windowed layer in a graph")
    layer()
    torch.cuda.synchronize()
    want, k1, v1 = x.clone(), cache.k.clone(), cache.v.clone()
    assert torch.isfinite(want).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(3):
        x.copy_(x0)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want)
        assert torch.equal(cache.k.view(torch.int16), k1.view(torch.int16))
        assert torch.equal(cache.v.view(torch.int16), v1.view(torch.int16))
        (x0 @ x0.T).sum().item()


@pytest.mark.parametrize("dtype,lens", [("bf16", [1, 1]), ("bf16", [1, 70]), ("f32", [1, 9])])
def test_pages_past_32_bit_offsets_and_shared_by_requests(dtype, lens):
    """A pool whose later elements lie past 2^31 (bytes past 2^32): the step's pages are the pool's last ones, and both
    requests' tables begin with the same pages (a prefix that they share)."""
    code, td, eps = (B.VFM_BF16, torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (B.VFM_F32, torch.float32, 2.0 ** -24)
    H, KH, dh, page = 4, 2, 128, 64
    n_pages = (1 << 18) + 64                                   # 2^24 slots and more of 128 per head
    lens, ctx, task = np.array(lens, np.int32), np.array([150, 200], np.int32), np.zeros(2, np.int32)
    last = n_pages - 1
    table = np.array([[last, last - 3, last - 1, 0, 0], [last, last - 3, last - 2, last - 5, last - 4]], np.int32)
    kp, vp = [torch.empty(KH, n_pages * page, dh, dtype=td, device="cuda") for _ in range(2)]
    rng = np.random.default_rng(17)
    for t in (kp, vp):                                          # the last pages alone are written
        t[:, -8 * page:] = torch.from_numpy(rng.standard_normal((KH, 8 * page, dh))).to(td).cuda()
    attn = B.make_attn(code, H, KH, dh)
    pb = B.Batch(task, lens, 1, ctx_len=ctx)
    qkv = torch.from_numpy(rng.standard_normal((pb.T, (H + 2 * KH) * dh))).to(td).cuda()
    kv = B.PagedKV(kp, vp, page, table)
    q, out = [torch.empty(pb.T, H * dh, dtype=td, device="cuda") for _ in range(2)]
    ws = torch.empty(max(1, B.vfm_attention_workspace(attn, pb.c)), dtype=torch.uint8, device="cuda")
    log(f"far pages {dtype} {lens}")
    B.vfm_kv_append(attn, pb.c, qkv, q, kv)
    B.vfm_attention_paged(attn, pb.c, q, kv, out, ws)
    torch.cuda.synchronize()
    rows, o = np64(qkv), np64(out)
    assert np.array_equal(np64(q), rows[:, :H * dh])            # no rotation: as they were
    at = 0
    for i, (m, c) in enumerate(zip(lens, ctx)):
        pos = np.arange(int(c + m))
        slots = torch.from_numpy(table[i, pos // page].astype(np.int64) * page + pos % page).cuda()
        k, v = np64(kp[:, slots]).transpose(1, 0, 2), np64(vp[:, slots]).transpose(1, 0, 2)
        r = rows[at:at + m].reshape(m, H + 2 * KH, dh)
        assert np.array_equal(k[c:], r[:, H:H + KH]) and np.array_equal(v[c:], r[:, H + KH:])
        ref, a, n = D.attention(r[:, :H], k, v, int(c), 0, 0, dh ** -0.5)
        dot = D.score_sizes(r[:, :H], k, dh ** -0.5)[:, :, None]
        lim = ((eps if dtype == "bf16" else 0.0) + (n[:, None, None] + 16) * 2.0 ** -24) * (a + np.abs(ref)) \
            + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
        assert np.all(np.abs(o[at:at + m].reshape(m, H, dh) - ref) <= lim)
        at += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windowed_layer_long_context_beside_a_prompt(dtype):
    """One row at 12000 with everything visible beside a prompt of 600 rows and a chunk: the step's workspace holds the
    long row's partial results, not the same number for every row."""
    w = _decoder(dtype, 64, d=1024)
    lens, ctx, task = [600, 1, 20], [0, 12000, 50], [1, 0, 2]
    cfg = R.cfg_for(w)
    cfg.attn = B.VFM_ATTN_MIXED

    def size(at):
        pb = B.Batch(np.array(task, np.int32), np.array(lens, np.int32), w.n_tasks, ctx_len=np.array([0, at, 50], np.int32))
        return B.vfm_workspace_size_windowed(cfg, pb.c, None, 0, 0)
    assert size(12000) <= size(100) + (16 << 20)
    _run_layer(w, lens, ctx, task, 64, 0, 0, rows=6)
