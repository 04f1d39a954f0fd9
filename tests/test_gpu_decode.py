"""GPU tests of decoding over a bounded KV cache through the C ABI: the rotary
append, attention with a sliding window and sinks, the draw of next tokens,
against plain 64-bit forms of the same inputs.

Tolerances.  A rounding to a type is off by at most u = finfo(type).eps / 2 of
the value.  Attention: an output is a sum of terms p_k v_k; with a = sum p |v|
and o the exact output, bf16 rounds each weight (u a) and the result (u |o|);
fp32 sums over n keys are off by at most n 2^-24 of their terms' sizes, in the
products and in the sum that divides them; and a score, an fp32 dot product of
dh terms, by (dh + 2) 2^-24 sum |q k|, twice, as the largest one is subtracted
(with the exponential's own 2 ulp).  Their sum is the bound of each element."""
import numpy as np
import pytest
import torch

from paper_2606_09643_amd import binding as B
from tests import decode_common as D
from tests.gpu_common import log
from tests.helpers import np64

pytestmark = pytest.mark.gpu
DT = {"bf16": (B.VFM_BF16, torch.bfloat16, 2.0 ** -8), "f32": (B.VFM_F32, torch.float32, 2.0 ** -24)}


class Cache:
    """A paged cache of requests of ctx[i] + lens[i] tokens: K / V per request
    (host float64, already of the type's values), their pages in random order,
    and everything that no row of its request sees set to `junk`."""

    def __init__(self, lens, ctx, KH, dh, page, window, sinks, dtype, seed, junk=float("nan"), spread=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.ctx, self.page = np.asarray(lens, np.int32), np.asarray(ctx, np.int32), page
        _, td, _ = DT[dtype]
        end = self.lens.astype(np.int64) + self.ctx
        need = -(-end // page)
        total = int(need.sum()) + 2
        perm = rng.permutation(total)
        self.table = np.full((len(lens), int(need.max()) + 1), -1, np.int32)
        pool = [torch.full((KH, total * page, dh), junk, dtype=td) for _ in range(2)]
        self.k, self.v, at = [], [], 0
        for i in range(len(lens)):
            pos = np.arange(end[i])
            rows = np.arange(self.ctx[i], end[i])
            seen = D.visible(rows[:, None], pos[None], window, sinks).any(0) if end[i] <= 20000 else np.ones(end[i], bool)
            pages = perm[at:at + need[i]]
            at += int(need[i])
            for j in range(int(need[i])):                 # a page without any seen key may be anything
                if seen[j * page:(j + 1) * page].any():
                    self.table[i, j] = pages[j]
            slots = torch.from_numpy(pages[pos // page] * page + pos % page)
            for c, (pl, dst) in enumerate(zip(pool, (self.k, self.v))):
                x = torch.from_numpy(rng.standard_normal((end[i], KH, dh)) * (spread if c == 0 else 1.0)).to(td)
                dst.append(np64(x))
                x[~torch.from_numpy(seen)] = junk
                pl[:, slots] = x.permute(1, 0, 2)
        self.kp, self.vp = pool[0].cuda(), pool[1].cuda()
        self.kv = B.PagedKV(self.kp, self.vp, page, self.table)

    def slots(self, i, pos):
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page


def _tasks(n, seed):
    return np.random.default_rng(seed).integers(0, 5, n).astype(np.int32)


def _attend(c, task, H, KH, dh, window, sinks, dtype, q, scale=0.0, only=None, ldo=None, ws_fill=255):
    """out [T, ldo] of the requests `only` (all), rows in plan order; q: per request host float64 [m, H, dh]."""
    code, td, _ = DT[dtype]
    ids = np.arange(len(c.lens)) if only is None else np.asarray(only)
    attn = B.make_attn(code, H, KH, dh, window=window, n_sink=sinks, scale=scale)
    pb = B.Batch(task[ids], c.lens[ids], 5, ctx_len=c.ctx[ids])
    kv = B.PagedKV(c.kp, c.vp, c.page, c.table[ids])
    order = np.argsort(task[ids], kind="stable")
    qd = torch.from_numpy(np.concatenate([q[ids[o]].reshape(-1, H * dh) for o in order])).to(td).cuda()
    out = torch.full((pb.T + 1, ldo or H * dh), 77.0, dtype=td, device="cuda")
    ws = torch.full((max(1, B.vfm_attention_workspace(attn, pb.c)),), ws_fill, dtype=torch.uint8, device="cuda")
    B.vfm_attention_paged(attn, pb.c, qd, kv, out, ws)
    torch.cuda.synchronize()
    assert torch.all(out[pb.T:] == 77) and torch.all(out[:, H * dh:] == 77)
    o = out[:pb.T, :H * dh].float().cpu().numpy().astype(np.float64)
    cu = np.concatenate([[0], np.cumsum(c.lens[ids[order]])])
    return {int(ids[o_]): o[cu[p]:cu[p + 1]].reshape(-1, H, dh) for p, o_ in enumerate(order)}


def _check(c, got, q, window, sinks, dtype, scale):
    _, _, u = DT[dtype]
    worst = 0.0
    for i, o in got.items():
        ref, a, n = D.attention(q[i], c.k[i], c.v[i], int(c.ctx[i]), window, sinks, scale)
        dh = ref.shape[-1]
        dot = D.score_sizes(q[i], c.k[i], scale)[:, :, None]
        nn = n[:, None, None]
        tol = (u if dtype == "bf16" else 0.0) * (a + np.abs(ref)) + (nn + 16) * 2.0 ** -24 * (a + np.abs(ref)) \
            + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
        assert np.isfinite(o).all(), (i, "not finite")
        far = np.abs(o - ref) / tol
        worst = max(worst, float(far.max()))
        assert far.max() <= 1, (i, int(c.lens[i]), int(c.ctx[i]), np.unravel_index(far.argmax(), far.shape), far.max())
    return worst


RAGGED = [(1, 0), (1, 1), (1, 15), (1, 16), (1, 37), (1, 300), (2, 0), (3, 61), (5, 16), (17, 0), (17, 40), (33, 127),
          (64, 0), (70, 250), (130, 3), (1, 1500)]


@pytest.mark.parametrize("dtype,H,KH,dh,page,window,sinks", [
    ("bf16", 2, 2, 128, 64, 0, 0), ("bf16", 2, 2, 64, 16, 0, 0), ("bf16", 4, 1, 128, 16, 50, 3),
    ("bf16", 7, 1, 64, 32, 17, 1), ("bf16", 8, 2, 128, 1024, 64, 64), ("bf16", 8, 1, 64, 64, 1, 0),
    ("bf16", 8, 1, 128, 16, 1, 5), ("bf16", 40, 1, 64, 16, 100, 33), ("bf16", 64, 1, 128, 128, 33, 4),
    ("bf16", 20, 1, 128, 32, 200, 0), ("bf16", 3, 3, 128, 16, 16, 16), ("bf16", 2, 1, 64, 16, 4000, 9),
    ("f32", 2, 2, 128, 64, 0, 0), ("f32", 4, 2, 64, 16, 50, 3), ("f32", 7, 1, 128, 32, 17, 1),
    ("f32", 40, 1, 64, 16, 100, 33), ("f32", 2, 2, 64, 1024, 1, 0)])
def test_attention_ragged(dtype, H, KH, dh, page, window, sinks):
    """Every length and context in one batch: single rows, chunks, prompts;
    pages that end inside tiles, page entries and slots that nothing sees NaN."""
    log(f"attend {dtype} H {H} KH {KH} dh {dh} page {page} window {window} sinks {sinks}")
    lens, ctx = [l for l, _ in RAGGED], [x for _, x in RAGGED]
    c = Cache(lens, ctx, KH, dh, page, window, sinks, dtype, seed=H * dh + window)
    rng = np.random.default_rng(7)
    _, td, _ = DT[dtype]
    q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh)) * 1.5).to(td)) for m in lens]
    task = _tasks(len(lens), 3)
    got = _attend(c, task, H, KH, dh, window, sinks, dtype, q, ldo=H * dh + 8)
    log(f"  {_check(c, got, q, window, sinks, dtype, dh ** -0.5):.3f} of the tolerance")
    # alone and beside others: the same bits
    for only in ([2], [8], [13], [15, 12, 9]):
        alone = _attend(c, task, H, KH, dh, window, sinks, dtype, q, only=only, ws_fill=0)
        for i in only:
            assert np.array_equal(alone[i], got[i]), i


@pytest.mark.parametrize("dtype,H,KH,dh,page,window,sinks,lens,ctx", [
    ("bf16", 4, 1, 128, 64, 0, 0, [1, 1, 3], [9000, 4097, 12000]),
    ("bf16", 2, 2, 64, 16, 3000, 70, [1, 200, 1], [9000, 5000, 3001]),
    ("bf16", 4, 1, 128, 256, 0, 0, [150, 1], [6000, 20000]),
    ("f32", 2, 1, 64, 64, 0, 0, [1, 40], [9000, 5000])])
def test_attention_long_keys_are_cut_and_joined(dtype, H, KH, dh, page, window, sinks, lens, ctx):
    """Long contexts of few heads: the keys go to many blocks and are joined."""
    log(f"long {dtype} H {H} KH {KH} dh {dh} window {window} ctx {ctx}")
    c = Cache(lens, ctx, KH, dh, page, window, sinks, dtype, seed=5)
    rng = np.random.default_rng(8)
    _, td, _ = DT[dtype]
    q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh)) * 1.5).to(td)) for m in lens]
    task = _tasks(len(lens), 4)
    pb = B.Batch(task, c.lens, 5, ctx_len=c.ctx)
    assert B.vfm_attention_workspace(B.make_attn(DT[dtype][0], H, KH, dh, window=window, n_sink=sinks), pb.c) > 0
    got = _attend(c, task, H, KH, dh, window, sinks, dtype, q)
    log(f"  {_check(c, got, q, window, sinks, dtype, dh ** -0.5):.3f} of the tolerance")
    for i in range(len(lens)):
        assert np.array_equal(_attend(c, task, H, KH, dh, window, sinks, dtype, q, only=[i], ws_fill=0)[i], got[i])


@pytest.mark.parametrize("dtype,H,KH,dh", [("bf16", 4, 2, 128), ("bf16", 2, 1, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("lens,ctx,window", [([12], [40], 9), ([100], [70], 30), ([100], [0], 0)])
def test_attention_keys_that_only_some_rows_see(dtype, H, KH, dh, lens, ctx, window):
    """An infinity or a NaN in the V row (and in the K row) of a key reaches the
    rows that see it and no other."""
    c = Cache(lens, ctx, KH, dh, 16, window, 2, dtype, seed=11)
    rng = np.random.default_rng(9)
    _, td, _ = DT[dtype]
    q = [np64(torch.from_numpy(rng.standard_normal((lens[0], H, dh))).to(td))]
    task = np.zeros(1, np.int32)
    clean = _attend(c, task, H, KH, dh, window, 2, dtype, q)[0]
    m, x = lens[0], ctx[0]
    for what, at, val in (("v", x + m // 2, np.inf), ("v", x + m - 2, np.nan), ("k", x + m // 3, np.nan),
                          ("v", max(0, x - 5), -np.inf)):
        slot = int(c.slots(0, np.array([at]))[0])
        pool = c.vp if what == "v" else c.kp
        was = pool[:, slot].clone()
        d = 5
        pool[:, slot, d] = val
        got = _attend(c, task, H, KH, dh, window, 2, dtype, q)[0]
        pool[:, slot] = was
        see = D.visible(x + np.arange(m), at, window, 2)
        assert np.array_equal(got[~see], clean[~see]), (what, at)
        if what == "v":
            bad = got[see][:, :, d]
            assert np.all(np.isnan(bad)) if np.isnan(val) else np.all(bad == val), (what, at)
            others = np.delete(got[see], d, axis=2)
            assert np.array_equal(others, np.delete(clean[see], d, axis=2))
        else:
            assert np.isnan(got[see]).all()


@pytest.mark.parametrize("H,KH,dh,page,window,sinks,lens,ctx", [
    (32, 32, 64, 64, 0, 0, [2050], [0]), (64, 16, 128, 16, 90, 5, [1100, 1, 40], [333, 50, 0]),
    (56, 8, 64, 32, 300, 0, [1300], [70])])
def test_attention_prompts_of_wide_blocks(H, KH, dh, page, window, sinks, lens, ctx):
    """Prompts whose blocks fill the chip: rows at the blocks' and tiles' borders
    and a spread of others against the 64-bit form."""
    assert KH * -(-lens[0] * (H // KH) // 256) >= 256
    c = Cache(lens, ctx, KH, dh, page, window, sinks, "bf16", seed=21)
    rng = np.random.default_rng(12)
    q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh), dtype=np.float32) * 1.5).to(torch.bfloat16)) for m in lens]
    task = _tasks(len(lens), 4)
    got = _attend(c, task, H, KH, dh, window, sinks, "bf16", q)
    worst, m = 0.0, lens[0]
    heads = [0, H // 2 + 1, H - 1]
    for i in sorted({0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 257, m // 2, m - 2, m - 1} | set(rng.integers(0, m, 20).tolist())):
        see = D.visible(ctx[0] + i, np.arange(ctx[0] + m), window, sinks)
        for h in heads:
            k, v = c.k[0][see, h * KH // H], c.v[0][see, h * KH // H]
            p = np.exp((sc := k @ q[0][i, h] * dh ** -0.5) - sc.max())
            p /= p.sum()
            a, ref = p @ np.abs(v), p @ v
            dot = np.abs(q[0][i, h]).max() * np.abs(k).max() * dh ** 0.5
            tol = 2.0 ** -8 * (a + np.abs(ref)) + (see.sum() + 16) * 2.0 ** -24 * (a + np.abs(ref)) \
                + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
            far = np.abs(got[0][i, h] - ref) / tol
            worst = max(worst, float(far.max()))
            assert far.max() <= 1, (i, h, far.max())
    log(f"  {worst:.3f} of the tolerance")
    if len(lens) > 1:
        _check(c, {i: got[i] for i in range(1, len(lens))}, q, window, sinks, "bf16", dh ** -0.5)
    assert np.array_equal(_attend(c, task, H, KH, dh, window, sinks, "bf16", q, only=[0], ws_fill=0)[0], got[0])


@pytest.mark.parametrize("dh,lo,hi", [(64, 100, 700), (64, 1, 100), (128, 100, 700), (128, 1, 100)])
def test_attention_rows_alone_and_among_many(dh, lo, hi):
    """A step of more blocks than the chip holds at once, and rows of it alone: the 64-bit form's, and the same bits."""
    rng = np.random.default_rng(dh + hi)
    ctx = rng.integers(lo, hi, 40).tolist()
    c = Cache([1] * 40, ctx, 16, dh, 16, 0, 0, "bf16", seed=31)
    q = [np64(torch.from_numpy(rng.standard_normal((1, 16, dh), dtype=np.float32)).to(torch.bfloat16)) for _ in ctx]
    task = _tasks(40, 6)
    got = _attend(c, task, 16, 16, dh, 0, 0, "bf16", q)
    _check(c, got, q, 0, 0, "bf16", dh ** -0.5)
    for i in (0, 17, int(np.argmax(ctx)), int(np.argmin(ctx))):
        assert np.array_equal(_attend(c, task, 16, 16, dh, 0, 0, "bf16", q, only=[i], ws_fill=0)[i], got[i])


def test_attention_large_logits_and_scale():
    """Scores of hundreds (one key takes the whole weight) and a given scale."""
    for dtype in ("bf16", "f32"):
        H, KH, dh = 2, 1, 64
        c = Cache([1, 40], [200, 30], KH, dh, 32, 0, 0, dtype, seed=2, spread=8.0)
        rng = np.random.default_rng(1)
        q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh)) * 8).to(DT[dtype][1])) for m in (1, 40)]
        got = _attend(c, np.zeros(2, np.int32), H, KH, dh, 0, 0, dtype, q, scale=0.25)
        # the scores' own rounding is what counts here: 66 2^-24 (sum |q k|) 0.25 each
        log(f"  {dtype}: {_check(c, got, q, 0, 0, dtype, 0.25):.3f} of the tolerance")


def test_attention_rows_of_a_wider_matrix():
    """Queries as the first columns of [T, 3 d] rows, as a layer keeps them."""
    H = KH = 2
    dh = 64
    c = Cache([3, 40], [20, 0], KH, dh, 16, 10, 1, "bf16", seed=3)
    rng = np.random.default_rng(2)
    q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh))).to(torch.bfloat16)) for m in (3, 40)]
    ref = _attend(c, np.zeros(2, np.int32), H, KH, dh, 10, 1, "bf16", q)
    pb = B.Batch(np.zeros(2, np.int32), c.lens, 1, ctx_len=c.ctx)
    wide = torch.full((43, 3 * H * dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :H * dh] = torch.from_numpy(np.concatenate([x.reshape(-1, H * dh) for x in q])).to(torch.bfloat16).cuda()
    out = torch.zeros(43, H * dh, dtype=torch.bfloat16, device="cuda")
    attn = B.make_attn(B.VFM_BF16, H, KH, dh, window=10, n_sink=1)
    B.vfm_attention_paged(attn, pb.c, wide, c.kv, out)
    assert np.array_equal(np64(out).reshape(-1, H, dh), np.concatenate([ref[0], ref[1]]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_replayed_graph_and_other_stream(dtype):
    """A captured call, replayed with eager work between, and a call on another
    stream give the eager call's bits, also with several chunks to join."""
    H, KH, dh = 4, 2, 128
    lens, ctx = [1, 1, 150, 2], [3000, 10, 700, 500]
    c = Cache(lens, ctx, KH, dh, 64, 0, 0, dtype, seed=6)
    rng = np.random.default_rng(3)
    _, td, _ = DT[dtype]
    attn = B.make_attn(DT[dtype][0], H, KH, dh)
    pb = B.Batch(np.zeros(4, np.int32), c.lens, 1, ctx_len=c.ctx)
    qd = torch.from_numpy(rng.standard_normal((pb.T, H * dh))).to(td).cuda()
    ws = torch.empty(B.vfm_attention_workspace(attn, pb.c), dtype=torch.uint8, device="cuda")
    eager = torch.empty_like(qd)
    B.vfm_attention_paged(attn, pb.c, qd, c.kv, eager, ws)
    torch.cuda.synchronize()
    out = torch.zeros_like(qd)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = torch.zeros_like(qd)
        B.vfm_attention_paged(attn, pb.c, qd, c.kv, other, ws)
    s.synchronize()
    assert torch.equal(other, eager)
    with torch.cuda.graph(g):
        B.vfm_attention_paged(attn, pb.c, qd, c.kv, out, ws)
    for i in range(4):
        out.fill_(float(i))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


@pytest.mark.parametrize("dtype,H,KH,dh,page,theta", [
    ("bf16", 2, 2, 128, 64, 10000.0), ("bf16", 7, 1, 64, 16, 500000.0), ("bf16", 4, 2, 128, 32, 0.0),
    ("f32", 4, 2, 64, 16, 10000.0), ("f32", 3, 3, 128, 1024, 1.0)])
def test_append(dtype, H, KH, dh, page, theta):
    """Rotated q and k, copied v, slots of other positions left alone; positions
    up to a million; rows of a wider matrix.  The rotation is one rounding (u)
    of a sum of two products, whose fp32 factors are off by 2^-24 each, angle
    and products by 2^-23 of the terms."""
    lens, ctx = [1, 3, 40, 1, 2, 1], [0, 15, 100, 4095, 1000000 // page * page - 1, 7]
    code, td, u = DT[dtype]
    n, rng = len(lens), np.random.default_rng(4)
    need = [-(-(a + b) // page) for a, b in zip(lens, ctx)]
    table = np.full((n, max(need)), -5, np.int32)           # only the new positions' pages exist
    nxt = 0
    for i in range(n):
        for j in range(ctx[i] // page, need[i]):
            table[i, j] = nxt
            nxt += 1
    perm = rng.permutation(nxt + 2).astype(np.int32)
    table[table >= 0] = perm[table[table >= 0]]
    kp = torch.full((KH, (nxt + 2) * page, dh), 9.0, dtype=td, device="cuda")
    vp = torch.full_like(kp, 8.0)
    kv = B.PagedKV(kp, vp, page, table)
    task = np.array([2, 0, 1, 0, 2, 1], np.int32)
    pb = B.Batch(task, lens, 3, ctx_len=ctx)
    W = (H + 2 * KH) * dh
    host = torch.from_numpy(rng.standard_normal((pb.T, W))).to(td)
    qkv = torch.full((pb.T, W + 16), float("nan"), dtype=td, device="cuda")
    qkv[:, :W] = host.cuda()
    q_out = torch.full((pb.T, H * dh), 7.0, dtype=td, device="cuda")
    attn = B.make_attn(code, H, KH, dh, rope_theta=theta)
    B.vfm_kv_append(attn, pb.c, qkv, q_out, kv)
    order = np.argsort(task, kind="stable")
    at, written = 0, torch.zeros(kp.shape[1], dtype=torch.bool)
    x = np64(host).reshape(pb.T, H + 2 * KH, dh)
    gk, gv, gq = np64(kp), np64(vp), np64(q_out).reshape(pb.T, H, dh)
    for i in order:
        m = lens[i]
        pos = np.arange(ctx[i], ctx[i] + m)
        slots = table[i, pos // page].astype(np.int64) * page + pos % page
        written[torch.from_numpy(slots)] = True
        rows = x[at:at + m]
        ref = D.rotate(rows[:, :H + KH], pos, theta)
        size = np.abs(rows[:, :H + KH])
        size = size + np.roll(size, dh // 2, axis=-1)
        tol = (u * np.abs(ref) if dtype == "bf16" else 0.0) + 4 * 2.0 ** -23 * size if theta else 0 * ref
        assert np.all(np.abs(gq[at:at + m] - ref[:, :H]) <= tol[:, :H]), i
        assert np.all(np.abs(gk[:, slots].transpose(1, 0, 2) - ref[:, H:]) <= tol[:, H:]), i
        assert np.array_equal(gv[:, slots].transpose(1, 0, 2), rows[:, H + KH:])
        at += m
    assert torch.all(kp.cpu()[:, ~written] == 9) and torch.all(vp.cpu()[:, ~written] == 8)


def _draw(rows, temperature=None, top_k=None, top_p=None, min_p=None, u=None, want_logprob=True):
    """ids, logprob of ragged rows of outputs (one task per request)."""
    n = len(rows)
    sizes = np.array([len(r) for r in rows], np.int32)
    pb = B.Batch(np.arange(n, dtype=np.int32)[::-1].copy(), np.ones(n, np.int32), n, n_out=sizes[::-1].copy())
    out = torch.from_numpy(np.concatenate([np.asarray(r, np.float32) for r in rows] + [np.full(3, 1e30, np.float32)])).cuda()
    t = lambda a, d: None if a is None else torch.from_numpy(np.asarray(a, d)).cuda()
    sp = B.Sampling(t(temperature, np.float32), t(top_k, np.int32), t(top_p, np.float32), t(min_p, np.float32))
    ids = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    lp = torch.full((n,), 99.0, dtype=torch.float32, device="cuda") if want_logprob else None
    B.vfm_sample_tokens(pb.c, out, sp, t(u, np.float32), ids, lp)
    return ids.cpu().numpy(), lp.cpu().numpy() if want_logprob else None


def _check_draw(rows, temperature, top_k, top_p, min_p, u):
    """Every draw against the 64-bit form.  A weight is rounded by 2^-45 of the
    largest one, whose weight is 1, so a border of the running sum S >= 1 moves
    by less than n 2^-44 in all; only a target closer than that to one may give
    another output.  logprob: one rounding to fp32 (2^-24), and S off by n 2^-44."""
    ids, lp = _draw(rows, temperature, top_k, top_p, min_p, u)
    for i, r in enumerate(rows):
        r32 = np.asarray(r, np.float32)
        a, l, near = D.sample(r32, np.float32(temperature[i]), top_k[i], np.float32(top_p[i]), np.float32(min_p[i]),
                              np.float32(u[i]))
        room = len(r) * 2.0 ** -44
        if ids[i] != a:
            assert near <= room, (i, len(r), ids[i], a, near, temperature[i], top_k[i], top_p[i], min_p[i], u[i])
            continue
        if np.isnan(l):
            assert np.isnan(lp[i])
        else:
            assert abs(lp[i] - l) <= 2.0 ** -23 * abs(l) + room + 2.0 ** -40, (i, lp[i], l)


SIZES = [1, 2, 3, 5, 64, 255, 256, 257, 1000, 1023, 1024, 1025, 4095, 4096, 4097, 5000, 8193, 32000, 100003]


@pytest.mark.parametrize("spread", [0.05, 2.0, 12.0])
@pytest.mark.parametrize("size", ["small", "middle", "large"])
def test_sample_filters(spread, size):
    """Sizes around the blocks' shapes, every combination of filters."""
    rng = np.random.default_rng(int(spread * 100))
    sizes = {"small": [s for s in SIZES if s <= 1024], "middle": [s for s in SIZES if s <= 4096],
             "large": SIZES}[size]
    rows, par = [], []
    for s in sizes:
        for k in (0, 1, 3, 40, 600, 2000, 10 ** 6):
            for p in (1.0, 0.9, 0.3, 0.999):
                for m in (0.0, 0.05):
                    if rng.random() < (0.45 if s < 5000 else 0.12):
                        rows.append((rng.standard_normal(s) * spread).astype(np.float32))
                        par.append((rng.choice([0.7, 1.0, 2.0]), k, p, m, rng.random()))
    log(f"sample {size} spread {spread}: {len(rows)} rows")
    _check_draw(rows, *[list(x) for x in zip(*par)])


@pytest.mark.parametrize("spread", [0.3, 2.5])
def test_sample_middle_k(spread):
    """A top-k around the sizes of the lists that are put in order, with the other filters tighter or looser."""
    rng = np.random.default_rng(int(spread * 10))
    rows, par = [], []
    for s in (60, 300, 1000, 5000, 40000):
        for k in (55, 56, 57, 64, 100, 199, 256, 257, 513):
            for p, m in ((1.0, 0.0), (0.9, 0.0), (0.999, 0.02), (0.4, 0.02), (1.0, 0.3)):
                rows.append((rng.standard_normal(s) * spread).astype(np.float32))
                par.append((1.0, k, p, m, rng.random()))
    _check_draw(rows, *[list(x) for x in zip(*par)])


def test_sample_ties():
    """Equal outputs, few or thousands: the lowest indexes are kept first."""
    rng = np.random.default_rng(0)
    rows, par = [], []
    for s in (7, 300, 1024, 3000, 9000, 40000):
        for quantum in (0.5, 2.0, 0.0):
            for k, p, m in ((0, 1.0, 0.0), (1, 1.0, 0.0), (max(1, s // 3), 1.0, 0.0), (0, 0.5, 0.0), (0, 0.25, 0.1),
                            (s - 1, 0.7, 0.0), (s // 2 + 1, 0.125, 0.0)):
                l = rng.standard_normal(s)
                l = np.round(l / quantum) * quantum if quantum else np.full(s, 1.25)
                rows.append(l.astype(np.float32))
                par.append((1.0, k, p, m, rng.random()))
    _check_draw(rows, *[list(x) for x in zip(*par)])


def test_sample_close_values():
    """Thousands of different outputs so close that they share a bin, beside far ones."""
    rng = np.random.default_rng(1)
    rows, par = [], []
    for s in (2000, 6000, 50000):
        for k, p in ((s // 3, 1.0), (0, 0.4), (s // 2, 0.3), (1500, 0.9), (0, 1.0)):
            l = (1.0 + 1e-7 * rng.integers(0, 4000, s)).astype(np.float32)
            l[rng.integers(0, s, 5)] = -20.0
            rows.append(l)
            par.append((1.0, k, p, 0.0, rng.random()))
    _check_draw(rows, *[list(x) for x in zip(*par)])


def test_sample_special_values():
    """Masked outputs (lowest value, -inf, NaN), infinities, empty requests, and
    parameters out of range."""
    f = np.finfo(np.float32)
    rng = np.random.default_rng(2)
    x = rng.standard_normal(2000).astype(np.float32)
    low, inf, nan, hole = x.copy(), x.copy(), x.copy(), x.copy()
    low[::2], inf[1::2], nan[::3] = f.min, -np.inf, np.nan
    hole[5:1990] = f.min
    top = x.copy()
    top[[17, 400, 1999]] = np.inf
    rows = [low, inf, nan, hole, top, np.full(50, -np.inf, np.float32), np.full(9, np.nan, np.float32),
            np.zeros(0, np.float32), np.array([f.max, f.min, 0], np.float32), np.array([np.nan, -np.inf, np.nan], np.float32),
            np.array([-0.0, 0.0, -0.0], np.float32)]
    for T, k, p, m in ((1.0, 0, 1.0, 0.0), (1.0, 2, 0.8, 0.0), (0.5, 0, 0.9, 0.01), (1e-30, 0, 1.0, 0.0),
                       (1e30, 0, 0.5, 0.0), (np.inf, 3, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (-1.0, 5, 0.5, 0.5),
                       (np.nan, 0, 1.0, 0.0), (1.0, -3, np.nan, np.nan), (1.0, 0, 0.0, 0.0), (1.0, 0, -1.0, 0.0),
                       (1.0, 0, 1.0, 1.0), (1.0, 0, 1.0, 2.0), (1.0, 0, 2.0, -1.0)):
        for u in (0.0, 0.37, float(np.float32(1) - np.float32(2) ** -24), 1.0, 5.0, -0.5, np.nan):
            n = len(rows)
            ids, lp = _draw(rows, [T] * n, [k] * n, [p] * n, [m] * n, [u] * n)
            for i, r in enumerate(rows):
                a, l, near = D.sample(r, np.float32(T), k, np.float32(p), np.float32(m), u)
                assert ids[i] == a or near <= len(r) * 2.0 ** -44, (i, T, k, p, m, u, ids[i], a, near)
                if ids[i] == a:
                    assert np.isnan(lp[i]) if np.isnan(l) else abs(lp[i] - l) <= 2.0 ** -22 * abs(l) + 1e-9, (i, lp[i], l)


def test_sample_defaults_and_greedy():
    """No parameters: the plain softmax; temperature 0 is vfm_greedy_tokens."""
    rng = np.random.default_rng(3)
    rows = [rng.standard_normal(s).astype(np.float32) for s in (10, 700, 5000)]
    u = [0.2, 0.9, 0.5]
    ids, lp = _draw(rows, u=u)
    for i, r in enumerate(rows):
        a, l, _ = D.sample(r, 1.0, 0, 1.0, 0.0, np.float32(u[i]))
        assert ids[i] == a and abs(lp[i] - l) <= 2.0 ** -23 * abs(l) + 1e-9
    ids, _ = _draw(rows, temperature=[0.0] * 3, u=u, want_logprob=False)
    assert ids.tolist() == [int(r.argmax()) for r in rows]


def test_sample_frequencies():
    """Evenly spaced numbers give every output its share (to one number a border)."""
    w = np.array([1.0, 2.0, 4.0, 1.0, 8.0])
    n = 1600
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    ids, _ = _draw([np.log(w)] * n, temperature=[1.0] * n, u=u)
    assert np.all(np.abs(np.bincount(ids, minlength=5) - n * w / w.sum()) <= 2)


def test_sample_replayed_graph():
    rng = np.random.default_rng(5)
    sizes = np.array([50, 3000, 40000], np.int32)
    pb = B.Batch(np.arange(3, dtype=np.int32), np.ones(3, np.int32), 3, n_out=sizes)
    out = torch.from_numpy(rng.standard_normal(int(sizes.sum())).astype(np.float32)).cuda()
    sp = B.Sampling(top_k=torch.tensor([5, 0, 40], dtype=torch.int32, device="cuda"),
                    top_p=torch.tensor([1.0, 0.9, 0.8], device="cuda"))
    u = torch.zeros(3, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    B.vfm_sample_tokens(pb.c, out, sp, u, ids)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        B.vfm_sample_tokens(pb.c, out, sp, u, ids)
    for val in (0.1, 0.5, 0.9, 0.3):
        u.fill_(val)
        eager = torch.empty_like(ids)
        B.vfm_sample_tokens(pb.c, out, sp, u, eager)
        ids.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, eager)


@pytest.mark.parametrize("dtype,H,KH,dh", [("bf16", 4, 2, 128), ("bf16", 2, 1, 64), ("f32", 4, 2, 64), ("f32", 2, 1, 128)])
@pytest.mark.parametrize("sign,power", [(-1, 101), (1, 101), (-1, 33), (1, 33), (-1, 110), (1, 120)])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_attention_scores_of_any_size(dtype, H, KH, dh, sign, power, window):
    """Scores of 2^33 to 2^122, all of one sign.  Queries and keys have one dim that is not 0, so a score is one
    product of two short numbers, exact in fp32; two scores are equal or differ by 2^(power - 8) and more, of which
    2^23 times the scale still puts every weight but the largest ones' below 2^-1000.  An output is then the mean of
    the V rows with the largest score: one V row, bit for bit, or the mean of n, whose weights 1 are exact, off by
    the n additions, the division and the type's rounding."""
    _, td, u = DT[dtype]
    lens, ctx = [1, 1, 90, 3, 1], [60, 0, 200, 5000, 7000]
    c = Cache(lens, ctx, KH, dh, 16, window, 0, dtype, seed=4)
    rng = np.random.default_rng(power)
    steps = [rng.integers(128, 256, (n, KH)) for n in c.lens + c.ctx]     # 8 bits each
    for i, st in enumerate(steps):
        pos = np.arange(len(st))
        k = torch.zeros(KH, len(st), dh, dtype=td)
        k[:, :, 3] = torch.from_numpy((sign * st * 2.0 ** (power // 2 - 8)).T).to(td)
        there = c.table[i, pos // 16] >= 0
        c.kp[:, torch.from_numpy(c.slots(i, pos)[there]).cuda()] = k[:, torch.from_numpy(there)].cuda()
    q = [np.zeros((m, H, dh)) for m in lens]
    for x in q:
        x[:, :, 3] = 2.0 ** (power - power // 2)
    got = _attend(c, np.zeros(5, np.int32), H, KH, dh, window, 0, dtype, q)
    for i, m in enumerate(lens):
        for r in range(m):
            see = D.visible(ctx[i] + r, np.arange(ctx[i] + m), window, 0)
            for h in range(H):
                s = sign * steps[i][:, h * KH // H]
                best = see & (s == s[see].max())
                v, n = c.v[i][best, h * KH // H], int(best.sum())
                ref = v.mean(0)
                tol = 0.0 if n == 1 else (u if dtype == "bf16" else 0.0) * np.abs(ref) \
                    + 2 * (n + 2) * 2.0 ** -24 * np.abs(v).sum(0) / n
                assert np.all(np.abs(got[i][r, h] - ref) <= tol), (i, r, h, n, np.abs(got[i][r, h] - ref).max())


def _width(n):
    """Fixed-point bits of a weight in a row of n outputs: as many as 64-bit sums of n of them hold, at most 44."""
    return min(44, 63 - max(0, int(n - 1).bit_length()))


LARGE = [262143, 262144, 262145, 300000, 2 ** 19 - 1, 2 ** 19, 2 ** 19 + 1, 1000003, 2 ** 20 + 5]


@pytest.mark.parametrize("n", LARGE)
def test_sample_large_heads(n):
    """Rows whose pieces have more than 64 runs, around the sizes at which weights get fewer bits, every kind of
    filter, numbers u that land early and late.  A weight rounded by 2^-(s + 1) of the largest moves a border of the
    running sum S >= 1, and u S, by n 2^-(s + 1) each at most: a target farther than n 2^-s S from every border
    gives the 64-bit form's output."""
    rng = np.random.default_rng(n)
    x = (rng.standard_normal(n) * 2).astype(np.float32)
    par = [(1.0, 0, 1.0, 0.0, 0.9995), (0.8, 0, 1.0, 0.0, 0.013), (1.0, 0, 0.9, 0.0, 0.51), (1.3, 0, 1.0, 0.01, 0.98),
           (1.0, 150000, 1.0, 0.0, 0.77), (1.0, 150000, 0.8, 0.0, 0.999), (1.0, 3000, 0.95, 0.002, 0.3),
           (1.0, 40, 1.0, 0.0, 0.6), (0.0, 0, 1.0, 0.0, 0.5), (1.0, 0, 0.4, 0.0, float(np.float32(1) - np.float32(2) ** -24))]
    ids, lp = _draw([x] * len(par), *[list(c) for c in zip(*par)])
    room = n * 2.0 ** -_width(n)
    for i, (T, k, p, m, u) in enumerate(par):
        a, l, near = D.sample(x, np.float32(T), k, np.float32(p), np.float32(m), np.float32(u))
        assert ids[i] == a or near <= room, (i, ids[i], a, near)
        if ids[i] == a:
            assert abs(lp[i] - l) <= 2.0 ** -23 * abs(l) + room + 2.0 ** -40, (i, lp[i], l)


@pytest.mark.parametrize("n", LARGE)
@pytest.mark.parametrize("gap", [21.5, 22.9, 0.0])
def test_sample_large_flat_tails(n, gap):
    """One output at 0 and all others `gap` below it: each of them is next to nothing, together they are up to 5e-4
    of the sum, or with gap 0 all of it, 2^63 units.  The drawn output's stretch of the exact running sum holds u S up
    to the rounding of the weights, all of them by the same e <= 2^-(s + 1): n e at most.  logprob is off by fp32's
    rounding and by n e / S.  A top-p border in the tail moves by as much and by one weight."""
    s, T = _width(n), 1.0
    x = np.full(n, -gap, np.float32)
    x[n // 3] = 0.0
    tail = float(np.exp(np.float64(x[0])))
    room = n * 2.0 ** -(s + 1)
    w = np.full(n, tail)
    w[n // 3] = 1.0
    c = np.cumsum(w)
    S = float(c[-1])
    us = [1e-6, 2e-5, 0.3, 1 - 2e-5, 1 - 1e-6, float(np.float32(1) - np.float32(2) ** -24)]
    ids, lp = _draw([x] * len(us), [T] * len(us), u=us)
    for i, u in enumerate(us):
        t = float(np.float32(u)) * S
        a = int(ids[i])
        assert c[a] - w[a] - 2 * room <= t <= c[a] + 2 * room, (u, a, c[a] - w[a], t, room)
        ref = np.log(w[a] / S)
        assert abs(lp[i] - ref) <= 2.0 ** -23 * abs(ref) + room / S + 2.0 ** -40, (u, lp[i], ref)
    # top-p: half of the tail stays, by index
    if gap:
        p = float(np.float32(1 - 0.5 * (S - 1) / S))
        keep = np.zeros(n, bool)
        keep[n // 3] = True
        m = int(np.ceil((p * S - 1) / tail))
        keep[np.delete(np.arange(n), n // 3)[:m]] = True
        wk = np.where(keep, w, 0.0)
        ck = np.cumsum(wk)
        ids, lp = _draw([x] * len(us), [T] * len(us), top_p=[p] * len(us), u=us)
        for i, u in enumerate(us):
            a, t = int(ids[i]), float(np.float32(u)) * ck[-1]
            assert ck[a] - w[a] - 4 * room - tail <= t <= ck[a] + 4 * room + tail, (u, a, ck[a], t, room)
            ref = np.log(w[a] / ck[-1])
            assert abs(lp[i] - ref) <= 2.0 ** -23 * abs(ref) + 3 * room + tail, (u, lp[i], ref)


@pytest.mark.parametrize("dtype,H,KH,dh,window,lens,ctx", [
    ("bf16", 8, 1, 128, 0, [1] * 130, [20, 30000] + [40] * 127 + [9000]),
    ("bf16", 32, 8, 64, 0, [700, 1, 2, 40], [0, 20000, 100, 9000]),
    ("bf16", 32, 8, 128, 0, [5, 600, 1, 1], [30000, 10, 700, 12000]),
    ("bf16", 16, 16, 64, 6000, [1] * 600 + [33], [90] * 599 + [20000, 9000]),
    ("f32", 4, 2, 64, 0, [900, 1, 30], [0, 15000, 6000]), ("f32", 16, 2, 128, 0, [300, 2], [10, 12000])])
def test_attention_long_contexts_beside_others(dtype, H, KH, dh, window, lens, ctx):
    """Steps whose blocks and records, as rectangles over the longest request's chunks, would be mostly empty: every
    request has the bits that it has alone, the long ones the 64-bit form's values, and the workspace is that of
    the requests; replayed from a graph the same."""
    log(f"long beside others {dtype} H {H} KH {KH} dh {dh} {len(lens)} requests")
    c = Cache(lens, ctx, KH, dh, 64, window, 2 if window else 0, dtype, seed=13)
    rng = np.random.default_rng(14)
    code, td, _ = DT[dtype]
    sinks = 2 if window else 0
    q = [np64(torch.from_numpy(rng.standard_normal((m, H, dh), dtype=np.float32)).to(td)) for m in lens]
    n = len(lens)
    task = _tasks(n, 5)
    attn = B.make_attn(code, H, KH, dh, window=window, n_sink=sinks)
    pb = B.Batch(task, c.lens, 5, ctx_len=c.ctx)
    size = B.vfm_attention_workspace(attn, pb.c)
    got = _attend(c, task, H, KH, dh, window, sinks, dtype, q)
    order = np.argsort(ctx)
    some = sorted({0, 1, min(2, n - 1), n - 2, n - 1, int(order[-1]), int(order[-2]), int(np.argmax(lens))})
    alone = 0
    for i in some:
        pi = B.Batch(task[i:i + 1], c.lens[i:i + 1], 5, ctx_len=c.ctx[i:i + 1])
        alone += B.vfm_attention_workspace(attn, pi.c)
        assert np.array_equal(_attend(c, task, H, KH, dh, window, sinks, dtype, q, only=[i], ws_fill=0)[i], got[i]), i
    assert 0 < size <= 2 * alone + (16 << 20) + 1024 + 64 * (n + 1)
    few = {i: got[i] for i in some if lens[i] <= 5 or ctx[i] > 1000}
    log(f"  {_check(c, few, q, window, sinks, dtype, dh ** -0.5):.3f} of the tolerance")
    by = np.argsort(task, kind="stable")
    qd = torch.from_numpy(np.concatenate([q[o].reshape(-1, H * dh) for o in by])).to(td).cuda()
    eager, out = torch.empty_like(qd), torch.zeros_like(qd)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    B.vfm_attention_paged(attn, pb.c, qd, c.kv, eager, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.vfm_attention_paged(attn, pb.c, qd, c.kv, out, ws)
    for i in range(3):
        out.fill_(float(i))
        ws.fill_(170 + i)
        (qd.float() @ qd[:1].float().T).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


def test_attention_of_a_step_that_fills_a_launch():
    """300000 single rows beside a prompt, 32 heads of 64: 9.6 million blocks, which as rectangles with the prompt's
    would be more than a launch holds.  All requests read the same page, so every row has the bits of one alone."""
    H = KH = 32
    dh, page, n = 64, 16, 300000
    rng = np.random.default_rng(3)
    kp, vp = [torch.from_numpy(rng.standard_normal((KH, 5 * page, dh), dtype=np.float32)).to(torch.bfloat16).cuda() for _ in range(2)]
    attn = B.make_attn(B.VFM_BF16, H, KH, dh)
    row = torch.from_numpy(rng.standard_normal((65, H * dh), dtype=np.float32)).to(torch.bfloat16).cuda()

    def run(lens, ctx, q):
        lens, ctx = np.asarray(lens, np.int32), np.asarray(ctx, np.int32)
        pb = B.Batch(np.zeros(len(lens), np.int32), lens, 1, ctx_len=ctx)
        table = np.zeros((len(lens), 5), np.int32)
        table[-1] = np.arange(5)
        ws = torch.empty(max(1, B.vfm_attention_workspace(attn, pb.c)), dtype=torch.uint8, device="cuda")
        out = torch.full_like(q, 9.0)
        B.vfm_attention_paged(attn, pb.c, q, B.PagedKV(kp, vp, page, table), out, ws)
        torch.cuda.synchronize()
        return out, ws.numel()
    log("a step that fills a launch")
    one, _ = run([1, 64], [15, 0], row)
    many, size = run([1] * n + [64], [15] * n + [0], torch.cat([row[:1].expand(n, -1), row[1:]]))
    assert size >= 16 * (n + 2)
    assert torch.equal(many[:n], one[:1].expand(n, -1)) and torch.equal(many[n:], one[1:])
    k, v = [np64(t[:, :page]).transpose(1, 0, 2) for t in (kp, vp)]
    q = np64(row[:1]).reshape(1, H, dh)
    ref, a, _ = D.attention(q, k, v, page - 1, 0, 0, dh ** -0.5)
    dot = D.score_sizes(q, k, dh ** -0.5)[:, :, None]
    tol = 2.0 ** -8 * (a + np.abs(ref)) + (page + 16) * 2.0 ** -24 * (a + np.abs(ref)) + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
    assert np.all(np.abs(np64(one[:1]).reshape(1, H, dh) - ref) <= tol)
