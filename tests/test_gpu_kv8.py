"""GPU tests of decoding over an 8-bit cache through the C ABI: the append's scales and codes, and attention over them,
against plain 64-bit forms of the same inputs.

Tolerances.  Append: a scale and a code are one rounding of the rotated 64-bit value.  Its angle is pos theta^(-2i/dh): the
exponent's argument (up to 19 in base 2, 13.2 in base e) is a product of two rounded numbers, so the power is off by
2 * 19 ln 2 = 27 2^-53 in one form and 2 * 13.2 = 27 in the other, each with 4 roundings more: the two angles by less
than 64 2^-53 pos, the values by that times the pair's size.  q is off by that and one rounding to its type (u =
finfo(type).eps / 2).  Codes and scales are equal: a value that close to a tie is not among these inputs.
Attention: the cache's numbers are exact in bf16 and fp32, so the bound is that of the bf16 / fp32 cache's attention: with
a = sum p |v| and o the exact output, bf16 rounds each weight (u a) and the result (u |o|); fp32 sums over n keys are off by
n 2^-24 of their terms' sizes, in the products and in the sum that divides them, and a score by (dh + 2) 2^-24
sum |q k|, twice, with the exponential's own 2 ulp."""
import numpy as np
import pytest
import torch

from paper_2606_09643_amd import binding as B
from tests import decode_common as D
from tests import kv8_common as K
from tests.gpu_common import log
from tests.helpers import np64
from tests.test_gpu_decode import DT, RAGGED, _check, _tasks

pytestmark = pytest.mark.gpu
JUNK = 0x7F                                              # NaN


class Cache8:
    """An 8-bit paged cache of requests of ctx[i] + lens[i] tokens: numbers k / v per request (host float64), their
    pages in random order, everything that no row of its request sees NaN codes (scales of such runs 255)."""

    def __init__(self, lens, ctx, KH, dh, page, window, sinks, seed, spread=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.ctx, self.page, self.KH, self.dh = np.asarray(lens, np.int32), np.asarray(ctx, np.int32), page, KH, dh
        end = self.lens.astype(np.int64) + self.ctx
        need = -(-end // page)
        total = int(need.sum()) + 2
        perm = rng.permutation(total)
        self.table = np.full((len(lens), int(need.max()) + 1), -1, np.int32)
        pool = [np.full((KH, total * page, dh), JUNK, np.uint8) for _ in range(2)]
        exps = np.full((total * page // 16, KH, 2), 255, np.uint8)
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
            slots = pages[pos // page] * page + pos % page
            runs = np.unique(pos[seen] // 16)
            for c, dst in enumerate((self.k, self.v)):
                e = rng.integers(117, 123, (-(-end[i] // 16), KH)) + (int(round(np.log2(spread))) if c == 0 else 0)
                codes = K.to_codes(np.clip(rng.standard_normal((end[i], KH, dh), dtype=np.float32) * 90, -448, 448))
                dst.append(K.VALUES[codes] * 2.0 ** (e[pos // 16] - 127.0)[..., None])
                codes[~seen] = JUNK
                pool[c][:, slots] = codes.transpose(1, 0, 2)
                exps[slots[runs * 16] // 16, :, c] = e[runs]
        self.kp, self.vp, self.exps = (torch.from_numpy(x).cuda() for x in (*pool, exps))
        self.kv = B.PagedKVQ8(self.kp, self.vp, self.exps, page, self.table)

    def slots(self, i, pos):
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page


def _queries(lens, H, dh, dtype, seed, std=1.5):
    rng = np.random.default_rng(seed)
    return [np64(torch.from_numpy(rng.standard_normal((m, H, dh), dtype=np.float32) * std).to(DT[dtype][1])) for m in lens]


def _attend(c, task, H, KH, dh, window, sinks, dtype, q, scale=0.0, only=None, ldo=None, ws_fill=255):
    """Outputs of the requests `only` (all) by request; q: per request host float64 [m, H, dh]."""
    code, td, _ = DT[dtype]
    ids = np.arange(len(c.lens)) if only is None else np.asarray(only)
    attn = B.make_attn(code, H, KH, dh, window=window, n_sink=sinks, scale=scale)
    pb = B.Batch(task[ids], c.lens[ids], 5, ctx_len=c.ctx[ids])
    kv = B.PagedKVQ8(c.kp, c.vp, c.exps, c.page, c.table[ids])
    order = np.argsort(task[ids], kind="stable")
    qd = torch.from_numpy(np.concatenate([q[ids[o]].reshape(-1, H * dh) for o in order])).to(td).cuda()
    out = torch.full((pb.T + 1, ldo or H * dh), 77.0, dtype=td, device="cuda")
    ws = torch.full((max(1, B.vfm_attention_workspace_q8(attn, pb.c)),), ws_fill, dtype=torch.uint8, device="cuda")
    B.vfm_attention_paged_q8(attn, pb.c, qd, kv, out, ws)
    torch.cuda.synchronize()
    assert torch.all(out[pb.T:] == 77) and torch.all(out[:, H * dh:] == 77)
    o = out[:pb.T, :H * dh].float().cpu().numpy().astype(np.float64)
    cu = np.concatenate([[0], np.cumsum(c.lens[ids[order]])])
    return {int(ids[o_]): o[cu[p]:cu[p + 1]].reshape(-1, H, dh) for p, o_ in enumerate(order)}


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
class Pool8:
    """An 8-bit cache that appends go to, on the device and as 64-bit forms per request and head: junk throughout but for
    the ctx[i] tokens that request i has."""

    def __init__(self, ctx, room, KH, dh, page, seed):
        rng = np.random.default_rng(seed)
        n = len(ctx)
        self.page, self.KH, self.dh = page, KH, dh
        need = [-(-r // page) for r in room]
        self.table = np.full((n, max(need)), -5, np.int32)
        used = [(i, j) for i in range(n) for j in range(ctx[i] // page, need[i])]   # only the new positions' pages exist
        perm = rng.permutation(len(used) + 2)
        for (i, j), pg in zip(used, perm):
            self.table[i, j] = pg
        slots = (len(used) + 2) * page
        self.codes = [rng.integers(0, 256, (KH, slots, dh)).astype(np.uint8) for _ in range(2)]
        self.exps = rng.integers(0, 256, (slots // 16, KH, 2)).astype(np.uint8)
        for i in range(n):                                # the runs that rows of the sequence are in
            if ctx[i] % 16:
                run = np.arange(ctx[i] // 16 * 16, ctx[i])
                s = self.slots(i, run)
                self.exps[s[0] // 16] = rng.integers(110, 128, (KH, 2))
                for p in self.codes:
                    p[:, s] = K.to_codes(np.clip(rng.standard_normal((KH, len(run), dh)) * 100, -448, 448))
        self.kp, self.vp, self.ep = (torch.from_numpy(x.copy()).cuda() for x in (*self.codes, self.exps))
        self.kv = B.PagedKVQ8(self.kp, self.vp, self.ep, page, self.table)

    def slots(self, i, pos):
        return self.table[i, pos // self.page].astype(np.int64) * self.page + pos % self.page

    def append(self, i, ctx, k, v):
        """The 64-bit forms of request i's step: rows k, v [m, KH, dh] (rotated) after ctx tokens."""
        m = len(k)
        first = ctx // 16 * 16
        pos = np.arange(first, -(-(ctx + m) // 16) * 16)
        s = self.slots(i, pos)
        for c, rows in enumerate((k, v)):
            for h in range(self.KH):
                codes, exps = self.codes[c][h, s], self.exps[s[::16] // 16, h, c]
                K.append(codes, exps, rows[:, h], np.arange(ctx, ctx + m) - first, ctx - first)
                self.codes[c][h, s], self.exps[s[::16] // 16, h, c] = codes, exps

    def check(self):
        """The device's scales and codes against the forms', slots that nothing was written to among them."""
        assert np.array_equal(self.ep.cpu().numpy(), self.exps)
        for got, want, c in ((self.kp, self.codes[0], "k"), (self.vp, self.codes[1], "v")):
            got = got.cpu().numpy()
            differ = (got != want) & ~(np.isnan(K.VALUES[got]) & np.isnan(K.VALUES[want]))
            assert not differ.any(), (c, int(differ.sum()), np.argwhere(differ)[:4])


def _step(pool, task, lens, ctx, H, KH, dh, dtype, theta, x, wide=16):
    """One append of rows x [T, H + 2 KH, dh] (host, plan order), as views of wider rows; q_out [T, H, dh]."""
    code, td, _ = DT[dtype]
    pb = B.Batch(task, lens, int(max(task)) + 1, ctx_len=ctx)
    W = (H + 2 * KH) * dh
    qkv = torch.full((pb.T, W + wide), float("nan"), dtype=td, device="cuda")
    qkv[:, :W] = x.reshape(pb.T, W).cuda()
    q_out = torch.full((pb.T, H * dh), 7.0, dtype=td, device="cuda")
    B.vfm_kv_append_q8(B.make_attn(code, H, KH, dh, rope_theta=theta), pb.c, qkv, q_out, pool.kv)
    return np64(q_out).reshape(pb.T, H, dh)


def _follow(pool, task, lens, ctx, H, KH, theta, x, q_out, u):
    """The forms of that step; q_out against its form."""
    order, at, x = np.argsort(task, kind="stable"), 0, np64(x)
    for i in order:
        m = lens[i]
        q, k, v = K.rotated(x[at:at + m], H, KH, np.arange(ctx[i], ctx[i] + m), theta)
        pool.append(i, ctx[i], k, v)
        size = np.abs(x[at:at + m, :H])
        size = size + np.roll(size, size.shape[-1] // 2, axis=-1)
        far = 64 * 2.0 ** -53 * np.arange(ctx[i], ctx[i] + m)[:, None, None] * size + 4 * 2.0 ** -53 * size
        assert np.all(np.abs(q_out[at:at + m] - q) <= u * (np.abs(q) + far) + far), i
        at += m


@pytest.mark.parametrize("dtype,H,KH,dh,page,theta", [
    ("bf16", 2, 2, 128, 64, 10000.0), ("bf16", 7, 1, 64, 16, 500000.0), ("bf16", 4, 2, 128, 32, 0.0),
    ("bf16", 5, 5, 64, 128, 10000.0), ("f32", 4, 2, 64, 16, 10000.0), ("f32", 3, 3, 128, 1024, 1.0)])
def test_append(dtype, H, KH, dh, page, theta):
    """Steps one after another: single rows, chunks, rows behind others in a run, far positions; rows of sizes that make
    scales grow; whatever lies in slots that are not the sequence's takes no part and stays."""
    log(f"append8 {dtype} H {H} KH {KH} dh {dh} page {page} theta {theta}")
    rng = np.random.default_rng(H + dh)
    td, u = DT[dtype][1:]
    ctx = [0, 15, 100, 4095, 1000000 // page * page - 1, 7, 31]
    steps = [[1, 3, 40, 1, 2, 1, 17], [1] * 7, [2, 16, 1, 15, 33, 1, 1], [1] * 7]
    pool = Pool8(ctx, [c + sum(s[i] for s in steps) + 16 for i, c in enumerate(ctx)], KH, dh, page, 4)
    task = np.array([2, 0, 1, 0, 2, 1, 1], np.int32)
    for lens in steps:
        T = sum(lens)
        x = torch.from_numpy(rng.standard_normal((T, H + 2 * KH, dh)) * 4.0 ** rng.integers(-3, 4, (T, 1, 1))).to(td)
        q = _step(pool, task, lens, ctx, H, KH, dh, dtype, theta, x)
        _follow(pool, task, lens, ctx, H, KH, theta, x, q, u)
        pool.check()
        ctx = [c + m for c, m in zip(ctx, lens)]


@pytest.mark.parametrize("dtype,H,KH,dh", [("bf16", 3, 1, 128), ("f32", 2, 2, 64)])
def test_append_of_a_step_with_many_rows(dtype, H, KH, dh):
    """Prompts, a chunk, single rows, runs cut at either end."""
    rng = np.random.default_rng(8)
    td, u = DT[dtype][1:]
    lens, ctx = [1500, 1, 777, 16, 15, 1, 33, 2], [0, 5, 100, 16, 1, 64, 47, 15]
    task = np.array([1, 0, 1, 2, 0, 2, 0, 0], np.int32)
    pool = Pool8(ctx, [a + b + 16 for a, b in zip(lens, ctx)], KH, dh, 64, 5)
    T = sum(lens)
    x = torch.from_numpy(rng.standard_normal((T, H + 2 * KH, dh), dtype=np.float32)).to(td)
    q = _step(pool, task, lens, ctx, H, KH, dh, dtype, 10000.0, x, wide=0)
    _follow(pool, task, lens, ctx, H, KH, 10000.0, x, q, u)
    pool.check()


@pytest.mark.parametrize("dtype,H,KH,dh", [("bf16", 2, 1, 128), ("bf16", 3, 3, 64), ("f32", 1, 1, 128)])
@pytest.mark.parametrize("most", [2, 5, 20])
def test_append_of_a_step_with_many_short_requests(dtype, H, KH, dh, most):
    """Requests of a few rows each around the ends of runs: several runs begin in 16 rows of the batch."""
    rng = np.random.default_rng(most)
    td, u = DT[dtype][1:]
    lens = [int(n) for n in rng.integers(1, most + 1, 70)]
    ctx = [16 * int(c) + int(r) for c, r in zip(rng.integers(0, 30, 70), rng.integers(12, 18, 70))]
    pool = Pool8(ctx, [a + b + 16 for a, b in zip(lens, ctx)], KH, dh, 16, most)
    T = sum(lens)
    x = torch.from_numpy(rng.standard_normal((T, H + 2 * KH, dh), dtype=np.float32)).to(td)
    task = rng.integers(0, 5, 70).astype(np.int32)
    q = _step(pool, task, lens, ctx, H, KH, dh, dtype, 10000.0, x)
    _follow(pool, task, lens, ctx, H, KH, 10000.0, x, q, u)
    pool.check()


def test_append_of_two_requests_to_one_run():
    """Either's scale and codes of either are there, and nothing beside them is touched."""
    H, KH, dh = 2, 2, 64
    rng = np.random.default_rng(3)
    lens, x = [5, 3], torch.from_numpy(rng.standard_normal((8, H + 2 * KH, dh)) * np.repeat([1.0, 100.0], [5, 3])[:, None, None]).to(torch.bfloat16)
    pools = [Pool8([0, 0], [32, 32], KH, dh, 32, 4) for _ in range(3)]
    both = pools[2]
    table = both.table.copy()
    table[1] = table[0]
    both.kv = B.PagedKVQ8(both.kp, both.vp, both.ep, both.page, table)
    _step(both, np.zeros(2, np.int32), lens, [0, 0], H, KH, dh, "bf16", 0.0, x)
    for i, pool in enumerate(pools[:2]):                  # each alone on those pages
        rows = np64(x)[:5] if i == 0 else np64(x)[5:]
        _, k, v = K.rotated(rows, H, KH, np.arange(lens[i]), 0.0)
        pool.append(0, 0, k, v)
    for got, c in ((both.kp, 0), (both.vp, 1)):
        got = got.cpu().numpy()
        assert np.all((got == pools[0].codes[c]) | (got == pools[1].codes[c]))
    got = both.ep.cpu().numpy()
    assert np.all((got == pools[0].exps) | (got == pools[1].exps))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("theta", [0.0, 10000.0])
def test_append_special_values(dtype, theta):
    """Zeros, infinities and NaN, values near the types' ends and below e4m3's subnormals, values on the scales' borders."""
    H = KH = 1
    dh, td = 64, DT[dtype][1]
    big, tiny = float(torch.finfo(td).max), float(torch.finfo(td).tiny)
    rows = np.zeros((12, 3, dh))
    rows[1] = 448.0
    rows[2] = 1.75
    rows[3, :, :3] = np.inf, -np.inf, 1.0
    rows[4, :, 5] = np.nan
    rows[4, :, 6] = 3.0
    rows[5] = big
    rows[5, :, 1] = -big
    rows[6] = tiny
    rows[7] = np.nan
    rows[8, :, :8] = 448.0, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, -21.0
    rows[9] = -0.0
    rows[10, :, ::2] = 1e30
    rows[11] = 449.0
    x = torch.from_numpy(rows).to(td)
    for r in range(12):                                   # each alone in its run, then all behind each other in one
        pool = Pool8([0], [32], KH, dh, 16, r)
        _step(pool, np.zeros(1, np.int32), [1], [0], H, KH, dh, dtype, theta, x[r:r + 1])
        with np.errstate(invalid="ignore", over="ignore"):
            _, k, v = K.rotated(np64(x[r:r + 1]), H, KH, np.array([0]), theta)   # an infinity times the sine 0: NaN
        pool.append(0, 0, k, v)
        pool.check()
    pool = Pool8([0], [32], KH, dh, 16, 40)
    for r in range(12):
        _step(pool, np.zeros(1, np.int32), [1], [r], H, KH, dh, dtype, theta, x[r:r + 1])
        with np.errstate(invalid="ignore", over="ignore"):
            _, k, v = K.rotated(np64(x[r:r + 1]), H, KH, np.array([r]), theta)
        pool.append(0, r, k, v)
        pool.check()


def test_append_replayed_graph_and_other_stream():
    """A captured append, replayed with eager work between: the eager call's bits, and the same after a second time (a scale
    that has grown stays)."""
    H, KH, dh, lens, ctx = 4, 2, 128, [1, 20, 1], [3, 9, 40]
    x = torch.randn(22, (H + 2 * KH) * dh, dtype=torch.bfloat16, device="cuda")
    pb = B.Batch(np.zeros(3, np.int32), lens, 1, ctx_len=ctx)
    attn = B.make_attn(B.VFM_BF16, H, KH, dh, rope_theta=10000.0)
    pools = [Pool8(ctx, [64] * 3, KH, dh, 16, 7) for _ in range(3)]
    q = [torch.zeros(22, H * dh, dtype=torch.bfloat16, device="cuda") for _ in pools]
    B.vfm_kv_append_q8(attn, pb.c, x, q[0], pools[0].kv)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.vfm_kv_append_q8(attn, pb.c, x, q[1], pools[1].kv)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.vfm_kv_append_q8(attn, pb.c, x, q[2], pools[2].kv)
    for i in range(3):
        q[2].fill_(float(i))
        g.replay()
        torch.cuda.synchronize()
        for j in (1, 2):
            assert torch.equal(q[j], q[0])
            for a, b in zip((pools[j].kp, pools[j].vp, pools[j].ep), (pools[0].kp, pools[0].vp, pools[0].ep)):
                assert torch.equal(a, b), (i, j)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,H,KH,dh,page,window,sinks", [
    ("bf16", 2, 2, 128, 64, 0, 0), ("bf16", 2, 2, 64, 16, 0, 0), ("bf16", 4, 1, 128, 16, 50, 3),
    ("bf16", 7, 1, 64, 32, 17, 1), ("bf16", 8, 2, 128, 1024, 64, 64), ("bf16", 8, 1, 64, 64, 1, 0),
    ("bf16", 8, 1, 128, 16, 1, 5), ("bf16", 40, 1, 64, 16, 100, 33), ("bf16", 64, 1, 128, 128, 33, 4),
    ("bf16", 20, 1, 128, 32, 200, 0), ("bf16", 3, 3, 128, 16, 16, 16), ("bf16", 2, 1, 64, 16, 4000, 9),
    ("f32", 2, 2, 128, 64, 0, 0), ("f32", 4, 2, 64, 16, 50, 3), ("f32", 7, 1, 128, 32, 17, 1),
    ("f32", 40, 1, 64, 16, 100, 33), ("f32", 2, 2, 64, 1024, 1, 0)])
def test_attention_ragged(dtype, H, KH, dh, page, window, sinks):
    """Every length and context in one batch: single rows, chunks, prompts; pages and runs that end inside tiles, page
    entries, slots and scales that nothing sees NaN."""
    log(f"attend8 {dtype} H {H} KH {KH} dh {dh} page {page} window {window} sinks {sinks}")
    lens, ctx = [l for l, _ in RAGGED], [x for _, x in RAGGED]
    c = Cache8(lens, ctx, KH, dh, page, window, sinks, seed=H * dh + window)
    q = _queries(lens, H, dh, dtype, 7)
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
    log(f"long8 {dtype} H {H} KH {KH} dh {dh} window {window} ctx {ctx}")
    c = Cache8(lens, ctx, KH, dh, page, window, sinks, seed=5)
    q = _queries(lens, H, dh, dtype, 8)
    task = _tasks(len(lens), 4)
    pb = B.Batch(task, c.lens, 5, ctx_len=c.ctx)
    assert B.vfm_attention_workspace_q8(B.make_attn(DT[dtype][0], H, KH, dh, window=window, n_sink=sinks), pb.c) > 0
    got = _attend(c, task, H, KH, dh, window, sinks, dtype, q)
    log(f"  {_check(c, got, q, window, sinks, dtype, dh ** -0.5):.3f} of the tolerance")
    for i in range(len(lens)):
        assert np.array_equal(_attend(c, task, H, KH, dh, window, sinks, dtype, q, only=[i], ws_fill=0)[i], got[i])


@pytest.mark.parametrize("dtype,H,KH,dh", [("bf16", 4, 2, 128), ("bf16", 2, 1, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("lens,ctx,window", [([12], [40], 9), ([100], [70], 30), ([100], [0], 0)])
def test_attention_keys_that_only_some_rows_see(dtype, H, KH, dh, lens, ctx, window):
    """A NaN in the V row (and in the K row) of a key reaches the rows that see it and no other."""
    c = Cache8(lens, ctx, KH, dh, 16, window, 2, seed=11)
    q = _queries(lens, H, dh, dtype, 9, std=1.0)
    task = np.zeros(1, np.int32)
    clean = _attend(c, task, H, KH, dh, window, 2, dtype, q)[0]
    m, x = lens[0], ctx[0]
    for what, at, code in (("v", x + m // 2, 0x7F), ("v", x + m - 2, 0xFF), ("k", x + m // 3, 0x7F), ("v", max(0, x - 5), 0x7F)):
        slot = int(c.slots(0, np.array([at]))[0])
        pool = c.vp if what == "v" else c.kp
        was = pool[:, slot].clone()
        d = 5
        pool[:, slot, d] = code
        got = _attend(c, task, H, KH, dh, window, 2, dtype, q)[0]
        pool[:, slot] = was
        see = D.visible(x + np.arange(m), at, window, 2)
        assert np.array_equal(got[~see], clean[~see]), (what, at)
        if what == "v":
            assert np.all(np.isnan(got[see][:, :, d])), (what, at)
            assert np.array_equal(np.delete(got[see], d, axis=2), np.delete(clean[see], d, axis=2))
        else:
            assert np.isnan(got[see]).all()


@pytest.mark.parametrize("H,KH,dh,page,window,sinks,lens,ctx", [
    (32, 32, 64, 64, 0, 0, [2050], [0]), (64, 16, 128, 16, 90, 5, [1100, 1, 40], [333, 50, 0]),
    (56, 8, 64, 32, 300, 0, [1300], [70])])
def test_attention_prompts_of_wide_blocks(H, KH, dh, page, window, sinks, lens, ctx):
    """Prompts whose blocks fill the chip: rows at the blocks' and tiles' borders and a spread of others."""
    c = Cache8(lens, ctx, KH, dh, page, window, sinks, seed=21)
    rng = np.random.default_rng(12)
    q = _queries(lens, H, dh, "bf16", 12)
    task = _tasks(len(lens), 4)
    got = _attend(c, task, H, KH, dh, window, sinks, "bf16", q)
    worst, m = 0.0, lens[0]
    for i in sorted({0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 257, m // 2, m - 2, m - 1} | set(rng.integers(0, m, 20).tolist())):
        see = D.visible(ctx[0] + i, np.arange(ctx[0] + m), window, sinks)
        for h in (0, H // 2 + 1, H - 1):
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
    c = Cache8([1] * 40, ctx, 16, dh, 16, 0, 0, seed=31)
    q = _queries([1] * 40, 16, dh, "bf16", 3, std=1.0)
    task = _tasks(40, 6)
    got = _attend(c, task, 16, 16, dh, 0, 0, "bf16", q)
    _check(c, got, q, 0, 0, "bf16", dh ** -0.5)
    for i in (0, 17, int(np.argmax(ctx)), int(np.argmin(ctx))):
        assert np.array_equal(_attend(c, task, 16, 16, dh, 0, 0, "bf16", q, only=[i], ws_fill=0)[i], got[i])


@pytest.mark.parametrize("dtype,n,long", [("bf16", 65, 0), ("bf16", 200, 0), ("f32", 130, 0), ("bf16", 130, 30000), ("f32", 70, 30000)])
def test_attention_of_many_requests(dtype, n, long):
    """More requests than are looked at in one step of the search for a block's, prompts and single rows by turns; with one
    long context among them blocks are found in the table."""
    rng = np.random.default_rng(n)
    lens, ctx = rng.choice([1, 1, 2, 33, 70], n).tolist(), rng.integers(0, 40, n).tolist()
    if long:
        ctx[n // 2], lens[n // 2] = long, 1
    H, KH, dh = (4, 4, 64) if dtype == "bf16" else (2, 2, 64)
    c = Cache8(lens, ctx, KH, dh, 16, 0, 0, seed=n)
    q = _queries(lens, H, dh, dtype, 5)
    task = _tasks(n, 7)
    got = _attend(c, task, H, KH, dh, 0, 0, dtype, q)
    _check(c, got, q, 0, 0, dtype, dh ** -0.5)
    for i in (0, n // 2, n - 1):
        assert np.array_equal(_attend(c, task, H, KH, dh, 0, 0, dtype, q, only=[i], ws_fill=0)[i], got[i])


@pytest.mark.parametrize("H,KH,dh,page,window,sinks", [
    (2, 2, 64, 16, 0, 0), (4, 2, 128, 64, 0, 0), (3, 1, 64, 32, 0, 0), (4, 1, 128, 16, 0, 0), (4, 4, 64, 16, 130, 3),
    (4, 2, 64, 128, 199, 17), (2, 2, 128, 16, 513, 0), (4, 1, 64, 64, 1000, 70)])
def test_attention_single_fp32_rows(H, KH, dh, page, window, sinks):
    """Single rows of up to 4 queries on a key head, few and many keys, alone (where every request is one) and beside chunks."""
    log(f"single8 H {H} KH {KH} dh {dh} page {page} window {window} sinks {sinks}")
    ctx = [0, 1, 127, 128, 143, 144, 150, 191, 255, 256, 257, 700, 1023, 1024, 2500, 40, 300]
    lens = [1] * 15 + [9, 40]
    c = Cache8(lens, ctx, KH, dh, page, window, sinks, seed=dh + window)
    q = _queries(lens, H, dh, "f32", 4)
    task = _tasks(len(lens), 3)
    got = _attend(c, task, H, KH, dh, window, sinks, "f32", q, ldo=H * dh + 8)
    log(f"  {_check(c, got, q, window, sinks, 'f32', dh ** -0.5):.3f} of the tolerance")
    for only in ([4], [5], [14], [9, 11, 13], [12, 16], list(range(15))):
        alone = _attend(c, task, H, KH, dh, window, sinks, "f32", q, only=only, ws_fill=0)
        for i in only:
            assert np.array_equal(alone[i], got[i]), i


def test_attention_large_logits_and_scale():
    """Scores of hundreds (one key takes the whole weight) and a given scale."""
    for dtype in ("bf16", "f32"):
        H, KH, dh = 2, 1, 64
        c = Cache8([1, 40], [200, 30], KH, dh, 32, 0, 0, seed=2, spread=8.0)
        q = _queries([1, 40], H, dh, dtype, 1, std=8.0)
        got = _attend(c, np.zeros(2, np.int32), H, KH, dh, 0, 0, dtype, q, scale=0.25)
        log(f"  {dtype}: {_check(c, got, q, 0, 0, dtype, 0.25):.3f} of the tolerance")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_replayed_graph_and_other_stream(dtype):
    """A captured call, replayed with eager work between, and a call on another stream give the eager call's bits."""
    H, KH, dh = 4, 2, 128
    lens, ctx = [1, 1, 150, 2], [3000, 10, 700, 500]
    c = Cache8(lens, ctx, KH, dh, 64, 0, 0, seed=6)
    rng = np.random.default_rng(3)
    td = DT[dtype][1]
    attn = B.make_attn(DT[dtype][0], H, KH, dh)
    pb = B.Batch(np.zeros(4, np.int32), c.lens, 1, ctx_len=c.ctx)
    qd = torch.from_numpy(rng.standard_normal((pb.T, H * dh))).to(td).cuda()
    ws = torch.empty(B.vfm_attention_workspace_q8(attn, pb.c), dtype=torch.uint8, device="cuda")
    eager = torch.empty_like(qd)
    B.vfm_attention_paged_q8(attn, pb.c, qd, c.kv, eager, ws)
    torch.cuda.synchronize()
    out, other = torch.zeros_like(qd), torch.zeros_like(qd)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.vfm_attention_paged_q8(attn, pb.c, qd, c.kv, other, ws)
    s.synchronize()
    assert torch.equal(other, eager)
    with torch.cuda.graph(g):
        B.vfm_attention_paged_q8(attn, pb.c, qd, c.kv, out, ws)
    for i in range(4):
        out.fill_(float(i))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


def test_calls_on_two_streams_at_once():
    """Attention over one cache from two streams, each with its outputs and workspace, while an append fills another."""
    H, KH, dh = 8, 2, 64
    c = Cache8([1, 1, 150, 2], [9000, 10, 700, 500], KH, dh, 64, 0, 0, seed=6)
    pb = B.Batch(np.zeros(4, np.int32), c.lens, 1, ctx_len=c.ctx)
    gen = torch.Generator(device="cuda").manual_seed(1)
    calls = []
    for dtype in ("bf16", "f32"):
        code, td, _ = DT[dtype]
        attn = B.make_attn(code, H, KH, dh, rope_theta=10000.0)
        q = torch.randn(pb.T, H * dh, generator=gen, device="cuda").to(td)
        qkv = torch.randn(pb.T, (H + 2 * KH) * dh, generator=gen, device="cuda").to(td)
        ws = torch.empty(max(1, B.vfm_attention_workspace_q8(attn, pb.c)), dtype=torch.uint8, device="cuda")
        pool = Pool8(c.ctx, (c.lens + c.ctx).tolist(), KH, dh, 64, 9)
        first = [t.clone() for t in (pool.kp, pool.vp, pool.ep)]
        calls.append((attn, q, qkv, ws, pool, first, torch.empty_like(q), torch.empty_like(q)))

    def both(streams):
        for s, (attn, q, qkv, ws, pool, first, out, q_out) in zip(streams, calls):
            with torch.cuda.stream(s):
                for now, was in zip((pool.kp, pool.vp, pool.ep), first):
                    now.copy_(was)
                B.vfm_kv_append_q8(attn, pb.c, qkv, q_out, pool.kv)
                B.vfm_attention_paged_q8(attn, pb.c, q, c.kv, out, ws)
        torch.cuda.synchronize()
        return [t.clone() for x in calls for t in (x[4].kp, x[4].vp, x[4].ep, x[6], x[7])]

    torch.cuda.synchronize()
    want = both([torch.cuda.current_stream()] * 2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(both(streams), want))


@pytest.mark.parametrize("dtype,H,KH,dh,window,lens,ctx", [
    ("bf16", 8, 1, 128, 0, [1] * 130, [20, 30000] + [40] * 127 + [9000]),
    ("bf16", 32, 8, 64, 0, [700, 1, 2, 40], [0, 20000, 100, 9000]),
    ("bf16", 32, 8, 128, 0, [5, 600, 1, 1], [30000, 10, 700, 12000]),
    ("bf16", 16, 16, 64, 6000, [1] * 600 + [33], [90] * 599 + [20000, 9000]),
    ("f32", 4, 2, 64, 0, [900, 1, 30], [0, 15000, 6000]), ("f32", 16, 2, 128, 0, [300, 2], [10, 12000])])
def test_attention_long_contexts_beside_others(dtype, H, KH, dh, window, lens, ctx):
    """Steps whose blocks and records are the requests' own by a table: every request has the bits that it has alone, the
    long ones the 64-bit form's values; replayed from a graph the same."""
    log(f"long beside others, 8 bits {dtype} H {H} KH {KH} dh {dh} {len(lens)} requests")
    sinks = 2 if window else 0
    c = Cache8(lens, ctx, KH, dh, 64, window, sinks, seed=13)
    code, td, _ = DT[dtype]
    q = _queries(lens, H, dh, dtype, 14, std=1.0)
    n = len(lens)
    task = _tasks(n, 5)
    attn = B.make_attn(code, H, KH, dh, window=window, n_sink=sinks)
    pb = B.Batch(task, c.lens, 5, ctx_len=c.ctx)
    got = _attend(c, task, H, KH, dh, window, sinks, dtype, q)
    order = np.argsort(ctx)
    some = sorted({0, 1, min(2, n - 1), n - 2, n - 1, int(order[-1]), int(order[-2]), int(np.argmax(lens))})
    for i in some:
        assert np.array_equal(_attend(c, task, H, KH, dh, window, sinks, dtype, q, only=[i], ws_fill=0)[i], got[i]), i
    few = {i: got[i] for i in some if lens[i] <= 5 or ctx[i] > 1000}
    log(f"  {_check(c, few, q, window, sinks, dtype, dh ** -0.5):.3f} of the tolerance")
    by = np.argsort(task, kind="stable")
    qd = torch.from_numpy(np.concatenate([q[o].reshape(-1, H * dh) for o in by])).to(td).cuda()
    eager, out = torch.empty_like(qd), torch.zeros_like(qd)
    ws = torch.full((B.vfm_attention_workspace_q8(attn, pb.c),), 255, dtype=torch.uint8, device="cuda")
    B.vfm_attention_paged_q8(attn, pb.c, qd, c.kv, eager, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.vfm_attention_paged_q8(attn, pb.c, qd, c.kv, out, ws)
    for i in range(3):
        out.fill_(float(i))
        ws.fill_(170 + i)
        (qd.float() @ qd[:1].float().T).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i


@pytest.mark.parametrize("dtype,lens", [("bf16", [1, 1]), ("bf16", [1, 70]), ("f32", [1, 9])])
def test_pages_past_32_bit_offsets_and_shared_by_requests(dtype, lens):
    """A pool whose later codes lie past 2^32 bytes: the step's pages are the pool's last ones, and both requests' tables
    begin with the same pages (a prefix that they share)."""
    code, td, u = DT[dtype]
    H, KH, dh, page = 4, 2, 128, 64
    n_pages = (1 << 19) + 64                               # 2^25 slots and more of 128 bytes per head
    lens, ctx = np.array(lens, np.int32), np.array([150, 200], np.int32)
    last = n_pages - 1
    table = np.array([[last, last - 3, last - 1, 0, 0], [last, last - 3, last - 2, last - 5, last - 4]], np.int32)
    kp, vp = [torch.empty(KH, n_pages * page, dh, dtype=torch.uint8, device="cuda") for _ in range(2)]
    exps = torch.empty(n_pages * page // 16, KH, 2, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(17)
    for t in (kp, vp):                                     # the last pages alone are written
        t[:, -8 * page:] = torch.from_numpy(K.to_codes(rng.standard_normal((KH, 8 * page, dh)) * 80)).cuda()
    exps[-8 * page // 16:] = torch.from_numpy(rng.integers(118, 121, (8 * page // 16, KH, 2)).astype(np.uint8)).cuda()
    attn = B.make_attn(code, H, KH, dh)
    pb = B.Batch(np.zeros(2, np.int32), lens, 1, ctx_len=ctx)
    qkv = torch.from_numpy(rng.standard_normal((pb.T, (H + 2 * KH) * dh))).to(td).cuda()
    kv = B.PagedKVQ8(kp, vp, exps, page, table)
    q, out = [torch.empty(pb.T, H * dh, dtype=td, device="cuda") for _ in range(2)]
    ws = torch.empty(max(1, B.vfm_attention_workspace_q8(attn, pb.c)), dtype=torch.uint8, device="cuda")
    log(f"far pages, 8 bits {dtype} {lens}")
    B.vfm_kv_append_q8(attn, pb.c, qkv, q, kv)
    B.vfm_attention_paged_q8(attn, pb.c, q, kv, out, ws)
    torch.cuda.synchronize()
    rows, o, at = np64(qkv), np64(out), 0
    assert np.array_equal(np64(q), rows[:, :H * dh])       # no rotation: as they were
    for i, (m, c) in enumerate(zip(lens, ctx)):
        pos = np.arange(int(c + m))
        slots = table[i, pos // page].astype(np.int64) * page + pos % page
        sd = torch.from_numpy(slots).cuda()
        e = exps[sd // 16].cpu().numpy()
        k, v = [K.VALUES[t[:, sd].cpu().numpy()].transpose(1, 0, 2) * 2.0 ** (e[..., n] - 127.0)[..., None]
                for n, t in enumerate((kp, vp))]
        r = rows[at:at + m].reshape(m, H + 2 * KH, dh)
        for got, want, n in ((k[c:], r[:, H:H + KH], 0), (v[c:], r[:, H + KH:], 1)):
            half = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** (e[c:, :, n] - 137.0)[..., None])   # half an e4m3 step
            assert np.all(np.abs(got - want) <= half)
        ref, a, n = D.attention(r[:, :H], k, v, int(c), 0, 0, dh ** -0.5)
        dot = D.score_sizes(r[:, :H], k, dh ** -0.5)[:, :, None]
        lim = ((u if dtype == "bf16" else 0.0) + (n[:, None, None] + 16) * 2.0 ** -24) * (a + np.abs(ref)) \
            + a * 2 * ((dh + 2) * 2.0 ** -24 * dot + 2.0 ** -22)
        assert np.all(np.abs(o[at:at + m].reshape(m, H, dh) - ref) <= lim)
        at += m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [-100, -20, 12, 18, 40])
def test_attention_scales_of_any_size(dtype, shift):
    """Keys under scales of 2^-110 to 2^30: scores from nothing to 2^33 and more, where the largest takes the whole weight;
    values under the same scales come out times 2^shift.  Few rows and many."""
    H, KH, dh = 2, 1, 64
    lens, ctx = [1, 40], [200, 100]
    c = Cache8(lens, ctx, KH, dh, 32, 0, 0, seed=2)
    q = _queries(lens, H, dh, dtype, 1)
    task = np.zeros(2, np.int32)
    base = _attend(c, task, H, KH, dh, 0, 0, dtype, q)
    seen = c.exps != 255
    c.exps[..., 1] += (seen[..., 1] * shift).to(torch.uint8)        # wraps for negative shifts
    got = _attend(c, task, H, KH, dh, 0, 0, dtype, q)
    for i in range(2):
        assert np.array_equal(got[i], base[i] * 2.0 ** shift)
    c.v = [v * 2.0 ** shift for v in c.v]
    c.exps[..., 0] += (seen[..., 0] * shift).to(torch.uint8)
    c.k = [k * 2.0 ** shift for k in c.k]
    got = _attend(c, task, H, KH, dh, 0, 0, dtype, q)
    if shift > 0:                                          # rows whose two largest scores lie apart by more than rounding
        for i in range(2):
            for r in range(lens[i]):
                for h in range(H):
                    s = c.k[i][:ctx[i] + r + 1, 0] @ q[i][r, h] * dh ** -0.5
                    top = np.argsort(s)
                    size = np.abs(c.k[i][:ctx[i] + r + 1, 0]).max() * np.abs(q[i][r, h]).max() * dh ** 0.5
                    if s[top[-1]] - s[top[-2]] > 40 + (dh + 2) * 2.0 ** -23 * size:
                        v = c.v[i][top[-1], 0]
                        assert np.all(np.abs(got[i][r, h] - v) <= 2.0 ** -8 * np.abs(v) + 2.0 ** -20 * np.abs(c.v[i]).max())
    else:
        log(f"  {_check(c, got, q, 0, 0, dtype, dh ** -0.5):.3f} of the tolerance")


def test_attention_rows_of_a_wider_matrix():
    """Queries as the first columns of [T, 3 d] rows, as a layer keeps them."""
    H = KH = 2
    dh = 64
    c = Cache8([3, 40], [20, 0], KH, dh, 16, 10, 1, seed=3)
    q = _queries([3, 40], H, dh, "bf16", 2, std=1.0)
    ref = _attend(c, np.zeros(2, np.int32), H, KH, dh, 10, 1, "bf16", q)
    pb = B.Batch(np.zeros(2, np.int32), c.lens, 1, ctx_len=c.ctx)
    wide = torch.full((43, 3 * H * dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :H * dh] = torch.from_numpy(np.concatenate([x.reshape(-1, H * dh) for x in q])).to(torch.bfloat16).cuda()
    out = torch.zeros(43, H * dh, dtype=torch.bfloat16, device="cuda")
    attn = B.make_attn(B.VFM_BF16, H, KH, dh, window=10, n_sink=1)
    B.vfm_attention_paged_q8(attn, pb.c, wide, c.kv, out)
    assert np.array_equal(np64(out).reshape(-1, H, dh), np.concatenate([ref[0], ref[1]]))


def test_prompt_in_chunks_and_at_once():
    """A prompt appended in chunks that end on runs leaves the bits of one appended at once; in chunks that cut runs its
    numbers are within a rounding to the run's last scale."""
    H, KH, dh, n = 2, 2, 64, 100
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((n, H + 2 * KH, dh)) * 2.0 ** rng.integers(-2, 3, (n, 1, 1))).to(torch.bfloat16)
    pools = []
    for cuts in ([0, 100], [0, 16, 64, 96, 100], [0, 5, 17, 18, 47, 50, 99, 100]):
        pool = Pool8([0], [n], KH, dh, 16, 3)
        for a, b in zip(cuts, cuts[1:]):
            _step(pool, np.zeros(1, np.int32), [b - a], [a], H, KH, dh, "bf16", 10000.0, x[a:b])
        pools.append(pool)
    s = pools[0].slots(0, np.arange(n))
    e = pools[0].ep.cpu().numpy()[s // 16]
    for p in pools[1:]:
        assert np.array_equal(p.ep.cpu().numpy()[s // 16], e)
    for n_, t in enumerate(("kp", "vp")):
        one, same, cut = (getattr(p, t).cpu().numpy()[:, s] for p in pools)
        assert np.array_equal(one, same)
        a, b = K.VALUES[one], K.VALUES[cut]
        assert np.all(np.abs(a - b) <= 2.0 ** -9)          # e4m3's smallest number: what turns subnormal is rounded twice
