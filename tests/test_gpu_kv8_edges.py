"""GPU tests of the 8-bit cache's append and attention at the types' ends, and of the loop where masks fail or end.

Tolerances.  Append: a code and a rotated query are one rounding of the 64-bit value, below the types' normal numbers too.
The 64-bit form's angles differ by up to 64 2^-53 of the position, its values by far = that times the pair's size, and its
own 4 roundings.  Rounding is monotone, so a query lies between the rounded want - far and want + far, which are one number
unless a tie lies between them.  (An fp32 query at position 80000 is up to 2^18 steps of 2^-149, and far 2e-4 of a
step: of 1.5 million some are that close to a tie.  A code's steps are 2^14 times as large.)  A bf16 query below 2^-126 is
cut to 24 bits first (off by less than 2^-150) and rounded to a multiple of 2^-149 (by 2^-150 at most): 2^-149 beside far.
Attention where the largest score takes the whole weight: the other weights are below e^-40 each, 2^-57,
so the output is the value at that key up to n 2^-57 of the largest one, and a rounding of the result (2^-24 in fp32), two with
the division."""
import numpy as np
import pytest
import torch

from paper_2606_09643_amd import runner as R
from tests import kv8_common as K
from tests.gpu_common import log
from tests.helpers import np64
from tests.test_gpu_decode import DT
from tests.test_gpu_kv8 import Cache8, Pool8, _attend, _queries, _step
from tests.test_gpu_windowed import REQUESTS, SAMPLING, _decoder, _model

pytestmark = pytest.mark.gpu


def _once(y, bits):
    """y rounded once to that many significant bits, ties to even, under fp32's exponents (fewer bits below 2^-126)."""
    unit = 2.0 ** (np.maximum(np.frexp(y)[1] - 1, -126) - (bits - 1))
    return np.rint(y / unit) * unit


@pytest.mark.parametrize("dtype,H,KH,dh", [("f32", 6, 6, 128), ("f32", 8, 8, 64), ("bf16", 8, 1, 128), ("bf16", 12, 2, 64)])
@pytest.mark.parametrize("rows", [1, 2000])
def test_append_below_the_normal_numbers(dtype, H, KH, dh, rows):
    """Rotated values below 2^-126, where fp32 has fewer bits than the number's own 24: codes are rounded once."""
    log(f"append8 subnormal {dtype} H {H} KH {KH} dh {dh} rows {rows}")
    rng = np.random.default_rng(H + dh)
    td = DT[dtype][1]
    n = 2000
    # whole multiples of the type's smallest number, up to 2^-131 (fp32) and 2^-126 (bf16)
    step, most = (2.0 ** -149, 1 << 18) if dtype == "f32" else (2.0 ** -133, 1 << 7)
    x = torch.from_numpy(rng.integers(-most, most + 1, (n, H + 2 * KH, dh)) * step).to(td)
    lens = [n] if rows > 1 else [1] * n
    ctx = [5] if rows > 1 else [16 * int(c) for c in rng.integers(1, 5000, n)]
    task = np.zeros(len(lens), np.int32)
    pool = Pool8(ctx, [a + b + 16 for a, b in zip(lens, ctx)], KH, dh, 16, 3)
    q = _step(pool, task, lens, ctx, H, KH, dh, dtype, 10000.0, x)
    at, either, host = 0, 0, np64(x)
    for i, m in enumerate(lens):
        want, k, v = K.rotated(host[at:at + m], H, KH, np.arange(ctx[i], ctx[i] + m), 10000.0)
        pool.append(i, ctx[i], k, v)
        size = np.abs(host[at:at + m, :H])
        size = size + np.roll(size, dh // 2, axis=-1)
        far = (64 * np.arange(ctx[i], ctx[i] + m)[:, None, None] + 4) * 2.0 ** -53 * size + (2.0 ** -149 if dtype == "bf16" else 0.0)
        lo, hi = (_once(want + d, 24 if dtype == "f32" else 8) for d in (-far, far))
        differ = (q[at:at + m] < lo) | (q[at:at + m] > hi)
        assert not differ.any(), (i, int(differ.sum()))
        either += int((lo != hi).sum())
        at += m
    assert either < 1e-3 * n * H * dh
    pool.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [12, 18, 40])
def test_attention_of_the_largest_score_alone(dtype, shift):
    """Scores so far apart that the largest takes the whole weight, of few rows and many: the output is that key's value."""
    log(f"attend8 {dtype} shift {shift}")
    H, KH, dh = 2, 1, 64
    lens, ctx = [1, 40], [200, 100]
    c = Cache8(lens, ctx, KH, dh, 32, 0, 0, seed=2)
    q = _queries(lens, H, dh, dtype, 1)
    c.exps[..., 0] += ((c.exps[..., 0] != 255) * shift).to(torch.uint8)
    got = _attend(c, np.zeros(2, np.int32), H, KH, dh, 0, 0, dtype, q)
    u, checked = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23), [0, 0]
    for i in range(2):
        k, v = c.k[i][:, 0] * 2.0 ** shift, c.v[i][:, 0]
        for r in range(lens[i]):
            for h in range(H):
                s = k[:ctx[i] + r + 1] @ q[i][r, h] * dh ** -0.5
                top = np.argsort(s)
                size = np.abs(k).max() * np.abs(q[i][r, h]).max() * dh ** 0.5
                if s[top[-1]] - s[top[-2]] > 40 + (dh + 2) * 2.0 ** -23 * size:
                    want = v[top[-1]]
                    assert np.all(np.abs(got[i][r, h] - want) <= u * np.abs(want) + 2.0 ** -40 * np.abs(v).max()), (i, r, h)
                    checked[i] += 1
    assert checked[0] > 0 and checked[1] > 20, checked


@pytest.mark.parametrize("dtype,window", [("bf16", 40), ("f32", None)])
def test_loop_goes_on_after_a_failed_mask_and_ends_at_an_empty_one(dtype, window):
    """Steps that a mask function's error ended behind their layers are taken again: rows that were appended twice, penalties,
    drawn and greedy tokens are those without the failure.  A mask that leaves nothing ends its request alone."""
    w = _decoder(dtype, 64)
    model, emb, prompts = _model(w)
    n = int(model.heads.n_out[0])

    def grammar(bad, last):
        calls = []

        def allowed(answer):
            calls.append(len(answer))
            if len(calls) in bad:
                raise RuntimeError("the grammar's own")
            ok = np.ones(n, bool) if len(answer) < last else np.zeros(n, bool)
            ok[answer] = False
            return ok
        return allowed

    def run(bad):
        log(f"loop {dtype} window {window}, failing calls {bad}")
        cb = R.ContinuousBatcher(model, emb, page_size=16, n_pages=24, max_seqs=3, max_step_tokens=48, max_pages=9,
                                 kv8=True, window=window)
        adjust = [R.AdjustParams(1.3, 0.2, 0.1, allowed=grammar(bad, 99)), R.AdjustParams(1.2, bias={5: 1.0}), None,
                  R.AdjustParams(allowed=grammar((), 2)), R.AdjustParams(frequency=0.3, allowed=grammar(bad, 7))]
        for rid, ((task, _, n_new), pr) in enumerate(zip(REQUESTS, prompts)):
            cb.submit(rid, task, pr, n_new, sampling=SAMPLING[rid], adjust=adjust[rid])
        failed = 0
        while cb.waiting or cb.running:
            try:
                cb.step()
            except RuntimeError:
                failed += 1
        assert cb.committed == 0 and cb.alloc.count(0)[1] == 24
        return cb.tokens(), failed
    plain, failed = run(())
    assert failed == 0 and [len(plain[r]) for r in range(5)] == [40, 30, 70, 3, 8]
    assert plain[3][2] == plain[4][7] == -1 and min(plain[0] + plain[3][:2] + plain[4][:7]) >= 0
    assert len(set(plain[0])) == 40
    assert run((1, 2, 5, 6)) == (plain, 8)
