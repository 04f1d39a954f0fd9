"""GPU tests of the adjustment of head outputs (penalties, biases, masks) through the C ABI, against the plain 64-bit form.

Tolerance: an output is one rounding to fp32 of a 64-bit result, so it is off by 2^-24 of itself; the 64-bit operations
(a product with a reciprocal, a fused multiply-add, two sums) are off by 4 2^-53 of their terms, which the sum of the
terms' sizes bounds."""
import numpy as np
import pytest
import torch

from paper_2606_09643_amd import binding as B
from tests import kv8_common as K

pytestmark = pytest.mark.gpu


class Rows:
    """Ragged head outputs and what is to be done to them, per request a dict of kv8_common.adjust's arguments."""

    def __init__(self, rows, par, words=None, lists=("hist", "bias", "mask"), unit=("r", "p", "f"), prompts=True, batch=True):
        n = len(rows)
        self.rows, self.par = [np.asarray(r, np.float32) for r in rows], par
        sizes = np.array([len(r) for r in rows], np.int32)
        if batch:
            self.pb = B.Batch(np.arange(n, dtype=np.int32)[::-1].copy(), np.ones(n, np.int32), n, n_out=sizes[::-1].copy())
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        get = lambda k, d: np.array([p.get(k, d) for p in par], np.float32)  # noqa: E731
        t = {}
        for name, k, d in (("repetition", "r", 1.0), ("presence", "p", 0.0), ("frequency", "f", 0.0)):
            if k in unit:
                t[name] = dev(get(k, d))
        if "hist" in lists:
            h = [np.asarray(p.get("hist", ()), np.int32) for p in par]
            begin = np.cumsum([0] + [len(x) + i % 3 for i, x in enumerate(h)])           # gaps: every alignment
            flat = np.full(begin[-1] + 1, 1, np.int32)
            for b, x in zip(begin, h):
                flat[b:b + len(x)] = x
            t.update(hist=dev(flat), hist_begin=dev(begin[:-1].astype(np.int64)),
                     hist_len=dev(np.array([len(x) for x in h], np.int32)))
            if prompts:
                t["n_prompt"] = dev(np.array([p.get("n_prompt", 0) for p in par], np.int32))
        if "bias" in lists:
            b = [list(p.get("bias", ())) for p in par]
            begin = np.cumsum([0] + [len(x) for x in b])
            t.update(bias_id=dev(np.array([i for x in b for i, _ in x] + [0], np.int32)),
                     bias=dev(np.array([v for x in b for _, v in x] + [9.0], np.float32)),
                     bias_begin=dev(begin[:-1].astype(np.int64)), bias_len=dev(np.array([len(x) for x in b], np.int32)))
        if "mask" in lists:
            words = words or -(-int(sizes.max()) // 32)
            of = [i for i, p in enumerate(par) if p.get("allowed") is not None]
            row = np.full(n, -1, np.int32)
            row[of] = np.arange(len(of))[::-1]
            m = np.zeros((max(1, len(of)), words), np.int32)
            for i in of:
                m[row[i]] = K.mask_words(par[i]["allowed"], words)
            t.update(mask=dev(m), mask_row=dev(row))
        self.tensors, self.adjust = t, B.OutputAdjust(**t)

    def flat(self):
        return torch.from_numpy(np.concatenate(self.rows + [np.full(5, 1e30, np.float32)])).cuda()

    def run(self, place, stream=None):
        out = self.flat()
        to = out if place else torch.full_like(out, 5.0)
        B.vfm_adjust_outputs(self.pb.c, out, self.adjust, None if place else to, stream)
        assert place or torch.equal(out.nan_to_num(3.0), self.flat().nan_to_num(3.0))
        tail = to[-5:].cpu().numpy()
        assert np.all(tail == (np.float32(1e30) if place else 5.0))
        return to.cpu().numpy()

    def check(self, got):
        at = 0
        for i, (r, p) in enumerate(zip(self.rows, self.par)):
            g = got[at:at + len(r)].astype(np.float64)
            at += len(r)
            p = {k: (np.float64(np.float32(v)) if k in "rpf" else v) for k, v in p.items()}
            if "bias" in p:
                p["bias"] = [(j, np.float64(np.float32(v))) for j, v in p["bias"]]
            with np.errstate(over="ignore"):
                want = K.adjust(r, **p)
                want32 = want.astype(np.float32)
            fine = np.isfinite(want32)
            assert np.array_equal(np.isnan(g), np.isnan(want)), i
            assert np.array_equal(g[~fine & ~np.isnan(want)], want32[~fine & ~np.isnan(want)].astype(np.float64)), i
            on = lambda k, d: p.get(k, d) if p.get(k, d) > 0 or k != "r" and p.get(k, d) < 0 else d  # noqa: E731
            terms = np.abs(r.astype(np.float64)) * max(on("r", 1.0), 1 / on("r", 1.0), 1.0) \
                + abs(on("p", 0.0)) + abs(on("f", 0.0)) * len(p.get("hist", ())) + 100.0
            tol = 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -53 * terms + 2.0 ** -149
            far = np.abs(g[fine] - want[fine]) / tol[fine]
            assert far.size == 0 or far.max() <= 1, (i, len(r), far.max())
            # what nothing applies to keeps its bits
            same = np.ones(len(r), bool)
            h = np.asarray(p.get("hist", ()), np.int64)
            same[h[(h >= 0) & (h < len(r))]] = False
            for j, _ in p.get("bias", ()):
                if 0 <= j < len(r):
                    same[j] = False
            if p.get("allowed") is not None:
                same &= p["allowed"] if p["allowed"].any() else False
            assert np.array_equal(g[same].astype(np.float32).view(np.int32), r[same].view(np.int32)), i


def _par(rng, n, hist, biases=5, allow=None, out_of=0.05):
    h = (n * rng.random(hist) ** 3).astype(np.int64)
    stray = rng.random(hist) < out_of
    h[stray] = rng.choice([-1, n, n + 7, 2 ** 31 - 1, -2 ** 31], int(stray.sum()))
    p = {"r": rng.choice([0.7, 1.0, 1.3]), "p": rng.choice([0.0, 0.6, -0.4]), "f": rng.choice([0.0, 0.25]), "hist": h,
         "n_prompt": int(rng.integers(0, hist + 2)),
         "bias": [(int(j), float(v)) for j, v in zip(rng.integers(-2, n + 2, biases), rng.choice([-np.inf, 3.0, -2.5, 100.0], biases))]}
    if allow is not None:
        p["allowed"] = rng.random(n) < allow
    return p


SIZES = [1, 2, 3, 4, 5, 7, 31, 32, 33, 64, 255, 1000, 1020, 1021, 1023, 1024, 1025, 2047, 4099, 8189, 8192, 8193, 32000]


@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("hist", [0, 1, 6, 700, 5000])
def test_adjust_ragged(place, hist):
    """Rows of every size and alignment beside each other, with and without masks, histories and biases; ids that stray."""
    print(f"adjust ragged hist {hist} place {place}", flush=True)
    rng = np.random.default_rng(hist)
    rows = [rng.standard_normal(n) * 4 for n in SIZES + SIZES[::-1]]
    par = [_par(rng, len(r), hist if i % 4 else hist // 3, biases=int(i % 6), allow=[None, 0.5, 0.01, 1.0][i % 4])
           for i, r in enumerate(rows)]
    b = Rows(rows, par)
    b.check(b.run(place))


@pytest.mark.parametrize("n_req", [1, 3, 70])
def test_adjust_large_heads(n_req):
    """Many slices of a request, with small and large blocks; a history longer than the head."""
    rng = np.random.default_rng(n_req)
    rows = [rng.standard_normal(100003 if i < 3 else 30011) * 4 for i in range(n_req)]
    par = [_par(rng, len(r), 150000 if i == 0 else 3000, biases=300, allow=0.3 if i % 2 else None) for i, r in enumerate(rows)]
    b = Rows(rows, par)
    for place in (True, False):
        b.check(b.run(place))


def test_adjust_what_is_given_alone():
    """Each group alone, none at all, penalties without a prompt's length, masks without enough words."""
    rng = np.random.default_rng(5)
    rows = [rng.standard_normal(n) for n in (50, 1500, 3)]
    for lists, unit in (((), ()), (("hist",), ("r",)), (("hist",), ("p",)), (("hist",), ("f",)), (("hist",), ()),
                        (("bias",), ()), (("mask",), ()), (("hist", "mask"), ("r", "f")), (("bias", "hist"), ("p",))):
        par = []
        for r in rows:
            p = _par(rng, len(r), 40, allow=0.5)
            par.append({k: v for k, v in p.items() if k in unit or k in ("hist",) and "hist" in lists
                        or k == "bias" and "bias" in lists or k == "allowed" and "mask" in lists})
        b = Rows(rows, par, lists=lists, unit=unit, prompts=False)
        for place in (True, False):
            b.check(b.run(place))
    for p in par:                                        # outputs past the mask's words are not allowed
        p["allowed"] = None
    par[1]["allowed"] = np.ones(1500, bool)
    b = Rows(rows, par, words=20)
    par[1]["allowed"] = np.arange(1500) < 640
    b.check(b.run(True))


def test_adjust_special_values():
    """Infinities and NaN among the outputs, masks that leave nothing (one with bits behind the row's end), parameters out
    of range, lists that reach out of their arrays, mask rows that do not exist."""
    rng = np.random.default_rng(6)
    n = 1030
    rows = [rng.standard_normal(n).astype(np.float32) for _ in range(8)]
    for r in rows:
        r[[0, 5, 9]] = np.inf, -np.inf, np.nan
        r[[11, 12, 13]] = 0.0, -0.0, 3.4e38
    par = [_par(rng, n, 60, biases=3, out_of=0.2) for _ in rows]
    par[0].update(r=-1.0, p=np.nan, f=np.nan)
    par[1].update(r=np.nan, f=-0.5)
    par[2].update(allowed=np.zeros(n, bool))
    par[3].update(allowed=np.arange(n) == 9)             # only the NaN
    par[4].update(hist=[0, 5, 9, 11, 12, 13] * 3, n_prompt=6, r=2.0, p=0.5)
    par[5].update(hist=[13] * 9, r=0.5, p=0.0, f=0.0)    # past fp32's range
    par[6].update(allowed=np.arange(n) >= 1024)
    b = Rows(rows, par, words=40)
    w = b.tensors["mask"][b.tensors["mask_row"][2].item()]
    w[n // 32] = -64                                     # bits of outputs that the row does not have (1030 % 32 = 6)
    w[33:] = -1
    for place in (True, False):
        b.check(b.run(place))
    # lists out of their arrays: what is there counts, the rest is not read
    rows, par = rows[:3], [dict(par[i]) for i in (4, 4, 4)]
    b = Rows(rows, par, lists=("hist", "mask"))
    total = b.tensors["hist"].numel()
    b.tensors["hist_begin"].copy_(torch.tensor([total - 2, -1, total]))
    b.tensors["hist_len"].fill_(2 ** 31 - 1)
    b.tensors["mask_row"].copy_(torch.tensor([1, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32))
    last = b.tensors["hist"][-2:].cpu().tolist()
    b.par = [{**par[0], "hist": last, "n_prompt": par[0]["n_prompt"], "bias": []}, {}, {}]
    b.check(b.run(False))
    b.tensors["hist_len"].fill_(-5)
    b.par = [{}, {}, {}]
    b.check(b.run(True))


def test_masked_rows_give_no_token():
    """A mask that leaves nothing: neither draw nor greedy pick answers with a token; one that leaves one: that one."""
    n = 300
    rng = np.random.default_rng(7)
    rows = [rng.standard_normal(n) for _ in range(3)]
    par = [{"allowed": np.zeros(n, bool)}, {"allowed": np.arange(n) == 277}, {}]
    b = Rows(rows, par)
    out = torch.from_numpy(b.run(True)).cuda()
    ids, u = torch.full((3,), 99, dtype=torch.int32, device="cuda"), torch.full((3,), 0.3, device="cuda")
    B.vfm_sample_tokens(b.pb.c, out, B.Sampling(), u, ids)
    assert ids[:2].tolist() == [-1, 277] and 0 <= int(ids[2]) < n
    B.vfm_greedy_tokens(b.pb.c, out, ids)
    assert ids.tolist() == [-1, 277, int(np.argmax(rows[2].astype(np.float32)))]


def test_adjust_replayed_graph_and_other_stream():
    rng = np.random.default_rng(9)
    rows = [rng.standard_normal(n) for n in (32000, 5, 900)]
    b = Rows(rows, [_par(rng, len(r), 500, allow=0.2) for r in rows])
    want = torch.from_numpy(b.run(False)).cuda()
    out, to = b.flat(), torch.zeros_like(want)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.vfm_adjust_outputs(b.pb.c, out, b.adjust, to)
    s.synchronize()
    assert torch.equal(to[:-5].nan_to_num(7.0), want[:-5].nan_to_num(7.0))
    with torch.cuda.graph(g):
        B.vfm_adjust_outputs(b.pb.c, out, b.adjust, to)
    for i in range(3):
        to.fill_(float(i))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(to[:-5].nan_to_num(7.0), want[:-5].nan_to_num(7.0)), i


@pytest.mark.parametrize("n,n_req", [(50000, 1), (3000, 3), (20000, 260)])
def test_adjust_lists_past_16_bits(n, n_req):
    """One request of more tokens than 16 bits count, of one output mostly, and one of more biases than 15 bits count,
    several for the same output; beside requests with short lists."""
    rng = np.random.default_rng(n)
    rows = [rng.standard_normal(n) * 4 for _ in range(n_req)]
    par = [_par(rng, n, 50, allow=0.5) for _ in rows]
    hist = np.full(200000, n - 2, np.int64)
    hist[::100] = rng.integers(0, n, 2000)
    par[0].update(hist=hist, n_prompt=1000, f=0.01, p=0.1, r=1.3)
    par[-1]["bias"] = [(int(j), float(v)) for j, v in zip(rng.integers(0, n, 70000), rng.standard_normal(70000).round(2))]
    if n_req > 1:
        par[1].update(hist=np.full(65536, 5, np.int64), n_prompt=0, f=0.001, r=1.0)
    b = Rows(rows, par)
    for place in (True, False):
        b.check(b.run(place))
