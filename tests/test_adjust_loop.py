"""The continuous-batching loop's handling of masks that follow the generated tokens (no GPU): the device's calls are stood
in for by plain ones on the CPU, whose head outputs favour the same order of tokens at every step."""
import numpy as np
import pytest
import torch

from paper_2606_09643_amd import binding as B
from paper_2606_09643_amd import runner as R
from paper_2606_09643_amd import workloads as wl

N_OUT = np.array([40, 100, 33], np.int32)


def _scores(n):
    return torch.from_numpy(((np.arange(n) * 37) % 101).astype(np.float32))


class _Table:
    c = None


class _Model:
    def __init__(self):
        self.w = wl.WORKLOADS[5].replace(n_layers=1, d=256, n_heads=2, head_dim=128, d_ff=512, n_tasks=3)
        self.n_layers, self.cfg, self.c_layers = 1, R.cfg_for(self.w), [None]
        self.heads, self.head_tab, self.final = wl.Heads(N_OUT, [], []), _Table(), {"w": None}

    def lora_c(self, i):
        return None


@pytest.fixture
def loop(monkeypatch):
    """Makes loops on the CPU; the requests' outputs of the latest step are in `rows`."""
    batches, RealBatch = [], B.Batch

    def batch(*args, **kw):
        batches.append(RealBatch(*args, **{**kw, "non_blocking": False}))
        return batches[-1]

    def rows(out):
        off = batches[-1].out_off()
        return [out[a:b] for a, b in zip(off, off[1:])]

    def head(cfg, w, b, heads, pb, x, out, ws):
        for o in rows(out):
            o.copy_(_scores(len(o)))

    def adjust(pb, out, a):
        t = a.tensors
        for i, o in enumerate(rows(out)):
            if t["mask"] is not None and int(t["mask_row"][i]) >= 0:
                words = t["mask"][int(t["mask_row"][i])].numpy().view(np.uint8)
                ok = torch.from_numpy(np.unpackbits(words, bitorder="little")[:len(o)].astype(bool))
                o[~ok] = -float("inf") if ok.any() else float("nan")

    def greedy(pb, out, ids):
        for i, o in enumerate(rows(out)):
            ids[i] = -1 if torch.isnan(o).all() else int(o.argmax())

    nothing = lambda *a, **kw: None  # noqa: E731
    for name, call in (("Batch", batch), ("vfm_workspace_size_q8", lambda *a: 1), ("vfm_embed_forward", nothing),
                       ("vfm_layer_forward_q8", nothing), ("vfm_head_forward", head), ("vfm_adjust_outputs", adjust),
                       ("vfm_greedy_tokens", greedy)):
        monkeypatch.setattr(B, name, call)

    def make(**kw):
        args = dict(page_size=16, n_pages=30, max_seqs=4, max_step_tokens=64, max_pages=6, device="cpu", kv8=True)
        cb = R.ContinuousBatcher(_Model(), emb=None, **{**args, **kw})
        cb._h2d = lambda a: torch.from_numpy(np.ascontiguousarray(a))
        return cb
    return make


class _NoRepeat:
    """No token twice; keeps the lists it was asked for, and fails at the calls `bad` in the way `how`."""

    def __init__(self, n, bad=(), how="raise"):
        self.n, self.bad, self.how, self.calls, self.lists = n, set(bad), how, 0, []

    def __call__(self, answer):
        self.calls += 1
        if self.calls - 1 in self.bad:
            if self.how == "raise":
                raise RuntimeError("the grammar's own")
            return np.ones(self.n + 1, bool)
        self.lists.append(list(answer))
        ok = np.ones(self.n, bool)
        ok[answer] = False
        return ok


@pytest.mark.parametrize("how,error", [("raise", RuntimeError), ("shape", ValueError)])
def test_a_step_whose_mask_failed_can_be_taken_again(loop, how, error):
    """The function's error reaches the caller; stepped again, every mask is asked for with the tokens that there are, each
    once, and all requests end with the tokens that they have without the failure."""
    def run(bad):
        cb, gram = loop(), [_NoRepeat(40, bad, how), _NoRepeat(100), None]
        for rid, g in enumerate(gram):
            cb.submit(rid, rid, np.arange(5 + rid, dtype=np.int32), 7 + rid, adjust=g and R.AdjustParams(allowed=g))
        failed = 0
        while cb.waiting or cb.running:
            try:
                cb.step()
            except error:
                failed += 1
        return cb.tokens(), gram, failed
    plain, gram, failed = run(())
    assert failed == 0 and [len(plain[r]) for r in range(3)] == [7, 8, 9]
    for rid in range(2):
        assert len(set(plain[rid])) == len(plain[rid])
        assert gram[rid].lists == [plain[rid][:j] for j in range(len(plain[rid]))]
    got, gram, failed = run((0, 3, 4, 8))
    assert failed == 4 and got == plain
    assert gram[0].lists == [plain[0][:j] for j in range(7)]
    # the second request's function answers anew in a step that is taken again, from the same list
    assert all(x == plain[1][:len(x)] for x in gram[1].lists)


def test_a_request_whose_mask_leaves_nothing_ends(loop):
    """Its last token is -1, no function is asked with that token in its list, its pages and slot are free again, and the
    requests beside it go on as they do without it."""
    def grammar(n, stop, lists):
        def allowed(answer):
            lists.append(list(answer))
            ok = np.zeros(n, bool)
            if len(answer) < stop:
                ok[len(answer) * 3 % n] = True
            return ok
        return allowed

    def run(stops):
        cb, lists = loop(max_seqs=2), [[] for _ in stops]
        for rid, stop in enumerate(stops):
            cb.submit(rid, rid % 3, np.arange(20, dtype=np.int32), 30,
                      adjust=R.AdjustParams(1.5, allowed=grammar(int(N_OUT[rid % 3]), stop, lists[rid])))
        cb.submit(9, 1, np.arange(5, dtype=np.int32), 6)
        cb.submit(10, 0, np.arange(5, dtype=np.int32), 6, adjust=R.AdjustParams(allowed=np.zeros(40, bool)))
        done = cb.run()
        assert cb.committed == 0 and cb.alloc.count(0)[1] == 30 and len(cb.free_slots) == 2
        assert cb._hist_free == [(cb._hist.numel(), 0)]
        return done, lists, cb.steps
    stops = [4, 0, 100, 29, 30]
    done, lists, steps = run(stops)
    for rid, stop in enumerate(stops):
        want = [j * 3 % int(N_OUT[rid % 3]) for j in range(min(stop, 30))] + [-1] * (stop < 30)
        assert done[rid] == want, rid
        assert lists[rid] == [want[:j] for j in range(len(want))]
    assert done[10] == [-1] and done[9] == [int(_scores(100).argmax())] * 6
    assert run([100] * 5)[0][9] == done[9]


def test_parameters_that_fp32_does_not_hold_are_refused():
    """A penalty goes to the device as fp32: one that is infinite or zero there would be another penalty.  Outputs are whole
    numbers."""
    for kw in (dict(repetition=1e39), dict(repetition=1e-46), dict(presence=1e39), dict(frequency=-1e39),
               dict(bias={1: 1e39}), dict(bias={1: 0.0, 2: -4e38}), dict(bias={1.5: 1.0}), dict(bias={"1": 1.0})):
        with pytest.raises(ValueError):
            R.AdjustParams(**kw)
    top = float(np.finfo(np.float32).max)
    a = R.AdjustParams(top, -top, top, bias={np.int64(3): top, 4: -np.inf, 2.0: np.inf, 5: 1e-50})
    assert a.penalizes and a.bias_id.tolist() == [3, 4, 2, 5] and a.bias.tolist() == [top, -np.inf, np.inf, 0.0]
    assert R.AdjustParams(1e-45).repetition == 1e-45 and R.AdjustParams(presence=1e-50).penalizes


def test_histories_of_finished_sequences_are_given_back(loop):
    """Prompts on the device stay as they are while their sequences run, beside sequences that come and go."""
    cb, rng, live = loop(), np.random.default_rng(0), []
    for rid in range(300):
        s = R._Seq(rid, 0, rng.integers(0, 9, rng.integers(1, 40)), int(rng.integers(1, 30)), 16)
        cb._place_history(s)
        live.append(s)
        if len(live) > 7:
            gone = live.pop(int(rng.integers(0, len(live))))
            cb._give_history(gone.hist, len(gone.prompt) + gone.max_new)
        spans = sorted((x.hist, x.hist + len(x.prompt) + x.max_new) for x in live)
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and spans[-1][1] <= cb._hist.numel()
        for x in live:
            assert np.array_equal(cb._hist[x.hist:x.hist + len(x.prompt)].numpy(), x.prompt)
    assert cb._hist.numel() <= 4 * 8 * 69
    for s in live:
        cb._give_history(s.hist, len(s.prompt) + s.max_new)
    assert cb._hist_free == [(cb._hist.numel(), 0)]
