"""Host-side scheduling of the continuous-batching loop (no GPU): which
prompts join the running batch under the sequence slots, the per-step token
budget and the page commitments, FIFO and BFQ admission, and that a request
that can never fit is refused up front."""
import numpy as np
import pytest

from paper_2606_09643_amd import binding as B
from paper_2606_09643_amd import runner as R
from paper_2606_09643_amd import workloads as wl


class _StubModel:
    """Just what the batcher reads before a step runs."""

    def __init__(self):
        self.w = wl.WORKLOADS[5].replace(n_layers=1, d=256, n_heads=2, head_dim=128, d_ff=512, n_tasks=3)
        self.n_layers = 1
        self.cfg = R.cfg_for(self.w)


def _batcher(**kw):
    args = dict(page_size=16, n_pages=12, max_seqs=3, max_step_tokens=64, max_pages=6, device="cpu")
    args.update(kw)
    return R.ContinuousBatcher(_StubModel(), emb=None, **args)


def test_fifo_admission_respects_slots_tokens_and_pages():
    cb = _batcher()
    # budgets (pages of 16 for prompt + new - 1 tokens): 1, 2, 1, 3, 2
    for rid, (L, n) in enumerate([(5, 6), (17, 3), (1, 8), (33, 4), (9, 9)]):
        cb.submit(rid, rid % 3, np.zeros(L, np.int32), n)
    new = cb._admit(0.0)
    # slots: 3; tokens 5 + 17 + 1 = 23 <= 64; pages 1 + 2 + 1 = 4 <= 12
    assert [s.rid for s in new] == [0, 1, 2] and cb.committed == 4
    assert [s.rid for s in cb.waiting] == [3, 4]
    assert cb._admit(0.0) == []                      # no slot free
    # a finished sequence frees its slot and pages
    s0 = cb.running[0]
    cb.alloc.release(s0.slot)
    cb.free_slots.append(s0.slot)
    cb.committed -= s0.budget
    cb.running.remove(s0)
    new = cb._admit(0.0)                             # 2 decode rows + 33 prompt tokens <= 64
    assert [s.rid for s in new] == [3] and cb.committed == 6


def test_fifo_admission_stops_at_the_first_prompt_that_does_not_fit():
    cb = _batcher(max_step_tokens=40, chunk_prompts=False)
    for rid, L in enumerate([30, 20, 5]):
        cb.submit(rid, 0, np.zeros(L, np.int32), 2)
    assert [s.rid for s in cb._admit(0.0)] == [0]    # 30 + 20 > 40: FIFO does not skip ahead
    assert [s.rid for s in cb.waiting] == [1, 2]


def test_chunked_prompts_join_with_what_is_left_of_the_budget():
    cb = _batcher(max_step_tokens=40, max_pages=6)
    for rid, L in enumerate([30, 20, 5]):
        cb.submit(rid, 0, np.zeros(L, np.int32), 2)
    # 30 tokens, then 10 of the 20-token prompt; the third has no token left this step
    assert [s.rid for s in cb._admit(0.0)] == [0, 1]
    assert [s.rid for s in cb.waiting] == [2]


def test_page_commitment_holds_back_prompts():
    cb = _batcher(n_pages=4, max_pages=4, max_step_tokens=1000)
    cb.submit(0, 0, np.zeros(40, np.int32), 10)      # 49 tokens: 4 pages
    cb.submit(1, 1, np.zeros(3, np.int32), 2)        # 1 page
    assert [s.rid for s in cb._admit(0.0)] == [0]
    assert cb.committed == 4 and [s.rid for s in cb.waiting] == [1]


def test_bfq_admission_takes_whole_batches_in_tag_order():
    bfq = B.BFQ([1.0, 1.0, 1.0], [0.0, 1.0, 1.5], b_max=2)
    cb = _batcher(bfq=bfq, max_seqs=4)
    for rid, task in enumerate([0, 0, 1, 2]):
        cb.submit(rid, task, np.zeros(4, np.int32), 3)
    new = cb._admit(0.0)
    # start tags: task 0: 0, 1; task 1: 0; task 2: 0 -> batches (0, 2) then (3, 1)
    assert [s.rid for s in new] == [0, 2, 3, 1]
    assert cb.waiting == []


def test_requests_that_can_never_fit_are_refused():
    cb = _batcher(max_pages=2)
    with pytest.raises(ValueError):
        cb.submit(0, 0, np.zeros(40, np.int32), 1)   # 40 tokens need 3 pages of 16
    with pytest.raises(ValueError):
        cb.submit(1, 0, np.zeros(0, np.int32), 1)    # empty prompt


def test_windowed_sequences_hold_a_ring_of_pages():
    """Pages of 16, window 40, 20 sinks: 2 pages for the sinks and, with at most 40 new rows a step, ring pages for
    79 positions in a row, which touch at most 6."""
    cb = _batcher(n_pages=32, max_pages=8, max_step_tokens=64, window=40, n_sink=20)
    assert cb.chunk and cb.max_chunk == 40
    cb.submit(0, 0, np.zeros(200, np.int32), 10000)      # far more positions than the pool has
    cb.submit(1, 0, np.zeros(3, np.int32), 20)           # 22 positions: no ring needed
    cb.submit(2, 0, np.zeros(1, np.int32), 10000)        # window - 1 + 1 positions: 4 pages
    a, b, c = cb._admit(0.0)
    assert [s.budget for s in (a, b, c)] == [8, 2, 6] and cb.committed == 16
    rng = np.random.default_rng(0)
    for s, most in ((a, 40), (c, 1)):
        ctx, owner = 0, {}                               # physical page -> the logical page that was written last
        while ctx < 3000:
            n = min(int(rng.integers(1, most + 1)), len(s.prompt) - ctx) if ctx < len(s.prompt) else 1
            t = cb._tables([s, b], [ctx + n, 5])
            assert t.shape[1] == -(-(ctx + n) // 16)
            for j in range(ctx // 16, t.shape[1]):
                owner[int(t[0, j])] = j
            first = max(0, ctx - 40 + 1) // 16
            for j in list(range(first, t.shape[1])) + [j for j in (0, 1) if j < t.shape[1]]:
                assert owner[int(t[0, j])] == j          # a page that some row sees still holds its positions
            ctx += n
        assert len(owner) <= s.budget == cb.alloc.count(s.slot)[0]
    held = {int(p) for s in (a, b, c) for p in cb.alloc.table([s.slot])[0][:cb.alloc.count(s.slot)[0]]}
    assert len(held) == sum(cb.alloc.count(s.slot)[0] for s in (a, b, c))      # no page belongs to two


def test_windowed_prompts_take_bounded_chunks():
    cb = _batcher(n_pages=32, max_pages=8, max_step_tokens=64, window=40)
    cb.submit(0, 0, np.zeros(100, np.int32), 2)
    cb.submit(1, 0, np.zeros(100, np.int32), 2)
    a, b = cb._admit(0.0)
    assert cb._rows(a, 64) == 40 and cb._rows(b, 24) == 24


def test_windows_and_sampling_parameters_are_refused():
    for kw in (dict(window=0), dict(window=16, n_sink=-1), dict(max_chunk=0)):
        with pytest.raises(ValueError):
            _batcher(**kw)
    for kw in (dict(temperature=-0.5), dict(temperature=float("nan")), dict(top_k=-1), dict(top_k=2 ** 31),
               dict(top_p=-0.1), dict(min_p=float("nan"))):
        with pytest.raises(ValueError):
            R.SamplingParams(**kw)


def test_requests_without_a_seed_draw_their_own_numbers():
    """Two requests with the default parameters do not share a run of uniform numbers; a given seed repeats its own."""
    def numbers(seq):
        return [float(seq.rng.random(dtype=np.float32)) for _ in range(20)]
    cb = _batcher(n_pages=32, max_pages=8)
    same = R.SamplingParams(1.0)
    for rid, sp in enumerate([R.SamplingParams(), R.SamplingParams(), same, same, R.SamplingParams(seed=3),
                              R.SamplingParams(seed=3)]):
        cb.submit(rid, 0, np.zeros(3, np.int32), 2, sampling=sp)
    runs = [numbers(cb.requests[rid]) for rid in range(6)]
    for i in range(4):
        for j in range(i):
            assert runs[i] != runs[j], (i, j)
    assert runs[4] == runs[5] == [float(x) for x in np.random.default_rng(3).random(20, dtype=np.float32)]


def test_windows_that_the_library_refuses_are_refused_up_front():
    for kw in (dict(window=(1 << 30) + 1), dict(window=1 << 33), dict(window=16, n_sink=(1 << 30) + 1), dict(window=2.5),
               dict(window=float("inf")), dict(window=float("nan")), dict(window=16, n_sink=0.5)):
        with pytest.raises(ValueError):
            _batcher(**kw)
    assert _batcher(window=1 << 30, max_step_tokens=64).max_chunk == 64
