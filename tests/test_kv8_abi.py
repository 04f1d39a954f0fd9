"""Host-side checks of the calls over an 8-bit cache and of the adjustment of head outputs (no GPU): every call below is
refused, or answered from the plan alone, before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2606_09643_amd import binding as B
from tests import kv8_common as K
from tests import test_decode_abi as A
from tests.test_decode_abi import BAD_ATTN, DH, H, KH, PTR, TABLE, _attn, _batch, _kv


def _kv8(table=TABLE, exps=PTR, **kw):
    t, k = _kv(table, **kw)
    return t, B.vfm_kv_pages_q8(k, exps)


def _attend(attn=None, batch=None, kv=None, q=PTR, ldq=H * DH, out=PTR, ldo=H * DH, ws=PTR, nb=1 << 40):
    host, b = batch if batch is not None else _batch()
    t, k = kv if kv is not None else _kv8()
    return B.lib().vfm_attention_paged_q8(C.byref(attn if attn is not None else _attn()), C.byref(b), q, ldq,
                                          C.byref(k), out, ldo, ws, nb, 1)


def _append(attn=None, batch=None, kv=None, qkv=PTR, ld=(H + 2 * KH) * DH, q_out=PTR):
    host, b = batch if batch is not None else _batch()
    t, k = kv if kv is not None else _kv8()
    return B.lib().vfm_kv_append_q8(C.byref(attn if attn is not None else _attn()), C.byref(b), qkv, ld, q_out,
                                    C.byref(k), 1)


@pytest.mark.parametrize("bad,status", BAD_ATTN)
def test_attention_descriptions_are_refused(bad, status):
    assert _attend(attn=_attn(**bad), ldq=1 << 20, ldo=1 << 20) == status
    assert _append(attn=_attn(**bad), ld=1 << 20) == status
    host, b = _batch()
    n = C.c_size_t()
    assert B.lib().vfm_attention_workspace_q8(C.byref(_attn(**bad)), C.byref(b), C.byref(n)) == status


def test_arguments_are_refused():
    lib, (host, b) = B.lib(), _batch()
    assert lib.vfm_attention_paged_q8(C.byref(_attn()), C.byref(b), PTR, 256, None, PTR, 256, PTR, 0, 1) == B.VFM_ERR_ARG
    assert lib.vfm_kv_append_q8(C.byref(_attn()), C.byref(b), PTR, 512, PTR, None, 1) == B.VFM_ERR_ARG
    for bad in (dict(q=None), dict(out=None), dict(q=PTR + 8), dict(out=PTR + 2), dict(kv=_kv8(exps=None)),
                dict(kv=_kv8(exps=PTR + 2))):
        assert _attend(**bad) == B.VFM_ERR_ARG, bad
    for bad in (dict(qkv=None), dict(q_out=None), dict(qkv=PTR + 8), dict(q_out=PTR + 8), dict(kv=_kv8(exps=None)),
                dict(kv=_kv8(exps=PTR + 8))):
        assert _append(**bad) == B.VFM_ERR_ARG, bad
    for bad in (dict(ldq=H * DH - 8), dict(ldo=H * DH - 8), dict(ldq=H * DH + 4), dict(ldo=H * DH + 1)):
        assert _attend(**bad) == B.VFM_ERR_SHAPE, bad
    for bad in (dict(ld=(H + 2 * KH) * DH - 8), dict(ld=(H + 2 * KH) * DH + 4)):
        assert _append(**bad) == B.VFM_ERR_SHAPE, bad
    long = _batch(lens=(1, 1), ctx=(5000, 0))
    kv = _kv8(np.zeros((2, 400)), n_pages=1)
    need = B.vfm_attention_workspace_q8(_attn(), long[1])
    assert need > 0
    for bad in (dict(ws=None), dict(nb=need - 1), dict(ws=PTR + 16)):
        assert _attend(batch=long, kv=kv, **bad) == B.VFM_ERR_WORKSPACE, bad


def test_caches_and_pages_are_refused():
    for bad in (dict(page=8), dict(page=48), dict(page=2048), dict(k=None), dict(v=None), dict(k=PTR + 4)):
        assert _attend(kv=_kv8(**bad)) == B.VFM_ERR_ARG, bad
        assert _append(kv=_kv8(**bad)) == B.VFM_ERR_ARG, bad
    for bad in (dict(n_pages=0), dict(max_pages=0), dict(n_pages=1 << 27), dict(max_pages=2)):
        assert _attend(kv=_kv8(**bad)) == B.VFM_ERR_SHAPE, bad
        assert _append(kv=_kv8(**bad)) == B.VFM_ERR_SHAPE, bad
    batch = _batch(lens=(1,), ctx=(100,), tasks=(0,))
    for window, n_sink, seen in ((0, 0, range(7)), (20, 0, (5, 6)), (17, 1, (0, 5, 6))):
        for j in seen:
            for bad in (-1, 50):
                t = np.arange(8).reshape(1, 8).copy()
                t[0, j] = bad
                assert _attend(attn=_attn(window=window, n_sink=n_sink), batch=batch, kv=_kv8(t), nb=0, ws=None) \
                    == B.VFM_ERR_SHAPE, (j, bad)
    t = np.full((1, 8), -1)
    assert _append(batch=batch, kv=_kv8(t)) == B.VFM_ERR_SHAPE
    t[0, 6] = 50
    assert _append(batch=batch, kv=_kv8(t)) == B.VFM_ERR_SHAPE
    far = _batch(lens=(2,), ctx=((1 << 30) - 1,), tasks=(0,))
    assert _attend(attn=_attn(window=5), batch=far) == B.VFM_ERR_SHAPE
    assert _append(batch=far) == B.VFM_ERR_SHAPE


def test_layer_is_refused():
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    cfg = R.cfg_for(wl.WORKLOADS[5])
    cfg.attn = B.VFM_ATTN_MIXED
    W = B.vfm_layer_weights(*[PTR] * len(B.vfm_layer_weights._fields_))
    host, b = _batch()
    t, k = _kv8()

    def call(cfg=cfg, batch=b, kv=k, window=16, n_sink=4, ws=PTR, nb=1 << 40, x=PTR):
        return B.lib().vfm_layer_forward_q8(C.byref(cfg), C.byref(W), None, C.byref(batch), x, C.byref(kv), window,
                                            n_sink, ws, nb, 1)
    assert call(window=-1) == B.VFM_ERR_ARG and call(n_sink=-1) == B.VFM_ERR_ARG and call(x=None) == B.VFM_ERR_ARG
    assert call(kv=_kv8(exps=None)[1]) == B.VFM_ERR_ARG
    bidir = B.vfm_cfg.from_buffer_copy(cfg)
    bidir.attn = B.VFM_ATTN_BIDIR
    host0, b0 = _batch(ctx=(0, 0))
    assert call(cfg=bidir, batch=b0) == B.VFM_ERR_UNSUPPORTED
    dec = B.vfm_cfg.from_buffer_copy(cfg)
    dec.attn = B.VFM_ATTN_DECODE
    assert call(cfg=dec) == B.VFM_ERR_UNSUPPORTED
    bad = TABLE.copy()
    bad[0, 6] = -1
    t2, k2 = _kv8(bad)
    assert call(kv=k2) == B.VFM_ERR_SHAPE
    n = C.c_size_t()
    lib = B.lib()
    assert lib.vfm_workspace_size_q8(C.byref(cfg), C.byref(b), None, -1, 0, C.byref(n)) == B.VFM_ERR_ARG
    assert lib.vfm_workspace_size_q8(C.byref(cfg), C.byref(b), None, 16, 0, None) == B.VFM_ERR_ARG
    need = B.vfm_workspace_size_q8(cfg, b, None, 16, 4)
    assert need > 0


def test_batches_larger_than_a_launch_are_refused():
    n = 1 << 24
    host = B.vfm_plan(np.zeros(1, np.int32), np.array([n]), 1, ctx_len=np.array([0]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    assert _append(batch=(host, b), kv=_kv8(np.zeros((1, n // 1024)), page=1024, n_pages=1)) == B.VFM_ERR_UNSUPPORTED


def _adjust(batch=None, out=PTR, adjusted=PTR, **kw):
    host, b = batch if batch is not None else _batch()
    a = B.vfm_adjust(**kw)
    return B.lib().vfm_adjust_outputs(C.byref(b), out, C.byref(a), adjusted, 1)


def test_adjustments_are_refused():
    host, b = _batch()
    assert B.lib().vfm_adjust_outputs(None, PTR, C.byref(B.vfm_adjust()), PTR, 1) == B.VFM_ERR_ARG
    assert B.lib().vfm_adjust_outputs(C.byref(b), PTR, None, PTR, 1) == B.VFM_ERR_ARG
    lists = dict(hist=PTR, hist_begin=PTR, hist_len=PTR), dict(bias=PTR, bias_id=PTR, bias_begin=PTR, bias_len=PTR), \
        dict(mask=PTR, mask_row=PTR, n_masks=1, mask_words=1)
    for bad in (dict(out=None), dict(adjusted=None), dict(out=PTR + 4), dict(adjusted=PTR + 8)):
        assert _adjust(**bad) == B.VFM_ERR_ARG, bad
    for whole in lists:
        head = next(iter(whole))
        for n in whole:
            if n != head and not n.startswith(("n_", "mask_words")):
                assert _adjust(**{**whole, n: None}) == B.VFM_ERR_ARG, n
    for bad in ({**lists[0], "n_hist": -1}, {**lists[1], "n_bias": -1}, {**lists[2], "n_masks": -1},
                {**lists[2], "mask_words": 0}):
        assert _adjust(**bad) == B.VFM_ERR_SHAPE, bad


def test_adjustments_larger_than_a_launch_are_refused():
    n = (1 << 23) + 1
    host = B.vfm_plan(np.zeros(n, np.int32), np.ones(n, np.int32), 1, n_out=np.array([2]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    assert _adjust(batch=(host, b)) == B.VFM_ERR_UNSUPPORTED
    del host, b
    # many short rows beside one long one: the blocks are those of the longest
    n = 1 << 20
    tasks = np.zeros(n, np.int32)
    tasks[-1] = 1
    host = B.vfm_plan(tasks, np.ones(n, np.int32), 2, n_out=np.array([2, 1 << 27]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    assert _adjust(batch=(host, b)) == B.VFM_ERR_UNSUPPORTED


def test_binding_checks_operands():
    host, b = _batch(lens=(1, 2), ctx=(3, 0))
    a = _attn()
    kp = torch.zeros(KH, 10 * 16, DH, dtype=torch.uint8)
    ex = torch.zeros(10, KH, 2, dtype=torch.uint8)
    table = np.arange(2 * 4).reshape(2, 4)
    for bad in (dict(k=kp.float()), dict(v=kp.to(torch.int8)), dict(exps=ex.int())):
        with pytest.raises(ValueError):
            B.PagedKVQ8(**{**dict(k=kp, v=kp, exps=ex, page_size=16, table=table, device="cpu"), **bad})
    kv = B.PagedKVQ8(kp, kp.clone(), ex, 16, table, device="cpu")
    assert B.PagedKVQ8(kp.view(torch.float8_e4m3fn), kp, ex, 16, table, device="cpu").layout == kv.layout is not None
    q = torch.zeros(3, H * DH, dtype=torch.bfloat16)
    qkv = torch.zeros(3, (H + 2 * KH) * DH, dtype=torch.bfloat16)
    for bad in (q[:2], q.float(), q[:, :-8], torch.zeros(3, DH, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            B.vfm_attention_paged_q8(a, b, bad, kv, q.clone(), None, stream=1)
        with pytest.raises(ValueError):
            B.vfm_attention_paged_q8(a, b, q, kv, bad, None, stream=1)
        with pytest.raises(ValueError):
            B.vfm_kv_append_q8(a, b, bad, q, kv, stream=1)
    # operands that would pass but for their device never reach the library
    for call in (lambda: B.vfm_attention_paged_q8(a, b, q, kv, q.clone(), None, stream=1),
                 lambda: B.vfm_kv_append_q8(a, b, qkv, q, kv, stream=1),
                 lambda: B.vfm_adjust_outputs(b, torch.zeros(14), B.OutputAdjust(), stream=1)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    for layout in (ex[:9], ex.permute(2, 1, 0), torch.zeros(10, 2, KH + 1, dtype=torch.uint8)):
        assert B.PagedKVQ8(kp, kp, layout, 16, table, device="cpu").layout is None


def test_binding_checks_adjustments():
    i32, f32, i64 = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.int32, torch.float32, torch.int64))
    good = dict(repetition=f32(2), hist=i32(9), hist_begin=i64(2), hist_len=i32(2), bias=f32(3), bias_id=i32(3),
                bias_begin=i64(2), bias_len=i32(2), mask=i32(1, 4), mask_row=i32(2))
    assert B.OutputAdjust(**good).n == 2
    for bad in (dict(repetition=i32(2)), dict(hist=i64(9)), dict(hist_begin=i32(2)), dict(mask=i32(4)),
                dict(mask=torch.zeros(1, 4)), dict(bias=None, bias_id=f32(3)), dict(hist_len=None), dict(bias_id=None),
                dict(mask_row=None), dict(nonsense=f32(2)), dict(bias_id=i32(2)), dict(repetition=f32(4)[::2]),
                dict(mask=i32(1, 0))):
        with pytest.raises(ValueError):
            B.OutputAdjust(**{**good, **bad})
    host, b = _batch()
    with pytest.raises(ValueError):                      # for fewer requests than the batch has
        B.vfm_adjust_outputs(b, f32(14), B.OutputAdjust(repetition=f32(1)), stream=1)


def test_plain_forms():
    """The 64-bit forms that the GPU tests hold kernels to: codes against torch's e4m3, exponents at their borders."""
    x = np.concatenate([np.random.default_rng(0).standard_normal(20000) * 60, K.VALUES[:127], -K.VALUES[:127],
                        (K.VALUES[:126] + K.VALUES[1:127]) / 2, [448.0, -448.0, 0.0, -0.0, 2.0 ** -10, 2.0 ** -11]])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(K.to_codes(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert np.array_equal(np.nan_to_num(K.VALUES, nan=7.0),
                          np.nan_to_num(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), nan=7.0))
    for a, e in ((0.0, 1), (448.0, 127), (np.nextafter(448.0, 500), 128), (1.75, 119), (1.0, 119), (1.7500001, 120),
                 (K.TOP, 247), (2.0 ** -126, 1)):
        assert K.exponent_of(a) == e, a
    got = K.adjust([1.0, -1.0, 2.0, 0.5], r=2.0, p=0.5, f=0.25, hist=[0, 1, 1, 9, -3, 0], n_prompt=1,
                   bias=[(2, 5.0), (2, 1.0), (77, 1.0)], allowed=np.array([True, True, True, False]))
    assert got.tolist() == [0.5 - 0.75, -2.0 - 1.0, 3.0, -np.inf]
    assert np.isnan(K.adjust([1.0, 2.0], allowed=np.zeros(2, bool))).all()
    assert K.mask_words(np.arange(40) % 2 == 1, 2).view(np.uint32).tolist() == [0xAAAAAAAA, 0xAA]
    assert A.PTR == PTR


class _Model:
    """Just what the batcher reads before a step runs."""

    def __init__(self):
        from paper_2606_09643_amd import runner as R
        from paper_2606_09643_amd import workloads as wl
        self.w = wl.WORKLOADS[5].replace(n_layers=1, d=256, n_heads=2, head_dim=128, d_ff=512, n_tasks=3)
        self.n_layers, self.cfg = 1, R.cfg_for(self.w)
        self.heads = wl.Heads(np.array([7, 100, 33], np.int32), [], [])


def test_adjust_parameters_are_refused():
    from paper_2606_09643_amd import runner as R
    for kw in (dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=float("nan")), dict(repetition=float("inf")),
               dict(presence=float("nan")), dict(frequency=float("inf")), dict(bias={-1: 1.0}), dict(bias={2: float("nan")})):
        with pytest.raises(ValueError):
            R.AdjustParams(**kw)
    cb = R.ContinuousBatcher(_Model(), emb=None, page_size=16, n_pages=12, max_seqs=3, max_step_tokens=64, max_pages=6,
                             device="cpu", kv8=True)
    assert cb.k[0].dtype == torch.uint8 and cb.exps[0].shape == (12, 2, 2)
    for task, a in ((0, R.AdjustParams(bias={7: 1.0})), (1, R.AdjustParams(allowed=np.ones(99))),
                    (2, R.AdjustParams(allowed=np.ones((1, 33))))):
        with pytest.raises(ValueError):
            cb.submit(0, task, np.zeros(3, np.int32), 2, adjust=a)
    cb.submit(0, 1, np.zeros(3, np.int32), 2, adjust=R.AdjustParams(bias={99: -np.inf}, allowed=np.ones(100)))
    assert cb.waiting[0].adjust.penalizes is False


def test_histories_have_their_own_room():
    """Parts of the device's token buffer: none overlap while their sequences run, those of finished ones are used again."""
    from paper_2606_09643_amd import runner as R
    cb = R.ContinuousBatcher(_Model(), emb=None, page_size=16, n_pages=40, max_seqs=8, max_step_tokens=64, max_pages=6,
                             device="cpu", kv8=True)
    cb._h2d = lambda a: torch.from_numpy(np.ascontiguousarray(a))
    rng = np.random.default_rng(0)
    live, total = [], 0
    for rid in range(200):
        s = R._Seq(rid, 0, rng.integers(0, 9, rng.integers(1, 40)), int(rng.integers(1, 30)), 16)
        cb._place_history(s)
        live.append(s)
        total = max(total, sum(len(x.prompt) + x.max_new for x in live))
        if len(live) > 7:
            gone = live.pop(int(rng.integers(0, len(live))))
            cb._hist_free.append((len(gone.prompt) + gone.max_new, gone.hist))
        spans = sorted((x.hist, x.hist + len(x.prompt) + x.max_new) for x in live)
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and spans[-1][1] <= cb._hist.numel()
        for x in live:
            assert np.array_equal(cb._hist[x.hist:x.hist + len(x.prompt)].numpy(), x.prompt)
    assert cb._hist.numel() <= 16 * total


def test_loop_device_tokens_of_finished_sequences_are_used_again():
    """Parts do not overlap while they are taken, free neighbours become one, and the buffer stays bounded."""
    from paper_2606_09643_amd import runner as R
    cb = R.ContinuousBatcher(_Model(), emb=None, page_size=16, n_pages=12, max_seqs=3, max_step_tokens=64, max_pages=6,
                             device="cpu")
    rng, live = np.random.default_rng(0), []
    for i in range(4000):
        if len(live) == 8 or (live and rng.random() < 0.4):
            cb._give_history(*live.pop(int(rng.integers(len(live)))))
        else:
            n = int(rng.integers(1, 200))
            live.append((cb._take_history(n), n))
        parts = sorted([(b, n) for b, n in live] + [(b, n) for n, b in cb._hist_free])
        assert parts[0][0] == 0 and all(a + n == b for (a, n), (b, _) in zip(parts, parts[1:]))
        assert sum(parts[-1]) == cb._hist.numel()
    assert cb._hist.numel() <= 4 * 8 * 200
    for part in live:
        cb._give_history(*part)
    assert cb._hist_free == [(cb._hist.numel(), 0)]
