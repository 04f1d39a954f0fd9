"""Host-side checks of the bounded-cache decoding calls (no GPU): every call
below is refused, or answered from the plan alone, before anything is launched."""
import ctypes as C

import numpy as np
import pytest

from paper_2606_09643_amd import binding as B

PTR = 1 << 20          # an aligned address that is never read: the calls are refused before a launch
H, KH, DH = 4, 2, 64


def _batch(lens=(1, 40), ctx=(100, 0), tasks=(0, 0)):
    host = B.vfm_plan(np.array(tasks), np.array(lens), 1 + max(tasks), ctx_len=np.array(ctx),
                      n_out=np.full(1 + max(tasks), 7))
    return host, B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)


def _kv(table, page=16, n_pages=50, k=PTR, v=PTR, max_pages=None):
    t = np.ascontiguousarray(table, np.int32)
    return t, B.vfm_kv_pages(k, v, n_pages, page, t.shape[1] if max_pages is None else max_pages,
                             t.ctypes.data_as(C.POINTER(C.c_int32)), PTR)


def _attn(**kw):
    a = dict(dtype=B.VFM_BF16, n_heads=H, n_kv_heads=KH, head_dim=DH, window=0, n_sink=0, scale=0.0, rope_theta=0.0)
    a.update(kw)
    return B.make_attn(**a)


TABLE = np.arange(2 * 8).reshape(2, 8)


def _attend(attn=None, batch=None, kv=None, q=PTR, ldq=H * DH, out=PTR, ldo=H * DH, ws=PTR, nb=1 << 40):
    host, b = batch if batch is not None else _batch()
    t, k = kv if kv is not None else _kv(TABLE)
    a = attn if attn is not None else _attn()
    return B.lib().vfm_attention_paged(C.byref(a), C.byref(b), q, ldq, C.byref(k), out, ldo, ws, nb, 1)


def _append(attn=None, batch=None, kv=None, qkv=PTR, ld=(H + 2 * KH) * DH, q_out=PTR):
    host, b = batch if batch is not None else _batch()
    t, k = kv if kv is not None else _kv(TABLE)
    a = attn if attn is not None else _attn()
    return B.lib().vfm_kv_append(C.byref(a), C.byref(b), qkv, ld, q_out, C.byref(k), 1)


BAD_ATTN = [
    (dict(dtype=7), B.VFM_ERR_ARG), (dict(head_dim=96), B.VFM_ERR_UNSUPPORTED), (dict(n_heads=0), B.VFM_ERR_SHAPE),
    (dict(n_heads=2048, n_kv_heads=2048), B.VFM_ERR_SHAPE), (dict(n_kv_heads=3), B.VFM_ERR_SHAPE),
    (dict(n_kv_heads=0), B.VFM_ERR_SHAPE), (dict(n_heads=65, n_kv_heads=1), B.VFM_ERR_UNSUPPORTED),
    (dict(window=-1), B.VFM_ERR_ARG), (dict(window=(1 << 30) + 1), B.VFM_ERR_ARG), (dict(n_sink=-1), B.VFM_ERR_ARG),
    (dict(scale=-0.1), B.VFM_ERR_ARG), (dict(scale=float("nan")), B.VFM_ERR_ARG),
    (dict(scale=float("inf")), B.VFM_ERR_ARG), (dict(rope_theta=-1.0), B.VFM_ERR_ARG),
    (dict(rope_theta=float("nan")), B.VFM_ERR_ARG)]


@pytest.mark.parametrize("bad,status", BAD_ATTN)
def test_attention_descriptions_are_refused(bad, status):
    wide = dict(ldq=1 << 20, ldo=1 << 20)
    assert _attend(attn=_attn(**bad), **wide) == status
    assert _append(attn=_attn(**bad), ld=1 << 20) == status
    host, b = _batch()
    n = C.c_size_t()
    assert B.lib().vfm_attention_workspace(C.byref(_attn(**bad)), C.byref(b), C.byref(n)) == status


def test_attention_arguments_are_refused():
    lib, (host, b), (t, k) = B.lib(), _batch(), _kv(TABLE)
    n = C.c_size_t()
    assert lib.vfm_attention_workspace(None, C.byref(b), C.byref(n)) == B.VFM_ERR_ARG
    assert lib.vfm_attention_workspace(C.byref(_attn()), None, C.byref(n)) == B.VFM_ERR_ARG
    assert lib.vfm_attention_workspace(C.byref(_attn()), C.byref(b), None) == B.VFM_ERR_ARG
    assert lib.vfm_attention_paged(C.byref(_attn()), C.byref(b), PTR, 256, None, PTR, 256, PTR, 0, 1) == B.VFM_ERR_ARG
    for bad in (dict(q=None), dict(out=None), dict(q=PTR + 8), dict(out=PTR + 2)):
        assert _attend(**bad) == B.VFM_ERR_ARG, bad
    for bad in (dict(ldq=H * DH - 8), dict(ldo=H * DH - 8), dict(ldq=H * DH + 4), dict(ldo=H * DH + 1)):
        assert _attend(**bad) == B.VFM_ERR_SHAPE, bad
    # a long context of few heads needs records: workspace missing, small or unaligned
    long = _batch(lens=(1, 1), ctx=(5000, 0))
    kv = _kv(np.zeros((2, 400)), n_pages=1)
    need = B.vfm_attention_workspace(_attn(), long[1])
    assert need > 0
    for bad in (dict(ws=None), dict(nb=need - 1), dict(ws=PTR + 16)):
        assert _attend(batch=long, kv=kv, **bad) == B.VFM_ERR_WORKSPACE, bad


def test_caches_are_refused():
    for bad in (dict(page=8), dict(page=48), dict(page=2048), dict(k=None), dict(v=None), dict(k=PTR + 4)):
        assert _attend(kv=_kv(TABLE, **bad)) == B.VFM_ERR_ARG, bad
        assert _append(kv=_kv(TABLE, **bad)) == B.VFM_ERR_ARG, bad
    for bad in (dict(n_pages=0), dict(max_pages=0), dict(n_pages=1 << 27), dict(max_pages=2)):
        assert _attend(kv=_kv(TABLE, **bad)) == B.VFM_ERR_SHAPE, bad
        assert _append(kv=_kv(TABLE, **bad)) == B.VFM_ERR_SHAPE, bad


@pytest.mark.parametrize("window,n_sink,seen", [(0, 0, range(7)), (20, 0, (5, 6)), (1, 0, (6,)), (16, 0, (5, 6)),
                                                (17, 1, (0, 5, 6)), (5, 17, (0, 1, 6)), (5, 100, range(7)),
                                                (1000, 0, range(7))])
def test_pages_that_rows_see_have_to_exist(window, n_sink, seen):
    """One row at position 100 (pages of 16: 0 .. 6): a bad id in a seen page is
    refused, one in any other page is not looked at.  The calls with a good table
    stop at the workspace or the next argument check, never at a launch: out NULL."""
    batch = _batch(lens=(1,), ctx=(100,), tasks=(0,))
    for j in range(8):
        for bad in (-1, 50):
            t = np.arange(8).reshape(1, 8).copy()
            t[0, j] = bad
            st = _attend(attn=_attn(window=window, n_sink=n_sink), batch=batch, kv=_kv(t), nb=0, ws=None) \
                if j in seen else None
            if j in seen:
                assert st == B.VFM_ERR_SHAPE, (j, bad)
    # the append looks at the new position's page alone
    t = np.full((1, 8), -1)
    assert _append(batch=batch, kv=_kv(t)) == B.VFM_ERR_SHAPE
    t[0, 6] = 50
    assert _append(batch=batch, kv=_kv(t)) == B.VFM_ERR_SHAPE


def test_append_arguments_are_refused():
    for bad in (dict(qkv=None), dict(q_out=None), dict(qkv=PTR + 8), dict(q_out=PTR + 8)):
        assert _append(**bad) == B.VFM_ERR_ARG, bad
    for bad in (dict(ld=(H + 2 * KH) * DH - 8), dict(ld=(H + 2 * KH) * DH + 4)):
        assert _append(**bad) == B.VFM_ERR_SHAPE, bad


def test_far_positions_are_refused():
    batch = _batch(lens=(2,), ctx=((1 << 30) - 1,), tasks=(0,))
    assert _attend(attn=_attn(window=5), batch=batch) == B.VFM_ERR_SHAPE
    assert _append(batch=batch) == B.VFM_ERR_SHAPE


def test_workspace_follows_the_request_alone():
    """The records' chunk count comes from a request's own sizes; a batch takes
    the largest."""
    a = _attn(n_heads=32, n_kv_heads=32, head_dim=128)
    one = B.vfm_attention_workspace(a, _batch(lens=(1,), ctx=(2000,), tasks=(0,))[1])
    two = B.vfm_attention_workspace(a, _batch(lens=(1, 1), ctx=(2000, 3), tasks=(0, 0))[1])
    assert 0 < one < two <= 2 * one + 512
    assert B.vfm_attention_workspace(a, _batch(lens=(1,), ctx=(100,), tasks=(0,))[1]) == 0
    # a window bounds the keys, and with them the chunks
    w = _attn(n_heads=32, n_kv_heads=32, head_dim=128, window=128, n_sink=4)
    assert B.vfm_attention_workspace(w, _batch(lens=(1,), ctx=(100000,), tasks=(0,))[1]) == 0


def test_sample_arguments_are_refused():
    lib, (host, b) = B.lib(), _batch()
    s = B.vfm_sampling(None, None, None, None)
    ok = [C.byref(b), PTR, C.byref(s), PTR, PTR, None, 1]
    for i in (0, 1, 2, 3, 4):
        bad = list(ok)
        bad[i] = None
        assert lib.vfm_sample_tokens(*bad) == B.VFM_ERR_ARG, i


def test_windowed_layer_is_refused():
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    w = wl.WORKLOADS[5]
    cfg = R.cfg_for(w)
    cfg.attn = B.VFM_ATTN_MIXED
    W = B.vfm_layer_weights(*[PTR] * len(B.vfm_layer_weights._fields_))
    host, b = _batch()
    t, k = _kv(TABLE)

    def call(cfg=cfg, batch=b, kv=k, window=16, n_sink=4, ws=PTR, nb=1 << 40, x=PTR):
        return B.lib().vfm_layer_forward_windowed(C.byref(cfg), C.byref(W), None, C.byref(batch), x, C.byref(kv), window,
                                                  n_sink, ws, nb, 1)
    assert call(window=-1) == B.VFM_ERR_ARG and call(n_sink=-1) == B.VFM_ERR_ARG and call(x=None) == B.VFM_ERR_ARG
    bidir = B.vfm_cfg.from_buffer_copy(cfg)
    bidir.attn = B.VFM_ATTN_BIDIR
    host0, b0 = _batch(ctx=(0, 0))
    assert call(cfg=bidir, batch=b0) == B.VFM_ERR_UNSUPPORTED
    dec = B.vfm_cfg.from_buffer_copy(cfg)
    dec.attn = B.VFM_ATTN_DECODE
    assert call(cfg=dec) == B.VFM_ERR_UNSUPPORTED
    bad = TABLE.copy()
    bad[0, 6] = -1
    t2, k2 = _kv(bad)
    assert call(kv=k2) == B.VFM_ERR_SHAPE
    n = C.c_size_t()
    lib = B.lib()
    assert lib.vfm_workspace_size_windowed(C.byref(cfg), C.byref(b), None, -1, 0, C.byref(n)) == B.VFM_ERR_ARG
    assert lib.vfm_workspace_size_windowed(C.byref(cfg), C.byref(b), None, 16, 0, None) == B.VFM_ERR_ARG
    assert B.vfm_workspace_size_windowed(cfg, b, None, 16, 4) > 0


def test_binding_checks_operands():
    import torch
    host, b = _batch(lens=(1, 2), ctx=(3, 0))
    a = _attn()
    kp = torch.zeros(KH, 10 * 16, DH, dtype=torch.bfloat16)
    kv = B.PagedKV(kp, kp.clone(), 16, np.arange(2 * 4).reshape(2, 4), device="cpu")
    q = torch.zeros(3, H * DH, dtype=torch.bfloat16)
    for bad in (q[:2], q.float(), q[:, :-8], q.t().contiguous().t(), torch.zeros(3, DH, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            B.vfm_attention_paged(a, b, bad, kv, q.clone(), None, stream=1)
        with pytest.raises(ValueError):
            B.vfm_attention_paged(a, b, q, kv, bad, None, stream=1)
        with pytest.raises(ValueError):
            B.vfm_kv_append(a, b, bad, q, kv, stream=1)
    with pytest.raises(ValueError):                      # a pool of another head count
        B.vfm_attention_paged(_attn(n_kv_heads=4), b, q, kv, q.clone(), None, stream=1)
    with pytest.raises(ValueError):
        B.Sampling(top_k=torch.zeros(2))
    with pytest.raises(ValueError):
        B.Sampling(temperature=torch.zeros(2, dtype=torch.int32))
    u = torch.zeros(2)
    out, ids = torch.zeros(14), torch.zeros(2, dtype=torch.int32)
    for bad in (dict(out=torch.zeros(13)), dict(u=torch.zeros(1)), dict(ids=torch.zeros(2)), dict(logprob=ids),
                dict(sampling=B.Sampling(top_p=torch.zeros(1)))):
        args = dict(out=out, sampling=B.Sampling(), u=u, ids=ids, logprob=None)
        args.update(bad)
        with pytest.raises(ValueError):
            B.vfm_sample_tokens(b, args["out"], args["sampling"], args["u"], args["ids"], args["logprob"], stream=1)


def test_binding_refuses_host_memory():
    """Operands that would pass but for their device never reach the library."""
    import torch
    host, b = _batch(lens=(1, 2), ctx=(3, 0))
    a = _attn()
    kp = torch.zeros(KH, 10 * 16, DH, dtype=torch.bfloat16)
    kv = B.PagedKV(kp, kp.clone(), 16, np.arange(2 * 4).reshape(2, 4), device="cpu")
    q, qkv = torch.zeros(3, H * DH, dtype=torch.bfloat16), torch.zeros(3, (H + 2 * KH) * DH, dtype=torch.bfloat16)
    for call in (lambda: B.vfm_attention_paged(a, b, q, kv, q.clone(), None, stream=1),
                 lambda: B.vfm_kv_append(a, b, qkv, q, kv, stream=1),
                 lambda: B.vfm_sample_tokens(b, torch.zeros(14), B.Sampling(), torch.zeros(2),
                                             torch.zeros(2, dtype=torch.int32), stream=1)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


def test_sample_refuses_huge_heads():
    host = B.vfm_plan(np.array([0]), np.array([1]), 1, n_out=np.array([(1 << 30) + 1]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    s = B.vfm_sampling(None, None, None, None)
    assert B.lib().vfm_sample_tokens(C.byref(b), PTR, C.byref(s), PTR, PTR, None, 1) == B.VFM_ERR_SHAPE


def test_head_offsets_past_int32_are_refused():
    """Offsets of head outputs are 32-bit: a batch whose requests have 2^31 and more of them together would
    have offsets before the buffer, so it has no plan (and no call on heads or draws ever sees one)."""
    def plan(n_out, tasks):
        return B.vfm_plan(np.array(tasks), np.ones(len(tasks)), len(n_out), n_out=np.array(n_out))
    for n_out, tasks in (([1 << 30], [0, 0, 0]), ([1 << 30], [0, 0]), ([(1 << 31) - 1, 1], [0, 1]),
                         ([600000], [0] * 3580)):
        with pytest.raises(RuntimeError, match="vfm_plan"):
            plan(n_out, tasks)
    host = plan([(1 << 30), (1 << 30) - 1], [0, 1])          # 2^31 - 1 outputs: the last offset still fits
    assert host[6] == (1 << 31) - 1


def _ws(a, lens, ctx):
    host, b = _batch(lens=lens, ctx=ctx, tasks=[0] * len(lens))          # b points into host
    return B.vfm_attention_workspace(a, b)


@pytest.mark.parametrize("heads,kv_heads,dh,dtype,lens,ctx", [
    (32, 8, 128, B.VFM_BF16, [2048, 1], [0, 20000]), (32, 8, 128, B.VFM_BF16, [8192, 1], [0, 20000]),
    (32, 8, 128, B.VFM_BF16, [16384, 32], [0, 20000]), (32, 1, 128, B.VFM_BF16, [8192, 1], [0, 100000]),
    (32, 8, 128, B.VFM_BF16, [8192, 1], [0, 131072]), (8, 1, 128, B.VFM_BF16, [1] * 256, [100] * 255 + [60000]),
    (32, 32, 128, B.VFM_BF16, [1] * 200 + [4000], [50] * 199 + [4000, 0]), (8, 4, 64, B.VFM_F32, [4096, 1], [0, 20000]),
    (4, 2, 64, B.VFM_F32, [1000, 70, 1], [0, 9000, 30000])])
def test_workspace_is_that_of_the_requests(heads, kv_heads, dh, dtype, lens, ctx):
    """Only requests whose keys are cut need room, each as much as alone: a long context beside prompts or short rows
    costs its own records (up to twice as much, or 16 MB, where one stride for all is simpler), not a share for
    every row of the step."""
    a = _attn(n_heads=heads, n_kv_heads=kv_heads, head_dim=dh, dtype=dtype)
    alone = sum(_ws(a, [m], [c]) for m, c in set(zip(lens, ctx)) for _ in range(list(zip(lens, ctx)).count((m, c))))
    both = _ws(a, lens, ctx)
    assert 0 < both <= 2 * alone + (16 << 20) + 1024 + 64 * (len(lens) + 1)
    rows = sum(lens) * heads * dh * (2 if dtype == B.VFM_BF16 else 4)
    assert both <= rows + 2 * alone + (16 << 20)


def test_windowed_layer_workspace_beside_a_long_context():
    """A prompt of 8191 rows and one row at 4000 in the layer: no more than the layer over the whole cache takes."""
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    cfg = R.cfg_for(wl.WORKLOADS[5])
    cfg.attn = B.VFM_ATTN_MIXED
    host, b = _batch(lens=[8191, 1], ctx=[0, 4000], tasks=[0, 0])
    assert B.vfm_workspace_size_windowed(cfg, b, None, 0, 0) <= B.vfm_workspace_size(cfg, b) + (16 << 20)


@pytest.mark.parametrize("heads,kv_heads,dtype,lens,ctx", [
    (64, 1, B.VFM_F32, [70000, 1], [0, 100000]), (64, 1, B.VFM_BF16, [140000, 1], [0, 200000]),
    (16, 1, B.VFM_BF16, [1] * 70000, [20] * 69999 + [400000]), (32, 32, B.VFM_BF16, [1] * 300000 + [64], [20] * 300001)])
def test_valid_steps_are_not_refused_for_empty_blocks(heads, kv_heads, dtype, lens, ctx):
    """A launch holds 2^24 blocks; blocks that a long context's chunks or a prompt would add to the others do not count."""
    a = _attn(n_heads=heads, n_kv_heads=kv_heads, head_dim=64, dtype=dtype)
    assert _ws(a, lens, ctx) > 0


@pytest.mark.parametrize("bad", [(1 << 32) + 5, 1 << 31, 1 << 33, -(1 << 32) + 7, 5.5])
def test_numbers_past_32_bits_are_refused(bad):
    """A ctypes int32 keeps the low bits of what it is given: 2^32 + 5 would be a window of 5."""
    for name in ("n_heads", "n_kv_heads", "head_dim", "window", "n_sink"):
        with pytest.raises((ValueError, TypeError)):
            _attn(**{name: bad})
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    cfg = R.cfg_for(wl.WORKLOADS[5])
    cfg.attn = B.VFM_ATTN_MIXED
    host, b = _batch()
    for window, n_sink in ((bad, 4), (16, bad)):
        with pytest.raises((ValueError, TypeError)):
            B.vfm_workspace_size_windowed(cfg, b, None, window, n_sink)
        with pytest.raises((ValueError, TypeError)):
            B.vfm_layer_forward_windowed(cfg, None, None, b, None, None, window, n_sink, None, stream=1)
    assert B.make_attn(B.VFM_BF16, np.int64(H), KH, DH, window=np.int32(7)).window == 7


def test_batches_larger_than_a_launch_are_refused():
    """A launch holds 2^32 - 1 threads: steps of 2^24 rows and more (the append's block of 256 threads each) and
    draws of 2^22 requests from heads of more than 1024 outputs (1024 threads each) are refused before anything runs."""
    n = 1 << 24
    host = B.vfm_plan(np.zeros(1, np.int32), np.array([n]), 1, ctx_len=np.array([0]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    kv = _kv(np.zeros((1, n // 1024)), page=1024, n_pages=1)
    assert _append(batch=(host, b), kv=kv) == B.VFM_ERR_UNSUPPORTED
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    cfg = R.cfg_for(wl.WORKLOADS[5])
    cfg.attn = B.VFM_ATTN_CAUSAL
    W = B.vfm_layer_weights(*[PTR] * len(B.vfm_layer_weights._fields_))
    assert B.lib().vfm_layer_forward_windowed(C.byref(cfg), C.byref(W), None, C.byref(b), PTR, C.byref(kv[1]), 16, 0, None,
                                              0, 1) == B.VFM_ERR_UNSUPPORTED
    del host, b
    n = 1 << 22
    tasks = np.zeros(n, np.int32)
    tasks[-1] = 1
    host = B.vfm_plan(tasks, np.ones(n, np.int32), 2, n_out=np.array([2, 1025]))
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, host.size)
    s = B.vfm_sampling(None, None, None, None)
    assert B.lib().vfm_sample_tokens(C.byref(b), PTR, C.byref(s), PTR, PTR, None, 1) == B.VFM_ERR_UNSUPPORTED


@pytest.mark.parametrize("m,G,KH", [(1 << 30, 64, 1), (1 << 30, 64, 16), (1 << 30, 1, 64), (1 << 26, 64, 16),
                                    ((1 << 30) - 1, 7, 100)])
@pytest.mark.parametrize("dtype", [B.VFM_F32, B.VFM_BF16])
def test_requests_of_any_length_have_a_plan(m, G, KH, dtype):
    """Rows times heads past 2^32 are refused, or need no workspace, without a fault of the host.  (Of the plan only the
    header and the arrays per request are read, so the arrays per row need not exist.)"""
    host = np.zeros(64, np.int32)
    host[:3] = 1, 1, m
    host[B.VFM_PLAN_HEADER + 3] = m                              # cu_seqlens[1], behind order[1] and task[1]
    b = B.vfm_batch(host.ctypes.data_as(C.POINTER(C.c_int32)), PTR, 1 << 34)
    n = C.c_size_t()
    st = B.lib().vfm_attention_workspace(C.byref(_attn(dtype=dtype, n_heads=G * KH, n_kv_heads=KH)), C.byref(b), C.byref(n))
    assert (st, n.value) in ((B.VFM_OK, 0), (B.VFM_ERR_UNSUPPORTED, 0))


@pytest.mark.parametrize("window,n_sink,seen", [(20, 0, (5, 6)), (1, 0, (6,)), (16, 0, (5, 6)), (17, 1, (0, 5, 6)),
                                                (5, 17, (0, 1, 6)), (5, 100, range(7)), (0, 0, range(7))])
def test_pages_that_no_row_sees_are_not_looked_at(window, n_sink, seen):
    """One row at position 100 (pages of 16: 0 .. 6) of a windowed layer without a workspace, so that no call gets to a
    launch: a bad id in a seen page is refused as such, one in any other page is not what the call is refused for."""
    from paper_2606_09643_amd import runner as R
    from paper_2606_09643_amd import workloads as wl
    cfg = R.cfg_for(wl.WORKLOADS[5])
    cfg.attn = B.VFM_ATTN_MIXED
    W = B.vfm_layer_weights(*[PTR] * len(B.vfm_layer_weights._fields_))
    host, b = _batch(lens=(1,), ctx=(100,), tasks=(0,))

    def status(t):
        t, k = _kv(t)
        return B.lib().vfm_layer_forward_windowed(C.byref(cfg), C.byref(W), None, C.byref(b), PTR, C.byref(k), window, n_sink,
                                                  None, 0, None)
    good = status(np.arange(8).reshape(1, 8))
    assert good in (B.VFM_ERR_WORKSPACE, B.VFM_ERR_HIP)
    for j in range(8):
        for bad in (-1, 50):
            t = np.arange(8).reshape(1, 8).copy()
            t[0, j] = bad
            assert status(t) == (B.VFM_ERR_SHAPE if j in seen else good), (j, bad)
