"""Scored decode calls (capped scores, distance bias, sliding window over both partitions) against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["short", "persistent"])
def kernel(request):
    """Small calls go to the cluster kernel; asking for a cut of its own (here: at least 3 tiles per share) keeps the persistent one."""
    spd.spd_set_split(3 if request.param == "persistent" else 0, False)
    yield request.param
    spd.spd_set_split(0, False)


def slopes_of(hq):
    return (2.0 ** (-8.0 * torch.arange(1, hq + 1, dtype=torch.float64) / hq)).float()


def workload(lin, lout, hq, hkv, d, dtype, seed, qscale=1.0):
    w = wl.make_workload(dict(batch=len(lin), hq=hq, hkv=hkv, d=d, dtype=dtype, lin=("const", 0), lout=("const", 0), seed=seed),
                         lengths=(np.array(lin), np.array(lout)), slack=True)
    w.q = (w.q.float() * qscale).to(w.dtype)
    return w


def setup(w, cap, window, alibi):
    g = w.to("cuda")
    shape = spd.make_shape(w.batch, w.num_q_heads, w.num_kv_heads, w.head_dim, w.dtype, w.sm_scale)
    sl = slopes_of(w.num_q_heads) if alibi else None
    return g, shape, spd.make_score(cap, window, None if sl is None else sl.cuda()), sl, spd.alloc_workspace(shape)


def close(got, want, tol, what):
    err = (got.cpu().double() - want).abs()
    lim = tol[..., None] + (ref.half_step(got.dtype) * want.abs() if got.dtype != torch.float32 else 0)
    assert bool((err <= lim).all()), (what, float(err.max()), float((err - lim).max()))


LENGTHS = ([0, 40, 0, 17, 16, 0, 300, 1, 65], [0, 0, 25, 0, 16, 1, 33, 1, 0])
SHAPES = [("bf16", 128, 8, 1), ("bf16", 128, 4, 4), ("bf16", 64, 4, 2), ("bf16", 64, 16, 1), ("f32", 64, 8, 8), ("f32", 128, 8, 2), ("f32", 64, 8, 1),
          ("f32", 128, 2, 1)]


@pytest.mark.parametrize("dtype,d,hq,hkv", SHAPES)
@pytest.mark.parametrize("cap,window,alibi", [(0.0, 0, False), (20.0, 0, False), (0.0, 0, True), (0.0, 1, False), (0.0, 17, True), (5.0, 33, True),
                                              (50.0, 300, False), (0.0, 100000, False)])
def test_fused_and_halves(kernel, dtype, d, hq, hkv, cap, window, alibi):
    w = workload(*LENGTHS, hq, hkv, d, dtype, seed=d + hq, qscale=3.0)
    g, shape, score, sl, ws = setup(w, cap, window, alibi)
    want, _, _, _, tol = ref.decode(w, cap, window, sl)
    for out_dtype in (torch.float32, torch.bfloat16):
        out = torch.full((w.batch, hq, d), float("nan"), dtype=out_dtype, device="cuda")
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        close(out, want, tol, "fused")
    assert bool((out[0] == 0).all())
    # the two halves: the private partial is the 64-bit one, and merged by the service call it gives the same output
    part = spd.alloc_partial(shape)
    spd.spd_partial_attn_scored(shape, score, g.q, g.priv, g.pub.seq_lens, part, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    wa, _, wm, wl_, wt = ref.decode(w, cap, window, sl, parts=(True, False))
    o, m, l = (t.cpu().double() for t in part)
    empty = torch.isinf(wm)
    assert bool((m[empty] == -float("inf")).all()) and bool((l[empty] == 0).all()) and bool((o[empty] == 0).all())
    full = ~empty
    a = o[full] / l[full][:, None]
    assert bool(((a - wa[full]).abs() <= wt[full][:, None]).all())
    lse = m[full] + l[full].log()
    e = wt[full] + 1e-5                 # wt bounds twice the weights' relative error times max|v| (above 1/2 everywhere here)
    assert bool(((lse - (wm[full] + wl_[full].log())).abs() <= 2 * e).all())
    out = torch.full((w.batch, hq, d), float("nan"), dtype=torch.float32, device="cuda")
    spd.spd_service_attn_merge_scored(shape, score, g.q, g.pub, g.priv.seq_lens, part, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, 2 * tol, "merged halves")


def test_plain_options_give_the_plain_call():
    w = workload([700, 33, 2000], [5, 90, 17], 8, 2, 128, "bf16", seed=1)
    g, shape, score, _, ws = setup(w, 0.0, 0, False)
    a, b = (torch.empty((3, 8, 128), device="cuda") for _ in range(2))
    try:
        spd.spd_set_split(0, True)
        spd.spd_decode_step(shape, g.q, g.priv, g.pub, a, ws)
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, b, ws)
    finally:
        spd.spd_set_split(0, False)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 16, 17, 100, 257])
def test_what_lies_in_front_of_the_window_is_never_used(dtype, window):
    """Pages in front of the window carry indices outside the pool, rows in front of it NaN and infinities."""
    lin, lout = [500, 64, 33, 0, 300, 17], [40, 0, 15, 400, 1, 16]
    w = workload(lin, lout, 8, 4, 128, dtype, seed=window)
    want, _, _, _, tol = ref.decode(w, 0.0, window)
    for u in range(w.batch):
        n = lin[u] + lout[u]
        first = max(0, n - window)
        for part, base, m in ((w.priv, 0, lin[u]), (w.pub, lin[u], lout[u])):
            lo = int(part.page_indptr[u])
            for t in range(m):
                if base + t < first:
                    pg = int(part.page_indices[lo + t // 16])
                    part.k_pool[pg, :, t % 16] = float("nan") if t % 2 else float("inf")
                    part.v_pool[pg, :, t % 16] = float("inf") if t % 2 else float("nan")
        for part, base, m in ((w.priv, 0, lin[u]), (w.pub, lin[u], lout[u])):
            lo = int(part.page_indptr[u])
            for pgi in range((m + 15) // 16):
                if base + min(m, 16 * pgi + 16) <= first:
                    part.page_indices[lo + pgi] = -1 if pgi % 2 else part.num_pages + 5
    g, shape, score, _, ws = setup(w, 0.0, window, False)
    for share in (0, 1, 3):               # 0: the cluster kernel
        try:
            spd.spd_set_split(share, False)
            out = torch.full((w.batch, 8, 128), float("nan"), device="cuda")
            spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
            assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        finally:
            spd.spd_set_split(0, False)
        close(out, want, tol, f"window {window} share {share}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_inside_the_window_is_not_hidden(kernel, dtype):
    w = workload([300, 40], [10, 40], 4, 2, 64, dtype, seed=31)
    want, _, _, _, tol = ref.decode(w, 0.0, 64)
    pg = int(w.priv.page_indices[int(w.priv.page_indptr[0]) + 290 // 16])
    w.priv.k_pool[pg, 0, 290 % 16] = float("nan")               # KV head 0 of user 0: query heads 0 and 1
    w.priv.v_pool[pg, 1, 290 % 16] = float("nan")
    g, shape, score, _, ws = setup(w, 0.0, 64, False)
    out = torch.zeros((2, 4, 64), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    assert not bool(torch.isfinite(out[0]).any())
    close(out[1], want[1], tol[1], "bystander")


@pytest.mark.parametrize("min_tiles", [1, 7, 1 << 30])
def test_any_cut_of_long_sequences(min_tiles):
    w = workload([3000, 1, 5000], [100, 700, 3], 8, 2, 128, "bf16", seed=21, qscale=2.0)
    g, shape, score, sl, ws = setup(w, 30.0, 2500, True)
    want, _, _, _, tol = ref.decode(w, 30.0, 2500, sl)
    out = torch.full((3, 8, 128), float("nan"), device="cuda")
    try:
        spd.spd_set_split(min_tiles, False)
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    finally:
        spd.spd_set_split(0, False)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, tol, "cut")


def test_stored_plan_belongs_to_its_window():
    w = workload([900, 50, 1700], [60, 300, 2], 8, 2, 128, "bf16", seed=22)
    g, shape, score, sl, ws = setup(w, 0.0, 500, True)
    want, _, _, _, tol = ref.decode(w, 0.0, 500, sl)
    out = torch.empty((3, 8, 128), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws, plan=spd.SPD_PLAN_STORE)
    for _ in range(3):
        out.fill_(float("nan"))
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws, plan=spd.SPD_PLAN_REUSE)
        close(out, want, tol, "reused plan")
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    other = spd.make_score(0.0, 499, sl.cuda())
    spd.spd_decode_step_scored(shape, other, g.q, g.priv, g.pub, out, ws, plan=spd.SPD_PLAN_REUSE)
    assert spd.spd_query_device_status(ws)[0] == 7


def test_bad_pages_and_lengths_are_contained(kernel):
    w = workload([200, 100, 90, 300], [20, 30, 5, 8], 8, 2, 128, "bf16", seed=23)
    want, _, _, _, tol = ref.decode(w, 0.0, 128)
    w.priv.page_indices[int(w.priv.page_indptr[0]) + 7] = w.priv.num_pages        # tokens 112 .. 127 of user 0: inside its window
    w.pub.seq_lens[2] = 10000
    g, shape, score, _, ws = setup(w, 0.0, 128, False)
    out = torch.full((4, 8, 128), float("nan"), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (4, 0)
    assert bool((out[[0, 2]] == 0).all())
    close(out[[1, 3]], want[[1, 3]], tol[[1, 3]], "bystanders")
    # a negative length of the other partition
    part = spd.alloc_partial(shape)
    peers = torch.tensor([20, 30, -1, 8], dtype=torch.int32, device="cuda")
    spd.spd_partial_attn_scored(shape, score, g.q, g.priv, peers, part, ws)
    assert spd.spd_query_device_status(ws) == (4, 0)
    assert bool((part[1][2] == -float("inf")).all()) and bool((part[2][2] == 0).all())


def test_captured_and_replayed_on_another_stream(kernel):
    w = workload([700, 80, 0], [40, 9, 33], 8, 2, 128, "bf16", seed=24)
    g, shape, score, sl, ws = setup(w, 10.0, 200, True)
    want, _, _, _, tol = ref.decode(w, 10.0, 200, sl)
    out, st = torch.empty((3, 8, 128), device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws, stream=st)
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws, stream=st)
    for _ in range(3):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        close(out, want, tol, "replay")
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 1), ("bf16", 64, 4, 4), ("f32", 64, 8, 2), ("f32", 128, 16, 1)])
def test_clusters_of_every_size(dtype, d, hq, hkv):
    """One user to so many that a sequence gets a single CTA; users with nothing cached, with one token, and with the longest sequence."""
    for B in (1, 2, 5, 18, 37):
        lin = [(37 * u * u + 900 * (u == 0)) % 1200 for u in range(B)]
        lout = [(11 * u) % 40 for u in range(B)]
        w = workload(lin, lout, hq, hkv, d, dtype, seed=B)
        g, shape, score, sl, ws = setup(w, 15.0, 0, True)
        want, _, _, _, tol = ref.decode(w, 15.0, 0, sl)
        out = torch.full((B, hq, d), float("nan"), device="cuda")
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        close(out, want, tol, f"{B} users")


def test_two_streams_side_by_side():
    """Two batches with a workspace each, called in turn on two streams; every result is right."""
    jobs = []
    for s in range(2):
        w = workload([300 + 50 * s, 40, 90], [5, 60, 0], 8, 2, 128, "bf16", seed=40 + s)
        g, shape, score, sl, ws = setup(w, 0.0, 128, True)
        want, _, _, _, tol = ref.decode(w, 0.0, 128, sl)
        jobs.append((g, shape, score, ws, torch.empty((3, 8, 128), device="cuda"), torch.cuda.Stream(), want, tol))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, shape, score, ws, out, st, _, _ in jobs:
            spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws, stream=st)
    torch.cuda.synchronize()
    for _, _, _, ws, out, st, want, tol in jobs:
        close(out, want, tol, "side by side")
        assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)
