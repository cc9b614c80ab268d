"""Attention behind a launch that appends: the lengths it grows as its last act are the ones that the next call reads, whichever
workspace either of them uses.  What the calls ask of the stream is read off a captured graph's edges; nothing in it is run."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, setup, workload

pytestmark = pytest.mark.gpu


class EdgeData(C.Structure):
    _fields_ = [("from_port", C.c_ubyte), ("to_port", C.c_ubyte), ("type", C.c_ubyte), ("reserved", C.c_ubyte * 5)]


def edges_of(calls, stream, kernels=None):
    """Captures the calls on one stream (not run): for each of their kernels but the first, whether it may start before the one in front
    has ended.  kernels: how many there are, if not one per call."""
    L = C.CDLL("libcuda.so.1")
    st, graph, n = C.c_void_p(stream.cuda_stream), C.c_void_p(), C.c_size_t()
    assert L.cuStreamBeginCapture_v2(st, 1) == 0                     # capture mode: this thread's calls only
    try:
        for call in calls:
            call()
    finally:
        assert L.cuStreamEndCapture(st, C.byref(graph)) == 0
    assert L.cuGraphGetNodes(graph, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert L.cuGraphGetNodes(graph, nodes, C.byref(n)) == 0
    assert L.cuGraphGetEdges_v2(graph, None, None, None, C.byref(n)) == 0
    frm, to, data = (C.c_void_p * n.value)(), (C.c_void_p * n.value)(), (EdgeData * n.value)()
    assert L.cuGraphGetEdges_v2(graph, frm, to, data, C.byref(n)) == 0
    after = {a: (b, e.type) for a, b, e in zip(frm, to, data)}
    at, out = (set(nodes) - set(to)).pop(), []
    while at in after:
        at, kind = after[at]
        assert kind in (0, 1)
        out.append(kind == 1)                                       # CU_GRAPH_DEPENDENCY_TYPE_PROGRAMMATIC
    assert L.cuGraphDestroy(graph) == 0
    assert len(out) == (kernels or len(calls)) - 1
    return out


@pytest.fixture
def overlap():
    spd.spd_set_programmatic_launch(True)
    yield


@pytest.fixture
def job():
    w = workload([300, 4, 90], [15, 3, 31], 8, 2, 128, "bf16", 12)
    g, shape, score, _, ws = setup(w, 20.0, 64, False)
    k_new, v_new = (torch.randn((3, 2, 128), device="cuda").bfloat16() for _ in range(2))
    out, part = torch.empty((3, 8, 128), device="cuda"), spd.alloc_partial(shape)
    spd.spd_partial_attn(shape, g.q, g.priv, part, ws)
    torch.cuda.synchronize()
    other, st = spd.alloc_workspace(shape), torch.cuda.Stream()
    step = dict(q=g.q, k_new=k_new, v_new=v_new, priv=g.priv, pub=g.pub, out=out)
    appends = {
        "step": lambda x, s=st: spd.spd_decode_step_append(shape, g.q, k_new, v_new, g.priv, g.pub, out, x, stream=s),
        "service": lambda x, s=st: spd.spd_service_attn_merge_append(shape, g.q, k_new, v_new, g.pub, part, out, x, stream=s),
    }
    reads = {
        "plain": lambda x, s=st: spd.spd_decode_step(shape, g.q, g.priv, g.pub, out, x, stream=s),
        "service": lambda x, s=st: spd.spd_service_attn_merge(shape, g.q, g.pub, part, out, x, stream=s),
        "scored": lambda x, s=st: spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, x, stream=s),
        "scored stored": lambda x, s=st: spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, x, plan=spd.SPD_PLAN_STORE, stream=s),
        "scored half": lambda x, s=st: spd.spd_partial_attn_scored(shape, score, g.q, g.priv, g.pub.seq_lens, part, x, stream=s),
    }
    return shape, ws, other, st, appends, reads, step


@pytest.mark.parametrize("read", ["plain", "service", "scored", "scored stored", "scored half"])
@pytest.mark.parametrize("append", ["step", "service"])
@pytest.mark.parametrize("same", [True, False], ids=["one workspace", "two workspaces"])
def test_a_call_behind_an_append_waits_for_its_end(overlap, job, append, read, same):
    shape, ws, other, st, appends, reads, _ = job
    wa, wr = ws, ws if same else other
    got = edges_of([lambda: appends[append](wa), lambda: reads[read](wr), lambda: reads[read](wr)], st)
    assert got == [False, True]            # the second call has nothing to wait for but the first


def test_an_append_on_one_stream_says_nothing_about_another(overlap, job):
    shape, ws, other, st, appends, reads, _ = job
    st2 = torch.cuda.Stream()
    edges_of([lambda: reads["plain"](ws), lambda: appends["step"](ws)], st)
    assert edges_of([lambda: reads["scored"](other, st2)] * 3, st2) == [True, True]
    assert edges_of([lambda: reads["scored"](other)] * 3, st) == [True, True]


def test_the_layers_of_a_token_step_still_overlap(overlap, job):
    shape, ws, other, st, appends, reads, step = job
    lens = [step["pub"].seq_lens.clone() for _ in range(3)]
    p = step["pub"]
    layers = [(step["q"], step["k_new"], step["v_new"], step["priv"], wl.PagedKV(p.k_pool, p.v_pool, p.page_indptr, p.page_indices, x), step["out"])
              for x in lens]
    got = edges_of([lambda: spd.spd_token_step(shape, layers, ws, same_lengths=True, stream=st), lambda: reads["scored"](other),
                    lambda: reads["plain"](ws)], st, kernels=5)
    assert got == [True, True, False, True]


def test_results_behind_appends_with_workspaces_of_their_own():
    """Ten tokens: append with one workspace, scored and plain step with two others, all on one stream without a wait on the host."""
    w = workload([300, 4, 90], [15, 0, 31], 8, 2, 128, "bf16", 12)
    g, shape, score, _, ws = setup(w, 20.0, 64, False)
    wss = [ws, spd.alloc_workspace(shape), spd.alloc_workspace(shape)]
    gen = torch.Generator().manual_seed(2)
    st = torch.cuda.Stream()
    k_new, v_new = (torch.randn((10, 3, 2, 128), generator=gen).bfloat16().cuda() for _ in range(2))
    big = wl.make_paged_kv(np.array([64, 64, 64]), 2, 128, torch.bfloat16, np.random.default_rng(3), gen, "cpu", poison=False)
    n0 = torch.tensor([15, 0, 31], dtype=torch.int32)
    big.seq_lens.copy_(n0)
    pub = big.to("cuda")
    outs = torch.empty((10, 2, 3, 8, 128), device="cuda")
    other = torch.empty_like(outs[0, 0])
    torch.cuda.synchronize()
    for s in range(10):
        spd.spd_decode_step_append(shape, g.q, k_new[s], v_new[s], g.priv, pub, other, wss[0], stream=st)
        if s % 2:
            spd.spd_decode_step(shape, g.q, g.priv, pub, outs[s, 1], wss[2], stream=st)
            spd.spd_decode_step_scored(shape, score, g.q, g.priv, pub, outs[s, 0], wss[1], stream=st)
        else:
            spd.spd_decode_step_scored(shape, score, g.q, g.priv, pub, outs[s, 0], wss[1], stream=st)
            spd.spd_decode_step(shape, g.q, g.priv, pub, outs[s, 1], wss[2], stream=st)
    for x in wss:
        assert spd.spd_query_device_status(x, st) == (spd.SPD_OK, -1)
    grown = pub.to("cpu")
    for s in range(10):
        grown.seq_lens.copy_(n0 + s + 1)
        x = wl.Workload("grown", 3, 8, 2, 128, 16, torch.bfloat16, w.sm_scale, w.q, w.priv, grown)
        for i, (cap, window) in enumerate(((20.0, 64), (0.0, 0))):
            want, _, _, _, tol = ref.decode(x, cap, window, None)
            close(outs[s, i], want, tol, (s, i))
