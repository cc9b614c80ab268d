"""Prompt attention with capped scores, distance bias and interval masks against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, slopes_of

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
P_WEIGHT = {"bf16": 2.0 ** -8, "f32": 0.0}      # weights are rounded to bf16 once on the tensor cores


def prompts(lens, hq, hkv, d, dtype, seed, qscale=1.0, wide=False):
    gen = torch.Generator().manual_seed(seed)
    T = int(sum(lens))
    if wide:
        row = torch.randn((T, (hq + 2 * hkv) * d + 8), generator=gen).to(DT[dtype])
        q, k, v = row[:, :hq * d].view(T, hq, d), row[:, hq * d:(hq + hkv) * d].view(T, hkv, d), row[:, (hq + hkv) * d:(hq + 2 * hkv) * d].view(T, hkv, d)
    else:
        q, k, v = (torch.randn((T, h, d), generator=gen).to(DT[dtype]) for h in (hq, hkv, hkv))
    q.mul_(qscale)
    return q, k, v, torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))


def documents(lens, seed, longest=60):
    rng = np.random.default_rng(seed)
    out = []
    for n in lens:
        cuts = np.concatenate([[0], np.cumsum(rng.integers(1, longest, n + 1))])
        out.append(cuts[np.searchsorted(cuts, np.arange(n), side="right") - 1])
    return torch.from_numpy(np.concatenate(out + [np.zeros(0)]).astype(np.int32))


def run(q, k, v, ip, d, cap=0.0, window=0, slopes=None, prefix=None, doc=None, out_dtype=torch.float32, scale=None, stream=None):
    B, (T, hq), hkv = len(ip) - 1, q.shape[:2], k.shape[1]
    shape = spd.make_shape(B, hq, hkv, d, q.dtype, scale or d ** -0.5)
    ws = spd.alloc_workspace(shape)
    row = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda").copy_(q)
    kk = torch.empty_strided(k.shape, k.stride(), dtype=q.dtype, device="cuda").copy_(k)
    vv = torch.empty_strided(v.shape, v.stride(), dtype=q.dtype, device="cuda").copy_(v)
    out = torch.full((T, hq, d), float("nan"), dtype=out_dtype, device="cuda")
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    spd.spd_prefill_attn_scored(shape, spd.make_score(cap, window, cu(slopes)), row, kk, vv, ip.cuda(), out, ws, prefix_lens=cu(prefix),
                                doc_start=cu(doc), stream=stream)
    return out, spd.spd_query_device_status(ws, stream)


LENS = [1, 63, 64, 65, 0, 130, 300]
OPTIONS = [dict(), dict(cap=20.0), dict(cap=3.0), dict(alibi=True), dict(window=1), dict(window=70), dict(window=7, alibi=True, cap=10.0), dict(prefix=True),
           dict(docs=True), dict(docs=True, window=20, alibi=True), dict(prefix=True, window=40, alibi=True), dict(prefix=True, docs=True, cap=30.0)]


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 4, 2), ("bf16", 128, 3, 3), ("bf16", 64, 8, 1), ("f32", 64, 2, 2), ("f32", 128, 4, 1)])
@pytest.mark.parametrize("opt", OPTIONS, ids=lambda o: "_".join(f"{k}{v}" for k, v in o.items()) or "plain")
def test_options(dtype, d, hq, hkv, opt):
    q, k, v, ip = prompts(LENS, hq, hkv, d, dtype, seed=len(opt) + d, qscale=3.0 if "cap" in opt else 1.0)
    sl = slopes_of(hq) if opt.get("alibi") else None
    prefix = torch.tensor([1, 70, 64, 10, 3, -4, 200], dtype=torch.int32) if opt.get("prefix") else None
    doc = documents(LENS, 3) if opt.get("docs") else None
    want, tol = ref.prefill(q, k, v, LENS, d ** -0.5, opt.get("cap", 0.0), opt.get("window", 0), sl,
                            None if prefix is None else prefix.clamp(min=0), doc, P_WEIGHT[dtype])
    for out_dtype in (torch.float32, torch.bfloat16):
        out, status = run(q, k, v, ip, d, opt.get("cap", 0.0), opt.get("window", 0), sl, prefix, doc, out_dtype)
        assert status == (spd.SPD_OK, -1)
        close(out, want, tol, opt)


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 2, 1), ("bf16", 128, 1, 1), ("bf16", 64, 2, 2), ("f32", 128, 1, 1)])
@pytest.mark.parametrize("opt", [dict(cap=40.0), dict(window=333, alibi=True), dict(prefix=True), dict(docs=True, cap=15.0)], ids=str)
def test_long_prompts(dtype, d, hq, hkv, opt):
    """Prompts of many blocks; a sample of the rows, block edges among them."""
    lens = [2100, 1025]
    q, k, v, ip = prompts(lens, hq, hkv, d, dtype, seed=77, qscale=3.0 if "cap" in opt else 1.0, wide=True)
    sl = slopes_of(hq) if opt.get("alibi") else None
    prefix = torch.tensor([1500, 1025], dtype=torch.int32) if opt.get("prefix") else None
    doc = documents(lens, 5, longest=900) if opt.get("docs") else None
    T = sum(lens)
    rows = set(range(0, T, 61)) | {e + x for e in (0, 128, 256, 1024, 1500, 2048, 2100, 2228, 3124) for x in (-1, 0, 1) if 0 <= e + x < T}
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, opt.get("cap", 0.0), opt.get("window", 0), sl, prefix, doc, P_WEIGHT[dtype], rows)
    out, status = run(q, k, v, ip, d, opt.get("cap", 0.0), opt.get("window", 0), sl, prefix, doc)
    assert status == (spd.SPD_OK, -1) and bool(torch.isfinite(out).all())
    r = sorted(rows)
    close(out[r], want[r], tol[r], opt)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_rows_that_see_nothing_give_zeros(dtype, d):
    """doc_start above the row (padding): the row is 0, its neighbours are not touched; a whole prompt of padding too."""
    lens, hq, hkv = [200, 300, 40], 2, 1
    q, k, v, ip = prompts(lens, hq, hkv, d, dtype, seed=4)
    doc = torch.zeros(540, dtype=torch.int32)
    doc[100:130] = 1 << 30
    doc[200:500] = 301
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, doc=doc, weight=P_WEIGHT[dtype])
    out, status = run(q, k, v, ip, d, doc=doc)
    assert status == (spd.SPD_OK, -1)
    assert bool((out[100:130] == 0).all()) and bool((out[200:500] == 0).all())
    close(out, want, tol, "padding")


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 2, 1), ("bf16", 128, 1, 1), ("bf16", 64, 2, 2), ("f32", 64, 1, 1)])
@pytest.mark.parametrize("opt", [dict(), dict(window=50), dict(docs=True)], ids=str)
def test_hidden_keys_may_hold_anything(dtype, d, hq, hkv, opt):
    """NaN and infinities in rows of k and v: rows that do not see them are as without them; rows that do are not finite."""
    lens = [150, 70, 290]
    q, k, v, ip = prompts(lens, hq, hkv, d, dtype, seed=14)
    doc = documents(lens, 8) if opt.get("docs") else None
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, window=opt.get("window", 0), doc=doc, weight=P_WEIGHT[dtype])
    spoiled = {60: float("nan"), 149: float("inf"), 219: float("nan"), 150 + 70 + 200: float("inf")}
    for r, x in spoiled.items():
        v[r], k[r] = x, float("nan")
    clean = torch.ones(sum(lens), dtype=torch.bool)
    t0 = 0
    for n in lens:
        lo, hi = ref.intervals(n, opt.get("window", 0), 0, None if doc is None else doc[t0:t0 + n])
        for r in spoiled:
            if t0 <= r < t0 + n:
                clean[t0:t0 + n] &= ~((lo <= r - t0) & (hi >= r - t0))
        t0 += n
    out, status = run(q, k, v, ip, d, window=opt.get("window", 0), doc=doc)
    assert status == (spd.SPD_OK, -1)
    close(out[clean], want[clean], tol[clean], opt)
    assert not bool(torch.isfinite(out[~clean]).any(dim=-1).any())


def test_large_scores_and_small_scales():
    lens = [140, 33]
    q, k, v, ip = prompts(lens, 2, 1, 128, "bf16", seed=15, qscale=8.0)
    want, tol = ref.prefill(q, k, v, lens, 1.0, cap=1.0, weight=2.0 ** -8)          # scores of several hundred, capped at 1
    out, _ = run(q, k, v, ip, 128, cap=1.0, scale=1.0)
    close(out, want, tol, "deep in the cap")
    want, tol = ref.prefill(q, k, v, lens, 1.0, weight=2.0 ** -8)                    # one key takes nearly all
    out, _ = run(q, k, v, ip, 128, scale=1.0)
    close(out, want, tol, "peaked")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_inconsistent_offsets_are_contained(dtype, d):
    lens = [100, 50, 80]
    q, k, v, ip = prompts(lens, 2, 1, d, dtype, seed=16)
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, weight=P_WEIGHT[dtype])
    for bad, first in ((torch.tensor([0, 100, 90, 230]), 1), (torch.tensor([0, 100, 5000, 230]), 1), (torch.tensor([0, 100, 150, 229]), 2)):
        out, status = run(q, k, v, bad.int(), d)
        assert status == (4, first)
        close(out[:100], want[:100], tol[:100], "users in front")
        if first == 1:
            assert bool(torch.isnan(out[100:]).all())


def test_captured_and_replayed():
    lens, hq, hkv, d = [300, 129], 4, 2, 128
    q, k, v, ip = prompts(lens, hq, hkv, d, "bf16", seed=17)
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, window=90, weight=2.0 ** -8)
    shape = spd.make_shape(2, hq, hkv, d, torch.bfloat16, d ** -0.5)
    ws, out, st = spd.alloc_workspace(shape), torch.empty((429, hq, d), device="cuda"), torch.cuda.Stream()
    a = [t.cuda() for t in (q, k, v, ip)]
    score = spd.make_score(window=90)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        spd.spd_prefill_attn_scored(shape, score, *a, out, ws, stream=st)
    for _ in range(2):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        close(out, want, tol, "replay")
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
