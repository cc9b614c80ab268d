"""Scored calls at drawn shapes, at the ends of their ranges, and side by side."""
import random

import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, setup, slopes_of, workload
from tests.test_gpu_prefill_scored import DT, P_WEIGHT, documents, prompts, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(24))
def test_prompts_of_drawn_shapes(seed):
    r = random.Random(seed)
    dtype, d, hkv = r.choice(["bf16", "bf16", "f32"]), r.choice([64, 128]), r.choice([1, 2, 3])
    hq = hkv * r.choice([1, 2, 4, 8, 16])
    lens = [r.choice([0, 1, 2, 79, 80, 81, 127, 128, 129, r.randrange(1, 400)]) for _ in range(r.choice([1, 2, 7, 40]))]
    if sum(lens) == 0:
        lens[0] = 5
    cap, window = r.choice([0.0, 0.0, 2.0, 30.0, 90.0]), r.choice([0, 0, 1, 80, r.randrange(1, 300)])
    q, k, v, ip = prompts(lens, hq, hkv, d, dtype, seed, qscale=3.0 if cap else 1.0, wide=r.random() < 0.5)
    sl = slopes_of(hq) * r.choice([1.0, 4.0, -0.05]) if r.random() < 0.4 else None
    prefix = torch.tensor([r.randrange(-1, n + 2) for n in lens], dtype=torch.int32) if r.random() < 0.4 else None
    doc = documents(lens, seed, longest=r.choice([5, 90, 300])) if r.random() < 0.4 else None
    T = sum(lens)
    rows = set(r.sample(range(T), min(T, 60))) | {0, T - 1}
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5, cap, window, sl, None if prefix is None else prefix.clamp(min=0), doc, P_WEIGHT[dtype], rows)
    out, status = run(q, k, v, ip, d, cap, window, sl, prefix, doc, r.choice([torch.float32, torch.bfloat16]))
    assert status == (spd.SPD_OK, -1) and bool(torch.isfinite(out.float()).all())
    at = sorted(rows)
    close(out[at], want[at], tol[at], (seed, lens))


@pytest.mark.parametrize("seed", range(16))
def test_decode_of_drawn_shapes(seed):
    r = random.Random(100 + seed)
    dtype, d, hkv = r.choice(["bf16", "bf16", "f32"]), r.choice([64, 128]), r.choice([1, 2, 3])
    hq = hkv * r.choice([1, 2, 4, 8, 16])
    B = r.choice([1, 3, 20])
    most = r.choice([5, 40, 700, 3000])
    lin, lout = [r.randrange(0, most) for _ in range(B)], [r.randrange(0, 50) for _ in range(B)]
    cap, window, alibi = r.choice([0.0, 4.0, 70.0]), r.choice([0, 0, 1, 33, r.randrange(1, 2000)]), r.random() < 0.5
    w = workload(lin, lout, hq, hkv, d, dtype, seed, qscale=2.0)
    g, shape, score, sl, ws = setup(w, cap, window, alibi)
    want, _, _, _, tol = ref.decode(w, cap, window, sl)
    out = torch.full((B, hq, d), float("nan"), device="cuda")
    for knob in (0, 2):
        try:
            spd.spd_set_split(knob, False)
            spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
        finally:
            spd.spd_set_split(0, False)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        close(out, want, tol, (seed, knob))


def test_no_prompt_tokens_and_one_prompt_token():
    shape = spd.make_shape(2, 4, 2, 128, torch.bfloat16, 0.1)
    ws, ip = spd.alloc_workspace(shape), torch.zeros(3, dtype=torch.int32, device="cuda")
    e = lambda h: torch.empty((0, h, 128), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    spd.spd_prefill_attn_scored(shape, spd.make_score(), e(4), e(2), e(2), ip, e(4), ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    q, k, v, ip = prompts([0, 1], 4, 2, 128, "bf16", 3)
    out, status = run(q, k, v, ip, 128)
    assert status == (spd.SPD_OK, -1)
    assert torch.equal(out.cpu(), v.float().repeat_interleave(2, dim=1))       # one key: its weight is exactly 1


def test_rows_behind_the_last_prompt_are_left_alone():
    q, k, v, ip = prompts([50, 70], 2, 1, 128, "bf16", 4)
    shape = spd.make_shape(2, 2, 1, 128, torch.bfloat16, 128 ** -0.5)
    ws = spd.alloc_workspace(shape)
    pad = torch.full((300, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = pad[:120]
    spd.spd_prefill_attn_scored(shape, spd.make_score(), q.cuda(), k.cuda(), v.cuda(), ip.cuda(), out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    assert bool((pad[120:] == 7.0).all()) and not bool((out == 7.0).all(dim=-1).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_beyond_32_bit_offsets(dtype):
    """Pages near the end of a pool of more than 4 GiB: appended to, then read."""
    B, hq, hkv, d = 2, 8, 8, 128
    es = 2 if dtype == "bf16" else 4
    pages = (9 << 29) // (hkv * 16 * d * es) + 8                       # 4.5 GiB each for K and V
    kp, vp = (torch.zeros((pages, hkv, 16, d), dtype=DT[dtype], device="cuda") for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    part = wl.PagedKV(kp, vp, i32(0, 2, 4), i32(pages - 1, 3, pages - 4, pages - 2), i32(0, 0))
    small = wl.PagedKV(kp[:1].clone(), vp[:1].clone(), i32(0, 1, 1), i32(0), i32(0, 0))
    gen = torch.Generator().manual_seed(1)
    lens = [20, 31]
    k, v = (torch.randn((51, hkv, d), generator=gen).to(DT[dtype]) for _ in range(2))
    q = torch.randn((B, hq, d), generator=gen).to(DT[dtype])
    shape = spd.make_shape(B, hq, hkv, d, DT[dtype], d ** -0.5)
    ws, score = spd.alloc_workspace(shape), spd.make_score(20.0)
    spd.spd_append_kv_rope(shape, None, None, k.cuda(), v.cuda(), part, ws, tok_indptr=i32(0, 20, 51))
    assert part.seq_lens.tolist() == lens
    assert torch.equal(kp[pages - 2, :, 14].cpu(), k[50]) and torch.equal(vp[pages - 1, :, 15].cpu(), v[15])
    out = torch.empty((B, hq, d), device="cuda")
    spd.spd_decode_step_scored(shape, score, q.cuda(), part, small, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    t0 = 0
    for u, n in enumerate(lens):
        for h in range(hq):
            want, _, _, _, S = ref.attend(q[u, h], k[t0:t0 + n, h], v[t0:t0 + n, h], torch.ones(n, dtype=torch.bool), d ** -0.5, 20.0)
            tol = ref.bound(float(v.abs().max()), d, S, n, 20.0, 0.0, 2.0 ** -16 if dtype == "bf16" else 0.0)
            assert float((out[u, h].cpu().double() - want).abs().max()) <= tol
        t0 += n


def test_two_prompt_calls_side_by_side():
    """Two batches on two streams, a workspace each, again and again: the work counters do not meet."""
    jobs = []
    for s in range(2):
        lens = [300 + 100 * s, 77, 513]
        q, k, v, ip = prompts(lens, 8, 2, 128, "bf16", 50 + s)
        rows = set(range(0, sum(lens), 97))
        want, tol = ref.prefill(q, k, v, lens, 128 ** -0.5, cap=25.0, window=200, weight=2.0 ** -8, rows=rows)
        shape = spd.make_shape(3, 8, 2, 128, torch.bfloat16, 128 ** -0.5)
        jobs.append(([t.cuda() for t in (q, k, v, ip)], shape, spd.alloc_workspace(shape), torch.empty_like(q, dtype=torch.float32, device="cuda"),
                     torch.cuda.Stream(), sorted(rows), want, tol))
    torch.cuda.synchronize()
    score = spd.make_score(25.0, 200)
    for _ in range(25):
        for a, shape, ws, out, st, _, _, _ in jobs:
            spd.spd_prefill_attn_scored(shape, score, *a, out, ws, stream=st)
    torch.cuda.synchronize()
    for _, _, ws, out, st, rows, want, tol in jobs:
        assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)
        close(out[rows], want[rows], tol[rows], "side by side")


def test_same_call_gives_the_same_bits():
    """Prompt attention hands its items out in whatever order the CTAs come; no result depends on it."""
    q, k, v, ip = prompts([700, 33, 260], 8, 4, 128, "bf16", 60)
    first, _ = run(q, k, v, ip, 128, cap=30.0, window=150, slopes=slopes_of(8))
    for _ in range(5):
        again, _ = run(q, k, v, ip, 128, cap=30.0, window=150, slopes=slopes_of(8))
        assert torch.equal(first, again)


def test_another_device_than_the_current_one_is_refused():
    q, k, v, ip = prompts([4], 2, 1, 64, "f32", 1)
    shape = spd.make_shape(1, 2, 1, 64, torch.float32, 0.1)
    ws = spd.alloc_workspace(shape)
    with pytest.raises(ValueError):
        spd.spd_prefill_attn_scored(shape, spd.make_score(), q, k, v, ip, q.clone(), ws)      # host tensors
    with pytest.raises(ValueError):
        spd.spd_prefill_attn_scored(shape, spd.make_score(), q.cuda().double(), k.cuda(), v.cuda(), ip.cuda(), q.cuda(), ws)
    with pytest.raises(ValueError):
        spd.spd_prefill_attn_scored(shape, spd.make_score(), q.cuda(), k.cuda(), v.cuda(), ip.cuda().long(), q.cuda(), ws)
    with pytest.raises(ValueError):
        spd.spd_prefill_attn_scored(shape, spd.make_score(), q.cuda(), k.cuda(), v.cuda(), ip, q.cuda(), ws)      # offsets on the host
    with pytest.raises(ValueError):
        spd.spd_prefill_attn_scored(shape, spd.make_score(), q.cuda(), k.cuda()[:1].expand(4, 1, 64), v.cuda(), ip.cuda(), q.cuda(), ws)
    for rows in (torch.zeros(320).cuda().as_strided((4, 2, 64), (64, 64, 1)), torch.zeros(4, 64, 2).cuda().transpose(1, 2)):      # overlapping, not packed
        with pytest.raises(ValueError):
            spd.spd_prefill_attn_scored(shape, spd.make_score(), rows, k.cuda(), v.cuda(), ip.cuda(), q.cuda(), ws)
    w = workload([5], [3], 2, 1, 64, "f32", 1)
    g, shape, score, _, ws = setup(w, 0.0, 0, False)
    out = torch.empty((1, 2, 64), device="cuda")
    for bad in (dict(q=w.q), dict(q=g.q.double()), dict(q=g.q[:, :1]), dict(priv=w.priv), dict(pub=w.pub), dict(out=out.cpu()), dict(out=out[:, :1])):
        a = dict(dict(q=g.q, priv=g.priv, pub=g.pub, out=out), **bad)
        with pytest.raises(ValueError):
            spd.spd_decode_step_scored(shape, score, a["q"], a["priv"], a["pub"], a["out"], ws)


@pytest.mark.parametrize("cap,scale", [(50.0, 1 / 16), (51.0, 64 ** -0.5), (100.0, 64 ** -0.5), (1000.0, 64 ** -0.5), (50.0, 1e-4), (0.01, 1.0), (1e-3, 3.0),
                                       (1e30, 0.1), (1e-30, 0.1)])
@pytest.mark.parametrize("alibi", [False, True])
def test_caps_over_their_range(cap, scale, alibi):
    """Every size of cap over scores from far below it to far above."""
    lens, hq, hkv, d = [170, 90], 4, 2, 64
    q, k, v, ip = prompts(lens, hq, hkv, d, "bf16", 70)
    q *= torch.logspace(-2, 1.5, q.shape[0])[torch.randperm(q.shape[0], generator=torch.Generator().manual_seed(1))][:, None, None].bfloat16()
    sl = slopes_of(hq) if alibi else None
    # Where the cap is far above the scores its error is 2.3e-6 = 2^-18.7 < 6 x 2^-21 of the greatest score (the polynomials'; the
    # other form only serves blocks in which some score reaches the cap) and not 2^-21 of the cap.
    top = scale * max(float((q[t0:t0 + n].double().flatten(0, 1) @ k[t0:t0 + n].double().flatten(0, 1).T).abs().max()) for t0, n in ((0, 170), (170, 90)))
    eff = min(cap, 6 * top)
    want, tol = ref.prefill(q, k, v, lens, scale, cap, 0, sl, weight=P_WEIGHT["bf16"], cap_error=eff)
    shape = spd.make_shape(2, hq, hkv, d, torch.bfloat16, scale)
    ws, out = spd.alloc_workspace(shape), torch.empty(q.shape, device="cuda")
    spd.spd_prefill_attn_scored(shape, spd.make_score(cap, 0, None if sl is None else sl.cuda()), q.cuda(), k.cuda(), v.cuda(), ip.cuda(), out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, tol, (cap, scale))
    # the same rows as generated tokens: the last token of each prompt over its keys
    w = workload(lens, [0, 0], hq, hkv, d, "bf16", 71, qscale=4.0)
    w.sm_scale = scale
    g, shape, score, sl, ws = setup(w, cap, 0, alibi)
    # the cubic is off by 2 / 15 / 16^4 = 2.1e-6 of the score, the full form by 2^-22 of the cap <= 16 scores: 8 x 2^-21 of the greatest
    top = scale * float(w.q.double().abs().sum(-1).max()) * 8.0            # |q.k| <= |q|_1 max|k|, and no k exceeds 8
    want, _, _, _, tol = ref.decode(w, cap, 0, sl, cap_error=min(cap, 8 * top))
    out = torch.empty((2, hq, d), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, tol, ("decode", cap, scale))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_short_and_long_calls_in_turns(dtype, d):
    """Calls of the cluster kernel between calls of the persistent one that store, derive and reuse their cut, back to back on one
    stream and workspace: whatever is still running when the next one starts, nobody reads what is being written."""
    w = workload([900, 3, 2500, 0, 64, 1200], [30, 0, 77, 5, 1, 400], 8, 4, d, dtype, 11)
    g, shape, _, _, ws = setup(w, 0.0, 0, False)
    plain, near = spd.make_score(), spd.make_score(30.0, 40)
    outs = {}
    for name, score, args in (("plain", plain, (0.0, 0)), ("near", near, (30.0, 40))):
        outs[name] = ref.decode(w, *args, None)
    turns = [("plain", spd.SPD_PLAN_STORE), ("near", spd.SPD_PLAN_PER_CALL), ("plain", spd.SPD_PLAN_STORE), ("plain", spd.SPD_PLAN_REUSE),
             ("near", spd.SPD_PLAN_STORE), ("plain", spd.SPD_PLAN_STORE), ("near", spd.SPD_PLAN_PER_CALL), ("near", spd.SPD_PLAN_PER_CALL)] * 8
    calls = [(kind, plan, torch.full((w.batch, 8, d), float("nan"), device="cuda")) for kind, plan in turns]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for kind, plan, out in calls:
        spd.spd_decode_step_scored(shape, plain if kind == "plain" else near, g.q, g.priv, g.pub, out, ws, plan=plan, stream=st)
    assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)
    for kind, _, out in calls:
        want, _, _, _, tol = outs[kind]
        close(out, want, tol, kind)


def test_scored_call_behind_an_appending_launch():
    """The lengths that an appending launch writes as its last act are the ones that the scored call behind it reads."""
    w = workload([300, 4, 90], [15, 0, 31], 8, 2, 128, "bf16", 12)
    g, shape, score, _, ws = setup(w, 20.0, 64, False)
    gen = torch.Generator().manual_seed(2)
    st = torch.cuda.Stream()
    k_new, v_new = (torch.randn((10, 3, 2, 128), generator=gen).bfloat16().cuda() for _ in range(2))
    big = wl.make_paged_kv(np.array([64, 64, 64]), 2, 128, torch.bfloat16, np.random.default_rng(3), gen, "cpu", poison=False)
    n0 = torch.tensor([15, 0, 31], dtype=torch.int32)
    big.seq_lens.copy_(n0)
    pub = big.to("cuda")
    outs = [torch.empty((3, 8, 128), device="cuda") for _ in range(10)]
    other = torch.empty_like(outs[0])
    torch.cuda.synchronize()
    for s in range(10):
        spd.spd_decode_step_append(shape, g.q, k_new[s], v_new[s], g.priv, pub, other, ws, stream=st)
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, pub, outs[s], ws, stream=st)
    assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)
    grown = pub.to("cpu")
    for s in range(10):
        grown.seq_lens.copy_(n0 + s + 1)
        x = wl.Workload("grown", 3, 8, 2, 128, 16, torch.bfloat16, w.sm_scale, w.q, w.priv, grown)
        want, _, _, _, tol = ref.decode(x, 20.0, 64, None)
        close(outs[s], want, tol, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_users_than_a_cta_caches(dtype):
    B, hq, hkv, d = 1500, 2, 1, 64
    r = random.Random(5)
    lin, lout = [r.choice([0, 1, 15, 16, 40, 90]) for _ in range(B)], [r.choice([0, 1, 17, 33]) for _ in range(B)]
    w = workload(lin, lout, hq, hkv, d, dtype, 21)
    g, shape, score, sl, ws = setup(w, 20.0, 30, True)
    want, _, _, _, tol = ref.decode(w, 20.0, 30, sl)
    out = torch.full((B, hq, d), float("nan"), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, tol, "many users")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_tiny_prompts(dtype):
    r = random.Random(6)
    lens = [r.choice([0, 0, 1, 2, 3, 5]) for _ in range(900)]
    q, k, v, ip = prompts(lens, 2, 1, 64, dtype, 22)
    want, tol = ref.prefill(q, k, v, lens, 64 ** -0.5, 0.0, 2, None, weight=P_WEIGHT[dtype])
    out, status = run(q, k, v, ip, 64, window=2)
    assert status == (spd.SPD_OK, -1)
    close(out, want, tol, "tiny prompts")


@pytest.mark.parametrize("dtype,cap,alibi", [("bf16", 0.0, True), ("bf16", 30.0, False), ("f32", 0.0, True)])
def test_one_very_long_prompt(dtype, cap, alibi):
    n, hq, hkv, d = 70001, 2, 1, 64
    q, k, v, ip = prompts([n], hq, hkv, d, dtype, 23)
    sl = slopes_of(hq) / 64 if alibi else None                     # down to 2^-14: the bias reaches over the whole prompt
    rows = {0, 1, 79, 80, 4095, 32768, 65535, 65536, 69999, n - 1}
    want, tol = ref.prefill(q, k, v, [n], d ** -0.5, cap, 0, sl, weight=P_WEIGHT[dtype], rows=rows)
    out, status = run(q, k, v, ip, d, cap=cap, slopes=sl)
    assert status == (spd.SPD_OK, -1)
    at = sorted(rows)
    close(out[at], want[at], tol[at], "long prompt")


@pytest.mark.parametrize("dtype,cap,window,alibi", [("bf16", 0.0, 0, True), ("bf16", 50.0, 200000, False), ("f32", 20.0, 0, True)])
def test_one_very_long_cache(dtype, cap, window, alibi):
    w = workload([300007, 5], [13, 100], 4, 1, 64, dtype, 24)
    g, shape, score, _, ws = setup(w, cap, window, False)
    sl = slopes_of(4) / 4096 if alibi else None
    score = spd.make_score(cap, window, None if sl is None else sl.cuda())
    want, _, _, _, tol = ref.decode(w, cap, window, sl)
    out = torch.full((2, 4, 64), float("nan"), device="cuda")
    spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    close(out, want, tol, "long cache")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,hq,hkv", [([300, 129, 0, 200, 257], 8, 2), ([70] * 40, 4, 4), ([9, 31, 1, 0, 25] * 12, 8, 8)])
def test_fp32_tiles_of_every_kind(lens, hq, hkv, d):
    """The three shapes of the fp32 kernel: two groups of threads per tile, one group, and half tiles; what is hidden is spoiled, and a
    visible key that is NaN spoils exactly the rows that see it."""
    T = sum(lens)
    q, k, v, ip = prompts(lens, hq, hkv, d, "f32", 80)
    doc = documents(lens, 81, longest=90)
    prefix = torch.tensor([n // 3 for n in lens], dtype=torch.int32)
    rows = set(random.Random(1).sample(range(T), min(T, 150)))
    for kw in (dict(cap=15.0, slopes=slopes_of(hq)), dict(window=70, prefix=prefix), dict(doc=doc)):
        want, tol = ref.prefill(q, k, v, lens, d ** -0.5, kw.get("cap", 0.0), kw.get("window", 0), kw.get("slopes"), kw.get("prefix"), kw.get("doc"), rows=rows)
        out, status = run(q, k, v, ip, d, kw.get("cap", 0.0), kw.get("window", 0), kw.get("slopes"), kw.get("prefix"), kw.get("doc"))
        assert status == (spd.SPD_OK, -1)
        at = sorted(rows)
        close(out[at], want[at], tol[at], kw.keys())
    # one spoiled key in the longest prompt: causal rows in front of it are as before, rows from it on are NaN
    clean, _ = run(q, k, v, ip, d)
    u = max(range(len(lens)), key=lambda i: lens[i])
    t0, bad = int(ip[u]), lens[u] // 2
    for spoil in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if spoil == "k" else v2)[t0 + bad] = float("nan")
        out, _ = run(q, k2, v2, ip, d)
        hit = torch.zeros(T, dtype=torch.bool)
        hit[t0 + bad:t0 + lens[u]] = True
        assert bool(out[hit.cuda()].isnan().all()), spoil
        assert torch.equal(out[~hit.cuda()], clean[~hit.cuda()]), spoil
