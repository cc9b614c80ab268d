"""Attention of drafted tokens (trees and runs over both partitions, windows with sinks, capped and biased scores) against the 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import drafted_reference as dr

pytestmark = pytest.mark.gpu

# drafted, private and public context tokens per user: nothing cached, one partition empty, no drafted tokens, ends inside and at the end of a page
MIX = ([3, 1, 7, 0, 16, 5, 33, 2, 9], [0, 40, 0, 17, 16, 0, 300, 1, 65], [0, 0, 25, 0, 16, 1, 33, 1, 0])
SHAPES = [("bf16", 128, 8, 2), ("bf16", 128, 4, 4), ("bf16", 64, 16, 2), ("bf16", 64, 24, 1), ("bf16", 128, 2, 1), ("f32", 64, 8, 8), ("f32", 128, 8, 2),
          ("f32", 64, 16, 1)]


def ok(d):
    assert spd.spd_query_device_status(d.ws) == (spd.SPD_OK, -1)


@pytest.mark.parametrize("dtype,d,hq,hkv", SHAPES)
@pytest.mark.parametrize("kind", ["tree", "run"])
@pytest.mark.parametrize("cap,window,sinks,alibi", [(0.0, 0, 0, False), (20.0, 0, 0, False), (0.0, 0, 0, True), (0.0, 1, 0, False), (0.0, 17, 3, True),
                                                    (5.0, 33, 40, True), (50.0, 300, 1, False), (0.0, 100000, 5, False)])
def test_fused_and_halves(dtype, d, hq, hkv, kind, cap, window, sinks, alibi):
    w = dr.batch(*MIX, hq, hkv, d, dtype, seed=d + hq, kind=kind, qscale=3.0)
    g = dr.OnDevice(w, cap, window, sinks, alibi)
    want, _, _, _, tol = dr.expected(w, cap, window, sinks, g.slopes)
    for out_dtype in (torch.float32, torch.bfloat16):
        dr.close(g.fused(out_dtype), want, tol, "fused")
    out, part = g.halves()
    dr.close(out, want, tol, "halves")
    _, O, m, l, _ = dr.expected(w, cap, window, sinks, g.slopes, parts=(True, False))
    mg, lg = part[1].cpu().double(), part[2].cpu().double()
    none = l == 0
    assert bool((lg[none] == 0).all()) and bool((mg[none] == -float("inf")).all()) and bool((part[0].cpu()[none] == 0).all())
    scale = torch.exp(mg[~none] - m[~none])                # the partial's reference may differ from the maximum by its own rounding
    assert bool(((scale - 1).abs() < 1e-3).all())
    assert bool(((lg[~none] * scale - l[~none]).abs() <= 4e-3 * l[~none]).all())
    ok(g)


@pytest.mark.parametrize("kind", ["star", "chain"])
@pytest.mark.parametrize("n", [1, 31, 64, 65, 200, 256])
def test_tree_shapes(kind, n):
    w = dr.batch([n, max(1, n // 2)], [100, 7], [3, 50], 4, 1, 64, "bf16", seed=n, kind=kind)
    g = dr.OnDevice(w, window=40, sinks=5)
    want, _, _, _, tol = dr.expected(w, window=40, sinks=5)
    dr.close(g.fused(), want, tol)
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 16), (700, 20)])
def test_long_runs(dtype, window, sinks):
    """Parts of prompts behind a cache: many tiles of rows, each with keys of its own."""
    w = dr.batch([333, 1, 700], [500, 20, 0], [0, 3, 0], 4, 2, 64, dtype, seed=5, kind="run")
    g = dr.OnDevice(w, window=window, sinks=sinks)
    rows = set(range(0, 1034, 37)) | {332, 333, 334, 1033}
    want, _, _, _, tol = dr.expected(w, window=window, sinks=sinks, rows=rows)
    at = torch.tensor(sorted(rows))
    dr.close(g.fused()[at.cuda()], want[at], tol[at])
    ok(g)


@pytest.mark.parametrize("dtype,d,hq", [("bf16", 128, 8), ("f32", 64, 4)])
def test_cut_sequences(dtype, d, hq):
    """Few users with long caches: every item is cut over many CTAs and joined; twice the same bits."""
    w = dr.batch([6, 2], [5000, 3001], [77, 0], hq, 1, d, dtype, seed=11)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    a, b = g.fused(), g.fused()
    assert torch.equal(a, b)
    dr.close(a, want, tol)
    dr.close(g.halves()[0], want, tol)
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_per_user_needs_no_offsets(dtype):
    w = dr.batch([1] * 5, [30, 0, 4000, 100, 17], [0, 0, 9, 40, 200], 8, 2, 64, dtype, seed=3, kind="run")
    g = dr.OnDevice(w, window=50, sinks=4)
    want, _, _, _, tol = dr.expected(w, window=50, sinks=4)
    out = g.fused()
    dr.close(out, want, tol)
    g.drafts["tok_indptr"] = None
    assert torch.equal(g.fused(), out)
    ok(g)


def test_agrees_with_the_scored_step():
    """One token without sinks is what the scored step computes, in its own rounding."""
    w = dr.batch([1] * 4, [300, 20, 1, 77], [5, 0, 3, 90], 16, 2, 128, "bf16", seed=8, kind="run")
    g = dr.OnDevice(w, cap=30.0, window=64, alibi=True)
    out, other = g.fused(), g.out()
    spd.spd_decode_step_scored(g.shape, g.score, g.q, g.priv, g.pub, other, g.ws)
    _, _, _, _, tol = dr.expected(w, 30.0, 64, 0, g.slopes)
    dr.close(out, other.cpu().double(), 2 * tol)
    ok(g)


def test_partials_merge_by_rows():
    w = dr.batch([4, 7], [90, 33], [20, 2], 4, 2, 64, "bf16", seed=21)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    part, out = g.partial(), g.out()
    spd.spd_partial_attn_drafted(g.shape, g.score, g.q, g.priv, g.pub.seq_lens, part, g.ws, **g.drafts)
    rows = spd.make_shape(g.T, 4, 2, 64, torch.bfloat16, w.sm_scale)
    empty = (torch.zeros_like(part[0]), torch.full_like(part[1], -float("inf")), torch.zeros_like(part[2]))
    spd.spd_service_attn_merge_drafted(g.shape, g.score, g.q, g.pub, g.priv.seq_lens, empty, out, g.ws, **g.drafts)
    public = dr.expected(w, parts=(False, True))
    dr.close(out, public[0], public[4], "an empty partial changes nothing")
    spd.spd_merge_partials(rows, [part], out)
    private = dr.expected(w, parts=(True, False))
    dr.close(out, private[0], private[4], "the private half alone")
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_hidden_keys_never_enter(dtype, value):
    """A drafted token that is not finite reaches itself and what comes after it, nobody else; context in front of the window nobody."""
    n, lp = 6, 70
    w = dr.batch([n, 3], [lp, 20], [10, 0], 4, 1, 64, dtype, seed=31)
    w.trees[0] = np.array([-1, 0, -1, 2, 1, 2])
    w.parents = torch.from_numpy(np.concatenate(w.trees).astype(np.int32))
    window, sinks = 30, 2
    want, _, _, _, tol = dr.expected(w, window=window, sinks=sinks)
    spoiled = []
    for part, x in ((w.pub, 10 + 2), (w.priv, 5), (w.priv, lp - 19)):       # token 2; hidden from all; seen by the roots alone
        page = int(part.page_indices[int(part.page_indptr[0]) + x // 16])
        part.v_pool[page, :, x % 16] = value
        spoiled.append((page, x % 16))
    w.priv.k_pool[int(w.priv.page_indices[int(w.priv.page_indptr[0])]), :, 9] = float("nan")      # hidden too
    out = dr.OnDevice(w, window=window, sinks=sinks).fused().cpu()
    ctx, depth = lp + 10, [0, 1, 0, 1, 2, 1]
    line = {0: [0], 1: [0, 1], 2: [2], 3: [2, 3], 4: [0, 1, 4], 5: [2, 5]}
    for i in range(n):
        hit = 2 in line[i] or ctx + depth[i] - (lp - 19) < window
        if hit:
            assert not bool(torch.isfinite(out[i]).any()), i
        else:
            dr.close(out[i:i + 1], want[i:i + 1], tol[i:i + 1], i)
    dr.close(out[n:], want[n:], tol[n:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype):
    w = dr.batch([2, 2], [40, 0], [0, 0], 2, 1, 64, dtype, seed=41, kind="run")
    w.q.copy_(torch.ones_like(w.q))
    for part in (w.priv, w.pub):
        part.k_pool[torch.isfinite(part.k_pool)] = -float("inf")
    out = dr.OnDevice(w).fused()
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_flagged_users(dtype):
    w = dr.batch([3, 4, 2, 5, 2], [100, 30, 60, 20, 40], [0, 9, 4, 2, 0], 4, 2, 64, dtype, seed=51)
    want, _, _, _, tol = dr.expected(w)
    g = dr.OnDevice(w)
    starts = w.indptr.tolist()

    def run(first):
        out = g.fused()
        code, bad = spd.spd_query_device_status(g.ws)
        assert (code, bad) == (4, first)
        return out

    keep = g.priv.page_indices.clone()
    g.priv.page_indices[int(g.priv.page_indptr[1])] = 1 << 30                   # user 1
    g.drafts["parents"][starts[3] + 2] = 2                                       # user 3: its own parent
    out = run(1)
    for u in range(5):
        a, b = starts[u], starts[u + 1]
        if u in (1, 3):
            assert bool((out[a:b] == 0).all())
        else:
            dr.close(out[a:b], want[a:b], tol[a:b], u)
    g.priv.page_indices.copy_(keep)
    g.drafts["parents"][starts[3] + 2] = -2
    assert bool((run(3)[starts[3]:starts[4]] == 0).all())
    g.drafts["parents"][starts[3] + 2] = 1
    g.pub.seq_lens[4] = 1                                                        # fewer public tokens than drafted ones
    out = run(4)
    assert bool((out[starts[4]:] == 0).all())
    dr.close(out[:starts[3]], want[:starts[3]], tol[:starts[3]])
    g.pub.seq_lens[4] = 2
    g.drafts["tok_indptr"][3] = starts[2] - 1                                    # not monotone: user 2 and all behind it are left out
    out = run(2)
    dr.close(out[:starts[2]], want[:starts[2]], tol[:starts[2]])
    assert bool(torch.isnan(out[starts[2]:]).all())


def test_wide_trees_are_flagged():
    w = dr.batch([257, 3], [10, 10], [0, 0], 2, 1, 64, "bf16", seed=61, kind="chain")
    g = dr.OnDevice(w)
    out = g.fused()
    assert spd.spd_query_device_status(g.ws) == (4, 0)
    assert bool((out[:257] == 0).all()) and bool(torch.isfinite(out[257:]).all())


def test_graph_and_streams():
    w = dr.batch([5, 9, 1], [700, 30, 64], [3, 0, 16], 8, 2, 128, "bf16", seed=71)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    out, side = g.out(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g.fused(out=out)
    side.synchronize()
    dr.close(out, want, tol)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.fused(out=out)
    out.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    dr.close(out, want, tol)
    ok(g)


def test_users_beyond_the_threads():
    """More users than a CTA has threads, many of them without drafted tokens."""
    rng = np.random.default_rng(81)
    counts = rng.integers(0, 3, 700)
    w = dr.batch(counts, rng.integers(0, 40, 700), rng.integers(0, 20, 700), 2, 1, 64, "bf16", seed=81)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    dr.close(g.fused(), want, tol)
    ok(g)


def test_nothing_drafted():
    w = dr.batch([0, 0], [10, 20], [3, 0], 2, 1, 64, "f32", seed=91)
    g = dr.OnDevice(w)
    assert g.fused().numel() == 0
    ok(g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_outputs_at_odd_multiples_of_16_bytes(dtype):
    w = dr.batch([3, 9], [40, 600], [5, 0], 8, 2, 128, "bf16", seed=93)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    es = torch.finfo(dtype).bits // 8
    room = torch.full((12 * 8 * 128 + 64,), float("nan"), dtype=dtype, device="cuda")
    out = room[16 // es:16 // es + 12 * 8 * 128].view(12, 8, 128)
    assert out.data_ptr() % 32 == 16
    dr.close(g.fused(out=out), want, tol)
    assert bool(torch.isnan(room[:16 // es]).all()) and bool(torch.isnan(room[16 // es + out.numel():]).all())
    ok(g)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 20)])
def test_what_shared_memory_held_before(window, sinks):
    """Runs whose tiles of rows end in front of the partition's end leave parts of their last block unloaded: nothing of what an earlier
    call left there (here: rows that are not finite) may enter."""
    spoil = dr.batch([40, 40], [500, 300], [0, 0], 4, 2, 128, "bf16", seed=95, kind="run")
    for part in (spoil.priv, spoil.pub):
        part.v_pool.fill_(float("nan"))
    s = dr.OnDevice(spoil)
    w = dr.batch([500, 300, 77], [333, 70, 9], [0, 3, 0], 4, 2, 128, "bf16", seed=96, kind="run")
    g = dr.OnDevice(w, window=window, sinks=sinks)
    first = g.fused()
    rows = set(range(0, 877, 23))
    want, _, _, _, tol = dr.expected(w, window=window, sinks=sinks, rows=rows)
    at = torch.tensor(sorted(rows))
    dr.close(first[at.cuda()], want[at], tol[at])
    for _ in range(3):
        s.fused()
        assert torch.equal(g.fused(), first)
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(136, 1), (128, 1), (40, 1), (48, 2)])
def test_wide_groups(dtype, hq, hkv):
    """Groups that fill a tile of rows, leave some of it empty, or are cut."""
    w = dr.batch([3, 1, 9], [20, 90, 0], [4, 0, 7], hq, hkv, 64, dtype, seed=hq)
    g = dr.OnDevice(w, window=40, sinks=2)
    want, _, _, _, tol = dr.expected(w, window=40, sinks=2)
    dr.close(g.fused(), want, tol)
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_without_pages(dtype):
    w = dr.batch([4, 2], [0, 0], [9, 30], 4, 2, 64, dtype, seed=97)
    w.priv.k_pool, w.priv.v_pool = w.priv.k_pool[:0].contiguous(), w.priv.v_pool[:0].contiguous()
    w.priv.page_indptr, w.priv.page_indices = torch.zeros(3, dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    g = dr.OnDevice(w)
    want, _, _, _, tol = dr.expected(w)
    dr.close(g.fused(), want, tol)
    dr.close(g.halves()[0], want, tol)
    ok(g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_users_many_heads_drawn(dtype):
    rng = np.random.default_rng(98)
    for seed in range(12):
        B, hkv, g = int(rng.integers(1, 9)), int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 8, 16]))
        d, kind = int(rng.choice([64, 128])), str(rng.choice(["tree", "run", "star", "chain"]))
        counts = rng.integers(0, int(rng.choice([2, 20, 70])), B)
        if counts.sum() == 0:
            counts[0] = 1
        w = dr.batch(counts, rng.integers(0, int(rng.choice([5, 200, 900])), B), rng.integers(0, 90, B), hkv * g, hkv, d, dtype, seed=seed, kind=kind, qscale=2.0)
        args = float(rng.choice([0.0, 20.0, 1e-3, 1e6])), int(rng.choice([0, 5, 70, 2**31 - 1])), int(rng.choice([0, 3, 50, 2**31 - 1]))
        h = dr.OnDevice(w, *args, alibi=bool(rng.integers(0, 2)))
        rows = set(rng.integers(0, h.T, 12).tolist())
        want, _, _, _, tol = dr.expected(w, *args, h.slopes, rows=rows)
        at = torch.tensor(sorted(rows))
        dr.close(h.fused(torch.bfloat16)[at.cuda()], want[at], tol[at], seed)
        dr.close(h.halves()[0][at.cuda()], want[at], tol[at], seed)
        ok(h)
