"""Append with rotation: rotated rows, cache rows bit for bit, lengths, refusals on the device, streams and graphs."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(B, hq, hkv, d, dtype, runs, held, seed, slack=2, wide=False):
    """Tokens (CPU), the partition that takes them (CPU) and the offsets; wide: q, k and v are parts of one wider row per token."""
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    runs, held = np.asarray(runs), np.asarray(held)
    T = int(runs.sum())
    part = wl.make_paged_kv(held + runs, hkv, d, DT[dtype], rng, gen, "cpu", slack_pages=np.full(B, slack), poison=False)
    part.seq_lens = torch.from_numpy(held.astype(np.int32))
    if wide:
        row = torch.randn((T, (hq + 2 * hkv) * d + 16), generator=gen).to(DT[dtype])
        q, k, v = row[:, :hq * d].view(T, hq, d), row[:, hq * d:(hq + hkv) * d].view(T, hkv, d), row[:, (hq + hkv) * d:(hq + 2 * hkv) * d].view(T, hkv, d)
    else:
        q, k, v = (torch.randn((T, h, d), generator=gen).to(DT[dtype]) for h in (hq, hkv, hkv))
    ip = torch.from_numpy(np.concatenate([[0], np.cumsum(runs)]).astype(np.int32))
    return q, k, v, part, ip


def wide_to(t, dev):
    """Copy that keeps a strided view's strides."""
    base = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=dev)
    return base.copy_(t)


def expect(part, ip, k, v, ok=None):
    """The pools after the append (bit for bit) and the grown lengths."""
    kp, vp, lens = part.k_pool.clone(), part.v_pool.clone(), part.seq_lens.clone()
    for u in range(len(lens)):
        a, b, held = int(ip[u]), int(ip[u + 1]), int(part.seq_lens[u])
        if ok is not None and not ok[u]:
            continue
        for i in range(b - a):
            pg = int(part.page_indices[int(part.page_indptr[u]) + (held + i) // 16])
            kp[pg, :, (held + i) % 16], vp[pg, :, (held + i) % 16] = k[a + i], v[a + i]
        lens[u] = held + b - a
    return kp, vp, lens


def positions_of(part, ip, base, pairs):
    p = torch.cat([torch.arange(int(ip[u]), int(ip[u + 1])) - int(ip[u]) + int(part.seq_lens[u]) + (int(base[u]) if base is not None else 0)
                   for u in range(len(part.seq_lens))])
    return p.double()[:, None].expand(-1, pairs)


CASES = [
    # dtype, d, hq, hkv, rot, interleaved, runs (None: one token each), held, wide
    ("bf16", 128, 8, 2, 128, False, None, [0, 1, 15, 16, 17, 300], False),
    ("bf16", 128, 32, 8, 128, False, [1, 0, 37, 16, 5, 130], [0, 9, 15, 16, 0, 1], False),
    ("bf16", 64, 5, 5, 32, True, [3, 70, 1], [0, 14, 31], True),
    ("bf16", 64, 16, 2, 16, False, None, [40, 0, 7], True),
    ("f32", 64, 8, 8, 64, False, [33, 1, 2], [0, 0, 100], False),
    ("f32", 128, 4, 1, 96, True, None, [5], True),
    ("f32", 128, 2, 2, 128, False, [513], [16], True),
]


@pytest.mark.parametrize("dtype,d,hq,hkv,rot,inter,runs,held,wide", CASES)
def test_rows_cache_and_lengths(dtype, d, hq, hkv, rot, inter, runs, held, wide):
    B = len(held)
    q, k, v, part, ip = make(B, hq, hkv, d, dtype, runs if runs is not None else [1] * B, held, seed=rot + B, wide=wide)
    T = q.shape[0]
    base = torch.arange(B, dtype=torch.int32) * 13001 + 5
    inv = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float()
    pos = positions_of(part, ip, base, rot // 2)
    want_q, want_k = ref.rotate(q, pos, inv, inter), ref.rotate(k, pos, inv, inter)
    g = part.to("cuda")
    shape = spd.make_shape(B, hq, hkv, d, DT[dtype], 1.0)
    ws = spd.alloc_workspace(shape)
    q_out = torch.full((T, hq, d), float("nan"), dtype=DT[dtype], device="cuda")
    k_out = torch.full((T, hkv, d), float("nan"), dtype=DT[dtype], device="cuda")
    spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda(), interleaved=inter), wide_to(q, "cuda"), wide_to(k, "cuda"), wide_to(v, "cuda"), g, ws,
                           q_out=q_out, k_out=k_out, tok_indptr=None if runs is None else ip.cuda(), pos_base=base.cuda())
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    for got, want, x in ((q_out, want_q, q), (k_out, want_k, k)):
        err = (got.cpu().double() - want).abs()
        assert bool((err <= ref.rotate_bound(x, inv, inter, DT[dtype], want)).all()), float(err.max())
    kp, vp, lens = expect(part, ip, k_out.cpu(), v)
    assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp)      # every other slot is as it was
    assert torch.equal(g.seq_lens.cpu(), lens)


def test_far_positions_keep_their_angles():
    """Positions near 2^31: the angle is reduced in 64 bits, so the fastest pair still turns right."""
    B, hq, hkv, d = 3, 2, 1, 64
    q, k, v, part, ip = make(B, hq, hkv, d, "f32", [1, 1, 1], [0, 3, 40], seed=5)
    pos = torch.tensor([[2147483647, 1000003, 131071]], dtype=torch.int32)
    inv = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    want = ref.rotate(q, pos[0].double()[:, None].expand(-1, 32), inv, False, 1.25)
    shape, g = spd.make_shape(B, hq, hkv, d, torch.float32, 1.0), part.to("cuda")
    ws = spd.alloc_workspace(shape)
    qg = q.cuda()
    spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda(), scale=1.25), qg, k.cuda(), v.cuda(), g, ws, q_out=qg, positions=pos.cuda())   # in place
    assert bool(((qg.cpu().double() - want).abs() <= ref.rotate_bound(q, inv, False, torch.float32, want, 1.25)).all())


@pytest.mark.parametrize("runs", [None, [40, 3, 0, 7]])
def test_several_axes(runs):
    B, hq, hkv, d, sec = 4, 6, 3, 128, (16, 24, 24)
    q, k, v, part, ip = make(B, hq, hkv, d, "bf16", runs or [1] * B, [0, 5, 16, 33], seed=9)
    T = q.shape[0]
    pos = torch.randint(-50, 5000, (3, T), generator=torch.Generator().manual_seed(1)).int()
    inv = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float()
    per_pair = torch.cat([pos[a].double()[:, None].expand(-1, n) for a, n in enumerate(sec)], 1)
    shape, g = spd.make_shape(B, hq, hkv, d, torch.bfloat16, 1.0), part.to("cuda")
    ws = spd.alloc_workspace(shape)
    q_out, kg = torch.empty_like(q, device="cuda"), k.cuda()
    spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda(), sections=sec), q.cuda(), kg, v.cuda(), g, ws, q_out=q_out, k_out=kg,
                           tok_indptr=None if runs is None else ip.cuda(), positions=pos.cuda())
    for got, x in ((q_out, q), (kg, k)):
        want = ref.rotate(x, per_pair, inv, False)
        assert bool(((got.cpu().double() - want).abs() <= ref.rotate_bound(x, inv, False, torch.bfloat16, want)).all())
    kp, vp, lens = expect(part, ip, kg.cpu(), v)
    assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp) and torch.equal(g.seq_lens.cpu(), lens)


@pytest.mark.parametrize("runs", [None, [17, 1, 0]])
def test_without_rotation_and_where_lengths_go(runs):
    B, hkv, d = 3, 4, 64
    q, k, v, part, ip = make(B, 8, hkv, d, "bf16", runs or [1] * B, [0, 15, 32], seed=3)
    shape = spd.make_shape(B, 8, hkv, d, torch.bfloat16, 1.0)
    ws = spd.alloc_workspace(shape)
    kp, vp, lens = expect(part, ip, k, v)
    for where in ("in place", "other", None):
        g = part.to("cuda")
        other = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        spd.spd_append_kv_rope(shape, None, None, k.cuda(), v.cuda(), g, ws, tok_indptr=None if runs is None else ip.cuda(),
                               new_lens=other if where == "other" else where)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp)
        assert torch.equal(g.seq_lens.cpu(), lens if where == "in place" else part.seq_lens)
        assert other.tolist() == (lens.tolist() if where == "other" else [-7] * B)


@pytest.mark.parametrize("ragged", [False, True])
def test_users_without_room_or_with_bad_pages_keep_their_length(ragged):
    """User 1 is full, user 3 lists a page outside the pool, user 4 a negative length: flagged, the others served."""
    B, hq, hkv, d = 6, 4, 2, 64
    runs = [20, 20, 20, 20, 20, 20] if ragged else [1] * B
    q, k, v, part, ip = make(B, hq, hkv, d, "bf16", runs, [5, 16, 0, 16, 7, 30], seed=8, slack=0)
    part.seq_lens[1] = 16 * int(part.page_indptr[2] - part.page_indptr[1])
    part.page_indices[int(part.page_indptr[3]) + 1] = part.num_pages
    part.seq_lens[4] = -2
    ok = [True, False, True, False, False, True]
    inv = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    shape, g = spd.make_shape(B, hq, hkv, d, torch.bfloat16, 1.0), part.to("cuda")
    ws = spd.alloc_workspace(shape)
    k_out, q_out = torch.empty_like(k, device="cuda"), torch.empty_like(q, device="cuda")
    spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda()), q.cuda(), k.cuda(), v.cuda(), g, ws, q_out=q_out, k_out=k_out,
                           tok_indptr=ip.cuda() if ragged else None)
    assert spd.spd_query_device_status(ws) == (4, 1)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    kp, vp, lens = expect(part, ip, k_out.cpu(), v, ok)
    assert torch.equal(g.seq_lens.cpu(), lens)
    for u in [u for u in range(B) if ok[u]] + [1]:              # what a served user holds; user 1's full cache is untouched
        pages = part.page_indices[int(part.page_indptr[u]):int(part.page_indptr[u + 1])].long()
        assert torch.equal(g.k_pool.cpu()[pages], kp[pages]) and torch.equal(g.v_pool.cpu()[pages], vp[pages])
    want = ref.rotate(q, positions_of(part, ip, None, 32), inv, False)      # rotated rows are there for everybody
    assert bool(((q_out.cpu().double() - want).abs() <= ref.rotate_bound(q, inv, False, torch.bfloat16, want)).all())


@pytest.mark.parametrize("ip,bad", [([0, 5, 3, 9], 1), ([1, 4, 6, 9], 0), ([0, 4, 6, 8], 2)])
def test_inconsistent_offsets_write_nothing(ip, bad):
    B, hkv, d = 3, 2, 64
    q, k, v, part, _ = make(B, 4, hkv, d, "f32", [3, 3, 3], [2, 2, 2], seed=4)
    shape, g = spd.make_shape(B, 4, hkv, d, torch.float32, 1.0), part.to("cuda")
    ws = spd.alloc_workspace(shape)
    k_out = torch.full_like(k, 3.0).cuda()
    spd.spd_append_kv_rope(shape, None, None, k.cuda(), v.cuda(), g, ws, k_out=k_out, tok_indptr=torch.tensor(ip, dtype=torch.int32).cuda())
    assert spd.spd_query_device_status(ws) == (4, bad)
    assert torch.equal(g.k_pool.cpu(), part.k_pool) and torch.equal(g.v_pool.cpu(), part.v_pool)
    assert torch.equal(g.seq_lens.cpu(), part.seq_lens) and bool((k_out == 3.0).all())


def test_no_tokens_and_many_users():
    B, hkv, d = 700, 1, 64
    runs = [0] * B
    q, k, v, part, ip = make(B, 1, hkv, d, "bf16", runs, [3] * B, seed=6)
    shape, g = spd.make_shape(B, 1, hkv, d, torch.bfloat16, 1.0), part.to("cuda")
    ws = spd.alloc_workspace(shape)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    spd.spd_append_kv_rope(shape, None, None, k.cuda(), v.cuda(), g, ws, tok_indptr=ip.cuda(), new_lens=lens)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1) and lens.tolist() == [3] * B
    runs = (np.arange(B) % 5).tolist()                          # many short runs, some empty
    q, k, v, part, ip = make(B, 1, hkv, d, "bf16", runs, (np.arange(B) % 40).tolist(), seed=7)
    g = part.to("cuda")
    spd.spd_append_kv_rope(shape, None, None, k.cuda(), v.cuda(), g, ws, tok_indptr=ip.cuda())
    kp, vp, want = expect(part, ip, k, v)
    assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp) and torch.equal(g.seq_lens.cpu(), want)


@pytest.mark.parametrize("ragged", [False, True])
def test_side_stream_and_graph_replay(ragged):
    """Captured on a side stream and replayed: each replay appends behind what the one before left."""
    B, hq, hkv, d, n = 4, 4, 2, 128, 3
    runs = [2, 0, 5, 1] if ragged else [1] * B
    q, k, v, part, ip = make(B, hq, hkv, d, "bf16", runs, [0, 14, 16, 33], seed=12, slack=3)
    shape, g = spd.make_shape(B, hq, hkv, d, torch.bfloat16, 1.0), part.to("cuda")
    ws, st = spd.alloc_workspace(shape), torch.cuda.Stream()
    inv = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    args = [x.cuda() for x in (q, k, v)]
    q_out, k_out, ipg = torch.empty_like(args[0]), torch.empty_like(args[1]), ip.cuda()
    rope = spd.make_rope(inv)
    call = lambda: spd.spd_append_kv_rope(shape, rope, *args, g, ws, q_out=q_out, k_out=k_out, tok_indptr=ipg if ragged else None, stream=st)  # noqa: E731
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    now = part
    for _ in range(n):
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        kp, vp, lens = expect(now, ip, k_out.cpu(), v)
        want = ref.rotate(k, positions_of(now, ip, None, 64), inv.cpu(), False)
        assert bool(((k_out.cpu().double() - want).abs() <= ref.rotate_bound(k, inv.cpu(), False, torch.bfloat16, want)).all())
        assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp) and torch.equal(g.seq_lens.cpu(), lens)
        now = wl.PagedKV(kp, vp, part.page_indptr, part.page_indices, lens)
    assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)


def test_a_replayed_call_starts_without_old_flags():
    """Runs appended in place from a graph: a user refused for a bad page in one replay is served in the next once its table is mended."""
    q, k, v, part, ip = make(3, 4, 2, 64, "bf16", [20, 20, 5], [3, 10, 0], seed=31)
    g, shape = part.to("cuda"), spd.make_shape(3, 4, 2, 64, torch.bfloat16, 0.1)
    ws, st, kg, vg, ipg = spd.alloc_workspace(shape), torch.cuda.Stream(), k.cuda(), v.cuda(), ip.cuda()
    at = int(part.page_indptr[1]) + 1
    g.page_indices[at] = -7
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        spd.spd_append_kv_rope(shape, None, None, kg, vg, g, ws, tok_indptr=ipg, stream=st)
    with torch.cuda.stream(st):
        graph.replay()
    torch.cuda.synchronize()
    assert g.seq_lens.tolist() == [23, 10, 5]
    g.page_indices[at] = part.page_indices[at]
    g.seq_lens.copy_(part.seq_lens)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        graph.replay()
    torch.cuda.synchronize()
    kp, vp, lens = expect(part, ip, k, v)
    assert g.seq_lens.tolist() == lens.tolist() == [23, 30, 5]
    assert torch.equal(g.k_pool.cpu(), kp) and torch.equal(g.v_pool.cpu(), vp)
    assert spd.spd_query_device_status(ws) == (4, 1)              # the first replay's, still to be read


def test_positions_may_be_the_lengths_themselves():
    """One token per user at the position its cache ends at: positions, seq_lens and new_lens one array, with and without offsets."""
    for ragged in (False, True):
        q, k, v, part, ip = make(5, 4, 2, 128, "bf16", [1] * 5, [0, 17, 3, 90, 1000], seed=32)
        g, shape = part.to("cuda"), spd.make_shape(5, 4, 2, 128, torch.bfloat16, 0.1)
        inv = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float()
        ws, qo = spd.alloc_workspace(shape), torch.empty_like(q, device="cuda")
        spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda()), q.cuda(), k.cuda(), v.cuda(), g, ws, q_out=qo,
                               tok_indptr=ip.cuda() if ragged else None, positions=g.seq_lens)
        assert g.seq_lens.tolist() == [1, 18, 4, 91, 1001] and spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        want = ref.rotate(q, part.seq_lens.double()[:, None].expand(-1, 64), inv, False)
        assert bool(((qo.cpu().double() - want).abs() <= ref.rotate_bound(q, inv, False, torch.bfloat16, want)).all())
        if ragged:
            with pytest.raises(spd.SpdError):
                other = g.seq_lens.clone()
                spd.spd_append_kv_rope(shape, spd.make_rope(inv.cuda()), q.cuda(), k.cuda(), v.cuda(), g, ws, q_out=qo, tok_indptr=ip.cuda(),
                                       positions=other, new_lens=other)
