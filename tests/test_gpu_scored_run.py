"""The scored calls together, as a serving loop uses them: prompts are rotated, attended to and handed to the private cache; then
token after token is rotated, appended to the public cache and attended over both partitions, eagerly and from a CUDA graph."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, slopes_of

pytestmark = pytest.mark.gpu


class Layer:
    """One layer's caches: room for the prompts and for `tokens` generated tokens per user, nothing cached yet."""

    def __init__(self, lens, tokens, hkv, d, dtype, seed):
        rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        B = len(lens)
        self.priv = wl.make_paged_kv(np.asarray(lens), hkv, d, dtype, rng, gen, "cpu", poison=False).to("cuda")
        self.pub = wl.make_paged_kv(np.full(B, tokens), hkv, d, dtype, rng, gen, "cpu", poison=False).to("cuda")
        for part in (self.priv, self.pub):
            part.k_pool.fill_(float("nan"))
            part.v_pool.fill_(float("nan"))
            part.seq_lens.zero_()


def cpu(part):
    return part.to("cpu")


@pytest.mark.parametrize("dtype,d,hq,hkv,cap,window,alibi,graph", [
    (torch.bfloat16, 128, 8, 2, 30.0, 0, False, False),
    (torch.bfloat16, 128, 4, 4, 0.0, 50, False, True),
    (torch.bfloat16, 64, 8, 4, 0.0, 0, True, True),
    (torch.float32, 64, 4, 2, 20.0, 33, True, False),
])
def test_prompts_then_tokens(dtype, d, hq, hkv, cap, window, alibi, graph):
    lens, steps, layers = [70, 1, 0, 200], 20, 2
    B, T = len(lens), sum(lens)
    ip = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    gen = torch.Generator().manual_seed(5)
    randn = lambda *s: torch.randn(s, generator=gen).to(dtype)  # noqa: E731
    shape = spd.make_shape(B, hq, hkv, d, dtype, d ** -0.5)
    ws = spd.alloc_workspace(shape)
    inv = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float()
    rope = None if alibi else spd.make_rope(inv.cuda())            # a model has rotary positions or a distance bias
    sl = slopes_of(hq) if alibi else None
    score = spd.make_score(cap, window, None if sl is None else sl.cuda())
    weight = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0

    caches = [Layer(lens, steps, hkv, d, dtype, seed) for seed in range(layers)]
    for ly in caches:
        q, k, v = randn(T, hq, d), randn(T, hkv, d), randn(T, hkv, d)
        qg, kg, vg = q.cuda(), k.cuda(), v.cuda()
        spd.spd_append_kv_rope(shape, rope, qg if rope else None, kg, vg, ly.priv, ws, q_out=qg if rope else None, k_out=kg, tok_indptr=ip)
        out = torch.full((T, hq, d), float("nan"), dtype=dtype, device="cuda")
        spd.spd_prefill_attn_scored(shape, score, qg, kg, vg, ip, out, ws)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        assert ly.priv.seq_lens.tolist() == lens
        want, tol = ref.prefill(qg.cpu(), kg.cpu(), v, lens, d ** -0.5, cap, window, sl, weight=weight)
        close(out, want, tol, "prompts")

    # every step's new rows of every layer, and one buffer for what is fed to the calls
    new = [[(randn(B, hq, d), randn(B, hkv, d), randn(B, hkv, d)) for _ in caches] for _ in range(steps)]
    feed = [tuple(torch.empty_like(t).cuda() for t in x) for x in new[0]]
    q_rot = [torch.empty_like(f[0]) for f in feed]
    outs = [torch.empty((B, hq, d), dtype=dtype, device="cuda") for _ in caches]
    st = torch.cuda.Stream()

    def step():
        for ly, (q, k, v), qr, out in zip(caches, feed, q_rot, outs):
            spd.spd_append_kv_rope(shape, rope, q if rope else None, k, v, ly.pub, ws, q_out=qr if rope else None,
                                   pos_base=ly.priv.seq_lens if rope else None, stream=st)
            spd.spd_decode_step_scored(shape, score, qr if rope else q, ly.priv, ly.pub, out, ws, stream=st)
    torch.cuda.synchronize()
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured, stream=st):
            step()
    for s in range(steps):
        for f, x in zip(feed, new[s]):
            for a, b in zip(f, x):
                a.copy_(b)
        torch.cuda.synchronize()
        if graph:
            with torch.cuda.stream(st):
                captured.replay()
        else:
            step()
        st.synchronize()
        for ly, (q, k, v), qr, out in zip(caches, new[s], q_rot, outs):
            assert ly.pub.seq_lens.tolist() == [s + 1] * B
            if rope:
                pos = (torch.tensor(lens) + s).double()[:, None].expand(-1, d // 2)
                turned = ref.rotate(q, pos, inv, False)
                assert bool(((qr.cpu().double() - turned).abs() <= ref.rotate_bound(q, inv, False, dtype, turned)).all())
            if s % 7 == 0 or s == steps - 1:
                w = wl.Workload("run", B, hq, hkv, d, 16, dtype, d ** -0.5, qr.cpu() if rope else q, cpu(ly.priv), cpu(ly.pub))
                want, _, _, _, tol = ref.decode(w, cap, window, sl)
                close(out, want, tol, f"step {s}")
                for u in range(B):                                  # the new rows sit where they belong
                    kk, vv = wl.gather_dense(w.pub, u, 0)
                    assert torch.equal(vv[s], v[u, 0]) and bool(torch.isfinite(kk).all())
    assert spd.spd_query_device_status(ws, st) == (spd.SPD_OK, -1)


def test_decode_follows_a_prompt_as_prompt_attention_would():
    """The last row of a prompt through prompt attention, and the same token as a generated one through the two caches."""
    lens, hq, hkv, d = [150, 33, 1], 8, 2, 128
    T, B = sum(lens), 3
    gen = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn((T, h, d), generator=gen).bfloat16().cuda() for h in (hq, hkv, hkv))
    shape = spd.make_shape(B, hq, hkv, d, torch.bfloat16, d ** -0.5)
    ws, score = spd.alloc_workspace(shape), spd.make_score(10.0, 60)
    ip = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    whole = torch.empty((T, hq, d), device="cuda")
    spd.spd_prefill_attn_scored(shape, score, q, k, v, ip, whole, ws)
    ly = Layer(lens, 4, hkv, d, torch.bfloat16, 3)
    last = (ip[1:] - 1).long()
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[last] = False
    short = torch.from_numpy(np.concatenate([[0], np.cumsum(np.array(lens) - 1)]).astype(np.int32)).cuda()
    spd.spd_append_kv_rope(shape, None, None, k[keep], v[keep], ly.priv, ws, tok_indptr=short)
    spd.spd_append_kv_rope(shape, None, None, k[last], v[last], ly.pub, ws)
    out = torch.empty((B, hq, d), device="cuda")
    spd.spd_decode_step_scored(shape, score, q[last], ly.priv, ly.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    # prompt attention rounds its weights to bf16 once: half a step of the greatest |v|; the rest is far smaller
    assert float((out - whole[last]).abs().max()) <= (2.0 ** -8 + 2.0 ** -12) * float(v.abs().max())
