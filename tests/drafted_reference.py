"""Plain 64-bit form of the calls for drafted tokens, and the batches that their tests use.  Error bounds: tests/scored_reference.py; weights that are
rounded to bf16 for the product with V count 2^-8 once."""
import math

import numpy as np
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import scored_reference as ref


def slopes_of(hq):
    return (2.0 ** (-8.0 * torch.arange(1, hq + 1, dtype=torch.float64) / hq)).float()


def trees(counts, seed, kind="tree"):
    """Parents per user: a random tree, a run, a star (all tokens right behind the context), or a run given as a tree."""
    rng = np.random.default_rng(seed)
    if kind == "star":
        return [np.full(n, -1) for n in counts]
    if kind in ("run", "chain"):
        return [np.arange(n) - 1 for n in counts]
    return [np.array([int(rng.integers(-1, i)) if i else -1 for i in range(n)], dtype=np.int64) for n in counts]


def batch(counts, lin, lout, hq, hkv, d, dtype, seed, kind="tree", qscale=1.0):
    """A workload whose public partitions end with the drafted tokens: lout counts the public tokens in front of them."""
    counts, lin, lout = (np.asarray(x) for x in (counts, lin, lout))
    w = wl.make_workload(dict(batch=len(counts), hq=hq, hkv=hkv, d=d, dtype=dtype, lin=("const", 0), lout=("const", 0), seed=seed),
                         lengths=(lin, lout + counts), slack=True)
    T = int(counts.sum())
    gen = torch.Generator().manual_seed(seed + 1000)
    w.q = (torch.randn((T, hq, d), generator=gen) * qscale).to(w.dtype)
    w.counts, w.kind, w.trees = counts, kind, trees(counts, seed, kind)
    w.indptr = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    w.parents = None if kind == "run" else torch.from_numpy(np.concatenate(w.trees + [np.zeros(0)]).astype(np.int32))
    return w


class OnDevice:
    def __init__(self, w, cap=0.0, window=0, sinks=0, alibi=False, device="cuda"):
        self.w, self.q = w, w.q.to(device)
        self.priv, self.pub = w.priv.to(device), w.pub.to(device)
        self.shape = spd.make_shape(len(w.counts), w.num_q_heads, w.num_kv_heads, w.head_dim, w.dtype, w.sm_scale)
        self.slopes = slopes_of(w.num_q_heads) if alibi else None
        self.score = spd.make_score(cap, window, None if self.slopes is None else self.slopes.to(device))
        self.ws = spd.alloc_drafted_workspace(self.shape, device)
        self.drafts = dict(tok_indptr=w.indptr.to(device), parents=None if w.parents is None else w.parents.to(device), sinks=sinks)
        self.T = w.q.shape[0]

    def out(self, dtype=torch.float32):
        return torch.full((self.T, self.w.num_q_heads, self.w.head_dim), float("nan"), dtype=dtype, device=self.q.device)

    def partial(self):
        hq, d = self.w.num_q_heads, self.w.head_dim
        return tuple(torch.full((self.T, hq) + x, float("nan"), device=self.q.device) for x in ((d,), (), ()))

    def fused(self, dtype=torch.float32, out=None):
        out = self.out(dtype) if out is None else out
        spd.spd_decode_step_drafted(self.shape, self.score, self.q, self.priv, self.pub, out, self.ws, **self.drafts)
        return out

    def halves(self, dtype=torch.float32):
        part, out = self.partial(), self.out(dtype)
        spd.spd_partial_attn_drafted(self.shape, self.score, self.q, self.priv, self.pub.seq_lens, part, self.ws, **self.drafts)
        spd.spd_service_attn_merge_drafted(self.shape, self.score, self.q, self.pub, self.priv.seq_lens, part, out, self.ws, **self.drafts)
        return out, part


def expected(w, cap=0.0, window=0, sinks=0, slopes=None, parts=(True, True), rows=None):
    """(out, O, m, l, tol) in 64 bits: rows [T, Hq(, D)].  rows: only these rows of q (others stay 0)."""
    T, Hq, D = w.q.shape
    g = Hq // w.num_kv_heads
    out, O = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
    m, l, tol = torch.full((T, Hq), -math.inf, dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64)
    weight = 0.0 if w.dtype == torch.float32 else 2.0 ** -8
    t0 = 0
    for u, tree in enumerate(w.trees):
        n, lp, lq = len(tree), int(w.priv.seq_lens[u]), int(w.pub.seq_lens[u])
        ctx = lp + lq - n
        depth, line = np.zeros(n, dtype=np.int64), np.zeros((n, n), dtype=bool)
        for i, p in enumerate(tree):
            if p >= 0:
                depth[i], line[i] = depth[p] + 1, line[p]
            line[i, i] = True
        where = torch.cat([torch.arange(ctx), ctx + torch.from_numpy(depth)])
        here = torch.cat([torch.full((lp,), parts[0]), torch.full((lq,), parts[1])])
        kv = []
        for h in range(w.num_kv_heads):
            a = [wl.gather_dense(x, u, h) if c else (torch.zeros((0, D), dtype=w.dtype),) * 2 for x, c in ((w.priv, lp), (w.pub, lq))]
            kv.append((torch.cat([a[0][0], a[1][0]]), torch.cat([a[0][1], a[1][1]])))
        for i in range(n):
            if rows is not None and t0 + i not in rows:
                continue
            pos = ctx + int(depth[i])
            far = pos - where
            seen = here & torch.cat([torch.ones(ctx, dtype=torch.bool), torch.from_numpy(line[i])])
            if window:
                seen = seen & ((far < window) | (where < sinks))
            for h in range(Hq):
                k, v = kv[h // g]
                sl = float(slopes[h]) if slopes is not None else 0.0
                out[t0 + i, h], O[t0 + i, h], m[t0 + i, h], l[t0 + i, h], S = ref.attend(w.q[t0 + i, h], k, v, seen, w.sm_scale, cap, sl, far.double())
                if bool(seen.any()):
                    tol[t0 + i, h] = ref.bound(float(v[seen].abs().max()), D, S, int(seen.sum()), cap, abs(sl) * float(far[seen].abs().max()), weight)
        t0 += n
    return out, O, m, l, tol


def close(got, want, tol, what=""):
    err = (got.cpu().double() - want).abs()
    lim = tol[..., None] + (ref.half_step(got.dtype) * want.abs() if got.dtype != torch.float32 else 2.0 ** -24 * want.abs())
    assert bool((err <= lim).all()), (what, float(err.max()), float((err - lim).max()))
