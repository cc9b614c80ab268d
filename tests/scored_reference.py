"""Plain 64-bit forms of the scored calls (capped scores, distance bias, window and interval masks) and of the append with
rotation, with the error bounds that the tests use.  Test-side only: nothing here runs on the library's path.

Error bounds.  An output is sum_j p_j v_j / sum_j p_j; a relative error of at most e on every weight p_j moves it by at most
2 e max|v|.  A weight's relative error is the absolute error of its score (exp' = exp) plus what its own evaluation costs:
  score   D 2^-24 S          D products summed in fp32, S = scale * sum_d |q_d k_d|
          2^-21 cap          the cap's special-function steps (relative to the cap; cap_error in its place where a test knows better)
          2^-23 slope dist   product and sum of the distance bias
  weight  2^-21              exponential (2 ulp) and the change of the running maximum
Rounding the weights to bf16 for the product with V touches the numerator alone and counts once: 2^-8 (prompt attention on the
tensor cores), or 2^-16 where a bf16 head and a remainder are used (decode on the tensor cores).
The sums over n keys add n 2^-24 at most, and an output rounded to a type half a step of it, eps / 2.
"""
import math

import torch


def bound(vmax, D, S, n, cap=0.0, bias=0.0, weight=0.0):
    e = D * 2.0 ** -24 * S + 2.0 ** -21 * cap + 2.0 ** -23 * bias + 2.0 ** -21 + n * 2.0 ** -24
    return (2.0 * e + weight) * vmax


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def scores(q, k, scale, cap, slope, dist):
    """q [D], k [n, D] in float64."""
    s = scale * (k @ q)
    if cap:
        s = cap * torch.tanh(s / cap)
    return s - slope * dist


def attend(q, k, v, seen, scale, cap=0.0, slope=0.0, dist=None):
    """One row in 64 bits -> (output, unnormalised O, m, l, S).  Hidden keys are left out, so what they hold is irrelevant."""
    D = q.shape[0]
    k, v = k[seen].double(), v[seen].double()
    q = q.double()
    if k.shape[0] == 0:
        z = torch.zeros(D, dtype=torch.float64)
        return z, z, -math.inf, 0.0, 0.0
    d = torch.zeros(k.shape[0], dtype=torch.float64) if dist is None else dist[seen].double()
    s = scores(q, k, scale, cap, slope, d)
    m = float(s.max())
    p = torch.exp(s - m)
    O, l = p @ v, float(p.sum())
    return O / l, O, m, l, float(scale * (k.abs() @ q.abs()).max())


def decode(w, cap=0.0, window=0, slopes=None, parts=(True, True), cap_error=None):
    """Every user and head of a workload (CPU tensors): (out, O, m, l, tol) over the partitions in `parts`, positions counted over both."""
    from paper_2409_19134_b200 import workloads as wl
    B, Hq, Hkv, D = w.batch, w.num_q_heads, w.num_kv_heads, w.head_dim
    g = Hq // Hkv
    out, O = torch.zeros((B, Hq, D), dtype=torch.float64), torch.zeros((B, Hq, D), dtype=torch.float64)
    m, l, tol = (torch.zeros((B, Hq), dtype=torch.float64) for _ in range(3))
    for u in range(B):
        na, nb = int(w.priv.seq_lens[u]), int(w.pub.seq_lens[u])
        n = na + nb
        pos = torch.cat([torch.arange(na) if parts[0] else torch.arange(0), torch.arange(na, n) if parts[1] else torch.arange(0)])
        dist = (n - 1 - pos).double()
        seen = dist < window if window else torch.ones_like(dist, dtype=torch.bool)
        for h in range(Hkv):
            kv = [wl.gather_dense(p, u, h) for p, c, on in zip((w.priv, w.pub), (na, nb), parts) if on and c]
            none = torch.zeros((0, D), dtype=w.dtype)
            k, v = torch.cat([x[0] for x in kv] or [none]), torch.cat([x[1] for x in kv] or [none])
            vmax = float(v[seen].abs().max()) if bool(seen.any()) else 0.0
            for j in range(h * g, (h + 1) * g):
                sl = float(slopes[j]) if slopes is not None else 0.0
                out[u, j], O[u, j], m[u, j], l[u, j], S = attend(w.q[u, j], k, v, seen, w.sm_scale, cap, sl, dist)
                bias = abs(sl) * float(dist[seen].max()) if bool(seen.any()) else 0.0
                tol[u, j] = bound(vmax, D, S, int(seen.sum()), cap if cap_error is None else cap_error, bias, 0.0 if w.dtype == torch.float32 else 2.0 ** -16)
    return out, O, m, l, tol


def intervals(n, window=0, prefix=0, doc=None):
    """First and last key that each of n rows sees."""
    i = torch.arange(n)
    lo = torch.zeros(n, dtype=torch.int64) if doc is None else doc.long().clamp(min=0)
    if window:
        lo = torch.maximum(lo, i - window + 1)
    lo = lo.clamp(min=0)
    prefix = min(prefix, n)
    return lo, torch.where(i < prefix, torch.full_like(i, prefix - 1), i)


def prefill(q, k, v, lens, scale, cap=0.0, window=0, slopes=None, prefix=None, doc=None, weight=0.0, rows=None, cap_error=None):
    """Packed prompts on the CPU -> (out [T,Hq,D], tol [T,Hq]) in float64; rows: only these packed rows (others stay 0)."""
    T, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, tol = torch.zeros((T, Hq, D), dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64)
    t0 = 0
    for u, n in enumerate(lens):
        lo, hi = intervals(n, window, int(prefix[u]) if prefix is not None else 0, None if doc is None else doc[t0:t0 + n])
        j = torch.arange(n)
        for i in range(n):
            if rows is not None and t0 + i not in rows:
                continue
            seen = (j >= lo[i]) & (j <= hi[i])
            dist = (i - j).abs().double()
            for h in range(Hq):
                sl = float(slopes[h]) if slopes is not None else 0.0
                kk, vv = k[t0:t0 + n, h // g], v[t0:t0 + n, h // g]
                out[t0 + i, h], _, _, _, S = attend(q[t0 + i, h], kk, vv, seen, scale, cap, sl, dist)
                if bool(seen.any()):
                    tol[t0 + i, h] = bound(float(vv[seen].abs().max()), D, S, int(seen.sum()), cap if cap_error is None else cap_error, abs(sl) * float(dist[seen].max()), weight)
        t0 += n
    return out, tol


def rotate(x, pos, inv_freq, interleaved, scale=1.0):
    """x [T,H,D], pos [T, pairs] in float64."""
    y = x.double().clone()
    n = inv_freq.numel()
    a = torch.arange(n) * (2 if interleaved else 1)
    b = a + (1 if interleaved else n)
    ang = (pos * inv_freq.double())[:, None, :]
    c, s = ang.cos() * scale, ang.sin() * scale
    xa, xb = x[..., a].double(), x[..., b].double()
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    return y


def rotate_bound(x, inv_freq, interleaved, dtype, ref, scale=1.0):
    """Half a step of the output type, plus three fp32 roundings (product, fused product and sum, sine and cosine with their angle:
    4 ulp together with the angle's 2^-24 turns = 2 pi 2^-24) on the pair's magnitude."""
    n = inv_freq.numel()
    a = torch.arange(n) * (2 if interleaved else 1)
    b = a + (1 if interleaved else n)
    mag = torch.zeros_like(ref)
    pair = (x[..., a].double().abs() + x[..., b].double().abs()) * abs(scale)
    mag[..., a], mag[..., b] = pair, pair
    return half_step(dtype) * ref.abs() + mag * 14 * 2.0 ** -24
