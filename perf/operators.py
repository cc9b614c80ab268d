"""Timed cases of the operators that give the partitioned cache its positions and score shapes.

  append : `spd_append_kv_rope`      rotation of q and k by position, k and v rows into the paged cache
  decode : `spd_decode_step_scored`  one token per user over both partitions; capped scores, distance bias, window
  prefill: `spd_prefill_attn_scored` prompts; the same scores, and window, prefix and document masks

`run` computes a case with elementary torch operations in 32 bits (angles in 64), or with the library's calls where `own` is true.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_workspaces = {}      # one workspace per shape, as a serving process keeps it


def listed():
    return [
        # --- append: one new token per user of a small batch (paper-scale layer), the smallest call
        dict(name="append_token_8", op="append", batch=8, hq=32, hkv=8, d=128, dtype="bf16", run_lo=1, run_hi=1, held_lo=1, held_hi=128,
             rot=128, inter=False, axes=1, len_seed=1),
        # one new token per user of the many-user service batch
        dict(name="append_token_512", op="append", batch=512, hq=64, hkv=8, d=128, dtype="bf16", run_lo=1, run_hi=1, held_lo=0, held_hi=2048,
             rot=128, inter=False, axes=1, len_seed=2),
        # image prompts: three position axes, neighbouring channels paired, half of the channels rotated, fp32
        dict(name="append_image_prompts", op="append", batch=5, hq=8, hkv=8, d=64, dtype="f32", run_lo=37, run_hi=700, held_lo=0, held_hi=50,
             rot=32, inter=True, axes=3, len_seed=3),
        # hand-over of eight long prompts
        dict(name="append_long_prompts", op="append", batch=8, hq=32, hkv=8, d=128, dtype="bf16", run_lo=2048, run_hi=8192, held_lo=0, held_hi=0,
             rot=128, inter=False, axes=1, len_seed=4),
        # --- decode: the tiny fp32 configuration, distance bias and capped scores
        dict(name="decode_tiny_f32", op="decode", batch=4, hq=8, hkv=8, d=64, dtype="f32", in_lo=256, in_hi=256, out_lo=32, out_hi=32,
             cap=30.0, alibi=True, window=0, len_seed=5),
        # a handful of users with long prompts read through a sliding window: latency
        dict(name="decode_window_8", op="decode", batch=8, hq=32, hkv=8, d=128, dtype="bf16", in_lo=4096, in_hi=32768, out_lo=1, out_hi=256,
             cap=0.0, alibi=False, window=1024, len_seed=6),
        # the grouped-query service batch with capped scores
        dict(name="decode_cap_128", op="decode", batch=128, hq=32, hkv=8, d=128, dtype="bf16", in_lo=2048, in_hi=8192, out_lo=1, out_hi=1024,
             cap=50.0, alibi=False, window=0, len_seed=7),
        # few users, very long prompts, distance bias: each sequence split over many SMs and joined
        dict(name="decode_alibi_long", op="decode", batch=8, hq=32, hkv=8, d=128, dtype="bf16", in_lo=32768, in_hi=131072, out_lo=1, out_hi=256,
             cap=0.0, alibi=True, window=0, len_seed=8),
        # --- prefill: the tiny fp32 configuration's prompts, capped scores and distance bias
        dict(name="prefill_tiny_f32", op="prefill", batch=4, hq=8, hkv=8, d=64, dtype="f32", lo=256, hi=256, cap=30.0, alibi=True, window=0,
             prefix=False, docs=False, len_seed=9),
        # many ragged prompts made of packed documents, distance bias
        dict(name="prefill_docs_ragged", op="prefill", batch=24, hq=16, hkv=4, d=64, dtype="bf16", lo=33, hi=1000, cap=0.0, alibi=True, window=0,
             prefix=False, docs=True, len_seed=10),
        # prompts with a bidirectional prefix and a sliding window
        dict(name="prefill_prefix_window", op="prefill", batch=3, hq=32, hkv=8, d=128, dtype="bf16", lo=1500, hi=4097, cap=0.0, alibi=False,
             window=1000, prefix=True, docs=False, len_seed=11),
        # one long prompt with capped scores
        dict(name="prefill_cap_long", op="prefill", batch=1, hq=32, hkv=8, d=128, dtype="bf16", lo=8192, hi=8192, cap=50.0, alibi=False, window=0,
             prefix=False, docs=False, len_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "prefill"])
    f32 = rng.random() < 0.2
    d = rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 8])
    case = dict(op=op, hq=hkv * group, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", len_seed=rng.randrange(1 << 20))
    if op == "append":
        axes = rng.choice([1, 1, 3])
        ragged = rng.random() < 0.5
        case.update(batch=_log_int(rng, 1, 24 if ragged else 400), run_lo=1, run_hi=_log_int(rng, 2, 4000) if ragged else 1,
                    held_lo=0, held_hi=_log_int(rng, 1, 300), rot=rng.choice([d, d, 32]), inter=rng.random() < 0.3, axes=axes)
    elif op == "decode":
        case.update(batch=_log_int(rng, 1, 96))
        longest = _log_int(rng, 16, 16000000 // (case["batch"] * hkv * max(1, group // 2)) + 32)
        longest = min(longest, 60000)
        case.update(in_lo=rng.choice([0, longest // 4]), in_hi=longest, out_lo=0, out_hi=_log_int(rng, 1, 600),
                    cap=rng.choice([0.0, 20.0, 50.0]), alibi=rng.random() < 0.4, window=rng.choice([0, 0, _log_int(rng, 1, 5000)]))
    else:
        if f32:
            case.update(hq=min(16, hkv * group))
            case["hkv"] = min(case["hkv"], case["hq"])
        hi = _log_int(rng, 2, 1500 if f32 else 6000)
        batch = max(1, min(32, _log_int(rng, 1, 1 + 1200000000 // (hi * hi * case["hq"]))))
        case.update(batch=batch, lo=rng.choice([1, hi // 2 + 1]), hi=hi, cap=rng.choice([0.0, 20.0, 50.0]), alibi=rng.random() < 0.3,
                    window=rng.choice([0, 0, _log_int(rng, 1, 2000)]), prefix=rng.random() < 0.3, docs=rng.random() < 0.3)
    return case


# ---------------------------------------------------------------------------------------------------------------------
# sizes that follow from the case alone
def _lengths(case):
    rng = np.random.default_rng(case["len_seed"])
    B = case["batch"]
    if case["op"] == "append":
        return rng.integers(case["run_lo"], case["run_hi"] + 1, B), rng.integers(case["held_lo"], case["held_hi"] + 1, B)
    if case["op"] == "decode":
        lp, lo = rng.integers(case["in_lo"], case["in_hi"] + 1, B), rng.integers(case["out_lo"], case["out_hi"] + 1, B)
        return lp, np.where(lp + lo == 0, 1, lo)      # a query's own token is always cached
    return (rng.integers(case["lo"], case["hi"] + 1, B),)


def _intervals(case):
    """Per row of the packed prompts: document start (within the prompt), prefix length of its prompt, first and last visible key."""
    (lens,) = _lengths(case)
    rng = np.random.default_rng([case["len_seed"], 7])
    los, his, docs, prefs = [], [], [], []
    for n in lens:
        i = np.arange(n)
        start = np.zeros(n, dtype=np.int64)
        if case["docs"]:                               # documents of 1 to about 300 tokens, packed one after another
            cuts = np.cumsum(rng.integers(1, 300, n + 1))
            cuts = np.concatenate([[0], cuts[cuts < n]])
            start = cuts[np.searchsorted(cuts, i, side="right") - 1]
        pre = int(rng.integers(0, n + 1)) // 2 if case["prefix"] else 0
        lo = np.maximum(start, i - case["window"] + 1) if case["window"] else start
        los.append(np.maximum(lo, 0)); his.append(np.where(i < pre, pre - 1, i))
        docs.append(start); prefs.append(pre)
    cat = lambda v: np.concatenate(v).astype(np.int64)  # noqa: E731
    return lens, cat(los), cat(his), cat(docs), np.array(prefs, dtype=np.int64)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d, B = case["hq"], case["hkv"], case["d"], case["batch"]
    if case["op"] == "append":
        T = int(_lengths(case)[0].sum())
        # q, k, v read; q, the packed k, and the cache rows of k and v written
        return {"bytes": T * d * es * ((hq + 2 * hkv) + (hq + hkv) + 2 * hkv), "flops": T * (hq + hkv) * case["rot"] * 3}
    if case["op"] == "decode":
        lp, lo = _lengths(case)
        n = int(np.minimum(lp + lo, case["window"] or (1 << 60)).sum())
        return {"bytes": n * 2 * hkv * d * es + B * hq * d * 2 * es, "flops": 4 * d * hq * n}
    lens, lo, hi, _, _ = _intervals(case)
    T = int(lens.sum())
    return {"bytes": T * d * es * (2 * hq + 2 * hkv), "flops": 4 * d * hq * int(np.maximum(hi - lo + 1, 0).sum())}


# ---------------------------------------------------------------------------------------------------------------------
class _Part:
    """One paged partition: pools [pages, hkv, 16, d], tables and lengths on the device."""


def _part(lens, room, hkv, d, dtype, rng, gen, dev):
    p = _Part()
    need = np.maximum(-(-np.asarray(room) // PAGE), 1)
    indptr = np.concatenate([[0], np.cumsum(need)])
    pages = int(indptr[-1]) + 3
    p.k_pool = torch.randn((pages, hkv, PAGE, d), generator=gen, device=dev, dtype=torch.float32).to(dtype)
    p.v_pool = torch.randn((pages, hkv, PAGE, d), generator=gen, device=dev, dtype=torch.float32).to(dtype)
    p.page_indptr = torch.from_numpy(indptr.astype(np.int32)).to(dev)
    p.page_indices = torch.from_numpy(rng.permutation(pages)[:int(indptr[-1])].astype(np.int32)).to(dev)
    p.seq_lens = torch.from_numpy(np.asarray(lens).astype(np.int32)).to(dev)
    return p


def _randn(shape, dtype, gen, dev, scale=1.0):
    return (torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng([seed, 1])
    dtype, B, hq, hkv, d = DTYPES[case["dtype"]], case["batch"], case["hq"], case["hkv"], case["d"]
    st = dict(case=case, dev=dev)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(dev)  # noqa: E731
    if case["op"] == "append":
        runs, held = _lengths(case)
        T = int(runs.sum())
        pairs, axes = case["rot"] // 2, case["axes"]
        st["part"] = _part(held, held + runs, hkv, d, dtype, rng, gen, dev)
        st["new_lens"] = torch.zeros(B, dtype=torch.int32, device=dev)
        st["q"] = _randn((T, hq, d), dtype, gen, dev)
        st["k"] = _randn((T, hkv, d), dtype, gen, dev)
        st["v"] = _randn((T, hkv, d), dtype, gen, dev)
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
        st["indptr"] = i32(np.concatenate([[0], np.cumsum(runs)]))
        st["inv_freq"] = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().to(dev)
        first = rng.integers(0, 100000, B)                                     # tokens of the other partition in front of this one
        st["pos_base"] = i32(first)
        st["sections"], st["positions"] = None, None
        if axes == 3:                                                          # time, height and width of a patch
            st["sections"] = (pairs - 2 * (pairs // 3), pairs // 3, pairs // 3)
            t = np.arange(T)
            st["positions"] = i32(np.stack([t // 400 + 3, t // 20 % 20, t % 20]))
        st["axis"] = torch.from_numpy(np.repeat(np.arange(3), st["sections"] or (pairs, 0, 0))).to(dev)
        st["user"] = torch.from_numpy(np.repeat(np.arange(B), runs)).to(dev)
        st["one"] = case["run_hi"] == 1
    elif case["op"] == "decode":
        lp, lo = _lengths(case)
        st["q"] = _randn((B, hq, d), dtype, gen, dev, 4.0 if case["cap"] else 1.0)    # scores that reach into the cap
        st["priv"] = _part(lp, lp, hkv, d, dtype, rng, gen, dev)
        st["pub"] = _part(lo, lo, hkv, d, dtype, rng, gen, dev)
        first = np.maximum(lp + lo - (case["window"] or (1 << 60)), 0)
        st["spans"] = int(np.maximum(lp - first, 0).max()), int((lo - np.maximum(first - lp, 0)).max())
        st["out"] = torch.empty((B, hq, d), dtype=dtype, device=dev)
    else:
        lens, _, _, docs, prefs = _intervals(case)
        T = int(lens.sum())
        st["q"] = _randn((T, hq, d), dtype, gen, dev, 4.0 if case["cap"] else 1.0)
        st["k"] = _randn((T, hkv, d), dtype, gen, dev)
        st["v"] = _randn((T, hkv, d), dtype, gen, dev)
        st["indptr"] = i32(np.concatenate([[0], np.cumsum(lens)]))
        st["doc_start"] = i32(docs) if case["docs"] else None
        st["prefix"] = i32(prefs) if case["prefix"] else None
        st["longest"] = int(lens.max())
        st["out"] = torch.empty((T, hq, d), dtype=dtype, device=dev)
    if case["op"] != "append":
        st["slopes"] = (2.0 ** (-8.0 * torch.arange(1, hq + 1, dtype=torch.float64) / hq)).float().to(dev) if case["alibi"] else None
    return st


# ---------------------------------------------------------------------------------------------------------------------
def _append_plain(st):
    case, part = st["case"], st["part"]
    pairs, T = case["rot"] // 2, st["q"].shape[0]
    user = st["user"]
    slot = part.seq_lens.long()[user] + torch.arange(T, device=st["dev"]) - st["indptr"].long()[user]      # position within the partition
    pos = st["positions"].double()[st["axis"]].T if st["positions"] is not None else (st["pos_base"].long()[user] + slot).double()[:, None]
    angle = pos * st["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def rotate(x):
        y = x.float()
        if case["inter"]:
            a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = y[..., :pairs], y[..., pairs:2 * pairs]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        return torch.cat([turned, y[..., 2 * pairs:]], dim=-1).to(x.dtype)

    q, k = rotate(st["q"]), rotate(st["k"])
    page = part.page_indices.long()[part.page_indptr.long()[user] + slot // PAGE]
    part.k_pool[page, :, slot % PAGE] = k
    part.v_pool[page, :, slot % PAGE] = st["v"]
    lens = part.seq_lens + st["indptr"][1:] - st["indptr"][:-1]
    return {"q": q, "k": k, "k_pool": part.k_pool, "v_pool": part.v_pool, "lens": lens}


def _visible(part, first, span):
    """K and V rows [first, len) of every user, padded to `span` rows in 32 bits, and which of them are there."""
    at = first[:, None] + torch.arange(span, device=first.device)
    there = at < part.seq_lens.long()[:, None]
    where = (part.page_indptr.long()[:-1, None] + at // PAGE).clamp(max=max(part.page_indices.numel() - 1, 0))
    page = part.page_indices.long()[where]
    rows = lambda pool: torch.where(there[:, :, None, None], pool[page, :, at % PAGE].float(), 0.0)  # noqa: E731
    return rows(part.k_pool), rows(part.v_pool), at, there


def _decode_plain(st):
    case = st["case"]
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    lp, lo = st["priv"].seq_lens.long(), st["pub"].seq_lens.long()
    last = lp + lo - 1
    first = (last + 1 - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(lp)
    k1, v1, at1, there1 = _visible(st["priv"], torch.minimum(first, lp), st["spans"][0])
    k2, v2, at2, there2 = _visible(st["pub"], (first - lp).clamp(min=0), st["spans"][1])
    k, v, there = torch.cat([k1, k2], 1), torch.cat([v1, v2], 1), torch.cat([there1, there2], 1)
    dist = last[:, None] - torch.cat([at1, at2 + lp[:, None]], 1)
    q = st["q"].float().view(B, hkv, hq // hkv, d)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    if st["slopes"] is not None:
        s = s - st["slopes"].view(1, hkv, hq // hkv, 1) * dist[:, None, None, :].float()
    s = s.masked_fill(~there[:, None, None, :], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p, v.transpose(1, 2)) / p.sum(-1, keepdim=True)
    return o.reshape(B, hq, d).to(st["q"].dtype)


def _prefill_plain(st):
    case = st["case"]
    B, hq, hkv, d, n = case["batch"], case["hq"], case["hkv"], case["d"], st["longest"]
    start, T = st["indptr"].long(), st["q"].shape[0]
    lens = start[1:] - start[:-1]
    i = torch.arange(n, device=st["dev"])
    row = (start[:-1, None] + i).clamp(max=T - 1)                              # packed row of token i of each prompt, padded
    q = st["q"].float()[row].view(B, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)
    k = st["k"].float()[row].permute(0, 2, 3, 1)[:, :, None]
    v = st["v"].float()[row].permute(0, 2, 1, 3)[:, :, None]
    lo = st["doc_start"].long()[row] if st["doc_start"] is not None else torch.zeros_like(row)
    if case["window"]:
        lo = torch.maximum(lo, i - case["window"] + 1)
    hi = i.expand(B, n)
    if st["prefix"] is not None:
        pre = torch.minimum(st["prefix"].long(), lens)[:, None]
        hi = torch.where(i < pre, pre - 1, hi)
    seen = (i >= lo[:, :, None]) & (i <= hi[:, :, None]) & (i < lens[:, None, None])     # [B, row, key]
    s = torch.matmul(q, k).mul_(1.0 / math.sqrt(d))
    if case["cap"]:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    if st["slopes"] is not None:
        s -= st["slopes"].view(hkv, hq // hkv, 1, 1) * (i[:, None] - i).abs().float()
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    user = torch.searchsorted(start[1:], torch.arange(T, device=st["dev"]), right=True)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)[user, torch.arange(T, device=st["dev"]) - start[user]].to(st["q"].dtype)


# ---------------------------------------------------------------------------------------------------------------------
def _shape(st, spd):
    case = st["case"]
    dtype = DTYPES[case["dtype"]]
    key = (case["batch"], case["hq"], case["hkv"], case["d"], dtype)
    if key not in _workspaces:
        shape = spd.make_shape(*key, 1.0 / math.sqrt(case["d"]))
        _workspaces[key] = shape, spd.alloc_workspace(shape)
    return _workspaces[key]


def _run_own(st):
    from paper_2409_19134_b200 import binding as spd
    case = st["case"]
    shape, ws = _shape(st, spd)
    if case["op"] == "append":
        rope = spd.make_rope(st["inv_freq"], interleaved=case["inter"], sections=st["sections"])
        spd.spd_append_kv_rope(shape, rope, st["q"], st["k"], st["v"], st["part"], ws, q_out=st["q_out"], k_out=st["k_out"],
                               tok_indptr=None if st["one"] else st["indptr"], positions=st["positions"],
                               pos_base=None if st["positions"] is not None else st["pos_base"], new_lens=st["new_lens"])
        return {"q": st["q_out"], "k": st["k_out"], "k_pool": st["part"].k_pool, "v_pool": st["part"].v_pool, "lens": st["new_lens"]}
    score = spd.make_score(logit_cap=case["cap"], window=case["window"], alibi_slopes=st["slopes"])
    if case["op"] == "decode":
        spd.spd_decode_step_scored(shape, score, st["q"], st["priv"], st["pub"], st["out"], ws)
    else:
        spd.spd_prefill_attn_scored(shape, score, st["q"], st["k"], st["v"], st["indptr"], st["out"], ws, prefix_lens=st["prefix"],
                                    doc_start=st["doc_start"])
    return st["out"]


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append_plain, "decode": _decode_plain, "prefill": _prefill_plain}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
def _exact_append(st):
    case, part = st["case"], st["part"]
    runs, held = _lengths(case)
    pairs, inter = case["rot"] // 2, case["inter"]
    q, k, v = (st[n].double() for n in ("q", "k", "v"))
    kp, vp = part.k_pool.double(), part.v_pool.double()
    a_at = torch.arange(pairs, device=st["dev"]) * (2 if inter else 1)
    b_at = a_at + (1 if inter else pairs)
    axis_of = [0] * pairs if st["sections"] is None else sum(([a] * n for a, n in enumerate(st["sections"])), [])
    done = 0
    for u in range(case["batch"]):
        n, h = int(runs[u]), int(held[u])
        if st["positions"] is None:
            pos = (int(st["pos_base"][u]) + h + torch.arange(n, device=st["dev"], dtype=torch.float64))[:, None].expand(n, pairs)
        else:
            pos = torch.stack([st["positions"][a, done:done + n].double() for a in axis_of], 1)
        turn = torch.polar(torch.ones_like(pos), pos * st["inv_freq"].double())[:, None, :]
        for x in (q, k):
            y = x[done:done + n]
            z = torch.complex(y[..., a_at], y[..., b_at]) * turn
            y[..., a_at], y[..., b_at] = z.real, z.imag
        lo = int(part.page_indptr[u])
        at = h + torch.arange(n, device=st["dev"])
        pages = part.page_indices[lo + at // PAGE].long()
        kp[pages, :, at % PAGE], vp[pages, :, at % PAGE] = k[done:done + n], v[done:done + n]
        done += n
    return {"q": q, "k": k, "k_pool": kp, "v_pool": vp, "lens": None}


def _exact_scores(q, k, dist, case, slopes):
    s = (q @ k.T) / math.sqrt(case["d"])
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    return s if slopes is None else s - slopes * dist


def _exact_decode(st):
    case = st["case"]
    lp, lo = _lengths(case)
    g = case["hq"] // case["hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["dev"])
    for u in range(case["batch"]):
        n = int(lp[u] + lo[u])
        rows = [[], []]
        for part, m in ((st["priv"], int(lp[u])), (st["pub"], int(lo[u]))):
            a, b = int(part.page_indptr[u]), int(part.page_indptr[u + 1])
            pages = part.page_indices[a:b].long()
            for r, pool in zip(rows, (part.k_pool, part.v_pool)):
                r.append(pool[pages].transpose(0, 1).reshape(case["hkv"], -1, case["d"])[:, :m])
        k, v = (torch.cat(r, 1) for r in rows)
        f = max(0, n - case["window"]) if case["window"] else 0
        dist = n - 1 - torch.arange(f, n, device=st["dev"], dtype=torch.float64)
        for h in range(case["hkv"]):
            sl = None if st["slopes"] is None else st["slopes"][h * g:(h + 1) * g, None].double()
            s = _exact_scores(st["q"][u, h * g:(h + 1) * g].double(), k[h, f:].double(), dist, case, sl)
            out[u, h * g:(h + 1) * g] = torch.softmax(s, -1) @ v[h, f:].double()
    return out


def _exact_prefill(st):
    case = st["case"]
    lens, lo, hi, _, _ = _intervals(case)
    g = case["hq"] // case["hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["dev"])
    lo, hi = torch.from_numpy(lo).to(st["dev"]), torch.from_numpy(hi).to(st["dev"])
    t = 0
    for n in (int(x) for x in lens):
        j = torch.arange(n, device=st["dev"])
        for a in range(0, n, 2048):
            b = min(n, a + 2048)
            hidden = (j < lo[t + a:t + b, None]) | (j > hi[t + a:t + b, None])
            dist = (j[a:b, None] - j).abs().double()
            for h in range(case["hq"]):
                sl = None if st["slopes"] is None else st["slopes"][h].double()
                s = _exact_scores(st["q"][t + a:t + b, h].double(), st["k"][t:t + n, h // g].double(), dist, case, sl)
                s = s.masked_fill(hidden, -math.inf)
                out[t + a:t + b, h] = torch.nan_to_num(torch.softmax(s, -1)) @ st["v"][t:t + n, h // g].double()
        t += n
    return out


def exact(case, seed):
    return {"append": _exact_append, "decode": _exact_decode, "prefill": _exact_prefill}[case["op"]](prepare(case, seed))
