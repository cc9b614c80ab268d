"""Timed cases of the calls that draft several tokens ahead over the partitioned cache and of those that hand its pages round.

  attend: `spd_decode_step_drafted`  trees or runs of drafted tokens over both partitions (also in the protocol's two halves:
          `spd_partial_attn_drafted`, `spd_service_attn_merge_drafted`); capped scores, distance bias, window with sinks
  keep  : `spd_keep_drafted`         accepted branches moved to the front of the drafted rows in every layer's pools
  fork  : `spd_pages_release`, `spd_pages_fork`, `spd_pages_copy`   samples that start from one prompt's pages
  turn  : `spd_pages_release`, `spd_pages_take`                     users that leave, users that come and tokens to come

`run` computes a case with elementary torch operations in 32 bits, or with the library's calls where `own` is true.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NOTHING = 1 << 30     # a first token behind all others: nothing of the slot is meant
_workspaces = {}      # one workspace per shape, as a serving process keeps it


def listed():
    return [
        # --- attend: the tiny fp32 configuration, small trees, capped scores and distance bias: the smallest call
        dict(name="tree_tiny_f32", op="attend", batch=4, hq=8, hkv=8, d=64, dtype="f32", n_lo=12, n_hi=12, tree=True, in_lo=256, in_hi=256,
             out_lo=1, out_hi=32, cap=30.0, alibi=True, window=0, sinks=0, halves=False, len_seed=1),
        # a paper-scale layer, ragged trees, computed in the protocol's two halves
        dict(name="tree_small_halves", op="attend", batch=8, hq=32, hkv=8, d=128, dtype="bf16", n_lo=5, n_hi=16, tree=True, in_lo=300, in_hi=700,
             out_lo=1, out_hi=128, cap=0.0, alibi=False, window=0, sinks=0, halves=True, len_seed=2),
        # the service batch with a tree of drafted tokens for each user
        dict(name="tree_many", op="attend", batch=64, hq=32, hkv=8, d=128, dtype="bf16", n_lo=26, n_hi=26, tree=True, in_lo=1024, in_hi=8192,
             out_lo=1, out_hi=1024, cap=0.0, alibi=False, window=0, sinks=0, halves=False, len_seed=3),
        # few users, long prompts, wide trees: rows fill the tensor cores
        dict(name="tree_long", op="attend", batch=4, hq=32, hkv=8, d=128, dtype="bf16", n_lo=64, n_hi=64, tree=True, in_lo=32768, in_hi=80000,
             out_lo=1, out_hi=256, cap=0.0, alibi=False, window=0, sinks=0, halves=False, len_seed=4),
        # one token per user through a window behind four sinks
        dict(name="token_sinks", op="attend", batch=64, hq=32, hkv=8, d=128, dtype="bf16", n_lo=1, n_hi=1, tree=False, in_lo=4096, in_hi=12288,
             out_lo=1, out_hi=512, cap=0.0, alibi=False, window=2048, sinks=4, halves=False, len_seed=5),
        # a part of two prompts behind what the cache holds, window and sinks, capped scores
        dict(name="run_sinks", op="attend", batch=2, hq=32, hkv=8, d=128, dtype="bf16", n_lo=1500, n_hi=2100, tree=False, in_lo=700, in_hi=5000,
             out_lo=0, out_hi=0, cap=50.0, alibi=False, window=1500, sinks=16, halves=False, len_seed=6),
        # --- keep: a handful of users, two layers
        dict(name="keep_small", op="keep", batch=8, hkv=8, d=128, dtype="bf16", n_lo=5, n_hi=16, tree=True, held_lo=1, held_hi=500, layers=2,
             len_seed=7),
        # every user of the many-user batch, trees of 64 tokens, sixteen layers
        dict(name="keep_many", op="keep", batch=512, hkv=8, d=128, dtype="bf16", n_lo=33, n_hi=64, tree=True, held_lo=0, held_hi=300, layers=16,
             len_seed=8),
        # --- fork: seven more samples of one prompt, two layers
        dict(name="fork_few", op="fork", prompts=1, samples=7, hkv=8, d=128, dtype="bf16", lo=500, hi=500, layers=2, spare=60, len_seed=9),
        # four beams for each of 96 prompts, eight layers
        dict(name="fork_many", op="fork", prompts=96, samples=384, hkv=8, d=128, dtype="bf16", lo=64, hi=1500, layers=8, spare=2000, len_seed=10),
        # --- turn: one user of eight leaves, another one comes
        dict(name="turn_few", op="turn", batch=8, gone=1, lo=100, hi=900, spare=200, len_seed=11),
        # the many-user batch over a large pool, a quarter of the users new
        dict(name="turn_many", op="turn", batch=512, gone=128, lo=16, hi=8000, spare=120000, len_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "keep", "fork", "turn"])
    f32 = rng.random() < 0.2
    d, hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8])
    case = dict(op=op, len_seed=rng.randrange(1 << 20))
    if op != "turn":
        case.update(hkv=hkv, d=d, dtype="f32" if f32 else "bf16")
    if op == "attend":
        g = rng.choice([1, 2, 4, 8])
        form = rng.choice(["tree", "tree", "token", "run"])
        n = {"tree": rng.randint(1, 100), "token": 1, "run": _log_int(rng, 2, 500 if f32 else 2000)}[form]
        batch = _log_int(rng, 1, {"tree": 64, "token": 128, "run": 4}[form])
        longest = _log_int(rng, 16, min(40000, 4000000000 // (batch * hkv * g * (n + 8) * d) + 64, 300000000 // (batch * hkv * d) + 64))
        window = rng.choice([0, 0, _log_int(rng, 1, 3000)])
        case.update(batch=batch, hq=hkv * g, n_lo=rng.choice([n, max(1, n // 2)]), n_hi=n, tree=form == "tree", in_lo=rng.choice([0, longest // 3]),
                    in_hi=longest, out_lo=0, out_hi=_log_int(rng, 1, 400), cap=rng.choice([0.0, 0.0, 20.0, 50.0]), alibi=rng.random() < 0.3,
                    window=window, sinks=rng.choice([0, rng.randint(1, 40)]) if window else 0, halves=rng.random() < 0.25)
    elif op == "keep":
        n = rng.randint(1, 64)
        case.update(batch=_log_int(rng, 1, 300), n_lo=1, n_hi=n, tree=rng.random() < 0.8, held_lo=0, held_hi=_log_int(rng, 1, 300), layers=rng.randint(1, 8))
    elif op == "fork":
        prompts = _log_int(rng, 1, 64)
        case.update(prompts=prompts, samples=prompts * rng.randint(1, 4), lo=1, hi=_log_int(rng, 2, 1500), layers=rng.randint(1, 6),
                    spare=_log_int(rng, 1, 1000))
    else:
        batch = _log_int(rng, 2, 500)
        case.update(batch=batch, gone=rng.randint(1, batch), lo=1, hi=_log_int(rng, 2, 8000), spare=_log_int(rng, 1, 50000))
    return case


# ---------------------------------------------------------------------------------------------------------------------
# sizes that follow from the case alone
def _ints(rng, lo, hi, n):
    return rng.integers(lo, hi + 1, n)


def _sizes(case):
    """attend: drafted, private and public context tokens per user; keep: drafted, held; fork: lengths, source; turn: lengths, new lengths."""
    rng = np.random.default_rng(case["len_seed"])
    if case["op"] == "attend":
        B = case["batch"]
        return _ints(rng, case["n_lo"], case["n_hi"], B), _ints(rng, case["in_lo"], case["in_hi"], B), _ints(rng, case["out_lo"], case["out_hi"], B)
    if case["op"] == "keep":
        return _ints(rng, case["n_lo"], case["n_hi"], case["batch"]), _ints(rng, case["held_lo"], case["held_hi"], case["batch"])
    if case["op"] == "fork":
        return _ints(rng, case["lo"], case["hi"], case["prompts"]), np.sort(_ints(rng, 0, case["prompts"] - 1, case["samples"]))
    gone = np.zeros(case["batch"], dtype=bool)
    gone[rng.permutation(case["batch"])[:case["gone"]]] = True
    return _ints(rng, case["lo"], case["hi"], case["batch"]), _ints(rng, case["lo"], case["hi"], case["batch"]), gone


def _parents(case, counts):
    """A tree for each user, as a drafting model leaves it: tokens by depth, better ones with more children.  Runs: every token's parent is the one before."""
    rng = np.random.default_rng([case["len_seed"], 3])
    trees = []
    for n in counts:
        i = np.arange(n)
        trees.append(np.minimum(np.maximum((i * rng.uniform(0.3, 0.8, n)).astype(np.int64) - 1, -1), i - 1) if case["tree"] else i - 1)
    return trees


def _chosen(case, trees):
    """The last accepted token of each user's tree, -1 where none is; and how many are accepted with it."""
    rng = np.random.default_rng([case["len_seed"], 4])
    last = np.array([int(rng.integers(0, len(t))) if rng.random() < 0.9 else -1 for t in trees])
    paths = []
    for t, x in zip(trees, last):
        path = []
        while x >= 0:
            path.append(int(x))
            x = t[x]
        paths.append(path[::-1])
    return last, paths


def _seen_keys(case):
    """Keys that some row of a user sees, and pairs of a row and a key that it sees, over all users."""
    counts, lp, lq = _sizes(case)
    trees = _parents(case, counts)
    keys = pairs = 0
    W, S = case["window"] or (1 << 40), case["sinks"]
    for n, ctx, tree in zip(counts, (lp + lq).tolist(), trees):
        depth = np.zeros(n, dtype=np.int64)
        for i, p in enumerate(tree.tolist()):
            depth[i] = depth[p] + 1 if p >= 0 else 0
        back = np.minimum(ctx, np.maximum(W - 1 - depth, 0)) # context tokens inside a row's window
        front = np.minimum(S, ctx - back)                    # sinks in front of it
        own = np.minimum(depth + 1, W)
        late = np.clip(np.minimum(depth + 1 - own, S - ctx), 0, None)
        pairs += int((back + front + own + late).sum())
        keys += int(min(ctx, back.max() + min(S, ctx))) + int(n)
    return keys, pairs


def work(case):
    if case["op"] == "turn":
        lens, new, gone = _sizes(case)
        pages = int(_pages_held(lens).sum()) + case["spare"]
        moved = int(-(-lens[gone] // PAGE).sum()) + int(-(-new[gone] // PAGE).sum())
        return {"bytes": 4 * pages + 16 * moved + 16 * case["batch"], "flops": 0}
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attend":
        keys, pairs = _seen_keys(case)
        T = int(_sizes(case)[0].sum())
        return {"bytes": keys * 2 * case["hkv"] * case["d"] * es + 2 * T * case["hq"] * case["d"] * es, "flops": 4 * case["d"] * case["hq"] * pairs}
    row = case["hkv"] * case["d"] * es * 2 * case["layers"]
    if case["op"] == "keep":
        _, paths = _chosen(case, _parents(case, _sizes(case)[0]))
        moved = sum(sum(i != x for i, x in enumerate(p)) for p in paths)
        return {"bytes": 2 * moved * row + 8 * int(_sizes(case)[0].sum()) + 16 * case["batch"], "flops": 0}
    lens, source = _sizes(case)
    listed = -(-lens[source] // PAGE)
    return {"bytes": 2 * int((lens[source] % PAGE > 0).sum()) * PAGE * row + 20 * int(listed.sum()), "flops": 0}


def _pages_held(lens):
    return -(-np.asarray(lens) // PAGE)


# ---------------------------------------------------------------------------------------------------------------------
class _Part:
    """One paged partition: pools [pages, hkv, 16, d], tables and lengths on the device."""


def _part(lens, hkv, d, dtype, rng, gen, dev, layers=1):
    p = _Part()
    need = np.maximum(_pages_held(lens), 1)
    indptr = np.concatenate([[0], np.cumsum(need)])
    pages = int(indptr[-1]) + 3
    p.pools = [_randn((pages, hkv, PAGE, d), dtype, gen, dev) for _ in range(2 * layers)]
    p.k_pool, p.v_pool = p.pools[0], p.pools[1]
    p.page_indptr = torch.from_numpy(indptr.astype(np.int32)).to(dev)
    p.page_indices = torch.from_numpy(rng.permutation(pages)[:int(indptr[-1])].astype(np.int32)).to(dev)
    p.seq_lens = torch.from_numpy(np.asarray(lens).astype(np.int32)).to(dev)
    return p


def _randn(shape, dtype, gen, dev, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=dev).normal_(generator=gen)
    return x * scale if scale != 1.0 else x


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng([seed, 1])
    st = dict(case=case, dev=dev)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(dev)  # noqa: E731
    starts = lambda c: np.concatenate([[0], np.cumsum(c)])  # noqa: E731
    if case["op"] == "attend":
        counts, lp, lq = _sizes(case)
        dtype, T = DTYPES[case["dtype"]], int(counts.sum())
        st["q"] = _randn((T, case["hq"], case["d"]), dtype, gen, dev, 4.0 if case["cap"] else 1.0)    # scores that reach into the cap
        st["priv"] = _part(lp, case["hkv"], case["d"], dtype, rng, gen, dev)
        st["pub"] = _part(lq + counts, case["hkv"], case["d"], dtype, rng, gen, dev)
        st["indptr"] = i32(starts(counts))
        st["parents"] = i32(np.concatenate(_parents(case, counts))) if case["tree"] else None
        st["most"], st["one"] = int(counts.max()), case["n_hi"] == 1
        reach = (case["window"] - 1 if case["window"] else 1 << 40)
        st["span"] = int(np.minimum(lp + lq, reach).max())
        st["slopes"] = (2.0 ** (-8.0 * torch.arange(1, case["hq"] + 1, dtype=torch.float64) / case["hq"])).float().to(dev) if case["alibi"] else None
        st["out"] = torch.empty((T, case["hq"], case["d"]), dtype=dtype, device=dev)
        if case["halves"]:
            st["partial"] = tuple(torch.empty((T, case["hq"]) + x, device=dev) for x in ((case["d"],), (), ()))
    elif case["op"] == "keep":
        counts, held = _sizes(case)
        trees = _parents(case, counts)
        st["part"] = _part(held + counts, case["hkv"], case["d"], DTYPES[case["dtype"]], rng, gen, dev, case["layers"])
        st["indptr"] = i32(starts(counts))
        st["parents"] = i32(np.concatenate(trees)) if case["tree"] else None
        st["last"], st["most"] = i32(_chosen(case, trees)[0]), int(counts.max())
        st["new_lens"], st["kept"] = torch.zeros(case["batch"], dtype=torch.int32, device=dev), torch.zeros(int(counts.sum()), dtype=torch.int32, device=dev)
    elif case["op"] == "fork":
        lens, source = _sizes(case)
        P, S = case["prompts"], case["samples"]
        room = np.concatenate([_pages_held(lens), _pages_held(lens[source]) + 2])
        indptr = starts(room)
        pages = int(_pages_held(lens).sum()) + S + case["spare"]
        perm = rng.permutation(pages)
        table, refs = np.full(int(indptr[-1]), -1), np.zeros(pages)
        table[:int(indptr[P])] = perm[:int(indptr[P])]
        refs[perm[:int(indptr[P])]] = 1
        st.update(page_indptr=i32(indptr), page_indices=i32(table), refs=i32(refs), seq_lens=i32(np.concatenate([lens, np.zeros(S)])),
                  source=i32(np.concatenate([np.full(P, -1), source])), gone_from=i32(np.concatenate([np.full(P, NOTHING), np.zeros(S)])),
                  copies=torch.zeros((P + S, 2), dtype=torch.int32, device=dev))
        st["pools"] = [_randn((pages, case["hkv"], PAGE, case["d"]), DTYPES[case["dtype"]], gen, dev) for _ in range(2 * case["layers"])]
    else:
        lens, new, gone = _sizes(case)
        indptr = starts(np.maximum(_pages_held(lens + 1), _pages_held(new)))
        pages = int(np.maximum(_pages_held(lens + 1), _pages_held(new)).sum()) + case["spare"]
        perm, table, refs, used = rng.permutation(pages), np.full(int(indptr[-1]), -1), np.zeros(pages), 0
        for u, n in enumerate(_pages_held(lens).tolist()):
            table[indptr[u]:indptr[u] + n] = perm[used:used + n]
            used += n
        refs[perm[:used]] = 1
        st.update(page_indptr=i32(indptr), page_indices=i32(table), refs=i32(refs), gone_from=i32(np.where(gone, 0, NOTHING)),
                  have=i32(np.where(gone, 0, lens)), want=i32(np.where(gone, new, lens + 1)))
    return st


# ---------------------------------------------------------------------------------------------------------------------
def _ancestors(st, B, n):
    """[B, n, n]: whether token j is i itself or above it in its user's tree (padded to n tokens), and how far i lies below its root."""
    dev, start = st["dev"], st["indptr"].long()
    i = torch.arange(n, device=dev)
    there = i < (start[1:] - start[:-1])[:, None]
    if st["parents"] is None:
        up = (i[:, None] >= i).expand(B, n, n)
    else:
        parent = torch.where(there, st["parents"].long()[(start[:-1, None] + i).clamp(max=st["parents"].numel() - 1)], -1)
        step = (parent[:, :, None] == i).double() + torch.eye(n, dtype=torch.float64, device=dev)
        up = torch.linalg.matrix_power(step, n) > 0
    return up, up.sum(-1) - 1, there


def _attend_plain(st):
    case, priv, pub, dev = st["case"], st["priv"], st["pub"], st["dev"]
    B, hq, hkv, d, n = case["batch"], case["hq"], case["hkv"], case["d"], st["most"]
    start, T = st["indptr"].long(), st["q"].shape[0]
    lp = priv.seq_lens.long()
    ctx = lp + pub.seq_lens.long() - (start[1:] - start[:-1])
    up, depth, row_there = _ancestors(st, B, n)
    pos = ctx[:, None] + depth                                                    # [B, row]
    # keys: sinks in front of the widest window, the context from there on, the drafted tokens
    first = (ctx - st["span"]).clamp(min=0)
    sink = torch.arange(case["sinks"], device=dev).expand(B, -1)
    tail = first[:, None] + torch.arange(st["span"], device=dev)
    own = ctx[:, None] + torch.arange(n, device=dev)
    at = torch.cat([sink, tail, own], 1)                                          # place in the cache
    there = torch.cat([sink < first[:, None], tail < ctx[:, None], row_there], 1)
    where_ = torch.cat([sink, tail, pos], 1)                                      # position, by depth where drafted

    def rows(a, b):
        def of(part, x):
            page = part.page_indices.long()[(part.page_indptr.long()[:-1, None] + x // PAGE).clamp(max=part.page_indices.numel() - 1)]
            return page.clamp(min=0), x % PAGE
        inside = there & (at < lp[:, None])
        p1, s1 = of(priv, torch.where(inside, at, 0))
        p2, s2 = of(pub, torch.where(there & ~inside, at - lp[:, None], 0))
        x = torch.where(inside[:, :, None, None], a[p1, :, s1], b[p2, :, s2]).float()
        return torch.where(there[:, :, None, None], x, 0.0)

    k, v = rows(priv.k_pool, pub.k_pool), rows(priv.v_pool, pub.v_pool)           # [B, key, hkv, d]
    dist = pos[:, :, None] - where_[:, None, :]                                   # [B, row, key]
    seen = there[:, None, :].expand_as(dist)
    if case["window"]:
        seen = seen & ((dist < case["window"]) | (where_ < case["sinks"])[:, None, :])
    seen = torch.cat([seen[:, :, :-n], seen[:, :, -n:] & up], 2)
    row = (start[:-1, None] + torch.arange(n, device=dev)).clamp(max=T - 1)
    q = st["q"].float()[row].view(B, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(d)).view(B, hkv, hq // hkv, n, -1)
    if case["cap"]:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    if st["slopes"] is not None:
        s -= st["slopes"].view(hkv, hq // hkv, 1, 1) * dist[:, None, None].float()
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, -1, p.shape[-1]), v.transpose(1, 2)).view(B, hkv, hq // hkv, n, d) / torch.where(total == 0, 1.0, total)
    user = torch.searchsorted(start[1:], torch.arange(T, device=dev), right=True)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, d)[user, torch.arange(T, device=dev) - start[user]].to(st["q"].dtype)


def _keep_plain(st):
    case, part, dev = st["case"], st["part"], st["dev"]
    B, n = case["batch"], st["most"]
    start = st["indptr"].long()
    up, depth, there = _ancestors(st, B, n)
    last = st["last"].long()
    base = part.seq_lens.long() - (start[1:] - start[:-1])
    kept = up[torch.arange(B, device=dev), last.clamp(min=0)] & (last >= 0)[:, None]            # [B, token]
    rank = kept.cumsum(1) - 1
    user, token = kept.nonzero(as_tuple=True)
    to = rank[user, token]

    def slot(x):
        x = base[user] + x
        return part.page_indices.long()[part.page_indptr.long()[user] + x // PAGE], x % PAGE

    (p1, s1), (p2, s2) = slot(token), slot(to)
    for pool in part.pools:
        pool[p2, :, s2] = pool[p1, :, s1]
    names = torch.full_like(st["kept"], -1)
    names[start[user] + to] = token.int()
    return {"pools": part.pools, "new_lens": (base + kept.sum(1)).int(), "kept": names}


def _slots(st):
    """Slot of each table entry, and its place in the slot."""
    start = st["page_indptr"].long()
    e = torch.arange(st["page_indices"].numel(), device=st["dev"])
    slot = torch.searchsorted(start[1:], e, right=True)
    return slot, e - start[slot]


def _release_plain(st, first):
    slot, e = _slots(st)
    pages, refs = st["page_indices"], st["refs"]
    gone = (e >= (first.long()[slot] + PAGE - 1) // PAGE) & (pages >= 0)
    refs.index_add_(0, pages.clamp(min=0).long(), -gone.int())
    pages.masked_fill_(gone, -1)


def _take_plain(st, want):
    """A fresh page for every entry marked in `want`: the lowest pages that nobody lists, in the order of the entries."""
    pages, refs = st["page_indices"], st["refs"]
    free = torch.argsort((refs != 0).int(), stable=True)
    fresh = free[(want.cumsum(0) - 1).clamp(min=0, max=free.numel() - 1)]
    pages.copy_(torch.where(want, fresh, pages.long()).int())
    refs.index_add_(0, fresh, want.int())


def _fork_plain(st):
    start, lens, pages, refs = st["page_indptr"].long(), st["seq_lens"], st["page_indices"], st["refs"]
    _release_plain(st, st["gone_from"])
    slot, e = _slots(st)
    src = st["source"].long()
    new, n = src[slot] >= 0, lens.long()[src.clamp(min=0)]
    theirs = pages[(start[src.clamp(min=0)][slot] + e).clamp(max=pages.numel() - 1)]
    shared = new & (e < n[slot] // PAGE)
    part = new & (e == n[slot] // PAGE) & (n[slot] % PAGE > 0)
    pages.copy_(torch.where(shared, theirs, pages))
    refs.index_add_(0, theirs.clamp(min=0).long(), (shared & (theirs >= 0)).int())
    _take_plain(st, part)
    st["copies"].fill_(-1)
    st["copies"][slot[part]] = torch.stack([theirs[part], pages[part]], 1)
    lens.copy_(torch.where(src >= 0, n.int(), lens))
    pairs = st["copies"][st["copies"][:, 0] >= 0].long()
    for pool in st["pools"]:
        pool[pairs[:, 1]] = pool[pairs[:, 0]]
    return {"pools": st["pools"], "table": pages, "refs": refs, "lens": lens, "copies": st["copies"]}


def _turn_plain(st):
    _release_plain(st, st["gone_from"])
    slot, e = _slots(st)
    first, last = (st["have"].long() + PAGE - 1) // PAGE, (st["want"].long() + PAGE - 1) // PAGE
    _take_plain(st, (e >= first[slot]) & (e < last[slot]) & (st["page_indices"] < 0))
    return {"table": st["page_indices"], "refs": st["refs"]}


# ---------------------------------------------------------------------------------------------------------------------
def _shape(case, spd):
    B = case["prompts"] + case["samples"] if case["op"] == "fork" else case["batch"]
    key = (B, case.get("hq", case.get("hkv", 1)), case.get("hkv", 1), case.get("d", 128), DTYPES[case.get("dtype", "bf16")], case["op"])
    if key not in _workspaces:
        shape = spd.make_shape(*key[:5], 1.0 / math.sqrt(key[3]))
        _workspaces[key] = shape, spd.alloc_drafted_workspace(shape) if case["op"] == "attend" else spd.alloc_workspace(shape)
    return _workspaces[key]


def _run_own(st):
    from paper_2409_19134_b200 import binding as spd
    case = st["case"]
    shape, ws = _shape(case, spd)
    if case["op"] == "attend":
        score = spd.make_score(logit_cap=case["cap"], window=case["window"], alibi_slopes=st["slopes"])
        drafts = dict(tok_indptr=None if st["one"] else st["indptr"], parents=st["parents"], sinks=case["sinks"])
        if case["halves"]:
            spd.spd_partial_attn_drafted(shape, score, st["q"], st["priv"], st["pub"].seq_lens, st["partial"], ws, **drafts)
            spd.spd_service_attn_merge_drafted(shape, score, st["q"], st["pub"], st["priv"].seq_lens, st["partial"], st["out"], ws, **drafts)
        else:
            spd.spd_decode_step_drafted(shape, score, st["q"], st["priv"], st["pub"], st["out"], ws, **drafts)
        return st["out"]
    if case["op"] != "turn" and "handle" not in st:        # kept as long as the cache's pools, like the pools themselves
        st["handle"] = spd.make_pools(shape, st["pools"] if case["op"] == "fork" else st["part"].pools)
    if case["op"] == "keep":
        spd.spd_keep_drafted(shape, st["handle"], st["part"], st["indptr"], st["last"], ws, parents=st["parents"], new_lens=st["new_lens"],
                             kept=st["kept"])
        return {"pools": st["part"].pools, "new_lens": st["new_lens"], "kept": st["kept"]}
    spd.spd_pages_release(shape, st["refs"], st["page_indptr"], st["page_indices"], st["gone_from"], ws)
    if case["op"] == "fork":
        spd.spd_pages_fork(shape, st["refs"], st["page_indptr"], st["page_indices"], st["seq_lens"], st["source"], st["copies"], ws)
        spd.spd_pages_copy(shape, st["handle"], st["copies"], ws)
        return {"pools": st["pools"], "table": st["page_indices"], "refs": st["refs"], "lens": st["seq_lens"], "copies": st["copies"]}
    spd.spd_pages_take(shape, st["refs"], st["page_indptr"], st["page_indices"], st["have"], st["want"], ws)
    return {"table": st["page_indices"], "refs": st["refs"]}


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _attend_plain, "keep": _keep_plain, "fork": _fork_plain, "turn": _turn_plain}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
def _exact_attend(st):
    case = st["case"]
    counts, lp, lq = _sizes(case)
    trees = _parents(case, counts)
    g, W, S = case["hq"] // case["hkv"], case["window"] or (1 << 40), case["sinks"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["dev"])
    t0 = 0
    for u in range(case["batch"]):
        n, ctx = int(counts[u]), int(lp[u] + lq[u])
        rows = [[], []]
        for part, m in ((st["priv"], int(lp[u])), (st["pub"], int(lq[u]) + n)):
            a, b = int(part.page_indptr[u]), int(part.page_indptr[u + 1])
            for r, pool in zip(rows, (part.k_pool, part.v_pool)):
                r.append(pool[part.page_indices[a:b].long()].transpose(0, 1).reshape(case["hkv"], -1, case["d"])[:, :m])
        k, v = (torch.cat(r, 1) for r in rows)
        line = np.zeros((n, n), dtype=bool)
        place = np.zeros(n, dtype=np.int64)
        for i, p in enumerate(trees[u].tolist()):
            if p >= 0:
                line[i], place[i] = line[p], place[p] + 1
            line[i, i] = True
        line, place = torch.from_numpy(line).to(st["dev"]), torch.from_numpy(place).to(st["dev"]) + ctx
        at = torch.cat([torch.arange(ctx, device=st["dev"]), place])
        for a in range(0, n, 256):
            b = min(n, a + 256)
            far = place[a:b, None] - at
            hidden = (far >= W) & (at >= S)
            hidden[:, ctx:] |= ~line[a:b]
            for h in range(case["hq"]):
                s = st["q"][t0 + a:t0 + b, h].double() @ k[h // g].double().T / math.sqrt(case["d"])
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if st["slopes"] is not None:
                    s = s - st["slopes"][h].double() * far
                out[t0 + a:t0 + b, h] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v[h // g].double()
        t0 += n
    return out


def _exact_keep(st):
    case, part = st["case"], st["part"]
    counts, held = _sizes(case)
    _, paths = _chosen(case, _parents(case, counts))
    table, ip = part.page_indices.cpu().numpy(), part.page_indptr.cpu().numpy()
    src, dst = [], []
    for u, path in enumerate(paths):
        for i, x in enumerate(path):
            for at, to in ((int(held[u]) + x, src), (int(held[u]) + i, dst)):
                to.append(int(table[ip[u] + at // PAGE]) * PAGE + at % PAGE)
    src, dst = (torch.tensor(x, dtype=torch.int64, device=st["dev"]) for x in (src, dst))
    pools = []
    for pool in part.pools:
        flat = pool.transpose(1, 2).reshape(-1, case["hkv"], case["d"]).double()
        flat[dst] = flat[src]
        pools.append(flat.view(-1, PAGE, case["hkv"], case["d"]).transpose(1, 2))
    return {"pools": pools, "new_lens": None, "kept": None}


def _exact_fork(st):
    lens, source = _sizes(st["case"])
    table, ip, refs = (st[x].cpu().numpy() for x in ("page_indices", "page_indptr", "refs"))
    free = np.flatnonzero(refs == 0).tolist()
    pairs = [(int(table[ip[s] + lens[s] // PAGE]), 0) for s in source if lens[s] % PAGE]
    pairs = [(a, free[i]) for i, (a, _) in enumerate(pairs)]
    pools = [pool.double() for pool in st["pools"]]
    for pool in pools:
        for a, b in pairs:
            pool[b] = pool[a]
    return {"pools": pools, "table": None, "refs": None, "lens": None, "copies": None}


def exact(case, seed):
    if case["op"] == "turn":
        return None
    st = prepare(case, seed)
    if case["op"] != "attend" and sum(p.numel() for p in st.get("pools") or st["part"].pools) > 4e9:
        return None                     # twice as many bytes as the card has room for beside the pools
    return {"attend": _exact_attend, "keep": _exact_keep, "fork": _exact_fork}[case["op"]](st)
