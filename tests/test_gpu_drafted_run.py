"""The calls for drafted tokens and for pages as a server uses them: pages taken, drafts appended, verified, kept and released round after round over a
private and a public cache, then samples that start from one user's cache -- against caches kept as plain rows on the host."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import workloads as wl
from tests import drafted_reference as dr
from tests import scored_reference as ref

pytestmark = pytest.mark.gpu
PAGE, HQ, HKV, D = 16, 8, 2, 64


def i32(a):
    return torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()


class Server:
    """Users with a private prompt and a public cache in two layers that share their tables; rows of everything on the host too."""

    def __init__(self, dtype, prompts, room, pages, seed, window=0, sinks=0):
        self.dtype, self.B, self.window, self.sinks = dtype, len(prompts), window, sinks
        self.gen, self.rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.shape = spd.make_shape(self.B, HQ, HKV, D, dtype, D ** -0.5)
        self.ws = spd.alloc_drafted_workspace(self.shape)
        self.score = spd.make_score(window=window)
        self.rows = [[[[self.randn(n, HKV) for _ in range(2)] for _ in range(2)] for n in prompts] for _ in range(1)][0]      # [user][layer][k, v]: prompt and what follows
        self.prompt = list(prompts)
        self.refs, self.ip = torch.zeros(pages, dtype=torch.int32, device="cuda"), i32(np.arange(self.B + 1) * room)
        self.ix = torch.full((self.B * room,), -1, dtype=torch.int32, device="cuda")
        nan = lambda n: torch.full((n, HKV, PAGE, D), float("nan"), dtype=dtype, device="cuda")  # noqa: E731
        self.pub = [wl.PagedKV(nan(pages), nan(pages), self.ip, self.ix, torch.zeros(self.B, dtype=torch.int32, device="cuda")) for _ in range(2)]
        self.lens = self.pub[0].seq_lens
        self.pub[1].seq_lens = self.lens                       # one length for both layers
        need = [-(-n // PAGE) for n in prompts]
        tables = i32(np.concatenate([[0], np.cumsum(need)])), i32(self.rng.permutation(sum(need))) if sum(need) else i32([])
        self.priv = []
        for layer in range(2):
            part = wl.PagedKV(nan(sum(need)), nan(sum(need)), *tables, torch.zeros(self.B, dtype=torch.int32, device="cuda"))
            k, v = (torch.cat([self.rows[u][layer][x] for u in range(self.B)]).cuda() for x in range(2))
            spd.spd_append_kv_rope(self.shape, None, None, k, v, part, self.ws, tok_indptr=i32(np.concatenate([[0], np.cumsum(prompts)])))
            self.priv.append(part)
        self.pools = spd.make_pools(self.shape, [p for part in self.pub for p in (part.k_pool, part.v_pool)])

    def randn(self, n, heads):
        return torch.randn((n, heads, D), generator=self.gen).to(self.dtype)

    def table(self):
        return self.shape, self.refs, self.ip, self.ix

    def draft(self, counts, kind):
        self.trees = dr.trees(counts, int(self.rng.integers(1 << 30)), kind)
        self.counts, self.tok = counts, i32(np.concatenate([[0], np.cumsum(counts)]))
        self.parents = None if kind == "run" else i32(np.concatenate(self.trees + [np.zeros(0)]))
        T = int(sum(counts))
        self.q = [self.randn(T, HQ) for _ in range(2)]
        self.new = [[self.randn(T, HKV) for _ in range(2)] for _ in range(2)]
        self.held = [r[0][0].shape[0] - n for r, n in zip(self.rows, self.prompt)]         # public tokens in front of the draft
        self.on = [t.cuda() for t in self.q], [[t.cuda() for t in kv] for kv in self.new]
        self.out = [torch.full((T, HQ, D), float("nan"), device="cuda") for _ in range(2)]

    def step(self, want):
        """One round on the device: pages, append and attention in both layers.  want: public tokens with the draft."""
        spd.spd_pages_take(*self.table(), self.lens, want, self.ws)
        for layer in range(2):
            k, v = self.on[1][layer]
            spd.spd_append_kv_rope(self.shape, None, None, k, v, self.pub[layer], self.ws, tok_indptr=self.tok, new_lens="in place" if layer == 1 else None)
            if layer == 0:                                     # the first layer attends over the lengths that the second one's append will write
                self.pub[0].seq_lens = want
            spd.spd_decode_step_drafted(self.shape, self.score, self.on[0][layer], self.priv[layer], self.pub[layer], self.out[layer], self.ws, tok_indptr=self.tok,
                                        parents=self.parents, sinks=self.sinks)
            self.pub[0].seq_lens = self.lens

    def check(self):
        t0 = 0
        for u, tree in enumerate(self.trees):
            n, ctx = len(tree), self.rows[u][0][0].shape[0]
            line, depth = np.zeros((n, n), dtype=bool), np.zeros(n, dtype=np.int64)
            for i, p in enumerate(tree):
                if p >= 0:
                    line[i], depth[i] = line[p], depth[p] + 1
                line[i, i] = True
            where = torch.cat([torch.arange(ctx), ctx + torch.from_numpy(depth)])
            for layer in range(2):
                k, v = (torch.cat([self.rows[u][layer][x], self.new[layer][x][t0:t0 + n]]) for x in range(2))
                for i in range(n):
                    seen = torch.cat([torch.ones(ctx, dtype=torch.bool), torch.from_numpy(line[i])])
                    if self.window:
                        seen &= (ctx + int(depth[i]) - where < self.window) | (where < self.sinks)
                    for h in range(HQ):
                        kk, vv = k[:, h // (HQ // HKV)], v[:, h // (HQ // HKV)]
                        want, _, _, _, S = ref.attend(self.q[layer][t0 + i, h], kk, vv, seen, D ** -0.5)
                        tol = ref.bound(float(vv[seen].abs().max()), D, S, int(seen.sum()), weight=0.0 if self.dtype == torch.float32 else 2.0 ** -8)
                        err = (self.out[layer][t0 + i, h].cpu().double() - want).abs().max()
                        assert float(err) <= tol + 2.0 ** -24 * float(want.abs().max()), (u, layer, i, h, float(err), tol)
            t0 += n

    def keep(self):
        last = [int(self.rng.integers(-1, n)) if n else -1 for n in self.counts]
        kept = torch.zeros(int(sum(self.counts)), dtype=torch.int32, device="cuda")
        spd.spd_keep_drafted(self.shape, self.pools, self.pub[1], self.tok, i32(last), self.ws, parents=self.parents, kept=kept)
        t0, names = 0, kept.cpu().tolist()
        for u, (tree, x) in enumerate(zip(self.trees, last)):
            path = []
            while x >= 0:
                path.append(x)
                x = int(tree[x])
            path.reverse()
            assert names[t0:t0 + len(tree)] == path + [-1] * (len(tree) - len(path))
            for layer in range(2):
                for x in range(2):
                    self.rows[u][layer][x] = torch.cat([self.rows[u][layer][x], self.new[layer][x][t0:t0 + len(tree)][path]])
            t0 += len(tree)
        spd.spd_pages_release(*self.table(), self.lens, self.ws)                       # what the rejected tokens had
        assert self.lens.tolist() == [r[0][0].shape[0] - n for r, n in zip(self.rows, self.prompt)]
        if self.window:                                                                 # and what lies hidden for good
            first = [max(0, self.sinks - n) for n in self.prompt]
            hidden = [max(0, r[0][0].shape[0] + 1 - self.window - n) for r, n in zip(self.rows, self.prompt)]
            spd.spd_pages_release(*self.table(), i32(first), self.ws, to_tokens=i32(hidden))
        self.ok()

    def ok(self):
        assert spd.spd_query_device_status(self.ws) == (spd.SPD_OK, -1)
        listed = self.ix[self.ix >= 0].cpu()
        assert torch.equal(torch.bincount(listed.long(), minlength=self.refs.numel()), self.refs.cpu().long())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 20)])
def test_rounds(dtype, window, sinks):
    s = Server(dtype, [40, 0, 17, 100], 20, 50, seed=3, window=window, sinks=sinks)
    for counts, kind in (([7, 12, 1, 0], "tree"), ([30, 5, 33, 9], "run"), ([40, 40, 40, 40], "tree"), ([1, 1, 1, 1], "run"), ([25, 3, 17, 30], "chain"), ([20, 60, 2, 8], "star")):
        s.draft(counts, kind)
        s.step(i32(np.array(s.held) + np.array(counts)))
        s.check()
        s.keep()


def test_samples_of_one_user():
    """Three users become copies of the first one in the middle of a page; what they draft afterwards is their own."""
    s = Server(torch.bfloat16, [0, 0, 0, 0], 12, 40, seed=5)
    s.draft([53, 0, 0, 0], "run")
    s.step(i32([53, 0, 0, 0]))
    s.keep()
    n, copies = int(s.lens[0]), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    spd.spd_pages_fork(*s.table(), s.lens, i32([-1, 0, 0, 0]), copies, s.ws)
    spd.spd_pages_copy(s.shape, s.pools, copies, s.ws)
    assert s.lens.tolist() == [n] * 4 and (n % PAGE == 0) == bool((copies == -1).all())
    s.rows = [s.rows[0]] + [[[x.clone() for x in kv] for kv in s.rows[0]] for _ in range(3)]
    s.ok()
    for counts, kind in (([5, 9, 33, 1], "tree"), ([2, 20, 3, 40], "run")):
        s.draft(counts, kind)
        s.step(i32(np.array(s.held) + np.array(counts)))
        s.check()
        s.keep()
    spd.spd_pages_release(*s.table(), i32([0] * 4), s.ws)
    s.ok()
    assert int(s.refs.sum()) == 0


def test_a_round_from_a_graph():
    s = Server(torch.bfloat16, [33, 70], 12, 30, seed=7)
    s.draft([10, 21], "tree")
    want, back = i32(np.array(s.held) + np.array([10, 21])), s.lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(want)
    torch.cuda.current_stream().wait_stream(side)
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.lens.copy_(back)
        s.step(want)
    for out in s.out:
        out.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    s.check()
    s.keep()


def test_two_streams():
    """Two batches side by side, each on a stream and a workspace of its own."""
    ws = [dr.batch([5, 17, 1], [700, 30, 64], [3, 0, 16], 8, 2, 128, "bf16", seed=71), dr.batch([33, 2], [90, 1500], [0, 40], 8, 2, 128, "bf16", seed=72)]
    gs = [dr.OnDevice(w) for w in ws]
    want = [dr.expected(w) for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(30):
        for g, s, o in zip(gs, streams, outs):
            with torch.cuda.stream(s):
                o.append(g.fused())
    torch.cuda.synchronize()
    for o, x in zip(outs, want):
        dr.close(o[0], x[0], x[4])
        assert all(torch.equal(o[0], y) for y in o)


def test_two_graphs_on_one_workspace():
    """Two captured calls of one shape that share a workspace, replayed in turns on one stream, with eager calls in between."""
    ws = [dr.batch([5, 17, 1], [700, 30, 64], [3, 0, 16], 8, 2, 128, "bf16", seed=73), dr.batch([33, 2, 9], [90, 1500, 0], [0, 40, 7], 8, 2, 128, "bf16", seed=74)]
    gs = [dr.OnDevice(w) for w in ws]
    gs[1].ws = gs[0].ws
    want, outs, graphs = [dr.expected(w) for w in ws], [g.out() for g in gs], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for g, o in zip(gs, outs):
            g.fused(out=o)
    torch.cuda.current_stream().wait_stream(side)
    for g, o in zip(gs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            g.fused(out=o)
    for i in range(20):
        for o in outs:
            o.fill_(float("nan"))
        graphs[i % 2].replay()
        eager = gs[0].fused()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, outs[0])
    for o, x in zip(outs, want):
        dr.close(o, x[0], x[4])
    assert spd.spd_query_device_status(gs[0].ws) == (spd.SPD_OK, -1)
