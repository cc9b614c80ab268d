"""Pages taken, shared, copied and released on the device, and the rows of accepted drafted tokens, against plain loops."""
import numpy as np
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import drafted_reference as dr

pytestmark = pytest.mark.gpu
PAGE = 16


class Table:
    """Tables and counts on the host, with the loops that say what each call does, and their copies on the device."""

    def __init__(self, room, pages, seed, held=None, dtype=torch.bfloat16, hkv=2, d=64):
        rng = np.random.default_rng(seed)
        self.B, self.pages = len(room), pages
        self.indptr = np.concatenate([[0], np.cumsum(room)])
        self.indices, self.refs = np.full(int(self.indptr[-1]), -1), np.zeros(pages, dtype=np.int64)
        self.lens = np.zeros(self.B, dtype=np.int64) if held is None else np.array(held)
        perm = rng.permutation(pages)
        used = 0
        for u, n in enumerate(self.lens):
            k = -(-int(n) // PAGE)
            self.indices[self.indptr[u]:self.indptr[u] + k] = perm[used:used + k]
            used += k
        self.refs[perm[:used]] = 1
        self.shape = spd.make_shape(self.B, hkv, hkv, d, dtype, 1.0)
        self.ws = spd.alloc_workspace(self.shape)
        self.upload()

    def upload(self):
        i32 = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()  # noqa: E731
        self.g_refs, self.g_indptr, self.g_indices, self.g_lens = i32(self.refs), i32(self.indptr), i32(self.indices), i32(self.lens)

    def args(self):
        return self.shape, self.g_refs, self.g_indptr, self.g_indices

    def row(self, u):
        return self.indices[self.indptr[u]:self.indptr[u + 1]]

    def release(self, first, last=None):
        for u in range(self.B):
            row = self.row(u)
            end = len(row) if last is None else min(len(row), int(last[u]) // PAGE)
            for e in range(-(-int(first[u]) // PAGE), end):
                if row[e] >= 0:
                    self.refs[row[e]] -= 1
                    row[e] = -1

    def take(self, first, last):
        free = np.flatnonzero(self.refs == 0).tolist()
        short = []
        wanted = 0
        total = len(free)
        for u in range(self.B):
            row = self.row(u)
            want = [e for e in range(-(-int(first[u]) // PAGE), -(-int(last[u]) // PAGE)) if row[e] == -1]
            wanted += len(want)
            if want and wanted > total:
                short.append(u)
                continue
            for e in want:
                row[e] = free.pop(0)
                self.refs[row[e]] = 1
        return short

    def fork(self, source):
        free = np.flatnonzero(self.refs == 0).tolist()
        copies = np.full((self.B, 2), -1)
        for u, s in enumerate(source):
            if s < 0:
                continue
            n = int(self.lens[s])
            for e in range(n // PAGE):
                self.row(u)[e] = self.row(s)[e]
                if self.row(s)[e] >= 0:
                    self.refs[self.row(s)[e]] += 1
            if n % PAGE:
                page = free.pop(0)
                self.refs[page] = 1
                copies[u] = self.row(s)[n // PAGE], page
                self.row(u)[n // PAGE] = page
            self.lens[u] = n
        return copies

    def same(self, status=(spd.SPD_OK, -1)):
        assert spd.spd_query_device_status(self.ws) == status
        assert np.array_equal(self.g_refs.cpu().numpy(), self.refs)
        assert np.array_equal(self.g_indices.cpu().numpy(), self.indices)
        assert np.array_equal(self.g_lens.cpu().numpy(), self.lens)


def i32(a):
    return torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()


@pytest.mark.parametrize("B,pages,most", [(1, 40, 30), (7, 300, 30), (300, 9001, 25), (3, 70001, 8000), (1500, 20000, 9), (2, 5, 1)])
def test_take_and_release(B, pages, most):
    rng = np.random.default_rng(B + pages)
    t = Table(rng.integers(1, most + 1, B), pages, seed=B, held=np.zeros(B))
    for step in range(4):
        room = np.diff(t.indptr) * PAGE
        last = (rng.random(B) * (room + 1)).astype(np.int64)
        first = (rng.random(B) * last).astype(np.int64)
        a, b = i32(first), i32(last)
        spd.spd_pages_take(*t.args(), a, b, t.ws)
        assert t.take(first, last) == []
        t.same()
        if step == 3:                                    # to the tables' end, other users nothing at all
            first = np.where(rng.random(B) < 0.5, 0, 1 << 30)
            spd.spd_pages_release(*t.args(), i32(first), t.ws)
            t.release(first)
        else:
            first = (rng.random(B) * room).astype(np.int64)
            last = (first + rng.random(B) * 200).astype(np.int64)
            spd.spd_pages_release(*t.args(), i32(first), t.ws, to_tokens=i32(last))
            t.release(first, last)
        t.same()


def test_take_without_enough_pages():
    t = Table([4] * 6, 13, seed=1)
    first, last = np.zeros(6), np.array([64, 0, 50, 48, 16, 0])      # 4, 0, 4, 3, 1 pages; the fourth leaves 2 that the last could do with
    spd.spd_pages_take(*t.args(), i32(first), i32(last), t.ws)
    assert t.take(first, last) == []
    t.same()
    t.release([0, 1 << 30, 0, 1 << 30, 1 << 30, 1 << 30])
    t.upload()
    last = np.array([16, 33, 64, 0, 64, 48])                          # 1, 3, 4 pages of 9; then 3 and 3, of which there is only one left
    spd.spd_pages_take(*t.args(), i32(first), i32(last), t.ws)
    assert t.take(first, last) == [4, 5]
    t.same((8, 4))
    with pytest.raises(spd.SpdError, match="SPD_ERR_NO_PAGE"):
        spd._check(8, "take")


def test_bad_requests_leave_users_alone():
    t = Table([3, 3, 3, 3], 20, seed=2, held=[0, 40, 0, 0])
    spd.spd_pages_take(*t.args(), i32([0, 0, 0, -1]), i32([10, 40, 49, 20]), t.ws)        # 49 tokens do not fit three pages
    t.take([0, 0, 0, 0], [10, 40, 0, 0])
    t.same((4, 2))
    t.refs[t.row(1)[1]] = 0                                              # a page that nobody lists, they say
    t.row(1)[2] = 20                                                     # a page that is not there
    t.upload()
    spd.spd_pages_release(*t.args(), i32([0, 0, 0, 0]), t.ws)
    t.refs[t.row(0)[0]] -= 1
    t.refs[t.row(1)[0]] -= 1
    t.row(0)[0], t.row(1)[0], t.row(1)[1] = -1, -1, -1
    t.same((4, 1))


@pytest.mark.parametrize("dtype,hkv,d,layers", [(torch.bfloat16, 8, 128, 2), (torch.float32, 1, 64, 1), (torch.bfloat16, 3, 64, 70)])
@pytest.mark.parametrize("held", [[500, 16, 0, 33, 1], [48, 1, 15, 17, 0]])
def test_fork_and_copy(dtype, hkv, d, layers, held):
    n = len(held)
    source = [-1] * n + [0, 0, 3, 2, 4, 1]
    t = Table([-(-x // PAGE) + 2 for x in held] + [35] * 6, 120, seed=3, held=held + [0] * 6, dtype=dtype, hkv=hkv, d=d)
    gen = torch.Generator(device="cuda").manual_seed(4)
    pools = [torch.randn((t.pages, hkv, PAGE, d), generator=gen, device="cuda").to(dtype) for _ in range(2 * layers)]
    want = [p.clone() for p in pools]
    copies = torch.full((t.B, 2), 7, dtype=torch.int32, device="cuda")
    for handle in (pools, spd.make_pools(t.shape, pools)):
        spd.spd_pages_fork(*t.args(), t.g_lens, i32(source), copies, t.ws)
        spd.spd_pages_copy(t.shape, handle, copies, t.ws)
        pairs = t.fork(source)
        t.same()
        assert np.array_equal(copies.cpu().numpy(), pairs)
        for a, b in pairs:
            if a >= 0:
                for p in want:
                    p[b] = p[a]
        for p, q in zip(pools, want):
            assert torch.equal(p, q)
        gone = [1 << 30] * n + [0] * 6
        t.release(gone)
        spd.spd_pages_release(*t.args(), i32(gone), t.ws)
        t.lens[n:] = 0
        t.g_lens[n:] = 0
        t.same()


def test_fork_refusals():
    held = [40, 20, 33, 0, 0, 0, 0, 0, 10]
    t = Table([4, 4, 4, 4, 1, 4, 4, 4, 4], 60, seed=5, held=held)
    t.row(7)[1] = 3 if t.refs[3] else int(np.flatnonzero(t.refs)[0])          # in use where the copy's pages would go
    t.refs[t.row(7)[1]] += 1
    t.upload()
    copies = torch.zeros((t.B, 2), dtype=torch.int32, device="cuda")
    source = [-1, -1, -1, 0, 0, 3, 6, 0, 9]      # fine; too little room; from one that is being copied; itself; in use; not a user
    spd.spd_pages_fork(*t.args(), t.g_lens, i32(source), copies, t.ws)
    pairs = t.fork([-1, -1, -1, 0, -1, -1, -1, -1, -1])
    t.same((4, 4))
    assert np.array_equal(copies.cpu().numpy(), pairs)
    t = Table([3, 3, 3], 4, seed=6, held=[40, 0, 0])                            # one free page for two copies
    spd.spd_pages_fork(*t.args(), t.g_lens, i32([-1, 0, 0]), copies[:3], t.ws)
    pairs = t.fork([-1, 0, -1])
    t.same((8, 2))
    assert np.array_equal(copies[:3].cpu().numpy(), pairs)


def test_copy_leaves_bad_pairs_out():
    shape = spd.make_shape(1, 2, 2, 64, torch.float32, 1.0)
    ws = spd.alloc_workspace(shape)
    pool = torch.randn((6, 2, 16, 64), device="cuda")
    want = pool.clone()
    want[4] = pool[1]
    spd.spd_pages_copy(shape, [pool], i32([[-1, -1], [1, 4], [0, 6], [-1, 2], [3, 3]]), ws)
    assert spd.spd_query_device_status(ws) == (4, 2)
    assert torch.equal(pool, want)
    spd.spd_pages_copy(shape, [pool], i32(np.zeros((0, 2))), ws)
    spd.spd_pages_copy(shape, [], i32([[0, 1]]), ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1) and torch.equal(pool, want)


def keep_by_loops(w, last, pools):
    """Rows moved in `pools` (lists of host pools sharing w.pub's tables); returns new lengths and the tokens kept."""
    lens, names = [], []
    for u, tree in enumerate(w.trees):
        n, ln = len(tree), int(w.pub.seq_lens[u])
        path, x = [], int(last[u])
        while x >= 0:
            path.append(x)
            x = int(tree[x])
        path.reverse()
        at = lambda t: (int(w.pub.page_indices[int(w.pub.page_indptr[u]) + t // PAGE]), t % PAGE)  # noqa: E731
        for i, x in enumerate(path):
            (p1, s1), (p2, s2) = at(ln - n + x), at(ln - n + i)
            for pool in pools:
                pool[p2, :, s2] = pool[p1, :, s1].clone()
        lens.append(ln - n + len(path))
        names += path + [-1] * (n - len(path))
    return lens, names


@pytest.mark.parametrize("dtype,hq,hkv,d,layers", [("bf16", 8, 8, 128, 2), ("f32", 4, 1, 128, 1), ("bf16", 3, 3, 64, 66)])
@pytest.mark.parametrize("kind", ["tree", "chain", "star", "run"])
def test_keep(dtype, hq, hkv, d, layers, kind):
    counts = [5, 0, 1, 64, 17, 33, 2, 256 if kind == "chain" else 90]
    w = dr.batch(counts, [0] * 8, [0, 7, 15, 3, 16, 31, 100, 1], hq, hkv, d, dtype, seed=7, kind=kind)
    rng = np.random.default_rng(8)
    last = [int(rng.integers(0, n)) if n and u != 6 else -1 for u, n in enumerate(counts)]
    gen = torch.Generator().manual_seed(9)
    pools = [torch.randn(w.pub.k_pool.shape, generator=gen).to(w.dtype) for _ in range(2 * layers)]
    on = [p.cuda() for p in pools]
    lens, names = keep_by_loops(w, last, pools)
    shape = spd.make_shape(8, hq, hkv, d, w.dtype, 1.0)
    ws, g = spd.alloc_workspace(shape), w.pub.to("cuda")
    kept, new = torch.full((sum(counts),), 9, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    parents = None if w.parents is None else w.parents.cuda()
    spd.spd_keep_drafted(shape, on[:0], g, w.indptr.cuda(), i32(last), ws, parents=parents, new_lens=new, kept=kept)
    spd.spd_keep_drafted(shape, on, g, w.indptr.cuda(), i32(last), ws, parents=parents, total_tokens=sum(counts))
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    assert new.tolist() == lens == g.seq_lens.tolist() and kept.tolist() == names
    for a, b in zip(on, pools):
        assert torch.equal(a.cpu(), b)


def test_keep_refusals():
    w = dr.batch([4, 3, 5, 2, 6], [0] * 5, [10, 20, 0, 5, 3], 2, 2, 64, "bf16", seed=11)
    pools = [p.clone().nan_to_num(0.0) for p in (w.pub.k_pool, w.pub.v_pool)]
    on = [p.cuda() for p in pools]
    shape = spd.make_shape(5, 2, 2, 64, torch.bfloat16, 1.0)
    ws, g = spd.alloc_workspace(shape), w.pub.to("cuda")
    last = [2, 3, 4, 1, 5]                                  # user 1 has three tokens
    parents = w.parents.clone()
    at = w.indptr.tolist()
    parents[at[2] + 1] = 3                                  # user 2: a parent behind its child
    g.page_indices[int(g.page_indptr[4])] = -5              # user 4: a page that is not there
    g.seq_lens[3] = 1                                       # user 3: shorter than its draft
    kept = torch.zeros(20, dtype=torch.int32, device="cuda")
    lens, names = keep_by_loops(w, [2, -1, -1, -1, -1], pools)
    spd.spd_keep_drafted(shape, on, g, w.indptr.cuda(), i32(last), ws, parents=parents.cuda(), kept=kept)
    assert spd.spd_query_device_status(ws) == (4, 1)
    assert g.seq_lens.tolist() == [lens[0], 23, 5, 1, 9]
    assert kept.tolist() == names[:4] + [-1] * 16
    for a, b in zip(on, pools):
        assert torch.equal(a.cpu(), b)


def test_captured():
    """Release, take, fork and copy in one graph: every replay works on the state that it finds."""
    t = Table([8, 8, 8], 50, seed=12, held=[100, 0, 0])
    pools = [torch.randn((50, 2, 16, 64), device="cuda").bfloat16() for _ in range(2)]
    copies, source, gone = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), i32([-1, 0, 0]), i32([1 << 30, 0, 0])
    handle = spd.make_pools(t.shape, pools)

    def step():
        spd.spd_pages_release(*t.args(), gone, t.ws)
        spd.spd_pages_fork(*t.args(), t.g_lens, source, copies, t.ws)
        spd.spd_pages_copy(t.shape, handle, copies, t.ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
    t.fork([-1, 0, 0])
    t.same()
    for a, b in copies.tolist()[1:]:
        assert all(torch.equal(p[a], p[b]) for p in pools)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_beyond_32_bits(dtype):
    """Pools of more than 2^32 bytes: attention, kept rows and copies at their far end."""
    hkv, d = 8, 128
    page = hkv * PAGE * d * (2 if dtype == torch.bfloat16 else 4)
    n = 2**32 // page + 40
    w = dr.batch([6, 3], [70, 0], [20, 33], 16, hkv, d, "bf16" if dtype == torch.bfloat16 else "f32", seed=13)
    want, _, _, _, tol = dr.expected(w)
    g = dr.OnDevice(w)
    far = {}
    for name, part in (("priv", g.priv), ("pub", g.pub)):
        pools = [torch.empty((n, hkv, PAGE, d), dtype=dtype, device="cuda") for _ in range(2)]
        shift = n - part.k_pool.shape[0]
        for pool, small in zip(pools, (part.k_pool, part.v_pool)):
            pool[shift:] = small
        part.k_pool, part.v_pool = pools
        part.page_indices += shift
        far[name] = shift
    dr.close(g.fused(), want, tol)
    dr.close(g.halves()[0], want, tol)
    pools = [g.pub.k_pool, g.pub.v_pool]
    small = [p[far["pub"]:].cpu() for p in pools]
    w.pub.page_indices = g.pub.page_indices.cpu() - far["pub"]
    lens, names = keep_by_loops(w, [5, 1], small)
    spd.spd_keep_drafted(g.shape, pools, g.pub, g.drafts["tok_indptr"], i32([5, 1]), g.ws, parents=g.drafts["parents"])
    assert spd.spd_query_device_status(g.ws) == (spd.SPD_OK, -1) and g.pub.seq_lens.tolist() == lens
    used = torch.cat([(p[far["pub"]:].cpu() == s) | (torch.isnan(s) & torch.isnan(p[far["pub"]:].cpu())) for p, s in zip(pools, small)])
    assert bool(used.all())
    spd.spd_pages_copy(g.shape, pools, i32([[n - 1, 1], [int(g.pub.page_indices[0]), n - 30]]), g.ws)
    assert spd.spd_query_device_status(g.ws) == (spd.SPD_OK, -1)
    for p in pools:
        for a, b in ((n - 1, 1), (int(g.pub.page_indices[0]), n - 30)):
            assert bool(((p[a] == p[b]) | (torch.isnan(p[a]) & torch.isnan(p[b]))).all())


def test_take_from_a_large_pool_in_rounds():
    """Pages are given out and come back until every page of a pool of many chunks has been used, by users of very different sizes."""
    rng = np.random.default_rng(14)
    t = Table(rng.integers(1, 4000, 40), 40001, seed=14)
    for _ in range(6):
        first = np.zeros(40)
        last = np.minimum(np.diff(t.indptr) * PAGE, rng.integers(0, 64000, 40))
        spd.spd_pages_take(*t.args(), i32(first), i32(last), t.ws)
        short = t.take(first, last)
        t.same((8, short[0]) if short else (spd.SPD_OK, -1))
        gone = np.where(rng.random(40) < 0.4, 0, 1 << 30)
        spd.spd_pages_release(*t.args(), i32(gone), t.ws)
        t.release(gone)
        t.same()


def test_keep_looks_at_the_pages_of_runs():
    """Tokens of a run stay where they are, but not on a page that is not there."""
    counts, lout = [40, 40, 40, 20, 5, 30], [10, 10, 10, 16, 3, 0]
    w = dr.batch(counts, [0] * 6, lout, 2, 2, 64, "bf16", seed=15, kind="run")
    on = [p.cuda() for p in (w.pub.k_pool, w.pub.v_pool)]
    shape = spd.make_shape(6, 2, 2, 64, torch.bfloat16, 1.0)
    ws, g = spd.alloc_workspace(shape), w.pub.to("cuda")
    first = w.pub.page_indptr.tolist()
    g.page_indices[first[0] + 2] = -1                       # tokens 32 .. 47 of user 0, of which 10 .. 30 stay
    g.page_indices[first[1] + 1] = -1                       # tokens 16 .. 31 of user 1, of which 10 .. 16 stay
    g.page_indices[first[2] + 1] = on[0].shape[0]           # user 2: the same, behind the pool's end
    g.page_indices[first[3]] = -1                           # user 3: in front of the drafted tokens
    last = [20, 6, 39, 19, -1, 29]
    g.page_indices[first[4]] = -1                           # user 4: nothing stays
    g.seq_lens[5] = 9                                       # user 5: shorter than its draft
    kept = torch.full((175,), 9, dtype=torch.int32, device="cuda")
    spd.spd_keep_drafted(shape, on, g, w.indptr.cuda(), i32(last), ws, kept=kept)
    assert spd.spd_query_device_status(ws) == (4, 1)           # and users 2 and 5
    assert g.seq_lens.tolist() == [31, 50, 50, 36, 3, 9]
    names = [list(range(x + 1)) + [-1] * (n - x - 1) for n, x in zip(counts, [20, -1, -1, 19, -1, -1])]
    assert kept.tolist() == sum(names, [])
    for a, b in zip(on, (w.pub.k_pool, w.pub.v_pool)):
        assert torch.equal(a.cpu().nan_to_num(7.0), b.nan_to_num(7.0))


def test_tables_that_are_not_there():
    """No pages and no entries, though the offsets list some: users that have any are refused, nothing is read."""
    shape = spd.make_shape(3, 2, 2, 64, torch.bfloat16, 1.0)
    ws, none, indptr = spd.alloc_workspace(shape), torch.zeros(0, dtype=torch.int32, device="cuda"), i32([0, 0, 2, 5])
    lens, copies = i32([0, 20, 0]), i32(np.zeros((3, 2)))
    spd.spd_pages_take(shape, none, indptr, none, i32([0, 0, 0]), i32([0, 0, 20]), ws)
    assert spd.spd_query_device_status(ws) == (4, 1)
    spd.spd_pages_release(shape, none, indptr, none, i32([0, 0, 0]), ws)
    assert spd.spd_query_device_status(ws) == (4, 1)
    spd.spd_pages_fork(shape, none, indptr, none, lens, i32([-1, -1, 1]), copies, ws)
    assert spd.spd_query_device_status(ws) == (4, 2)
    assert lens.tolist() == [0, 20, 0] and copies.tolist() == [[-1, -1]] * 3
    spd.spd_pages_fork(shape, none, indptr, none, lens, i32([-1, 0, 0]), copies, ws)      # of a user without tokens, into entries that are not there
    assert spd.spd_query_device_status(ws) == (4, 1)
    empty = i32([0, 0, 0, 0])                                                             # nobody lists anything: nothing to do
    spd.spd_pages_take(shape, none, empty, none, i32([0, 0, 0]), i32([0, 0, 0]), ws)
    spd.spd_pages_release(shape, none, empty, none, i32([0, 0, 0]), ws)
    spd.spd_pages_fork(shape, none, empty, none, i32([0, 0, 0]), i32([-1, 0, -1]), copies, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    held = i32([3, -1, -1, -1, -1])                                                       # entries, but no pool: a page that is listed is out of range
    spd.spd_pages_release(shape, none, indptr, held, i32([0, 0, 0]), ws)
    assert spd.spd_query_device_status(ws) == (4, 1) and held.tolist() == [3, -1, -1, -1, -1]


def test_workspace_for_a_pool_of_many_pages():
    """Four bytes per page do not fit every shape's workspace: the size call says what does."""
    shape, pages = spd.make_shape(2, 1, 1, 64, torch.bfloat16, 1.0), 6_000_001
    assert spd.spd_pages_workspace_size(shape, 0) == spd.spd_workspace_size(shape)
    refs, indptr, indices = torch.ones(pages, dtype=torch.int32, device="cuda"), i32([0, 3, 5]), i32([-1] * 5)
    refs[[5, 4_000_000, pages - 2, pages - 1]] = 0
    size = spd.spd_pages_workspace_size(shape, pages)
    assert size > spd.spd_workspace_size(shape)
    with pytest.raises(spd.SpdError, match="SPD_ERR_WORKSPACE"):
        spd.spd_pages_take(shape, refs, indptr, indices, i32([0, 0]), i32([40, 16]), torch.zeros(size - 1, dtype=torch.uint8, device="cuda"))
    ws = spd.alloc_pages_workspace(shape, pages)
    assert ws.numel() == size
    spd.spd_pages_take(shape, refs, indptr, indices, i32([0, 0]), i32([40, 16]), ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    assert indices.tolist() == [5, 4_000_000, pages - 2, pages - 1, -1] and int(refs.sum()) == pages
