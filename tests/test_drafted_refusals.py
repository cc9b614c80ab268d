"""What the calls for drafted tokens and for pages refuse before any device is touched: the library's own checks, and those of the Python calls
(tensors are stand-ins there, and the library is one that notes the call)."""
import ctypes as C

import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import build as spd_build
from tests.test_scored_refusals import FakePart, FakeStream, FakeTensor, calls  # noqa: F401

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 0x100000          # an aligned address that nobody reads: every call below is refused on the host
SHAPE = spd.make_shape(2, 8, 2, 64, torch.bfloat16, 0.125)


@pytest.fixture(scope="module")
def lib():
    spd_build.build()
    return spd.lib()


def test_struct_and_status(lib):
    assert C.sizeof(spd.Drafts) == 32 and spd.Drafts.sinks.offset == 24
    assert "pages" in spd.status_string(8) and "SPD_ERR_NO_PAGE" in str(spd.SpdError(8, "x"))
    assert set(("spd_decode_step_drafted", "spd_partial_attn_drafted", "spd_service_attn_merge_drafted", "spd_keep_drafted", "spd_pages_take",
                "spd_pages_release", "spd_pages_fork", "spd_pages_copy")) <= set(spd.EXPORTS)


def test_drafted_arguments_are_checked(lib):
    sc, kv, part = spd.Score(0.0, 0, None), spd.PagedKV(P, P, 4, P, P, P), spd.Partial(P, P, P)

    def every(code, shape=SHAPE, score=sc, drafts=spd.Drafts(5, P, P, 0), q=P, kv=kv, lens=P, part=part, out=P, dt=0, ws=P, only=None):
        got = {"fused": lambda: lib.spd_decode_step_drafted(shape, score, drafts, q, kv, kv, out, dt, ws, 1 << 40, None),
               "private": lambda: lib.spd_partial_attn_drafted(shape, score, drafts, q, kv, lens, part, ws, 1 << 40, None),
               "public": lambda: lib.spd_service_attn_merge_drafted(shape, score, drafts, q, kv, lens, part, out, dt, ws, 1 << 40, None)}
        for name, call in got.items():
            if only is None or name in only:
                assert call() == code, name
    every(INVALID, drafts=None)
    every(INVALID, drafts=spd.Drafts(-1, P, None, 0))
    every(INVALID, drafts=spd.Drafts(1 << 31, P, None, 0))
    every(INVALID, drafts=spd.Drafts(5, None, None, 0))                  # five tokens of two users
    every(INVALID, drafts=spd.Drafts(5, P, None, -1))
    every(INVALID, score=None)
    for cap, window in ((-1.0, 0), (float("nan"), 0), (0.0, -1)):
        every(INVALID, score=spd.Score(cap, window, None))
    every(INVALID, score=spd.Score(0.0, 0, P + 2))
    every(INVALID, q=None)
    every(INVALID, q=P + 8)
    every(INVALID, ws=None)
    every(INVALID, ws=P + 16)
    every(INVALID, kv=None)
    every(INVALID, kv=spd.PagedKV(P, P, -1, P, P, P))
    every(INVALID, kv=spd.PagedKV(P + 64, P, 4, P, P, P))
    every(INVALID, kv=spd.PagedKV(P, None, 4, P, P, P))
    every(INVALID, kv=spd.PagedKV(P, P, 4, None, P, P))
    every(INVALID, kv=spd.PagedKV(P, P, 4, P, P, None))
    every(UNSUPPORTED, kv=spd.PagedKV(P, P, 1 << 27, P, P, P))
    every(INVALID, lens=None, only=("private", "public"))
    every(INVALID, part=spd.Partial(None, P, P), only=("private", "public"))
    every(INVALID, part=spd.Partial(P + 8, P, P), only=("private", "public"))
    every(INVALID, part=spd.Partial(P, P + 2, P), only=("private", "public"))
    every(INVALID, out=None, only=("fused", "public"))
    every(INVALID, out=P + 8, only=("fused", "public"))
    every(UNSUPPORTED, dt=7, only=("fused", "public"))
    for bad, code in ((spd.make_shape(2, 8, 2, 96, torch.bfloat16, 0.125), UNSUPPORTED), (spd.make_shape(0, 8, 2, 64, torch.bfloat16, 0.125), INVALID),
                      (spd.make_shape(2, 9, 2, 64, torch.bfloat16, 0.125), UNSUPPORTED), (spd.make_shape(2, 8, 2, 64, torch.bfloat16, -1.0), UNSUPPORTED),
                      (spd.make_shape(2, 8, 2, 64, torch.bfloat16, float("nan")), INVALID), (spd.make_shape(2, 8, 2, 64, torch.bfloat16, 0.125, page_size=32), UNSUPPORTED)):
        every(code, shape=bad)
    n = C.c_size_t(0)
    assert lib.spd_drafted_workspace_size(SHAPE, None) == INVALID
    assert lib.spd_drafted_workspace_size(spd.make_shape(2, 8, 2, 96, torch.bfloat16, 1.0), C.byref(n)) == UNSUPPORTED


def test_pages_arguments_are_checked(lib):
    size = 1 << 40

    def table(name, n=8, refs=P, ip=P, ix=P, a=P, b=P, c=P, ws=P, size=size, shape=SHAPE):
        f = getattr(lib, "spd_pages_" + name)
        return f(shape, n, refs, ip, ix, a, b, c, ws, size, None) if name == "fork" else f(shape, n, refs, ip, ix, a, b, ws, size, None)
    for name in ("take", "release", "fork"):
        for bad in (dict(n=-1), dict(n=(1 << 30) + 1), dict(refs=None), dict(refs=P + 4), dict(ip=None), dict(ix=None), dict(a=None), dict(ws=None), dict(ws=P + 64)):
            assert table(name, **bad) == INVALID, (name, bad)
        assert table(name, size=256) == WORKSPACE
        assert table(name, n=1 << 24, size=1 << 24) == WORKSPACE             # four bytes per page
        assert table(name, shape=spd.make_shape(2, 8, 3, 64, torch.bfloat16, 1.0)) == UNSUPPORTED
    assert table("take", b=None) == INVALID and table("fork", b=None) == INVALID and table("fork", c=None) == INVALID
    pools = (C.c_void_p * 2)(P, P)

    def copy(n=2, pools=pools, pages=8, m=3, pairs=P, ws=P, size=size, shape=SHAPE):
        return lib.spd_pages_copy(shape, n, pools, pages, m, pairs, ws, size, None)
    for bad in (dict(n=-1), dict(pools=None), dict(pools=(C.c_void_p * 2)(P, None)), dict(pools=(C.c_void_p * 2)(P, P + 64)), dict(pages=-1), dict(m=-1),
                dict(pairs=None), dict(ws=None), dict(ws=P + 64)):
        assert copy(**bad) == INVALID, bad
    assert copy(size=16) == WORKSPACE

    def keep(T=5, ip=P, up=P + 256, last=P + 512, n=2, pools=pools, pages=8, pi=P, px=P, lens=P + 1024, new=P + 1024, kept=None, ws=P, size=size, shape=SHAPE):
        return lib.spd_keep_drafted(shape, T, ip, up, last, n, pools, pages, pi, px, lens, new, kept, ws, size, None)
    for bad in (dict(T=-1), dict(T=1 << 31), dict(ip=None), dict(last=None), dict(n=-1), dict(pools=None), dict(pools=(C.c_void_p * 2)(None, P)), dict(pages=-1),
                dict(pi=None), dict(lens=None), dict(ws=None), dict(ws=P + 64), dict(kept=P), dict(kept=P + 256), dict(kept=P + 512), dict(kept=P + 1024),
                dict(new=P), dict(new=P + 512), dict(new=P + 2048, kept=P + 2048)):
        assert keep(**bad) == INVALID, bad
    assert keep(size=16) == WORKSPACE


# ---- the Python calls
B, HQ, HKV, D, BF16, T = 3, 8, 2, 64, torch.bfloat16, 6
FAKE = spd.make_shape(B, HQ, HKV, D, BF16, 0.125)
I32 = dict(dtype=torch.int32)


def part():
    return FakePart(B, 5, HKV, D, BF16)


def fused(**kw):
    a = dict(dict(score=spd.make_score(), q=FakeTensor(T, HQ, D, dtype=BF16), priv=part(), pub=part(), out=FakeTensor(T, HQ, D), ws=FakeTensor(1 << 20, dtype=torch.uint8),
                  tok_indptr=FakeTensor(B + 1, **I32), parents=FakeTensor(T, **I32), sinks=0), **kw)
    spd.spd_decode_step_drafted(FAKE, a["score"], a["q"], a["priv"], a["pub"], a["out"], a["ws"], tok_indptr=a["tok_indptr"], parents=a["parents"], sinks=a["sinks"],
                                stream=FakeStream)


def halves(**kw):
    a = dict(dict(q=FakeTensor(T, HQ, D, dtype=BF16), kv=part(), lens=FakeTensor(B, **I32), part=[FakeTensor(T, HQ, D), FakeTensor(T, HQ), FakeTensor(T, HQ)],
                  out=FakeTensor(T, HQ, D), ws=FakeTensor(1 << 20, dtype=torch.uint8)), **kw)
    sc, ip = spd.make_score(), FakeTensor(B + 1, **I32)
    spd.spd_partial_attn_drafted(FAKE, sc, a["q"], a["kv"], a["lens"], a["part"], a["ws"], tok_indptr=ip, stream=FakeStream)
    spd.spd_service_attn_merge_drafted(FAKE, sc, a["q"], a["kv"], a["lens"], a["part"], a["out"], a["ws"], tok_indptr=ip, stream=FakeStream)


def test_python_drafted_calls_check_their_tensors(calls):  # noqa: F811
    fused()
    halves()
    assert calls == ["spd_decode_step_drafted", "spd_partial_attn_drafted", "spd_service_attn_merge_drafted"]
    del calls[:]
    q, p = FakeTensor(T, HQ, D, dtype=BF16), part()
    for bad in (dict(q=q.but(dtype=torch.float32)), dict(q=q.but(shape=(T, HQ - 1, D))), dict(q=q.but(dev=-1)), dict(q=q.but(dev=1)),
                dict(q=q.but(strides=(2 * HQ * D, D, 1))), dict(out=FakeTensor(T, HQ, D - 1)), dict(out=FakeTensor(T, HQ, D, dev=1)),
                dict(tok_indptr=FakeTensor(B, **I32)), dict(tok_indptr=FakeTensor(B + 1, dtype=torch.int64)), dict(tok_indptr=FakeTensor(B + 1, dev=-1, **I32)),
                dict(tok_indptr=None), dict(parents=FakeTensor(T - 1, **I32)), dict(parents=FakeTensor(T, dtype=torch.int64)), dict(parents=FakeTensor(T, dev=1, **I32)),
                dict(sinks=-1), dict(sinks=1 << 31), dict(ws=FakeTensor(1 << 20)), dict(ws=FakeTensor(1 << 20, dtype=torch.uint8, dev=1)),
                dict(priv=p.but(seq_lens=FakeTensor(B + 1, **I32))), dict(pub=p.but(k_pool=p.k_pool.but(dtype=torch.float32))),
                dict(pub=p.but(v_pool=p.v_pool.but(dev=1)))):
        with pytest.raises(ValueError):
            fused(**bad)
    for bad in (dict(lens=FakeTensor(T, **I32)), dict(lens=FakeTensor(B, dev=1, **I32)), dict(part=[FakeTensor(B, HQ, D), FakeTensor(T, HQ), FakeTensor(T, HQ)]),
                dict(part=[FakeTensor(T, HQ, D, dtype=BF16), FakeTensor(T, HQ), FakeTensor(T, HQ)])):
        with pytest.raises(ValueError):
            halves(**bad)
    assert calls == []


def test_python_page_calls_check_their_tensors(calls):  # noqa: F811
    pool = FakeTensor(7, HKV, 16, D, dtype=BF16)
    refs, ip, ix, u = FakeTensor(7, **I32), FakeTensor(B + 1, **I32), FakeTensor(9, **I32), FakeTensor(B, **I32)
    pairs, ws = FakeTensor(4, 2, **I32), FakeTensor(1 << 20, dtype=torch.uint8)
    fine = dict(refs=refs, ip=ip, ix=ix, a=u, b=u, pairs=FakeTensor(B, 2, **I32), ws=ws)

    def every(**kw):
        a = dict(fine, **kw)
        yield lambda: spd.spd_pages_take(FAKE, a["refs"], a["ip"], a["ix"], a["a"], a["b"], a["ws"], stream=FakeStream)
        yield lambda: spd.spd_pages_release(FAKE, a["refs"], a["ip"], a["ix"], a["a"], a["ws"], to_tokens=a["b"], stream=FakeStream)
        yield lambda: spd.spd_pages_fork(FAKE, a["refs"], a["ip"], a["ix"], a["a"], a["b"], a["pairs"], a["ws"], stream=FakeStream)
    for call in every():
        call()
    spd.spd_pages_copy(FAKE, [pool, pool], pairs, ws, stream=FakeStream)
    spd.spd_keep_drafted(FAKE, spd.make_pools(FAKE, [pool]), FakePart(B, 7, HKV, D, BF16), ip, u, ws, parents=FakeTensor(T, **I32), kept=FakeTensor(T, **I32),
                         stream=FakeStream)
    assert calls == ["spd_pages_take", "spd_pages_release", "spd_pages_fork", "spd_pages_copy", "spd_keep_drafted"]
    del calls[:]
    for bad in (dict(refs=refs.but(dtype=torch.int64)), dict(refs=refs.but(dev=-1)), dict(refs=refs.but(strides=(2,))), dict(ip=FakeTensor(B, **I32)),
                dict(ix=ix.but(dtype=torch.int64)), dict(ix=ix.but(dev=1)), dict(a=FakeTensor(B + 1, **I32)), dict(a=u.but(dev=-1)), dict(b=u.but(dtype=torch.int64)),
                dict(ws=FakeTensor(1 << 20))):
        for call in every(**bad):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        spd.spd_pages_fork(FAKE, refs, ip, ix, u, u, FakeTensor(B, 3, **I32), ws, stream=FakeStream)
    for pools in ([pool, pool.but(dtype=torch.float32)], [pool, pool.but(shape=(6, HKV, 16, D))], [pool, pool.but(dev=1)], [pool.but(strides=(4096, 1024, 64, 2))],
                  [pool.but(shape=(7, 1, 16, D))]):
        with pytest.raises(ValueError):
            spd.spd_pages_copy(FAKE, pools, pairs, ws, stream=FakeStream)
    with pytest.raises(ValueError):
        spd.spd_pages_copy(spd.make_shape(B, HQ, 1, D, BF16, 1.0), spd.make_pools(FAKE, [pool]), pairs, ws, stream=FakeStream)      # made for another shape
    keep = dict(part=FakePart(B, 7, HKV, D, BF16), ip=ip, last=u, parents=FakeTensor(T, **I32), kept=FakeTensor(T, **I32), new="in place")
    for bad in (dict(last=FakeTensor(T, **I32)), dict(last=u.but(dev=1)), dict(kept=FakeTensor(T + 1, **I32)), dict(parents=FakeTensor(T, dtype=torch.int64)),
                dict(ip=FakeTensor(B, **I32)), dict(new=FakeTensor(T, **I32)), dict(parents=None, kept=None)):
        a = dict(keep, **bad)
        with pytest.raises(ValueError):
            spd.spd_keep_drafted(FAKE, [pool], a["part"], a["ip"], a["last"], ws, parents=a["parents"], kept=a["kept"], new_lens=a["new"], stream=FakeStream)
    assert calls == []


@pytest.mark.parametrize("other", [spd.make_shape(B, HQ, HKV // 2, 2 * D, BF16, 1.0), spd.make_shape(B, HQ, 2 * HKV, D, BF16, 1.0),
                                   spd.make_shape(B, HQ, HKV, D, torch.float32, 1.0)])
def test_pools_made_for_other_rows_are_refused(calls, other):  # noqa: F811
    """Pages of as many elements, cut into other heads."""
    handle, u = spd.make_pools(FAKE, [FakeTensor(7, HKV, 16, D, dtype=BF16)]), FakeTensor(B, **I32)
    ws, pairs = FakeTensor(1 << 20, dtype=torch.uint8), FakeTensor(4, 2, **I32)
    spd.spd_pages_copy(FAKE, handle, pairs, ws, stream=FakeStream)
    assert calls == ["spd_pages_copy"]
    with pytest.raises(ValueError):
        spd.spd_pages_copy(other, handle, pairs, ws, stream=FakeStream)
    with pytest.raises(ValueError):
        spd.spd_keep_drafted(other, handle, FakePart(B, 7, HKV, D, BF16), FakeTensor(B + 1, **I32), u, ws, parents=FakeTensor(T, **I32), stream=FakeStream)
    assert calls == ["spd_pages_copy"]


def test_pages_workspace_size_checks_its_arguments(lib):
    n = C.c_size_t(0)
    assert "spd_pages_workspace_size" in spd.EXPORTS
    assert lib.spd_pages_workspace_size(SHAPE, 8, None) == INVALID and lib.spd_pages_workspace_size(None, 8, C.byref(n)) == INVALID
    assert lib.spd_pages_workspace_size(SHAPE, -1, C.byref(n)) == INVALID and lib.spd_pages_workspace_size(SHAPE, (1 << 30) + 1, C.byref(n)) == INVALID
    assert lib.spd_pages_workspace_size(spd.make_shape(2, 8, 3, 64, torch.bfloat16, 1.0), 8, C.byref(n)) == UNSUPPORTED
