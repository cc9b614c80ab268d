"""What the Python calls refuse before an address reaches the library: pools, tables, lengths, partials and workspaces that do not fit the
shape, and tensors that are not on the device the call runs on.  No GPU: tensors are stand-ins, and the library is one that notes the call."""
import math

import pytest
import torch

from paper_2409_19134_b200 import binding as spd


class FakeTensor:
    """As much of a tensor as the wrappers look at; device -1 is the host."""

    def __init__(self, *shape, dtype=torch.float32, dev=0, strides=None):
        self.shape, self.dtype, self._dev = torch.Size(shape), dtype, dev
        self._strides = strides or tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))
        self.is_cuda, self.device = dev >= 0, torch.device("cuda", dev) if dev >= 0 else torch.device("cpu")

    def but(self, **kw):
        return FakeTensor(*kw.pop("shape", self.shape), **dict(dict(dtype=self.dtype, dev=self._dev), **kw))

    def numel(self):
        return math.prod(self.shape)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._strides

    def is_contiguous(self):
        return self._strides == FakeTensor(*self.shape)._strides if self.shape else True

    def get_device(self):
        return self._dev

    def data_ptr(self):
        return 0x100000 if self.numel() else 0


class FakePart:
    def __init__(self, B, pages, hkv, d, dtype, listed=4):
        i32 = dict(dtype=torch.int32)
        self.k_pool, self.v_pool = FakeTensor(pages, hkv, 16, d, dtype=dtype), FakeTensor(pages, hkv, 16, d, dtype=dtype)
        self.page_indptr, self.page_indices, self.seq_lens = FakeTensor(B + 1, **i32), FakeTensor(listed, **i32), FakeTensor(B, **i32)

    def but(self, **kw):
        p = FakePart.__new__(FakePart)
        p.__dict__.update(self.__dict__, **kw)
        return p


@pytest.fixture
def calls(monkeypatch):
    """Names of the library functions that were reached."""
    reached = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0
    monkeypatch.setattr(spd, "lib", lambda: Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return reached


class FakeStream:
    cuda_stream = 0


B, HQ, HKV, D, BF16 = 3, 8, 2, 64, torch.bfloat16
SHAPE = spd.make_shape(B, HQ, HKV, D, BF16, 0.125)
I32 = dict(dtype=torch.int32)


def part():
    return FakePart(B, 5, HKV, D, BF16)


def bad_parts():
    p = part()
    yield "pool of another type", p.but(k_pool=p.k_pool.but(dtype=torch.float32), v_pool=p.v_pool.but(dtype=torch.float32))
    yield "v pool of another type", p.but(v_pool=p.v_pool.but(dtype=torch.float32))
    yield "fewer kv heads", p.but(k_pool=p.k_pool.but(shape=(5, 1, 16, D)), v_pool=p.v_pool.but(shape=(5, 1, 16, D)))
    yield "smaller head_dim", p.but(k_pool=p.k_pool.but(shape=(5, HKV, 16, 32)), v_pool=p.v_pool.but(shape=(5, HKV, 16, 32)))
    yield "fewer v pages", p.but(v_pool=p.v_pool.but(shape=(4, HKV, 16, D)))
    yield "strided pool", p.but(k_pool=p.k_pool.but(strides=(2 * HKV * 16 * D, 16 * D, D, 1)))
    yield "short lengths", p.but(seq_lens=FakeTensor(B - 1, **I32))
    yield "short table", p.but(page_indptr=FakeTensor(B, **I32))
    yield "64-bit lengths", p.but(seq_lens=FakeTensor(B, dtype=torch.int64))
    yield "64-bit pages", p.but(page_indices=FakeTensor(4, dtype=torch.int64))
    yield "strided lengths", p.but(seq_lens=FakeTensor(B, strides=(2,), **I32))
    for dev in (-1, 1):
        for name in ("k_pool", "v_pool", "page_indptr", "page_indices", "seq_lens"):
            yield f"{name} on device {dev}", p.but(**{name: getattr(p, name).but(dev=dev)})


def fused(**kw):
    a = dict(dict(score=spd.make_score(), q=FakeTensor(B, HQ, D, dtype=BF16), priv=part(), pub=part(), out=FakeTensor(B, HQ, D),
                  ws=FakeTensor(1 << 20, dtype=torch.uint8)), **kw)
    spd.spd_decode_step_scored(SHAPE, a["score"], a["q"], a["priv"], a["pub"], a["out"], a["ws"], stream=FakeStream)


def partial():
    return [FakeTensor(B, HQ, D), FakeTensor(B, HQ), FakeTensor(B, HQ)]


def private_half(**kw):
    a = dict(dict(score=spd.make_score(), q=FakeTensor(B, HQ, D, dtype=BF16), priv=part(), lens=FakeTensor(B, **I32), part=partial(),
                  ws=FakeTensor(1 << 20, dtype=torch.uint8)), **kw)
    spd.spd_partial_attn_scored(SHAPE, a["score"], a["q"], a["priv"], a["lens"], a["part"], a["ws"], stream=FakeStream)


def public_half(**kw):
    a = dict(dict(score=spd.make_score(), q=FakeTensor(B, HQ, D, dtype=BF16), pub=part(), lens=FakeTensor(B, **I32), part=partial(),
                  out=FakeTensor(B, HQ, D), ws=FakeTensor(1 << 20, dtype=torch.uint8)), **kw)
    spd.spd_service_attn_merge_scored(SHAPE, a["score"], a["q"], a["pub"], a["lens"], a["part"], a["out"], a["ws"], stream=FakeStream)


T = 6


def prompts(**kw):
    a = dict(dict(score=spd.make_score(), q=FakeTensor(T, HQ, D, dtype=BF16), k=FakeTensor(T, HKV, D, dtype=BF16), v=FakeTensor(T, HKV, D, dtype=BF16),
                  ip=FakeTensor(B + 1, **I32), out=FakeTensor(T, HQ, D), ws=FakeTensor(1 << 20, dtype=torch.uint8), prefix=FakeTensor(B, **I32),
                  doc=FakeTensor(T, **I32)), **kw)
    spd.spd_prefill_attn_scored(SHAPE, a["score"], a["q"], a["k"], a["v"], a["ip"], a["out"], a["ws"], prefix_lens=a["prefix"], doc_start=a["doc"],
                                stream=FakeStream)


def append(**kw):
    a = dict(dict(rope=spd.make_rope(FakeTensor(32)), q=FakeTensor(T, HQ, D, dtype=BF16), k=FakeTensor(T, HKV, D, dtype=BF16),
                  v=FakeTensor(T, HKV, D, dtype=BF16), part=part(), ws=FakeTensor(1 << 20, dtype=torch.uint8), q_out=FakeTensor(T, HQ, D, dtype=BF16),
                  k_out=FakeTensor(T, HKV, D, dtype=BF16), ip=FakeTensor(B + 1, **I32), pos=None, base=FakeTensor(B, **I32), new=FakeTensor(B, **I32)), **kw)
    spd.spd_append_kv_rope(SHAPE, a["rope"], a["q"], a["k"], a["v"], a["part"], a["ws"], q_out=a["q_out"], k_out=a["k_out"], tok_indptr=a["ip"],
                           positions=a["pos"], pos_base=a["base"], new_lens=a["new"], stream=FakeStream)


ALL = {fused: "spd_decode_step_scored", private_half: "spd_partial_attn_scored", public_half: "spd_service_attn_merge_scored",
       prompts: "spd_prefill_attn_scored", append: "spd_append_kv_rope"}


@pytest.mark.parametrize("call", ALL, ids=lambda f: f.__name__)
def test_fitting_tensors_reach_the_library(call, calls):
    call()
    assert calls == [ALL[call]]


@pytest.mark.parametrize("what", [name for name, _ in bad_parts()])
@pytest.mark.parametrize("call,which", [(fused, "priv"), (fused, "pub"), (private_half, "priv"), (public_half, "pub"), (append, "part")],
                         ids=lambda x: x if isinstance(x, str) else x.__name__)
def test_partitions_that_do_not_fit_the_shape_are_refused(call, which, what, calls):
    with pytest.raises(ValueError):
        call(**{which: dict(bad_parts())[what]})
    assert not calls


@pytest.mark.parametrize("call", [private_half, public_half], ids=lambda f: f.__name__)
def test_partials_that_do_not_fit_are_refused(call, calls):
    for i in range(3):
        good = partial()[i]
        for bad in (good.but(dev=-1), good.but(dev=1), good.but(dtype=BF16), good.but(shape=(B - 1, *good.shape[1:])),
                    good.but(strides=tuple(2 * s for s in good.stride()))):
            with pytest.raises(ValueError):
                call(part=[bad if j == i else t for j, t in enumerate(partial())])
    assert not calls


@pytest.mark.parametrize("dev", [-1, 1])
@pytest.mark.parametrize("call,names", [(fused, "q out ws"), (private_half, "q lens ws"), (public_half, "q lens out ws"),
                                        (prompts, "q k v ip out ws prefix doc"), (append, "q k v ws q_out k_out ip base new")],
                         ids=lambda x: "" if isinstance(x, str) else x.__name__)
def test_tensors_of_another_device_are_refused(call, names, dev, calls):
    for name in names.split():
        t = {"q": FakeTensor(B, HQ, D, dtype=BF16) if call in (fused, private_half, public_half) else FakeTensor(T, HQ, D, dtype=BF16),
             "k": FakeTensor(T, HKV, D, dtype=BF16), "v": FakeTensor(T, HKV, D, dtype=BF16), "ip": FakeTensor(B + 1, **I32),
             "out": FakeTensor(T, HQ, D) if call is prompts else FakeTensor(B, HQ, D), "ws": FakeTensor(1 << 20, dtype=torch.uint8),
             "lens": FakeTensor(B, **I32), "prefix": FakeTensor(B, **I32), "doc": FakeTensor(T, **I32), "q_out": FakeTensor(T, HQ, D, dtype=BF16),
             "k_out": FakeTensor(T, HKV, D, dtype=BF16), "base": FakeTensor(B, **I32), "new": FakeTensor(B, **I32)}[name]
        call(**{name: t})
        assert calls.pop() == ALL[call], name
        with pytest.raises(ValueError):
            call(**{name: t.but(dev=dev)})
        assert not calls, name


def test_options_on_another_device_or_of_another_size_are_refused(calls):
    for call in (fused, private_half, public_half, prompts):
        call(score=spd.make_score(alibi_slopes=FakeTensor(HQ)))
        assert calls.pop() == ALL[call]
        for slopes in (FakeTensor(HQ - 1), FakeTensor(HQ, dev=1)):
            with pytest.raises(ValueError):
                call(score=spd.make_score(alibi_slopes=slopes))
    with pytest.raises(ValueError):
        append(rope=spd.make_rope(FakeTensor(32, dev=1)))
    for bad in (FakeTensor(HQ, dev=-1), FakeTensor(HQ, dtype=torch.float64), FakeTensor(HQ, strides=(2,))):
        with pytest.raises(ValueError):
            spd.make_score(alibi_slopes=bad)
        with pytest.raises(ValueError):
            spd.make_rope(bad)
    with pytest.raises(ValueError):
        spd.make_rope(FakeTensor(4, 8))
    with pytest.raises(ValueError):
        fused(ws=FakeTensor(1 << 18, dtype=torch.float32))
    assert not calls
