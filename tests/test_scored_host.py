"""CPU-side checks of the scored calls and the append with rotation: what the host refuses, before any device is touched."""
import ctypes as C

import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from paper_2409_19134_b200 import build as spd_build
from tests import scored_reference as ref

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    spd_build.build()
    return spd.lib()


def test_struct_layouts(lib):
    assert C.sizeof(spd.Score) == 16 and C.sizeof(spd.Tokens) == 48
    assert C.sizeof(spd.Rope) == 40 and spd.Rope.inv_freq.offset == 32


SHAPE = spd.make_shape(2, 8, 2, 64, torch.bfloat16, 0.125)
P = 0x100000          # an aligned address that nobody reads: every call below is refused on the host


def test_score_options_are_checked(lib):
    kv = spd.PagedKV(P, P, 4, P, P, P)
    part = spd.Partial(P, P, P)
    for cap, window in ((-1.0, 0), (float("nan"), 0), (float("inf"), 0), (1e-38, 0), (0.0, -1)):
        sc = spd.Score(cap, window, None)
        assert lib.spd_decode_step_scored(SHAPE, sc, P, kv, kv, P, 0, 0, P, 1 << 30, None) == INVALID
        assert lib.spd_partial_attn_scored(SHAPE, sc, P, kv, P, part, 0, P, 1 << 30, None) == INVALID
        assert lib.spd_service_attn_merge_scored(SHAPE, sc, P, kv, P, part, P, 0, 0, P, 1 << 30, None) == INVALID
        assert lib.spd_prefill_attn_scored(SHAPE, sc, 4, spd.Tokens(P, P, P, 0, 0, 0), P, None, None, P, 0, P, 1 << 30, None) == INVALID
    sc = spd.Score(0.0, 0, None)
    assert lib.spd_decode_step_scored(SHAPE, None, P, kv, kv, P, 0, 0, P, 1 << 30, None) == INVALID
    assert lib.spd_decode_step_scored(SHAPE, sc, P, kv, None, P, 0, 0, P, 1 << 30, None) == INVALID
    assert lib.spd_decode_step_scored(SHAPE, sc, P, kv, kv, None, 0, 0, P, 1 << 30, None) == INVALID
    assert lib.spd_decode_step_scored(SHAPE, sc, P, kv, kv, P, 0, 3, P, 1 << 30, None) == INVALID        # plan mode
    assert lib.spd_decode_step_scored(SHAPE, sc, P, kv, kv, P, 5, 0, P, 1 << 30, None) == UNSUPPORTED    # output type
    assert lib.spd_partial_attn_scored(SHAPE, sc, P, kv, None, part, 0, P, 1 << 30, None) == INVALID     # lengths of the other half
    assert lib.spd_service_attn_merge_scored(SHAPE, sc, P, kv, None, part, P, 0, 0, P, 1 << 30, None) == INVALID
    odd = spd.make_shape(2, 8, 2, 96, torch.bfloat16, 0.125)
    assert lib.spd_decode_step_scored(odd, sc, P, kv, kv, P, 0, 0, P, 1 << 30, None) == UNSUPPORTED


def test_prefill_arguments_are_checked(lib):
    sc = spd.Score(0.0, 0, None)

    def call(shape=SHAPE, n=4, tok=spd.Tokens(P, P, P, 0, 0, 0), ip=P, out=P, dt=0, ws=P, size=1 << 30):
        return lib.spd_prefill_attn_scored(shape, sc, n, tok, ip, None, None, out, dt, ws, size, None)
    for bad in (dict(n=-1), dict(tok=None), dict(ip=None), dict(out=None), dict(ws=None), dict(ws=P + 16), dict(out=P + 8), dict(n=1 << 31),
                dict(tok=spd.Tokens(None, P, P, 0, 0, 0)), dict(tok=spd.Tokens(P, P + 2, P, 0, 0, 0)),
                dict(tok=spd.Tokens(P, P, P, 8 * 64 - 8, 0, 0)),          # rows would overlap
                dict(tok=spd.Tokens(P, P, P, 0, 2 * 64 + 4, 0))):          # not a multiple of 16 bytes
        assert call(**bad) == INVALID, bad
    assert call(size=16) == WORKSPACE
    assert call(dt=9) == UNSUPPORTED
    for scale in (0.0, -0.5, float("inf")):
        assert call(shape=spd.make_shape(2, 8, 2, 64, torch.bfloat16, scale)) == UNSUPPORTED


def test_append_arguments_are_checked(lib):
    good = dict(rotary_dim=64, interleaved=0, num_axes=1, sections=(C.c_int32 * 4)(), scale=1.0, inv_freq=P)

    def call(rope=good, n=2, tok=spd.Tokens(P, P, P, 0, 0, 0), ip=None, pos=None, base=None, q_out=P + 4096, k_out=None, kp=P, pages=4, indptr=P,
             lens=P, ws=P, size=1 << 30, shape=SHAPE, new_lens=None):
        r = spd.Rope(**rope) if rope is not None else None
        return lib.spd_append_kv_rope(shape, r, n, tok, ip, pos, base, q_out, k_out, kp, P, pages, indptr, P, lens, new_lens, ws, size, None)
    for bad in (dict(n=3), dict(n=-1, ip=P), dict(tok=None), dict(tok=spd.Tokens(P, None, P, 0, 0, 0)), dict(tok=spd.Tokens(None, P, P, 0, 0, 0)),
                dict(q_out=None), dict(kp=None), dict(kp=P + 64), dict(pages=0), dict(indptr=None), dict(lens=None), dict(ws=None),
                dict(pos=P, base=P), dict(rope=dict(good, num_axes=3)), dict(rope=dict(good, inv_freq=None)), dict(rope=dict(good, interleaved=2)),
                dict(rope=dict(good, scale=float("nan"))), dict(rope=dict(good, scale=float("inf"))),
                dict(rope=dict(good, num_axes=3, sections=(C.c_int32 * 4)(16, 8, 9, 0)), pos=P),
                dict(rope=dict(good, num_axes=2, sections=(C.c_int32 * 4)(40, -8, 0, 0)), pos=P),
                dict(tok=spd.Tokens(P, P, P, 8 * 64 + 8, 0, 0), q_out=P),            # in place over strided rows
                dict(tok=spd.Tokens(P, P, P, 0, 2 * 64 + 8, 0), k_out=P),
                dict(base=P + 256, new_lens=P + 256),                                  # lengths written over the positions' base
                dict(ip=P, pos=P + 512, new_lens=P + 512),                             # ... over positions that others still read
                dict(rope=None), dict(rope=None, q_out=None, pos=P), dict(k_out=P + 4)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(rope=dict(good, rotary_dim=80)), dict(rope=dict(good, rotary_dim=24)), dict(rope=dict(good, rotary_dim=0)),
                dict(rope=dict(good, num_axes=5), pos=P), dict(rope=dict(good, num_axes=0))):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(size=1024) == WORKSPACE
    # a workspace that ends where the status query would still clear (flags of 2 users, then tickets of 4 sequences) is too small
    sizes = [n for n in range(0, 1 << 20, 256) if call(size=n, rope=dict(good, rotary_dim=64), k_out=P + 4) == WORKSPACE]
    assert call(size=sizes[-1] + 256, k_out=P + 4) == INVALID
    small, large = spd.make_shape(2, 2, 2, 64, torch.bfloat16, 0.125), spd.make_shape(2, 512, 512, 64, torch.bfloat16, 0.125)
    assert call(size=sizes[-1] + 256, shape=small, k_out=P + 4) == INVALID
    assert call(size=sizes[-1] + 256, shape=large, k_out=P + 4) == WORKSPACE


def test_reference_forms_agree_with_torch():
    """The 64-bit forms that the GPU tests lean on, against torch's own softmax on one dense case."""
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn((9, h, 16), generator=gen) for h in (2, 1, 1))
    out, _ = ref.prefill(q, k, v, [4, 5], 0.25, cap=2.0, window=3, slopes=torch.tensor([0.5, 0.25]), prefix=torch.tensor([0, 3]))
    lo, hi = ref.intervals(5, 3, 3)
    assert lo.tolist() == [0, 0, 0, 1, 2] and hi.tolist() == [2, 2, 2, 3, 4]
    i = torch.arange(5)
    s = 2.0 * torch.tanh(0.25 * q[4:, 1].double() @ k[4:, 0].double().T / 2.0) - 0.25 * (i[:, None] - i).abs()
    s = s.masked_fill((i < lo[:, None]) | (i > hi[:, None]), -torch.inf)
    assert torch.allclose(out[4:, 1], torch.softmax(s, -1) @ v[4:, 0].double())


def test_python_wrappers_refuse_what_the_structs_would_bend():
    """A window beyond 32 bits would wrap; addresses of host tensors would fault."""
    for window in (1 << 31, 1 << 32, -(1 << 32)):
        with pytest.raises(ValueError):
            spd.make_score(window=window)
    for call in (lambda: spd._rows(torch.zeros(5, 2, 64), 2, 64, 5, torch.float32), lambda: spd._i32(torch.zeros(3, dtype=torch.int32), 3),
                 lambda: spd._packed(torch.zeros(8), 8)):
        with pytest.raises(ValueError):
            call()
