"""Capped scores of drafted tokens over the whole range of caps, with error bounds relative to the scores where the cap is far above them, and
rows whose bits must not depend on what lies beside them."""
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import drafted_reference as dr
from tests import scored_reference as ref

pytestmark = pytest.mark.gpu


def ok(d):
    assert spd.spd_query_device_status(d.ws) == (spd.SPD_OK, -1)


# The cap's own error.  Caps that the polynomials' coefficients carry (up to about 200 at head_dim 128 and 300 at 64, with the scale of these batches): 2^-21 of the
# cap, as a maximum or a block with greater scores goes by the special-function unit.  Larger ones: an odd polynomial that is off by 3.2e-6 of
# the score, and five roundings of 2^-24, below 2^-18 of the score; beyond the cap itself 2^-21 of it.
def cap_error(cap, S):
    return 2.0 ** -21 * cap if cap < 300 else min(2.0 ** -21 * cap, 2.0 ** -18 * S)


def score_error(D, S, cap, bias):
    return D * 2.0 ** -24 * S + cap_error(cap, S) + 2.0 ** -23 * bias


def bound(vmax, D, S, n, cap, bias, weight):
    return (2.0 * (score_error(D, S, cap, bias) + 2.0 ** -21 + n * 2.0 ** -24) + weight) * vmax


@pytest.mark.parametrize("cap", [0.01, 20.0, 150.0, 210.0, 300.0, 1e3, 1e4, 1e5, 1e6, 1e8, 1e30])
@pytest.mark.parametrize("d,kind,window", [(64, "tree", 0), (64, "run", 130), (128, "tree", 100), (128, "run", 0)])
@pytest.mark.parametrize("alibi", [False, True])
def test_caps_over_their_range(cap, d, kind, window, alibi, monkeypatch):
    """Scores from far below every cap to far above the small ones, side by side in a tile; blocks seen whole and blocks with masks."""
    w = dr.batch([9, 40, 3], [400, 170, 90], [37, 20, 0], 4, 2, d, "bf16", seed=d, kind=kind)
    w.q *= torch.logspace(-2, 1.5, 52)[torch.randperm(52, generator=torch.Generator().manual_seed(1))][:, None, None].bfloat16()
    g = dr.OnDevice(w, cap, window, 5 if window else 0, alibi)
    args = cap, window, 5 if window else 0, g.slopes

    monkeypatch.setattr(ref, "bound", bound)
    want, _, _, _, tol = dr.expected(w, *args)
    dr.close(g.fused(), want, tol, "fused")
    out, part = g.halves()
    dr.close(out, want, tol, "halves")
    ok(g)
    # the private half's maxima say how exact the scores are, without the rounding of the weights; 2^-22: there and back between natural and log2 units
    monkeypatch.setattr(ref, "bound", lambda vmax, D, S, n, cap, bias, weight: score_error(D, S, cap, bias))
    _, _, m, l, err = dr.expected(w, *args, parts=(True, False))
    seen = l > 0
    assert bool(((part[1].cpu().double() - m).abs()[seen] <= (err + 2.0 ** -22 * m.abs())[seen]).all())


@pytest.mark.parametrize("alibi", [False, True])
def test_huge_caps_change_nothing(alibi, monkeypatch):
    """At 1e8 a score is capped by less than its own rounding."""
    w = dr.batch([9, 40], [400, 170], [37, 20], 4, 2, 128, "bf16", seed=3)
    monkeypatch.setattr(ref, "bound", bound)
    outs, tols = [], []
    for cap in (0.0, 1e8):
        g = dr.OnDevice(w, cap, 0, 0, alibi)
        outs.append(g.fused())
        tols.append(dr.expected(w, cap, 0, 0, g.slopes)[4])
        ok(g)
    dr.close(outs[1], outs[0].cpu().double(), tols[0] + tols[1])


@pytest.mark.parametrize("kind,window", [("tree", 0), ("run", 90)])
def test_scales_that_leave_nothing_of_the_quotient(kind, window, monkeypatch):
    """sm_scale / cap below fp32's range: scores of ordinary size stay what they are without a cap."""
    w = dr.batch([9, 40], [400, 170], [37, 20], 4, 2, 64, "bf16", seed=4, kind=kind)
    w.sm_scale, w.q = 1e-20, (w.q.float() * 1e19).bfloat16()
    g = dr.OnDevice(w, 1e30, window)
    monkeypatch.setattr(ref, "bound", bound)
    want, _, _, _, tol = dr.expected(w, 1e30, window)
    dr.close(g.fused(), want, tol)
    ok(g)


def capped(w, cap=20.0, window=0):
    g = dr.OnDevice(w, cap, window)
    out = g.fused()
    ok(g)
    return out


@pytest.mark.parametrize("kind,window", [("tree", 0), ("run", 0), ("run", 60)])
@pytest.mark.parametrize("cap", [20.0, 1e4])
def test_a_neighbour_does_not_choose_the_arithmetic(kind, window, cap):
    """A tile's rows behind a user's last token hold the next user's q: whatever it is, the first user's bits stay."""
    outs = []
    for scale in (0.01, 1.0, 1e3, float("nan")):
        w = dr.batch([5, 30], [400, 200], [9, 3], 8, 2, 128, "bf16", seed=17, kind=kind)
        w.q[5:] *= scale
        outs.append(capped(w, cap, window)[:5])
    assert all(torch.equal(outs[0], x) for x in outs[1:])


def test_what_shared_memory_held_chooses_no_arithmetic():
    """Groups of 24 leave 8 rows of a tile without a query: whatever an earlier call left there, the bits stay."""
    w = dr.batch([5, 3], [400, 200], [9, 3], 24, 1, 64, "bf16", seed=18)
    outs = []
    for scale in (0.01, 1e3, float("nan")):
        other = dr.batch([64, 64], [9000, 9000], [0, 0], 4, 1, 64, "bf16", seed=19, kind="run")      # all rows of both tiles, on every SM
        other.q *= scale
        dr.OnDevice(other).fused()
        outs.append(capped(w))
    assert all(torch.equal(outs[0], x) for x in outs[1:])
