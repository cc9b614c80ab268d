"""Capped prompts whose weights sit on few keys: rounding the weights to bf16 must not show where the values that they average agree."""
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import scored_reference as ref
from tests.test_gpu_prefill_scored import prompts, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap", [8.0, 30.0, 50.0])
@pytest.mark.parametrize("d,hq,hkv", [(128, 2, 1), (64, 1, 1)])
def test_rounded_weights_are_summed_as_they_are_used(d, hq, hkv, cap):
    """With the same rounded weights w (1 + e), |e| <= 2^-8, above and below, the output is off by sum w e (v - out) / sum w (1 + e), at most
    2^-8 / (1 - 2^-8) sum p |v - out|; and by what the scores' own errors make of it, as elsewhere."""
    n = 260
    q, k, v, ip = prompts([n], hq, hkv, d, "bf16", seed=96, qscale=6.0)
    v.add_(4.0)                                              # values that agree to a quarter
    want, tol = ref.prefill(q, k, v, [n], d ** -0.5, cap)
    out, status = run(q, k, v, ip, d, cap=cap)
    assert status == (spd.SPD_OK, -1)
    got = out.cpu().double()
    for i in range(n):
        for h in range(hq):
            kk, vv = k[:i + 1, h // (hq // hkv)].double(), v[:i + 1, h // (hq // hkv)].double()
            s = ref.scores(q[i, h].double(), kk, d ** -0.5, cap, 0.0, torch.zeros(i + 1).double())
            p = torch.softmax(s, 0)
            lim = p @ (vv - want[i, h]).abs() * (2.0 ** -8 / (1 - 2.0 ** -8)) + tol[i, h]
            assert bool(((got[i, h] - want[i, h]).abs() <= lim).all()), (i, h)
