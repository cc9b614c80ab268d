"""Scored calls where a visible key scores minus infinity, and prompts whose V rows are spoiled or huge."""
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close
from tests.test_gpu_prefill_scored import P_WEIGHT, prompts, run

pytestmark = pytest.mark.gpu


def shut_out(q, k, keys):
    """Gives the keys a score of minus infinity with every query: one channel of theirs is infinite, where all queries are negative."""
    q[..., 0] = -q[..., 0].abs() - 0.125
    k[keys] = 0
    k[keys, :, 0] = float("inf")


@pytest.mark.parametrize("spoiled", [False, True])
@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 2, 1), ("bf16", 64, 1, 1), ("f32", 64, 2, 2)])
def test_prompt_keys_that_score_minus_infinity_weigh_nothing(dtype, d, hq, hkv, spoiled):
    """The first key (and one further on) is visible but weighs nothing: rows are as if they did not see it; a row that sees nothing else is
    zero.  With a spoiled V row in the prompt, which sends the rows of its tile through their keys one by one, too."""
    n = 300
    q, k, v, ip = prompts([n], hq, hkv, d, dtype, seed=90)
    shut_out(q, k, [0])
    if spoiled:
        v[150] = float("nan")
    want, tol = ref.prefill(q, k, v, [n], d ** -0.5, doc=torch.ones(n, dtype=torch.int32), weight=P_WEIGHT[dtype])
    out, status = run(q, k, v, ip, d)
    assert status == (spd.SPD_OK, -1)
    good = 150 if spoiled else n
    close(out[:good], want[:good], tol[:good], "keys of no weight")
    assert bool((out[0] == 0).all()) and bool(out[good:].isnan().all())
