"""Scored calls between plain ones on one workspace: the plain calls' shares keep following the measured streaming rates."""
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, setup, workload

pytestmark = pytest.mark.gpu
MAX_GRID = 256


def rate_table(ws):
    """[third][CTA][share weight, cycles] as the launches left them, behind the workspace's header."""
    return ws[256:256 + 3 * MAX_GRID * 8].view(torch.float32).view(3, MAX_GRID, 2).cpu()


@pytest.mark.parametrize("window_layers", [1, 2, 3, 5])
def test_window_layers_between_global_ones(window_layers):
    """One global layer after some with a short window, token after token: every third of the table is written, so each global layer finds
    rates that an earlier one measured."""
    n = [12000 + 16 * u for u in range(8)]
    w = workload(n, [1] * 8, 8, 8, 64, "bf16", seed=1)
    g, shape, near, _, ws = setup(w, 0.0, 64, False)
    out = torch.empty((8, 8, 64), device="cuda")
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for _ in range(6):
        spd.spd_decode_step(shape, g.q, g.priv, g.pub, out, ws)
        for _ in range(window_layers):
            spd.spd_decode_step_scored(shape, near, g.q, g.priv, g.pub, out, ws)
    assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
    table = rate_table(ws)
    assert bool((table[:, :sms] > 0).all())
    want, _, _, _, tol = ref.decode(w, 0.0, 64, None)
    close(out, want, tol, "the last window layer")
