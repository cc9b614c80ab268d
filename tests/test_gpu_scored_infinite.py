"""Scored calls where a visible key scores minus infinity, and prompts whose V rows are spoiled or huge."""
import pytest
import torch

from paper_2409_19134_b200 import binding as spd
from tests import scored_reference as ref
from tests.test_gpu_decode_scored import close, setup, workload
from tests.test_gpu_decode_scored import kernel  # noqa: F401
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


def decode_job(dtype, d, hq, hkv):
    """Two users of 320 tokens whose first 40 score minus infinity: 40 of 300 private ones; all 20 private and 20 of 300 public ones."""
    w = workload([300, 20], [20, 300], hq, hkv, d, dtype, seed=91)
    w.q[..., 0] = -w.q[..., 0].abs() - 0.125
    for u in range(2):
        for part, base, m in ((w.priv, 0, (300, 20)[u]), (w.pub, (300, 20)[u], (20, 300)[u])):
            for t in range(m):
                if base + t < 40:
                    page = int(part.page_indices[int(part.page_indptr[u]) + t // 16])
                    part.k_pool[page, :, t % 16] = 0
                    part.k_pool[page, :, t % 16, 0] = float("inf")
    want, O, m, l, tol = ref.decode(w, window=280)          # as if the 40 were out of sight
    return setup(w, 0.0, 0, False), want, tol


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 2, 2), ("f32", 128, 2, 1), ("f32", 64, 8, 1)])
def test_decode_keys_that_score_minus_infinity_weigh_nothing(kernel, dtype, d, hq, hkv):  # noqa: F811
    """Whole tiles, pieces and a whole partition of such keys, in front of others that count."""
    (g, shape, score, _, ws), want, tol = decode_job(dtype, d, hq, hkv)
    for share in ((0,) if kernel == "short" else (3, 1)):
        spd.spd_set_split(share, False)
        out = torch.full((2, hq, d), float("nan"), device="cuda")
        spd.spd_decode_step_scored(shape, score, g.q, g.priv, g.pub, out, ws)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        close(out, want, tol, ("fused", share))
        part = spd.alloc_partial(shape)
        spd.spd_partial_attn_scored(shape, score, g.q, g.priv, g.pub.seq_lens, part, ws)
        assert bool((part[0][1] == 0).all()) and bool((part[1][1] == -float("inf")).all()) and bool((part[2][1] == 0).all())
        out = torch.full((2, hq, d), float("nan"), device="cuda")
        spd.spd_service_attn_merge_scored(shape, score, g.q, g.pub, g.priv.seq_lens, part, out, ws)
        assert spd.spd_query_device_status(ws) == (spd.SPD_OK, -1)
        close(out, want, 2 * tol, ("halves", share))


@pytest.mark.parametrize("n,d,hq", [(9000, 128, 2), (700001, 64, 1)])
def test_a_spoiled_row_at_the_end_of_a_long_prompt(n, d, hq):
    """The rows of the last tile are done again one by one over all their keys; everybody else waits for them as long as it takes."""
    q, k, v, ip = prompts([n], hq, 1, d, "bf16", seed=92)
    bad = n - 70                                          # the last tile's rows in front of it do not see it
    v[bad] = float("nan")
    out, status = run(q, k, v, ip, d)
    assert status == (spd.SPD_OK, -1)
    rows = {0, 1, 4095, n // 2, n - 300, bad - 20, bad - 1}
    want, tol = ref.prefill(q, k, v, [n], d ** -0.5, weight=P_WEIGHT["bf16"], rows=rows)
    at = sorted(rows)
    close(out[at], want[at], tol[at], "rows in front of the spoiled one")
    assert bool(out[bad:].isnan().all()) and bool(torch.isfinite(out[:bad]).all())


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,hq", [(128, 2), (64, 1)])
@pytest.mark.parametrize("cap,side,size", [(50.0, 1, 1e17), (50.0, 1, 1e36), (20.0, 1, 1e32), (50.0, -1, 1e-30), (0.0, 0, 1e37), (60.0, 1, 1e37)])
def test_rows_of_v_far_from_one(cap, side, size, d, hq, out_dtype):
    """Finite rows of v whose products with the weights, taken relative to another score than the row's greatest, leave fp32's range: the
    output is an average of them all the same.  side: all scores deep in the cap's upper or lower end, or spread over some units."""
    lens = [300, 33]
    q, k, v, ip = prompts(lens, hq, 1, d, "bf16", seed=93, qscale=4.0 if side == 0 else 1.0)
    if side:
        q.copy_(q.abs() + 1)
        k.copy_(side * (k.abs() + 1))
    v.mul_(size)
    assert bool(torch.isfinite(v).all())
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5 * (8 if side else 1), cap, weight=P_WEIGHT["bf16"])
    out, status = run(q, k, v, ip, d, cap=cap, scale=d ** -0.5 * (8 if side else 1), out_dtype=out_dtype)
    assert status == (spd.SPD_OK, -1)
    close(out, want, tol, (cap, size))


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("n,d,hq", [(512, 128, 2), (300, 64, 1), (70001, 64, 1)])
def test_one_channel_of_a_key_that_everybody_sees_is_nan(n, d, hq, cap):
    """That channel is NaN for every row, the others are as without it; nothing is to be gained by doing rows again."""
    q, k, v, ip = prompts([n], hq, 1, d, "bf16", seed=94)
    rows = set(range(n)) if n < 1000 else {0, 1, 255, 256, n // 2, n - 1}
    want, tol = ref.prefill(q, k, v, [n], d ** -0.5, cap, weight=P_WEIGHT["bf16"], rows=rows)
    v[0, 0, 3] = float("nan")
    out, status = run(q, k, v, ip, d, cap=cap)
    assert status == (spd.SPD_OK, -1) and bool(out[:, :, 3].isnan().all())
    at, rest = sorted(rows), [c for c in range(d) if c != 3]
    close(out[at][..., rest], want[at][..., rest], tol[at], "other channels")


@pytest.mark.parametrize("d,hq", [(128, 2), (64, 1)])
def test_tiny_rows_of_v_under_moderately_low_scores(d, hq):
    """All scores near -20, v near the smallest normal numbers: sums relative to a score of 0 would be left with a few bits."""
    lens = [300, 33]
    q, k, v, ip = prompts(lens, hq, 1, d, "bf16", seed=95)
    q.copy_(q.abs() + 1)
    k.copy_(-k.abs() - 1)
    v.mul_(1e-37)
    want, tol = ref.prefill(q, k, v, lens, d ** -0.5 * 8, 20.0, weight=P_WEIGHT["bf16"])
    out, status = run(q, k, v, ip, d, cap=20.0, scale=d ** -0.5 * 8)
    assert status == (spd.SPD_OK, -1)
    close(out, want, tol, "tiny")
