"""rt_paged_attention where scores are far from ordinary: so large that float32
has no whole numbers for them left, up to its largest and lowest ones, or far below others that count."""
import math

import pytest
import torch

from tests import serve_reference as S
from tests.test_gpu_attention import _inputs, _run

pytestmark = pytest.mark.gpu


def _near_mean(got, cache, batch, q):
    """Rows whose scores are all equal, in float32 too (the same operations on
    the same numbers): weights are equal, so a row is the mean of the values it
    sees.  Off by u = half a step in the rounded weight, 2^-24 for each addition
    of the sums (as serve_reference counts them), u in the output."""
    u, e, g = torch.finfo(q.dtype).eps / 2, 2.0 ** -24, q.shape[1] // cache["k"].shape[1]
    qs = batch["q_start"].tolist()
    for i, kl in enumerate(batch["kv_len"].tolist()):
        vs, n = S.gather(cache, batch, i)[1], qs[i + 1] - qs[i]
        for t in range(n):
            mine = vs[:, :kl - n + t + 1].repeat_interleave(g, 0)
            ref, mag = mine.mean(1), mine.abs().mean(1)
            tol = (u + 2 * (kl / 4 + 72) * e) * mag * (1 + u) + u * ref.abs() + 2.0 ** -24
            near = (got[qs[i] + t].double() - ref).abs() <= tol
            assert bool(near.all()), (i, t, int((~near).sum()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,kv", [(3, 12), (40, 49), (150, 159), (40, 1500)])
@pytest.mark.parametrize("value", [900, 1014, 1100, 2900, 4500, 5736, 5748, 7800, 8000, 30000])
def test_scores_beyond_whole_numbers(dtype, rows, kv, value):
    """q and k of 128 equal elements: scores of 2^23.6 to 2^33.8 powers of two
    (2^24 at 1,014, 2^29 at 5,736, 10^9 at 7,828), all the same."""
    cache, batch, q = _inputs([rows], [kv], 2, 1, 128, 64, dtype, 1)
    cache["k"].fill_(value)
    q.fill_(value)
    _near_mean(_run(cache, batch, q), cache, batch, q)


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("rows,kv", [(1, 50), (1, 700), (1, 6000), (20, 700), (40, 49), (40, 3000), (150, 200)])
def test_scores_at_the_ends_of_float32(rows, kv, sign):
    """Scores of +-2.9e38, which float32 does not hold in powers of two (1.44
    times as much), are scores like others, in one run and in several, by the
    row's place and by a tree's words."""
    cache, batch, q = _inputs([rows], [kv], 4, 2, 64, 64, torch.bfloat16, 1)
    cache["k"].fill_(0)
    cache["k"][..., 0] = sign * 1.7e19
    q.fill_(0)
    q[..., 0] = 1.7e19
    _near_mean(_run(cache, batch, q, scale=1.0), cache, batch, q)
    if rows <= 64:
        tree = torch.tensor([(2 << t) - 1 for t in range(rows)], dtype=torch.int64)
        _near_mean(_run(cache, batch, q, scale=1.0, tree=tree), cache, batch, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new,kv", [(1, 4000), (20, 4000), (40, 4000), (64, 1500)])
@pytest.mark.parametrize("down", [14.5, 18.7, 22.45, 25.2, 28.3])
def test_small_weights_add_up(dtype, new, kv, down):
    """The first place outweighs every other 2^down times, but its values are
    0: the others make the result.  Beside a thousand sequences without rows, so
    that runs are long.  On top of serve_reference's bound a weight that float16
    holds with fewer bits is off by at most 2^-33 of the largest."""
    rows, kvs = [0] * 1100, [0] * 1100
    rows[700], kvs[700] = new, kv
    cache, batch, q = _inputs(rows, kvs, 1, 1, 64, 64, dtype, 1)
    cache["k"].fill_(0)
    cache["v"].abs_()
    page = int(batch["page_table"][700, 0])
    cache["k"][page, 0, 0, 0] = 8.0
    cache["v"][page, 0, 0, :, 0] = 0.0
    q.fill_(0)
    q[..., 0] = 1.0
    scale = down * math.log(2.0) / 8.0
    got = _run(cache, batch, q, scale=scale)
    ref, mag, big = S.attend(cache, batch, q, scale)
    tol = S.attend_tolerance(ref, mag, big, dtype, kv, 64)
    if dtype is torch.float16:
        tol += kv * 2.0 ** -33 * float(cache["v"].max())
    near = (got.double() - ref).abs() <= tol
    assert bool(near.all()), (int((~near).sum()), float(((got.double() - ref).abs() / mag).max()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [3, 40])
def test_rows_by_place_hold_their_weights_in_float32(dtype, rows):
    """Next to values that some rows do not see and that are not finite, rows go
    over their places one by one, with no matrix product and no rounding of
    weights: serve_reference's bound without that part."""
    cache, batch, q = _inputs([rows], [rows + 6], 4, 2, 64, 16, dtype, 3)
    clean = {k: v.clone() for k, v in cache.items()}
    place = rows + 5  # the last row's own
    page = int(batch["page_table"][0, place // 16])
    cache["v"][page, :, place % 16 // 8, :, place % 8] = math.inf
    got = _run(cache, batch, q)[:-1]
    ref, mag, big = (x[:-1] for x in S.attend(clean, batch, q, 0.125))
    u = torch.finfo(dtype).eps / 2
    tol = S.attend_tolerance(ref, mag, big, dtype, rows + 6, 64) - u * mag * (1 + u)
    near = (got.double() - ref).abs() <= tol
    assert bool(near.all()), int((~near).sum())
