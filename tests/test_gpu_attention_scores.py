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
@pytest.mark.parametrize("rows", [1, 20, 40, 150])
def test_the_largest_weight_is_exact(dtype, rows):
    """A row that sees one place (a prompt's first), or one that outweighs the
    others 2^30 times, gets that place's values bit for bit."""
    cache, batch, q = _inputs([rows], [rows], 6, 2, 128, 64, dtype, 3, 2.0)
    vs = S.gather(cache, batch, 0)[1]
    one = vs[:, 0].to(dtype).repeat_interleave(3, 0)
    assert torch.equal(_run(cache, batch, q)[0], one)
    q[..., 0] = 40.0
    cache["k"][..., 0] = 0.0
    page = int(batch["page_table"][0, 0])
    cache["k"][page, :, 0, 0] = 11.0  # 440 / 11.3 above the others' few units: 2^56 and up
    got = _run(cache, batch, q)
    assert torch.equal(got, one.expand_as(got))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [700, 715, 718, 1008, 1012, 1013, 1014, 1015])
def test_rising_scores_beyond_whole_numbers(dtype, value):
    """Scores of 2^22.9 to 2^24 powers of two that rise by 10 to 20 more behind
    the first 64 places, whose values are 0: those behind outweigh them at least
    500 times (float32's steps of 1 there among it)."""
    cache, batch, q = _inputs([40], [200], 2, 1, 128, 64, dtype, 1)
    cache["v"].fill_(1)
    page = int(batch["page_table"][0, 0])
    cache["v"][page] = 0
    for up in range(80, 161, 5):
        cache["k"].fill_(value)
        cache["k"][..., 127] = up  # times 1 and 0.1275: 10.2 to 20.4 powers of two
        cache["k"][page, ..., 127] = 0
        q.fill_(value)
        q[..., 127] = 1.0
        got = _run(cache, batch, q).double()
        assert bool(((got >= 0.99) & (got <= 1)).all()), (up, float(got.min()), float(got.max()))


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
