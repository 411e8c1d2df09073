"""rt_paged_attention over batches as a caller's arrays may hold them: rows
that start before the tensors or end behind them."""
import pytest
import torch

from tests import serve_reference as S
from tests.test_gpu_attention import _check, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("start", [-1, -1000, -2 ** 31])
@pytest.mark.parametrize("n,hq", [(3, 1), (64, 3), (65, 1), (65, 3), (1100, 2)])
@pytest.mark.parametrize("long", [60, 4000])
def test_rows_before_and_behind_the_tensors(n, hq, long, start):
    """The first sequence is said to start before row 0, the last to end
    behind the last row: rejected, their rows are NaN as far as they lie in the
    tensors, and the others are served as without them."""
    new = [150] + [1 + (i * 37) % 20 for i in range(1, n - 1)] + [140]
    kv = [150] + [new[i] + (long if i == n // 2 else i % 7) for i in range(1, n - 1)] + [140]
    cache, batch, q = _inputs(new, kv, hq, 1, 64, 64, torch.bfloat16, 8, 2.0)
    want = _run(cache, batch, q)
    wrong = dict(batch, q_start=batch["q_start"].clone())
    wrong["q_start"][0] = start
    wrong["q_start"][-1] += 9
    got = _run(cache, wrong, q)
    assert torch.isnan(got[:150]).all() and torch.isnan(got[-140:]).all()
    assert torch.equal(got[150:-140], want[150:-140])
    if n <= 65:
        _check(want, cache, batch, q)
