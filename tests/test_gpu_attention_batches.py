"""rt_paged_attention over batches as a caller's arrays may hold them: rows
that start before the tensors or end behind them, and beside other sequences of
all kinds; token trees in float16."""
import pytest
import torch

from tests import serve_reference as S
from tests.test_gpu_attention import _check, _inputs, _run, _tree

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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,rows", [(3, 1), (3, 40), (70, 1), (70, 16), (70, 40), (70, 150), (1100, 1), (1100, 40)])
def test_other_sequences_change_nothing(n, rows, dtype):
    """A sequence's output, bit for bit, whatever the other sequences hold
    (within the same bounds), whether they are rejected or have no rows."""
    new = [1 + i % 3 for i in range(n)]
    new[n // 2] = rows
    kv = [m + (i * 61) % 900 for i, m in enumerate(new)]
    kv[0] = 900
    kv[n // 2] = 700
    cache, batch, q = _inputs(new, kv, 4, 2, 64, 64, dtype, 8, 2.0)
    lo = int(batch["q_start"][n // 2])
    want = _run(cache, batch, q)[lo:lo + rows]
    assert torch.isfinite(want).all()
    for lengths in ([m for m in new], [900] * n, [-1] * n, [901 if i % 2 else m + 5 for i, m in enumerate(new)]):
        lengths[n // 2] = 700
        got = _run(cache, dict(batch, kv_len=torch.tensor(lengths, dtype=torch.int32),
                               page_table=batch["page_table"].clamp(max=cache["k"].shape[0] - 1)), q)
        assert torch.equal(got[lo:lo + rows], want)
    alone = batch["q_start"].clone()
    alone[:n // 2] = lo
    alone[n // 2 + 1:] = lo + rows
    got = _run(cache, dict(batch, q_start=alone), q)
    assert torch.equal(got[lo:lo + rows], want)
    assert (got[:lo] == 7.0).all() and (got[lo + rows:] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 16), (4, 4, 64, 64), (16, 1, 128, 32), (3, 1, 64, 128)])
def test_trees_in_float16(hq, hkv, d, page):
    new = [21, 1, 0, 64, 5, 33]
    kv = [400, 1, 7, 64, 900, 65]
    cache, batch, q = _inputs(new, kv, hq, hkv, d, page, torch.float16, 9, 2.0)
    tree = _tree(new, 3)
    _check(_run(cache, batch, q, tree=tree), cache, batch, q, tree)
    new, kv = [4, 2, 8], [1500, 9, 300]  # few rows, in runs
    cache, batch, q = _inputs(new, kv, hkv, hkv, d, page, torch.float16, 9, 2.0)
    tree = _tree(new, 4)
    _check(_run(cache, batch, q, tree=tree), cache, batch, q, tree)
