"""Host-side parts of the measured calibration (CPU): slowdown fit, physics,
frequencies, the refusals of an instance's batches."""
import math

import numpy as np
import pytest
import torch

from paper_2609_16206_amd import experiments as E
from paper_2609_16206_amd import instance as I
from paper_2609_16206_amd import workload as W


def test_shape_is_the_measured_constants_own():
    assert I.Shape().kv_bytes_per_token == 36864


@pytest.mark.parametrize("beta", [0.0, 0.029 / 7, 0.3])
def test_slowdown_is_recovered(beta):
    b = np.array([1, 2, 4, 8, 16, 32, 64])
    assert abs(E.fit_batch_slowdown(b, 5e6 * (1 + beta * (b - 1))) - beta) < 1e-12


def test_slowdown_edges():
    assert E.fit_batch_slowdown([1, 4], [10.0, 8.0]) == 0.0  # faster together: no slowdown below 0
    assert E.fit_batch_slowdown([1], [10.0]) == 0.0
    with pytest.raises(ValueError, match="lone request"):
        E.fit_batch_slowdown([2, 4], [10.0, 12.0])


def test_physics_of_curves_makes_a_point():
    p, o = np.array([16, 256, 4096]), np.array([2, 33, 129])
    cur = dict(prompt_len=p, prefill_ns=4e6 + 900.4 * p, out_len=o, decode_ns=5e6 * (o - 1.0))
    ph = E.measured_physics(cur, 36864)
    assert ph == dict(pre_base_ns=4000000, pre_tok_ns=900, dec_tok_ns=5000000, kv_bytes_per_token=36864)
    pt = W.make_point(2, 4, physics=ph)
    assert (pt["pre_base_ns"], pt["pre_tok_ns"], pt["dec_tok_ns"]) == (4000000, 900, 5000000)
    assert pt["xfer_tok_ns"] == W.xfer_tok_ns(36864)
    # a fit through the origin from below stays a legal point
    low = E.measured_physics(dict(cur, prefill_ns=1000.0 * p - 5.0), 36864)
    assert low["pre_base_ns"] == 0 and low["pre_tok_ns"] == 1000


@pytest.mark.parametrize("rot,base,factor", [(128, 1e6, 1.0), (64, 1e4, 4.0), (2, 1e4, 1.0)])
def test_frequencies(rot, base, factor):
    f = I.rope_frequencies(rot, base, factor, device="cpu")
    assert f.dtype == torch.float64 and f.shape == (rot // 2,)
    for j in range(rot // 2):
        assert math.isclose(float(f[j]), base ** (-2 * j / rot) / factor, rel_tol=1e-14)


def test_batches_and_refusals():
    inst = I.Instance(I.Shape(1, 2, 1, 64, 16, 24, 50), max_seqs=3, max_len=100, page_size=32, device="cpu")
    assert inst.max_len == 128 and inst.page_table.tolist() == [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]]
    b = inst.batch([1, 7], [128, 7])
    assert b["q_start"].tolist() == [0, 1, 8] and b["kv_len"].tolist() == [128, 7]
    assert (b["max_q"], b["max_kv"]) == (7, 128) and b["page_table"].shape == (2, 4)
    for new, total, kw in [([1], [129], {}), ([0], [4], {}), ([5], [4], {}), ([1] * 4, [1] * 4, {}), ([1], [1, 2], {}),
                           ([1], [1], dict(max_kv=129))]:
        with pytest.raises(ValueError):
            inst.batch(new, total, **kw)


def test_measured_goes_with_calibrate_only():
    with pytest.raises(SystemExit):
        E.main(["policies", "--measured"])


def test_tokens_must_match_the_batch():
    """Too few or too many tokens come back before anything runs on them: rows
    beyond the tensors would end the process on the GPU."""
    inst = I.Instance(I.Shape(1, 2, 1, 64, 16, 24, 50), max_seqs=3, max_len=100, page_size=32, device="cpu")
    for n in (0, 7, 9):
        with pytest.raises(ValueError, match="8 tokens"):
            inst.forward(torch.zeros(n, dtype=torch.int32), inst.batch([1, 7], [128, 7]))
    with pytest.raises(ValueError, match="2 tokens"):
        I.Decoder(inst, torch.zeros(1, dtype=torch.int32), [3, 4], 5, graph=False).step()
