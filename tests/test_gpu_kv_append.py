"""rt_kv_append against the float64 form: layouts of the rotation, ragged and
padded batches, group and page borders, strided views, refused data."""
import math

import numpy as np
import pytest
import torch

from tests import serve_reference as S

pytestmark = pytest.mark.gpu


def _freq(rot, factor=1.0):
    return torch.from_numpy(10000.0 ** (-np.arange(0, rot, 2) / rot) / factor)


def _run(cache, batch, k, v, q=None, q_out=None, rope=None, positions=None, **kw):
    from paper_2609_16206_amd import rt_router as R
    c, b = S.to_gpu(cache), S.to_gpu(batch)
    g = [None if t is None else t.cuda() for t in (k, v, q, q_out, positions)]
    if rope is not None:
        rope = dict(rope, inv_freq=rope["inv_freq"].cuda())
    R.rt_kv_append(c, b, g[0], g[1], q=g[2], q_out=g[3], rope=rope, positions=g[4], **kw)
    torch.cuda.synchronize()
    return c["k"].cpu(), c["v"].cpu(), None if q is None else g[3].cpu()


def _near(got, ref, src_scale, dtype):
    """Within one rounding of the type, plus float32 arithmetic: the angle is
    off by 2 pi 2^-26 = 9.4e-8, sine and cosine by 2 steps of 2^-24, their
    scale, the two products and the sum by 2^-24 each; under 4e-7 of the
    pair's magnitude in all."""
    u = torch.finfo(dtype).eps / 2
    tiny = float(torch.finfo(dtype).smallest_normal) * u * 2
    tol = u * ref.abs() + 4e-7 * src_scale * (1 + u) + tiny
    bad = (got.double() - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} values off, worst {(got.double() - ref).abs().max()}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,page,rot,inter", [(16, 2, 128, 64, 128, False), (8, 8, 64, 16, 64, True),
                                                     (5, 1, 128, 32, 64, False), (6, 3, 64, 128, 16, True),
                                                     (4, 2, 128, 1024, 48, True), (3, 3, 64, 16, 0, False)])
def test_append_matches_float64(dtype, hq, hkv, d, page, rot, inter):
    new = [1, 0, 7, 8, 9, 33, 1, 100, 0, 3]
    kv = [1, 5, 7, 16, 12, 40, 700, 131, 0, 18]
    batch, n_pages, rows = S.make_batch(new, kv, page, 3, pad_rows=3, front_rows=2, stride_extra=1)
    cache = S.make_cache(n_pages, hkv, d, page, dtype, 4)
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn(rows, (hq + 2 * hkv) * d, generator=g).to(dtype)
    q, k, v = (x.view(rows, -1, d) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
    q_out = torch.full((rows, hq, d), 7.0, dtype=dtype)
    f = _freq(rot, 4.0) if rot else None
    rope = None if f is None else dict(inv_freq=f, interleaved=inter, scale=1.25)
    kc, vc, qo = _run(cache, batch, k, v, q, q_out, rope)
    rk, rv, rq = S.append(cache, batch, k, v, q, f, inter, 1.25)
    assert torch.equal(vc.double(), rv)
    scale = 1.25 * 2 * float(qkv.double().abs().max())
    _near(kc, rk, scale, dtype)
    live = ~torch.isnan(rq[:, 0, 0])
    assert int(live.sum()) == sum(new)
    _near(qo[live], rq[live], scale, dtype)
    assert (qo[~live] == 7.0).all()  # rows of no sequence
    # places that no row went to are untouched, bit for bit
    same = rk == cache["k"].double()
    assert torch.equal(kc[same], cache["k"][same])


@pytest.mark.parametrize("pos", [0, 1, 131071, 5_000_000, 2**31 - 1])
def test_far_positions(pos):
    """Angles stay right where float32 positions would not: the reference
    angle is a float64 product too (error 2^-53 of up to 2^31 radians)."""
    batch, n_pages, rows = S.make_batch([1], [9], 16, 0)
    cache = S.make_cache(n_pages, 1, 64, 16, torch.float16, 1)
    k = torch.randn(rows, 1, 64, generator=torch.Generator().manual_seed(2)).half()
    f = _freq(64)
    p = torch.tensor([pos], dtype=torch.int32)
    kc, _, _ = _run(cache, batch, k, k, rope=dict(inv_freq=f), positions=p)
    rk, _, _ = S.append(cache, batch, k, k, inv_freq=f, positions=p)
    # the product's own rounding, twice over: 2^31 2^-52 = 4.8e-7 radians at most
    _near(kc, rk, 2 * float(k.double().abs().max()) * (1 + pos * 2.0 ** -52 / 4e-7), torch.float16)


def test_in_place_queries_and_head_major_views():
    """q_out in q's memory, and tensors whose heads lie outside the tokens."""
    hq, hkv, d, rows = 4, 2, 64, 50
    batch, n_pages, n = S.make_batch([rows], [rows + 30], 32, 1)
    cache = S.make_cache(n_pages, hkv, d, 32, torch.bfloat16, 2)
    g = torch.Generator().manual_seed(3)
    from paper_2609_16206_amd import rt_router as R
    q = torch.randn(hq, rows, d, generator=g).bfloat16()
    k, v = torch.randn(hkv, rows, d, generator=g).bfloat16(), torch.randn(hkv, rows, d, generator=g).bfloat16()
    f = _freq(64)
    c, b = S.to_gpu(cache), S.to_gpu(batch)
    qg = q.cuda().transpose(0, 1)
    R.rt_kv_append(c, b, k.cuda().transpose(0, 1), v.cuda().transpose(0, 1), q=qg, q_out=qg,
                   rope=dict(inv_freq=f.cuda()))
    torch.cuda.synchronize()
    rk, rv, rq = S.append(cache, batch, k.transpose(0, 1), v.transpose(0, 1), q.transpose(0, 1), f)
    _near(c["k"].cpu(), rk, 10, torch.bfloat16)
    assert torch.equal(c["v"].cpu().double(), rv)
    _near(qg.cpu(), rq, 10, torch.bfloat16)


def test_many_rows_and_long_search():
    """More sequences than one round of the search covers, several of them
    without rows, and the launch of four rows a workgroup."""
    rng = np.random.default_rng(0)
    new = rng.integers(0, 4, 5000)
    kv = new + rng.integers(0, 30, 5000)
    batch, n_pages, rows = S.make_batch(new.tolist(), kv.tolist(), 16, 1)
    cache = S.make_cache(n_pages, 1, 64, 16, torch.bfloat16, 2)
    k = torch.randn(rows, 1, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    kc, vc, _ = _run(cache, batch, k, k)
    rk, rv, _ = S.append(cache, batch, k, k)
    assert torch.equal(kc.double(), rk) and torch.equal(vc.double(), rv)


@pytest.mark.parametrize("what", ["kv short", "kv long", "q long", "backwards", "behind", "negative page", "big page"])
def test_rejected_rows_write_nothing(what):
    """Rows of a sequence the call cannot use: q_out NaN, cache untouched; the
    other sequence is served."""
    from paper_2609_16206_amd import rt_router as R
    batch, n_pages, rows = S.make_batch([9, 9], [30, 20], 16, 1)
    cache = S.make_cache(n_pages, 1, 64, 16, torch.bfloat16, 2)
    x = torch.randn(rows, 1, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    ref = S.append(cache, batch, x, x, x)
    bad = list(range(9))
    if what == "kv short":
        batch["kv_len"][0] = 8
    elif what == "kv long":
        batch["kv_len"][0] = 31
    elif what == "q long":
        batch["max_q"] = 8
        bad = list(range(18))
    elif what == "backwards":
        batch["q_start"] = torch.tensor([9, 0, 9], dtype=torch.int32)  # sequence 0 has no rows, the last 9 none
        bad = []
    elif what == "behind":
        batch["q_start"] = torch.tensor([0, 9, 19], dtype=torch.int32)
        bad = list(range(9, 18))
    elif what == "negative page":
        batch["page_table"][0, 1] = -1  # places 16 .. 31: all nine
    else:
        batch["page_table"][0, 1] = n_pages
    out = torch.full((rows, 1, 64), 7.0, dtype=torch.bfloat16)
    kc, vc, qo = _run(cache, batch, x, x, x, out)
    assert torch.isnan(qo[bad]).all()
    if what == "backwards":
        return  # memory is safe; which rows belong to whom is not defined
    good = [r for r in range(18) if r not in bad]
    assert torch.equal(qo[good].double(), ref[2][good])
    only = {r: (pg, sl) for r, _, _, pg, sl in S.rows_of(S.make_batch([9, 9], [30, 20], 16, 1)[0], 16)}
    for r in bad:
        pg, sl = only[r]
        assert torch.equal(kc[pg, :, sl], cache["k"][pg, :, sl])
        assert torch.equal(vc[pg, :, sl // 8, :, sl % 8], cache["v"][pg, :, sl // 8, :, sl % 8])
    for r in good:
        pg, sl = only[r]
        assert torch.equal(kc[pg, :, sl].double(), ref[0][pg, :, sl])
        assert torch.equal(vc[pg, :, sl // 8, :, sl % 8].double(), ref[1][pg, :, sl // 8, :, sl % 8])


def test_empty_calls():
    batch, n_pages, rows = S.make_batch([], [], 16, 1)
    cache = S.make_cache(n_pages, 1, 64, 16, torch.bfloat16, 2)
    x = torch.zeros(0, 1, 64, dtype=torch.bfloat16)
    kc, _, _ = _run(cache, batch, x, x)
    assert torch.equal(kc, cache["k"])
    batch, n_pages, rows = S.make_batch([0, 0], [0, 4], 16, 1)
    kc, _, _ = _run(cache, batch, x, x)
    assert torch.equal(kc, cache["k"])


@pytest.mark.parametrize("start", [[9, 0, 9], [0, 18, 9], [18, 9, 0], [5, -7, 30], [2 ** 31 - 1, -2 ** 31, 18]])
@pytest.mark.parametrize("pad", [0, 3000])
def test_rows_out_of_order_write_only_dealt_places(start, pad):
    """Starts that decrease or lie far outside: whose row is whose is not
    defined, but a row of q_out is the rotated one, NaN or as it was, and of
    the cache only places that the table deals to the two sequences change."""
    batch, n_pages, rows = S.make_batch([9, 9], [30, 20], 16, 1, pad_rows=pad)
    cache = S.make_cache(n_pages, 1, 64, 16, torch.bfloat16, 2)
    x = torch.randn(rows, 1, 64, generator=torch.Generator().manual_seed(3)).bfloat16()
    batch["q_start"] = torch.tensor(start, dtype=torch.int32)
    batch["max_q"] = rows
    out = torch.full((rows, 1, 64), 7.0, dtype=torch.bfloat16)
    kc, vc, qo = _run(cache, batch, x, x, x, out)
    for r in range(rows):
        assert torch.equal(qo[r], x[r]) or (qo[r] == 7.0).all() or torch.isnan(qo[r]).all()
    dealt = {(int(batch["page_table"][i, p // 16]), p % 16) for i, n in enumerate((30, 20)) for p in range(n)}
    for pg in range(n_pages):
        for sl in range(16):
            if (pg, sl) not in dealt:
                assert torch.equal(kc[pg, :, sl], cache["k"][pg, :, sl])
                assert torch.equal(vc[pg, :, sl // 8, :, sl % 8], cache["v"][pg, :, sl // 8, :, sl % 8])
