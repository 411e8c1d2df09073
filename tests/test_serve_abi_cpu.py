"""The serving operators' refusals, without a GPU: argument errors come back
before anything is launched, struct layouts match the header, and calls with
nothing to do return."""
import ctypes as C
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rt_router.h")
PTR = 1 << 20  # a pointer that is never read


@pytest.fixture(scope="module")
def rt():
    from paper_2609_16206_amd import build as b
    if not os.path.exists(b.LIB):
        b.build()
    from paper_2609_16206_amd import rt_router
    return rt_router


def _cache(rt, **kw):
    c = rt.rt_kv_cache(dtype=0, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, k=PTR, v=PTR)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(rt, **kw):
    b = rt.rt_kv_batch(n_seqs=2, n_tokens=3, q_start=PTR, kv_len=PTR, page_table=PTR, table_stride=4, max_q=2, max_kv=50)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _heads(rt, **kw):
    h = rt.rt_heads(data=PTR, token_stride=256, head_stride=64)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


CACHE_ERRORS = [(dict(dtype=2), "EINVAL"), (dict(dtype=-1), "EINVAL"), (dict(n_kv_heads=0), "EINVAL"),
                (dict(n_kv_heads=1025), "ERANGE"), (dict(head_dim=96), "EUNSUPPORTED"), (dict(head_dim=0), "EINVAL"),
                (dict(page_size=8), "EINVAL"), (dict(page_size=48), "EINVAL"), (dict(page_size=2048), "EINVAL"),
                (dict(n_pages=0), "EINVAL"), (dict(n_pages=1 << 31), "EINVAL"), (dict(k=None), "EINVAL"),
                (dict(v=PTR + 8), "EINVAL")]
BATCH_ERRORS = [(dict(n_seqs=-1), "EINVAL"), (dict(n_tokens=-1), "EINVAL"), (dict(max_q=-1), "EINVAL"),
                (dict(max_kv=-1), "EINVAL"), (dict(n_tokens=1 << 31), "ERANGE"), (dict(n_seqs=1 << 31), "ERANGE"),
                (dict(max_kv=(1 << 28) + 1, table_stride=1 << 40), "ERANGE"), (dict(table_stride=3), "EINVAL"),
                (dict(q_start=None), "EINVAL"), (dict(kv_len=None), "EINVAL"), (dict(page_table=None), "EINVAL"),
                (dict(table_stride=1 << 62), "ERANGE")]
IN_ERRORS = [(dict(data=None), "EINVAL"), (dict(data=PTR + 2), "EINVAL"), (dict(token_stride=-64), "EINVAL"),
             (dict(head_stride=4), "EINVAL"), (dict(token_stride=1 << 62), "ERANGE")]
OUT_ERRORS = IN_ERRORS + [(dict(token_stride=64), "EINVAL"), (dict(head_stride=0), "EINVAL"),
                          (dict(token_stride=0), "EINVAL"), (dict(head_stride=56), "EINVAL")]


def _attend(rt, cache=None, batch=None, hq=4, scale=0.125, q=None, tree=None, out=None, ws=PTR, nb=1 << 40):
    ref = lambda x: None if x is False else C.byref(x)
    return rt._lib.rt_paged_attention(ref(_cache(rt) if cache is None else cache),
                                      ref(_batch(rt) if batch is None else batch), hq, scale,
                                      ref(_heads(rt) if q is None else q), tree,
                                      ref(_heads(rt) if out is None else out), ws, nb, None)


def _append(rt, cache=None, batch=None, rope=None, hq=4, q=None, q_out=None, k=None, v=None):
    ref = lambda x: None if x is False else C.byref(x)
    return rt._lib.rt_kv_append(ref(_cache(rt) if cache is None else cache), ref(_batch(rt) if batch is None else batch),
                                None if rope is None else C.byref(rope), None, hq,
                                ref(_heads(rt) if q is None else q), ref(_heads(rt, data=2 * PTR) if q_out is None else q_out),
                                ref(_heads(rt) if k is None else k), ref(_heads(rt) if v is None else v), None)


def test_layouts_match_the_header(rt, tmp_path):
    names = ["rt_kv_cache", "rt_kv_batch", "rt_heads", "rt_rope"]
    lines = ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void){"]
    for s in names:
        lines.append(f'printf("{s} %zu\\n", sizeof({s}));')
        for f, _ in getattr(rt, s)._fields_:
            lines.append(f'printf("{s}.{f} %zu\\n", offsetof({s}, {f}));')
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-std=c11", str(src), "-o", str(exe)], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines())
    for s in names:
        cls = getattr(rt, s)
        assert int(got[s]) == C.sizeof(cls), s
        for f, _ in cls._fields_:
            assert int(got[f"{s}.{f}"]) == getattr(cls, f).offset, (s, f)
    # and the forms the calls pack, field by field
    c = rt.rt_kv_cache.from_buffer_copy(rt._CACHE.pack(1, 2, 3, 4, 5, 6, 7))
    assert (c.dtype, c.n_kv_heads, c.head_dim, c.page_size, c.n_pages, c.k, c.v) == (1, 2, 3, 4, 5, 6, 7)
    b = rt.rt_kv_batch.from_buffer_copy(rt._BATCH.pack(1, 2, 3, 4, 5, 6, 7, 8))
    assert (b.n_seqs, b.n_tokens, b.q_start, b.kv_len, b.page_table, b.table_stride, b.max_q, b.max_kv) == (1, 2, 3, 4, 5, 6, 7, 8)
    h = rt.rt_heads.from_buffer_copy(rt._HEADS.pack(1, 2, 3))
    assert (h.data, h.token_stride, h.head_stride) == (1, 2, 3)
    r = rt.rt_rope.from_buffer_copy(rt._ROPE.pack(1, 2, True, 4.5))
    assert (r.inv_freq, r.rot_dim, r.interleaved, r.scale) == (1, 2, 1, 4.5)


@pytest.mark.parametrize("change,err", CACHE_ERRORS)
def test_cache_errors(rt, change, err):
    code = getattr(rt, "RT_" + err)
    assert _attend(rt, cache=_cache(rt, **change)) == code
    assert "rt_paged_attention" in rt.rt_last_error()
    assert _append(rt, cache=_cache(rt, **change)) == code


@pytest.mark.parametrize("change,err", BATCH_ERRORS)
def test_batch_errors(rt, change, err):
    code = getattr(rt, "RT_" + err)
    assert _attend(rt, batch=_batch(rt, **change)) == code
    assert _append(rt, batch=_batch(rt, **change)) == code


@pytest.mark.parametrize("change,err", IN_ERRORS)
def test_input_row_errors(rt, change, err):
    code, h = getattr(rt, "RT_" + err), _heads(rt, **change)
    assert _attend(rt, q=h) == code
    assert _append(rt, q=h) == code and _append(rt, k=h) == code and _append(rt, v=h) == code


@pytest.mark.parametrize("change,err", OUT_ERRORS)
def test_output_row_errors(rt, change, err):
    code, h = getattr(rt, "RT_" + err), _heads(rt, **change)
    assert _attend(rt, out=h) == code
    assert _append(rt, q_out=h) == code


def test_attention_errors(rt):
    nan, inf = float("nan"), float("inf")
    assert _attend(rt, cache=False) == rt.RT_EINVAL and _attend(rt, batch=False) == rt.RT_EINVAL
    assert _attend(rt, q=False) == rt.RT_EINVAL and _attend(rt, out=False) == rt.RT_EINVAL
    for hq in (0, -2, 3):
        assert _attend(rt, hq=hq) == rt.RT_EINVAL
    assert _attend(rt, hq=130) == rt.RT_ERANGE
    for s in (0.0, -1.0, nan, inf):
        assert _attend(rt, scale=s) == rt.RT_EINVAL
    assert _attend(rt, batch=_batch(rt, max_q=65), tree=PTR) == rt.RT_ERANGE
    big = _batch(rt, max_kv=100_000, table_stride=10_000)
    n = C.c_int64()
    assert rt._lib.rt_paged_attention_workspace(C.byref(_cache(rt)), C.byref(big), 4, C.byref(n)) == rt.RT_OK
    assert n.value > 0
    assert _attend(rt, batch=big, ws=None) == rt.RT_EINVAL
    assert _attend(rt, batch=big, nb=n.value - 1) == rt.RT_EINVAL
    assert _attend(rt, batch=big, ws=PTR + 4) == rt.RT_EINVAL
    assert rt._lib.rt_paged_attention_workspace(C.byref(_cache(rt)), C.byref(big), 4, None) == rt.RT_EINVAL
    assert rt._lib.rt_paged_attention_workspace(None, C.byref(big), 4, C.byref(n)) == rt.RT_EINVAL
    for b in (_batch(rt, n_seqs=0), _batch(rt, n_tokens=0)):
        assert _attend(rt, batch=b, q=False, out=False, ws=None, nb=0) == rt.RT_OK


def test_append_errors(rt):
    def rope(**kw):
        r = rt.rt_rope(inv_freq=PTR, rot_dim=32, interleaved=0, scale=1.0)
        for k, v in kw.items():
            setattr(r, k, v)
        return r
    for bad in (dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=80), dict(interleaved=2),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(inv_freq=None)):
        assert _append(rt, rope=rope(**bad)) == rt.RT_EINVAL, bad
    assert _append(rt, cache=False) == rt.RT_EINVAL and _append(rt, batch=False) == rt.RT_EINVAL
    assert _append(rt, k=False) == rt.RT_EINVAL and _append(rt, v=False) == rt.RT_EINVAL
    assert _append(rt, q_out=False) == rt.RT_EINVAL
    assert _append(rt, hq=0) == rt.RT_EINVAL
    assert _append(rt, q_out=_heads(rt, token_stride=512)) == rt.RT_EINVAL  # q's memory, other strides: PTR is q's
    for b in (_batch(rt, n_seqs=0), _batch(rt, n_tokens=0)):
        assert _append(rt, batch=b) == rt.RT_OK


def _sample(rt, dtype=2, rows=2, vocab=100, logits=PTR, stride=100, bits=PTR, out=PTR, ws=PTR, nb=1 << 40):
    return rt._lib.rt_sample_tokens(dtype, rows, vocab, logits, stride, None, None, None, None, bits, out, ws, nb, None)


def test_sample_errors(rt):
    for bad in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(stride=99), dict(logits=None),
                dict(bits=None), dict(out=None), dict(logits=PTR + 2), dict(dtype=0, logits=PTR + 1)):
        assert _sample(rt, **bad) == rt.RT_EINVAL, bad
    assert _sample(rt, vocab=262145, stride=1 << 20) == rt.RT_ERANGE
    assert _sample(rt, rows=1 << 31) == rt.RT_ERANGE
    assert _sample(rt, stride=1 << 60, rows=100) == rt.RT_ERANGE
    assert _sample(rt, rows=0, logits=None, bits=None, out=None, ws=None, nb=0) == rt.RT_OK
    n = C.c_int64()
    assert rt._lib.rt_sample_workspace(2, 100, None) == rt.RT_EINVAL
    assert rt._lib.rt_sample_workspace(-1, 100, C.byref(n)) == rt.RT_EINVAL
    assert rt._lib.rt_sample_workspace(1, 262145, C.byref(n)) == rt.RT_ERANGE
    assert rt._lib.rt_sample_workspace(1, 262144, C.byref(n)) == rt.RT_OK and n.value >= 0


def test_binding_refuses_cpu_tensors(rt):
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    c = dict(k=torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16), v=torch.zeros(1, 2, 2, 64, 8, dtype=torch.bfloat16))
    b = dict(q_start=torch.zeros(2, dtype=torch.int32), kv_len=torch.zeros(1, dtype=torch.int32),
             page_table=torch.zeros(1, 1, dtype=torch.int32), max_q=1, max_kv=1)
    for call in (lambda: rt.rt_kv_append(c, b, x, x), lambda: rt.rt_paged_attention(c, b, x, x),
                 lambda: rt.rt_sample_tokens(torch.zeros(2, 9), torch.zeros(2, dtype=torch.int64),
                                             torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()


@pytest.mark.parametrize("change", [dict(max_q=2 ** 31), dict(max_kv=2 ** 40), dict(max_kv=65), dict(q_start=torch.zeros(2)),
                                    dict(kv_len=torch.zeros(3, dtype=torch.int32)),
                                    dict(page_table=torch.zeros(2, 8, dtype=torch.int32)[:, ::2])])
def test_binding_refuses_batches_it_cannot_pass(rt, change):
    ok = dict(q_start=torch.zeros(3, dtype=torch.int32), kv_len=torch.zeros(2, dtype=torch.int32),
              page_table=torch.zeros(2, 4, dtype=torch.int32), max_q=1, max_kv=64)
    assert len(rt._kv_batch(ok, 5, 16)) == C.sizeof(rt.rt_kv_batch)
    with pytest.raises((TypeError, ValueError)):
        rt._kv_batch(dict(ok, **change), 5, 16)


def test_binding_refuses_rows_it_cannot_pass(rt):
    x = torch.zeros(4, 3, 64, dtype=torch.bfloat16)
    assert rt._heads(x, "q", torch.bfloat16, 4, 64) == rt._HEADS.pack(x.data_ptr(), 192, 64)
    for t, n, d, h in [(x.half(), 4, 64, None), (x, 5, 64, None), (x, 4, 128, None), (x, 4, 64, 2), (x[0], 4, 64, None),
                       (x.transpose(1, 2), 4, 3, None)]:
        with pytest.raises((TypeError, ValueError)):
            rt._heads(t, "q", torch.bfloat16, n, d, h)
    with pytest.raises(TypeError, match="GPU"):
        rt._same_gpu([("q", x)])


def test_limits_of_a_launch(rt):
    """Sizes that a launch cannot take come back before it, and the largest
    sizes that it can are planned."""
    n = C.c_int64()
    plan = lambda hq=4, hkv=2, **kw: rt._lib.rt_paged_attention_workspace(  # noqa: E731
        C.byref(_cache(rt, n_kv_heads=hkv)), C.byref(_batch(rt, **kw)), hq, C.byref(n))
    assert plan(n_seqs=(1 << 23) - 1) == rt.RT_OK and plan(n_seqs=1 << 23) == rt.RT_ERANGE  # 2 KV heads: 2^24 pairs
    assert "too many" in rt.rt_last_error()
    assert _attend(rt, batch=_batch(rt, n_seqs=1 << 23)) == rt.RT_ERANGE
    # tiles of 128 rows of prompts: n_tokens / 128 + n_seqs of each KV head
    many = dict(max_q=200, max_kv=200, table_stride=20, n_seqs=1 << 22)
    assert plan(hq=2, n_tokens=(1 << 29) - 128, **many) == rt.RT_OK
    assert plan(hq=2, n_tokens=1 << 29, **many) == rt.RT_ERANGE
    # few rows in several runs are launched by sequence, head and run
    runs = dict(max_kv=40000, table_stride=3000)
    assert plan(n_seqs=(1 << 24) - 1, **runs) == rt.RT_OK and plan(n_seqs=1 << 24, **runs) == rt.RT_ERANGE
    assert plan(n_tokens=(1 << 29) - 1024) == rt.RT_ERANGE  # n_tokens * n_q_heads
    assert plan(n_tokens=(1 << 29) - 1025) == rt.RT_OK
    for tokens in ((1 << 26) - 3, (1 << 31) - 2):  # an append's rows by four
        assert _append(rt, batch=_batch(rt, n_tokens=tokens)) == rt.RT_ERANGE
        assert "n_tokens" in rt.rt_last_error()
    assert _append(rt, hq=65537) == rt.RT_EINVAL
    assert _append(rt, batch=_batch(rt, n_tokens=(1 << 31) - 1)) == rt.RT_ERANGE


def test_scales_that_overflow_are_refused(rt):
    """Scores are held in powers of two, 1.44 to a score's unit: scale times that
    has to be a float32."""
    for scale in (2.0 ** 127 * 1.01, 3e38, 3.4e38):
        assert _attend(rt, scale=scale) == rt.RT_ERANGE
        assert "2^127" in rt.rt_last_error()
    # (the largest scale passes this check: the next one refuses the rows)
    assert _attend(rt, scale=2.0 ** 127, batch=_batch(rt, max_q=65), tree=PTR) == rt.RT_ERANGE
    assert "tree" in rt.rt_last_error()
