"""The serving operators together: prompts in chunks beside single tokens,
append -> attention -> draw, against float64 at every step; the instance that
the measured calibration runs them in, eager and replayed."""
import time

import numpy as np
import pytest
import torch

from tests import serve_reference as S

pytestmark = pytest.mark.gpu


def _rotated(x, pos, f):
    a = pos.double()[:, None, None] * f
    h = f.numel()
    lo, hi, rest = x[..., :h].double(), x[..., h:2 * h].double(), x[..., 2 * h:].double()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin(), rest], -1)


def _pairs(x, rot):
    """|a| + |b| of each value's rotated pair (|x| where nothing is rotated)."""
    s = x[..., :rot // 2].abs() + x[..., rot // 2:rot].abs()
    return torch.cat([s, s, x[..., rot:].abs()], -1)


@pytest.mark.parametrize("dtype,hq,hkv,d,page,rot", [(torch.bfloat16, 8, 2, 128, 16, 128), (torch.float16, 3, 3, 64, 64, 32)])
def test_chunks_and_single_tokens_together(dtype, hq, hkv, d, page, rot):
    """Three requests: a prompt in chunks of odd sizes, one prefilled at once,
    one that starts with a single token and later brings a tree-less draft of
    three; pages are dealt as they are needed, none in order.  Every step's
    attention is compared with float64 over the unrounded history.

    Bound: a rotated key or query is rounded once (u = half a step) behind a
    rotation in 32 bits (within 6 * 2^-24 of its pair's |a| + |b|), so with the
    pairs' sums in place of the values a score moves by at most 2.1 u times
    their product, and a weight by twice that, beside serve_reference's bound."""
    from paper_2609_16206_amd import rt_router as R
    plan = [[130, 1, 1], [77, 0, 1], [1, 60, 3], [0, 1, 1], [1, 1, 1]]
    total = [sum(s[i] for s in plan) for i in range(3)]
    g = torch.Generator().manual_seed(hq)
    q, k, v = ([torch.randn(t, h, d, generator=g).to(dtype) for t in total] for h in (hq, hkv, hkv))
    f = 1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    width = -(-max(total) // page)
    order = torch.randperm(3 * width, generator=g).to(torch.int32)
    table = torch.randint(0, 3 * width, (3, width), generator=g, dtype=torch.int32)
    cache = R.alloc_kv_cache(3 * width, hkv, d, page, dtype)
    for t in cache.values():
        t.fill_(float("nan"))  # places that nothing was appended to must not count
    at, dealt = [0, 0, 0], 0
    w = torch.randn(hq * d, 700, generator=g)
    u = torch.finfo(dtype).eps / 2
    for step, new in enumerate(plan):
        upto = [a + n for a, n in zip(at, new)]
        for i in range(3):
            for pg in range(-(-at[i] // page), -(-upto[i] // page)):
                table[i, pg] = order[dealt]
                dealt += 1
        cut = lambda x: torch.cat([x[i][at[i]:upto[i]] for i in range(3)])  # noqa: E731
        qkv = torch.cat([cut(q), cut(k), cut(v)], 1).cuda()  # as a fused projection leaves them
        qq, kk, vv = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        batch = dict(q_start=torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda(),
                     kv_len=torch.tensor(upto, dtype=torch.int32).cuda(), page_table=table.cuda(), max_q=max(new),
                     max_kv=max(upto))
        R.rt_kv_append(cache, batch, kk, vv, q=qq, q_out=qq, rope=dict(inv_freq=f.cuda()))
        out = torch.empty(sum(new), hq, d, dtype=dtype, device="cuda")
        R.rt_paged_attention(cache, batch, qq, out)
        logits = out.float().flatten(1) @ w.cuda()
        bits = torch.from_numpy(np.random.default_rng(step).integers(-2 ** 63, 2 ** 63 - 1, sum(new), dtype=np.int64))
        rows = sum(new)
        prm = dict(temperature=torch.full((rows,), 0.8), top_k=torch.full((rows,), 40, dtype=torch.int32),
                   top_p=torch.full((rows,), 0.9))
        token = torch.empty(rows, dtype=torch.int32, device="cuda")
        R.rt_sample_tokens(logits, bits.cuda(), token, **{n: t.cuda() for n, t in prm.items()})
        assert torch.equal(token.cpu(), S.sample(logits.cpu(), bits, **prm))
        got, row = out.cpu().double(), 0
        for i in range(3):
            pos = torch.arange(upto[i])
            kr, qr = _rotated(k[i][:upto[i]], pos, f), _rotated(q[i][at[i]:upto[i]], pos[at[i]:], f)
            for r in range(new[i]):
                n = at[i] + r + 1
                for h in range(hq):
                    ks, vs = kr[:n, h * hkv // hq], v[i][:n, h * hkv // hq].double()
                    p = torch.softmax(ks @ qr[r, h] * d ** -0.5, 0)
                    ref, mag = p @ vs, p @ vs.abs()
                    big = float((ks.abs() @ qr[r, h].abs()).max()) * d ** -0.5
                    moved = float((_pairs(ks, rot) @ _pairs(qr[r, h], rot)).max()) * d ** -0.5 * 2.1 * u
                    tol = S.attend_tolerance(ref, mag, torch.tensor(big), dtype, n, d) + 2 * moved * mag
                    assert ((got[row, h] - ref).abs() <= tol).all(), (step, i, r, h)
                row += 1
        at = upto


def test_workspace_comes_from_the_calls_own_stream():
    """Memory that the current stream has freed, and whose last use may still
    be pending there, is not taken for a call on another stream."""
    from paper_2609_16206_amd import rt_router as R
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        x = torch.empty(5 << 20, dtype=torch.uint8, device="cuda")
        freed = x.data_ptr()
        del x
        assert R._workspace(None, 5 << 20, 0, stream)[0] != freed
    assert R._workspace(None, 5 << 20, 0, None)[0] == freed  # (the current stream's own may be)


def test_two_streams_at_once():
    """The same calls on two streams, each with a workspace of its own, give
    what they give alone."""
    from paper_2609_16206_amd import rt_router as R
    g = torch.Generator().manual_seed(0)
    kv = [3000, 5, 1700]
    batch, n_pages, rows = S.make_batch([1, 1, 1], kv, 64, 3)
    cache = S.to_gpu(S.make_cache(n_pages, 2, 128, 64, torch.bfloat16, 4))
    b = S.to_gpu(batch)
    q = [torch.randn(3, 8, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
    logits = [torch.randn(64, 20000, generator=g).cuda() for _ in range(2)]
    bits = torch.arange(64, dtype=torch.int64).mul_(2 ** 57 + 12345).cuda()
    prm = dict(top_k=torch.full((64,), 50, dtype=torch.int32).cuda(), top_p=torch.full((64,), 0.9).cuda())

    def run(i, stream=None):
        o, t = torch.empty_like(q[i]), torch.empty(64, dtype=torch.int32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        R.rt_paged_attention(cache, b, q[i], o, stream=stream)
        R.rt_sample_tokens(logits[i], bits, t, stream=stream, **prm)
        return o, t
    alone = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        both = [run(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for x, y in zip(alone, both):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


SMALL = dict(layers=2, q_heads=4, kv_heads=2, head_dim=64, hidden=256, ffn=384, vocab=1999)


def _plain_logits(inst, tokens):
    """float64 logits behind the last of one request's tokens, no cache."""
    s = inst.shape
    norm = lambda x: x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    d, g, n = s.head_dim, s.q_heads // s.kv_heads, len(tokens)
    x = inst.embed.cpu().double()[tokens]
    pos, f = torch.arange(n), inst.inv_freq.cpu()
    for w in inst.layers:
        w = {k: v.cpu().double() for k, v in w.items()}
        qkv = (norm(x) @ w["qkv"].T).view(n, -1, d)
        q, k = _rotated(qkv[:, :s.q_heads], pos, f), _rotated(qkv[:, s.q_heads:s.q_heads + s.kv_heads], pos, f)
        v = qkv[:, s.q_heads + s.kv_heads:]
        o = torch.empty(n, s.q_heads, d, dtype=torch.float64)
        for h in range(s.q_heads):
            sc = q[:, h] @ k[:, h // g].T * d ** -0.5
            o[:, h] = torch.softmax(sc.masked_fill(~torch.ones(n, n).tril().bool(), -torch.inf), 1) @ v[:, h // g]
        x = x + o.flatten(1) @ w["out"].T
        gate, up = (norm(x) @ w["up"].T).chunk(2, 1)
        x = x + (gate * torch.sigmoid(gate) * up) @ w["down"].T
    return norm(x[-1]) @ inst.head.cpu().double().T


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_instance_in_chunks_matches_the_plain_decoder(dtype):
    """Bound, in norms: at most 2 x 9 + 2 roundings of u on the way to the
    logits, none magnified by more than 2 (random weights of unit gain; a
    score's error reaches a weight twice): 40 u of the logits' norm."""
    from paper_2609_16206_amd import instance as I
    inst = I.Instance(I.Shape(**SMALL), max_seqs=3, max_len=160, dtype=dtype, page_size=16)
    g = torch.Generator().manual_seed(3)
    tok = [torch.randint(0, 1999, (n,), generator=g) for n in (150, 40, 9)]
    inst.forward(torch.cat([tok[0][:97], tok[1][:39], tok[2][:1]]).cuda(), inst.batch([97, 39, 1], [97, 39, 1]))
    got = inst.forward(torch.cat([tok[0][97:], tok[1][39:], tok[2][1:]]).cuda(), inst.batch([53, 1, 8], [150, 40, 9]))
    for i in range(3):
        ref = _plain_logits(inst, tok[i])
        err = (got[i].cpu().double() - ref).norm() / ref.norm()
        assert err <= 40 * torch.finfo(dtype).eps / 2, (i, float(err))


def test_decoder_replays_its_eager_steps():
    """Captured and eager decoding of the same requests draw the same tokens
    at every step, with the program's own work between the replays; another
    captured decoder that steps in between changes nothing."""
    from paper_2609_16206_amd import instance as I
    inst = I.Instance(I.Shape(**SMALL), max_seqs=5, max_len=96, page_size=32)
    g = torch.Generator().manual_seed(5)
    held = [33, 1, 64, 7, 50]
    prompt = torch.randint(0, 1999, (sum(held),), generator=g).cuda()
    first = torch.randint(0, 1999, (5,), generator=g).cuda()
    runs = []
    for graph in (False, True, True):
        inst.forward(prompt, inst.batch(held, held))
        kw = dict(seed=11, temperature=0.9, top_k=50, top_p=0.95, graph=graph)
        dec = I.Decoder(inst, first, held, 12, **kw)
        other = I.Decoder(I.Instance(inst.shape, max_seqs=5, max_len=96, seed=1), first, [1] * 5, 12,
                          **kw) if len(runs) == 2 else None
        out = []
        for step in range(12):
            dec.step()
            out.append(dec.tokens.cpu())
            torch.randn(500, 500, device="cuda").mul_(2).sum().item()
            if other is not None:
                other.step()
        assert dec.batch["kv_len"].tolist() == [h + 12 for h in held]
        with pytest.raises(RuntimeError, match="room"):
            dec.step()
        runs.append(torch.stack(out))
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])
    assert len(set(runs[0].flatten().tolist())) > 20  # (draws, not one token again and again)


def test_measured_calibration_end_to_end():
    """Curves measured on a small instance make a point that simulates."""
    from paper_2609_16206_amd import experiments as E
    from paper_2609_16206_amd import instance as I
    from paper_2609_16206_amd import workload as W
    inst = I.Instance(I.Shape(**SMALL), max_seqs=4, max_len=160)
    cur = I.measure(inst, prompts=(16, 64, 160), outputs=(2, 9), batches=(1, 4), context=100, repeats=2)
    assert all((np.asarray(v) > 0).all() for v in cur.values())
    ph = E.measured_physics(cur, inst.shape.kv_bytes_per_token)
    pt = W.make_point(2, 3, n_classes=3, physics=ph, service="batched",
                      beta_dec=E.fit_batch_slowdown(cur["batch"], cur["step_ns"]))
    rows = E.run_cells([E.Cell("measured", pt, W.chat(4.0))], replicas=2, requests=200)
    assert 0 <= rows[0]["mean"] <= 1


def test_measured_prefill_is_the_gpus_time():
    """Host time between launches, here 50 ms a call, is no part of a prefill's
    latency (a decode step's has none either: both are replayed)."""
    from paper_2609_16206_amd import instance as I

    class SlowHost(I.Instance):
        def forward(self, tokens, batch):
            time.sleep(0.05)
            return super().forward(tokens, batch)
    inst = SlowHost(I.Shape(**SMALL), max_seqs=1, max_len=160)
    cur = I.measure(inst, prompts=(16, 100), outputs=(2,), batches=(1,), context=100, repeats=3)
    assert all(0 < t < 2e7 for k in ("prefill_ns", "decode_ns", "step_ns") for t in cur[k])


def test_an_instance_keeps_its_gpu():
    """Made on "cuda", it names that GPU: what its calls allocate later lies
    there, whichever is current then."""
    from paper_2609_16206_amd import instance as I
    inst = I.Instance(I.Shape(**SMALL), max_seqs=1, max_len=64)
    assert inst.device == torch.device("cuda", torch.cuda.current_device())
    assert inst.batch([1], [1])["kv_len"].device == inst.device
