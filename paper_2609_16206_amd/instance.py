"""A serving instance to calibrate on: the decoder that the measured constants
stand for (36,864 KV bytes a token), with random weights, a paged cache and the
library's serving operators, and the latency curves measured on it.

The paper takes its service constants from a benchmark of the machines that
serve (Section III-B); this is that benchmark for the GPU at hand.  A layer is
norm, one projection to q, k and v, rt_kv_append, rt_paged_attention, output
projection, norm and a gated feed-forward; a step ends in rt_sample_tokens.
The plain matrix products are torch's.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, List, Sequence

import numpy as np
import torch
import torch.nn.functional as F

from . import rt_router as R


@dataclass(frozen=True)
class Shape:
    """36 layers x 2 (k, v) x 2 KV heads x 128 x 2 bytes = 36,864 bytes a token."""
    layers: int = 36
    q_heads: int = 16
    kv_heads: int = 2
    head_dim: int = 128
    hidden: int = 2048
    ffn: int = 11008
    vocab: int = 151936

    @property
    def kv_bytes_per_token(self) -> int:
        return self.layers * 2 * self.kv_heads * self.head_dim * 2


def rope_frequencies(rot_dim: int, base: float = 1e6, factor: float = 1.0, device="cuda") -> torch.Tensor:
    """Angles per position of the rotated pairs, float64 [rot_dim / 2]:
    base ** (-2 j / rot_dim) / factor.  A factor above 1 slows every pair at every
    position alike, so that positions up to that many times the trained ones turn
    no further than those."""
    j = torch.arange(rot_dim // 2, dtype=torch.float64)
    return (base ** (-2.0 * j / rot_dim) / factor).to(device)


class Instance:
    """Weights, cache and page table of `max_seqs` requests of up to `max_len`
    tokens each.  Request i's pages are i * w .. (i + 1) * w - 1."""

    def __init__(self, shape: Shape = Shape(), max_seqs: int = 64, max_len: int = 8192, dtype=torch.bfloat16,
                 page_size: int = 64, seed: int = 0, device="cuda"):
        self.shape, self.dtype, self.max_seqs = shape, dtype, max_seqs
        s, g = shape, torch.Generator(device).manual_seed(seed)

        def weight(n_out, n_in):
            w = torch.randn(n_out, n_in, generator=g, device=device, dtype=torch.float32)
            return (w * n_in ** -0.5).to(dtype)

        d = s.head_dim
        self.embed = torch.randn(s.vocab, s.hidden, generator=g, device=device).to(dtype)
        self.device = self.embed.device  # (with its number: the current GPU may be another one later)
        self.head = weight(s.vocab, s.hidden)
        self.layers = [dict(qkv=weight((s.q_heads + 2 * s.kv_heads) * d, s.hidden),
                            out=weight(s.hidden, s.q_heads * d), up=weight(2 * s.ffn, s.hidden),
                            down=weight(s.hidden, s.ffn)) for _ in range(s.layers)]
        w = -(-max_len // page_size)
        self.max_len = w * page_size
        self.page_table = torch.arange(max_seqs * w, dtype=torch.int32, device=device).view(max_seqs, w)
        self.caches = [R.alloc_kv_cache(max_seqs * w, s.kv_heads, d, page_size, dtype, device)
                       for _ in range(s.layers)]
        self.inv_freq = rope_frequencies(d, device=device)

    def batch(self, new: Sequence[int], total: Sequence[int], max_kv: int = 0) -> Dict:
        """The batch in which requests 0 .. n - 1 bring new[i] tokens each and
        then hold total[i]; max_kv: room for later steps on the same batch."""
        if len(new) != len(total) or len(new) > self.max_seqs:
            raise ValueError(f"new and total must have one entry for each of at most {self.max_seqs} requests")
        if any(not 1 <= a <= b <= self.max_len for a, b in zip(new, total)):
            raise ValueError(f"1 <= new <= total <= {self.max_len} must hold for every request")
        if max_kv > self.max_len:
            raise ValueError(f"max_kv must be at most {self.max_len}")
        i32 = dict(dtype=torch.int32, device=self.device)
        return dict(q_start=torch.tensor([0] + list(np.cumsum(new)), **i32), kv_len=torch.tensor(list(total), **i32),
                    page_table=self.page_table[:len(new)], n_tokens=sum(new), max_q=max(list(new) + [0]),
                    max_kv=max(list(total) + [0, max_kv]))

    def forward(self, tokens: torch.Tensor, batch: Dict) -> torch.Tensor:
        """Appends the tokens (below vocab) of every request and returns the
        logits [requests, vocab] behind each one's last token."""
        s, n, d = self.shape, tokens.numel(), self.shape.head_dim
        if n != batch.get("n_tokens", n):
            raise ValueError(f"the batch brings {batch['n_tokens']} tokens, got {n}")
        hq, hkv = s.q_heads, s.kv_heads
        rope = dict(inv_freq=self.inv_freq)
        x = self.embed[tokens]
        for w, cache in zip(self.layers, self.caches):
            qkv = (F.rms_norm(x, (s.hidden,), eps=1e-6) @ w["qkv"].t()).view(n, hq + 2 * hkv, d)
            q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            R.rt_kv_append(cache, batch, k, v, q=q, q_out=q, rope=rope)
            o = torch.empty(n, hq, d, dtype=self.dtype, device=self.device)
            R.rt_paged_attention(cache, batch, q, o)
            x = x + o.view(n, hq * d) @ w["out"].t()
            gate, up = (F.rms_norm(x, (s.hidden,), eps=1e-6) @ w["up"].t()).chunk(2, dim=1)
            x = x + (F.silu(gate) * up) @ w["down"].t()
        last = x[batch["q_start"][1:].long() - 1]
        return F.rms_norm(last, (s.hidden,), eps=1e-6) @ self.head.t()


class Decoder:
    """Decode steps of requests that an Instance holds: each step appends every
    request's last token and draws its next one.  `graph`: the step is captured
    once and replayed (its buffers are this object's own).  `tokens` holds the
    last tokens, `batch["kv_len"]` the tokens in the cache."""

    def __init__(self, inst: Instance, tokens: torch.Tensor, held: Sequence[int], steps: int, seed: int = 0,
                 temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0, graph: bool = True):
        n = len(held)
        self.inst, self.steps, self.left = inst, steps, steps
        self.batch = inst.batch([1] * n, [h + 1 for h in held], max(held) + steps)
        self.batch["kv_len"] -= 1  # (a step adds one first)
        self.held = self.batch["kv_len"].clone()
        self.tokens = tokens.to(torch.int32).clone()
        g = torch.Generator(inst.device).manual_seed(seed)
        self.bits = torch.randint(-2 ** 63, 2 ** 63 - 1, (n,), generator=g, dtype=torch.int64, device=inst.device)
        full = lambda v, t: torch.full((n,), v, dtype=t, device=inst.device)  # noqa: E731
        self.settings = dict(temperature=full(temperature, torch.float32), top_k=full(top_k, torch.int32),
                             top_p=full(top_p, torch.float32))
        self.graph = None
        if graph:
            with torch.cuda.device(inst.device):
                self._capture()

    def _capture(self) -> None:
        own = (self.tokens, self.batch["kv_len"], self.bits)
        kept = [t.clone() for t in own]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # libraries set themselves up outside the capture
            self._step()
            for t, k in zip(own, kept):
                t.copy_(k)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._step()

    def rewind(self) -> None:
        """Back to the number of cached tokens at the start."""
        self.batch["kv_len"].copy_(self.held)
        self.left = self.steps

    def _step(self) -> None:
        self.batch["kv_len"].add_(1)
        self.bits.mul_(6364136223846793005).add_(1442695040888963407)  # (a generator modulo 2^64)
        R.rt_sample_tokens(self.inst.forward(self.tokens, self.batch), self.bits, self.tokens, **self.settings)

    def step(self) -> None:
        if self.left < 1:
            raise RuntimeError("the requests have no room for another step")
        self.left -= 1
        if self.graph is None:
            self._step()
        else:
            self.graph.replay()


def _median_ns(calls: Sequence) -> float:
    """Median time of the calls, each between two events."""
    t: List[float] = []
    for call in calls:
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        t.append(a.elapsed_time(b) * 1e6)  # ms to ns
    return float(np.median(t))


def measure(inst: Instance, prompts: Sequence[int] = (16, 64, 256, 512, 1024, 2048, 4096, 8192),
            outputs: Sequence[int] = (2, 9, 33, 65, 129), batches: Sequence[int] = (1, 2, 4, 8, 16, 32, 64),
            context: int = 512, repeats: int = 5, seed: int = 0) -> Dict[str, np.ndarray]:
    """The latency curves that fit_service_constants and fit_batch_slowdown
    take, measured on the instance: prefill latency of one prompt with its first
    token, the time of a lone request's o - 1 decode steps, and the time of a
    decode step with b requests of `context` tokens each.  All of it is replayed
    from graphs: the GPU's time, without the host's between launches (16 tokens
    of the default shape 5.0 ms, launched one by one 5.7 to 6.3)."""
    dev = inst.device
    g = torch.Generator(dev).manual_seed(seed)
    vocab = inst.shape.vocab
    draw = lambda n: torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32, device=dev)  # noqa: E731
    with torch.cuda.device(dev):
        bits, token = torch.zeros(1, dtype=torch.int64, device=dev), torch.empty(1, dtype=torch.int32, device=dev)
        prefill = []
        for p in prompts:
            b, t = inst.batch([p], [p]), draw(p)
            call = lambda: R.rt_sample_tokens(inst.forward(t, b), bits, token)  # noqa: E731,B023
            call()  # libraries set themselves up outside the capture
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            graph.replay()
            prefill.append(_median_ns([graph.replay] * repeats))
            del graph  # (and its memory)
        fill = max(1, 8192 // context)  # requests whose context is written at once
        n = max(list(batches) + [1])
        for first in range(0, n, fill):
            m = min(fill, n - first)
            b = inst.batch([context] * m, [context] * m)
            b["page_table"] = inst.page_table[first:first + m]
            inst.forward(draw(m * context), b)
        decode, step = [], []
        for o in outputs:
            dec = Decoder(inst, draw(1), [context], o - 1, seed)

            def run():
                dec.rewind()
                for _ in range(o - 1):  # noqa: B023
                    dec.step()
            run()
            decode.append(_median_ns([run] * repeats))
        for m in batches:
            dec = Decoder(inst, draw(m), [context] * m, 3 * repeats + 1, seed)
            dec.step()
            step.append(_median_ns([dec.step] * (3 * repeats)))
    return dict(prompt_len=np.asarray(prompts), prefill_ns=np.asarray(prefill), out_len=np.asarray(outputs),
                decode_ns=np.asarray(decode), batch=np.asarray(batches), step_ns=np.asarray(step))
