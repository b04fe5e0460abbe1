"""A served decoder stack: attention over a 4-bit paged cache in front of the per-layer top-k MoE module.

    x <- x + W_o attention(rope(W_qkv norm(x)))          keys and values live in the layer's 4-bit cache
    x <- x + MoE_l(norm(x); k_l)

for batches of requests of different lengths, prompts and single tokens in one step.  The projections are plain library
products; everything else between them is this package's kernels: ``tables`` once a step, then per layer ``append``
(rotary positions, 4-bit storage), ``attention`` and the MoE layer with that layer's own number of active experts.

    python -m paper_2509_02753_b200.decoder [workload] [requests] [prompt tokens] [steps]

runs prompts and decoding steps of a model with that workload's MoE shapes and seeded weights and prints the time of each.
"""
from __future__ import annotations

import sys
import time
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding as B
from . import kv_cache as K
from . import synth


@dataclass
class Attention:
    """Shape of a layer's attention.  window > 0: a token sees the last `window` tokens and the first `sinks`."""
    n_heads: int
    n_kv_heads: int
    head_dim: int
    rope_dim: int
    layout: str = "half"
    window: int = 0
    sinks: int = 0
    k_scale: float = 1.0
    v_scale: float = 1.0


class Request:
    """Tokens in the cache, and the row of the block table."""

    def __init__(self, row: int):
        self.row, self.length = row, 0


def rms_norm(x: torch.Tensor, eps: float = 1e-6) -> torch.Tensor:
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps)).to(x.dtype)


class Decoder:
    """layers: one dict per layer with "qkv" [(n_heads + 2 n_kv_heads) head_dim, d], "o" [d, n_heads head_dim] and the MoE
    weights of ``binding.make_weights``; k_vec: the active experts of each layer."""

    def __init__(self, layers: Sequence[dict], k_vec: Sequence[int], plan: B.MoEPlan, attn: Attention, *, renorm: bool, n_pages: int, page_size: int,
                 max_requests: int, max_tokens: int, max_context: int, base: float = 10000.0, scaling: Optional[dict] = None):
        self.layers, self.k_vec, self.moe, self.attn, self.renorm = layers, list(k_vec), plan, attn, renorm
        dtype = plan.dtype
        self.kv = K.KVPlan(n_heads=attn.n_heads, n_kv_heads=attn.n_kv_heads, head_dim=attn.head_dim, page_size=page_size, dtype=dtype,
                           max_requests=max_requests, max_tokens=max_tokens)
        self.weights = [B.make_weights(w) for w in layers]
        self.caches = [self.kv.new_cache(n_pages) for _ in layers]
        self.turns = K.rope_table(attn.rope_dim, max_context, base=base, **(scaling or {}))
        self.page = page_size
        self.width = -(-max_context // page_size)
        self.max_context = max_context
        self.table = torch.full((max_requests, self.width), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros((max_requests,), dtype=torch.int32, device="cuda")
        self.requests = [Request(i) for i in range(max_requests)]
        self.free = list(range(n_pages))

    def close(self):
        self.kv.close()

    def _fresh(self, new: Sequence[int]) -> int:
        return sum(-(-(r.length + n) // self.page) - -(-r.length // self.page) for r, n in zip(self.requests, new))

    def finish(self, row: int) -> None:
        """Gives a request's pages back; the row serves another request from its first token on."""
        held = -(-self.requests[row].length // self.page)
        self.free += self.table[row, :held].tolist()
        self.table[row].fill_(-1)
        self.lengths[row] = 0
        self.requests[row].length = 0

    def step(self, x: torch.Tensor, new: Sequence[int]) -> torch.Tensor:
        """One step: x [sum(new), d] are the hidden states of the new tokens, request after request (new[i] of request i, 0
        for one that pauses).  Returns the stack's output for them, [sum(new), d]."""
        T = x.shape[0]
        assert T == sum(new) and len(new) == len(self.requests)
        if any(n < 0 for n in new):
            raise ValueError("a negative number of new tokens")
        if T == 0:
            return x
        need = self._fresh(new)
        if need > len(self.free):
            raise MemoryError(f"{need} pages wanted, {len(self.free)} free")
        if any(r.length + n > self.max_context for r, n in zip(self.requests, new)):
            raise ValueError("a request passes max_context")
        a, dev = self.attn, x.device
        fresh = torch.tensor(self.free[:need], dtype=torch.int32, device=dev)
        kv_len, cu, position, slot, _ = self.kv.tables(self.lengths, torch.tensor(list(new), dtype=torch.int32, device=dev), fresh, self.table, T)
        for layer, weights, cache, k in zip(self.layers, self.weights, self.caches, self.k_vec):
            qkv = torch.matmul(rms_norm(x), layer["qkv"].t()).view(T, a.n_heads + 2 * a.n_kv_heads, a.head_dim)
            q, key, value = qkv.split((a.n_heads, a.n_kv_heads, a.n_kv_heads), 1)
            q = self.kv.append(q, key, value, slot, cache, positions=position, turns=self.turns, layout=a.layout, k_scale=a.k_scale, v_scale=a.v_scale)
            o = self.kv.attention(q, cu, kv_len, self.table, cache, max_new=max(new), window=a.window, sinks=a.sinks, k_scale=a.k_scale, v_scale=a.v_scale)
            x = x + torch.matmul(o.view(T, -1), layer["o"].t())
            x = x + self.moe.layer_forward(rms_norm(x), weights, k, self.renorm)
        del self.free[:need]
        self.lengths = kv_len
        for r, n in zip(self.requests, new):
            r.length += n
        return x

    def check(self) -> None:
        """Raises if a kernel met a bad index or a wait ran out since the last check; synchronises."""
        status, bits = self.kv.device_status()
        if status != 0:
            raise B.MoEError(f"cache operators (status bits {bits})", status)
        if self.moe.device_status() != 0:
            raise B.MoEError("moe layer", -8)


def make_attention_weights(attn: Attention, d: int, layer: int, dtype: torch.dtype, seed: int = 0) -> dict:
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + layer)
    rows = (attn.n_heads + 2 * attn.n_kv_heads) * attn.head_dim
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5  # noqa: E731
    return {"qkv": normal(rows, d).to(dtype), "o": normal(d, attn.n_heads * attn.head_dim).to(dtype)}


def build(workload: str, attn: Attention, *, layers: int, dtype: torch.dtype, requests: int, max_tokens: int, max_context: int, page_size: int = 64,
          seed: int = 0) -> Decoder:
    """A decoder of `layers` layers with the workload's MoE shapes, seeded weights, and its per-layer numbers of experts."""
    wl = synth.WORKLOADS[workload]
    k_vec: List[int] = (synth.make_k_vector(wl, seed) * layers)[:layers]
    plan = B.MoEPlan(wl.d, wl.E, wl.I, max_tokens, max(k_vec), dtype, I_shared=wl.I_shared, shared_gate=wl.shared_gate)
    weights = [{**synth.make_layer(wl, i % wl.L, dtype, "cuda", seed), **make_attention_weights(attn, wl.d, i, dtype, seed)} for i in range(layers)]
    pages = requests * -(-max_context // page_size)
    return Decoder(weights, k_vec, plan, attn, renorm=wl.renorm, n_pages=pages, page_size=page_size, max_requests=requests, max_tokens=max_tokens,
                   max_context=max_context)


def attention_of(wl: synth.Workload) -> Attention:
    """Heads of 128 dimensions as wide as the model, four (or the next larger number that divides) to a key/value head."""
    heads = wl.d // 128
    return Attention(n_heads=heads, n_kv_heads=max(n for n in range(1, max(1, heads // 4) + 1) if heads % n == 0), head_dim=128, rope_dim=128)


def main(argv: Sequence[str]) -> None:
    workload = argv[0] if argv else "olmoe"
    requests, prompt, steps = (int(argv[i]) if len(argv) > i else v for i, v in ((1, 16), (2, 1024), (3, 64)))
    wl = synth.WORKLOADS[workload]
    attn = attention_of(wl)
    dec = build(workload, attn, layers=min(wl.L, 8), dtype=torch.bfloat16, requests=requests, max_tokens=requests * prompt, max_context=prompt + steps)
    x = synth.make_tokens(wl, requests * prompt, torch.bfloat16, "cuda")

    def timed(f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        return time.perf_counter() - t

    dec.step(x, [prompt] * requests)           # the first step loads the kernels
    dec.check()
    for row in range(requests):
        dec.finish(row)
    first = timed(lambda: dec.step(x, [prompt] * requests))
    token = x[:requests].contiguous()
    each = timed(lambda: [dec.step(token, [1] * requests) for _ in range(steps)]) / steps
    dec.check()
    cache = sum(c.numel() for c in dec.caches) / 2 ** 20
    print(f"{workload}: {len(dec.layers)} layers, k = {dec.k_vec}, {requests} requests, cache {cache:.0f} MiB in 4 bits")
    print(f"prompts of {prompt} tokens: {first * 1e3:.2f} ms, {requests * prompt / first:.0f} tokens/s")
    print(f"a token of every request: {each * 1e3:.3f} ms, {requests / each:.0f} tokens/s")
    dec.close()


if __name__ == "__main__":
    main(sys.argv[1:])
