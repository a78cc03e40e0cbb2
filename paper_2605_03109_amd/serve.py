"""The attention half of a decoder block as it is served: gated maps q, k, v, the paged cache in 4 bits, attention over
it, the gated map o.  One `step` takes the new tokens of a batch of requests, prompts and single tokens alike; lengths,
tables and the free list stay on the device and nothing is waited for.

``python -m paper_2605_03109_amd.serve`` runs prompts and decode steps of synthetic tokens through one block (the
shapes of an OPT-6.7B layer by default) and prints one JSON line with the times of both.
"""
from __future__ import annotations

import argparse
import collections
import json
import sys
import time
from typing import Dict, Optional

import torch

from paper_2605_03109_amd import gsi


class AttentionBlock:
    """Weights W[m, d] and bases U[d, k] (one for the input of q, k, v, one for that of o), a cache of `n_pages` pages for up
    to `requests` requests of up to `max_len` tokens.  Requests keep their pages; tokens behind the last page or past `max_len` have no place in
    the cache, and `missing` says so: it is the number of pages that were not there, summed over the steps (on the device, 0 where nothing was lost;
    a step whose `status[1]` is not 0 has lost tokens, and its requests are to be dropped or given again)."""

    KEPT = 8  # step sizes whose buffers are kept, in order of use

    def __init__(self, weights: Dict[str, torch.Tensor], U_in: torch.Tensor, U_out: torch.Tensor, heads: int, kv_heads: int,
                 requests: int, n_pages: int, max_len: int, page: int = 64, eps: float = 0.05):
        dev = U_in.device
        self.heads, self.kv_heads, self.dim = heads, kv_heads, weights["q"].shape[0] // heads
        self.eps, self.max_len = eps, max_len
        self.U_in, self.U_out = U_in, U_out
        self.W = weights
        self.M = {name: gsi.build_image(W, U_out if name == "o" else U_in) for name, W in weights.items()}
        self.cache = gsi.KvCache.empty(n_pages, kv_heads, self.dim, page, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        self.table = torch.full((requests, -(-max_len // page)), -1, **i32)
        self.kv_len = torch.zeros(requests, **i32)
        self.free = torch.arange(n_pages, **i32)
        self._count = torch.tensor([n_pages, 0], **i32)  # free pages, missing ones
        self._change = torch.tensor([-1, 1], **i32)      # of them, by the tables' status
        self.status = torch.zeros(2, **i32)              # of the last step: pages taken, pages that were not there
        self._place = torch.arange(n_pages, device=dev)
        self._stacks: collections.OrderedDict[tuple, tuple] = collections.OrderedDict()

    @property
    def n_free(self) -> torch.Tensor:
        return self._count[:1]

    @n_free.setter
    def n_free(self, n: torch.Tensor) -> None:
        self._count = torch.cat([n.view(1), self._count[1:]])

    @property
    def missing(self) -> torch.Tensor:
        return self._count[1:]

    def _stacks_for(self, T: int) -> tuple:
        # buffers by stream too: memory that one gives back is used again behind the work of its own stream only
        key = T, torch.cuda.current_stream(self.U_in.device).cuda_stream
        if key in self._stacks:
            self._stacks.move_to_end(key)
        else:
            while len(self._stacks) >= self.KEPT:
                self._stacks.popitem(last=False)
            f32 = dict(dtype=torch.float32, device=self.U_in.device)
            X = torch.empty((T, self.U_in.shape[0]), **f32)
            A = torch.empty((T, self.heads, self.dim), **f32)
            qkv = gsi.LayerStack([{"U": self.U_in, "X": X}],
                                 [{"W": self.W[n], "M": self.M[n], "input_id": 0} for n in "qkv"], T, self.eps)
            out = gsi.LayerStack([{"U": self.U_out, "X": A.view(T, -1)}], [{"W": self.W["o"], "M": self.M["o"], "input_id": 0}],
                                 T, self.eps)
            self._stacks[key] = (X, A, qkv, out)
        return self._stacks[key]

    def step(self, X: torch.Tensor, n_new: torch.Tensor, max_q: int, max_len: Optional[int] = None) -> torch.Tensor:
        """X[T, d] (fp32): the step's tokens, request by request; n_new[requests] int32: how many each has; max_q, max_len: the most
        that one has, new and altogether.  Returns the output of map o, [T, d] (valid until the next step of T tokens; a step of a size that is
        not among the last KEPT sets its buffers up first)."""
        T = X.shape[0]
        x, attended, qkv, out = self._stacks_for(T)
        x.copy_(X)
        self.kv_len, start, slots, _, self.status = gsi.kv_tables(self.kv_len, n_new, self.free, self.n_free, self.table, T, self.cache.page)
        # what was taken leaves the front of the free list
        self.free = self.free[(self._place + self.status[0]).clamp(max=self.free.numel() - 1)]
        self._count = torch.addcmul(self._count, self.status, self._change)
        qkv.run()
        q, k, v = (m["Y"].view(T, -1, self.dim) for m in qkv.maps_t)
        gsi.kv_append(self.cache, k, v, slots)
        gsi.kv_attention(self.cache, q, start, self.kv_len, self.table, max_q=max_q, max_len=max_len or self.max_len, O=attended)
        out.run()
        return out.maps_t[0]["Y"]


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=32)
    ap.add_argument("--k", type=int, default=256, help="rank of the bases")
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--steps", type=int, default=32, help="decode steps behind the prompts")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        print("serve.py: no GPU visible", file=sys.stderr)
        return 3
    from paper_2605_03109_amd import workload_device as wd

    g = torch.Generator(device="cuda").manual_seed(260503109)
    d, dim = args.d, args.d // args.heads
    rows = {"q": args.heads * dim, "k": args.kv_heads * dim, "v": args.kv_heads * dim, "o": d}
    W = {n: wd.make_weight(m, args.heads * dim if n == "o" else d, g) for n, m in rows.items()}
    U = [wd.make_basis64(w, args.k, g).to(torch.bfloat16) for w in (d, args.heads * dim)]
    lens = [max(1, args.prompt - (args.prompt * i) // (2 * args.requests)) for i in range(args.requests)]
    page, max_len = 64, args.prompt + args.steps
    block = AttentionBlock(W, U[0], U[1], args.heads, args.kv_heads, args.requests, sum(-(-(n + args.steps) // page) for n in lens), max_len, page)
    n_new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    one = torch.ones_like(n_new)
    prompt, tokens = torch.randn(sum(lens), d, generator=g, device="cuda"), torch.randn(args.requests, d, generator=g, device="cuda")

    def timed(f) -> float:
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        return time.perf_counter() - t

    def decode():
        for _ in range(args.steps):
            block.step(tokens, one, 1)

    state = block.kv_len, block.free, block._count
    block.step(prompt, n_new, args.prompt), block.step(tokens, one, 1)  # first calls
    block.kv_len, block.free, block._count = state
    block.table.fill_(-1)
    prompt_s = timed(lambda: block.step(prompt, n_new, args.prompt))
    decode_s = timed(decode)
    if int(block.missing):
        print("serve.py: the cache had too few pages, tokens were lost", file=sys.stderr)
        return 1
    print(json.dumps({"workload": f"attention half of a block, d {d}, {args.heads} heads over {args.kv_heads}, rank {args.k}, {args.requests} requests",
                      "prompt_tokens": sum(lens), "prompt_ms": round(prompt_s * 1e3, 3), "decode_steps": args.steps,
                      "decode_us_per_step": round(decode_s / args.steps * 1e6, 1),
                      "cache_bytes_per_token": args.kv_heads * dim * 2 * 17 // 32, "data": "synthetic"}))
    return 0


if __name__ == "__main__":
    sys.exit(main())
