"""An attention layer that serves drafted tokens over a paged cache and calibrates its heads' rotations on the way.

`AttentionLayer` runs the operators of `attention` as a server would, one step for a batch of sequences: norms and positions of queries and
keys, the new keys and values into the cache, attention of every new token over its sequence and those drafted tokens it follows.  The
step's output rows are the per-head activations in front of the output projection, one of the sites whose rotations the paper calibrates
(App. A); a `binding.Calibrator` with as many heads takes those of the tokens that stay.

    python -m paper_2605_10793_amd.layer [--bits 4] [--sequences 8] [--prompt 512] [--steps 24]

feeds random prompts in chunks, calibrates on them, then drafts a tree of tokens a step and commits one of its paths.
"""
from __future__ import annotations

import argparse
import time
from typing import Optional

import torch

from . import attention, binding


class AttentionLayer:
    """table: int32 [sequences, columns], the pages of `cache` that each sequence may use.  q_weight, k_weight: of the per-head norms.
    calibrator: takes the outputs of the tokens that are committed, or None; it may have been made on any stream of the cache's device."""

    def __init__(self, plan: attention.Rotary, q_weight, k_weight, cache: attention.KVCache, table, eps: float = 1e-6,
                 calibrator: Optional[binding.Calibrator] = None):
        self.plan, self.q_weight, self.k_weight, self.cache, self.table, self.eps = plan, q_weight, k_weight, cache, table, eps
        if calibrator is not None and calibrator.device != cache.device:
            raise ValueError(f"the calibrator is on cuda:{calibrator.device}, the cache on cuda:{cache.device}")
        self.calibrator = calibrator
        self.prefix = torch.zeros(table.shape[0], dtype=torch.int32, device=table.device)      # committed tokens
        self._last = None

    def step(self, fused, start, depth=None, mask=None, max_query: int = 64, max_context: Optional[int] = None):
        """New tokens of every sequence, at most 64 each: fused [tokens, heads + 2 cache heads, width] holds their queries, keys and values,
        start (int32 [sequences + 1]) the first row of each sequence.  A tree of drafted tokens has its tokens' depths (int64) and masks
        (attention.tree_attention); without them they are a chain.  max_query: the most of a sequence, so that every token has a result.  Returns
        [tokens, heads, width].  Nothing is committed."""
        tokens, kv = fused.shape[0], self.cache.heads
        if tokens > self.table.shape[0] * max_query:
            raise ValueError(f"{tokens} tokens are more than {max_query} for each of {self.table.shape[0]} sequences")
        heads = fused.shape[1] - 2 * kv
        q, k, v = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
        rows = torch.arange(tokens, dtype=torch.int32, device=fused.device)
        sequence = torch.searchsorted(start[1:], rows, right=True).clamp_(max=self.table.shape[0] - 1)      # (rows of no sequence: the last)
        first = self.prefix if depth is not None else self.prefix - start[:-1]
        positions = first[sequence] + (rows.long() if depth is None else depth)
        q_out, k_out = attention.qk_norm_rotary(self.plan, q, k, self.q_weight, self.k_weight, positions, eps=self.eps)
        attention.append(self.cache, k_out, v, start, self.prefix, self.table)
        out = attention.tree_attention(q_out, self.cache, start, self.prefix, self.table, mask=mask, max_query=max_query, max_context=max_context)
        self._last = q, k, v, k_out, positions, out
        return out

    def commit(self, start, rows=None):
        """The tokens of the last step that stay.  rows (int64): their row numbers there, each sequence's from its root on, start (int32
        [sequences + 1]) the first entry of each sequence; None: all rows, as they were passed.  Kept keys and values move to the places
        behind the committed ones, and their outputs go to the calibrator."""
        _, _, v, k_out, _, out = self._last
        if rows is not None:
            out = out[rows]
            attention.append(self.cache, k_out[rows], v[rows], start, self.prefix, self.table)
        if self.calibrator is not None and out.shape[0]:
            self._calibrate(out)
        start = start.clamp(0, out.shape[0])           # as the operators read it
        self.prefix += (start[1:] - start[:-1]).clamp_(min=0)

    def _calibrate(self, out):
        """The calibrator reads `out` on its own stream: not before it is written, and done before its memory may change."""
        cal, x = self.calibrator, out.flatten(1)
        if cal.stream == torch._C._cuda_getCurrentRawStream(cal.device):
            cal.step_batch_heads(x, 0, out.shape[1])
            return
        here = torch.cuda.current_stream(out.device)
        there = torch.cuda.ExternalStream(cal.stream, out.device) if cal.stream else torch.cuda.default_stream(out.device)
        there.wait_stream(here)
        cal.step_batch_heads(x, 0, out.shape[1])
        here.wait_stream(there)

    def gradients(self, q_grad, k_grad):
        """From the gradients of the last step's normed and rotated queries and keys: those of its projections and of the two weights."""
        q, k, _, _, positions, _ = self._last
        return attention.qk_norm_rotary_backward(self.plan, q, k, self.q_weight, self.k_weight, positions, q_grad, k_grad, eps=self.eps)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--bits", type=int, default=4, choices=(16, 8, 4))
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512, help="tokens of each prompt")
    ap.add_argument("--steps", type=int, default=24, help="drafting steps")
    args = ap.parse_args()
    heads, kv, width, page, B = 32, 8, 128, 64, args.sequences
    dev = "cuda:0"
    g = torch.Generator(device=dev)
    g.manual_seed(0)
    spread = torch.exp(0.7 * torch.randn(heads + 2 * kv, width, device=dev, generator=g))       # uneven channels, as activations have them

    def draw(tokens):
        return (torch.randn(tokens, heads + 2 * kv, width, device=dev, generator=g) * spread).to(torch.bfloat16)

    # A tree of 15 drafted tokens a sequence: each follows the token (i - 1) / 2 of it.
    nodes, path = 15, [0, 2, 5, 11]
    above = [0]
    for i in range(1, nodes):
        above.append(above[(i - 1) // 2] | 1 << (i - 1) // 2)
    mask = torch.tensor([a | 1 << i for i, a in enumerate(above)] * B, device=dev)
    depth = torch.tensor([bin(a).count("1") for a in above] * B, device=dev)

    def runs(n):
        return torch.arange(B + 1, dtype=torch.int32, device=dev) * n

    most = args.prompt + args.steps * len(path) + nodes
    columns = -(-most // page)
    cache = attention.KVCache.empty(B * columns, kv, page, width, args.bits, dev)
    table = torch.arange(B * columns, dtype=torch.int32, device=dev).view(B, columns)
    R0 = torch.eye(width).repeat(heads, 1, 1).numpy()
    weight = torch.ones(width, dtype=torch.bfloat16, device=dev)
    cal = binding.Calibrator(heads * width, heads, "bf16", R0, max_tokens=64 * B)
    layer = AttentionLayer(attention.Rotary(width, 500000.0, device=dev), weight, weight, cache, table, calibrator=cal)
    try:
        for at in range(0, args.prompt, 64):
            n = min(64, args.prompt - at)
            layer.step(draw(n * B), runs(n), max_query=n, max_context=most)
            layer.commit(runs(n))
        before = cal.objective().mean() / (args.prompt * B)
        cal.update_rotation()
        print(f"{B} prompts of {args.prompt} tokens in a {args.bits}-bit cache; objective a token and head {before:.4g}, rotations updated")
        kept = torch.tensor([b * nodes + i for b in range(B) for i in path], device=dev)
        rows = [draw(nodes * B) for _ in range(args.steps)]
        torch.cuda.synchronize()
        t = time.perf_counter()
        for x in rows:
            layer.step(x, runs(nodes), depth, mask, max_query=nodes, max_context=most)
            layer.commit(runs(len(path)), kept)
        torch.cuda.synchronize()
        ms = (time.perf_counter() - t) * 1e3 / max(args.steps, 1)
        print(f"{args.steps} steps of {nodes} drafted tokens a sequence, {len(path)} kept: {ms:.3f} ms a step, {int(layer.prefix[0])} tokens a sequence; "
              f"objective {cal.objective().mean() / max(args.steps * len(kept), 1):.4g}")
    finally:
        cal.close()


if __name__ == "__main__":
    main()
