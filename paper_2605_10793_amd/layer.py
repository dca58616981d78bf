"""An attention layer that serves drafted tokens over a paged cache and calibrates its heads' rotations on the way, and that trains on packed sequences.

`AttentionLayer` runs the operators of `attention` as a server would, one step for a batch of sequences: norms and positions of queries and
keys, the new keys and values into the cache, attention of every new token over its sequence and those drafted tokens it follows.  The
step's output rows are the per-head activations in front of the output projection, one of the sites whose rotations the paper calibrates
(App. A); a `binding.Calibrator` with as many heads takes those of the tokens that stay.

    python -m paper_2605_10793_amd.layer [--bits 4] [--sequences 8] [--prompt 512] [--chunk 64] [--steps 24] [--beams 0]

feeds random prompts in chunks, calibrates on them, then drafts a tree of tokens a step and commits one of its paths; with --beams, every sequence goes on
from a random one of each group of that many after every step.
"""
from __future__ import annotations

import argparse
import random
import time
from typing import Optional

import torch

from . import attention, binding


class AttentionLayer:
    """table: int32 [sequences, columns], the pages of `cache` that each sequence may use.  q_weight, k_weight: of the per-head norms.
    calibrator: takes the outputs of the tokens that are committed, or None; it may have been made on any stream of the cache's device.  window, cap,
    slopes: of the attention (attention.chunk_attention); they leave no masks to trees of drafted tokens."""

    def __init__(self, plan: attention.Rotary, q_weight, k_weight, cache: attention.KVCache, table, eps: float = 1e-6,
                 calibrator: Optional[binding.Calibrator] = None, window: int = 0, cap: float = 0.0, slopes=None):
        self.plan, self.q_weight, self.k_weight, self.cache, self.table, self.eps = plan, q_weight, k_weight, cache, table, eps
        if calibrator is not None and calibrator.device != cache.device:
            raise ValueError(f"the calibrator is on cuda:{calibrator.device}, the cache on cuda:{cache.device}")
        self.calibrator = calibrator
        self.prefix = torch.zeros(table.shape[0], dtype=torch.int32, device=table.device)      # committed tokens
        self._ahead = None             # by how much the sequences' next positions lie ahead of that; None: nowhere
        self.window, self.cap, self.slopes = window, cap, slopes
        self._last = self._trained = None
        self._moved = False            # whether sequences went on from others, or dropped tokens, since the last step

    def step(self, fused, start, depth=None, mask=None, max_query: int = 64, max_context: Optional[int] = None):
        """New tokens of every sequence, at most max_query each (64 at most of a tree): fused [tokens, heads + 2 cache heads, width] holds their queries, keys and
        values, start (int32 [sequences + 1], 0 or more) the first row of each sequence, in their order; a start below one before it: a sequence of none, as if
        that had been repeated.  A tree of drafted tokens has its tokens' depths (int64) and masks
        (attention.tree_attention); without them they are a chain.  max_query: the most of a sequence, so that every token has a result.  Returns
        [tokens, heads, width].  Nothing is committed."""
        tokens, kv = fused.shape[0], self.cache.heads
        if tokens > self.table.shape[0] * max_query:
            raise ValueError(f"{tokens} tokens are more than {max_query} for each of {self.table.shape[0]} sequences")
        options = bool(self.window or self.cap or self.slopes is not None)
        if mask is not None and options:
            raise ValueError("a layer with a window, capped scores or slopes takes chains of tokens, no trees")
        q, k, v = self._split(fused)
        rows = torch.arange(tokens, dtype=torch.int32, device=fused.device)
        # (rows of no sequence: the last; where a start falls, those behind it begin where rows end)
        sequence = torch.searchsorted(start.cummax(0).values[1:-1], rows, right=True)
        first = self.prefix if self._ahead is None else self.prefix + self._ahead
        if depth is None:
            first = first - start[:-1]
        positions = first[sequence] + (rows.long() if depth is None else depth)
        q_out, k_out = attention.qk_norm_rotary(self.plan, q, k, self.q_weight, self.k_weight, positions, eps=self.eps)
        attention.append(self.cache, k_out, v, start, self.prefix, self.table)
        if options or (mask is None and max_query > 64):
            out = attention.chunk_attention(q_out, self.cache, start, self.prefix, self.table, window=self.window, cap=self.cap, slopes=self.slopes,
                                            max_query=max_query, max_context=max_context)
        else:
            out = attention.tree_attention(q_out, self.cache, start, self.prefix, self.table, mask=mask, max_query=max_query, max_context=max_context)
        self._last, self._moved = (q, k, v, k_out, positions, out), False
        return out

    def _split(self, fused):
        heads = fused.shape[1] - 2 * self.cache.heads
        return fused[:, :heads], fused[:, heads:heads + self.cache.heads], fused[:, heads + self.cache.heads:]

    def branch(self, parents, table):
        """Every sequence goes on from one of them, parents (int64 [sequences]), in the pages of `table` (as large as the present one): the parent's full pages
        stand in front of it, shared, whatever it holds there, and the page that the parent has begun is copied to the one behind them.  That and what
        follows must be pages that nothing else uses (attention.Pages keeps count)."""
        if table.shape != self.table.shape:
            raise ValueError(f"table must be {list(self.table.shape)}, as the present one")
        page, sequences = self.cache.page_tokens, self.table.shape[0]
        prefix, old = self.prefix[parents], self.table[parents]
        full = (prefix // page)[:, None]
        at = torch.arange(page, dtype=torch.int32, device=prefix.device)
        tokens = torch.where(at < (prefix % page)[:, None], full * page + at, -1)          # (-1: no token, nothing is moved)
        start = torch.arange(sequences + 1, dtype=torch.int32, device=prefix.device) * page
        begun = table.gather(1, full.long().clamp_(max=table.shape[1] - 1))
        attention.gather(self.cache, tokens.flatten(), start, old, begun)
        self.table = torch.where(torch.arange(table.shape[1], device=prefix.device) < full, old, table)
        self.prefix, self._moved = prefix, True
        if self._ahead is not None:
            self._ahead = self._ahead[parents]

    @property
    def position(self):
        """Of each sequence (int32), the position that its next token gets: the number of committed tokens, unless `keep` was told another."""
        return self.prefix.clone() if self._ahead is None else self.prefix + self._ahead

    def keep(self, tokens, start, table, position=None):
        """The sequences keep these of their tokens (as in attention.gather), in the pages of `table`, which nothing reads.  The keys keep their positions: where
        tokens were dropped that others stood behind, `position` (int32 [sequences]) says where those that follow stand, for them to be as far from each key as
        they would have been: `layer.position`, if they follow the last one.  None: they get positions from the number of tokens that are left on, which is right
        where a sequence keeps its first ones.  Windows and slopes go by the tokens that are left."""
        attention.gather(self.cache, tokens, start, self.table, table)
        start = start.clamp(0, tokens.shape[0])        # as gather reads it
        self.table, self.prefix, self._moved = table, start[1:] - start[:-1], True
        self._ahead = None if position is None else position - self.prefix

    def packed(self, fused, start, first=None, last=None):
        """Whole sequences, packed, for training: fused as in step, start (int32 [sequences + 1], any number of them, not falling) the first row of each, first and
        last the bounds of what tokens see (attention.attention).  Returns [tokens, heads, width], which a calibrator may take as it takes a step's; the cache is not
        used."""
        q, k, v = self._split(fused)
        rows = torch.arange(fused.shape[0], dtype=torch.int32, device=fused.device)
        positions = (rows - start[(torch.searchsorted(start, rows, right=True) - 1).clamp_(min=0)]).long()
        q_out, k_out = attention.qk_norm_rotary(self.plan, q, k, self.q_weight, self.k_weight, positions, eps=self.eps)
        bounds = dict(first=first, last=last, window=self.window, cap=self.cap, slopes=self.slopes)
        out, lse = attention.attention(q_out, k_out, v, start, lse=True, **bounds)
        self._trained = q, k, v, q_out, k_out, positions, start, bounds, out, lse
        return out

    def packed_gradients(self, grad):
        """From the gradient of what `packed` returned last: those of fused, of q_weight and of k_weight."""
        q, k, v, q_out, k_out, positions, start, bounds, out, lse = self._trained
        dq, dk, dv = attention.attention_backward(q_out, k_out, v, out, lse, grad, start, **bounds)
        dq, dk, dq_weight, dk_weight = attention.qk_norm_rotary_backward(self.plan, q, k, self.q_weight, self.k_weight, positions, dq, dk, eps=self.eps)
        return torch.cat([dq, dk, dv], 1), dq_weight, dk_weight

    def commit(self, start, rows=None):
        """The tokens of the last step that stay.  rows (int64): their row numbers there, each sequence's from its root on, start (int32
        [sequences + 1]) the first entry of each sequence; None: all rows, as they were passed.  Kept keys and values move to the places
        behind the committed ones, and their outputs go to the calibrator.  Not after a branch or `keep`, which take committed tokens alone."""
        if self._moved:
            raise ValueError("the last step's tokens were not committed before sequences went on from others or dropped tokens")
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
    ap.add_argument("--chunk", type=int, default=64, help="tokens of a prompt that go at a time")
    ap.add_argument("--steps", type=int, default=24, help="drafting steps")
    ap.add_argument("--beams", type=int, default=0, help="sequences of a group that go on from random ones of it after every step (0: each by itself)")
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
    cache = attention.KVCache.empty(B * columns * (2 if args.beams else 1), kv, page, width, args.bits, dev)
    pages = attention.Pages(cache.pages)
    held = [pages.take(columns) for _ in range(B)]
    table = torch.tensor(held, dtype=torch.int32, device=dev)
    R0 = torch.eye(width).repeat(heads, 1, 1).numpy()
    weight = torch.ones(width, dtype=torch.bfloat16, device=dev)
    cal = binding.Calibrator(heads * width, heads, "bf16", R0, max_tokens=max(64, args.chunk) * B)
    layer = AttentionLayer(attention.Rotary(width, 500000.0, device=dev), weight, weight, cache, table, calibrator=cal)
    try:
        for at in range(0, args.prompt, args.chunk):
            n = min(args.chunk, args.prompt - at)
            layer.step(draw(n * B), runs(n), max_query=n, max_context=most)
            layer.commit(runs(n))
        before = cal.objective().mean() / (args.prompt * B)
        cal.update_rotation()
        print(f"{B} prompts of {args.prompt} tokens in a {args.bits}-bit cache; objective a token and head {before:.4g}, rotations updated")
        kept = torch.tensor([b * nodes + i for b in range(B) for i in path], device=dev)
        rows = [draw(nodes * B) for _ in range(args.steps)]
        choose = random.Random(0)
        torch.cuda.synchronize()
        t, committed = time.perf_counter(), args.prompt
        for x in rows:
            layer.step(x, runs(nodes), depth, mask, max_query=nodes, max_context=most)
            layer.commit(runs(len(path)), kept)
            committed += len(path)
            if args.beams:
                parents = [b // args.beams * args.beams + choose.randrange(min(args.beams, B - b // args.beams * args.beams)) for b in range(B)]
                shared = [held[p][:committed // page] for p in parents]
                for x in shared:
                    pages.share(x)
                fresh = [x + pages.take(columns - len(x)) for x in shared]
                for x in held:
                    pages.release(x)
                held = fresh
                layer.branch(torch.tensor(parents, device=dev), torch.tensor(held, dtype=torch.int32, device=dev))
        torch.cuda.synchronize()
        ms = (time.perf_counter() - t) * 1e3 / max(args.steps, 1)
        print(f"{args.steps} steps of {nodes} drafted tokens a sequence, {len(path)} kept: {ms:.3f} ms a step, {int(layer.prefix[0])} tokens a sequence; "
              f"objective {cal.objective().mean() / max(args.steps * len(kept), 1):.4g}")
    finally:
        cal.close()


if __name__ == "__main__":
    main()
