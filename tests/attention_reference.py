"""Attention and its gradients from their definition in 64 bits on the CPU, with what 32-bit sums and bf16 factors may be off by."""
import math

import torch

HALF = 2.0 ** -8          # a rounding to bf16, relative


def attend(q, k, v, seen, place, scale, cap=0.0, slopes=None, grad=None, sizes=None):
    """One sequence: q [rows, heads, width] at `place` [rows], k, v [keys, key heads, width], seen [rows, keys].  Returns a dict of values and their
    tolerances: out, lse, and with `grad` dq, dk, dv.  sizes: for keys and values held as codes, what their entries are summed from at most, [keys, key heads]
    each (an offset, and a step times up to 128 + 255): 32-bit sums are off by parts of that, not of the values that are left."""
    q, k, v = q.double(), k.double(), v.double()
    heads, kv, width = q.shape[1], k.shape[1], q.shape[2]
    group = heads // kv
    distance = (place.double()[:, None] - torch.arange(k.shape[0], dtype=torch.float64)).abs()
    res = {n: torch.zeros(s, dtype=torch.float64) for n, s in
           (("out", q.shape), ("out_tol", q.shape), ("lse", q.shape[:2]), ("lse_tol", q.shape[:2]), ("dq", q.shape), ("dq_tol", q.shape), ("dk", k.shape),
            ("dk_tol", k.shape), ("dv", v.shape), ("dv_tol", v.shape))}
    for h in range(heads):
        qh, kh, vh = q[:, h], k[:, h // group], v[:, h // group]
        u = scale * qh @ kh.T
        s = u if cap == 0 else cap * torch.tanh(u / cap)
        near = 1 - torch.tanh(u / cap) ** 2 if cap else torch.ones_like(u)
        if slopes is not None:
            s = s - slopes[h].double() * distance
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=torch.float64)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
        # A score: a sum of `width` products and a few operations in 32 bits, each 2^-24 of what is summed at most.  The exponent of 2 it becomes is off
        # by that over ln 2, the weight by that again; the weight and the sum each by a few more units.
        visible = torch.where(seen, torch.ones_like(s), torch.zeros_like(s))
        size = (abs(scale) * qh.abs() @ kh.abs().T + (cap if cap else 0.0) + (slopes[h].double() * distance if slopes is not None else 0.0)) * visible
        if sizes is not None:
            size = torch.maximum(size, abs(scale) * qh.abs().sum(-1, keepdim=True) * sizes[0][:, h // group].double()[None] * visible)
        eps = (width + 16) * 2.0 ** -24 * size.amax(-1, keepdim=True) + 2.0 ** -20 if s.shape[1] else torch.zeros_like(top)
        o, a = p @ vh, p @ vh.abs()
        res["out"][:, h] = o
        # weights rounded, and divided by their sum as rounded; then the result
        res["out_tol"][:, h] = 1.02 * (HALF * (a + o.abs()) + HALF * o.abs() + 2 * eps * a) + 1e-30
        if sizes is not None:      # a chain of sums over blocks of 64 keys, 32 of them in one product
            res["out_tol"][:, h] += (s.shape[1] / 64 + 64) * 2.0 ** -24 * (sizes[1][:, h // group].double() * visible).amax(-1, keepdim=True)
        res["lse"][:, h] = (top + torch.log(total))[:, 0]
        res["lse_tol"][:, h] = (1.02 * HALF + 2 * eps[:, 0] + 2.0 ** -22 * torch.where(top == -math.inf, torch.zeros_like(top), top).abs()[:, 0])
        if grad is None:
            continue
        g = grad[:, h].double()
        dp = g @ vh.T
        d = (g * o).sum(-1, keepdim=True)
        ds = p * (dp - d) * near
        # D takes the result; weights come from an lse whose sum was of rounded weights, and are rounded as factors
        d_tol = (g.abs() * res["out_tol"][:, h]).sum(-1, keepdim=True) + (width + 16) * 2.0 ** -24 * (g.abs() * o.abs()).sum(-1, keepdim=True)
        p_tol = p * (2 * HALF + 2 * eps) * 1.02
        ds_tol = 1.02 * (p * near * (d_tol + (width + 16) * 2.0 ** -24 * (g.abs() @ vh.abs().T)) + ds.abs() * (2 * HALF + 2 * eps) + p * (dp - d).abs() * 2.0 ** -20)
        res["dq"][:, h] = scale * ds @ kh
        res["dq_tol"][:, h] = abs(scale) * ds_tol @ kh.abs() + HALF * res["dq"][:, h].abs()
        res["dk"][:, h // group] += scale * ds.T @ qh
        res["dk_tol"][:, h // group] += abs(scale) * ds_tol.T @ qh.abs()
        res["dv"][:, h // group] += p.T @ g
        res["dv_tol"][:, h // group] += p_tol.T @ g.abs()
    for n in ("dk", "dv"):
        res[n + "_tol"] += HALF * res[n].abs()
    return res


def seen_of(count, first, last, window, committed=0):
    """[count, committed + count] truth values: which keys tokens committed, committed + 1, ... see.  first, last: lists, or None."""
    length = committed + count
    place, j = torch.arange(committed, length)[:, None], torch.arange(length)[None]
    lo = torch.zeros(count, 1, dtype=torch.long) if first is None else torch.as_tensor(first)[:, None]
    hi = place + 1 if last is None else torch.as_tensor(last)[:, None]
    if window:
        lo = torch.maximum(lo, place - window + 1)
    return (j >= lo) & (j < hi)


def close(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    same = (got == want) | (off <= tol) | (torch.isnan(want) & torch.isnan(got))
    if not bool(same.all()):
        at = tuple(int(x) for x in torch.nonzero(~same)[0])
        raise AssertionError(f"{what}: {int((~same).sum())} of {same.numel()} off, first at {at}: {float(got[at])} for {float(want[at])}, tolerance {float(tol[at])}")
