"""The attention layer around the calibrated heads, over libconqur.so (the C ABI declared in include/conqur.h).

Argument marshalling only, like `binding`: every step runs in the library's HIP kernels, PyTorch supplies device memory and
the stream (the current one of the tensors' device).  Nothing synchronises, nothing falls back to the CPU.

  Rotary                              the plan of a rotary position encoding (frequencies on the device)
  rotary                              positions into queries and keys, or back out of their gradients
  qk_norm_rotary, .._backward         per-head norms and positions in one pass, and that pass's gradients
  KVCache, append                     a paged cache of keys and values in bf16 or in 8- or 4-bit zero-point codes
  tree_attention                      attention of new tokens (a tree of drafted ones, a chain, a single one) over the cache

Rows are [tokens, heads, width] tensors of any token and head stride, e.g. slices of a fused projection's output.  All tensors of a call, its
plan and its cache lie on one device.  Nothing here is recorded for autograd: tensors that require gradients are refused where gradients are
enabled.
"""
from __future__ import annotations

import ctypes
import struct
import threading
from typing import Optional, Tuple

import torch
from torch import _C, bfloat16, contiguous_format, empty_like, float32, int32, int64

from . import binding

SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}

MOST_CONTEXT = (1 << 31) - 1       # tokens of a sequence that a call counts

# The HOST structs of the header, field by field (conqur_heads: pointer, two strides, heads).
_HEADS = "QqqQ"
_ROTARY = struct.Struct("=" + 6 * _HEADS + "QQQQ" + "Q" + "IIIII" + "ff" + "I")
_CACHE_BATCH = "QQQQQIIII" + "QQQqII"
_APPEND = struct.Struct("=" + _CACHE_BATCH + 4 * _HEADS + "Q")
_TREE = struct.Struct("=" + _CACHE_BATCH + 2 * _HEADS + "QQQQQ" + "If")
_ABSENT = (0, 0, 0, 0)
_NOTHING = (None, 0, 0)


def _check(status: int, what: str) -> None:
    if status != binding.OK:
        raise binding.ConqurError(status, f"{what} failed")


# A decode step makes three of these calls a layer, so what Python does around each counts as much as a small kernel: tensors are looked at with
# as few attribute reads as the checks need, torch's names are taken once, and the stream is asked for by device index (a pass of `rotary`
# 15.1 -> 10 us, of which the launch is 3.7).

def _rows(x, name: str, dtype, device: int, shape) -> Tuple[int, int, int, int]:
    stride = x.stride()
    if x.shape != shape or len(shape) != 3 or stride[2] != 1 or x.dtype is not dtype:
        raise ValueError(f"{name} must be a {list(shape)} device tensor of {dtype} with unit stride along the width")
    if x.get_device() != device:
        _elsewhere(x, name, device)
    return x.data_ptr(), stride[0], stride[1], shape[1]


def _vector(x, name: str, dtype, device: int, n: int) -> int:
    if x.dtype is not dtype or x.shape != (n,) or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} device tensor of {n} entries")
    if x.get_device() != device:
        _elsewhere(x, name, device)
    return x.data_ptr()


def _elsewhere(x, name: str, device: int):
    """A kernel takes addresses as they are: what lies on the host or on another GPU must not get that far."""
    raise ValueError(f"{name} lies on {x.device}, where a tensor on " + ("a GPU" if device < 0 else f"cuda:{device}") + " is needed")


def _no_gradient(what: str, instead: str) -> None:
    """These calls are not part of autograd's graph: a result would end it without a word."""
    raise ValueError(f"{what} records nothing for autograd: {instead}; call it under torch.no_grad() or on detached tensors")


def _run(call, device: int, *args) -> int:
    """A library call's status, on a device and its current stream."""
    if device == _C._cuda_getDevice():
        return call(*args, _C._cuda_getCurrentRawStream(device))
    with torch.cuda.device(device):
        return call(*args, _C._cuda_getCurrentRawStream(device))


def _like(x):
    return None if x is None else empty_like(x, memory_format=contiguous_format)


class Rotary:
    """Frequencies of a rotary position encoding over the first `part` entries of a head.  interleaved: pairs (2j, 2j + 1) instead of
    (j, j + part/2).  scaling: "none", "linear", "base", "bands" or "ramp", for contexts `factor` times the trained `context`
    (conqur_rotary_scaling in the header says what `low` and `high` are)."""

    def __init__(self, part: int, theta: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, low: float = 1.0,
                 high: float = 4.0, context: float = 8192.0, device: str = "cuda"):
        if scaling not in SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(SCALINGS)}")
        turns = torch.empty(max(part // 2, 1), dtype=torch.float64)
        magnitude = ctypes.c_float()
        _check(binding.load().conqur_rotary_frequencies(part, SCALINGS[scaling], theta, factor, low, high, context, turns.data_ptr(),
                                                        ctypes.byref(magnitude)), "conqur_rotary_frequencies")
        self.part, self.layout, self.magnitude = part, 1 if interleaved else 0, magnitude.value
        self.turns = turns.to(device)


def _rotary_call(plan, q, k, positions, q_out, k_out, q_grad=None, k_grad=None, q_weight=None, k_weight=None, transposed=0, eps=0.0) -> bytes:
    dtype = q.dtype
    if dtype is not bfloat16 and dtype is not float32:
        raise ValueError("queries and keys must be bf16 or fp32")
    shape, k_shape = q.shape, None if k is None else k.shape
    if len(shape) != 3 or (k is not None and (len(k_shape) != 3 or k_shape[0] != shape[0] or k_shape[2] != shape[2])):
        raise ValueError("queries and keys must be [tokens, heads, width], with as many tokens and as wide")
    tokens, _, width = shape
    device = q.get_device()
    if device < 0:
        _elsewhere(q, "q", device)
    if plan.turns.get_device() != device:
        _elsewhere(plan.turns, "the plan", device)
    same, k_same = (dtype, device, shape), (dtype, device, k_shape)
    return _ROTARY.pack(*_rows(q, "q", *same), *(_ABSENT if k is None else _rows(k, "k", *k_same)),
                        *_rows(q_out, "the result of q", *same), *(_ABSENT if k is None else _rows(k_out, "the result of k", *k_same)),
                        *(_ABSENT if q_grad is None else _rows(q_grad, "the gradient of q", *same)),
                        *(_ABSENT if k_grad is None else _rows(k_grad, "the gradient of k", *k_same)),
                        0 if q_weight is None else _vector(q_weight, "q_weight", dtype, device, width),
                        0 if k_weight is None else _vector(k_weight, "k_weight", dtype, device, width),
                        _vector(positions, "positions", int64, device, tokens), plan.turns.data_ptr(), tokens, width, plan.part, plan.layout,
                        1 if dtype is bfloat16 else 0, transposed, plan.magnitude, eps, 0)


def rotary(plan: Rotary, q, positions, k=None, out=None, k_out=None, transposed: bool = False):
    """Queries (and keys) rotated by their positions (int64, one per token), into new tensors unless `out` / `k_out` are given (they may
    be the inputs).  transposed: the transposed rotation, for gradients.  Returns the result of q, or of (q, k)."""
    if (q.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
        _no_gradient("rotary", "transposed=True takes gradients back")
    if out is None:
        out = _like(q)
    if k_out is None and k is not None:
        k_out = _like(k)
    call = _rotary_call(plan, q, k, positions, out, k_out, transposed=1 if transposed else 0)
    _check(_run(binding.load().conqur_rotary, q.get_device(), call), "conqur_rotary")
    return out if k is None else (out, k_out)


def qk_norm_rotary(plan: Rotary, q, k, q_weight, k_weight, positions, eps: float = 1e-6, out=None, k_out=None):
    """rotary(w x / sqrt(mean x^2 + eps)) of queries and keys, in one pass; returns (q, k)."""
    if (q.requires_grad or k.requires_grad or q_weight.requires_grad or k_weight.requires_grad) and torch.is_grad_enabled():
        _no_gradient("qk_norm_rotary", "qk_norm_rotary_backward gives its gradients")
    if out is None:
        out = _like(q)
    if k_out is None:
        k_out = _like(k)
    call = _rotary_call(plan, q, k, positions, out, k_out, q_weight=q_weight, k_weight=k_weight, eps=eps)
    _check(_run(binding.load().conqur_qk_norm_rotary, q.get_device(), call), "conqur_qk_norm_rotary")
    return out, k_out


def qk_norm_rotary_backward(plan: Rotary, q, k, q_weight, k_weight, positions, q_grad, k_grad, eps: float = 1e-6):
    """Gradients of qk_norm_rotary at inputs q, k, for the gradients q_grad, k_grad of its results: (of q, of k, of q_weight, of k_weight), the
    last two in fp32."""
    lib = binding.load()
    dq, dk = _like(q), _like(k)
    call = _rotary_call(plan, q, k, positions, dq, dk, q_grad, k_grad, q_weight, k_weight, eps=eps)
    width = q.shape[2]
    dw = torch.empty((2, width), dtype=float32, device=q.device)
    size = lib.conqur_qk_norm_rotary_workspace(width)
    workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
    at = dw.data_ptr()
    _check(_run(lib.conqur_qk_norm_rotary_backward, q.get_device(), call, at, at + 4 * width, workspace.data_ptr(), size),
           "conqur_qk_norm_rotary_backward")
    return dq, dk, dw[0], dw[1]


class KVCache:
    """A pool of pages.  bits 16: k [pages, heads, page_tokens, width] and v [pages, heads, width, page_tokens] in bf16; bits 8: uint8 codes in
    the same layout; bits 4: two codes a byte, width/2 bytes in place of width.  Codes have k_scale and v_scale [pages, heads, page_tokens,
    2] in fp32, (step, offset) of every token.  page_tokens: a power of two, 16 to 256; width 64 or 128.  `empty` allocates one."""

    def __init__(self, k, v, k_scale=None, v_scale=None, bits: int = 16):
        if bits not in (16, 8, 4):
            raise ValueError("bits must be 16, 8 or 4")
        dtype = bfloat16 if bits == 16 else torch.uint8
        if k.dim() != 4 or not k.is_cuda or k.dtype != dtype or not k.is_contiguous():
            raise ValueError(f"k must be a contiguous 4-D device tensor of {dtype}")
        pages, heads, page_tokens, n = k.shape
        if tuple(v.shape) != (pages, heads, n, page_tokens) or v.dtype != dtype or v.device != k.device or not v.is_contiguous():
            raise ValueError("k must be [pages, heads, page_tokens, n] and v [pages, heads, n, page_tokens], contiguous, of one type and device")
        for s in (k_scale, v_scale):
            if bits == 16:
                if s is not None:
                    raise ValueError("a bf16 cache has no scales")
            elif s is None or s.dtype != float32 or tuple(s.shape) != (pages, heads, page_tokens, 2) or s.device != k.device or not s.is_contiguous():
                raise ValueError("codes need contiguous fp32 k_scale and v_scale [pages, heads, page_tokens, 2]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page_tokens, self.bits = pages, heads, page_tokens, bits
        self.width = n * 2 if bits == 4 else n
        self.device = k.get_device()
        self._fields = (k.data_ptr(), v.data_ptr(), 0 if k_scale is None else k_scale.data_ptr(), 0 if v_scale is None else v_scale.data_ptr(),
                        pages, heads, self.width, page_tokens, bits)

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, width: int, bits: int = 16, device: str = "cuda") -> "KVCache":
        n, dtype = (width // 2, torch.uint8) if bits == 4 else (width, torch.uint8 if bits == 8 else bfloat16)
        k = torch.empty((pages, heads, page_tokens, n), dtype=dtype, device=device)
        v = torch.empty((pages, heads, n, page_tokens), dtype=dtype, device=device)
        scales = [None if bits == 16 else torch.empty((pages, heads, page_tokens, 2), dtype=float32, device=device) for _ in range(2)]
        return cls(k, v, *scales, bits=bits)


def _batch(start, prefix, table, device: int) -> Tuple:
    sequences, stride = prefix.shape[0], table.stride()
    if table.dim() != 2 or table.dtype is not int32 or stride[1] != 1 or table.shape[0] != sequences:
        raise ValueError("table must be a [sequences, columns] int32 device tensor with unit column stride")
    if table.get_device() != device:
        _elsewhere(table, "table", device)
    columns = table.shape[1]
    return (_vector(start, "start", int32, device, sequences + 1), _vector(prefix, "prefix", int32, device, sequences), table.data_ptr(),
            stride[0] if sequences > 1 else max(stride[0], columns), columns, sequences)


def append(cache: KVCache, k, v, start, prefix, table, values: bool = False, k_values=None, v_values=None):
    """New keys and values (bf16) into the cache.  Sequence b's rows are [start[b], start[b + 1]) and become its tokens prefix[b] and on;
    token i lies in slot i % page_tokens of page table[b, i // page_tokens] (int32 device tensors).  A start below the one before it: no rows;
    not with more than 512 sequences, whose starts must not fall.  values (8 or 4 bits): also returns
    what the cache holds of them, (k_values, v_values), in the given or in new bf16 tensors, where rows of
    tokens without a place are not written."""
    if (k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        _no_gradient("append", "it has no gradient")
    tokens = k.shape[0]
    device = cache.device
    same = (bfloat16, device, (tokens, cache.heads, cache.width))
    if values:
        k_values = _like(k) if k_values is None else k_values
        v_values = _like(v) if v_values is None else v_values
    call = _APPEND.pack(*cache._fields, *_batch(start, prefix, table, device), *_rows(k, "k", *same), *_rows(v, "v", *same),
                        *(_ABSENT if k_values is None else _rows(k_values, "k_values", *same)),
                        *(_ABSENT if v_values is None else _rows(v_values, "v_values", *same)), tokens)
    _check(_run(binding.load().conqur_cache_append, device, call), "conqur_cache_append")
    return (k_values, v_values) if values else None


class _Kept(threading.local):
    """The workspaces of tree_attention, each thread its own, by device and stream.  A call's launches meet in it: the calls of one thread on one
    stream come one behind the other, whatever their caches, those of two threads may be enqueued between each other's launches."""

    def __init__(self):
        self.rooms = {}


_kept = _Kept()


def tree_attention(q, cache: KVCache, start, prefix, table, mask=None, max_query: int = 64, max_context: Optional[int] = None,
                   scale: Optional[float] = None, out=None):
    """Attention of new tokens q (bf16 [tokens, heads, width]; packed as in `append`, which has put their keys and values into the cache) over
    the committed tokens and those new ones that mask (int64, bit j: new token j of the sequence) names; None: each sees itself and those
    before it.  max_query: most new tokens of a sequence (up to 64); max_context: most tokens, committed and new (default: what the table
    holds; a closer bound shares the work out better).  scale: 1 / sqrt(width) unless given.  Returns out.  Rows beyond max_query of a sequence
    and rows of no sequence have no result: they stay as they are in `out`; in a new tensor, rows beyond 64 of a sequence are zeros, and all of them
    where there are more tokens than sequences of max_query hold."""
    if q.requires_grad and torch.is_grad_enabled():
        _no_gradient("tree_attention", "it has no gradient")
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, width]")
    device = cache.device
    if _C._cuda_getDevice() != device:       # (what is asked below is asked of the current device)
        with torch.cuda.device(device):
            return tree_attention(q, cache, start, prefix, table, mask, max_query, max_context, scale, out)
    tokens, heads, _ = q.shape
    width = cache.width
    if out is None:
        out = _like(q)
        # (a max_query below 64 is the caller's word, unless the tokens are too many for it)
        if tokens > max_query and (max_query >= 64 or tokens > prefix.shape[0] * max_query):
            out.zero_()
    same = (bfloat16, device, (tokens, heads, width))
    fields = (*cache._fields, *_batch(start, prefix, table, device), *_rows(q, "q", *same), *_rows(out, "out", *same),
              0 if mask is None else _vector(mask, "mask", int64, device, tokens), tokens,
              min(table.shape[1] * cache.page_tokens, MOST_CONTEXT) if max_context is None else max_context)
    tail = (max_query, width ** -0.5 if scale is None else scale)
    lib = binding.load()
    at = device, _C._cuda_getCurrentRawStream(device)
    # (a graph keeps the room it was captured with: it takes its own, from its memory pool)
    capturing = _C._cuda_isCurrentStreamCapturing()
    rooms = _kept.rooms
    have = _NOTHING if capturing else rooms.get(at, _NOTHING)
    status = lib.conqur_tree_attention(_TREE.pack(*fields, *have[1:], *tail), at[1])
    if status == binding.EINVAL:       # perhaps for want of room alone: one that is large enough stays
        size = lib.conqur_tree_attention_workspace(_TREE.pack(*fields, 0, 0, *tail))
        if size > have[2]:
            room = torch.empty(size, dtype=torch.uint8, device=q.device)
            have = (room, room.data_ptr(), size)
            if not capturing:
                rooms[at] = have
            status = lib.conqur_tree_attention(_TREE.pack(*fields, *have[1:], *tail), at[1])
    _check(status, "conqur_tree_attention")
    return out
