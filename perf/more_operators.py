"""Attention over packed sequences and over chunks of new tokens, and moves of cached tokens, as cases that can be timed and compared.

`run` computes a case with elementary torch operations in 32 bits while `own` is false, and through the library's public
entry points (`paper_2605_10793_amd.attention`) where it is true.  Kinds:

  packed    attention of packed sequences over themselves; `train`: with the gradients of queries, keys and values
  chunk     attention of new tokens, from one to thousands of a sequence, over a paged cache that holds them already
  gather    tokens of a cache's sequences moved into other pages: a fork's last page, or the tokens that a sequence keeps

Scores.  A token at position p of its sequence gives key j the score cap * tanh(u / cap) - slope * |p - j|, u = q k_j / sqrt(width) (no cap:
u; no slopes: no distance), for keys from max(first, p - window + 1) on up to, not including, last; without bounds of its own a token sees
itself and all before it.

Layouts.  Queries, keys and values are [tokens, heads, width], here slices of one fused projection's output.  A cache is a
pool of pages: keys [pages, heads, page tokens, width], values [pages, heads, width, page tokens]; codes of 4 bits lie two in
a byte, entry j in the low half and entry j + width/2 in the high half; per page, head and token a (step, offset) pair of
32-bit floats, value = step * code + offset.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ------------------------------------------------------------------------------------------------ cases

def _packed(train, batch, fewest, most, q_heads, k_heads, width, mask, cap, slopes, name=None):
    c = dict(kind="packed", train=train, batch=batch, fewest=fewest, most=most, q_heads=q_heads, k_heads=k_heads, width=width, mask=mask, cap=cap,
             slopes=slopes)
    return dict(c, name=name) if name else c


def _chunk(batch, fewest, most, shortest, longest, q_heads, k_heads, width, bits, page, mask, cap, slopes, name=None):
    c = dict(kind="chunk", batch=batch, fewest=fewest, most=most, shortest=shortest, longest=longest, q_heads=q_heads, k_heads=k_heads, width=width,
             bits=bits, page=page, mask=mask, cap=cap, slopes=slopes)
    return dict(c, name=name) if name else c


def _gather(what, batch, shortest, longest, heads, width, bits, page, name=None):
    c = dict(kind="gather", what=what, batch=batch, shortest=shortest, longest=longest, heads=heads, width=width, bits=bits, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short question by itself: all launch latency
        _packed(False, 1, 77, 77, 32, 8, 128, "causal", 0.0, False, "attend_short"),
        # eight calibration sequences of 2048 tokens
        _packed(False, 8, 2048, 2048, 32, 8, 128, "causal", 0.0, False, "attend_calibration"),
        # four sequences packed with documents of uneven lengths and padded at their ends, scores capped
        _packed(False, 4, 2500, 4001, 16, 16, 64, "documents", 30.0, False, "attend_documents_capped"),
        # a training step's forward and backward on two calibration sequences
        _packed(True, 2, 2048, 2048, 32, 8, 128, "causal", 0.0, False, "train_calibration"),
        # prefixes that are seen from both sides, a bias that grows with distance, uneven lengths
        _packed(True, 5, 301, 1999, 24, 4, 64, "prefix", 0.0, True, "train_prefix_slopes"),
        # a single token of a single sequence, capped: latency again
        _chunk(1, 1, 1, 777, 777, 32, 8, 128, 16, 64, "causal", 50.0, False, "chunk_one_token"),
        # batched decoding within a window over uneven contexts, 16-bit cache
        _chunk(64, 1, 1, 501, 8190, 32, 8, 128, 16, 64, "window", 0.0, False, "chunk_decode_window"),
        # some drafted tokens of many sequences, 4-bit cache, a distance bias
        _chunk(32, 1, 7, 501, 8190, 32, 8, 128, 4, 64, "causal", 0.0, True, "chunk_few_4bit"),
        # four prompts' next 1024 tokens or fewer behind what is committed
        _chunk(4, 700, 1024, 0, 8000, 32, 8, 128, 16, 64, "causal", 0.0, False, "chunk_prompt"),
        # the next tokens of a long prompt, an image's among them, over an 8-bit cache
        _chunk(1, 777, 777, 30011, 30011, 32, 8, 128, 8, 128, "span", 0.0, False, "chunk_long_8bit"),
        # 64 beams forked from their parents: the pages that are not full are copied
        _gather("fork", 64, 500, 8000, 8, 128, 16, 64, "gather_fork"),
        # sequences of a 4-bit cache that drop a quarter of their tokens
        _gather("keep", 32, 500, 8000, 8, 128, 4, 64, "gather_keep_4bit"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["packed", "packed", "chunk", "chunk", "chunk", "gather"])
    width = rng.choice([64, 128, 128])
    k_heads = rng.choice([1, 2, 4, 8])
    if kind == "gather":
        return _gather(rng.choice(["fork", "keep"]), _log(rng, 1, 64), _log(rng, 1, 500), _log(rng, 500, 8000), k_heads, width, rng.choice([16, 16, 8, 4]),
                       rng.choice([16, 32, 64, 128, 256]))
    group = rng.choice([1, 2, 4, 4, 5, 8])
    q_heads = k_heads * group
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    slopes = rng.random() < 0.3
    if kind == "packed":
        train = rng.random() < 0.6
        width = rng.choice([64, 128, 128, 80])
        batch = _log(rng, 1, 16)
        most = _log(rng, 1, 4096)
        # no more pairs than the listed training step has
        while batch * most * most * q_heads * width > 2 * 2048 * 2048 * 32 * 128:
            most = most * 2 // 3
        return _packed(train, batch, rng.randint(max(1, most // 4), most), most, q_heads, k_heads, width,
                       rng.choice(["causal", "documents", "prefix", "window"]), cap, slopes)
    batch = _log(rng, 1, 64)
    most = rng.choice([1, _log(rng, 1, 16), _log(rng, 8, 1024)])
    most = max(1, min(most, 4096 // batch))
    longest = _log(rng, 1, max(1, min(32768, 270000 // batch, 250_000_000_000 // (batch * most * q_heads * width * 4))))
    bits = rng.choice([16, 16, 8, 4])
    return _chunk(batch, rng.randint(1, most), most, rng.randint(0, longest), longest, q_heads, k_heads, width, bits, rng.choice([16, 32, 64, 128, 256]),
                  rng.choice(["causal", "causal", "window", "span"]), cap, slopes)


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], uneven steps, in a mixed order, the same for every seed."""
    v = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    step = 7 if n % 7 else 5 if n % 5 else 3 if n % 3 else 1
    return [v[i * step % n] for i in range(n)]


def _counts(c):
    """New tokens of every sequence (packed: all of its tokens)."""
    return _spread(c["fewest"], c["most"], c["batch"])


def _committed(c):
    """Tokens that every sequence's cache holds before the new ones."""
    return [0] * c["batch"] if c["kind"] == "packed" else _spread(c["shortest"], c["longest"], c["batch"])


def _window(c):
    """Keys that a token sees at most, itself among them: half of the longest sequence.  0: no limit."""
    if c["mask"] != "window":
        return 0
    return max(1, (c["most"] + (0 if c["kind"] == "packed" else c["longest"])) // 2)


def _bounds(c):
    """first and last key of every token + 1, by sequence, as lists; None where each sees itself and all before it."""
    if c["mask"] in ("causal", "window"):
        return None
    both = []
    for n, a in zip(_counts(c), _committed(c)):
        if c["mask"] == "documents":      # documents of 5/16 of the sequence or what is left, the last tokens padding that sees nothing
            size, pad = max(1, n * 5 // 16), n // 9
            first = [i // size * size if i < n - pad else 0 for i in range(n)]
            last = [i + 1 if i < n - pad else 0 for i in range(n)]
        elif c["mask"] == "prefix":       # a quarter of the sequence is seen by all of it
            first, last = [0] * n, [max(i + 1, n // 4) for i in range(n)]
        else:                             # span: the second quarter of the new tokens sees its whole self
            lo, hi = n // 4, n // 2
            first, last = [0] * n, [a + (hi if lo <= i < hi else i + 1) for i in range(n)]
        both.append((first, last))
    return both


def _seen(c):
    """Pairs of tokens and keys that are seen, and keys that any token sees."""
    pairs = keys = 0
    bounds, w = _bounds(c), _window(c)
    for b, (n, a) in enumerate(zip(_counts(c), _committed(c))):
        lo, hi = a + n, 0
        for i in range(n):
            f, t = (bounds[b][0][i], bounds[b][1][i]) if bounds else (max(0, a + i + 1 - w) if w else 0, a + i + 1)
            if t > f:
                pairs += t - f
                lo, hi = min(lo, f), max(hi, t)
        keys += max(0, hi - lo)
    return pairs, keys


def _kept(c):
    """Tokens moved of every sequence."""
    return [n - n // c["page"] * c["page"] if c["what"] == "fork" else max(1, n * 3 // 4) for n in _committed(c)]


def work(case):
    c = case
    if c["kind"] == "gather":
        row = c["width"] * c["bits"] // 8 + (0 if c["bits"] == 16 else 8)      # a key or a value of one head in the cache
        tokens = sum(_kept(c))
        return {"bytes": 4 * tokens * c["heads"] * row + 4 * tokens, "flops": 0}
    pairs, keys = _seen(c)
    tokens, q, k = sum(_counts(c)), c["q_heads"] * c["width"], c["k_heads"] * c["width"]
    if c["kind"] == "packed":
        if c["train"]:      # q, k, v, the result's gradient in; the result and three gradients out
            return {"bytes": 2 * tokens * (4 * q + 4 * k), "flops": 14 * pairs * q}
        return {"bytes": 2 * tokens * (2 * q + 2 * k), "flops": 4 * pairs * q}
    row = c["width"] * c["bits"] // 8 + (0 if c["bits"] == 16 else 8)
    return {"bytes": 2 * keys * c["k_heads"] * row + 4 * tokens * q, "flops": 4 * pairs * q}


# ------------------------------------------------------------------------------------------------ inputs

def _activations(gen, tokens, heads, width, spread=0.5):
    """Log-normal channel scales with two outlier channels a head, as projections of a transformer give."""
    scale = torch.exp(spread * torch.randn(heads, width, device=DEV, generator=gen))
    scale[:, 1] *= 8
    scale[:, width // 2 + 3] *= 5
    return torch.randn(tokens, heads, width, device=DEV, generator=gen) * scale


def _unit(x, size):
    return x / x.square().mean(-1, keepdim=True).sqrt() * size


def _quantise(rows, bits):
    """The zero-point quantiser over the last dimension of 32-bit rows: codes, steps and offsets."""
    lo, hi = rows.amin(-1, keepdim=True), rows.amax(-1, keepdim=True)
    step = (hi - lo) / (2 ** bits - 1)
    zero = -torch.round(lo / step)
    code = torch.clamp(torch.round(rows / step) + zero, 0, 2 ** bits - 1)
    return code, step, -(step * zero)


def _packed_codes(code, bits):
    code = code.to(torch.uint8)
    if bits == 8:
        return code
    half = code.shape[-1] // 2
    return code[..., :half] | code[..., half:] << 4


def _pool(c, gen, pages, heads):
    """A cache in use: pages full of keys and values of earlier tokens."""
    page, width, bits = c["page"], c["width"], c["bits"]
    out = []
    for which in ("k", "v"):
        x = _activations(gen, pages * page, heads, width).view(pages, page, heads, width).transpose(1, 2)
        x = x.to(torch.bfloat16)
        if bits == 16:
            out += [x.contiguous() if which == "k" else x.transpose(2, 3).contiguous(), None]
            continue
        code, step, offset = _quantise(x.float(), bits)
        code = _packed_codes(code, bits)
        out += [code.contiguous() if which == "k" else code.transpose(2, 3).contiguous(), torch.cat([step, offset], -1).contiguous()]
    return out


def _table(c, gen, lengths, spare=0):
    """Pages of every sequence in a mixed order; `spare` pages more.  The table, and the number of pages."""
    need = [max(1, (n + c["page"] - 1) // c["page"]) for n in lengths]
    columns, pages = max(need), sum(need) + 3 + spare
    order = torch.randperm(pages, device=DEV, generator=gen, dtype=torch.int32)
    first = torch.tensor([sum(need[:b]) for b in range(len(need))], device=DEV)
    at = torch.arange(columns, device=DEV)
    table = order[(first[:, None] + at).clamp(max=pages - 1)]
    return torch.where(at < torch.tensor(need, device=DEV)[:, None], table, torch.zeros_like(table)).contiguous(), pages


def _starts(counts):
    return torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device=DEV)


def _slopes(c):
    return torch.exp2(-8 * (1 + torch.arange(c["q_heads"], device=DEV, dtype=torch.float32)) / c["q_heads"]) if c["slopes"] else None


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 13)
    s = {"case": c}
    if c["kind"] == "gather":
        lengths, kept = _committed(c), _kept(c)
        both, pages = _table(c, gen, lengths + kept)
        s["table"], s["to_table"] = both[:c["batch"]], both[c["batch"]:]
        s["k_pool"], s["k_scale"], s["v_pool"], s["v_scale"] = _pool(c, gen, pages, c["heads"])
        if c["what"] == "fork":
            pick = [torch.arange(n - m, n) for n, m in zip(lengths, kept)]
        else:
            host = torch.Generator().manual_seed(seed * 31 + 7)
            pick = [torch.randperm(n, generator=host)[:m].sort().values for n, m in zip(lengths, kept)]
        s["tokens"], s["start"] = torch.cat(pick).to(torch.int32).to(DEV), _starts(kept)
    else:
        counts, committed, heads = _counts(c), _committed(c), c["q_heads"] + 2 * c["k_heads"]
        tokens, bounds = sum(counts), _bounds(c)
        s["start"], s["slopes"], s["window"] = _starts(counts), _slopes(c), _window(c)
        s["counts"], s["committed"] = counts, committed      # what a program knows of its batch
        for i, x in enumerate(("first", "last")):
            s[x] = torch.tensor(sum((b[i] for b in bounds), []), dtype=torch.int32, device=DEV) if bounds else None
        if c["kind"] == "packed":
            fused = _activations(gen, tokens, heads, c["width"])
            fused[:, :c["q_heads"]] = _unit(fused[:, :c["q_heads"]], 1.5)      # queries and keys as their norms leave them
            fused[:, c["q_heads"]:c["q_heads"] + c["k_heads"]] = _unit(fused[:, c["q_heads"]:c["q_heads"] + c["k_heads"]], 1.0)
            fused = fused.to(torch.bfloat16)
            s["q"], s["k"], s["v"] = fused[:, :c["q_heads"]], fused[:, c["q_heads"]:c["q_heads"] + c["k_heads"]], fused[:, c["q_heads"] + c["k_heads"]:]
            if c["train"]:
                s["grad"] = torch.randn(tokens, c["q_heads"], c["width"], device=DEV, generator=gen).to(torch.bfloat16)
        else:
            s["table"], pages = _table(c, gen, [a + n for a, n in zip(committed, counts)])
            s["k_pool"], s["k_scale"], s["v_pool"], s["v_scale"] = _pool(c, gen, pages, c["k_heads"])
            s["prefix"] = torch.tensor(committed, dtype=torch.int32, device=DEV)
            s["context"] = max(a + n for a, n in zip(committed, counts))
            s["q"] = _unit(_activations(gen, tokens, c["q_heads"], c["width"]), 1.5).to(torch.bfloat16)
    if own and c["kind"] != "packed":          # the handle that a program keeps for its cache
        from paper_2605_10793_amd import attention as A
        s["cache"] = A.KVCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], bits=c["bits"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_mask(s, at, n, committed, length):
    """Which keys the tokens [at, at + n) of a sequence see, [tokens, keys], and how far apart they are."""
    p = torch.arange(committed, committed + n, device=DEV)[:, None]
    j = torch.arange(length, device=DEV)
    seen = j < (p + 1 if s["last"] is None else s["last"][at:at + n, None])
    if s["first"] is not None:
        seen = seen & (j >= s["first"][at:at + n, None])
    if s["window"]:
        seen = seen & (j > p - s["window"])
    return seen, (p - j).abs().float()


def _plain_weights(s, q, k, seen, apart):
    """Softmax weights [key heads, group * tokens, keys] of 32-bit rows [key heads, group * tokens, width], and the scores' tanh."""
    c = s["case"]
    group = c["q_heads"] // c["k_heads"]
    u, t = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(c["width"]), None
    if c["cap"]:
        t = torch.tanh(u / c["cap"])
        u = c["cap"] * t
    u = u.view(c["k_heads"], group, *seen.shape)
    if s["slopes"] is not None:
        u = u - s["slopes"].view(c["k_heads"], group, 1, 1) * apart
    u = u.masked_fill(~seen, -math.inf)
    top = u.amax(-1, keepdim=True)
    p = torch.exp(u - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return (p / torch.where(total == 0, torch.ones_like(total), total)).flatten(1, 2), t


def _by_head(x, k_heads):
    """[tokens, heads, width] as 32-bit [key heads, group * tokens, width]."""
    n, h, w = x.shape
    return x.float().view(n, k_heads, h // k_heads, w).permute(1, 2, 0, 3).reshape(k_heads, -1, w)


def _by_token(x, n):
    k, rows, w = x.shape
    return x.view(k, rows // n, n, w).permute(2, 0, 1, 3).reshape(n, -1, w)


def _plain_packed(s):
    c, at = s["case"], 0
    out = [[] for _ in range(4 if c["train"] else 1)]
    for n in s["counts"]:
        rows = slice(at, at + n)
        q, k, v = (_by_head(s[x][rows], c["k_heads"]) for x in ("q", "k", "v"))
        p, t = _plain_weights(s, q, k, *_plain_mask(s, at, n, 0, n))
        o = torch.matmul(p, v)
        out[0].append(_by_token(o, n))
        if c["train"]:
            g = _by_head(s["grad"][rows], c["k_heads"])
            out[3].append(_by_token(torch.matmul(p.transpose(1, 2).contiguous(), g), n))
            d = torch.matmul(g, v.transpose(1, 2).contiguous())
            d = p * (d - (g * o).sum(-1, keepdim=True)) / math.sqrt(c["width"])
            if t is not None:
                d = d * (1 - t * t)
            out[1].append(_by_token(torch.matmul(d, k), n))
            out[2].append(_by_token(torch.matmul(d.transpose(1, 2).contiguous(), q), n))
        at += n
    return [torch.cat(x).to(torch.bfloat16) for x in out]


def _plain_values(s, which, b, length):
    """A sequence's keys or values in 32 bits, [heads, tokens, width]."""
    c = s["case"]
    pages = s["table"][b, :(length + c["page"] - 1) // c["page"]].long()
    x = s[which + "_pool"][pages]                              # [pages, heads, ...]
    x = x if which == "k" else x.transpose(2, 3)
    if c["bits"] == 4:
        x = torch.cat([x & 15, x >> 4], -1)
    x = x.float()
    if c["bits"] != 16:
        pair = s[which + "_scale"][pages]
        x = x * pair[..., :1] + pair[..., 1:]
    return x.transpose(0, 1).flatten(1, 2)[:, :length].contiguous()


def _plain_chunk(s):
    c, at, out = s["case"], 0, []
    for b, (n, a) in enumerate(zip(s["counts"], s["committed"])):
        q = _by_head(s["q"][at:at + n], c["k_heads"])
        k, v = _plain_values(s, "k", b, a + n), _plain_values(s, "v", b, a + n)
        p, _ = _plain_weights(s, q, k, *_plain_mask(s, at, n, a, a + n))
        out.append(_by_token(torch.matmul(p, v), n))
        at += n
    return [torch.cat(out).to(torch.bfloat16)]


def _plain_gather(s):
    c = s["case"]
    rows = torch.arange(s["tokens"].shape[0], device=DEV)
    b = torch.searchsorted(s["start"][1:].contiguous(), rows.int(), right=True)
    to, token = rows - s["start"].long()[b], s["tokens"].long()
    page, slot = s["table"][b, token // c["page"]].long(), token % c["page"]
    to_page, to_slot = s["to_table"][b, to // c["page"]].long(), to % c["page"]
    s["k_pool"][to_page, :, to_slot] = s["k_pool"][page, :, slot]
    s["v_pool"][to_page, :, :, to_slot] = s["v_pool"][page, :, :, slot]
    if c["bits"] == 16:
        return [s["k_pool"], s["v_pool"]]
    for x in ("k_scale", "v_scale"):
        s[x][to_page, :, to_slot] = s[x][page, :, slot]
    return [s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"]]      # codes are moved as they are: equal, bit for bit


# ------------------------------------------------------------------------------------------------ the library's calls

def _own_packed(A, s):
    c = s["case"]
    options = dict(first=s["first"], last=s["last"], window=s["window"], cap=c["cap"], slopes=s["slopes"])
    if not c["train"]:
        return A.attention(s["q"], s["k"], s["v"], s["start"], **options)
    out, lse = A.attention(s["q"], s["k"], s["v"], s["start"], lse=True, **options)
    return [out, *A.attention_backward(s["q"], s["k"], s["v"], out, lse, s["grad"], s["start"], **options)]


def _own_chunk(A, s):
    c = s["case"]
    return A.chunk_attention(s["q"], s["cache"], s["start"], s["prefix"], s["table"], first=s["first"], last=s["last"], window=s["window"], cap=c["cap"],
                             slopes=s["slopes"], max_query=c["most"], max_context=s["context"])


def _own_gather(A, s):
    A.gather(s["cache"], s["tokens"], s["start"], s["table"], s["to_table"])
    return [s["k_pool"], s["v_pool"]] if s["case"]["bits"] == 16 else [s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"]]


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2605_10793_amd import attention as A
        out = {"packed": _own_packed, "chunk": _own_chunk, "gather": _own_gather}[kind](A, state)
    else:
        out = {"packed": _plain_packed, "chunk": _plain_chunk, "gather": _plain_gather}[kind](state)
    return list(out) if isinstance(out, (list, tuple)) else [out]


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_head(c, s, b, at, n, committed, head, q, k, v):
    """One sequence's result for one query head, from the definition."""
    length = k.shape[0]
    u = (q @ k.T.contiguous()) * c["width"] ** -0.5
    if c["cap"]:
        u = torch.tanh(u / c["cap"]) * c["cap"]
    place = torch.arange(committed, committed + n, device=DEV, dtype=torch.float64)
    keys = torch.arange(length, device=DEV, dtype=torch.float64)
    if c["slopes"]:
        u = u - s["slopes"][head].double() * (place[:, None] - keys).abs()
    low, high = torch.zeros_like(place), place + 1
    bounds, w = _bounds(c), _window(c)
    if bounds:
        low, high = (torch.tensor(x, device=DEV, dtype=torch.float64) for x in bounds[b])
    if w:
        low = torch.maximum(low, place - (w - 1))
    hidden = (keys < low[:, None]) | (keys >= high[:, None])
    none = hidden.all(-1)
    u = torch.where(hidden & ~none[:, None], torch.full_like(u, -math.inf), u)      # (rows that see nothing: replaced below)
    return torch.where(none[:, None], torch.zeros_like(q), torch.softmax(u, -1) @ v)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "gather":
        outs = [s["k_pool"], s["v_pool"]] + ([] if c["bits"] == 16 else [s["k_scale"], s["v_scale"]])
        outs = [x.double() if x.is_floating_point() else x for x in outs]
        old = [x.clone() for x in outs]
        page, i, kept, tokens = c["page"], 0, _kept(c), s["tokens"].tolist()
        table, to_table = s["table"].tolist(), s["to_table"].tolist()
        source, target = [], []
        for b, m in enumerate(kept):
            source += [(table[b][t // page], t % page) for t in tokens[i:i + m]]
            target += [(to_table[b][t // page], t % page) for t in range(m)]
            i += m
        if source:
            sp, ss, tp, ts = (torch.tensor(x, device=DEV) for x in (*zip(*source), *zip(*target)))
            for j, (x, y) in enumerate(zip(outs, old)):
                if j == 1:
                    x.transpose(2, 3)[tp, :, ts] = y.transpose(2, 3)[sp, :, ss]
                else:
                    x[tp, :, ts] = y[sp, :, ss]
        return outs
    counts, committed, group, at = _counts(c), _committed(c), c["q_heads"] // c["k_heads"], 0
    tokens = sum(counts)
    out = torch.zeros(tokens, c["q_heads"], c["width"], dtype=torch.float64, device=DEV)
    grads = None
    if c["kind"] == "packed" and c["train"]:
        grads = [torch.zeros_like(out)] + [torch.zeros(tokens, c["k_heads"], c["width"], dtype=torch.float64, device=DEV) for _ in range(2)]
    for b, (n, a) in enumerate(zip(counts, committed)):
        for kh in range(c["k_heads"]):
            if c["kind"] == "packed":
                k, v = s["k"][at:at + n, kh].double(), s["v"][at:at + n, kh].double()
            else:
                length = a + n
                pages, both = s["table"][b, :(length + c["page"] - 1) // c["page"]].long(), []
                for which in ("k", "v"):
                    x = s[which + "_pool"][pages, kh]
                    x = x if which == "k" else x.mT
                    if c["bits"] == 4:
                        x = torch.stack([x % 16, x // 16], -2).flatten(-2)
                    x = x.double()
                    if c["bits"] != 16:
                        pair = s[which + "_scale"][pages, kh].double()
                        x = x * pair[..., 0, None] + pair[..., 1, None]
                    both.append(x.flatten(0, 1)[:length])
                k, v = both
            for h in range(kh * group, (kh + 1) * group):
                q = s["q"][at:at + n, h].double()
                if grads is None:
                    out[at:at + n, h] = _exact_head(c, s, b, at, n, a, h, q, k, v)
                    continue
                leaves = [x.detach().clone().requires_grad_() for x in (q, k, v)]
                with torch.enable_grad():
                    o = _exact_head(c, s, b, at, n, a, h, *leaves)
                    g = torch.autograd.grad(o, leaves, s["grad"][at:at + n, h].double())
                out[at:at + n, h] = o.detach()
                grads[0][at:at + n, h] = g[0]
                grads[1][at:at + n, kh] += g[1]
                grads[2][at:at + n, kh] += g[2]
        at += n
    return [out] if grads is None else [out, *grads]
