"""The attention-side operators of this library, as cases that can be timed and compared.

`run` computes a case with elementary torch operations in 32 bits while `own` is false, and through the library's public
entry points (`paper_2605_10793_amd.attention`) where it is true.  Kinds:

  rotary    positions rotated into queries and keys (or, transposed, out of their gradients)
  norm      queries and keys normalised per head and rotated in one pass; `backward`: that pass's gradients
  append    new keys and values put into the pages of a cache: 16-bit, or the zero-point codes of 8 or 4 bits, then with the
            values that the cache holds as outputs (what a quantisation-aware stream goes on with)
  tree      attention of drafted tokens (a tree of them for each sequence, or one token) over that cache

Layouts.  Queries, keys and values are [tokens, heads, width], here slices of one fused projection's output.  A cache is a
pool of pages: keys [pages, heads, page tokens, width], values [pages, heads, width, page tokens]; codes of 4 bits lie two in
a byte, entry j in the low half and entry j + width/2 in the high half; per page, head and token a (step, offset) pair of
32-bit floats, value = step * code + offset.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases

def _rotary(tokens, q_heads, k_heads, width, part, dtype, layout, scaling, transposed, first, name=None):
    c = dict(kind="rotary", tokens=tokens, q_heads=q_heads, k_heads=k_heads, width=width, part=part, dtype=dtype, layout=layout,
             scaling=scaling, transposed=transposed, first=first)
    return dict(c, name=name) if name else c


def _norm(tokens, q_heads, k_heads, width, part, dtype, layout, scaling, backward, first, name=None):
    c = dict(kind="norm", tokens=tokens, q_heads=q_heads, k_heads=k_heads, width=width, part=part, dtype=dtype, layout=layout,
             scaling=scaling, backward=backward, first=first)
    return dict(c, name=name) if name else c


def _append(batch, fewest, most, committed, heads, width, bits, page, name=None):
    c = dict(kind="append", batch=batch, fewest=fewest, most=most, committed=committed, heads=heads, width=width, bits=bits, page=page)
    return dict(c, name=name) if name else c


def _tree(batch, nodes, shortest, longest, q_heads, k_heads, width, bits, page, name=None):
    c = dict(kind="tree", batch=batch, nodes=nodes, shortest=shortest, longest=longest, q_heads=q_heads, k_heads=k_heads, width=width,
             bits=bits, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence on its way into attention: all launch latency
        _rotary(1, 32, 8, 128, 128, "bf16", "half", "none", False, 777, "rotary_one_token"),
        # two calibration sequences of 2048 tokens, half of every head rotated, far into a stretched context
        _rotary(4096, 32, 8, 128, 64, "bf16", "interleaved", "bands", False, 100000, "rotary_prompt_part"),
        # the way back in fp32, a width and a token count that fit no power of two
        _rotary(1999, 32, 32, 80, 80, "f32", "half", "linear", True, 0, "rotary_gradient_f32"),
        # a batch of 64 sequences decoding one token each
        _norm(64, 32, 8, 128, 128, "bf16", "half", "none", False, 3000, "norm_decode"),
        # a prompt batch
        _norm(8192, 32, 8, 128, 128, "bf16", "half", "ramp", False, 0, "norm_prompt"),
        # the same batch's gradients
        _norm(8192, 32, 8, 128, 128, "bf16", "half", "none", True, 0, "norm_gradient"),
        # the decoding batch's new keys and values into a 4-bit cache
        _append(64, 1, 1, 2900, 8, 128, 4, 64, "append_decode_4bit"),
        # eight prompts of uneven length, the longest 2048 tokens, into 16-bit pages
        _append(8, 517, 2048, 0, 8, 128, 16, 64, "append_prompts_16bit"),
        # a single short sequence: latency again
        _tree(1, 1, 777, 777, 32, 8, 128, 16, 64, "tree_one_token_short"),
        # batched decoding over uneven contexts, 16-bit cache
        _tree(64, 1, 501, 8190, 32, 8, 128, 16, 64, "tree_decode_batch"),
        # drafted trees of 48 tokens being verified for eight sequences, 8-bit cache
        _tree(8, 48, 1000, 16000, 32, 8, 128, 8, 64, "tree_verify_8bit"),
        # five drafted tokens at the end of a very long context, 4-bit cache
        _tree(2, 5, 120000, 131067, 32, 8, 128, 4, 128, "tree_long_4bit"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotary", "norm", "append", "tree", "tree"])
    if kind in ("rotary", "norm"):
        width = rng.choice([64, 80, 96, 128, 128, 256])
        part = rng.choice([width, width, width // 2])
        k_heads = rng.choice([1, 2, 4, 8, 16])
        q_heads = k_heads * rng.choice([1, 2, 4, 5, 8])
        q_heads = min(q_heads, 64)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        layout = rng.choice(["half", "half", "interleaved"])
        scaling = rng.choice(["none", "linear", "base", "bands", "ramp"])
        back = rng.random() < 0.4
        most = 8192 * 40 * 128 * 2 // ((q_heads + k_heads) * width * (4 if dtype == "f32" else 2))
        tokens = _log(rng, 1, min(16384, max(2, most)))
        first = _log(rng, 1, 500000)
        return (_rotary if kind == "rotary" else _norm)(tokens, q_heads, k_heads, width, part, dtype, layout, scaling, back, first)
    width = rng.choice([64, 128, 128])
    page = rng.choice([32, 64, 128, 256])
    bits = rng.choice([16, 16, 8, 4])
    k_heads = rng.choice([1, 2, 4, 8])
    batch = _log(rng, 1, 64)
    if kind == "append":
        if rng.random() < 0.5:
            return _append(batch, 1, _log(rng, 1, 64), _log(rng, 1, 8000), k_heads, width, bits, page)
        most = _log(rng, 2, min(4096, 16384 // batch))
        return _append(batch, rng.randint(1, most), most, _log(rng, 1, 500), k_heads, width, bits, page)
    nodes = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 2, 64)])
    group = rng.choice([1, 2, 4, 4, 7, 8])
    # no more products than the listed trees have, no more tokens held than the listed batch
    most = min(131072, 280000 // batch, 13_000_000_000 // (batch * nodes * k_heads * group * width))
    longest = _log(rng, 16, max(16, most))
    shortest = rng.randint(max(1, longest // 8), longest)
    return _tree(batch, nodes, shortest, longest, k_heads * group, k_heads, width, bits, page)


def _spread(lo, hi, n):
    """n whole numbers over [lo, hi], uneven steps, in a mixed order, the same for every seed."""
    v = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    step = 7 if n % 7 else 5 if n % 5 else 3 if n % 3 else 1
    return [v[i * step % n] for i in range(n)]


def _counts(c):
    """New tokens of every sequence."""
    if c["kind"] == "append":
        return _spread(c["fewest"], c["most"], c["batch"])
    return [c["nodes"]] * c["batch"]


def _committed(c):
    """Tokens that every sequence's cache holds already."""
    if c["kind"] == "append":
        return _spread(c["committed"] // 2, c["committed"], c["batch"])
    return _spread(c["shortest"], c["longest"], c["batch"])


def work(case):
    c = case
    if c["kind"] in ("rotary", "norm"):
        e = 4 if c["dtype"] == "f32" else 2
        values = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["width"]
        if c["kind"] == "rotary":
            return {"bytes": 2 * values * e + 8 * c["tokens"], "flops": 3 * values * c["part"] / c["width"]}
        if c["backward"]:
            return {"bytes": 3 * values * e + 8 * c["tokens"] + 2 * c["width"] * (e + 4), "flops": 14 * values}
        return {"bytes": 2 * values * e + 8 * c["tokens"] + 2 * c["width"] * e, "flops": 8 * values}
    row = c["width"] * c["bits"] // 8 + (0 if c["bits"] == 16 else 8)      # a key or a value of one head in the cache
    tokens = sum(_counts(c))
    heads = c["heads"] if c["kind"] == "append" else c["k_heads"]
    if c["kind"] == "append":
        values = 2 * tokens * heads * c["width"]
        return {"bytes": 2 * values + 2 * tokens * heads * row + (0 if c["bits"] == 16 else 2 * values), "flops": 6 * values}
    held = sum(a + b for a, b in zip(_committed(c), _counts(c)))
    seen = sum(n * (a + 1) for a, n in zip(_committed(c), _counts(c)))     # itself and the committed tokens at least
    return {"bytes": 2 * held * heads * row + 4 * tokens * c["q_heads"] * c["width"] + 12 * tokens,
            "flops": 4 * seen * c["q_heads"] * c["width"]}


# ------------------------------------------------------------------------------------------------ inputs

def _dtype(c):
    return torch.float32 if c.get("dtype") == "f32" else torch.bfloat16


def _activations(gen, tokens, heads, width, spread=0.5):
    """Log-normal channel scales with two outlier channels a head, as projections of a transformer give."""
    scale = torch.exp(spread * torch.randn(heads, width, device=DEV, generator=gen))
    scale[:, 1] *= 8
    scale[:, width // 2 + 3] *= 5
    return torch.randn(tokens, heads, width, device=DEV, generator=gen) * scale


def _scaling(name):
    """The arguments of a stretched context: factor, the two bounds, and the context the model was trained on."""
    return {"none": (1.0, 0.0, 0.0, 0.0), "linear": (4.0, 0.0, 0.0, 0.0), "base": (4.0, 0.0, 0.0, 0.0),
            "bands": (8.0, 1.0, 4.0, 8192.0), "ramp": (16.0, 1.0, 32.0, 4096.0)}[name]


THETA = 10000.0


def _frequencies(c):
    """Turns a position adds to every pair (float64), and the factor on the result."""
    factor, low, high, context = _scaling(c["scaling"])
    pairs = torch.arange(c["part"] // 2, dtype=torch.float64)
    theta, magnitude = THETA, 1.0
    if c["scaling"] == "base":
        theta = THETA * factor ** (c["part"] / max(1, c["part"] - 2))
    turns = torch.exp(-2 * pairs / c["part"] * math.log(theta)) / (2 * math.pi)
    if c["scaling"] == "linear":
        turns = turns / factor
    elif c["scaling"] == "bands":
        keep = ((turns * context - low) / (high - low)).clamp(0, 1)        # turns made within the trained context
        turns = keep * turns + (1 - keep) * turns / factor
    elif c["scaling"] == "ramp":
        first, last = (c["part"] * math.log(context / (r * 2 * math.pi)) / (2 * math.log(THETA)) for r in (high, low))
        first, last = max(0, math.floor(first)), min(c["part"] - 1, math.ceil(last))
        keep = 1 - ((pairs - first) / max(last - first, 1e-3)).clamp(0, 1)
        turns = keep * turns + (1 - keep) * turns / factor
        magnitude = 0.1 * math.log(factor) + 1
    return turns.to(DEV), magnitude


def _positions(c):
    """A batch of packed sequences: positions run up from `first` and start again, twice."""
    p = torch.arange(c["tokens"], dtype=torch.int64, device=DEV)
    return c["first"] + p % max(1, (c["tokens"] + 1) // 2)


def _ancestors(parents):
    """Bit j of entry i: node i sees node j, one of its ancestors or itself."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    return [m - (1 << 64) if m >> 63 else m for m in seen]


def _quantise(rows, bits):
    """The zero-point quantiser over the last dimension of 32-bit rows: codes, steps and offsets."""
    lo, hi = rows.amin(-1, keepdim=True), rows.amax(-1, keepdim=True)
    step = (hi - lo) / torch.full_like(lo, 2 ** bits - 1)
    flat = step == 0
    safe = torch.where(flat, torch.ones_like(step), step)
    zero = -torch.round(lo / safe)
    code = torch.clamp(torch.round(rows / safe) + zero, 0, 2 ** bits - 1)
    code = torch.where(flat, torch.zeros_like(code), code)
    offset = torch.where(flat, lo, -(step * zero))
    return code, step, offset


def _packed(code, bits):
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
        code = _packed(code, bits)
        out += [code.contiguous() if which == "k" else code.transpose(2, 3).contiguous(), torch.cat([step, offset], -1).contiguous()]
    return out


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 13)
    s = {"case": c}
    if c["kind"] in ("rotary", "norm"):
        heads, width, dt = c["q_heads"] + 2 * c["k_heads"], c["width"], _dtype(c)
        fused = _activations(gen, c["tokens"], heads, width).to(dt)
        s["q"], s["k"] = fused[:, :c["q_heads"]], fused[:, c["q_heads"]:c["q_heads"] + c["k_heads"]]
        s["positions"] = _positions(c)
        s["turns"], s["magnitude"] = _frequencies(c)
        if c["kind"] == "norm":
            s["q_weight"] = (1 + 0.3 * torch.randn(width, device=DEV, generator=gen)).to(dt)
            s["k_weight"] = (1 + 0.3 * torch.randn(width, device=DEV, generator=gen)).to(dt)
            if c["backward"]:
                s["q_grad"] = torch.randn(c["tokens"], c["q_heads"], width, device=DEV, generator=gen).to(dt)
                s["k_grad"] = torch.randn(c["tokens"], c["k_heads"], width, device=DEV, generator=gen).to(dt)
        if own:      # the plan that a program makes once for its model
            from paper_2605_10793_amd import attention as A
            factor, low, high, context = _scaling(c["scaling"])
            s["plan"] = A.Rotary(c["part"], THETA, interleaved=c["layout"] == "interleaved", scaling=c["scaling"], factor=factor, low=low,
                                 high=high, context=context, device=DEV)
        return s
    heads = c["heads"] if c["kind"] == "append" else c["k_heads"]
    counts, committed = _counts(c), _committed(c)
    need = [(a + n + c["page"] - 1) // c["page"] for a, n in zip(committed, counts)]
    columns, pages = max(need), sum(need) + 3
    order = torch.randperm(pages, device=DEV, generator=gen, dtype=torch.int32)
    first = torch.tensor([sum(need[:b]) for b in range(len(need))], device=DEV)
    at = torch.arange(columns, device=DEV)
    table = order[(first[:, None] + at).clamp(max=pages - 1)]
    s["table"] = torch.where(at < torch.tensor(need, device=DEV)[:, None], table, torch.zeros_like(table)).contiguous()
    s["k_pool"], s["k_scale"], s["v_pool"], s["v_scale"] = _pool(c, gen, pages, heads)
    s["prefix"] = torch.tensor(committed, dtype=torch.int32, device=DEV)
    s["start"] = torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device=DEV)
    tokens = sum(counts)
    # where every new token lies, for the plain form: its sequence and its place there
    s["seq"] = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV))
    s["place"] = torch.arange(tokens, device=DEV) - s["start"].long()[s["seq"]]
    if c["kind"] == "append":
        fused = torch.cat([_activations(gen, tokens, heads, c["width"]) for _ in range(2)], 1).to(torch.bfloat16)
        s["k"], s["v"] = fused[:, :heads], fused[:, heads:]
    else:
        q = _activations(gen, tokens, c["q_heads"], c["width"])
        s["q"] = (q / q.square().mean(-1, keepdim=True).sqrt() * 1.5).to(torch.bfloat16)
        parents = torch.rand(tokens, generator=torch.Generator().manual_seed(seed * 31 + 7)).tolist()
        masks = []
        for n in counts:          # every node hangs on one of the nodes shortly before it; the first is the root
            masks += _ancestors([-1 if i == 0 else max(0, i - 1 - int(parents[len(masks) + i] * 4)) for i in range(n)])
        s["mask"] = torch.tensor(masks, dtype=torch.int64, device=DEV)
        s["context"] = max(a + n for a, n in zip(committed, counts))
    if own:          # the handle that a program keeps for its cache
        from paper_2605_10793_amd import attention as A
        s["cache"] = A.KVCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], bits=c["bits"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _angles(s):
    """cos and sin of every token's pairs, [tokens, 1, pairs]; whole turns fall away before the angle is rounded to 32 bits."""
    t = s["positions"].double()[:, None] * s["turns"]
    a = (t - torch.floor(t)).float() * (2 * math.pi)
    return torch.cos(a)[:, None], torch.sin(a)[:, None]


def _rotated(s, x, transposed=False):
    """32-bit rows rotated by their positions."""
    c = s["case"]
    part, half = c["part"], c["part"] // 2
    cos, sin = _angles(s)
    if transposed:
        sin = -sin
    a, b = (x[..., 0:part:2], x[..., 1:part:2]) if c["layout"] == "interleaved" else (x[..., :half], x[..., half:part])
    m = s["magnitude"]
    u, v = (a * cos - b * sin) * m, (b * cos + a * sin) * m
    y = torch.stack([u, v], -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat([u, v], -1)
    return torch.cat([y, x[..., part:]], -1)


def _plain_rotary(s):
    dt = _dtype(s["case"])
    return [_rotated(s, s[x].float(), s["case"]["transposed"]).to(dt) for x in ("q", "k")]


def _plain_norm(s):
    c = s["case"]
    dt = _dtype(c)
    out, weights = [], []
    for x in ("q", "k"):
        v, w = s[x].float(), s[x + "_weight"].float()
        rstd = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
        unit = v * rstd
        if not c["backward"]:
            out.append(_rotated(s, unit * w).to(dt))
            continue
        g = _rotated(s, s[x + "_grad"].float(), True)
        weights.append((g * unit).sum((0, 1)))
        g = g * w
        out.append((rstd * (g - unit * (g * unit).mean(-1, keepdim=True))).to(dt))
    return out + weights


def _plain_append(s):
    c = s["case"]
    at = s["prefix"].long()[s["seq"]] + s["place"]
    page, slot = s["table"][s["seq"], at // c["page"]].long(), at % c["page"]
    if c["bits"] == 16:
        s["k_pool"][page, :, slot] = s["k"]
        s["v_pool"][page, :, :, slot] = s["v"]
        return [s["k_pool"], s["v_pool"]]
    out = []
    for x in ("k", "v"):
        code, step, offset = _quantise(s[x].float(), c["bits"])
        if x == "k":
            s["k_pool"][page, :, slot] = _packed(code, c["bits"])
        else:
            s["v_pool"][page, :, :, slot] = _packed(code, c["bits"])
        s[x + "_scale"][page, :, slot] = torch.cat([step, offset], -1)
        out.append((step * code + offset).to(torch.bfloat16))
    return out + [s["k_scale"], s["v_scale"]]


def _plain_values(s, which):
    """The cache's keys or values in 32 bits, [sequences, heads, tokens, width]."""
    c = s["case"]
    x = s[which + "_pool"][s["table"].long()]                              # [sequences, columns, heads, ...]
    x = x if which == "k" else x.transpose(3, 4)
    if c["bits"] == 4:
        x = torch.cat([x & 15, x >> 4], -1)
    x = x.float()
    if c["bits"] != 16:
        pair = s[which + "_scale"][s["table"].long()]
        x = x * pair[..., :1] + pair[..., 1:]
    return x.transpose(1, 2).flatten(2, 3).contiguous()


def _plain_tree(s):
    c = s["case"]
    batch, nodes, group = c["batch"], c["nodes"], c["q_heads"] // c["k_heads"]
    q = s["q"].float().view(batch, nodes, c["k_heads"], group, c["width"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    k, v = _plain_values(s, "k"), _plain_values(s, "v")
    p = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()) / math.sqrt(c["width"])
    j = torch.arange(k.shape[2], device=DEV) - s["prefix"][:, None]        # a drafted token's number, negative for committed ones
    bit = s["mask"].view(batch, nodes, 1) >> j.clamp(0, 63)[:, None] & 1
    seen = (j < 0)[:, None] | (j < nodes)[:, None] & (bit == 1)            # [sequences, nodes, tokens]
    p = p.view(batch, c["k_heads"], nodes, group, -1).masked_fill(~seen[:, None, :, None], -math.inf).flatten(2, 3)
    p = torch.exp(p - p.amax(-1, keepdim=True))                            # every node sees itself
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return o.view(batch, c["k_heads"], nodes, group, c["width"]).permute(0, 2, 1, 3, 4).reshape(-1, c["q_heads"], c["width"]).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the library's calls

def _own_rotary(A, s):
    return A.rotary(s["plan"], s["q"], s["positions"], k=s["k"], transposed=s["case"]["transposed"])


def _own_norm(A, s):
    if s["case"]["backward"]:
        return A.qk_norm_rotary_backward(s["plan"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"], s["q_grad"], s["k_grad"], EPS)
    return A.qk_norm_rotary(s["plan"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"], EPS)


def _own_append(A, s):
    c = s["case"]
    held = A.append(s["cache"], s["k"], s["v"], s["start"], s["prefix"], s["table"], values=c["bits"] != 16)
    return [s["k_pool"], s["v_pool"]] if c["bits"] == 16 else [*held, s["k_scale"], s["v_scale"]]


def _own_tree(A, s):
    return A.tree_attention(s["q"], s["cache"], s["start"], s["prefix"], s["table"], mask=s["mask"], max_query=s["case"]["nodes"],
                            max_context=s["context"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2605_10793_amd import attention as A
        out = {"rotary": _own_rotary, "norm": _own_norm, "append": _own_append, "tree": _own_tree}[kind](A, state)
    else:
        out = {"rotary": _plain_rotary, "norm": _plain_norm, "append": _plain_append, "tree": _plain_tree}[kind](state)
    return list(out) if isinstance(out, (list, tuple)) else [out]


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_turn(c, positions):
    """e^(i p f) of every token and pair as complex128, from the definitions, and the factor."""
    factor, low, high, context = _scaling(c["scaling"])
    part, freq, magnitude = c["part"], [], 1.0
    for j in range(part // 2):
        theta = THETA * factor ** (part / max(1, part - 2)) if c["scaling"] == "base" else THETA
        f = theta ** (-2.0 * j / part)
        if c["scaling"] == "linear":
            f /= factor
        elif c["scaling"] == "bands":
            wave = 2 * math.pi / f
            if wave > context / low:
                f /= factor
            elif wave >= context / high:
                keep = (context / wave - low) / (high - low)
                f = (1 - keep) * f / factor + keep * f
        elif c["scaling"] == "ramp":
            dim = lambda turns: part * math.log(context / (turns * 2 * math.pi)) / (2 * math.log(THETA))  # noqa: E731
            a, b = max(math.floor(dim(high)), 0), min(math.ceil(dim(low)), part - 1)
            away = min(1.0, max(0.0, (j - a) / max(b - a, 1e-3)))
            f = f / factor * away + f * (1 - away)
            magnitude = 0.1 * math.log(factor) + 1
        freq.append(f)
    angle = positions.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    return torch.polar(torch.ones_like(angle), angle)[:, None], magnitude


def _exact_rotate(c, x, turn, magnitude):
    part = c["part"]
    y = x.clone()
    if c["layout"] == "interleaved":
        z = torch.complex(x[..., 0:part:2], x[..., 1:part:2]) * turn * magnitude
        y[..., 0:part:2], y[..., 1:part:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :part // 2], x[..., part // 2:part]) * turn * magnitude
        y[..., :part // 2], y[..., part // 2:part] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] in ("rotary", "norm"):
        turn, magnitude = _exact_turn(c, s["positions"])
        out, weights = [], []
        for x in ("q", "k"):
            v = s[x].double()
            if c["kind"] == "rotary":
                out.append(_exact_rotate(c, v, turn.conj() if c["transposed"] else turn, magnitude))
                continue
            w = s[x + "_weight"].double()
            norm = torch.sqrt((v * v).sum(-1, keepdim=True) / c["width"] + EPS)
            if not c["backward"]:
                out.append(_exact_rotate(c, v / norm * w, turn, magnitude))
                continue
            g = _exact_rotate(c, s[x + "_grad"].double(), turn.conj(), magnitude)
            weights.append((g * v / norm).flatten(0, 1).sum(0))
            g = g * w
            out.append(g / norm - v * (g * v).sum(-1, keepdim=True) / (c["width"] * norm ** 3))
        return out + weights
    page = c["page"]
    counts, committed = _counts(c), _committed(c)
    if c["kind"] == "append":
        if c["bits"] == 16:      # copies: there is nothing to be exact about
            k, v = s["k_pool"].double(), s["v_pool"].double()
        else:
            top = 2 ** c["bits"] - 1
            held, pairs = [], []
            for x in ("k", "v"):
                y = s[x].double()
                lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
                # the integers are decided in 32 bits, by definition: an entry half way between two levels goes to neither in 64
                step = ((hi - lo).float() / torch.full_like(lo.float(), top))
                zero = -torch.round(lo.float() / step)
                code = (torch.round(y.float() / step) + zero).clamp(0, top)
                held.append(step.double() * (code - zero).double())
                pairs.append(torch.cat([(hi - lo) / top, -(hi - lo) / top * zero.double()], -1))
            k, v = s["k_scale"].double(), s["v_scale"].double()
        i = 0
        for b, n in enumerate(counts):
            at = torch.arange(committed[b], committed[b] + n, device=DEV)
            for p in range(committed[b] // page, (committed[b] + n - 1) // page + 1):
                pick = (at // page == p).nonzero()[:, 0]
                own_page, slots = int(s["table"][b, p]), at[pick] % page
                rows = i + pick
                if c["bits"] == 16:
                    k[own_page][:, slots] = s["k"][rows].double().transpose(0, 1)
                    v[own_page][:, :, slots] = s["v"][rows].double().permute(1, 2, 0)
                else:
                    k[own_page][:, slots] = pairs[0][rows].transpose(0, 1)
                    v[own_page][:, slots] = pairs[1][rows].transpose(0, 1)
            i += n
        return [k, v] if c["bits"] == 16 else [*held, k, v]
    group, out, i = c["q_heads"] // c["k_heads"], [], 0
    masks = s["mask"].tolist()
    for b, n in enumerate(counts):
        length = committed[b] + n
        pages = s["table"][b, :(length + page - 1) // page].long()
        both = []
        for which in ("k", "v"):
            x = s[which + "_pool"][pages]
            x = x if which == "k" else x.mT
            if c["bits"] == 4:
                x = torch.stack([x % 16, x // 16], -2).flatten(-2)
            x = x.double()
            if c["bits"] != 16:
                x = x * s[which + "_scale"][pages][..., 0, None].double() + s[which + "_scale"][pages][..., 1, None].double()
            both.append(x.movedim(1, 0).flatten(1, 2)[:, :length])
        hidden = torch.tensor([[j >= committed[b] and not masks[i + r] >> (j - committed[b]) & 1 for j in range(committed[b], length)]
                               for r in range(n)], device=DEV)
        rows = torch.empty(n, c["q_heads"], c["width"], dtype=torch.float64, device=DEV)
        for h in range(c["q_heads"]):
            w = s["q"][i:i + n, h].double() @ both[0][h // group].T.contiguous() * c["width"] ** -0.5
            w[:, committed[b]:][hidden] = -math.inf
            rows[:, h] = torch.softmax(w, -1) @ both[1][h // group]
        out.append(rows)
        i += n
    return [torch.cat(out)]
