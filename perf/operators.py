"""What the performance of the 8-bit transformer operators is measured on: the calls that a program makes which keeps its weights
and its keys and values in e4m3, over the range of sizes that it makes them at.

A case is one call of one operator:

* ``quantize``  rows of activations (or 128 x 128 blocks of weights) to e4m3 with a power-of-two scale for each block of 128,
* ``dense``     act(x w^T + bias) of two e4m3 matrices with a scale for each block of 128,
* ``rotary``    rotary positions of queries and keys, both layouts, part of the head, frequencies scaled for long contexts,
* ``append``    new keys and values into the pages of an e4m3 cache with a scale for each page and head,
* ``attend``    attention of new tokens over that cache.

``run`` computes them from elementary tensor operations, or (``own``) makes the framework's calls.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
E4M3 = torch.float8_e4m3fn
E4M3_MOST = 448.0


# ---- the cases -------------------------------------------------------------------------------------------------------
def _quantize(m, k, rows, kind):
    return {"op": "quantize", "m": m, "k": k, "rows": rows, "type": kind}


def _dense(m, n, k, kind, act, bias):
    return {"op": "dense", "m": m, "n": n, "k": k, "type": kind, "act": act, "bias": bias}


def _rotary(tokens, hq, hk, d, rot, kind, interleaved, scaled, far, inverse):
    return {"op": "rotary", "tokens": tokens, "hq": hq, "hk": hk, "d": d, "rot": rot, "type": kind, "interleaved": interleaved,
            "scaled": scaled, "far": far, "inverse": inverse}


def _append(batch, count, ragged, length, hk, d, block, kind):
    return {"op": "append", "batch": batch, "count": count, "ragged": ragged, "length": length, "hk": hk, "d": d, "block": block,
            "type": kind}


def _attend(batch, count, ragged, length, hq, hk, d, block, window, kind):
    return {"op": "attend", "batch": batch, "count": count, "ragged": ragged, "length": length, "hq": hq, "hk": hk, "d": d,
            "block": block, "window": window, "type": kind}


def listed():
    named = [
        # one token's activations in front of a projection: latency is all there is
        ("quantize_token", _quantize(1, 4096, 1, "bf16")),
        # the activations of a long prompt: one pass over memory
        ("quantize_prompt", _quantize(8192, 4096, 1, "bf16")),
        # a projection of eight sequences' next tokens: the weights are read once
        ("dense_tokens", _dense(8, 4096, 4096, "bf16", "none", False)),
        # a classifier-like layer whose sizes are multiples of nothing, results in 32 bits
        ("dense_ragged", _dense(333, 1000, 1960, "f32", "gelu", True)),
        # a projection of a long prompt: the tensor cores are the bound
        ("dense_prompt", _dense(8192, 4096, 4096, "bf16", "none", True)),
        # the queries and keys of sixteen sequences' next tokens
        ("rotary_tokens", _rotary(16, 32, 8, 128, 128, "bf16", False, False, 32768, False)),
        # a long prompt far into its context, interleaved pairs in half of each head, frequencies scaled
        ("rotary_prompt", _rotary(8192, 32, 8, 128, 64, "f16", True, True, 1 << 20, False)),
        # the next tokens of 64 sequences into pages that are partly filled
        ("append_tokens", _append(64, 1, False, 4096, 8, 128, 64, "bf16")),
        # four prompts of different lengths behind what the cache holds already
        ("append_prompts", _append(4, 2048, True, 4096, 8, 128, 64, "f16")),
        # the next tokens of 64 sequences of different lengths: grouped queries, bound by reading the cache
        ("attend_tokens", _attend(64, 1, True, 8192, 32, 8, 128, 64, 0, "bf16")),
        # the next token of one long sequence: the axis of the keys is all there is to share out
        ("attend_long", _attend(1, 1, False, 131072, 32, 8, 128, 128, 0, "bf16")),
        # two prompts in their second half: the tensor cores and the exponentials are the bound
        ("attend_prompts", _attend(2, 2048, False, 4096, 32, 8, 128, 64, 0, "bf16")),
    ]
    return [dict(c, name=n) for n, c in named]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("quantize", "dense", "dense", "rotary", "append", "attend", "attend", "attend"))
    if op == "quantize":
        while True:
            m, k = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)
            if m * k <= 1 << 25:
                return _quantize(m, k, rng.choice((1, 1, 128)), rng.choice(("f32", "f16", "bf16")))
    if op == "dense":
        while True:
            m, n, k = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
            if m * n * k <= 1 << 37:
                return _dense(m, n, k, rng.choice(("f32", "f16", "bf16")), rng.choice(("none", "none", "relu", "gelu")), rng.random() < 0.5)
    if op == "rotary":
        hk = rng.choice((1, 2, 4, 8, 12))
        d = rng.choice((32, 64, 80, 96, 128, 256))
        return _rotary(_log_int(rng, 1, 4096), hk * rng.choice((1, 2, 4)), hk, d, rng.choice((d, d, d // 2)), rng.choice(("f32", "f16", "bf16")),
                       rng.random() < 0.5, rng.random() < 0.5, _log_int(rng, 4096, 1 << 20), rng.random() < 0.25)
    if op == "append":
        batch = _log_int(rng, 1, 64)
        return _append(batch, rng.choice((1, 1, _log_int(rng, 2, max(2, 4096 // batch)))), rng.random() < 0.5, _log_int(rng, 64, 4096),
                       rng.choice((1, 2, 4, 8)), rng.choice((32, 64, 96, 128, 256)), rng.choice((16, 32, 64, 128)), rng.choice(("f16", "bf16", "f32")))
    while True:
        batch, hk = _log_int(rng, 1, 64), rng.choice((1, 2, 4, 8, 12))
        hq, d = hk * rng.choice((1, 2, 4, 7, 8)), rng.choice((32, 64, 64, 96, 128, 128, 128, 256))
        count = rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 16, 2048)))
        length = _log_int(rng, max(16, count), 65536)
        if batch * length * hk * d <= 1 << 27 and batch * count * length * hq * d <= 1 << 35:
            return _attend(batch, count, rng.random() < 0.5, length, hq, hk, d, rng.choice((16, 32, 64, 128)), rng.choice((0, 0, 0, _log_int(rng, 16, 4096))),
                           rng.choice(("f16", "bf16", "bf16")))


# ---- sizes of a ragged batch: they go by the case alone, so that its work does ----------------------------------------
def _sizes(case):
    """(new tokens, tokens in the cache with them) of each sequence."""
    if not case["ragged"]:
        return [(case["count"], max(case["length"], case["count"]))] * case["batch"]
    rng = random.Random("%d %d %d" % (case["batch"], case["count"], case["length"]))
    counts = [case["count"] if i == 0 or case["count"] == 1 else rng.randint(1, case["count"]) for i in range(case["batch"])]
    return [(c, max(c, case["length"] if i == 0 else rng.randint(1, case["length"]))) for i, c in enumerate(counts)]


def _pairs(count, length, window):
    """Keys that the queries of one sequence see, all in all."""
    first = length - count
    return sum(min(first + i + 1, window) for i in range(count)) if window else count * first + count * (count + 1) // 2


def _keys(count, length, window):
    """Keys of one sequence that any of its queries sees."""
    return min(length, count - 1 + window) if window else length


def work(case):
    op = case["op"]
    if op == "quantize":
        m, k = case["m"], case["k"]
        kb, mb = -(-k // 128), -(-m // case["rows"])
        return {"bytes": m * k * (BYTES[case["type"]] + 1) + 4 * kb * mb, "flops": 2 * m * k}
    if op == "dense":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // 128)
        return {"bytes": (m + n) * k + 4 * kb * (m + -(-n // 128)) + m * n * BYTES[case["type"]] + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    if op == "rotary":
        heads = case["hq"] + case["hk"]
        return {"bytes": 2 * case["tokens"] * heads * case["d"] * BYTES[case["type"]] + 4 * case["tokens"] + 4 * case["rot"],
                "flops": 3 * case["tokens"] * heads * case["rot"]}
    sizes = _sizes(case)
    tokens = sum(c for c, _ in sizes)
    hk, d = case["hk"], case["d"]
    if op == "append":
        pages = sum((n - 1) // case["block"] - (n - c) // case["block"] + 1 for c, n in sizes)
        return {"bytes": 2 * tokens * hk * d * (BYTES[case["type"]] + 1) + 2 * 2 * 4 * pages * hk + 4 * pages + 8 * len(sizes), "flops": 4 * tokens * hk * d}
    keys = sum(_keys(c, n, case["window"]) for c, n in sizes)
    pairs = sum(_pairs(c, n, case["window"]) for c, n in sizes)
    pages = sum(-(-_keys(c, n, case["window"]) // case["block"]) for c, n in sizes)
    return {"bytes": 2 * keys * hk * d + pages * (8 * hk + 4) + 2 * tokens * case["hq"] * d * BYTES[case["type"]] + 8 * len(sizes),
            "flops": 4 * pairs * case["hq"] * d}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _normal(gen, *shape):
    """Activations as they are: normal, with channels (the last axis) of different spread."""
    x = torch.randn(*shape, generator=gen, device=gen.device)
    return x * torch.exp(0.7 * torch.randn(shape[-1], generator=gen, device=gen.device))


def _power_scale(most):
    """The smallest power of two s, 2^-126 at least, with most <= 448 s (448 = 1.75 * 2^8)."""
    f, e = torch.frexp(most)
    e = torch.where(most > 0, (e - 9 + (f > 0.875).to(e.dtype)).clamp(min=-126), torch.full_like(e, -126))
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pitched(rows, cols, device):
    """An e4m3 matrix whose rows start on 16-byte boundaries, zeros to begin with."""
    return torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=device).view(E4M3)[:, :cols]


def _frequencies(rot, scaled):
    """Angles per position of the pairs, in 64 bits: 10000^(-2i/rot); scaled: slow ones divided by 8, the middle blended."""
    f = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaled:
        turns = 8192 * f / (2 * math.pi)                  # over the context of the training
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = f * keep + f / 8 * (1 - keep)
    return f


def _prepare_cache(case, gen):
    """Pages in the order that a long-running program leaves them in, filled, and the sizes of the batch."""
    dev, sizes = gen.device, _sizes(case)
    block, hk, d = case["block"], case["hk"], case["d"]
    need = [-(-n // block) for _, n in sizes]
    pages, most = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros(len(sizes), most, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s = {"table": table, "starts": torch.tensor([0] + [c for c, _ in sizes], device=dev).cumsum(0).to(torch.int32),
         "lengths": torch.tensor([n for _, n in sizes], dtype=torch.int32, device=dev), "most_new": max(c for c, _ in sizes)}
    for name in ("k", "v"):
        x = _normal(gen, pages, hk, block, d)
        scale = _power_scale(x.abs().amax(dim=(2, 3)))
        s[name + "_cache"] = (x / scale[:, :, None, None]).to(E4M3)
        s[name + "_scale"] = scale
        del x
    return s, sum(c for c, _ in sizes)


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    op, kind = case["op"], TYPES[case["type"]]
    s = {"case": case}
    if op == "quantize":
        s["x"] = _normal(gen, case["m"], case["k"]).to(kind)
        s["q"] = _pitched(case["m"], case["k"], dev)
        s["scales"] = torch.empty(-(-case["k"] // 128), -(-case["m"] // case["rows"]), device=dev)
    elif op == "dense":
        m, n, k = case["m"], case["n"], case["k"]
        s["x"], s["w"] = _pitched(m, k, dev), _pitched(n, k, dev)
        # the operands of a layer: what the quantisation of its activations and weights gives
        q, xs = _plain_quantize(_normal(gen, m, k), 1)
        s["x"].view(torch.uint8).copy_(q.view(torch.uint8))
        s["x_scale"] = xs
        q, ws = _plain_quantize(torch.randn(n, k, generator=gen, device=dev) / math.sqrt(k), 128)
        s["w"].view(torch.uint8).copy_(q.view(torch.uint8))
        s["w_scale"] = ws.t().contiguous() * (0.5 + torch.rand(ws.shape[1], ws.shape[0], generator=gen, device=dev))
        s["bias"] = torch.randn(n, generator=gen, device=dev) if case["bias"] else None
        s["y"] = torch.empty(m, n, dtype=kind, device=dev)
    elif op == "rotary":
        t, d = case["tokens"], case["d"]
        s["x"] = [_normal(gen, t, h, d).to(kind) for h in (case["hq"], case["hk"])]
        s["y"] = [torch.empty_like(x) for x in s["x"]]
        s["positions"] = torch.randint(0, case["far"], (t,), generator=gen, device=dev, dtype=torch.int32)
        s["frequencies"] = _frequencies(case["rot"], case["scaled"]).to(dev)
        s["factor"] = 0.1 * math.log(8.0) + 1.0 if case["scaled"] else 1.0
    else:
        more, tokens = _prepare_cache(case, gen)
        s.update(more)
        if op == "append":
            s["k"], s["v"] = (_normal(gen, tokens, case["hk"], case["d"]).to(kind) for _ in range(2))
        else:
            s["q"] = _normal(gen, tokens, case["hq"], case["d"]).to(kind)
            s["out"] = torch.empty_like(s["q"])
            s["scale"] = 1.0 / math.sqrt(case["d"])
    if own:
        s["call"] = _own_call(case, s)
    return s


def _own_call(case, s):
    """The handle that a program keeps: checked arguments of the call, and its workspace where it has one."""
    from paper_2201_05587_b200 import binding as B
    op = case["op"]
    if op == "quantize":
        return B.quantize(s["x"], s["q"], s["scales"], block_rows=case["rows"])
    if op == "dense":
        act = {"none": B.TT_ACT_NONE, "relu": B.TT_ACT_RELU, "gelu": B.TT_ACT_GELU_ERF}[case["act"]]
        return B.dense_quantized(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"], act=act)
    if op == "rotary":
        table = B.rotary_table(s["frequencies"])
        return B.rotary(s["x"], s["positions"], table, s["y"], interleaved=case["interleaved"], factor=s["factor"], inverse=case["inverse"])
    cache = B.Cache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"])
    if op == "append":
        return B.cache_append(cache, s["k"], s["v"], s["starts"], s["lengths"])
    return B.cache_attention(cache, s["q"], s["out"], s["starts"], s["lengths"], scale=s["scale"], window=case["window"], max_count=s["most_new"])


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        s["call"].run()
        if op == "quantize":
            return {"q": s["q"], "scales": s["scales"]}
        if op == "dense":
            return s["y"]
        if op == "rotary":
            return s["y"]
        if op == "append":
            return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}
        return s["out"]
    if op == "quantize":
        q, scales = _plain_quantize(s["x"], s["case"]["rows"])
        return {"q": q, "scales": scales}
    return {"dense": _plain_dense, "rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend}[op](s)


def _plain_quantize(x, rows):
    """e4m3 values [m, k] and scales [ceil(k / 128), ceil(m / rows)]."""
    m, k = x.shape
    kb, mb = -(-k // 128), -(-m // rows)
    x = torch.nn.functional.pad(x.float(), (0, kb * 128 - k, 0, mb * rows - m)).view(mb, rows, kb, 128)
    scale = _power_scale(torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=(1, 3)))
    q = (x / scale[:, None, :, None]).to(E4M3)
    return q.view(mb * rows, kb * 128)[:m, :k], scale.t().contiguous()


def _spread(scale, times, dim, size):
    return scale.repeat_interleave(times, dim=dim).narrow(dim, 0, size)


def _plain_act(y, act):
    if act == "relu":
        return torch.clamp(y, min=0)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain_dense(s):
    c = s["case"]
    x = s["x"].float() * _spread(s["x_scale"], 128, 0, c["k"]).t()
    w = s["w"].float() * _spread(_spread(s["w_scale"], 128, 0, c["n"]), 128, 1, c["k"])
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return _plain_act(y, c["act"]).to(TYPES[c["type"]])


def _plain_rotary(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["frequencies"][None, :]          # far positions: 32 bits lose the angle
    cos, sin = (torch.cos(angle) * s["factor"]).float()[:, None, :], (torch.sin(angle) * s["factor"]).float()[:, None, :]
    if c["inverse"]:
        sin = -sin

    def turned(x):
        v, rot = x.float(), c["rot"]
        a, b = (v[..., 0:rot:2], v[..., 1:rot:2]) if c["interleaved"] else (v[..., :rot // 2], v[..., rot // 2:rot])
        pair = (a * cos - b * sin, b * cos + a * sin)
        pair = torch.stack(pair, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(pair, dim=-1)
        return torch.cat((pair, v[..., rot:]), dim=-1).to(x.dtype)

    q, k = s["x"]
    return [turned(q), turned(k)]


def _places(s, block):
    """Of each new token: its sequence, its position, the page and the slot that it goes to."""
    starts, lengths = s["starts"].long(), s["lengths"].long()
    counts = starts[1:] - starts[:-1]
    total = s["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(counts.numel(), device=starts.device), counts, output_size=total)
    pos = lengths[seq] - counts[seq] + torch.arange(total, device=starts.device) - starts[seq]
    return counts, seq, pos, s["table"].long()[seq, pos // block], pos % block


def _plain_append(s):
    block = s["case"]["block"]
    counts, seq, pos, page, slot = _places(s, block)
    first = s["lengths"].long() - counts                                          # position of each sequence's first new token
    last = s["lengths"].long() - 1
    # the pages that receive tokens; a sequence that touches fewer names its last one again
    most = (s["most_new"] + block - 2) // block + 1
    index = torch.minimum((first // block)[:, None] + torch.arange(most, device=page.device), (last // block)[:, None])
    old_slots = torch.where(index == (first // block)[:, None], (first % block)[:, None], 0).flatten()      # tokens that they hold already
    touched = torch.gather(s["table"].long(), 1, index).flatten()

    def put(cache, scale, x):
        x = x.float()
        need = torch.zeros_like(scale).index_reduce_(0, page, torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=2), "amax")
        need, old = _power_scale(need[touched]), scale[touched]
        new = torch.where((old_slots > 0)[:, None], torch.maximum(old, need), need)
        held = cache.view(torch.uint8)[touched]
        again = (held.view(E4M3).float() * (old / new)[:, :, None, None]).to(E4M3).view(torch.uint8)
        mine = torch.arange(block, device=page.device)[None, :] < old_slots[:, None]
        cache.view(torch.uint8)[touched] = torch.where(mine[:, None, :, None], again, held)
        scale[touched] = new
        cache.view(torch.uint8)[page, :, slot] = (x / scale[page][:, :, None]).to(E4M3).view(torch.uint8)

    put(s["k_cache"], s["k_scale"], s["k"])
    put(s["v_cache"], s["v_scale"], s["v"])
    return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _plain_attend(s):
    c = s["case"]
    block, hk, d = c["block"], c["hk"], c["d"]
    table, starts, lengths = s["table"].long(), s["starts"].long(), s["lengths"].long()
    batch, group, most = table.shape[0], c["hq"] // hk, s["most_new"]
    counts = starts[1:] - starts[:-1]

    def keys(cache, scale):
        x = cache.view(torch.uint8)[table].view(E4M3).float() * scale[table][..., None, None]     # [batch, pages, heads, block, d]
        return x.transpose(1, 2).reshape(batch, hk, -1, d)

    k = keys(s["k_cache"], s["k_scale"])
    at = torch.arange(k.shape[2], device=k.device)
    held = at[None, :] < lengths[:, None]
    row = torch.arange(most, device=k.device)
    token = (starts[:-1, None] + row[None, :]).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][token].float().view(batch, most, hk, group, d).permute(0, 2, 1, 3, 4).reshape(batch, hk, most * group, d)
    pos = (lengths - counts)[:, None] + row[None, :]
    seen = held[:, None, :] & (at[None, None, :] <= pos[:, :, None])
    if c["window"]:
        seen = seen & (at[None, None, :] > pos[:, :, None] - c["window"])
    seen = seen.repeat_interleave(group, dim=1)[:, None]                                          # [batch, 1, rows, keys]
    scores = torch.where(seen, (q @ k.transpose(2, 3)) * s["scale"], float("-inf"))
    del k
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isfinite(top), top, 0.0))
    del scores
    v = torch.where(held[:, None, :, None], keys(s["v_cache"], s["v_scale"]), 0.0)
    total = p.sum(dim=-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, 1.0)
    o = o.view(batch, hk, most, group, d).permute(0, 2, 1, 3, 4).reshape(batch, most, c["hq"], d)
    mine = row[None, :] < counts[:, None]
    out = torch.empty_like(s["q"])
    out[token[mine]] = o[mine].to(out.dtype)
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def _powers(e):
    """2^e in 64 bits, to the bit."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_scale(most):
    """2^ceil(log2(most / 448)) of each, found by comparing with the powers themselves."""
    powers = _powers(torch.arange(-126, 128, device=most.device))
    return powers[torch.searchsorted(powers * E4M3_MOST, most.double().contiguous()).clamp(max=253)]


def _exact_e4m3(v):
    """The nearest value with four significant bits and no bit below 2^-9 (ties to even), |v| <= 448."""
    _, e = torch.frexp(v)
    step = _powers((e - 4).clamp(min=-9))
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x, rows = s["x"].double(), case["rows"]
        m, k = x.shape
        scales = torch.stack([torch.stack([x[i:i + rows, j:j + 128].abs().amax() for i in range(0, m, rows)]) for j in range(0, k, 128)]) \
            if rows > 1 else torch.stack([x[:, j:j + 128].abs().amax(dim=1) for j in range(0, k, 128)])
        scales = _exact_scale(scales)
        full = scales.repeat_interleave(rows, dim=1)[:, :m].repeat_interleave(128, dim=0)[:k].t()
        return {"q": _exact_e4m3(x / full), "scales": scales}
    if op == "dense":
        m, n, k = case["m"], case["n"], case["k"]
        x, w, y = s["x"].double(), s["w"].double(), torch.zeros(m, n, dtype=torch.float64, device=s["x"].device)
        for b in range(-(-k // 128)):
            at = slice(128 * b, min(k, 128 * b + 128))
            y += (x[:, at] * s["x_scale"][b].double()[:, None]) @ (w[:, at] * s["w_scale"][:, b].double().repeat_interleave(128)[:n, None]).t()
        if case["bias"]:
            y += s["bias"].double()
        return torch.relu(y) if case["act"] == "relu" else y * torch.special.ndtr(y) if case["act"] == "gelu" else y
    if op == "rotary":
        turn = torch.polar(torch.full((case["tokens"], case["rot"] // 2), s["factor"], dtype=torch.float64, device=s["positions"].device),
                           s["positions"].double()[:, None] * s["frequencies"] * (-1 if case["inverse"] else 1))[:, None, :]
        found = []
        for x in s["x"]:
            y, half = x.double().clone(), case["rot"] // 2
            a = slice(0, case["rot"], 2) if case["interleaved"] else slice(0, half)
            b = slice(1, case["rot"], 2) if case["interleaved"] else slice(half, case["rot"])
            z = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * turn
            y[..., a], y[..., b] = z.real, z.imag
            found.append(y)
        return found
    sizes, block, at = _sizes(case), case["block"], 0
    table = s["table"].cpu()
    if op == "append":
        found = {n: s[n].double() for n in ("k_cache", "v_cache", "k_scale", "v_scale")}
        for b, (count, length) in enumerate(sizes):
            for j in range((length - count) // block, (length - 1) // block + 1):
                lo, hi = max(length - count, j * block), min(length, (j + 1) * block)
                page, held = int(table[b, j]), lo - j * block
                for name in ("k", "v"):
                    x = s[name][at + lo - (length - count):at + hi - (length - count)].double().transpose(0, 1)       # [heads, tokens, d]
                    scale, old = _exact_scale(x.abs().amax(dim=(1, 2))), found[name + "_scale"][page]
                    if held:
                        scale = torch.maximum(scale, old)
                        found[name + "_cache"][page, :, :held] = _exact_e4m3(found[name + "_cache"][page, :, :held] * (old / scale)[:, None, None])
                    found[name + "_scale"][page] = scale
                    found[name + "_cache"][page, :, held:held + hi - lo] = _exact_e4m3(x / scale[:, None, None])
            at += count
        return found
    group = case["hq"] // case["hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for b, (count, length) in enumerate(sizes):
        pages = s["table"][b, :-(-length // block)].long()
        pos = torch.arange(length - count, length, device=out.device)[:, None]
        key = torch.arange(length, device=out.device)[None, :]
        hidden = (key > pos) | ((key <= pos - case["window"]) if case["window"] else (key < 0))
        for h in range(case["hk"]):
            k, v = ((s[n + "_cache"].view(torch.uint8)[pages, h].view(E4M3).double() * s[n + "_scale"][pages, h].double()[:, None, None]).reshape(-1, case["d"])[:length]
                    for n in ("k", "v"))
            for g in range(group):
                q = s["q"][at:at + count, h * group + g].double()
                out[at:at + count, h * group + g] = torch.softmax((q @ k.t() * s["scale"]).masked_fill(hidden, float("-inf")), dim=-1) @ v
        at += count
    return out
