"""Measured cases of the quantised operators for serving: products with 4-bit weights, and a cache of keys and values held in
8 bits with the attention that reads it.

``run`` computes either the operators' plain form (elementary torch operations in 32 bits) or, where ``own`` is true, makes the
package's calls.  Operators:

  linear     y = relu?( x_scale * x (scale (code - zero))^T + bias ): 4-bit codes, one scale (and zero point) per row and group
             of inputs; x float16, bfloat16 or int8
  append     new keys and values are quantised into blocks of the cache, one scale per block and head; returns what the touched
             blocks hold as values, and their scales
  attention  softmax attention of every sequence's last rows over its blocks in the cache

Lengths of a batch's sequences follow from the case alone: they fall evenly from the longest to the shortest.
"""
import math

import torch

own = False

DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "int8": torch.int8}

# ---- cases ----------------------------------------------------------------------------------------------------

def _linear(rows, inputs, outputs, group, dtype, zero_points=False, bias=False, relu=False, name=None):
    case = {"op": "linear", "rows": rows, "inputs": inputs, "outputs": outputs, "group": group, "dtype": dtype,
            "zero_points": zero_points, "bias": bias, "relu": relu}
    return dict(case, name=name) if name else case


def _append(sequences, new, shortest_new, before, kv_heads, head_dim, block, dtype, name=None):
    """`sequences` sequences with shortest_new..new new tokens each, behind 0..before older ones."""
    case = {"op": "append", "sequences": sequences, "new": new, "shortest_new": shortest_new, "before": before,
            "kv_heads": kv_heads, "head_dim": head_dim, "block": block, "dtype": dtype}
    return dict(case, name=name) if name else case


def _attention(sequences, rows, shortest_rows, length, shortest, kv_heads, group, head_dim, block, dtype, causal=True, window=0,
               name=None):
    """`sequences` sequences of shortest..length tokens in the cache, the last shortest_rows..rows of which ask."""
    case = {"op": "attention", "sequences": sequences, "rows": rows, "shortest_rows": shortest_rows, "length": length,
            "shortest": shortest, "kv_heads": kv_heads, "group": group, "head_dim": head_dim, "block": block, "dtype": dtype,
            "causal": causal, "window": window}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one row through a layer of the deepest channel count: a call's fixed cost
        _linear(1, 512, 512, 64, "float16", name="linear_one_small"),
        # one token through a wide projection, zero points as calibrated weights have them: the bytes of the weights
        _linear(1, 4096, 16384, 128, "bfloat16", zero_points=True, name="linear_one_wide"),
        # sixteen requests decoded together
        _linear(16, 8192, 8192, 64, "float16", name="linear_batch"),
        # the classifier behind the VGG-16-shaped stack: its int8 maps (512 x 7 x 7) at the benchmark's batch
        _linear(16, 25088, 4096, 128, "int8", bias=True, relu=True, name="linear_classifier"),
        # a class count and channel counts that divide nothing, more rows than one tile, small groups
        _linear(53, 1000, 1001, 32, "bfloat16", zero_points=True, bias=True, name="linear_ragged"),
        # a prompt of 4096 tokens
        _linear(4096, 4096, 8192, 128, "float16", name="linear_prompt"),
        # every request of a batch stores one token: most blocks hold older tokens, some scales grow
        _append(128, 1, 1, 63, 8, 128, 64, "bfloat16", name="append_tokens"),
        # prompts of unlike lengths enter the cache
        _append(8, 2048, 700, 0, 8, 128, 32, "float16", name="append_prompts"),
        # one request just begun, as many heads of queries as of keys, the smallest blocks: a call's fixed cost
        _attention(1, 1, 1, 101, 101, 8, 1, 64, 16, "float16", name="attention_one_small"),
        # a batch decoded together at unlike lengths, four heads of queries to one of keys
        _attention(64, 1, 1, 8192, 500, 8, 4, 128, 64, "bfloat16", name="attention_batch"),
        # one request at the end of a long document
        _attention(1, 1, 1, 131071, 131071, 8, 8, 128, 64, "bfloat16", name="attention_long"),
        # prompts, one of them behind a cached beginning
        _attention(2, 4096, 2500, 6100, 2500, 8, 4, 128, 64, "bfloat16", name="attention_prompt"),
    ]


def _log_int(rng, low, high):
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    largest = [work(case) for case in listed()]
    while True:
        case = {"linear": _draw_linear, "append": _draw_append, "attention": _draw_attention}[
            rng.choice(("linear", "linear", "linear", "append", "attention", "attention"))](rng)
        cost = work(case)
        if all(cost[unit] <= max(w[unit] for w in largest) for unit in cost):
            return case


def _draw_linear(rng):
    rows = 1 if rng.random() < 0.25 else _log_int(rng, 1, 4096)
    inputs, outputs = _log_int(rng, 32, 28672), _log_int(rng, 16, 28672)
    if rng.random() < 0.75:
        inputs, outputs = -(-inputs // 128) * 128, -(-outputs // 16) * 16
    return _linear(rows, inputs, outputs, rng.choice((32, 64, 128)), rng.choice(("float16", "bfloat16", "int8")),
                   rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.25)


def _draw_cache(rng):
    return rng.choice((1, 2, 4, 5, 8, 16)), rng.choice((64, 128, 128, 256)), rng.choice((16, 32, 64, 128)), rng.choice(("float16", "bfloat16"))


def _draw_append(rng):
    kv_heads, head_dim, block, dtype = _draw_cache(rng)
    new = 1 if rng.random() < 0.5 else _log_int(rng, 1, 8192)
    return _append(_log_int(rng, 1, 128), new, rng.randint(1, new), rng.randint(0, 300), kv_heads, head_dim, block, dtype)


def _draw_attention(rng):
    kv_heads, head_dim, block, dtype = _draw_cache(rng)
    group = rng.choice((1, 2, 4, 6, 8))
    if rng.random() < 0.5:   # tokens one by one, or a few guessed ahead
        sequences, length = _log_int(rng, 1, 64), _log_int(rng, 1, 131072)
        rows = 1 if rng.random() < 0.75 else min(length, rng.randint(2, 8))
    else:
        sequences, length = _log_int(rng, 1, 8), _log_int(rng, 1, 8192)
        rows = _log_int(rng, 1, min(4096, length))
    shortest = rng.randint(1, length)
    causal = rng.random() < 0.85
    window = rng.choice((0, 0, _log_int(rng, 1, length))) if causal else 0
    return _attention(sequences, rows, min(rows, shortest, rng.randint(1, rows)), length, shortest, kv_heads, group, head_dim, block,
                      dtype, causal, window)


# ---- sizes that follow from a case ------------------------------------------------------------------------------

def _fall(most, least, count):
    return [most - (most - least) * b // max(1, count - 1) for b in range(count)]


def _lengths(case):
    """(tokens in the cache after the call, of which new or asking) per sequence."""
    n = case["sequences"]
    if case["op"] == "append":
        new = _fall(case["new"], case["shortest_new"], n)
        before = [case["before"] * ((5 * b + 2) % 7) // 6 for b in range(n)]
        return [a + b for a, b in zip(before, new)], new
    lengths = _fall(case["length"], case["shortest"], n)
    return lengths, [min(a, b) for a, b in zip(lengths, _fall(case["rows"], case["shortest_rows"], n))]


def _touched(case):
    """For each sequence, the first and the last block (of its own) that receives new tokens."""
    lengths, new = _lengths(case)
    return [((a - n) // case["block"], (a - 1) // case["block"]) for a, n in zip(lengths, new)]


def _pairs(case):
    """Visible (row, token) pairs, per head of queries."""
    total = 0
    lengths, rows = _lengths(case)
    for length, n in zip(lengths, rows):
        if not case["causal"]:
            total += n * length
            continue
        first, window = length - n, case["window"]
        if window == 0:
            total += n * (first + 1) + n * (n - 1) // 2
        else:
            total += sum(min(window, p + 1) for p in range(first, length))
    return total


def work(case):
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inputs"], case["outputs"]
        groups = -(-k // case["group"])
        x_bytes, y_bytes = (1, 4) if case["dtype"] == "int8" else (2, 2)
        weights = n * k / 2 + n * groups * (2.5 if case["zero_points"] else 2)
        extra = (4 * n if case["bias"] else 0) + (4 * m if case["dtype"] == "int8" else 0)
        return {"bytes": int(weights + m * k * x_bytes + m * n * y_bytes + extra), "flops": 2 * m * n * k}
    lengths, new = _lengths(case)
    h, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        blocks = sum(last - first + 1 for first, last in _touched(case))
        held = blocks * case["block"] * h * d
        # keys and values in, codes and scales out; then the touched blocks' codes in and their values out
        return {"bytes": 2 * (sum(new) * h * d * 3 + blocks * h * 4) + 2 * (held * 5 + blocks * h * 4), "flops": 2 * 3 * sum(new) * h * d}
    seen = 0
    for length, n in zip(lengths, new):
        seen += min(length, case["window"] + n - 1) if case["window"] else length
    scales = 2 * 4 * h * sum(-(-length // case["block"]) for length in lengths)
    heads = h * case["group"]
    return {"bytes": 2 * seen * h * d + scales + 4 * sum(new) * heads * d, "flops": 4 * d * heads * _pairs(case)}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inputs"], case["outputs"]
        groups = -(-k // case["group"])
        if case["dtype"] == "int8":
            # half zeros, else 0..127: maps behind a ReLU
            x = torch.randint(-128, 128, (m, k), dtype=torch.int16, device="cuda", generator=gen).clamp_(min=0).to(torch.int8)
            state["x_scale"] = torch.rand(m, device="cuda", generator=gen) * 0.02 + 0.01
            scale_dtype = torch.float16
        else:
            # activations have channels of larger size
            x = torch.randn(m, k, device="cuda", generator=gen)
            x = (x * torch.exp(torch.randn(k, device="cuda", generator=gen) * 0.5)).to(DTYPES[case["dtype"]])
            state["x_scale"] = None
            scale_dtype = x.dtype
        # codes of normal weights: round(2.5 normal) around the zero point
        zero = torch.randint(5, 12, (n, groups), dtype=torch.uint8, device="cuda", generator=gen) if case["zero_points"] else None
        codes = torch.randn(n, k, device="cuda", generator=gen).mul_(2.5).round_()
        centre = 8 if zero is None else zero.float().repeat_interleave(case["group"], 1)[:, :k]
        state["codes"] = codes.add_(centre).clamp_(0, 15).to(torch.uint8)
        state["scales"] = ((torch.rand(n, groups, device="cuda", generator=gen) + 0.5) / (2.5 * math.sqrt(k))).to(scale_dtype)
        state["zero"] = zero
        state["bias"] = torch.randn(n, device="cuda", generator=gen) if case["bias"] else None
        state["x"] = x
        if own:
            import paper_1901_01965_amd as wg
            state["packed"] = wg.pack_int4_weights(state["codes"], state["scales"], state["zero"], group=case["group"])
        return state

    lengths, new = _lengths(case)
    h, d, block, dtype = case["kv_heads"], case["head_dim"], case["block"], DTYPES[case["dtype"]]
    counts = [-(-length // block) for length in lengths]
    blocks = sum(counts) + 2   # two that belong to nobody
    order = torch.randperm(blocks, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(len(lengths), max(counts), dtype=torch.int32, device="cuda")
    at = 0
    for b, count in enumerate(counts):
        table[b, :count] = order[at:at + count]
        at += count
    state["k"] = torch.randint(-127, 128, (blocks, h, block, d), dtype=torch.int8, device="cuda", generator=gen)
    state["v"] = torch.randint(-127, 128, (blocks, h, d, block), dtype=torch.int8, device="cuda", generator=gen)
    state["k_scale"] = torch.rand(blocks, h, device="cuda", generator=gen) * 0.02 + 0.015
    state["v_scale"] = torch.rand(blocks, h, device="cuda", generator=gen) * 0.02 + 0.015
    state["table"] = table
    state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    # a batch of single tokens needs no starts
    state["starts"] = None if max(new) == 1 else torch.tensor(starts, dtype=torch.int32, device="cuda")
    state["host"] = (lengths, starts)
    total = starts[-1]
    if case["op"] == "append":
        # keys and values as slices of one projection's output; keys have larger channels
        both = torch.randn(total, 2, h, d, device="cuda", generator=gen)
        both[:, 0] *= torch.exp(torch.randn(h, d, device="cuda", generator=gen) * 0.5)
        both = both.to(dtype)
        state["new_k"], state["new_v"] = both[:, 0], both[:, 1]
        blocks_of = [table[b, first:last + 1] for b, (first, last) in enumerate(_touched(case))]
        state["touched"] = torch.cat(blocks_of)
    else:
        state["q"] = (torch.randn(total, h * case["group"], d, device="cuda", generator=gen) * 1.5).to(dtype)
        state["scale"] = 1.0 / math.sqrt(d)
    if own:
        import paper_1901_01965_amd as wg
        state["cache"] = wg.Int8Cache(state["k"], state["v"], state["k_scale"], state["v_scale"])
    return state


# ---- passes ---------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        import paper_1901_01965_amd as wg
        if case["op"] == "linear":
            return wg.int4_linear(state["x"], state["packed"], bias=state["bias"], relu=case["relu"], x_scale=state["x_scale"])
        if case["op"] == "append":
            cache = state["cache"]
            wg.int8_cache_append(state["new_k"], state["new_v"], cache, state["table"], state["lengths"], state["starts"])
            k, v = wg.int8_cache_read(cache, state["touched"])
            return {"k": k, "v": v, "k_scale": cache.k_scale, "v_scale": cache.v_scale}
        return wg.int8_cache_attention(state["q"], state["cache"], state["table"], state["lengths"], state["starts"],
                                       scale=state["scale"], causal=case["causal"], window=case["window"])
    return {"linear": _plain_linear, "append": _plain_append, "attention": _plain_attention}[case["op"]](state, case)


def _plain_linear(state, case):
    k, group = case["inputs"], case["group"]
    zero = 8.0 if state["zero"] is None else state["zero"].float().repeat_interleave(group, 1)[:, :k]
    weights = (state["codes"].float() - zero) * state["scales"].float().repeat_interleave(group, 1)[:, :k]
    y = state["x"].float() @ weights.t()
    if state["x_scale"] is not None:
        y = y * state["x_scale"][:, None]
    if state["bias"] is not None:
        y = y + state["bias"]
    if case["relu"]:
        y = torch.where(y > 0, y, torch.zeros_like(y))
    return y if state["x"].dtype == torch.int8 else y.to(state["x"].dtype)


def _plain_append(state, case):
    # codes next to the border between two are told apart in 64 bits
    block, lengths, table = case["block"], state["lengths"].long(), state["table"].long()
    total = state["new_k"].shape[0]
    rows = torch.arange(total, device="cuda")
    if state["starts"] is None:
        sequence, position = rows, lengths - 1
    else:
        starts = state["starts"].long()
        sequence = torch.searchsorted(starts[1:].contiguous(), rows, right=True)
        position = lengths[sequence] - starts[sequence + 1] + rows
    at, slot = table[sequence, position // block], position % block
    touched, touches = torch.unique(at, return_inverse=True)
    first = torch.full_like(touched, block).scatter_reduce(0, touches, slot, "amin")
    out = {}
    for name, new, codes, scales in (("k", state["new_k"], state["k"], state["k_scale"]), ("v", state["new_v"], state["v"], state["v_scale"])):
        new = new.double()
        held = codes[touched] if name == "k" else codes[touched].transpose(2, 3)
        old = torch.where(first[:, None] > 0, scales[touched], torch.zeros_like(scales[touched]))
        largest = torch.zeros_like(old).scatter_reduce(0, touches[:, None].expand(-1, new.shape[1]), new.abs().amax(2).float(), "amax")
        scale = torch.maximum(old, (largest.double() / 127).float()).double()
        older = (torch.arange(block, device="cuda")[None, :] < first[:, None])[:, None, :, None]
        divisor = torch.where(scale > 0, scale, torch.ones_like(scale))
        held = held.double()
        held = torch.where(older, torch.round(held * old[:, :, None, None] / divisor[:, :, None, None]), held)
        held[touches, :, slot] = torch.round(new / divisor[touches][:, :, None]).clamp(-127, 127)
        scales[touched] = scale.float()
        codes[touched] = (held if name == "k" else held.transpose(2, 3)).to(torch.int8)
        want = state["touched"].long()
        values = codes[want].float() * scales[want][:, :, None, None]
        out[name] = values if name == "k" else values.transpose(2, 3).contiguous()
    out["k_scale"], out["v_scale"] = state["k_scale"], state["v_scale"]
    return out


def _plain_attention(state, case):
    block, h, g, d = case["block"], case["kv_heads"], case["group"], case["head_dim"]
    lengths, starts = state["host"]
    q, table = state["q"], state["table"].long()
    out = torch.empty_like(q)
    for b, length in enumerate(lengths):
        n = starts[b + 1] - starts[b]
        blocks = table[b, :-(-length // block)]
        # [h, tokens, d] and, for the second product, the same
        keys = (state["k"][blocks].float() * state["k_scale"][blocks][:, :, None, None]).permute(1, 0, 2, 3).reshape(h, -1, d)[:, :length]
        values = (state["v"][blocks].float() * state["v_scale"][blocks][:, :, None, None]).permute(1, 0, 3, 2).reshape(h, -1, d)[:, :length]
        keys, values = keys.transpose(1, 2).contiguous(), values.contiguous()
        step = max(1, (1 << 27) // (h * g * length))
        for i in range(0, n, step):
            part = q[starts[b] + i:starts[b] + min(n, i + step)].float()
            rows = part.shape[0]
            part = part.reshape(rows, h, g, d).permute(1, 0, 2, 3).reshape(h, rows * g, d)
            scores = torch.bmm(part, keys) * state["scale"]
            if case["causal"]:
                position = (length - n + i + torch.arange(rows, device="cuda")).repeat_interleave(g)[:, None]
                token = torch.arange(length, device="cuda")[None, :]
                hidden = token > position
                if case["window"]:
                    hidden = hidden | (token <= position - case["window"])
                scores.masked_fill_(hidden, float("-inf"))
            weights = torch.exp(scores - scores.amax(2, keepdim=True))
            mean = torch.bmm(weights, values) / weights.sum(2, keepdim=True)
            out[starts[b] + i:starts[b] + i + rows] = mean.reshape(h, rows, g, d).permute(1, 0, 2, 3).reshape(rows, h * g, d).to(q.dtype)
    return out


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        k, n, group = case["inputs"], case["outputs"], case["group"]
        x = state["x"].double()
        y = torch.zeros(x.shape[0], n, dtype=torch.float64, device="cuda")
        for j in range(-(-k // group)):
            part = slice(j * group, min(k, (j + 1) * group))
            zero = 8.0 if state["zero"] is None else state["zero"][:, j:j + 1].double()
            y += torch.mm(x[:, part], (state["codes"][:, part].double() - zero).t().contiguous()) * state["scales"][:, j].double()
        if state["x_scale"] is not None:
            y *= state["x_scale"].double()[:, None]
        if state["bias"] is not None:
            y += state["bias"].double()
        return y.clamp(min=0) if case["relu"] else y
    if case["op"] == "append":
        return _exact_append(state, case)
    return _exact_attention(state, case)


def _exact_append(state, case):
    """Block by block, in the order the sequences bring them; the scales are 32-bit numbers by definition."""
    block = case["block"]
    lengths, starts = state["host"]
    out = {"k": [], "v": [], "k_scale": state["k_scale"].double().clone(), "v_scale": state["v_scale"].double().clone()}
    table = state["table"].tolist()
    for b, (first, last) in enumerate(_touched(case)):
        base = lengths[b] - (starts[b + 1] - starts[b])   # position of the sequence's first new token
        for i in range(first, last + 1):
            page = table[b][i]
            begin, end = max(base, i * block), min(lengths[b], (i + 1) * block)
            rows = slice(starts[b] + begin - base, starts[b] + end - base)
            lo, hi = begin - i * block, end - i * block
            for name in ("k", "v"):
                new = state["new_" + name][rows].double().transpose(0, 1)   # [h, tokens, d]
                codes = state[name][page].double()
                codes = codes if name == "k" else codes.transpose(1, 2)
                old = state[name + "_scale"][page].double() * (lo > 0)
                scale = torch.maximum(old, (new.abs().amax((1, 2)) / 127.0).float().double())
                divisor = torch.where(scale > 0, scale, torch.ones_like(scale))[:, None, None]
                codes = codes.clone()
                codes[:, :lo] = torch.round(codes[:, :lo] * old[:, None, None] / divisor)
                codes[:, lo:hi] = torch.round(new / divisor).clamp(-127, 127)
                out[name].append(codes * scale[:, None, None])
                out[name + "_scale"][page] = scale
    out["k"], out["v"] = torch.stack(out["k"]), torch.stack(out["v"])
    return out


def _exact_attention(state, case):
    block, h, g, d = case["block"], case["kv_heads"], case["group"], case["head_dim"]
    lengths, starts = state["host"]
    out = torch.empty(state["q"].shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lengths):
        n = starts[b + 1] - starts[b]
        pages = state["table"][b, :-(-length // block)].long()
        for head in range(h):
            keys = state["k"][pages, head].double() * state["k_scale"][pages, head].double()[:, None, None]
            values = state["v"][pages, head].double() * state["v_scale"][pages, head].double()[:, None, None]
            keys = keys.reshape(-1, d)[:length].t().contiguous()
            values = values.transpose(1, 2).reshape(-1, d)[:length].contiguous()
            step = max(1, (1 << 26) // length)
            for query_head in range(head * g, (head + 1) * g):
                for i in range(0, n, step):
                    rows = slice(starts[b] + i, starts[b] + min(n, i + step))
                    scores = torch.mm(state["q"][rows, query_head].double(), keys) * state["scale"]
                    position = length - n + i + torch.arange(scores.shape[0], device="cuda")[:, None]
                    token = torch.arange(length, device="cuda")[None, :]
                    if case["causal"]:
                        scores[(token > position) | ((token <= position - case["window"]) if case["window"] else (token < 0))] = -math.inf
                    out[rows, query_head] = torch.mm(torch.softmax(scores, 1), values)
    return out
