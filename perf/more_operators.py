"""Operators around the denoising step: rotary positions, and a paged cache of keys and values in 8 bits that is
written, read back and attended to by a batch of sequences which may share a prefix.

`listed()` names the fixed cases, `draw()` gives more of the same ranges, `prepare()` makes what a
program holds before the call, `run()` is one pass - through the framework's entry points where `own`
is true, in elementary torch operations where it is not - `work()` what a pass cannot do without and
`exact()` the result in 64 bits.

What one pass is, by `kind`:
  rotary     rows of heads turned by their positions
  write      keys and values of some tokens into the cache, and back: the values it holds for them then
  read       a sequence's tokens out of the cache
  attention  rows of a batch of sequences over the cache: a prefix that all of them share, and their own keys

The cache holds e4m3 codes with one power of two to a token and head (`cache` "e4m3": the least 2^e, e >= -126, that
leaves the largest magnitude at 448 or less), or bfloat16 values as they are.
"""
from __future__ import annotations

import math

import torch

own = False

PART = 2 ** 15      # tokens that prepare() writes at a time


def _rotary(name, rows, heads, head_dim=128, dim=128, dtype="bf16", interleaved=False, base=500000.0, factor=1.0, original=0,
            last=4096, pad=0, inverse=False):
    return dict(name=name, kind="rotary", rows=rows, heads=heads, head_dim=head_dim, dim=dim, dtype=dtype, interleaved=interleaved,
                base=base, factor=factor, original=original, last=last, pad=pad, inverse=inverse)


def _cache(name, kind, rows, kv_heads, head_dim=128, page=64, cache="e4m3", dtype="bf16", scattered=False, skipped=0):
    return dict(name=name, kind=kind, rows=rows, kv_heads=kv_heads, head_dim=head_dim, page=page, cache=cache, dtype=dtype,
                scattered=scattered, skipped=skipped)


def _attention(name, seqs, rows, keys, heads, kv_heads, head_dim=128, prefix=0, page=64, cache="e4m3", causal=False, ragged=False):
    return dict(name=name, kind="attention", seqs=seqs, rows=rows, keys=keys, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                prefix=prefix, page=page, cache=cache, causal=causal, ragged=ragged)


def listed():
    return [
        # the queries and keys of one token of the LLaDA-8B shape (32 + 32 heads): latency
        _rotary("rotary_one", 1, 64),
        # float32 gradients of the Dream-7B shape's 28 + 4 heads, neighbours turn, half of the head, frequencies
        # stretched for a context 16 times longer, far positions
        _rotary("rotary_far", 2001, 32, dim=64, dtype="f32", interleaved=True, base=10000.0, factor=16.0, original=8192,
                last=131072, inverse=True),
        # the first step of 16 sequences of the LLaDA-8B shape: 24576 rows, queries beside keys
        _rotary("rotary_first", 24576, 64),
        # a partial step of the LLaDA-8B shape: 34 tokens here and there in a sequence: latency
        _cache("write_step", "write", 34, 32, scattered=True),
        # the first step of 16 sequences
        _cache("write_first", "write", 24576, 32),
        # one sequence of 512 + 256 tokens, for a layer that is computed elsewhere
        _cache("read_sequence", "read", 768, 32),
        # a long context of the Dream-7B shape
        _cache("read_long", "read", 131071, 4, page=256),
        # a single row over a short context, 28 heads on 4: latency
        _attention("attention_one", 1, 1, 1000, 28, 4),
        # a partial step of 16 sequences, up to 34 rows over up to 1536 positions each
        _attention("attention_step", 16, 34, 1536, 32, 32, ragged=True),
        # 64 samples of one long prompt, a row each: the prompt is read once for all
        _attention("attention_shared", 64, 1, 511, 28, 4, prefix=16384, ragged=True),
        # a single row over a long context in bfloat16
        _attention("attention_long", 1, 1, 131071, 28, 4, page=256, cache="bf16"),
        # the first step of 16 sequences: every row over every position of its sequence
        _attention("attention_full", 16, 1536, 1536, 32, 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(32, 32, 128), (28, 4, 128), (4, 4, 64), (8, 1, 128), (16, 2, 64), (12, 4, 128), (64, 8, 128)]


def draw(rng):
    what = rng.random()
    if what < 0.25:
        heads, kv_heads, head_dim = rng.choice(HEADS)
        factor = rng.choice([1.0, 1.0, 8.0, round(rng.uniform(1.5, 40.0), 2)])
        c = _rotary("", _log_int(rng, 1, 24576), heads + kv_heads, head_dim, rng.choice([head_dim, head_dim // 2, head_dim // 4 + 6]),
                    rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.4, rng.choice([10000.0, 500000.0, 1000000.0]), factor,
                    rng.choice([0, 8192]) if factor > 1 else 0, _log_int(rng, 64, 1000000), rng.choice([0, 0, 8, 3]), rng.random() < 0.3)
        c["rows"] = max(1, min(c["rows"], 24576 * 64 * 128 * 2 // (c["heads"] * head_dim * (4 if c["dtype"] == "f32" else 2))))
    elif what < 0.55:
        _, kv_heads, head_dim = rng.choice(HEADS)
        kind = rng.choice(["write", "write", "read"])
        rows = min(_log_int(rng, 1, 131072 if kind == "read" else 24576), 24576 * 32 * 128 // (kv_heads * head_dim))
        c = _cache("", kind, rows, kv_heads, head_dim, rng.choice([32, 64, 128, 256]), rng.choice(["e4m3", "e4m3", "bf16"]),
                   rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.4, rng.choice([0, 0, rng.randint(0, rows - 1)]))
    else:
        heads, kv_heads, head_dim = rng.choice(HEADS)
        seqs = _log_int(rng, 1, 64)
        rows = rng.choice([1, _log_int(rng, 1, 128), _log_int(rng, 1, 1536)])
        keys = max(1, min(_log_int(rng, 1, 131072), 24576 * 4096 // (seqs * kv_heads * head_dim)))
        prefix = rng.choice([0, _log_int(rng, 1, 32768)])
        room = 16 * 1536 * 1536 * 32 // (seqs * heads)      # rows x keys that cost no more than the largest listed case
        keys = min(keys, room)
        prefix = min(prefix, room - keys)
        c = _attention("", seqs, max(1, min(rows, room // (keys + prefix))), keys, heads, kv_heads, head_dim, prefix,
                       rng.choice([32, 64, 128, 256]), rng.choice(["e4m3", "e4m3", "bf16"]), rng.random() < 0.4, rng.random() < 0.5)
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
LOW, HIGH = 1.0, 32.0      # turns over the original length below which a frequency is stretched, and above which it is not


def _frequencies(case):
    """radians a position, of each pair: float64"""
    i = torch.arange(case["dim"] // 2, dtype=torch.float64)
    theta = case["base"] ** (-2.0 * i / case["dim"])
    if case["original"]:
        part = ((case["original"] * theta / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
    else:
        part = torch.zeros_like(theta)
    return theta * (part + (1 - part) / case["factor"])


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["original"] else 1.0


def _values(gen, shape):
    """keys or values: channels of different size, a few of them large, as models have them"""
    size = torch.exp(0.7 * torch.randn(shape[1:], device="cuda", generator=gen))
    return torch.randn(shape, device="cuda", generator=gen) * size


def _order(gen, n):
    return torch.randperm(n, device="cuda", generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case)
    if case["kind"] == "rotary":
        rows, heads, head_dim = case["rows"], case["heads"], case["head_dim"]
        # (the rows of a matrix of queries, keys and more beside them)
        x = torch.randn((rows, heads * head_dim + case["pad"]), device="cuda", generator=gen).to(DTYPES[case["dtype"]])
        state["x"] = x[:, :heads * head_dim].unflatten(1, (heads, head_dim))
        state["positions"] = torch.randint(0, case["last"], (rows,), device="cuda", generator=gen, dtype=torch.int32)
        state["theta"] = _frequencies(case).cuda()
        state["amplitude"] = _amplitude(case)
        if own:
            import paper_2603_18489_amd as ec
            state["plan"] = ec.rotary_plan(case["dim"], case["base"], case["interleaved"], case["factor"], case["original"], LOW, HIGH,
                                           state["amplitude"], device="cuda")
        return state
    kv_heads, head_dim, page = case["kv_heads"], case["head_dim"], case["page"]
    if case["kind"] in ("write", "read"):
        rows = case["rows"]
        pages = -(-(2 * rows if case["scattered"] else rows) // page) + 1
        table = _order(gen, pages)
        at = torch.arange(rows, device="cuda")
        if case["scattered"]:
            at = _order(gen, 2 * rows)[:rows].sort().values
        slots = table[at // page] * page + at % page
        if case["skipped"]:
            slots[rows - case["skipped"]:] = -1
        state["slots"] = slots.int()
    else:
        seqs, n, keys, prefix = case["seqs"], case["rows"], case["keys"], case["prefix"]
        width, shared = -(-keys // page), -(-prefix // page)
        pages = seqs * width + shared
        order = _order(gen, pages).int()
        state["table"] = order[shared:].reshape(seqs, width)
        state["prefix_table"] = order[:shared]
        least = (keys + 1) // 2 if case["ragged"] else keys
        state["lengths"] = torch.randint(least, keys + 1, (seqs,), device="cuda", generator=gen, dtype=torch.int32)
        # (rows from all to half of them, the same for every seed: the result's shape goes by them)
        count = n - 5 * torch.arange(seqs, device="cuda") % (n // 2 + 1) if case["ragged"] else torch.full((seqs,), n, device="cuda")
        starts = torch.zeros(seqs + 1, device="cuda", dtype=torch.int32)
        starts[1:] = count.cumsum(0)
        state["starts"] = starts
        q = torch.randn((int(starts[-1]), case["heads"], head_dim), device="cuda", generator=gen)
        # (queries of different sharpness, which look at many keys or at few)
        state["q"] = (q * torch.exp(0.5 * torch.randn(q.shape[:2] + (1,), device="cuda", generator=gen))).bfloat16()
    k, v = (_values(gen, ((pages * page if case["kind"] != "write" else rows), kv_heads, head_dim)) for _ in range(2))
    if case["kind"] == "write":
        state["k"], state["v"] = (t.to(DTYPES[case["dtype"]]) for t in (k, v))
    else:
        k *= 0.5
        state["k"], state["v"] = ((_quantize(t) if case["cache"] == "e4m3" else (t.bfloat16(), None)) for t in (k, v))
    if own:
        import paper_2603_18489_amd as ec
        state["cache"] = ec.kv_cache(pages, kv_heads, head_dim, page, DTYPES[case["cache"]], device="cuda")
        if case["kind"] != "write":
            every = torch.arange(pages * page, device="cuda", dtype=torch.int32)
            for part in every.split(PART):      # what the codes stand for is kept as it is
                ec.kv_write(state["cache"], *(_dequantize(*(t if t is None else t[part] for t in state[w])) for w in "kv"), part)
    return state


# ---- plain forms -------------------------------------------------------------------------------
def _quantize(x):
    """codes like x, and the powers of two (int32) of its rows; NaN where a row is not finite"""
    x = x.float()
    amax = x.abs().amax(dim=-1, keepdim=True)
    part, exponent = torch.frexp(amax)                        # amax = part 2^exponent, part in [0.5, 1)
    e = torch.where(part > 0.875, exponent - 8, exponent - 9).clamp(min=-126)
    e = torch.where(amax == 0, -126, e)
    code = torch.ldexp(x.double(), -e).float()                # (a power of two: exact, 448 at most)
    bad = ~torch.isfinite(amax)
    return torch.where(bad, math.nan, code).to(torch.float8_e4m3fn), torch.where(bad, 0, e)


def _dequantize(code, e):
    return code.float() if e is None else torch.ldexp(code.float(), e)


def _turn(x, positions, theta, dim, interleaved, amplitude, inverse):
    angle = positions.double()[:, None, None] * theta
    cos, sin = (amplitude * torch.cos(angle)).float(), (amplitude * torch.sin(angle)).float()
    sin = -sin if inverse else sin
    y = x.float().clone()
    half = dim // 2
    first, second = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, half), slice(half, dim))
    a, b = x[..., first].float(), x[..., second].float()
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y.to(x.dtype)


def _of_slots(kv, slots):
    code, e = kv
    at = slots.long().clamp(min=0)
    v = _dequantize(code[at], None if e is None else e[at])
    return torch.where((slots < 0)[:, None, None], 0.0, v)


def _attend(state):
    seqs, n, page, heads, kv_heads, hd = (state[f] for f in ("seqs", "rows", "page", "heads", "kv_heads", "head_dim"))
    group, scale = heads // kv_heads, 1 / math.sqrt(hd)
    q, starts, lengths = state["q"], state["starts"].long(), state["lengths"].long()
    inside = torch.arange(page, device=q.device)
    count = starts[1:] - starts[:-1]
    row = torch.arange(n, device=q.device)
    live = row < count[:, None]                                             # [seqs, n]
    at = torch.where(live, starts[:-1, None] + row, 0)
    # [seqs, kv heads, rows x heads of a group, head dim]
    qs = q[at].float().reshape(seqs, n, kv_heads, group, hd).permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, n * group, hd)
    scores, values = [], []
    if state["prefix"]:
        slots = (state["prefix_table"].long()[:, None] * page + inside).reshape(-1)[:state["prefix"]]
        k, v = (_of_slots(state[w], slots).transpose(0, 1) for w in "kv")   # [kv heads, keys, head dim]
        flat = qs.transpose(0, 1).reshape(kv_heads, seqs * n * group, hd)
        s = torch.matmul(flat, k.transpose(1, 2)).reshape(kv_heads, seqs, n * group, -1).transpose(0, 1)
        scores.append(s * scale)
        values.append(v)
    slots = (state["table"].long()[:, :, None] * page + inside).reshape(seqs, -1)[:, :state["keys"]]
    k, v = (_of_slots(state[w], slots.reshape(-1)).reshape(seqs, -1, kv_heads, hd).transpose(1, 2) for w in "kv")
    s = torch.matmul(qs, k.transpose(2, 3)) * scale
    limit = lengths[:, None].expand(seqs, n)
    if state["causal"]:
        limit = torch.minimum(limit, lengths[:, None] - count[:, None] + row + 1)
    key = torch.arange(s.shape[-1], device=q.device)
    hidden = key >= limit.repeat_interleave(group, dim=1)[:, None, :, None]
    scores.append(s.masked_fill_(hidden, -math.inf))
    s = torch.cat(scores, dim=-1)
    top = s.amax(dim=-1, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    first = state["prefix"]
    out = torch.matmul(p[..., first:], v)
    if first:
        flat = p[..., :first].transpose(0, 1).reshape(kv_heads, seqs * n * group, first)
        out += torch.matmul(flat, values[0]).reshape(kv_heads, seqs, n * group, hd).transpose(0, 1)
    out = torch.where(total > 0, out / total, 0.0)
    out = out.reshape(seqs, kv_heads, n, group, hd).permute(0, 2, 1, 3, 4).reshape(seqs, n, heads, hd)
    return out[live].to(torch.bfloat16)


def run(state):
    kind = state["kind"]
    if kind == "rotary":
        if own:
            import paper_2603_18489_amd as ec
            return ec.rotary(state["x"], state["positions"], state["plan"], inverse=state["inverse"])
        return _turn(*(state[f] for f in ("x", "positions", "theta", "dim", "interleaved", "amplitude", "inverse")))
    if kind == "attention":
        if own:
            import paper_2603_18489_amd as ec
            starts = dict(starts=state["starts"], max_rows=state["rows"]) if state["ragged"] else {}
            shared = dict(prefix=state["prefix_table"], prefix_len=state["prefix"]) if state["prefix"] else {}
            return ec.kv_attention(state["q"], state["cache"], state["table"], state["lengths"], max_keys=state["keys"],
                                   causal=state["causal"], **starts, **shared)
        return _attend(state)
    if own:
        import paper_2603_18489_amd as ec
        if kind == "write":
            ec.kv_write(state["cache"], state["k"], state["v"], state["slots"])
        return ec.kv_read(state["cache"], state["slots"], torch.bfloat16 if kind == "write" else DTYPES[state["dtype"]])
    slots = state["slots"]
    if kind == "read":
        return tuple(_of_slots(state[w], slots).to(DTYPES[state["dtype"]]) for w in "kv")
    values = (_dequantize(*_quantize(state[w])) if state["cache"] == "e4m3" else state[w] for w in "kv")
    return tuple(torch.where((slots < 0)[:, None, None], 0.0, t).to(torch.bfloat16) for t in values)


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"] == "rotary":
        n = case["rows"] * case["heads"] * case["head_dim"]
        # two products and a sum for each value that turns
        return {"bytes": 2 * n * size[case["dtype"]] + 4 * case["rows"], "flops": 3 * n * case["dim"] // case["head_dim"]}
    hd = case["head_dim"]
    token = 2 * case["kv_heads"] * (hd + 1 if case["cache"] == "e4m3" else 2 * hd)      # bytes of a token in the cache
    if case["kind"] in ("write", "read"):
        rows = case["rows"] - case["skipped"]
        n = 2 * case["rows"] * case["kv_heads"] * hd
        if case["kind"] == "read":
            return {"bytes": rows * token + n * size[case["dtype"]] + 4 * case["rows"], "flops": n}
        return {"bytes": n * size[case["dtype"]] + 2 * rows * token + 2 * n + 4 * case["rows"], "flops": 3 * n}
    share = 0.75 if case["ragged"] else 1.0       # (lengths and rows from a half to the whole)
    rows, keys = case["seqs"] * case["rows"] * share, case["keys"] * share
    pairs = rows * (case["prefix"] + keys)
    if case["causal"]:
        few, many = min(case["rows"] * share, keys), max(case["rows"] * share, keys)
        pairs -= rows * keys - case["seqs"] * few * (many - few / 2 if case["rows"] * share <= keys else few / 2)
    return {"bytes": (case["seqs"] * keys + case["prefix"]) * token + 2 * rows * case["heads"] * hd * 2,
            "flops": 4 * pairs * case["heads"] * hd}


# ---- results in 64 bits --------------------------------------------------------------------------
def _nearest(x):
    """float64 values -> the nearest ones on the grid of their row, by arithmetic on the grid's steps"""
    amax = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / 448))
    e = torch.where(448 * torch.exp2(e - 1) >= amax, e - 1, torch.where(448 * torch.exp2(e) < amax, e + 1, e)).clamp(min=-126)
    y = x * torch.exp2(-e)
    binade = torch.floor(torch.log2(torch.where(y == 0, 1.0, y.abs()))).clamp(min=-6)
    binade = torch.where(torch.exp2(binade) > y.abs(), binade - 1, binade).clamp(min=-6)
    step = torch.exp2(binade - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "rotary":
        x, half = state["x"].double(), case["dim"] // 2
        z = x[..., :case["dim"]]
        z = z.unflatten(-1, (half, 2)) if case["interleaved"] else torch.stack((z[..., :half], z[..., half:]), dim=-1)
        angle = state["positions"].double()[:, None] * state["theta"]
        angle = -angle if case["inverse"] else angle
        factor = torch.polar(torch.full_like(angle, state["amplitude"]), angle)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * factor[:, None])
        z = z.flatten(-2) if case["interleaved"] else torch.cat((z[..., 0], z[..., 1]), dim=-1)
        return torch.cat((z, x[..., case["dim"]:]), dim=-1)
    if case["kind"] in ("write", "read"):
        slots = state["slots"]
        gone = (slots < 0)[:, None, None]
        if case["kind"] == "write":
            both = (state[w].double() for w in "kv")
            if case["cache"] == "e4m3":
                both = (_nearest(t) for t in both)
            return tuple(torch.where(gone, 0.0, t) for t in both)
        at = torch.where(slots < 0, 0, slots).long()
        both = (state[w][0][at].double() * (1.0 if state[w][1] is None else torch.exp2(state[w][1][at].double())) for w in "kv")
        return tuple(torch.where(gone, 0.0, t) for t in both)
    page, hd, group = case["page"], case["head_dim"], case["heads"] // case["kv_heads"]
    starts, lengths = state["starts"].tolist(), state["lengths"].tolist()
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")

    def gather(table, n):
        at = torch.arange(n, device="cuda")
        at = table.long()[at // page] * page + at % page if n else at
        k, v = (state[w][0][at].double() for w in "kv")
        if case["cache"] == "e4m3":
            k, v = (t * torch.exp2(state[w][1][at].double()) for t, w in zip((k, v), "kv"))
        return k, v

    shared = gather(state["prefix_table"], case["prefix"])
    for b in range(case["seqs"]):
        mine = gather(state["table"][b], lengths[b])
        k, v = (torch.cat(t) for t in zip(shared, mine))
        rows = starts[b + 1] - starts[b]
        seen = torch.full((rows,), case["prefix"] + lengths[b], device="cuda")
        if case["causal"]:
            seen = torch.clamp(seen - rows + 1 + torch.arange(rows, device="cuda"), min=case["prefix"])
        hidden = torch.arange(len(k), device="cuda") >= seen[:, None]
        empty = (seen == 0)[:, None]
        for h in range(case["heads"]):
            s = torch.matmul(state["q"][starts[b]:starts[b + 1], h].double(), k[:, h // group].t()) / math.sqrt(hd)
            p = torch.softmax(s.masked_fill(hidden, -math.inf), dim=-1)
            out[starts[b]:starts[b + 1], h] = torch.where(empty, 0.0, torch.matmul(torch.where(empty, 0.0, p), v[:, h // group]))
    return out
