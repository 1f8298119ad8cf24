"""Operators around the denoising step: tokens drawn from rows of logits, and matrices in microscaled
4-bit floating point (MXFP4: e2m1 codes, one power-of-two scale to 32 values of a row).

`listed()` names the fixed cases, `draw()` gives more of the same ranges, `prepare()` makes what a
program holds before the call, `run()` is one pass - through the framework's entry points where `own`
is true, in elementary torch operations where it is not - `work()` what a pass cannot do without and
`exact()` the result in 64 bits.

What one pass is, by `kind`:
  sample      logits on the device and one uniform number a row -> a token a row, its probability among
              the tokens kept and among all, how many were kept and what share of the probability they hold
  round_trip  a matrix to 4 bits and back: the values its codes and scales stand for
  linear      x W^T with W in 4 bits; x in bfloat16 (`act` "bf16"), or brought to 4 bits first ("mxfp4")
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


def _sample(name, rows, vocab, dtype="f32", pad=0, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, pad=pad,
                temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def _trip(name, rows, k, dtype="bf16", pad=0):
    return dict(name=name, kind="round_trip", rows=rows, k=k, dtype=dtype, pad=pad)


def _linear(name, m, n, k, act="bf16", out="bf16", pad=0):
    return dict(name=name, kind="linear", m=m, n=n, k=k, act=act, out=out, pad=pad)


def listed():
    return [
        # one row of a small vocabulary, all three filters: latency
        _sample("sample_one", 1, 4096, temperature=0.7, top_k=50, top_p=0.95, min_p=0.02),
        # a block of masked positions of the LLaDA-8B shape, temperature alone
        _sample("sample_block", 32, 126464, temperature=0.8),
        # the Dream-7B shape with its usual low temperature and nucleus
        _sample("sample_nucleus", 34, 152064, temperature=0.2, top_p=0.95),
        # the rows of 16 sequences at once, bfloat16 logits (many equal values), every filter
        _sample("sample_batch", 544, 126464, dtype="bf16", temperature=1.0, top_k=1000, top_p=0.9, min_p=0.001),
        # activations of a partial step: latency
        _trip("round_trip_rows", 34, 4096),
        # a gate/up matrix of the LLaDA-8B shape, as trained in float32
        _trip("round_trip_weight", 24576, 4096, dtype="f32"),
        # a single row through a small square matrix: latency
        _linear("linear_one", 1, 4096, 4096),
        # a partial step's rows through gate and up of the LLaDA-8B shape: a weight stream
        _linear("linear_block", 34, 24576, 4096),
        # the block's rows through the LM head, float32 logits
        _linear("linear_head", 32, 126464, 4096, out="f32"),
        # 16 sequences' partial rows through gate and up of the Dream-7B shape, an odd number of rows
        _linear("linear_batch", 561, 37888, 3584),
        # a full step of one sequence with activations in 4 bits too
        _linear("linear4_full", 768, 24576, 4096, act="mxfp4"),
        # the first step of 16 sequences: 24576 rows
        _linear("linear4_first", 24576, 12288, 4096, act="mxfp4"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    what = rng.random()
    if what < 0.4:
        while True:
            rows, vocab = _log_int(rng, 1, 1200), _log_int(rng, 1000, 163840)
            if rows * vocab <= 544 * 126464:
                break
        filters = dict(top_k=rng.choice([0, 0, 1, 50, _log_int(rng, 2, 5000)]),
                       top_p=rng.choice([1.0, 0.9, 0.95, round(rng.uniform(0.05, 0.99), 3)]),
                       min_p=rng.choice([0.0, 0.0, 0.05, round(rng.uniform(0.001, 0.5), 3)]))
        c = _sample("", rows, vocab, dtype=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0, 0, 1, 3, 64]),
                    temperature=rng.choice([0.2, 0.7, 1.0, round(rng.uniform(0.1, 2.0), 2)]), **filters)
    elif what < 0.55:
        c = _trip("", _log_int(rng, 1, 24576), 32 * _log_int(rng, 1, 400), dtype=rng.choice(["bf16", "f32"]),
                  pad=rng.choice([0, 0, 8, 32, 5]))
        c["rows"] = min(c["rows"], 24576 * 4096 // c["k"])
    else:
        few = rng.random() < 0.5
        m = _log_int(rng, 1, 96) if few else _log_int(rng, 97, 8192)
        k = 32 * rng.choice([_log_int(rng, 4, 400), 128, 112, 384])
        n = rng.choice([_log_int(rng, 64, 40000), 16 * _log_int(rng, 4, 8000) if few else 4096, 24576])
        c = _linear("", m, n, k, act=rng.choice(["bf16", "bf16", "mxfp4"]), out=rng.choice(["bf16", "bf16", "f32"]),
                    pad=rng.choice([0, 0, 8, 64]))
        c["n"] = max(16, min(c["n"], 24576 * 12288 * 4096 // (m * k), 126464 * 4096 // k))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(gen, rows, cols, pad, dtype):
    """rows x cols with `pad` more columns in memory, normal"""
    return torch.randn((rows, cols + pad), device="cuda", generator=gen, dtype=torch.float32).to(DTYPES[dtype])[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case)
    if case["kind"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        # From nearly decided rows to nearly flat ones: a spread of 1 to 4 over the vocabulary, and 24
        # candidates that stand out by up to 18.
        z = torch.randn((rows, vocab + case["pad"]), device="cuda", generator=gen)
        z *= 1.0 + 3.0 * torch.rand((rows, 1), device="cuda", generator=gen)
        at = torch.randint(0, vocab, (rows, 24), device="cuda", generator=gen)
        lift = torch.rand((rows, 24), device="cuda", generator=gen) * 18.0 * torch.rand((rows, 1), device="cuda", generator=gen)
        z.scatter_add_(1, at, lift)
        state["logits"] = z.to(DTYPES[case["dtype"]])[:, :vocab]
        state["uniforms"] = torch.rand((rows,), device="cuda", generator=gen)
    elif case["kind"] == "round_trip":
        # channels of different size, as weights and activations have them
        x = torch.randn((case["rows"], case["k"] + case["pad"]), device="cuda", generator=gen)
        x *= 0.02 * torch.exp(torch.randn((1, case["k"] + case["pad"]), device="cuda", generator=gen))
        state["x"] = x.to(DTYPES[case["dtype"]])[:, :case["k"]]
    else:
        state["x"] = _rows(gen, case["m"], case["k"], case["pad"], "bf16")
        w = torch.randn((case["n"], case["k"]), device="cuda", generator=gen) * 0.02
        codes, scales = _quantize(w)
        state["codes"], state["scales"] = codes, scales
        if own:   # the matrix as the products read it: laid out once, when a model is loaded
            import paper_2603_18489_amd as ec
            state["w"] = ec.mxfp4_pack(ec.Mxfp4(codes, scales))
    return state


# ---- plain forms -------------------------------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantize(x):
    """codes uint8 [rows, k/2] (even k in the low four bits), scales uint8 [rows, k/32]"""
    rows, k = x.shape
    v = x.float().reshape(rows, k // 32, 32)
    amax = v.abs().amax(dim=-1)
    exponent = (torch.frexp(amax)[1] - 3).clamp(min=-127)          # frexp's mantissa is in [0.5, 1)
    exponent = torch.where(amax == 0, -127, exponent)
    y = torch.ldexp(v.double(), -exponent.unsqueeze(-1)).float()   # a power of two: exact, in [-8, 8]
    a = y.abs()
    two = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    code = two.clamp(max=7).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    bad = ~torch.isfinite(amax)
    code = torch.where(bad.unsqueeze(-1), 0, code)
    scale = torch.where(bad, 255, exponent + 127).to(torch.uint8)
    code = code.reshape(rows, k // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), scale


def _dequantize(codes, scales):
    rows, half = codes.shape
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device, dtype=torch.float32)
    v = table[torch.stack((codes & 15, codes >> 4), dim=-1).int()].reshape(rows, half // 16, 32)
    s = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    s = torch.where(scales == 255, math.nan, s)
    return (v * s.unsqueeze(-1)).reshape(rows, 2 * half)


def _draw_tokens(z, u, temperature, top_k, top_p, min_p):
    temperature, top_p, min_p = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    if temperature == 0:
        temperature, top_k = 1.0, 1
    rows, vocab = z.shape
    z = z.float()
    ranked, ids = torch.sort(z, dim=-1, descending=True, stable=True)
    top = ranked[:, :1].double()
    e = torch.exp((ranked.double() - top) / temperature)
    keep = ranked > -math.inf
    if top_k > 0:
        keep &= torch.arange(vocab, device=z.device) < top_k
    e_k = torch.where(keep, e, 0.0)
    if top_p < 1:
        keep = keep & (torch.cumsum(e_k, dim=-1) - e_k < top_p * e_k.sum(dim=-1, keepdim=True))
    keep = keep & (e >= min_p)
    kept = torch.zeros_like(keep).scatter_(1, ids, keep)
    e = torch.exp((z.double() - top) / temperature)
    e_kept = torch.where(kept, e, 0.0)
    total = e.sum(dim=-1)
    sums = torch.cumsum(e_kept, dim=-1)
    token = (sums <= u.double().unsqueeze(-1) * sums[:, -1:]).sum(dim=-1).clamp(max=vocab - 1)
    mine = e.gather(1, token.unsqueeze(-1)).squeeze(-1)
    share = sums[:, -1]
    stats = torch.stack((mine / share, mine / total, kept.sum(dim=-1).double(), share / total), dim=-1)
    return token.to(torch.int32), stats.float()


def run(state):
    if state["kind"] == "sample":
        filters = [state[f] for f in ("temperature", "top_k", "top_p", "min_p")]
        if own:
            import paper_2603_18489_amd as ec
            return ec.row_sample(state["logits"], state["uniforms"], *filters)
        return _draw_tokens(state["logits"], state["uniforms"], *filters)
    if state["kind"] == "round_trip":
        dtype = DTYPES[state["dtype"]]
        if own:
            import paper_2603_18489_amd as ec
            return ec.mxfp4_dequantize(ec.mxfp4_quantize(state["x"]), dtype)
        return _dequantize(*_quantize(state["x"])).to(dtype)
    dtype = DTYPES[state["out"]]
    if own:
        import paper_2603_18489_amd as ec
        x = ec.mxfp4_quantize(state["x"]) if state["act"] == "mxfp4" else state["x"]
        return ec.mxfp4_linear(x, state["w"], dtype)
    x = _dequantize(*_quantize(state["x"])) if state["act"] == "mxfp4" else state["x"].float()
    return torch.matmul(x, _dequantize(state["codes"], state["scales"]).t()).to(dtype)


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        # a difference, an exponential and a sum for each logit
        return {"bytes": n * size[case["dtype"]] + case["rows"] * (4 + 4 + 16), "flops": 3 * n}
    if case["kind"] == "round_trip":
        n = case["rows"] * case["k"]
        return {"bytes": 2 * n * size[case["dtype"]], "flops": 3 * n}
    m, n, k = case["m"], case["n"], case["k"]
    return {"bytes": 2 * m * k + n * k * 17 // 32 + m * n * size[case["out"]], "flops": 2 * m * n * k}


# ---- results in 64 bits --------------------------------------------------------------------------
def _exact_values(x):
    """the values nearest to a float64 matrix on the grid of its blocks, by search among all sixteen"""
    grid = np.array(E2M1)
    middle = (grid[1:] + grid[:-1]) / 2
    blocks = np.abs(x).reshape(-1, 32)
    top = blocks.max(axis=1)
    power = np.exp2(np.maximum(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 2, -127))[:, None]
    scaled = blocks / power
    low = np.searchsorted(middle, scaled.ravel(), side="left").reshape(scaled.shape)      # a tie goes down
    tie = (scaled == middle[np.minimum(low, 6)]) & (low < 7) & (low % 2 == 1)             # unless that code is odd
    return (np.copysign(grid[low + tie] * power, x.reshape(-1, 32))).reshape(x.shape)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "sample":
        if case["rows"] * case["vocab"] > 8e7:
            return None
        z, u = state["logits"].double().cpu().numpy(), state["uniforms"].double().cpu().numpy()
        t, p, m = (float(np.float32(case[f])) for f in ("temperature", "top_p", "min_p"))
        tokens, stats = np.zeros(len(z), dtype=np.int32), np.zeros((len(z), 4))
        for r, row in enumerate(z):
            e = np.exp((row - row.max()) / t)
            order = np.argsort(-row, kind="stable")
            if case["top_k"]:
                order = order[:case["top_k"]]
            run_up = np.cumsum(e[order])
            if p < 1:
                order = order[:1 + np.searchsorted(run_up[:-1], p * run_up[-1], side="left")]
            order = np.sort(order[e[order] >= m])
            run_up = np.cumsum(e[order])
            pick = min(np.searchsorted(run_up, u[r] * run_up[-1], side="right"), len(order) - 1)
            tokens[r] = order[pick]
            stats[r] = (e[tokens[r]] / run_up[-1], e[tokens[r]] / e.sum(), len(order), run_up[-1] / e.sum())
        return tokens, stats
    if case["kind"] == "round_trip":
        if case["rows"] * case["k"] > 1.1e8:
            return None
        return _exact_values(state["x"].double().cpu().numpy())
    w = state["codes"].cpu().numpy()
    w = np.stack((w & 15, w >> 4), axis=-1).reshape(len(w), -1)
    signed = np.array(E2M1 + tuple(-v for v in E2M1), dtype=np.float32)
    w = signed[w].reshape(len(w), -1, 32) * np.exp2(state["scales"].cpu().numpy().astype(np.float32) - 127)[..., None]
    w = torch.from_numpy(w.reshape(len(w), -1)).cuda().double()      # (exact in float32)
    x = state["x"].double()
    if case["act"] == "mxfp4":
        x = torch.from_numpy(_exact_values(x.cpu().numpy())).cuda()
    return torch.matmul(x, w.t())
