"""The operators on microscaled 4-bit floating point (MXFP4) as cases that can be timed and compared.

A block of 32 neighbouring values x of a row shares a power of two s = 2^(floor(log2 max|x|) - 2); each value is held as the
E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) nearest to x / s, ties to the even mantissa, 6 where x / s is
above it.  The last block of a row may be short.  NaN counts as 0, an infinity as the largest value; neither is in max|x|.

  quantize  a tensor into codes and scales and back into the values they stand for (`q8_mx4_quantize`, `q8_mx4_dequantize`)
  fake      the same rounding in training, values in and values out (`q8_mx4_fake_quantize`); in fp32 the straight-through
            gradient of the step as well (`q8_ste_backward`)
  linear    act(x_hat w_hat^T + b): an activation quantised as it comes in, a weight quantised when the model was loaded
            (`q8_mx4_linear`)
  experts   the same with one weight matrix per expert: slot t of expert e, offsets[e] <= t < offsets[e + 1], takes row
            rows[t] of the activations (row t without `rows`) (`q8_mx4_linear_grouped`); slots that no expert owns keep what the output held

Activations are ~ N(0, 1) with one entry in a hundred multiplied by 8, weights and biases ~ N(0, 0.02), as in
paper_1910_06188_b200/synth.py.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
BLOCK = 32


def listed():
    return [
        # the input of a BERT-Large layer on 64 x 384 tokens
        dict(name="quantize_24576x1024", op="quantize", M=24576, K=1024, dtype="fp32", ld=1024),
        # one of three projections side by side, rows that end inside a block
        dict(name="quantize_odd_1777x1000", op="quantize", M=1777, K=1000, dtype="fp16", ld=3000),
        # quantisation-aware training: the widest weight of BERT-Large with its gradient, and a batch's activations
        dict(name="fake_weight_4096x1024", op="fake", M=4096, K=1024, dtype="fp32", std=0.02),
        dict(name="fake_batch_12288x4096", op="fake", M=12288, K=4096, dtype="bf16", std=1.0),
        # a served model answering one token at a time: the smallest call there is
        dict(name="linear_token_1x1024", op="linear", M=1, K=1024, N=4096, dtype="fp32", act=1, bias=True, ld=1024),
        # a batch of single tokens against a wide layer: the weights are all there is to read
        dict(name="linear_decode_24x4096", op="linear", M=24, K=4096, N=16384, dtype="bf16", act=0, bias=False, ld=4096),
        # a short ragged batch; no size is a multiple of anything
        dict(name="linear_odd_509x1000", op="linear", M=509, K=1000, N=777, dtype="fp16", act=0, bias=True, ld=1010),
        # FFN1 of BERT-Large on 64 x 384 tokens, fp32 in and out as the encoder has it
        dict(name="linear_ffn1_24576", op="linear", M=24576, K=1024, N=4096, dtype="fp32", act=1, bias=True, ld=1024),
        # a long prompt through a large square layer
        dict(name="linear_prompt_4096", op="linear", M=4096, K=8192, N=8192, dtype="bf16", act=0, bias=False, ld=8192),
        # 16 tokens, two experts each of 64: few rows an expert, many experts without any
        dict(name="experts_decode_16x2", op="experts", tokens=16, top=2, E=64, K=1024, N=2048, dtype="bf16", act=0, bias=False,
             spread=1.0, spare=0, routing=1),
        # a prompt of 8192 tokens, two experts each of 32, unevenly spread
        dict(name="experts_prompt_8192x2", op="experts", tokens=8192, top=2, E=32, K=2048, N=4096, dtype="bf16", act=0, bias=False,
             spread=0.5, spare=0, routing=2),
        # ragged everywhere, slots in the experts' order already, some behind the last expert's
        dict(name="experts_odd_1000", op="experts", tokens=1000, top=0, E=7, K=520, N=300, dtype="fp32", act=1, bias=True,
             spread=1.0, spare=37, routing=3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["quantize", "fake", "linear", "linear", "experts", "experts"])
    dtype = rng.choice(["fp32", "fp16", "bf16"])
    if op in ("quantize", "fake"):
        K = _log_int(rng, 33, 8192)
        M = _log_int(rng, 1, min(24576, 25_000_000 // K))
        if op == "fake":
            return dict(op=op, M=M, K=K, dtype=dtype, std=rng.choice([0.02, 1.0]))
        return dict(op=op, M=M, K=K, dtype=dtype, ld=K + rng.choice([0, 0, 8, 13]))
    if op == "linear":
        K, N = _log_int(rng, 33, 8192), _log_int(rng, 8, 16384)
        M = _log_int(rng, 1, max(1, min(24576, 100_000_000 // N, 100_000_000 // K, int(2.5e11) // (N * K))))
        return dict(op=op, M=M, K=K, N=N, dtype=dtype, act=rng.randint(0, 1), bias=rng.random() < 0.5, ld=K + rng.choice([0, 0, 8, 13]))
    E, K = rng.randint(1, 64), _log_int(rng, 64, 2048)
    N = _log_int(rng, 64, min(4096, 260_000_000 // (E * K)))
    top = rng.choice([0, 1, 2])
    case = dict(op=op, tokens=_log_int(rng, 1, 8192), top=top, E=E, K=K, N=N, dtype=dtype, act=rng.randint(0, 1), bias=rng.random() < 0.5,
                spread=rng.choice([0.0, 0.5, 1.0]), spare=rng.choice([0, 5, 130]) if top == 0 else 0, routing=rng.randrange(1000))
    while case["tokens"] > 1 and E * int(_counts(case).max()) * max(N, K) > 300_000_000:
        case["tokens"] //= 2
    return case


# ---------------------------------------------------------------- inputs
def _slots(case):
    return case["tokens"] * max(1, case["top"])


def _counts(case):
    """How many slots each expert has: multinomial with uneven odds."""
    r = np.random.RandomState(case["routing"])
    odds = np.exp(case["spread"] * r.standard_normal(case["E"]))
    return r.multinomial(_slots(case) - case["spare"] if _slots(case) > case["spare"] else _slots(case), odds / odds.sum())


def _activation(g, M, ld, K, dtype):
    x = torch.randn((M, ld), generator=g, device="cuda")
    x *= 1 + 7 * (torch.rand((M, ld), generator=g, device="cuda") < 0.01)
    return x.to(DTYPES[dtype])[:, :K]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, K, dtype = case["op"], case["K"], case["dtype"]
    if op in ("quantize", "fake"):
        x = _activation(g, case["M"], case.get("ld", K), K, dtype)
        s = {"op": op, "x": x * case["std"] if op == "fake" else x}
        if op == "fake" and dtype == "fp32":
            s["g"] = torch.randn((case["M"], K), generator=g, device="cuda")
        return s
    if op == "linear":
        w = 0.02 * torch.randn((case["N"], K), generator=g, device="cuda")
        b = 0.02 * torch.randn(case["N"], generator=g, device="cuda") if case["bias"] else None
        return {"op": op, "x": _activation(g, case["M"], case["ld"], K, dtype), "w": w, "b": b, "act": case["act"]}
    E, N, T = case["E"], case["N"], _slots(case)
    counts = np.roll(_counts(case), int(seed) % E)
    s = {"op": op, "x": _activation(g, case["tokens"], K, K, dtype), "act": case["act"], "most": int(counts.max()),
         "w": 0.02 * torch.randn((E, N, K), generator=g, device="cuda"),
         "b": 0.02 * torch.randn((E, N), generator=g, device="cuda") if case["bias"] else None,
         "offsets": torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda(), "rows": None,
         "y": torch.randn((T, N), generator=g, device="cuda").to(DTYPES[dtype])}
    if case["top"]:  # which token each slot takes, any token up to `top` times
        s["rows"] = (torch.randperm(T, generator=g, device="cuda") // case["top"]).to(torch.int32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if "w" in s:  # the weight is quantised once, when a model is loaded
        if own:
            from paper_1910_06188_b200 import binding as q8

            s["w"] = q8.q8_mx4_quantize(s["w"])
        else:
            s["w"] = _rounded(s["w"])
    return s


# ---------------------------------------------------------------- the plain form
def _rounded(x):
    """The fp32 values that the codes and scales of x stand for."""
    K = x.shape[-1]
    v = x.float()
    v = torch.where(torch.isnan(v), torch.zeros_like(v), v)
    v = torch.nn.functional.pad(v, (0, -K % BLOCK)).unflatten(-1, (-1, BLOCK))
    m = torch.where(torch.isinf(v), torch.zeros_like(v), v.abs()).amax(-1, keepdim=True)
    e = ((m.view(torch.int32) >> 23) - 2).clamp(min=0) - 127  # the exponent of the maximum less 2, at least -127
    t = torch.ldexp(v.abs(), -e)  # exact: at least 4 and below 8 at the maximum
    q = 0.5 * ((t > 0.25).float() + (t >= 0.75) + (t > 1.25) + (t >= 1.75)) + (t > 2.5).float() + (t >= 3.5) + 2.0 * (t > 5.0)
    return torch.ldexp(torch.where(v < 0, -q, q), e).flatten(-2)[..., :K]


def _activated(y, act):
    return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5))) if act else y


def _plain(s):
    x = s["x"]
    if s["op"] == "quantize":
        return _rounded(x)
    if s["op"] == "fake":
        y = _rounded(x).to(x.dtype)
        return [y, s["g"].clone()] if "g" in s else y
    if s["op"] == "linear":
        y = _rounded(x) @ s["w"].t()
        return _activated(y if s["b"] is None else y + s["b"], s["act"]).to(x.dtype)
    # every expert's rows, padded to the longest run, through one batched product
    offsets, T, E = s["offsets"].long(), s["y"].shape[0], s["w"].shape[0]
    slot = torch.arange(T, device=x.device)
    e = torch.searchsorted(offsets, slot, right=True) - 1
    used = (e >= 0) & (e < E)
    e = e.clamp(0, E - 1)
    at = torch.where(used, e * s["most"] + slot - offsets[e], E * s["most"])  # one place more, for slots of no expert
    h = _rounded(x)
    h = h if s["rows"] is None else h[s["rows"].long()]
    padded = h.new_zeros(E * s["most"] + 1, h.shape[1]).index_copy(0, at, h)
    y = torch.bmm(padded[:-1].view(E, s["most"], -1), s["w"].transpose(1, 2))
    y = _activated(y if s["b"] is None else y + s["b"][:, None], s["act"]).flatten(0, 1)
    y = torch.where(used[:, None], y[at.clamp(max=E * s["most"] - 1)].to(x.dtype), s["y"])
    s["y"].copy_(y)
    return s["y"]


# ---------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_1910_06188_b200 import binding as q8

    if s["op"] == "quantize":
        return q8.q8_mx4_dequantize(q8.q8_mx4_quantize(s["x"]))
    if s["op"] == "fake":
        y = q8.q8_mx4_fake_quantize(s["x"])
        return [y, q8.q8_ste_backward(s["g"])] if "g" in s else y
    if s["op"] == "linear":
        return q8.q8_mx4_linear(s["x"], s["w"], s["b"], s["act"])
    return q8.q8_mx4_linear_grouped(s["x"], s["offsets"], s["w"], s["b"], s["act"], s["rows"], s["y"])


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op, K, size = case["op"], case["K"], BYTES[case["dtype"]]
    packed = lambda rows: rows * (K / 2 + math.ceil(K / BLOCK))  # noqa: E731
    if op == "quantize":  # the codes and scales are written, and read when they are turned back
        return {"bytes": case["M"] * K * (size + 4) + 2 * packed(case["M"]), "flops": 0}
    if op == "fake":
        return {"bytes": case["M"] * K * 2 * size * (2 if case["dtype"] == "fp32" else 1), "flops": 0}
    if op == "linear":
        M, N = case["M"], case["N"]
        return {"bytes": M * K * size + packed(N) + 4 * N * case["bias"] + M * N * size, "flops": 2 * M * N * K}
    counts, N = _counts(case), case["N"]
    used, hit = int(counts.sum()), int((counts > 0).sum())
    return {"bytes": case["tokens"] * K * size + packed(N * hit) + 4 * N * hit * case["bias"] + used * N * size
            + 4 * (case["E"] + 1) + 4 * used * (case["top"] > 0), "flops": 2 * used * N * K}


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_values(x):
    """Block by block: the scale from the logarithm, the element as a multiple of its binade's step."""
    rows, K = x.shape
    out = torch.zeros_like(x, dtype=torch.float64)
    for k in range(0, K, BLOCK):
        v = torch.nan_to_num(x[:, k:k + BLOCK].double(), nan=0.0, posinf=math.inf, neginf=-math.inf)
        finite = torch.where(torch.isinf(v), 0.0, v)
        mantissa, exponent = torch.frexp(finite.abs().max(dim=1, keepdim=True).values)
        scale = torch.pow(2.0, (exponent.double() - 3).clamp(min=-127))
        t = v.abs() / scale
        step = torch.pow(2.0, torch.floor(torch.log2(t.clamp(1.0, 4.0))) - 1)  # 0.5 below 2, 1 below 4, 2 from there on
        out[:, k:k + BLOCK] = torch.sign(v) * torch.round(t / step).mul(step).clamp(max=6.0) * scale
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if s["op"] == "quantize":
        return _exact_values(s["x"])
    if s["op"] == "fake":
        y = _exact_values(s["x"])
        return [y, s["g"].double()] if "g" in s else y

    def layer(x, w, b):
        y = _exact_values(x) @ _exact_values(w).t()
        y = y if b is None else y + b.double()
        return y * torch.special.ndtr(y) if s["act"] else y

    if s["op"] == "linear":
        return layer(s["x"], s["w"], s["b"])
    y, ends = s["y"].double(), s["offsets"].tolist()
    x = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        if hi > lo:
            y[lo:hi] = layer(x[lo:hi], s["w"][e], None if s["b"] is None else s["b"][e])
    return y
