"""The 8-bit path of a transformer's linear layers as timed cases: each operator in its plain form and as the library's call.

A case is a dict of plain values; `op` says which operator it is:

  linear    int8 / uint8 codes [n, k] times int8 weights [out, k], one scale per token (or one for all) and one per channel
  quantize  rows of real values, gated or not, to int8 codes with one scale per row
  norm      norm behind a block, its gate and scale, the residual sum, the norm of the next block, int8 codes with a scale per row
  logprobs  log probabilities of given tokens, entropy and the largest alternatives of rows of logits

Codes are returned as the values they stand for (code times scale).  A code is floor(v * i + 1/2) with i = 127 / max|v| rounded to
32 bits, its scale max|v| / 127 rounded to 32 bits; both are part of the operator's definition.
"""
from __future__ import annotations

import math

import torch

own = False

MOST_MACS = 8192 * 4096 * 8192      # of the largest listed product; a drawn one stays below it
MOST_ROWS = 4096 * 8192             # elements of the largest listed activation
MOST_LOGITS = 1024 * 50001

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "s32": 4}


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one generated token through a square projection: the weights are read once and nothing else counts
        {"name": "linear_token", "op": "linear", "n": 1, "k": 4096, "out": 4096, "x": "s8", "y": "bf16", "bias": False, "per_token": True},
        # what a decoding batch holds at some moment, an odd number of output channels, biased
        {"name": "linear_decode_ragged", "op": "linear", "n": 23, "k": 2048, "out": 8191, "x": "s8", "y": "f16", "bias": True, "per_token": True},
        # the fully connected layer of the residual networks with real-valued logits: unsigned codes, one scale for the batch
        {"name": "linear_fc_u8", "op": "linear", "n": 256, "k": 2048, "out": 1000, "x": "u8", "y": "f32", "bias": True, "per_token": False},
        # a prompt batch through the widening projection: bound by the matrix units
        {"name": "linear_prefill", "op": "linear", "n": 8192, "k": 4096, "out": 8192, "x": "s8", "y": "bf16", "bias": False, "per_token": True},
        # the gated activation in front of the narrowing projection; gate and value are halves of one tensor
        {"name": "quantize_gated", "op": "quantize", "n": 4096, "c": 8192, "t": "bf16", "act": "silu", "gated": True},
        # a weight matrix, one scale per output channel, extents that no vector width divides
        {"name": "quantize_weights", "op": "quantize", "n": 8191, "c": 2047, "t": "f32", "act": "none", "gated": False},
        # one generated token between two blocks
        {"name": "norm_token", "op": "norm", "n": 1, "c": 4096, "t": "bf16", "post": "none", "pre": "rms", "gate": "none"},
        # part of a prompt, layer norms, a gate per token, an odd width
        {"name": "norm_chunk", "op": "norm", "n": 777, "c": 1537, "t": "f16", "post": "none", "pre": "layer", "gate": "token"},
        # a prompt batch with norms on both sides of the block and a gate per channel
        {"name": "norm_prefill", "op": "norm", "n": 4096, "c": 8192, "t": "bf16", "post": "rms", "pre": "rms", "gate": "channel"},
        # the 32-bit logits of a classifying network, its five likeliest classes
        {"name": "logprobs_classes", "op": "logprobs", "n": 256, "v": 1000, "t": "s32", "tokens": 1, "top": 5},
        # a decoding batch over a large vocabulary with alternatives
        {"name": "logprobs_decode", "op": "logprobs", "n": 16, "v": 131072, "t": "bf16", "tokens": 1, "top": 20},
        # scoring a text: many rows, an odd vocabulary, one alternative
        {"name": "logprobs_score", "op": "logprobs", "n": 1024, "v": 50001, "t": "f32", "tokens": 1, "top": 1},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: products of 1..8192 tokens with 64..16384 inputs and 16..32768 outputs, rows of 16..16384 values, vocabularies of
    100..262144, each spread over its logarithm, with odd extents, every type and every option."""
    op = rng.choice(["linear", "linear", "quantize", "norm", "logprobs"])
    if op == "linear":
        n, k, out = _log_int(rng, 1, 8192), _log_int(rng, 64, 16384), _log_int(rng, 16, 32768)
        if rng.random() < 0.75:
            k = max(64, k // 64 * 64)
        if rng.random() < 0.6:
            out = max(16, out // 16 * 16)
        n = max(1, min(n, MOST_MACS // (k * out)))
        out = max(16, min(out, MOST_MACS // (k * n)))
        return {"op": op, "n": n, "k": k, "out": out, "x": rng.choice(["s8", "s8", "s8", "u8"]), "y": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "bias": rng.random() < 0.5, "per_token": rng.random() < 0.8}
    if op == "quantize":
        c = _log_int(rng, 16, 16384)
        n = max(1, min(_log_int(rng, 1, 16384), MOST_ROWS // c))
        t, act = rng.choice([("f32", "none"), ("bf16", "none"), ("f16", "none"), ("bf16", "silu"), ("f16", "silu"), ("bf16", "gelu")])
        return {"op": op, "n": n, "c": c, "t": t, "act": act, "gated": act != "none" and rng.random() < 0.7}
    if op == "norm":
        c = _log_int(rng, 64, 16384)
        n = max(1, min(_log_int(rng, 1, 8192), MOST_ROWS // c))
        return {"op": op, "n": n, "c": c, "t": rng.choice(["bf16", "f16"]), "post": rng.choice(["none", "rms", "layer"]),
                "pre": rng.choice(["rms", "layer"]), "gate": rng.choice(["none", "channel", "token"])}
    v = _log_int(rng, 100, 262144)
    n = max(1, min(_log_int(rng, 1, 4096), MOST_LOGITS // v))
    return {"op": op, "n": n, "v": v, "t": rng.choice(["s32", "f32", "f16", "bf16"]), "tokens": rng.randint(1, 4), "top": rng.randint(1, 20)}


# ------------------------------------------------------------------ what a program has in hand before the call

FL_LOGITS = 12                      # fractional bits of the 32-bit logits
EPS = 1e-5
BRANCH = 0.25                       # the factor of a block's output in the residual sum


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    s = dict(case)
    if case["op"] == "linear":
        n, k, out = case["n"], case["k"], case["out"]
        s["w"] = (normal(out, k) * 32).round_().clamp_(-127, 127).to(torch.int8)
        x = normal(n, k) * 32
        s["x"] = x.round_().clamp_(-127, 127).to(torch.int8) if case["x"] == "s8" else x.abs_().round_().clamp_(0, 255).to(torch.uint8)
        s["xs"] = torch.rand(n if case["per_token"] else 1, generator=g, device="cuda") * 0.05 + 0.005
        s["ws"] = torch.rand(out, generator=g, device="cuda") * 0.001 + 0.0005
        s["bias"] = normal(out) if case["bias"] else None
        s["out"] = torch.empty(n, out, dtype=TYPES[case["y"]], device="cuda")
    elif case["op"] == "quantize":
        n, c, t = case["n"], case["c"], TYPES[case["t"]]
        both = normal(n, 2 * c if case["gated"] else c, dtype=t)
        s["x"], s["u"] = both[:, :c], both[:, c:] if case["gated"] else None
        s["q"], s["scale"] = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        s["y"] = torch.empty(n, c, dtype=t, device="cuda")
    elif case["op"] == "norm":
        n, c, t = case["n"], case["c"], TYPES[case["t"]]
        s["x"], s["r"] = normal(n, c, dtype=t), (normal(n, c) * 2 + 0.1).to(t)
        s["g"] = {"none": lambda: None, "channel": lambda: normal(1, c, dtype=t), "token": lambda: normal(n, c, dtype=t)}[case["gate"]]()
        s["post_w"] = normal(c) * 0.1 + 1 if case["post"] != "none" else None
        s["pre_w"] = normal(c) * 0.1 + 1
        s["pre_b"] = normal(c) * 0.1 if case["pre"] == "layer" else None
        s["q"], s["scale"] = torch.empty(n, c, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        s["y"], s["sum"] = torch.empty(n, c, dtype=t, device="cuda"), torch.empty(n, c, dtype=t, device="cuda")
    else:
        n, v = case["n"], case["v"]
        z = normal(n, v) * 3
        s["logits"] = (z * 2.0 ** FL_LOGITS).round_().to(torch.int32) if case["t"] == "s32" else z.to(TYPES[case["t"]])
        s["tokens"] = torch.randint(0, v, (n, case["tokens"]), generator=g, device="cuda")
        s["lp"], s["entropy"] = torch.empty(n, case["tokens"], device="cuda"), torch.empty(n, device="cuda")
        s["top_lp"] = torch.empty(n, case["top"], device="cuda")
        s["top_ids"] = torch.empty(n, case["top"], dtype=torch.int64, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return {"linear": _linear, "quantize": _quantize, "norm": _norm, "logprobs": _logprobs}[s["op"]](s)


def _library():
    from paper_2202_05239_b200 import api
    return api


def _linear(s):
    if own:
        _library().f8_linear_scaled(s["x"], s["xs"], s["w"], s["ws"], s["out"], bias=s["bias"])
        return s["out"]
    y = (s["x"].float() @ s["w"].float().t()) * s["xs"][:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(TYPES[s["y"]])


def _codes(v, t):
    """The values that the codes of the rows of v stand for, and the scales."""
    a = v.abs().amax(dim=1, keepdim=True)
    top = torch.full_like(a, 127.0)     # tensors on both sides of a division: a plain number's reciprocal would be multiplied by
    inverse, scale = top / a, a / top
    q = torch.floor(v.double() * inverse.double() + 0.5).clamp(-127, 127).float()
    return (q * scale).to(t), scale[:, 0]


def _quantize(s):
    if own:
        api = _library()
        act = {"none": api.F8_ACT_NONE, "silu": api.F8_ACT_SILU, "gelu": api.F8_ACT_GELU}[s["act"]]
        api.f8_quantize_rows(s["x"], s["q"], s["scale"], y=s["y"], u=s["u"], act=act)
        return {"values": s["y"], "scale": s["scale"]}
    v = s["x"].float()
    if s["act"] == "silu":
        v = v / (1 + torch.exp(-v))
    elif s["act"] == "gelu":
        v = 0.5 * v * (1 + torch.erf(v * 0.7071067811865476))
    if s["u"] is not None:
        v = v * s["u"].float()
    values, scale = _codes(v, TYPES[s["t"]])
    return {"values": values, "scale": scale}


def _normed(v, kind, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + EPS) * w
    return v if b is None else v + b


def _norm(s):
    if own:
        api = _library()
        kind = {"none": api.F8_NORM_NONE, "rms": api.F8_NORM_RMS, "layer": api.F8_NORM_LAYER}
        api.f8_norm_quantize(s["x"], s["q"], s["scale"], y=s["y"], residual=s["r"], residual_out=s["sum"], gate=s["g"],
                             post_norm=kind[s["post"]], post_w=s["post_w"], pre_norm=kind[s["pre"]], pre_w=s["pre_w"], pre_b=s["pre_b"],
                             eps=EPS, branch_scale=BRANCH)
        return {"sum": s["sum"], "values": s["y"], "scale": s["scale"]}
    v = _normed(s["x"].float(), s["post"], s["post_w"], None)
    if s["g"] is not None:
        v = v * s["g"].float()
    v = s["r"].float() + BRANCH * v
    values, scale = _codes(_normed(v, s["pre"], s["pre_w"], s["pre_b"]), TYPES[s["t"]])
    return {"sum": v.to(TYPES[s["t"]]), "values": values, "scale": scale}


def _logprobs(s):
    if own:
        _library().f8_token_logprobs(s["logits"], s["tokens"], s["lp"], entropy=s["entropy"], top_logprobs=s["top_lp"], top_ids=s["top_ids"],
                                     fl=FL_LOGITS if s["t"] == "s32" else 0)
        return {"lp": s["lp"], "entropy": s["entropy"], "top_lp": s["top_lp"], "top_ids": s["top_ids"]}
    z = s["logits"].float()
    if s["t"] == "s32":
        z = z * 2.0 ** -FL_LOGITS
    d = z - z.amax(dim=1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(dim=1, keepdim=True)
    lp = d - torch.log(total)
    entropy = torch.log(total)[:, 0] - (e * d).sum(dim=1) / total[:, 0]
    ids = torch.sort(s["logits"], dim=1, descending=True, stable=True).indices[:, :s["top"]]
    return {"lp": lp.gather(1, s["tokens"]), "entropy": entropy, "top_lp": lp.gather(1, ids), "top_ids": ids}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "linear":
        n, k, out = case["n"], case["k"], case["out"]
        scales = 4 * ((n if case["per_token"] else 1) + out * (2 if case["bias"] else 1))
        return {"bytes": n * k + out * k + scales + n * out * SIZE[case["y"]], "flops": 2 * n * k * out}
    if case["op"] == "quantize":
        n, c, b = case["n"], case["c"], SIZE[case["t"]]
        return {"bytes": n * c * (b * (3 if case["gated"] else 2) + 1) + 4 * n, "flops": 4 * n * c}
    if case["op"] == "norm":
        n, c, b = case["n"], case["c"], SIZE[case["t"]]
        gate = {"none": 0, "channel": c * b, "token": n * c * b}[case["gate"]]
        return {"bytes": n * c * (4 * b + 1) + gate + 4 * n + 4 * c * ((case["post"] != "none") + 1 + (case["pre"] == "layer")), "flops": 12 * n * c}
    n, v = case["n"], case["v"]
    return {"bytes": n * v * SIZE[case["t"]] + n * (12 * case["tokens"] + 4 + 12 * case["top"]), "flops": 4 * n * v}


# ------------------------------------------------------------------ the definition, in 64 bits

def _exact_codes(v):
    peak = v.abs().max(dim=1).values.float().double()
    i, scale = (127.0 / peak).float().double(), (peak / 127.0).float().double()
    return (v * i.unsqueeze(1) + 0.5).floor().clamp(min=-127, max=127) * scale.unsqueeze(1), scale


def _exact_norm(v, kind, w, b):
    if kind == "none":
        return v
    mu = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    v = (v - mu) * ((v - mu).square().mean(1, keepdim=True) + EPS).rsqrt() * w.double()
    return v if b is None else v + b.double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        y = torch.matmul(s["x"].double(), s["w"].double().T)
        y = y * torch.outer(s["xs"].double().expand(case["n"]), s["ws"].double())
        return y if s["bias"] is None else y + s["bias"].double()
    if case["op"] == "quantize":
        v = s["x"].double()
        if case["act"] == "silu":
            v = v * torch.special.expit(v)
        elif case["act"] == "gelu":
            v = v * torch.special.ndtr(v)
        if s["u"] is not None:
            v = v * s["u"].double()
        values, scale = _exact_codes(v)
        return {"values": values, "scale": scale}
    if case["op"] == "norm":
        branch = _exact_norm(s["x"].double(), case["post"], s["post_w"], None)
        if s["g"] is not None:
            branch = branch * s["g"].double()
        total = s["r"].double() + branch * BRANCH
        values, scale = _exact_codes(_exact_norm(total, case["pre"], s["pre_w"], s["pre_b"]))
        return {"sum": total, "values": values, "scale": scale}
    z = s["logits"].double() * (2.0 ** -FL_LOGITS if case["t"] == "s32" else 1.0)
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    p = torch.exp(z - lse)
    top = torch.sort(z, dim=1, descending=True, stable=True).values[:, :case["top"]]
    return {"lp": torch.gather(z, 1, s["tokens"]) - lse, "entropy": lse[:, 0] - (p * z).sum(1), "top_lp": top - lse, "top_ids": None}
