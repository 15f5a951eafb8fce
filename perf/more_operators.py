"""What the operators around a pruned block's products are timed on: the product with an epilogue (the block's
down product) and its gradients, dropout without a stored mask, the norm with an output in 8 bits, and products of
8-bit tokens with 8-bit weights.

`listed()` names the fixed cases and `draw(rng)` gives another one of the same ranges.  A case is a dict of plain
values.  Throughout, tokens x n is the input and a weight is n x m.

  op       "linear":            Z = X W + bias, Y = residual + D(act(Z))
           "linear_backward":   dZ = act'(Z) D(dY), dX = dZ W^T, dW = X^T dZ, dbias = column sums of dZ
           "dropout" / "dropout_backward":  residual + D(x), and D(dy)
           "norm8":             r = x + scale * gate * w_post * b/rms(b), y = w_pre * r/rms(r), y in 8 bits
           "q8" / "q8_gated":   residual + act(x W + bias), and act(x Wg) * (x Wu), x and the weights in 8 bits
  tokens, n, m
  dtype    "f32", "bf16" or "f16" (of what is not in 8 bits)
  act      "none", "silu", "gelu" or "relu"
  bias, residual      whether there is one
  saved    linear: also return Z
  p        share of entries that D drops; the others are divided by 1 - p
  gate     norm8: "channel" (one value per channel) or "token" (one per token and channel)

In 8 bits: every 32 neighbouring entries of a row (of x; of W along n, column by column) are e4m3 codes times one power
of two, the smallest with which the largest of them fits.

D keeps entry (t, c) if word c % 4 of Philox4x32-10 (Salmon et al. 2011), counter (c / 4, t, offset, offset's high half),
key (seed, its high half), is at least p * 2^32.

With `own` false, `run` computes the operators in elementary torch operations in 32 bits; with `own` true
it calls paper_2405_02086_amd.binding.
"""
import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-6


def _linear(name, tokens, n, m, dtype, **more):
    c = {"name": name, "op": "linear", "tokens": tokens, "n": n, "m": m, "dtype": dtype, "act": "none", "bias": False,
         "residual": False, "saved": False, "p": 0.0}
    c.update(more)
    return c


def _dropout(name, op, tokens, n, dtype, p, residual):
    return {"name": name, "op": op, "tokens": tokens, "n": n, "dtype": dtype, "p": p, "residual": residual}


def _norm8(name, tokens, n, dtype, gate):
    return {"name": name, "op": "norm8", "tokens": tokens, "n": n, "dtype": dtype, "gate": gate}


def _q8(name, op, tokens, n, m, dtype, act, bias=False, residual=False):
    return {"name": name, "op": op, "tokens": tokens, "n": n, "m": m, "dtype": dtype, "act": act, "bias": bias,
            "residual": residual}


def listed():
    return [
        # The smallest layer with everything but a residual: launches and host time.
        _linear("linear_small_f32", 16, 256, 128, "f32", act="gelu", bias=True),
        # One token through a wide block's down product, added to the residual stream.
        _linear("linear_token_bf16", 1, 16384, 4096, "bf16", residual=True),
        # The same for the forward half of a training step, with dropout on the block's result.
        _linear("linear_prompt_bf16", 4096, 16384, 4096, "bf16", residual=True, p=0.1),
        # Odd sizes throughout (no row is 16-byte aligned), pre-activations kept for the backward pass.
        _linear("linear_odd_saved_f16", 777, 2731, 1001, "f16", act="gelu", bias=True, saved=True),
        # The backward half of that training step.
        _linear("linear_backward_bf16", 4096, 16384, 4096, "bf16", op="linear_backward", residual=True, p=0.1),
        # The paper's matrix shape as a layer in fp32 with bias and activation.
        _linear("linear_backward_f32", 1000, 1000, 10000, "f32", op="linear_backward", act="gelu", bias=True),
        # Dropout on a block's result on its way into the residual stream, a batch of prompts.
        _dropout("dropout_prompt_bf16", "dropout", 16384, 4096, "bf16", 0.1, True),
        # The gradient of a small dropout, rows of odd length.
        _dropout("dropout_backward_odd_f32", "dropout_backward", 333, 1001, "f32", 0.5, False),
        # Between two blocks of a decoder that answers in 8 bits, one token.
        _norm8("norm8_token_bf16", 1, 4096, "bf16", "channel"),
        # The same over a batch of prompts.
        _norm8("norm8_prompt_bf16", 16384, 4096, "bf16", "channel"),
        # One token through the two input matrices of a block in 8 bits.
        _q8("q8_gated_token_bf16", "q8_gated", 1, 4096, 16384, "bf16", "silu"),
        # A prompt through the matrix behind it.
        _q8("q8_prompt_bf16", "q8", 4096, 16384, 4096, "bf16", "none", residual=True),
    ]


_MOST_FLOPS = 4 * 4096 * 16384 * 4096
_MOST_ENTRIES = 16384 * 4096


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi):
    """A power of two, an odd multiple of eight or an odd number."""
    v = _log_uniform(rng, lo, hi)
    kind = rng.choice(("power", "eight", "odd"))
    if kind == "power":
        return int(2 ** min(math.floor(math.log2(hi)), max(math.ceil(math.log2(lo)), round(math.log2(v)))))
    step = 8 if kind == "eight" else 1
    return step * (2 * max(0, round((v / step - 1) / 2)) + 1)


def _tokens(rng, hi, most):
    """A power of two or an odd number."""
    v = max(1, min(round(_log_uniform(rng, 1, hi)), most))
    return v if v & (v - 1) == 0 else v - 1 + v % 2


def draw(rng):
    op = rng.choice(("linear", "linear", "linear_backward", "linear_backward", "dropout", "dropout_backward", "norm8", "norm8",
                     "q8", "q8_gated"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op.startswith("linear"):
        n, m = _size(rng, 64, 16384), _size(rng, 64, 16384)
        # (fp32 products run at a tenth of the 16-bit rate)
        tokens = _tokens(rng, 8192, _MOST_FLOPS // (4 * n * m * (8 if dtype == "f32" else 1)))
        act = rng.choice(("none", "none", "silu", "gelu", "relu"))
        c = _linear("", tokens, n, m, dtype, op=op, act=act, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                    saved=op == "linear" and rng.random() < 0.3, p=rng.choice((0.0, 0.0, 0.1, 0.25, 0.5)))
    elif op.startswith("dropout"):
        n = _size(rng, 64, 16384)
        residual = op == "dropout" and rng.random() < 0.5
        c = _dropout("", op, _tokens(rng, 16384, 2 * _MOST_ENTRIES // (_BYTES[dtype] * n)), n, dtype,
                     rng.choice((0.05, 0.1, 0.5, 0.9)), residual)
    elif op == "norm8":
        n = _size(rng, 64, 16384)
        c = _norm8("", _tokens(rng, 16384, 2 * _MOST_ENTRIES // (_BYTES[dtype] * n)), n, dtype, rng.choice(("channel", "token")))
    else:
        n, m = _size(rng, 64, 16384), _size(rng, 64, 16384)
        tokens = _tokens(rng, 8192, _MOST_FLOPS // (4 * n * m))
        gated = op == "q8_gated"
        c = _q8("", op, tokens, n, m, dtype, rng.choice(("silu", "gelu", "relu") + (() if gated else ("none", "none"))),
                not gated and rng.random() < 0.5, not gated and rng.random() < 0.5)
    del c["name"]
    return c


def work(case):
    t, n, e, op = case["tokens"], case["n"], _BYTES[case["dtype"]], case["op"]
    if op == "linear":
        m = case["m"]
        return {"bytes": e * (t * n + n * m + t * m * (1 + case["residual"] + case["saved"]) + m * case["bias"]),
                "flops": 2 * t * n * m}
    if op == "linear_backward":
        m = case["m"]
        return {"bytes": e * (2 * t * n + 2 * n * m + t * m * (1 + (case["act"] != "none"))) + 4 * m * case["bias"],
                "flops": 4 * t * n * m}
    if op.startswith("dropout"):
        return {"bytes": e * t * n * (2 + case["residual"]), "flops": 3 * t * n}
    if op == "norm8":
        rows = 4 if case["gate"] == "token" else 3
        return {"bytes": n * (e * (rows * t + (2 if case["gate"] == "token" else 3)) + t * 33 / 32), "flops": 12 * t * n}
    m, mats = case["m"], 2 if op == "q8_gated" else 1
    return {"bytes": 33 / 32 * (t * n + mats * n * m) + e * (t * m * (1 + case["residual"]) + m * case["bias"]),
            "flops": 2 * mats * t * n * m}


# ---------------------------------------------------------------- inputs

def _eight_bits(v):
    """Rows in 8 bits: codes (float8_e4m3fn) of the entries filled up with zeros to whole groups of 128, scales
    (float8_e8m0fnu) of every 32 of them."""
    rows, n = v.shape
    wide = -(-n // 128) * 128
    full = torch.zeros(rows, wide, device=v.device)
    full[:, :n] = v
    g = full.view(rows, wide // 32, 32)
    e = _exponent(g.abs().amax(2))
    codes = (g * torch.exp2(-e)[:, :, None]).view(rows, wide).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _exponent(top):
    """The smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8), not below -127."""
    fraction, e = torch.frexp(top)                # top = fraction * 2^e, fraction in [0.5, 1)
    e = e.float() - 9 + (fraction > 0.875).float()
    return torch.where(top > 0, e, torch.full_like(e, -127.0)).clamp_min(-127.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t, n, dtype, op = case["tokens"], case["n"], _DTYPES[case["dtype"]], case["op"]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    s = {"case": case}
    if op.startswith(("linear", "dropout")):
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=gen, device="cuda"))
        s["offset"] = int(torch.randint(0, 2 ** 40, (1,), generator=gen, device="cuda"))
    if op.startswith("linear"):
        m = case["m"]
        s["X"], s["W"] = normal(t, n), normal(n, m, scale=n ** -0.5)
        if case["bias"]:
            s["bias"] = normal(m, scale=0.5)
        if op == "linear":
            if case["residual"]:
                s["residual"] = normal(t, m, scale=2.0)
        else:
            s["dY"] = normal(t, m)
            if case["act"] != "none":
                s["Z"] = normal(t, m)
    elif op.startswith("dropout"):
        s["x"] = normal(t, n)
        if case["residual"]:
            s["residual"] = normal(t, n, scale=2.0)
    elif op == "norm8":
        # a residual stream of growing size, and a few channels that stand out in every token
        s["b"] = normal(t, n, scale=0.7)
        out = torch.ones(n, device="cuda")
        out[torch.randint(0, n, (max(1, n // 256),), generator=gen, device="cuda")] = 8.0
        s["x"] = (torch.randn(t, n, generator=gen, device="cuda") * 2 * out).to(dtype)
        s["w_post"], s["w_pre"] = normal(n, scale=0.1) + 1, normal(n, scale=0.1) + 1
        s["gate"] = normal(t, n) if case["gate"] == "token" else normal(n)
        s["scale"] = 0.5
    else:
        m = case["m"]
        s["x8"] = _eight_bits(torch.randn(t, n, generator=gen, device="cuda"))
        s["W8"] = [_eight_bits(torch.randn(m, n, generator=gen, device="cuda") * n ** -0.5)
                   for _ in range(2 if op == "q8_gated" else 1)]
        if case["bias"]:
            s["bias"] = normal(m, scale=0.5)
        if case["residual"]:
            s["residual"] = normal(t, m, scale=2.0)
    if own:
        # what a program of this framework holds on to beside its data: scratch, and the views of packed matrices
        from paper_2405_02086_amd import binding as mp
        if op.startswith("linear"):
            s["workspace"] = mp.Workspace(mp.linear_workspace_bytes(t, n, case["m"], dtype, backward=op == "linear_backward"))
        elif op.startswith("q8"):
            s["x"] = mp.Q8(n, *s["x8"])
            s["W"] = [mp.Q8(n, *w) for w in s["W8"]]
            s["workspace"] = mp.Workspace(mp.q8_workspace_bytes(t, n, case["m"], gated=op == "q8_gated"))
    return s


# ---------------------------------------------------------------- the plain forms

def _act(kind, g):
    if kind == "silu":
        return g / (1 + torch.exp(-g))
    if kind == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * (g > 0) if kind == "relu" else g


def _act_slope(kind, g):
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p * (1 + g * (1 - p))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    return (g > 0).to(g.dtype) if kind == "relu" else torch.ones_like(g)


_LOW = 0xffffffff


def _kept(tokens, cols, s):
    """Where D keeps an entry: ten rounds of Philox4x32 on 64-bit integers, whose products wrap at 2^64."""
    quads = -(-cols // 4)
    c0 = torch.arange(quads, device="cuda").expand(tokens, quads)
    c1 = torch.arange(tokens, device="cuda")[:, None].expand(tokens, quads)
    c2, c3 = torch.full_like(c0, s["offset"] & _LOW), torch.full_like(c0, s["offset"] >> 32)
    k0, k1 = s["seed"] & _LOW, s["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack((c0, c1, c2, c3), -1).view(tokens, quads * 4)[:, :cols]
    return words >= min(round(s["case"]["p"] * 2 ** 32), _LOW)


def _drop(v, s):
    p = s["case"]["p"]
    return torch.where(_kept(v.shape[0], v.shape[1], s), v * (1 / (1 - p)), torch.zeros_like(v)) if p > 0 else v


def _plain_linear(s, case, dtype):
    z = s["X"].float() @ s["W"].float()
    if case["bias"]:
        z = z + s["bias"].float()
    y = _drop(_act(case["act"], z), s)
    if case["residual"]:
        y = s["residual"].float() + y
    return {"Y": y.to(dtype), "Z": z.to(dtype)} if case["saved"] else {"Y": y.to(dtype)}


def _plain_linear_backward(s, case, dtype):
    dz = _drop(s["dY"].float(), s)
    if case["act"] != "none":
        dz = dz * _act_slope(case["act"], s["Z"].float())
    out = {"dX": (dz @ s["W"].float().t()).to(dtype), "dW": (s["X"].float().t() @ dz).to(dtype)}
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    return out


def _plain_dropout(s, case, dtype):
    y = _drop(s["x"].float(), s)
    return {"y": (s["residual"].float() + y if case["residual"] else y).to(dtype)}


def _rstd(z):
    return 1 / torch.sqrt((z * z).mean(1, keepdim=True) + _EPS)


def _plain_norm8(s, case, dtype):
    x, b = s["x"].float(), s["b"].float()
    r = x + s["scale"] * s["gate"].float() * (b * _rstd(b) * s["w_post"].float())
    codes, scales = _eight_bits(r * _rstd(r) * s["w_pre"].float())
    return {"r": r.to(dtype), "y": codes[:, :case["n"]], "scales": scales}


def _wide(codes, scales, n):
    rows, wide = codes.shape
    return (codes.float().view(rows, wide // 32, 32) * scales.float()[:, :, None]).view(rows, wide)[:, :n]


def _plain_q8(s, case, dtype):
    x = _wide(*s["x8"], case["n"])
    y = x @ _wide(*s["W8"][0], case["n"]).t()
    if case["bias"]:
        y = y + s["bias"].float()
    y = _act(case["act"], y)
    if case["op"] == "q8_gated":
        y = y * (x @ _wide(*s["W8"][1], case["n"]).t())
    return (s["residual"].float() + y if case["residual"] else y).to(dtype)


_PLAIN = {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "dropout": _plain_dropout,
          "dropout_backward": _plain_dropout, "norm8": _plain_norm8, "q8": _plain_q8, "q8_gated": _plain_q8}


# ---------------------------------------------------------------- the framework's calls

def _own(s, case, dtype):
    from paper_2405_02086_amd import binding as mp
    op = case["op"]
    if op.startswith(("linear", "dropout")):
        drop = mp.Dropout(case["p"], s["seed"], s["offset"]) if case["p"] > 0 else None
    if op == "linear":
        z = torch.empty(case["tokens"], case["m"], dtype=dtype, device="cuda") if case["saved"] else None
        y = mp.linear(s["X"], s["W"], bias=s.get("bias"), residual=s.get("residual"), act=case["act"], dropout=drop, z_out=z,
                      workspace=s["workspace"])
        return {"Y": y, "Z": z} if case["saved"] else {"Y": y}
    if op == "linear_backward":
        dx, dw, dbias = mp.linear_backward(s["dY"], s["X"], s["W"], Z=s.get("Z"), act=case["act"], dropout=drop,
                                           need_dbias=case["bias"], workspace=s["workspace"])
        return {"dX": dx, "dW": dw, "dbias": dbias} if case["bias"] else {"dX": dx, "dW": dw}
    if op == "dropout":
        return {"y": mp.dropout(s["x"], drop, residual=s.get("residual"))}
    if op == "dropout_backward":
        return {"y": mp.dropout_backward(s["x"], drop)}
    if op == "norm8":
        r, y = mp.block_norm8(s["x"], s["b"], s["w_post"], s["gate"], s["w_pre"], scale=s["scale"], eps=_EPS)
        return {"r": r, "y": y.codes[:, :case["n"]], "scales": y.scales}
    if op == "q8":
        return mp.q8_linear(s["x"], s["W"][0], bias=s.get("bias"), residual=s.get("residual"), act=case["act"], dtype=dtype,
                            workspace=s["workspace"])
    return mp.q8_gated(s["x"], s["W"][0], s["W"][1], act=case["act"], dtype=dtype, workspace=s["workspace"])


def run(state):
    case = state["case"]
    dtype = _DTYPES[case["dtype"]]
    return _own(state, case, dtype) if own else _PLAIN[case["op"]](state, case, dtype)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_act(kind, g):
    if kind == "silu":
        return g * torch.special.expit(g)
    if kind == "gelu":
        return g * torch.special.ndtr(g)
    return torch.clamp_min(g, 0) if kind == "relu" else g


def _exact_kept(tokens, cols, s):
    """The generator again, with numbers of 32 bits as a high and a low half of 16 and the constants' products summed by halves."""
    def times(halves, constant):
        (h, l), (ch, cl) = halves, (constant >> 16, constant & 0xffff)
        low = l * cl
        mid = h * cl + (low >> 16)
        mid2 = l * ch + (mid & 0xffff)
        high = h * ch + (mid >> 16) + (mid2 >> 16)
        return (high >> 16, high & 0xffff), (mid2 & 0xffff, low & 0xffff)

    def split(v):
        return v >> 16, v & 0xffff

    quads = -(-cols // 4)
    shape = (tokens, quads)
    column, token = torch.arange(quads, device="cuda")[None].expand(shape), torch.arange(tokens, device="cuda")[:, None].expand(shape)
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    x = [split(column), split(token)] + [tuple(torch.full(shape, h, device="cuda") for h in split(v))
                                         for v in (s["offset"] % 2 ** 32, s["offset"] // 2 ** 32)]
    for r in range(10):
        keys = [split((k + r * w) % 2 ** 32) for k, w in zip(key, (0x9E3779B9, 0xBB67AE85))]
        (h0, l0), (h1, l1) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
        x = [tuple(a ^ b ^ c for a, b, c in zip(h1, x[1], keys[0])), l1, tuple(a ^ b ^ c for a, b, c in zip(h0, x[3], keys[1])), l0]
    share = torch.stack([h * 65536 + l for h, l in x], 2).reshape(tokens, quads * 4)[:, :cols].double() / 2.0 ** 32
    return share >= round(s["case"]["p"] * 2 ** 32) / 2.0 ** 32


def _exact_drop(v, s):
    p = s["case"]["p"]
    return v * _exact_kept(*v.shape, s).double() / (1 - p) if p > 0 else v


def _exact_rms_norm(z):
    return z / torch.sqrt(torch.linalg.vector_norm(z, dim=1, keepdim=True) ** 2 / z.shape[1] + _EPS)


def _exact_codes(y):
    """Values of the codes and of the scales: multiples of an e4m3 binade's step, 2^-3 of its power of two and 2^-9 at the least."""
    rows, n = y.shape
    groups = -(-n // 128) * 4
    y = torch.cat((y, y.new_zeros(rows, groups * 32 - n)), 1).view(rows, groups, 32)
    top = y.abs().amax(2)
    scale = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(-127, 127))
    # (a logarithm next to a whole number)
    scale = torch.where(top > 448 * scale, 2 * scale, torch.where((top <= 224 * scale) & (scale > 2.0 ** -127), scale / 2, scale))
    v = y / scale[:, :, None]
    binade = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))))
    step = binade / 8
    return (torch.round(v / step) * step).view(rows, groups * 32)[:, :n], scale


def exact(case, seed):
    """What `run` returns, by definition and in 64 bits; gradients by differentiating the forward definition."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    with torch.enable_grad():
        if op == "linear":
            z = s["X"].double() @ s["W"].double()
            if case["bias"]:
                z = z + s["bias"].double()
            y = _exact_drop(_exact_act(case["act"], z), s)
            if case["residual"]:
                y = y + s["residual"].double()
            return {"Y": y, "Z": z} if case["saved"] else {"Y": y}
        if op == "linear_backward":
            x, w = s["X"].double().requires_grad_(), s["W"].double().requires_grad_()
            z = x @ w
            at = (s["Z"].double() if case["act"] != "none" else z.detach()).requires_grad_()
            dz = torch.autograd.grad(_exact_drop(_exact_act(case["act"], at), s), at, s["dY"].double())[0]
            dx, dw = torch.autograd.grad(z, (x, w), dz)
            return {"dX": dx, "dW": dw, "dbias": dz.sum(0)} if case["bias"] else {"dX": dx, "dW": dw}
        if op.startswith("dropout"):
            y = _exact_drop(s["x"].double(), s)
            return {"y": y + s["residual"].double() if case["residual"] else y}
        if op == "norm8":
            r = s["x"].double() + s["scale"] * s["gate"].double() * (_exact_rms_norm(s["b"].double()) * s["w_post"].double())
            codes, scale = _exact_codes(_exact_rms_norm(r) * s["w_pre"].double())
            return {"r": r, "y": codes, "scales": scale}
        x, *weights = ((codes.double().unflatten(1, (-1, 32)) * scales.double()[:, :, None]).flatten(1) for codes, scales in [s["x8"]] + s["W8"])
        y = x @ weights[0].t()
        if case["bias"]:
            y = y + s["bias"].double()
        y = _exact_act(case["act"], y)
        if op == "q8_gated":
            y = y * (x @ weights[1].t())
        return y + s["residual"].double() if case["residual"] else y
