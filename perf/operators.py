"""The dense feed-forward block: trained in bf16, served in bf16 or in 8-bit integers, from one token to a long prefill.

A case names the operator and its sizes:

  forward    GatedFFN.forward(x): y = (silu(x Wg^T) * (x Wu^T)) Wd^T, weights and activations in bf16
  backward   GatedFFN.backward(x, dy): the gradients of x and of both weights; nothing was kept from the forward pass
  linear     Int8Linear.forward(x): x is rounded to 8-bit integers with one scale per token, the weight has one per
             output channel; the result comes in bf16 or fp32
  int8_ffn   Int8FFN.forward(x): the block of `forward` on the product of `linear`

H is the model's width, I the block's inner width (for `linear`: H inputs, I outputs), T the number of tokens.
Widths are those of this repository's workloads (experts, which run densely as always-on ones or in draft models) and
generic odd ones.  Activations are N(0,1) with a spread of scales over the channels, weights N(0,0.02), output
gradients N(0,0.01).
"""
import math

import torch

own = False

FORWARD, BACKWARD, LINEAR, INT8_FFN = "forward", "backward", "linear", "int8_ffn"


def _case(name, op, T, H, I, out="bf16"):
    return {"name": name, "op": op, "T": T, "H": H, "I": I, "out": out}


def listed():
    return [
        # one token through the smallest expert shape: a call whose latency counts
        _case("ffn_token", FORWARD, 1, 2048, 768),
        # a decode batch through the widest block: a stream of weights
        _case("ffn_decode", FORWARD, 16, 4096, 14336),
        # a ragged prefill chunk
        _case("ffn_chunk", FORWARD, 1023, 4096, 6400),
        # a long prefill through the widest block
        _case("ffn_prefill", FORWARD, 8192, 4096, 14336),
        # fine-tuning on one short sequence, small expert
        _case("grad_short", BACKWARD, 257, 2048, 1408),
        # nothing a multiple of a tile
        _case("grad_odd", BACKWARD, 777, 1096, 2744),
        # a training step's micro-batch through the widest block
        _case("grad_batch", BACKWARD, 4096, 4096, 14336),
        # one token through one projection
        _case("int8_token", LINEAR, 1, 7168, 2048),
        # a prefill chunk, ragged in tokens and in outputs, result kept in fp32
        _case("int8_chunk", LINEAR, 1023, 4096, 14333, "f32"),
        # decode batches of the block in 8 bits: a few sequences, a few dozen
        _case("int8_ffn_decode", INT8_FFN, 7, 4096, 14336),
        _case("int8_ffn_batch", INT8_FFN, 64, 5120, 1408),
        # a long prefill of the block in 8 bits
        _case("int8_ffn_prefill", INT8_FFN, 8192, 4096, 14336),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, min(hi, step * round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)))


def draw(rng):
    op = rng.choice((FORWARD, BACKWARD, LINEAR, INT8_FFN))
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        step = 8 if op in (FORWARD, BACKWARD) else 16
        c = {"op": op, "T": _log(rng, 1, 16384), "H": _log(rng, 256, 8192, step), "I": _log(rng, 256, 16384, step), "out": "bf16"}
        if op == LINEAR:
            c["I"] = _log(rng, 256, 16384)
            c["out"] = rng.choice(("bf16", "f32"))
        w = work(c)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return c


def _normal(shape, gen, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _rows_to_int8(w):
    """One scale per row: what a user's conversion of a checkpoint does."""
    scale = w.float().abs().amax(1) / 127.0
    return torch.round(w.float() / scale[:, None]).to(torch.int8), scale


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, T, H, I = case["op"], case["T"], case["H"], case["I"]
    s = {"op": op, "out": case["out"]}
    spread = torch.exp(_normal((H,), gen, 0.5, torch.float32))
    s["x"] = (_normal((T, H), gen, 1.0, torch.float32) * spread).to(torch.bfloat16)
    if op == LINEAR:
        s["weight"], s["weight_scale"] = _rows_to_int8(_normal((I, H), gen, 0.02))
        return s
    s["gate_up"] = _normal((2 * I, H), gen, 0.02)
    s["down"] = _normal((H, I), gen, 0.02)
    if op == BACKWARD:
        s["dy"] = _normal((T, H), gen, 0.01)
    if op == INT8_FFN:
        s["gate_up"], s["gate_up_scale"] = _rows_to_int8(s["gate_up"])
        s["down"], s["down_scale"] = _rows_to_int8(s["down"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2609_21483_b200 as weave
        if s["op"] == LINEAR:
            s["layer"] = weave.Int8Linear(s["weight"], s["weight_scale"], max_tokens=case["T"])
        elif s["op"] == INT8_FFN:
            s["layer"] = weave.Int8FFN(s["gate_up"], s["gate_up_scale"], s["down"], s["down_scale"], max_tokens=case["T"])
        else:
            s["layer"] = weave.GatedFFN(s["gate_up"], s["down"], max_tokens=case["T"], backward=s["op"] == BACKWARD)
    return s


# ---- the plain forms

def _dtype(s):
    return torch.float32 if s["out"] == "f32" else torch.bfloat16


def _gated(g, u):
    return g / (1.0 + torch.exp(-g)) * u


def _forward(s):
    g, u = (s["x"].float() @ s["gate_up"].float().T).chunk(2, dim=1)
    return (_gated(g, u) @ s["down"].float().T).to(torch.bfloat16)


def _backward(s):
    x, dy, gate_up, down = (s[k].float() for k in ("x", "dy", "gate_up", "down"))
    g, u = (x @ gate_up.T).chunk(2, dim=1)
    sig = 1.0 / (1.0 + torch.exp(-g))
    dh = dy @ down
    dgu = torch.cat([dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig], dim=1)
    return {"dx": (dgu @ gate_up).to(torch.bfloat16), "dgate_up": (dgu.T @ x).to(torch.bfloat16),
            "ddown": (dy.T @ (g * sig * u)).to(torch.bfloat16)}


def _tokens_to_int8(x):
    # the integer nearest to x / scale: quotients next to a half are common (x has 8 bits), so they are held in 64 bits
    # (and so is the scale's own division: by a Python number torch would multiply with a reciprocal rounded to fp32)
    scale = (x.double().abs().amax(1) / 127.0).float()
    return torch.nan_to_num(torch.round(x.double() / scale.double()[:, None])), scale


def _product(x, weight, weight_scale):
    """x in 8-bit integers times weight^T.  The sums pass 2^24, so they are held in 64 bits; the scales in 32."""
    q, scale = _tokens_to_int8(x)
    return (q @ weight.double().T).float() * (scale[:, None] * weight_scale[None, :])


def _int8_ffn(s):
    g, u = _product(s["x"], s["gate_up"], s["gate_up_scale"]).chunk(2, dim=1)
    # the gated product is a bf16 tensor before it is rounded to 8 bits: part of the operator's definition
    return _product(_gated(g, u).to(torch.bfloat16), s["down"], s["down_scale"]).to(torch.bfloat16)


def run(state):
    s = state
    if own:
        layer = s["layer"]
        if s["op"] == BACKWARD:
            dx, dgate_up, ddown = layer.backward(s["x"], s["dy"])
            return {"dx": dx, "dgate_up": dgate_up, "ddown": ddown}
        if s["op"] == LINEAR:
            return layer.forward(s["x"], out_dtype=_dtype(s))
        return layer.forward(s["x"])
    if s["op"] == FORWARD:
        return _forward(s)
    if s["op"] == BACKWARD:
        return _backward(s)
    if s["op"] == LINEAR:
        return _product(s["x"], s["weight"], s["weight_scale"]).to(_dtype(s))
    return _int8_ffn(s)


def work(case):
    """Inputs and weights read once, results written once, and the products.  The backward pass has x and dy alone,
    so it cannot do without the two projections of the forward pass: eight products of T x H x I."""
    op, T, H, I = case["op"], float(case["T"]), float(case["H"]), float(case["I"])
    if op == FORWARD:
        return {"bytes": 6 * H * I + 4 * T * H, "flops": 6 * T * H * I}
    if op == BACKWARD:
        return {"bytes": 12 * H * I + 6 * T * H, "flops": 16 * T * H * I}
    if op == LINEAR:
        return {"bytes": H * I + 4 * I + 2 * T * H + T * I * (4 if case["out"] == "f32" else 2), "flops": 2 * T * H * I}
    return {"bytes": 3 * H * I + 4 * (2 * I + H) + 4 * T * H, "flops": 6 * T * H * I}


# ---- the definitions in 64 bits

def _exact_quantised(x):
    """(integers, scales) in 64 bits; the scale itself is a 32-bit number by definition."""
    x = x.double()
    scale = (x.abs().max(dim=1, keepdim=True).values / 127.0).float().double()
    return torch.where(scale > 0, (x / scale).round(), torch.zeros_like(x)), scale


def _exact_product(x, weight, weight_scale):
    q, scale = _exact_quantised(x)
    return torch.einsum("tk,nk->tn", q, weight.double()) * scale * weight_scale.double()


def exact(case, seed):
    s = _inputs(case, seed)
    op, I = s["op"], case["I"]
    if op == LINEAR:
        return _exact_product(s["x"], s["weight"], s["weight_scale"])
    if op == INT8_FFN:
        gu = _exact_product(s["x"], s["gate_up"], s["gate_up_scale"])
        h = (gu[:, :I] * torch.sigmoid(gu[:, :I]) * gu[:, I:]).to(torch.bfloat16)
        return _exact_product(h, s["down"], s["down_scale"])
    x, w, down = s["x"].double(), s["gate_up"].double(), s["down"].double()
    g = torch.einsum("th,ih->ti", x, w[:I])
    u = torch.einsum("th,ih->ti", x, w[I:])
    sig = torch.sigmoid(g)
    if op == FORWARD:
        return torch.einsum("ti,hi->th", g * sig * u, down)
    dy = s["dy"].double()
    dh = torch.einsum("th,hi->ti", dy, down)
    dg, du = dh * u * (sig + g * sig * (1.0 - sig)), dh * g * sig
    return {"dx": torch.einsum("ti,ih->th", dg, w[:I]) + torch.einsum("ti,ih->th", du, w[I:]),
            "dgate_up": torch.cat([torch.einsum("ti,th->ih", dg, x), torch.einsum("ti,th->ih", du, x)]),
            "ddown": torch.einsum("th,ti->hi", dy, g * sig * u)}
