"""The operators around 8-bit projections of a decoder, as cases that can be timed.

8-bit format: e4m3 codes and power-of-two scales. A block of 128 consecutive elements of a row of activations, or of 128 x
128 elements of a weight, shares the scale 2^e with the least e >= -127 for which no finite element exceeds 448 * 2^e (-127
for a block of zeros); an element is stored as the e4m3 value nearest to v / 2^e (ties to even), and as NaN if it is not finite.

The kinds of a case (`case["kind"]`):
  norm        s = x + residual, rounded to the inputs' type; y = s / sqrt(mean(s^2) + eps) * weight, in 8 bits and, where
              `both`, in the inputs' type as well (what factorised projections read)
  norm_grad   for L = sum(dy * y) and a gradient `ds` that arrives at s from the residual branch: dL/ds, dL/dweight (fp32)
  linear      Y = X W^T of an 8-bit weight, in bf16. X comes in 8 bits (as the norm leaves it), or, with `transposed`, as a gradient in
              bf16, which the pass quantises first: the input gradient of the projection, DX = DY W
  gated       silu(X Wg^T) * (X Wu^T) of two 8-bit weights, in 8 bits: what the down projection reads
  gated_grad  for gate and up as the forward pass saved them and the gradient dh of silu(gate) * up: their gradients, in
              8 bits, as the input gradient of the pair reads them

Widths are those of the projections in `workloads/configs.py` (hidden width 5120, query width 8192, key/value width 1024, MLP
width 25600) and generic odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

_BLOCK = 128
_EPS = 1e-6
_PROJECTIONS = {"q": (5120, 8192), "k": (5120, 1024), "o": (8192, 5120), "up": (5120, 25600), "down": (25600, 5120)}
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_MOST_FLOPS = 2.0 * 8192 * 5120 * 25600      # of a drawn product: that of the largest listed one
_MOST_VALUES = 8192 * 5120                   # of a drawn elementwise case


def listed():
    return [
        # before the projections of one generated token
        {"name": "norm_decode_1", "kind": "norm", "tokens": 1, "width": 5120, "type": "bf16", "both": False},
        # before the projections of a long prompt, some of them factorised
        {"name": "norm_prefill_8192", "kind": "norm", "tokens": 8192, "width": 5120, "type": "bf16", "both": True},
        # fine-tuning: a micro-batch, and a small odd one in fp32
        {"name": "norm_grad_1024", "kind": "norm_grad", "tokens": 1024, "width": 5120, "type": "bf16"},
        {"name": "norm_grad_f32_odd", "kind": "norm_grad", "tokens": 333, "width": 1001, "type": "f32"},
        # one generated token through the query projection
        {"name": "linear_q_decode_1", "kind": "linear", "tokens": 1, "in": 5120, "out": 8192, "transposed": False},
        # verification of eight drafted tokens, down projection
        {"name": "linear_down_verify_8", "kind": "linear", "tokens": 8, "in": 25600, "out": 5120, "transposed": False},
        # fine-tuning: input gradient of the down projection, an odd micro-batch
        {"name": "linear_down_input_gradient_1001", "kind": "linear", "tokens": 1001, "in": 25600, "out": 5120, "transposed": True},
        # a long prompt through the up projection
        {"name": "linear_up_prefill_8192", "kind": "linear", "tokens": 8192, "in": 5120, "out": 25600, "transposed": False},
        # gate and up projections of an MLP block: one generated token, and a prompt of ragged length
        {"name": "gated_decode_1", "kind": "gated", "tokens": 1, "in": 5120, "out": 25600},
        {"name": "gated_prompt_777", "kind": "gated", "tokens": 777, "in": 5120, "out": 25600},
        # fine-tuning: back through silu(gate) * up, a small odd micro-batch and a whole one
        {"name": "gated_grad_77", "kind": "gated_grad", "tokens": 77, "width": 25600, "type": "bf16"},
        {"name": "gated_grad_1024", "kind": "gated_grad", "tokens": 1024, "width": 25600, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "linear", "linear", "linear", "gated", "gated", "gated_grad"])
    if kind in ("norm", "norm_grad", "gated_grad"):
        usual = [1024, 5120, 8192] if kind != "gated_grad" else [25600]
        width = rng.choice(usual) if rng.random() < 0.5 else _log_int(rng, 64, 16384)
        case = {"kind": kind, "tokens": min(_log_int(rng, 1, 8192), max(1, _MOST_VALUES // width)), "width": width,
                "type": rng.choice(["bf16", "bf16", "f32"])}
        if kind == "norm":
            case["both"] = rng.random() < 0.5
        return case
    if rng.random() < 0.6:
        n_in, n_out = _PROJECTIONS["up" if kind == "gated" else rng.choice(sorted(_PROJECTIONS))]
    else:
        n_in, n_out = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
    case = {"kind": kind, "in": n_in, "out": n_out}
    if kind == "linear":
        case["transposed"] = rng.random() < 0.3
    most = int(_MOST_FLOPS / (2 * n_in * n_out * (2 if kind == "gated" else 1)))
    case["tokens"] = max(1, min(_log_int(rng, 1, 8192), most))
    return case


# ---------------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    """Activations N(0, 1) with a few channels that are 30 times larger, as the residual stream of a trained decoder has them;
    weights N(0, 1 / inputs); gradients of size 1e-3."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, tokens = case["kind"], case["tokens"]

    def normal(rows, cols, size=1.0, dtype=torch.bfloat16, outliers=False):
        v = torch.randn((rows, cols), generator=gen, device="cuda")
        if outliers:
            v[:, torch.randint(0, cols, (max(1, cols // 500),), generator=gen, device="cuda")] *= 30
        return (v * size).to(dtype)

    if kind in ("norm", "norm_grad"):
        width, dtype = case["width"], _TYPES[case["type"]]
        weight = (1 + 0.2 * torch.randn((width,), generator=gen, device="cuda")).to(dtype)
        made = {"x": normal(tokens, width, 1.0, dtype, True), "weight": weight}
        if kind == "norm":
            made["residual"] = normal(tokens, width, 3.0, dtype, True)
        else:
            made["dy"], made["ds"] = normal(tokens, width, 1e-3, dtype), normal(tokens, width, 1e-3, dtype)
        return made
    if kind == "gated_grad":
        width, dtype = case["width"], _TYPES[case["type"]]
        return {"gate_up": normal(tokens, 2 * width, 2.0, dtype), "dh": normal(tokens, width, 1e-3, dtype)}
    n_in, n_out = case["in"], case["out"]
    made = {"weights": [normal(n_out, n_in, n_in ** -0.5) for _ in range(2 if kind == "gated" else 1)]}
    if case.get("transposed"):
        made["dy"] = normal(tokens, n_out, 1e-3)
    else:
        made["x"] = normal(tokens, n_in, 1.0, outliers=True)
    return made


# ---------------------------------------------------------------------------------------------------------------------------
# plain form
# ---------------------------------------------------------------------------------------------------------------------------
def _quantise(v, rows=1):
    """Codes and scales of fp32 [n, k], in blocks of `rows` x 128."""
    n, k = v.shape
    nb, kb = -(-n // rows), -(-k // _BLOCK)
    if nb * rows != n or kb * _BLOCK != k:
        v = torch.nn.functional.pad(v, (0, kb * _BLOCK - k, 0, nb * rows - n))
    v = v.reshape(nb, rows, kb, _BLOCK)
    most = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(dim=(1, 3), keepdim=True)
    part, e = torch.frexp(most)                                       # most = part * 2^e, part in [0.5, 1)
    e = torch.where(most > 0, e - 9 + (part > 0.875).to(e.dtype), -127).clamp(min=-127)
    inverse = ((127 - e) << 23).view(torch.float32)
    codes = (v * inverse).to(torch.float8_e4m3fn).reshape(nb * rows, kb * _BLOCK)[:n, :k]
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).reshape(nb, kb)


def _dequantise(codes, scales, rows=1):
    n, k = codes.shape
    scales = scales.to(torch.float32).repeat_interleave(_BLOCK, dim=1)[:, :k]
    if rows > 1:
        scales = scales.repeat_interleave(rows, dim=0)[:n]
    return codes.to(torch.float32) * scales


def _plain_norm(s, weight):
    return s * torch.rsqrt((s * s).mean(dim=1, keepdim=True) + _EPS) * weight


def _plain(state):
    kind = state["kind"]
    if kind == "norm":
        s = (state["x"].float() + state["residual"].float()).to(state["x"].dtype)
        y = _plain_norm(s.float(), state["weight"].float())
        codes, scales = _quantise(y)
        out = {"sum": s, "codes": codes, "scales": scales}
        if state["both"]:
            out["y"] = y.to(s.dtype)
        return out
    if kind == "norm_grad":
        s, dy = state["x"].float(), state["dy"].float()
        r = torch.rsqrt((s * s).mean(dim=1, keepdim=True) + _EPS)
        unit, g = s * r, dy * state["weight"].float()
        ds = r * (g - unit * (g * unit).mean(dim=1, keepdim=True)) + state["ds"].float()
        return {"ds": ds.to(state["x"].dtype), "dweight": (dy * unit).sum(dim=0)}
    if kind == "gated_grad":
        gate, up = state["gate_up"].float().chunk(2, dim=1)
        dh, sig = state["dh"].float(), torch.sigmoid(gate)
        dgate, dup = dh * up * sig * (1 + gate * (1 - sig)), dh * gate * sig
        (gc, gs), (uc, us) = _quantise(dgate), _quantise(dup)
        return {"gate_codes": gc, "gate_scales": gs, "up_codes": uc, "up_scales": us}
    weights = [_dequantise(c, s, _BLOCK) for c, s in state["weights"]]
    if state["transposed"]:
        codes, scales = _quantise(state["dy"].float())
        return (_dequantise(codes, scales) @ weights[0]).to(torch.bfloat16)
    x = _dequantise(*state["x"])
    if kind == "linear":
        return (x @ weights[0].t()).to(torch.bfloat16)
    gate, up = x @ weights[0].t(), x @ weights[1].t()
    codes, scales = _quantise(gate * torch.sigmoid(gate) * up)
    return {"codes": codes, "scales": scales}


# ---------------------------------------------------------------------------------------------------------------------------
# the framework's form
# ---------------------------------------------------------------------------------------------------------------------------
def _own(state):
    import paper_2602_01613_amd as tn
    kind = state["kind"]
    if kind == "norm":
        got = tn.rms_norm(state["x"], state["weight"], _EPS, residual=state["residual"], outputs="both" if state["both"] else "fp8")
        out = {"sum": got.sum, "codes": got.fp8.values(), "scales": got.fp8.block_scales()}
        if state["both"]:
            out["y"] = got.y
        return out
    if kind == "norm_grad":
        ds, dweight = tn.rms_norm_gradients(state["dy"], state["x"], state["weight"], _EPS, dsum=state["ds"])
        return {"ds": ds, "dweight": dweight}
    if kind == "gated_grad":
        d = tn.silu_gate_gradients(state["gate_up"], state["dh"], outputs="fp8").fp8
        return {"gate_codes": d.values(0), "gate_scales": d.block_scales(0), "up_codes": d.values(1), "up_scales": d.block_scales(1)}
    if kind == "linear":
        return state["layer"](state["dy"] if state["transposed"] else state["x"])
    h = state["layer"].gated(state["x"])
    return {"codes": h.values(), "scales": h.block_scales()}


def prepare(case, seed):
    made = _inputs(case, seed)
    kind = case["kind"]
    state = {"kind": kind}
    if kind in ("norm", "norm_grad", "gated_grad"):
        state.update(made, both=case.get("both", False))
        return state
    state["transposed"] = case.get("transposed", False)
    if own:
        import paper_2602_01613_amd as tn
        state["layer"] = tn.Fp8Linear(made["weights"], case["tokens"], transpose=state["transposed"])
    else:
        state["weights"] = [_quantise(w.float(), _BLOCK) for w in made["weights"]]
    if state["transposed"]:
        state["dy"] = made["dy"]
    else:
        state["x"] = tn.quantize_fp8(made["x"]) if own else _quantise(made["x"].float())
    return state


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------------------------------------------------------
def _exact_blocks(v, tall):
    """(values of the codes, scales), both in 64 bits: per row, or per 128 rows where `tall`."""
    codes, scales = torch.zeros_like(v), []
    for j in range(0, v.shape[1], _BLOCK):
        part = v[:, j:j + _BLOCK]
        most = part.abs().amax(dim=1)
        if tall:
            most = torch.stack([m.max() for m in most.split(_BLOCK)])
        e = torch.ceil(torch.log2((most / 448).clamp(min=2.0 ** -127)))
        e = torch.where(448 * torch.exp2(e - 1) >= most, e - 1, e)     # log2 may be off by its last bit
        e = torch.where(448 * torch.exp2(e) < most, e + 1, e).clamp(min=-127)
        scales.append(torch.exp2(e))
        q = part / (scales[-1].repeat_interleave(_BLOCK)[:v.shape[0]] if tall else scales[-1])[:, None]
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
        codes[:, j:j + _BLOCK] = torch.round(q / step) * step
    return codes, torch.stack(scales, dim=1)


def _exact_values(v, tall=False):
    codes, scales = _exact_blocks(v.double(), tall)
    n, k = codes.shape
    for b in range(scales.shape[1]):
        s = scales[:, b].repeat_interleave(_BLOCK)[:n] if tall else scales[:, b]
        codes[:, b * _BLOCK:(b + 1) * _BLOCK] *= s[:, None]
    return codes


def exact(case, seed):
    made = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        s = (made["x"].double() + made["residual"].double()).to(made["x"].dtype).double()
        y = s / torch.sqrt((s ** 2).sum(dim=1, keepdim=True) / case["width"] + _EPS) * made["weight"].double()
        codes, scales = _exact_blocks(y, False)
        out = {"sum": s, "codes": codes, "scales": scales}
        if case["both"]:
            out["y"] = y
        return out
    if kind == "norm_grad":
        # y_i = w_i s_i / n with n = sqrt(mean(s^2) + eps); dn/ds_j = s_j / (width * n)
        s, dy, w = made["x"].double(), made["dy"].double(), made["weight"].double()
        n = torch.sqrt((s ** 2).sum(dim=1, keepdim=True) / case["width"] + _EPS)
        along = (dy * w * s).sum(dim=1, keepdim=True)
        return {"ds": dy * w / n - s * along / (case["width"] * n ** 3) + made["ds"].double(), "dweight": (dy * s / n).sum(dim=0)}
    if kind == "gated_grad":
        width = case["width"]
        gate, up, dh = made["gate_up"][:, :width].double(), made["gate_up"][:, width:].double(), made["dh"].double()
        decay = torch.exp(-gate)
        dgate = dh * up * (1 + decay + gate * decay) / (1 + decay) ** 2
        (gc, gs), (uc, us) = _exact_blocks(dgate, False), _exact_blocks(dh * gate / (1 + decay), False)
        return {"gate_codes": gc, "gate_scales": gs, "up_codes": uc, "up_scales": us}
    weights = [_exact_values(w, True) for w in made["weights"]]
    if case.get("transposed"):
        return torch.matmul(_exact_values(made["dy"]), weights[0])
    x = _exact_values(made["x"])
    if kind == "linear":
        return torch.matmul(x, weights[0].t())
    gate, up = torch.matmul(x, weights[0].t()), torch.matmul(x, weights[1].t())
    codes, scales = _exact_blocks(gate / (1 + torch.exp(-gate)) * up, False)
    return {"codes": codes, "scales": scales}


def work(case):
    """Bytes: 8-bit operands with their scales, other tensors in their own type, gradients of weights in fp32. FLOPs: the
    products, and a handful for each value of the elementwise operators."""
    kind, tokens = case["kind"], case["tokens"]
    blocks = lambda n: -(-n // _BLOCK)                                  # noqa: E731
    eight = lambda rows, cols: rows * (cols + blocks(cols))            # noqa: E731
    elt = 4 if case.get("type") == "f32" else 2
    if kind == "norm":
        width = case["width"]
        nbytes = elt * (tokens * width * (4 if case["both"] else 3) + width) + eight(tokens, width)
        return {"bytes": nbytes, "flops": 7 * tokens * width}
    if kind == "norm_grad":
        width = case["width"]
        return {"bytes": elt * (4 * tokens * width + width) + 4 * width, "flops": 13 * tokens * width}
    if kind == "gated_grad":
        width = case["width"]
        return {"bytes": elt * 3 * tokens * width + 2 * eight(tokens, width), "flops": 14 * tokens * width}
    n_in, n_out, n = case["in"], case["out"], 2 if kind == "gated" else 1
    weights = n * (n_in * n_out + blocks(n_in) * blocks(n_out))
    flops = 2 * n * tokens * n_in * n_out
    if kind == "gated":
        return {"bytes": weights + eight(tokens, n_in) + eight(tokens, n_out), "flops": flops + 7 * tokens * n_out}
    if case["transposed"]:
        return {"bytes": weights + 2 * tokens * (n_in + n_out), "flops": flops}
    return {"bytes": weights + eight(tokens, n_in) + 2 * tokens * n_out, "flops": flops}
