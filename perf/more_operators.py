"""What factors are fine-tuned with beside frozen 4-bit projections, as cases that can be timed: products of weights in 4 bits with group
scales, their input gradients, the norm of the factors' gradients, and the AdamW step that updates them.

4-bit weights: W[f][k] = (code[f][k] - zero[f][k // group]) * scale[f][k // group], codes and zeros whole numbers from 0 to 15 (two codes to a
byte, the even k in the low half), scales in 16 bits, groups of 32, 64 or 128 inputs; without zeros they are 8.

AdamW, step t (the count before it, and one) on the gradients g of many tensors, with n the root of the sum of all g^2:
  g <- g * max_norm / n where n > max_norm
  m <- beta1 * m + (1 - beta1) * g,   v <- beta2 * v + (1 - beta2) * g^2
  p <- p * (1 - lr * decay) - lr * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
Parameters in bf16 are roundings of an fp32 master, which is what the step updates. The state is one buffer over all tensors, each tensor
starting at a multiple of 128. In 8 bits it holds m and the root of v as e4m3 codes, with a power-of-two scale for each 128: 2^e with the least
e >= -127 for which nothing finite in the block exceeds 448 * 2^e. A value between two codes takes the farther one from zero if the part of the
step by which it exceeds the nearer, plus (h + 1/2) / 2^16, reaches one, where h is a whole number below 2^16 that a hash of the seed, the step
and the place gives: nothing is lost on average, however small the steps of a state are beside those of its codes.

The kinds of a case (`case["kind"]`):
  linear      Y = X W^T in bf16
  gated       silu(X Wg^T) * (X Wu^T) in bf16
  gradient    DX = sum over the tensors of DY_i W_i in bf16: the input gradient of one projection, or of two that read the same inputs
  norm        the root of the sum of the squares of all gradients
  adamw       the step, with the norm and the clipping where `clip`

Widths are those of the projections in `workloads/configs.py` (hidden width 5120, query width 8192, key/value width 1024, MLP width 25600) and
generic odd ones; the factors are those of its trains, rings and Tucker layers.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_PROJECTIONS = {"q": (5120, 8192), "k": (5120, 1024), "o": (8192, 5120), "up": (5120, 25600), "down": (25600, 5120)}
_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_MOST_FLOPS = 2.0 * 8192 * 5120 * 25600      # of a drawn product: that of the largest listed one
_BLOCK = 128
_LR, _BETA1, _BETA2, _EPS, _DECAY, _MAX_NORM, _SEED, _COUNT = 1e-5, 0.9, 0.999, 1e-8, 0.01, 1.0, 1234567, 1000

# numbers of values of a layer's tensors: trains 5120 -> 8192 of rank 64, rings 25600 -> 5120 of rank 32, Tucker layers 5120 -> 25600 of ranks
# 64, 64, 32, 32
_LAYERS = {
    "train": (8 * 8 * 64, 64 * 16 * 10 * 64, 64 * 8 * 8 * 64, 64 * 8 * 8),
    "ring": (32 * 8 * 10 * 32, 32 * 10 * 16 * 32, 32 * 8 * 10 * 32, 32 * 8 * 16 * 32),
    "tucker": (64 * 64 * 32 * 32, 160 * 64, 160 * 64, 64 * 32, 80 * 32),
}
_MOST_LAYERS = 64


def listed():
    return [
        # one generated token through the query projection
        {"name": "linear_q_decode_1", "kind": "linear", "tokens": 1, "in": 5120, "out": 8192, "group": 128, "zeros": True, "scale": "bf16"},
        # verification of eight drafted tokens, down projection
        {"name": "linear_down_verify_8", "kind": "linear", "tokens": 8, "in": 25600, "out": 5120, "group": 64, "zeros": False, "scale": "f16"},
        # a short odd batch through a small odd projection
        {"name": "linear_odd_33", "kind": "linear", "tokens": 33, "in": 1001, "out": 777, "group": 32, "zeros": True, "scale": "f16"},
        # a long prompt through the up projection
        {"name": "linear_up_prefill_8192", "kind": "linear", "tokens": 8192, "in": 5120, "out": 25600, "group": 128, "zeros": True, "scale": "bf16"},
        # gate and up projections of an MLP block: one generated token, and a prompt of ragged length
        {"name": "gated_decode_1", "kind": "gated", "tokens": 1, "in": 5120, "out": 25600, "group": 128, "zeros": True, "scale": "bf16"},
        {"name": "gated_prompt_777", "kind": "gated", "tokens": 777, "in": 5120, "out": 25600, "group": 128, "zeros": False, "scale": "bf16"},
        # fine-tuning: input gradient of the down projection, an odd micro-batch; of gate and up together, a small one
        {"name": "gradient_down_1001", "kind": "gradient", "tensors": 1, "tokens": 1001, "in": 25600, "out": 5120, "group": 128, "zeros": True, "scale": "bf16"},
        {"name": "gradient_gate_up_77", "kind": "gradient", "tensors": 2, "tokens": 77, "in": 5120, "out": 25600, "group": 64, "zeros": True, "scale": "bf16"},
        # the gradients of one train's cores, and of all factors that are fine-tuned
        {"name": "norm_train", "kind": "norm", "layout": "train", "layers": 1, "grad": "f32"},
        {"name": "norm_mixed_64", "kind": "norm", "layout": "mixed", "layers": 64, "grad": "f32"},
        # one Tucker layer fine-tuned with states in 32 bits; all factors with states in 8 bits and clipping
        {"name": "adamw_tucker", "kind": "adamw", "layout": "tucker", "layers": 1, "grad": "f32", "param": "bf16", "bits": 32, "clip": False},
        {"name": "adamw_mixed_64_8bit", "kind": "adamw", "layout": "mixed", "layers": 64, "grad": "f32", "param": "bf16", "bits": 8, "clip": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "gated", "gated", "gradient", "gradient", "norm", "adamw", "adamw", "adamw"])
    if kind in ("norm", "adamw"):
        layout = rng.choice(["train", "ring", "tucker", "mixed", "odd"])
        case = {"kind": kind, "layout": layout, "layers": _log_int(rng, 1, _MOST_LAYERS // (4 if layout == "tucker" else 1)), "grad": rng.choice(["f32", "f32", "bf16"])}
        if layout == "odd":
            case["sizes"] = rng.randrange(1 << 20)
        if kind == "adamw":
            case.update(param=rng.choice(["bf16", "bf16", "f32"]), bits=rng.choice([8, 32]), clip=rng.random() < 0.5)
        return case
    if rng.random() < 0.6:
        n_in, n_out = _PROJECTIONS["up" if kind == "gated" else rng.choice(sorted(_PROJECTIONS))]
    else:
        n_in, n_out = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
    case = {"kind": kind, "in": n_in, "out": n_out, "group": rng.choice([32, 64, 128, 128]), "zeros": rng.random() < 0.6, "scale": rng.choice(["bf16", "bf16", "f16"])}
    if kind == "gradient":
        case["tensors"] = rng.choice([1, 2])
    most = int(_MOST_FLOPS / (2 * n_in * n_out * _tensors(case)))
    case["tokens"] = max(1, min(_log_int(rng, 1, 8192), most))
    return case


def _tensors(case):
    return 2 if case["kind"] == "gated" else case.get("tensors", 1)


def _sizes(case):
    """Numbers of values of the tensors of a `norm` or `adamw` case."""
    layout, layers = case["layout"], case["layers"]
    if layout == "odd":
        rng = random.Random(case["sizes"])
        return [_log_int(rng, 1, 1 << 20) for _ in range(4 * layers)]
    names = ("train", "ring", "tucker") if layout == "mixed" else (layout,)
    return [n for i in range(layers) for n in _LAYERS[names[i % len(names)]]]


# ---------------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------------
def _weights_and_rows(case, gen):
    """Activations N(0, 1) with a few channels that are 30 times larger, as the residual stream of a trained decoder has them;
    gradients of size 1e-3; weights of size 1 / sqrt(inputs) whose groups differ in size and in where they have their zero."""
    n_in, n_out, group, tokens = case["in"], case["out"], case["group"], case["tokens"]
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")      # noqa: E731
    groups, made = -(-n_in // group), {"weights": []}
    for _ in range(_tensors(case)):
        zeros = (8 + 1.5 * normal(n_out, groups)).round_().clamp_(0, 15).to(torch.uint8) if case["zeros"] else None
        codes = normal(n_out, n_in + n_in % 2).mul_(2.5)
        centre = zeros.repeat_interleave(group, dim=1)[:, :n_in] if case["zeros"] else 8
        codes[:, :n_in] += centre
        codes = codes.round_().clamp_(0, 15).to(torch.uint8)
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
        scales = (0.4 * n_in ** -0.5 * torch.exp(0.3 * normal(n_out, groups))).to(_TYPES[case["scale"]])
        made["weights"].append((codes.contiguous(), scales, zeros))
    if case["kind"] == "gradient":
        made["rows"] = (1e-3 * normal(tokens, n_out * _tensors(case))).bfloat16()
    else:
        x = normal(tokens, n_in)
        x[:, torch.randint(0, n_in, (max(1, n_in // 500),), generator=gen, device="cuda")] *= 30
        made["rows"] = x.bfloat16()
    return made


def _places(sizes):
    """(place of each tensor in the state, length of the state)"""
    places, end = [], 0
    for n in sizes:
        places.append(end)
        end += -(-n // _BLOCK) * _BLOCK
    return places, end


def _tensors_and_state(case, gen):
    """Gradients whose size differs from tensor to tensor, by a power of ten at the most; parameters of the size of a core's;
    the state of a run that is _COUNT steps old. One buffer for each, laid out like the state, with zeros between the tensors."""
    sizes = _sizes(case)
    places, length = _places(sizes)
    normal = lambda: torch.randn((length,), generator=gen, device="cuda")      # noqa: E731
    counts = torch.tensor(sizes, device="cuda")
    which = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), -(-counts // _BLOCK) * _BLOCK, output_size=length)
    there = torch.arange(length, device="cuda") - torch.tensor(places, device="cuda")[which] < counts[which]
    spread = 10 ** torch.rand((len(sizes),), generator=gen, device="cuda")
    size = 1e-4 * spread[which] * there
    made = {"sizes": sizes, "places": places, "grad": (normal() * size).to(_TYPES[case["grad"]])}
    if case["kind"] == "adamw":
        made["master"] = normal().mul_(0.04) * there
        made["params"] = made["master"].to(_TYPES[case["param"]])
        made["first"] = normal() * 0.25 * size
        made["second"] = size * size * torch.exp(0.3 * normal())
        if case["bits"] == 8:
            made["first"], made["first_scales"] = _nearest(made["first"])
            made["second"], made["second_scales"] = _nearest(made["second"].sqrt_())
        made["count"] = torch.tensor(_COUNT, dtype=torch.int64, device="cuda")
    return made


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return _tensors_and_state(case, gen) if case["kind"] in ("norm", "adamw") else _weights_and_rows(case, gen)


def _block_exponents(v):
    """Biased exponents of the scales of the blocks of v [blocks, 128], as int32 [blocks, 1]."""
    most = v.abs().amax(dim=1, keepdim=True)
    part, e = torch.frexp(most)                                       # most = part * 2^e, part in [0.5, 1)
    return torch.where(most > 0, e - 9 + (part > 0.875).to(e.dtype), -127).clamp(min=-127) + 127


def _scales(e):
    return e.to(torch.uint8).view(torch.float8_e8m0fnu).reshape(-1)


def _nearest(v):
    v = v.reshape(-1, _BLOCK)
    e = _block_exponents(v)
    codes = (v * ((254 - e) << 23).view(torch.float32)).to(torch.float8_e4m3fn)
    return codes.reshape(-1), _scales(e)


# ---------------------------------------------------------------------------------------------------------------------------
# plain form
# ---------------------------------------------------------------------------------------------------------------------------
def _dequantise(state, codes, scales, zeros):
    n, group = state["in"], state["group"]
    q = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1)[:, :n].float()
    q -= 8.0 if zeros is None else zeros.repeat_interleave(group, dim=1)[:, :n].float()
    return q * scales.float().repeat_interleave(group, dim=1)[:, :n]


def _plain_product(state):
    x = state["rows"].float()
    weights = [_dequantise(state, *w) for w in state["weights"]]
    if state["kind"] == "gradient":
        return sum(part @ w for part, w in zip(x.chunk(len(weights), dim=1), weights)).bfloat16()
    if state["kind"] == "linear":
        return (x @ weights[0].t()).bfloat16()
    gate, up = x @ weights[0].t(), x @ weights[1].t()
    return (gate * torch.sigmoid(gate) * up).bfloat16()


def _plain_norm(grad):
    return grad.double().square().sum().sqrt().float()


def _mix(x):
    """32 bits to 32 bits, in the low half of int64."""
    x = ((x ^ (x >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xB7E15163) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _hash(count, length):
    """32 bits for each place of a state, for the step that makes the count `count`."""
    place = torch.arange(length, dtype=torch.int64, device="cuda")
    key = _mix(_mix(torch.full_like(count, _SEED)) ^ count)
    return _mix((place & 0xFFFFFFFF) ^ _mix(key ^ (place >> 32)))


def _towards_both(v, h):
    """v in 8 bits, with 16 random bits h for each value: codes and scales."""
    v = v.reshape(-1, _BLOCK)
    e = _block_exponents(v)
    y = v * ((254 - e) << 23).view(torch.float32)
    size = y.abs()
    low = size < 2.0 ** -6                                            # below the least normal code all steps are alike
    bits = torch.where(low, size + 2.0 ** -6, size).view(torch.int32) + h.reshape(-1, _BLOCK).to(torch.int32) * 16 + 8
    codes = (bits >> 20) - torch.where(low, 968, 960) + torch.where(y < 0, 128, 0)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn).reshape(-1), _scales(e)


def _values(codes, scales):
    return (codes.float().reshape(-1, _BLOCK) * scales.float()[:, None]).reshape(-1)


def _plain_step(state):
    g = state["grad"].float()
    out = {}
    if state["clip"]:
        out["norm"] = _plain_norm(state["grad"])
        g = g * torch.where(out["norm"] > _MAX_NORM, _MAX_NORM / out["norm"], 1.0)
    state["count"] += 1
    t, eight = state["count"].double(), state["bits"] == 8
    m = _values(state["first"], state["first_scales"]) if eight else state["first"]
    v = _values(state["second"], state["second_scales"]).square() if eight else state["second"]
    m = _BETA1 * m + (1 - _BETA1) * g
    v = _BETA2 * v + (1 - _BETA2) * g * g
    move = _LR * (m / (1 - _BETA1 ** t).float()) / ((v / (1 - _BETA2 ** t).float()).sqrt() + _EPS)
    master = state["master"] if state["param"] == "bf16" else state["params"]
    master.copy_(master * (1 - _LR * _DECAY) - move)
    if state["param"] == "bf16":
        state["params"].copy_(master)
        out["master"] = master
    if eight:
        h = _hash(state["count"], m.numel())
        codes, scales = _towards_both(m, h & 0xFFFF)
        state["first"].copy_(codes), state["first_scales"].copy_(scales)
        codes, scales = _towards_both(v.sqrt(), h >> 16)
        state["second"].copy_(codes), state["second_scales"].copy_(scales)
        out.update(first_scales=state["first_scales"], second_scales=state["second_scales"])
    else:
        state["first"].copy_(m), state["second"].copy_(v)
    out.update(params=state["params"], first=state["first"], second=state["second"], count=state["count"])
    return out


def _plain(state):
    if state["kind"] == "norm":
        return _plain_norm(state["grad"])
    return _plain_step(state) if state["kind"] == "adamw" else _plain_product(state)


# ---------------------------------------------------------------------------------------------------------------------------
# the framework's form
# ---------------------------------------------------------------------------------------------------------------------------
def _own(state):
    kind = state["kind"]
    if kind == "norm":
        return state["optimizer"].gradient_norm(state["grads"])
    if kind == "adamw":
        norm = state["optimizer"].step(state["grads"], max_norm=_MAX_NORM if state["clip"] else None)
        out = {"params": state["params"], **state["optimizer"].state_dict()}
        if state["clip"]:
            out["norm"] = norm
        return out
    return state["layer"].gated(state["rows"]) if kind == "gated" else state["layer"](state["rows"])


def prepare(case, seed):
    made = _inputs(case, seed)
    state = {**case, **made}
    if not own:
        return state
    import paper_2602_01613_amd as tn
    if case["kind"] in ("norm", "adamw"):
        views = lambda flat: [flat[p:p + n] for p, n in zip(made["places"], made["sizes"])]      # noqa: E731
        state["grads"] = views(made["grad"])
        state["optimizer"] = tn.AdamW(views(made.get("params", made["grad"])), lr=_LR, betas=(_BETA1, _BETA2), eps=_EPS, weight_decay=_DECAY,
                                      state_bits=case.get("bits", 32), seed=_SEED)
        if case["kind"] == "adamw":
            keys = ["first", "second", "count"] + ["master"] * (case["param"] == "bf16") + ["first_scales", "second_scales"] * (case["bits"] == 8)
            state["optimizer"].load_state_dict({k: made[k] for k in keys})
    else:
        codes, scales, zeros = zip(*made["weights"])
        state["layer"] = tn.Int4Linear(codes, case["tokens"], transpose=case["kind"] == "gradient", group=case["group"], scales=scales,
                                       zeros=zeros if case["zeros"] else None, in_features=case["in"])
    return state


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------------------------------------------------------
def _exact_weight(case, codes, scales, zeros):
    rows, n = codes.shape[0], case["in"]
    w = torch.empty((rows, 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    w[:, 0::2], w[:, 1::2] = codes % 16, codes // 16
    of = torch.arange(n, device=codes.device) // case["group"]
    return (w[:, :n] - (8.0 if zeros is None else zeros.double()[:, of])) * scales.double()[:, of]


def _exact_product(case, made):
    x, total = made["rows"].double(), 0.0
    outputs = []
    for i, w in enumerate(made["weights"]):
        w = _exact_weight(case, *w)
        if case["kind"] == "gradient":
            total = total + torch.matmul(x[:, i * case["out"]:(i + 1) * case["out"]], w)
        else:
            outputs.append(torch.matmul(x, w.t()))
    if case["kind"] == "gradient":
        return total
    return outputs[0] if case["kind"] == "linear" else outputs[0] / (1 + torch.exp(-outputs[0])) * outputs[1]


def _exact_hash(length, count):
    """The hash with Python's whole numbers for what all places share."""
    def shared(x):
        x = (x ^ x >> 16) * 0x9E3779B1 % 2 ** 32
        x = (x ^ x >> 15) * 0xB7E15163 % 2 ** 32
        return x ^ x >> 16
    # (places below 2^32 only: the states of the cases are shorter)
    x = torch.arange(length, device="cuda") ^ shared(shared(shared(_SEED) ^ count))
    for shift, factor in ((16, 0x9E3779B1), (15, 0xB7E15163)):
        x = torch.bitwise_xor(x, x >> shift)
        x = ((x * (factor >> 16) % 65536 * 65536) + x * (factor & 0xFFFF)) % 2 ** 32
    return torch.bitwise_xor(x, x >> 16)


def _exact_codes(v, h):
    v = v.reshape(-1, _BLOCK)
    most = v.abs().max(dim=1, keepdim=True).values
    e = torch.ceil(torch.log2((most / 448).clamp(min=2.0 ** -127)))
    e = torch.where(448 * torch.exp2(e - 1) >= most, e - 1, e)         # log2 may be off by its last bit
    e = torch.where(448 * torch.exp2(e) < most, e + 1, e).clamp(min=-127)
    y = v.abs() / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    nearer = torch.floor(y / step)
    farther = y / step - nearer + (h.reshape(-1, _BLOCK).double() + 0.5) / 65536 >= 1
    return (torch.sign(v) * (nearer + farther) * step).reshape(-1), torch.exp2(e).reshape(-1)


def exact(case, seed):
    made = _inputs(case, seed)
    if case["kind"] not in ("norm", "adamw"):
        return _exact_product(case, made)
    g = made["grad"].double()
    norm = torch.linalg.vector_norm(g)
    if case["kind"] == "norm":
        return norm
    out = {}
    if case["clip"]:
        out["norm"] = norm
        g = g * min(1.0, _MAX_NORM / float(norm))
    t, eight = _COUNT + 1, case["bits"] == 8
    m, v = made["first"].to(torch.float64), made["second"].to(torch.float64)
    if eight:
        of = torch.arange(m.numel(), device="cuda") // _BLOCK
        m, v = m * made["first_scales"].to(torch.float64)[of], (v * made["second_scales"].to(torch.float64)[of]) ** 2
    m, v = m + (1 - _BETA1) * (g - m), v + (1 - _BETA2) * (g ** 2 - v)
    p = (made["master"] if case["param"] == "bf16" else made["params"]).double()
    p = p - _LR * (_DECAY * p + m / (1 - _BETA1 ** t) / (torch.sqrt(v / (1 - _BETA2 ** t)) + _EPS))
    out["params"], out["count"] = p, t
    if case["param"] == "bf16":
        out["master"] = p
    if eight:
        h = _exact_hash(m.numel(), t)
        m, out["first_scales"] = _exact_codes(m, h % 65536)
        v, out["second_scales"] = _exact_codes(torch.sqrt(v), h // 65536)
    out["first"], out["second"] = m, v
    return out


def work(case):
    """Bytes: codes two to a byte, zeros likewise, scales in 16 bits, other tensors in their own type; of a step each gradient once, parameters,
    masters and states in and out (bf16 parameters out). FLOPs: the products, and a handful for each value of the others."""
    kind = case["kind"]
    if kind in ("norm", "adamw"):
        values = sum(_sizes(case))
        grad = 4 if case["grad"] == "f32" else 2
        if kind == "norm":
            return {"bytes": grad * values + 4, "flops": 2 * values}
        states = 16 if case["bits"] == 32 else 4 * (1 + 1 / _BLOCK)
        return {"bytes": values * (grad + (10 if case["param"] == "bf16" else 8) + states), "flops": values * (20 if case["bits"] == 32 else 60)}
    n_in, n_out, tokens, n = case["in"], case["out"], case["tokens"], _tensors(case)
    weights = n * n_out * (n_in / 2 + -(-n_in // case["group"]) * (2.5 if case["zeros"] else 2))
    outputs = n_out if kind == "gated" else n * n_out
    return {"bytes": weights + 2 * tokens * (n_in + outputs), "flops": 2 * n * tokens * n_in * n_out + (7 * tokens * n_out if kind == "gated" else 0)}
