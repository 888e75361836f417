"""Products of 4-bit weights against 64 bits: forwards, gated and input gradient, every kernel form, odd sizes, strides, what is not finite,
graphs, streams. Marshalling and comparison only; the oracle is oracle/int4_oracle.py."""
import numpy as np
import pytest
import torch

import oracle.int4_oracle as I
import paper_2602_01613_amd as tn
from fp8_util import half_unit, host
from int4_util import FORM_CASES, GROUP_CASES, LONG_ROWS

pytestmark = pytest.mark.gpu

SCALE = {"bf16": torch.bfloat16, "f16": torch.float16}


def make(m, n, group, n_tensors=1, zeros=True, scale="bf16", seed=0):
    rng = np.random.default_rng(seed)
    groups, made = -(-n // group), []
    for _ in range(n_tensors):
        codes = rng.integers(0, 16, (m, n), dtype=np.uint8)
        z = rng.integers(0, 16, (m, groups), dtype=np.uint8) if zeros else None
        s = torch.from_numpy(np.exp2(rng.uniform(-9, -5, (m, groups))) * rng.choice([-1, 1], (m, groups))).to(SCALE[scale])
        made.append((codes, s, z))
    return made


def layer_of(made, n, group, tokens, **more):
    dev = lambda a: torch.from_numpy(a).cuda()      # noqa: E731
    zeros = None if made[0][2] is None else [dev(z) for _, _, z in made]
    return tn.Int4Linear([dev(I.pack(c)) for c, _, _ in made], tokens, group=group, scales=[s.cuda() for _, s, _ in made], zeros=zeros, in_features=n, **more)


def weights_of(made, group):
    return [I.weight(c, s.double().numpy(), z, group) for c, s, z in made]


def rows(tokens, cols, seed=1, size=1.0):
    return (torch.randn((tokens, cols), generator=torch.Generator().manual_seed(seed)) * size).bfloat16()


def bounds(made, group, x, exact_codes):
    """How far an fp32 sum may be from the 64-bit one, before its rounding to bf16, for each tensor [tokens, m].

    Streamed: products of 16 + code and of 16 + zero with x are exact, and every sum of n terms in fp32 is off by at most n * 2^-23 of the sum of their
    magnitudes (2^-23, not 2^-24, as additions inside the matrix cores may cut off); n: a group's, the correction, the groups', the waves'. In tiles each weight
    is rounded to fp16, 2^-11 of it at the most, and k terms are summed."""
    x = np.abs(host(x))
    result = []
    for c, s, z in made:
        k = c.shape[1]
        if exact_codes:
            terms = c.astype(np.float64) + 32 + (8 if z is None else np.repeat(z, group, axis=1)[:, :k])
            w = terms * np.repeat(np.abs(s.double().numpy()), group, axis=1)[:, :k]
            result.append((group + 4 + k / group + 16) * 2.0 ** -23 * (x @ w.T))
        else:
            w = np.abs(I.weight(c, s.double().numpy(), z, group))
            result.append((2.0 ** -11 + (k + 16) * 2.0 ** -23) * (x @ w.T))
    return result


def check(y, ref, off):
    got = host(y)
    assert np.isfinite(got).all()
    bad = np.abs(got - ref) > off + half_unit(np.abs(ref) + off, "bf16")
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


def streamed(m, n, n_tensors, tokens, gated, group):
    return tn.int4_plan_query(m, n, n_tensors, tokens, gated, tn.TN_INT4_PLAN_STREAM_TOKENS, group=group) > 0


# tokens, outputs, inputs, group, zeros, scales, tensors
CASES = [
    (1, 1, 1, 32, True, "bf16", 1), (1, 16, 128, 128, True, "bf16", 1), (1, 64, 256, 64, False, "f16", 1), (3, 100, 130, 32, True, "f16", 1), (7, 257, 1001, 128, True, "bf16", 2),
    (16, 64, 640, 64, True, "f16", 1), (17, 48, 1280, 32, False, "bf16", 1), (31, 130, 512, 128, True, "bf16", 2), (33, 777, 1001, 32, True, "f16", 1),
    (48, 80, 2048, 64, True, "bf16", 1), (64, 300, 129, 128, False, "f16", 1), (65, 300, 384, 32, True, "bf16", 1), (65, 64, 4096, 64, True, "f16", 1),
    (100, 1000, 1000, 128, True, "bf16", 2), (129, 256, 5120, 128, False, "bf16", 1), (200, 513, 640, 64, True, "bf16", 1), (300, 2000, 256, 32, False, "f16", 1),
    (513, 5120, 256, 128, True, "bf16", 1), (777, 700, 1100, 128, True, "f16", 1), (1025, 4100, 384, 64, True, "bf16", 2), (2100, 3000, 128, 32, True, "bf16", 1),
    (1, 5120, 25600, 128, True, "bf16", 1), (130, 128, 25600, 64, True, "bf16", 1),
]


@pytest.mark.parametrize("tokens,m,n,group,zeros,scale,tensors", CASES)
def test_forward(tokens, m, n, group, zeros, scale, tensors):
    made = make(m, n, group, tensors, zeros, scale)
    layer, x = layer_of(made, n, group, tokens), rows(tokens, n)
    y = layer(x.cuda())
    assert y.dtype == torch.bfloat16 and tuple(y.shape) == (tokens, tensors * m)
    off = bounds(made, group, x, streamed(m, n, tensors, tokens, False, group))
    for i, w in enumerate(weights_of(made, group)):
        check(y[:, i * m:(i + 1) * m], host(x) @ w.T, off[i])


@pytest.mark.parametrize("tokens,m,n,group,zeros,scale,tensors", CASES)
def test_input_gradient(tokens, m, n, group, zeros, scale, tensors):
    made = make(m, n, group, tensors, zeros, scale, seed=3)
    layer, dy = layer_of(made, n, group, tokens, transpose=True), rows(tokens, tensors * m, 4, 1e-3)
    dx = layer(dy.cuda())
    assert tuple(dx.shape) == (tokens, n)
    ref, most = 0.0, 0.0
    for i, w in enumerate(weights_of(made, group)):
        part = host(dy)[:, i * m:(i + 1) * m]
        ref, most = ref + part @ w, most + np.abs(part) @ np.abs(w)
    check(dx, ref, (2.0 ** -11 + (tensors * m + 16) * 2.0 ** -23) * most)


@pytest.mark.parametrize("tokens,m,n,group,zeros,scale,tensors", [c for c in CASES if c[1] * c[2] < 10 ** 7])
def test_gated(tokens, m, n, group, zeros, scale, tensors):
    """|silu'| <= 1.1 and |silu(v)| <= |v|: errors of gate and up pass on with up and with gate; the product and the sigmoid add 2^-20."""
    made = make(m, n, group, 2, zeros, scale, seed=5)
    layer, x = layer_of(made, n, group, tokens), rows(tokens, n, 6)
    gate, up = (host(x) @ w.T for w in weights_of(made, group))
    og, ou = bounds(made, group, x, streamed(m, n, 2, tokens, True, group))
    ref = I.silu_gate(gate, up)
    check(layer.gated(x.cuda()), ref, 1.1 * og * (np.abs(up) + ou) + np.abs(gate) * ou + 2.0 ** -20 * (np.abs(ref) + 1e-30))


@pytest.mark.parametrize("kind,tokens,m,n,group", FORM_CASES)
def test_every_form(kind, tokens, m, n, group):
    made = make(m, n, group, 2 if kind == "gated" else 1, tokens % 2 == 1, "f16" if m % 8 else "bf16", seed=tokens + m)
    w = weights_of(made, group)
    if kind == "back":
        layer, dy = layer_of(made, n, group, tokens, transpose=True), rows(tokens, m, 4, 1e-3)
        check(layer(dy.cuda()), host(dy) @ w[0], (2.0 ** -11 + (m + 16) * 2.0 ** -23) * (np.abs(host(dy)) @ np.abs(w[0])))
        return
    layer, x = layer_of(made, n, group, tokens), rows(tokens, n)
    off = bounds(made, group, x, streamed(m, n, len(made), tokens, kind == "gated", group))
    sums = [host(x) @ v.T for v in w]
    if kind == "plain":
        check(layer(x.cuda()), sums[0], off[0])
    else:
        ref = I.silu_gate(*sums)
        check(layer.gated(x.cuda()), ref, 1.1 * off[0] * (np.abs(sums[1]) + off[1]) + np.abs(sums[0]) * off[1] + 2.0 ** -20 * (np.abs(ref) + 1e-30))


def test_relative_error_is_that_of_one_rounding():
    """Random weights and activations: a rounding to bf16 is off by 2^-8 of a value's power of two at the most and evenly spread, 2^-8 / sqrt(3) in the mean square of that, which
    the values exceed: below 2^-8 / sqrt(3) of them. The weights' roundings to fp16, 2^-11, and the sums' add less than a tenth of it."""
    for tokens, transpose in ((8, False), (500, False), (500, True)):
        made = make(1024, 2048, 128, 1)
        layer, x = layer_of(made, 2048, 128, tokens, transpose=transpose), rows(tokens, 1024 if transpose else 2048)
        w = weights_of(made, 128)[0]
        ref = host(x) @ (w if transpose else w.T)
        assert np.linalg.norm(host(layer(x.cuda())) - ref) <= 1.1 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(ref)


@pytest.mark.parametrize("transpose", [False, True])
def test_rows_and_scales_of_any_size_in_tiles(transpose):
    """Tokens from 2^-120 to 2^120, one of zeros, one with channels 2^30 apart; features whose scales are 2^60 apart: each row and feature has its own power of two."""
    m, n, tokens = 96, 512, 70
    made = make(m, n, 128, 1)
    codes, s, z = made[0]
    grow = torch.exp2(torch.arange(m) % 60 - 30.0)[:, None] if not transpose else torch.exp2(torch.arange(4) * 20.0 - 40)[None, :]
    made = [(codes, (s.float() * grow).bfloat16(), z)]
    layer = layer_of(made, n, 128, tokens, transpose=transpose)
    x = rows(tokens, m if transpose else n).float() * torch.exp2(torch.linspace(-120, 80, tokens).round())[:, None]
    x[3] = 0
    x[4, ::7] *= 2.0 ** 30
    x = x.bfloat16()
    w = weights_of(made, 128)[0]
    w = w if transpose else w.T
    most = np.abs(host(x)) @ np.abs(w) + w.shape[0] * 2.0 ** -35 * np.abs(host(x)).max(axis=1, keepdims=True) * np.abs(w).max(axis=0, keepdims=True)
    y = layer(x.cuda())
    check(y, host(x) @ w, (2.0 ** -11 + (w.shape[0] + 16) * 2.0 ** -23) * most + 2.0 ** -133)
    assert bool((y[3] == 0).all())


@pytest.mark.parametrize("tokens", [1, 20, 64, 65, 200])
@pytest.mark.parametrize("lead,pad", [(1, 3), (8, 0), (0, 8), (4, 4)])
def test_strides_and_what_lies_beside(tokens, lead, pad):
    """Rows inside a wider tensor, aligned or not; what is beside the output stays as it was; NaN beside the input is not read."""
    m, n = 130, 384
    made = make(m, n, 64, 1)
    layer, x = layer_of(made, n, 64, tokens), rows(tokens, n)
    wide = torch.full((tokens, lead + n + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, lead:lead + n] = x.cuda()
    out = torch.full((tokens + 2, lead + m + pad + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    y = layer(wide[:, lead:lead + n], out=out[1:1 + tokens, lead:lead + m])
    assert torch.equal(y, layer(x.cuda()))
    out[1:1 + tokens, lead:lead + m] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("n", [100, 384])
@pytest.mark.parametrize("tokens", [2, 40, 100])
def test_not_finite(tokens, n):
    """An infinity or a NaN of a token shows in its row as the definition has it, and in no other row."""
    m, group = 70, 32
    made = make(m, n, group, 1)
    w = weights_of(made, group)[0]
    layer, x = layer_of(made, n, group, tokens), rows(tokens, n)
    clean = layer(x.cuda())
    x[0, 5], x[1, n - 1] = float("inf"), float("nan")
    y = layer(x.cuda())
    assert torch.equal(y[2:], clean[2:])
    with np.errstate(invalid="ignore"):
        ref = host(x) @ w.T
    for t in (0, 1):
        assert np.array_equal(np.isnan(host(y[t])), np.isnan(ref[t])) and np.array_equal(host(y[t])[np.isinf(ref[t])], ref[t][np.isinf(ref[t])])
    # gradients
    back, dy = layer_of(made, n, group, tokens, transpose=True), rows(tokens, m)
    clean = back(dy.cuda())
    dy[1, 3] = float("-inf")
    dx = back(dy.cuda())
    assert torch.equal(dx[2:], clean[2:]) and torch.equal(dx[0], clean[0])
    with np.errstate(invalid="ignore"):
        ref = (host(dy) @ w)[1]
    assert np.array_equal(np.isnan(host(dx[1])), np.isnan(ref)) and np.array_equal(host(dx[1])[np.isinf(ref)], ref[np.isinf(ref)])


def test_values_whose_code_sums_overflow():
    """x near the top of bf16 with small scales: the sums of 16 + code overflow, those of the weights do not."""
    codes = np.full((16, 128), 9, dtype=np.uint8)
    s = torch.full((16, 1), 2.0 ** -20).bfloat16()
    layer = layer_of([(codes, s, None)], 128, 128, 1)
    x = torch.full((1, 128), 2.0 ** 126).bfloat16()
    check(layer(x.cuda()), np.full((1, 16), 128 * 2.0 ** 106), 2.0 ** 113 * 128 * 2.0 ** -23)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,group", [(1, 1, 32), (33, 129, 64), (70, 1001, 32), (64, 256, 128)])
def test_quantised_at_create(m, n, group, dtype):
    rng = np.random.default_rng(7)
    w = (rng.standard_normal((m, n)) * np.exp2(rng.integers(-20, 20, (m, 1)))).astype(np.float32)
    w[0] = 0
    if m > 8:
        w[1] = np.abs(w[1])
        w[2] = -np.abs(w[2])
        w[3, n // 2], w[4, 0] = np.inf, np.nan
        w[5] = 1e-41
    t = torch.from_numpy(w).to(dtype)
    codes, scales, zeros = I.quantize(t.float().numpy(), group)
    for transpose in (False, True):
        layer = tn.Int4Linear([t.cuda()], 4, group=group, transpose=transpose)
        c, s, z = (v.cpu().numpy() for v in layer.quantized_tensor())
        assert np.array_equal(I.unpack(c, n), codes) and np.array_equal(z, zeros) and np.array_equal(s, scales, equal_nan=True)
    # half a step in a group of one sign or with zero inside, one where rounding moves the zero; the scale's own rounding adds 15 * 2^-8 of a step
    fine = np.isfinite(t.float().numpy()).all(axis=1) & (np.abs(w) > 1e-30).all(axis=1)
    err = np.abs(I.weight(codes, scales, zeros, group) - t.double().numpy())[fine]
    assert (err <= (1 + 15 * 2.0 ** -8) * np.repeat(scales.astype(np.float64), group, axis=1)[fine, :n]).all()


def test_given_codes_come_back():
    for n in (1, 65, 300):
        for scale in SCALE:
            made = make(90, n, 32, 2, True, scale)
            for transpose in (False, True):
                layer = layer_of(made, n, 32, 1, transpose=transpose)
                for i, (codes, s, z) in enumerate(made):
                    c, sc, zz = layer.quantized_tensor(i)
                    assert np.array_equal(I.unpack(c.cpu().numpy(), n), codes) and torch.equal(sc.cpu(), s.float()) and np.array_equal(zz.cpu().numpy(), z)


def test_same_from_call_to_call():
    made = make(600, 1100, 64, 2)
    layer = layer_of(made, 1100, 64, 300)
    for tokens in (1, 50, 300):
        x = rows(tokens, 1100).cuda()
        a, b = layer(x), layer.gated(x)
        for _ in range(3):
            assert torch.equal(layer(x), a) and torch.equal(layer.gated(x), b)


def test_no_tokens():
    made = make(40, 50, 32, 2)
    layer, back = layer_of(made, 50, 32, 5), layer_of(made, 50, 32, 5, transpose=True)
    x = torch.empty((0, 50), dtype=torch.bfloat16, device="cuda")
    assert tuple(layer(x).shape) == (0, 80) and tuple(layer.gated(x).shape) == (0, 40)
    assert tuple(back(torch.empty((0, 80), dtype=torch.bfloat16, device="cuda")).shape) == (0, 50)


@pytest.mark.parametrize("tokens", [1, 60, 200])
def test_graphs_and_streams(tokens):
    """Two captured calls of one layer, replayed on two streams at once and between eager work, give what eager calls give."""
    made = make(513, 1001, 128, 2)
    layer, back = layer_of(made, 1001, 128, tokens), layer_of(made, 1001, 128, tokens, transpose=True)
    xs = [rows(tokens, 1001, s).cuda() for s in (1, 2)]
    gs = [rows(tokens, 1026, s).cuda() for s in (3, 4)]
    want = [(layer.gated(x), layer(x), back(g)) for x, g in zip(xs, gs)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x, g in zip(xs, gs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append((layer.gated(x), layer(x), back(g)))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for out in outs:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        layer(xs[0])
        torch.cuda.synchronize()
        for out, ref in zip(outs, want):
            for t, r in zip(out, ref):
                assert torch.equal(t, r)


def test_eager_calls_on_two_streams():
    made = make(700, 1001, 64, 1)
    layer = layer_of(made, 1001, 64, 200)
    xs = [rows(200, 1001, s).cuda() for s in range(4)]
    want = [layer(x) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for s, x in zip(streams, xs):
        with torch.cuda.stream(s):
            got.append(layer(x))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    made = make(64, 128, 128, 2)
    layer, back = layer_of(made, 128, 128, 8), layer_of(made, 128, 128, 8, transpose=True)
    x = rows(8, 128).cuda()
    for bad in (x.float(), x[:, :100], x.t().contiguous().t(), x.cpu(), torch.zeros((9, 128), dtype=torch.bfloat16, device="cuda"), x[0]):
        with pytest.raises(ValueError):
            layer(bad)
    with pytest.raises(ValueError):
        back.gated(x)
    with pytest.raises(ValueError):
        layer(x, out=torch.empty((8, 127), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(tn.TNLinearError):
        layer(x, out=x)                                      # [8, 128] is what the pair of 64 outputs gives
    buffer = torch.zeros((16, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(tn.TNLinearError):
        layer(buffer[:8], out=buffer[7:15])
    layer(buffer[:8], out=buffer[8:])
    layer.close()
    with pytest.raises(RuntimeError):
        layer(x)


@pytest.mark.parametrize("scale", ["bf16", "f16"])
def test_a_layer_made_of_anothers_tensors_holds_the_same(scale):
    """Scales come back in fp32, and scale_dtype is the type that holds them exactly."""
    layer = layer_of(make(90, 300, 32, 1, True, scale), 300, 32, 1)
    assert layer.scale_dtype == SCALE[scale]
    codes, scales, zeros = layer.quantized_tensor()
    again = tn.Int4Linear([codes], 1, transpose=True, group=32, scales=[scales.to(layer.scale_dtype)], zeros=[zeros], in_features=300)
    assert all(torch.equal(a, b) for a, b in zip(again.quantized_tensor(), (codes, scales, zeros)))
    assert tn.Int4Linear([torch.ones((4, 64), device="cuda")], 1).scale_dtype == torch.bfloat16


@pytest.mark.parametrize("tokens", [1, 20, 64, 65, 200])
def test_input_and_output_beside_each_other_in_one_buffer(tokens):
    """Columns of the same rows share no element: outputs go beside the inputs, to either side, and nothing else is written."""
    m, n = 130, 384
    layer, x = layer_of(make(m, n, 64, 1), n, 64, tokens), rows(tokens, n).cuda()
    want = layer(x)
    for x_at, y_at in ((0, n), (m, 0), (m + 5, 3)):
        wide = torch.full((tokens, m + n + 9), 7.0, dtype=torch.bfloat16, device="cuda")
        wide[:, x_at:x_at + n] = x
        expect = wide.clone()
        expect[:, y_at:y_at + m] = want
        layer(wide[:, x_at:x_at + n], out=wide[:, y_at:y_at + m])
        assert torch.equal(wide, expect)


def dense(x, w):
    """x @ w in 64 bits: on the GPU, where hundreds of such products take no time."""
    return host(torch.matmul(x.cuda().double(), torch.from_numpy(np.ascontiguousarray(w)).cuda()))


@pytest.mark.parametrize("kind,tokens,m,n,group", [(*c[:4], g) for c in GROUP_CASES for g in c[4]])
def test_every_kernel(kind, tokens, m, n, group):
    made = make(m, n, group, 2 if kind == "gated" else 1, group != 64, "f16" if tokens % 2 else "bf16", seed=tokens + m + group)
    w = weights_of(made, group)
    if kind == "back":
        layer, dy = layer_of(made, n, group, tokens, transpose=True), rows(tokens, m, 4, 1e-3)
        check(layer(dy.cuda()), dense(dy, w[0]), (2.0 ** -11 + (m + 16) * 2.0 ** -23) * dense(dy.abs(), np.abs(w[0])))
        return
    layer, x = layer_of(made, n, group, tokens), rows(tokens, n)
    exact_codes = streamed(m, n, len(made), tokens, kind == "gated", group)
    off = []
    for (c, s, z), v in zip(made, w):          # as in bounds()
        terms = (c + 32.0 + (8 if z is None else np.repeat(z, group, axis=1)[:, :n])) * np.repeat(np.abs(s.double().numpy()), group, axis=1)[:, :n] if exact_codes else np.abs(v)
        off.append(((group + 4 + n / group + 16) * 2.0 ** -23 if exact_codes else 2.0 ** -11 + (n + 16) * 2.0 ** -23) * dense(x.abs(), terms.T))
    sums = [dense(x, v.T) for v in w]
    if kind == "plain":
        check(layer(x.cuda()), sums[0], off[0])
    else:
        ref = I.silu_gate(*sums)
        check(layer.gated(x.cuda()), ref, 1.1 * off[0] * (np.abs(sums[1]) + off[1]) + np.abs(sums[0]) * off[1] + 2.0 ** -20 * (np.abs(ref) + 1e-30))


@pytest.mark.parametrize("tokens,m,n,tensors,transposed,ranges,runs", LONG_ROWS)
def test_every_run_of_long_rows(tokens, m, n, tensors, transposed, ranges, runs):
    """Rows of one value each, which together have one in every run of 8 inputs: an output is that value, from 2^-20 to 2^20, times a weight rounded to fp16, and each row's power of two hangs
    on a run of its own. Then rows full of values: a run that was lost or taken twice among r of them is off by sqrt(1 / r) in the mean square, 1.2 % or more; the roundings
    are 2^-8 / sqrt(3), and the weights' a tenth of that, as above."""
    made = make(m, n, 128, tensors, True, "f16", seed=runs)
    layer = layer_of(made, n, 128, tokens, transpose=transposed)
    w = weights_of(made, 128)
    w = np.concatenate(w) if transposed else w[0].T              # [inputs, outputs]
    own = m if transposed else n                                 # inputs of a tensor: runs start anew with each, at a multiple of 128
    per = -(-own // 128) * 16
    rng = np.random.default_rng(8)
    run = np.arange(tokens) % (tensors * per)
    column = run // per * own + np.minimum(run % per * 8 + rng.integers(0, 8, tokens), own - 1)
    assert len(np.unique(column)) >= tensors * -(-own // 8)
    value = torch.from_numpy(rng.standard_normal(tokens) * np.exp2(rng.integers(-20, 21, tokens))).bfloat16()
    x = torch.zeros((tokens, tensors * own), dtype=torch.bfloat16, device="cuda")
    x[torch.arange(tokens), torch.from_numpy(column)] = value.cuda()
    ref = host(value)[:, None] * w[column]
    check(layer(x), ref, 2.0 ** -11 * np.abs(ref))
    x = torch.randn((tokens, tensors * own), generator=torch.Generator(device="cuda").manual_seed(9), dtype=torch.bfloat16, device="cuda")
    y = layer(x)
    some = torch.arange(0, tokens, tokens // 61)
    ref = dense(x[some], w)
    assert np.linalg.norm(host(y[some]) - ref) <= 1.1 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(ref)


@pytest.mark.parametrize("scale", ["f16", "bf16"])
@pytest.mark.parametrize("transpose", [False, True])
def test_scales_of_one_feature_far_apart_in_tiles(transpose, scale):
    """Scales from 1 to 2^-24 of the largest of a feature (transposed: of a group of features) in fp16, to 2^-30 in bf16, and tokens that read one of them alone: a weight is off by 2^-11 of itself and by
    2^-31 of the largest scale. The sums of the token's 32 values add 2^-23 for each."""
    m, n, group, tokens = 96, 512, 32, 192
    codes, s, z = make(m, n, group, 1, seed=12)[0]
    down = torch.arange(m)[:, None] / (m - 1) if transpose else torch.arange(n // group)[None, :] / (n // group - 1)
    s = (torch.sign(s.float()) * (1 + torch.rand(s.shape, generator=torch.Generator().manual_seed(1))) * torch.exp2(-torch.round((24 if scale == "f16" else 30) * down))).to(SCALE[scale])
    made = [(codes, s, z)]
    layer, w = layer_of(made, n, group, tokens, transpose=transpose), weights_of(made, group)[0]
    assert tn.int4_plan_query(m, n, 1, tokens, False, tn.TN_INT4_PLAN_TILE_TOKENS, transpose, group) > 0
    x = rows(tokens, m if transpose else n).float()
    own = (torch.arange(m)[None, :] if transpose else torch.arange(n)[None, :] // group) == torch.arange(tokens)[:, None] % (m if transpose else n // group)
    x = (x * own).bfloat16()
    size = np.abs(s.double().numpy())
    most = np.repeat(size.max(axis=0), group) if transpose else size.max(axis=1)             # of each output
    w = w if transpose else w.T
    sums = np.abs(host(x)) @ np.abs(w)
    check(layer(x.cuda()), host(x) @ w, (2.0 ** -11 + 48 * 2.0 ** -23) * sums + 2.0 ** -31 * np.abs(host(x)).sum(axis=1, keepdims=True) * most)


@pytest.mark.parametrize("transpose", [False, True])
def test_more_tokens_than_one_launch_converts(transpose):
    """Rows become fp16 2^19 at a time."""
    m, n, tokens = 24, 40, (1 << 19) + 4099
    made = make(m, n, 32, 2 if transpose else 1, seed=13)
    layer = layer_of(made, n, 32, tokens, transpose=transpose)
    w = weights_of(made, 32)
    w = np.concatenate(w) if transpose else w[0].T
    x = torch.randn((tokens, len(w)), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    check(layer(x), dense(x, w), (2.0 ** -11 + (len(w) + 16) * 2.0 ** -23) * dense(x.abs(), np.abs(w)))
