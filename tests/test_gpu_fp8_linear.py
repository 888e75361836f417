"""Products of 8-bit weights with 8-bit activations against 64 bits on the same codes."""
import numpy as np
import pytest
import torch

import oracle.fp8_oracle as Q
import paper_2602_01613_amd as tn
from fp8_util import FORM_CASES, check_eight_bit, check_padding, dev, exponents, half_unit, host, on_gpu, rounded
from paper_2602_01613_amd import fp8

pytestmark = pytest.mark.gpu

def weights_of(rng, m, n, count, dtype="bf16"):
    return [rounded(rng.standard_normal((m, n)) * n ** -0.5, dtype) for _ in range(count)]


def activations(rng, rows, cols):
    v = rng.standard_normal((rows, cols))
    v[:, rng.integers(0, cols, max(1, cols // 300))] *= 30
    return v


def eight(v, rows=1):
    return Q.dequantize(*Q.quantize(v, rows), rows)


def sums_off(x8, w8):
    """What the matrix cores' sums may be off by: the products of 8 consecutive k are aligned to the largest of them and cut off (towards
    zero) at 2^-13 of it, which costs each of the seven others less than that; sums of groups are fp32's."""
    pad = -x8.shape[1] % 8
    most = lambda v: np.abs(np.pad(v, ((0, 0), (0, pad)))).reshape(v.shape[0], -1, 8).max(axis=2)      # noqa: E731
    return (7 * 2.0 ** -13 + 2.0 ** -18) * (most(x8) @ most(w8).T)


def check_product(got, x8, w8):
    ref = x8 @ w8.T
    err = np.abs(host(got) - ref)
    bound = half_unit(ref, "bf16") + sums_off(x8, w8)
    assert np.isfinite(host(got)).all() and (err <= bound).all(), (err - bound).max()
    if ref.size >= 64:         # all of it: a rounding to bf16 is 2^-8 at the most, and one lost k in 5120 would be 1.4e-2
        assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(ref)


# tokens around the sizes of fragments and tiles; features and inputs of one, of a block less and more, and of whole tiles
TOKENS = [1, 2, 15, 16, 17, 33, 64, 65, 100, 128, 129, 200, 257, 300, 520]
SHAPES = [(1, 1), (64, 64), (127, 129), (128, 128), (300, 200), (777, 1001), (1024, 640), (260, 5120)]


@pytest.mark.parametrize("m,n", SHAPES)
def test_forward(m, n):
    rng = np.random.default_rng(m * 10007 + n)
    w = weights_of(rng, m, n, 1)
    layer, w8 = tn.Fp8Linear([dev(w[0])], max(TOKENS)), eight(w[0], 128)
    x = rounded(activations(rng, max(TOKENS), n))
    x8 = eight(x)
    for tokens in TOKENS:
        rows = tn.quantize_fp8(dev(x[:tokens]))
        y = layer(rows)
        check_product(y, x8[:tokens], w8)
        assert torch.equal(y, layer(rows)) and torch.equal(y, layer(dev(x[:tokens])))


@pytest.mark.parametrize("m,n", [(5, 9), (128, 256), (200, 300), (640, 1001)])
@pytest.mark.parametrize("count", [1, 2])
def test_transposed(m, n, count):
    """Gradients of the outputs to that of the inputs: two tensors' gradients are two segments, and their shares are added."""
    rng = np.random.default_rng(m * 31 + n + count)
    w = weights_of(rng, m, n, count)
    layer, w8 = tn.Fp8Linear([dev(v) for v in w], 300, transpose=True), np.concatenate([eight(v, 128) for v in w])
    assert (layer.M, layer.N) == (n, count * m)
    for tokens in (1, 16, 20, 70, 130, 300):
        dy = rounded(rng.standard_normal((tokens, count * m)) * 1e-3)
        x8 = np.concatenate([eight(dy[:, i * m:(i + 1) * m]) for i in range(count)], axis=1)
        check_product(layer(dev(dy)), x8, w8.T)


@pytest.mark.parametrize("m,n", [(1, 5), (128, 128), (130, 300), (640, 1000), (1025, 512)])
def test_pair_and_gated(m, n):
    rng = np.random.default_rng(m * 17 + n)
    w = weights_of(rng, m, n, 2)
    layer, w8 = tn.Fp8Linear([dev(v) for v in w], 520), [eight(v, 128) for v in w]
    assert (layer.M, layer.N) == (2 * m, n)
    for tokens in (1, 7, 16, 17, 40, 65, 130, 257, 520):
        x = rounded(activations(rng, tokens, n))
        x8, rows = eight(x), tn.quantize_fp8(dev(x))
        check_product(layer(rows), x8, np.concatenate(w8))
        got = layer.gated(rows)
        check_padding(got)
        gate, up = x8 @ w8[0].T, x8 @ w8[1].T
        # what the sums may be off by, through silu(gate) * up
        eg, eu = sums_off(x8, w8[0]), sums_off(x8, w8[1])
        ref = Q.silu_gate(gate, up)
        off = 1.1 * np.abs(up) * eg + np.abs(Q.silu_gate(gate, 1.0)) * eu + 1.1 * eg * eu + 2.0 ** -20 * np.abs(ref)
        codes, exps = host(got.values()), exponents(got.block_scales())
        blocks = range(0, m, 128)
        most = np.stack([np.abs(ref[:, b:b + 128]).max(axis=1) for b in blocks], axis=1)
        slack = np.stack([off[:, b:b + 128].max(axis=1) for b in blocks], axis=1)
        assert ((exps >= Q.block_exponent(np.maximum(most - slack, 0))) & (exps <= Q.block_exponent(most + slack))).all()
        scale = np.repeat(np.exp2(exps.astype(np.float64)), 128, axis=1)[:, :m]
        bound = 2.0 ** -4 * (np.abs(ref) + off) + 2.0 ** -10 * scale + off
        assert (np.abs(Q.dequantize(codes, exps) - ref) <= bound).all()
        again = layer.gated(rows, out=tn.Fp8Rows.empty(tokens, m))
        assert torch.equal(again.codes.view(torch.uint8), got.codes.view(torch.uint8)) and torch.equal(again.scales.view(torch.uint8), got.scales.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("m,n", [(1, 1), (130, 257), (256, 128)])
def test_quantised_weights(m, n, transpose, dtype):
    """Codes and scales bit for bit, out of a layer as they went in, and a layer made from them gives the same results."""
    rng = np.random.default_rng(m + n)
    w = [rounded(rng.standard_normal((m, n)) * np.exp2(rng.integers(-20, 20, (m, n)) / 4), dtype) for _ in range(2)]
    if m > 1:
        w[1][:128, :128] = 0
    layer = tn.Fp8Linear([dev(v, dtype) for v in w], 40, transpose)
    parts = [layer.quantized_tensor(i) for i in range(2)]
    for i in range(2):
        codes, exps = Q.quantize(w[i], 128)
        assert np.array_equal(host(parts[i][0]), codes) and np.array_equal(exponents(parts[i][1]), exps)
    twin = tn.Fp8Linear([p[0] for p in parts], 40, transpose, scales=[p[1] for p in parts])
    x = dev(rng.standard_normal((33, layer.N)))
    assert torch.equal(layer(x), twin(x))
    assert layer.query(tn.TN_QUERY_PARAM_COUNT) == 2 * m * n
    layer.close()
    with pytest.raises(RuntimeError):
        layer(x)


@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_what_is_not_finite_stays_in_its_rows(tokens):
    rng = np.random.default_rng(tokens)
    x = rounded(rng.standard_normal((tokens, 300)))
    x[tokens // 2, 17], x[tokens - 1, 299] = np.inf, np.nan
    w = weights_of(rng, 200, 300, 2)
    layer = tn.Fp8Linear([dev(v) for v in w], tokens)
    bad = np.zeros(tokens, dtype=bool)
    bad[[tokens // 2, tokens - 1]] = True
    y = host(layer(dev(x)))
    assert np.isnan(y[bad]).all() and np.isfinite(y[~bad]).all()
    codes = host(layer.gated(dev(x)).values())
    assert np.isnan(codes[bad]).all() and np.isfinite(codes[~bad]).all()


def test_scales_far_apart():
    """Blocks of one row and of one weight that differ by 2^40: their exponents are added by the instruction, not multiplied out."""
    rng = np.random.default_rng(11)
    x, w = rng.standard_normal((20, 512)), rng.standard_normal((256, 512))
    for b in range(4):
        x[:, b * 128:(b + 1) * 128] *= 2.0 ** (20 * b - 40)
        w[:, b * 128:(b + 1) * 128] *= 2.0 ** (40 - 20 * b)
    w[128:] *= 2.0 ** -60
    check_product(tn.Fp8Linear([dev(w)], 20)(dev(x)), eight(rounded(x)), eight(rounded(w), 128))


@pytest.mark.parametrize("tokens", [5, 50, 400])
def test_into_rows_of_a_wider_tensor(tokens):
    rng = np.random.default_rng(3)
    w = weights_of(rng, 133, 260, 1)
    layer, x = tn.Fp8Linear([dev(w[0])], tokens), dev(rng.standard_normal((tokens, 260)))
    y = torch.full((tokens, 401), 7.0, dtype=torch.bfloat16, device="cuda")
    got = layer(x, out=y[:, 5:138])
    assert torch.equal(y[:, 5:138], layer(x)) and got.data_ptr() == y[:, 5:].data_ptr()
    assert (y[:, :5] == 7).all() and (y[:, 138:] == 7).all()


def test_no_tokens():
    layer = tn.Fp8Linear([dev(np.ones((10, 20)))] * 2, 1)
    e = torch.empty((0, 20), dtype=torch.bfloat16, device="cuda")
    assert layer(e).shape == (0, 20) and layer.gated(e).codes.shape == (0, 128)


def test_more_tokens_than_the_handle_was_made_for():
    rng = np.random.default_rng(4)
    w, x = weights_of(rng, 256, 1024, 1), rng.standard_normal((700, 1024))
    check_product(tn.Fp8Linear([dev(w[0])], 1)(dev(x)), eight(rounded(x)), eight(w[0], 128))


def test_ranges_of_inputs_in_a_shared_workspace():
    """Sizes whose inputs are split (partial sums in the workspace): a block that two layers share, blocks too small for it, and the layer's own."""
    rng = np.random.default_rng(14)
    m, n, tokens = 300, 4000, 70
    w, x = weights_of(rng, m, n, 2), rounded(rng.standard_normal((tokens, n)))
    x8, w8 = eight(x), np.concatenate([eight(v, 128) for v in w])
    block = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    layers = [tn.Fp8Linear([dev(v) for v in w], tokens, workspace=s) for s in (block, block, block[:256], None)]
    assert layers[0].query(tn.TN_QUERY_WORKSPACE_BYTES) == 1 << 24 and layers[3].query(tn.TN_QUERY_WORKSPACE_BYTES) > 0
    gated = []
    for layer in layers:
        check_product(layer(dev(x)), x8, w8)
        gated.append(host(layer.gated(dev(x)).values()))
    for g in gated[1:]:                       # other orders of the sums: a code here and there is its neighbour
        assert (g != gated[0]).mean() < 1e-2
    with pytest.raises(ValueError):
        tn.Fp8Linear([dev(w[0])], 1, workspace=block.cpu())


def test_output_offsets_past_32_bits():
    rng = np.random.default_rng(5)
    tokens, m, n = (1 << 31) // 8200 + 300, 8200, 128
    w = weights_of(rng, m, n, 1)
    layer = tn.Fp8Linear([dev(w[0])], tokens)
    x = torch.ones((tokens, n), dtype=torch.bfloat16, device="cuda")
    last = dev(rng.standard_normal((5, n)))
    x[-5:] = last
    y = layer(x)
    assert y.numel() > 1 << 31
    check_product(y[-5:], eight(host(last)), eight(w[0], 128))
    assert torch.equal(y[:1].expand(4, m), y[tokens // 2:tokens // 2 + 4])


def test_on_a_stream_of_its_own_and_in_a_graph():
    rng = np.random.default_rng(6)
    w = weights_of(rng, 640, 1500, 2)
    layer, back = tn.Fp8Linear([dev(v) for v in w], 200), tn.Fp8Linear([dev(v) for v in w], 200, transpose=True)
    xs = [dev(rng.standard_normal((t, 1500))) for t in (1, 40, 200)]
    dys = [dev(rng.standard_normal((t, 1280))) for t in (1, 40, 200)]

    def work():
        return [o for x in xs for o in (layer(x), layer.gated(x).codes.view(torch.uint8))] + [back(d) for d in dys]
    ref = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = work()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(4):
        for t in xs + dys:
            t.copy_(torch.roll(t, 1, 1))
        eager = [t.clone() for t in work()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i


def test_binding_refuses():
    w = dev(np.ones((10, 20)))
    layer, one = tn.Fp8Linear([w, w], 4), tn.Fp8Linear([w], 4)
    back = tn.Fp8Linear([w, w], 4, transpose=True)
    x = dev(np.ones((2, 20)))
    q = tn.quantize_fp8(w)
    scales = torch.zeros((1, 1), dtype=torch.float8_e8m0fnu, device="cuda")
    bad = [lambda: tn.Fp8Linear([], 1), lambda: tn.Fp8Linear([w, w, w], 1), lambda: tn.Fp8Linear([w, w.float()], 1), lambda: tn.Fp8Linear([w.half()], 1),
           lambda: tn.Fp8Linear([w.t()], 1), lambda: tn.Fp8Linear([w.cpu()], 1), lambda: tn.Fp8Linear([w], 1, scales=[scales]),
           lambda: tn.Fp8Linear([q.values()], 1), lambda: tn.Fp8Linear([q.values().contiguous()], 1, scales=[scales[:, :0]]),
           lambda: layer(dev(np.ones((2, 21)))), lambda: layer(x.half()), lambda: layer(tn.quantize_fp8(dev(np.ones((2, 21))))),
           lambda: layer(tn.quantize_fp8(x, 2)), lambda: back(tn.quantize_fp8(x)), lambda: layer(x, out=torch.empty(2, 20, device="cuda")),
           lambda: layer(x, out=torch.empty(3, 20, dtype=torch.bfloat16, device="cuda")), lambda: one.gated(x), lambda: back.gated(x),
           lambda: layer.gated(x, out=tn.Fp8Rows.empty(2, 11))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(tn.TNLinearError):
        tn.Fp8Linear([w], 0)
    with pytest.raises(tn.TNLinearError):
        layer.quantized_tensor(2)
    with pytest.raises(tn.TNLinearError):
        layer.query(999)


def test_binding_refuses_another_gpu(monkeypatch):
    """A layer is used on the GPU that it lives on, with tensors there."""
    w, x = dev(np.ones((128, 256))), dev(np.ones((2, 256)))
    elsewhere = lambda shape, dtype: on_gpu(torch.empty(shape, dtype=dtype, device="cuda"), 1)      # noqa: E731
    far, far_w, far_y = (elsewhere(s, torch.bfloat16) for s in ((2, 256), (128, 256), (2, 256)))
    far8 = tn.Fp8Rows(elsewhere((2, 256), torch.float8_e4m3fn), elsewhere((2, 4), torch.float8_e8m0fnu), 256)
    out8 = tn.Fp8Rows(elsewhere((2, 128), torch.float8_e4m3fn), elsewhere((2, 4), torch.float8_e8m0fnu), 128)
    block = elsewhere((1 << 20,), torch.uint8)
    far_codes, far_scales = elsewhere((128, 256), torch.float8_e4m3fn), elsewhere((1, 2), torch.float8_e8m0fnu)
    layer = tn.Fp8Linear([w, w], 4)
    codes, scales = layer.quantized_tensor(0)
    for call in (lambda: tn.Fp8Linear([far_w], 4), lambda: tn.Fp8Linear([w, far_w], 4), lambda: tn.Fp8Linear([w], 4, workspace=block),
                 lambda: tn.Fp8Linear([codes], 4, scales=[far_scales]), lambda: tn.Fp8Linear([far_codes], 4, scales=[scales]),
                 lambda: layer(far), lambda: layer(far8), lambda: layer(x, out=far_y), lambda: layer.gated(far8), lambda: layer.gated(x, out=out8)):
        with pytest.raises(ValueError):
            call()
    rows = tn.quantize_fp8(x)
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 1)
    for call in (lambda: layer(rows), lambda: layer.gated(rows), lambda: layer.quantized_tensor(0), lambda: layer(x), lambda: tn.Fp8Linear([w], 4)):
        with pytest.raises(ValueError):
            call()
    monkeypatch.undo()
    assert torch.equal(layer(rows), layer(x))


def test_gated_refuses_its_input_as_output():
    """Square weights: the rows of input and output have one size, and other workgroups still read the input when one writes."""
    w = dev(np.eye(256))
    layer, rows = tn.Fp8Linear([w, w], 40), tn.quantize_fp8(dev(np.ones((80, 256))))
    part = lambda a, b: tn.Fp8Rows(rows.codes[a:b], rows.scales[a:b], 256)      # noqa: E731
    before = rows.codes.view(torch.uint8).clone()
    for x, out in ((rows, rows), (part(0, 40), part(39, 79)), (part(20, 60), part(0, 40))):
        with pytest.raises(tn.TNLinearError):
            layer.gated(x, out=out)
    assert torch.equal(rows.codes.view(torch.uint8), before)
    want = layer.gated(part(0, 40))
    got = layer.gated(part(0, 40), out=part(40, 80))                  # beside each other is no overlap
    assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(got.scales.view(torch.uint8), want.scales.view(torch.uint8))


def exact_rows(codes, scales, rows=1):
    """Codes and scales in 64 bits, on the GPU."""
    n, k = codes.shape
    scale = scales.contiguous().view(torch.uint8).double().sub(127).exp2()
    return codes.double() * scale.repeat_interleave(rows, 0)[:n].repeat_interleave(128, 1)[:, :k]


def sums_off_gpu(x8, w8):
    pad = -x8.shape[1] % 8
    most = lambda v: torch.nn.functional.pad(v.abs(), (0, pad)).reshape(v.shape[0], -1, 8).amax(dim=2)      # noqa: E731
    return (7 * 2.0 ** -13 + 2.0 ** -18) * (most(x8) @ most(w8).t().contiguous())


@pytest.mark.parametrize("gated,m,n,tokens", FORM_CASES)
def test_every_form(gated, m, n, tokens):
    """Each kernel a product may take, at sizes that choose it, against 64 bits on the layer's own codes."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + n + tokens)
    weights = [(torch.randn((m, n), generator=gen, device="cuda") / n ** 0.5).bfloat16() for _ in range(1 + gated)]
    layer = tn.Fp8Linear(weights, tokens)
    rows = tn.quantize_fp8(torch.randn((tokens, n), generator=gen, device="cuda").bfloat16())
    x8, w8 = exact_rows(rows.values(), rows.block_scales()), [exact_rows(*layer.quantized_tensor(i), 128) for i in range(1 + gated)]
    sums, off = [x8 @ w.t() for w in w8], [sums_off_gpu(x8, w) for w in w8]
    if not gated:
        y = layer(rows).double()
        unit = torch.exp2(torch.floor(torch.log2(sums[0].abs().clamp(min=2.0 ** -120))) - 8)          # half a unit in bf16's last place
        err = (y - sums[0]).abs()
        assert (err <= 2 * unit + off[0]).all()                                                       # (twice: ref and y may differ in their powers of two)
        assert err.norm() <= 2.0 ** -8 * sums[0].norm()
        assert torch.equal(layer(rows).double(), y)
        return
    got = layer.gated(rows)
    check_padding(got)
    (gate, up), (eg, eu) = sums, off
    sig = torch.sigmoid(gate)
    ref = gate * sig * up
    off = 1.1 * up.abs() * eg + (gate * sig).abs() * eu + 1.1 * eg * eu + 2.0 ** -20 * ref.abs()
    values = exact_rows(got.values(), got.block_scales())
    scale = got.block_scales().contiguous().view(torch.uint8).double().sub(127).exp2()
    wide = scale.repeat_interleave(128, 1)[:, :m]
    assert ((values - ref).abs() <= 2.0 ** -4 * (ref.abs() + off) + 2.0 ** -10 * wide + off).all()
    pad = -m % 128
    most = torch.nn.functional.pad(ref.abs(), (0, pad)).reshape(tokens, -1, 128).amax(dim=2)
    slack = torch.nn.functional.pad(off, (0, pad)).reshape(tokens, -1, 128).amax(dim=2)
    assert ((most - slack) <= 448 * scale).all() and ((most + slack) > 224 * scale).all()
    assert (values - ref).norm() <= 2.0 ** -4 * ref.norm()
    again = layer.gated(rows)
    assert torch.equal(again.codes.view(torch.uint8), got.codes.view(torch.uint8)) and torch.equal(again.scales.view(torch.uint8), got.scales.view(torch.uint8))
