"""Norm, silu(gate) * up, their gradients and quantisation against the 64-bit oracle, at the sizes and values where they can go wrong."""
import numpy as np
import pytest
import torch

import oracle.fp8_oracle as Q
import paper_2602_01613_amd as tn
from fp8_util import check_eight_bit, check_padding, dev, exponents, half_unit, host, rounded

pytestmark = pytest.mark.gpu

EPS = 1e-6
# one token to many, widths below and above a block, a wave's chunks, and each form of the kernels
SIZES = [(1, 1), (3, 7), (1, 128), (2, 129), (5, 512), (4, 513), (9, 1001), (2, 2048), (3, 2056), (1, 5120), (7, 5120), (2, 6144), (2, 8191), (2, 8192),
         (2, 9000), (1, 16384)]


def close(got, ref, dtype, extra):
    """One rounding to the type, and `extra` (64 bits, or a number) of fp32 arithmetic."""
    err = np.abs(got - ref)
    bound = half_unit(ref, dtype) + extra
    assert np.isfinite(got).all() and (err <= bound).all(), (err - bound).max()


def rng_of(*key):
    return np.random.default_rng(sum((i + 1) * 7919 * int(k) for i, k in enumerate(key)) % (1 << 32))


def activations(rng, rows, cols, size=1.0):
    v = rng.standard_normal((rows, cols)) * size
    v[:, rng.integers(0, cols, max(1, cols // 300))] *= 30
    return v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rms_norm(rows, cols, dtype):
    rng = rng_of(rows, cols, 1)
    x, res = rounded(activations(rng, rows, cols), dtype), rounded(activations(rng, rows, cols, 3.0), dtype)
    w = rounded(1 + 0.2 * rng.standard_normal(cols), dtype)
    got = tn.rms_norm(dev(x, dtype), dev(w, dtype), EPS, residual=dev(res, dtype), outputs="both")
    s = rounded(x + res, dtype)
    assert np.array_equal(host(got.sum), s)
    ref = Q.rms_norm(s, w, EPS)
    # fp32: a sum of `cols` squares over lanes (errors of each sign average; 2^-21 holds for any order here), a square root, two products
    close(host(got.y), ref, dtype, 2.0 ** -20 * np.abs(ref))
    check_eight_bit(got.fp8, ref)
    check_padding(got.fp8)
    # the outputs do not depend on which others are asked for
    only8, only = tn.rms_norm(dev(x, dtype), dev(w, dtype), EPS, residual=dev(res, dtype), outputs="fp8"), tn.rms_norm(got.sum, dev(w, dtype), EPS)
    assert torch.equal(only8.fp8.codes.view(torch.uint8), got.fp8.codes.view(torch.uint8)) and only8.y is None
    assert torch.equal(only.y, got.y) and only.sum is None and only.fp8 is None


def test_rms_norm_without_weight_strided_and_in_place():
    rng = rng_of(5)
    wide = rounded(activations(rng, 6, 3 * 700))
    x, res = dev(wide)[:, 700:1400], dev(wide)[:, 1400:]
    s = rounded(wide[:, 700:1400] + wide[:, 1400:])
    ref = Q.rms_norm(s, None, EPS)
    y = torch.full((6, 900), 7.0, dtype=torch.bfloat16, device="cuda")
    got = tn.rms_norm(x, None, EPS, residual=res, out=tn.RowOutput(y[:, :700], None, res))
    assert got.sum is res and np.array_equal(host(res), s)
    close(host(y[:, :700]), ref, "bf16", 2.0 ** -20 * np.abs(ref))
    assert (y[:, 700:] == 7).all()
    z = dev(s)
    tn.rms_norm(z, None, EPS, out=tn.RowOutput(z, None))
    assert torch.equal(z, y[:, :700])


@pytest.mark.parametrize("rows,cols", [(6, 300), (5, 700), (3, 9000)])
def test_rms_norm_in_place_of_both_inputs(rows, cols):
    """sum and y where x and residual were, either way round; one tensor for both is refused."""
    rng = rng_of(rows, cols, 13)
    x, res, w = (dev(v) for v in (activations(rng, rows, cols), activations(rng, rows, cols), 1 + 0.2 * rng.standard_normal(cols)))
    ref = tn.rms_norm(x, w, EPS, residual=res, outputs="both")
    for swap in (False, True):
        x2, res2 = x.clone(), res.clone()
        y, total = (res2, x2) if swap else (x2, res2)
        got = tn.rms_norm(x2, w, EPS, residual=res2, outputs="both", out=tn.RowOutput(y, None, total))
        assert got.y is y and got.sum is total and torch.equal(y, ref.y) and torch.equal(total, ref.sum)
        assert torch.equal(got.fp8.codes.view(torch.uint8), ref.fp8.codes.view(torch.uint8))
    before = x.clone()
    with pytest.raises(tn.TNLinearError):
        tn.rms_norm(x, w, EPS, residual=res, out=tn.RowOutput(x, None, x))
    assert torch.equal(x, before)


def test_rms_norm_rows_of_zeros_and_of_what_is_not_finite():
    x = np.zeros((5, 300))
    x[1, 7], x[2, 7], x[3] = np.inf, np.nan, 1e-30
    x[4, :128] = 3.0
    got = tn.rms_norm(dev(x, "f32"), None, EPS, outputs="both")
    y, codes, exps = host(got.y), host(got.fp8.values()), exponents(got.fp8.block_scales())
    assert not y[0].any() and not codes[0].any() and (exps[0] == -127).all()
    assert not y[1, :7].any() and np.isnan(y[1, 7]) and np.isnan(codes[1, 7]) and not codes[1, :7].any()      # 0 / inf, inf / inf
    assert np.isnan(y[2]).all() and np.isnan(codes[2]).all()
    np.testing.assert_allclose(y[3], 1e-27, rtol=1e-6)                                                          # eps alone
    assert (exps[4] == [Q.block_exponent(y[4, 0]), -127, -127]).all() and not codes[4, 128:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES + [(600, 40), (1100, 129), (2000, 1)])
def test_rms_norm_gradients(rows, cols, dtype):
    rng = rng_of(rows, cols, 2)
    s, dy, ds = (rounded(v, dtype) for v in (activations(rng, rows, cols), rng.standard_normal((rows, cols)) * 1e-3, rng.standard_normal((rows, cols)) * 1e-3))
    w = rounded(1 + 0.2 * rng.standard_normal(cols), dtype)
    dx, dw = tn.rms_norm_gradients(dev(dy, dtype), dev(s, dtype), dev(w, dtype), EPS, dsum=dev(ds, dtype))
    ref, ref_dw = Q.rms_norm_gradients(dy, s, w, EPS, ds)
    r = 1 / np.sqrt((s * s).mean(axis=1, keepdims=True) + EPS)
    u, g = s * r, dy * w
    # fp32: the mean of g * u is off by 2^-20 of the mean of |g * u| at most; each term by a few roundings of its own size
    extra = 2.0 ** -20 * (r * np.abs(g) + r * np.abs(u) * np.abs(g * u).mean(axis=1, keepdims=True) + np.abs(ds))
    close(host(dx), ref, dtype, extra)
    assert dw.dtype == torch.float32
    close(host(dw), ref_dw, "f32", 2.0 ** -20 * np.abs(dy * u).sum(axis=0))
    # alone, and into a given tensor
    alone, none = tn.rms_norm_gradients(dev(dy, dtype), dev(s, dtype), dev(w, dtype), EPS, dweight=False)
    close(host(alone), ref - ds, dtype, extra)
    assert none is None
    mine = dev(ds, dtype)
    again, dw2 = tn.rms_norm_gradients(dev(dy, dtype), dev(s, dtype), dev(w, dtype), EPS, dsum=mine, dx=mine)
    assert again is mine and torch.equal(mine, dx) and torch.equal(dw, dw2)


def test_rms_norm_gradients_against_differences():
    """Central differences of the kernel's own fp32 forward, along random directions."""
    rng = rng_of(77)
    rows, cols = 4, 333
    x, w, dy = rng.standard_normal((rows, cols)), 1 + 0.2 * rng.standard_normal(cols), rng.standard_normal((rows, cols))
    dx, dw = tn.rms_norm_gradients(dev(dy, "f32"), dev(x, "f32"), dev(w, "f32"), EPS)
    loss = lambda x_, w_: (host(tn.rms_norm(dev(x_, "f32"), dev(w_, "f32"), EPS).y) * rounded(dy, "f32")).sum()      # noqa: E731
    step = 1e-2                                # error of the difference: step^2 and 2^-24 * |loss terms| / step, each under 1e-3 of the slopes' size
    for _ in range(4):
        vx, vw = rng.standard_normal((rows, cols)), rng.standard_normal(cols)
        slope = (host(dx) * vx).sum()
        assert abs((loss(x + step * vx, w) - loss(x - step * vx, w)) / (2 * step) - slope) < 2e-3 * np.linalg.norm(host(dx)) * np.linalg.norm(vx)
        slope = (host(dw) * vw).sum()
        assert abs((loss(x, w + step * vw) - loss(x, w - step * vw)) / (2 * step) - slope) < 2e-3 * np.linalg.norm(host(dw)) * np.linalg.norm(vw)


def test_gradients_of_no_rows():
    e = torch.empty((0, 70), dtype=torch.bfloat16, device="cuda")
    dx, dw = tn.rms_norm_gradients(e, e, dev(np.ones(70)), EPS)
    assert dx.shape == (0, 70) and not dw.any()
    assert tn.rms_norm(e, None, EPS, residual=e, outputs="both").fp8.codes.shape == (0, 128)
    assert tn.silu_gate(e, "both").y.shape == (0, 35) and tn.silu_gate_gradients(e, e[:, :35], "both").fp8.codes.shape == (0, 256)
    assert tn.quantize_fp8(e, 2).scales.shape == (0, 4)


GATE_SIZES = [(1, 1), (3, 7), (2, 128), (5, 129), (17, 500), (40, 1001), (3, 25600)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", GATE_SIZES)
def test_silu_gate_and_gradients(rows, cols, dtype):
    rng = rng_of(rows, cols, 3)
    gate_up = rounded(rng.standard_normal((rows, 2 * cols)) * 3, dtype)
    gate, up, dh = gate_up[:, :cols], gate_up[:, cols:], rounded(rng.standard_normal((rows, cols)) * 1e-3, dtype)
    got = tn.silu_gate(dev(gate_up, dtype), "both")
    ref = Q.silu_gate(gate, up)
    close(host(got.y), ref, dtype, 2.0 ** -20 * np.abs(ref))
    check_eight_bit(got.fp8, ref)
    check_padding(got.fp8)
    grads = tn.silu_gate_gradients(dev(gate_up, dtype), dev(dh, dtype), "both")
    dg, du = Q.silu_gate_gradients(gate, up, dh)
    # 1 + gate * (1 - sig) crosses zero near gate = -1.28: the error there is that of its terms, up to 1 + |gate|, times dh * up * sig
    sig = 1 / (1 + np.exp(-gate))
    extra = 2.0 ** -20 * np.abs(dh * up * sig) * (1 + np.abs(gate))
    close(host(grads.y[:, :cols]), dg, dtype, extra)
    close(host(grads.y[:, cols:]), du, dtype, 2.0 ** -20 * np.abs(du))
    codes, exps = host(grads.fp8.values(0)), exponents(grads.fp8.block_scales(0))
    scale = np.repeat(np.exp2(exps.astype(np.float64)), 128, axis=1)[:, :cols]
    assert (np.abs(Q.dequantize(codes, exps) - dg) <= 2.0 ** -4 * np.abs(dg) + 2.0 ** -10 * scale + 1.1 * extra).all()
    check_eight_bit(grads.fp8, du, segment=1)
    check_padding(grads.fp8)
    mine = dev(gate_up, dtype)
    tn.silu_gate_gradients(mine, dev(dh, dtype), out=tn.RowOutput(mine, None))
    assert torch.equal(mine, grads.y)


def test_silu_gate_at_the_ends():
    gate = np.array([[0.0, -200.0, 200.0, -88.5, -1e30, 1e30, np.inf, -np.inf, np.nan, 1.0]])
    up = np.array([[2.0, 3.0, 2.0, 1.0, 2.0, 1e-30, 1.0, 1.0, 1.0, np.inf]])
    both = dev(np.concatenate([gate, up], axis=1), "f32")
    got = tn.silu_gate(both, "both")
    y = host(got.y)[0]
    assert y[0] == 0 and y[1] == 0 and y[2] == 400 and y[4] == 0 and abs(y[3]) < 1e-35
    np.testing.assert_allclose(y[5], 1.0, rtol=1e-6)
    assert y[6] == np.inf and np.isnan(y[7]) and np.isnan(y[8]) and y[9] == np.inf
    codes = host(got.fp8.values())[0]
    assert np.isnan(codes[6:]).all() and np.isfinite(codes[:6]).all()
    assert exponents(got.fp8.block_scales())[0, 0] == Q.block_exponent(400.0)
    g = host(tn.silu_gate_gradients(both, dev(np.ones((1, 10)), "f32")).y)[0]
    assert g[0] == 1.0 and abs(g[1]) < 1e-30 and g[2] == 2.0 and g[4] == 0 and np.isnan(g[8])


def gates_everywhere(dtype):
    """Every bf16 value within +-128 and, in fp32, dense runs of values where exp(-gate) leaves fp32's range and between: [rows, 1000]."""
    bits = torch.arange(0x4300 + 1, dtype=torch.int32)                         # 0 .. 128
    v = (bits << 16).view(torch.float32).double().numpy()
    v = np.concatenate([v, -v])
    if dtype == "f32":
        v = np.concatenate([v, np.linspace(-105, -80, 20001), np.linspace(80, 105, 4001), np.linspace(-128, 128, 8001)])
    return np.resize(rounded(v, dtype), (-(-v.size // 1000), 1000))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_silu_gate_and_gradients_of_every_gate(dtype):
    """Finite for finite gates, and within what fp32 and one rounding take off: 2^-20 of each term as above, and 1 / (1 + exp(-gate)) itself to
    2^-126, the least that a reciprocal that drops subnormal results has to be off by."""
    gate = gates_everywhere(dtype)
    rng = rng_of(12)
    up, dh = (rounded(v, dtype) for v in (rng.standard_normal(gate.shape), rng.standard_normal(gate.shape)))
    both = np.concatenate([gate, up], axis=1)
    got, grads = tn.silu_gate(dev(both, dtype), "both"), tn.silu_gate_gradients(dev(both, dtype), dev(dh, dtype), "both")
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-gate))
    off = 2.0 ** -20 * sig + 2.0 ** -126
    slack = 2.0 ** -126                                                        # of a result so small itself
    ref, (dg, du) = Q.silu_gate(gate, up), Q.silu_gate_gradients(gate, up, dh)
    close(host(got.y), ref, dtype, off * np.abs(gate * up) + slack)
    close(host(grads.y[:, :1000]), dg, dtype, off * np.abs(dh * up) * (1 + np.abs(gate)) + slack)
    close(host(grads.y[:, 1000:]), du, dtype, off * np.abs(dh * gate) + slack)
    # 8 bits: of the values in fp32, bit for bit, whatever the inputs' type
    wide, wide_grads = tn.silu_gate(dev(both, "f32"), "both"), tn.silu_gate_gradients(dev(both, "f32"), dev(dh, "f32"), "both")
    for rows8, twin, segment, values in ((got.fp8, wide.fp8, 0, wide.y), (grads.fp8, wide_grads.fp8, 0, wide_grads.y[:, :1000]),
                                         (grads.fp8, wide_grads.fp8, 1, wide_grads.y[:, 1000:])):
        codes, exps = Q.quantize(host(values))
        for r in (rows8, twin):
            assert np.array_equal(host(r.values(segment)), codes) and np.array_equal(exponents(r.block_scales(segment)), exps)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,segments", [(1, 1, 1), (3, 127, 1), (2, 128, 2), (5, 129, 2), (4, 1001, 3), (70, 640, 1), (2, 25600, 2)])
def test_quantize(rows, cols, segments, dtype):
    """Given values: codes and scales are the format's, bit for bit; sizes from fp32's least to its largest."""
    rng = rng_of(rows, cols, segments, 4)
    x = rounded(rng.standard_normal((rows, cols * segments)) * np.exp2(rng.integers(-40, 40, (rows, cols * segments)) / 4), dtype)
    x[rng.random(x.shape) < 0.02] = 0
    if cols > 300:
        x[0, 0], x[0, 200], x[rows - 1, 5] = np.inf, -np.inf, np.nan
        x[-1, 256:300] *= 2.0 ** -130
        x[-1] = rounded(x[-1], dtype)
    got = tn.quantize_fp8(dev(x, dtype), segments)
    check_padding(got)
    for i in range(segments):
        codes, exps = Q.quantize(x[:, i * cols:(i + 1) * cols])
        assert np.array_equal(exponents(got.block_scales(i)), exps)
        mine = host(got.values(i))
        assert np.array_equal(np.isnan(mine), np.isnan(codes)) and np.array_equal(np.nan_to_num(mine), np.nan_to_num(codes))


def test_quantize_at_the_steps_of_the_scale():
    """Largest magnitudes at, just below and just above 448 * 2^e, subnormal blocks, the largest fp32, ties between codes."""
    tops = []
    for e in (-120, -10, 0, 100):
        top = np.float32(448.0 * 2.0 ** e)
        tops += [top, np.nextafter(top, np.float32(0)), np.nextafter(top, np.float32(np.inf))]
    tops += [np.float32(3.4028234e38), np.float32(1e-45), np.float32(1e-39), np.float32(2.0 ** -126)]
    x = np.zeros((len(tops), 128), dtype=np.float32)
    for i, t in enumerate(tops):
        x[i] = t * (1 - np.arange(128, dtype=np.float32) / 128)
        x[i, ::3] *= -1
    codes, exps = Q.quantize(x.astype(np.float64))
    got = tn.quantize_fp8(torch.from_numpy(x).cuda())
    assert np.array_equal(exponents(got.block_scales()), exps) and np.array_equal(host(got.values()), codes)


def test_offsets_past_32_bits():
    rows, cols = (1 << 31) // 8192 + 9, 8192
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x.fill_(1.0)
    last = dev(rng_of(8).standard_normal((4, cols)))
    x[-4:] = last
    small = tn.rms_norm(last, None, EPS, outputs="both")
    got = tn.rms_norm(x, None, EPS, outputs="both")
    assert torch.equal(got.y[-4:], small.y) and torch.equal(got.fp8.codes[-4:].view(torch.uint8), small.fp8.codes.view(torch.uint8))
    assert torch.equal(got.fp8.scales[-4:].view(torch.uint8), small.fp8.scales.view(torch.uint8))
    del got
    q = tn.quantize_fp8(x)
    assert torch.equal(q.codes[-4:].view(torch.uint8), tn.quantize_fp8(last).codes.view(torch.uint8))
    del q
    h = tn.silu_gate(x, "y").y
    assert torch.equal(h[-4:], tn.silu_gate(last, "y").y)


def test_more_rows_than_one_launch_takes():
    """2^32 threads and more in a launch are refused by the runtime, so long inputs go in runs of rows. Rows repeat here with a prime period:
    each has the bits that a short call gives it."""
    period = 4099

    def repeats(small, rows, make):
        x = small.repeat(-(-rows // period), 1)[:rows]
        got, want = make(x), make(small)
        del x
        for g, w in zip(got, want):
            g, w = g.view(torch.uint8), w.view(torch.uint8)
            whole = rows // period * period
            assert g.shape[0] == rows and torch.equal(g[whole:], w[:rows - whole])
            g = g[:whole].view(-1, *w.shape)
            for at in range(0, g.shape[0], 4096):
                assert bool((g[at:at + 4096] == w).all())

    def norm(x):
        n = tn.rms_norm(x, None, EPS, residual=x, outputs="both")
        return n.y, n.sum, n.fp8.codes, n.fp8.scales

    def quantised(x):
        q = tn.quantize_fp8(x)
        return q.codes, q.scales

    small = dev(rng_of(10).standard_normal((period, 8)))
    repeats(small, (1 << 21) + 5, norm)                                            # the norm's runs have 2^21 rows
    repeats(small, (1 << 26) + 5, lambda x: (tn.rms_norm(x, None, EPS).y,))        # a wave to a row: 2^32 threads
    rows = (1 << 28) + 5                                                            # 16 lanes to a row: 2^32 threads
    repeats(small[:, :2].contiguous(), rows, lambda x: (tn.silu_gate(x, "y").y,))
    repeats(small[:, :2].contiguous(), rows, lambda x: (tn.silu_gate_gradients(x, x[:, 1:], "y").y,))
    repeats(small[:, :1].contiguous(), (1 << 27) + 5, quantised)                   # two runs, with codes


def test_on_a_stream_of_its_own_and_in_a_graph():
    rng = rng_of(9)
    x, res, w = dev(activations(rng, 33, 1500)), dev(activations(rng, 33, 1500)), dev(np.ones(1500))
    dy = dev(rng.standard_normal((33, 1500)))

    def work():
        n = tn.rms_norm(x, w, EPS, residual=res, outputs="both")
        dx, dw = tn.rms_norm_gradients(dy, n.sum, w, EPS)
        g = tn.silu_gate_gradients(x, dy[:, :750], "both")
        return [n.y, n.sum, n.fp8.codes.view(torch.uint8), n.fp8.scales.view(torch.uint8), dx, dw, g.y, g.fp8.codes.view(torch.uint8),
                tn.silu_gate(x, "both").fp8.codes.view(torch.uint8), tn.quantize_fp8(x).codes.view(torch.uint8)]
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
        x.copy_(torch.roll(x, 1, 0))
        eager = [t.clone() for t in work()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i


def test_binding_refuses():
    x, w = dev(np.ones((4, 256))), dev(np.ones(256))
    bad = [lambda: tn.rms_norm(x.half(), None), lambda: tn.rms_norm(x[0], None), lambda: tn.rms_norm(x, w[:255]), lambda: tn.rms_norm(x, w.float()),
           lambda: tn.rms_norm(x, w, residual=x[:3]), lambda: tn.rms_norm(x, w, residual=x.float()), lambda: tn.rms_norm(x.t(), None),
           lambda: tn.rms_norm(x[:1].expand(4, 256), w), lambda: tn.rms_norm(x, w, outputs="all"),
           lambda: tn.rms_norm(x, w, outputs="fp8", out=tn.RowOutput(None, tn.Fp8Rows.empty(4, 255))),
           lambda: tn.rms_norm(x, w, out=tn.RowOutput(x.float(), None)),
           lambda: tn.rms_norm_gradients(x[:, :255], x, w), lambda: tn.rms_norm_gradients(x, x, w, dsum=x[:2]), lambda: tn.rms_norm_gradients(x, x, w, dx=x.float()),
           lambda: tn.silu_gate(x[:, :255]), lambda: tn.silu_gate_gradients(x, x), lambda: tn.quantize_fp8(x, 3), lambda: tn.quantize_fp8(x, 0),
           lambda: tn.quantize_fp8(x, out=tn.Fp8Rows.empty(4, 128)), lambda: tn.quantize_fp8(x.t())]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: tn.rms_norm(x, w, eps=-1.0), lambda: tn.rms_norm(dev(np.ones((1, 16385))), None)):
        with pytest.raises(tn.TNLinearError):
            call()
