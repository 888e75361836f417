"""Operators around 8-bit projections, what needs no GPU: the oracle's own pins, the C ABI's refusals and layout, the binding's checks."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle.fp8_oracle as Q
import paper_2602_01613_amd as tn
from paper_2602_01613_amd import fp8

HERE = os.path.dirname(os.path.abspath(__file__))
INVALID, UNSUPPORTED = -1, -2


def test_e4m3_rounding_is_the_formats():
    """Against a search over all codes, decoded from their bit fields; ties to the even code."""
    table = {}
    for c in range(0x7f):
        e, m = c >> 3, c & 7
        table[c] = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
    codes, values = np.array(list(table)), np.array(list(table.values()))
    assert values.max() == Q.E4M3_MAX
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(0, 448, 2000), np.exp2(rng.uniform(-12, 8.8, 4000)), values, (values[1:] + values[:-1]) / 2])
    d = np.abs(v[:, None] - values[None, :])
    best = d.min(axis=1, keepdims=True)
    pick = np.where(d == best, (codes & 1)[None, :] * 1000 + codes[None, :], 10 ** 6).argmin(axis=1)
    assert np.array_equal(Q.e4m3_round(v), values[pick])
    assert np.array_equal(Q.e4m3_round(-v), -values[pick])
    t = torch.from_numpy(v).to(torch.float32).to(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(Q.e4m3_round(v.astype(np.float32)), t)


def test_block_exponent_is_the_least_that_holds():
    rng = np.random.default_rng(1)
    a = np.concatenate([np.exp2(rng.uniform(-110, 120, 3000)), 448 * np.exp2(np.arange(-100, 100.0)), np.nextafter(448, 500) * np.exp2(np.arange(-100, 100.0))])
    e = Q.block_exponent(a).astype(np.float64)
    assert (a <= 448 * np.exp2(e)).all() and (a > 448 * np.exp2(e - 1)).all()
    assert Q.block_exponent(np.array([0.0, 2.0 ** -126, 2.0 ** -149])).tolist() == [-127, -127, -127]


def test_gradient_formulas_against_differences():
    rng = np.random.default_rng(2)
    s, dy, w = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    dx, dw = Q.rms_norm_gradients(dy, s, w, 1e-3)
    f = lambda s_, w_: (dy * Q.rms_norm(s_, w_, 1e-3)).sum()      # noqa: E731
    step = 1e-6
    for i in range(3):
        for j in range(7):
            d = np.zeros((3, 7))
            d[i, j] = step
            assert abs((f(s + d, w) - f(s - d, w)) / (2 * step) - dx[i, j]) < 1e-7
    for j in range(7):
        d = np.zeros(7)
        d[j] = step
        assert abs((f(s, w + d) - f(s, w - d)) / (2 * step) - dw[j]) < 1e-7
    gate, up, dh = rng.standard_normal((3, 5)) * 3, rng.standard_normal((3, 5)), rng.standard_normal((3, 5))
    dg, du = Q.silu_gate_gradients(gate, up, dh)
    num_g = dh * (Q.silu_gate(gate + step, up) - Q.silu_gate(gate - step, up)) / (2 * step)
    num_u = dh * (Q.silu_gate(gate, up + step) - Q.silu_gate(gate, up - step)) / (2 * step)
    assert np.abs(num_g - dg).max() < 1e-7 and np.abs(num_u - du).max() < 1e-7


def test_header_declares_what_the_binding_exports():
    text = open(os.path.join(os.path.dirname(HERE), "include", "tn_fp8.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(tn_(?:fp8|rms|silu)_[a-z_0-9]+)\s*\(", text))
    assert declared == set(tn.FP8_EXPORTED_SYMBOLS)
    lib = tn.load_library()
    for name in declared:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("cols,segments,codes,scales", [(1, 1, 128, 4), (128, 1, 128, 4), (129, 1, 256, 4), (5120, 1, 5120, 40),
                                                        (25600, 2, 51200, 400), (1001, 2, 2048, 16), (600, 3, 1920, 16)])
def test_row_strides(cols, segments, codes, scales):
    a, b = ctypes.c_int64(0), ctypes.c_int64(0)
    assert fp8._library().tn_fp8_row_strides(cols, segments, ctypes.byref(a), ctypes.byref(b)) == 0
    assert (a.value, b.value) == (codes, scales)
    assert fp8._library().tn_fp8_row_strides(cols, segments, None, None) == 0


def test_row_strides_refusals():
    f = fp8._library().tn_fp8_row_strides
    assert f(0, 1, None, None) == INVALID and f(5, 0, None, None) == INVALID
    assert f(1 << 40, 1, None, None) == UNSUPPORTED and f(5, 1 << 20, None, None) == UNSUPPORTED


# A valid call of each row operator with addresses that are never reached: every entry of `bad` makes it wrong
A = 1 << 20
ROW_CALLS = {
    "tn_fp8_quantize": (dict(dtype=1, rows=2, cols=10, segments=1, x=A, x_stride=10, codes=A, scales=A, stream=None),
                        [("dtype", 2), ("dtype", -1), ("rows", -1), ("cols", 0), ("segments", 0), ("x", None), ("x_stride", 9), ("x", A + 1),
                         ("codes", None), ("scales", None), ("codes", A + 8), ("scales", A + 2)]),
    "tn_rms_norm": (dict(dtype=1, rows=2, cols=10, x=A, x_stride=10, residual=A, residual_stride=10, weight=A, eps=1e-6, sum=A, sum_stride=10,
                         y=A, y_stride=10, codes=A, scales=A, stream=None),
                    [("dtype", 2), ("rows", -1), ("cols", 0), ("x", None), ("x", A + 1), ("x_stride", 9), ("residual_stride", 9), ("residual", A + 1),
                     ("weight", A + 1), ("eps", -1.0), ("eps", float("nan")), ("sum_stride", 9), ("sum", A + 1), ("y_stride", 9), ("y", A + 1),
                     ("codes", None), ("scales", None), ("codes", A + 4), ("scales", A + 1)]),
    "tn_rms_norm_gradients": (dict(dtype=0, rows=2, cols=10, dy=A, dy_stride=10, s=A, s_stride=10, weight=A, eps=1e-6, dsum=A, dsum_stride=10,
                                   dx=A, dx_stride=10, dweight=A, workspace=A, workspace_bytes=1 << 30, stream=None),
                              [("dtype", 3), ("rows", -1), ("cols", 0), ("dy", None), ("s", None), ("dx", None), ("dy_stride", 9), ("s_stride", 9),
                               ("dsum_stride", 9), ("dx_stride", 9), ("dy", A + 2), ("s", A + 2), ("dx", A + 2), ("dsum", A + 2), ("weight", A + 2),
                               ("dweight", A + 2), ("workspace", None), ("workspace", A + 8), ("workspace_bytes", 79), ("eps", -1.0)]),
    "tn_silu_gate": (dict(dtype=1, rows=2, cols=10, gate_up=A, gate_up_stride=20, y=A, y_stride=10, codes=A, scales=A, stream=None),
                     [("dtype", 2), ("rows", -1), ("cols", 0), ("gate_up", None), ("gate_up", A + 1), ("gate_up_stride", 19), ("y", A + 1),
                      ("y_stride", 9), ("codes", None), ("scales", None), ("codes", A + 1), ("scales", A + 1)]),
    "tn_silu_gate_gradients": (dict(dtype=1, rows=2, cols=10, gate_up=A, gate_up_stride=20, dh=A, dh_stride=10, y=A, y_stride=20, codes=A, scales=A,
                                    stream=None),
                               [("dtype", 2), ("rows", -1), ("cols", 0), ("gate_up", None), ("dh", None), ("gate_up_stride", 19), ("dh_stride", 9),
                                ("dh", A + 1), ("y", A + 1), ("y_stride", 19), ("codes", None), ("scales", None)]),
}


@pytest.mark.parametrize("name", sorted(ROW_CALLS))
def test_row_operators_refuse(name):
    good, bad = ROW_CALLS[name]
    fn = getattr(fp8._library(), name)
    for key, value in bad:
        assert key in good
        assert fn(*{**good, key: value}.values()) == INVALID, (key, value)
    assert fn(*{**good, "rows": (1 << 30) + 1}.values()) == UNSUPPORTED
    assert fn(*{**good, "cols": 1 << 30}.values()) == UNSUPPORTED
    if name != "tn_rms_norm_gradients":                       # its dweight is written for no rows too
        assert fn(*{**good, "rows": 0}.values()) == 0


def test_nothing_asked_for_is_refused():
    lib = fp8._library()
    assert lib.tn_rms_norm(*{**ROW_CALLS["tn_rms_norm"][0], "sum": None, "y": None, "codes": None, "scales": None}.values()) == INVALID
    assert lib.tn_silu_gate(*{**ROW_CALLS["tn_silu_gate"][0], "y": None, "codes": None, "scales": None}.values()) == INVALID
    assert lib.tn_silu_gate_gradients(*{**ROW_CALLS["tn_silu_gate_gradients"][0], "y": None, "codes": None, "scales": None}.values()) == INVALID


def test_norm_refuses_one_place_for_two_outputs():
    lib = fp8._library()
    good = ROW_CALLS["tn_rms_norm"][0]
    for where in (A, A + 4096):
        assert lib.tn_rms_norm(*{**good, "sum": where, "y": where, "residual": A}.values()) == INVALID
        assert lib.tn_rms_norm(*{**good, "sum": where, "y": where, "codes": None, "scales": None}.values()) == INVALID


def test_norm_workspace():
    f = fp8._library().tn_rms_norm_gradients_workspace
    assert f(-1, 5) == INVALID and f(5, 0) == INVALID and f(5, 1 << 30) == UNSUPPORTED and f((1 << 30) + 1, 5) == UNSUPPORTED
    assert f(0, 5) == 0 and f(1, 5) >= 20 and f(1 << 30, 100) <= 1 << 24


def _desc(**change):
    d = fp8._Desc()
    fields = dict(dtype=1, n_tensors=1, out_features=10, in_features=10, max_tokens=1, flags=0, stream=None, tensors=[A], scales=None)
    fields.update(change)
    keep = []
    for key in ("tensors", "scales"):
        if fields[key] is not None:
            arr = (ctypes.c_void_p * len(fields[key]))(*fields[key])
            keep.append(arr)
            fields[key] = arr
    for key, value in fields.items():
        if value is not None:
            setattr(d, key, value)
    return d, keep


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(n_tensors=0), INVALID), (dict(n_tensors=3, tensors=[A] * 3), INVALID),
    (dict(out_features=0), INVALID), (dict(in_features=-4), INVALID), (dict(max_tokens=0), INVALID), (dict(flags=2), INVALID),
    (dict(tensors=None), INVALID), (dict(tensors=[None]), INVALID), (dict(tensors=[A + 1]), INVALID), (dict(dtype=2), INVALID),
    (dict(dtype=2, scales=[None]), INVALID), (dict(n_tensors=2, tensors=[A, None]), INVALID),
    (dict(workspace=A + 16, workspace_bytes=1024), INVALID), (dict(workspace=A, workspace_bytes=0), INVALID), (dict(workspace_bytes=1024), INVALID),
    (dict(out_features=1 << 23), UNSUPPORTED), (dict(in_features=1 << 40), UNSUPPORTED), (dict(max_tokens=1 << 40), UNSUPPORTED)])
def test_layer_descriptions_refused(change, status):
    h = ctypes.c_void_p(0)
    d, keep = _desc(**change)
    assert fp8._library().tn_fp8_linear_create(ctypes.byref(h), ctypes.byref(d)) == status
    assert not h.value


def test_null_handles():
    lib = fp8._library()
    d, keep = _desc()
    value = ctypes.c_int64(0)
    assert lib.tn_fp8_linear_create(None, ctypes.byref(d)) == INVALID
    assert lib.tn_fp8_linear_create(ctypes.byref(ctypes.c_void_p(0)), None) == INVALID
    assert lib.tn_fp8_linear_forward(None, A, A, A, 10, 1, None) == INVALID
    assert lib.tn_fp8_linear_gated(None, A, A, A, A, 1, None) == INVALID
    assert lib.tn_fp8_linear_tensor(None, 0, A, A, None) == INVALID
    assert lib.tn_fp8_linear_query(None, tn.TN_QUERY_OUT_FEATURES, ctypes.byref(value)) == INVALID
    assert lib.tn_fp8_linear_destroy(None) == 0


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(2, 8), torch.zeros(8)
    for call in (lambda: tn.rms_norm(x, w), lambda: tn.quantize_fp8(x), lambda: tn.silu_gate(x), lambda: tn.silu_gate_gradients(x, x[:, :4]),
                 lambda: tn.rms_norm_gradients(x, x, w), lambda: tn.Fp8Rows(torch.zeros(1, 128, dtype=torch.float8_e4m3fn), torch.zeros(1, 4), 8)):
        with pytest.raises(ValueError):
            call()
    if not torch.cuda.is_available():
        with pytest.raises(RuntimeError):
            tn.Fp8Linear([x], 1)


def test_rows_in_host_memory_cannot_be_made():
    with pytest.raises(ValueError):
        tn.Fp8Rows.empty(2, 200, device="cpu")


def test_binding_refuses_tensors_of_another_gpu(monkeypatch):
    """Kernels go to the current GPU's stream: a tensor elsewhere, or a current GPU that is not the tensors', is refused before any launch."""
    from fp8_util import on_gpu
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 0)
    monkeypatch.setattr(fp8, "_library", lambda: pytest.fail("reached the library"))
    made = [[on_gpu(torch.empty(shape, dtype=torch.bfloat16), i) for shape in ((4, 256), (256,), (4, 512))] for i in range(2)]
    e = [(on_gpu(torch.empty((4, 256), dtype=torch.float8_e4m3fn), i), on_gpu(torch.empty((4, 4), dtype=torch.float8_e8m0fnu), i)) for i in range(2)]
    (x, w, wide), (far, far_w, far_wide) = made
    far8 = tn.Fp8Rows(*e[1], 256)
    calls = [lambda: tn.rms_norm(far, far_w), lambda: tn.rms_norm(x, far_w), lambda: tn.rms_norm(x, w, residual=far),
             lambda: tn.rms_norm(x, w, out=tn.RowOutput(far, None)), lambda: tn.rms_norm(x, w, outputs="fp8", out=tn.RowOutput(None, far8)),
             lambda: tn.rms_norm(x, w, residual=x, out=tn.RowOutput(x, None, far)),
             lambda: tn.rms_norm_gradients(far, far, far_w), lambda: tn.rms_norm_gradients(far, x, w), lambda: tn.rms_norm_gradients(x, x, far_w, dweight=False),
             lambda: tn.rms_norm_gradients(x, x, w, dsum=far), lambda: tn.rms_norm_gradients(x, x, w, dx=far),
             lambda: tn.silu_gate(far_wide), lambda: tn.silu_gate(wide, out=tn.RowOutput(far, None)),
             lambda: tn.silu_gate_gradients(wide, far), lambda: tn.silu_gate_gradients(far_wide, far),
             lambda: tn.quantize_fp8(far), lambda: tn.quantize_fp8(x, out=far8), lambda: tn.Fp8Rows(e[0][0], e[1][1], 256)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()


TILES = [(64, 256), (96, 256), (128, 256), (160, 256), (192, 256), (224, 256), (256, 256), (64, 128), (96, 128), (128, 128), (192, 128), (256, 128)]


def test_every_form_of_a_product_is_among_the_tested_sizes():
    from fp8_util import FORM_CASES
    seen, several = set(), set()
    for gated, m, n, tokens in FORM_CASES:
        ask = lambda what: tn.fp8_plan_query(m, n, 1 + gated, tokens, bool(gated), what)      # noqa: E731
        tile = (ask(tn.TN_FP8_PLAN_TILE_TOKENS), ask(tn.TN_FP8_PLAN_TILE_FEATURES))
        ranges, fused, pieces = ask(tn.TN_FP8_PLAN_RANGES), ask(tn.TN_FP8_PLAN_FUSED), ask(tn.TN_FP8_PLAN_STREAM_PIECES)
        assert (tile == (0, 0)) == (pieces > 0) and ranges >= 1 and not (fused and (ranges > 1 or not gated))
        kind = "fused" if fused else "partial" if gated or ranges > 1 else "output"
        seen.add((kind, pieces) if pieces else (kind, tile))
        if not pieces:
            blocks = -(-m // 128) * 128 * (1 + gated)
            items = -(-tokens // tile[0]) * -(-blocks // tile[1]) * ranges
            if items > 256 * (2 if sum(tile) <= 256 else 1):
                several.add((kind, tile))
    want = {("output", t) for t in TILES} | {("partial", t) for t in TILES[:10]} | {("partial", (256, 128)), ("partial", (192, 128))}
    want |= {("fused", t) for t in TILES[:7]} | {(k, g) for k in ("output", "partial") for g in (1, 2, 4)}
    assert not want - seen, want - seen
    assert len({t for k, t in several if k == "output"}) >= 8 and len({t for k, t in several if k == "fused"}) >= 5, several


def test_plan_queries_refuse():
    lib = fp8._library()
    value = ctypes.c_int64(0)
    d, keep = _desc(tensors=None, n_tensors=2)
    ask = lambda tokens=1, gated=0, what=0, desc=d: lib.tn_fp8_linear_plan_query(ctypes.byref(desc) if desc else None, tokens, gated, what, ctypes.byref(value))      # noqa: E731
    assert ask() == 0 and ask(gated=1) == 0
    assert ask(tokens=0) == INVALID and ask(what=99) == INVALID and ask(desc=None) == INVALID and ask(tokens=1 << 40) == UNSUPPORTED
    one, keep1 = _desc(tensors=None)
    back, keep2 = _desc(tensors=None, n_tensors=2, flags=tn.TN_FLAG_TRANSPOSE)
    assert ask(gated=1, desc=one) == INVALID and ask(gated=1, desc=back) == INVALID and ask(desc=back) == 0
    assert lib.tn_fp8_linear_plan_query(ctypes.byref(d), 1, 0, 0, None) == INVALID
