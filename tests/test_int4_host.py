"""Projections with 4-bit weights, what needs no GPU: the oracle's own pins, the C ABI's refusals, the binding's checks, the choice of a kernel."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle.int4_oracle as I
import paper_2602_01613_amd as tn
from paper_2602_01613_amd import fp8, int4

HERE = os.path.dirname(os.path.abspath(__file__))
INVALID, UNSUPPORTED = -1, -2
A = 1 << 20


def test_oracle_packs_and_dequantises():
    rng = np.random.default_rng(0)
    for n in (1, 2, 7, 130):
        codes = rng.integers(0, 16, (5, n), dtype=np.uint8)
        packed = I.pack(codes)
        assert packed.shape == (5, (n + 1) // 2) and np.array_equal(I.unpack(packed, n), codes)
        assert packed[0, 0] & 15 == codes[0, 0] and (n < 2 or packed[0, 0] >> 4 == codes[0, 1])
    codes, scales = rng.integers(0, 16, (3, 70), dtype=np.uint8), rng.standard_normal((3, 3))
    zeros = rng.integers(0, 16, (3, 3), dtype=np.uint8)
    w = I.weight(codes, scales, zeros, 32)
    for f in range(3):
        for k in range(70):
            assert w[f, k] == (int(codes[f, k]) - int(zeros[f, k // 32])) * scales[f, k // 32]
    assert np.array_equal(I.weight(codes, scales, None, 32), I.weight(codes, scales, np.full((3, 3), 8), 32))


def test_oracle_quantises_within_its_step():
    rng = np.random.default_rng(1)
    w = rng.standard_normal((40, 200)).astype(np.float32)
    w[0], w[1], w[2] = 0, np.abs(w[1]), -np.abs(w[2])
    codes, scales, zeros = I.quantize(w, 64)
    assert codes.max() <= 15 and zeros.max() <= 15 and (codes[0] == 8).all() and (zeros[0] == 8).all() and (scales[0] == 0).all()
    assert (zeros[1] == 0).all() and (zeros[2] == 15).all()
    err = np.abs(I.weight(codes, scales, zeros, 64) - w)
    assert (err <= (1 + 15 * 2.0 ** -8) * np.repeat(scales, 64, axis=1)[:, :200]).all()
    assert np.array_equal(I.bf16(np.float32([1.00390625, 1.01171875])), np.float32([1.0, 1.015625]))          # ties to even


def test_header_declares_what_the_binding_exports():
    text = open(os.path.join(os.path.dirname(HERE), "include", "tn_int4.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(tn_int4_[a-z_0-9]+)\s*\(", text))
    assert declared == set(tn.INT4_EXPORTED_SYMBOLS)
    lib = tn.load_library()
    for name in declared:
        assert hasattr(lib, name), name


def _desc(**change):
    d = int4._Desc()
    fields = dict(dtype=3, n_tensors=1, out_features=10, in_features=10, group=32, scale_dtype=1, tensors=[A], scales=[A], zeros=None, flags=0, stream=None)
    fields.update(change)
    keep = []
    for key in ("tensors", "scales", "zeros"):
        if fields[key] is not None:
            arr = (ctypes.c_void_p * len(fields[key]))(*fields[key])
            keep.append(arr)
            fields[key] = arr
    for key, value in fields.items():
        if value is not None:
            setattr(d, key, value)
    return d, keep


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(n_tensors=0), INVALID), (dict(n_tensors=3, tensors=[A] * 3, scales=[A] * 3), INVALID),
    (dict(out_features=0), INVALID), (dict(in_features=-4), INVALID), (dict(group=16), INVALID), (dict(group=256), INVALID), (dict(group=0), INVALID),
    (dict(scale_dtype=0), INVALID), (dict(scale_dtype=2), INVALID), (dict(flags=2), INVALID), (dict(tensors=None), INVALID), (dict(tensors=[None]), INVALID),
    (dict(scales=None), INVALID), (dict(scales=[None]), INVALID), (dict(scales=[A + 1]), INVALID), (dict(zeros=[None]), INVALID),
    (dict(dtype=0, tensors=[A + 2]), INVALID), (dict(dtype=1, tensors=[A + 1]), INVALID), (dict(n_tensors=2, tensors=[A, None], scales=[A, A]), INVALID),
    (dict(out_features=1 << 23), UNSUPPORTED), (dict(in_features=1 << 40), UNSUPPORTED), (dict(out_features=1 << 20, in_features=1 << 13), UNSUPPORTED),
    (dict(out_features=1 << 13, in_features=1 << 20, flags=128), UNSUPPORTED)])
def test_layer_descriptions_refused(change, status):
    h = ctypes.c_void_p(0)
    d, keep = _desc(**change)
    assert int4._library().tn_int4_linear_create(ctypes.byref(h), ctypes.byref(d)) == status
    assert not h.value


def test_null_handles():
    lib = int4._library()
    d, keep = _desc()
    value = ctypes.c_int64(0)
    assert lib.tn_int4_linear_create(None, ctypes.byref(d)) == INVALID
    assert lib.tn_int4_linear_create(ctypes.byref(ctypes.c_void_p(0)), None) == INVALID
    assert lib.tn_int4_linear_workspace(None, A, 10, 1, 0) == INVALID
    assert lib.tn_int4_linear_forward(None, A, 10, A, 10, 1, None, 0, None) == INVALID
    assert lib.tn_int4_linear_gated(None, A, 10, A, 10, 1, None, 0, None) == INVALID
    assert lib.tn_int4_linear_tensor(None, 0, A, A, A, None) == INVALID
    assert lib.tn_int4_linear_query(None, tn.TN_QUERY_OUT_FEATURES, ctypes.byref(value)) == INVALID
    assert lib.tn_int4_linear_destroy(None) == 0


def test_plan_queries_refuse():
    lib = int4._library()
    value = ctypes.c_int64(0)
    d, keep = _desc(tensors=None, n_tensors=2)
    ask = lambda tokens=1, gated=0, what=0, desc=d: lib.tn_int4_linear_plan_query(ctypes.byref(desc) if desc else None, tokens, gated, what, ctypes.byref(value))      # noqa: E731
    assert ask() == 0 and ask(gated=1) == 0
    assert ask(tokens=0) == INVALID and ask(what=99) == INVALID and ask(desc=None) == INVALID and ask(tokens=1 << 40) == UNSUPPORTED
    one, keep1 = _desc(tensors=None)
    back, keep2 = _desc(tensors=None, n_tensors=2, flags=tn.TN_FLAG_TRANSPOSE)
    assert ask(gated=1, desc=one) == INVALID and ask(gated=1, desc=back) == INVALID and ask(desc=back) == 0
    assert lib.tn_int4_linear_plan_query(ctypes.byref(d), 1, 0, 0, None) == INVALID


def test_binding_refuses(monkeypatch):
    """Arguments that do not fit are refused before the library is reached."""
    from fp8_util import on_gpu
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 0)
    monkeypatch.setattr(int4, "_library", lambda: pytest.fail("reached the library"))
    here = lambda shape, dtype, gpu=0: on_gpu(torch.zeros(shape, dtype=dtype), gpu)      # noqa: E731
    codes, s, z = here((4, 5), torch.uint8), here((4, 1), torch.bfloat16), here((4, 1), torch.uint8)
    ok = dict(tensors=[codes], max_tokens=1, transpose=False, group=128, scales=[s], zeros=[z], in_features=None)
    int4._description(**ok)
    int4._description(**{**ok, "in_features": 9})
    int4._description(**{**ok, "tensors": [here((4, 10), torch.float32)], "scales": None, "zeros": None})
    for change in (dict(tensors=[]), dict(tensors=[codes] * 3), dict(tensors=[codes, here((4, 6), torch.uint8)]), dict(max_tokens=0), dict(group=100), dict(scales=None),
                   dict(scales=[s, s]), dict(scales=[here((4, 1), torch.float32)]), dict(scales=[here((4, 2), torch.bfloat16)]), dict(scales=[here((4, 1), torch.bfloat16, 1)]),
                   dict(zeros=[here((4, 1), torch.int8)]), dict(zeros=[z, z]), dict(zeros=[here((3, 1), torch.uint8)]), dict(in_features=8), dict(in_features=11),
                   dict(tensors=[here((4, 5), torch.uint8, 1)]), dict(tensors=[here((4, 5), torch.int8)]), dict(tensors=[torch.zeros((4, 5), dtype=torch.uint8)]),
                   dict(tensors=[here((4, 10), torch.float32)]), dict(tensors=[here((4, 10), torch.float32)], scales=None, zeros=[z]),
                   dict(tensors=[here((4, 10), torch.float32)], scales=None, zeros=None, in_features=9), dict(tensors=[here((4, 10), torch.float16)], scales=None, zeros=None),
                   dict(tensors=[here((5, 4), torch.uint8).t()])):
        with pytest.raises(ValueError):
            int4._description(**{**ok, **change})
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 1)
    with pytest.raises(ValueError):
        int4._description(**ok)


def test_needs_a_gpu():
    if not torch.cuda.is_available():
        with pytest.raises(RuntimeError):
            tn.Int4Linear([torch.zeros(4, 4)], 1)


TILES = (32, 64, 96, 128, 160, 192)


def test_every_form_of_a_product_is_among_the_tested_sizes():
    from int4_util import FORM_CASES
    seen = set()
    for kind, tokens, m, n, group in FORM_CASES:
        ask = lambda what: tn.int4_plan_query(m, n, 2 if kind == "gated" else 1, tokens, kind == "gated", what, kind == "back", group)      # noqa: E731
        tile, ranges, stream = ask(tn.TN_INT4_PLAN_TILE_TOKENS), ask(tn.TN_INT4_PLAN_RANGES), (ask(tn.TN_INT4_PLAN_STREAM_TOKENS), ask(tn.TN_INT4_PLAN_STREAM_PIECES))
        assert (tile == 0) == (stream[0] > 0) == (stream[1] > 0) and (tile or ranges == 1)
        seen.add((kind, tile, ranges > 1) if tile else (kind,) + stream)
    want = {(k, t, s) for k in ("plain", "gated", "back") for t in TILES for s in (False, True)}
    want |= {("plain", 16, 1), ("plain", 16, 2), ("plain", 16, 4), ("plain", 32, 4), ("gated", 16, 2), ("gated", 16, 4), ("gated", 32, 4)}
    assert not want - seen, want - seen


def test_a_given_output_counts_as_written(monkeypatch):
    """For autograd, which may have saved it."""
    from fp8_util import on_gpu

    class Library:
        def __getattr__(self, name):
            return lambda *args: 0
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 0)
    for name, value in (("_lib", Library()), ("_library", Library), ("_stream", lambda gpu: 99)):
        monkeypatch.setattr(int4, name, value)
    layer = tn.Int4Linear.__new__(tn.Int4Linear)
    for name, value in dict(_handle=123, _gpu=0, _device="cpu", max_tokens=8, n_tensors=2, transpose=False, shape=(6, 10), M=12, N=10).items():
        setattr(layer, name, value)
    x, y, h = (on_gpu(torch.zeros(shape, dtype=torch.bfloat16), 0) for shape in ((3, 10), (3, 12), (3, 6)))
    assert layer(x, out=y) is y and layer.gated(x, out=h) is h
    assert (x._version, y._version, h._version) == (0, 1, 1)
    with pytest.raises(ValueError):
        layer(x, out=h)
    assert h._version == 1
    assert layer(x)._version == 0 and layer.gated(x)._version == 0


BESIDE = """
import ctypes, json
import paper_2602_01613_amd as tn
from paper_2602_01613_amd import int4
import test_int4_host as host
lib = int4._library()
mem = ctypes.create_string_buffer(1 << 20)
at = (ctypes.addressof(mem) + 255) // 256 * 256
space = at + (1 << 19)
desc, keep = host._desc(out_features=20, in_features=32, tensors=[at], scales=[at])
h = ctypes.c_void_p(0)
assert lib.tn_int4_linear_create(ctypes.byref(h), ctypes.byref(desc)) == 0
def status(x_at, x_stride, y_at, y_stride, tokens):
    base = at + 4096
    return lib.tn_int4_linear_forward(h, base + 2 * x_at, x_stride, base + 2 * y_at, y_stride, tokens, space, 1 << 18, None)
print("RESULT " + json.dumps([status(*case) for case in json.loads(CASES)]))
"""


def test_input_and_output_may_lie_beside_each_other():
    """Against the sets of their elements, where the strides are equal; of different strides, against the spans."""
    import json
    import subprocess
    import sys
    import tempfile
    cases = [(x, s, y, s, t) for s in (32, 40, 52, 55, 60, 104) for t in (1, 2, 5) for x, y in
             [(0, d) for d in (0, 19, 20, 31, 32, 35, 40, 51, 52, 60, 84, 104, 136, 300)] + [(d, 0) for d in (1, 19, 20, 23, 25, 28, 32, 40, 52, 72, 75, 124, 300)]]
    cases += [(0, 64, 32, 65, 3), (0, 64, 160, 65, 3), (0, 64, 159, 65, 3), (200, 64, 0, 90, 3), (199, 64, 0, 90, 3)]
    with tempfile.TemporaryDirectory() as folder:
        out = os.path.join(folder, "libfake_hip.so")
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I/opt/rocm/include", os.path.join(HERE, "fake_hip.cpp"), "-o", out])
        env = dict(os.environ, LD_PRELOAD=out, PYTHONPATH=os.pathsep.join([HERE, os.path.dirname(HERE)]))
        r = subprocess.run([sys.executable, "-c", f"CASES = {json.dumps(json.dumps(cases))}\n" + BESIDE], cwd=os.path.dirname(HERE), env=env, capture_output=True, text=True, timeout=300)
    lines = [l for l in r.stdout.splitlines() if l.startswith("RESULT ")]
    assert lines, r.stderr[-800:]
    for (x, sx, y, sy, t), status in zip(cases, json.loads(lines[0][7:])):
        if sx == sy:
            mine, other = ({at + i * sx + c for i in range(t) for c in range(cols)} for at, cols in ((x, 32), (y, 20)))
            apart = not mine & other
        else:
            apart = x >= y + (t - 1) * sy + 20 or y >= x + (t - 1) * sx + 32
        assert status == (0 if apart else INVALID), (x, sx, y, sy, t, status)


def _kernels(path):
    """(name, notes) of the gfx950 kernels in a library that was built here: the metadata of its code objects."""
    import struct

    import msgpack
    data = open(path, "rb").read()
    at = data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        n, p = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(n):
            start, size, length = struct.unpack_from("<QQQ", data, p)
            target, p = data[p + 24:p + 24 + length], p + 24 + length
            if b"gfx950" not in target or not size:
                continue
            elf = data[at + start:at + start + size]
            headers, (step, count) = struct.unpack_from("<Q", elf, 32)[0], struct.unpack_from("<HH", elf, 54)
            for i in range(count):
                kind, _, where, _, _, held = struct.unpack_from("<IIQQQQ", elf, headers + i * step)
                end = where + held if kind == 4 else 0                    # 4: notes
                while where < end:
                    name, size_of, what = struct.unpack_from("<III", elf, where)
                    body = where + 12 + (name + 3) // 4 * 4
                    if what == 32:                                        # AMDGPU metadata
                        for kernel in msgpack.unpackb(elf[body:body + size_of])["amdhsa.kernels"]:
                            yield kernel[".name"], kernel
                    where = body + (size_of + 3) // 4 * 4
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 24)


def test_no_kernel_keeps_registers_in_memory():
    """A register that does not fit goes to scratch memory, and comes back from it in the inner loop."""
    found = {name: k for name, k in _kernels(tn.library_path()) if re.search(r"int4_|adamw_|gradient_norm", name)}
    assert sum("int4_stream_kernel" in n for n in found) == 21 and sum("int4_gemm_kernel" in n for n in found) == 78 and len(found) > 105
    spilled = [n for n, k in found.items() if k[".vgpr_spill_count"] or k[".sgpr_spill_count"] or k[".private_segment_fixed_size"]]
    assert not spilled, spilled


def test_every_compiled_kernel_is_among_the_tested_sizes():
    """Tiles by tokens, output, direction and groups to 128 inputs (transposed: groups of features to a wave's 64), streams by tokens, pieces, output and groups."""
    from int4_util import GROUP_CASES
    seen = set()
    for kind, tokens, m, n, groups in GROUP_CASES:
        for group in groups:
            ask = lambda what: tn.int4_plan_query(m, n, 2 if kind == "gated" else 1, tokens, kind == "gated", what, kind == "back", group)      # noqa: E731
            tile, ranges = ask(tn.TN_INT4_PLAN_TILE_TOKENS), ask(tn.TN_INT4_PLAN_RANGES)
            sub = 128 // group if kind != "back" else 2 if group == 32 else 1
            seen.add((kind, tile, ranges > 1, sub) if tile else (kind, ask(tn.TN_INT4_PLAN_STREAM_TOKENS), ask(tn.TN_INT4_PLAN_STREAM_PIECES), sub))
            blocks = -(-(m if kind == "back" else n) // 128)
            assert -(-blocks // ranges) >= 6, (kind, tokens, m, n, group)
    want = {(k, t, s, u) for k in ("plain", "gated") for t in TILES for s in (False, True) for u in (1, 2, 4)} | {("back", t, s, u) for t in TILES for s in (False, True) for u in (1, 2)}
    want |= {("plain", t, p, u) for t, p in ((16, 1), (16, 2), (16, 4), (32, 4)) for u in (1, 2, 4)} | {("gated", t, p, u) for t, p in ((16, 2), (16, 4), (32, 4)) for u in (1, 2, 4)}
    assert not want - seen, want - seen


def test_long_rows_are_as_long_as_they_are_meant_to_be():
    from int4_util import LONG_ROWS
    for tokens, m, n, tensors, transposed, ranges, runs in LONG_ROWS:
        assert tn.int4_plan_query(m, n, tensors, tokens, False, tn.TN_INT4_PLAN_TILE_TOKENS, transposed) > 0
        assert tn.int4_plan_query(m, n, tensors, tokens, False, tn.TN_INT4_PLAN_RANGES, transposed) == ranges
        blocks = tensors * -(-m // 128) if transposed else -(-n // 128)
        assert -(-blocks // ranges) * 16 == runs
    runs = [r[-1] for r in LONG_ROWS]
    assert any(512 < r <= 1024 for r in runs) and any(1024 < r <= 3328 for r in runs) and any(r > 3328 for r in runs)
    assert any(t == 2 and back and -(-m // 128) * 16 > 3328 for _, m, _, t, back, _, _ in LONG_ROWS)          # the second tensor's part begins behind what threads hold


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_bound_of_weights_in_tiles(kind):
    """A scale as fp16 under the power of two that puts the largest into [2^10, 2^11), times a code, rounded again: off by 2^-11 of the weight and, of scales below 2^-24 of the largest, by
    2^-31 of that largest. Half of the latter would not do."""
    rng = np.random.default_rng(2)
    bits = 11 if kind == "f16" else 8
    largest = np.exp2(rng.uniform(0, 1, 1 << 18))
    part, e = np.frexp(largest * np.exp2(-rng.uniform(0, 40, largest.size)))
    scale = np.ldexp(np.round(part * 2 ** bits) / 2 ** bits, e)
    half = (scale * 1024).astype(np.float16)
    assert (half.astype(np.float64) / 1024 == scale)[scale >= 2.0 ** -24 * largest].all()
    codes = np.arange(1, 16)[:, None]
    off = np.abs((codes.astype(np.float16) * half).astype(np.float64) / 1024 - codes * scale) - 2.0 ** -11 * codes * scale
    assert 2.0 ** -32 < (off / largest).max() <= 2.0 ** -31
