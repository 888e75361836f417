"""The AdamW step, what needs no GPU: the oracle's own pins, the C ABI's refusals, the binding's checks."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import oracle.adamw_oracle as O
import paper_2602_01613_amd as tn
from paper_2602_01613_amd import adamw, fp8

HERE = os.path.dirname(os.path.abspath(__file__))
INVALID, UNSUPPORTED = -1, -2
A = 1 << 20


def test_oracle_step_against_torch():
    rng = np.random.default_rng(0)
    p = torch.from_numpy(rng.standard_normal(50)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
    mine, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        mine, m, v = O.step(mine, g, m, v, t, 0.01, 0.9, 0.99, 1e-6, 0.1)
        assert np.abs(mine - p.detach().numpy()).max() < 1e-13


def test_rounding_is_right_on_average_and_to_a_neighbour():
    """At every point between two codes the share that goes up is the part of the way, to the 2^-16 of the random numbers."""
    h = np.arange(1 << 16, dtype=np.uint64)
    for value in (1.0, 1.03, 100.0, 447.9, 448.0, 0.011, 2.0 ** -9, 2.0 ** -11, 0.0):
        v = np.concatenate([np.full(127 * 512, value), [448.0] * 512]).reshape(128, 512).T.reshape(-1)          # the scale is 1
        codes, e = O.quantize(v, np.resize(h, v.size))
        assert (e == 0).all()
        mine = codes.reshape(-1, 128)[:, :127]
        _, _, below, part, step = O.neighbours(v)
        assert np.isin(mine, [below[0, 0], below[0, 0] + step[0, 0]]).all()
        assert abs(mine.mean() - value) <= step[0, 0] * 2.0 ** -7         # (65024 of the 65536 numbers, in order)
    assert np.array_equal(O.quantize(-v, np.resize(h, v.size))[0], -codes)


def test_roots_least_part_of_m_holds_for_every_past_and_is_reached():
    rng = np.random.default_rng(0)
    for beta1, beta2 in ((0.9, 0.999), (0.9, 0.95), (0.0, 0.9)):
        least = O.least_root(beta1, beta2)
        pasts = [np.ones(200), rng.standard_normal(200), (beta1 / beta2) ** np.arange(200)[::-1], np.eye(200)[150]]
        parts = []
        for past in pasts:
            m = v = 0.0
            for g in past:
                _, m, v = O.step(0.0, g, m, v, 1, 0.0, beta1, beta2, 1.0, 0.0)
                assert v ** 0.5 >= least * abs(m) * (1 - 1e-12)
            parts.append(v ** 0.5 / max(abs(m), 1e-30))
        assert abs(parts[2] / least - 1) < 1e-3            # the gradients that make the two sides alike
    assert O.least_root(0.99, 0.9) == 0.0


def test_hash_is_even_and_its_halves_and_steps_are_apart():
    """Means and correlations of 2^18 numbers, within five standard errors of what independent even ones have."""
    n = 1 << 18
    places = np.arange(n)
    series = []
    for seed, step, base in ((0, 1, 0), (0, 2, 0), (1, 1, 0), (0, 1, 1 << 32)):
        h = O.hash_of(seed, step, places + base)
        series += [h & np.uint64(0xFFFF), h >> np.uint64(16)]
    x = np.array(series, dtype=np.float64) / 65536 - 0.5
    assert np.abs(x.mean(axis=1)).max() < 5 * (1 / 12 / n) ** 0.5
    assert np.abs(np.corrcoef(x) - np.eye(8)).max() < 5 / n ** 0.5
    assert np.abs([np.corrcoef(r[:-d], r[d:])[0, 1] for r in x for d in (1, 2, 8, 128)]).max() < 5.5 / n ** 0.5
    over = np.array([O.hash_of(9, t, places[:512]) & np.uint64(0xFFFF) for t in range(512)], dtype=np.float64) / 65536 - 0.5
    assert abs((over[:-1] * over[1:]).mean()) * 12 < 5 / over.size ** 0.5


def test_header_declares_what_the_binding_exports():
    text = open(os.path.join(os.path.dirname(HERE), "include", "tn_adamw.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(tn_adamw_[a-z_0-9]+)\s*\(", text))
    assert declared == set(tn.ADAMW_EXPORTED_SYMBOLS)
    lib = tn.load_library()
    for name in declared:
        assert hasattr(lib, name), name


def test_state_values():
    f = adamw._state_values
    assert f([1]) == 128 and f([0]) == 0 and f([128, 129, 0, 5]) == 128 + 256 + 128
    raw = adamw._library().tn_adamw_state_values
    one = (ctypes.c_int64 * 1)
    assert raw(0, one(5)) == INVALID and raw(1, None) == INVALID and raw(1, one(-1)) == INVALID and raw(1, one(1 << 50)) == UNSUPPORTED
    assert raw((1 << 20) + 1, one(5)) == UNSUPPORTED


def _desc(**change):
    d = adamw._Desc()
    fields = dict(n_tensors=2, state_bits=8, sizes=[5, 6], dtypes=[0, 1], params=[A, A + 256], decays=[0.0, 0.0], first=A, second=A, first_scales=A, second_scales=A,
                  master=A, count=A, beta1=0.9, beta2=0.99, eps=1e-8, seed=0, init_master=0, stream=None)
    fields.update(change)
    types = dict(sizes=ctypes.c_int64, dtypes=ctypes.c_int32, params=ctypes.c_void_p, decays=ctypes.c_float)
    keep = []
    for key, kind in types.items():
        if fields[key] is not None:
            arr = (kind * len(fields[key]))(*fields[key])
            keep.append(arr)
            fields[key] = ctypes.cast(arr, ctypes.POINTER(kind))
    for key, value in fields.items():
        if value is not None:
            setattr(d, key, value)
    return d, keep


@pytest.mark.parametrize("change,status", [
    (dict(n_tensors=0), INVALID), (dict(state_bits=16), INVALID), (dict(sizes=None), INVALID), (dict(sizes=[5, -1]), INVALID), (dict(dtypes=None), INVALID),
    (dict(dtypes=[0, 2]), INVALID), (dict(params=None), INVALID), (dict(params=[A, None]), INVALID), (dict(params=[A + 2, A]), INVALID), (dict(params=[A, A + 1]), INVALID),
    (dict(decays=None), INVALID), (dict(first=None), INVALID), (dict(second=A + 64), INVALID), (dict(first_scales=None), INVALID), (dict(second_scales=None), INVALID),
    (dict(master=None), INVALID), (dict(master=A + 4), INVALID), (dict(count=None), INVALID), (dict(count=A + 4), INVALID), (dict(beta1=1.0), INVALID), (dict(beta2=-0.1), INVALID),
    (dict(beta1=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(sizes=[1 << 41, 5]), UNSUPPORTED)])
def test_descriptions_refused(change, status):
    h = ctypes.c_void_p(0)
    d, keep = _desc(**change)
    assert adamw._library().tn_adamw_create(ctypes.byref(h), ctypes.byref(d)) == status
    assert not h.value


def test_null_handles():
    lib = adamw._library()
    d, keep = _desc()
    assert lib.tn_adamw_create(None, ctypes.byref(d)) == INVALID and lib.tn_adamw_create(ctypes.byref(ctypes.c_void_p(0)), None) == INVALID
    grads, kinds = (ctypes.c_void_p * 1)(A), (ctypes.c_int32 * 1)(0)
    assert lib.tn_adamw_workspace(None) == INVALID
    assert lib.tn_adamw_gradient_norm(None, grads, kinds, A, A, 1 << 20, None) == INVALID
    assert lib.tn_adamw_step(None, grads, kinds, 0.1, None, 0.0, None, 0, None, 0, None) == INVALID
    assert lib.tn_adamw_destroy(None) == 0


def test_binding_refuses(monkeypatch):
    """Parameters and numbers that do not fit are refused before the library is reached."""
    from fp8_util import on_gpu
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 0)
    here = lambda shape, dtype=torch.float32, gpu=0: on_gpu(torch.zeros(shape, dtype=dtype), gpu)      # noqa: E731
    p = here(100)
    assert adamw._check_params([p, here(5, torch.bfloat16), here(0)]) == 0
    for bad in ([], [p, p], [p, on_gpu(p[90:95], 0)], [here(4, torch.float16)], [torch.zeros(4)], [here((4, 5)).t()], [here(4, gpu=1)], [p, here(4, gpu=1)], [None]):
        with pytest.raises(ValueError):
            adamw._check_params(bad)
    ok = dict(n=2, lr=0.1, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0, state_bits=8, seed=0)
    assert adamw._check_numbers(**ok) == [0.0, 0.0] and adamw._check_numbers(**{**ok, "weight_decay": [0.1, 0]}) == [0.1, 0.0]
    nan, inf = float("nan"), float("inf")
    for change in (dict(lr=-1), dict(lr=nan), dict(lr=inf), dict(betas=(0.9,)), dict(betas=(1.0, 0.9)), dict(betas=(0.9, nan)), dict(eps=-1), dict(eps=nan), dict(state_bits=4),
                   dict(weight_decay=[0.1]), dict(weight_decay=nan), dict(weight_decay=[0.1, -0.1]), dict(seed=-1), dict(seed=2 ** 32)):
        with pytest.raises(ValueError):
            adamw._check_numbers(**{**ok, **change})


def test_needs_a_gpu():
    if not torch.cuda.is_available():
        with pytest.raises(RuntimeError):
            tn.AdamW([torch.zeros(4)])


class _Recorder:
    """A library whose functions note their calls and succeed."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name,) + args) or 0


def _optimizer(monkeypatch, params, **more):
    """(an optimizer of these tensors, which say that they are on GPU 0, its library's calls)"""
    lib = _Recorder()
    monkeypatch.setattr(fp8, "_current_gpu", lambda: 0)
    for name, value in (("_lib", lib), ("_library", lambda: lib), ("_stream", lambda gpu: 99)):
        monkeypatch.setattr(adamw, name, value)
    opt = tn.AdamW.__new__(tn.AdamW)
    state = {"first": torch.zeros(128), "second": torch.zeros(128), "count": torch.zeros((), dtype=torch.int64), "master": torch.zeros(128)}
    fields = dict(_handle=123, _gpu=0, params=params, lr=0.1, betas=(0.9, 0.99), eps=1e-8, weight_decay=[0.0] * len(params), state_bits=32, seed=0, _state=state,
                  _sizes=[p.numel() for p in params], _shapes=[p.shape for p in params], _param_pointers=[p.data_ptr() for p in params],
                  _all_f32=(ctypes.c_int32 * len(params))(), _workspace_bytes=256, _device="cpu")
    for name, value in {**fields, **more}.items():
        setattr(opt, name, value)
    return opt, lib.calls


def test_reset_master_keeps_the_handle(monkeypatch):
    """Captured steps have the addresses of the handle's tables: it is neither destroyed nor made anew."""
    from fp8_util import on_gpu
    opt, calls = _optimizer(monkeypatch, [on_gpu(torch.zeros(5, dtype=torch.bfloat16), 0)])
    opt.reset_master()
    assert calls == [("tn_adamw_reset_master", 123, 99)] and opt._handle == 123
    opt.close()
    with pytest.raises(RuntimeError):
        opt.reset_master()


def test_reset_master_refuses_no_handle():
    assert adamw._library().tn_adamw_reset_master(None, None) == INVALID


RESET = """
import ctypes, json, os
import paper_2602_01613_amd as tn
from paper_2602_01613_amd import adamw
import test_adamw_host as host
lib = adamw._library()
hip = ctypes.CDLL(os.environ['LD_PRELOAD'])
hip.fake_hip_take_launches.restype = ctypes.c_char_p
take = lambda: [l.split()[0] for l in hip.fake_hip_take_launches().decode().splitlines()]
mem = ctypes.create_string_buffer(65536)
at = (ctypes.addressof(mem) + 255) // 256 * 256
found = []
for dtypes, sizes in (([0, 1], [5, 6]), ([0, 0], [5, 6]), ([0, 1], [5, 0])):
    d, keep = host._desc(dtypes=dtypes, sizes=sizes, params=[at, at + 256], first=at, second=at, first_scales=at, second_scales=at, master=at, count=at, init_master=0)
    h = ctypes.c_void_p(0)
    assert lib.tn_adamw_create(ctypes.byref(h), ctypes.byref(d)) == 0
    made = take()
    assert lib.tn_adamw_reset_master(h, None) == 0
    found.append([made, take()])
    assert lib.tn_adamw_destroy(h) == 0
print("RESULT " + json.dumps(found))
"""


def test_reset_master_is_one_launch_where_a_parameter_is_in_bf16():
    import json
    import subprocess
    import sys
    import tempfile
    with tempfile.TemporaryDirectory() as folder:
        out = os.path.join(folder, "libfake_hip.so")
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I/opt/rocm/include", os.path.join(HERE, "fake_hip.cpp"), "-o", out])
        env = dict(os.environ, LD_PRELOAD=out, PYTHONPATH=os.pathsep.join([HERE, os.path.dirname(HERE)]))
        r = subprocess.run([sys.executable, "-c", RESET], cwd=os.path.dirname(HERE), env=env, capture_output=True, text=True, timeout=300)
    lines = [l for l in r.stdout.splitlines() if l.startswith("RESULT ")]
    assert lines, r.stderr[-800:]
    (mixed_made, mixed), (_, f32), (_, empty) = json.loads(lines[0][7:])
    assert mixed_made == [] and len(mixed) == 1 and "adamw_master_kernel" in mixed[0] and f32 == [] and empty == []


def test_a_step_raises_the_parameters_versions(monkeypatch):
    """What autograd saved before a step is not taken for the same after it; a step that was refused changes nothing."""
    from fp8_util import on_gpu
    params = [on_gpu(torch.zeros(5), 0), on_gpu(torch.zeros(3, dtype=torch.bfloat16), 0)]
    opt, calls = _optimizer(monkeypatch, params)
    before = [p._version for p in params]
    grads = [on_gpu(torch.zeros(5), 0), on_gpu(torch.zeros(3), 0)]
    with pytest.raises(ValueError):
        opt.step(grads, lr=-1.0)
    assert [p._version for p in params] == before and not calls
    opt.step(grads)
    assert [c[0] for c in calls] == ["tn_adamw_step"]
    assert [p._version for p in params] == [v + 1 for v in before] and [g._version for g in grads] == [0, 0]


def test_a_given_norm_tensor_counts_as_written(monkeypatch):
    from fp8_util import on_gpu
    opt, calls = _optimizer(monkeypatch, [on_gpu(torch.zeros(5), 0)])
    out = on_gpu(torch.zeros(()), 0)
    assert opt.gradient_norm([on_gpu(torch.zeros(5), 0)], out=out) is out
    assert [c[0] for c in calls] == ["tn_adamw_gradient_norm"] and out._version == 1


def test_a_parameter_whose_memory_moved_is_refused(monkeypatch):
    """The handle has the addresses of the parameters as they were: neither a step nor reset_master() may go there."""
    from fp8_util import on_gpu
    opt, calls = _optimizer(monkeypatch, [on_gpu(torch.zeros(5, dtype=torch.bfloat16), 0)])
    grads = [on_gpu(torch.zeros(5), 0)]
    opt.step(grads)
    opt.reset_master()
    assert [c[0] for c in calls] == ["tn_adamw_step", "tn_adamw_reset_master"]
    opt.params[0] = on_gpu(torch.zeros(5, dtype=torch.bfloat16), 0)
    for call in (lambda: opt.step(grads), opt.reset_master):
        with pytest.raises(RuntimeError, match="not where it was"):
            call()
    assert len(calls) == 2
