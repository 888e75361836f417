"""Gradients of the norm where a workgroup takes several rows: the row requested ahead, sums over rows, outputs in place of an input."""
import numpy as np
import pytest
import torch

import oracle.fp8_oracle as Q
import paper_2602_01613_amd as tn
from fp8_util import dev, half_unit, host, rounded
from paper_2602_01613_amd import fp8

pytestmark = pytest.mark.gpu

EPS = 1e-6


def groups_of(rows, cols):
    """Workgroups of a call: each leaves a row of fp32 sums in the workspace."""
    need = fp8._library().tn_rms_norm_gradients_workspace(rows, cols)
    assert need > 0 and need % (4 * cols) == 0
    return need // (4 * cols)


def check(got, ref, bound):
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= bound).all(), (err - bound).max()


# whole chunks of 8, one to a thread (the next row is requested ahead): two, three and four rows, odd and even numbers of them, the last round
# full, all but empty and in between; parts of a chunk at the end of a row; two chunks to a thread, whole and not
SIZES = [(257, 5120), (512, 5120), (600, 5120), (771, 5120), (1024, 5120), (1300, 1024), (5200, 40), (2561, 8),
         (2700, 129), (1300, 1001), (700, 5121), (600, 8200), (520, 9001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_several_rows_to_a_workgroup(rows, cols, dtype):
    groups = groups_of(rows, cols)
    assert rows > groups
    rng = np.random.default_rng(rows * 20011 + cols)
    s = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-3, 4, (rows, 1)))           # rows of different sizes: one taken for another shows
    s[:, rng.integers(0, cols, max(1, cols // 300))] *= 30
    s, dy, ds = (rounded(v, dtype) for v in (s, rng.standard_normal((rows, cols)) * 1e-3, rng.standard_normal((rows, cols)) * 1e-3))
    w = rounded(1 + 0.2 * rng.standard_normal(cols), dtype)
    d = {k: dev(v, dtype) for k, v in (("s", s), ("dy", dy), ("ds", ds), ("w", w))}
    dx, dw = tn.rms_norm_gradients(d["dy"], d["s"], d["w"], EPS, dsum=d["ds"])
    ref, ref_dw = Q.rms_norm_gradients(dy, s, w, EPS, ds)
    r = 1 / np.sqrt((s * s).mean(axis=1, keepdims=True) + EPS)
    u, g = s * r, dy * w
    # fp32: the mean of g * u to 2^-20 of the mean of |g * u|; each term to a few roundings of its own size
    extra = 2.0 ** -20 * (r * np.abs(g) + r * np.abs(u) * np.abs(g * u).mean(axis=1, keepdims=True) + np.abs(ds))
    check(host(dx), ref, half_unit(ref, dtype) + extra)
    # a column's sum: a term to 2^-21 of itself, and one rounding of 2^-24 for each of the additions in a row (a workgroup's rows, every 32nd
    # workgroup, five to join them), whose running sums are no larger than the sum of magnitudes
    in_a_row = -(-rows // groups) + -(-groups // 32) + 5
    check(host(dw), ref_dw, (in_a_row + 8) * 2.0 ** -24 * np.abs(dy * u).sum(axis=0))
    # a row's result does not depend on the rows before it
    for i in (0, groups - 1, groups, rows - 1):
        one, _ = tn.rms_norm_gradients(d["dy"][i:i + 1], d["s"][i:i + 1], d["w"], EPS, dsum=d["ds"][i:i + 1], dweight=False)
        assert torch.equal(one[0], dx[i]), i
    for key in ("s", "dy", "ds"):                             # in place of each input
        now = {**d, key: d[key].clone()}
        again, dw2 = tn.rms_norm_gradients(now["dy"], now["s"], now["w"], EPS, dsum=now["ds"], dx=now[key])
        assert again is now[key] and torch.equal(again, dx) and torch.equal(dw2, dw)
    alone, dw3 = tn.rms_norm_gradients(d["dy"], d["s"], d["w"], EPS)
    check(host(alone), ref - ds, half_unit(ref - ds, dtype) + extra)
    assert torch.equal(dw3, dw)


@pytest.mark.parametrize("cols", [1000, 1001])
def test_several_rows_of_wider_tensors(cols):
    rows = 1400
    assert rows > groups_of(rows, cols)
    rng = np.random.default_rng(cols)
    wide = dev(rng.standard_normal((rows, 3 * cols + 1)))
    dy, s, ds = wide[:, :cols], wide[:, cols:2 * cols], wide[:, 2 * cols:3 * cols]
    dx, dw = tn.rms_norm_gradients(dy.contiguous(), s.contiguous(), dev(np.ones(cols)), EPS, dsum=ds.contiguous())
    out = torch.full((rows, cols + 7), 7.0, dtype=torch.bfloat16, device="cuda")
    _, dw2 = tn.rms_norm_gradients(dy, s, dev(np.ones(cols)), EPS, dsum=ds, dx=out[:, 3:3 + cols])
    assert torch.equal(out[:, 3:3 + cols], dx) and torch.equal(dw2, dw)
    assert (out[:, :3] == 7).all() and (out[:, 3 + cols:] == 7).all()


def test_several_rows_against_differences():
    """The formula's gradient of more rows than there are workgroups, along a direction, from the kernel's own fp32 forward."""
    rows, cols = 2600, 72
    assert rows > groups_of(rows, cols)
    rng = np.random.default_rng(7)
    x, w, dy = (rounded(v, "f32") for v in (rng.standard_normal((rows, cols)), 1 + 0.2 * rng.standard_normal(cols), rng.standard_normal((rows, cols))))
    dx, dw = tn.rms_norm_gradients(dev(dy, "f32"), dev(x, "f32"), dev(w, "f32"), EPS)
    loss = lambda x_, w_: (host(tn.rms_norm(dev(x_, "f32"), dev(w_, "f32"), EPS).y) * dy).sum()      # noqa: E731
    step = 1e-2                                # (as with few rows: the third-order term and the differences' rounding are each under 1e-3)
    vx, vw = rng.standard_normal((rows, cols)), rng.standard_normal(cols)
    slope = (host(dx) * vx).sum()
    assert abs((loss(x + step * vx, w) - loss(x - step * vx, w)) / (2 * step) - slope) < 2e-3 * np.linalg.norm(host(dx)) * np.linalg.norm(vx)
    slope = (host(dw) * vw).sum()
    assert abs((loss(x, w + step * vw) - loss(x, w - step * vw)) / (2 * step) - slope) < 2e-3 * np.linalg.norm(host(dw)) * np.linalg.norm(vw)
