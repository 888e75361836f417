"""Helpers shared by the tests of the operators around 8-bit projections (marshalling and comparison only)."""
import numpy as np
import torch

import oracle.fp8_oracle as Q

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SIGNIFICANT = {"bf16": 8, "f32": 24}          # bits of the significand


def half_unit(ref, dtype):
    """What one rounding to the type may take off: half a unit in the last place of ref (of its neighbour's, at a power of two)."""
    _, ex = np.frexp(np.abs(ref) * (1 + 2.0 ** -12))      # |ref| < 2^ex: units of 2^(ex - bits)
    return np.exp2(ex - SIGNIFICANT[dtype] - 1.0)


def dev(a, dtype="bf16"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TORCH[dtype])


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def rounded(a, dtype="bf16"):
    """a, rounded to dtype, in 64 bits: what both sides are given."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TORCH[dtype]).to(torch.float64).numpy()


class OnGpu(torch.Tensor):
    """A tensor that says that it is on GPU `gpu`, wherever its memory is: for the checks of arguments."""
    gpu = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.gpu


def on_gpu(t, gpu):
    t = t.as_subclass(OnGpu)
    t.gpu = gpu
    return t


def exponents(scales):
    return scales.contiguous().view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def check_padding(rows8):
    """Codes and scale bytes where there is no value are zero."""
    p = rows8.codes.shape[1] // rows8.segments
    codes = rows8.codes.view(torch.uint8).cpu().numpy().reshape(rows8.rows, rows8.segments, p)
    assert not codes[:, :, rows8.cols:].any()
    blocks = p // 128 * rows8.segments
    assert not rows8.scales.view(torch.uint8).cpu().numpy()[:, blocks:].any()


def check_eight_bit(rows8, ref, segment=0, rel=1e-5):
    """Codes and scales of values that the kernel computed in fp32, each within `rel` of `ref` (64 bits): every block has
    the scale of the reference unless its largest magnitude is that near to a power-of-two step of the scale, every value lies
    within half a step of e4m3 (2^-4 of it, 2^-10 of the scale below the least normal) of the reference, and nearly all codes agree."""
    codes, exps = host(rows8.values(segment)), exponents(rows8.block_scales(segment))
    ref_codes, ref_exps = Q.quantize(ref)
    for shift in (-rel, rel):
        _, near = Q.quantize(ref * (1 + shift))
        ref_exps = np.where(exps == near, near, ref_exps)
    assert np.array_equal(exps, ref_exps)
    got = Q.dequantize(codes, exps)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(codes), ~fine)
    scale = np.repeat(np.exp2(exps.astype(np.float64)), 128, axis=1)[:, :ref.shape[1]]
    bound = (2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * scale) * (1 + 2 * rel) + rel * np.abs(ref)
    assert (np.abs(got - ref)[fine] <= bound[fine]).all()
    differ = (codes != ref_codes)[fine].mean() if fine.any() else 0.0
    assert differ <= 2e-3 + 128.5 * (exps != Q.quantize(ref)[1]).sum() / ref.size, differ


# (gated, out_features, in_features, tokens): a call of each form a product has - every tile with its own output, with partial sums of
# ranges and with silu(gate) * up; streamed with each number of pieces - and tiles of which a workgroup takes several
FORM_CASES = [
    (0, 100, 100, 1), (0, 4100, 100, 1), (0, 25600, 100, 8),
    (0, 520, 256, 2048), (0, 520, 100, 4096), (0, 300, 100, 12000), (0, 12000, 2048, 400), (0, 520, 100, 6000), (0, 12000, 4096, 600),
    (0, 10000, 256, 777), (0, 300, 1000, 12000), (0, 6000, 512, 1700), (0, 10000, 100, 1300), (0, 1500, 2048, 4096), (0, 5120, 100, 3000),
    (0, 300, 3000, 777), (0, 1500, 5120, 200), (0, 2600, 5120, 80), (0, 6000, 12000, 256), (0, 100, 12000, 4096), (0, 4100, 12000, 600),
    (0, 3000, 25600, 300), (0, 6000, 8192, 160), (0, 3000, 12000, 1300), (0, 12000, 12000, 200), (0, 300, 25600, 2048), (0, 1500, 25600, 1000),
    (1, 100, 512, 1), (1, 2600, 512, 1), (1, 8192, 1000, 8),
    (1, 100, 100, 1), (1, 25600, 256, 80), (1, 520, 1000, 6000), (1, 300, 256, 12000), (1, 520, 512, 8192), (1, 25600, 100, 200), (1, 520, 100, 12000),
    (1, 100, 3000, 600), (1, 2048, 5120, 24), (1, 520, 8192, 80), (1, 520, 25600, 400), (1, 5120, 3000, 100), (1, 520, 25600, 777),
    (0, 1500, 100, 4096), (0, 4100, 256, 4096), (0, 2600, 100, 6000), (0, 25600, 4096, 600), (0, 25600, 256, 777), (0, 4100, 1000, 4096),
    (0, 2600, 512, 8192), (0, 4100, 256, 6000), (0, 2600, 2048, 6000), (0, 10000, 100, 3000),
    (1, 8192, 1000, 5), (0, 25600, 1000, 6), (0, 5120, 4096, 16),
    (1, 300, 100, 6000), (1, 12000, 1000, 600), (1, 10000, 1000, 777), (1, 2600, 512, 4096), (1, 16000, 256, 777), (1, 5120, 100, 3000),
]
