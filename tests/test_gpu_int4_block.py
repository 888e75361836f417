"""The example that runs the operators together: an MLP block with frozen 4-bit projections forwards and back, and a step of its adapter."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "int4_finetune.py")


def test_block_and_its_step():
    """A rounding to bf16 is off by 2^-8 / sqrt(3) = 0.23 % in the mean square at the most. The longest way has gate and up, their product, its projection or
    gradient, two sums and a factorised layer's three steps: 8 of them one after another, and silu's slope, which is below 1.1, twice as often in the gradients: below 16 of
    them even if all went one way. The norm of the gradients is off by no more than they are. A first step moves each master by lr * g / (|g| + eps), which fp32
    rounds at the master's size: 2^-24 * 4 / lr = 2.4e-4."""
    spec = importlib.util.spec_from_file_location("int4_finetune", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    for hidden, width, tokens, group in ((640, 1300, 77, 128), (256, 512, 1, 32), (512, 384, 300, 64)):
        errors = module.check(hidden, width, tokens, group)
        assert errors.pop("move") <= 1e-3, errors
        assert all(e < 16 * 2.0 ** -8 / 3 ** 0.5 for e in errors.values()), errors


def test_the_way_back_has_the_weights_of_the_way_there():
    """A checkpoint's fp16 scales have more bits than bf16 holds."""
    import torch

    import paper_2602_01613_amd as tn
    spec = importlib.util.spec_from_file_location("int4_finetune", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    gen = torch.Generator().manual_seed(5)
    codes = torch.randint(0, 256, (48, 150), generator=gen, dtype=torch.uint8).cuda()
    scales = torch.rand((48, 10), generator=gen).half().cuda()
    layer = tn.Int4Linear([codes], 4, group=32, scales=[scales])
    back = module.Block._transposed(layer)
    assert all(torch.equal(a, b) for a, b in zip(back.quantized_tensor(), layer.quantized_tensor()))
    assert torch.equal(back.quantized_tensor()[1], scales.float())
