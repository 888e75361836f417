"""Sizes shared by the tests of projections with 4-bit weights."""

# (kind, tokens, outputs, inputs, group): a call of each form a product has - streamed with each number of pieces and tokens; every tile with its own output,
# with partial sums of ranges and with silu(gate) * up; forwards and transposed ("back")
FORM_CASES = [
    ("plain", 1, 40, 100, 32), ("plain", 33, 6000, 100, 64), ("plain", 33, 10000, 100, 32), ("plain", 33, 25600, 100, 128), ("plain", 8, 8192, 640, 64),
    ("plain", 20, 25600, 640, 32), ("plain", 3, 300, 25600, 128),
    ("gated", 1, 40, 100, 64), ("gated", 33, 6000, 100, 32), ("gated", 33, 10000, 100, 32), ("gated", 5, 1024, 2048, 128), ("gated", 24, 10000, 640, 64),
    ("plain", 77, 40, 100, 128), ("plain", 77, 40, 1000, 32), ("plain", 3000, 520, 100, 64), ("plain", 3000, 40, 2048, 128), ("plain", 130, 25600, 100, 32),
    ("plain", 3000, 40, 5120, 64), ("plain", 200, 25600, 100, 64), ("plain", 4096, 40, 5120, 32), ("plain", 3000, 2600, 100, 32), ("plain", 3000, 520, 2048, 64),
    ("plain", 1000, 10000, 100, 128), ("plain", 3000, 40, 12000, 32), ("plain", 600, 10000, 640, 64),
    ("gated", 77, 40, 100, 32), ("gated", 77, 40, 1000, 128), ("gated", 3000, 300, 100, 64), ("gated", 3000, 40, 2048, 32), ("gated", 130, 12800, 100, 128),
    ("gated", 3000, 40, 5120, 64), ("gated", 200, 12800, 100, 32), ("gated", 4096, 40, 5120, 128), ("gated", 130, 25600, 100, 64), ("gated", 130, 1500, 12000, 32),
    ("gated", 2048, 2600, 100, 64), ("gated", 3000, 40, 12000, 128), ("gated", 400, 5120, 640, 32),
    ("back", 1, 40, 100, 32), ("back", 1, 1500, 100, 64), ("back", 3000, 40, 640, 32), ("back", 3000, 1500, 100, 128), ("back", 777, 40, 5120, 64),
    ("back", 777, 12800, 100, 32), ("back", 1300, 40, 5120, 32), ("back", 1300, 12800, 100, 64), ("back", 777, 40, 12000, 128), ("back", 777, 12800, 300, 32),
    ("back", 2048, 40, 5120, 64), ("back", 3000, 25600, 100, 32), ("back", 600, 640, 10000, 32),
]
