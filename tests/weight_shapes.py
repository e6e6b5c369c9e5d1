"""Sizes of weight gradients that reach each of the kernel's workgroup shapes (waves and tiles along the channels, then along
the outputs), as (shape, slots an expert has, width, outputs, types).  test_slot_rules.py has the library's rule say so for
each; test_gpu_weight_shapes.py runs them."""

# from one slot over the ends of a step (32 or 64 slots) to an expert that hundreds of ranges share
FEW = [1, 33, 0, 65, 32, 64, 31, 130]
MANY = FEW + [200_003, 1000, 0, 80_001]
EXPERTS = [700 + 37 * i for i in range(70)] + [150_000, 0, 1]        # more than the 64 that a wave knows at a time
TYPES = ("f32", "bf16", "f16")

CASES = [
    ((4, 2, 2, 4), MANY, 256, 256, TYPES),                # one whole tile
    ((4, 2, 2, 4), MANY, 200, 250, TYPES),                # a tile that ends inside a chunk of outputs
    ((4, 2, 2, 4), EXPERTS, 129, 131, TYPES),
    ((4, 2, 2, 4), FEW + [50_000, 3], 300, 515, TYPES),   # six tiles
    ((2, 2, 4, 2), MANY, 128, 256, TYPES),
    ((2, 2, 4, 2), MANY, 100, 250, TYPES),
    ((2, 2, 4, 2), EXPERTS, 33, 133, TYPES),
    ((2, 2, 4, 2), FEW + [150_000, 3], 7, 300, TYPES),    # two tiles
    ((2, 2, 2, 2), MANY, 128, 128, ("f32", "f16")),
    ((2, 2, 2, 2), MANY + [300_000], 128, 128, ("bf16",)),
    ((2, 2, 2, 2), MANY, 100, 101, ("f32", "f16")),
    ((2, 2, 2, 2), EXPERTS + [300_000], 65, 67, ("bf16",)),
    ((2, 2, 2, 2), FEW + [3000, 5], 640, 650, TYPES),     # many tiles, few slots
    ((2, 2, 2, 1), FEW + [3000], 128, 128, ("f32", "f16")),
    ((2, 2, 2, 1), EXPERTS, 100, 47, TYPES),
    ((1, 2, 4, 1), FEW + [3000], 128, 128, ("bf16",)),
    ((1, 2, 4, 1), EXPERTS, 47, 100, TYPES),
    ((2, 1, 2, 1), EXPERTS, 40, 43, TYPES),
    ((4, 1, 1, 1), EXPERTS, 100, 31, TYPES),
    ((4, 1, 1, 1), EXPERTS, 100, 7, TYPES),               # fewer outputs than a chunk
]
PARAMS = [(shape, sizes, width, out, dtype) for shape, sizes, width, out, types in CASES for dtype in types]
IDS = ["x".join(map(str, shape)) + f"-{sum(sizes)}in{len(sizes)}-{width}x{out}-{dtype}"
       for shape, sizes, width, out, dtype in PARAMS]
EMPTY = 77                      # slots behind the last expert's
