"""Sizes at which the feed-forward products take each of their tiles, with workgroups that go on to further tiles of several steps, ragged last tiles, and splits: what test_ffn_tiles_host
holds the plans to and test_gpu_ffn_tiles computes.  Tiles are rows x columns of products; of the gated unit's, half of the columns belong to either matrix."""

# rows, in_dim, out_dim, group, fmt, scales, out; (rows, columns) of a tile, whether there are more tiles than compute units, whether the last ones are split
LINEAR = [
    ((4100, 640, 4100, 128, "fp8", "fp32", "bf16"), (256, 128), True, False),
    ((4100, 384, 6001, 128, "fp8", "bf16", "bf16"), (256, 256), True, False),
    ((4100, 384, 4100, 128, "fp8", "fp32", "bf16"), (128, 128), True, False),
    ((8200, 384, 133, 128, "int4", "fp32", "bf16"), (128, 128), False, False),
    ((4100, 768, 4100, 256, "fp8", "bf16", "bf16"), (256, 128), True, False),
    ((4100, 2048, 4100, 128, "int4", "fp32", "bf16"), (256, 128), True, True),
    ((8200, 2048, 4100, 128, "fp8", "fp32", "bf16"), (256, 256), True, True),
    ((8200, 384, 1500, 128, "fp8", "fp32", "fp32"), (256, 128), True, False),
    ((8200, 2048, 1030, 128, "fp8", "bf16", "fp32"), (256, 128), True, True),
    ((8200, 400, 1500, 400, "fp8", "fp32", "fp32"), (256, 128), True, False),
    ((1030, 2048, 4100, 128, "int4", "fp32", "fp32"), (128, 128), True, True),
    ((777, 4096, 4100, 128, "fp8", "fp32", "bf16"), (128, 128), False, False),
]
# rows, in_dim, width, group, fmt, scales, act; the same.  Forward and, of the products that are computed again, backward.
GATED = [
    ((8200, 384, 1500, 128, "fp8", "fp32", "silu"), (256, 128), True, False),
    ((8200, 400, 1500, 400, "fp8", "bf16", "gelu"), (256, 128), True, False),
    ((8200, 512, 1501, 256, "int4", "fp32", "silu"), (256, 128), True, False),
    ((8200, 384, 1030, 128, "fp8", "fp32", "gelu"), (128, 128), True, False),
    ((777, 2048, 4100, 128, "fp8", "bf16", "silu"), (128, 128), False, False),
]
# matrices, rows, in_dim, width of the gradients of some of these; the tiles' shape (0 .. 3: 128 x 128, 128, 192, 256 x 256), whether grad_input's and grad_weights' last tiles are split
GRADIENTS = [
    ((1, 4100, 640, 4100), 0, True, True),
    ((1, 8200, 384, 133), 0, False, True),
    ((2, 8200, 384, 1500), 0, False, True),
    ((1, 1030, 2048, 4100), 2, True, False),
    ((2, 8200, 512, 1501), 2, False, True),
    ((1, 777, 4096, 4100), 3, True, True),
    ((1, 8200, 2048, 4100), 3, True, True),
    ((2, 777, 2048, 4100), 3, True, True),
]
