"""Sizes at which the cross entropy's tiled kernels have tiles of 256, of 128 and
of both, its classes in one piece and in several, forward and backward: (rows,
columns, classes, types of x, the weight and dweight, tile and pieces forward,
tile of the logits and of the products and pieces backward; None: not run)."""

F, B = "f32", "bf16"

TILES = [
    ([2100, 1500], 1030, 8200, B, B, B, (256, 1), None),
    ([2100], 1700, 8200, F, F, F, (256, 1), (256, 256, 1)),
    ([2100, 0, 700], 1701, 8201, B, F, F, (256, 1), (256, 256, 1)),
    ([2050, 1], 3301, 8193, B, B, B, (256, 1), (256, 256, 1)),
    ([1270], 3300, 17001, F, B, B, (256, 1), (256, 256, 1)),
    ([2300], 2400, 8200, B, F, B, (256, 1), (256, 256, 1)),
    # the logits' sums are short, the gradients' long
    ([901, 450], 1003, 30011, B, F, F, (256, 1), (128, 256, 1)),
    ([531], 1088, 16853, B, B, F, (128, 1), (128, 128, 1)),
    # several pieces: labels in each, the last one shorter, and not of whole tiles
    ([4096, 17], 4100, 33201, B, B, B, (256, 3), (256, 256, 1)),
    ([4000], 3301, 40001, F, F, F, (256, 3), (256, 256, 2)),
]
