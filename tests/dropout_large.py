"""Sizes at which dropout goes past the caches (more than 256 MB, rows on whole 16
bytes), and at which a lane has more than one turn of two vectors: (rows, columns,
type, residual, elements behind a row, past the caches)."""

LARGE = [
    ([2100, 0, 6400], 4096, "f32", False, 0, True),
    ([8500], 4096, "f32", True, 8, True),
    ([4200, 4200, 4199, 4201], 4096, "bf16", False, 0, True),
    ([11500, 3], 4104, "bf16", True, 8, True),
    # rows that end inside a vector, or begin between 16 bytes: through the caches
    ([34000, 11], 1003, "f32", True, 5, False),
    ([70000], 1003, "bf16", False, 0, False),
    ([45000], 1003, "bf16", True, 3, False),
    ([36000], 1000, "f32", False, 3, False),
]
