"""Calls with rows on both sides of the sizes from which norms and rotations take other kernels (test infrastructure)."""

# kind, tokens, q_heads, kv_heads, dim, dims, heads that a lane group of the call takes
ROTATE = [("bf16", 5119, 11, 3, 128, 128, 1), ("bf16", 5120, 11, 3, 128, 128, 8), ("bf16", 3413, 20, 3, 80, 32, 1), ("bf16", 3414, 20, 3, 80, 32, 8),
          ("bf16", 40959, 5, 0, 17, 6, 1), ("bf16", 40960, 5, 0, 17, 6, 8), ("bf16", 20000, 1, 1, 256, 130, 8), ("f32", 4095, 20, 3, 80, 32, 1), ("f32", 4096, 20, 3, 80, 32, 4),
          ("f32", 9000, 11, 3, 128, 64, 1)]

# kind, q_heads, kv_heads, dim, dims, page, rows of the sequences (a row of none follows them), whether queries are launched apart from the cache
APPEND = [("bf16", 12, 2, 128, 128, 64, [9000, 0, 7381, 1], False), ("bf16", 12, 2, 128, 128, 64, [9000, 1, 7381, 1], True), ("bf16", 3, 3, 40, 24, 16, [65534], False),
          ("bf16", 3, 3, 40, 24, 16, [60000, 5535], True), ("f32", 12, 1, 128, 64, 32, [1, 10920], False), ("f32", 12, 1, 128, 64, 32, [10000, 922], True),
          ("f32", 13, 1, 80, 32, 16, [10081], False), ("f32", 13, 1, 80, 32, 16, [81, 10001], True)]


def lanes_of_a_head(dim, dims):
    """Lanes side by side that have a head: a power of two of units of four pairs, and of eight further elements."""
    units = -(-dims // 8) + -(-(dim - dims) // 8)
    return 1 << (units - 1).bit_length()


def workgroups(tokens, heads, each, dim, dims):
    """Of a launch whose lane groups take `each` heads of a token."""
    return -(-tokens * -(-heads // each) // (256 // lanes_of_a_head(dim, dims)))
