"""Calls of tree_attn at its edges, shared by the GPU tests and the tests without a GPU that say which kernel takes them."""

# sequences, new tokens, heads (of 2 kv-heads), max_len, the kernel: which one is taken goes by max_len, not by the lengths, so that a short sequence can be given to the
# kernel for many rows.  Few rows in groups of 8 and 16; many in one, two and three blocks.
SHAPES = [(1, 1, 4, 1100, "few8"), (1, 5, 4, 1100, "few16"), (8, 30, 8, 5000, "wide"), (4, 40, 8, 6000, "wide"), (6, 64, 12, 2500, "wide")]
