"""Shapes of the GPU tests in which linear_blocks_wide_kernel (many tokens) runs between other kernels, or on rows that lie far apart, by
the kernel that the plan takes for them (tests/test_blocks_plan_neighbours.py holds the plan to that)."""
# tokens of a layer, channels, columns: few and many tokens of one layer, whose widths W4A8 layers take too
LAYER = (4096, 1024)
FEW_TOKENS, MANY_TOKENS = (1, 16, 77), (520, 1100, 2048)
EXPERTS = 4

# 8 MB from a row to the next: rows, channels, columns
FAR_FEW, FAR_MANY = (5, 4112, 272), (520, 4112, 272)
