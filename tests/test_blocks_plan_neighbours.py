"""The shapes of tests/test_gpu_wide_neighbours.py reach the kernels that they are there for."""
from blocks_neighbours import EXPERTS, FAR_FEW, FAR_MANY, FEW_TOKENS, LAYER, MANY_TOKENS
from test_blocks_plan import plan  # noqa: F401  (the fixture)


def test_the_shapes_reach_the_kernels_that_they_are_there_for(plan):  # noqa: F811
    for tokens, wide in ((FEW_TOKENS, 0), (MANY_TOKENS, 1)):
        for p in plan([(m, 1, *LAYER, 148, 0) for m in tokens] + [(m, EXPERTS, *LAYER, 148, 1) for m in tokens]):
            assert p["wide"] == wide, tokens
    for (rows, N, K), wide in ((FAR_FEW, 0), (FAR_MANY, 1)):
        for p in plan([(rows, 1, N, K, 148, 0), (rows, 2, N, K, 148, 1)]):
            assert p["wide"] == wide, rows
    # the layer between others has clusters that share K as well as the wide kernel, which takes all of tensor memory
    assert any(p["cut"] > 1 for p in plan([(m, 1, *LAYER, 148, 0) for m in FEW_TOKENS]))
