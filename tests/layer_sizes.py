"""Sizes of the GPU tests that reach the launches which small calls do not; a host test asks the library's
plans whether they do."""

# (N, d, f) of the gated feed-forward block.  Together with the small sizes of test_gpu_layer_ffn.py they reach
# every tile, ring and split of every product that the plans choose.
FFN_PATHS = [
    (15, 3328, 6080), (49, 88, 17288), (55, 1928, 664), (61, 1544, 6152), (64, 1536, 6144), (71, 4704, 9704),
    (261, 8, 11744), (5003, 3584, 14336), (9548, 3560, 232),
]
