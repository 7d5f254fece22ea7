"""Sizes of the GPU tests that reach the launches which small calls do not; a host test asks the library's
plans whether they do."""

# (N, d, f) of the gated feed-forward block.  Together with the small sizes of test_gpu_layer_ffn.py they reach
# every tile, ring and split of every product that the plans choose.
FFN_PATHS = [
    (15, 3328, 6080), (49, 88, 17288), (55, 1928, 664), (61, 1544, 6152), (64, 1536, 6144), (71, 4704, 9704),
    (261, 8, 11744), (5003, 3584, 14336), (9548, 3560, 232),
]

# (N, heads of queries, of keys, D, rot, interleaved, type) of the head norms.  Every width class of a head (lanes
# 1 to 64) in both types, through the caches and past them: calls whose waves take several passes (forward) and
# several tokens (backward).
_F, _B = "f32", "bf16"
QK_PATHS = [
    (8203, 130, 65, 8, 0, False, _B), (8209, 70, 3, 8, 0, False, _F),
    (8203, 70, 33, 16, 16, False, _B), (8209, 61, 40, 16, 16, True, _F),
    (8203, 50, 17, 24, 16, False, _B), (8209, 33, 18, 32, 32, False, _F),
    (8203, 35, 9, 64, 64, False, _B), (8209, 17, 9, 56, 32, True, _F),
    (8203, 17, 5, 128, 128, False, _B), (8209, 10, 3, 72, 64, False, _F),
    (8203, 7, 3, 256, 64, False, _B), (8209, 4, 2, 200, 192, True, _F),
    (8203, 3, 2, 512, 512, False, _B), (8209, 2, 1, 264, 256, False, _F),
    (9001, 600, 61, 8, 0, False, _B), (9001, 400, 200, 8, 0, False, _F),
    (9001, 280, 70, 16, 16, True, _B), (9001, 200, 100, 16, 16, False, _F),
    (9001, 140, 30, 32, 32, False, _B), (9001, 140, 50, 24, 16, False, _F),
    (9001, 70, 20, 56, 48, False, _B), (9001, 35, 9, 64, 64, False, _F),
    (28481, 28, 4, 128, 128, False, _B), (9001, 21, 4, 128, 128, False, _F),
    (9001, 20, 6, 200, 64, True, _B), (9001, 9, 2, 256, 256, False, _F),
    (9001, 9, 2, 512, 128, False, _B), (9001, 5, 2, 512, 512, True, _F),
]

# (N, d, type in, type out, residual) of dropout calls past the caches.
DROP_PAST = [
    (30011, 2056, _B, _B, True), (30011, 2056, _F, _F, True), (30011, 2056, _B, _B, False),
    (30011, 2056, _F, _F, False), (30011, 2056, _F, _B, False), (30011, 2056, _B, _F, False),
]
