"""Sizes of linear layers whose products run the larger tiles' main loops, and the copies onto
16-byte chunks.  Which of them do is asserted on the host (test_linear_tiles_cpu.py); their results
are checked on the GPU (test_gpu_linear_tiles.py)."""

# m x n x k of a product by element bytes, its tile and whether k is split: each with ragged edges
# of m and n, a rest of k behind the last whole stage, and more stages than twice the tile's depth
PRODUCTS = [
    (2, (3848, 2408, 360), 256, False),
    (2, (2728, 712, 6408), 256, True),
    (2, (2952, 656, 360), 128, False),
    (2, (1104, 264, 3208), 128, True),
    (4, (3848, 3736, 168), 256, False),
    (4, (2728, 712, 6408), 256, True),
    (4, (4128, 712, 168), 128, False),
    (4, (1552, 656, 1608), 128, True),
]

# rows, n_in, n_out off the chunks, large enough for copies onto them; by element bytes the tiles of
# x W^T, dz W and dz^T x
COPIED = [
    ((1409, 1201, 1303), {2: (64, 64, 64), 4: (64, 64, 64)}),
    ((3851, 365, 3739), {2: (256, 128, 128), 4: (256, 64, 64)}),
    ((3851, 3739, 365), {2: (128, 256, 128), 4: (64, 256, 64)}),
    ((365, 3739, 3851), {2: (128, 128, 256), 4: (64, 64, 256)}),
]


def layer_of(which, m, n, k):
    """rows, n_in, n_out of the layer whose forward (0), dx (1) or dweight (2) is m x n x k."""
    return [(m, k, n), (m, n, k), (k, n, m)][which]
