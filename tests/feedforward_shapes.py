"""Sizes at which every tile of the feed-forward products runs its whole loop: more steps than lie in LDS (and, in
8 bits, than two groups of scales), sums, rows and columns that end inside a step or a tile, rows that are read as
they are (K a multiple of 8) and rows that are copied.  test_feedforward_tiles.py holds them to the rule that picks
the tile, test_gpu_feedforward.py runs them."""

# (M, K, F): tile of the gated block's forward, bf16 and 8 bits
GATED = {(300, 1144, 517): 64, (300, 1100, 500): 64, (999, 1096, 2730): 128, (1100, 1290, 2050): 128,
         (2050, 1064, 3000): 256, (3001, 1301, 2500): 256}

# (M, K, F): tiles of its gradients' products, with respect to x and to the weights
BACKWARD = {(700, 136, 333): (64, 64), (700, 139, 333): (64, 64), (3001, 2600, 1300): (128, 128),
            (2100, 2050, 1030): (128, 128), (3001, 3000, 2100): (256, 256), (2900, 3101, 1490): (256, 256)}

# (M, K, F) with more than 2^31 elements of dg and du together: the same
BACKWARD_LONG = {(20_001, 3_000, 55_000): (256, 256)}

# (M, N, K): tile of the 8-bit product
PRODUCT8 = {(700, 1001, 1300): 64, (2001, 2100, 1160): 128, (4090, 8189, 1300): 256}
