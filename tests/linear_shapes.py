"""Sizes at which every tile of the linear layer's products runs its whole loop: sums, rows and columns that end inside a step
or a tile, rows that are read as they are (K a multiple of 8) and rows that are copied, sums by halves and in slices.
test_linear_tiles.py holds them to the rule that picks the tile, test_gpu_linear.py runs them."""

# (M, K, N): (tile, parts of the sum, whether in slices) of the forward
FORWARD16 = {(1300, 1000, 1500): (64, 1, False), (130, 2053, 135): (64, 2, False), (999, 2730, 1000): (64, 2, False),
             (2050, 1064, 3000): (128, 1, False), (2100, 513, 2100): (128, 1, False), (999, 1096, 2730): (128, 2, False),
             (1100, 1290, 2050): (128, 2, False), (3000, 3001, 3000): (256, 1, False), (3000, 3000, 3001): (256, 1, False),
             (70, 8200, 65): (64, 1, True)}

# from 8 bits
FORWARD8 = {(700, 1144, 517): (64, 1, False), (300, 2048, 300): (64, 2, False), (2001, 1160, 2100): (128, 1, False),
            (2040, 2048, 2030): (128, 2, False), (2000, 3048, 2000): (128, 2, False), (4090, 8190, 4090): (256, 1, False),
            (70, 8200, 65): (64, 1, True)}

# (M, K, N): of the gradients' products, with respect to x and to the weights
BACKWARD = {(1000, 1100, 1300): ((64, 1, False), (64, 1, False)), (700, 139, 333): ((64, 1, False), (64, 2, False)),
            (513, 1000, 1100): ((64, 2, False), (64, 1, False)), (2900, 3101, 1490): ((128, 1, False), (128, 1, False)),
            (1500, 1500, 1501): ((128, 2, False), (128, 2, False)), (3001, 2600, 1300): ((128, 1, False), (128, 2, False)),
            (3001, 3003, 3002): ((256, 1, False), (256, 1, False)), (5000, 300, 900): ((64, 1, False), (64, 1, True)),
            (20_000, 130, 500): ((64, 1, False), (64, 1, True)), (70, 65, 8200): ((64, 1, True), (64, 1, False))}
