"""Sizes of the gated projections and their gradients that go through the tiles and shares named beside them: tests on the
GPU run them, and one on the CPU asks the rules whether they still go there."""
# (m, k, n), 8-bit operands: tile, and whether all, the last or none of the tiles are split
EIGHT_BITS = {(3500, 1000, 2041): (256, "none"), (4352, 4104, 2176): (256, "last"), (1500, 8200, 1500): (256, "all"),
              (300, 8200, 700): (128, "all"), (130, 1000, 300): (128, "none")}
# (m, k, n), both weights' gradients by launches of their own beside that of x: the same of the weights' product.
# n of 850 and 851 have 896 columns in the products, so that the second weight begins inside a tile.
GRADIENTS = {(600, 4712, 850): (256, "none"), (610, 4709, 851): (256, "none"), (2127, 3458, 2943): (256, "last")}
# the weights' gradients without that of x
WEIGHTS = {(8200, 2200, 1100): (256, "all"), (610, 4709, 851): (256, "none")}
# one weight's gradient alone
ONE_WEIGHT = {(1200, 4352, 2176): (256, "none"), (4352, 4352, 1024): (256, "all")}
# all gradients, both products in one launch: whether the sums of dx's product are split, and those of the weights'
ONE_LAUNCH = {(300, 264, 520): ("all", "none"), (4352, 4352, 1024): ("none", "last")}
