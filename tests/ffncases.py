"""Sizes that send calls of include/topoep_ffn.h to the kernels that small ones do
not reach: tiles of 256 x 256 with a remainder in each axis and more than six stages of the inner one, and a few rows of
so many weights that every wave has a tile of its own.  tests/test_ffn_launches.py checks
that they do."""
from itertools import accumulate

# T, H, I of dense blocks; what each is for
DENSE_LARGE = [(2050, 456, 2184),      # gate and up
               (2050, 456, 4104),      # the hidden axis' gradient
               (2050, 4104, 456),      # down, and x's gradient
               (450, 2056, 4104),      # the gradients of down
               (450, 2056, 2064)]      # the gradients of up

# T, H, I, E, L, k of routed ones
ROUTED_LARGE = [(2050, 456, 1032, 2, 2, 2),    # gate and up
                (2050, 456, 2056, 2, 2, 2),    # the hidden axis' gradient, with the weights'
                (2050, 2056, 456, 3, 2, 3),    # down, and x's gradient
                (300, 1544, 2824, 3, 3, 2),    # the gradients of down
                (300, 2056, 1032, 2, 2, 1)]    # the gradients of up

# a few rows, dense or 1, 3 and 8 on average for each expert; inner axes of more than four steps of 256 bytes
DENSE_FEW = [(1, 584, 8200), (7, 584, 8200), (15, 584, 8200), (3, 16392, 584), (6, 16392, 584), (16, 16392, 584),
             (3, 584, 520), (6, 520, 584), (16, 584, 584)]
ROUTED_FEW = [(64, 552, 520, 64, 64, 1), (48, 552, 520, 64, 64, 4), (171, 552, 520, 64, 64, 3), (100, 264, 136, 256, 70, 2)]

# M, N, K of the 8-bit product, gated or not
INT8_LARGE = [(2050, 4104, 912, False), (2050, 4368, 912, True)]
INT8_FEW = [(1, 16400, 1104, False), (5, 16400, 1104, False), (16, 16400, 1104, False), (2, 16400, 1104, True),
            (8, 16400, 1104, True), (11, 16400, 1104, True)]
# the groups' ends, N, K, gated
INT8_GROUPS = [([0, 1501, 1502, 4003], 2310, 912, False), ([0, 1501, 1502, 4003], 2182, 912, True)]
# and 64 of them that have none, the mean, three times the mean and none in turn
INT8_GROUPS += [(list(accumulate([0] + [0, mean, 3 * mean, 0] * 16)), 272, 1168, gated)
                for mean in (1, 3, 9) for gated in (False, True)]
