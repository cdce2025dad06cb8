"""The weight stream of the experts' products for a few rows (forward) at sizes where several warps share an output, where a
warp's ring of copies goes round and on into its next outputs, and where an expert's weights are read more than once."""
import pytest
import torch

import paper_2209_13258_b200 as P
from test_gpu_experts import Problem

pytestmark = pytest.mark.gpu

# warps to an output (WK), stages of 64 of K for each, on 148 SMs; the ring has four stages
STREAMED = [
    (1, 2, 8, "even", 8192, 2048),      # one token's first layer: WK 2, 16 stages
    (1, 2, 8, "even", 2048, 8192),      # its second layer: WK 8, 16 stages
    (8, 8, 8, "even", 512, 1024),       # WK 8, two stages; every expert has eight rows
    (1, 1, 4, "even", 136, 1032),       # WK 8: 3 3 3 3 3 2 0 0 stages, and K ends inside one
    (3, 2, 4, "skewed", 72, 840),       # WK 4: 4 4 4 2
    (7, 1, 1, "one", 24, 8200),         # WK 16, the last warp with nothing
    (5, 3, 9, "holes", 1000, 600),      # WK 4: 3 3 3 1; dropped choices
    (8, 2, 64, "skewed", 8192, 264),    # WK 1, a warp walks several outputs; 5 stages
    (8, 4, 32, "holes", 4104, 2056),    # WK 2, a group walks several outputs; 17 and 16 stages
    (8, 8, 8, "even", 4096, 4104),      # WK 4, a group walks several outputs
    (8, 16, 16, "one", 1024, 520),      # WK 2: 128 rows of one expert, 16 readings of its weights
    (8, 2, 3, "one", 40, 3336),         # WK 16: 16 rows of one expert, two readings
    (33, 1, 3, "skewed", 200, 2600),    # WK 16: 3 ... 3 2 0 0; from here on 16 rows to a reading
    (100, 1, 16, "one", 512, 512),      # WK 4: 100 rows of one expert, seven readings
    (64, 2, 16, "one", 128, 2048),      # WK 16: 128 rows, eight readings
    (64, 2, 16, "skewed", 128, 2048),
    (79, 2, 68, "one", 480, 400),       # WK 1, 7 stages: 158 rows, ten readings
    (79, 2, 68, "holes", 480, 400),
    (48, 2, 16, "skewed", 8, 12000),    # WK 16, 12 stages, half an output
    (512, 1, 32, "one", 256, 8192),     # too many readings in the worst case: the tile kernel
    (200, 1, 20, "one", 136, 4096),
]


@pytest.mark.parametrize("T,k,E,how,N,K", STREAMED)
def test_shared_outputs_rings_and_readings(T, k, E, how, N, K):
    p = Problem(T, k, E, how, N, K, seed=1)
    for act in (P.ACT_NONE, P.ACT_GELU_TANH):
        p.check_forward(act)


def test_the_same_bits_again():
    """The warps' sums meet in a fixed order."""
    p = Problem(8, 2, 8, "skewed", 2048, 4104, seed=2)
    first = p.forward(P.ACT_GELU_TANH, save=True)
    for _ in range(20):
        again = p.forward(P.ACT_GELU_TANH, save=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
