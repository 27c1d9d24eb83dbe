"""Sums of attention weights: queries that saw nothing."""
import numpy as np
import pytest
import torch

from test_gpu_evict import check_weights, weights_case

pytestmark = pytest.mark.gpu

# heads and the queries of three requests, one for each kernel: one query a request (whole rows of four and eight heads where they are in 4 bits), several queries in one
# block of columns, many over short lists, many by tiles
QUERIES = [(8, 8, [1, 1, 1]), (8, 4, [1, 1, 1]), (6, 3, [5, 2, 4]), (8, 2, [30, 9, 3]), (40, 2, [2, 1, 3]), (4, 1, [19, 40, 2])]


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("hq,hkv,queries", QUERIES)
def test_a_query_that_saw_nothing_gives_nothing_whatever_it_holds(cuda, hq, hkv, queries, positions, bits):
    """Rows behind the last query of a padded batch: LSE = -inf, and q was never written."""
    c = weights_case(cuda, [300, 77, 131], queries, hq, hkv, bits, hq, positions)
    nothing = np.arange(sum(queries)) % 2 == 1
    c["LSE"][nothing] = -np.inf
    c["LSE"][0, hq // 2] = -np.inf                                    # and one head of a query
    c["q"][nothing] = 0
    c["q"][0, hq // 2] = 0
    c["q_dev"][torch.from_numpy(nothing).to(cuda)] = float("nan")
    c["q_dev"][0, hq // 2, ::2] = float("inf")
    check_weights(c, decay=0.5, by_offsets=True)
