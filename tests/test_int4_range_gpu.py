"""The 4-bit product over the range of its inputs (needs a B200): tolerances as in test_int4_gpu.py, (K + 3) 2^-23 of the sum of the terms'
magnitudes, whatever the entries of x beside one another are, and half a step of the output type."""
import pytest
import torch

import paper_2602_04879_b200 as dppo
from test_int4_gpu import DEV, F32, check_product, packed, product_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,group,N", [(33, 2048, 128, 40000), (48, 2048, 64, 40000), (61, 700, 128, 60000), (64, 4096, 64, 20000)])
def test_product_of_33_to_64_rows_by_pairs_of_ctas_repeats(M, K, group, N):
    """Tens of tiles to a pair of CTAs, whose exchanged sums are read while the other goes on to the next tile: the same bits every time, and the
    right ones."""
    x, codes, scale = product_case(M, N, K, group, seed=3 * M + K)
    q, s, xd = packed(codes), scale.to(DEV), x.to(DEV)
    cols = torch.arange(0, N, N // 100)
    a, st = dppo.dppo_matvec_int4(xd, q, s, group)
    assert int(st.item()) == 0
    check_product(a[:, cols.to(DEV)], x, codes[cols], scale[cols], group, F32)
    for _ in range(40):
        assert torch.equal(dppo.dppo_matvec_int4(xd, q, s, group)[0], a)
