"""The 4-bit product over the range of its inputs (needs a B200): tolerances as in test_int4_gpu.py, (K + 3) 2^-23 of the sum of the terms'
magnitudes, whatever the entries of x beside one another are, and half a step of the output type."""
import pytest
import torch

import paper_2602_04879_b200 as dppo
from test_int4_gpu import BF, DEV, F32, check_product, packed, product_case

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


def outlier_case(M, N, K, group, seed, lift, code):
    """x with an entry of 2^lift beside standard normal ones in each group, at another place in each, whose weights' codes are `code`."""
    x, codes, scale = product_case(M, N, K, group, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    x = torch.randn((M, K), generator=g).to(BF)
    for k0 in range(0, K, group):
        k = k0 + int(torch.randint(0, min(group, K - k0), (1,), generator=g))
        x[:, k] = 1.5 * 2.0 ** lift
        codes[:, k] = code
    return x, codes, scale


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 16])
@pytest.mark.parametrize("K,group,N", [(2048, 128, 300), (777, 64, 300), (1024, 32, 300), (9000, 32, 200)])
def test_product_with_an_entry_that_stands_out_of_its_group(M, K, group, N):
    """Where the large entry's weight is zero its group's sum is that of the others, and an fp32 sum has it to their last place."""
    for lift in (0, 8, 12, 16, 20, 22, 24, 30, 60, 120):
        x, codes, scale = outlier_case(M, N, K, group, 17 * M + lift, lift, 8)
        y, st = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
        assert int(st.item()) == 0
        check_product(y, x, codes, scale, group, F32)


@pytest.mark.parametrize("M", [1, 4, 5])
@pytest.mark.parametrize("K,group", [(2048, 128), (777, 64), (500, 32)])
def test_product_with_entries_of_every_size(M, K, group):
    """Magnitudes spread evenly over their exponents, by which a few entries of a group make up its sum, whichever codes they meet."""
    N = 300
    for low, high in ((-40, 0), (-100, 20), (0, 60), (-130, -90)):
        x, codes, scale = product_case(M, N, K, group, seed=high)
        g = torch.Generator().manual_seed(M + high)
        x = (torch.randn((M, K), generator=g) * torch.exp2(low + (high - low) * torch.rand((M, K), generator=g))).to(BF)
        codes[: N // 2][:, x[0].abs().float() > 2.0 ** ((low + high) / 2)] = 8
        y, st = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
        assert int(st.item()) == 0
        check_product(y, x, codes, scale, group, F32)


@pytest.mark.parametrize("M", [1, 3, 5])
@pytest.mark.parametrize("x_by,scale_by", [(-110, 0), (-110, 40), (-125, 60), (-60, -40), (100, -100), (112, -30)])
def test_product_of_tiny_and_huge_numbers(M, x_by, scale_by):
    """Results within fp32's ordinary range from x and scales that are not.  (The sums of groups are in it too: 64 terms of at most 4.5 x 2^3 x 8 x
    2^112 are below 2^127.)"""
    N, K, group = 200, 700, 64
    x, codes, scale = product_case(M, N, K, group, seed=x_by + 200)
    x, scale = (x.float() * 2.0 ** x_by).to(BF), (scale.float() * 2.0 ** scale_by).to(BF)
    y, st = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
    assert int(st.item()) == 0
    check_product(y, x, codes, scale, group, F32)
