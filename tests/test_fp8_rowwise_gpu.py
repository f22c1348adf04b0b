"""Row-wise 8-bit quantisation at sizes on either side of the whole-tile kernel (needs a B200): against the two-way form, which always
takes whole tiles, and against the definition."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows,cols", [(130, 19000), (2300, 2111), (37000, 128), (37760, 100), (128, 37761), (1, 40000), (1700, 2048)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_rowwise_alone_equals_both_ways(rows, cols, dtype, fmt):
    g = torch.Generator().manual_seed(rows)
    x = (torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())).to(dtype)
    xd = x.to(DEV)
    one, both = dppo.dppo_fp8_quantize(xd, fmt), dppo.dppo_fp8_quantize(xd, fmt, transposed=True)
    torch.cuda.synchronize()
    assert int(one["status"].item()) == 0 and torch.equal(one["scale"], both["scale"])
    assert torch.equal(one["q"].contiguous().view(torch.uint8), both["q"].contiguous().view(torch.uint8))
    val, sc, y = R.quantize(x[:140].double().numpy(), "e4m3" if fmt == torch.float8_e4m3fn else "e5m2", 1)
    assert np.array_equal(one["scale"][:140].cpu().numpy(), sc.astype(np.float32))
    got = one["q"][:140].float().cpu().numpy().astype(np.float64)
    bad = got != val                       # fp32 inputs: 7/8 x and the quotient round by 2^-24 each, next to a tie either neighbour will do
    assert not bad.any() or (dtype == torch.float32 and np.all(np.abs(y[bad] - 0.5 * (got[bad] + val[bad])) <= 2.0 ** -23 * np.abs(y[bad])))


@pytest.mark.parametrize("rows,cols", [(1, 151936), (4, 151936), (16, 37889), (64, 40000), (65, 40000), (64, 40007), (200, 40003), (66, 40008)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_rows_of_a_wide_matrix(rows, cols, dtype):
    """Few rows, and rows on no 16-byte boundary, take the kernel with a row per thread however many columns there are."""
    g = torch.Generator().manual_seed(rows + cols)
    xd = (torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())).to(dtype).to(DEV)
    one, both = dppo.dppo_fp8_quantize(xd), dppo.dppo_fp8_quantize(xd, transposed=True)
    assert int(one["status"].item()) == 0 and torch.equal(one["scale"], both["scale"])
    assert torch.equal(one["q"].contiguous().view(torch.uint8), both["q"].contiguous().view(torch.uint8))
