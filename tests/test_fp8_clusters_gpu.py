"""8-bit products whose tiles are shared along K by clusters of every size from two to eight CTAs, odd ones among them, whose shares of the
tile's rows and of the blocks differ (needs a B200).  Tolerance: 128 + blocks + 3 roundings of 2^-23 of the terms' magnitudes, as one
rounding per addition in the tensor cores and the fp32 sums, and one more for each CTA's part."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("M,N,K", [(921, 1998, 6000), (546, 1001, 1500), (984, 1058, 6000), (53, 2724, 1500), (551, 512, 2500), (214, 2791, 6000),
                                   (430, 448, 6000), (365, 1288, 6000), (865, 182, 2500), (523, 546, 6000), (59, 1660, 6000), (50, 2711, 6000), (30, 1215, 2500),
                                   (1362, 772, 4100), (546, 1001, 9000), (775, 377, 9000), (302, 576, 4100), (346, 1280, 9000), (200, 2048, 20000)])
@pytest.mark.parametrize("b_br,out", [(128, torch.float32), (1, torch.bfloat16)])
def test_tiles_shared_by_clusters_of_any_size(M, N, K, b_br, out):
    g = torch.Generator().manual_seed(M + N)
    a = dppo.dppo_fp8_quantize(torch.randn((M, K), generator=g).to(DEV), torch.float8_e5m2)
    b = dppo.dppo_fp8_quantize(torch.randn((N, K), generator=g).to(DEV), block_rows=b_br)
    wide = torch.full((M + 1, N + 5), -3.0, dtype=out, device=DEV)
    C, status = dppo.dppo_gemm_tn_fp8(a["q"], a["scale"], b["q"], b["scale"], 1, b_br, C=wide[:M, :N])
    again, _ = dppo.dppo_gemm_tn_fp8(a["q"], a["scale"], b["q"], b["scale"], 1, b_br, out)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(again, C) and bool((wide[:, N:] == -3).all()) and bool((wide[M] == -3).all())
    host = lambda q: q.float().cpu().numpy().astype(np.float64)  # noqa: E731
    ref, mag = R.product(host(a["q"]), a["scale"].double().cpu().numpy(), 1, host(b["q"]), b["scale"].double().cpu().numpy(), b_br)
    step = 2.0 ** -24 if out == torch.float32 else 2.0 ** -8
    tol = (128 + -(-K // 128) + 3 + 8) * 2.0 ** -23 * mag + step * np.abs(ref)
    assert np.all(np.abs(C.double().cpu().numpy() - ref) <= tol)
