"""The rollout-side calls on a stream that is not the current one (needs a B200)."""
import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_calls_on_another_stream_wait_for_nothing_on_the_current_one():
    """While the current stream is busy, the calls run on theirs; what they allocate and clear (the status word) is in order with
    their kernels."""
    g = torch.Generator().manual_seed(31)
    z = torch.randn((6, 3000), generator=g).to(DEV)
    z[2, 5] = float("nan")
    u = torch.rand(6, generator=g, dtype=torch.float64).to(DEV)
    ref = dppo.dppo_sample(z, u, K=4)
    a = dppo.dppo_fp8_quantize(torch.randn((50, 300), generator=g).to(DEV))
    refq = dppo.dppo_fp8_quantize(z)
    refc, _ = dppo.dppo_gemm_tn_fp8(a["q"], a["scale"], a["q"], a["scale"], b_block_rows=1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.cuda.Event()
    torch.cuda._sleep(200_000_000)
    busy.record()
    out = dppo.dppo_sample(z, u, K=4, stream=side)
    q = dppo.dppo_fp8_quantize(z, stream=side)
    C, st = dppo.dppo_gemm_tn_fp8(a["q"], a["scale"], a["q"], a["scale"], b_block_rows=1, stream=side)
    side.synchronize()
    assert not busy.query()
    torch.cuda.synchronize()
    assert int(out["status"].item()) == binding.STATUS_NONFINITE_ROW and int(q["status"].item()) == binding.STATUS_NONFINITE_ROW and int(st.item()) == 0
    assert all(torch.equal(out[n], ref[n]) for n in ("sampled_ids", "mu_logp", "mu_topk_ids", "mu_topk_p"))
    assert torch.equal(q["q"].view(torch.uint8), refq["q"].view(torch.uint8)) and torch.equal(C, refc)


def test_a_status_word_of_another_type_is_refused():
    z, u = torch.zeros((2, 8), device=DEV), torch.zeros(2, dtype=torch.float64, device=DEV)
    for bad in (torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int32)):
        with pytest.raises(AssertionError):
            dppo.dppo_sample(z, u, status=bad)
        with pytest.raises(AssertionError):
            dppo.dppo_fp8_quantize(z, status=bad)
