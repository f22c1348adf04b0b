"""The give-up path of the bounded waits of the policy loss and of the product with 4-bit weights (needs a B200): with
``test_inject = DPPO_INJECT_NO_COPIES`` the producers issue nothing, every wait runs out after ``wait_limit_us`` and the call returns with
DPPO_STATUS_WAIT_LIMIT; the next call is an ordinary one."""
import time

import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LIMIT_US = 20000


@pytest.mark.parametrize("form", [binding.KL_K3, binding.KL_PI_REF, binding.KL_REF_PI])
@pytest.mark.parametrize("T", [3, 300])
def test_policy_loss_gives_up_and_the_next_call_is_fine(T, form):
    """Rows shared by clusters of CTAs (few rows), and a CTA to a row."""
    g = torch.Generator(device=DEV).manual_seed(5)
    z = 3 * torch.randn((T, 40000), generator=g, device=DEV)
    y = z + 0.3 * torch.randn(z.shape, generator=g, device=DEV)
    ids = torch.randint(0, 40000, (T,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.randn(T, generator=g, device=DEV)
    lp = dppo.dppo_token_logp(z, ids)["logp"]
    kw = dict(ref_logits=y, ref_logp=lp, kl_form=form, wait_limit_us=LIMIT_US)
    want = dppo.dppo_policy_kl_fwd_bwd(z, ids, lp, adv, **kw)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    out = dppo.dppo_policy_kl_fwd_bwd(z, ids, lp, adv, test_inject=binding.INJECT_NO_COPIES, **kw)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    assert int(out["status"].item()) & binding.STATUS_WAIT_LIMIT
    out = dppo.dppo_policy_kl_fwd_bwd(z, ids, lp, adv, **kw)
    assert int(out["status"].item()) == 0 and int(want["status"].item()) == 0
    assert all(torch.equal(out[n], want[n]) for n in ("loss", "kl", "mask", "dlogits"))


@pytest.mark.parametrize("M,K,group", [(1, 2048, 128), (1, 9000, 32), (16, 9000, 64), (61, 2048, 128), (20, 33000, 64)])
def test_product_gives_up_and_the_next_call_is_fine(M, K, group):
    """A CTA and a pair of CTAs to a tile, x whole and in parts, both kinds of products."""
    N = 9000
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn((M, K), generator=g, device=DEV).bfloat16()
    w = dppo.dppo_int4_quantize(torch.randn((N, K), generator=g, device=DEV).bfloat16(), group)
    q, scale = w["q"], w["scale"]
    want, st = dppo.dppo_matvec_int4(x, q, scale, group)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    _, bad = dppo.dppo_matvec_int4(x, q, scale, group, wait_limit_us=LIMIT_US, test_inject=binding.INJECT_NO_COPIES)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    assert int(bad.item()) & binding.STATUS_WAIT_LIMIT
    got, st2 = dppo.dppo_matvec_int4(x, q, scale, group)
    assert int(st.item()) == 0 and int(st2.item()) == 0 and torch.equal(got, want)
