"""The give-up path of the policy loss's bounded waits (needs a B200): with ``test_inject = DPPO_INJECT_NO_COPIES`` the producers issue nothing, every
wait runs out after ``wait_limit_us`` and the call returns with DPPO_STATUS_WAIT_LIMIT; the next call is an ordinary one."""
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
