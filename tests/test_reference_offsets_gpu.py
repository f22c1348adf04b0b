"""Log-probabilities, gradients and the KL term of logits far from zero (needs a B200).  Softmax does not depend on a common offset; fp32 holds the
differences of these rows exactly, so the tolerances are those of test_reference_losses_gpu.py with the sizes of the rows before the
offset, and 2^-53 of the offset for a log-sum-exp that is handed over in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from oracle import reference_oracle as R
from test_reference_losses_gpu import DEV, F32, FORMS, U, check_grad, check_policy, eps, host, pi_tol, placed, policy_case, pref_case, run_policy, run_pref

pytestmark = pytest.mark.gpu
OFFSETS = [2.0 ** 12, -2.0 ** 16, 2.0 ** 18, 3.0 * 2.0 ** 19]


def moved(t, by):
    """t rounded to eighths, and the same `by` further up: exact in fp32 up to 2^21."""
    t = (t.float() * 8).round() / 8
    out = t + by
    assert torch.equal(out.double() - by, t.double())
    return t, out


@pytest.mark.parametrize("by", OFFSETS)
def test_gradient_of_log_probabilities_of_offset_logits(by):
    T, V = 5, 3000
    c = policy_case(T, V, F32, seed=3, masked=False)
    z, far = moved(c["z"], by)
    ids, g = c["ids"].to(DEV), torch.randn(T, generator=torch.Generator().manual_seed(4))
    o = dppo.dppo_token_logp(far.to(DEV), ids)
    d = dppo.dppo_token_logp_bwd(far.to(DEV), ids, o["lse"], g.to(DEV))["dlogits"]
    zh, w = z.double().numpy(), np.abs(g.double().numpy())[:, None]
    want = R.token_logp(zh, c["ids"].numpy())
    assert np.all(np.abs(host(o["logp"]) - want) <= eps(V) + U * np.abs(want))
    check_grad(d, R.logp_gradient(zh, c["ids"].numpy(), g.double().numpy()), w * (pi_tol(zh, V) + abs(by) * 2.0 ** -53), F32)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("by,ref_by", [(b, r) for b in OFFSETS for r in (b, -b, 0.0)])
@pytest.mark.parametrize("ring", [True, False])
def test_policy_loss_of_offset_logits(by, ref_by, form, ring):
    c = policy_case(6, 3000, F32, seed=5, masked=False)
    c["z"], z = moved(c["z"], by)
    c["y"], y = moved(c["y"], ref_by)
    lp = torch.from_numpy(R.token_logp(c["z"].double().numpy(), c["ids"].numpy()))
    c["mu"], c["ref"] = (lp - 0.1).float(), (lp - 0.2).float()
    z = z.to(DEV) if ring else placed(z, 3003, 1)[0]
    o = run_policy(c, form, z=z, y=y.to(DEV), mask=False)
    assert int(o["status"].item()) == 0
    check_policy(c, o, form)


@pytest.mark.parametrize("by", OFFSETS)
def test_preference_loss_of_offset_logits(by):
    c = pref_case([0, 3, 5, 6, 9], 9, 2000, F32, seed=6)
    c["z"], far = moved(c["z"], by)
    c["ref"] = torch.from_numpy(R.token_logp(c["z"].double().numpy(), c["ids"].numpy()) - 0.2).float()
    o, w = run_pref(c, z=far.to(DEV)), R.preference(c["z"].double().numpy(), c["ids"].numpy(), c["cu"].tolist(), np.ones(9, bool), "sigmoid", float(np.float32(0.2)),
                                                    ref_logp=c["ref"].double().numpy())
    coef = np.abs(w["coef"])[:, None]
    # the coefficient: a quarter of beta times what the two sums of nine log-probabilities are off by, and its own rounding
    rel = 0.25 * 0.2 * 9 * (eps(2000) + 2.0 ** -53 * abs(by)) / 0.2 + U
    check_grad(o["dlogits"], w["dlogits"], coef * (pi_tol(c["z"].double().numpy(), 2000) + abs(by) * 2.0 ** -53 + rel), F32)
