"""Corners of dppo_sample's documented ranges (needs a B200): the last double below one, temperatures at either end of fp32."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LAST = 1.0 - 2.0 ** -53


def test_last_uniform_before_a_tail_without_weight():
    """The largest uniform number, and a tail of whole chunks whose weights are below 2^-1000: where rounding leaves the running sum at
    or below its target, the token is still one that weighs something."""
    T, V, live = 400, 20000, 12000
    g = torch.Generator().manual_seed(21)
    z = 480.0 + 3.0 * torch.randn((T, V), generator=g)
    z[:, live:] = -250.0 - 12.0 * torch.rand((T, V - live), generator=g)
    for rows in (T, 20):
        out = dppo.dppo_sample(z[:rows].to(DEV), torch.full((rows,), LAST, dtype=torch.float64, device=DEV), K=3)
        ids, logp = out["sampled_ids"].cpu(), out["mu_logp"].cpu()
        assert int(out["status"].item()) == 0
        assert bool((ids >= 0).all()) and bool((ids < live).all())
        # what lies behind it weighs no more than 2^-53 of the mass and the error of the sums, which is less than 1e-11 of it
        w = torch.exp(z[:rows, :live].double() - 480.0)
        behind = torch.stack([w[t, int(ids[t]) + 1:].sum() / w[t].sum() for t in range(rows)])
        assert float(behind.max()) < 2.0 ** -53 + 1e-11 and bool(torch.isfinite(logp).all())


@pytest.mark.parametrize("k", [50, 600])
def test_last_uniform_in_a_list_of_tokens_without_weight(k):
    """top_k lists tokens of weight zero, among them the highest ids: none of them is drawn."""
    T, V = 64, 5000
    g = torch.Generator().manual_seed(22)
    z = -1e4 * (1.0 + torch.rand((T, V), generator=g))
    z[:, 100:130] = 3.0 * torch.randn((T, 30), generator=g)
    out = dppo.dppo_sample(z.to(DEV), torch.full((T,), LAST, dtype=torch.float64, device=DEV), top_k=torch.full((T,), k, dtype=torch.int32, device=DEV), K=k)
    ids = out["sampled_ids"].cpu().numpy()
    assert np.all((ids >= 100) & (ids < 130)) and bool(torch.isfinite(out["mu_logp"]).all()) and int(out["status"].item()) == 0


@pytest.mark.parametrize("tau", [3.4e38, 1e36, 6e35, 4e35, 1e30, 1e-30, 1e-44])
@pytest.mark.parametrize("settings", [{}, {"top_p": 0.6}, {"min_p": 0.5}, {"top_k": 1500}])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures_at_either_end(tau, settings, dtype):
    """Temperatures so high that 2^-1000 of the maximum lies below all floats (a logit of -inf still weighs nothing), and so low that
    only the maximum weighs anything.  The running sums are off by less than 1e-11 of the mass: ids are compared where no
    decision is closer than that."""
    V, K = 6000, 20
    g = torch.Generator().manual_seed(23)
    z = torch.stack([3.0 * torch.randn(V, generator=g), 1e38 * torch.randn(V, generator=g).clamp(-3, 3), torch.full((V,), torch.finfo(dtype).min), torch.zeros(V)])
    z[:, torch.rand(V, generator=g) < 0.7] = float("-inf")
    z = z.to(dtype)
    T = z.shape[0]
    u = torch.rand(T, generator=g, dtype=torch.float64)
    temps = torch.full((T,), tau)
    s = {n: torch.full((T,), v, dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in settings.items()}
    out = dppo.dppo_sample(z.to(DEV), u.to(DEV), temperature=temps.to(DEV), K=K, **{n: v.to(DEV) for n, v in s.items()})
    assert int(out["status"].item()) == 0
    for t in range(T):
        ora = R.sample_row(z[t].float().numpy(), u[t].item(), temperature=temps[t].item(), K=K, **{n: v[t].item() for n, v in s.items()})
        assert np.array_equal(out["mu_topk_ids"][t].cpu().numpy(), ora["top_ids"])
        if ora["margin"] < 1e-11:
            continue
        assert int(out["sampled_ids"][t]) == ora["id"], (t, ora["margin"])
        assert abs(float(out["mu_logp"][t]) - ora["logp"]) <= 2.0 ** -24 * abs(ora["logp"]) + 1e-11
        assert np.all(np.abs(out["mu_topk_p"][t].cpu().numpy() - ora["top_p"]) <= 2.0 ** -24 * ora["top_p"] + 1e-11)
