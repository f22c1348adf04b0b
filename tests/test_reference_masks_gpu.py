"""The policy loss with masked vocabularies over rows of several slots of the ring, so that a thread meets masked stretches before, between and
behind live ones, and with the kernel for any layout (needs a B200).  Tolerances: those of test_reference_losses_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from oracle import reference_oracle as R
from paper_2602_04879_b200 import binding
from test_reference_losses_gpu import BF, DEV, F32, FORMS, check_policy, placed, policy_case, run_policy

pytestmark = pytest.mark.gpu
LOWEST_BF16 = torch.finfo(BF).min


def live_entries(kind, T, V, g):
    """Which entries a mask leaves, [T,V] bool: everything behind a long stretch, everything in front of one, one in a hundred, or whole blocks
    of a few thousand by turns; the last two differ from row to row."""
    j = torch.arange(V)[None, :]
    t = torch.arange(T)[:, None]
    if kind == "front":
        return (j >= V * 2 // 5).expand(T, V)
    if kind == "back":
        return (j < V // 3).expand(T, V)
    if kind == "few":
        return torch.rand((T, V), generator=g) < 0.01
    return (j // 4100 + t) % 3 == 0


def masked_case(kind, T, V, dtype, seed):
    c = policy_case(T, V, dtype, seed=seed, masked=False)
    g = torch.Generator().manual_seed(seed + 1)
    live = live_entries(kind, T, V, g).clone()
    for t in range(T):
        some = torch.nonzero(live[t])[:, 0]
        # half of the tokens the likeliest that is live, half of them any
        c["ids"][t] = some[int(c["z"][t, some].float().argmax())] if t % 2 else some[int(torch.randint(0, len(some), (1,), generator=g))]
    return c, live


def with_mask(c, live, value, in_z, in_y):
    """The case with `value` in the entries that are not live, and the rows as the oracle is to see them."""
    c = dict(c, z=c["z"].clone(), y=c["y"].clone())
    for name, yes in (("z", in_z), ("y", in_y)):
        if yes:
            c[name][~live] = value
    h = {n: c[n].double().numpy() for n in ("z", "y")}
    for n in h:
        h[n][h[n] <= LOWEST_BF16] = -np.inf
    lp = torch.from_numpy(R.token_logp(h["z"], c["ids"].numpy()))
    c["mu"], c["ref"] = (lp - 0.1).float(), (lp - 0.2).float()
    return c, h["z"], h["y"]


SIZES = [(3, 151936, BF), (3, 60000, F32), (150, 20488, BF), (150, 9000, F32)]
VALUES = [float("-inf"), "lowest", -3e38, -1e38, -1e9]


@pytest.mark.parametrize("kind", ["front", "back", "few", "blocks"])
@pytest.mark.parametrize("T,V,dtype", SIZES)
def test_vocabulary_masked_alike_in_both_policies(T, V, dtype, kind):
    case, live = masked_case(kind, T, V, dtype, seed=V + T)
    for value in VALUES:
        value = torch.finfo(dtype).min if value == "lowest" else value
        c, zh, yh = with_mask(case, live, value, True, True)
        for form in FORMS:
            o = run_policy(c, form, mask=False, dlogits_f32=True)
            assert int(o["status"].item()) == 0, (form, value)
            check_policy(c, o, form, zh=zh, yh=yh)


@pytest.mark.parametrize("kind", ["front", "back", "few", "blocks"])
@pytest.mark.parametrize("T,V,dtype", SIZES)
def test_vocabulary_masked_in_the_policy_alone(T, V, dtype, kind):
    """KL(pi || rho) is finite, and so is k3; KL(rho || pi) is infinite where the mask is."""
    case, live = masked_case(kind, T, V, dtype, seed=V + T + 10)
    for value in VALUES:
        value = torch.finfo(dtype).min if value == "lowest" else value
        c, zh, yh = with_mask(case, live, value, True, False)
        for form in ("pi_ref", "k3"):
            o = run_policy(c, form, mask=False, dlogits_f32=True)
            assert int(o["status"].item()) == 0, (form, value)
            check_policy(c, o, form, zh=zh, yh=yh)
        if value < -1e37:
            o = run_policy(c, "ref_pi", mask=False)
            assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW, value
            assert float(o["loss"].item()) == 0 and not o["kl"].any() and not o["dlogits"].any()


@pytest.mark.parametrize("T,V,dtype", SIZES)
def test_vocabulary_masked_in_the_reference_alone(T, V, dtype):
    case, live = masked_case("blocks", T, V, dtype, seed=V + T + 20)
    for value in (float("-inf"), -3e38):
        c, zh, yh = with_mask(case, live, value, False, True)
        o = run_policy(c, "pi_ref", mask=False)
        assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW
        assert float(o["loss"].item()) == 0 and not o["kl"].any() and not o["dlogits"].any()
        o = run_policy(c, "ref_pi", mask=False, dlogits_f32=True)
        assert int(o["status"].item()) == 0
        check_policy(c, o, "ref_pi", zh=zh, yh=yh)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("alone", [False, True])
def test_masked_vocabulary_in_rows_off_16_byte_boundaries(dtype, alone):
    """The kernel for any layout."""
    T, V = 5, 20001
    for kind in ("front", "few"):
        case, live = masked_case(kind, T, V, dtype, seed=77)
        for value in (float("-inf"), -3e38, -1e38):
            c, zh, yh = with_mask(case, live, value, True, not alone)
            z, _ = placed(c["z"], V + 2, 1)
            for form in ("pi_ref", "k3") if alone else FORMS:
                o = run_policy(c, form, z=z, mask=False, dlogits_f32=True)
                assert int(o["status"].item()) == 0, (form, value)
                check_policy(c, o, form, zh=zh, yh=yh)


def test_masked_log_probabilities_of_long_rows():
    for dtype in (BF, F32):
        case, live = masked_case("front", 4, 151936, dtype, seed=5)
        for value in VALUES:
            c, zh, _ = with_mask(case, live, torch.finfo(dtype).min if value == "lowest" else value, True, False)
            o = dppo.dppo_token_logp(c["z"].to(DEV), c["ids"].to(DEV))
            want = R.token_logp(zh, c["ids"].numpy())
            assert int(o["status"].item()) == 0
            assert np.all(np.abs(o["logp"].double().cpu().numpy() - want) <= (151936 / 512 + 96) * 2.0 ** -24 + 2.0 ** -24 * np.abs(want))
