"""Ratios and loss terms at the end of fp32's range (needs a B200): a row whose term is infinite in fp32 is dropped, so that no gradient holds a
NaN; one whose ratio alone is that large is not."""
import numpy as np
import pytest
import torch

from paper_2602_04879_b200 import binding
from test_reference_losses_gpu import BF, F32, FORMS, check_policy, policy_case, run_policy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dtype,V", [(F32, 700), (BF, 20488)])
def test_rows_whose_term_leaves_fp32_are_dropped(dtype, V, form):
    c = policy_case(6, V, dtype, seed=91, masked=False)
    c["adv"] = torch.tensor([1.0, -1.0, -2.0, 0.5, 0.0, -1e30])
    mu = c["mu"].clone()
    c["mu"][1] = mu[1] - 100.0               # r around e^100, A < 0: no clip on that side
    c["mu"][5] = mu[5] - 30.0                # r |A| = 1e43
    c["mu"][3] = mu[3] - 200.0               # r around e^200 with A > 0: clipped, the term is (1 + eps_high) A
    c["mu"][4] = mu[4] - 100.0               # and with A = 0: no term
    o = run_policy(c, form, mask=False, dlogits_f32=True)
    assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW
    k = dict(c, mu=mu.clone(), adv=c["adv"].clone())
    k["mu"][3] = mu[3] - 3.0                 # the same term and gradient, with a ratio that the tolerances can go by
    k["adv"][5] = 0.0
    check_policy(k, o, form, valid=np.array([1, 0, 1, 1, 1, 0], bool), scale=1.0 / 6)


def test_calls_from_several_threads_share_nothing():
    """Few rows, shared by clusters of every size: the first calls of each shape ask the device how many of them it runs."""
    import threading
    cases = [policy_case(T, V, BF, seed=T + V, masked=False) for T, V in ((3, 9000), (30, 20488), (70, 40000), (2, 151936))]
    wrong = []

    def work(i):
        st = torch.cuda.Stream("cuda:0")
        try:
            with torch.cuda.stream(st):
                first = run_policy(cases[i], "pi_ref", mask=False)
                for _ in range(30):
                    o = run_policy(cases[i], "pi_ref", mask=False)
                    if not all(torch.equal(o[n], first[n]) for n in ("loss", "kl", "dlogits")):
                        wrong.append((i, "result"))
                check_policy(cases[i], first, "pi_ref")
        except Exception as e:             # noqa: BLE001 (reported below)
            wrong.append((i, repr(e)[:300]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]
