"""CPU-only: refusals of the policy loss that its neighbours make too."""
from test_reference_host_logic import B, _policy  # noqa: F401 (B: the fixture)


def test_policy_refuses_a_negative_wait_limit(B):  # noqa: F811
    assert _policy(B, opts=B.DppoOpts(wait_limit_us=-1)) == -11
    assert _policy(B, T=0, opts=B.DppoOpts(wait_limit_us=-5)) == -11
