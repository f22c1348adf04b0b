"""CPU-only checks of the losses against a reference policy and the 4-bit weights: refusals before anything is launched, and the
float64 restatement against differences and library routines."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import reference_oracle as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def B():
    from paper_2602_04879_b200 import build
    build.build_library()
    from paper_2602_04879_b200 import binding as b
    return b


def _logp(B, **over):
    a = dict(z=0x100000, T=4, V=64, ld=64, dt=B.BF16, ids=0x20000, tok=None, lp=0x30000, lse=0x40000, status=0x50000)
    a.update(over)
    return B.lib().dppo_token_logp(P(a["z"]), a["T"], a["V"], a["ld"], a["dt"], P(a["ids"]), P(a["tok"]), P(a["lp"]), P(a["lse"]), P(a["status"]), None)


def _bwd(B, **over):
    a = dict(z=0x100000, T=4, V=64, ld=64, dt=B.BF16, ids=0x20000, tok=None, lse=0x40000, c=0x30000, odt=0, d=0x200000, ldd=64, status=0x50000)
    a.update(over)
    return B.lib().dppo_token_logp_bwd(P(a["z"]), a["T"], a["V"], a["ld"], a["dt"], P(a["ids"]), P(a["tok"]), P(a["lse"]), P(a["c"]), a["odt"], P(a["d"]),
                                       a["ldd"], P(a["status"]), None)


def _policy(B, **over):
    a = dict(z=0x100000, T=4, V=64, ld=64, dt=B.BF16, y=0x300000, ldy=64, ref=0x21000, ids=0x20000, mu=0x22000, adv=0x23000, tok=None, form=B.KL_PI_REF, beta=0.1,
             lo=0.2, hi=0.2, opts=None, loss=0x30000, kl=0x31000, mask=0x32000, d=0x200000, ldd=64, stats=None, status=0x50000, ws=0x60000, n=1 << 20)
    a.update(over)
    o = a["opts"]
    return B.lib().dppo_policy_kl_fwd_bwd(P(a["z"]), a["T"], a["V"], a["ld"], a["dt"], P(a["y"]), a["ldy"], P(a["ref"]), P(a["ids"]), P(a["mu"]), P(a["adv"]),
                                          P(a["tok"]), a["form"], a["beta"], a["lo"], a["hi"], ctypes.byref(o) if o is not None else None, P(a["loss"]),
                                          P(a["kl"]), P(a["mask"]), P(a["d"]), a["ldd"], P(a["stats"]), P(a["status"]), P(a["ws"]), a["n"], None)


def _pref(B, **over):
    a = dict(z=0x100000, T=4, V=64, ld=64, dt=B.BF16, ids=0x20000, tok=None, ref=None, cu=0x21000, P=1, var=B.PREF_SIGMOID, beta=0.1, e=0.0, m=0.0, avg=0, opts=None,
             loss=0x30000, rew=0x31000, lp=0x32000, d=0x200000, ldd=64, status=0x50000, ws=0x60000, n=1 << 20)
    a.update(over)
    o = a["opts"]
    return B.lib().dppo_preference_fwd_bwd(P(a["z"]), a["T"], a["V"], a["ld"], a["dt"], P(a["ids"]), P(a["tok"]), P(a["ref"]), P(a["cu"]), a["P"], a["var"],
                                           a["beta"], a["e"], a["m"], a["avg"], ctypes.byref(o) if o is not None else None, P(a["loss"]), P(a["rew"]),
                                           P(a["lp"]), P(a["d"]), a["ldd"], P(a["status"]), P(a["ws"]), a["n"], None)


@pytest.mark.parametrize("call", [_logp, _bwd, _policy, _pref])
def test_rows_that_are_refused(B, call):
    assert call(B, T=-1) == -2 and call(B, V=0) == -2 and call(B, V=2 ** 30 + 1, ld=2 ** 31) == -2 and call(B, T=2 ** 27 + 1) == -2
    assert call(B, dt=2) == -3 and call(B, dt=-1) == -3
    for name in ("z", "ids", "status"):
        assert call(B, **{name: None}) == -1
    assert call(B, ld=63) == -6
    assert call(B, z=0x100001) == -7 and call(B, ids=0x20002) == -7 and call(B, status=0x50001) == -7 and call(B, dt=B.F32, z=0x100002) == -7


def test_logp_refusals(B):
    assert _logp(B, T=0) == 0 and _logp(B, T=0, z=None, ids=None, lp=None) == 0
    assert _logp(B, lp=None) == -1
    assert _logp(B, lp=0x30002) == -7 and _logp(B, lse=0x40004) == -7
    assert _bwd(B, T=0) == 0
    assert _bwd(B, lse=None) == -1 and _bwd(B, c=None) == -1 and _bwd(B, d=None) == -1
    assert _bwd(B, odt=2) == -3
    assert _bwd(B, ldd=63) == -6
    assert _bwd(B, d=0x200001) == -7 and _bwd(B, odt=1, d=0x200002) == -7 and _bwd(B, lse=0x40004) == -7 and _bwd(B, c=0x30001) == -7


@pytest.mark.parametrize("call", [_bwd, _policy, _pref])
def test_gradients_in_place_or_apart(B, call):
    row = 64 * 2
    assert call(B, d=0x100000 + row) == -9 and call(B, d=0x100000 + 3 * row + 32) == -9 and call(B, d=0x100000 - 2 * row) == -9
    assert call(B, d=0x100000, ldd=128) == -9
    f32 = {"odt": 1} if call is _bwd else {"opts": B.DppoOpts(dlogits_dtype=B.DLOGITS_F32)}
    assert call(B, d=0x100000, **f32) == -9


def test_policy_refusals(B):
    assert _policy(B, form=3) == -4 and _policy(B, form=-1) == -4
    assert _policy(B, beta=-0.1) == -11 and _policy(B, beta=float("nan")) == -11 and _policy(B, beta=float("inf")) == -11
    assert _policy(B, lo=-0.1) == -11 and _policy(B, hi=float("nan")) == -11
    assert _policy(B, opts=B.DppoOpts(dlogits_dtype=5)) == -3
    for name in ("mu", "adv", "loss", "kl", "mask", "d", "y"):
        assert _policy(B, **{name: None}) == -1, name
    assert _policy(B, form=B.KL_K3, ref=None) == -1 and _policy(B, form=B.KL_REF_PI, y=None) == -1
    assert _policy(B, ldd=63) == -6 and _policy(B, ldy=10) == -6
    for name in ("mu", "adv", "loss", "kl", "ref", "stats"):
        assert _policy(B, **{name: 0x70002}) == -7, name
    assert _policy(B, y=0x300001) == -7
    assert _policy(B, ws=None) == -8 and _policy(B, ws=0x60010) == -8 and _policy(B, n=100) == -8
    assert _policy(B, y=0x200000) == -9 and _policy(B, y=0x200000 + 130) == -9      # the gradient over the reference logits


def test_preference_refusals(B):
    assert _pref(B, P=-1) == -2 and _pref(B, P=2 ** 24 + 1) == -2
    assert _pref(B, var=3) == -4 and _pref(B, var=-1) == -4
    assert _pref(B, beta=0.0) == -11 and _pref(B, beta=float("nan")) == -11 and _pref(B, m=float("inf")) == -11
    assert _pref(B, e=-0.1) == -11 and _pref(B, e=0.6) == -11 and _pref(B, e=0.1, var=B.PREF_IPO) == -11 and _pref(B, e=float("nan")) == -11
    for name in ("cu", "loss", "rew", "lp", "d"):
        assert _pref(B, **{name: None}) == -1, name
    assert _pref(B, cu=0x21004) == -7 and _pref(B, rew=0x31001) == -7 and _pref(B, lp=0x32002) == -7 and _pref(B, ref=0x33001) == -7
    assert _pref(B, ws=None) == -8 and _pref(B, ws=0x60010) == -8 and _pref(B, n=100) == -8
    assert B.dppo_preference_workspace_bytes(0, 0) == 256 and B.dppo_preference_workspace_bytes(1, 1) == 256 * 6
    assert B.dppo_preference_workspace_bytes(-5, -5) == 256


def _quant(B, **over):
    a = dict(x=0x100000, rows=4, cols=256, ld=256, dt=B.BF16, g=128, q=0x200000, ldq=128, s=0x300000, lds=2, v=None, ldv=256, status=0x50000)
    a.update(over)
    return B.lib().dppo_int4_quantize(P(a["x"]), a["rows"], a["cols"], a["ld"], a["dt"], a["g"], P(a["q"]), a["ldq"], P(a["s"]), a["lds"], P(a["v"]), a["ldv"],
                                      P(a["status"]), None)


def test_int4_quantize_refusals(B):
    assert _quant(B, rows=0) == 0 and _quant(B, cols=0) == 0
    assert _quant(B, rows=-1) == -2 and _quant(B, cols=-1) == -2 and _quant(B, rows=2 ** 20, cols=2 ** 20) == -2 and _quant(B, cols=2 ** 30 + 1, rows=1) == -2
    assert _quant(B, dt=2) == -3 and _quant(B, g=16) == -11 and _quant(B, g=96) == -11
    for name in ("x", "q", "s", "status"):
        assert _quant(B, **{name: None}) == -1
    assert _quant(B, ld=255) == -6 and _quant(B, ldq=127) == -6 and _quant(B, lds=1) == -6 and _quant(B, v=0x400000, ldv=255) == -6
    assert _quant(B, x=0x100001) == -7 and _quant(B, s=0x300001) == -7 and _quant(B, v=0x400001) == -7 and _quant(B, status=0x50002) == -7
    assert _quant(B, q=0x100010) == -9 and _quant(B, s=0x200010) == -9 and _quant(B, s=0x100010) == -9 and _quant(B, v=0x100010) == -9
    assert _quant(B, v=0x200000) == -9 and _quant(B, v=0x300000) == -9 and _quant(B, v=0x100000, ldv=512) == -9


def _matvec(B, **over):
    a = dict(x=0x100000, ldx=256, q=0x200000, ldq=128, s=0x300000, lds=2, g=128, M=4, N=8, K=256, y=0x400000, dt=B.F32, ldy=8, status=0x50000, opts=None)
    a.update(over)
    o = a["opts"]
    return B.lib().dppo_matvec_int4(P(a["x"]), a["ldx"], P(a["q"]), a["ldq"], P(a["s"]), a["lds"], a["g"], a["M"], a["N"], a["K"], P(a["y"]), a["dt"], a["ldy"],
                                    P(a["status"]), ctypes.byref(o) if o is not None else None, None)


def test_matvec_refusals(B):
    assert _matvec(B, M=0) == 0 and _matvec(B, N=0) == 0
    for name in ("M", "N", "K"):
        assert _matvec(B, **{name: -1}) == -2 and _matvec(B, **{name: 2 ** 30 + 1}) == -2
    assert _matvec(B, dt=2) == -3 and _matvec(B, g=8) == -11 and _matvec(B, opts=B.DppoOpts(wait_limit_us=-1)) == -11
    for name in ("x", "q", "s", "y", "status"):
        assert _matvec(B, **{name: None}) == -1
    assert _matvec(B, ldx=255) == -6 and _matvec(B, ldq=127) == -6 and _matvec(B, lds=1) == -6 and _matvec(B, ldy=7) == -6
    assert _matvec(B, x=0x100001) == -7 and _matvec(B, s=0x300001) == -7 and _matvec(B, y=0x400002) == -7 and _matvec(B, status=0x50001) == -7
    assert _matvec(B, y=0x100010) == -9 and _matvec(B, y=0x200010) == -9 and _matvec(B, y=0x300000) == -9


def test_binding_repeats_the_header(B):
    hdr = open(os.path.join(ROOT, "include", "dppo.h")).read()
    for name, value in (("KL_PI_REF", B.KL_PI_REF), ("KL_REF_PI", B.KL_REF_PI), ("KL_K3", B.KL_K3), ("PREF_SIGMOID", B.PREF_SIGMOID), ("PREF_IPO", B.PREF_IPO),
                        ("PREF_HINGE", B.PREF_HINGE), ("STATUS_BAD_SEQUENCES", B.STATUS_BAD_SEQUENCES)):
        assert int(re.search(rf"DPPO_{name}\s*=\s*(\d+)", hdr).group(1)) == value


# ------------------------------------------------------------------------------------------------------- the restatement
def _case(seed, T=6, V=11):
    rng = np.random.default_rng(seed)
    z = 2 * rng.standard_normal((T, V))
    ids = rng.integers(0, V, T)
    return rng, z, ids


@pytest.mark.parametrize("form", ["pi_ref", "ref_pi", "k3"])
def test_policy_gradient_against_differences(form):
    """Central differences of the loss: with h = 1e-5 the truncation is of the order h^2 = 1e-10 and the rounding 1e-16 / h = 1e-11."""
    rng, z, ids = _case(1)
    y = z + 0.5 * rng.standard_normal(z.shape)
    lp = R.token_logp(z, ids)
    a = dict(ids=ids, mu_logp=lp + 0.3 * rng.standard_normal(6), adv=rng.standard_normal(6), valid=np.array([1, 1, 0, 1, 1, 1], bool), form=form, beta=0.7, eps_low=0.2,
             eps_high=0.25, y=y, ref_logp=lp + 0.3 * rng.standard_normal(6))
    out = R.policy_kl(z, **a)
    assert 0 < out["mask"].sum() < 5                         # clipped rows and others
    h, num = 1e-5, np.zeros_like(z)
    for i in np.ndindex(z.shape):
        e = np.zeros_like(z)
        e[i] = h
        num[i] = (R.policy_kl(z + e, **a)["loss"] - R.policy_kl(z - e, **a)["loss"]) / (2 * h)
    assert np.abs(num - out["dlogits"]).max() < 1e-8


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("ipo", 0.0), ("hinge", 0.0)])
@pytest.mark.parametrize("average", [False, True])
def test_preference_gradient_against_differences(kind, smoothing, average):
    rng, z, ids = _case(2, T=12)
    cu = [1, 4, 6, 6, 8, 9, 11]                              # the second pair has an empty sequence and does not count
    a = dict(ids=ids, cu=cu, valid=rng.random(12) < 0.9, kind=kind, beta=0.3, smoothing=smoothing, margin=0.05, average=average,
             ref_logp=R.token_logp(z, ids) + 0.2 * rng.standard_normal(12))
    out = R.preference(z, **a)
    assert out["reward"][2] == 0 and (out["coef"][6:8] == 0).all() and out["coef"][0] == out["coef"][11] == 0
    h, num = 1e-5, np.zeros_like(z)
    for i in np.ndindex(z.shape):
        e = np.zeros_like(z)
        e[i] = h
        num[i] = (R.preference(z + e, **a)["loss"] - R.preference(z - e, **a)["loss"]) / (2 * h)
    assert np.abs(num - out["dlogits"]).max() < 1e-8 * max(1.0, np.abs(out["dlogits"]).max())


def test_losses_against_torch():
    torch = pytest.importorskip("torch")
    rng, z, ids = _case(3)
    y = z + rng.standard_normal(z.shape)
    Z, Y = torch.tensor(z, requires_grad=True), torch.tensor(y)
    lz, ly = torch.log_softmax(Z, 1), torch.log_softmax(Y, 1)
    every = np.ones(6, bool)
    for form, ref in (("pi_ref", torch.nn.functional.kl_div(ly, lz, reduction="batchmean", log_target=True)),
                      ("ref_pi", torch.nn.functional.kl_div(lz, ly, reduction="batchmean", log_target=True))):
        out = R.policy_kl(z, ids, np.zeros(6), np.zeros(6), every, form, 1.0, 0.2, 0.2, y=y)
        assert abs(out["loss"] - ref.item()) < 1e-12
        assert np.abs(out["dlogits"] - torch.autograd.grad(ref, Z, retain_graph=True)[0].numpy()).max() < 1e-12
    cu = [0, 2, 3, 5, 6]
    lp = lz.gather(1, torch.tensor(ids)[:, None])[:, 0]
    h = 0.2 * torch.stack([lp[0:2].sum() - lp[2:3].sum(), lp[3:5].sum() - lp[5:6].sum()])
    ref = -torch.nn.functional.logsigmoid(h).mean()
    out = R.preference(z, ids, cu, every, "sigmoid", 0.2)
    assert abs(out["loss"] - ref.item()) < 1e-12 and np.abs(out["dlogits"] - torch.autograd.grad(ref, Z)[0].numpy()).max() < 1e-12


def test_int4_restatement():
    rng = np.random.default_rng(4)
    for bits in (8,):
        x = rng.standard_normal(1000) * np.exp2(rng.integers(-30, 30, 1000))
        torch = pytest.importorskip("torch")
        assert np.array_equal(R.round_bits(x.astype(np.float32).astype(np.float64), bits), torch.tensor(x.astype(np.float32)).to(torch.bfloat16).double().numpy())
    x = rng.standard_normal((5, 77))
    code, scale, val = R.int4_quantize(x, 32)
    assert code.min() >= 1 and code.max() <= 15 and scale.shape == (5, 3)
    # at most half a step off, and 7.03 steps (a scale rounded down by 2^-9) clip to 7
    assert np.abs(val - x).max() <= 0.5 * scale.max() * (1 + 1e-12)
    assert np.array_equal(R.unpack(R.pack(code), 77), code)
    y, mag = R.int4_product(rng.standard_normal((3, 77)), code, scale, 32)
    assert y.shape == (3, 5) and (mag >= np.abs(y)).all()
