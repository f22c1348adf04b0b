"""Log-probabilities of tokens, the clipped policy loss with a KL term and the loss over pairs of sequences against float64 (needs a
B200).

Tolerances, u = 2^-24.  A thread adds up at most V / 512 pairs of terms, warps and CTAs a few dozen more sums, an exponential is good to 2^-22
= 4 u and its argument to 2 u of its size (30 at most for entries that count): a row's sum is good to eps(V) = (V / 512 + 96) u, and so is
lse.  logp: eps, and half a step of fp32.  A gradient entry c (1[a] - pi): pi carries eps and its own exponential's error, (eps + (4 + 2 x) u) pi
with x = lse - z (pi x <= 1/e), then half a step of the output type.  KL: its terms are pi times a difference of at most `spread`, the two lse
cancel up to eps each: 3 eps (1 + spread).  Its gradient pi (l - KL): that, and the difference's own roundings, 4 u of |z| + |y| + |c|.
Half a step: 2^-24 (fp32) and 2^-8 (bf16), relative; the loss sums rows in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding
from oracle import reference_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32
FORMS = {"pi_ref": binding.KL_PI_REF, "ref_pi": binding.KL_REF_PI, "k3": binding.KL_K3}
KINDS = {"sigmoid": binding.PREF_SIGMOID, "ipo": binding.PREF_IPO, "hinge": binding.PREF_HINGE}


def eps(V):
    return (V / 512 + 96) * U


def host(t):
    return t.detach().double().cpu().numpy()


def rows(T, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = spread * torch.randn((T, V), generator=g)
    z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += 8 * torch.rand(T, generator=g)
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    ids[::2] = z[::2].argmax(1).to(torch.int32)              # half of the tokens likely, half of them not
    return z.to(dtype), ids, g


def placed(t, stride=None, offset=0, fill=float("nan")):
    """The matrix t on the device in rows of `stride` elements, `offset` elements behind a 16-byte boundary, the rest filled."""
    T, V = t.shape
    stride = stride or V
    buf = torch.full((offset + T * stride + 64,), fill, dtype=t.dtype, device=DEV)
    out = torch.as_strided(buf, (T, V), (stride, 1), offset)
    out.copy_(t)
    return out, buf


def check_grad(d, want, tol, dtype):
    got = host(d)
    lim = tol + HALF[dtype] * np.abs(want) * (1 + 1e-3) + 1e-36
    bad = np.abs(got - want) > lim
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], lim[bad][:4])


def pi_tol(z, V):
    """error of pi, entrywise"""
    l = R.log_softmax(z)
    p = np.exp(l)
    x = np.where(p > 0, -l, 0.0)
    return p * (eps(V) + (4 + 2 * np.minimum(x, 200)) * U)


SIZES = [(1, 1), (3, 2), (5, 7), (4, 33), (7, 1000), (3, 4097), (2, 20481), (2, 50257), (1, 151936)]


# ------------------------------------------------------------------------------------------------------------- logp
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_logp_forward_and_backward(T, V, dtype):
    z, ids, g = rows(T, V, dtype, seed=V + T)
    c = torch.randn(T, generator=g)
    zd, _ = placed(z, V + 5, 3)
    o = dppo.dppo_token_logp(zd, ids.to(DEV))
    d = dppo.dppo_token_logp_bwd(zd, ids.to(DEV), o["lse"], c.to(DEV), dlogits_f32=True)["dlogits"]
    same = dppo.dppo_token_logp_bwd(zd, ids.to(DEV), o["lse"], c.to(DEV))["dlogits"]
    assert int(o["status"].item()) == 0
    zh, want = z.double().numpy(), R.token_logp(z.double().numpy(), ids.numpy())
    assert np.all(np.abs(host(o["logp"]) - want) <= eps(V) + U * np.abs(want))
    assert np.all(np.abs(host(o["lse"]) - (zh[np.arange(T), ids.numpy()] - want)) <= eps(V))
    tol = pi_tol(zh, V) * np.abs(c.double().numpy())[:, None]
    ref = R.logp_gradient(zh, ids.numpy(), c.double().numpy())
    check_grad(d, ref, tol, F32)
    check_grad(same, ref, tol, dtype)


def test_logp_of_very_confident_tokens_keeps_its_relative_accuracy():
    for dtype in (BF, F32):
        z = torch.zeros((6, 3000), dtype=dtype)
        ids = torch.tensor([0, 1, 7, 8, 2999, 1500], dtype=torch.int32)
        z[torch.arange(6), ids.long()] = torch.tensor([12.0, 16.0, 20.0, 24.0, 28.0, 32.0]).to(dtype)
        o = dppo.dppo_token_logp(z.to(DEV), ids.to(DEV))
        d = dppo.dppo_token_logp_bwd(z.to(DEV), ids.to(DEV), o["lse"], torch.ones(6, device=DEV), dlogits_f32=True)["dlogits"]
        za = z[torch.arange(6), ids.long()].double().numpy()
        want = -np.log1p(2999 * np.exp(-za))
        assert np.all(np.abs(host(o["logp"]) - want) <= (eps(3000) + U) * np.abs(want))
        got = host(d)[np.arange(6), ids.numpy()]
        # lse is handed over as a 64-bit number: off by half a step, 2^-53 of it, which 1 - pi(a) = 1 - exp(z_a - lse) takes on as it is
        assert np.all(np.abs(got + np.expm1(want)) <= (2 * eps(3000) + U) * np.abs(np.expm1(want)) + 2.0 ** -53 * za)


def test_logp_masked_rows_and_dropped_rows():
    z, ids, _ = rows(9, 777, BF, seed=5)
    z[1] = float("nan")                                      # masked: never read
    z[2, 5] = float("nan")
    z[3, 6] = float("inf")
    z[4] = float("-inf")
    z[5] = torch.finfo(BF).min                               # a row of the type's lowest value has no distribution either
    z[6, 10:] = torch.finfo(BF).min                          # but entries of it are a mask
    ids[6] = 3
    z[7, 100:300] = float("-inf")
    ids[7] = 150                                             # the token itself masked
    ids[1], ids[0] = -100, 777
    mask = torch.ones(9, dtype=torch.uint8)
    mask[1] = 0
    want = R.token_logp(z[[6, 7, 8]].double().numpy(), ids[[6, 7, 8]].numpy())
    o = dppo.dppo_token_logp(z.to(DEV), ids.to(DEV), mask.to(DEV))
    assert int(o["status"].item()) == binding.STATUS_BAD_SAMPLED_ID | binding.STATUS_NONFINITE_ROW
    lp, lse = host(o["logp"]), host(o["lse"])
    assert np.all(lp[:6] == 0) and lse[1] == 0 and np.isnan(lse[[0, 2, 3, 4, 5]]).all() and np.isfinite(lse[6:]).all()
    assert want[1] == -np.inf and lp[7] == -np.inf
    assert np.all(np.abs(lp[[6, 8]] - want[[0, 2]]) <= eps(777) + U * np.abs(want[[0, 2]]))
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    c = torch.full((9,), 0.5, device=DEV)
    c[8] = 0.0
    d = dppo.dppo_token_logp_bwd(z.to(DEV), ids.to(DEV), o["lse"], c, mask.to(DEV), status=st)["dlogits"]
    assert int(st.item()) == binding.STATUS_BAD_SAMPLED_ID | binding.STATUS_NONFINITE_ROW
    assert (host(d)[[0, 1, 2, 3, 4, 5, 8]] == 0).all()
    zh = z[[6, 7]].double().numpy()
    zh[zh < -1e38] = -np.inf
    with np.errstate(invalid="ignore"):
        check_grad(d[6:8], R.logp_gradient(zh, ids[6:8].numpy(), np.full(2, 0.5)), pi_tol(zh, 777), BF)


def test_logp_without_rows_and_long_rows():
    o = dppo.dppo_token_logp(torch.empty((0, 50), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV))
    assert o["logp"].shape == (0,) and int(o["status"].item()) == 0
    for dtype in (BF, F32):
        V = 700001                                           # longer than anything is unrolled for
        z, ids, _ = rows(2, V, dtype, seed=9)
        o = dppo.dppo_token_logp(z.to(DEV), ids.to(DEV))
        want = R.token_logp(z.double().numpy(), ids.numpy())
        assert np.all(np.abs(host(o["logp"]) - want) <= eps(V) + U * np.abs(want))


# ----------------------------------------------------------------------------------------------------------- policy
def policy_case(T, V, dtype, seed, masked=True):
    z, ids, g = rows(T, V, dtype, seed)
    y = (z.float() + 0.4 * torch.randn((T, V), generator=g)).to(dtype)
    lp = torch.from_numpy(R.token_logp(z.double().numpy(), ids.numpy()))
    mu = (lp + 0.4 * torch.randn(T, generator=g, dtype=torch.float64)).clamp(max=-1e-6).float()
    adv = torch.randn(T, generator=g)
    ref = (lp + 0.3 * torch.randn(T, generator=g, dtype=torch.float64)).clamp(max=0).float()
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8) if masked else torch.ones(T, dtype=torch.uint8)
    return dict(z=z, y=y, ids=ids, mu=mu, adv=adv, ref=ref, mask=mask)


def run_policy(c, form, z=None, y=None, mask=True, **kw):
    t = {n: c[n].to(DEV) for n in ("ids", "mu", "adv", "ref", "mask")}
    a = dict(kl_form=FORMS[form], kl_coef=0.3, eps_low=0.2, eps_high=0.25)
    a.update(kw)
    z = c["z"].to(DEV) if z is None else z
    a["ref_logp" if form == "k3" else "ref_logits"] = t["ref"] if form == "k3" else (c["y"].to(DEV) if y is None else y)
    return dppo.dppo_policy_kl_fwd_bwd(z, t["ids"], t["mu"], t["adv"], t["mask"] if mask else None, **a)


def check_policy(c, o, form, valid=None, scale=None, dtype=None, zh=None, yh=None, eps_low=0.2, eps_high=0.25, beta=0.3):
    zh = c["z"].double().numpy() if zh is None else zh
    yh = c["y"].double().numpy() if yh is None else yh
    V = zh.shape[1]
    valid = c["mask"].numpy() != 0 if valid is None else valid
    w = R.policy_kl(zh, c["ids"].numpy(), c["mu"].double().numpy(), c["adv"].double().numpy(), valid, form, beta, eps_low, eps_high, y=yh,
                    ref_logp=c["ref"].double().numpy(), scale=scale)
    e, n = eps(V), max(1, int(valid.sum()))
    s = scale or 1.0 / n
    near = (np.abs(w["r"] - (1 + eps_high)) <= 3 * e * w["r"]) | (np.abs(w["r"] - (1 - eps_low)) <= 3 * e * w["r"])
    assert not near[valid].any()                             # no row within rounding of the clip: masks must be equal
    assert np.array_equal(o["mask"].cpu().numpy(), w["mask"])
    if form == "k3":
        x = np.where(valid, np.abs(np.expm1(c["ref"].double().numpy() - R.token_logp(zh, c["ids"].numpy()))), 0)
        tol_kl = (e + U) * x + e * e
    else:
        tol_kl = 3 * e * (1 + w["spread"])
    assert np.all(np.abs(host(o["kl"]) - w["kl"]) <= tol_kl + U * np.abs(w["kl"]))
    adv = np.abs(c["adv"].double().numpy())
    tol_row = s * (beta * tol_kl + 2 * e * w["r"] * adv) + 2 * U * np.abs(w["terms"])
    assert abs(float(o["loss"].item()) - w["loss"]) <= tol_row.sum() + U * abs(w["loss"])
    pt = np.zeros(zh.shape)
    with np.errstate(invalid="ignore"):
        lz, p = R.log_softmax(zh[valid]), np.exp(R.log_softmax(zh[valid]))
    g = np.abs(w["mask"] * w["r"] * adv)[:, None]
    pz = np.zeros(zh.shape)
    pz[valid] = pi_tol(zh[valid], V)
    P = np.zeros(zh.shape)
    P[valid] = p
    if form == "k3":
        x = np.abs(np.expm1(np.where(valid, c["ref"].double().numpy() - R.token_logp(zh, c["ids"].numpy()), 0)))[:, None]
        hot = np.zeros(zh.shape)
        hot[np.arange(len(zh)), c["ids"].numpy()] = 1
        size = g + beta * x
        pt = s * (size * pz + (2 * e * (g + beta * (1 + x)) + 2 * U * size) * np.abs(P - hot))
    elif form == "pi_ref":
        l = np.zeros(zh.shape)
        with np.errstate(invalid="ignore"):
            l[valid] = lz - R.log_softmax(yh[valid])
        l = np.where(P > 0, np.abs(l), 0)
        kl = w["kl"][:, None]
        far = 4 * U * (np.where(P > 0, np.abs(zh), 0) + np.where(P > 0, np.abs(yh), 0) + 50)
        pt = s * ((g + beta * (l + kl)) * (pz + 4 * U * P) + P * (2 * e * g + beta * (tol_kl[:, None] + 2 * e + far)))
    else:
        q, qz = np.zeros(zh.shape), np.zeros(zh.shape)
        q[valid], qz[valid] = np.exp(R.log_softmax(yh[valid])), pi_tol(yh[valid], V)
        pt = s * ((g + beta) * (pz + 4 * U * P) + 2 * e * g * P + beta * (qz + 4 * U * q))
    hot = np.zeros(zh.shape)
    hot[np.arange(len(zh)), c["ids"].numpy()] = 1
    pt += s * hot * 4 * e * (g + beta)                       # the token's own entry
    pt[~valid] = 0
    check_grad(o["dlogits"], w["dlogits"], pt, dtype or o["dlogits"].dtype)
    return w


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (5, 7), (9, 33), (20, 1000), (6, 4097), (3, 20483), (3, 50257), (2, 151936)])
def test_policy_loss(T, V, dtype, form):
    c = policy_case(T, V, dtype, seed=7 * V + T, masked=T > 3)
    o = run_policy(c, form, dlogits_f32=True, want_stats=True)
    assert int(o["status"].item()) == 0
    w = check_policy(c, o, form)
    same = run_policy(c, form, mask=False) if not (c["mask"] == 0).any() else run_policy(c, form)
    check_policy(c, same, form)
    st = host(o["stats"])
    assert st[0] == int(c["mask"].sum()) and st[1] == int(((w["mask"] == 0) & (c["mask"].numpy() != 0)).sum())
    assert abs(st[2] - w["kl"].sum()) <= 1e-4 * (1 + w["kl"].sum())


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dtype,V", [(BF, 170001), (F32, 90001), (F32, 170001)])
def test_policy_loss_of_rows_too_long_for_registers(dtype, V, form):
    c = policy_case(2, V, dtype, seed=V, masked=False)
    # the second row's sums move to a larger maximum in its last part, in both tensors
    c["z"][1, -3:] += 12
    c["y"][1, -3:] += 12
    c["ref"] = torch.from_numpy(R.token_logp(c["z"].double().numpy(), c["ids"].numpy())).float() - 0.2
    c["mu"] = c["ref"] + 0.1
    o = run_policy(c, form)
    assert int(o["status"].item()) == 0
    check_policy(c, o, form)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lay", [(0, 1000, 0, 1000, 0, 1000), (1, 1003, 1, 1003, 1, 1003), (3, 1001, 0, 1000, 5, 1002), (8, 1008, 1, 1016, 16, 1024)])
def test_policy_loss_in_any_layout(lay, dtype, form):
    """Row starts on and off 16-byte boundaries, alike and unlike in the three tensors; what lies between the rows stays."""
    zo, zs, yo, ys, do, ds = lay
    c = policy_case(6, 1000, dtype, seed=11)
    z, _ = placed(c["z"], zs, zo)
    y, _ = placed(c["y"], ys, yo)
    d, buf = placed(torch.zeros((6, 1000), dtype=dtype), ds, do, fill=7.0)
    check_policy(c, run_policy(c, form, z=z, y=y, dlogits=d), form)
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (6, 1000), (ds, 1), do).fill_(True)
    assert (buf[~inside] == 7.0).all()
    d32, _ = placed(torch.zeros((6, 1000)), ds, do, fill=7.0)
    check_policy(c, run_policy(c, form, z=z, y=y, dlogits=d32, dlogits_f32=True), form)


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("V", [1001, 170003])
def test_policy_gradient_in_place_and_repeatable(form, V):
    c = policy_case(5, V, BF, seed=13)
    a, b = run_policy(c, form), run_policy(c, form)
    z = c["z"].to(DEV)
    p = run_policy(c, form, z=z, dlogits=z)
    for n in ("loss", "kl", "mask", "dlogits"):
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], p[n]), n


def test_policy_kl_of_policies_that_differ_by_a_constant_or_not_at_all():
    """Offsets between the two rows of logits cancel: KL and gradient are those of equal policies, zero up to eps of the lse."""
    c = policy_case(4, 5000, F32, seed=17, masked=False)
    c["adv"].zero_()
    for off in (0.0, 8.0, -64.0):
        c["y"] = (c["z"] * 256).round() / 256 + off
        c["z"] = (c["z"] * 256).round() / 256
        for form in ("pi_ref", "ref_pi"):
            o = run_policy(c, form, kl_coef=1.0)
            assert np.abs(host(o["kl"])).max() <= 3 * eps(5000)
            assert np.abs(host(o["dlogits"])).max() <= 0.25 * (6 * eps(5000) + 4 * U * 100)


@pytest.mark.parametrize("form", ["pi_ref", "ref_pi"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("apart", ["wide", "halves", "one entry"])
def test_policy_of_policies_that_live_on_different_entries(apart, dtype, form):
    """Entries whose probability vanishes under one policy and counts under the other: their exponentials cannot come from one another."""
    T, V = 4, 20488
    c = policy_case(T, V, dtype, seed=31, masked=False)
    z, y = c["z"].float(), c["y"].float()
    if apart == "wide":
        g = torch.Generator().manual_seed(32)
        z, y = z + 30 * torch.randn(z.shape, generator=g), y + 30 * torch.randn(y.shape, generator=g)
    elif apart == "halves":
        z[:, ::2] -= 150
        y[:, 1::2] -= 90
    else:
        y[:, 4321] += 120
        z[:, 4322] -= 120
    c["z"], c["y"] = z.to(dtype), y.to(dtype)
    check_policy(c, run_policy(c, form), form)


def test_policy_masked_vocabulary_infinities_and_dropped_rows():
    for dtype in (BF, F32):
        c = policy_case(8, 3001, dtype, seed=19, masked=False)
        low = torch.finfo(dtype).min
        for t in (c["z"], c["y"]):
            t[0, 2000:] = float("-inf")
            t[1, ::2] = low
            t[7, 1:] = float("-inf")                         # a single token has all the mass
        c["ids"][:2] = torch.tensor([1999, 1], dtype=torch.int32)
        c["ids"][7] = 0
        c["z"][2, 5:9] = float("-inf")                       # pi has none where rho has some: fine for KL(pi || rho) only
        c["y"][3, 5:9] = float("-inf")                       # and the other way round
        c["ids"][2:4] = 20
        c["z"][4, 0], c["y"][5, 0], c["z"][6, 1] = float("nan"), float("nan"), float("inf")
        c["mu"] = torch.from_numpy(np.nan_to_num(R.token_logp(np.nan_to_num(c["z"].double().numpy(), nan=0, posinf=0, neginf=-1e300), c["ids"].numpy()))).float() - 0.1
        zh, yh = c["z"].double().numpy(), c["y"].double().numpy()
        zh[zh <= -3e38], yh[yh <= -3e38] = -np.inf, -np.inf
        for form, gone in (("pi_ref", [3, 4, 5, 6]), ("ref_pi", [2, 4, 5, 6])):
            o = run_policy(c, form, mask=False)
            assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW
            valid = np.ones(8, bool)
            valid[gone] = False
            zz, yy = zh.copy(), yh.copy()
            zz[gone], yy[gone] = 0, 0
            check_policy(c, o, form, valid=valid, scale=1.0 / 8, zh=zz, yh=yy)
        o = run_policy(c, "k3", mask=False)
        valid = np.array([1, 1, 1, 1, 0, 1, 0, 1], bool)
        zz = zh.copy()
        zz[~valid] = 0
        check_policy(c, o, "k3", valid=valid, scale=1.0 / 8, zh=zz, yh=None)


def test_policy_masked_rows_bad_ids_and_empty_calls():
    c = policy_case(6, 500, BF, seed=23, masked=False)
    c["mask"][1] = 0
    c["z"][1], c["y"][1], c["ids"][1] = float("nan"), float("nan"), -100
    c["ids"][3] = 500
    for form in FORMS:
        o = run_policy(c, form)
        assert int(o["status"].item()) == binding.STATUS_BAD_SAMPLED_ID
        valid = np.array([1, 0, 1, 0, 1, 1], bool)
        z, y, k = c["z"].double().numpy(), c["y"].double().numpy(), dict(c, ids=c["ids"].clone())
        z[~valid], y[~valid] = 0, 0
        k["ids"][[1, 3]] = 0
        check_policy(k, o, form, valid=valid, scale=1.0 / 5, zh=z, yh=y)
        c2 = dict(c, mask=torch.zeros(6, dtype=torch.uint8))
        o = run_policy(c2, form)
        assert float(o["loss"].item()) == 0 and (o["dlogits"] == 0).all() and (o["kl"] == 0).all() and int(o["status"].item()) == 0
        e = {n: t[:0] for n, t in c.items()}
        o = run_policy(e, form, mask=False)
        assert float(o["loss"].item()) == 0 and o["dlogits"].shape == (0, 500)


def test_policy_without_a_clip_and_with_a_given_scale():
    c = policy_case(12, 300, F32, seed=29)
    inf = float("inf")
    for form in FORMS:
        check_policy(c, run_policy(c, form, eps_low=inf, eps_high=inf, loss_scale=0.01), form, scale=float(np.float32(0.01)), eps_low=inf, eps_high=inf)
        check_policy(c, run_policy(c, form, kl_coef=0.0), form, beta=0.0)


def test_policy_loss_against_its_own_differences():
    """The kernel's gradient along a direction against the kernel's loss at two points: h^2 / 6 of the third derivative (of the order of the
    loss itself) and the loss's rounding, 2 u (|loss| + terms) / (2 h)."""
    c = policy_case(16, 64, F32, seed=31, masked=False)
    g = torch.Generator().manual_seed(1)
    v = torch.randn((16, 64), generator=g)
    v /= v.norm()
    h = 2.0 ** -7
    for form in FORMS:
        kw = dict(eps_low=float("inf"), eps_high=float("inf"), kl_coef=1.0)
        z = c["z"].to(DEV)
        d = run_policy(c, form, z=z, **kw)["dlogits"]
        up, dn = (float(run_policy(c, form, z=z + s * h * v.to(DEV), **kw)["loss"].item()) for s in (1, -1))
        want = float((d.double().cpu() * v.double()).sum())
        assert abs((up - dn) / (2 * h) - want) <= h * h + (4 * U * 4 + 2 * eps(64)) / (2 * h)


# ------------------------------------------------------------------------------------------------------- preference
def pref_case(cu, T, V, dtype, seed, masked=False):
    z, ids, g = rows(T, V, dtype, seed)
    lp = torch.from_numpy(R.token_logp(z.double().numpy(), ids.numpy()))
    ref = (lp + 0.3 * torch.randn(T, generator=g, dtype=torch.float64)).float()
    mask = (torch.rand(T, generator=g) < 0.7).to(torch.uint8) if masked else None
    return dict(z=z, ids=ids, cu=torch.tensor(cu, dtype=torch.int64), ref=ref, mask=mask)


def run_pref(c, kind="sigmoid", z=None, **kw):
    a = dict(beta=0.2, variant=KINDS[kind])
    a.update(kw)
    return dppo.dppo_preference_fwd_bwd(c["z"].to(DEV) if z is None else z, c["ids"].to(DEV), c["cu"].to(DEV), c["ref"].to(DEV) if c["ref"] is not None else None,
                                        c["mask"].to(DEV) if c["mask"] is not None else None, **a)


def check_pref(c, o, kind="sigmoid", beta=0.2, label_smoothing=0.0, margin=0.0, average=False, loss_scale=None, zh=None):
    zh = c["z"].double().numpy() if zh is None else zh
    T, V = zh.shape
    valid = np.ones(T, bool) if c["mask"] is None else c["mask"].numpy() != 0
    cu, ids = c["cu"].tolist(), c["ids"].numpy()
    w = R.preference(zh, ids, cu, valid, kind, beta, label_smoothing, margin, average, None if c["ref"] is None else c["ref"].double().numpy(), loss_scale)
    e = eps(V)
    assert np.all(np.abs(host(o["logp"]) - w["logp"]) <= e + U * np.abs(w["logp"]))
    n = np.array([valid[cu[q]:cu[q + 1]].sum() for q in range(len(cu) - 1)])
    tol_R = beta * e * (np.minimum(n, 1) if average else n)
    assert np.all(np.abs(host(o["reward"]) - w["reward"]) <= tol_R + U * np.abs(w["reward"]))
    tol_h = tol_R[0::2] + tol_R[1::2]
    # how fast the loss and its derivative go with h
    if kind == "ipo":
        h = np.abs(w["reward"][0::2] - w["reward"][1::2] - margin) / beta + 0.5 / beta
        by, by2 = (2 * h / beta), 2 / beta ** 2
    else:
        by, by2 = 1.0, (0.25 if kind == "sigmoid" else 0.0)
    count = max(1, int(((n[0::2] > 0) & (n[1::2] > 0)).sum()))
    s = loss_scale or 1.0 / count
    assert abs(float(o["loss"].item()) - w["loss"]) <= s * (by * tol_h).sum() + U * abs(w["loss"])
    c_tol = np.zeros(T)
    for q in range(len(cu) - 1):
        if n[q]:
            c_tol[cu[q]:cu[q + 1]] = s * beta * by2 * tol_h[q // 2] / (n[q] if average else 1)
    inside = np.zeros(T, bool)
    inside[cu[0]:cu[-1]] = True
    use = inside & valid
    tol = np.zeros(zh.shape)
    P = np.exp(R.log_softmax(zh[use]))
    hot = np.zeros(P.shape)
    hot[np.arange(len(P)), ids[use]] = 1
    coef = np.abs(w["coef"][use])[:, None]
    tol[use] = coef * (pi_tol(zh[use], V) + 2 * U * P) + (c_tol[use][:, None] + U * coef) * np.abs(P - hot) + coef * hot * 3 * e
    check_grad(o["dlogits"], w["dlogits"], tol, o["dlogits"].dtype)


@pytest.mark.parametrize("kind,kw", [("sigmoid", {}), ("sigmoid", dict(label_smoothing=0.125, margin=0.25)), ("ipo", {}), ("hinge", {})])
@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("dtype,V", [(BF, 1000), (F32, 777), (BF, 50257)])
def test_preference_loss(kind, kw, average, dtype, V):
    cu, T = ([2, 5, 6, 13, 20], 23) if V > 10000 else ([2, 5, 6, 6, 9, 9, 9, 40, 41, 74, 107, 108], 110)
    if len(cu) % 2 == 0:
        cu = cu[:-1]
    c = pref_case(cu, T, V, dtype, seed=V, masked=V == 777)
    o = run_pref(c, kind, average=average, **kw)
    assert int(o["status"].item()) == 0
    check_pref(c, o, kind, average=average, **kw)
    check_pref(c, run_pref(c, kind, average=average, dlogits_f32=True, loss_scale=0.5, **kw), kind, average=average, loss_scale=0.5, **kw)


@pytest.mark.parametrize("P", [1, 15, 16, 17, 40, 1500])
def test_preference_counts_of_pairs(P):
    """More and fewer sequences than a CTA has warps, and than it has threads; sequences of one row, of none, and a long one."""
    rng = np.random.default_rng(P)
    n = rng.integers(0, 4, 2 * P)
    n[rng.integers(0, 2 * P)] = 300
    cu = np.concatenate([[1], 1 + np.cumsum(n)]).tolist()
    c = pref_case(cu, cu[-1] + 3, 40, F32, seed=P, masked=P % 2 == 0)
    o = run_pref(c)
    assert int(o["status"].item()) == 0
    check_pref(c, o)
    assert (o["dlogits"][0] == 0).all() and (o["dlogits"][cu[-1]:] == 0).all()


def test_preference_without_a_reference_without_pairs_without_rows():
    c = pref_case([0, 4, 9], 9, 100, F32, seed=3)
    c["ref"] = None
    check_pref(c, run_pref(c, average=True, margin=0.1), average=True, margin=0.1)
    c["cu"] = torch.tensor([3], dtype=torch.int64)
    o = run_pref(c)
    assert float(o["loss"].item()) == 0 and (o["dlogits"] == 0).all() and (o["logp"] == 0).all() and o["reward"].numel() == 0 and int(o["status"].item()) == 0
    e = dict(z=c["z"][:0], ids=c["ids"][:0], cu=torch.zeros(3, dtype=torch.int64), ref=None, mask=None)
    o = run_pref(e)
    assert float(o["loss"].item()) == 0 and (o["reward"] == 0).all() and int(o["status"].item()) == 0


@pytest.mark.parametrize("cu", [[0, 5, 4, 6, 9], [-1, 2, 4, 6, 9], [0, 2, 4, 6, 10], [0, 5, 9, 3, 4, 6, 8], [2 ** 40, 2 ** 40, 2 ** 40], [-2 ** 62, 0, 2 ** 62]])
def test_preference_refuses_sequences_that_are_none(cu):
    c = pref_case([0, 4, 9], 9, 100, BF, seed=4)
    c["cu"] = torch.tensor(cu, dtype=torch.int64)
    o = run_pref(c)
    assert int(o["status"].item()) == binding.STATUS_BAD_SEQUENCES
    assert float(o["loss"].item()) == 0 and (o["dlogits"] == 0).all() and (o["reward"] == 0).all()


def test_preference_drops_pairs_with_broken_rows():
    c = pref_case([1, 4, 6, 9, 12, 14, 15, 17, 19], 20, 200, BF, seed=6)
    z, ids = c["z"], c["ids"]
    z[0], z[19], ids[0], ids[19] = float("nan"), float("nan"), -100, 10 ** 6      # outside the sequences: not looked at
    z[7, 3] = float("nan")                                   # second pair
    ids[13] = 200                                            # third pair
    o = run_pref(c)
    assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW | binding.STATUS_BAD_SAMPLED_ID
    good = dict(c, z=z.clone(), ids=ids.clone())
    good["z"][[0, 7, 19]] = 0
    good["ids"][[0, 13, 19]] = 0
    mask = torch.ones(20, dtype=torch.uint8)
    mask[6:15] = 0
    w = dict(good, mask=mask)
    # logp of the sound rows of dropped pairs is given all the same
    lp = host(o["logp"])
    assert np.all(np.abs(lp[[6, 8, 9, 12]] - R.token_logp(good["z"].double().numpy(), good["ids"].numpy())[[6, 8, 9, 12]]) <= 1e-4) and lp[7] == lp[13] == 0
    o["logp"][6:15] = 0
    check_pref(w, o)
    # a token of probability zero: its pair's h is infinite
    c = pref_case([0, 4, 9], 9, 100, BF, seed=7)
    c["z"][2, c["ids"][2]] = float("-inf")
    o = run_pref(c)
    assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW and float(o["loss"].item()) == 0 and (o["dlogits"] == 0).all()


def test_preference_in_place_repeatable_and_in_any_layout():
    c = pref_case([0, 6, 11, 15, 17], 17, 1001, BF, seed=8, masked=True)
    a, b = run_pref(c), run_pref(c)
    z, _ = placed(c["z"], 1009, 3)
    d, buf = placed(torch.zeros((17, 1001), dtype=BF), 1005, 6, fill=7.0)
    p = run_pref(c, z=z, dlogits=d)
    assert torch.isnan(z).sum() == 0
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (17, 1001), (1005, 1), 6).fill_(True)
    assert (buf[~inside] == 7.0).all()
    z2 = c["z"].to(DEV)
    q = run_pref(c, z=z2, dlogits=z2)
    for n in ("loss", "reward", "logp", "dlogits"):
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], q[n]), n
    check_pref(c, p)


def test_preference_loss_against_its_own_differences():
    c = pref_case([0, 6, 11, 15, 17], 17, 64, F32, seed=9)
    g = torch.Generator().manual_seed(1)
    v = torch.randn((17, 64), generator=g)
    v /= v.norm()
    h = 2.0 ** -6
    for kind in ("sigmoid", "ipo"):
        z = c["z"].to(DEV)
        o = run_pref(c, kind)
        up, dn = (float(run_pref(c, kind, z=z + s * h * v.to(DEV))["loss"].item()) for s in (1, -1))
        want = float((o["dlogits"].double().cpu() * v.double()).sum())
        size = abs(float(o["loss"].item())) + 1
        assert abs((up - dn) / (2 * h) - want) <= size * (h * h + (4 * U + 8 * eps(64)) / (2 * h))


# --------------------------------------------------------------------------------------- streams, graphs, and together
def test_calls_on_another_stream_wait_for_nothing_on_the_current_one():
    c, f = policy_case(6, 3000, F32, seed=41), pref_case([0, 2, 3, 5, 6], 6, 3000, F32, seed=42)
    ids, zd, yd = c["ids"].to(DEV), c["z"].to(DEV), c["y"].to(DEV)
    t = {n: c[n].to(DEV) for n in ("mu", "adv", "ref", "mask")}
    fd = {n: f[n].to(DEV) for n in ("z", "ids", "cu", "ref")}
    ones = torch.ones(6, device=DEV)

    def calls(**kw):
        l = dppo.dppo_token_logp(zd, ids, **kw)
        return (l["logp"], dppo.dppo_token_logp_bwd(zd, ids, l["lse"], ones, **kw)["dlogits"],
                dppo.dppo_policy_kl_fwd_bwd(zd, ids, t["mu"], t["adv"], t["mask"], ref_logits=yd, kl_form=dppo.KL_PI_REF, **kw)["dlogits"],
                dppo.dppo_preference_fwd_bwd(fd["z"], fd["ids"], fd["cu"], fd["ref"], **kw)["dlogits"])
    want = calls()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.cuda.Event()
    torch.cuda._sleep(400_000_000)
    busy.record()
    got = calls(stream=side)
    side.synchronize()
    assert not busy.query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_replayed_on_new_inputs():
    c1, c2 = policy_case(30, 2000, BF, seed=51), policy_case(30, 2000, BF, seed=52)
    cu = torch.tensor([0, 7, 15, 20, 29], device=DEV)
    names = ("z", "y", "ids", "mu", "adv", "ref", "mask")
    t = {n: c1[n].to(DEV) for n in names}
    st = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step():
        lp = dppo.dppo_token_logp(t["y"], t["ids"], t["mask"], status=st)["logp"]
        a = dppo.dppo_policy_kl_fwd_bwd(t["z"], t["ids"], t["mu"], t["adv"], t["mask"], ref_logp=lp, kl_form=dppo.KL_K3, status=st)
        b = dppo.dppo_policy_kl_fwd_bwd(t["z"], t["ids"], t["mu"], t["adv"], t["mask"], ref_logits=t["y"], kl_form=dppo.KL_REF_PI, status=st)
        p = dppo.dppo_preference_fwd_bwd(t["z"], t["ids"], cu, lp, t["mask"], status=st)
        return [a["loss"], a["dlogits"], b["loss"], b["kl"], b["dlogits"], p["loss"], p["reward"], p["dlogits"]]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for n in names:
        t[n].copy_(c2[n])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_rows_and_offsets_beyond_2_to_31_elements():
    """A row that starts behind element 2^31 of its tensor, in both tensors and the gradient."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    V, stride = 1001, (1 << 30) + 8
    buf = torch.empty(2 * stride + 2048, dtype=BF, device=DEV)
    out = torch.empty(2 * stride + 2048, dtype=BF, device=DEV)
    c = policy_case(3, V, BF, seed=61, masked=False)
    z, d = torch.as_strided(buf, (3, V), (stride, 1), 0), torch.as_strided(out, (3, V), (stride, 1), 0)
    z.copy_(c["z"])
    check_policy(c, run_policy(c, "pi_ref", z=z, y=z.clone().copy_(c["y"]), dlogits=d, mask=False), "pi_ref")
    f = pref_case([0, 1, 3], 3, V, BF, seed=62)
    z.copy_(f["z"])
    check_pref(f, run_pref(f, z=z, dlogits=d))
