"""Drawing tokens from rows of logits against the float64 restatement (needs a B200).

Tolerances.  The sums are 64-bit and the exponentials good to 1.3e-12 relative, so the running sums are off by less than 1e-11
of the whole mass: ids are compared wherever no decision of the exact computation is closer than that to flipping.  mu_logp and
the record's probabilities are rounded to fp32 once: 2^-24 relative, plus 1e-11 for what goes before."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EDGE = 1e-11


def _rows(T, V, dtype, seed, sigma=3.0, peak=8.0):
    g = torch.Generator().manual_seed(seed)
    z = sigma * torch.randn((T, V), generator=g)
    z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += peak * torch.rand(T, generator=g)
    return z.to(dtype)


def _uniform(T, seed):
    return torch.rand(T, generator=torch.Generator().manual_seed(seed + 77), dtype=torch.float64)


def _settings(T, seed, kinds):
    g = torch.Generator().manual_seed(seed + 5)
    s = {}
    if "t" in kinds:
        s["temperature"] = 0.3 + 1.2 * torch.rand(T, generator=g)
        s["temperature"][::7] = 0.0
    if "k" in kinds:
        s["top_k"] = torch.randint(-1, 60, (T,), generator=g, dtype=torch.int32)
    if "K" in kinds:
        s["top_k"] = torch.randint(1000, 3000, (T,), generator=g, dtype=torch.int32)
    if "p" in kinds:
        s["top_p"] = 0.3 + 0.75 * torch.rand(T, generator=g)
    if "P" in kinds:
        s["top_p"] = 0.9 + 0.0999 * torch.rand(T, generator=g)
    if "m" in kinds:
        s["min_p"] = 0.2 * torch.rand(T, generator=g) ** 3
    return s


def _on_gpu(z, u, K, s, mask=None, **kw):
    return dppo.dppo_sample(z if z.is_cuda else z.to(DEV), u.to(DEV), K=K, token_mask=None if mask is None else mask.to(DEV),
                            **{n: v.to(DEV) for n, v in s.items()}, **kw)


def _check(out, z, u, K, s, mask=None, rows=None, status=0):
    torch.cuda.synchronize()
    assert int(out["status"].item()) == status
    zh = z.float().cpu().numpy()
    ids, logp = out["sampled_ids"].cpu().numpy(), out["mu_logp"].cpu().numpy()
    tid = out["mu_topk_ids"].cpu().numpy() if K else None
    tp = out["mu_topk_p"].cpu().numpy() if K else None
    compared = 0
    for t in rows if rows is not None else range(zh.shape[0]):
        one = {n: v[t].item() for n, v in s.items()}
        ora = R.sample_row(zh[t], u[t].item(), K=K, **one) if mask is None or mask[t] else None
        if ora is None:
            assert ids[t] == 0 and logp[t] == 0 and (not K or (not tid[t].any() and not tp[t].any())), t
            continue
        assert 0 <= ids[t] < zh.shape[1]
        if K:
            assert np.array_equal(tid[t], ora["top_ids"]), (t, tid[t], ora["top_ids"])
        if ora["margin"] < EDGE:
            continue
        compared += 1
        assert ids[t] == ora["id"], (t, ids[t], ora["id"], ora["margin"], one)
        assert abs(logp[t] - ora["logp"]) <= 2.0 ** -24 * abs(ora["logp"]) + EDGE, (t, logp[t], ora["logp"])
        if K:
            assert np.all(np.abs(tp[t] - ora["top_p"]) <= 2.0 ** -24 * ora["top_p"] + EDGE), t
    return compared


@pytest.mark.parametrize("kinds", ["", "t", "k", "p", "m", "tkpm", "tPm", "P", "K", "tKp", "Km"])
@pytest.mark.parametrize("T,V,dtype,K", [(40, 4096, torch.float32, 20), (33, 50257, torch.bfloat16, 64), (9, 151936, torch.bfloat16, 0),
                                         (150, 1001, torch.float32, 5)])
def test_sampling_matches_the_definition(T, V, dtype, K, kinds):
    z, u, s = _rows(T, V, dtype, seed=V + T), _uniform(T, V), _settings(T, V, kinds)
    assert _check(_on_gpu(z, u, K, s), z, u, K, s) >= T - 1


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 31, 255, 256, 257, 1024, 8191, 20481])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_odd_sizes_and_full_width_records(V, dtype):
    T, K = 12, min(V, 1024)
    z, u, s = _rows(T, V, dtype, seed=V), _uniform(T, V), _settings(T, V, "tpm")
    assert _check(_on_gpu(z, u, K, s), z, u, K, s) >= T - 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 3, 8])
def test_rows_of_a_wider_tensor_at_any_offset(dtype, offset):
    """Row strides above V, rows that start at any element; what lies beside the rows is NaN and must not be looked at."""
    T, V = 10, 3001
    wide = torch.full((T, V + 37), float("nan"), dtype=dtype)
    z = _rows(T, V, dtype, seed=offset)
    wide[:, offset:offset + V] = z
    w, u, s = wide.to(DEV)[:, offset:offset + V], _uniform(T, 3), _settings(T, 3, "tp")
    assert w.stride(0) == V + 37
    assert _check(_on_gpu(w, u, 16, s), z, u, 16, s) >= T - 1


def test_a_row_does_not_depend_on_how_many_share_the_call():
    """1 to 100 rows a call: eight, four, two or one SM per row; the same ids, and values equal up to the order of 64-bit additions."""
    z, u, s = _rows(100, 151936, torch.bfloat16, seed=4), _uniform(100, 4), _settings(100, 4, "tP")
    whole = _on_gpu(z, u, 20, s)
    for T in (1, 18, 19, 37, 74, 75):
        part = _on_gpu(z[:T], u[:T], 20, {n: v[:T] for n, v in s.items()})
        assert torch.equal(part["sampled_ids"], whole["sampled_ids"][:T]) and torch.equal(part["mu_topk_ids"], whole["mu_topk_ids"][:T])
        assert torch.allclose(part["mu_logp"], whole["mu_logp"][:T], rtol=2.0 ** -23, atol=1e-11)
        again = _on_gpu(z[:T], u[:T], 20, {n: v[:T] for n, v in s.items()})
        assert all(torch.equal(part[n], again[n]) for n in part)


def test_more_rows_than_sms():
    """Above 148 rows a CTA has fewer threads and a row to itself: the same ids as when SMs share the rows."""
    for V, dtype in ((151936, torch.bfloat16), (4097, torch.float32)):
        z, u, s = _rows(300, V, dtype, seed=6), _uniform(300, 6), _settings(300, 6, "tkP")
        whole = _on_gpu(z, u, 30, s)
        part = _on_gpu(z[200:260], u[200:260], 30, {n: v[200:260] for n, v in s.items()})
        assert torch.equal(part["sampled_ids"], whole["sampled_ids"][200:260]) and torch.equal(part["mu_topk_ids"], whole["mu_topk_ids"][200:260])
        _check(whole, z, u, 30, s, rows=range(0, 300, 7))


NEG = float("-inf")


def _special_rows(dtype, V=6000):
    """Rows that a mask, a tie or an order makes awkward, each with what is special about it."""
    g = torch.Generator().manual_seed(11)
    base = 2.0 * torch.randn(V, generator=g)
    rows = []

    def add(z):
        rows.append(z.to(dtype))
    add(torch.where(torch.arange(V) == 4321, base, NEG))                       # one token left
    add(torch.where(torch.arange(V) % 500 == 3, base, NEG))                    # fewer tokens left than the record holds
    low = torch.finfo(dtype).min
    add(torch.where(torch.arange(V) % 700 == 1, base, torch.full((V,), low)))  # masked with the type's lowest value
    add(torch.full((V,), low))                                                 # nothing but that: uniform
    add(torch.full((V,), 0.25))                                                # all equal: more ties than the list holds
    add(torch.where(torch.arange(V) < 5000, torch.full((V,), 3.0), base - 9))  # five thousand ties at the top
    add(torch.sort(base).values)                                               # ascending, descending: the largest in few groups
    add(torch.sort(base, descending=True).values)
    add(torch.zeros(V) * torch.where(torch.arange(V) % 2 == 0, 1.0, -1.0))     # +0 and -0 are equal
    add(base * 1e4)                                                            # weights far below the smallest double
    add(base * 1e-4)
    add(torch.where(torch.arange(V) == 7, torch.full((V,), 3e38), base))
    add(torch.where(torch.arange(V) % 3 == 0, base, NEG))
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("setting", [{}, {"top_k": 3}, {"top_k": 40}, {"top_k": 1024}, {"top_k": 1500}, {"top_k": 4500}, {"top_p": 0.5}, {"top_p": 0.999},
                                     {"min_p": 0.3}, {"min_p": 1.0}, {"top_k": 2000, "top_p": 0.7}, {"temperature": 0.01}, {"temperature": 0.0},
                                     {"temperature": 50.0, "top_p": 0.9, "min_p": 1e-3}, {"top_p": 0.0}])
def test_masked_tied_and_ordered_rows(dtype, setting):
    z = _special_rows(dtype)
    T, K = z.shape[0], 30
    for seed in (1, 2):
        u = _uniform(T, seed)
        s = {n: torch.full((T,), v, dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in setting.items()}
        _check(_on_gpu(z, u, K, s), z, u, K, s)


def test_ends_of_the_unit_interval():
    z = _rows(8, 5000, torch.float32, seed=2)
    z[0, :100] = NEG
    z[1, -100:] = NEG
    first = torch.zeros(8, dtype=torch.float64)
    out = _on_gpu(z, first, 0, {})
    assert out["sampled_ids"].tolist() == [100] + [0] * 7
    s = {"top_k": torch.full((8,), 50, dtype=torch.int32)}
    out = _on_gpu(z, first, 0, s)
    assert out["sampled_ids"].tolist() == [int(torch.topk(r, 50).indices.min()) for r in z]
    last = torch.full((8,), 1.0 - 2.0 ** -53, dtype=torch.float64)
    out = _on_gpu(z, last, 0, s)
    assert out["sampled_ids"].tolist() == [int(torch.topk(r, 50).indices.max()) for r in z]
    out = _on_gpu(z, last, 0, {})
    assert all(np.isfinite(z[t, i].item()) for t, i in enumerate(out["sampled_ids"].tolist()))


def test_dropped_rows_and_status_bits():
    z = _rows(8, 3000, torch.float32, seed=9)
    u = _uniform(8, 9)
    z[1, 77] = float("nan")
    z[2, 2999] = float("inf")
    z[3] = NEG
    z[4, 5] = -float("nan")
    mask = torch.tensor([1, 1, 1, 1, 1, 0, 1, 1], dtype=torch.uint8)
    out = _on_gpu(z, u, 4, {}, mask)
    _check(out, z, u, 4, {}, mask, status=binding.STATUS_NONFINITE_ROW)
    # a masked row may hold anything: it is not read
    z[5] = float("nan")
    only = torch.tensor([1, 0, 0, 0, 0, 0, 1, 1], dtype=torch.uint8)
    _check(_on_gpu(z, u, 4, {}, only), z, u, 4, {}, only)
    good = _rows(6, 500, torch.float32, seed=1)
    bad = {"temperature": [-1.0, float("nan"), float("inf")], "top_p": [-0.1, float("nan")], "min_p": [-0.1, 1.5, float("nan")]}
    for name, values in bad.items():
        for v in values:
            s = {name: torch.tensor([0.5, 0.5, v, 0.5, 0.5, 0.5])}
            out = _on_gpu(good, u[:6], 4, s)
            torch.cuda.synchronize()
            assert int(out["status"].item()) == binding.STATUS_BAD_SAMPLING
            assert out["sampled_ids"][2] == 0 and out["mu_logp"][2] == 0 and not out["mu_topk_p"][2].any()
            s[name][2] = 0.5
            _check(_on_gpu(good, u[:6], 4, s), good, u[:6], 4, s)
    for v in (1.0, -1e-300, float("nan")):
        uu = u[:6].clone()
        uu[3] = v
        out = _on_gpu(good, uu, 0, {})
        torch.cuda.synchronize()
        assert int(out["status"].item()) == binding.STATUS_BAD_SAMPLING and out["sampled_ids"][3] == 0


def test_empty_batch_and_outputs_of_the_caller():
    out = _on_gpu(torch.empty((0, 100)), torch.empty(0, dtype=torch.float64), 5, {})
    assert out["sampled_ids"].shape == (0,) and out["mu_topk_ids"].shape == (0, 5)
    z, u = _rows(3, 400, torch.float32, seed=3), _uniform(3, 3)
    # the outputs are views into larger buffers whose other entries stay as they were
    ids = torch.full((5,), -7, dtype=torch.int32, device=DEV)
    lp = torch.full((5,), -7.0, device=DEV)
    ti = torch.full((5, 6), -7, dtype=torch.int32, device=DEV)
    tp = torch.full((5, 6), -7.0, device=DEV)
    out = _on_gpu(z, u, 6, {}, out=dict(sampled_ids=ids[1:4], mu_logp=lp[1:4], mu_topk_ids=ti[1:4], mu_topk_p=tp[1:4]))
    _check(out, z, u, 6, {})
    assert all(b[0].eq(-7).all() and b[4].eq(-7).all() for b in (ids, lp, ti, tp))


def test_long_rows_beyond_the_usual_vocabulary():
    for V, dtype in ((1 << 20, torch.bfloat16), ((1 << 21) + 3, torch.float32)):
        z, u = _rows(2, V, dtype, seed=5), _uniform(2, 5)
        for kinds in ("", "P", "k"):
            s = _settings(2, 6, kinds)
            _check(_on_gpu(z, u, 10, s), z, u, 10, s)


def test_graph_replay_other_streams_and_concurrent_calls():
    z, u, s = _rows(30, 50257, torch.bfloat16, seed=8).to(DEV), _uniform(30, 8).to(DEV), _settings(30, 8, "tkp")
    s = {n: v.to(DEV) for n, v in s.items()}
    ref = dppo.dppo_sample(z, u, K=8, **s)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = dppo.dppo_sample(z, u, K=8, status=st, **s)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[n], ref[n]) for n in ("sampled_ids", "mu_logp", "mu_topk_ids", "mu_topk_p"))
    u2 = _uniform(30, 9)
    u.copy_(u2)
    g.replay()
    torch.cuda.synchronize()
    _check(out, z.cpu(), u2, 8, {n: v.cpu() for n, v in s.items()})
    ref = {n: v.clone() for n, v in out.items()}
    side = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for q in side:
        q.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(q):
            outs += [dppo.dppo_sample(z, u, K=8, **s) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(o[n], ref[n]) for o in outs for n in ("sampled_ids", "mu_logp", "mu_topk_ids", "mu_topk_p"))


@pytest.mark.parametrize("K", [20])
def test_the_record_feeds_the_loss(K):
    """Sampled, then evaluated under the same logits: ratio 1, no divergence beyond fp32, nothing masked, for every variant that
    reads the record."""
    z, u, adv = _rows(64, 32000, torch.bfloat16, seed=1).to(DEV), _uniform(64, 1).to(DEV), torch.ones(64, device=DEV)
    o = dppo.dppo_sample(z, u, K=K)
    for variant in (dppo.BINARY_TV, dppo.BINARY_KL, dppo.TOPK_TV, dppo.TOPK_KL):
        r = dppo.dppo_loss_fwd_bwd(z, o["sampled_ids"], o["mu_logp"], adv, None, variant, K, 1e-4, o["mu_topk_ids"], o["mu_topk_p"], want_stats=True)
        torch.cuda.synchronize()
        assert int(r["status"].item()) == 0 and bool(r["mask"].all()) and float(r["divergence"].abs().max()) <= 1e-5
        assert abs(float(r["loss"].item()) + 1.0) <= 1e-5                      # -mean(r A) with r = 1, A = 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("setting,rest", [({"top_p": 0.9999}, -30.0), ({"top_k": 4096}, -30.0), ({"top_k": 4096, "top_p": 0.9999}, -30.0),
                                          ({"top_p": 0.9999, "temperature": 1e36}, -3e38)])
def test_a_full_list_of_the_largest_weight_in_one_chunk(dtype, setting, rest):
    """4096 tokens of weight 1 side by side, as many as the sorted list holds, in one of a long row's chunks, and a few hundred light ones
    all over the row: the cut takes in the whole list, whose weights add up within that chunk."""
    V = 1 << 20
    g = torch.Generator().manual_seed(33)
    z = torch.full((3, V), NEG)
    z[:, ::1500] = rest
    for t, first in enumerate((64, 3 * 4352 + 100, 200 * 4224 + 50)):     # chunks of 4352 elements in bf16, of 4224 in fp32
        z[t, (first // 4352 * 4352 if dtype == torch.bfloat16 else first // 4224 * 4224) + 64:][:4096] = 0.25
    if "temperature" in setting:
        z = torch.where(z == 0.25, torch.randn((3, V), generator=g), z)   # so hot that unlike logits all weigh 1
    z, u = z.to(dtype), _uniform(3, 33)
    s = {n: torch.full((3,), v, dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in setting.items()}
    assert _check(_on_gpu(z, u, 30, s), z, u, 30, s) >= 2


VARIANTS = (dppo.BINARY_TV, dppo.BINARY_KL, dppo.TOPK_TV, dppo.TOPK_KL)


def test_the_readme_example_compares_like_distributions():
    """The README's lines as they stand, with the trainer's logits equal to the rollout's: no divergence beyond fp32, nothing masked."""
    import os
    import textwrap
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    lines = textwrap.dedent(text[text.index("The rollout side"):].split("```python\n")[1].split("```")[0]).rstrip()
    first, loss = lines.rsplit("\n", 1)
    g = torch.Generator().manual_seed(3)
    T, d, V = 96, 256, 1000
    ns = dict(dppo=dppo, torch=torch, W=(0.2 * torch.randn((V, d), generator=g)).to(torch.bfloat16).to(DEV), uniform=_uniform(T, 3).to(DEV),
              hidden=torch.randn((T, d), generator=g).to(torch.bfloat16).to(DEV), adv=torch.where(torch.rand(T, generator=g) < 0.5, -1.0, 1.0).to(DEV),
              tau=torch.full((T,), 0.7, device=DEV), p=torch.full((T,), 0.9, device=DEV))
    exec(first, ns)
    ns["logits"] = ns["z"]
    exec(loss, ns)
    assert int(ns["r"]["status"].item()) == 0 and int(ns["o"]["status"].item()) == 0
    assert bool(ns["r"]["mask"].all()) and float(ns["r"]["divergence"].abs().max()) <= 1e-5


def test_a_record_at_another_temperature_feeds_the_loss_on_scaled_logits():
    """The record is softmax(z / tau)'s.  Against logits divided by tau in fp32, each off by at most e = 2^-24 max |z / tau|, so that a
    log probability is off by at most 2 e, the loss finds a ratio of 1 and no divergence: within its own 1e-5 (divergence) and 1e-4
    (loss) and what 2 e does to them."""
    T, V, K = 64, 32000, 20
    z, u = _rows(T, V, torch.float32, seed=1), _uniform(T, 1)
    tau = 0.4 + 1.2 * torch.rand(T, generator=torch.Generator().manual_seed(2))
    scaled = z / tau[:, None]
    e = 2.0 ** -24 * float(scaled.abs().max())
    o = _on_gpu(z, u, K, {"temperature": tau})
    for variant in VARIANTS:
        r = dppo.dppo_loss_fwd_bwd(scaled.to(DEV), o["sampled_ids"], o["mu_logp"], torch.ones(T, device=DEV), None, variant, K, 1e-3, o["mu_topk_ids"], o["mu_topk_p"])
        torch.cuda.synchronize()
        assert int(r["status"].item()) == 0 and bool(r["mask"].all()) and float(r["divergence"].abs().max()) <= 1e-5 + 4 * e
        assert abs(float(r["loss"].item()) + 1.0) <= 1e-4 + 2 * e


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_record_with_cuts_against_the_loss_oracle(dtype):
    """Cut-off tokens stand in the record with probability 0.  The loss takes the record as it is: the truncated distribution against the
    whole softmax, which differ by the mass that was cut."""
    from oracle import dppo_oracle as O
    from parity_util import check_dlogits, check_loss, check_scalars
    T, V, K = 48, 3000, 20
    z, u = _rows(T, V, dtype, seed=12, sigma=1.5), _uniform(T, 12)
    g = torch.Generator().manual_seed(13)
    s = {"top_k": torch.randint(1, 40, (T,), generator=g, dtype=torch.int32), "top_p": 0.5 + 0.5 * torch.rand(T, generator=g)}
    o = _on_gpu(z, u, K, s)
    assert bool((o["mu_topk_p"] == 0).any()) and float(o["mu_topk_p"].sum(1).min()) > 0
    adv = torch.where(torch.rand(T, generator=g) < 0.5, -1.0, 1.0)
    host = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731
    zs = (z + 0.05 * torch.randn((T, V), generator=g)).to(dtype)
    for variant in VARIANTS:
        r = dppo.dppo_loss_fwd_bwd(zs.to(DEV), o["sampled_ids"], o["mu_logp"], adv.to(DEV), None, variant, K, 0.3, o["mu_topk_ids"], o["mu_topk_p"])
        torch.cuda.synchronize()
        assert int(r["status"].item()) == 0
        ora = O.dppo_loss_fwd_bwd(host(zs.float()), o["sampled_ids"].cpu().numpy(), host(o["mu_logp"]), host(adv), None, variant, K, 0.3, None,
                                  o["mu_topk_ids"].cpu().numpy(), host(o["mu_topk_p"]))
        check_scalars(r["divergence"].cpu().numpy(), r["mask"].cpu().numpy(), ora, {"token_mask": None}, 0.3)
        check_loss(float(r["loss"].item()), ora["loss"], dtype == torch.bfloat16)
        check_dlogits(r["dlogits"], ora["dlogits"], dtype == torch.bfloat16)
        if variant == dppo.BINARY_TV:
            assert float(r["divergence"].mean()) > 0.05


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top_p", [0.0, 1e-45, 1e-30])
@pytest.mark.parametrize("top_k,temperature", [(1025, 1.0), (1500, 1.0), (5000, 30.0), (4500, 1e5), (3000, 0.01)])
def test_a_top_p_of_nothing_within_a_long_top_k(dtype, top_p, top_k, temperature):
    """A prefix of at least 0 of the mass still holds one token, also where ties or a high temperature put more tokens next to the
    largest than the list holds, so that the cut is bracketed.  One row alone, rows that share the call, and one CTA per row."""
    z = _special_rows(dtype)
    T = z.shape[0]
    u = _uniform(T, 17)

    def settings(n):
        return {"top_k": torch.full((n,), top_k, dtype=torch.int32), "top_p": torch.full((n,), top_p), "temperature": torch.full((n,), temperature)}
    out = _on_gpu(z, u, 30, settings(T))
    _check(out, z, u, 30, settings(T))
    many = _on_gpu(z.repeat(20, 1), u.repeat(20), 30, settings(20 * T))
    assert torch.equal(many["sampled_ids"].view(20, T), out["sampled_ids"].expand(20, T))
    for t in (3, 4, 5):
        one = _on_gpu(z[t:t + 1], u[t:t + 1], 0, settings(1))
        assert int(one["sampled_ids"][0]) == int(out["sampled_ids"][t]) == int(z[t].float().argmax())


def test_more_than_2_31_logits():
    """16384 rows of 151936: rows behind element 2^31 are what a call on them alone draws, and what the definition says."""
    T, V, K = 16384, 151936, 20
    g = torch.Generator(device=DEV).manual_seed(5)
    z = torch.empty((T, V), dtype=torch.bfloat16, device=DEV)
    for i in range(0, T, 2048):
        z[i:i + 2048] = 3.0 * torch.randn((2048, V), generator=g, device=DEV)
    u, s = _uniform(T, 5), _settings(T, 5, "tkP")
    out = _on_gpu(z, u, K, s)
    first = T - 400
    assert first * V > 2 ** 31
    tail = _on_gpu(z[first:], u[first:], K, {n: v[first:] for n, v in s.items()})
    assert int(out["status"].item()) == 0 and all(torch.equal(out[n][first:], tail[n]) for n in ("sampled_ids", "mu_logp", "mu_topk_ids", "mu_topk_p"))
    rows = torch.tensor([0, 7000, 14135, 14136, T - 1])
    few = {n: v[rows.to(DEV)] for n, v in out.items() if n != "status"}
    _check(dict(few, status=out["status"]), z[rows.to(DEV)], u[rows], K, {n: v[rows] for n, v in s.items()})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_longest_rows(dtype):
    """V = 2^30, the documented limit: equal weights everywhere, whose running sums are exact, and a thousand tokens far apart."""
    V = 1 << 30
    z = torch.full((2, V), 0.5, dtype=dtype, device=DEV)
    u = torch.tensor([0.999999999, 0.123456789], dtype=torch.float64)
    out = _on_gpu(z, u, 0, {})
    assert out["sampled_ids"].tolist() == [int(x * V) for x in u.tolist()] and int(out["status"].item()) == 0
    assert float((out["mu_logp"].double().cpu() + np.log(V)).abs().max()) <= 2.0 ** -24 * np.log(V) + EDGE
    where = torch.arange(1023, V, 1 << 20)
    z.fill_(NEG)
    vals = 2.0 * torch.randn((2, where.numel()), generator=torch.Generator().manual_seed(6))
    z[:, where.to(DEV)] = vals.to(dtype).to(DEV)
    for s in ({}, {"top_k": torch.full((2,), 100, dtype=torch.int32)}, {"top_p": torch.full((2,), 0.9)}, {"min_p": torch.full((2,), 0.05)}):
        out = _on_gpu(z, u, 10, s)
        assert int(out["status"].item()) == 0
        for t in range(2):
            ora = R.sample_row(vals[t].to(dtype).float().numpy(), u[t].item(), K=10, **{n: v[t].item() for n, v in s.items()})
            assert out["mu_topk_ids"][t].tolist() == where[ora["top_ids"]].tolist()
            if ora["margin"] >= EDGE:
                assert int(out["sampled_ids"][t]) == int(where[ora["id"]])
                assert abs(float(out["mu_logp"][t]) - ora["logp"]) <= 2.0 ** -24 * abs(ora["logp"]) + EDGE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("setting", [{"top_p": 0.6}, {"top_k": 1500}, {"top_k": 12000}, {"top_k": 12000, "top_p": 0.6}, {"top_k": 12000, "top_p": 0.6, "min_p": 0.999}])
def test_each_way_to_a_cut(dtype, setting):
    """Rows whose cut lies in the first list; below it, among tokens that a step of the histogram tells apart; among more tokens of one
    step than the list holds (the cut is bracketed); among as many equal ones.  By mass and by count, rows that share SMs and rows
    that do not."""
    V, few = 50257, 4
    g = torch.Generator().manual_seed(41)
    at = torch.randperm(V, generator=g)
    z = torch.full((few, V), -20.0)
    z[0] = 4.0 * torch.randn(V, generator=g)
    z[1, at[:14000]] = 2.0 + 3.0 * torch.rand(14000, generator=g)
    z[2, at[:20000]] = 1.0 + 0.01 * torch.rand(20000, generator=g)
    z[3, at[:20000]] = 1.0
    z, u = z.to(dtype), _uniform(few, 41)

    def settings(n):
        return {k: torch.full((n,), v, dtype=torch.int32 if k == "top_k" else torch.float32) for k, v in setting.items()}
    out = _on_gpu(z, u, 30, settings(few))
    assert _check(out, z, u, 30, settings(few)) >= few - 1
    many = _on_gpu(z.repeat(50, 1), u.repeat(50), 30, settings(50 * few))
    assert torch.equal(many["sampled_ids"].view(50, few), out["sampled_ids"].expand(50, few))
    assert torch.equal(many["mu_topk_ids"][-few:], out["mu_topk_ids"])
