"""Cases for the losses against a reference policy and the 4-bit LM head: log-probabilities of given tokens (forward and backward),
the clipped policy loss with a KL term, the loss over pairs of preferred and rejected sequences, rounding weights to 4 bits with a
scale per group, and the product of a few rows with such weights.

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes inputs on the GPU from a seed, ``run`` makes
one pass: in elementary torch operations, or through the library where ``own`` is true.  ``exact`` gives the same outputs from the
definitions in 64 bits, ``work`` the bytes and operations that a pass cannot do without.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------------------- cases
def _logp(name, T, V, dtype, backward, masked):
    return {"name": name, "op": "logp", "T": T, "V": V, "dtype": dtype, "backward": backward, "masked": masked}


def _policy(name, T, V, dtype, kl, masked):
    return {"name": name, "op": "policy", "T": T, "V": V, "dtype": dtype, "kl": kl, "masked": masked}


def _preference(name, pairs, rows, V, dtype, kind, average):
    return {"name": name, "op": "preference", "pairs": pairs, "rows": rows, "V": V, "dtype": dtype, "kind": kind, "average": average}


def _quantize(name, rows, cols, dtype, group):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "group": group}


def _matvec(name, M, N, K, group, out):
    return {"name": name, "op": "matvec", "M": M, "N": N, "K": K, "group": group, "out": out}


def listed():
    return [
        # the reference model's pass over one response: log-probabilities only
        _logp("logp_response_513", 513, 151936, "bf16", False, False),
        # log-probabilities and their gradient for a loss that the user writes, fp32 rows that start at any 4-byte boundary
        _logp("logp_step_f32_odd", 777, 50257, "f32", True, True),
        # a toy step: latency is what counts
        _policy("policy_k3_toy", 256, 4096, "f32", "k3", False),
        # a block of response tokens, KL at the sampled tokens: the usual form of the loss
        _policy("policy_k3_4096", 4096, 151936, "bf16", "k3", True),
        # the same block with the reference policy's logits at hand: KL over the whole vocabulary
        _policy("policy_kl_4096", 4096, 151936, "bf16", "pi_ref", False),
        # the other direction over a vocabulary whose rows start anywhere
        _policy("policy_kl_reversed_odd", 1000, 50257, "bf16", "ref_pi", True),
        # a micro-batch of two short pairs
        _preference("preference_2_short", 2, 93, 32000, "bf16", "sigmoid", False),
        # a micro-batch of long answers
        _preference("preference_16", 16, 6000, 151936, "bf16", "sigmoid", False),
        # the LM head for the rollout after an optimiser step, with the values it stands for
        _quantize("quantize_lm_head", 151936, 2048, "bf16", 128),
        # a small layer of odd sizes in fp32
        _quantize("quantize_odd_f32", 1001, 777, "f32", 32),
        # logits of one request's decoding step
        _matvec("logits_decode_1", 1, 151936, 2048, 128, "bf16"),
        # logits of a server's batch
        _matvec("logits_decode_61", 61, 151936, 2048, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "policy", "policy", "preference", "quantize", "matvec", "matvec"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = rng.choice([151936, 128256, 50257, 32000, _log_int(rng, 1000, 262144)])
    most = 4096 * 151936 * 2 // (V * SIZE[dtype])
    if op == "logp":
        c = _logp("", _log_int(rng, 1, most), V, dtype, rng.random() < 0.5, rng.random() < 0.5)
    elif op == "policy":
        c = _policy("", _log_int(rng, 1, most), V, dtype, rng.choice(["k3", "pi_ref", "ref_pi"]), rng.random() < 0.5)
    elif op == "preference":
        pairs = _log_int(rng, 1, 64)
        c = _preference("", pairs, _log_int(rng, 4 * pairs, max(4 * pairs + 1, min(6000, most))), V, dtype, rng.choice(["sigmoid", "ipo", "hinge"]), rng.random() < 0.3)
    elif op == "quantize":
        cols = rng.choice([1024, 2048, 4096, _log_int(rng, 64, 8192)])
        c = _quantize("", _log_int(rng, 16, 151936 * 2048 // max(cols, 2048)), cols, dtype, rng.choice([32, 64, 128]))
    else:
        K = rng.choice([1024, 2048, 4096, _log_int(rng, 64, 8192)])
        c = _matvec("", _log_int(rng, 1, 64), _log_int(rng, 64, 151936 * 2048 // max(K, 2048)), K, rng.choice([32, 64, 128]), rng.choice(["bf16", "f32"]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _logits(T, V, dtype, g):
    """Rows of unlike sharpness: normal noise over a head that falls off like a power of the rank, and one token lifted by
    anything from nothing to near certainty."""
    z = torch.randn((T, V), generator=g, device=DEV).mul_(3.0)
    start = torch.randint(0, V, (T, 1), generator=g, device=DEV)
    z -= 1.1 * torch.log1p(((torch.arange(V, device=DEV) * 7919 + start) % V).to(torch.float32))
    z[torch.arange(T, device=DEV), start[:, 0]] += 14.0 * torch.rand(T, generator=g, device=DEV)
    return z.to(TYPES[dtype])


def _near(z, by, g):
    """The logits of a policy a little way off, in the same type."""
    out = torch.empty_like(z)
    for i in range(0, z.shape[0], 512):
        part = z[i:i + 512]
        out[i:i + 512] = part.float() + by * torch.randn(part.shape, generator=g, device=DEV)
    return out


def _drawn(z, g):
    """A token per row, drawn from the row's distribution."""
    ids = [(p := z[i:i + 512].float()).sub_(torch.empty_like(p).exponential_(generator=g).log_()).argmax(1) for i in range(0, z.shape[0], 512)]
    return torch.cat(ids).to(torch.int32)


def _logp_of(z, ids):
    """fp32 log-probabilities of the tokens, as a model's earlier pass has stored them."""
    return torch.cat([torch.log_softmax(z[i:i + 512].float(), 1).gather(1, ids[i:i + 512, None].long())[:, 0] for i in range(0, z.shape[0], 512)])


def _token_mask(T, masked, g):
    return (torch.rand(T, generator=g, device=DEV) < 0.8).to(torch.uint8) if masked else None


def _lengths(pairs, rows, g):
    """Rows of the 2 * pairs sequences, one at least each, unlike one another; they end a little before the last row."""
    w = torch.rand(2 * pairs, generator=g, device=DEV, dtype=torch.float64) + 0.05
    n = 1 + torch.floor(w / w.sum() * (rows - 2 * pairs) * 0.98).long()
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.cumsum(n, 0)])


def _pack(codes):
    """Codes 0 .. 15 two to a byte, the even column in the low half; rows of a whole number of 16 bytes."""
    rows, cols = codes.shape
    wide = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.uint8, device=codes.device)
    wide[:, :cols] = codes
    return (wide[:, 0::2] | (wide[:, 1::2] << 4)).contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 29)
    op = case["op"]
    s = {"op": op}
    if op in ("logp", "policy"):
        T = case["T"]
        z = _logits(T, case["V"], case["dtype"], g)
        s.update(logits=z, ids=_drawn(z, g), token_mask=_token_mask(T, case["masked"], g))
        if op == "logp":
            s.update(backward=case["backward"], dlogp=torch.randn(T, generator=g, device=DEV) / T)
        else:
            # the rollout policy is a step or two behind the trainer's, the reference policy further off
            s.update(kl=case["kl"], kl_coef=0.05, eps_low=0.2, eps_high=0.28, advantages=torch.randn(T, generator=g, device=DEV),
                     mu_logp=_logp_of(z, s["ids"]) + 0.15 * torch.randn(T, generator=g, device=DEV), ref_logits=None, ref_logp=None)
            if case["kl"] == "k3":
                s["ref_logp"] = _logp_of(z, s["ids"]) + 0.3 * torch.randn(T, generator=g, device=DEV)
            else:
                s["ref_logits"] = _near(z, 0.3, g)
    elif op == "preference":
        z = _logits(case["rows"], case["V"], case["dtype"], g)
        ids = _drawn(z, g)
        s.update(logits=z, ids=ids, cu_seqlens=_lengths(case["pairs"], case["rows"], g), kind=case["kind"], average=case["average"], beta=0.1,
                 ref_logp=_logp_of(z, ids) + 0.2 * torch.randn(case["rows"], generator=g, device=DEV), smoothing=0.05 if case["kind"] == "sigmoid" else 0.0)
    elif op == "quantize":
        w = 0.02 * torch.randn((case["rows"], case["cols"]), generator=g, device=DEV)
        s.update(w=(w * torch.exp(0.5 * torch.randn((case["rows"], 1), generator=g, device=DEV))).to(TYPES[case["dtype"]]), group=case["group"])
    else:
        M, N, K, G = case["M"], case["N"], case["K"], case["group"]
        codes = torch.empty((N, K), dtype=torch.uint8, device=DEV)
        for i in range(0, N, 8192):
            part = codes[i:i + 8192]
            part.copy_(torch.clamp(torch.round(2.8 * torch.randn(part.shape, generator=g, device=DEV)), -7, 7) + 8)
        s.update(x=torch.randn((M, K), generator=g, device=DEV).to(torch.bfloat16), q=_pack(codes),
                 scale=(0.02 * torch.exp(0.3 * torch.randn((N, -(-K // G)), generator=g, device=DEV))).to(torch.bfloat16), group=G, out=TYPES[case["out"]], K=K)
    if own:     # what a training or decoding loop keeps between its steps
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
def _lse(z):
    """Log-sum-exp of the rows, 64 bits (a ratio next to the clip border, a KL that is a small difference)."""
    out = []
    for i in range(0, z.shape[0], 512):
        p = z[i:i + 512].double()
        m = p.amax(1, keepdim=True)
        out.append(m[:, 0] + torch.log(torch.exp(p - m).sum(1)))
    return torch.cat(out)


def _at(z, ids):
    return z.gather(1, ids[:, None].long())[:, 0].double()


def _valid(s):
    return torch.ones(s["logits"].shape[0], dtype=torch.bool, device=DEV) if s["token_mask"] is None else s["token_mask"] != 0


def _gradient(z, lse, ids, c):
    """c_t (1[j = a_t] - pi_tj) in the type of z."""
    d = torch.exp(z.float() - lse.float()[:, None]).mul_(-c.float()[:, None])
    d[torch.arange(z.shape[0], device=DEV), ids.long()] += c.float()
    return d.to(z.dtype)


def _plain_logp(s):
    z, ok = s["logits"], _valid(s)
    lse = _lse(z)
    out = {"logp": torch.where(ok, _at(z, s["ids"]) - lse, 0.0).float()}
    if s["backward"]:
        out["dlogits"] = _gradient(z, lse, s["ids"], torch.where(ok, s["dlogp"], 0.0))
    return out


def _plain_policy(s):
    z, y, ok = s["logits"], s["ref_logits"], _valid(s)
    T = z.shape[0]
    scale = 1.0 / torch.clamp(ok.sum(), min=1).double()
    lse, adv = _lse(z), s["advantages"].double()
    lp = _at(z, s["ids"]) - lse
    r = torch.exp(lp - s["mu_logp"].double())
    clipped = ((adv > 0) & (r > 1 + s["eps_high"])) | ((adv < 0) & (r < 1 - s["eps_low"]))
    keep = ok & ~clipped
    surrogate = torch.minimum(r * adv, torch.clamp(r, 1 - s["eps_low"], 1 + s["eps_high"]) * adv)
    g = torch.where(keep, scale * r * adv, 0.0)
    b = scale * s["kl_coef"]
    if s["kl"] == "k3":
        x = s["ref_logp"].double() - lp
        kl = torch.exp(x) - x - 1
        d = _gradient(z, lse, s["ids"], torch.where(ok, b * (1 - torch.exp(x)) - g, 0.0))
    else:
        lse_y = _lse(y)
        kl = torch.empty(T, dtype=torch.float64, device=DEV)
        d = torch.empty_like(z)
        for i in range(0, T, 512):
            e = min(T, i + 512)
            lz, ly = z[i:e].float() - lse[i:e, None].float(), y[i:e].float() - lse_y[i:e, None].float()
            wide = (z[i:e].double() - y[i:e].double()) - (lse - lse_y)[i:e, None]
            if s["kl"] == "pi_ref":
                kl[i:e] = (torch.exp(lz).double() * wide).sum(1)
                part = torch.exp(lz) * (g[i:e, None] + b * (wide - kl[i:e, None])).float()
            else:
                kl[i:e] = -(torch.exp(ly).double() * wide).sum(1)
                part = torch.exp(lz) * (g[i:e, None] + b).float() - b * torch.exp(ly)
            part[torch.arange(e - i, device=DEV), s["ids"][i:e].long()] -= g[i:e].float()
            d[i:e] = torch.where(ok[i:e, None], part, 0.0)
    loss = (torch.where(ok, s["kl_coef"] * kl - surrogate, 0.0).sum() * scale).float()
    return {"loss": loss.reshape(1), "kl": torch.where(ok, kl, 0.0).float(), "mask": keep.to(torch.uint8), "dlogits": d}


def _plain_preference(s):
    z, cu, beta, e = s["logits"], s["cu_seqlens"], s["beta"], s["smoothing"]
    P = (cu.numel() - 1) // 2
    lse = _lse(z)
    lp = _at(z, s["ids"]) - lse
    n = (cu[1:] - cu[:-1]).double()
    rows = torch.arange(z.shape[0], device=DEV)
    seq = torch.searchsorted(cu, rows, right=True) - 1                  # sequence of each row; 2 P behind the last one
    inside = seq < 2 * P
    seq = torch.where(inside, seq, 0)
    R = torch.zeros(2 * P, dtype=torch.float64, device=DEV).index_add_(0, seq, torch.where(inside, lp - s["ref_logp"].double(), 0.0))
    weight = 1.0 / n if s["average"] else torch.ones_like(n)
    R = beta * weight * R
    h = R[0::2] - R[1::2]
    if s["kind"] == "sigmoid":
        pair = (1 - e) * torch.log1p(torch.exp(-h)) + e * torch.log1p(torch.exp(h))
        dh = torch.sigmoid(h) - (1 - e)
    elif s["kind"] == "ipo":
        pair = (h / beta - 0.5 / beta) ** 2
        dh = 2 * (h / beta - 0.5 / beta) / beta
    else:
        pair = torch.clamp(1 - h, min=0)
        dh = torch.where(h < 1, -1.0, 0.0)
    c = torch.stack([dh, -dh], 1).reshape(-1) * beta * weight / P       # derivative by each of the sequence's log-probabilities
    return {"loss": pair.mean().float().reshape(1), "reward": R.float(), "logp": torch.where(inside, lp, 0.0).float(),
            "dlogits": _gradient(z, lse, s["ids"], torch.where(inside, c[seq], 0.0))}


def _to_bits(x, bits):
    """x (64 bits) rounded to so many significant bits, ties to even."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)


def _groups(w, G):
    rows, cols = w.shape
    return torch.nn.functional.pad(w, (0, -cols % G)).view(rows, -1, G)


def _plain_quantize(s):
    w, G = s["w"], s["group"]
    rows, cols = w.shape
    values, scales = torch.empty_like(w), []
    for i in range(0, rows, 8192):
        v = _groups(w[i:i + 8192].double(), G)
        scale = _to_bits(torch.clamp(v.abs().amax(2), min=2.0 ** -100) / 7, 8)
        code = torch.clamp(torch.round(v / scale[:, :, None]), -7, 7)
        values[i:i + 8192] = (code * scale[:, :, None]).reshape(v.shape[0], -1)[:, :cols].float().to(w.dtype)
        scales.append(scale.to(torch.bfloat16))
    return {"values": values, "scale": torch.cat(scales)}


def _weights(s):
    """The values that packed codes and scales stand for, fp32."""
    q, K = s["q"], s["K"]
    code = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1)[:, :K].float() - 8
    return code * s["scale"].float().repeat_interleave(s["group"], 1)[:, :K]


def _plain_matvec(s):
    return {"y": (s["x"].float() @ _weights(s).t()).to(s["out"])}


def run(state):
    s = state
    if not own:
        return {"logp": _plain_logp, "policy": _plain_policy, "preference": _plain_preference, "quantize": _plain_quantize, "matvec": _plain_matvec}[s["op"]](s)
    import paper_2602_04879_b200 as dppo
    if s["op"] == "logp":
        o = dppo.dppo_token_logp(s["logits"], s["ids"], s["token_mask"], status=s["status"])
        if not s["backward"]:
            return {"logp": o["logp"]}
        b = dppo.dppo_token_logp_bwd(s["logits"], s["ids"], o["lse"], s["dlogp"], s["token_mask"], status=s["status"])
        return {"logp": o["logp"], "dlogits": b["dlogits"]}
    if s["op"] == "policy":
        form = {"k3": dppo.KL_K3, "pi_ref": dppo.KL_PI_REF, "ref_pi": dppo.KL_REF_PI}[s["kl"]]
        o = dppo.dppo_policy_kl_fwd_bwd(s["logits"], s["ids"], s["mu_logp"], s["advantages"], s["token_mask"], ref_logits=s["ref_logits"], ref_logp=s["ref_logp"],
                                        kl_form=form, kl_coef=s["kl_coef"], eps_low=s["eps_low"], eps_high=s["eps_high"], status=s["status"])
        return {n: o[n] for n in ("loss", "kl", "mask", "dlogits")}
    if s["op"] == "preference":
        kind = {"sigmoid": dppo.PREF_SIGMOID, "ipo": dppo.PREF_IPO, "hinge": dppo.PREF_HINGE}[s["kind"]]
        o = dppo.dppo_preference_fwd_bwd(s["logits"], s["ids"], s["cu_seqlens"], s["ref_logp"], variant=kind, beta=s["beta"], label_smoothing=s["smoothing"],
                                         average=s["average"], status=s["status"])
        return {n: o[n] for n in ("loss", "reward", "logp", "dlogits")}
    if s["op"] == "quantize":
        o = dppo.dppo_int4_quantize(s["w"], s["group"], values=True, status=s["status"])
        return {"values": o["values"], "scale": o["scale"]}
    y, _ = dppo.dppo_matvec_int4(s["x"], s["q"], s["scale"], s["group"], out_dtype=s["out"], status=s["status"])
    return {"y": y}


# --------------------------------------------------------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["rows"] * case["cols"]
        # each weight read once; its half byte, its value and the group's scale written
        return {"bytes": int(n * (2 * SIZE[case["dtype"]] + 0.5)) + 2 * case["rows"] * -(-case["cols"] // case["group"]), "flops": 3 * n}
    if op == "matvec":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * (K // 2) + 2 * N * -(-K // case["group"]) + 2 * M * K + M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    T, size = case["rows"] if op == "preference" else case["T"], SIZE[case["dtype"]]
    n = T * case["V"]
    # every logit (and reference logit) read once, every gradient written once; an exponential and an addition a logit
    if op == "logp":
        return {"bytes": n * size * (2 if case["backward"] else 1) + 12 * T, "flops": 2 * n}
    if op == "policy":
        return {"bytes": n * size * (2 if case["kl"] == "k3" else 3) + 24 * T, "flops": (4 if case["kl"] == "k3" else 9) * n}
    return {"bytes": n * size * 2 + 20 * T, "flops": 4 * n}


# -------------------------------------------------------------------------------------------------------------- exact
def _exact_row_block(z, ids):
    """(log-probabilities of all tokens, those of the given ones), 64 bits."""
    l = torch.log_softmax(z.double(), dim=1)
    return l, l.gather(1, ids[:, None].long())[:, 0]


def _blocks(T, V):
    n = max(1, (1 << 27) // V)
    return [(i, min(T, i + n)) for i in range(0, T, n)]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "matvec":
        out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=DEV)
        for i in range(0, case["N"], 8192):
            part = dict(s, q=s["q"][i:i + 8192], scale=s["scale"][i:i + 8192])
            q = part["q"].long()
            w = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.float64, device=DEV)
            w[:, 0::2], w[:, 1::2] = (q % 16) - 8, q.div(16, rounding_mode="floor") - 8
            w = w[:, :case["K"]]
            for k in range(0, case["K"], case["group"]):
                w[:, k:k + case["group"]] *= part["scale"][:, k // case["group"], None].double()
            out[:, i:i + 8192] = s["x"].double() @ w.t()
        return {"y": out}
    if op == "quantize":
        w, G = s["w"], case["group"]
        values = torch.empty(w.shape, dtype=torch.float64, device=DEV)
        scales = torch.empty((w.shape[0], -(-w.shape[1] // G)), dtype=torch.float64, device=DEV)
        for k in range(0, w.shape[1], G):
            v = w[:, k:k + G].double()
            top = torch.clamp(v.abs().max(1).values, min=2.0 ** -100) / 7
            step = torch.exp2(torch.floor(torch.log2(top)) - 7)         # top is no power of two: seven is in it, or in none of its values
            sc = torch.round(top / step) * step
            scales[:, k // G] = sc
            y = v / sc[:, None]
            low = torch.floor(y)
            up = (y - low > 0.5) | ((y - low == 0.5) & (low % 2 == 1))
            values[:, k:k + G] = torch.clamp(low + up, -7, 7) * sc[:, None]
        return {"values": values, "scale": scales}
    z, ids = s["logits"], s["ids"]
    T, V = z.shape
    if op == "logp":
        ok = torch.ones(T, dtype=torch.bool, device=DEV) if s["token_mask"] is None else s["token_mask"] != 0
        lp, d = [], []
        for i, e in _blocks(T, V):
            l, a = _exact_row_block(z[i:e], ids[i:e])
            lp.append(a * ok[i:e])
            if s["backward"]:
                c = s["dlogp"][i:e].double() * ok[i:e]
                p = torch.exp(l) * -c[:, None]
                p.scatter_add_(1, ids[i:e, None].long(), c[:, None])
                d.append(p)
        return {"logp": torch.cat(lp), **({"dlogits": torch.cat(d)} if s["backward"] else {})}
    if op == "policy":
        ok = torch.ones(T, dtype=torch.bool, device=DEV) if s["token_mask"] is None else s["token_mask"] != 0
        n = max(1, int(ok.sum()))
        # too large for gradients in 64 bits: only the values of the rows
        wide = T * V <= 1 << 29
        kls, d, loss = [], [], 0.0
        for i, e in _blocks(T, V):
            l, a = _exact_row_block(z[i:e], ids[i:e])
            A, okb = s["advantages"][i:e].double(), ok[i:e].double()
            r = torch.exp(a - s["mu_logp"][i:e].double())
            lo, hi = r * A, torch.clamp(r, 1 - s["eps_low"], 1 + s["eps_high"]) * A
            dlp = -torch.where(lo <= hi, lo, torch.zeros_like(lo)) / n      # derivative of the surrogate's term by log pi(a)
            if s["kl"] == "k3":
                ratio = torch.exp(s["ref_logp"][i:e].double() - a)
                kl = ratio - torch.log(ratio) - 1
                dlp = dlp + s["kl_coef"] / n * (1 - ratio)
                grad = -torch.exp(l) * dlp[:, None]
            else:
                ly = torch.log_softmax(s["ref_logits"][i:e].double(), dim=1)
                p = torch.exp(l)
                if s["kl"] == "pi_ref":
                    kl = (p * (l - ly)).sum(1)
                    grad = -p * dlp[:, None] + s["kl_coef"] / n * p * (l - ly - kl[:, None])
                else:
                    kl = (torch.exp(ly) * (ly - l)).sum(1)
                    grad = -p * dlp[:, None] + s["kl_coef"] / n * (p - torch.exp(ly))
            kls.append(kl * okb)
            loss = loss + ((s["kl_coef"] * kl - torch.minimum(lo, hi)) * okb).sum() / n
            if wide:
                grad.scatter_add_(1, ids[i:e, None].long(), dlp[:, None])
                d.append(grad * okb[:, None])
        return {"loss": loss.reshape(1), "kl": torch.cat(kls), "mask": None, "dlogits": torch.cat(d) if wide else None}
    # preference
    cu, beta, eps = s["cu_seqlens"].tolist(), s["beta"], s["smoothing"]
    P = (len(cu) - 1) // 2
    wide = T * V <= 1 << 29
    lp = torch.cat([_exact_row_block(z[i:e], ids[i:e])[1] for i, e in _blocks(T, V)])
    R = torch.zeros(2 * P, dtype=torch.float64, device=DEV, requires_grad=True)
    ratio = lp - s["ref_logp"].double()
    total = torch.stack([beta * (ratio[cu[i]:cu[i + 1]].mean() if s["average"] else ratio[cu[i]:cu[i + 1]].sum()) for i in range(2 * P)])
    with torch.enable_grad():
        h = (total + R)[0::2] - (total + R)[1::2]
        if s["kind"] == "sigmoid":
            pair = -(1 - eps) * torch.nn.functional.logsigmoid(h) - eps * torch.nn.functional.logsigmoid(-h)
        elif s["kind"] == "ipo":
            pair = (h / beta - 1 / (2 * beta)).square()
        else:
            pair = torch.relu(1 - h)
        loss = pair.sum() / P
        by_reward, = torch.autograd.grad(loss, R)
    c = torch.zeros(T, dtype=torch.float64, device=DEV)
    inside = torch.zeros(T, dtype=torch.float64, device=DEV)
    for i in range(2 * P):
        c[cu[i]:cu[i + 1]] = by_reward[i] * beta / (cu[i + 1] - cu[i] if s["average"] else 1)
        inside[cu[i]:cu[i + 1]] = 1
    d = []
    if wide:
        for i, e in _blocks(T, V):
            l, _ = _exact_row_block(z[i:e], ids[i:e])
            p = -torch.exp(l) * c[i:e, None]
            p.scatter_add_(1, ids[i:e, None].long(), c[i:e, None])
            d.append(p)
    return {"loss": loss.detach().reshape(1), "reward": total, "logp": lp * inside, "dlogits": torch.cat(d) if wide else None}
