"""Cases for the operators around a rollout step and its update: drawing tokens from a row of logits (with the record
that the DPPO loss reads), rounding tensors to 8-bit floating point with a scale for each block of 128, and the matrix
product of such tensors (logits of the LM head, gradients of the hidden states and of the LM head).

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes inputs on the GPU from a seed,
``run`` makes one pass: in elementary torch operations, or through the library where ``own`` is true.  ``exact`` gives the
same outputs from the definitions in 64 bits, ``work`` the bytes and operations that a pass cannot do without.
"""
import math

import torch

own = False
DEV = "cuda"
G = 128                                   # elements that share a scale
BIG = {"e4m3": 448.0, "e5m2": 57344.0}    # largest finite value of the 8-bit types
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------- cases
def _sample(name, T, V, dtype, filters, K):
    return {"name": name, "op": "sample", "T": T, "V": V, "dtype": dtype, "filters": filters, "K": K}


def _quantize(name, rows, cols, dtype, fmt, block_rows, both, data):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "fmt": fmt, "block_rows": block_rows,
            "both": both, "data": data}


def _product(name, M, N, K, a_fmt, b_block_rows, out, data):
    return {"name": name, "op": "product", "M": M, "N": N, "K": K, "a_fmt": a_fmt, "b_block_rows": b_block_rows, "out": out, "data": data}


def listed():
    return [
        # one request, one token: the row of a single decoding step with the usual chat settings; latency is what counts
        _sample("sample_decode_1", 1, 151936, "bf16", "chat", 0),
        # a decoding step of a server's batch: every request has its own settings (greedy ones among them); the top-20 record
        _sample("sample_decode_61_mixed", 61, 151936, "bf16", "mixed", 20),
        # rollouts as the trainer wants them: temperature 1, nothing cut off, the top-64 record for the Top-K divergence
        _sample("sample_rollout_2048", 2048, 151936, "bf16", "none", 64),
        # nucleus sampling alone from fp32 rows that start at any 4-byte boundary
        _sample("sample_top_p_f32", 256, 50257, "f32", "top_p", 0),
        # hidden states of one decoding step, in front of the LM head
        _quantize("quantize_hidden_61", 61, 2048, "bf16", "e4m3", 1, False, "normal"),
        # the LM head after an optimiser step: one scale for each 128 x 128, and transposed for the hidden states' gradient
        _quantize("quantize_lm_head", 151936, 2048, "bf16", "e4m3", 128, True, "weight"),
        # the loss's gradient with respect to the logits, along the vocabulary and (for the LM head's gradient) along the rows
        _quantize("quantize_dlogits", 2048, 151936, "bf16", "e5m2", 1, True, "dlogits"),
        # logits of one decoding step of a server's batch
        _product("logits_decode_61", 61, 151936, 2048, "e4m3", 128, "bf16", "weight"),
        # logits of a block of response tokens in training
        _product("logits_4096", 4096, 151936, 2048, "e4m3", 128, "bf16", "weight"),
        # gradient of the hidden states: dlogits . W, a sum over the vocabulary
        _product("dhidden_2048", 2048, 2048, 151936, "e5m2", 128, "f32", "dlogits"),
        # gradient of the LM head: dlogits^T . hidden, a sum over the rows
        _product("dlmhead_2048", 151936, 2048, 2048, "e5m2", 1, "f32", "dlogits"),
        # a small layer of odd sizes
        _product("product_odd", 333, 1001, 777, "e4m3", 1, "f32", "normal"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "quantize", "product"])
    if op == "sample":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        V = rng.choice([151936, 128256, 50257, 32000, _log_int(rng, 1000, 262144)])
        most = min(4096, 2048 * 151936 * 2 // (V * (2 if dtype == "bf16" else 4)))
        T = _log_int(rng, 1, most)
        c = _sample("", T, V, dtype, rng.choice(["none", "chat", "mixed", "top_p", "top_k", "min_p"]), rng.choice([0, 0, 20, 64, rng.randint(1, 100)]))
    elif op == "quantize":
        cols = rng.choice([2048, 151936, _log_int(rng, 100, 160000)])
        rows = _log_int(rng, 1, max(2, min(160000, 2048 * 151936 // cols)))
        c = _quantize("", rows, cols, rng.choice(["bf16", "f32"]), rng.choice(["e4m3", "e5m2"]), rng.choice([1, 128]), rng.random() < 0.5,
                      rng.choice(["normal", "weight", "dlogits"]))
    else:
        kind = rng.choice(["logits", "dhidden", "dlmhead", "layer"])
        if kind == "logits":
            c = _product("", _log_int(rng, 1, 4096), rng.choice([151936, 50257, _log_int(rng, 1000, 151936)]), rng.choice([1024, 2048, 777]), "e4m3", 128,
                         rng.choice(["bf16", "f32"]), "weight")
        elif kind == "dhidden":
            c = _product("", _log_int(rng, 16, 2048), rng.choice([1024, 2048]), _log_int(rng, 8192, 151936), rng.choice(["e4m3", "e5m2"]), 128, "f32", "dlogits")
        elif kind == "dlmhead":
            c = _product("", _log_int(rng, 8192, 151936), rng.choice([1024, 2048]), _log_int(rng, 100, 2048), rng.choice(["e4m3", "e5m2"]), 1, "f32", "dlogits")
        else:
            c = _product("", _log_int(rng, 16, 4096), _log_int(rng, 64, 4096), _log_int(rng, 64, 8192), "e4m3", rng.choice([1, 128]),
                         rng.choice(["bf16", "f32"]), "normal")
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _logits(T, V, dtype, g):
    """Rows of unlike sharpness: normal noise over a head that falls off like a power of the rank, and one token lifted by
    anything from nothing to near certainty."""
    z = 3.0 * torch.randn((T, V), generator=g, device=DEV)
    start = torch.randint(0, V, (T, 1), generator=g, device=DEV)
    z -= 1.1 * torch.log1p(((torch.arange(V, device=DEV) * 7919 + start) % V).to(torch.float32))
    lift = 14.0 * torch.rand(T, generator=g, device=DEV)
    z[torch.arange(T, device=DEV), start[:, 0]] += lift
    return z.to(TYPES[dtype])


def _settings(T, filters, g):
    """Per-row settings as a server holds them; None where the batch does not use one."""
    def uni(lo, hi):
        return lo + (hi - lo) * torch.rand(T, generator=g, device=DEV)

    def full(v, dtype=torch.float32):
        return torch.full((T,), v, dtype=dtype, device=DEV)
    s = {"temperature": None, "top_k": None, "top_p": None, "min_p": None}
    if filters == "chat":
        s.update(temperature=full(0.7), top_k=full(20, torch.int32), top_p=full(0.95))
    elif filters == "top_p":
        s.update(temperature=full(0.9), top_p=uni(0.8, 0.95))
    elif filters == "top_k":
        s.update(temperature=uni(0.6, 1.2), top_k=torch.randint(1, 400, (T,), generator=g, device=DEV, dtype=torch.int32))
    elif filters == "min_p":
        s.update(temperature=uni(0.6, 1.5), min_p=uni(0.01, 0.1))
    elif filters == "mixed":
        off = lambda p: torch.rand(T, generator=g, device=DEV) < p  # noqa: E731
        s.update(temperature=torch.where(off(0.15), full(0.0), uni(0.6, 1.2)),
                 top_k=torch.where(off(0.4), full(0, torch.int32), torch.randint(1, 200, (T,), generator=g, device=DEV, dtype=torch.int32)),
                 top_p=torch.where(off(0.4), full(1.0), uni(0.8, 0.99)),
                 min_p=torch.where(off(0.6), full(0.0), uni(0.02, 0.1)))
    return s


def _values(rows, cols, data, g):
    """fp32 values as the path meets them: hidden states, weights of a layer, or a loss gradient (a probability row times a
    small factor, with one large entry of the other sign)."""
    x = torch.randn((rows, cols), generator=g, device=DEV)
    if data == "weight":
        return x.mul_(0.02)
    if data == "dlogits":
        x = torch.softmax(2.0 * x, dim=1)
        x[torch.arange(rows, device=DEV), torch.randint(0, cols, (rows,), generator=g, device=DEV)] -= 1.0
        return x.mul_(torch.randn((rows, 1), generator=g, device=DEV) / rows)
    return x


def _padded(t, multiple=16):
    """The same values in rows that start on a multiple of 16 bytes, as the 8-bit tensors of the path are kept."""
    wide = -(-t.shape[1] // multiple) * multiple
    if wide == t.shape[1]:
        return t.contiguous()
    out = torch.zeros((t.shape[0], wide), dtype=torch.uint8, device=DEV).view(t.dtype)
    out[:, :t.shape[1]] = t
    return out[:, :t.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 17)
    if case["op"] == "sample":
        T = case["T"]
        s = {"logits": _logits(T, case["V"], case["dtype"], g), "uniform": torch.rand(T, generator=g, device=DEV, dtype=torch.float64),
             "K": case["K"], **_settings(T, case["filters"], g)}
        if own:     # what a decoding loop keeps between its steps
            s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    elif case["op"] == "quantize":
        s = {"x": _values(case["rows"], case["cols"], case["data"], g).to(TYPES[case["dtype"]]), "fmt": case["fmt"], "block_rows": case["block_rows"],
             "both": case["both"]}
        if own:
            s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    else:
        M, N, K = case["M"], case["N"], case["K"]
        a = _values(M, K, case["data"] if case["data"] == "dlogits" else "normal", g)
        b = _values(N, K, "weight" if case["b_block_rows"] == G else "normal", g)
        qa, sa = _blocks(a, case["a_fmt"], 1)
        qb, sb = _blocks(b, "e4m3", case["b_block_rows"])
        # the scales as the quantiser lays them out: the block index along K is the slow one
        s = {"a": _padded(qa), "a_scale": sa.t().contiguous().t(), "b": _padded(qb), "b_scale": sb.t().contiguous().t(),
             "b_block_rows": case["b_block_rows"], "out": TYPES[case["out"]]}
        if own:
            s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    s["op"] = case["op"]
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
def _blocks(x, fmt, block_rows):
    """(8-bit values, scales): groups of block_rows x 128 along the last dimension share scale = amax / largest value; the
    value stored is x / scale, rounded to nearest even.  The quotient is formed as (7/8 x) / (amax / 2^n), largest value =
    7/8 2^n: one rounding, and none at all where it lies half way between two 8-bit values."""
    rows, cols = x.shape
    x = x.to(torch.float32)
    pad = torch.nn.functional.pad(x, (0, -cols % G, 0, -rows % block_rows))
    v = pad.view(pad.shape[0] // block_rows, block_rows, pad.shape[1] // G, G)
    amax = v.abs().amax(dim=(1, 3))
    amax = torch.clamp(amax, min=2.0 ** -100)           # groups of zeros and of tiny values: the scale stays a normal number
    q = ((0.875 * v) / (amax * (0.875 / BIG[fmt]))[:, None, :, None]).reshape(pad.shape)[:rows, :cols]
    return q.to(F8[fmt]), amax / BIG[fmt]


def _plain_sample(s):
    z, order = torch.sort(s["logits"].to(torch.float32), dim=1, descending=True, stable=True)
    T, V = z.shape
    rank = torch.arange(V, device=z.device)
    one = torch.ones(T, dtype=torch.float64, device=z.device)
    temp = one if s["temperature"] is None else s["temperature"].double()
    k = torch.where(temp == 0, 1, V) if s["top_k"] is None else torch.where(temp == 0, 1, torch.where(s["top_k"] > 0, s["top_k"].long(), V))
    p = one if s["top_p"] is None else s["top_p"].double()
    m = 0 * one if s["min_p"] is None else s["min_p"].double()
    temp = torch.where(temp == 0, one, temp)
    w = torch.exp((z.double() - z[:, :1].double()) / temp[:, None])
    w = torch.where(rank < k[:, None], w, 0.0)
    mass = torch.cumsum(w, dim=1)
    keep = (rank == 0) | (p >= 1)[:, None] | (mass - w < p[:, None] * mass[:, -1:])
    w = torch.where(keep & (w >= m[:, None]), w, 0.0)
    c = torch.cumsum(torch.zeros_like(w).scatter_(1, order, w), dim=1)        # over the tokens in the order of their ids
    total = c[:, -1:]
    ids = (c <= s["uniform"][:, None] * total).sum(dim=1).clamp(max=V - 1)
    za = s["logits"].gather(1, ids[:, None]).double()
    logp = ((za - z[:, :1].double()) / temp[:, None] - torch.log(total))[:, 0]
    out = {"sampled_ids": ids.to(torch.int32), "mu_logp": logp.float()}
    if s["K"]:
        out["mu_topk_ids"] = order[:, :s["K"]].to(torch.int32)
        out["mu_topk_p"] = (w[:, :s["K"]] / total).float()
    return out


def _plain_quantize(s):
    q, scale = _blocks(s["x"], s["fmt"], s["block_rows"])
    out = {"q": q, "scale": scale}
    if s["both"]:
        out["qt"], out["qt_scale"] = _blocks(s["x"].t(), s["fmt"], s["block_rows"])
    return out


def _spread(scale, rows, cols, block_rows):
    return scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(G, 1)[:, :cols]


def _plain_product(s):
    a = s["a"].to(torch.float32) * _spread(s["a_scale"], *s["a"].shape, 1)
    b = s["b"].to(torch.float32) * _spread(s["b_scale"], *s["b"].shape, s["b_block_rows"])
    return {"c": (a @ b.t()).to(s["out"])}


def run(state):
    s = state
    if own:
        import paper_2602_04879_b200 as dppo
        if s["op"] == "sample":
            o = dppo.dppo_sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], K=s["K"], status=s["status"])
            return {n: o[n] for n in ("sampled_ids", "mu_logp") + (("mu_topk_ids", "mu_topk_p") if s["K"] else ())}
        if s["op"] == "quantize":
            o = dppo.dppo_fp8_quantize(s["x"], F8[s["fmt"]], s["block_rows"], transposed=s["both"], status=s["status"])
            return {n: o[n] for n in ("q", "scale") + (("qt", "qt_scale") if s["both"] else ())}
        c, _ = dppo.dppo_gemm_tn_fp8(s["a"], s["a_scale"], s["b"], s["b_scale"], b_block_rows=s["b_block_rows"], out_dtype=s["out"], status=s["status"])
        return {"c": c}
    return {"sample": _plain_sample, "quantize": _plain_quantize, "product": _plain_product}[s["op"]](s)


# --------------------------------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == "sample":
        n = case["T"] * case["V"]
        # every logit is read once and costs an exponential and an addition; what comes back is a few words a row
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + case["T"] * (16 + 8 * case["K"]), "flops": 2 * n}
    if case["op"] == "quantize":
        n, sides = case["rows"] * case["cols"], 2 if case["both"] else 1
        scales = -(-case["rows"] // case["block_rows"]) * -(-case["cols"] // G) + (-(-case["cols"] // case["block_rows"]) * -(-case["rows"] // G) if case["both"] else 0)
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + sides * n + 4 * scales, "flops": 2 * n}
    M, N, K, kb = case["M"], case["N"], case["K"], -(-case["K"] // G)
    return {"bytes": M * K + N * K + 4 * kb * (M + -(-N // case["b_block_rows"])) + M * N * (2 if case["out"] == "bf16" else 4), "flops": 2 * M * N * K}


# -------------------------------------------------------------------------------------------------------------- exact
def _round8(y, fmt):
    """y (float64) rounded to the nearest value of the 8-bit type, ties to even, by its exponent and step."""
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    e = torch.frexp(y)[1].to(torch.float64) - 1
    step = torch.exp2(torch.clamp(e, min=low) - bits)
    return torch.clamp(torch.round(y / step) * step, -BIG[fmt], BIG[fmt])


def _exact_blocks(x, fmt, block_rows):
    rows, cols = x.shape
    amax = torch.nn.functional.pad(x.abs(), (0, -cols % G)).view(rows, -1, G).amax(dim=2)
    if block_rows > 1:
        amax = torch.nn.functional.pad(amax, (0, 0, 0, -rows % block_rows)).view(-1, block_rows, amax.shape[1]).amax(dim=1)
    amax = torch.clamp(amax, min=2.0 ** -100)
    return _round8(x * BIG[fmt] / _spread(amax, rows, cols, block_rows), fmt), amax / BIG[fmt]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        if case["rows"] * case["cols"] > 1 << 28:       # in blocks of rows that hold whole groups the wide tensors would be too large
            x, n = s["x"], 8192
            parts = [_exact_blocks(x[i:i + n].double(), case["fmt"], case["block_rows"]) for i in range(0, case["rows"], n)]
            out = {"q": torch.cat([q for q, _ in parts]), "scale": torch.cat([c for _, c in parts])}
            del parts
            if case["both"]:
                parts = [_exact_blocks(x[:, i:i + n].t().double(), case["fmt"], case["block_rows"]) for i in range(0, case["cols"], n)]
                out["qt"], out["qt_scale"] = torch.cat([q for q, _ in parts]), torch.cat([c for _, c in parts])
            return out
        q, scale = _exact_blocks(s["x"].double(), case["fmt"], case["block_rows"])
        out = {"q": q, "scale": scale}
        if case["both"]:
            out["qt"], out["qt_scale"] = _exact_blocks(s["x"].double().t(), case["fmt"], case["block_rows"])
        return out
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        c = torch.zeros((M, N), dtype=torch.float64, device=DEV)
        for k in range(0, K, 16 * G):                   # panels of whole groups, added up in 64 bits
            ke = min(K, k + 16 * G)
            a = s["a"][:, k:ke].double() * _spread(s["a_scale"].double()[:, k // G:], M, ke - k, 1)
            b = s["b"][:, k:ke].double() * _spread(s["b_scale"].double()[:, k // G:], N, ke - k, s["b_block_rows"])
            c += a @ b.t()
        return {"c": c}
    # sampling, row after row: the kept set as a threshold on the sorted probabilities
    K, logp, top = case["K"], [], []
    for t in range(case["T"]):
        row = s["logits"][t].double()
        tau = 1.0 if s["temperature"] is None else float(s["temperature"][t])
        k = 0 if s["top_k"] is None else int(s["top_k"][t])
        p = 1.0 if s["top_p"] is None else float(s["top_p"][t])
        m = 0.0 if s["min_p"] is None else float(s["min_p"][t])
        ids = torch.argsort(row, descending=True, stable=True)
        if tau == 0.0:
            tau, k = 1.0, 1
        prob = torch.softmax(row[ids[:k] if 0 < k < row.numel() else ids] / tau, dim=0)
        n = prob.numel()
        if p < 1.0:
            n = int((torch.cumsum(prob, 0) < p).sum()) + 1
        n = min(max(n, 1), prob.numel())
        if m > 0.0:
            n = min(n, int((prob >= m * prob[0]).sum()))
        kept = prob[:n] / prob[:n].sum()
        in_order = torch.sort(ids[:n]).values
        by_id = torch.zeros_like(row)
        by_id[ids[:n]] = kept
        c = torch.cumsum(by_id[in_order], 0)
        pick = in_order[min(int((c <= float(s["uniform"][t])).sum()), n - 1)]
        logp.append(torch.log(by_id[pick]))
        if K:
            top.append(by_id[ids[:K]])
    out = {"sampled_ids": None, "mu_logp": torch.stack(logp)}
    if K:
        out["mu_topk_ids"], out["mu_topk_p"] = None, torch.stack(top)
    return out
