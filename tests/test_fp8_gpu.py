"""8-bit quantisation with a scale per block of 128 and the matrix product of such matrices against float64 (needs a B200).

Tolerances.  Scales are one correctly rounded fp32 division: equal to the float64 quotient rounded to fp32.  8-bit values of bf16
inputs are equal to the exact ones: 7/8 x is exact, the quotient is correctly rounded to fp32, and a quotient of two 8-bit
mantissas that is not a tie is further from one than 2^-14, so rounding twice does no harm.  For fp32 inputs 7/8 x and the
quotient round by 2^-24 each: values may differ where the exact quotient is within 2^-23 (relative) of a tie.
Product: a block's terms are added in fp32 by the tensor cores (at most one unit in the last place, 2^-23, of the magnitudes
added so far for each of the 128 terms), the block sums once each, the scales round three times: (128 + blocks + 3) 2^-23 of the
sum of magnitudes, plus half a step of the output type."""
import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding
from oracle import rollout_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def _values(rows, cols, dtype, seed):
    """Blocks of unlike magnitude, zeros, a block of zeros, tiny and large values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-12, 12, (rows, 1), generator=g).float())
    x *= (torch.rand((rows, cols), generator=g) > 0.1)
    x[rows // 2] = 0.0
    x[:, : min(cols, 128)] *= 1e-3
    if rows > 3:
        x[3] *= 1e-35
        x[1] *= 2.0 ** 100
    return x.to(dtype)


def _host(q):
    return q.to(torch.float32).cpu().numpy().astype(np.float64)


def _check_quantized(q, scale, x, fmt, block_rows, exact):
    val, sc, y = R.quantize(x, fmt, block_rows)
    assert np.array_equal(scale.cpu().numpy(), sc.astype(np.float32))
    got = _host(q)
    bad = got != val
    if exact:
        assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], val[bad][:3], y[bad][:3])
    elif bad.any():
        # both neighbours of a quotient that is within 2^-23 of the middle between them
        assert np.all(np.abs(y[bad] - 0.5 * (got[bad] + val[bad])) <= 2.0 ** -23 * np.abs(y[bad]))


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 128), (128, 128), (129, 257), (61, 2048), (300, 1001), (1, 5000), (2000, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_matches_the_definition(rows, cols, dtype, fmt, block_rows):
    x = _values(rows, cols, dtype, seed=rows + cols)
    xd, xh = x.to(DEV), x.double().numpy()
    both = dppo.dppo_fp8_quantize(xd, F8[fmt], block_rows, transposed=True)
    one = dppo.dppo_fp8_quantize(xd, F8[fmt], block_rows)
    tr = dppo.dppo_fp8_quantize(xd, F8[fmt], block_rows, rowwise=False, transposed=True)
    torch.cuda.synchronize()
    assert all(int(o["status"].item()) == 0 for o in (both, one, tr))
    exact = dtype == torch.bfloat16
    _check_quantized(both["q"], both["scale"], xh, fmt, block_rows, exact)
    _check_quantized(both["qt"], both["qt_scale"], np.ascontiguousarray(xh.T), fmt, block_rows, exact)
    assert torch.equal(one["q"].float(), both["q"].float()) and torch.equal(one["scale"], both["scale"]) and one["qt"] is None
    assert torch.equal(tr["qt"].float(), both["qt"].float()) and torch.equal(tr["qt_scale"], both["qt_scale"]) and tr["q"] is None
    if block_rows == 128:
        assert torch.equal(both["qt"].float(), both["q"].float().t())


def test_every_tie_rounds_to_even():
    """x = amax t / B for every middle t between two neighbouring 8-bit values, and the values themselves, at several amax."""
    for fmt in ("e4m3", "e5m2"):
        vals = torch.arange(0, 0x7f if fmt == "e4m3" else 0x7c, dtype=torch.uint8).view(F8[fmt]).float()
        mids = torch.cat([0.5 * (vals[1:] + vals[:-1]), vals])
        for amax in (448.0, 7.0, 1.75, 0.875, 7 * 2.0 ** -30, 57344.0):
            x = mids * (amax / R.MAX8[fmt])
            n = -(-x.numel() // 120) * 120
            x = torch.nn.functional.pad(x, (0, n - x.numel())).view(-1, 120)
            x = torch.cat([x, torch.full((x.shape[0], 8), amax)], 1).contiguous()
            assert torch.equal(x * R.MAX8[fmt] / amax, torch.cat([x[:, :120] * R.MAX8[fmt] / amax, torch.full((x.shape[0], 8), R.MAX8[fmt])], 1))
            o = dppo.dppo_fp8_quantize(x.to(DEV), F8[fmt])
            _check_quantized(o["q"], o["scale"], x.double().numpy(), fmt, 1, exact=True)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_reads_and_writes_its_own_places_only(block_rows):
    rows, cols = 150, 333
    wide = torch.full((rows, cols + 11), float("nan"), dtype=torch.bfloat16)
    x = _values(rows, cols, torch.bfloat16, seed=2)
    for off in (0, 1, 5, 8):
        wide[:] = float("nan")
        wide[:, off:off + cols] = x
        w = wide.to(DEV)[:, off:off + cols]
        o = dppo.dppo_fp8_quantize(w, block_rows=block_rows, transposed=True)
        torch.cuda.synchronize()
        assert int(o["status"].item()) == 0
        _check_quantized(o["q"], o["scale"], x.double().numpy(), "e4m3", block_rows, True)
    # bytes behind the rows stay as they were, for pitches that allow wide stores and pitches that do not; scales in either order
    L = binding.lib()
    for pitch, pitch_t in ((cols + 3, rows + 10), (336, 152), (cols, rows)):
        q = torch.full((rows + 1, pitch), 0x55, dtype=torch.uint8, device=DEV)
        qt = torch.full((cols + 1, pitch_t), 0x55, dtype=torch.uint8, device=DEV)
        nr, nk, nrt, nkt = -(-rows // block_rows), 3, -(-cols // block_rows), 2
        sc = torch.full((nr + 1, nk + 2), -1.0, device=DEV)
        sct = torch.full((nrt + 1, nkt + 2), -1.0, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        xd = x.to(DEV)
        rc = L.dppo_fp8_quantize(xd.data_ptr(), rows, cols, cols, binding.BF16, binding.E4M3, block_rows, q.data_ptr(), pitch, sc.data_ptr(), nk + 2, 1,
                                 qt.data_ptr(), pitch_t, sct.data_ptr(), nkt + 2, 1, st.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == 0 and int(st.item()) == 0
        assert bool((q[:rows, cols:] == 0x55).all()) and bool((q[rows] == 0x55).all()) and bool((qt[:cols, rows:] == 0x55).all()) and bool((qt[cols] == 0x55).all())
        assert bool((sc[:nr, nk:] == -1).all()) and bool((sc[nr] == -1).all()) and bool((sct[:nrt, nkt:] == -1).all()) and bool((sct[nrt] == -1).all())
        assert torch.equal(q[:rows, :cols], o["q"].contiguous().view(torch.uint8)) and torch.equal(qt[:cols, :rows], o["qt"].contiguous().view(torch.uint8))
        assert torch.equal(sc[:nr, :nk], o["scale"]) and torch.equal(sct[:nrt, :nkt], o["qt_scale"])


@pytest.mark.parametrize("value", [float("nan"), -float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_a_block_with_a_non_finite_value_is_nan(value, block_rows):
    x = _values(200, 300, torch.float32, seed=1)
    x[140, 200] = value
    o = dppo.dppo_fp8_quantize(x.to(DEV), block_rows=block_rows, transposed=True)
    torch.cuda.synchronize()
    assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW
    hit = torch.zeros(200, 300, dtype=torch.bool)
    hit[140 if block_rows == 1 else slice(128, 200), 128:256] = True
    assert torch.equal(o["q"].float().isnan().cpu(), hit)
    hit_t = torch.zeros(300, 200, dtype=torch.bool)
    hit_t[200 if block_rows == 1 else slice(128, 256), 128:200] = True
    assert torch.equal(o["qt"].float().isnan().cpu(), hit_t)
    assert int(o["scale"].isnan().sum()) == 1 and int(o["qt_scale"].isnan().sum()) == 1


def _operand(rows, K, fmt, block_rows, seed, spread_bits=6):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, K), generator=g) * torch.exp2(spread_bits * torch.rand((rows, 1), generator=g))
    o = dppo.dppo_fp8_quantize(x.to(DEV), F8[fmt], block_rows)
    return o["q"], o["scale"]


def _check_product(C, A, sa, abr, B, sb, bbr):
    ref, mag = R.product(_host(A), sa.double().cpu().numpy(), abr, _host(B), sb.double().cpu().numpy(), bbr)
    got = C.double().cpu().numpy()
    kb = -(-A.shape[1] // 128)
    tol = (128 + kb + 3) * 2.0 ** -23 * mag + (2.0 ** -8 * np.abs(ref) if C.dtype == torch.bfloat16 else 2.0 ** -24 * np.abs(ref))
    worst = np.abs(got - ref) - tol
    assert worst.max() <= 0, (np.argwhere(worst > 0)[:4], np.abs(got - ref).max())


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 256, 128), (128, 256, 128), (128, 256, 256), (127, 255, 130), (129, 257, 384), (61, 1000, 2048), (300, 520, 777),
                                   (33, 128, 5000), (512, 512, 1024), (1000, 3, 640), (3, 4096, 100)])
@pytest.mark.parametrize("a_br,b_br", [(1, 128), (1, 1), (128, 128), (128, 1)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_matches_float64(M, N, K, a_br, b_br, out):
    A, sa = _operand(M, K, "e4m3", a_br, seed=M + K)
    B, sb = _operand(N, K, "e4m3", b_br, seed=N + K + 1)
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, a_br, b_br, out)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and C.dtype == out
    _check_product(C, A, sa, a_br, B, sb, b_br)
    again, _ = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, a_br, b_br, out)
    assert torch.equal(again, C)


@pytest.mark.parametrize("fa,fb", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
def test_product_of_either_format(fa, fb):
    A, sa = _operand(200, 700, fa, 1, seed=5)
    B, sb = _operand(300, 700, fb, 128, seed=6)
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    _check_product(C, A, sa, 1, B, sb, 128)


def test_product_with_more_tiles_than_sms_and_strided_everything():
    """Several tiles per CTA; operands and output inside wider buffers; scales with the other stride order."""
    M, N, K = 1300, 7000, 520
    A, sa = _operand(M, K, "e4m3", 1, seed=1)
    B, sb = _operand(N, K, "e4m3", 128, seed=2)
    wa = torch.full((M, K + 40), 0x7f, dtype=torch.uint8, device=DEV)          # NaN behind every row
    wa[:, :K] = A.contiguous().view(torch.uint8)
    wb = torch.full((N, K + 24), 0x7f, dtype=torch.uint8, device=DEV)
    wb[:, :K] = B.contiguous().view(torch.uint8)
    A2, B2 = wa.view(torch.float8_e4m3fn)[:, :K], wb.view(torch.float8_e4m3fn)[:, :K]
    for dt, extra in ((torch.float32, 0), (torch.float32, 4), (torch.float32, 5), (torch.bfloat16, 8), (torch.bfloat16, 1)):
        wc = torch.full((M + 1, N + extra), -3.0, dtype=dt, device=DEV)
        C, status = dppo.dppo_gemm_tn_fp8(A2, sa.contiguous(), B2, sb.contiguous(), C=wc[:M, :N])
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        _check_product(C, A, sa, 1, B, sb, 128)
        assert bool((wc[:M, N:] == -3).all()) and bool((wc[M] == -3).all())


@pytest.mark.parametrize("M,N,K", [(1, 256, 20000), (64, 1024, 8192), (70, 300, 4100), (200, 100, 9000), (500, 1000, 1500), (61, 30000, 300), (129, 37000, 256)])
@pytest.mark.parametrize("b_br", [1, 128])
def test_product_of_few_tiles_and_of_ragged_rounds(M, N, K, b_br):
    """Clusters of two to eight CTAs that share a tile along K, and tiles narrower than 256 columns (their columns cross the 128-blocks
    of the scales)."""
    A, sa = _operand(M, K, "e4m3", 1, seed=M)
    B, sb = _operand(N, K, "e4m3", b_br, seed=N)
    for out in (torch.float32, torch.bfloat16):
        C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, 1, b_br, out)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        _check_product(C, A, sa, 1, B, sb, b_br)
        assert torch.equal(dppo.dppo_gemm_tn_fp8(A, sa, B, sb, 1, b_br, out)[0], C)
    wide = torch.full((M + 1, N + 3), -3.0, device=DEV)
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, 1, b_br, C=wide[:M, :N])
    _check_product(C, A, sa, 1, B, sb, b_br)
    assert bool((wide[:, N:] == -3).all()) and bool((wide[M] == -3).all())


def test_product_over_an_empty_sum_and_of_nothing():
    sa, sb = torch.empty((5, 0), device=DEV), torch.empty((1, 0), device=DEV)
    A, B = (torch.empty((n, 0), dtype=torch.float8_e4m3fn, device=DEV) for n in (5, 7))
    C = torch.full((5, 9), -2.0, device=DEV)
    out, _ = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, C=C[:, :7])
    torch.cuda.synchronize()
    assert bool((out == 0).all()) and bool((C[:, 7:] == -2).all())
    A = torch.empty((0, 128), dtype=torch.float8_e4m3fn, device=DEV)
    out, _ = dppo.dppo_gemm_tn_fp8(A, torch.empty((0, 1), device=DEV), *_operand(7, 128, "e4m3", 128, 1))
    assert out.shape == (0, 7)


def test_nan_blocks_reach_only_their_rows():
    A, sa = _operand(140, 300, "e4m3", 1, seed=1)
    B, sb = _operand(260, 300, "e4m3", 1, seed=2)
    sa = sa.clone()
    sa[131, 1] = float("nan")
    C, _ = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, b_block_rows=1)
    assert bool(C[131].isnan().all()) and int(C.isnan().sum()) == 260


@pytest.mark.parametrize("M,K", [(300, 500), (100, 5000)])
def test_product_gives_up_and_the_next_call_is_fine(M, K):
    """A CTA per tile, and a cluster that shares its tiles (all of it meets at its barriers and leaves)."""
    A, sa = _operand(M, K, "e4m3", 1, seed=3)
    B, sb = _operand(520, K, "e4m3", 128, seed=4)
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, wait_limit_us=20000, test_inject=binding.INJECT_NO_COPIES)
    torch.cuda.synchronize()
    assert int(status.item()) & binding.STATUS_WAIT_LIMIT
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, wait_limit_us=20000)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    _check_product(C, A, sa, 1, B, sb, 128)


def test_graph_replay_and_concurrent_products():
    x = torch.randn((200, 640), generator=torch.Generator().manual_seed(1)).to(DEV)
    w = dppo.dppo_fp8_quantize(torch.randn((400, 640), generator=torch.Generator().manual_seed(2)).to(DEV), block_rows=128)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step():
        q = dppo.dppo_fp8_quantize(x, status=st)
        return dppo.dppo_gemm_tn_fp8(q["q"], q["scale"], w["q"], w["scale"], status=st)[0]
    ref = step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    x.neg_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, -ref) and int(st.item()) == 0
    x.neg_()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += [step() for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)


def test_lm_head_step_in_8_bits_end_to_end():
    """As they are used: hidden states -> 8-bit logits -> sampled tokens with their record -> DPPO loss -> 8-bit gradients of the hidden
    states and of the LM head.  The gradients are held to the formulas on the quantised operands, and to central differences of
    the loss along a random direction (of the unquantised function: 8-bit operands move it by 2^-4 relative per entry)."""
    g = torch.Generator().manual_seed(3)
    T, d, V = 96, 256, 1000
    H, W = torch.randn((T, d), generator=g).to(torch.bfloat16).to(DEV), (0.08 * torch.randn((V, d), generator=g)).to(torch.bfloat16).to(DEV)
    u = torch.rand(T, generator=g, dtype=torch.float64).to(DEV)
    adv = torch.where(torch.rand(T, generator=g) < 0.5, -1.0, 1.0).to(DEV)
    qh = dppo.dppo_fp8_quantize(H)
    qw = dppo.dppo_fp8_quantize(W, block_rows=128, transposed=True)
    z8, _ = dppo.dppo_gemm_tn_fp8(qh["q"], qh["scale"], qw["q"], qw["scale"], out_dtype=torch.bfloat16)
    o = dppo.dppo_sample(z8, u, K=20)
    Hq = _host(qh["q"]) * R.spread(qh["scale"].double().cpu().numpy(), T, d, 1)
    Wq = _host(qw["q"]) * R.spread(qw["scale"].double().cpu().numpy(), V, d, 128)
    # the trainer's logits: the bf16 weights; the update
    z, _ = dppo.dppo_gemm_tn_bf16(H, W)
    r = dppo.dppo_loss_fwd_bwd(z, o["sampled_ids"], o["mu_logp"], adv, None, dppo.TOPK_KL, 20, 1e9, o["mu_topk_ids"], o["mu_topk_p"])
    dq = dppo.dppo_fp8_quantize(r["dlogits"], torch.float8_e5m2, transposed=True)
    dH, _ = dppo.dppo_gemm_tn_fp8(dq["q"], dq["scale"], qw["qt"], qw["qt_scale"])                         # dlogits . W
    ht = dppo.dppo_fp8_quantize(H, rowwise=False, transposed=True)
    dW, _ = dppo.dppo_gemm_tn_fp8(dq["qt"], dq["qt_scale"], ht["qt"], ht["qt_scale"], b_block_rows=1)     # dlogits^T . hidden
    torch.cuda.synchronize()
    assert all(int(x["status"].item()) == 0 for x in (qh, qw, o, r, dq, ht))
    _check_product(z8, qh["q"], qh["scale"], 1, qw["q"], qw["scale"], 128)
    _check_product(dH, dq["q"], dq["scale"], 1, qw["qt"], qw["qt_scale"], 128)
    _check_product(dW, dq["qt"], dq["qt_scale"], 1, ht["qt"], ht["qt_scale"], 1)
    assert np.abs(z8.double().cpu().numpy() - Hq @ Wq.T).max() <= 2.0 ** -8 * np.abs(Hq @ Wq.T).max() + 1e-3
    # loss(H, W) = -mean(exp(log pi(a) - log mu(a)) A) in float64; its slope along a direction by central differences
    Hd, Wd = H.double().cpu().numpy(), W.double().cpu().numpy()
    a, lmu, A = o["sampled_ids"].cpu().numpy(), o["mu_logp"].double().cpu().numpy(), adv.double().cpu().numpy()

    def loss(h, w):
        zz = h @ w.T
        m = zz.max(1)
        lp = zz[np.arange(T), a] - m - np.log(np.exp(zz - m[:, None]).sum(1))
        return -(np.exp(lp - lmu) * A).mean()
    rng = np.random.default_rng(0)
    for got, base, which in ((dH, Hd, 0), (dW, Wd, 1)):
        G = got.double().cpu().numpy()
        dl = r["dlogits"].double().cpu().numpy()
        if which == 0:
            other, ref = Wd, dl @ Wd
            mag = np.abs(dl) @ np.abs(Wd)
        else:
            other, ref = Hd, dl.T @ Hd
            mag = np.abs(dl).T @ np.abs(Hd)
        # operands rounded by at most half a step: e5m2 2^-3, e4m3 2^-4 relative (plus what falls below the smallest step of a block,
        # 2^-17 resp. 2^-10 of its amax); bound on every entry of the gradient
        floor = 2.0 ** -10 * (np.abs(dl).max() * np.abs(other).sum(0).max() + np.abs(other).max() * np.abs(dl).sum(1 if which == 0 else 0).max())
        assert np.all(np.abs(G - ref) <= (2.0 ** -3 + 2.0 ** -4 + 2.0 ** -7) * mag + floor)
        # the formula's own slope against differences (step 1e-5: 64-bit, error of order 1e-9), then the 8-bit one by the same bound
        D = rng.standard_normal(base.shape)
        eps = 1e-5
        args = lambda s: (base + s * eps * D, other) if which == 0 else (other, base + s * eps * D)  # noqa: E731
        slope = (loss(*args(1)) - loss(*args(-1))) / (2 * eps)
        # dlogits was formed from fp32 logits of bf16 operands: z is off by at most (256 + 1) 2^-24 of its magnitudes, so is the slope
        assert abs((ref * D).sum() - slope) <= 1e-4 * (np.abs(ref) * np.abs(D)).sum()


@pytest.mark.parametrize("M,N,K", [(200, 300, 151936), (1500, 5000, 4100), (130, 40000, 1000)])
@pytest.mark.parametrize("a_br,b_br", [(1, 128), (1, 1), (128, 128), (128, 1)])
def test_every_block_meets_its_own_scales(M, N, K, a_br, b_br):
    """Elements of +1 and -1 and scales of 1/2, 1 and 2 that change from block to block: every sum on the way is a multiple of 1/4 below
    2^20, exact in fp32 in any order, so one scale of another block would show.  Tiles shared along K, several tiles per CTA, many K
    blocks in a row."""
    g = torch.Generator(device=DEV).manual_seed(M)
    kb = -(-K // 128)

    def operand(rows, br):
        q = (torch.randint(0, 2, (rows, -(-K // 16) * 16), generator=g, device=DEV) * 2 - 1).float().to(torch.float8_e4m3fn)[:, :K]
        return q, torch.exp2(torch.randint(-1, 2, (-(-rows // br), kb), generator=g, device=DEV).float())

    def exact(q, scale, br):
        return q.double() * scale.double().repeat_interleave(br, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :K]
    A, sa = operand(M, a_br)
    B, sb = operand(N, b_br)
    assert 4 * K < 2 ** 20
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, a_br, b_br)
    assert int(status.item()) == 0
    assert torch.equal(C.double(), exact(A, sa, a_br) @ exact(B, sb, b_br).t())


@pytest.mark.parametrize("M,N,K", [(40, 1, 256), (40, 3, 256), (129, 77, 130), (300, 78, 777), (70, 79, 128), (33, 130, 256), (257, 255, 384), (40, 257, 256), (1000, 1001, 640),
                                   (200, 20001, 300), (64, 37, 8192)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b_br", [1, 128])
def test_product_into_columns_of_a_wider_matrix(M, N, K, out, b_br):
    """C's rows start on 16-byte boundaries and end anywhere: what stands behind their last column stays as it was."""
    A, sa = _operand(M, K, "e4m3", 1, seed=M)
    B, sb = _operand(N, K, "e4m3", b_br, seed=N)
    whole, _ = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, 1, b_br, torch.float32)
    piece = 16 // torch.empty((), dtype=out).element_size()
    wide = torch.full((M + 1, -(-N // piece) * piece + piece), -3.0, dtype=out, device=DEV)
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, 1, b_br, C=wide[:M, :N])
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(C, whole.to(out))
    assert bool((wide[:M, N:] == -3).all()) and bool((wide[M] == -3).all())


def test_8_bit_gradients_against_differences():
    """dHidden and dW of the 8-bit step against central differences of the loss itself, along a direction made of the entries with little
    cancellation, so that the operands' rounding leaves less than the slope: a gradient of zero, or of the other sign, fails.

    An element rounds by at most 2^-3 (e5m2) or 2^-4 (e4m3) of itself, or, below the smallest normal value, by half a step of its block:
    2^-17 / 57344 < 2^-32 or 2^-10 / 448 < 2^-18 of the block's largest.  The product adds (128 + blocks + 3) 2^-23 of the magnitudes.
    dlogits come from fp32 logits, off by at most (256 + 1) 2^-24 of their magnitudes: 1e-4 of the slope's terms with room to spare."""
    g = torch.Generator().manual_seed(3)
    T, d, V = 96, 256, 1000
    H, W = torch.randn((T, d), generator=g).to(torch.bfloat16).to(DEV), (0.08 * torch.randn((V, d), generator=g)).to(torch.bfloat16).to(DEV)
    u = torch.rand(T, generator=g, dtype=torch.float64).to(DEV)
    adv = torch.where(torch.rand(T, generator=g) < 0.5, -1.0, 1.0).to(DEV)
    qw = dppo.dppo_fp8_quantize(W, block_rows=128, transposed=True)
    z, _ = dppo.dppo_gemm_tn_bf16(H, W)
    o = dppo.dppo_sample(z, u, K=20)
    r = dppo.dppo_loss_fwd_bwd(z, o["sampled_ids"], o["mu_logp"], adv, None, dppo.TOPK_KL, 20, 1e9, o["mu_topk_ids"], o["mu_topk_p"])
    dq = dppo.dppo_fp8_quantize(r["dlogits"], torch.float8_e5m2, transposed=True)
    dH, _ = dppo.dppo_gemm_tn_fp8(dq["q"], dq["scale"], qw["qt"], qw["qt_scale"])
    ht = dppo.dppo_fp8_quantize(H, rowwise=False, transposed=True)
    dW, _ = dppo.dppo_gemm_tn_fp8(dq["qt"], dq["qt_scale"], ht["qt"], ht["qt_scale"], b_block_rows=1)
    torch.cuda.synchronize()
    Hd, Wd, dl = H.double().cpu().numpy(), W.double().cpu().numpy(), r["dlogits"].double().cpu().numpy()
    a, lmu, A = o["sampled_ids"].cpu().numpy(), o["mu_logp"].double().cpu().numpy(), adv.double().cpu().numpy()
    _check_slopes(dH.double().cpu().numpy(), dW.double().cpu().numpy(), Hd, Wd, dl, a, lmu, A)


def _check_slopes(dH, dW, Hd, Wd, dl, a, lmu, A):
    T = Hd.shape[0]

    def loss(h, w):
        zz = h @ w.T
        m = zz.max(1)
        lp = zz[np.arange(T), a] - m - np.log(np.exp(zz - m[:, None]).sum(1))
        return -(np.exp(lp - lmu) * A).mean()
    for G, left, other, at in ((dH, dl, Wd, lambda s: (Hd + s, Wd)), (dW, dl.T, Hd, lambda s: (Hd, Wd + s))):
        ref, mag = left @ other, np.abs(left) @ np.abs(other)
        blocks = -(-left.shape[1] // 128)
        bound = (2.0 ** -3 + 2.0 ** -4 + 2.0 ** -7 + (128 + blocks + 3) * 2.0 ** -22) * mag
        bound += 2.0 ** -17 * np.abs(other).max() * np.abs(left).sum(1, keepdims=True) + 2.0 ** -31 * np.abs(left).max() * np.abs(other).sum(0)
        D = np.where(bound < 0.5 * np.abs(ref), np.sign(ref), 0.0)
        assert (D != 0).sum() >= 200
        eps = 1e-5
        slope = (loss(*at(eps * D)) - loss(*at(-eps * D))) / (2 * eps)
        tol = (bound * np.abs(D)).sum() + 1e-4 * (mag * np.abs(D)).sum()
        assert tol < 0.6 * slope
        assert abs((G * D).sum() - slope) <= tol


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_more_than_2_31_elements(block_rows):
    """[16389, 151936]: blocks behind element 2^31, as stored and transposed, are what a call on their rows alone gives."""
    rows, cols, first = 16389, 151936, 16256
    g = torch.Generator(device=DEV).manual_seed(7)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    for i in range(0, rows, 2048):
        x[i:i + 2048] = torch.randn((min(2048, rows - i), cols), generator=g, device=DEV)
    assert first * cols > 2 ** 31 and first % 128 == 0
    o = dppo.dppo_fp8_quantize(x, torch.float8_e5m2, block_rows, transposed=True)
    one = dppo.dppo_fp8_quantize(x, torch.float8_e5m2, block_rows)
    t = dppo.dppo_fp8_quantize(x[first:], torch.float8_e5m2, block_rows, transposed=True)
    bits = lambda q: q.contiguous().view(torch.uint8)  # noqa: E731
    assert int(o["status"].item()) == 0 and torch.equal(bits(o["q"][first:]), bits(t["q"])) and torch.equal(o["scale"][first // block_rows:], t["scale"])
    assert torch.equal(bits(o["qt"][:, first:]), bits(t["qt"])) and torch.equal(o["qt_scale"][:, first // 128:], t["qt_scale"])
    assert torch.equal(bits(one["q"][first:]), bits(t["q"])) and torch.equal(one["scale"], o["scale"])


@pytest.mark.parametrize("M,N,K,out", [(16389, 151936, 256, torch.bfloat16), (43500, 50257, 128, torch.bfloat16), (43500, 50257, 128, torch.float32), (151936, 128, 16384, torch.float32)])
def test_product_beyond_2_31_elements(M, N, K, out):
    """Outputs by bulk tensor stores and by plain ones, and an operand, of more than 2^31 elements: the last rows, with elements of +1 and
    -1 whose sums are exact in fp32."""
    g = torch.Generator(device=DEV).manual_seed(8)

    def operand(rows):
        return ((torch.randint(0, 256, (rows, K), generator=g, dtype=torch.uint8, device=DEV) & 0x80) | 0x38).view(torch.float8_e4m3fn)
    A, B = operand(M), operand(N)
    sa = torch.exp2(torch.randint(-1, 2, (M, K // 128), generator=g, device=DEV).float())
    sb = torch.exp2(torch.randint(-1, 2, (-(-N // 128), K // 128), generator=g, device=DEV).float())
    C, status = dppo.dppo_gemm_tn_fp8(A, sa, B, sb, out_dtype=out)
    assert int(status.item()) == 0 and max(M * N, M * K) > 2 ** 31
    for first in (0, M - 300):
        a = A[first:first + 300].double() * sa[first:first + 300].double().repeat_interleave(128, 1)
        for n in range(0, N, 16384):
            b = B[n:n + 16384].double() * sb.double().repeat_interleave(128, 0)[n:min(N, n + 16384)].repeat_interleave(128, 1)
            assert torch.equal(C[first:first + 300, n:n + 16384], (a @ b.t()).float().to(out))
