"""4-bit weights with a scale per group and their product with a few rows against float64 (needs a B200).

Tolerances.  Scales and codes are equal to the exact ones: the scale is rounded once, a code is decided by the sign of |x| - (k + 1/2) scale, which
one fma gives exactly.  Values are code times scale (12 bits, exact in fp32) rounded once to x's type.  Product: the terms x (code - 8) are exact
(12 bits); they are added up in fp32, in any order, a rounding (2^-24, or 2^-23 where a tensor core truncates) for each of at most K
additions of the group sums, the scaling and the sum over the groups: (K + 3) 2^-23 of the sum of the terms' magnitudes, and half a step of
the output type (2^-24, 2^-8)."""
import threading

import numpy as np
import pytest
import torch

import paper_2602_04879_b200 as dppo
from paper_2602_04879_b200 import binding
from oracle import reference_oracle as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def weights(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-10, 10, (rows, 1), generator=g).float())
    x *= torch.rand((rows, cols), generator=g) > 0.1
    x[rows // 2] = 0.0
    if rows > 4:
        x[1] *= 2.0 ** 100
        x[3] *= 2.0 ** -120
    return x.to(dtype)


def check_quantized(o, x, group):
    code, scale, val = R.int4_quantize(x.double().numpy(), group)
    assert np.array_equal(o["scale"].double().cpu().numpy(), scale)
    assert np.array_equal(R.unpack(o["q"].cpu().numpy(), x.shape[1]), code)
    if x.shape[1] % 2:
        assert (o["q"][:, -1] >> 4 == 0).all()
    if o["values"] is not None:
        assert torch.equal(o["values"].cpu(), torch.from_numpy(val.astype(np.float32)).to(x.dtype))


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 32), (3, 31), (7, 129), (61, 2048), (300, 1001), (1, 5000), (2000, 3), (33, 777)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize_matches_the_definition(rows, cols, dtype, group):
    x = weights(rows, cols, dtype, seed=rows + cols)
    o = dppo.dppo_int4_quantize(x.to(DEV), group, values=True)
    assert int(o["status"].item()) == 0
    check_quantized(o, x, group)
    assert torch.equal(dppo.dppo_int4_quantize(x.to(DEV), group)["q"], o["q"])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ties_go_to_even_and_neighbours_do_not(dtype):
    """x = (k + 1/2) scale exactly, and the numbers of the type on either side of it."""
    rows = []
    for s in (1.0, 1.5, 0.8203125, 2.0 ** -20 * 1.1640625):
        mids = torch.tensor([(k + 0.5) * s for k in range(7)], dtype=torch.float64)
        x = mids.to(dtype)
        both = torch.cat([x, torch.nextafter(x, x * 0), torch.nextafter(x, x * 2)])
        row = torch.zeros(64, dtype=dtype)
        row[:21], row[21:42] = both, -both
        row[63] = 7 * s
        rows.append(row)
    x = torch.stack(rows)
    o = dppo.dppo_int4_quantize(x.to(DEV), 64, values=True)
    assert np.array_equal(o["scale"].float().cpu().numpy()[:, 0], np.array([1.0, 1.5, 0.8203125, 2.0 ** -20 * 1.1640625], np.float32))
    check_quantized(o, x, 64)


def test_many_fp32_groups_round_their_scale_once():
    g = torch.Generator().manual_seed(3)
    x = torch.randn((40000, 32), generator=g)
    # amax / 7 next to the middle of two bf16 numbers, where a first rounding to fp32 would land on it
    m = (torch.randint(256, 512, (40000,), generator=g).double() + 0.5) / 256
    x[:, 0] = (7 * m).float() * 4
    x[::2, 0] = torch.nextafter(x[::2, 0], torch.zeros(20000))
    check_quantized(dppo.dppo_int4_quantize(x.to(DEV), 32, values=True), x, 32)


def test_groups_that_are_not_finite():
    x = weights(6, 300, BF, seed=9)
    x[0, 5], x[2, 200], x[4, 299] = float("nan"), float("inf"), float("-inf")
    o = dppo.dppo_int4_quantize(x.to(DEV), 128, values=True)
    assert int(o["status"].item()) == binding.STATUS_NONFINITE_ROW
    bad = torch.zeros((6, 3), dtype=torch.bool)
    bad[0, 0] = bad[2, 1] = bad[4, 2] = True
    assert torch.equal(torch.isnan(o["scale"].cpu()), bad)
    wide = bad.repeat_interleave(128, 1)[:, :300]
    assert torch.equal(torch.isnan(o["values"].cpu()), wide)
    clean = torch.where(wide, torch.ones_like(x), x)
    ref = dppo.dppo_int4_quantize(clean.to(DEV), 128, values=True)
    assert torch.equal(o["values"].cpu()[~wide], ref["values"].cpu()[~wide])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantize_reads_and_writes_its_own_places_only(dtype):
    """Strides and offsets off the fast path's boundaries, through the C entry point; values over x itself."""
    rows, cols, group = 9, 203, 32
    x = weights(rows, cols, dtype, seed=21)
    want = dppo.dppo_int4_quantize(x.to(DEV), group, values=True)
    for off, ldx, ldq, lds, ldv in ((0, 208, 104, 8, 208), (1, 205, 103, 7, 211), (8, 216, 112, 9, 204)):
        xb = torch.full((off + rows * ldx,), float("nan"), dtype=dtype, device=DEV)
        torch.as_strided(xb, (rows, cols), (ldx, 1), off).copy_(x)
        q = torch.full((off + rows * ldq + 16,), 0xAB, dtype=torch.uint8, device=DEV)
        s = torch.full((off + rows * lds,), 3.0, dtype=BF, device=DEV)
        v = torch.full((off + rows * ldv,), 3.0, dtype=dtype, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        es = x.element_size()

        def call(values, ldvalues):
            return binding.lib().dppo_int4_quantize(xb.data_ptr() + off * es, rows, cols, ldx, binding._dtype_code(x), group, q.data_ptr() + off, ldq,
                                                    s.data_ptr() + 2 * off, lds, values, ldvalues, st.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert call(v.data_ptr() + off * es, ldv) == 0
        for buf, w, ld in ((q, want["q"], ldq), (s, want["scale"], lds), (v, want["values"], ldv)):
            inside = torch.zeros_like(buf, dtype=torch.bool)
            torch.as_strided(inside, tuple(w.shape), (ld, 1), off).fill_(True)
            assert torch.equal(torch.as_strided(buf, tuple(w.shape), (ld, 1), off), w)
            assert (buf[~inside] == (0xAB if buf is q else 3.0)).all()
        assert call(xb.data_ptr() + off * es, ldx) == 0
        assert torch.equal(torch.as_strided(xb, (rows, cols), (ldx, 1), off), want["values"])
        assert int(st.item()) == 0


# ---------------------------------------------------------------------------------------------------------- product
def product_case(M, N, K, group, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 16, (N, K), generator=g, dtype=torch.uint8)
    scale = (0.02 * torch.exp(torch.randn((N, -(-K // group)), generator=g))).to(BF)
    x = (torch.randn((M, K), generator=g) * torch.exp2(torch.randint(-4, 4, (M, 1), generator=g).float())).to(BF)
    return x, codes, scale


def packed(codes, lead=0, pitch=None):
    """Packed codes on the device: rows on 16-byte boundaries, or `pitch` bytes apart from `lead` bytes on; the half byte behind an odd row's
    end, and the bytes behind it, hold rubbish."""
    q = R.pack(codes.numpy())
    if codes.shape[1] % 2:
        q[:, -1] |= 0xE0
    n, b = q.shape
    pitch = pitch or -(-b // 16) * 16
    buf = torch.full((lead + n * pitch + 16,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.as_strided(buf, (n, b), (pitch, 1), lead)
    out.copy_(torch.from_numpy(q))
    return out


def check_product(y, x, codes, scale, group, out):
    want, mag = R.int4_product(x.double().numpy(), codes.numpy(), scale.double().numpy(), group)
    got = y.double().cpu().numpy()
    tol = (x.shape[1] + 3) * 2.0 ** -23 * mag + {F32: 2.0 ** -24, BF: 2.0 ** -8}[out] * np.abs(want)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 32), (1, 100, 2048), (2, 129, 777), (7, 1000, 128), (8, 333, 1001), (9, 64, 4096), (16, 257, 640), (17, 300, 512),
                                   (33, 130, 96), (61, 1111, 2048), (64, 128, 160), (65, 40, 300), (130, 77, 256), (1, 70000, 64), (3, 5, 20000)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_product(M, N, K, group):
    x, codes, scale = product_case(M, N, K, group, seed=M + N + K)
    q = packed(codes)
    for out in (F32, BF):
        y, st = dppo.dppo_matvec_int4(x.to(DEV), q, scale.to(DEV), group, out_dtype=out)
        assert int(st.item()) == 0
        check_product(y, x, codes, scale, group, out)


@pytest.mark.parametrize("M,K,group", [(64, 1024, 32), (61, 1024, 64), (33, 4096, 128), (16, 9000, 32), (7, 700, 128)])
def test_product_of_many_tiles(M, K, group):
    """Tens of tiles to an SM, several blocks of rows of x, x in parts and in pairs of SMs: a sample of the columns."""
    N = 40000
    x, codes, scale = product_case(M, N, K, group, seed=M + K)
    q, s, xd = packed(codes), scale.to(DEV), x.to(DEV)
    cols = torch.arange(0, N, 397)
    a, st = dppo.dppo_matvec_int4(xd, q, s, group)
    assert int(st.item()) == 0
    check_product(a[:, cols.to(DEV)], x, codes[cols], scale[cols], group, F32)
    for _ in range(3):
        assert torch.equal(dppo.dppo_matvec_int4(xd, q, s, group)[0], a)


@pytest.mark.parametrize("M,K,group,N", [(1, 9000, 32, 40000), (3, 9000, 32, 40000), (4, 4096, 32, 40000), (1, 16000, 64, 20000),
                                         (3, 33000, 32, 9000), (1, 70000, 128, 700), (20, 33000, 64, 5000)])
def test_product_of_few_rows_and_long_ones_repeats(M, K, group, N):
    """Rows of the weights that come and go while the products before them are still under way; rows of x too long for shared memory."""
    x, codes, scale = product_case(M, N, K, group, seed=M + K)
    q, s, xd = packed(codes), scale.to(DEV), x.to(DEV)
    cols = torch.arange(0, N, max(1, N // 40))
    a, st = dppo.dppo_matvec_int4(xd, q, s, group)
    assert int(st.item()) == 0
    check_product(a[:, cols.to(DEV)], x, codes[cols], scale[cols], group, F32)
    for _ in range(25):
        assert torch.equal(dppo.dppo_matvec_int4(xd, q, s, group)[0], a)


def test_product_in_any_layout():
    """Row strides and offsets of every operand; what lies beside y stays."""
    M, N, K, group = 5, 70, 333, 64
    x, codes, scale = product_case(M, N, K, group, seed=5)
    for lead, pitch, xo, ldx, so, lds, yo, ldy in ((0, 176, 0, 336, 0, 8, 0, 72), (3, 171, 1, 335, 1, 7, 1, 71), (16, 192, 8, 344, 8, 16, 4, 80)):
        q = packed(codes, lead, pitch)
        xb = torch.full((xo + M * ldx,), float("nan"), dtype=BF, device=DEV)
        xv = torch.as_strided(xb, (M, K), (ldx, 1), xo).copy_(x)
        sb = torch.full((so + N * lds,), float("nan"), dtype=BF, device=DEV)
        sv = torch.as_strided(sb, tuple(scale.shape), (lds, 1), so).copy_(scale)
        for out in (F32, BF):
            yb = torch.full((yo + M * ldy,), 7.0, dtype=out, device=DEV)
            yv = torch.as_strided(yb, (M, N), (ldy, 1), yo)
            dppo.dppo_matvec_int4(xv, q, sv, group, y=yv)
            check_product(yv, x, codes, scale, group, out)
            inside = torch.zeros_like(yb, dtype=torch.bool)
            torch.as_strided(inside, (M, N), (ldy, 1), yo).fill_(True)
            assert (yb[~inside] == 7.0).all()


@pytest.mark.parametrize("M,group,K", [(3, 32, 1000), (1, 64, 1500), (4, 32, 2048), (2, 64, 255), (20, 32, 700)])
def test_product_with_scales_in_padded_rows(M, group, K):
    """Rows of scales on the boundaries at which a chunk's are fetched together, with a last chunk that is not whole, and off them; what lies
    between the rows is not used."""
    N, groups = 300, -(-K // group)
    x, codes, scale = product_case(M, N, K, group, seed=K)
    q, xd = packed(codes), x.to(DEV)
    up = -(-groups // 8) * 8
    for so, lds in ((0, up), (0, up + 8), (8, up + 16), (0, up + 4), (4, up + 4), (1, up), (0, groups + 1), (2, up + 2)):
        sb = torch.full((so + N * lds,), float("nan"), dtype=BF, device=DEV)
        sv = torch.as_strided(sb, (N, groups), (lds, 1), so).copy_(scale)
        y, st = dppo.dppo_matvec_int4(xd, q, sv, group)
        assert int(st.item()) == 0
        check_product(y, x, codes, scale, group, F32)


@pytest.mark.parametrize("M", [1, 61])
def test_product_special_values(M):
    """Infinities and NaN in x stay in their row, in a scale in their column; K = 0; all-zero rows."""
    N, K, group = 50, 300, 32
    x, codes, scale = product_case(M, N, K, group, seed=6)
    clean = [dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)[0]]
    scale[7, 3] = float("nan")
    y, _ = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
    assert torch.isnan(y[:, 7]).all() and torch.equal(torch.cat([y[:, :7], y[:, 8:]], 1), torch.cat([clean[0][:, :7], clean[0][:, 8:]], 1))
    scale[7, 3] = 1.0
    x[M - 1, 299] = float("nan")
    y, _ = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
    assert torch.isnan(y[M - 1]).all() and torch.isfinite(y[:M - 1]).all()
    x[M - 1] = 0
    y, _ = dppo.dppo_matvec_int4(x.to(DEV), packed(codes), scale.to(DEV), group)
    assert (y[M - 1] == 0).all()
    y, _ = dppo.dppo_matvec_int4(x[:, :0].to(DEV), packed(codes)[:, :0], scale[:, :0].to(DEV), group)
    assert (y == 0).all()


def test_product_repeats_its_bits_and_rows_do_not_mix():
    x, codes, scale = product_case(13, 500, 1024, 128, seed=8)
    q, s = packed(codes), scale.to(DEV)
    a, b = (dppo.dppo_matvec_int4(x.to(DEV), q, s)[0] for _ in range(2))
    assert torch.equal(a, b)
    x2 = x.clone()
    x2[5] = 1.0
    c = dppo.dppo_matvec_int4(x2.to(DEV), q, s)[0]
    keep = [m for m in range(13) if m != 5]
    assert torch.equal(c[keep], a[keep])


def test_product_captured_and_on_another_stream():
    x, codes, scale = product_case(4, 700, 2048, 128, seed=10)
    q, s, xd = packed(codes), scale.to(DEV), x.to(DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    want, _ = dppo.dppo_matvec_int4(xd, q, s, status=st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = dppo.dppo_matvec_int4(xd, q, s, status=st)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    wq = dppo.dppo_int4_quantize(xd, 32)["q"]                # (a kernel's first launch loads it, and waits for the device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    busy = torch.cuda.Event()
    busy.record()
    z, _ = dppo.dppo_matvec_int4(xd, q, s, stream=side)
    w = dppo.dppo_int4_quantize(xd, 32, stream=side)
    side.synchronize()
    assert not busy.query()
    torch.cuda.synchronize()
    assert torch.equal(z, want) and torch.equal(w["q"], wq)


def test_product_from_several_threads():
    """Calls that take unlike amounts of shared memory, from threads with a stream each."""
    cases = []
    for K in (512, 2048, 4096, 700):
        x, codes, scale = product_case(16, 900, K, 64, seed=K)
        q, s, xd = packed(codes), scale.to(DEV), x.to(DEV)
        cases.append((xd, q, s, dppo.dppo_matvec_int4(xd, q, s, 64)[0]))
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        xd, q, s, want = cases[i]
        st = torch.cuda.Stream(DEV)
        try:
            with torch.cuda.stream(st):
                for _ in range(200):
                    if not torch.equal(dppo.dppo_matvec_int4(xd, q, s, 64)[0], want):
                        wrong.append((i, "result"))
        except Exception as e:             # noqa: BLE001 (reported below)
            wrong.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:3]


def test_rollout_in_4_bits_and_its_update_end_to_end():
    """The LM head rounded to 4 bits, logits of a decoding step, tokens drawn from them, the trainer's logits from the values that the codes stand
    for and from the weights themselves, and the clipped loss with a KL term between the two."""
    g = torch.Generator().manual_seed(77)
    V, d, T = 1500, 256, 24
    W = (0.05 * torch.randn((V, d), generator=g)).to(BF).to(DEV)
    hidden = torch.randn((T, d), generator=g).to(BF).to(DEV)
    w4 = dppo.dppo_int4_quantize(W, 64, values=True)
    z4, st = dppo.dppo_matvec_int4(hidden, w4["q"], w4["scale"], 64)
    check_product(z4, hidden.cpu(), torch.from_numpy(R.unpack(w4["q"].cpu().numpy(), d)), w4["scale"].cpu(), 64, F32)
    o = dppo.dppo_sample(z4, torch.rand(T, generator=g, dtype=torch.float64).to(DEV), K=0, status=st)
    lp = dppo.dppo_token_logp(z4, o["sampled_ids"], status=st)["logp"]
    # the record's log mu and the log-probability of the same token under the same row
    assert (lp - o["mu_logp"]).abs().max().item() <= (V / 512 + 96) * 2.0 ** -24 + 2.0 ** -23 * o["mu_logp"].abs().max().item()
    z = (hidden.float() @ W.float().t())
    adv = torch.randn(T, generator=g).to(DEV)
    r = dppo.dppo_policy_kl_fwd_bwd(z, o["sampled_ids"], o["mu_logp"], adv, ref_logits=z4, kl_form=dppo.KL_PI_REF, kl_coef=0.1, status=st)
    w = R.policy_kl(z.double().cpu().numpy(), o["sampled_ids"].cpu().numpy(), o["mu_logp"].double().cpu().numpy(), adv.double().cpu().numpy(), np.ones(T, bool), "pi_ref",
                    float(np.float32(0.1)), 0.2, 0.2, y=z4.double().cpu().numpy())
    assert int(st.item()) == 0
    assert np.abs(r["kl"].double().cpu().numpy() - w["kl"]).max() <= 3 * (V / 512 + 96) * 2.0 ** -24 * (1 + w["spread"].max())
    d = r["dlogits"].double().cpu().numpy()
    assert np.abs(d - w["dlogits"]).max() <= 1e-4 * np.abs(w["dlogits"]).max()
