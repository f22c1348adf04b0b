"""CPU-only checks of the rollout-side entry points: refusals before anything is launched, and the float64 restatement."""
import ctypes
import os
import re
import subprocess
import sys

import numpy as np
import pytest

from oracle import rollout_oracle as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2602_04879_b200 import build
    build.build_library()
    from paper_2602_04879_b200 import binding as b
    return b


P = ctypes.c_void_p


def _sample(B, **over):
    a = dict(logits=0x10000, T=4, V=64, ld=64, dt=B.BF16, u=0x20000, tau=None, k=None, p=None, m=None, tok=None, K=0, ids=0x30000, lp=0x40000,
             ti=None, tp=None, status=0x50000)
    a.update(over)
    return B.lib().dppo_sample(P(a["logits"]), a["T"], a["V"], a["ld"], a["dt"], P(a["u"]), P(a["tau"]), P(a["k"]), P(a["p"]), P(a["m"]), P(a["tok"]),
                               a["K"], P(a["ids"]), P(a["lp"]), P(a["ti"]), P(a["tp"]), P(a["status"]), None)


def test_sample_refusals(binding):
    B = binding
    assert _sample(B, T=0) == 0                                     # nothing to do, nothing launched
    assert _sample(B, T=-1) == -2 and _sample(B, V=0) == -2 and _sample(B, K=-1) == -2 and _sample(B, K=65) == -2
    assert _sample(B, V=2 ** 31, ld=2 ** 31) == -2
    assert _sample(B, dt=2) == -3
    assert _sample(B, K=1025, V=5000, ld=5000) == -11
    for name in ("logits", "u", "ids", "lp", "status"):
        assert _sample(B, **{name: None}) == -1
    assert _sample(B, K=4) == -5 and _sample(B, K=4, ti=0x60000) == -5
    assert _sample(B, ld=63) == -6
    assert _sample(B, logits=0x10001) == -7 and _sample(B, u=0x20004) == -7
    assert _sample(B, dt=B.F32, logits=0x10002) == -7


def _quantize(B, **over):
    a = dict(x=0x10000, rows=4, cols=256, ld=256, dt=B.BF16, fmt=B.E4M3, br=1, q=0x20000, ldq=256, s=0x30000, sr=1, sk=4, qt=None, ldqt=16, st=None,
             str_=1, stk=256, status=0x50000)
    a.update(over)
    return B.lib().dppo_fp8_quantize(P(a["x"]), a["rows"], a["cols"], a["ld"], a["dt"], a["fmt"], a["br"], P(a["q"]), a["ldq"], P(a["s"]), a["sr"], a["sk"],
                                     P(a["qt"]), a["ldqt"], P(a["st"]), a["str_"], a["stk"], P(a["status"]), None)


def test_quantize_refusals(binding):
    B = binding
    assert _quantize(B, rows=0) == 0 and _quantize(B, cols=0) == 0
    assert _quantize(B, rows=-1) == -2 and _quantize(B, cols=-1) == -2 and _quantize(B, rows=2 ** 20, cols=2 ** 20, ld=2 ** 20, ldq=2 ** 20) == -2
    assert _quantize(B, dt=2) == -3 and _quantize(B, fmt=2) == -3 and _quantize(B, fmt=-1) == -3
    assert _quantize(B, br=64) == -11
    assert _quantize(B, x=None) == -1 and _quantize(B, q=None) == -1 and _quantize(B, s=None) == -1 and _quantize(B, qt=0x60000) == -1
    assert _quantize(B, status=None) == -1
    assert _quantize(B, ld=255) == -6 and _quantize(B, ldq=255) == -6 and _quantize(B, qt=0x60000, st=0x70000, ldqt=3) == -6
    assert _quantize(B, sk=3) == -6 and _quantize(B, sr=0) == -6 and _quantize(B, sr=1, sk=1) == -6 and _quantize(B, sr=-1) == -6      # scales that share a place
    assert _quantize(B, rows=200, sk=200, qt=0x60000, st=0x70000, ldqt=208, stk=255) == -6
    assert _quantize(B, x=0x10001) == -7 and _quantize(B, s=0x30002) == -7


def _product(B, **over):
    a = dict(A=0x10000, lda=256, fa=B.E4M3, abr=1, sa=0x20000, sar=1, sak=4, Bm=0x30000, ldb=256, fb=B.E4M3, bbr=128, sb=0x40000, sbr=1, sbk=1,
             M=4, N=8, K=256, C=0x50000, cdt=B.F32, ldc=8, status=0x60000, opts=None)
    a.update(over)
    o = a["opts"]
    return B.lib().dppo_gemm_tn_fp8(P(a["A"]), a["lda"], a["fa"], a["abr"], P(a["sa"]), a["sar"], a["sak"], P(a["Bm"]), a["ldb"], a["fb"], a["bbr"],
                                    P(a["sb"]), a["sbr"], a["sbk"], a["M"], a["N"], a["K"], P(a["C"]), a["cdt"], a["ldc"], P(a["status"]),
                                    ctypes.byref(o) if o is not None else None, None)


def test_product_refusals(binding):
    B = binding
    assert _product(B, M=0) == 0 and _product(B, N=0) == 0
    assert _product(B, M=-1) == -2 and _product(B, N=-1) == -2 and _product(B, K=-1) == -2
    assert _product(B, fa=2) == -3 and _product(B, fb=-1) == -3 and _product(B, cdt=2) == -3
    assert _product(B, abr=2) == -11 and _product(B, bbr=64) == -11 and _product(B, opts=B.DppoOpts(wait_limit_us=-1)) == -11
    for name in ("A", "Bm", "sa", "sb", "C"):
        assert _product(B, **{name: None}) == -1
    assert _product(B, lda=240) == -6 and _product(B, ldb=128) == -6 and _product(B, ldc=7) == -6 and _product(B, sak=-1) == -6
    assert _product(B, A=0x10008) == -7 and _product(B, Bm=0x30001) == -7 and _product(B, lda=264) == -7 and _product(B, ldb=257) == -7
    assert _product(B, C=0x50002) == -7 and _product(B, sa=0x20001) == -7


def test_binding_repeats_the_header(binding):
    hdr = open(os.path.join(ROOT, "include", "dppo.h")).read()
    assert int(re.search(r"#define\s+DPPO_SAMPLE_MAX_TOPK\s+(\d+)", hdr).group(1)) == binding.SAMPLE_MAX_TOPK
    assert int(re.search(r"DPPO_STATUS_BAD_SAMPLING\s*=\s*(\d+)", hdr).group(1)) == binding.STATUS_BAD_SAMPLING


def test_sampling_restatement():
    """The restatement itself: its frequencies over a grid of uniform numbers are the probabilities of the definition."""
    rng = np.random.default_rng(0)
    z = rng.standard_normal(40) * 2
    grid = (np.arange(4000) + 0.5) / 4000
    for s in ({}, {"temperature": 0.7}, {"top_k": 5}, {"top_p": 0.8}, {"min_p": 0.2}, {"top_k": 10, "top_p": 0.9, "min_p": 0.05}):
        w = np.exp((z - z.max()) / s.get("temperature", 1.0))
        order = np.argsort(-z, kind="stable")
        keep = np.zeros(40, bool)
        keep[order[: s.get("top_k", 40)]] = True
        if "top_p" in s:
            mass, run = w[keep].sum(), 0.0
            for j in order:
                if keep[j]:
                    keep[j] = run < s["top_p"] * mass
                    run += w[j]
        if "min_p" in s:
            keep &= w >= s["min_p"]
        p = np.where(keep, w, 0) / w[keep].sum()
        out = [R.sample_row(z, u, K=40, **s) for u in grid]
        freq = np.bincount([o["id"] for o in out], minlength=40) / 4000
        assert np.abs(freq - p).max() <= 1.0 / 4000 + 1e-12            # a cell of mass p holds p 4000 grid points, give or take one
        assert np.allclose(out[0]["top_p"][np.argsort(out[0]["top_ids"])], p) and out[0]["kept"] == keep.sum()
        assert all(abs(o["logp"] - np.log(p[o["id"]])) < 1e-12 for o in out)
    assert R.sample_row(z, 0.9, temperature=0.0)["id"] == int(np.argmax(z)) and R.sample_row(np.full(4, -np.inf), 0.5) is None


def test_rounding_restatement():
    torch = pytest.importorskip("torch")
    for fmt, dt, top in (("e4m3", torch.float8_e4m3fn, 0x7f), ("e5m2", torch.float8_e5m2, 0x7c)):
        vals = torch.arange(0, top, dtype=torch.uint8).view(dt).float().numpy().astype(np.float64)
        assert np.array_equal(R.round8(vals, fmt), vals) and np.array_equal(R.round8(-vals, fmt), -vals)
        mids = 0.5 * (vals[1:] + vals[:-1])
        even = np.where(np.arange(mids.size) % 2 == 0, vals[:-1], vals[1:])           # the code with a zero last bit
        assert np.array_equal(R.round8(mids, fmt), even)
        assert np.array_equal(R.round8(mids * (1 + 1e-12), fmt), vals[1:]) and np.array_equal(R.round8(mids * (1 - 1e-12), fmt), vals[:-1])
        assert R.round8(np.array([1e9]), fmt)[0] == R.MAX8[fmt]


def test_import_where_torch_has_no_cuda():
    """The package imports where torch was built without CUDA (such a build has no raw-stream query), and refuses at the call."""
    pytest.importorskip("torch")
    code = ("import torch\n"
            "for n in [n for n in dir(torch._C) if 'urrentRawStream' in n]: delattr(torch._C, n)\n"
            "import paper_2602_04879_b200 as dppo\n"
            "for call in (lambda: dppo.dppo_sample(torch.zeros(2, 4), torch.zeros(2, dtype=torch.float64)), lambda: dppo.dppo_fp8_quantize(torch.zeros(2, 4))):\n"
            "    try:\n        call()\n    except AssertionError:\n        pass\n    else:\n        raise SystemExit('CPU tensors were taken')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
