"""Refusals of the 8-bit operators and of the sampler with parameters per row, and their 64-bit references. No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import ops8_reference as ref
import paper_2605_08696_b200 as P

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, -1, -2, -3
A = 1 << 20                      # a 16-byte aligned address; nothing is launched in any of these calls


def _norm(**kw):
    a = dict(R=2, d=128, x=A, xt=0, xs=128, dl=None, dt=0, ds=0, g=A, eps=1e-5, h=None, hs=0, q=A, qs=128, s=A, sr=1, sb=2)
    a.update(kw)
    return P.load_library().srm_k_rms_norm_fp8(*[a[k] for k in ("R", "d", "x", "xt", "xs", "dl", "dt", "ds", "g", "eps", "h", "hs",
                                                               "q", "qs", "s", "sr", "sb")], None)


def _quant(**kw):
    a = dict(R=2, K=128, x=A, xt=1, xs=128, br=1, q=A, qs=128, s=A, sr=1, sb=2)
    a.update(kw)
    return P.load_library().srm_k_quant_fp8(*[a[k] for k in ("R", "K", "x", "xt", "xs", "br", "q", "qs", "s", "sr", "sb")], None)


def _gemm(**kw):
    a = dict(M=2, N=8, K=128, A=A, as_=128, sa=A, sar=1, sab=2, W=A, ws=128, sw=A, swr=1, swb=1, bias=None, acc=0, out=A, ot=0, os=8, st=None)
    a.update(kw)
    return P.load_library().srm_k_gemm_fp8(*[a[k] for k in ("M", "N", "K", "A", "as_", "sa", "sar", "sab", "W", "ws", "sw", "swr",
                                                           "swb", "bias", "acc", "out", "ot", "os", "st")], None)


def _sample(**kw):
    a = dict(R=2, V=8, l=A, lt=0, ls=8, u=A, T=None, k=None, p=None, m=None, tok=A, st=None)
    a.update(kw)
    return P.load_library().srm_k_sample(*[a[k] for k in ("R", "V", "l", "lt", "ls", "u", "T", "k", "p", "m", "tok", "st")], None)


@pytest.mark.parametrize("call,kw,code", [
    (_norm, dict(R=-1), INVALID), (_norm, dict(d=0), INVALID), (_norm, dict(xt=3), INVALID), (_norm, dict(dl=A, dt=9, ds=128), INVALID),
    (_norm, dict(eps=-1.0), INVALID), (_norm, dict(eps=float("nan")), INVALID), (_norm, dict(h=A, hs=128), INVALID),
    (_norm, dict(d=120), UNSUPPORTED), (_norm, dict(d=16400), UNSUPPORTED), (_norm, dict(x=None), INVALID), (_norm, dict(q=None), INVALID),
    (_norm, dict(g=None), INVALID), (_norm, dict(s=None), INVALID), (_norm, dict(xs=127), INVALID), (_norm, dict(x=A + 4), ALIGNMENT),
    (_norm, dict(xs=130), ALIGNMENT), (_norm, dict(qs=136), ALIGNMENT), (_norm, dict(q=A + 8), ALIGNMENT), (_norm, dict(g=A + 4), ALIGNMENT),
    (_norm, dict(s=A + 2), ALIGNMENT), (_norm, dict(sr=0), INVALID), (_norm, dict(d=256, xs=256, qs=256, sb=0), INVALID), (_norm, dict(dl=A + 2, ds=128), ALIGNMENT),
    (_norm, dict(dl=A, ds=128, h=A, hs=64), INVALID), (_norm, dict(R=0, x=None), OK),
    (_quant, dict(R=-2), INVALID), (_quant, dict(K=0), INVALID), (_quant, dict(K=100), UNSUPPORTED), (_quant, dict(br=2), INVALID),
    (_quant, dict(br=0), INVALID), (_quant, dict(xt=-1), INVALID), (_quant, dict(x=None), INVALID), (_quant, dict(x=A + 2), ALIGNMENT),
    (_quant, dict(xs=132), ALIGNMENT), (_quant, dict(qs=132), ALIGNMENT), (_quant, dict(qs=112), INVALID), (_quant, dict(s=None), INVALID),
    (_quant, dict(K=144, xs=144, qs=144, sb=0), INVALID), (_quant, dict(R=1 << 40), UNSUPPORTED), (_quant, dict(R=0, q=None), OK),
    (_gemm, dict(M=-1), INVALID), (_gemm, dict(N=0), INVALID), (_gemm, dict(K=0), INVALID), (_gemm, dict(K=24), UNSUPPORTED),
    (_gemm, dict(ot=2), INVALID), (_gemm, dict(acc=2), INVALID), (_gemm, dict(acc=1, ot=1), UNSUPPORTED), (_gemm, dict(A=None), INVALID),
    (_gemm, dict(W=None), INVALID), (_gemm, dict(sa=None), INVALID), (_gemm, dict(sw=None), INVALID), (_gemm, dict(out=None), INVALID),
    (_gemm, dict(A=A + 1), ALIGNMENT), (_gemm, dict(W=A + 8), ALIGNMENT), (_gemm, dict(as_=136), ALIGNMENT), (_gemm, dict(ws=120), INVALID),
    (_gemm, dict(out=A + 2), ALIGNMENT), (_gemm, dict(out=A + 1, ot=1), ALIGNMENT), (_gemm, dict(os=7), INVALID), (_gemm, dict(sar=-1), INVALID),
    (_gemm, dict(N=200, os=200, swr=-1), INVALID), (_gemm, dict(bias=A + 2), ALIGNMENT), (_gemm, dict(M=0, A=None), OK),
    (_gemm, dict(M=(1 << 30) + 1), UNSUPPORTED), (_gemm, dict(K=(1 << 20) + 16), UNSUPPORTED), (_gemm, dict(st=A + 2), ALIGNMENT),
    (_sample, dict(R=-1), INVALID), (_sample, dict(V=0), INVALID), (_sample, dict(V=262145, ls=262145), UNSUPPORTED), (_sample, dict(lt=5), INVALID),
    (_sample, dict(l=None), INVALID), (_sample, dict(u=None), INVALID), (_sample, dict(tok=None), INVALID), (_sample, dict(ls=7), INVALID),
    (_sample, dict(l=A + 2), ALIGNMENT), (_sample, dict(l=A + 1, lt=1), ALIGNMENT), (_sample, dict(T=A + 1), ALIGNMENT),
    (_sample, dict(st=A + 2), ALIGNMENT), (_sample, dict(R=0, u=None), OK),
])
def test_refusals(call, kw, code):
    assert call(**kw) == code


def test_the_binding_refuses_before_the_library_is_asked():
    x = torch.zeros(4, 256)
    q, s = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 2)
    g = torch.ones(256)
    for bad in (lambda: P.k_rms_norm_fp8(x, g, q, s),                                 # not on a GPU
                lambda: P.k_rms_norm_fp8(x, g, q, s[:, :1]), lambda: P.k_rms_norm_fp8(x, g[:100], q, s),
                lambda: P.k_rms_norm_fp8(x.t(), g, q, s), lambda: P.k_rms_norm_fp8(x, g, q, s, sum_out=x.bfloat16()),
                lambda: P.k_rms_norm_fp8(x.double(), g, q, s), lambda: P.k_quant_fp8(x, q, s, block_rows=64),
                lambda: P.k_quant_fp8(x, q, s, block_rows=128), lambda: P.k_quant_fp8(x, q[:3], s),
                lambda: P.k_gemm_fp8(q, s, q, s[:1], torch.zeros(4, 4).half()), lambda: P.k_gemm_fp8(q, s, q, s, torch.zeros(4, 4)),
                lambda: P.k_gemm_fp8(q, s, q[:, :128], s[:1], torch.zeros(4, 4)), lambda: P.k_gemm_fp8(q, s, q, s[:1], torch.zeros(4, 5)),
                lambda: P.k_sample(x, torch.zeros(4), torch.zeros(4, dtype=torch.int64)), lambda: P.k_sample(x, torch.zeros(3), torch.zeros(4, dtype=torch.int32)),
                lambda: P.k_sample(x, torch.zeros(4), torch.zeros(4, dtype=torch.int32), top_k=torch.zeros(4)),
                lambda: P.k_sample(x, None, torch.zeros(4, dtype=torch.int32)), lambda: P.k_sample(x[0], torch.zeros(4), torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(ValueError):
            bad()


def test_e4m3_table_is_torch_s():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3_table(), want, equal_nan=True)


def test_sample_reference_on_rows_worked_out_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.25, 0.15]))
    # whole distribution: ids ascending, borders 0.1 0.5 0.6 0.85 1
    for u, tok in ((0.0, 0), (0.0999, 0), (0.11, 1), (0.499, 1), (0.55, 2), (0.84, 3), (0.99, 4)):
        assert ref.sample_row(l, u)[0] == tok
    assert list(ref.sample_row(l, 0.5, top_k=3)[1]) == [1, 3, 4]
    assert list(ref.sample_row(l, 0.5, top_k=4)[1]) == [0, 1, 3, 4]                 # equal logits: the lowest id
    assert list(ref.sample_row(l, 0.5, top_p=0.6)[1]) == [1, 3]
    assert list(ref.sample_row(l, 0.5, top_k=2, top_p=0.6)[1]) == [1]               # 0.4 / 0.65 reaches 0.6
    assert list(ref.sample_row(l, 0.5, min_p=0.3)[1]) == [1, 3, 4]
    assert list(ref.sample_row(l, 0.5, T=0.5, min_p=0.3)[1]) == [1, 3]              # 0.25^2 / 0.4^2 = 0.39, 0.15^2 / 0.4^2 = 0.14
    assert ref.sample_row(l, 0.99, T=0.0)[0] == 1 and ref.sample_row(np.full(4, -np.inf), 0.5)[0] == 0
