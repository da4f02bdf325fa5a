"""Forms of the 8-bit operators and the sampler that a caller may use and the other tests leave out, against 64-bit forms: outputs
that have no tensor map together with bias and accumulation, scales in every order, quotients on rounding borders, matrices of
more than 2^31 elements, and clusters inside a captured graph."""
import numpy as np
import pytest
import torch

import ops8_reference as ref
from test_gpu_ops8 import DEV, E4M3, NORM_REL, U, _P, _check_codes, _codes, _gemm_bounds, _operands

pytestmark = pytest.mark.gpu


# ---- the product: any output, any scales ----------------------------------------------------------------------------

@pytest.mark.parametrize("M,N,K", [(40, 301, 1024), (300, 521, 656), (520, 1027, 272), (1030, 2051, 128)])
@pytest.mark.parametrize("pitch,first", [(0, 0), (3, 1), (64, 2)])
@pytest.mark.parametrize("bias,accumulate,out_dtype", [(True, True, torch.float32), (False, True, torch.float32), (True, False, torch.bfloat16)])
def test_gemm_into_any_rows_with_bias_and_accumulation(M, N, K, pitch, first, bias, accumulate, out_dtype):
    """Outputs with odd pitches and odd first columns; what lies around them stays."""
    a, sa, w, sw = _operands(M, N, K, M + N + K + pitch, "plain")
    g = torch.Generator(device=DEV).manual_seed(4)
    b = torch.randn(N, generator=g, device=DEV) * 1e4 if bias else None
    big = (torch.randn(M + 2, N + first + pitch, generator=g, device=DEV) * 1e4).to(out_dtype)
    kept, out = big.clone(), big[1: M + 1, first: first + N]
    extra = ([b.double().cpu().numpy()[None, :] * np.ones((M, 1))] if bias else []) + ([out.double().cpu().numpy()] if accumulate else [])
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    _P().k_gemm_fp8(a, sa, w, sw, out, bias=b, accumulate=accumulate, status=st)
    want, bound = _gemm_bounds(a, sa, w, sw, out_dtype, extra)
    assert int(st) == 0 and np.all(np.abs(out.double().cpu().numpy() - want) <= bound)
    kept[1: M + 1, first: first + N] = out
    assert torch.equal(big, kept)


@pytest.mark.parametrize("M", [1, 20, 700])
@pytest.mark.parametrize("order", ["rows", "columns", "apart", "one_per_row", "one_per_block"])
def test_gemm_reads_scales_in_any_order(M, order):
    N, K = 1300, 1168
    a, sa, w, sw = _operands(M, N, K, M, "plain")

    def laid(s):
        R, C = s.shape
        t = {"rows": lambda: torch.empty(R, C, device=DEV), "columns": lambda: torch.empty(C, R, device=DEV).t(),
             "apart": lambda: torch.empty(R, 3, C, 5, device=DEV)[:, 1, :, 2], "one_per_row": lambda: torch.empty(R, 1, device=DEV).expand(R, C),
             "one_per_block": lambda: torch.empty(1, C, device=DEV).expand(R, C)}[order]()
        if order == "one_per_row":
            t[:, :1].copy_(s[:, :1])
        elif order == "one_per_block":
            t[:1].copy_(s[:1])
        else:
            t.copy_(s)
        return t

    sa, sw = laid(sa), laid(sw)
    out = torch.empty(M, N, device=DEV)
    _P().k_gemm_fp8(a, sa, w, sw, out)
    want, bound = _gemm_bounds(a, sa, w, sw, torch.float32)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound)


# ---- quantisation: quotients rounded once ---------------------------------------------------------------------------

@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_codes_are_those_of_quotients_rounded_once(xt, block_rows):
    """The codes of x / s with the division's own rounding in fp32 (numpy's, of the scale that the kernel wrote), exactly. bf16 and
    fp16 values over the scale of such a maximum often lie on the border between two codes; fp32 values are put next to borders."""
    R, K = 2048, 1024
    g = torch.Generator(device=DEV).manual_seed(17)
    x = torch.randn(R, K, generator=g, device=DEV).mul_(torch.exp(3 * torch.randn(R, 1, generator=g, device=DEV))).to(xt)
    if xt == torch.float32:
        codes = torch.arange(127, dtype=torch.uint8, device=DEV).view(E4M3).float()
        border = (codes[:-1] + codes[1:]) / 2
        at = border[torch.randint(0, 126, (R, K), generator=g, device=DEV)]
        s = (x.abs().view(R, K // 128, 128).amax(2) / 448).repeat_interleave(128, 1)
        near = (at * s).view(torch.int32) + torch.randint(-2, 3, (R, K), generator=g, device=DEV, dtype=torch.int32)
        x = torch.where(torch.rand(R, K, generator=g, device=DEV) < 0.8, near.view(torch.float32), x)
    q, sc = torch.empty(R, K, dtype=E4M3, device=DEV), torch.empty(R // block_rows, K // 128, device=DEV)
    _P().k_quant_fp8(x, q, sc, block_rows=block_rows)
    xs, s = x.float().cpu().numpy(), np.repeat(np.repeat(sc.cpu().numpy(), block_rows, 0), 128, 1)
    with np.errstate(invalid="ignore"):                      # (in fp16 a few of these values are infinities)
        quot = torch.from_numpy(np.clip(xs / s, np.float32(-448), np.float32(448)))
    # the NaN of an infinity over its infinite scale is a NaN code; which of the two says nothing (IEEE 754 leaves the sign open)
    got, want = (np.where((c & 127) == 127, 127, c) for c in (_codes(q), _codes(quot.to(E4M3))))
    assert np.array_equal(got == 127, np.isnan(quot.numpy())) and np.array_equal(got, want)


# ---- more than 2^31 elements ----------------------------------------------------------------------------------------

def _ends(R, mark):
    """Rows around the one that holds element 2^31 - 1, and the last ones."""
    return [*range(mark - 3, mark + 4), R - 2, R - 1]


def test_quantisation_and_norm_beyond_32_bits():
    R, d = 140001, 16384                                     # 2.29e9 elements; row 131072 begins at 2^31
    P, rows = _P(), _ends(140001, 131072)
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(R, d, generator=g, device=DEV, dtype=torch.bfloat16)
    w = 1 + 0.1 * torch.randn(d, generator=g, device=DEV)
    q, s = torch.empty(R, d, dtype=E4M3, device=DEV), torch.empty(d // 128, R, device=DEV).t()
    xd = x[rows].double().cpu().numpy()
    P.k_quant_fp8(x, q, s)
    _check_codes(_codes(q[rows]), s[rows].double().cpu().numpy(), xd, ref.block_scales(xd, 1), 1, 3 * U)
    P.k_rms_norm_fp8(x, w, q, s, delta=x, sum_out=x)         # in place: every row twice itself
    h = x[rows].double().cpu().numpy()
    assert np.array_equal(h, 2 * xd)
    y = ref.rms_norm(h, w.double().cpu().numpy(), float(np.float32(1e-5)))
    _check_codes(_codes(q[rows]), s[rows].double().cpu().numpy(), y, ref.block_scales(y, 1), 1, NORM_REL)
    t = torch.empty(-(-R // 128), d // 128, device=DEV)
    P.k_quant_fp8(x, q, t, block_rows=128)
    for b in (1023, 1024, R // 128):
        xd = x[128 * b: 128 * b + 128].double().cpu().numpy()
        _check_codes(_codes(q[128 * b: 128 * b + 128]), t[b: b + 1].double().cpu().numpy(), xd, ref.block_scales(xd, 128), 128, 3 * U)


def test_product_and_selection_beyond_32_bits():
    """An A of 2^31 bytes and more against few and many columns, and an output of more than 2^31 elements with its selection."""
    P = _P()
    M, K, rows = 140001, 16384, _ends(140001, 131072)
    a, sa, w, sw = _operands(M, 300, K, 7, "plain")
    for N in (24, 300):
        out = torch.empty(M, N, device=DEV)
        P.k_gemm_fp8(a, sa, w[:N], sw[: -(-N // 128)], out)
        want, bound = _gemm_bounds(a[rows], sa[rows], w[:N], sw[: -(-N // 128)], torch.float32)
        assert np.all(np.abs(out[rows].double().cpu().numpy() - want) <= bound)
    del a, out
    M, N, K = 70001, 32000, 128
    rows = _ends(70001, 67108)                               # 2^31 elements end in row 67108
    a, sa, w, sw = _operands(M, N, K, 5, "plain")
    sa.mul_(1e-3)
    g = torch.Generator(device=DEV).manual_seed(1)
    u, k, p = torch.rand(M, generator=g, device=DEV), torch.full((M,), 40, dtype=torch.int32, device=DEV), torch.full((M,), 0.9, device=DEV)
    one, none = torch.ones(M, device=DEV), torch.zeros(M, device=DEV)
    for out_dtype in (torch.bfloat16, torch.float32):
        out, tok = torch.empty(M, N, dtype=out_dtype, device=DEV), torch.empty(M, dtype=torch.int32, device=DEV)
        P.k_gemm_fp8(a, sa, w, sw, out)
        P.k_sample(out, u, tok, top_k=k, top_p=p)
        want, bound = _gemm_bounds(a[rows], sa[rows], w, sw, out_dtype)
        assert np.all(np.abs(out[rows].double().cpu().numpy() - want) <= bound)
        assert torch.equal(tok[rows], ref.sample_rows(out[rows], u[rows], one[rows], k[rows], p[rows], none[rows]))
        del out


# ---- a captured graph with clusters in both kernels -----------------------------------------------------------------

@pytest.mark.parametrize("R,V", [(1, 131072), (6, 50001)])
def test_clusters_in_a_captured_graph(R, V):
    """A few rows' product (K shared out in clusters) and selection (a cluster a row), captured and replayed with new inputs."""
    P = _P()
    K = 2048
    a, sa, w, sw = _operands(R, V, K, R, "plain")
    sa.mul_(1e-4)
    g = torch.Generator(device=DEV).manual_seed(3)
    out, tok = torch.empty(R, V, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)
    u, st = torch.rand(R, generator=g, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    par = [torch.full((R,), 0.9, device=DEV), torch.full((R,), 60, dtype=torch.int32, device=DEV), torch.full((R,), 0.95, device=DEV),
           torch.full((R,), 0.01, device=DEV)]

    def step():
        P.k_gemm_fp8(a, sa, w, sw, out, status=st)
        P.k_sample(out, u, tok, temperature=par[0], top_k=par[1], top_p=par[2], min_p=par[3], status=st)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        u.copy_(torch.rand(R, generator=g, device=DEV))
        sa.mul_(0.9)
        out.fill_(float("nan"))
        tok.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        want, bound = _gemm_bounds(a, sa, w, sw, torch.float32)
        assert int(st) == 0 and np.all(np.abs(out.double().cpu().numpy() - want) <= bound)
        assert torch.equal(tok, ref.sample_rows(out, u, *par))
