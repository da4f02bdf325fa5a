"""The 8-bit operators and the sampler with parameters per row against plain 64-bit implementations (ops8_reference)."""
import numpy as np
import pytest
import torch

import ops8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
U = 2.0 ** -24                # half a step of fp32, relative
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _P():
    import paper_2605_08696_b200 as P
    return P


def _rows(R, C, dtype, layout):
    """An [R, C] view whose rows lie apart (in a wider buffer, 16-byte pitch), or a plain matrix, and the whole buffer."""
    if layout == "plain":
        t = torch.empty(R, C, dtype=dtype, device=DEV)
        return t, t
    big = torch.empty(R + 2, C + 48, dtype=dtype, device=DEV)
    return big[1: R + 1, 16: 16 + C], big


def _scales(R, C, layout):
    """[R, C] scales, row after row, column after column, or both strides larger than they need be."""
    if layout == "plain":
        return torch.full((C, R), -1.0, device=DEV).t()
    if layout == "rows":
        return torch.full((R, C), -1.0, device=DEV)
    return torch.full((2 * C + 1, 3 * R + 2), -1.0, device=DEV).t()[1: 1 + 3 * R: 3, 1::2][:R, :C]


def _codes(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


VALUE = ref.e4m3_table()


def _check_codes(q, s, want, want_s, block_rows, rel):
    """Codes and scales of a matrix against its exact values over its exact scales: a code is within half a step (2^-4 relative,
    2^-10 among the subnormals) of the exact quotient, up to the relative error `rel` of the quotients themselves."""
    R, K = want.shape
    assert np.all(np.abs(s - want_s) <= rel * want_s)
    got = VALUE[q]
    quot = want / ref.spread(want_s, block_rows, R, K)
    err = np.abs(got - quot)
    bound = np.maximum(np.abs(quot) * 2.0 ** -4, 2.0 ** -10) * (1 + 1e-9) + 2 * rel * np.abs(quot)
    assert np.all(err <= bound), float((err - bound).max())
    assert np.all(np.abs(got) <= 448)


# ---- RMS norm -------------------------------------------------------------------------------------------------

# Relative error of a normed value and of its block's scale: each square 1, a thread's chain of at most 16 sums, 10 levels of
# a tree, the mean 1 and eps 1, halved by the root: 15; rsqrtf 2 ulp: 4; the two products 2; the division by 448 1: 22 roundings.
NORM_REL = 24 * U


@pytest.mark.parametrize("R,d", [(1, 16), (1, 1024), (3, 64), (5, 144), (37, 512), (9, 1040), (130, 1536), (4, 4096), (3, 5008), (2, 16384)])
@pytest.mark.parametrize("xt,dt", [("fp32", None), ("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp32"), ("bf16", None), ("fp32", "fp16")])
def test_rms_norm(R, d, xt, dt):
    g = torch.Generator(device=DEV).manual_seed(R * 100003 + d)
    layout = "apart" if (R + d // 16) % 2 else "plain"
    x, _ = _rows(R, d, TYPES[xt], layout)
    x.copy_(torch.randn(R, d, generator=g, device=DEV) * torch.exp(torch.randn(d, generator=g, device=DEV)))
    delta = None
    if dt is not None:
        delta, _ = _rows(R, d, TYPES[dt], layout)
        delta.copy_(torch.randn(R, d, generator=g, device=DEV))
    w = torch.randn(d, generator=g, device=DEV)
    q, qbig = _rows(R, d, E4M3, layout)
    qbig.view(torch.uint8).fill_(0x55)
    h, hbig = _rows(R, d, TYPES[xt], layout)
    hbig.fill_(7.0)
    s = _scales(R, -(-d // 128), "strided" if layout == "apart" else "rows" if d % 128 else "plain")
    _P().k_rms_norm_fp8(x, w, q, s, delta=delta, sum_out=h if dt is not None else None, eps=1e-5)
    torch.cuda.synchronize()
    want_h = x if dt is None else (x.float() + delta.float()).to(TYPES[xt])
    if dt is not None:
        assert torch.equal(h, want_h)
    # (eps reaches the kernel as fp32)
    y = ref.rms_norm(want_h.double().cpu().numpy(), w.double().cpu().numpy(), float(np.float32(1e-5)))
    _check_codes(_codes(q), s.double().cpu().numpy(), y, ref.block_scales(y, 1), 1, NORM_REL)
    if layout == "apart":                     # what lies around the rows is left as it was
        qbig[1: R + 1, 16: 16 + d].view(torch.uint8).fill_(0x55)
        assert bool((qbig.view(torch.uint8) == 0x55).all())
        if dt is not None:
            hbig[1: R + 1, 16: 16 + d] = 7.0
            assert bool((hbig == 7.0).all())


def test_rms_norm_in_place_and_special_rows():
    P = _P()
    R, d = 6, 384
    g = torch.Generator(device=DEV).manual_seed(5)
    x0 = torch.randn(R, d, generator=g, device=DEV)
    x0[1] = 0.0                                # zeros: eps alone under the root
    x0[2, 5], x0[3, 300], x0[4] = float("nan"), float("inf"), x0[4] * 1e-20
    x0[5] *= 1e15
    delta = torch.zeros(R, d, device=DEV, dtype=torch.bfloat16)
    w = torch.ones(d, device=DEV)
    x = x0.clone()
    q, s = torch.empty(R, d, dtype=E4M3, device=DEV), torch.empty(R, 3, device=DEV)
    P.k_rms_norm_fp8(x, w, q, s, delta=delta, sum_out=x, eps=1e-5)
    assert torch.equal(x[[0, 1, 4, 5]], x0[[0, 1, 4, 5]])
    code, sc = _codes(q), s.cpu().numpy()
    assert np.all(code[1] == 0) and np.all(sc[1] == np.float32(2.0 ** -100))
    assert np.all((code[2] & 127) == 127) and np.all(np.isnan(sc[2]))               # a NaN reaches the whole row
    assert (code[3, 300] & 127) == 127 and np.isnan(sc[3, 2])
    rows = [0, 4, 5]
    y = ref.rms_norm(x0[rows].double().cpu().numpy(), np.ones(d), float(np.float32(1e-5)))
    _check_codes(code[rows], sc[rows].astype(np.float64), y, ref.block_scales(y, 1), 1, NORM_REL)


# ---- quantisation ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("R,K", [(1, 16), (1, 128), (2, 4096), (127, 144), (128, 128), (129, 400), (300, 1536), (1000, 80)])
@pytest.mark.parametrize("xt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant(R, K, xt, block_rows):
    g = torch.Generator(device=DEV).manual_seed(R * 7 + K)
    layout = "apart" if R % 2 else "plain"
    x, _ = _rows(R, K, TYPES[xt], layout)
    x.copy_(torch.randn(R, K, generator=g, device=DEV) * torch.exp(2 * torch.randn(R, 1, generator=g, device=DEV)))
    x[0, : min(K, 128)] = 0.0                  # a row (and at block_rows 1 a block) of zeros
    q, qbig = _rows(R, K, E4M3, layout)
    qbig.view(torch.uint8).fill_(0x55)
    s = _scales(-(-R // block_rows), -(-K // 128), "strided" if R % 2 else "plain")
    _P().k_quant_fp8(x, q, s, block_rows=block_rows)
    torch.cuda.synchronize()
    xd = x.double().cpu().numpy()
    want_s = ref.block_scales(xd, block_rows)
    assert np.array_equal(s.cpu().numpy(), want_s.astype(np.float32))               # amax is exact, one rounding
    # the reciprocal of the scale and the product with it: two roundings; the scale's own: one
    _check_codes(_codes(q), s.double().cpu().numpy(), xd, want_s, block_rows, 3 * U)
    if layout == "apart":
        qbig[1: R + 1, 16: 16 + K].view(torch.uint8).fill_(0x55)
        assert bool((qbig.view(torch.uint8) == 0x55).all())


def test_quant_rounds_to_nearest_even_and_saturates():
    """With a largest magnitude of 448 the scale is 1 and the codes are those of torch's rounding, halfway cases among them."""
    v = torch.cat([torch.tensor([448.0, -448.0, 0.0, -0.0]), torch.arange(0, 12, 2.0 ** -10)[:12284]]).to(DEV)
    x = v.view(96, 128).clone()
    x[:, 0] = 448.0
    q, s = torch.empty(96, 128, dtype=E4M3, device=DEV), torch.empty(96, 1, device=DEV)
    _P().k_quant_fp8(x, q, s)
    assert bool((s == 1).all()) and np.array_equal(_codes(q), _codes(x.to(E4M3)))


def test_quant_of_non_finite_blocks():
    x = torch.ones(2, 256, device=DEV)
    x[0, 3], x[1, 200] = float("nan"), float("-inf")
    q, s = torch.empty(2, 256, dtype=E4M3, device=DEV), torch.empty(2, 2, device=DEV)
    _P().k_quant_fp8(x, q, s)
    s, c = s.cpu().numpy(), _codes(q)
    assert np.isnan(s[0, 0]) and np.all((c[0, :128] & 127) == 127) and s[0, 1] == np.float32(1 / 448) and np.all(c[0, 128:] == 0x7e)
    assert np.isinf(s[1, 1]) and (c[1, 200] & 127) == 127 and np.all(c[1, :128] == 0x7e)


# ---- the product ----------------------------------------------------------------------------------------------

def _operands(M, N, K, seed, layout):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def codes(R):
        t, _ = _rows(R, K, E4M3, layout)
        c = torch.randint(0, 256, (R, K), generator=g, device=DEV).to(torch.uint8)
        t.copy_(torch.where((c & 127) == 127, torch.zeros_like(c), c).view(E4M3))
        return t

    a, w = codes(M), codes(N)
    sa, sw = _scales(M, -(-K // 128), layout if layout != "apart" else "strided"), _scales(-(-N // 128), -(-K // 128), "rows")
    sa.copy_(torch.exp(torch.randn(sa.shape, generator=g, device=DEV)))
    sw.copy_(torch.exp(torch.randn(sw.shape, generator=g, device=DEV)))
    return a, sa, w, sw


def _gemm_bounds(a, sa, w, sw, out_dtype, extra=None):
    """The exact product and how far the kernel's may be: the products are exact; 128 of them are added in fp32, the scales'
    product is rounded once, the sums over the blocks (and bias and old output) add one rounding each, in any order; an adder
    that cuts off instead of rounding costs twice as much; last the output's own rounding."""
    A, W = VALUE[_codes(a)], VALUE[_codes(w)]
    SA, SW = sa.double().cpu().numpy(), sw.double().cpu().numpy()
    want, size = ref.gemm(A, SA, W, SW), ref.gemm(np.abs(A), SA, np.abs(W), SW)
    for e in extra or ():
        want, size = want + e, size + np.abs(e)
    bound = (128 + sa.shape[1] + 4) * 2 * U * size
    if out_dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    return want, bound


SHAPES = [(1, 1, 16), (1, 128, 128), (2, 5, 4096), (3, 257, 144), (7, 96, 2048), (16, 32, 1024), (17, 1000, 272), (33, 136, 6144), (64, 8000, 512),
          (65, 384, 1552), (128, 128, 128), (129, 300, 2064), (200, 2048, 640), (255, 513, 640), (256, 256, 256), (300, 520, 1152), (511, 4096, 512),
          (520, 1024, 1536), (1000, 264, 96), (1025, 1544, 384), (2100, 2056, 272), (65, 4104, 144), (70, 4099, 400), (100, 6144, 656),
          (384, 2050, 256), (385, 129, 128), (400, 257, 1040), (2000, 100, 272)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["plain", "apart"])
def test_gemm(M, N, K, out_dtype, layout):
    a, sa, w, sw = _operands(M, N, K, M * 31 + N * 7 + K, layout)
    out, big = _rows(M, N, out_dtype, layout)
    big.fill_(-3.0)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    _P().k_gemm_fp8(a, sa, w, sw, out, status=st)
    torch.cuda.synchronize()
    assert int(st) == 0
    want, bound = _gemm_bounds(a, sa, w, sw, out_dtype)
    err = np.abs(out.double().cpu().numpy() - want)
    assert np.all(err <= bound), float((err / np.maximum(bound, 1e-300)).max())
    if layout == "apart":
        big[1: M + 1, 16: 16 + N] = -3.0
        assert bool((big == -3.0).all())


@pytest.mark.parametrize("M,N,K", [(1, 24, 144), (40, 300, 1024), (300, 520, 1152), (600, 1024, 512), (2050, 1032, 256)])
@pytest.mark.parametrize("bias,accumulate,out_dtype", [(True, False, torch.float32), (True, True, torch.float32), (False, True, torch.float32),
                                                       (True, False, torch.bfloat16)])
def test_gemm_bias_and_accumulation(M, N, K, bias, accumulate, out_dtype):
    a, sa, w, sw = _operands(M, N, K, M + N + K, "plain")
    g = torch.Generator(device=DEV).manual_seed(3)
    b = torch.randn(N, generator=g, device=DEV) * 1e4 if bias else None
    out = (torch.randn(M, N, generator=g, device=DEV) * 1e4).to(out_dtype)
    extra = ([b.double().cpu().numpy()[None, :] * np.ones((M, 1))] if bias else []) + ([out.double().cpu().numpy()] if accumulate else [])
    _P().k_gemm_fp8(a, sa, w, sw, out, bias=b, accumulate=accumulate)
    want, bound = _gemm_bounds(a, sa, w, sw, out_dtype, extra)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("M,N", [(5, 200), (300, 520)])
def test_gemm_non_finite_values_stay_in_their_rows_and_columns(M, N):
    a, sa, w, sw = _operands(M, N, 640, 9, "plain")
    a.view(torch.uint8)[2, 300] = 0x7f
    sa[4, 1] = float("inf")
    w.view(torch.uint8)[N - 1, 7] = 0xff
    out = torch.empty(M, N, device=DEV)
    _P().k_gemm_fp8(a, sa, w, sw, out)
    bad = ~torch.isfinite(out)
    want = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    want[2], want[4], want[:, N - 1] = True, True, True
    assert torch.equal(bad, want)


def test_gemm_twice_gives_the_same_bits():
    for M, N, K in [(1, 1024, 4096), (40, 1000, 1040), (300, 520, 1152), (1100, 1024, 512)]:
        a, sa, w, sw = _operands(M, N, K, 1, "plain")
        o1, o2 = torch.empty(M, N, device=DEV), torch.empty(M, N, device=DEV)
        _P().k_gemm_fp8(a, sa, w, sw, o1)
        _P().k_gemm_fp8(a, sa, w, sw, o2)
        assert torch.equal(o1, o2)


# ---- sampling -------------------------------------------------------------------------------------------------

def _sample_case(R, V, seed, dtype, spread=2.0):
    rng = np.random.default_rng(seed)
    l = rng.normal(size=(R, V)) * rng.choice([0.1, 1.0, spread, 4.0], size=(R, 1))
    for r in range(R):
        l[r, rng.integers(0, V, size=5)] += rng.uniform(0, 12)
    l = torch.from_numpy(l).to(DEV).to(dtype)
    par = dict(temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.7], size=R, p=[.1, .2, .3, .3, .1]).astype(np.float32),
               top_k=rng.choice([0, -1, 1, 2, 20, 50, 300, V, V + 7], size=R).astype(np.int32),
               top_p=rng.choice([0.0, 0.2, 0.8, 0.9, 0.99, 1.0, 1.5], size=R).astype(np.float32),
               min_p=rng.choice([0.0, 0.0, 1e-4, 0.02, 0.3, 1.0, 2.0], size=R).astype(np.float32))
    u = rng.random(R).astype(np.float32)
    u[0] = 0.0
    u[R - 1] = 1 - 2.0 ** -24
    return l, u, par


def _run_sample(l, u, par, status=None):
    tok = torch.full((l.shape[0],), -7, dtype=torch.int32, device=DEV)
    dev = {k: torch.from_numpy(v).to(DEV) for k, v in par.items()}
    _P().k_sample(l, torch.from_numpy(u).to(DEV), tok, status=status, **dev)
    torch.cuda.synchronize()
    return tok.cpu().numpy()


def _want_tokens(l, u, par):
    ln = l.double().cpu().numpy()
    g = lambda k, d: par[k] if k in par else np.full(len(u), d)  # noqa: E731
    return np.array([ref.sample_row(ln[r], float(u[r]), float(g("temperature", 1.0)[r]), int(g("top_k", 0)[r]), float(g("top_p", 1.0)[r]),
                                    float(g("min_p", 0.0)[r]))[0] for r in range(len(u))])


@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (40, 31), (64, 33), (200, 256), (100, 1000), (64, 2049), (300, 8000), (24, 32000), (16, 32769),
                                 (8, 50257), (4, 131072), (2, 262144)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_sample(R, V, dtype):
    l, u, par = _sample_case(R, V, R * 1009 + V, dtype)
    assert np.array_equal(_run_sample(l, u, par), _want_tokens(l, u, par))


@pytest.mark.parametrize("only", [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("top_k", "top_p"), ("top_p", "min_p")])
@pytest.mark.parametrize("V", [999, 8000, 32000])
def test_sample_with_some_parameters_missing(only, V):
    l, u, par = _sample_case(60, V, 11 + V, torch.float32)
    par = {k: v for k, v in par.items() if k in only}
    assert np.array_equal(_run_sample(l, u, par), _want_tokens(l, u, par))


@pytest.mark.parametrize("V", [300, 8000, 32000, 40000])
def test_sample_where_logits_tie(V):
    """Few distinct values: borders inside groups of equal logits, decided by the lowest id; and rows of one value, where every
    cumulative mass is a whole number and u falls on borders exactly."""
    rng = np.random.default_rng(V)
    R = 48
    l = rng.integers(-3, 4, size=(R, V)).astype(np.float32)
    l[:8] = 1.25
    l[8:12] = np.float32(-3.4028235e38)        # a type's lowest value is a value like others
    l[12:16, ::2] = np.float32(-3.4028235e38)
    l[16:20, 3] = 0.0
    l[16:20, 1] = -0.0
    _, u, par = _sample_case(R, V, 3, torch.float32)
    u[:8] = (rng.integers(0, V, size=8) / V).astype(np.float32)
    par["temperature"][:16] = 1.0
    par["top_k"][:4], par["top_p"][:4], par["min_p"][:4] = 0, 1.0, 0.0
    lt = torch.from_numpy(l).to(DEV)
    assert np.array_equal(_run_sample(lt, u, par), _want_tokens(lt, u, par))


def test_sample_masked_rows_and_non_finite_logits():
    V, R = 5000, 9
    rng = np.random.default_rng(1)
    l = rng.normal(size=(R, V)).astype(np.float32)
    l[0] = -np.inf                              # nothing left
    l[1, :] = -np.inf
    l[1, 4321] = -2.0                           # one token left
    l[2, rng.random(V) < 0.9] = -np.inf
    l[3, ::3] = np.nan
    l[4, [7, 9, 4000]] = np.inf                 # plus infinity takes all of the mass
    l[5] = np.nan
    l[6, 4999] = 90.0
    u = rng.random(R).astype(np.float32)
    u[4] = 0.5
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    lt = torch.from_numpy(l).to(DEV)
    tok = _run_sample(lt, u, {}, status=st)
    assert int(st) == 4                         # SRM_STATUS_NONFINITE
    assert tok[0] == 0 and tok[1] == 4321 and tok[5] == 0 and tok[4] == 9 and tok[6] == 4999
    rows = [2, 3, 6, 7, 8]
    assert np.array_equal(tok[rows], _want_tokens(lt[rows], u[rows], {}))
    st.zero_()
    _run_sample(lt[6:].contiguous(), u[6:], {}, status=st)
    assert int(st) == 0                         # minus infinity alone, and finite rows, raise nothing
    _run_sample(lt[1:3].contiguous(), u[1:3], {}, status=st)
    assert int(st) == 0


@pytest.mark.parametrize("V", [1000, 32000])
def test_sample_with_a_nan_beside_the_largest_logit(V):
    """One NaN masks its own token and nothing around it, wherever it stands."""
    R = 64
    g = torch.Generator(device=DEV).manual_seed(V)
    l = torch.randn(R, V, generator=g, device=DEV)
    at = torch.randint(1, V - 1, (R,), generator=g, device=DEV)
    rows = torch.arange(R, device=DEV)
    l[rows, at] = 30.0
    l[rows, at + torch.where(rows % 2 == 0, 1, -1)] = float("nan")
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    tok = torch.empty(R, dtype=torch.int32, device=DEV)
    for T in (0.0, 1.0):
        _P().k_sample(l, torch.full((R,), 0.5, device=DEV), tok, temperature=torch.full((R,), T, device=DEV), status=st)
        assert torch.equal(tok, at.int()) and int(st) == 4


def test_sample_odd_parameters():
    """NaN parameters have no effect (temperature: greedy, u: 0); u of 1 or more picks the last token kept; tiny and huge
    temperatures."""
    V = 777
    l, _, _ = _sample_case(8, V, 21, torch.float32)
    nan = np.float32("nan")
    u = np.array([0.3, nan, 1.0, 5.0, 0.6, 0.6, 0.6, 0.2], np.float32)
    par = dict(temperature=np.array([nan, 1, 1, 1, 1e-30, 1e30, 2e-38, np.inf], np.float32), top_p=np.full(8, nan, np.float32),
               min_p=np.full(8, nan, np.float32), top_k=np.full(8, 10, np.int32))
    tok = _run_sample(l, u, par)
    want = _want_tokens(l, np.nan_to_num(u), {**par, "temperature": np.where(np.isnan(par["temperature"]), 0, par["temperature"]),
                                              "top_p": np.ones(8), "min_p": np.zeros(8)})
    assert np.array_equal(tok, want)


def test_sample_leaves_other_rows_and_reads_strided_logits():
    l, u, par = _sample_case(10, 1000, 2, torch.float32)
    big = torch.full((12, 1003), 50.0, device=DEV)
    big[1:11, 1:1001] = l
    tok = torch.full((12,), -7, dtype=torch.int32, device=DEV)
    dev = {k: torch.from_numpy(v).to(DEV) for k, v in par.items()}
    _P().k_sample(big[1:11, 1:1001], torch.from_numpy(u).to(DEV), tok[1:11], **dev)
    assert int(tok[0]) == int(tok[11]) == -7
    assert np.array_equal(tok[1:11].cpu().numpy(), _want_tokens(l, u, par))


@pytest.mark.parametrize("kind", ["normal", "flat", "ties", "const", "two", "peaky", "masked", "huge", "half_and_half"])
@pytest.mark.parametrize("V", [3, 140, 2300, 9001, 33000, 122484])
def test_sample_distributions(kind, V):
    """Rows of every shape and all combinations of parameters, among them exact ties of a nucleus' mass (half of a whole number of
    equal weights), nuclei that reach into the last tokens, limits beyond any list, temperatures that leave only the maximum or
    make all weights equal; unaligned rows."""
    R = max(8, min(400, 1600000 // V))
    g = torch.Generator(device=DEV).manual_seed(V + len(kind))
    rand = lambda: torch.rand(R, V, generator=g, device=DEV)  # noqa: E731
    x = torch.randn(R, V, generator=g, device=DEV)
    x = {"normal": lambda: x * 2, "flat": lambda: x * 1e-3, "ties": lambda: (x * 3).round(), "const": lambda: torch.full_like(x, 0.75),
         "two": lambda: torch.where(rand() < 0.5, 1.0, 0.9999), "peaky": lambda: x * 6,
         "masked": lambda: torch.where(rand() < 0.9, -float("inf"), x * 2), "huge": lambda: x * 1e30,
         "half_and_half": lambda: torch.where(torch.arange(V, device=DEV) % 2 == 0, 0.5, -0.25).expand(R, V)}[kind]().clone()
    x[:, 0] = 0.5
    l = torch.empty(R, V + 3, device=DEV)[:, V % 4 % 3: V % 4 % 3 + V]
    l.copy_(x)

    def pick(values, dtype=torch.float32):
        return torch.tensor(values, device=DEV)[torch.randint(0, len(values), (R,), generator=g, device=DEV)].to(dtype)

    T = pick([0.3, 0.7, 1.0, 1.0, 2.0, 1e-3, 50.0, 1e20])
    k = pick([0, 0, 0, 1, 2, 20, 50, 100, 128, 200, 257, 300, 700, 1024, 1500, 5000, V], torch.int32)
    p = pick([1.0, 1.0, 0.9, 0.95, 0.5, 0.5, 0.25, 0.1, 0.999, 1 - 2.0 ** -24, 1e-6])
    m = pick([0.0, 0.0, 0.0, 1e-6, 1e-3, 0.02, 0.1, 0.5, 1.0])
    u = torch.rand(R, generator=g, device=DEV)
    tok = torch.empty(R, dtype=torch.int32, device=DEV)
    _P().k_sample(l, u, tok, temperature=T, top_k=k, top_p=p, min_p=m)
    assert torch.equal(tok, ref.sample_rows(l, u, T, k, p, m))


def test_offsets_beyond_32_bits():
    """Logits of more than 2^31 elements (4.5 GB in bf16): the product writes and the sampler reads the rows behind that mark as it
    does the same rows in a small matrix."""
    M, N, K = 70001, 32000, 128
    a, sa, w, sw = _operands(M, N, K, 5, "plain")
    sa.mul_(1e-3)
    u = torch.rand(M, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    tok = torch.empty(M, dtype=torch.int32, device=DEV)
    P = _P()
    P.k_gemm_fp8(a, sa, w, sw, out)
    k, p = torch.full((M,), 40, dtype=torch.int32, device=DEV), torch.full((M,), 0.9, device=DEV)
    P.k_sample(out, u, tok, top_k=k, top_p=p)
    for rows in (slice(0, 300), slice(67050, 67350), slice(M - 300, M)):          # row 67108 is where 2^31 elements end
        o2, t2 = torch.empty(300, N, dtype=torch.bfloat16, device=DEV), torch.empty(300, dtype=torch.int32, device=DEV)
        P.k_gemm_fp8(a[rows], sa[rows], w, sw, o2)
        P.k_sample(o2, u[rows], t2, top_k=k[rows], top_p=p[rows])
        assert torch.equal(out[rows], o2) and torch.equal(tok[rows], t2)


@pytest.mark.parametrize("M,N", [(8390003, 24), (3, 8390003)])
def test_gemm_of_more_tiles_than_a_grid_counts_in_one_direction(M, N):
    a, sa, w, sw = _operands(M, N, 16, 6, "plain")
    out = torch.full((M, N), float("nan"), device=DEV)
    _P().k_gemm_fp8(a, sa, w, sw, out)
    for at in (0, 65535 * 128 - 128, max(M, N) - 131):                    # 65535 tiles of 128 end at 8388480
        m, n = (slice(at, at + 131), slice(0, N)) if M > N else (slice(0, M), slice(at // 128 * 128, at + 131))
        want, bound = _gemm_bounds(a[m], sa[m], w[n], sw[n.start // 128: -(-n.stop // 128)], torch.float32)
        assert np.all(np.abs(out[m, n].double().cpu().numpy() - want) <= bound)
    assert bool(torch.isfinite(out).all())


def test_one_scale_for_all():
    """Scales of the product's operands may be broadcast (strides of 0)."""
    M, N, K = 300, 520, 640
    a, sa, w, sw = _operands(M, N, K, 8, "plain")
    one, two = torch.full((1, 1), 0.5, device=DEV), torch.full((1, 1), 0.25, device=DEV)
    for rows in (M, 40):
        o1, o2 = torch.empty(rows, N, device=DEV), torch.empty(rows, N, device=DEV)
        _P().k_gemm_fp8(a[:rows], one.expand(rows, 5), w, two.expand(5, 5), o1)
        _P().k_gemm_fp8(a[:rows], torch.full((rows, 5), 0.5, device=DEV), w, torch.full((5, 5), 0.25, device=DEV), o2)
        assert torch.equal(o1, o2)


# ---- all together ---------------------------------------------------------------------------------------------

def _tail(P, b):
    P.k_rms_norm_fp8(b["x"], b["g"], b["q"], b["s"], delta=b["delta"], sum_out=b["h"])
    P.k_gemm_fp8(b["q"], b["s"], b["w"], b["ws"], b["logits"], status=b["status"])
    P.k_sample(b["logits"], b["u"], b["tok"], temperature=b["T"], top_k=b["k"], top_p=b["p"], min_p=b["m"], status=b["status"])


def _tail_buffers(P, R, d, V, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    kb = -(-d // 128)
    wf = r(V, d).mul_(0.2).bfloat16()
    b = dict(x=r(R, d), delta=r(R, d).bfloat16(), g=1 + 0.1 * r(d), h=torch.empty(R, d, device=DEV), wf=wf,
             q=torch.empty(R, d, dtype=E4M3, device=DEV), s=torch.empty(kb, R, device=DEV).t(),
             w=torch.empty(V, d, dtype=E4M3, device=DEV), ws=torch.empty(-(-V // 128), kb, device=DEV), logits=torch.empty(R, V, device=DEV),
             u=torch.rand(R, generator=g, device=DEV), tok=torch.empty(R, dtype=torch.int32, device=DEV),
             T=torch.full((R,), 0.7, device=DEV), k=torch.full((R,), 50, dtype=torch.int32, device=DEV),
             p=torch.full((R,), 0.9, device=DEV), m=torch.full((R,), 0.01, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    P.k_quant_fp8(wf, b["w"], b["ws"], block_rows=128)
    return b


@pytest.mark.parametrize("R,d,V", [(1, 1024, 32000), (29, 512, 8000), (300, 1536, 4000)])
def test_the_tail_of_a_decode_step(R, d, V):
    """Norm, product and selection one after the other, as a decode step ends: each stage against the 64-bit form of what it was
    given, and the logits against those of the matrices that were never quantised."""
    P = _P()
    b = _tail_buffers(P, R, d, V, R + V)
    _tail(P, b)
    torch.cuda.synchronize()
    assert int(b["status"]) == 0
    h = (b["x"] + b["delta"].float()).double().cpu().numpy()
    assert np.array_equal(b["h"].double().cpu().numpy(), h)
    want, bound = _gemm_bounds(b["q"], b["s"], b["w"], b["ws"], torch.float32)
    assert np.all(np.abs(b["logits"].double().cpu().numpy() - want) <= bound)
    par = dict(temperature=b["T"].cpu().numpy(), top_k=b["k"].cpu().numpy(), top_p=b["p"].cpu().numpy(), min_p=b["m"].cpu().numpy())
    assert np.array_equal(b["tok"].cpu().numpy(), _want_tokens(b["logits"], b["u"].cpu().numpy(), par))
    # every factor is off by at most 2^-4 of itself, a little more among a block's smallest values: together below 2^-3 + 2^-8 of
    # the sum of magnitudes, and subnormal codes add at most 2^-10 / 448 of a block's largest value each
    y = ref.rms_norm(h, b["g"].double().cpu().numpy(), float(np.float32(1e-5)))
    wd = b["wf"].double().cpu().numpy()
    sub = 2.0 ** -10
    ya = np.abs(y) + sub * ref.spread(ref.block_scales(y, 1), 1, R, d)
    wa = np.abs(wd) + sub * ref.spread(ref.block_scales(wd, 128), 128, V, d)
    tol = (ya * (1 + 2.0 ** -4)) @ (wa * (1 + 2.0 ** -4)).T - np.abs(y) @ np.abs(wd).T
    assert np.all(np.abs(b["logits"].double().cpu().numpy() - y @ wd.T) <= tol + 1e-4)


def test_the_tail_captured_into_graphs_and_on_other_streams():
    """Two captured graphs with buffers of their own, replayed on two streams at once, give what the eager calls give, and follow
    new inputs."""
    P = _P()
    shapes = [(5, 512, 8000), (260, 1024, 2056)]
    bufs = [_tail_buffers(P, *s, seed=i) for i, s in enumerate(shapes)]
    for b in bufs:
        _tail(P, b)
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for b in bufs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            _tail(P, b)
        graphs.append(gr)
    for b in bufs:                              # new inputs
        b["x"].mul_(-1.25)
        b["u"].copy_(1 - b["u"])
    want = []
    for b in bufs:
        _tail(P, b)
        want.append({k: b[k].clone() for k in ("q", "s", "h", "logits", "tok")})
        for k in ("q", "s", "h", "logits", "tok"):
            b[k].view(torch.uint8).zero_() if k == "q" else b[k].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    for b, w in zip(bufs, want):
        assert int(b["status"]) == 0
        for k in ("s", "h", "logits", "tok"):
            assert torch.equal(b[k], w[k]), k
        assert torch.equal(b["q"].view(torch.uint8), w["q"].view(torch.uint8))


def test_no_rows_and_refusals_on_the_device():
    P = _P()
    e = lambda *s, **k: torch.empty(*s, device=DEV, **k)  # noqa: E731
    P.k_rms_norm_fp8(e(0, 128), e(128), e(0, 128, dtype=E4M3), e(0, 1))
    P.k_quant_fp8(e(0, 128), e(0, 128, dtype=E4M3), e(0, 1))
    P.k_gemm_fp8(e(0, 128, dtype=E4M3), e(0, 1), e(8, 128, dtype=E4M3), e(1, 1), e(0, 8))
    P.k_sample(e(0, 8), e(0), e(0, dtype=torch.int32))
    for code, bad in ((P.ERR_UNSUPPORTED, lambda: P.k_quant_fp8(e(4, 24), e(4, 24, dtype=E4M3), e(4, 1))),
                      (P.ERR_UNSUPPORTED, lambda: P.k_gemm_fp8(e(4, 128, dtype=E4M3), e(4, 1), e(8, 128, dtype=E4M3), e(1, 1),
                                                               e(4, 8, dtype=torch.bfloat16), accumulate=True)),
                      (P.ERR_ALIGNMENT, lambda: P.k_quant_fp8(e(4, 40)[:, 1:17], e(4, 16, dtype=E4M3), e(4, 1)))):
        with pytest.raises(P.SRMError) as err:
            bad()
        assert err.value.code == code
