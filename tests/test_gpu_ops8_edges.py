"""Ends of the ranges that the 8-bit operators and the sampler with parameters per row take, against 64-bit forms."""
import numpy as np
import pytest
import torch

import ops8_reference as ref
from test_gpu_ops8 import DEV, NORM_REL, _P, _check_codes, _codes

pytestmark = pytest.mark.gpu
INF = float("inf")


def _pick(g, R, values, dtype=torch.float32):
    return torch.tensor(values, device=DEV)[torch.randint(0, len(values), (R,), generator=g, device=DEV)].to(dtype)


def _tokens(l, u, T, k, p, m):
    tok = torch.full((l.shape[0],), -7, dtype=torch.int32, device=DEV)
    _P().k_sample(l, u, tok, temperature=T, top_k=k, top_p=p, min_p=m)
    return tok


# ---- sampling at the highest temperatures -------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["equal", "normal", "lowest", "widest"])
@pytest.mark.parametrize("mask", ["none", "minus_infinity", "nan"])
@pytest.mark.parametrize("R,V", [(256, 100), (200, 2300), (200, 9001), (2, 100000)])
def test_sample_at_high_temperatures(R, V, kind, mask):
    """A masked token (minus infinity, NaN) has no mass at any temperature, up to infinity, where all others have the same; and
    logits further apart than the largest fp32 number have the weights of their difference."""
    g = torch.Generator(device=DEV).manual_seed(V + 7 * len(kind) + len(mask))
    rand = lambda: torch.rand(R, V, generator=g, device=DEV)  # noqa: E731
    l = {"equal": lambda: torch.full((R, V), 0.75, device=DEV), "normal": lambda: torch.randn(R, V, generator=g, device=DEV) * 3,
         "lowest": lambda: torch.where(rand() < 0.5, torch.finfo(torch.float32).min, 2.0),
         "widest": lambda: (rand() * 2 - 1) * torch.finfo(torch.float32).max}[kind]()
    if mask != "none":
        l = torch.where(rand() < 0.5, -INF if mask == "minus_infinity" else float("nan"), l)
        l[:, 0] = 0.75
    for T in ([1e30, 1e36, 8e36], [2e37, 1e38], [3.4028235e38, INF]):
        for _ in range(3 if R < 8 else 1):
            args = (torch.rand(R, generator=g, device=DEV), _pick(g, R, T), _pick(g, R, [0, 0, 0, 20, 60, 1500], torch.int32),
                    _pick(g, R, [0.1, 0.5, 0.9, 0.9, 0.999, 1.0]), _pick(g, R, [0.0, 0.0, 0.0, 1e-3, 0.5, 1.0]))
            assert torch.equal(_tokens(l, *args), ref.sample_rows(l, *args))


def test_masked_half_of_a_row_at_infinite_temperature():
    """Fifty tokens of equal weight, 0.9 of their mass: the first 45, whatever stands in the masked places."""
    l = torch.full((2, 100), 0.75, device=DEV)
    l[0, 1::2], l[1, 1::2] = -INF, float("nan")
    n = 4000
    l = l.repeat_interleave(n, 0)
    u = torch.linspace(0, 1 - 2.0 ** -24, n, device=DEV).repeat(2)
    tok = torch.empty(2 * n, dtype=torch.int32, device=DEV)
    _P().k_sample(l, u, tok, temperature=torch.full((2 * n,), INF, device=DEV), top_p=torch.full((2 * n,), 0.9, device=DEV))
    for t in tok.view(2, n):
        assert t.unique().tolist() == list(range(0, 90, 2))


# ---- random numbers at and next to zero ----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V", [(300, 100), (200, 2300), (200, 9001), (2, 100000)])
def test_sample_with_random_numbers_near_zero(R, V, dtype):
    """u = 0 picks the lowest id that is kept, however little it weighs (as long as that is a number in 64 bits), and a tiny u the
    id that its mass falls on."""
    g = torch.Generator(device=DEV).manual_seed(V)
    l = (torch.randn(R, V, generator=g, device=DEV) * _pick(g, R, [2.0, 15.0, 40.0])[:, None]).to(dtype)
    l[:, 3] = -INF
    for us in ([0.0], [1e-45, 1e-40, 1e-36, 1e-30], [1e-25, 1e-20, 2.0 ** -40, 2.0 ** -24]):
        for _ in range(4 if R < 8 else 1):
            args = (_pick(g, R, us), _pick(g, R, [0.3, 1.0, 3.0]), _pick(g, R, [0, 0, 20, 50, 300, 1500, V], torch.int32),
                    _pick(g, R, [1.0, 1.0, 1.0, 0.9]), _pick(g, R, [0.0, 0.0, 1e-40, 1e-36, 1e-30, 1e-10]))
            assert torch.equal(_tokens(l, *args), ref.sample_rows(l, *args))


# ---- RMS norm: rows that are not finite, and the least rows without eps ---------------------------------------------

@pytest.mark.parametrize("d", [16, 384, 5008, 16384])
@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16, torch.float16])
def test_rms_norm_of_rows_that_are_not_finite(d, xt):
    """A NaN, an infinity, or squares beyond fp32 make the whole row's codes and scales NaN, and no other row's."""
    g = torch.Generator(device=DEV).manual_seed(d)
    x = torch.randn(9, d, generator=g, device=DEV).to(xt)
    delta = torch.randn(9, d, generator=g, device=DEV)
    x[1, d - 1], x[2, 0], x[3, d // 2] = INF, -INF, float("nan")
    delta[5, 7] = INF
    x[6, 3], delta[6, 3] = 6e4, 6e4                          # beyond fp16, a value like others in the other types
    delta[7, 1] = 1e25                                       # its square is beyond fp32 (and it is beyond fp16)
    w = torch.randn(d, generator=g, device=DEV)
    kb = -(-d // 128)
    q, s, h = torch.empty(9, d, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(9, kb, device=DEV), torch.empty_like(x)
    _P().k_rms_norm_fp8(x, w, q, s, delta=delta, sum_out=h, eps=1e-5)
    bad = [1, 2, 3, 5, 7] + ([6] if xt == torch.float16 else [])
    good = [r for r in range(9) if r not in bad]
    assert torch.equal(h.nan_to_num(nan=1.5), (x.float() + delta).to(xt).nan_to_num(nan=1.5))
    assert bool(((q.view(torch.uint8)[bad] & 127) == 127).all()) and bool(s[bad].isnan().all())
    want = ref.rms_norm(h[good].double().cpu().numpy(), w.double().cpu().numpy(), float(np.float32(1e-5)))
    _check_codes(_codes(q[good].view(torch.uint8)), s[good].double().cpu().numpy(), want, ref.block_scales(want, 1), 1, NORM_REL)


@pytest.mark.parametrize("d", [16, 400, 16384])
@pytest.mark.parametrize("rms", [1e-17, 1e-12, 1.0, 1e16])
def test_rms_norm_without_eps(d, rms):
    """eps = 0: rows with a root mean square from 1e-17 on, values spread over twelve powers of ten, are as exact as others (below
    that squares leave fp32's range); a row of zeros has no norm."""
    g = torch.Generator(device=DEV).manual_seed(d + 1)
    x = torch.randn(5, d, generator=g, device=DEV).double() * 10.0 ** (-12 * torch.rand(5, d, generator=g, device=DEV).double())
    x = (x / (x * x).mean(1, keepdim=True).sqrt() * (1.001 * rms)).clamp(-1e17, 1e17).float()
    x[4] = 0
    w = torch.randn(d, generator=g, device=DEV)
    q, s = torch.empty(5, d, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(5, -(-d // 128), device=DEV)
    _P().k_rms_norm_fp8(x, w, q, s, eps=0.0)
    assert bool(((q.view(torch.uint8)[4] & 127) == 127).all()) and bool(s[4].isnan().all())
    want = ref.rms_norm(x[:4].double().cpu().numpy(), w.double().cpu().numpy(), 0.0)
    _check_codes(_codes(q[:4].view(torch.uint8)), s[:4].double().cpu().numpy(), want, ref.block_scales(want, 1), 1, NORM_REL)


# ---- a nucleus that ends a few 1e-12 of the mass beside a group of equal logits -------------------------------------

def _close_row(nA, nB, V, gap):
    """Logits of nA tokens at 0, nB at -1 and a few near -16, and a top_p, so that the first group misses top_p's part of the whole
    mass by `gap` of the whole (negative: exceeds it): what two exponentials in 64 bits tell apart."""
    w = np.exp(-1.0)
    p = np.float32(nA / (nA + nB * w))
    while float(p) * (nA + nB * w) > nA * (1 - 1e-8):
        p = np.nextafter(p, np.float32(0))
    total = nA / (float(p) - gap)                    # nA = (p - gap) total
    nC = 50
    c = np.float32(np.log((total - nA - nB * w) / nC))
    l = np.full(V, -np.inf, np.float32)
    l[: 2 * nA: 2] = 0                               # ids of the first group lie below the second's
    l[2 * nA: 2 * nA + nB] = -1
    l[V - nC:] = c
    total = nA + nB * w + nC * np.exp(float(c))
    return l, p, (float(p) * total - nA) / total


@pytest.mark.parametrize("nA,nB,V", [(1500, 3000, 9001), (2000, 1200, 33000), (5000, 20000, 120000)])
def test_sample_decides_borders_to_64_bits(nA, nB, V):
    rows = [_close_row(nA, nB, V, gap) for gap in (4e-12, -4e-12, 1e-12, -1e-12)]
    for _, _, gap in rows:
        assert 5e-13 < abs(gap) < 8e-12
    l = torch.from_numpy(np.stack([r[0] for r in rows])).to(DEV)
    R = len(rows)
    p, u = torch.tensor([float(r[1]) for r in rows], device=DEV), torch.full((R,), 1 - 2.0 ** -24, device=DEV)
    one, none, k = torch.ones(R, device=DEV), torch.zeros(R, device=DEV), torch.zeros(R, dtype=torch.int32, device=DEV)
    # the last token kept: the first id of the second group where the first one's mass is too little, else the first group's last
    want = torch.tensor([2 * nA if r[2] > 0 else 2 * nA - 2 for r in rows], dtype=torch.int32, device=DEV)
    assert torch.equal(ref.sample_rows(l, u, one, k, p, none), want)
    for n in (1, 100):                               # both launch forms for the longer rows
        ln, un, pn, on, zn, kn = (t.repeat_interleave(n, 0) for t in (l, u, p, one, none, k))
        assert torch.equal(_tokens(ln, un, on, kn, pn, zn), want.repeat_interleave(n))
