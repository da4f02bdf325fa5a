"""The 8-bit product of many rows and the sampler's cluster kernels beside other work: short products one after the other on two
streams, and clusters whose blocks start late and out of step. Every result is compared with the 64-bit form."""
import numpy as np
import pytest
import torch

import ops8_reference as ref
from test_gpu_ops8 import DEV, _P, _gemm_bounds, _operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [16, 128, 256, 400, 640, 1168])
def test_short_products_of_many_rows_on_two_streams(K, out_dtype):
    """A tile of one to nine blocks of K (fewer and more than there are stages), the code of each kernel cold at first."""
    P = _P()
    shapes = [(520, 256, K), (400, 4100, K), (1300, 2056, K)]
    ops = [_operands(*s, seed=K + i, layout="plain") for i, s in enumerate(shapes)]
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    outs = [[torch.full(s[:2], float("nan"), dtype=out_dtype, device=DEV) for _ in range(2)] for s in shapes]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for o, pair in zip(ops, outs):
            for stream, out in zip(streams, pair):
                with torch.cuda.stream(stream):
                    P.k_gemm_fp8(*o, out, status=st)
    torch.cuda.synchronize()
    assert int(st) == 0
    for o, pair in zip(ops, outs):
        assert torch.equal(pair[0], pair[1])
        want, bound = _gemm_bounds(*o, out_dtype)
        assert np.all(np.abs(pair[0].double().cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("R,V", [(1, 131072), (3, 262144), (9, 60001), (17, 40000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sampler_clusters_beside_other_work(R, V, dtype):
    """Few rows and long vocabularies (a cluster of blocks each), while another stream keeps the SMs busy."""
    P = _P()
    g = torch.Generator(device=DEV).manual_seed(R + V)
    l = (torch.randn(R, V, generator=g, device=DEV) * 2).to(dtype)
    busy, side = torch.randn(4096, 4096, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    for k, p, m in ((0, 0.9, 0.0), (50, 1.0, 0.0), (50, 0.8, 0.02), (0, 1.0, 0.1), (0, 1.0, 0.0), (1500, 0.95, 0.0), (1, 1.0, 0.0), (20, 0.3, 0.0)):
        par = [torch.full((R,), 0.8, device=DEV), torch.full((R,), k, dtype=torch.int32, device=DEV), torch.full((R,), p, device=DEV),
               torch.full((R,), m, device=DEV)]
        us = [torch.rand(R, generator=g, device=DEV) for _ in range(12)]
        toks = [torch.empty(R, dtype=torch.int32, device=DEV) for _ in us]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(6):
                busy = torch.tanh(busy @ busy.t() * 1e-2)
        for u, tok in zip(us, toks):
            P.k_sample(l, u, tok, temperature=par[0], top_k=par[1], top_p=par[2], min_p=par[3])
        torch.cuda.synchronize()
        for u, tok in zip(us, toks):
            assert torch.equal(tok, ref.sample_rows(l, u, *par))
