"""The 8-bit product of many rows beside other work: short products one after the other on two streams, compared with the 64-bit
form."""
import numpy as np
import pytest
import torch

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
