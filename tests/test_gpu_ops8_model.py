"""The sampler with parameters per row and the 8-bit operators on a model of the library: its decode step's logits, its weights and
its normed activations."""
import numpy as np
import pytest
import torch

import ops8_reference as ref
import srm_inputs as I
from helpers import custom_shape
from test_gpu_ops8 import DEV, E4M3, _P, _gemm_bounds

pytestmark = pytest.mark.gpu


def _model():
    shape = custom_shape(n_layers=2, d_model=512, vocab=8000, n_ctx=48, dtype="bf16", seed=4)
    return shape, _P().SRM(shape, I.make_weights(shape, alpha_std=0.5, beta_std=0.5), device=DEV)


@pytest.mark.parametrize("B", [1, 37])
def test_decoding_with_each_sample_s_own_parameters(B):
    P, (shape, m) = _P(), _model()
    g = torch.Generator(device=DEV).manual_seed(B)
    prompts = torch.randint(0, shape.vocab, (B, 16), generator=g, device=DEV, dtype=torch.int32)
    st, ws, greedy = m.new_state(B), m.new_workspace(B, 16), P.Sampling("greedy")
    tok, _ = m.prefill(st, prompts, greedy, ws, want_logits=True)
    T = 0.5 + torch.rand(B, generator=g, device=DEV)
    k = torch.randint(0, 60, (B,), generator=g, device=DEV, dtype=torch.int32)
    p, mp = 0.7 + 0.4 * torch.rand(B, generator=g, device=DEV), 0.05 * torch.rand(B, generator=g, device=DEV)
    for step in range(1, 25):
        _, logits = m.decode_step(st, tok, greedy, step, ws, want_logits=True)
        u = torch.rand(B, generator=g, device=DEV)
        tok = torch.empty(B, dtype=torch.int32, device=DEV)
        P.k_sample(logits, u, tok, temperature=T, top_k=k, top_p=p, min_p=mp)
        assert torch.equal(tok, ref.sample_rows(logits, u, T, k, p, mp))
    assert st.status() == 0


@pytest.mark.parametrize("R", [1, 50, 400])
def test_a_model_s_projections_in_8_bits(R):
    """Up projection (with its bias) and LM head of normed activations, weights and activations quantised: the products of the
    codes as they are, and beside the products of the bf16 matrices, from which every factor is off by at most 2^-4 of itself (and
    2^-10 / 448 of its block's largest value among the subnormal codes)."""
    P, (shape, m) = _P(), _model()
    d = shape.d_model
    x = torch.randn(R, d, generator=torch.Generator(device=DEV).manual_seed(R), device=DEV) * 2 + 1
    a = torch.empty(R, d, dtype=m.act_dtype, device=DEV)
    m.k_final_norm(x, a)
    q, s = torch.empty(R, d, dtype=E4M3, device=DEV), torch.empty(d // 128, R, device=DEV).t()
    P.k_quant_fp8(a, q, s)
    for layer, tid, bias_tid in ((0, P.binding.T_W1, P.binding.T_B1), (-1, P.binding.T_W_LM, None)):
        W = m.tensor(layer, tid)
        b = m.tensor(layer, bias_tid).float().contiguous() if bias_tid else None
        N = W.shape[0]
        wq, ws = torch.empty(N, d, dtype=E4M3, device=DEV), torch.empty(-(-N // 128), d // 128, device=DEV)
        P.k_quant_fp8(W, wq, ws, block_rows=128)
        out, st = torch.empty(R, N, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        P.k_gemm_fp8(q, s, wq, ws, out, bias=b, status=st)
        extra = [b.double().cpu().numpy()[None, :] * np.ones((R, 1))] if bias_tid else []
        want, bound = _gemm_bounds(q, s, wq, ws, torch.float32, extra)
        got = out.double().cpu().numpy()
        assert int(st) == 0 and np.all(np.abs(got - want) <= bound)
        ad, wd = a.double().cpu().numpy(), W.double().cpu().numpy()
        sub = 2.0 ** -10
        am = np.abs(ad) + sub * ref.spread(ref.block_scales(ad, 1), 1, R, d)
        wm = np.abs(wd) + sub * ref.spread(ref.block_scales(wd, 128), 128, N, d)
        tol = (am * (1 + 2.0 ** -4)) @ (wm * (1 + 2.0 ** -4)).T - np.abs(ad) @ np.abs(wd).T
        whole = ad @ wd.T + (extra[0] if extra else 0.0)
        assert np.all(np.abs(got - whole) <= tol + bound)
