"""The 8-bit tail of a decode step, as cases that can be timed and compared: RMS norm into 8 bits, quantisation by
blocks of 128, the 8-bit product with block scales, and sampling with each row's own parameters.

With `own` false every operator is computed in its plain form (elementary torch operations); with `own` true through
the public calls of `paper_2605_08696_b200`. Sizes are those of the repository's configurations (widths 512, 1024 and
1536, hidden widths four times that, vocabularies of 8000 and 32000, batches from a single sample to a rollout's
16384) and what lies around and between them.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -100
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # one interactive sample: the norm in front of a projection, nothing but latency
        dict(name="norm_token", op="norm", rows=1, d=1024, x="fp32", delta="bf16"),
        # a rollout batch whose size is no multiple of anything
        dict(name="norm_rollout_16001", op="norm", rows=16001, d=1536, x="fp32", delta="bf16"),
        # hidden activations of a serving batch on their way into the down projection
        dict(name="quant_hidden_500", op="quant", rows=500, k=4096, x="bf16", block_rows=1),
        # the LM head of the rollout model, once per weight update
        dict(name="quant_lm_head", op="quant", rows=32000, k=1536, x="bf16", block_rows=128),
        # logits of one sample
        dict(name="lm_head_token", op="gemm", m=1, n=32000, k=1024, out="fp32"),
        # a handful of conversations, down projection: few tiles, a long sum
        dict(name="down_27", op="gemm", m=27, n=1024, k=4096, out="bf16"),
        # a mid-sized batch, up projection of the rollout model
        dict(name="up_777", op="gemm", m=777, n=6144, k=1536, out="bf16"),
        # the throughput benchmark's logits
        dict(name="lm_head_4096", op="gemm", m=4096, n=32000, k=1024, out="fp32"),
        # the rollout batch's up projection
        dict(name="up_16384", op="gemm", m=16384, n=6144, k=1536, out="bf16"),
        # one sample of a large vocabulary
        dict(name="sample_token", op="sample", rows=1, vocab=131072, logits="fp32"),
        # a serving batch of the small configuration, requests with their own parameters
        dict(name="sample_serving_250", op="sample", rows=250, vocab=8000, logits="bf16"),
        # the throughput benchmark's batch
        dict(name="sample_4096", op="sample", rows=4096, vocab=32000, logits="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "quant", "gemm", "gemm", "sample", "sample"))
    if op == "norm":
        d = 16 * _log(rng, 4, 512)
        return dict(op=op, rows=_log(rng, 1, min(20000, 16001 * 1536 // d)), d=d, x=rng.choice(("fp32", "fp32", "bf16", "fp16")),
                    delta=rng.choice(("none", "fp32", "bf16")))
    if op == "quant":
        k = 16 * _log(rng, 4, 512)
        return dict(op=op, rows=_log(rng, 1, min(32000, 32000 * 1536 // k)), k=k, x=rng.choice(("fp32", "bf16", "fp16")) if k <= 768 else "bf16",
                    block_rows=rng.choice((1, 128)))
    if op == "gemm":
        n, k = _log(rng, 100, 32000), 16 * _log(rng, 8, 400)
        m = _log(rng, 1, min(16384, 4096 * 32000 * 1024 // (n * k), 4096 * 32000 // n))
        return dict(op=op, m=m, n=n, k=k, out=rng.choice(("fp32", "bf16")))
    v = _log(rng, 1000, 131072)
    return dict(op=op, rows=_log(rng, 1, min(8192, 4096 * 32000 // v)), vocab=v, logits=rng.choice(("fp32", "fp32", "bf16")))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _blocks(n):
    return -(-n // 128)


def _quantised(x, block_rows):
    """e4m3 values and block scales of a matrix, for inputs (scales stored block after block)."""
    q, s = _plain_quant(x, block_rows)
    return q, s.t().contiguous().t()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*size, std=1.0):
        return torch.randn(*size, generator=g, device="cuda").mul_(std)

    def uniform(*size):
        return torch.rand(*size, generator=g, device="cuda")

    op = case["op"]
    s = dict(op=op)
    if op == "norm":
        R, d = case["rows"], case["d"]
        # a residual stream: channels of different size, a few of them large
        size = torch.exp(normal(d, std=0.5)) * torch.where(uniform(d) < 0.01, 12.0, 1.0)
        s["x"] = (normal(R, d) * size).to(TYPES[case["x"]])
        s["delta"] = None if case["delta"] == "none" else normal(R, d, std=0.3).to(TYPES[case["delta"]])
        s["g"] = 1.0 + normal(d, std=0.1)
        s["eps"] = 1e-5
        s["h"] = torch.empty_like(s["x"]) if s["delta"] is not None else None
        s["q"] = torch.empty(R, d, dtype=torch.float8_e4m3fn, device="cuda")
        s["scales"] = torch.empty(_blocks(d), R, device="cuda").t()
    elif op == "quant":
        R, K, br = case["rows"], case["k"], case["block_rows"]
        s["x"] = (normal(R, K) * torch.exp(normal(R, 1, std=0.5))).to(TYPES[case["x"]])
        s["block_rows"] = br
        s["q"] = torch.empty(R, K, dtype=torch.float8_e4m3fn, device="cuda")
        s["scales"] = torch.empty(_blocks(K), -(-R // br), device="cuda").t()
    elif op == "gemm":
        M, N, K = case["m"], case["n"], case["k"]
        a = normal(M, K) * torch.where(uniform(K) < 0.01, 8.0, 1.0)
        s["a"], s["a_scales"] = _quantised(a, 1)
        s["w"], s["w_scales"] = _quantised(normal(N, K, std=0.02), 128)
        s["out"] = torch.empty(M, N, dtype=TYPES[case["out"]], device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        # rows from confident to undecided: a broad floor, and a few tokens that stand out of it by a row's own amount
        logits = normal(R, V, std=1.5)
        for _ in range(6):
            at = torch.randint(0, V, (R, 1), generator=g, device="cuda")
            logits.scatter_(1, at, 4.0 + 10.0 * uniform(R, 1))
        s["logits"] = logits.to(TYPES[case["logits"]])

        def pick(values):
            at = torch.randint(0, len(values), (R,), generator=g, device="cuda")
            return torch.tensor(values, device="cuda")[at]

        # requests of several kinds side by side; 0, 1 and 0 leave top-k, top-p and min-p without effect
        s["temperature"] = pick([0.6, 0.7, 0.8, 1.0])
        s["top_k"] = pick([0, 0, 20, 50, 100]).to(torch.int32)
        s["top_p"] = pick([0.8, 0.9, 0.9, 0.95, 1.0])
        s["min_p"] = pick([0.0, 0.0, 0.02, 0.1])
        s["u"] = uniform(R)
        s["tokens"] = torch.empty(R, dtype=torch.int32, device="cuda")
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _spread(scales, block_rows, rows, cols):
    """A scale for every element of a rows x cols matrix."""
    s = scales.repeat_interleave(128, 1)[:, :cols]
    return s if block_rows == 1 else s.repeat_interleave(block_rows, 0)[:rows]


def _plain_quant(x, block_rows):
    R, K = x.shape
    rb, kb = -(-R // block_rows), _blocks(K)
    x = x.float()
    padded = torch.zeros(rb * block_rows, kb * 128, device=x.device)
    padded[:R, :K] = x
    amax = padded.view(rb, block_rows, kb, 128).abs().amax((1, 3))
    scales = (amax / E4M3_MAX).clamp(min=LEAST_SCALE)
    q = (x / _spread(scales, block_rows, R, K)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q, scales


def _plain_norm(s):
    h = s["x"] if s["delta"] is None else (s["x"].float() + s["delta"].float()).to(s["x"].dtype)
    f = h.float()
    y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + s["eps"]) * s["g"]
    q, scales = _plain_quant(y, 1)
    return [q, scales] if s["delta"] is None else [q, scales, h]


def _plain_gemm(s):
    (M, K), N = s["a"].shape, s["w"].shape[0]
    a = s["a"].float() * _spread(s["a_scales"], 1, M, K)
    w = s["w"].float() * _spread(s["w_scales"], 128, N, K)
    return (a @ w.t()).to(s["out"].dtype)


def _plain_sample(s):
    # in 64 bits: which token a random number falls on is decided at borders between sums of thousands of weights
    logits = s["logits"].double()
    R, V = logits.shape
    ordered, ids = torch.sort(logits, dim=1, descending=True, stable=True)      # equal logits: lowest id first
    w = torch.exp((ordered - ordered[:, :1]) / s["temperature"].double()[:, None])
    rank = torch.arange(V, device=w.device)[None]
    k = s["top_k"].long()[:, None]
    kept = (k <= 0) | (rank < k)
    w = torch.where(kept, w, 0.0)
    before = torch.nn.functional.pad(w.cumsum(1), (1, 0))
    p = s["top_p"].double()[:, None]
    kept &= (p >= 1) | (before[:, :-1] < p * before[:, -1:]) | (rank == 0)
    kept &= w >= s["min_p"].double()[:, None]
    cdf = torch.zeros_like(w).scatter_(1, ids, torch.where(kept, w, 0.0)).cumsum(1)
    target = s["u"].double()[:, None] * cdf[:, -1:]
    return (cdf <= target).sum(1).to(torch.int32)


def run(state):
    s = state
    if own:
        import paper_2605_08696_b200 as srm
        if s["op"] == "norm":
            srm.k_rms_norm_fp8(s["x"], s["g"], s["q"], s["scales"], delta=s["delta"], sum_out=s["h"], eps=s["eps"])
            return [s["q"], s["scales"]] if s["delta"] is None else [s["q"], s["scales"], s["h"]]
        if s["op"] == "quant":
            srm.k_quant_fp8(s["x"], s["q"], s["scales"], block_rows=s["block_rows"])
            return [s["q"], s["scales"]]
        if s["op"] == "gemm":
            srm.k_gemm_fp8(s["a"], s["a_scales"], s["w"], s["w_scales"], s["out"])
            return s["out"]
        srm.k_sample(s["logits"], s["u"], s["tokens"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                     min_p=s["min_p"])
        return s["tokens"]
    if s["op"] == "norm":
        return _plain_norm(s)
    if s["op"] == "quant":
        return list(_plain_quant(s["x"], s["block_rows"]))
    return _plain_gemm(s) if s["op"] == "gemm" else _plain_sample(s)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_quotients(y, block_rows):
    """Largest magnitudes over 448 of blocks of block_rows x 128, and every element over its block's."""
    R, K = y.shape
    rb, kb = -(-R // block_rows), _blocks(K)
    rows = torch.arange(R, device=y.device) // block_rows
    cols = torch.arange(K, device=y.device) // 128
    by_cols = torch.stack([y[:, 128 * j: 128 * j + 128].abs().amax(1) for j in range(kb)], 1)
    scales = torch.zeros(rb, kb, dtype=torch.float64, device=y.device).index_reduce_(0, rows, by_cols, "amax")
    scales = (scales / 448).clamp(min=2.0 ** -100)
    return y / scales[rows][:, cols], scales


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "norm":
        h = s["x"].double()
        if s["delta"] is not None:
            h = h + s["delta"].double()
        stored = h.to(s["x"].dtype).double()              # the norm is that of the stored sum
        y = stored / ((stored ** 2).sum(1, keepdim=True) / h.shape[1] + s["eps"]).sqrt() * s["g"].double()
        q, scales = _exact_quotients(y, 1)
        return [q, scales] if s["delta"] is None else [q, scales, h]
    if s["op"] == "quant":
        return list(_exact_quotients(s["x"].double(), s["block_rows"]))
    if s["op"] == "gemm":
        M, K = s["a"].shape
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        rows = torch.arange(s["w"].shape[0], device="cuda") // 128
        for b in range(_blocks(K)):
            a = s["a"][:, 128 * b: 128 * b + 128].double() * s["a_scales"][:, b: b + 1].double()
            w = s["w"][:, 128 * b: 128 * b + 128].double() * s["w_scales"][rows, b, None].double()
            out.addmm_(a, w.t())
        return out
    return None           # token ids: whole numbers, no rounding to measure


def work(case):
    op = case["op"]
    if op == "norm":
        R, d = case["rows"], case["d"]
        per = BYTES[case["x"]] + 1 + (0 if case["delta"] == "none" else BYTES[case["x"]] + BYTES[case["delta"]])
        return {"bytes": R * d * per + 4 * R * _blocks(d) + 4 * d, "flops": 8 * R * d}
    if op == "quant":
        R, K = case["rows"], case["k"]
        return {"bytes": R * K * (BYTES[case["x"]] + 1) + 4 * -(-R // case["block_rows"]) * _blocks(K), "flops": 3 * R * K}
    if op == "gemm":
        M, N, K = case["m"], case["n"], case["k"]
        scales = 4 * _blocks(K) * (M + _blocks(N))
        return {"bytes": M * K + N * K + scales + BYTES[case["out"]] * M * N, "flops": 2 * M * N * K}
    R, V = case["rows"], case["vocab"]
    return {"bytes": R * V * BYTES[case["logits"]] + 24 * R, "flops": 4 * R * V}
