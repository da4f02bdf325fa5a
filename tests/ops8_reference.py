"""Plain 64-bit implementations of the 8-bit operators and of the sampler with parameters per row (numpy; test
infrastructure only), written from their definitions in include/srm.h."""
import numpy as np

E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -100


def e4m3_table():
    """Value of each of the 256 codes of e4m3 (no infinities; 0x7f and 0xff are NaN)."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if (c & 127) == 127 else (-x if c & 128 else x)
    return v


def block_scales(x, block_rows):
    """[ceil(R / block_rows), ceil(K / 128)] scales of a matrix, in 64 bits."""
    R, K = x.shape
    return np.array([[max(np.abs(x[i: i + block_rows, j: j + 128]).max() / E4M3_MAX, LEAST_SCALE) for j in range(0, K, 128)]
                     for i in range(0, R, block_rows)])


def spread(scales, block_rows, R, K):
    return np.repeat(np.repeat(scales, block_rows, 0)[:R], 128, 1)[:, :K]


def rms_norm(h, g, eps):
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * g


def gemm(a, sa, w, sw):
    """a, w: the values of the codes (64 bits); sa [M, kb], sw [ceil(N / 128), kb]."""
    (M, K), N = a.shape, w.shape[0]
    return (a * spread(sa, 1, M, K)) @ (w * spread(sw, 128, N, K)).T


def sample_row(l, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Token of one row; parameters as the kernel gets them (fp32 values), arithmetic in 64 bits. Returns (token, kept ids in
    ascending order, cumulative masses of them over the whole)."""
    l = np.where(np.isnan(l), -np.inf, l).astype(np.float64)
    ids = np.flatnonzero(l > -np.inf)
    if len(ids) == 0:
        return 0, ids, np.zeros(0)
    order = ids[np.lexsort((ids, -l[ids]))]
    top = l[order[0]]
    if not T >= 2.0 ** -100:
        return int(order[0]), order[:1], np.ones(1)
    with np.errstate(invalid="ignore"):
        w = np.where(l[order] == top, 1.0, np.exp((l[order] - top) / T))
    n = len(order) if top_k <= 0 else min(top_k, len(order))
    total = w[:n].sum()
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
        n = max(1, int((before < top_p * total).sum()))
    if min_p > 0:
        n = int((w[:n] >= min(min_p, 1.0)).sum())
    kept = np.sort(order[:n])
    mass = w[:n][np.argsort(order[:n], kind="stable")]
    cdf = np.cumsum(mass)
    u = u if u > 0 else 0.0
    k = int((cdf <= u * cdf[-1]).sum())
    return int(kept[min(k, n - 1)]), kept, cdf / cdf[-1]


def sample_rows(l, u, T, top_k, top_p, min_p):
    """Tokens of many rows at once: torch tensors, 64 bits, every parameter a vector."""
    import torch
    l = l.double()
    l = torch.where(l != l, -float("inf"), l)
    o, ids = torch.sort(l, dim=1, descending=True, stable=True)
    top = o[:, :1]
    w = torch.where(o == top, 1.0, torch.exp((o - top) / T.double()[:, None]))
    rank = torch.arange(l.shape[1], device=l.device)[None]
    k = top_k.long()[:, None]
    kept = ((k <= 0) | (rank < k)) & (o > -float("inf"))
    w = torch.where(kept, w, 0.0)
    before = torch.nn.functional.pad(w.cumsum(1), (1, 0))
    p = top_p.double()[:, None]
    kept &= (p >= 1) | (before[:, :-1] < p * before[:, -1:]) | (rank == 0)
    m = min_p.double().clamp(max=1)[:, None]
    kept &= (m <= 0) | (w >= m)
    mass = torch.zeros_like(w).scatter_(1, ids, torch.where(kept, w, 0.0))
    cdf = mass.cumsum(1)
    tok = torch.minimum((cdf <= u.double()[:, None] * cdf[:, -1:]).sum(1), torch.where(mass > 0, rank, -1).amax(1))
    return torch.where(T >= 2.0 ** -100, tok, ids[:, 0]).int()
