"""Plain definitions in 64 bits of the operators around the index calls, and
builders of their inputs.  Nothing here uses the library."""
import numpy as np
import torch

LATENT, ROPE, BLK = 512, 64, 32
DIM = LATENT + ROPE
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """x rounded to bf16, as float64 numpy."""
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).bfloat16().double().numpy()


def quantise(x):
    """x [n, 512] float64 (bf16 values) -> codes uint8 [n, 256], scales uint8 [n, 16]."""
    n = x.shape[0]
    blocks = x.reshape(n, LATENT // BLK, BLK)
    finite = np.isfinite(blocks).all(-1)
    amax = np.where(finite, np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(-1), 0.0)
    e = np.full(amax.shape, -127, dtype=np.int64)
    pos = amax > 0
    e[pos] = np.ceil(np.log2(amax[pos] / 6.0)).astype(np.int64)
    # log2 may round across a power of two: settle it with exact products
    e = np.where(pos & (amax > 6.0 * np.exp2(e.astype(float))), e + 1, e)
    e = np.where(pos & (amax <= 6.0 * np.exp2(e - 1.0)), e - 1, e)
    e = np.maximum(e, -127)
    m = np.abs(np.where(np.isfinite(blocks), blocks, 0)) / np.exp2(e.astype(float))[..., None]
    # the nearest of the grid, the even code of two equally near
    d = np.abs(m[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    even = np.where((d == near) & (np.arange(8) % 2 == 0), np.arange(8), 99).min(-1)
    code = np.where(even < 99, np.where((d == near).sum(-1) > 1, even, d.argmin(-1)), d.argmin(-1))
    code = code + 8 * (np.signbit(blocks) & np.isfinite(blocks))
    code = np.where(finite[..., None], code, 0).reshape(n, LATENT).astype(np.uint8)
    scales = np.where(finite, e + 127, 255).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales


def values(codes, scales):
    """codes [..., 256], scales [..., 16] -> float64 [..., 512]."""
    signed = np.concatenate([GRID, -GRID])
    v = np.empty(codes.shape[:-1] + (LATENT,))
    v[..., 0::2] = signed[codes & 15]
    v[..., 1::2] = signed[codes >> 4]
    two = np.exp2(scales.astype(np.float64) - 127)
    two = np.where(scales == 255, np.nan, two)
    return v * np.repeat(two, BLK, axis=-1)


def random_cache(rows, rng, spread=0.5):
    x = bf16(rng.standard_normal((rows, LATENT)) * np.exp(spread * rng.standard_normal((1, LATENT))))
    codes, scales = quantise(x)
    return codes, scales, bf16(rng.standard_normal((rows, ROPE)))


def attend_rows(q, latent, rope, scale, allowed):
    """q [h, 576], keys latent [n, 512] / rope [n, 64], allowed [n] bool ->
    out [h, 512], lse [h], weight [n] (summed over heads), bound [h] (scale * max_s sum |q k|),
    spread [h, 512] (sum_s p |latent|)."""
    h = q.shape[0]
    k = np.concatenate([latent, rope], 1)[allowed]
    v = latent[allowed]
    weight = np.zeros(latent.shape[0])
    if k.shape[0] == 0:
        return np.zeros((h, LATENT)), np.full(h, -np.inf), weight, np.zeros(h), np.zeros((h, LATENT))
    with np.errstate(invalid="ignore", over="ignore"):
        z = scale * (q @ k.T)
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(-1, keepdims=True)
        p = p / total
        weight[allowed] = p.sum(0)
        bound = abs(scale) * (np.abs(q) @ np.abs(k).T).max(-1)
        return p @ v, (top + np.log(total))[:, 0], weight, bound, p @ np.abs(v)


def evict(acc, n, keep, sink, recent):
    """Kept positions of one sequence (a list, ascending)."""
    if n <= keep:
        return list(range(n))
    mine = set(range(sink)) | set(range(n - recent, n))
    a = acc[:n].astype(np.float64)
    rank = np.where(np.isnan(a), np.where(np.signbit(a), -np.inf, np.inf), a)
    order = sorted(range(n), key=lambda s: (-(2 if np.isnan(a[s]) and not np.signbit(a[s]) else
                                              -2 if np.isnan(a[s]) else 0), -rank[s], s))
    for s in order:
        if len(mine) >= keep:
            break
        mine.add(s)
    return sorted(mine)


def e4m3_value(code):
    code = np.asarray(code).astype(np.int64)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e > 0, (8 + m) * np.exp2(e - 10.0), m * np.exp2(-9.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code & 128, -v, v)


def e4m3_ulp(v):
    """Spacing of E4M3 values around |v| (the smaller one at a power of two)."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return np.exp2(np.minimum(e, 8) - 3)
