"""The bound that the attention's outputs are held to, and inputs at which it is
sharp.  Nothing here uses the library."""
import numpy as np

import ops_ref as ref


def out_bound(o, spread, E, n):
    """Of outputs o [h, 512] over n keys with spread = sum p |latent|, scores off by
    at most E [h].  A weight is held as two bf16: the high part is off by at most
    2^-8 of it, the low part by 2^-8 of that.  Products are added 16 keys at a time,
    twice (high and low parts), each addition off by at most 2^-23 of the sum of
    magnitudes; exp2, the weights' sum and its reciprocal stay below 2^-21.  The
    output is rounded to bf16."""
    return 2.0 ** -8 * np.abs(o) + (2.0 ** -16 + (n / 8 + 16) * 2.0 ** -23 + 2 * E + 2.0 ** -21)[:, None] * spread


def cancelling_pairs(rows, rng):
    """Cache rows (codes, scales, rope) in pairs: row 2 j has the latent 2 m and the
    position part 0, row 2 j + 1 has -3 m and -1 in the first position value.  A
    query that is 1 there and 0 elsewhere, with scale log 1.5, gives them weights
    of 3 : 2, so that outputs over whole pairs vanish."""
    sign = rng.choice([-1.0, 1.0], (1, ref.LATENT))
    m = rng.choice([0.5, 1.0, 2.0], (rows // 2, ref.LATENT)) * sign
    m[:, ::ref.BLK] = 2.0 * sign[:, ::ref.BLK]  # 2 m and 3 m up to 4 and 6: every block's scale is 1
    x = np.stack((2 * m, -3 * m), 1).reshape(rows, ref.LATENT)
    signed = np.concatenate([ref.GRID, -ref.GRID])
    code = np.abs(np.abs(x)[..., None] - signed[:8]).argmin(-1) + 8 * (x < 0)
    code = code.astype(np.uint8)
    rope = np.zeros((rows, ref.ROPE))
    rope[1::2, 0] = -1
    return code[:, 0::2] | (code[:, 1::2] << 4), np.full((rows, ref.LATENT // ref.BLK), 127, np.uint8), rope
