"""The attention's output bound on the CPU: it holds for weights of two bf16 and
fails for weights of one, so a kernel that lost the low part would not pass."""
import math

import numpy as np

import ops_ref as ref
from ops_edges import cancelling_pairs, out_bound


def test_bound_tells_weights_of_one_bf16_from_two():
    rng = np.random.default_rng(5)
    codes, scales, rope = cancelling_pairs(512, rng)
    latent = ref.values(codes, scales)
    q = np.zeros((1, 576))
    q[0, 512] = 1
    scale = float(np.float32(math.log(1.5)))
    o, _, _, bound, spread = ref.attend_rows(q, latent, rope, scale, np.ones(512, bool))
    assert np.abs(o).max() < 1e-5 * spread.min()
    tol = out_bound(o, spread, 2.0 ** -18 * bound, 512)
    z = scale * (q @ np.concatenate([latent, rope], 1).T)[0]
    e = np.exp(z - z.max())
    one = ref.bf16(e)
    two = one + ref.bf16(e - one)
    off = [np.abs(w @ latent / e.sum() - o) for w in (one, two)]
    assert np.all(off[0] > 4 * tol) and np.all(off[1] <= tol)
