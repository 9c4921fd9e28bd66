"""GPU tests of the norm with fp8 output near the ends of fp32, against its
definition in 64 bits."""
import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import host, say

pytestmark = pytest.mark.gpu


def _norm_edges(x, w, eps, group, label):
    """Codes and scales of finite rows whose values and scales may be anywhere in
    fp32's range.  A result below 2^-126 is rounded to a multiple of 2^-149, by
    half of that; the scale is at least 2^-149 where a group has a value."""
    say("norm edges", label, x.dtype, group)
    codes, scale, _ = pv.pivot_rmsnorm_fp8(x.cuda(), w.cuda(), eps, group=group)
    h, d = x.double().numpy(), x.shape[-1]
    y = h / np.sqrt((h ** 2).mean(-1, keepdims=True) + eps) * w.double().numpy()
    got, scale = ref.e4m3_value(host(codes)), host(scale).astype(np.float64)
    for g, lo in enumerate(range(0, d, group or d)):
        part, s = y[:, lo:lo + (group or d)], scale[:, g]
        amax = np.abs(part).max(-1)
        want = np.where(amax > 0, np.maximum(amax / 448, 2.0 ** -149), 1.0)
        assert np.all(np.abs(s - want) <= 4e-6 * want + 2.0 ** -149), (label, g, s, want)
        v = np.clip(part / s[:, None], -448, 448)
        off = np.abs(got[:, lo:lo + (group or d)] - v)
        room = ref.e4m3_ulp(v) / 2 + 1e-5 * np.abs(v) + 1.01 * 2.0 ** -150 / s[:, None]
        assert np.all(off <= room), (label, g, np.nanmax(off - room), np.isnan(off).sum())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("dim", [384, 3000, 9000])
def test_norm_of_tiny_and_huge_outputs(dim, group, dtype):
    """Groups (or whole rows) of outputs so small that their scale, or its
    reciprocal, is no normal number, beside normal groups and exact zeros; and
    outputs near the largest numbers."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(dim)
    x = torch.randn((3, dim), generator=g).to(dt)
    x[:, 5::9] = 0
    for size in (1e-35, 1e-36, 1e-37, 1e-38, 1e-40, 2.0 ** -133, 1e35):
        w = (1 + 0.3 * torch.rand(dim, generator=g)) * size
        if group:
            w[:128] = 1
        _norm_edges(x, w.to(dt), 1e-6, group, f"weights {size}")
    if dtype == "fp32":
        for size in (1e-42, 2.0 ** -149):
            w = torch.full((dim,), size)
            if group:
                w[:128] = 1
            _norm_edges(x, w, 1e-6, group, f"weights {size}")
    # the product of input and weight leaves fp32's range, the output does not
    for std, size in ((1e12, 1e30), (1e-10, 1e-30)):
        _norm_edges((x.float() * std).to(dt), ((1 + 0.3 * torch.rand(dim, generator=g)) * size).to(dt), 0.0, group,
                    f"rows {std} weights {size}")


def test_norm_of_more_rows_than_one_launch_holds():
    """2^24 rows and some: 2^32 threads are more than a launch takes."""
    rows, dim = (1 << 24) + 5, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, dim), generator=g, device="cuda").bfloat16()
    w = torch.ones(dim, dtype=torch.bfloat16, device="cuda")
    say("norm of many rows")
    codes, scale, h = pv.pivot_rmsnorm_fp8(x, w, 1e-6, residual=x)
    assert torch.equal(h, x + x)  # twice a bf16 value is one
    some = torch.cat([torch.arange(i, min(i + 64, rows), device="cuda")
                      for i in (0, (1 << 21) - 32, (1 << 22) - 32, (1 << 23) + 1, rows - 64)])
    for got, want in zip((codes, scale), pv.pivot_rmsnorm_fp8(x[some], w, 1e-6, residual=x[some])):
        assert torch.equal(got[some], want)
    y = 2 * x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)
    want = y.abs().amax(-1, keepdim=True) / 448
    assert bool(((scale - want).abs() <= 4e-6 * want).all())


@pytest.mark.parametrize("rows", [1, 5])
def test_norm_in_place(rows):
    """The sums in place of x or of the residual, of rows that are not padded (or of one row)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    wide = torch.randn((rows, 700), generator=g, device="cuda").bfloat16()
    w = torch.ones(300, dtype=torch.bfloat16, device="cuda")
    x, r = (torch.randn((rows, 300), generator=g, device="cuda").bfloat16() for _ in range(2))
    for a, b, first in ((x, r, True), (x, r, False), (x, wide[:, :300], True), (wide[:, 9:309], r, False)):
        want = pv.pivot_rmsnorm_fp8(a, w, 1e-6, residual=b)
        a, b = (a.clone(), b) if first else (a, b.clone())
        say("norm in place", rows)
        got = pv.pivot_rmsnorm_fp8(a, w, 1e-6, residual=b, residual_out=a if first else b)
        assert got[2] is (a if first else b) and all(torch.equal(s, t) for s, t in zip(got, want))
