"""GPU tests of the products with 4-bit weights against their definition in 64
bits, at the bound of draft_ref.linear_bound."""
import numpy as np
import pytest
import torch

import draft_ref as plain
import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


def _weights(n, k, rng, spread=1.0):
    x = rng.standard_normal((n, k)) * np.exp(spread * rng.standard_normal((1, k))) / np.sqrt(k)
    return plain.quantise(ref.bf16(x))


def _fp8(x, group):
    """E4M3FN codes and scales of x, and the values they stand for."""
    r, k = x.shape
    g = group or k
    parts = -(-k // g)
    padded = np.zeros((r, parts * g))
    padded[:, :k] = x
    scale = (np.abs(padded.reshape(r, parts, g)).max(-1) / 448).astype(np.float32)
    scale[scale == 0] = 1
    each = np.repeat(scale, g, 1)[:, :k].astype(np.float64)
    codes = torch.from_numpy((x / each).clip(-448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
    return codes, scale, codes.double().numpy() * each


def _inputs(rows, k, kind, rng):
    x = rng.standard_normal((rows, k)) * (1 + 5 * (rng.random((1, k)) > 0.98))
    if kind == "bf16":
        x = ref.bf16(x)
        return torch.from_numpy(x).bfloat16().cuda(), {}, x
    group = 128 if kind == "blocks" else 0
    codes, scale, x = _fp8(x, group)
    return codes.cuda(), dict(x_scale=dev(scale), group=group), x


def _check(got, x, codes, scales, bf16, label):
    y, s = plain.linear(x, codes, scales)
    got = got.double().cpu().numpy().reshape(y.shape)
    tol = plain.linear_bound(x.shape[1], s, y, bf16)
    assert np.all(np.abs(got - y) <= tol), (label, (np.abs(got - y) / tol).max())


SIZES = [
    # rows, n, k
    (1, 1, 32), (1, 5, 64), (2, 17, 96), (1, 16, 128), (3, 33, 160), (15, 40, 256), (16, 100, 512), (17, 64, 544),
    (1, 300, 1024), (2, 1000, 1056), (32, 15, 2048), (33, 31, 2080), (1, 70, 4096), (16, 129, 4128), (26, 203, 5024),
    (4, 50, 8192), (5, 49, 8224), (64, 48, 1024), (64, 130, 6144), (65, 20, 512), (130, 37, 2176), (1, 18, 16416),
    (31, 16, 12320), (1, 9000, 32), (7, 5000, 288), (1100, 40, 128),
]


@pytest.mark.parametrize("rows,n,k", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "row", "blocks"])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_linear4(rows, n, k, kind, out):
    rng = np.random.default_rng(rows * 7 + n + k)
    codes, scales = _weights(n, k, rng)
    x, kw, plain_x = _inputs(rows, k, kind, rng)
    say("linear4", rows, n, k, kind, out)
    y = pv.pivot_linear4(x, dev(codes), dev(scales), dtype=out, **kw)
    assert y.shape == (rows, n) and y.dtype == out
    _check(y, plain_x, codes, scales, out == torch.bfloat16, (rows, n, k, kind))


def test_strides_and_dimensions():
    """Rows of wider tensors on both sides that start anywhere; deeper inputs; what
    lies between the output's rows stays."""
    rng = np.random.default_rng(3)
    n, k = 45, 352
    codes, scales = _weights(n, k, rng)
    wide = torch.from_numpy(rng.standard_normal((9, 777))).bfloat16().cuda()
    out = torch.full((9, 101), 7.0, dtype=torch.float32, device="cuda")
    say("linear4 strided")
    y = pv.pivot_linear4(wide[:, 3:355], dev(codes), dev(scales), dtype=torch.float32, out=out[:, 50:95])
    assert y.data_ptr() == out[:, 50:].data_ptr()
    _check(out[:, 50:95], wide[:, 3:355].double().cpu().numpy(), codes, scales, False, "strided")
    assert (out[:, :50] == 7).all() and (out[:, 95:] == 7).all()
    c8, s8, x8 = _fp8(rng.standard_normal((6, k)), 128)
    big = torch.zeros((6, 400), dtype=torch.uint8, device="cuda")
    big[:, 5:5 + k] = c8.view(torch.uint8).cuda()
    say("linear4 fp8 bytes at odd addresses, bf16 rows at odd places")
    out = torch.zeros((6, 47), dtype=torch.bfloat16, device="cuda")
    pv.pivot_linear4(big[:, 5:5 + k], dev(codes), dev(scales), x_scale=dev(s8), group=128, out=out[:, 1:46])
    _check(out[:, 1:46], x8, codes, scales, True, "bytes")
    x = torch.from_numpy(rng.standard_normal((2, 3, k))).bfloat16().cuda()
    y = pv.pivot_linear4(x, dev(codes), dev(scales))
    assert y.shape == (2, 3, n)
    _check(y, x.double().cpu().numpy().reshape(6, k), codes, scales, True, "deeper")
    y = pv.pivot_linear4(x[0, 0], dev(codes), dev(scales))
    assert y.shape == (n,)
    assert pv.pivot_linear4(x[:0], dev(codes), dev(scales)).shape == (0, 3, n)
    assert pv.pivot_linear4(x, dev(codes[:0]), dev(scales[:0])).shape == (2, 3, 0)


@pytest.mark.parametrize("k,rows", [(160, 3), (4096, 20), (4224, 40)])
def test_special_values(k, rows):
    """A NaN or an infinity of x stays in its row, one of the weights in its column;
    the scales' ends; rows of zeros."""
    rng = np.random.default_rng(k)
    n = 50
    codes, scales = _weights(n, k, rng)
    x = ref.bf16(rng.standard_normal((rows, k)))
    x[1] = 0
    scales[7, 1] = 255        # NaN
    scales[9, :] = 0          # 2^-127
    scales[11, :] = 1
    codes[13] = 0
    codes[14, 3] = (codes[14, 3] & 0xF0) | 7
    scales[14, 0] = 253       # 6 * 2^126: infinite in bf16
    x[rows - 1, k - 1] = np.nan
    codes[:, k // 2 - 1] = codes[:, k // 2 - 1] & 0x0F | 0x20   # times 1
    say("linear4 special", k, rows)
    y = pv.pivot_linear4(torch.from_numpy(x).bfloat16().cuda(), dev(codes), dev(scales), dtype=torch.float32)
    got = host(y).astype(np.float64)
    assert np.isnan(got[rows - 1]).all() and np.isnan(got[:, 7]).all()
    rest = np.setdiff1d(np.arange(n), [7, 14])
    assert np.isfinite(got[:rows - 1][:, rest]).all()
    assert np.all(~np.isfinite(got[0, 14]))
    finite = np.delete(np.arange(rows), rows - 1)
    _check(y[:rows - 1][:, torch.from_numpy(rest).cuda()], x[finite], codes[rest], scales[rest], False, "special")
    assert (got[1, rest] == 0).all()


def test_scale_of_a_row_may_be_anything():
    rng = np.random.default_rng(5)
    codes, scales = _weights(20, 256, rng)
    c8, s8, x8 = _fp8(rng.standard_normal((4, 256)), 128)
    s8[0, 0], s8[1] = np.nan, 0.0
    say("linear4 scales")
    y = host(pv.pivot_linear4(c8.cuda(), dev(codes), dev(scales), x_scale=dev(s8), group=128, dtype=torch.float32))
    assert np.isnan(y[0]).all() and (y[1] == 0).all()
    _check(torch.from_numpy(y[2:]), x8[2:], codes, scales, False, "scales")


@pytest.mark.parametrize("rows", [1, 6, 30, 64])
def test_every_fp8_code(rows):
    """Every code's value, subnormal ones and both zeros among them, as a sum and alone; a
    NaN code makes its row NaN."""
    k = 288
    codes, scales = plain.quantise(np.ones((3, k)))
    x = np.tile((np.arange(k) % 256).astype(np.uint8), (rows, 1))
    x[:, (x[0] & 127) == 127] = 0
    x[rows - 1, k - 1] = 0xFF
    value = ref.e4m3_value(x)
    say("linear4 fp8 codes", rows)
    y = pv.pivot_linear4(dev(x), dev(codes), dev(scales), x_scale=torch.ones((rows, 1), device="cuda"), dtype=torch.float32)
    assert np.isnan(host(y)[rows - 1]).all() and not np.isnan(host(y)[:rows - 1]).any()
    if rows > 1:
        _check(y[:rows - 1], value[:rows - 1], codes, scales, False, "codes")
    eye = np.zeros((256, 256))
    np.fill_diagonal(eye, 1)
    codes, scales = plain.quantise(eye)
    x = np.zeros((rows, 256), np.uint8)
    x[0] = np.arange(256)
    x[0, [127, 255]] = 0
    y = pv.pivot_linear4(dev(x), dev(codes), dev(scales), x_scale=torch.full((rows, 1), 2.0, device="cuda"), dtype=torch.float32)
    assert np.array_equal(host(y)[0], 2 * ref.e4m3_value(x[0]).astype(np.float32))


def test_weights_past_32_bits():
    """4.6 GB of codes: a sum over k cut into eight parts, columns at both ends."""
    n, k = 140001, 65536
    g = torch.Generator(device="cuda").manual_seed(2)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(120, 124, (n, k // 32), generator=g, device="cuda", dtype=torch.uint8)
    x = torch.randn((2, k), generator=g, device="cuda").bfloat16()
    say("linear4 past 32 bits")
    y = pv.pivot_linear4(x, codes, scales, dtype=torch.float32)
    at = torch.tensor([0, 1, 65535, 131071, 131072, 139990, 140000], device="cuda")
    _check(y[:, at], x.double().cpu().numpy(), host(codes[at]), host(scales[at]), False, "far")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,k", [(1, 32), (3, 96), (70, 512), (129, 1056)])
def test_pack(dtype, n, k):
    rng = np.random.default_rng(n + k)
    w = torch.from_numpy(rng.standard_normal((n, k + 5)) * np.exp(4 * rng.standard_normal((n, 1)))).to(dtype)
    w[0, 2:34] = 0
    w[n // 2, 2 + k - 1] = float("inf")
    w[n - 1, 3] = float("nan")
    say("pack", dtype, n, k)
    codes, scales = pv.pivot_linear4_pack(w.cuda()[:, 2:2 + k])
    want = plain.quantise(w[:, 2:2 + k].double().numpy())
    assert np.array_equal(host(scales), want[1])
    assert np.array_equal(plain.values(host(codes), want[1]), plain.values(*want), equal_nan=True)
    assert np.array_equal(host(codes)[want[1].repeat(16, 1) == 255], want[0][want[1].repeat(16, 1) == 255])


def test_pack_extremes():
    """Every power of two of fp32 with both sides of the scale's step, and ties."""
    x = np.zeros((254, 32))
    for e in range(-126, 128):
        m = (1.0, 1.5, np.nextafter(np.float32(1.5), np.float32(2)), 1.99)[e % 4]
        x[e + 126, 0] = m * 2.0 ** e
        x[e + 126, 1:9] = -m * 2.0 ** e * np.array([0.0416015625, 0.125, 0.2083, 0.25, 0.4166, 0.5833, 0.75, 0.91])
    x[-1, 0] = np.finfo(np.float32).max
    x = x.astype(np.float32)
    small = np.float32([1e-45, 3e-39, 7e-38, 2e-38])
    x[:4, 9] = small
    say("pack extremes")
    codes, scales = pv.pivot_linear4_pack(dev(x))
    want = plain.quantise(x.astype(np.float64))
    assert np.array_equal(host(scales), want[1])
    assert np.array_equal(plain.values(host(codes), want[1]), plain.values(*want))


def test_same_bits_on_other_streams_and_in_a_graph():
    """Two streams at once, each with its workspace; a captured call replayed between
    eager ones.  64 rows of 6144: the sum over k is cut, so the workspace is used."""
    rng = np.random.default_rng(9)
    n, k = 700, 6144
    codes, scales = (dev(t) for t in _weights(n, k, rng))
    xs = [torch.from_numpy(rng.standard_normal((64, k))).bfloat16().cuda() for _ in range(2)]
    say("linear4 streams")
    want = [pv.pivot_linear4(x, codes, scales) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(pv.pivot_linear4(x, codes, scales))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    a = pv.pivot_linear4_args()
    x, out = xs[0].clone(), torch.empty((64, n), dtype=torch.bfloat16, device="cuda")
    a.n_rows, a.n, a.k, a.x, a.ld_x, a.codes, a.scales = 64, n, k, 1, k, 1, 1
    a.ld_out = n
    need = pv.lib().pivot_linear4_workspace_size(a)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    say("linear4 graph")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pv.pivot_linear4(x, codes, scales, out=out, ws=ws)
    for i in range(4):
        x.copy_(xs[i % 2])
        out.zero_()
        graph.replay()
        eager = pv.pivot_linear4(xs[1 - i % 2], codes, scales)
        torch.cuda.synchronize()
        assert torch.equal(out, want[i % 2]) and torch.equal(eager, want[1 - i % 2])
