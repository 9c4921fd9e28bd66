"""GPU tests of the products with 4-bit weights where a workgroup passes many tiles:
the rings in LDS are loaded again, the places of the waves' sums are taken again, and
the counters go on.  Every instance of the kernel that a call can pick runs (rows up
to 16, 32, 64; chunks of k a wave; kinds of rows; scales as words or bytes), and all
columns are compared with the product in 64 bits, at the bound of
draft_ref.linear_bound."""
import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import say

pytestmark = pytest.mark.gpu

CUS, WAVES = 256, 8


def cut(rows, k, blocks):
    """How linear4.hip cuts a call (plan_of): 16-row tiles a workgroup, chunks a wave, waves
    that share k, workgroups that share k, workgroups that may share the tiles."""
    mt = 1 if rows <= 16 else 2 if rows <= 32 else 4
    most = {1: 8, 2: 5, 4: 2 if blocks else 3}[mt]
    chunks = -(-k // 128)
    splits = -(-chunks // (WAVES * most))
    mine = -(-chunks // splits)
    kc = -(-mine // WAVES)
    waves = -(-mine // kc)
    kw = 8 if waves > 4 else 4 if waves > 2 else waves
    return mt, kc, kw, splits, max(1, CUS // (splits * -(-rows // (16 * mt))))


def ring(mt, kc, words):
    """Tiles on their way, places of sums, and how much later a tile is added up (Ring)."""
    sums = 4 if mt == 1 else 3
    tile = 1024 * kc + 256 * (-(-kc // 4) if words else kc)
    fit = (160 * 1024 - 512 - sums * WAVES * mt * 1024) // (WAVES * tile)
    return min(fit, 6), sums, sums - 2


def columns(rows, k, blocks, words):
    """A number of weight rows that is no multiple of 16, of tiles that do not divide by the
    workgroups, for every workgroup more steps than its ring and its sums have places."""
    mt, kc, kw, splits, groups = cut(rows, k, blocks)
    depth, sums, lag = ring(mt, kc, words)
    steps, nw = max(depth, sums) + lag + sums + 2, WAVES // kw
    tiles = steps * nw * groups + groups // 3 + 1
    assert tiles // groups // nw >= steps and tiles % groups
    return 16 * tiles - 5


GRID = torch.from_numpy(np.concatenate([ref.GRID, -ref.GRID]))


def check(y, x, codes, scales, k, bf16, label):
    """y against x w^T, x float64 [rows, k], in pieces of weight rows."""
    grid = GRID.cuda()
    n = codes.shape[0]
    step = max(1, (1 << 27) // k)
    steps = min(k, 1024) / 8 + 8 + k / 2048 + 4   # draft_ref.linear_bound
    for i in range(0, n, step):
        c = codes[i:i + step].long()
        w = torch.stack((grid[c & 15], grid[c >> 4]), -1).view(c.shape[0], k)
        w = w * torch.exp2(scales[i:i + step].double() - 127).repeat_interleave(32, 1)
        want, size = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
        tol = steps * 2.0 ** -23 * size + (2.0 ** -8 if bf16 else 2.0 ** -24) * want.abs() + 1e-37
        off = (y[:, i:i + step].double() - want).abs()
        assert bool((off <= tol).all()), (label, i, (off / tol).max().item())


def operands(rows, n, k, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(117, 125, (n, k // 32), generator=g, device="cuda", dtype=torch.uint8)
    x = torch.randn((rows, k), generator=g, device="cuda")
    if kind == "bf16":
        x = x.bfloat16()
        return x, {}, x.double(), codes, scales
    group = 128 if kind == "blocks" else k
    parts = -(-k // group)
    padded = torch.zeros((rows, parts * group), device="cuda")
    padded[:, :k] = x
    scale = padded.view(rows, parts, group).abs().amax(-1) / 448
    each = scale.repeat_interleave(group, 1)[:, :k]
    c8 = (x / each).clamp(-448, 448).to(torch.float8_e4m3fn)
    kw = dict(x_scale=scale, group=128 if kind == "blocks" else 0)
    return c8, kw, c8.double() * each.double(), codes, scales


def run(rows, k, kind, words, out, label, shift=None, seed=1):
    n = columns(rows, k, kind == "blocks", words)
    x, kw, plain_x, codes, scales = operands(rows, n, k, kind, seed)
    if shift is not None:  # rows that start anywhere are loaded straight into registers
        wide = torch.zeros((rows, k + 24), dtype=x.dtype, device="cuda")
        wide.view(torch.uint8 if kind != "bf16" else torch.bfloat16)[:, shift:shift + k] = \
            x.view(torch.uint8 if kind != "bf16" else torch.bfloat16)
        x = wide[:, shift:shift + k]
    if not words and k % 128 == 0:  # scales that start at an odd address
        backing = torch.empty(scales.numel() + 1, dtype=torch.uint8, device="cuda")
        backing[1:] = scales.view(-1)
        scales = backing[1:].view(scales.shape)
    say("linear4 pipeline", label, rows, n, k, kind, "words" if words else "bytes")
    y = pv.pivot_linear4(x, codes, scales, dtype=out, **kw)
    check(y, plain_x, codes, scales, k, out == torch.bfloat16, (label, rows, k, kind))


INSTANCES = [(mt, kc, kind, words) for mt, most in ((1, 8), (2, 5), (4, 3)) for kc in range(1, most + 1)
             for kind in ("bf16", "row", "blocks") for words in (True, False) if not (mt == 4 and kc == 3 and kind == "blocks")]


@pytest.mark.parametrize("mt,kc,kind,words", INSTANCES)
def test_every_instance_over_many_tiles(mt, kc, kind, words):
    """The last wave's last chunk is beyond k, or partly."""
    rows = {1: 13, 2: 29, 4: 61}[mt]
    k = 1024 * kc - (128 if words else 32)
    assert cut(rows, k, kind == "blocks")[:4] == (mt, kc, 8, 1)
    run(rows, k, kind, words, torch.float32 if kc % 2 else torch.bfloat16, (mt, kc))


@pytest.mark.parametrize("rows,k", [(1, 4096), (16, 2048), (17, 5120), (32, 1024), (33, 2048), (64, 1024), (16, 8192)])
@pytest.mark.parametrize("words", [True, False])
def test_whole_chunks(rows, k, words):
    """k that all waves share evenly; scales that are words, and the same from an odd address."""
    run(rows, k, "bf16", words, torch.bfloat16, "whole")


@pytest.mark.parametrize("rows,k,kw", [(2, 96, 1), (16, 256, 2), (30, 224, 2), (64, 480, 4), (9, 512, 4), (50, 32, 1)])
@pytest.mark.parametrize("kind", ["bf16", "row", "blocks"])
def test_waves_that_take_other_tiles(rows, k, kw, kind):
    """Short k: 1, 2 or 4 waves share a tile, the others take other ones."""
    assert cut(rows, k, kind == "blocks")[2] == kw
    run(rows, k, kind, k % 128 == 0, torch.float32, "short")


@pytest.mark.parametrize("rows,k,splits", [(3, 16416, 3), (16, 8320, 2), (31, 12288, 3), (64, 6144, 2), (100, 4192, 2)])
@pytest.mark.parametrize("kind", ["bf16", "blocks"])
def test_sums_cut_over_workgroups(rows, k, splits, kind):
    if rows > 32 and kind == "blocks":
        splits = -(-(-(-k // 128)) // 16)
    assert cut(rows, k, kind == "blocks")[3] == splits
    run(rows, k, kind, k % 128 == 0, torch.bfloat16, "cut")


@pytest.mark.parametrize("rows,k,kind,shift", [(13, 2048, "bf16", 3), (29, 1952, "row", 5), (61, 1920, "blocks", 1), (64, 2944, "bf16", 7)])
def test_rows_that_start_anywhere(rows, k, kind, shift):
    run(rows, k, kind, k % 128 == 0, torch.float32, "anywhere", shift)


@pytest.mark.parametrize("rows,k", [(2, 4096), (29, 2048), (64, 1920)])
def test_the_same_bits_every_time(rows, k):
    """Waves count each other's sums in, in whatever order they come."""
    n = columns(rows, k, False, True)
    x, kw, _, codes, scales = operands(rows, n, k, "bf16", 3)
    say("linear4 pipeline, same bits", rows, k)
    first = pv.pivot_linear4(x, codes, scales, dtype=torch.float32)
    for _ in range(8):
        assert torch.equal(pv.pivot_linear4(x, codes, scales, dtype=torch.float32), first)
