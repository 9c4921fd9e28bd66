"""GPU tests of calls whose rows need more than the 2^32 threads that one launch
counts: the 4-bit cache's write and read, the eviction's moves, the
select, and the encoder."""
import numpy as np
import pytest
import torch

import ops_ref as ref
import paper_2607_24593_amd as pv
from gpu_util import host, say

pytestmark = pytest.mark.gpu

ROWS = (1 << 26) + 3  # a wave a row


@pytest.fixture
def room():
    """At least 140 GB of free device memory, given back afterwards."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 140 << 30:
        pytest.skip("needs 140 GB of device memory")
    yield
    torch.cuda.empty_cache()


def _cache(rows):
    parts = (torch.zeros((rows, 256), dtype=torch.uint8, device="cuda"),
             torch.zeros((rows, 16), dtype=torch.uint8, device="cuda"),
             torch.zeros((rows, 64), dtype=torch.bfloat16, device="cuda"))
    return parts, pv.make_cache4(*parts, pv.make_row_map(seq_stride=rows, rows=rows))


def test_cache_write_of_many_rows(room):
    parts, cache = _cache(ROWS)
    latent = torch.zeros((ROWS, 512), dtype=torch.bfloat16, device="cuda")
    rope = torch.zeros((ROWS, 64), dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 7, 255, 1 << 24, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, ROWS - 1], device="cuda")
    rng = np.random.default_rng(1)
    x, r = ref.bf16(rng.standard_normal((len(some), 512))), ref.bf16(rng.standard_normal((len(some), 64)))
    latent[some], rope[some] = torch.from_numpy(x).bfloat16().cuda(), torch.from_numpy(r).bfloat16().cuda()
    say("cache write of many rows")
    pv.pivot_cache4_write(latent, rope, cache, [0], ROWS)
    codes, scales = ref.quantise(x)
    got = [host(t[some]) for t in parts[:2]]
    assert np.array_equal(got[1], scales)
    assert np.array_equal(ref.values(got[0], got[1]), ref.values(codes, scales))
    assert np.array_equal(parts[2][some].double().cpu().numpy(), r)


def test_cache_read_of_many_rows(room):
    parts, cache = _cache(16)
    rng = np.random.default_rng(2)
    x, r = ref.bf16(rng.standard_normal((16, 512))), ref.bf16(rng.standard_normal((16, 64)))
    pv.pivot_cache4_write(torch.from_numpy(x).bfloat16().cuda(), torch.from_numpy(r).bfloat16().cuda(), cache, [0], 16)
    idx = torch.full((1, ROWS), 3, dtype=torch.int32, device="cuda")
    some = torch.tensor([0, 1 << 25, (1 << 26) - 1, 1 << 26, ROWS - 1], device="cuda")
    idx[0, some] = torch.arange(5, dtype=torch.int32, device="cuda") + 8
    say("cache read of many rows")
    out = pv.pivot_cache4_read(cache, idx)[0]
    want = pv.pivot_cache4_read(cache, torch.arange(16, dtype=torch.int32, device="cuda")[None])[0]
    assert torch.equal(out[some], want[8:13])
    near = torch.tensor([5, (1 << 25) + 1, (1 << 26) + 1], device="cuda")
    assert torch.equal(out[near], want[3].expand(3, -1))


def test_evict_moves_of_many_sequences():
    batch = (1 << 24) + 3
    acc = torch.rand((batch, 2), device="cuda")
    src = torch.arange(2 * batch, dtype=torch.int32, device="cuda")
    dst = torch.zeros(batch, dtype=torch.int32, device="cuda")
    say("evict moves of many sequences")
    kept, out_acc = pv.pivot_evict(acc, [2] * batch, 1, [(src, dst)], pv.make_row_map(seq_stride=2, rows=2 * batch),
                                   pv.make_row_map(seq_stride=1, rows=batch))
    want = (acc[:, 1] > acc[:, 0]).int()
    assert torch.equal(kept[:, 0], want) and torch.equal(out_acc[:, 0], acc.amax(1))
    assert torch.equal(dst, 2 * torch.arange(batch, dtype=torch.int32, device="cuda") + want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_of_many_rows(dtype):
    """2^23 rows and some, 512 threads each."""
    rows, ld, m = (1 << 23) + 9, 24, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    perm = torch.randperm(ld, generator=g, device="cuda")
    scores = (torch.arange(rows, device="cuda")[:, None] * 5 + perm) % ld  # a different order in every row
    select = pv.pivot_topk_rows if dtype == torch.float32 else pv.pivot_topk_rows_bf16
    say("select of many rows", dtype)
    out = select(scores.to(dtype), ld, 0, m)
    want = scores.topk(m, dim=1).indices.int()
    assert torch.equal(out.sort(1).values, want.sort(1).values)


def test_encode_of_many_values(room):
    n = (1 << 34) + 5  # 4 a thread
    x = torch.ones(n, device="cuda")
    say("encode of many values")
    out = pv.pivot_encode_e4m3(x)
    del x
    assert all(bool((out[i:i + (1 << 31)] == 0x38).all()) for i in range(0, n, 1 << 31))  # 1.0
