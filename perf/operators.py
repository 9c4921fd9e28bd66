"""What is measured of the operators around the index calls: the norm that makes
the fp8 rows, the 4-bit latent cache that is written and read, the attention
over that cache (over index sets or the whole prefix), and the eviction by the
attention's accumulated weights.

`run` computes them in their plain form, from elementary torch operations in 32
bits, or, with `own` set, through the entry points of paper_2607_24593_amd.

A cached token is a row of 512 latent values in 4 bits (OCP MXFP4: E2M1 codes,
the even value in the low nibble, and one power-of-two scale per 32 values) and
64 position values in bf16.  All heads of a query attend to the same rows; the
values are the latent part of the keys.
"""
import math

import numpy as np
import torch

own = False

LATENT, ROPE = 512, 64
DIM = LATENT + ROPE
BLOCK = 32
ROW_BYTES = LATENT // 2 + LATENT // BLOCK + 2 * ROPE  # 400
KEY_BYTES = 128 + 4                                    # an fp8 indexer key and its scale
SCALE = 1.0 / math.sqrt(DIM)
EPS = 1e-6
SHARED = 8  # neighbouring queries whose sets overlap


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one token's hidden state in a decode step: launches and latency
        dict(name="norm-1x4096-bf16", op="norm", rows=1, dim=4096, dtype="bf16", group=0),
        # a decode batch with drafts, an odd width, scales per block of 128
        dict(name="norm-260x5003-bf16-blocks", op="norm", rows=260, dim=5003, dtype="bf16", group=128),
        # a prefill chunk with the residual stream held in fp32
        dict(name="norm-8192x6144-fp32", op="norm", rows=8192, dim=6144, dtype="fp32", group=0),
        # one new token of each of 32 requests into a paged cache
        dict(name="cache-32x1-paged", op="cache", batch=32, shortest=4001, longest=32768, n_q=1, page=64),
        # an 8192-token prompt chunk into a contiguous cache
        dict(name="cache-1x8192", op="cache", batch=1, shortest=40000, longest=40000, n_q=8192, page=0),
        # a chat user's decode step with one draft over the 2048 keys that the index call chose
        dict(name="attend-1x6k-sparse", op="attend", heads=128, batch=1, shortest=6001, longest=6001, n_q=2, topk=2048,
             page=0, acc=False),
        # a full decode batch of long contexts (decode-32x128k-fp8), its sets' weights accumulated
        dict(name="attend-32x128k-sparse-acc", op="attend", heads=128, batch=32, shortest=131072, longest=131072, n_q=2,
             topk=2048, page=0, acc=True),
        # a prompt chunk of 1003 queries, each with a set of its own
        dict(name="attend-prefill-1003-sparse", op="attend", heads=128, batch=1, shortest=32768, longest=32768,
             n_q=1003, topk=2048, page=0, acc=False),
        # ragged decode over whole prefixes in a paged pool: one of eight shards of 128 heads, weights accumulated
        dict(name="attend-8-ragged-dense-acc", op="attend", heads=16, batch=8, shortest=9001, longest=40000, n_q=1,
             topk=0, page=64, acc=True),
        # one long context read whole by all heads and a draft
        dict(name="attend-1x128k-dense", op="attend", heads=128, batch=1, shortest=131072, longest=131072, n_q=2,
             topk=0, page=0, acc=False),
        # one request over its budget: 20000 tokens down to 8192
        dict(name="evict-1x20k", op="evict", batch=1, shortest=20000, longest=20000, keep=8192, page=0),
        # a batch of ragged requests in a paged pool, cut to 4096 tokens each
        dict(name="evict-32-ragged-paged", op="evict", batch=32, shortest=3000, longest=32768, keep=4096, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "cache", "attend", "attend", "attend", "evict"])
    if op == "norm":
        dim = rng.choice([_log(rng, 256, 8192), 128 * rng.randint(2, 64)])
        rows = min(_log(rng, 1, 16384), 8192 * 6144 // dim)
        return dict(op=op, rows=rows, dim=dim, dtype=rng.choice(["bf16", "bf16", "fp32"]), group=rng.choice([0, 0, 128]))
    batch = _log(rng, 1, 48)
    longest = min(_log(rng, 500, 131072), (3 << 20) // batch)
    shortest = rng.choice([longest, max(200, longest // rng.randint(2, 12))])
    shortest = min(shortest, longest)
    page = rng.choice([0, 0, 16, 64, 256])
    if op == "cache":
        n_q = min(_log(rng, 1, 8192), shortest, max(1, 8192 // batch))
        return dict(op=op, batch=batch, shortest=shortest, longest=longest, n_q=n_q, page=page)
    if op == "evict":
        batch = min(batch, 32)
        return dict(op=op, batch=batch, shortest=shortest, longest=longest, keep=_log(rng, 100, min(longest, 8192)),
                    page=page)
    heads = rng.choice([8, 16, 16, 32, 64, 128, 128, rng.randint(1, 128)])
    acc = rng.choice([False, False, True])
    if rng.random() < 0.5:  # over index sets
        topk = rng.choice([512, 1024, 2048, 2048, _log(rng, 100, 2048)])
        n_q = rng.choice([1, 2, 2, 4, _log(rng, 5, 1500)])
        n_q = max(1, min(n_q, shortest, int(2.4e8 / (batch * heads * topk)), int(2.0e6 / (batch * topk))))
    else:
        topk = 0
        n_q = rng.choice([1, 1, 2, 3, 4])
        longest = max(200, min(longest, int(3.0e7 / (batch * heads * n_q)), (1 << 20) // batch))
        shortest = max(100, min(shortest, longest))
    return dict(op=op, heads=heads, batch=batch, shortest=shortest, longest=longest, n_q=n_q, topk=topk, page=page,
                acc=acc)


def _lengths(c):
    """Cached tokens of each request, from the shortest to the longest."""
    b, lo, hi = c["batch"], c["shortest"], c["longest"]
    return [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]


def work(c):
    if c["op"] == "norm":
        n = c["rows"] * c["dim"]
        e = 2 if c["dtype"] == "bf16" else 4
        groups = -(-c["dim"] // c["group"]) if c["group"] else 1
        return {"bytes": n * (3 * e + 1) + c["dim"] * e + c["rows"] * groups * 4, "flops": 8 * n}
    lens = _lengths(c)
    if c["op"] == "cache":  # written, then read back
        n = c["batch"] * c["n_q"]
        return {"bytes": n * (2 * 2 * DIM + 4), "flops": n * LATENT * 4}
    if c["op"] == "evict":
        kept = sum(min(n, c["keep"]) for n in lens)
        return {"bytes": 4 * sum(lens) + kept * (ROW_BYTES + 2 * KEY_BYTES + 2 * DIM + 8), "flops": sum(lens)}
    rows = c["batch"] * c["n_q"]
    io = rows * c["heads"] * (2 * DIM + 2 * LATENT + 4)
    if c["topk"]:
        # a group of neighbouring queries: its first set, and about a quarter of each further one
        pairs = sum(min(c["topk"], n - c["n_q"] + i + 1) for n in lens for i in range(c["n_q"]))
        groups, last = divmod(c["n_q"], SHARED)
        new = groups * (1 + 0.25 * (SHARED - 1)) + (1 + 0.25 * (last - 1) if last else 0)
        read = sum(min(n, int(c["topk"] * new)) for n in lens)
        io += 4 * rows * c["topk"] + (8 * read if c["acc"] else 0)
    else:
        pairs = sum(n - c["n_q"] + i + 1 for n in lens for i in range(c["n_q"]))
        read = sum(lens)
        io += 4 * read if c["acc"] else 0
    return {"bytes": io + read * ROW_BYTES, "flops": 2.0 * (DIM + LATENT) * pairs * c["heads"]}


# ------------------------------------------------------------------ the cache's numbers, in plain operations
def _quantise(x):
    """x [n, 512] -> codes uint8 [n, 256], scales uint8 [n, 16]."""
    v = x.float().reshape(-1, LATENT // BLOCK, BLOCK)
    amax = v.abs().amax(-1)
    mant, e = torch.frexp(amax)                   # amax = mant 2^e, mant in [1/2, 1)
    e = e - 3 + (mant > 0.75).int()               # smallest power of two with amax / 2^e <= 6
    e = torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    inv = ((127 - e).clamp(1, 254) << 23).view(torch.float32)
    m = v.abs() * inv.unsqueeze(-1)
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int()
            + (m >= 3.5).int() + (m > 5.0).int())
    code = (code + 8 * (v < 0).int()).reshape(-1, LATENT // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales, table):
    """codes [..., 256], scales [..., 16] -> fp32 [..., 512]."""
    both = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1)
    two = torch.where(scales == 0, torch.full((), 2.0 ** -127, device=codes.device),
                      (scales.int() << 23).view(torch.float32))
    lead = codes.shape[:-1]
    return (both.reshape(*lead, LATENT // BLOCK, BLOCK) * two.unsqueeze(-1)).reshape(*lead, LATENT)


# ------------------------------------------------------------------ inputs
def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std


def _pool(c, g, spare=0):
    """Rows of a cache for every request (contiguous, or pages of a pool in a
    random order, with `spare` rows a request on pages of their own)."""
    lens, b, page = _lengths(c), c["batch"], c["page"]
    per = max(lens) + 1
    if page:
        need, extra = -(-max(lens) // page), -(-spare // page)
        order = torch.randperm(b * (need + extra) + 3, generator=g, device="cuda").int()
        return (b * (need + extra) + 3) * page, order[:b * need].reshape(b, need).contiguous(), \
            order[b * need:b * (need + extra)].reshape(b, extra).contiguous()
    return b * per, None, None


def _cache(rows, g):
    codes = torch.empty((rows, LATENT // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, LATENT // BLOCK), dtype=torch.uint8, device="cuda")
    step = 1 << 18
    for r in range(0, rows, step):
        n = min(step, rows - r)
        # a latent's channels differ in size
        x = _normal((n, LATENT), g) * torch.exp(0.5 * _normal((1, LATENT), g))
        codes[r:r + n], scales[r:r + n] = _quantise(x)
    return codes, scales, _normal((rows, ROPE), g).bfloat16()


def _sets(c, lens, g):
    """Index sets of every query: the top of scores that neighbours mostly share."""
    out = []
    for n in lens:
        m, k = c["n_q"], c["topk"]
        if m == 1:
            score = _normal((1, n), g)
        else:
            score = torch.repeat_interleave(_normal((-(-m // SHARED), n), g), SHARED, 0)[:m] + 0.4 * _normal((m, n), g)
        pos = torch.arange(n - m, n, device="cuda")
        score.masked_fill_(torch.arange(n, device="cuda") > pos[:, None], -math.inf)
        top, idx = torch.topk(score, min(k, n), sorted=False)
        idx = idx.int().masked_fill(top == -math.inf, -1)
        idx = torch.cat((idx, idx.new_full((m, k - idx.shape[1]), -1)), 1)
        # short rows keep their padding at the end
        out.append(torch.gather(idx, 1, (idx < 0).int().sort(dim=1, stable=True).indices))
    return torch.stack(out).contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 2654435761 % (1 << 62) + 17)
    st = dict(c)
    if c["op"] == "norm":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        x = _normal((c["rows"], c["dim"]), g, 0.5)
        # a few channels of a residual stream are much larger than the others
        st["residual"] = (_normal((c["rows"], c["dim"]), g) * (1 + 20 * (_normal((1, c["dim"]), g) > 2.6))).to(dt)
        st["x"] = x.to(dt)
        st["weight"] = (1 + 0.2 * _normal((c["dim"],), g)).to(dt)
        return st
    lens = _lengths(c)
    st["lens"] = lens
    st["pos0"] = [n - c.get("n_q", 1) for n in lens]
    st["len_dev"] = torch.tensor(lens, dtype=torch.int64, device="cuda")
    st["table"] = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    rows, table, spare = _pool(c, g, c.get("keep", 0) if c["op"] == "evict" else 0)
    st["stride"] = rows // c["batch"] if table is None else 0
    st["pages"] = table
    if c["op"] == "cache":
        st["cache"] = (torch.zeros((rows, LATENT // 2), dtype=torch.uint8, device="cuda"),
                       torch.zeros((rows, LATENT // BLOCK), dtype=torch.uint8, device="cuda"),
                       torch.zeros((rows, ROPE), dtype=torch.bfloat16, device="cuda"))
        n = c["batch"] * c["n_q"]
        st["latent"] = (_normal((n, LATENT), g) * torch.exp(0.5 * _normal((1, LATENT), g))).bfloat16()
        st["rope"] = _normal((n, ROPE), g).bfloat16()
        st["idx"] = (torch.tensor(st["pos0"], device="cuda")[:, None]
                     + torch.arange(c["n_q"], device="cuda")).int().contiguous()
        return st
    st["cache"] = _cache(rows, g)
    if c["op"] == "evict":
        m = c["keep"]
        st["sink"], st["recent"] = min(4, m // 4), m // 8
        st["acc"] = torch.exp(2 * _normal((c["batch"], max(lens)), g))
        st["keys"] = torch.randint(0, 127, (rows, 128), generator=g, device="cuda").to(torch.uint8)
        st["key_scale"] = torch.exp(_normal((rows,), g))
        if table is None:  # contiguous requests move to a cache of their own
            st["to"] = tuple(torch.zeros((c["batch"] * m,) + t.shape[1:], dtype=t.dtype, device="cuda")
                             for t in st["cache"] + (st["keys"], st["key_scale"]))
        else:              # paged ones to fresh pages of the same pool
            st["to"] = st["cache"] + (st["keys"], st["key_scale"])
        st["to_pages"] = spare
        kept = torch.tensor([min(n, m) for n in lens], device="cuda")
        slot = torch.arange(m, device="cuda")
        st["slots"] = torch.where(slot < kept[:, None], slot, -1).int().contiguous()
        return st
    st["q"] = (_normal((c["batch"], c["n_q"], c["heads"], DIM), g, 2.0)).bfloat16()
    st["idx"] = _sets(c, lens, g) if c["topk"] else None
    st["acc"] = torch.zeros((c["batch"], max(lens)), device="cuda") if c["acc"] else None
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return {"norm": _norm, "cache": _write_read, "attend": _attend, "evict": _evict}[st["op"]](st)


def _lib():
    import paper_2607_24593_amd as pv
    return pv


def _map(st, batch_rows, pages):
    pv = _lib()
    if pages is not None:
        return pv.make_row_map(block_table=pages, page_size=st["page"], rows=st["cache"][0].shape[0])
    return pv.make_row_map(seq_stride=batch_rows, rows=batch_rows * st["batch"])


def _norm(st):
    if own:
        codes, scale, h = _lib().pivot_rmsnorm_fp8(st["x"], st["weight"], EPS, residual=st["residual"],
                                                   group=st["group"])
        return codes.view(torch.float8_e4m3fn), scale, h
    h = st["x"].float() + st["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * st["weight"].float()
    rows, dim = y.shape
    group = st["group"] or dim
    n = -(-dim // group)
    yg = torch.nn.functional.pad(y, (0, n * group - dim)).reshape(rows, n, group)
    amax = yg.abs().amax(-1)
    scale = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
    codes = (yg / scale.unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn).reshape(rows, n * group)[:, :dim]
    return codes, scale, h.to(st["x"].dtype)


def _rows(st, pos, pages, stride):
    """Cache rows of positions pos [B, n] (negative ones count as 0)."""
    pos = pos.clamp(min=0).long()
    if pages is None:
        return torch.arange(pos.shape[0], device=pos.device)[:, None] * stride + pos
    return torch.gather(pages.long(), 1, pos // st["page"]) * st["page"] + pos % st["page"]


def _read(st, cache, pos, pages, stride):
    row = _rows(st, pos, pages, stride)
    got = torch.cat((_values(cache[0][row], cache[1][row], st["table"]), cache[2][row].float()), -1)
    return torch.where((pos >= 0).unsqueeze(-1), got, torch.zeros((), device=pos.device)).bfloat16()


def _write_read(st):
    if own:
        pv = _lib()
        cache = pv.make_cache4(*st["cache"], _map(st, st["stride"], st["pages"]))
        pv.pivot_cache4_write(st["latent"], st["rope"], cache, st["pos0"], st["n_q"])
        return pv.pivot_cache4_read(cache, st["idx"])
    codes, scales = _quantise(st["latent"])
    row = _rows(st, st["idx"], st["pages"], st["stride"]).reshape(-1)
    for to, new in zip(st["cache"], (codes, scales, st["rope"])):
        to[row] = new
    return _read(st, st["cache"], st["idx"], st["pages"], st["stride"])


def _attend(st):
    acc = st["acc"]
    if acc is not None:
        acc.zero_()  # the window of queries whose weights count begins here
    if own:
        pv = _lib()
        cache = pv.make_cache4(*st["cache"], _map(st, st["stride"], st["pages"]))
        out, lse = pv.pivot_cache4_attend(st["q"], cache, st["pos0"], st["lens"], SCALE, idx=st["idx"], acc=acc)
        return (out, lse) if acc is None else (out, lse, acc)
    b, m, heads = st["q"].shape[:3]
    at = st["len_dev"][:, None] - m + torch.arange(m, device="cuda")          # [B, m] positions
    q = st["q"].float()
    if st["idx"] is not None:
        k = st["topk"]
        pos = st["idx"].reshape(b, m * k)
        row = _rows(st, pos, st["pages"], st["stride"]).reshape(b, m, k)
        seen = ((st["idx"] >= 0) & (st["idx"] <= at.unsqueeze(-1))).unsqueeze(2)  # [B, m, 1, k]
    else:
        k = max(st["lens"])
        pos = torch.minimum(torch.arange(k, device="cuda").expand(b, k), st["len_dev"][:, None] - 1)
        row = _rows(st, pos, st["pages"], st["stride"]).reshape(b, 1, k)
        seen = (torch.arange(k, device="cuda") <= at.unsqueeze(-1)).unsqueeze(2)
    latent = _values(st["cache"][0][row], st["cache"][1][row], st["table"])
    key = torch.cat((latent, st["cache"][2][row].float()), -1)                # [B, m or 1, k, 576]
    if st["idx"] is None:                                                    # all queries of a request in one product
        z = torch.matmul(q.reshape(b, m * heads, DIM), key[:, 0].transpose(1, 2)).reshape(b, m, heads, k)
    else:
        z = torch.matmul(q, key.transpose(2, 3))
    z = (z * SCALE).masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    if st["idx"] is None:
        out = torch.matmul(p.reshape(b, m * heads, k), latent[:, 0]).reshape(b, m, heads, LATENT)
    else:
        out = torch.matmul(p, latent)
    lse = (top + torch.log(total)).squeeze(-1)
    if acc is None:
        return out.bfloat16(), lse
    weight = p.sum(2)                                                         # [B, m, k]
    if st["idx"] is None:
        acc += weight.sum(1)
    else:
        acc.scatter_add_(1, pos.clamp(min=0).long(), weight.reshape(b, m * k))
    return out.bfloat16(), lse, acc


def _evict(st):
    m, b = st["keep"], st["batch"]
    pages, to_pages = st["pages"], st["to_pages"]
    src = st["cache"] + (st["keys"], st["key_scale"])
    if own:
        pv = _lib()
        there = _map(st, m, to_pages)
        kept, acc = pv.pivot_evict(st["acc"], st["lens"], m, list(zip(src, st["to"])), _map(st, st["stride"], pages),
                                   there, sink=st["sink"], recent=st["recent"])
        back = pv.pivot_cache4_read(pv.make_cache4(*st["to"][:3], there), st["slots"])
    else:
        n = st["acc"].shape[1]
        pos, size = torch.arange(n, device="cuda"), st["len_dev"][:, None]
        held = (pos < st["sink"]) | (pos >= size - st["recent"])
        value = st["acc"].masked_fill(held, math.inf).masked_fill(pos >= size, -math.inf)
        order = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :m]
        order = torch.where(order < size, order, n).sort(dim=1).values
        order = torch.nn.functional.pad(order, (0, m - order.shape[1]), value=n)
        kept = torch.where(order < n, order, -1).int()
        acc = torch.where(kept >= 0, torch.gather(st["acc"], 1, kept.clamp(min=0).long()), 0.0)
        row = _rows(st, kept, pages, st["stride"])[kept >= 0]
        to = _rows(st, st["slots"], to_pages, m)[kept >= 0]
        for x, y in zip(src, st["to"]):
            y[to] = x[row]
        back = _read(st, st["to"], st["slots"], to_pages, m)
    # the indexer's keys of the kept tokens, where they are now
    keys, key_scale = st["to"][3].view(torch.float8_e4m3fn), st["to"][4]
    if pages is None:
        return kept, acc, back, keys, key_scale
    return kept, acc, back


# ------------------------------------------------------------------ the definitions in 64 bits
_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _exact_values(codes, scales):
    signed = torch.tensor(np.concatenate([_GRID, -_GRID]), device=codes.device)
    v = torch.empty(codes.shape[:-1] + (LATENT,), dtype=torch.float64, device=codes.device)
    v[..., 0::2] = signed[codes.remainder(16).long()]
    v[..., 1::2] = signed[codes.div(16, rounding_mode="floor").long()]
    two = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=codes.device), scales.double() - 127)
    return v * two.repeat_interleave(BLOCK, -1)


def _exact_place(st, b, pos, pages, stride):
    if pages is None:
        return b * stride + pos
    return pages[b].long()[pos // st["page"]] * st["page"] + pos % st["page"]


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "norm":
        h = st["x"].double() + st["residual"].double()
        y = h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * st["weight"].double()
        group = c["group"] or c["dim"]
        scale = torch.stack([y[:, i:i + group].abs().max(-1).values / 448 for i in range(0, c["dim"], group)], -1)
        return y / scale.repeat_interleave(group, -1)[:, :c["dim"]], scale, h
    if c["op"] == "cache":
        x = st["latent"].double().reshape(-1, LATENT // BLOCK, BLOCK)
        two = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 6)))
        grid = torch.tensor(_GRID, device="cuda")
        m = (x / two).abs()
        above = torch.searchsorted(grid, m.contiguous()).clamp(1, 7)
        lo, hi = grid[above - 1], grid[above]
        up = (hi - m < m - lo) | ((hi - m == m - lo) & (above % 2 == 0))
        v = torch.where(up, hi, lo).copysign(x) * two
        return torch.cat((v.reshape(-1, LATENT), st["rope"].double()), 1).reshape(c["batch"], c["n_q"], DIM)
    lens = st["lens"]
    if c["op"] == "evict":
        m = c["keep"]
        kept = torch.full((c["batch"], m), -1, dtype=torch.int64, device="cuda")
        acc = torch.zeros((c["batch"], m), dtype=torch.float64, device="cuda")
        back = torch.zeros((c["batch"], m, DIM), dtype=torch.float64, device="cuda")
        keys = torch.zeros((c["batch"], m, 128), dtype=torch.float64, device="cuda")
        key_scale = torch.zeros((c["batch"], m), dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            a = st["acc"][b, :n].cpu().numpy()
            mine = set(range(min(st["sink"], n))) | set(range(max(0, n - st["recent"]), n))
            for s in np.argsort(-a, kind="stable").tolist():
                if len(mine) >= min(m, n):
                    break
                mine.add(s)
            at = torch.tensor(sorted(mine), device="cuda")
            k = len(mine)
            row = _exact_place(st, b, at, st["pages"], st["stride"])
            kept[b, :k] = at
            acc[b, :k] = st["acc"][b, at].double()
            back[b, :k, :LATENT] = _exact_values(st["cache"][0][row], st["cache"][1][row])
            back[b, :k, LATENT:] = st["cache"][2][row].double()
            keys[b, :k] = st["keys"][row].view(torch.float8_e4m3fn).double()
            key_scale[b, :k] = st["key_scale"][row].double()
        if st["pages"] is None:
            return kept, acc, back, keys.reshape(-1, 128), key_scale.reshape(-1)
        return kept, acc, back
    if work(c)["flops"] > 2e12:
        return None
    b_, m, heads = st["q"].shape[:3]
    out = torch.zeros((b_, m, heads, LATENT), dtype=torch.float64, device="cuda")
    lse = torch.full((b_, m, heads), -math.inf, dtype=torch.float64, device="cuda")
    acc = torch.zeros((b_, max(lens)), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if not c["topk"]:
            row = _exact_place(st, b, torch.arange(n, device="cuda"), st["pages"], st["stride"])
            v = _exact_values(st["cache"][0][row], st["cache"][1][row])
            k = torch.cat((v, st["cache"][2][row].double()), 1)
        for i in range(m):
            if c["topk"]:
                at = st["idx"][b, i].long()
                at = at[at >= 0]
                row = _exact_place(st, b, at, st["pages"], st["stride"])
                v = _exact_values(st["cache"][0][row], st["cache"][1][row])
                k = torch.cat((v, st["cache"][2][row].double()), 1)
            else:
                at = torch.arange(n - m + i + 1, device="cuda")
            z = st["q"][b, i].double() @ k[:at.numel()].T * SCALE
            lse[b, i] = torch.logsumexp(z, -1)
            p = torch.exp(z - lse[b, i][:, None])
            out[b, i] = p @ v[:at.numel()]
            acc[b].index_add_(0, at, p.sum(0))
    return (out, lse, acc) if c["acc"] else (out, lse)
