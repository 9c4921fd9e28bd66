"""What is measured of the operators that a decode step with drafted tokens adds:
products of few rows with weights in 4 bits, attention for a tree of drafted
tokens over the 4-bit latent cache with the acceptance of one of its paths, and
the pages of a cache that sequences share (forked, grown, copied, freed and
compacted).

`run` computes them in their plain form, from elementary torch operations in 32
bits, or, with `own` set, through the entry points of paper_2607_24593_amd.

4-bit numbers are OCP MXFP4: E2M1 codes, the even value in the low nibble, and
one power-of-two scale (E8M0) per 32 values.  A cached token is a row of 512 such
latent values and 64 position values in bf16; all heads attend to the same rows.
"""
import math

import numpy as np
import torch

own = False

LATENT, ROPE = 512, 64
DIM = LATENT + ROPE
BLOCK = 32
ROW_BYTES = LATENT // 2 + LATENT // BLOCK + 2 * ROPE   # 400
KEY_BYTES = 128 + 4                                     # an fp8 indexer key and its scale
TOKEN_BYTES = ROW_BYTES + KEY_BYTES                     # 532
SCALE = 1.0 / math.sqrt(DIM)


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one token's projection in a decode step: latency
        dict(name="linear-1x4096x4096-bf16", op="linear", rows=1, k=4096, n=4096, x="bf16", group=0, out="bf16"),
        # the queries of 128 heads of a token and its draft, from the norm's fp8 rows
        dict(name="linear-2x4096x73728-fp8", op="linear", rows=2, k=4096, n=73728, x="fp8", group=0, out="bf16"),
        # a tree of 26 drafts, odd sizes, scales per block of 128, fp32 for what adds it up
        dict(name="linear-26x5024x8203-fp8-blocks", op="linear", rows=26, k=5024, n=8203, x="fp8", group=128, out="fp32"),
        # a decode batch of 64 rows through a wide layer
        dict(name="linear-64x6144x24576-bf16", op="linear", rows=64, k=6144, n=24576, x="bf16", group=0, out="bf16"),
        # a chat user's tree of 26 drafts over the 2048 keys that each node's index call chose
        dict(name="tree-1x6k-26-sparse", op="tree", heads=128, batch=1, shortest=6001, longest=6001, nodes=26, topk=2048,
             page=0, acc=False),
        # ragged requests in a paged pool, 12 drafts each: one of eight shards of 128 heads, weights accumulated
        dict(name="tree-8-ragged-12-dense-acc", op="tree", heads=16, batch=8, shortest=9001, longest=40000, nodes=12,
             topk=0, page=64, acc=True),
        # a decode batch with small trees over short contexts
        dict(name="tree-32x1500-7-dense", op="tree", heads=32, batch=32, shortest=300, longest=1500, nodes=7, topk=0,
             page=16, acc=False),
        # one long context and a wide tree, all heads
        dict(name="tree-1x128k-64-dense", op="tree", heads=128, batch=1, shortest=131072, longest=131072, nodes=64,
             topk=0, page=0, acc=False),
        # the accepted paths of a batch's trees, moved to where the next step expects them
        dict(name="accept-32x64-paged", op="accept", batch=32, shortest=3000, longest=16384, nodes=64, depth=9, page=64),
        # a step of parallel samples: losers freed, winners forked, all grown by their drafts, shared last pages copied
        dict(name="pages-step-32x4", op="step", batch=32, samples=4, shortest=500, longest=4000, new=33, page=64,
             spare=0.3),
        # a large pool of long contexts in which two prompts of 64K tokens are admitted
        dict(name="pages-step-big-pool", op="step", batch=2, samples=1, shortest=20000, longest=65536, new=65536, page=16,
             spare=3.0),
        # a pool after many requests have gone: pages at its end move into its holes
        dict(name="pages-compact-600k", op="compact", batch=48, shortest=4000, longest=16384, page=64, gone=0.35,
             moves=3000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "tree", "tree", "tree", "accept", "step", "compact"])
    if op == "linear":
        x, group = rng.choice([("bf16", 0), ("bf16", 0), ("fp8", 0), ("fp8", 128)])
        k = 32 * rng.choice([_log(rng, 8, 400), 16 * rng.randint(1, 24)])
        n = rng.choice([_log(rng, 50, 73728), 64 * rng.randint(4, 512)])
        n = min(n, 4096 * 73728 // k)
        rows = rng.choice([1, 2, 4, _log(rng, 1, 64), _log(rng, 1, 64)])
        return dict(op=op, rows=rows, k=k, n=n, x=x, group=group, out=rng.choice(["bf16", "bf16", "fp32"]))
    page = rng.choice([0, 0, 16, 64, 256])
    batch = _log(rng, 1, 48)
    longest = min(_log(rng, 2, 131072), (1 << 20) // batch)
    shortest = min(longest, rng.choice([longest, max(1, longest // rng.randint(2, 12))]))
    if op == "accept":
        nodes = _log(rng, 2, 200)
        return dict(op=op, batch=batch, shortest=shortest, longest=longest, nodes=nodes,
                    depth=rng.randint(1, min(nodes, 24)), page=page)
    if op in ("step", "compact"):
        page = rng.choice([16, 64, 64, 256])
        batch = min(batch, 40)
        longest = min(max(longest, 100), 400000 // batch)
        shortest = max(1, min(shortest, longest))
        if op == "step":
            return dict(op=op, batch=batch, samples=rng.randint(1, 5), shortest=shortest, longest=longest,
                        new=min(_log(rng, 1, 4000), 400000 // (6 * batch)), page=page, spare=rng.choice([0.1, 0.5, 2.0]))
        return dict(op=op, batch=batch, shortest=shortest, longest=longest, page=page, gone=rng.choice([0.1, 0.3, 0.6]),
                    moves=_log(rng, 10, 5000))
    heads = rng.choice([8, 16, 16, 32, 64, 128, 128, rng.randint(1, 128)])
    acc = rng.choice([False, False, True])
    nodes = _log(rng, 2, 100)
    if rng.random() < 0.4:  # over index sets
        topk = rng.choice([512, 1024, 2048, _log(rng, 100, 2048)])
        nodes = max(1, min(nodes, int(2.4e8 / (batch * heads * topk)), int(1.0e6 / (batch * topk))))
    else:
        topk = 0
        nodes = max(1, min(nodes, int(1.0e9 / (batch * heads * longest)) or 1))
        while batch * heads * nodes * (longest + nodes) > 1.07e9 and batch > 1:
            batch //= 2
    return dict(op="tree", heads=heads, batch=batch, shortest=shortest, longest=longest, nodes=nodes, topk=topk,
                page=page, acc=acc)


def _lengths(c):
    """Cached tokens of each request, from the shortest to the longest."""
    b, lo, hi = c["batch"], c["shortest"], c["longest"]
    return [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]


def _ceil(a, b):
    return -(-a // b)


def work(c):
    if c["op"] == "linear":
        r, k, n = c["rows"], c["k"], c["n"]
        groups = _ceil(k, c["group"]) if c["group"] else 1
        x = r * (2 * k if c["x"] == "bf16" else k + 4 * groups)
        return {"bytes": n * (k // 2 + k // BLOCK) + x + r * n * (2 if c["out"] == "bf16" else 4), "flops": 2.0 * r * n * k}
    lens = _lengths(c)
    if c["op"] == "accept":
        return {"bytes": 2 * c["batch"] * c["depth"] * TOKEN_BYTES + 4 * c["batch"] * c["depth"], "flops": 0.0}
    if c["op"] == "step":
        p, s = c["page"], c["samples"]
        tables = sum(_ceil(n, p) for n in lens) * s * 2 + sum(_ceil(n + c["new"], p) for n in lens) * (s + 1)
        copied = sum(s for n in lens if n % p) * p * TOKEN_BYTES
        return {"bytes": 4 * tables + 4 * _pool_pages(c) + 2 * copied, "flops": 0.0}
    if c["op"] == "compact":
        # what moves is about the part of the live pages that lies behind the holes
        live = (1 - c["gone"]) * sum(_ceil(n, c["page"]) for n in lens)
        moved = min(c["moves"], c["gone"] * live)
        return {"bytes": 2 * moved * c["page"] * TOKEN_BYTES + 8 * live, "flops": 0.0}
    rows, heads, m = c["batch"] * c["nodes"], c["heads"], c["nodes"]
    io = rows * heads * (2 * DIM + 2 * LATENT + 4)
    if c["topk"]:
        pairs = sum(m * min(c["topk"], n + m) for n in lens)
        # a sequence's sets overlap: the first, and about a quarter of each further one
        read = sum(min(n + m, int(c["topk"] * (1 + 0.25 * (m - 1)))) for n in lens)
        io += 4 * rows * c["topk"] + (8 * read if c["acc"] else 0)
    else:
        pairs = sum(m * (n + max(1, m // 4)) for n in lens)  # a node has few ancestors
        read = sum(n + m for n in lens)
        io += 8 * read if c["acc"] else 0
    return {"bytes": io + read * ROW_BYTES, "flops": 2.0 * (DIM + LATENT) * pairs * heads}


# ------------------------------------------------------------------ 4-bit numbers in plain operations
def _quantise(x):
    """x [n, k] -> codes uint8 [n, k / 2], scales uint8 [n, k / 32]."""
    n, k = x.shape
    v = x.float().reshape(n, k // BLOCK, BLOCK)
    amax = v.abs().amax(-1)
    mant, e = torch.frexp(amax)
    e = e - 3 + (mant > 0.75).int()
    e = torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    inv = ((127 - e).clamp(1, 254) << 23).view(torch.float32)
    m = v.abs() * inv.unsqueeze(-1)
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int()
            + (m >= 3.5).int() + (m > 5.0).int())
    code = (code + 8 * (v < 0).int()).reshape(n, k // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales, table):
    """codes [..., k / 2], scales [..., k / 32] -> fp32 [..., k]."""
    both = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1)
    two = torch.where(scales == 0, torch.full((), 2.0 ** -127, device=codes.device),
                      (scales.int() << 23).view(torch.float32))
    lead, k = codes.shape[:-1], 2 * codes.shape[-1]
    return (both.reshape(*lead, k // BLOCK, BLOCK) * two.unsqueeze(-1)).reshape(*lead, k)


def _grid(device="cuda"):
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=device)


# ------------------------------------------------------------------ inputs
def _normal(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std


def _cache(rows, g):
    codes = torch.empty((rows, LATENT // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, LATENT // BLOCK), dtype=torch.uint8, device="cuda")
    step = 1 << 18
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x = _normal((n, LATENT), g) * torch.exp(0.5 * _normal((1, LATENT), g))  # a latent's channels differ in size
        codes[r:r + n], scales[r:r + n] = _quantise(x)
    return codes, scales, _normal((rows, ROPE), g).bfloat16()


def _arrays(rows, g):
    """What a pool holds for each token: the cache's three arrays, the indexer's keys and their scales."""
    byte = lambda n: torch.randint(0, 119, (rows, n), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    return (byte(LATENT // 2), byte(LATENT // BLOCK), _normal((rows, ROPE), g).bfloat16(), byte(128),
            torch.exp(_normal((rows,), g)))


def _trees(c, g, cpu):
    """Masks [B, nodes, words] of trees in topological order: bit j of node i is
    set where j is i or an ancestor of it."""
    b, m = c["batch"], c["nodes"]
    seen = np.zeros((b, m, m), dtype=bool)
    for t in range(b):
        for i in range(m):
            if i > 0:
                # drafters extend late nodes more often than early ones; a few start at the root
                parent = int(i * (cpu.random() ** 0.5)) if cpu.random() > 0.1 else -1
                if parent >= 0:
                    seen[t, i] = seen[t, parent]
            seen[t, i, i] = True
    words = _ceil(m, 32)
    bits = np.zeros((b, m, 32 * words), dtype=np.uint64)
    bits[:, :, :m] = seen
    packed = (bits.reshape(b, m, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(packed.view(np.int32)).cuda()


def _bits(mask, m):
    """Masks [B, m, words] -> truth values [B, m, m]."""
    j = torch.arange(m, device=mask.device)
    return ((mask[..., j // 32] >> (j % 32)) & 1).bool()


def _sets(c, lens, seen, g):
    """Index sets of the trees' nodes: the top of scores that a sequence's nodes
    mostly share.  A node's ancestors and itself are among them, and a few drafts
    that it must not see."""
    out, m, k = [], c["nodes"], c["topk"]
    for b, base in enumerate(lens):
        n = base + m
        score = _normal((1, n), g) + 0.4 * _normal((m, n), g)
        score[:, base:] += 10.0 * seen[b]
        top, idx = torch.topk(score, min(k, n), sorted=False)
        idx = idx.int()
        out.append(torch.cat((idx, idx.new_full((m, k - idx.shape[1]), -1)), 1))
    return torch.stack(out).contiguous()


def _pool_pages(c):
    """Pages of the pool of a step: those of all sequences once they are grown, and spare ones."""
    p = c["page"]
    grown = sum(_ceil(n + c["new"], p) + c["samples"] * (_ceil(n + c["new"], p) - n // p) for n in _lengths(c))
    return int(grown * (1 + c["spare"])) + 3


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 2654435761 % (1 << 62) + 29)
    cpu = np.random.default_rng(seed % (1 << 62) + 31)
    st = dict(c)
    st["grid"] = _grid()
    if c["op"] == "linear":
        r, k, n = c["rows"], c["k"], c["n"]
        st["codes"] = torch.empty((n, k // 2), dtype=torch.uint8, device="cuda")
        st["scales"] = torch.empty((n, k // BLOCK), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 27) // k)
        spread = torch.exp(0.3 * _normal((1, k), g))  # some input channels weigh more than others
        for i in range(0, n, step):
            j = min(n, i + step)
            st["codes"][i:j], st["scales"][i:j] = _quantise(_normal((j - i, k), g, k ** -0.5) * spread)
        # normed rows: a few channels are much larger than the others
        x = _normal((r, k), g) * (1 + 8 * (_normal((1, k), g) > 2.6))
        if c["x"] == "bf16":
            st["rows_in"], st["row_scale"] = x.bfloat16(), None
        else:
            group = c["group"] or k
            parts = _ceil(k, group)
            y = torch.nn.functional.pad(x, (0, parts * group - k)).reshape(r, parts, group)
            scale = y.abs().amax(-1) / 448
            codes = (y / scale.unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn)
            st["rows_in"] = codes.reshape(r, parts * group)[:, :k].contiguous()
            st["row_scale"] = scale.contiguous()
        return st
    lens = _lengths(c)
    st["lens"] = lens
    st["len_dev"] = torch.tensor(lens, dtype=torch.int64, device="cuda")
    page, b = c["page"], c["batch"]
    if c["op"] in ("tree", "accept"):
        m = c["nodes"]
        per = max(lens) + m
        if page:
            need = _ceil(per, page)
            order = torch.randperm(b * need + 3, generator=g, device="cuda").int()
            st["pages"], st["stride"], rows = order[:b * need].reshape(b, need).contiguous(), 0, (b * need + 3) * page
        else:
            st["pages"], st["stride"], rows = None, per, b * per
        st["pool_rows"] = rows
        if c["op"] == "accept":
            st["arrays"] = _arrays(rows, g)
            # a path's nodes, ascending: the first ones as they lie, then later drafts; padded where it ends early
            path = np.full((b, c["depth"]), -1, dtype=np.int32)
            for t in range(b):
                d = min(c["depth"], int(cpu.integers(1, c["depth"] + 1)))
                keep = int(cpu.integers(0, d + 1)) if m >= c["depth"] + d else d
                later = cpu.choice(np.arange(c["depth"], m), d - keep, replace=False) if d > keep else []
                path[t, :d] = np.concatenate([np.arange(keep), np.sort(later)])
            st["path"] = torch.from_numpy(path).cuda()
            return st
        st["mask"] = _trees(c, g, cpu)
        st["cache"] = _cache(rows, g)
        st["n_k"] = [n + m for n in lens]
        st["q"] = _normal((b, m, c["heads"], DIM), g, 2.0).bfloat16()
        st["idx"] = _sets(c, lens, _bits(st["mask"], m), g) if c["topk"] else None
        st["acc"] = torch.zeros((b, max(st["n_k"])), device="cuda") if c["acc"] else None
        return st
    if c["op"] == "step":
        samples, new = c["samples"], c["new"]
        pages = _pool_pages(c)
        slots, width = b * (1 + samples), _ceil(max(lens) + new, page)
        table = np.full((slots, width), -1, dtype=np.int32)
        refs = np.zeros(pages, dtype=np.int32)
        order = cpu.permutation(pages)
        at = 0
        for t, n in enumerate(lens):  # slot t (1 + samples) is the sequence, its forks follow
            k = _ceil(n, page)
            table[t * (1 + samples), :k] = order[at:at + k]
            at += k
        refs[order[:at]] = 1
        parents = [t * (1 + samples) for t in range(b)]
        st["src"] = [s for s in parents for _ in range(samples)]
        st["dst"] = [s + 1 + i for s in parents for i in range(samples)]
        st["fork_len"] = [n for n in lens for _ in range(samples)]
        st["slots"] = [s + i for s in parents for i in list(range(1, 1 + samples)) + [0]]  # the sequence after its forks
        st["now"] = [n for n in lens for _ in range(1 + samples)]
        st["then"] = [n + new for n in st["now"]]
        st["kept"] = [n if i == samples else 0 for n in lens for i in range(1 + samples)]
        for name in ("src", "dst", "fork_len", "slots", "now", "then", "kept"):
            st[name + "_dev"] = torch.tensor(st[name], dtype=torch.int64, device="cuda")
        st["table"], st["refs"] = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
        st["arrays"] = _arrays(pages * page, g)
        return st
    # compact: a batch's pages lie anywhere, some sequences have gone, some share their first pages
    k = [_ceil(n, page) for n in lens]
    pages = sum(k) + 5
    order = cpu.permutation(pages)
    table = np.full((b, max(k)), -1, dtype=np.int32)
    refs = np.zeros(pages, dtype=np.int32)
    at = 0
    for t in range(b):
        mine = order[at:at + k[t]].copy()
        at += k[t]
        if cpu.random() < c["gone"]:
            continue
        if t > 0 and cpu.random() < 0.25 and table[t - 1, 0] >= 0:
            shared = min(k[t], k[t - 1]) // 2
            mine[:shared] = table[t - 1, :shared]
        table[t, :k[t]] = mine
        np.add.at(refs, mine, 1)
    st["table0"], st["refs0"] = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda()
    st["table"], st["refs"] = st["table0"].clone(), st["refs0"].clone()
    st["arrays"] = _arrays(pages * page, g)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return {"linear": _linear, "tree": _tree, "accept": _accept, "step": _step, "compact": _compact}[st["op"]](st)


def _lib():
    import paper_2607_24593_amd as pv
    return pv


def _linear(st):
    out = torch.bfloat16 if st["out"] == "bf16" else torch.float32
    if own:
        return _lib().pivot_linear4(st["rows_in"], st["codes"], st["scales"], x_scale=st["row_scale"], group=st["group"],
                                    dtype=out)
    x = st["rows_in"].float()
    if st["row_scale"] is not None:
        r, k = x.shape
        s = st["row_scale"]
        x = x * (torch.repeat_interleave(s, st["group"], 1)[:, :k] if st["group"] else s)
    n, k = st["n"], st["k"]
    step = max(1, (1 << 28) // k)
    y = [torch.matmul(x, _values(st["codes"][i:i + step], st["scales"][i:i + step], st["grid"]).t())
         for i in range(0, n, step)]
    return torch.cat(y, 1).to(out)


def _map(st):
    pv = _lib()
    if st["pages"] is not None:
        return pv.make_row_map(block_table=st["pages"], page_size=st["page"], rows=st["pool_rows"])
    return pv.make_row_map(seq_stride=st["stride"], rows=st["pool_rows"])


def _rows(st, pos):
    """Pool rows of positions pos [B, n] (negative ones count as 0)."""
    pos = pos.clamp(min=0).long()
    if st["pages"] is None:
        return torch.arange(pos.shape[0], device=pos.device)[:, None] * st["stride"] + pos
    return torch.gather(st["pages"].long(), 1, pos // st["page"]) * st["page"] + pos % st["page"]


def _tree(st):
    acc = st["acc"]
    if acc is not None:
        acc.zero_()  # the window of queries whose weights count begins here
    if own:
        pv = _lib()
        cache = pv.make_cache4(*st["cache"], _map(st))
        out, lse = pv.pivot_cache4_attend(st["q"], cache, st["lens"], st["n_k"], SCALE, idx=st["idx"], acc=acc,
                                          tree=st["mask"])
        return (out, lse) if acc is None else (out, lse, acc)
    b, m, heads = st["q"].shape[:3]
    base = st["len_dev"][:, None, None]                                       # [B, 1, 1]
    seen = _bits(st["mask"], m)                                               # [B, m, m]
    if st["idx"] is not None:
        k = st["topk"]
        pos = st["idx"].reshape(b, m * k)
        at = st["idx"].long()                                                 # [B, m, k]
    else:
        k = max(st["n_k"])
        at = torch.minimum(torch.arange(k, device="cuda").expand(b, 1, k), base + m - 1)
        pos = at.reshape(b, k)
        at = torch.where(torch.arange(k, device="cuda") < base + m, torch.arange(k, device="cuda"), -1).expand(b, m, k)
    draft = torch.gather(seen, 2, (at - base).clamp(0, m - 1))
    ok = (at >= 0) & ((at < base) | ((at - base < m) & draft))
    row = _rows(st, pos).reshape(b, -1, k)
    q = st["q"].float()
    latent = _values(st["cache"][0][row], st["cache"][1][row], st["grid"])
    key = torch.cat((latent, st["cache"][2][row].float()), -1)                # [B, m or 1, k, 576]
    if st["idx"] is None:
        z = torch.matmul(q.reshape(b, m * heads, DIM), key[:, 0].transpose(1, 2)).reshape(b, m, heads, k)
    else:
        z = torch.matmul(q, key.transpose(2, 3))
    del key
    z = (z * SCALE).masked_fill(~ok.unsqueeze(2), -math.inf)
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
    weight = p.sum(2)
    if st["idx"] is None:
        acc += weight.sum(1)
    else:
        acc.scatter_add_(1, pos.clamp(min=0).long(), weight.reshape(b, m * k))
    return out.bfloat16(), lse, acc


def _accept(st):
    if own:
        _lib().pivot_tree_accept(st["path"], st["lens"], st["arrays"], _map(st))
        return st["arrays"]
    path = st["path"].long()
    base = st["len_dev"][:, None]
    there = _rows(st, base + torch.arange(path.shape[1], device="cuda").expand_as(path))
    here = _rows(st, base + path.clamp(min=0))
    ok = path >= 0
    for x in st["arrays"]:
        x[there[ok]] = x[here[ok]]  # the right side is read whole before it is written
    return st["arrays"]


def _plain_grow(table, refs, page, slots, now, then):
    """Sequences in the order of the list: a last page that others hold too is
    copied (the last holder keeps it), new pages follow, all from the lowest free
    pages up; where those are too few nothing happens."""
    n = slots.numel()
    grows = then > now
    last = table[slots, ((now - 1) // page).clamp(min=0)].long()
    part = grows & (now % page > 0) & (last >= 0)
    last = torch.where(part, last, -1 - torch.arange(n, device="cuda"))
    rank = ((last[:, None] == last) & (torch.arange(n, device="cuda")[:, None] > torch.arange(n, device="cuda"))).sum(1)
    copies = part & (rank < refs[last.clamp(min=0)] - 1)
    first_new = (now + page - 1) // page
    fresh = torch.where(grows, (then + page - 1) // page - first_new, 0)
    need = copies.long() + fresh
    first = torch.cumsum(need, 0) - need
    free = torch.nonzero(refs == 0).flatten()
    total = need.sum()
    pairs = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    state = torch.stack((torch.clamp(total - free.numel(), min=0), free.numel() - total)).int()
    if int(total) > free.numel():
        state[1] = free.numel()
        return pairs, state
    who = torch.nonzero(copies).flatten()
    old, new = last[who], free[first[who]]
    pairs[who, 0], pairs[who, 1] = old.int(), new.int()
    refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    refs[new] = 1
    table[slots[who], (now[who] - 1) // page] = new.int()
    most = int(fresh.max())
    j = torch.arange(most, device="cuda")
    mine = j < fresh[:, None]
    which = free[(first + copies)[:, None].expand(n, most)[mine] + j.expand(n, most)[mine]]
    table[slots[:, None].expand(n, most)[mine], (first_new[:, None] + j)[mine]] = which.int()
    refs[which] = 1
    return pairs, state


def _step(st):
    table, refs, page, arrays = st["table"], st["refs"], st["page"], st["arrays"]
    if own:
        pv = _lib()
        pages = pv.make_pages(table, refs, page)
        pv.pivot_pages_free(pages, st["slots"], st["then"], st["kept"])
        pv.pivot_pages_fork(pages, st["src"], st["dst"], st["fork_len"])
        pairs, state = pv.pivot_pages_grow(pages, st["slots"], st["now"], st["then"])
        pv.pivot_pages_copy(pages, pairs, arrays)
        return table, refs, pairs, state, arrays
    width = torch.arange(table.shape[1], device="cuda")
    # free: of each sequence the pages behind those that it keeps
    slots = st["slots_dev"]
    held = table[slots]
    gone = (width >= ((st["kept_dev"] + page - 1) // page)[:, None]) & (held >= 0) \
        & (width < ((st["then_dev"] + page - 1) // page)[:, None])
    refs.index_add_(0, held[gone].long(), torch.full((int(gone.sum()),), -1, dtype=torch.int32, device="cuda"))
    table[slots] = torch.where(gone, -1, held)
    # fork: the pages of the source
    held = table[st["src_dev"]]
    shared = (width < ((st["fork_len_dev"] + page - 1) // page)[:, None]) & (held >= 0)
    table[st["dst_dev"]] = torch.where(shared, held, table[st["dst_dev"]])
    refs.index_add_(0, held[shared].long(), torch.ones(int(shared.sum()), dtype=torch.int32, device="cuda"))
    pairs, state = _plain_grow(table, refs, page, slots, st["now_dev"], st["then_dev"])
    _plain_copy(pairs, page, arrays)
    return table, refs, pairs, state, arrays


def _plain_copy(pairs, page, arrays):
    pairs = pairs[pairs[:, 0] >= 0].long()
    row = torch.arange(page, device="cuda")
    here, there = ((pairs[:, i, None] * page + row).flatten() for i in (0, 1))
    for x in arrays:
        x[there] = x[here]


def _compact(st):
    table, refs, page, arrays = st["table"], st["refs"], st["page"], st["arrays"]
    table.copy_(st["table0"])  # the pool as the requests that have gone left it
    refs.copy_(st["refs0"])
    if own:
        pv = _lib()
        pages = pv.make_pages(table, refs, page)
        pairs, state = pv.pivot_pages_compact(pages, st["moves"])
        pv.pivot_pages_copy(pages, pairs, arrays)
        return table, refs, pairs, state, arrays
    live, free = torch.nonzero(refs > 0).flatten().flip(0), torch.nonzero(refs == 0).flatten()
    n = min(live.numel(), free.numel(), st["moves"])
    here, there = live[:n], free[:n]
    down = here > there
    here, there = here[down], there[down]
    pairs = torch.full((st["moves"], 2), -1, dtype=torch.int32, device="cuda")
    pairs[:here.numel(), 0], pairs[:here.numel(), 1] = here.int(), there.int()
    refs[there] = refs[here]
    refs[here] = 0
    new = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    new[here] = there.int()
    table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()], table))
    _plain_copy(pairs, page, arrays)
    return table, refs, pairs, torch.tensor([here.numel(), live.numel()], dtype=torch.int32, device="cuda"), arrays


# ------------------------------------------------------------------ the definitions in 64 bits
_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _exact_values(codes, scales):
    signed = torch.tensor(np.concatenate([_GRID, -_GRID]), device=codes.device)
    v = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=codes.device)
    v[..., 0::2] = signed[codes.remainder(16).long()]
    v[..., 1::2] = signed[codes.div(16, rounding_mode="floor").long()]
    two = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=codes.device), scales.double() - 127)
    return v * two.repeat_interleave(BLOCK, -1)


def _exact_place(st, b, pos):
    if st["pages"] is None:
        return b * st["stride"] + pos
    return st["pages"][b].long()[pos // st["page"]] * st["page"] + pos % st["page"]


def _exact_arrays(arrays, moves):
    """The pool's arrays after rows have moved, one after the other."""
    out = []
    for x in arrays:
        y = x.cpu().clone()
        for here, there in moves:
            y[there] = y[here]
        out.append((y.double() if y.is_floating_point() else y).cuda())
    return tuple(out)


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "linear":
        x = st["rows_in"].double()
        if st["row_scale"] is not None:
            of = torch.arange(c["k"], device="cuda") // (c["group"] or c["k"])
            x = x * st["row_scale"].double()[:, of]
        y = torch.empty((c["rows"], c["n"]), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 27) // c["k"])
        for i in range(0, c["n"], step):
            y[:, i:i + step] = x @ _exact_values(st["codes"][i:i + step], st["scales"][i:i + step]).T
        return y
    lens = st["lens"]
    if c["op"] == "accept":
        moves = []
        for b, path in enumerate(st["path"].tolist()):
            for j, node in enumerate(path):
                if node >= 0:
                    moves.append(tuple(int(_exact_place(st, b, lens[b] + v)) for v in (node, j)))
        return _exact_arrays(st["arrays"], moves)
    if c["op"] in ("step", "compact"):
        page = c["page"]
        table, refs = st["table"].cpu().numpy(), st["refs"].cpu().numpy()
        if c["op"] == "step":
            pairs = np.full((len(st["slots"]), 2), -1, dtype=np.int32)
            for s, d, n in zip(st["src"], st["dst"], st["fork_len"]):
                for i in range(_ceil(n, page)):
                    table[d, i] = table[s, i]
                    refs[table[s, i]] += 1
            free = [int(p) for p in np.nonzero(refs == 0)[0]][::-1]
            before = len(free)
            for i, (s, a, z) in enumerate(zip(st["slots"], st["now"], st["then"])):
                at = table[s, a // page] if a % page else -1
                if at >= 0 and refs[at] > 1:
                    refs[at] -= 1
                    table[s, a // page] = free.pop()
                    refs[table[s, a // page]] = 1
                    pairs[i] = at, table[s, a // page]
                for j in range(_ceil(a, page), _ceil(z, page)):
                    table[s, j] = free.pop()
                    refs[table[s, j]] = 1
            state = [0, len(free)]
            assert before >= len(free)
        else:
            pairs = np.full((c["moves"], 2), -1, dtype=np.int32)
            n, live = 0, int((refs > 0).sum())
            low, high = 0, len(refs) - 1
            to = {}
            while n < c["moves"]:
                while low < high and refs[low] > 0:
                    low += 1
                while low < high and refs[high] == 0:
                    high -= 1
                if low >= high:
                    break
                pairs[n] = high, low
                to[high] = low
                refs[low], refs[high] = refs[high], 0
                n += 1
            table = np.vectorize(lambda p: to.get(p, p))(table).astype(np.int32)
            state = [n, live]
        moves = [(slice(h * page, h * page + page), slice(t * page, t * page + page)) for h, t in pairs.tolist() if h >= 0]
        whole = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return whole(table), whole(refs), whole(pairs), torch.tensor(state, dtype=torch.int32, device="cuda"), \
            _exact_arrays(st["arrays"], moves)
    if work(c)["flops"] > 4e12:
        return None
    b_, m, heads = st["q"].shape[:3]
    out = torch.zeros((b_, m, heads, LATENT), dtype=torch.float64, device="cuda")
    lse = torch.full((b_, m, heads), -math.inf, dtype=torch.float64, device="cuda")
    acc = torch.zeros((b_, max(st["n_k"])), dtype=torch.float64, device="cuda")
    masks = st["mask"].cpu().numpy().view(np.uint32)
    for b, n in enumerate(lens):
        row = _exact_place(st, b, torch.arange(n + m, device="cuda"))
        v = _exact_values(st["cache"][0][row], st["cache"][1][row])
        k = torch.cat((v, st["cache"][2][row].double()), 1)
        for i in range(m):
            drafts = [n + j for j in range(m) if masks[b, i, j // 32] >> (j % 32) & 1]
            if c["topk"]:
                mine = set(drafts)
                entries = st["idx"][b, i].tolist()
                at = torch.tensor([s for s in entries if 0 <= s < n or s in mine], dtype=torch.int64, device="cuda")
            else:
                at = torch.cat((torch.arange(n, device="cuda"), torch.tensor(drafts, device="cuda")))
            z = st["q"][b, i].double() @ k[at].T * SCALE
            lse[b, i] = torch.logsumexp(z, -1)
            p = torch.exp(z - lse[b, i][:, None])
            out[b, i] = p @ v[at]
            acc[b].index_add_(0, at, p.sum(0))
    return (out, lse, acc) if c["acc"] else (out, lse)
