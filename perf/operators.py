"""The operators beside the restricted head that a decode step needs, as cases that can be measured: a key/value
cache held in 8 bits (written, read back, attended over) and the sampling of tokens from the target's logits.

Where `own` is false, `run` computes them in plain torch operations; where it is true, by the package's calls.
Inputs are the same for both.

Kinds:
  write   new tokens of several sequences are quantised into a paged cache; the blocks they touched are read back
  read    a part of the cache goes back to a floating type, for a caller that needs it so
  attend  rows of queries against the cache: one token, a draft tree (a bit mask among its nodes), a causal chunk
  sample  a token for each row of logits by temperature, top-k, top-p and min-p from given random numbers

The cache: pages of 32 to 256 tokens, in blocks of 32; K and V of a block and head share a scale each.  Per page and
head, blocks follow one another; per block all of K (32 x dim bytes), then all of V:
  K  [dim / 32][half h][token m][16 dims: 32 s + 16 h + b]
  V  [dim / 32][half h][dim 32 s + d][16 tokens: 8 a + 4 h + i, a = 0..3 outer, i = 0..3 inner]
scales are fp32 [pages, heads, blocks of a page, 2 (K, V)].
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
FLOATS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a decode step of 64 sequences: one token each goes into the cache
        {"name": "append 64 x 1", "kind": "write", "S": 64, "rows": 1, "len": 2048, "heads": 8, "dim": 128, "cache": "e4m3",
         "page": 64, "type": "bf16"},
        # two prompts are filled in
        {"name": "prompt 2 x 8,000", "kind": "write", "S": 2, "rows": 8000, "len": 0, "heads": 8, "dim": 128, "cache": "int8",
         "page": 128, "type": "bf16"},
        # the cache of one short sequence of a small model, for a caller that works in 32 bits
        {"name": "read 1 x 700", "kind": "read", "S": 1, "rows": 700, "len": 0, "heads": 8, "dim": 64, "cache": "int8", "page": 32,
         "type": "fp32"},
        # four long prefixes handed over in bf16
        {"name": "read 4 x 16,384", "kind": "read", "S": 4, "rows": 16384, "len": 0, "heads": 8, "dim": 128, "cache": "e4m3",
         "page": 64, "type": "bf16"},
        # the next token of one short conversation: a call is launches and latency
        {"name": "one token, 1,000", "kind": "attend", "S": 1, "rows": 1, "len": 1000, "group": 4, "heads": 8, "dim": 64,
         "cache": "e4m3", "page": 32, "type": "bf16", "tree": False},
        # a decode step of a full batch
        {"name": "64 tokens, 4,096 each", "kind": "attend", "S": 64, "rows": 1, "len": 4096, "group": 4, "heads": 8, "dim": 128,
         "cache": "e4m3", "page": 64, "type": "bf16", "tree": False},
        # one token far into one long document
        {"name": "one token, 131,072", "kind": "attend", "S": 1, "rows": 1, "len": 131072, "group": 4, "heads": 8, "dim": 128,
         "cache": "int8", "page": 64, "type": "fp16", "tree": False},
        # the target verifies the 60-node draft trees of eight sequences
        {"name": "trees 8 x 60, 3,000 each", "kind": "attend", "S": 8, "rows": 60, "len": 3000, "group": 4, "heads": 8,
         "dim": 128, "cache": "e4m3", "page": 64, "type": "bf16", "tree": True},
        # a chunk of a prompt behind what is there already
        {"name": "chunk 2,048 on 8,192", "kind": "attend", "S": 1, "rows": 2048, "len": 10240, "group": 4, "heads": 8,
         "dim": 128, "cache": "e4m3", "page": 128, "type": "bf16", "tree": False},
        # one sequence's next token
        {"name": "sample 1 row", "kind": "sample", "M": 1, "V": 151936, "type": "fp32", "ids": False, "filter": "all"},
        # the tokens of one verified draft tree
        {"name": "sample 60 rows", "kind": "sample", "M": 60, "V": 151936, "type": "fp32", "ids": False, "filter": "all"},
        # 16 trees at once, of a target that leaves its logits in bf16
        {"name": "sample 960 rows", "kind": "sample", "M": 960, "V": 151936, "type": "bf16", "ids": False, "filter": "top_p"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attend", "attend", "attend", "attend", "sample", "sample", "sample"])
    if kind == "sample":
        M = _log(rng, 1, 512)
        V = _log(rng, 1000, 160000)
        return {"kind": kind, "M": M, "V": V, "type": rng.choice(["fp32", "fp32", "bf16", "fp16"]), "ids": rng.random() < 0.4,
                "filter": rng.choice(["all", "all", "top_k", "top_p", "min_p", "none"])}
    heads, dim = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 96, 128, 128, 128, 192, 256])
    c = {"kind": kind, "heads": heads, "dim": dim, "cache": rng.choice(["e4m3", "e4m3", "int8"]),
         "page": rng.choice([32, 64, 64, 128, 256])}
    if kind in ("write", "read"):
        # at most 16,384 tokens of 1,024 elements in all
        tokens = _log(rng, 1, 16384 * 1024 // max(1024, heads * dim))
        S = min(tokens, _log(rng, 1, 64))
        c.update(S=S, rows=max(1, tokens // S), len=0 if rng.random() < 0.3 else _log(rng, 1, 4096),
                 type=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
        return c
    mode = rng.choice(["token", "token", "tree", "chunk"])
    c.update(group=rng.choice([1, 2, 4, 4, 7, 8]), type=rng.choice(["bf16", "bf16", "fp16"]), tree=mode == "tree")
    if mode == "token":
        S = _log(rng, 1, 64)
        c.update(S=S, rows=1, len=_log(rng, 1, min(131072, 64 * 4096 * 1024 // max(1024, heads * dim) // S)))
    elif mode == "tree":
        S = _log(rng, 1, 8)
        rows = rng.randrange(2, 65)
        c.update(S=S, rows=rows, len=rows + _log(rng, 1, 3000 * 4 * 1024 // max(4096, c["group"] * heads * dim)))
    else:
        S = _log(rng, 1, 4)
        rows = max(1, _log(rng, 4, 512) // S)
        c.update(S=S, rows=rows, len=rows + _log(rng, 1, 8192 * 4 * 1024 // max(4096, c["group"] * heads * dim)))
    return c


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _spread(least, most, S, ragged):
    """S whole numbers in [least, most]: the largest first, the others anywhere in the upper half, or all the same.  They
    are the case's own, whatever the seed: a golden-ratio sequence."""
    if not ragged or S == 1:
        return [most] * S
    low = max(least, (most + 1) // 2)
    return [most] + [low + int((i * 0.6180339887) % 1.0 * (most - low + 1)) for i in range(1, S)]


def _sizes(case):
    """Where the rows of every sequence start, and how many there are."""
    S, ragged = case["S"], case["S"] > 1
    rows = _spread(1, case["rows"], S, ragged and case["rows"] > 1)
    if case["kind"] == "attend":                                      # they are the last of the sequence's tokens
        lens = _spread(1, case["len"], S, ragged)
        rows = [min(r, n) for r, n in zip(rows, lens)]
        return [n - r for n, r in zip(lens, rows)], rows
    return [0] * S if case["len"] == 0 else _spread(0, case["len"], S, ragged), rows


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(counts):
    return _i32([0] + torch.tensor(counts).cumsum(0).tolist())


def _cache(case, tokens, g):
    """A full cache: pages for `tokens` of every sequence in any order, with the values of a layer: codes, scales, page table."""
    H, D, page = case["heads"], case["dim"], case["page"]
    width = -(-max(tokens) // page)
    pages = case["S"] * width + 3
    table = torch.randperm(pages, generator=g, device=DEV)[:case["S"] * width].to(torch.int32).view(case["S"], width)
    shape = (pages, H, page // BLOCK, 2, BLOCK * D)
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    # what stands for one: a largest value of about 4 in a block of a bell-shaped distribution
    if case["cache"] == "e4m3":
        data = (x * 64).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        scales = torch.exp2(torch.randint(-7, -5, shape[:4], generator=g, device=DEV).float())
    else:
        data = (x * 28).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
        scales = (0.5 + torch.rand(shape[:4], generator=g, device=DEV)) / 28
    return data, scales, table.contiguous()


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["kind"] == "sample":
        M, V = case["M"], case["V"]
        z = torch.randn((M, V), generator=g, device=DEV).mul_(2.0)
        # the few tokens that a context allows
        top = torch.randint(0, V, (M, 40), generator=g, device=DEV)
        z.scatter_reduce_(1, top, 4.0 + 10.0 * torch.rand((M, 40), generator=g, device=DEV), "amax")
        z[:, V // 3:V // 3 + V // 50] = -math.inf                    # banned tokens
        s["logits"] = z.to(FLOATS[case["type"]])
        s["u"] = torch.rand(M, generator=g, device=DEV)
        s["ids"] = torch.randperm(2 * V, generator=g, device=DEV)[:V].to(torch.int32) if case["ids"] else None
        f = case["filter"]
        r = torch.rand((4, M), generator=g, device=DEV)
        s["temperature"] = torch.where(r[0] < 0.1, 0.0, 0.5 + r[0])           # one in ten greedy
        s["top_k"] = (2.0 + 98.0 * r[1]).to(torch.int32) if f in ("all", "top_k") else None
        s["top_p"] = 0.8 + 0.19 * r[2] if f in ("all", "top_p") else None
        s["min_p"] = 0.01 + 0.1 * r[3] if f in ("all", "min_p") else None
        return s
    S, H, D = case["S"], case["heads"], case["dim"]
    dtype = FLOATS[case["type"]]
    starts, rows = _sizes(case)
    if case["kind"] == "attend":
        lens = [a + r for a, r in zip(starts, rows)]
        s["data"], s["scales"], s["table"] = _cache(case, lens, g)
        s["lens"], s["row_off"], s["max_rows"], s["max_len"] = _i32(lens), _offsets(rows), max(rows), max(lens)
        T = sum(rows)
        s["q"] = torch.randn((T, H * case["group"], D), generator=g, device=DEV).to(dtype)
        s["tree"] = None
        if case["tree"]:
            # every node's parent is any node before it; it sees its ancestors and itself
            n = max(rows)
            parent = torch.rand(n, generator=g, device=DEV).mul(torch.arange(n, device=DEV)).long().tolist()
            bits = [1]
            for j in range(1, n):
                bits.append(bits[parent[j]] | 1 << j)
            bits = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64)
            s["tree"] = torch.cat([bits[:r] for r in rows]).to(DEV)
        return s
    s["data"], s["scales"], s["table"] = _cache(case, [a + r for a, r in zip(starts, rows)], g)
    s["starts"], s["row_off"], s["max_rows"] = _i32(starts), _offsets(rows), max(rows)
    if case["kind"] == "write":
        T = sum(rows)
        # K and V as a fused projection leaves them, beside each other
        kv = torch.randn((T, 2, H, D), generator=g, device=DEV).to(dtype)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        starts, rows = [a // BLOCK * BLOCK for a in starts], [r + a % BLOCK for a, r in zip(starts, rows)]
    s["read"] = (_i32(starts), _offsets(rows), max(rows), sum(rows))
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_values(data, scales, kind, D):
    """Codes of blocks [..., 2, 32 D] and their scales [..., 2]: fp32 values of K and V [..., 32 tokens, D]."""
    c = data.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).float()
    lead, n = c.shape[:-2], c.dim() - 2
    at = list(range(n))
    k = c[..., 0, :].reshape(*lead, D // 32, 2, 32, 16).permute(*at, n + 2, n, n + 1, n + 3).reshape(*lead, 32, D)
    v = c[..., 1, :].reshape(*lead, D // 32, 2, 32, 4, 4).permute(*at, n + 3, n + 1, n + 4, n, n + 2).reshape(*lead, 32, D)
    a = scales.abs()
    return k * a[..., 0, None, None], v * a[..., 1, None, None]


def _plain_codes(k, v, kind, D):
    """The other way for values that are codes already: [..., 32 tokens, D] each to bytes [..., 2, 32 D]."""
    lead, n = k.shape[:-2], k.dim() - 2
    at = list(range(n))
    k = k.reshape(*lead, 32, D // 32, 2, 16).permute(*at, n + 1, n + 2, n, n + 3).reshape(*lead, 32 * D)
    v = v.reshape(*lead, 4, 2, 4, D // 32, 32).permute(*at, n + 3, n + 1, n + 4, n, n + 2).reshape(*lead, 32 * D)
    return torch.stack([k, v], -2).to(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).view(torch.uint8)


def _plain_scale(amax, kind):
    if kind == "int8":
        return (amax / 127).clamp(min=2.0 ** -100)
    m, e = torch.frexp(amax)                                          # amax = m 2^e, m in [1/2, 1); 448 = 7/8 of 2^9
    return torch.ldexp(torch.ones_like(amax), torch.where(m <= 0.875, e - 9, e - 8).clamp(-100, 120))


def _plain_blocks(s, starts, row_off, max_rows):
    """Blocks that rows [starts, +n) of every sequence touch, the same number for all: page, block in it, the positions of
    its tokens [S, blocks, 32], the rows they belong to, and which of them are rows at all."""
    page = s["case"]["page"]
    per = (max_rows + BLOCK - 2) // BLOCK + 1
    first, n = starts.long() // BLOCK, (row_off[1:] - row_off[:-1]).long()
    block = first[:, None] + torch.arange(per, device=DEV)
    pos = block[..., None] * BLOCK + torch.arange(BLOCK, device=DEV)
    i = pos - starts.long()[:, None, None]
    mine = (i >= 0) & (i < n[:, None, None])
    at = (block // (page // BLOCK)).clamp(max=s["table"].shape[1] - 1)
    return s["table"].long().gather(1, at), block % (page // BLOCK), pos, (i + row_off[:-1].long()[:, None, None]) * mine, mine


def _plain_write(s):
    case = s["case"]
    kind, D = case["cache"], case["dim"]
    pg, blk, pos, row, mine = _plain_blocks(s, s["starts"], s["row_off"], s["max_rows"])
    used = mine.any(2)
    pg, blk, pos, row, mine = pg[used], blk[used], pos[used], row[used], mine[used]            # [blocks, ...]
    start = s["starts"].long()[:, None].expand(used.shape)[used]
    fresh = pos[:, 0] >= start
    old_scale = s["scales"][pg, :, blk]                                                       # [blocks, heads, 2]
    ok, ov = _plain_values(s["data"][pg, :, blk], old_scale, kind, D)
    kept = (pos < start[:, None])[:, None, :, None]
    mine4 = mine[:, None, :, None]
    codes, scales = [], []
    for x, old, so in ((s["k"], ok, old_scale[..., 0]), (s["v"], ov, old_scale[..., 1])):
        new = x[row].float().permute(0, 2, 1, 3)                                              # [blocks, heads, 32, D]
        amax = torch.where(mine4 & torch.isfinite(new), new.abs(), 0.0).amax((2, 3))
        sc = _plain_scale(amax, kind)
        sc = torch.where(fresh[:, None], sc, torch.maximum(sc, so.abs()))
        nan = (mine4 & torch.isnan(new)).any(3).any(2) | ((so < 0) & ~fresh[:, None])
        y = torch.where(mine4, new, torch.where(kept, old, 0.0)) / sc[..., None, None]
        y = y.clamp(-448, 448) if kind == "e4m3" else torch.where(torch.isnan(y), -128.0, y.round().clamp(-127, 127))
        codes.append(y)
        scales.append(torch.where(nan, -sc, sc))
    s["data"][pg, :, blk] = _plain_codes(codes[0], codes[1], kind, D)
    s["scales"][pg, :, blk] = torch.stack(scales, -1)


def _plain_read(s):
    case = s["case"]
    starts, row_off, max_rows, T = s["read"]
    pg, blk, pos, row, mine = _plain_blocks(s, starts, row_off, max_rows)
    k, v = _plain_values(s["data"][pg, :, blk], s["scales"][pg, :, blk], case["cache"], case["dim"])
    dtype = FLOATS[case["type"]]
    out = []
    for x in (k, v):
        o = torch.empty((T, case["heads"], case["dim"]), dtype=dtype, device=DEV)
        o[row[mine]] = x.permute(0, 1, 3, 2, 4)[mine].to(dtype)
        out.append(o)
    return out


def _plain_attend(s):
    case = s["case"]
    S, H, D, G = case["S"], case["heads"], case["dim"], case["group"]
    table, lens, row_off, n_max = s["table"].long(), s["lens"].long(), s["row_off"].long(), s["max_rows"]
    k, v = _plain_values(s["data"][table], s["scales"][table], case["cache"], D)              # [S, width, H, blocks, 32, D]
    L = table.shape[1] * case["page"]
    k = k.permute(0, 2, 1, 3, 4, 5).reshape(S, H, L, D)
    v = v.permute(0, 2, 1, 3, 4, 5).reshape(S, H, L, D)
    n = row_off[1:] - row_off[:-1]
    i = torch.arange(n_max, device=DEV)
    mine = i < n[:, None]
    row = torch.where(mine, row_off[:-1, None] + i, 0)
    q = s["q"][row].float().view(S, n_max, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, n_max * G, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    t = torch.arange(L, device=DEV)
    base = (lens - n)[:, None]
    if s["tree"] is None:
        seen = t <= (base + i)[..., None]
    else:
        j = t - base                                                                          # [S, L]: the tree's node
        bit = (s["tree"][row][..., None] >> j.clamp(0, 63)[:, None, :]) & 1
        seen = (j < 0)[:, None, :] | ((bit == 1) & (j >= 0)[:, None, :] & (j < n[:, None])[:, None, :])
    seen = seen[:, None, :, None, :].expand(S, 1, n_max, G, L).reshape(S, 1, n_max * G, L)
    x = x.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(x, 3)
    p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    o = torch.matmul(p, v).view(S, H, n_max, G, D).permute(0, 2, 1, 3, 4).reshape(S, n_max, H * G, D)
    lse = lse.view(S, H, n_max, G).permute(0, 2, 1, 3).reshape(S, n_max, H * G)
    return o[mine].to(s["q"].dtype), lse[mine]


def _plain_sample(s):
    z, ids = s["logits"], s["ids"]
    V = z.shape[1]
    z = z.double()
    z = torch.where(torch.isnan(z), -math.inf, z)
    if ids is not None:                                                                       # ties go to the smaller id
        by_id = torch.argsort(ids)
        z, ids = z[:, by_id], ids[by_id]
    z, at = torch.sort(z, dim=1, descending=True, stable=True)
    T = s["temperature"].double()[:, None]
    greedy = ~(T > 0)
    w = torch.exp((z - z[:, :1]) / torch.where(greedy, 1.0, T))
    w = torch.where(z == z[:, :1], 1.0, w)
    n = torch.arange(V, device=DEV)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        w = torch.where((n < k) | (k <= 0), w, 0.0)
    w = torch.where(greedy & (n > 0), 0.0, w)
    c = w.cumsum(1)
    keep = w > 0
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        keep &= (c - w < p * c[:, -1:]) | (p >= 1) | (n == 0)
    if s["min_p"] is not None:
        keep &= (w >= s["min_p"].double()[:, None]) | (n == 0)
    w = torch.where(keep, w, 0.0)
    c = w.cumsum(1)
    total = c[:, -1:]
    j = torch.minimum((c <= s["u"].double()[:, None] * total).sum(1), keep.sum(1) - 1).clamp(min=0)[:, None]
    got = at.gather(1, j)
    token = got if ids is None else ids.long()[got]
    none = z[:, :1] == -math.inf
    logprob = torch.log(w.gather(1, j) / total)
    return {"ids": torch.where(none, -1, token)[:, 0].to(torch.int32),
            "logprob": torch.where(none, math.nan, logprob)[:, 0].float()}


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2605_27390_amd as ev
        if kind == "sample":
            token, logprob = ev.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                       min_p=s["min_p"], ids=s["ids"])
            return {"ids": token, "logprob": logprob}
        cache = ev.KVCache(s["data"].shape[0], case["page"], case["heads"], case["dim"], case["cache"], data=s["data"],
                           scales=s["scales"])
        if kind == "attend":
            o, lse = ev.kv_attention(s["q"], cache, s["table"], s["lens"], s["row_off"], s["max_rows"], max_len=s["max_len"],
                                     tree=s["tree"])
            return {"out": o, "lse": lse}
        if kind == "write":
            ev.kv_write(cache, s["k"], s["v"], s["table"], s["starts"], s["row_off"], s["max_rows"])
        starts, row_off, max_rows, T = s["read"]
        k, v = ev.kv_read(cache, s["table"], starts, row_off, max_rows, T, FLOATS[case["type"]])
    elif kind == "sample":
        return _plain_sample(s)
    elif kind == "attend":
        o, lse = _plain_attend(s)
        return {"out": o, "lse": lse}
    else:
        if kind == "write":
            _plain_write(s)
        k, v = _plain_read(s)
    return {"k": k, "v": v, "scales": s["scales"]} if kind == "write" else {"k": k, "v": v}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["type"]]
    if case["kind"] == "sample":
        return {"bytes": case["M"] * (case["V"] * size + 12), "flops": 0}
    H, D = case["heads"], case["dim"]
    starts, rows = _sizes(case)
    tokens = sum(rows)
    if case["kind"] == "read":
        return {"bytes": 2 * tokens * H * D * (1 + size), "flops": 0}
    if case["kind"] == "write":
        # the new tokens in, as codes out; the blocks that they touched in again, and out as values
        back = tokens + sum(a % BLOCK for a in starts)
        return {"bytes": 2 * H * D * (tokens * (size + 1) + back * (1 + size)), "flops": 0}
    G = case["group"]
    seen = sum(n * a + n * (n + 1) // 2 for a, n in zip(starts, rows))
    return {"bytes": 2 * H * D * (sum(starts) + tokens) + tokens * G * H * (2 * D * size + 4), "flops": 4 * seen * G * H * D}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_sequence(s, b, n):
    """The first n tokens of sequence b in 64 bits: K and V [n, heads, D]."""
    case = s["case"]
    H, D, page = case["heads"], case["dim"], case["page"]
    per = page // BLOCK
    blocks = torch.arange(-(-n // BLOCK), device=DEV)
    p = s["table"][b].long()[blocks // per]
    raw = s["data"][p, :, blocks % per].view(torch.float8_e4m3fn if case["cache"] == "e4m3" else torch.int8)   # [N, H, 2, 32 D]
    sc = s["scales"][p, :, blocks % per].double().abs()
    m, d = torch.arange(32, device=DEV)[:, None], torch.arange(D, device=DEV)[None, :]
    out = []
    for w, at in ((0, (d // 32) * 1024 + (d // 16 % 2) * 512 + m * 16 + d % 16),
                  (1, (d // 32) * 1024 + (m // 4 % 2) * 512 + d % 32 * 16 + m // 8 * 4 + m % 4)):
        x = raw[:, :, w].view(torch.uint8)[:, :, at].view(raw.dtype).double() * sc[:, :, w, None, None]        # [N, H, 32, D]
        out.append(x.permute(0, 2, 1, 3).reshape(-1, H, D)[:n])
    return out


def _exact_round(x, scale, kind):
    """x as a code of this scale stands for it."""
    y = x / scale
    if kind == "int8":
        return torch.round(y).clamp(-127, 127) * scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(min=-6) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448) * scale


def _exact_write(s):
    case = s["case"]
    kind, H, D = case["cache"], case["heads"], case["dim"]
    per = case["page"] // BLOCK
    starts, off = s["starts"].tolist(), s["row_off"].tolist()
    ks, vs, scales = [], [], s["scales"].double()
    for b in range(case["S"]):
        n, a = off[b + 1] - off[b], starts[b]
        lead = a % BLOCK
        first = a - lead
        old = _exact_sequence(s, b, a) if lead else None
        for w, (x, dst) in enumerate(((s["k"], ks), (s["v"], vs))):
            new = x[off[b]:off[b] + n].double()
            whole = torch.cat([old[w][first:a], new]) if lead else new                         # [lead + n, H, D]
            N = -(-(lead + n) // BLOCK)
            pad = torch.zeros((N * BLOCK, H, D), dtype=torch.float64, device=DEV)
            pad[lead:lead + n] = new
            amax = pad.view(N, BLOCK, H, D).abs().amax((1, 3))                                # [N, H]
            if kind == "int8":
                sc = (amax / 127).clamp(min=2.0 ** -100)
            else:
                sc = torch.exp2(torch.ceil(torch.log2((amax / 448).clamp(min=2.0 ** -100))))
            blocks = torch.arange(N, device=DEV) + first // BLOCK
            p = s["table"][b].long()[blocks // per]
            if lead:
                sc[0] = torch.maximum(sc[0], s["scales"][p[0], :, blocks[0] % per, w].double().abs())
            scales[p, :, blocks % per, w] = sc
            per_token = sc.repeat_interleave(BLOCK, 0)[:lead + n][..., None]
            dst.append(_exact_round(whole, per_token, kind))
    return {"k": torch.cat(ks), "v": torch.cat(vs), "scales": scales}


def _exact_sample(s):
    # one row after the other, on the numbers that can be drawn
    out = []
    M = s["logits"].shape[0]
    for m in range(M):
        z = s["logits"][m].double()
        at = torch.nonzero(z > -math.inf)[:, 0]
        z = z[at]
        if not z.numel():
            out.append(math.nan)
            continue
        T = float(s["temperature"][m].double())
        if not T > 0:
            out.append(0.0)
            continue
        token = at if s["ids"] is None else s["ids"].long()[at]
        # decreasing logits, then smaller ids: sorted by the second key first
        o = torch.argsort(token)
        o = o[torch.argsort(z[o], descending=True, stable=True)]
        lw = (z[o] - z.max()) / T
        if s["top_k"] is not None and int(s["top_k"][m]) > 0:
            lw = lw[:int(s["top_k"][m])]
        prob = torch.softmax(lw, 0)
        if s["top_p"] is not None and float(s["top_p"][m]) < 1:
            before = torch.cumsum(prob, 0) - prob
            lw = lw[:max(1, int((before < s["top_p"][m].double()).sum()))]
        if s["min_p"] is not None:
            lw = lw[:max(1, int((torch.exp(lw) >= s["min_p"][m].double()).sum()))]
        lp = torch.log_softmax(lw, 0)
        j = min(int((torch.cumsum(lp.exp(), 0) <= s["u"][m].double()).sum()), lp.numel() - 1)
        out.append(float(lp[j]))
    return {"ids": None, "logprob": torch.tensor(out, dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(s)
    if kind == "write":
        return _exact_write(s)
    if kind == "read":
        starts, off = s["starts"].tolist(), s["row_off"].tolist()
        ks, vs = [], []
        for b in range(case["S"]):
            k, v = _exact_sequence(s, b, starts[b] + off[b + 1] - off[b])
            ks.append(k[starts[b]:])
            vs.append(v[starts[b]:])
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    H, G, D = case["heads"], case["group"], case["dim"]
    lens, off = s["lens"].tolist(), s["row_off"].tolist()
    outs, lses = [], []
    for b in range(case["S"]):
        n, L = off[b + 1] - off[b], lens[b]
        k, v = _exact_sequence(s, b, L)
        q = s["q"][off[b]:off[b + 1]].double()
        t = torch.arange(L, device=DEV)
        i = torch.arange(n, device=DEV)[:, None]
        if s["tree"] is None:
            seen = t[None, :] - (L - n) <= i
        else:
            j = t[None, :] - (L - n)
            seen = (j < 0) | ((s["tree"][off[b]:off[b + 1], None] >> j.clamp(min=0)) & 1).bool()
        o = torch.empty((n, H * G, D), dtype=torch.float64, device=DEV)
        lse = torch.empty((n, H * G), dtype=torch.float64, device=DEV)
        for h in range(H):
            for a in range(h * G, h * G + G):
                x = (q[:, a] @ k[:, h].t().contiguous()) / math.sqrt(D)
                x = x.masked_fill(~seen, -math.inf)
                lse[:, a] = torch.logsumexp(x, 1)
                o[:, a] = torch.softmax(x, 1) @ v[:, h].contiguous()
        outs.append(o)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
