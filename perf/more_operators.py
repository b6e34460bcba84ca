"""The operators of one step of a continuous batch, as cases that can be timed and compared.

Between steps sequences share and give back cache pages: `fork_pages` (a child takes a parent's pages, the last partly
filled one as a copy) and `release_pages` (pages of finished or cut sequences return to the free list).  A step then runs
`norm_rope_kv_append` (norms of q and k per head, rotary positions, k and v into the cache) and `chunk_attention` (the new
tokens of all sequences, packed: one of a decode, thousands of a prompt) per layer, and `shape_logits` (penalties, biases,
grammar masks, probabilities) once.  Each operator is here in a plain form (`own` false: elementary torch operations) and
as the library's call.
"""
import math

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # beam search or parallel sampling over a small batch: 8 children of 4 parents
        dict(name="fork small", op="fork", batch=32, forks=8, parents=4, block_size=16, ctx_lo=100, ctx_hi=4000, cut=False,
             spare_pool=64),
        # a long shared prompt fans out: 512 children take prefixes of 32 long parents
        dict(name="fork prefixes", op="fork", batch=640, forks=512, parents=32, block_size=16, ctx_lo=4096, ctx_hi=32768,
             cut=True, spare_pool=4096),
        # a few requests end
        dict(name="release small", op="release", batch=64, rows=6, block_size=16, ctx_lo=100, ctx_hi=8192, shared=0.0,
             cut=False, spare_pool=64),
        # a large batch is cut back or ends, half of the pages shared with sequences of the list or outside it
        dict(name="release large", op="release", batch=600, rows=512, block_size=16, ctx_lo=1000, ctx_hi=16384, shared=0.5,
             cut=True, spare_pool=1000),
        # decode step of 64 requests, whole head rotated
        dict(name="norm rope decode", op="norm", tokens=64, hq=32, hkv=8, dim=128, rot=128, interleaved=False, block_size=16,
             pos_hi=8192, kv="bf16", offset=0.0, weights=True),
        # packed prompts into an 8-bit cache, long positions
        dict(name="norm rope prefill 8-bit", op="norm", tokens=16381, hq=64, hkv=8, dim=128, rot=128, interleaved=False,
             block_size=32, pos_hi=131072, kv="fp8", offset=0.0, weights=True),
        # tiny: 4 requests of at most 256 tokens, up to 8 new ones each
        dict(name="chunk tiny", op="chunk", batch=4, hq=8, hkv=2, dim=64, block_size=16, ctx_lo=8, ctx_hi=256, long_share=1.0,
             new_lo=1, new_hi=8, kv="bf16"),
        # a serving step: decodes and a few pieces of prompts in one call
        dict(name="chunk mixed batch", op="chunk", batch=64, hq=32, hkv=8, dim=128, block_size=16, ctx_lo=256, ctx_hi=8192,
             long_share=0.0625, new_lo=300, new_hi=700, kv="bf16"),
        # fresh prompts and pieces of long ones
        dict(name="chunk prefill", op="chunk", batch=5, hq=64, hkv=8, dim=128, block_size=32, ctx_lo=2000, ctx_hi=16000,
             long_share=1.0, new_lo=2000, new_hi=6000, kv="bf16"),
        # long contexts in an 8-bit cache, most with one new token, some with a few
        dict(name="chunk 8-bit long", op="chunk", batch=48, hq=40, hkv=8, dim=128, block_size=16, ctx_lo=4096, ctx_hi=32768,
             long_share=0.25, new_lo=5, new_hi=64, kv="fp8"),
        # one decode step's sampling: 4 requests, everything switched on
        dict(name="logits decode", op="logits", batch=4, nodes=1, vocab=128256, dtype="bf16", history=4096, bias=16, mask=True,
             penalties=True, greedy=0.25, both=False),
        # rows of 16-node draft trees before their verification
        dict(name="logits trees", op="logits", batch=16, nodes=16, vocab=152064, dtype="bf16", history=8192, bias=0, mask=True,
             penalties=True, greedy=0.0, both=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["fork", "release", "norm", "chunk", "chunk", "chunk", "logits", "logits"])
    bs = rng.choice([16, 16, 32, 64, 128, 256])
    if op == "fork":
        forks = _log(rng, 1, 512)
        hi = max(2, min(_log(rng, 16, 65536), bs * 32768 * 16 // max(32, forks)))
        parents = rng.randint(1, min(32, forks))
        return dict(op=op, batch=forks + parents + rng.randint(0, 90), forks=forks, parents=parents, block_size=bs,
                    ctx_lo=rng.choice([0, max(1, hi // 4)]), ctx_hi=hi, cut=rng.random() < 0.5, spare_pool=_log(rng, 1, 4096))
    if op == "release":
        rows = _log(rng, 1, 512)
        hi = max(2, min(_log(rng, 16, 32768), bs * 1024 * 512 // rows))
        return dict(op=op, batch=rows + rng.randint(0, 88), rows=rows, block_size=bs, ctx_lo=rng.choice([0, max(1, hi // 4)]),
                    ctx_hi=hi, shared=rng.choice([0.0, 0.3, 0.9]), cut=rng.random() < 0.5, spare_pool=_log(rng, 1, 4096))
    hq, hkv = rng.choice([(32, 8), (40, 8), (64, 8), (8, 8), (8, 2), (16, 1)])
    dim = rng.choice([64, 128, 128, 128])
    kv = rng.choice(["bf16", "bf16", "fp8"]) if dim == 128 else "bf16"
    if op == "norm":
        return dict(op=op, tokens=_log(rng, 1, 16384), hq=hq, hkv=hkv, dim=dim,
                    rot=rng.choice([dim, dim, 16 * rng.randint(1, dim // 16)]), interleaved=rng.random() < 0.5,
                    block_size=bs, pos_hi=_log(rng, 64, 1 << 20), kv=kv, offset=rng.choice([0.0, 1.0]),
                    weights=rng.random() < 0.8)
    if op == "chunk":
        batch = _log(rng, 1, 96)
        share = rng.choice([0.0, 0.1, 0.5, 1.0])
        new_hi = _log(rng, 1, 6000)
        hi = _log(rng, 16, 32768)
        # at most the largest listed case's products, and a cache of at most 4 GB
        while batch * (max(share, 1 / batch) * new_hi + 1) * max(hi, new_hi) * hq > 64 * 11000 * 11000 and batch > 1:
            batch = (batch + 1) // 2
        while batch * (max(share, 1 / batch) * new_hi + 1) * max(hi, new_hi) * hq > 64 * 11000 * 11000:
            new_hi = (new_hi + 1) // 2
        hi = max(new_hi, min(hi, 1_000_000 // batch * 8 // hkv))
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, dim=dim, block_size=bs, ctx_lo=rng.choice([1, max(1, hi // 4)]),
                    ctx_hi=hi, long_share=share, new_lo=rng.choice([0, max(1, new_hi // 3)]), new_hi=new_hi, kv=kv)
    vocab = _log(rng, 500, 200000)
    nodes = rng.choice([1, 1, _log(rng, 2, 24)])
    batch = max(1, min(_log(rng, 1, 256), 256 * 152064 // (vocab * nodes)))
    return dict(op=op, batch=batch, nodes=nodes, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp32"]),
                history=_log(rng, 16, 16384), bias=rng.choice([0, 0, _log(rng, 1, 256)]), mask=rng.random() < 0.5,
                penalties=rng.random() < 0.7, greedy=rng.choice([0.0, 0.0, 0.5]), both=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(g, lo, hi, shape):
    """Whole numbers of [lo, hi]."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV, dtype=torch.int32)


def _quantiles(lo, hi, n):
    """n lengths spread evenly over the logarithm of [lo, hi]: a case's work does not depend on the seed."""
    a, b = math.log(max(1, lo)), math.log(max(1, lo, hi))
    x = [max(lo, min(hi, int(round(math.exp(a + (b - a) * (i + 0.5) / n))))) for i in range(n)]
    return x if lo > 0 or n < 4 else [0] + x[1:]


def _shuffled(g, values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)[torch.randperm(len(values), generator=g, device=DEV)]


def _table(g, blocks_of, width, spare):
    """Distinct shuffled blocks for every sequence: (table [B, width] padded with -1, free blocks, pool size)."""
    used = int(blocks_of.sum())
    pool = used + spare
    perm = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    first = torch.cumsum(blocks_of, 0) - blocks_of
    j = torch.arange(width, device=DEV)
    at = (first[:, None] + j).clamp(max=pool - 1)
    return torch.where(j < blocks_of[:, None], perm[at], -1).to(torch.int32).contiguous(), perm[used:].contiguous(), pool


def _pool(g, pool, c):
    shape = (pool, c["hkv"], c["block_size"], c["dim"])
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return (x * 16).to(torch.float8_e4m3fn).view(torch.uint8) if c["kv"] == "fp8" else x


def _i32(*shape):
    return torch.empty(shape, dtype=torch.int32, device=DEV)


def _prepare_fork(c, g):
    B, F, P, bs = c["batch"], c["forks"], c["parents"], c["block_size"]
    order = torch.randperm(B, generator=g, device=DEV)
    child, kin, others = order[:F], order[F:F + P], order[F + P:]
    ctx = torch.zeros(B, dtype=torch.int32, device=DEV)
    ctx[kin] = _shuffled(g, _quantiles(c["ctx_lo"], c["ctx_hi"], P))
    ctx[others] = _shuffled(g, _quantiles(1, 50, max(1, others.numel())))[: others.numel()]
    held = (ctx.long() + bs - 1) // bs
    table, free, pool = _table(g, held, max(1, (c["ctx_hi"] + bs - 1) // bs) + 2, F + c["spare_pool"])
    parent = kin[torch.arange(F, device=DEV) % P]
    share = torch.rand(F, generator=g, device=DEV, dtype=torch.float64)
    lens = (ctx[parent].double() * (0.5 + 0.5 * share)).int() if c["cut"] else None
    return dict(ctx=ctx, held=held.int(), table=table, free=free, pool=pool, parent=parent.int(), child=child.int(), lens=lens,
                head=torch.full((1,), min(3, c["spare_pool"]), dtype=torch.int32, device=DEV),
                shares=torch.zeros(pool, dtype=torch.int32, device=DEV),
                outs=dict(context_lens_out=_i32(B), blocks_held_out=_i32(B), free_head_out=_i32(1), shares_out=_i32(pool)),
                copy_src=_i32(F), copy_dst=_i32(F), granted=_i32(F))


def _prepare_release(c, g):
    B, n, bs = c["batch"], c["rows"], c["block_size"]
    order = torch.randperm(B, generator=g, device=DEV)
    ctx = torch.zeros(B, dtype=torch.int32, device=DEV)
    ctx[order[:n]] = _shuffled(g, _quantiles(c["ctx_lo"], c["ctx_hi"], n))
    ctx[order[n:]] = _shuffled(g, _quantiles(1, max(1, c["ctx_hi"] // 2), max(1, B - n)))[: B - n]
    held = (ctx.long() + bs - 1) // bs
    width = max(1, (c["ctx_hi"] + bs - 1) // bs) + 1
    table, _, pool = _table(g, held, width, c["spare_pool"])
    if c["shared"]:   # a share of the sequences have a prefix of another's pages
        kin = torch.randint(0, B, (B,), generator=g, device=DEV)
        u = torch.rand(B, generator=g, device=DEV)
        common = torch.where(u < c["shared"], (torch.minimum(held, held[kin]) * (u / c["shared"])).long(), 0)
        common[torch.arange(B, device=DEV) % 3 == 0] = 0     # these rows keep pages of their own
        kin = kin - kin % 3
        common = torch.minimum(common, held[kin])
        j = torch.arange(width, device=DEV)
        table = torch.where(j < common[:, None], table[kin], table).contiguous()
    live = torch.arange(width, device=DEV) < held[:, None]
    uses = torch.bincount(table[live].long(), minlength=pool)
    dead = torch.nonzero(uses == 0).view(-1).int()           # free pages
    free = torch.full((pool,), -1, dtype=torch.int32, device=DEV)
    head = pool - dead.numel()
    free[head:] = dead
    rows = order[:n].int()
    share = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    keep = (ctx[order[:n]].double() * torch.where(share < 0.3, share, 0.0)).int() if c["cut"] else None
    return dict(ctx=ctx, held=held.int(), table=table, free=free, pool=pool, rows=rows, keep=keep,
                head=torch.full((1,), head, dtype=torch.int32, device=DEV), shares=(uses - 1).clamp(min=0).int(),
                outs=dict(context_lens_out=_i32(B), blocks_held_out=_i32(B), free_head_out=_i32(1), shares_out=_i32(pool)))


def _prepare_norm(c, g):
    T, hq, hkv, D, bs = c["tokens"], c["hq"], c["hkv"], c["dim"], c["block_size"]
    # heads of different magnitude, as projections give them
    qkv = torch.randn((T, hq + 2 * hkv, D), generator=g, device=DEV)
    qkv *= torch.exp(torch.randn((1, hq + 2 * hkv, 1), generator=g, device=DEV))
    qkv = qkv.to(torch.bfloat16)
    blocks = (T + bs - 1) // bs + 2
    j = torch.arange(c["rot"] // 2, dtype=torch.float64)
    s = dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], eps=1e-6,
             inv_freq=(1.0 / (1e6 ** (2 * j / c["rot"]))).float().to(DEV), positions=_ints(g, 0, c["pos_hi"] - 1, (T,)),
             slots=torch.randperm(blocks * bs, generator=g, device=DEV)[:T].int(), blocks=blocks,
             q_out=torch.empty((T, hq, D), dtype=torch.bfloat16, device=DEV), k_scale=0.02, v_scale=0.02)
    s["qw"], s["kw"] = (((1 - c["offset"]) + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16)
                        if c["weights"] else None for _ in range(2))
    s["k_cache"], s["v_cache"] = (_pool(g, blocks, c) for _ in range(2))
    return s


def _chunk_lens(c):
    """(new tokens, contexts with them) of the case's sequences; the longest contexts do not go with the longest chunks."""
    B = c["batch"]
    n_long = max(1 if c["long_share"] else 0, round(B * c["long_share"]))
    new = [1] * (B - n_long) + (_quantiles(c["new_lo"], c["new_hi"], n_long) if n_long else [])
    ctx = _quantiles(c["ctx_lo"], c["ctx_hi"], B)
    ctx = [ctx[(i * 7 + 3) % B] if math.gcd(7, B) == 1 else ctx[B - 1 - i] for i in range(B)]
    return new, [max(t, n) for t, n in zip(ctx, new)]


def _prepare_chunk(c, g):
    B, hq, D, bs = c["batch"], c["hq"], c["dim"], c["block_size"]
    new, ctx = _chunk_lens(c)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(g.initial_seed())).tolist()
    new, ctx = [new[i] for i in order], [ctx[i] for i in order]
    lens = torch.tensor(ctx, dtype=torch.int32, device=DEV)
    held = (lens.long() + bs - 1) // bs
    table, _, pool = _table(g, held, (max(ctx) + bs - 1) // bs, 5)
    first = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().to(DEV)
    rows = sum(new) + 3                                       # a few padding rows behind the last sequence
    s = dict(new_host=new, ctx_host=ctx, ctx=lens, table=table, pool=pool, first=first, scale=1.0 / math.sqrt(D),
             q=torch.randn((rows, hq, D), generator=g, device=DEV).to(torch.bfloat16),
             out=torch.zeros((rows, hq, D), dtype=torch.bfloat16, device=DEV), k_scale=1 / 16, v_scale=1 / 16)
    s["k_cache"], s["v_cache"] = (_pool(g, pool, c) for _ in range(2))
    return s


def _parents(g, batch, nodes):
    """A tree per row: node 0 is the root, node i hangs below one of the nodes before it."""
    u = torch.rand((batch, nodes), generator=g, device=DEV)
    i = torch.arange(nodes, device=DEV, dtype=torch.float32)
    return torch.minimum((u * i).to(torch.int32), (i - 1).clamp(min=0).to(torch.int32)).sub_((i == 0).to(torch.int32))


def _prepare_logits(c, g):
    B, N, V, L = c["batch"], c["nodes"], c["vocab"], c["history"]
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    u = lambda *n: torch.rand(n, generator=g, device=DEV)  # noqa: E731
    words = (V + 31) // 32
    s = dict(logits=torch.randn((B, N, V), generator=g, device=DEV).mul_(3).to(t), temperature=0.5 + u(B),
             probs=torch.empty((B, N, V), device=DEV), out=torch.empty((B, N, V), device=DEV) if c["both"] else None)
    s["temperature"] = torch.where(u(B) < c["greedy"], 0.0, s["temperature"])
    # words repeat: a few make up most of a text
    s["history"] = (V * u(B, L) ** 4).int().clamp(max=V - 1) if c["penalties"] else None
    s["lens"] = _ints(g, L // 2, L, (B,)) if c["penalties"] else None
    s["prompt"] = (s["lens"] * u(B)).int() if c["penalties"] else None
    s["repetition"] = 1.0 + 0.3 * u(B) if c["penalties"] else None
    s["frequency"] = 0.3 * u(B) if c["penalties"] else None
    s["presence"] = 0.5 * u(B) if c["penalties"] else None
    tree = N > 1 and c["penalties"]
    s["parents"] = _parents(g, B, N).contiguous() if tree else None
    s["tokens"] = _ints(g, 0, V - 1, (B, N)) if tree else None
    s["bias_tokens"] = s["bias_values"] = s["mask"] = None
    if c["bias"]:
        s["bias_tokens"] = torch.stack([torch.randperm(V, generator=g, device=DEV)[: c["bias"]] for _ in range(B)]).int()
        s["bias_values"] = torch.randn(s["bias_tokens"].shape, generator=g, device=DEV) * 5
    if c["mask"]:     # what a grammar allows: at some places nearly everything, at others next to nothing
        a, b = (torch.randint(-2**31, 2**31, (B, N, words), generator=g, device=DEV, dtype=torch.int64).int() for _ in range(2))
        s["mask"] = torch.where(u(B, N, 1) < 0.5, a | b, a & b).contiguous()
    return s


def prepare(case, seed):
    c = dict(case)
    s = {"fork": _prepare_fork, "release": _prepare_release, "norm": _prepare_norm, "chunk": _prepare_chunk,
         "logits": _prepare_logits}[c["op"]](c, _gen(seed))
    s["case"] = c
    if own and c["op"] != "logits":
        from paper_2511_21862_b200 import batch, binding, spec
        hkv, D, bs = c.get("hkv", 1), c.get("dim", 128), c["block_size"]
        table = s.get("table")
        shape = s["shape"] = binding.Shape(c.get("batch", 1), c.get("hq", hkv), hkv, D, bs, s.get("pool", s.get("blocks")),
                                           1 if table is None else table.shape[1], hkv * bs * D, bs * D, D)
        if c["op"] in ("fork", "release"):
            n = c.get("forks", c.get("rows"))
            s["workspace"] = torch.empty(batch.pages_workspace_bytes(shape, n), dtype=torch.uint8, device=DEV)
        if c["op"] == "norm":
            s["rope"] = spec.Rope(c["rot"], c["interleaved"], s["inv_freq"], 1.0)
            s["norm"] = batch.HeadNorm(s["eps"], s["qw"], s["kw"], c["offset"])
        if c["op"] == "chunk":
            s["workspace"] = torch.empty(batch.chunk_workspace_bytes(shape, s["q"].shape[0], max(s["new_host"])), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _fork(s):
    bs = s["case"]["block_size"]
    parent, child = s["parent"].long(), s["child"].long()
    lens = s["ctx"][parent] if s["lens"] is None else torch.minimum(s["lens"], s["ctx"][parent])
    full, part = lens.long() // bs, (lens % bs > 0).long()
    upto = s["head"].long() + torch.cumsum(part, 0)
    ok = (part == 0) | (upto <= s["free"].numel())
    j = torch.arange(s["table"].shape[1], device=DEV)
    whole = (j < full[:, None]) & ok[:, None]
    tail = (j == full[:, None]) & (part > 0)[:, None] & ok[:, None]
    fresh = s["free"][(upto - 1).clamp(0, s["free"].numel() - 1)]
    kin = s["table"][parent]
    table = s["table"].clone()
    table[child] = torch.where(whole, kin, torch.where(tail, fresh[:, None], table[child]))
    shares = s["shares"] + torch.bincount(kin[whole].long(), minlength=s["pool"]).int()
    ctx, held = s["ctx"].clone(), s["held"].clone()
    ctx[child] = torch.where(ok, lens, ctx[child])
    held[child] = torch.where(ok, (full + part).int(), held[child])
    copies = ok & (part > 0)
    src = torch.gather(kin, 1, full.clamp(max=j.numel() - 1)[:, None])[:, 0]
    return dict(table=table, ctx=ctx, held=held, head=(s["head"] + (part * ok).sum()).int(), shares=shares,
                copy_src=torch.where(copies, src, -1).int(), copy_dst=torch.where(copies, fresh, -1).int(), granted=ok.int())


def _release(s):
    bs = s["case"]["block_size"]
    rows = s["rows"].long()
    keep = torch.zeros_like(s["rows"]) if s["keep"] is None else s["keep"]
    stay = torch.minimum((keep.long() + bs - 1) // bs, s["held"][rows].long())
    j = torch.arange(s["table"].shape[1], device=DEV)
    gone = (j >= stay[:, None]) & (j < s["held"][rows][:, None])
    ids = s["table"][rows][gone].long()                      # in the order of the list, then of the tables
    uses = torch.bincount(ids, minlength=s["pool"])
    left = s["shares"] - uses
    freed = (left < 0) & (uses > 0)
    # the first place at which a freed page stands
    at = torch.full((s["pool"],), ids.numel(), device=DEV).scatter_reduce_(0, ids, torch.arange(ids.numel(), device=DEV), "amin")
    out = ids[torch.sort(at[freed]).values].int()
    free = s["free"].clone()
    head = s["head"].long()
    free[torch.arange(out.numel(), device=DEV) + head - out.numel()] = out
    ctx, held = s["ctx"].clone(), s["held"].clone()
    ctx[rows] = torch.minimum(ctx[rows], keep)
    held[rows] = stay.int()
    return dict(free=free, ctx=ctx, held=held, head=(head - out.numel()).int(), shares=left.clamp(min=0).int())


def _turn(x, cos, sin, rot, interleaved):
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y[..., : rot // 2], y[..., rot // 2: rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _stored(x, scale, like):
    if like.dtype == torch.uint8:
        return (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.to(torch.bfloat16)


def _values(cache):
    """A cache as the values that it stands for (an 8-bit one without its scale)."""
    return cache.view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache


def _norm(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))

    def head(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
        if w is not None:
            x = x * (w.float() + c["offset"])
        return _turn(x, cos, sin, c["rot"], c["interleaved"])

    q, k = head(s["q"], s["qw"]).to(torch.bfloat16), head(s["k"], s["kw"])
    blk, off = s["slots"].long() // c["block_size"], s["slots"].long() % c["block_size"]
    s["k_cache"][blk, :, off] = _stored(k, s["k_scale"], s["k_cache"])
    s["v_cache"][blk, :, off] = _stored(s["v"].float(), s["v_scale"], s["v_cache"])
    return dict(q=q, k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]))


def _chunk(s):
    c = s["case"]
    hq, hkv, D, bs = c["hq"], c["hkv"], c["dim"], c["block_size"]
    G, fp8, out, at = hq // hkv, c["kv"] == "fp8", s["out"], 0
    out = out.clone()
    for b, (n, T) in enumerate(zip(s["new_host"], s["ctx_host"])):
        if n == 0:
            continue
        ids = s["table"][b, : (T + bs - 1) // bs].long()
        pos = torch.arange(T - n, T, device=DEV)
        for h in range(hkv):
            k, v = (_values(x[ids, h]).float().flatten(0, 1)[:T] for x in (s["k_cache"], s["v_cache"]))
            if fp8:
                k, v = k * s["k_scale"], v * s["v_scale"]
            q = s["q"][at:at + n, h * G:(h + 1) * G].float().reshape(-1, D)
            w = (q @ k.T).mul_(s["scale"]).view(n, G, T)
            if n > 1:
                w.masked_fill_((torch.arange(T, device=DEV) > pos[:, None])[:, None], -math.inf)
            w = w.sub_(w.amax(-1, keepdim=True)).exp_()
            w /= w.sum(-1, keepdim=True)
            out[at:at + n, h * G:(h + 1) * G] = (w.view(-1, T) @ v).view(n, G, D).to(torch.bfloat16)
        at += n
    return out


def _counts(s, dtype):
    """(truth values: the token is in the request's text, generated or drafted occurrences), both [B, N, V]."""
    c = s["case"]
    B, N, V, L = c["batch"], c["nodes"], c["vocab"], c["history"]
    j = torch.arange(L, device=DEV)
    live, fresh = j < s["lens"][:, None], (j >= s["prompt"][:, None]) & (j < s["lens"][:, None])
    at = s["history"].long()
    seen = torch.zeros((B, V), dtype=dtype, device=DEV).scatter_add_(1, at, live.to(dtype))
    made = torch.zeros((B, V), dtype=dtype, device=DEV).scatter_add_(1, at, fresh.to(dtype))
    seen, made = (x[:, None].expand(B, N, V).clone() if N > 1 else x[:, None] for x in (seen, made))
    if s["parents"] is not None:     # the drafts above a node and its own; the root is in the history
        up = torch.arange(N, device=DEV).expand(B, N)
        for _ in range(N):
            on = up > 0
            tok = torch.gather(s["tokens"].long(), 1, up.clamp(min=0))
            for x in (seen, made):
                x.scatter_add_(2, tok[:, :, None], on[:, :, None].to(dtype))
            up = torch.where(on, torch.gather(s["parents"].long(), 1, up.clamp(min=0)), up)
    return seen > 0, made


def _logits(s):
    c = s["case"]
    V = c["vocab"]
    x = s["logits"].float()
    if c["penalties"]:
        seen, made = _counts(s, torch.float32)
        r, f, p = (s[k][:, None, None] for k in ("repetition", "frequency", "presence"))
        x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
        x = x - f * made - p * (made > 0)
    if c["bias"]:
        at = s["bias_tokens"].long()[:, None].expand(-1, c["nodes"], -1)
        x = x.scatter_add(2, at, s["bias_values"][:, None].expand(-1, c["nodes"], -1))
    if c["mask"]:
        bit = (s["mask"][..., None] >> torch.arange(32, device=DEV)) & 1
        x = torch.where(bit.flatten(2)[..., :V] > 0, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    t = s["temperature"][:, None, None]
    w = torch.exp((x - top) / torch.where(t > 0, t, 1.0))
    w = w / w.sum(-1, keepdim=True)
    first = torch.arange(V, device=DEV) == torch.where(x == top, torch.arange(V, device=DEV), V).amin(-1, keepdim=True)
    w = torch.where(t > 0, w, first.float())
    w = torch.where(top > -math.inf, w, 0.0)
    return dict(probs=w, logits=x) if c["both"] else dict(probs=w)


# ------------------------------------------------------------------------------------------------ the library's calls
def _own(s):
    from paper_2511_21862_b200 import batch
    c = s["case"]
    op, fp8 = c["op"], c.get("kv") == "fp8"
    if op == "fork":
        batch.fork_pages(s["shape"], s["parent"], s["child"], s["ctx"], s["table"], s["held"], s["free"], s["head"], s["shares"],
                         s["copy_src"], s["copy_dst"], s["granted"], s["workspace"], shared_lens=s["lens"], **s["outs"])
        o = s["outs"]
        return dict(table=s["table"], ctx=o["context_lens_out"], held=o["blocks_held_out"], head=o["free_head_out"],
                    shares=o["shares_out"], copy_src=s["copy_src"], copy_dst=s["copy_dst"], granted=s["granted"])
    if op == "release":
        batch.release_pages(s["shape"], s["rows"], s["ctx"], s["table"], s["held"], s["free"], s["head"], s["shares"],
                            s["workspace"], keep_lens=s["keep"], **s["outs"])
        o = s["outs"]
        return dict(free=s["free"], ctx=o["context_lens_out"], held=o["blocks_held_out"], head=o["free_head_out"],
                    shares=o["shares_out"])
    if op == "norm":
        if fp8:
            batch.norm_rope_kv_append_fp8(s["shape"], s["rope"], s["norm"], s["q"], s["k"], s["v"], s["positions"], s["slots"],
                                          s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        else:
            batch.norm_rope_kv_append(s["shape"], s["rope"], s["norm"], s["q"], s["k"], s["v"], s["positions"], s["slots"],
                                      s["q_out"], s["k_cache"], s["v_cache"])
        return dict(q=s["q_out"], k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]))
    if op == "chunk":
        if fp8:
            batch.chunk_attention_fp8(s["shape"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["first"],
                                      max(s["new_host"]), s["scale"], s["k_scale"], s["v_scale"], s["out"], s["workspace"])
        else:
            batch.chunk_attention(s["shape"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["first"],
                                  max(s["new_host"]), s["scale"], s["out"], s["workspace"])
        return s["out"]
    batch.shape_logits(s["logits"], probs=s["probs"], out=s["out"], temperature=s["temperature"], repetition=s["repetition"],
                       frequency=s["frequency"], presence=s["presence"], history=s["history"], history_lens=s["lens"],
                       prompt_lens=s["prompt"], tokens=s["tokens"], parents=s["parents"], bias_tokens=s["bias_tokens"],
                       bias_values=s["bias_values"], mask=s["mask"])
    return dict(probs=s["probs"], logits=s["out"]) if c["both"] else dict(probs=s["probs"])


def run(state):
    if own:
        return _own(state)
    return {"fork": _fork, "release": _release, "norm": _norm, "chunk": _chunk, "logits": _logits}[state["case"]["op"]](state)


def work(case):
    c, op = case, case["op"]
    B = c.get("batch", 1)
    if op == "fork":
        # a child's entries are read at the parent and written, and a count is raised for each; lengths and pages held of all
        # sequences and all counts in and out
        lens = _quantiles(c["ctx_lo"], c["ctx_hi"], c["parents"])
        pages = sum(lens) / c["parents"] * c["forks"] * (0.75 if c["cut"] else 1.0) / c["block_size"]
        pool = (sum(lens) + 13 * (B - c["forks"] - c["parents"])) / c["block_size"] + c["forks"] + c["spare_pool"]
        return dict(bytes=8 * pages + 16 * B + 8 * pool + 24 * c["forks"], flops=pages)
    if op == "release":
        # the released entries and their places in the free list, all counts in and out, lengths and pages held of all
        pages = sum(_quantiles(c["ctx_lo"], c["ctx_hi"], c["rows"])) / c["block_size"]
        pool = pages + sum(_quantiles(1, max(1, c["ctx_hi"] // 2), max(1, B - c["rows"]))) / c["block_size"] + c["spare_pool"]
        return dict(bytes=8 * pages * (1 - 0.5 * c["shared"]) + 8 * pool + 16 * B + 8 * c["rows"], flops=pages)
    if op == "norm":
        cell = 1 if c["kv"] == "fp8" else 2
        rows = c["tokens"] * c["dim"]
        return dict(bytes=rows * (2 * c["hq"] * 2 + 2 * c["hkv"] * (2 + cell)) + 8 * c["tokens"],
                    flops=rows * (c["hq"] + c["hkv"]) * 4 + 3 * c["tokens"] * c["rot"] * (c["hq"] + c["hkv"]))
    if op == "chunk":
        cell = 1 if c["kv"] == "fp8" else 2
        new, ctx = _chunk_lens(c)
        pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(new, ctx))
        held = sum(t for n, t in zip(new, ctx) if n)
        return dict(bytes=2 * cell * c["hkv"] * c["dim"] * held + 4 * sum(new) * c["hq"] * c["dim"] + 4 * held / c["block_size"] +
                    12 * B, flops=4 * c["hq"] * c["dim"] * pairs)
    rows = B * c["nodes"]
    cell = 2 if c["dtype"] == "bf16" else 4
    return dict(bytes=rows * c["vocab"] * (cell + 4 * (2 if c["both"] else 1) + (0.125 if c["mask"] else 0)) +
                (3 * B * c["history"] if c["penalties"] else 0) + 8 * B * c["bias"], flops=8.0 * rows * c["vocab"])


# ------------------------------------------------------------------------------------------------ definitions in 64 bits
def exact(case, seed):
    """Normed and turned rows, attention rows (one head of a sequence at a time) and probabilities in 64 bits; the page
    operators give whole numbers."""
    op = case["op"]
    if op in ("fork", "release"):
        return None
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"norm": _exact_norm, "chunk": _exact_chunk, "logits": _exact_logits}[op](s, case)


def _exact_norm(s, c):
    bs, rot = c["block_size"], c["rot"]
    angle = torch.outer(s["positions"].to(torch.float64), s["inv_freq"].to(torch.float64))
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x, w):
        x = x.to(torch.float64)
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["dim"] + s["eps"])
        if w is not None:
            x = x * (w.to(torch.float64) + c["offset"])
        head, tail = x[..., :rot], x[..., rot:]
        if c["interleaved"]:
            z = torch.view_as_complex(head.unflatten(-1, (rot // 2, 2)).contiguous()) * turn
            head = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(head[..., : rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
            head = torch.cat([z.real, z.imag], -1)
        return torch.cat([head, tail], -1)

    def placed(cache, rows, scale):
        fp8 = cache.dtype == torch.uint8
        y = (cache.view(torch.float8_e4m3fn) if fp8 else cache).to(torch.float64).permute(0, 2, 1, 3).flatten(0, 1)
        y[s["slots"].long()] = (rows / scale).clamp(-448, 448) if fp8 else rows
        return y.unflatten(0, (-1, bs)).permute(0, 2, 1, 3).contiguous()

    return dict(q=turned(s["q"], s["qw"]), k_cache=placed(s["k_cache"], turned(s["k"], s["kw"]), s["k_scale"]),
                v_cache=placed(s["v_cache"], s["v"].to(torch.float64), s["v_scale"]))


def _exact_chunk(s, c):
    hq, hkv, bs = c["hq"], c["hkv"], c["block_size"]
    fp8, out = c["kv"] == "fp8", s["out"].to(torch.float64)
    first = s["first"].tolist()
    for b in range(c["batch"]):
        r0, n, T = first[b], first[b + 1] - first[b], int(s["ctx"][b])
        if n == 0:
            continue
        ids = s["table"][b, : (T + bs - 1) // bs].long()
        see = torch.arange(T, device=DEV) - (T - n) <= torch.arange(n, device=DEV)[:, None]
        for h in range(hq):
            k, v = ((x[ids, h // (hq // hkv)].view(torch.float8_e4m3fn).to(torch.float64) * sc if fp8 else
                     x[ids, h // (hq // hkv)].to(torch.float64)).reshape(-1, c["dim"])[:T]
                    for x, sc in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])))
            w = (s["q"][r0:r0 + n, h].to(torch.float64) @ k.T) * s["scale"]
            out[r0:r0 + n, h] = torch.softmax(w.masked_fill_(~see, -math.inf), -1) @ v
    return out


def _exact_logits(s, c):
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    x = s["logits"].to(torch.float64)
    if c["penalties"]:
        lens, prompt = s["lens"].tolist(), s["prompt"].tolist()
        tokens = s["tokens"].tolist() if s["tokens"] is not None else None
        up = s["parents"].tolist() if s["parents"] is not None else None
        for b in range(B):
            old, new = s["history"][b, : lens[b]].long(), s["history"][b, prompt[b]: lens[b]].long()
            for i in range(N):
                branch, k = [], i
                while up is not None and k > 0:
                    branch.append(tokens[b][k])
                    k = up[b][k]
                extra = torch.tensor(branch, dtype=torch.long, device=DEV)
                seen, made = (torch.bincount(torch.cat([t, extra]), minlength=V) for t in (old, new))
                r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
                y = x[b, i]
                y = torch.where(seen > 0, torch.where(y > 0, y / r, y * r), y)
                x[b, i] = y - f * made - p * (made > 0)
    if c["bias"]:
        for b in range(B):
            x[b, :, s["bias_tokens"][b].long()] += s["bias_values"][b].to(torch.float64)
    if c["mask"]:
        v = torch.arange(V, device=DEV)
        x[((s["mask"].long()[..., v // 32] >> (v % 32)) & 1) == 0] = -math.inf
    probs = torch.zeros_like(x)
    for b in range(B):
        t = float(s["temperature"][b])
        for i in range(N):
            if float(x[b, i].max()) == -math.inf:
                continue
            if t > 0:
                probs[b, i] = torch.softmax(x[b, i] / t, -1)
            else:
                probs[b, i, int(torch.nonzero(x[b, i] == x[b, i].max())[0])] = 1
    return dict(probs=probs, logits=x) if c["both"] else dict(probs=probs)
