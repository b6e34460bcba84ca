"""The operators of one speculative decoding step over the paged KV cache, as cases that can be timed and compared.

A step runs, in this order: `plan_slots` (blocks and slots for the new tokens), `rope_kv_append` (rotary positions of q
and k, k and v into the cache), `tree_attention` (every drafted token sees the context and its own branch),
`verify_drafts` (drafts against the target's probabilities) and `kv_keep_path` (the accepted branch moves together).
Each operator is here in a plain form (`own` false: elementary torch operations) and as the library's call.
"""
import math

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # 64 requests, each with a 16-node draft tree, about to run: the call before every speculative step
        dict(name="slots tree step", op="slots", batch=64, block_size=16, ctx_lo=256, ctx_hi=8192, new_lo=16, new_hi=16,
             row_len=16, tree=True),
        # a burst of prompts admitted at once, packed one behind the other
        dict(name="slots prompts", op="slots", batch=256, block_size=16, ctx_lo=1, ctx_hi=64, new_lo=8192, new_hi=32768,
             row_len=0, tree=False),
        # one speculative step of a small batch: 8 requests of 5 tokens, whole head rotated
        dict(name="rope small step", op="rope", tokens=40, hq=32, hkv=8, dim=128, rot=128, interleaved=False,
             block_size=16, pos_hi=8192, kv="bf16", stretch=1.0),
        # a prefill of 16384 packed tokens, long positions, scaled frequencies
        dict(name="rope prefill", op="rope", tokens=16384, hq=64, hkv=8, dim=128, rot=128, interleaved=False,
             block_size=32, pos_hi=131072, kv="bf16", stretch=8.0),
        # tiny: 4 requests of at most 256 tokens, 5 nodes each
        dict(name="tree tiny", op="tree", batch=4, hq=8, hkv=2, dim=64, block_size=16, ctx_lo=17, ctx_hi=256, nodes=5,
             ragged=False, kv="bf16"),
        # 64 requests of mixed lengths, 16 nodes each
        dict(name="tree mixed batch", op="tree", batch=64, hq=32, hkv=8, dim=128, block_size=16, ctx_lo=256, ctx_hi=8192,
             nodes=16, ragged=False, kv="bf16"),
        # few very long requests, wide trees
        dict(name="tree long", op="tree", batch=8, hq=64, hkv=8, dim=128, block_size=32, ctx_lo=32768, ctx_hi=65536,
             nodes=64, ragged=False, kv="bf16"),
        # 8-bit cache, five query heads per kv head, trees of different sizes in one padded batch
        dict(name="tree 8-bit ragged", op="tree", batch=32, hq=40, hkv=8, dim=128, block_size=16, ctx_lo=4096,
             ctx_hi=32768, nodes=8, ragged=True, kv="fp8"),
        # a chain of four drafts for 4 requests
        dict(name="verify chain", op="verify", batch=4, nodes=5, vocab=152064, chain=True, draft=True, ragged=False,
             noise=0.5),
        # 128 requests with 16-node trees drawn from a draft model
        dict(name="verify trees", op="verify", batch=128, nodes=16, vocab=128256, chain=False, draft=True, ragged=True,
             noise=0.5),
        # one layer's cache after the verification of a small batch
        dict(name="keep small", op="keep", batch=8, hkv=8, dim=128, block_size=16, ctx_lo=64, ctx_hi=2048, nodes=8,
             kv="bf16"),
        # ... and of a large one with long accepted branches
        dict(name="keep large", op="keep", batch=512, hkv=8, dim=128, block_size=16, ctx_lo=64, ctx_hi=512, nodes=32,
             kv="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["slots", "rope", "tree", "tree", "verify", "verify", "keep"])
    bs = rng.choice([16, 32, 64, 128, 256])
    if op == "slots":
        tree = rng.random() < 0.5
        batch = _log(rng, 1, 512)
        if tree:
            n = _log(rng, 1, 128)
            return dict(op=op, batch=batch, block_size=bs, ctx_lo=1, ctx_hi=_log(rng, 16, 16384), new_lo=rng.randint(0, n),
                        new_hi=n, row_len=n + rng.randint(0, 3), tree=True)
        n = min(_log(rng, 1, 32768), 4_000_000 // batch)
        return dict(op=op, batch=batch, block_size=bs, ctx_lo=1, ctx_hi=_log(rng, 16, 16384), new_lo=rng.randint(0, n),
                    new_hi=n, row_len=0, tree=False)
    hq, hkv = rng.choice([(32, 8), (40, 8), (64, 8), (8, 8), (8, 2), (16, 1)])
    if op == "rope":
        dim = rng.choice([64, 128])
        kv = rng.choice(["bf16", "bf16", "fp8"]) if dim == 128 else "bf16"
        return dict(op=op, tokens=_log(rng, 1, 16384), hq=hq, hkv=hkv, dim=dim,
                    rot=rng.choice([dim, dim, 16 * rng.randint(1, dim // 16)]), interleaved=rng.random() < 0.5,
                    block_size=bs, pos_hi=_log(rng, 64, 1 << 20), kv=kv, stretch=rng.choice([1.0, 4.0, 32.0]))
    if op == "tree":
        dim = rng.choice([64, 128, 128, 128])
        kv = rng.choice(["bf16", "bf16", "fp8"]) if dim == 128 else "bf16"
        nodes = _log(rng, 1, 200)
        batch = _log(rng, 1, 64)
        # the plain form holds batch * hq * nodes * longest scores: at most the largest listed case's
        top = min(65536, 8 * 64 * 64 * 65536 // (batch * hq * nodes), 8 * 8 * 65536 // (batch * hkv))
        hi = max(nodes + 1, _log(rng, 16, max(17, top)))
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, dim=dim, block_size=bs, ctx_lo=rng.choice([nodes, max(nodes, hi // 8)]),
                    ctx_hi=hi, nodes=nodes, ragged=rng.random() < 0.5, kv=kv)
    if op == "verify":
        vocab = _log(rng, 500, 152064)
        nodes = _log(rng, 1, 64)
        batch = min(_log(rng, 1, 256), max(1, 128 * 16 * 128256 // (nodes * vocab)))
        return dict(op=op, batch=batch, nodes=nodes, vocab=vocab, chain=rng.random() < 0.3, draft=rng.random() < 0.6,
                    ragged=rng.random() < 0.5, noise=rng.choice([0.1, 0.5, 1.5]))
    dim = rng.choice([64, 128])
    return dict(op=op, batch=_log(rng, 1, 512), hkv=hkv, dim=dim, block_size=bs, ctx_lo=0, ctx_hi=_log(rng, 16, 256),
                nodes=_log(rng, 2, 64), kv=rng.choice(["bf16", "fp8"]) if dim == 128 else "bf16")


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _ints(g, lo, hi, shape):
    """Whole numbers of [lo, hi]."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV, dtype=torch.int32)


def _log_ints(g, lo, hi, n):
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    lo1 = max(1, lo)
    x = torch.exp(math.log(lo1) + u * (math.log(max(hi, lo1)) - math.log(lo1))).round().to(torch.int32)
    return x.clamp(lo, max(hi, lo))


def _parents(g, batch, nodes):
    """A tree per row: node 0 is the root, node i hangs below one of the nodes before it."""
    u = torch.rand((batch, nodes), generator=g, device=DEV)
    i = torch.arange(nodes, device=DEV, dtype=torch.float32)
    return torch.minimum((u * i).to(torch.int32), (i - 1).clamp(min=0).to(torch.int32)).sub_((i == 0).to(torch.int32))


def _table(g, blocks_of, spare):
    """Distinct shuffled blocks for every sequence: (table [B, MB] padded with -1, free blocks, pool size)."""
    used, width = int(blocks_of.sum()), max(1, int(blocks_of.max()))
    pool = used + spare
    perm = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    first = torch.cumsum(blocks_of, 0) - blocks_of
    j = torch.arange(width, device=DEV)
    at = (first[:, None] + j).clamp(max=max(0, used - 1))
    return torch.where(j < blocks_of[:, None], perm[at], -1).to(torch.int32).contiguous(), perm[used:].contiguous(), pool


def _pool(g, pool, c, kv):
    shape = (pool, c["hkv"], c["block_size"], c["dim"])
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return (x * 16).to(torch.float8_e4m3fn).view(torch.uint8) if kv == "fp8" else x


def _prepare_slots(c, g):
    B, bs = c["batch"], c["block_size"]
    ctx = _log_ints(g, c["ctx_lo"], c["ctx_hi"], B)
    new = _ints(g, c["new_lo"], c["new_hi"], (B,))
    held = (ctx.long() + bs - 1) // bs
    total = (ctx.long() + new + bs - 1) // bs
    table, free, pool = _table(g, held, int((total - held).sum()) + B)
    wide = torch.full((B, (c["ctx_hi"] + c["new_hi"] + bs - 1) // bs), -1, dtype=torch.int32, device=DEV)
    wide[:, : table.shape[1]] = table[:, : wide.shape[1]]
    rows = B * (c["row_len"] or c["new_hi"])     # packed: room for the longest requests, the rest of the rows is padding
    out = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(ctx=ctx, new=new, table=wide, held=held.int(), free=free, head=torch.full((1,), 3, dtype=torch.int32, device=DEV),
             pool=pool, slot_map=out(rows), positions=out(rows), first=out(B + 1), granted=out(B), total=out(B),
             held_out=out(B), head_out=out(1))
    s["parents"] = _parents(g, B, c["row_len"]).contiguous() if c["tree"] else None
    return s


def _prepare_rope(c, g):
    T, hq, hkv, D, bs = c["tokens"], c["hq"], c["hkv"], c["dim"], c["block_size"]
    qkv = torch.randn((T, (hq + 2 * hkv) * D), generator=g, device=DEV).to(torch.bfloat16)
    blocks = (T + bs - 1) // bs + 2
    j = torch.arange(c["rot"] // 2, dtype=torch.float64)
    inv = 1.0 / (1e6 ** (2 * j / c["rot"]))
    ramp = (j / max(1, c["rot"] // 2 - 1)).clamp(0, 1)            # low frequencies stretched, high ones kept
    inv = inv * (1 - ramp) + inv / c["stretch"] * ramp
    s = dict(q=qkv[:, : hq * D].unflatten(1, (hq, D)), k=qkv[:, hq * D:(hq + hkv) * D].unflatten(1, (hkv, D)),
             v=qkv[:, (hq + hkv) * D:].unflatten(1, (hkv, D)), inv_freq=inv.float().to(DEV),
             magnitude=0.1 * math.log(c["stretch"]) + 1.0, positions=_ints(g, 0, c["pos_hi"] - 1, (T,)),
             slots=torch.randperm(blocks * bs, generator=g, device=DEV)[:T].int(), blocks=blocks,
             q_out=torch.empty((T, hq, D), dtype=torch.bfloat16, device=DEV), k_scale=0.03, v_scale=0.02)
    s["k_cache"], s["v_cache"] = (_pool(g, blocks, c, c["kv"]) for _ in range(2))
    return s


def _prepare_tree(c, g):
    B, N, hq, D, bs = c["batch"], c["nodes"], c["hq"], c["dim"], c["block_size"]
    ctx = _log_ints(g, c["ctx_lo"], c["ctx_hi"], B).clamp(min=N)    # the nodes included
    sizes = _ints(g, 1, N, (B,)) if c["ragged"] else torch.full((B,), N, dtype=torch.int32, device=DEV)
    table, _, pool = _table(g, (ctx.long() + bs - 1) // bs, 5)
    s = dict(ctx=ctx, sizes=sizes, table=table, pool=pool, parents=_parents(g, B, N).contiguous(), scale=1.0 / math.sqrt(D),
             q=torch.randn((B, N, hq, D), generator=g, device=DEV).to(torch.bfloat16),
             out=torch.zeros((B, N, hq, D), dtype=torch.bfloat16, device=DEV), k_scale=1 / 16, v_scale=1 / 16)
    s["k_cache"], s["v_cache"] = (_pool(g, pool, c, c["kv"]) for _ in range(2))
    return s


def _prepare_verify(c, g):
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    logits = torch.randn((B, N, V), generator=g, device=DEV).mul_(2.5)
    p = torch.softmax(logits, -1)
    logits += torch.randn((B, N, V), generator=g, device=DEV).mul_(c["noise"])
    q = torch.softmax(logits, -1)
    del logits
    parents = torch.arange(-1, N - 1, device=DEV, dtype=torch.int32).expand(B, N) if c["chain"] else _parents(g, B, N)
    parents = parents.contiguous()
    # every node's token is drawn from the draft's distribution at its parent
    cdf = torch.cumsum(q, -1)
    u = torch.rand((B, N), generator=g, device=DEV) * 0.999
    at = parents.clamp(min=0).long()
    rows = (torch.arange(B, device=DEV)[:, None] * N + at).view(-1)
    tokens = torch.empty(B * N, dtype=torch.int32, device=DEV)
    for k in range(0, B * N, 256):
        r = cdf.view(B * N, V)[rows[k:k + 256]]
        tokens[k:k + 256] = torch.searchsorted(r, u.view(-1)[k:k + 256, None] * r[:, -1:], right=True).view(-1).clamp(max=V - 1).int()
    del cdf
    out = lambda *n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(p=p, q=q if c["draft"] else None, parents=None if c["chain"] else parents, all_parents=parents,
                tokens=tokens.view(B, N), uniforms=torch.rand((B, N), generator=g, device=DEV),
                sizes=_ints(g, 0, N, (B,)) if c["ragged"] else None, path=out(B, N), out_tokens=out(B, N), accepted=out(B))


def _prepare_keep(c, g):
    B, N, bs = c["batch"], c["nodes"], c["block_size"]
    base = _ints(g, c["ctx_lo"], c["ctx_hi"], (B,))
    blocks = (base.long() + N + bs - 1) // bs
    table, _, pool = _table(g, blocks, B * ((c["ctx_hi"] + N + bs - 1) // bs) - int(blocks.sum()))
    # an accepted branch: the root and a random increasing run of nodes
    pick = torch.rand((B, N), generator=g, device=DEV) < 0.6
    pick[:, 0] = True
    count = pick.sum(1)
    order = torch.argsort((~pick).int(), dim=1, stable=True)
    path = torch.where(torch.arange(N, device=DEV) < count[:, None], order, -1).int()
    s = dict(base=base, table=table, pool=pool, path=path.contiguous(), accepted=(count - 1).int(),
             ctx_out=torch.empty(B, dtype=torch.int32, device=DEV))
    s["k_cache"], s["v_cache"] = (_pool(g, pool, c, c["kv"]) for _ in range(2))
    return s


def prepare(case, seed):
    c = dict(case)
    s = {"slots": _prepare_slots, "rope": _prepare_rope, "tree": _prepare_tree, "verify": _prepare_verify,
         "keep": _prepare_keep}[c["op"]](c, _gen(seed))
    s["case"] = c
    if own:
        from paper_2511_21862_b200 import binding, spec
        hkv, D, bs = c.get("hkv", 1), c.get("dim", 128), c.get("block_size", 16)
        if c["op"] != "verify":
            table = s.get("table")
            s["shape"] = binding.Shape(c.get("batch", 1), c.get("hq", hkv), hkv, D, bs, s.get("pool", s.get("blocks")),
                                       1 if table is None else table.shape[1], hkv * bs * D, bs * D, D)
        if c["op"] == "slots":
            s["workspace"] = torch.empty(spec.plan_slots_workspace_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
        if c["op"] == "rope":
            s["rope"] = spec.Rope(c["rot"], c["interleaved"], s["inv_freq"], s["magnitude"])
        if c["op"] == "tree":
            s["workspace"] = torch.empty(spec.tree_workspace_bytes(s["shape"], c["nodes"]), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _slots(s):
    c, bs = s["case"], s["case"]["block_size"]
    B, L = c["batch"], c["row_len"]
    ctx, new, held = s["ctx"].long(), s["new"].long(), s["held"].long()
    need = ((ctx + new + bs - 1) // bs - held).clamp(min=0)
    upto = torch.cumsum(need, 0)
    head = s["head"].long()
    ok = (need == 0) | (head + upto <= s["free"].numel())
    from_ = head + upto - need
    tok_first = torch.cumsum(new, 0) - new
    n = s["slot_map"].numel()
    r = torch.arange(n, device=DEV)
    if L:
        b, i = r // L, r % L
    else:
        b = torch.searchsorted(tok_first + new, r, right=True).clamp(max=B - 1)
        i = r - tok_first[b]
    live = (i < new[b]) & ok[b]
    t = ctx[b] + i
    blk = t // bs
    fresh = live & (blk >= held[b])
    at = (from_[b] + blk - held[b]).clamp(0, s["free"].numel() - 1)
    known = s["table"][b, blk.clamp(max=s["table"].shape[1] - 1)].long()
    block = torch.where(fresh, s["free"][at].long(), known)
    slot = torch.where(live, block * bs + t % bs, -1)
    table = s["table"].clone()
    w = torch.nonzero(fresh & ((t % bs == 0) | (i == 0))).view(-1)
    table[b[w], blk[w]] = block[w].int()
    pos = t
    if c["tree"]:
        pos = ctx[b] + _depth(s["parents"]).view(-1)[:n]
    first = torch.cat([tok_first, tok_first[-1:] + new[-1:]])
    if L:
        first = torch.arange(B + 1, device=DEV) * L
    return dict(table=table, slot_map=slot.int(), positions=torch.where(i < new[b], pos, -1).int(), first=first.int(),
                granted=torch.where(ok, new, 0).int(), total=(ctx + torch.where(ok, new, 0)).int(),
                held=torch.where(ok, held + need, held).int(),
                head=(head + torch.where(ok, need, 0).sum()).int())


def _ancestors(parents):
    """[B, N, N] truth values: node j is node i or above it."""
    B, N = parents.shape
    eye = torch.eye(N, device=DEV)
    a = eye + (parents[:, :, None] == torch.arange(N, device=DEV))
    for _ in range(max(1, (N - 1).bit_length())):
        a = (a @ a).clamp(max=1)
    return a > 0


def _depth(parents):
    return _ancestors(parents).sum(-1) - 1


def _turn(x, cos, sin, rot, interleaved):
    x = x.float()
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


def _rope(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = ((f(angle) * s["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    q = _turn(s["q"], cos, sin, c["rot"], c["interleaved"]).to(torch.bfloat16)
    k = _turn(s["k"], cos, sin, c["rot"], c["interleaved"])
    blk, off = s["slots"].long() // c["block_size"], s["slots"].long() % c["block_size"]
    s["k_cache"][blk, :, off] = _stored(k, s["k_scale"], s["k_cache"])
    s["v_cache"][blk, :, off] = _stored(s["v"].float(), s["v_scale"], s["v_cache"])
    return dict(q=q, k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]))


def _gathered(cache, table, scale):
    """[B, Hkv, tokens, D] in 32 bits."""
    x = _values(cache[table.clamp(min=0).long()]).float().permute(0, 2, 1, 3, 4).flatten(2, 3)
    return x * scale if cache.dtype == torch.uint8 else x


def _tree(s):
    c = s["case"]
    B, N, hq, hkv, D = c["batch"], c["nodes"], c["hq"], c["hkv"], c["dim"]
    q = s["q"].float().view(B, N, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D)
    w = torch.matmul(q, _gathered(s["k_cache"], s["table"], s["k_scale"]).transpose(-1, -2)).mul_(s["scale"])
    T = w.shape[-1]
    base = (s["ctx"] - s["sizes"]).long()
    node = torch.arange(T, device=DEV) - base[:, None]                                        # [B, T]
    seen = torch.gather(_ancestors(s["parents"]), 2, node.clamp(0, N - 1)[:, None].expand(B, N, T))
    seen = torch.where(node[:, None] < 0, True, seen & (node < s["sizes"][:, None])[:, None])
    w = w.view(B, hkv, hq // hkv, N, T).masked_fill_(~seen[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True)).exp_()
    w /= w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, hkv, -1, T), _gathered(s["v_cache"], s["table"], s["v_scale"]))
    o = o.view(B, hkv, hq // hkv, N, D).permute(0, 3, 1, 2, 4).reshape(B, N, hq, D).to(torch.bfloat16)
    live = torch.arange(N, device=DEV) < s["sizes"][:, None]
    return torch.where(live[:, :, None, None], o, s["out"])


def _verify(s):
    p, q, tokens, parents = s["p"], s["q"], s["tokens"].long(), s["all_parents"].long()
    B, N, V = p.shape
    rows = torch.arange(B, device=DEV)
    size = torch.full((B,), N, device=DEV) if s["sizes"] is None else s["sizes"].long()
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    spent = torch.zeros(B, dtype=torch.float64, device=DEV)      # sum of the masses so far: weights are max(p - spent q, 0)
    mass = torch.ones(B, dtype=torch.float64, device=DEV)
    dropped = torch.zeros((B, N), dtype=torch.bool, device=DEV)  # rejected siblings at the current node (without q)
    count = torch.zeros(B, dtype=torch.long, device=DEV)
    path = torch.full((B, N), -1, dtype=torch.long, device=DEV)
    path[:, 0] = torch.where(size > 0, 0, -1)
    out = torch.full((B, N + 1), -1, dtype=torch.long, device=DEV)
    for i in range(1, N):
        asked = (parents[:, i] == cur) & (i < size)
        x = tokens[:, i]
        px = p[rows, cur, x].double()
        if q is not None:
            qx = q[rows, cur, x].double()
            take = asked & (s["uniforms"][:, i].double() * mass * qx < (px - spent * qx).clamp(min=0))
        else:
            px = torch.where((dropped & (tokens == x[:, None])).any(1), 0.0, px)
            take = asked & (s["uniforms"][:, i].double() * mass < px)
        refused = asked & ~take
        if q is not None:
            spent = torch.where(refused, spent + mass, spent)
            rest = (p[rows, cur].double() - spent[:, None] * q[rows, cur].double()).clamp(min=0).sum(-1)
            mass = torch.where(refused, rest, mass)
        else:
            mass = torch.where(refused, mass - px, mass)
            dropped[:, i] = refused
        count = count + take
        out[rows, torch.where(take, count - 1, N)] = x
        path[rows, count] = torch.where(take, torch.full_like(cur, i), path[rows, count])
        cur = torch.where(take, i, cur)
        spent, mass = torch.where(take, 0.0, spent), torch.where(take, 1.0, mass)
        dropped &= ~take[:, None]
    w = p[rows, cur].double()
    if q is not None:
        w = (w - spent[:, None] * q[rows, cur].double()).clamp(min=0)
    else:
        w[rows[:, None].expand(B, N)[dropped], tokens[dropped]] = 0
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, p[rows, cur].double())
    sums = torch.cumsum(w, -1)
    t = s["uniforms"][:, 0].double() * sums[:, -1]
    drawn = torch.searchsorted(sums, t[:, None], right=True).view(-1).clamp(max=V - 1)
    live = size > 0
    out[rows, torch.where(live, count, N)] = drawn
    return dict(path=path.int(), tokens=out[:, :N].int(), accepted=count.int())


def _keep(s):
    c = s["case"]
    bs, N = c["block_size"], c["nodes"]
    j = torch.arange(N, device=DEV)
    live = j <= s["accepted"][:, None]
    b, k = torch.nonzero(live, as_tuple=True)
    src = s["base"][b].long() + s["path"][b, k].long()
    dst = s["base"][b].long() + k
    for cache in (s["k_cache"], s["v_cache"]):
        cache[s["table"][b, dst // bs].long(), :, dst % bs] = cache[s["table"][b, src // bs].long(), :, src % bs]
    return dict(k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]), ctx=(s["base"] + 1 + s["accepted"]).int())


# ------------------------------------------------------------------------------------------------ the library's calls
def _own(s):
    from paper_2511_21862_b200 import spec
    c = s["case"]
    op, fp8 = c["op"], c.get("kv") == "fp8"
    if op == "slots":
        spec.plan_slots(s["shape"], s["ctx"], s["new"], s["table"], s["held"], s["free"], s["head"], s["slot_map"],
                        s["positions"], s["first"], s["granted"], s["total"], s["workspace"], row_len=c["row_len"],
                        parents=s["parents"], blocks_held_out=s["held_out"], free_head_out=s["head_out"])
        return dict(table=s["table"], slot_map=s["slot_map"], positions=s["positions"], first=s["first"],
                    granted=s["granted"], total=s["total"], held=s["held_out"], head=s["head_out"])
    if op == "rope":
        if fp8:
            spec.rope_kv_append_fp8(s["shape"], s["rope"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"],
                                    s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        else:
            spec.rope_kv_append(s["shape"], s["rope"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"],
                                s["k_cache"], s["v_cache"])
        return dict(q=s["q_out"], k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]))
    if op == "tree":
        if fp8:
            spec.tree_attention_fp8(s["shape"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["parents"],
                                    s["scale"], s["k_scale"], s["v_scale"], s["out"], s["workspace"], tree_sizes=s["sizes"])
        else:
            spec.tree_attention(s["shape"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx"], s["parents"],
                                s["scale"], s["out"], s["workspace"], tree_sizes=s["sizes"])
        return s["out"]
    if op == "verify":
        spec.verify_drafts(s["p"], s["q"], s["tokens"], s["parents"], s["uniforms"], s["path"], s["out_tokens"],
                           s["accepted"], tree_sizes=s["sizes"])
        return dict(path=s["path"], tokens=s["out_tokens"], accepted=s["accepted"])
    keep = spec.kv_keep_path_fp8 if fp8 else spec.kv_keep_path
    keep(s["shape"], s["k_cache"], s["v_cache"], s["table"], s["base"], s["path"], s["accepted"], s["ctx_out"])
    return dict(k_cache=_values(s["k_cache"]), v_cache=_values(s["v_cache"]), ctx=s["ctx_out"])


def run(state):
    if own:
        return _own(state)
    return {"slots": _slots, "rope": _rope, "tree": _tree, "verify": _verify, "keep": _keep}[state["case"]["op"]](state)


def _middle(lo, hi):
    """Mean of a length drawn evenly over its logarithm."""
    lo = max(1, lo)
    return float(lo) if hi <= lo else (hi - lo) / math.log(hi / lo)


def work(case):
    c, op = case, case["op"]
    B = c.get("batch", 1)
    if op == "slots":
        new = B * (c["new_lo"] + c["new_hi"]) / 2
        rows = B * (c["row_len"] or c["new_hi"])
        # lengths and what is held in, five words a sequence out, slot and position of every row, every new block's id in and out
        return dict(bytes=32 * B + 8 * rows + 8 * new / c["block_size"] + (4 * rows if c["tree"] else 0), flops=8 * rows)
    if op == "rope":
        cell = 1 if c["kv"] == "fp8" else 2
        rows = c["tokens"] * c["dim"]
        return dict(bytes=rows * (2 * c["hq"] * 2 + 2 * c["hkv"] * (2 + cell)) + 8 * c["tokens"],
                    flops=3 * c["tokens"] * c["rot"] * (c["hq"] + c["hkv"]))
    if op == "tree":
        cell = 1 if c["kv"] == "fp8" else 2
        tokens = B * max(c["nodes"], _middle(c["ctx_lo"], c["ctx_hi"]))
        nodes = (1 + c["nodes"]) / 2 if c["ragged"] else c["nodes"]
        return dict(bytes=2 * cell * c["hkv"] * c["dim"] * tokens + 4 * B * nodes * c["hq"] * c["dim"] +
                    4 * tokens / c["block_size"] + 4 * B * nodes, flops=4 * c["hq"] * c["dim"] * nodes * tokens)
    if op == "verify":
        # one row of the target (and of the draft, where a token was refused) a sequence, and a few words a node
        return dict(bytes=B * (4 * c["vocab"] * (2 if c["draft"] else 1) + 28 * c["nodes"]), flops=4.0 * B * c["vocab"])
    cell = 1 if c["kv"] == "fp8" else 2
    moved = B * 0.6 * (c["nodes"] - 1)
    return dict(bytes=4 * cell * c["hkv"] * c["dim"] * moved + 8 * B * c["nodes"], flops=0)


# ------------------------------------------------------------------------------------------------ definitions in 64 bits
def exact(case, seed):
    """Rotary rows and attention rows in 64 bits, one sequence (one head pair) at a time; the other operators compute
    whole numbers or move values."""
    op = case["op"]
    if op not in ("rope", "tree"):
        return None
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return _exact_rope(s, case) if op == "rope" else _exact_tree(s, case)


def _exact_rope(s, c):
    bs, rot = c["block_size"], c["rot"]
    angle = torch.outer(s["positions"].to(torch.float64), s["inv_freq"].to(torch.float64))
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None]

    def rotated(x):
        x = x.to(torch.float64)
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

    return dict(q=rotated(s["q"]), k_cache=placed(s["k_cache"], rotated(s["k"]), s["k_scale"]),
                v_cache=placed(s["v_cache"], s["v"].to(torch.float64), s["v_scale"]))


def _exact_tree(s, c):
    B, N, hq, hkv, D, bs = (c[k] for k in ("batch", "nodes", "hq", "hkv", "dim", "block_size"))
    fp8 = c["kv"] == "fp8"
    out = s["out"].to(torch.float64)
    up = s["parents"].tolist()
    for b in range(B):
        T, n = int(s["ctx"][b]), int(s["sizes"][b])
        ids = s["table"][b, : (T + bs - 1) // bs].long()
        k, v = (x[ids].view(torch.float8_e4m3fn).to(torch.float64) * sc if fp8 else x[ids].to(torch.float64)
                for x, sc in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])))
        k, v = (x.permute(1, 0, 2, 3).flatten(1, 2)[:, :T] for x in (k, v))        # [Hkv, T, D]
        hide = torch.ones((n, n), dtype=torch.bool)
        for i in range(n):
            j = i
            while j >= 0:
                hide[i, j] = False
                j = up[b][j]
        for h in range(hkv):
            q = s["q"][b, :n, h * (hq // hkv):(h + 1) * (hq // hkv)].to(torch.float64)     # [n, G, D]
            w = (q.reshape(-1, D) @ k[h].T).view(n, hq // hkv, T) * s["scale"]
            w[:, :, T - n:].masked_fill_(hide.to(DEV)[:, None], -math.inf)
            w = torch.softmax(w, -1)
            out[b, :n, h * (hq // hkv):(h + 1) * (hq // hkv)] = (w.view(-1, T) @ v[h]).view(n, -1, D)
    return out
