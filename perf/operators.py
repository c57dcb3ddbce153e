"""The operators of a verification step beside the draft tree, as measurable cases.

One decoding step of a served model drafts a tree, runs the verifier over its
positions and keeps the accepted path.  The cases are what that step asks for
next to the tree itself:

* ``sample``: a next token for every position from the verifier's logits
  (temperature, top-k, top-p, min-p, one given random number a position);
* ``slots``: cache pages, slots and positions of the tokens that every
  sequence gains, from the lengths on the GPU;
* ``append``: these tokens' keys and values into the paged 8-bit cache;
* ``attend``: attention of the tree's positions over that cache and over the
  tree itself.

With ``own`` false run() computes them in plain torch operations, with ``own``
true by the library's calls.  Sizes follow the repository's Qwen3-shaped
workloads (a vocabulary of 151936, draft depth 16, budgets of 32 to 512) and
generic attention shapes.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3_MAX = 448.0
SCALE_MIN, SCALE_MAX = 2.0 ** -64, 2.0 ** 64


def listed():
    return [
        # one sequence, one token: the plain decoding loop's last call, where only latency counts
        dict(name="sample-decode", kind="sample", dt="bf16", b=1, n=1, V=151936, pad=0, how="k20"),
        # sixteen sequences with a tree of 32 nodes each, every request with settings of its own
        dict(name="sample-tree33-b16", kind="sample", dt="bf16", b=16, n=33, V=151936, pad=0, how="mixed"),
        # fp32 logits without a top-k, an odd vocabulary inside padded rows
        dict(name="sample-nucleus-f32", kind="sample", dt="f32", b=4, n=65, V=128815, pad=17, how="nucleus"),
        # the accepted paths of sixteen sequences: every decoding step
        dict(name="slots-accepted-b16", kind="slots", b=16, ctx=8192, add=17, page=64, accepted=True),
        # a batch of prompts of many lengths
        dict(name="slots-prompts-b256", kind="slots", b=256, ctx=0, add=4096, page=16, accepted=False),
        # keys and values of the accepted paths
        dict(name="append-accepted-b16", kind="append", dt="bf16", b=16, ctx=8192, add=17, page=64, heads=8, D=128),
        # of four long prompts
        dict(name="append-prompts-b4", kind="append", dt="bf16", b=4, ctx=0, add=8192, page=64, heads=8, D=128),
        # one token of one sequence: the smallest attention call
        dict(name="attend-decode", kind="attend", dt="bf16", b=1, n=1, ctx=4096, page=64, heads=8, group=4, D=128,
             tree=False),
        # single tokens of many sequences: reading the cache is all there is
        dict(name="attend-decode-b64", kind="attend", dt="bf16", b=64, n=1, ctx=8192, page=64, heads=8, group=4,
             D=128, tree=False),
        # a tree of 32 nodes over one long context
        dict(name="attend-tree33", kind="attend", dt="bf16", b=1, n=33, ctx=8192, page=64, heads=8, group=4, D=128,
             tree=True),
        # of sixteen sequences: the largest call, where the matrix products weigh as much as the reads
        dict(name="attend-tree33-b16", kind="attend", dt="bf16", b=16, n=33, ctx=16384, page=64, heads=8, group=4,
             D=128, tree=True),
        # a small fp32 model's tree, short ragged contexts in small pages
        dict(name="attend-tree17-f32", kind="attend", dt="f32", b=3, n=17, ctx=1003, page=16, heads=2, group=4, D=64,
             tree=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "slots", "append", "attend", "attend", "attend"])
    if kind == "sample":
        dt, V, n = rng.choice(["bf16", "bf16", "f32"]), _log(rng, 1000, 151936), _log(rng, 1, 129)
        b = _log(rng, 1, 64)
        while b * n * V * (2 if dt == "bf16" else 4) > 16 * 33 * 151936 * 2:
            b, n = max(1, b // 2), max(1, n * 3 // 4)
        return dict(kind=kind, dt=dt, b=b, n=n, V=V, pad=rng.choice([0, 0, 1, 8, 64]),
                    how=rng.choice(["k20", "mixed", "nucleus", "plain", "greedy"]))
    if kind == "slots":
        if rng.random() < 0.5:
            return dict(kind=kind, b=_log(rng, 1, 512), ctx=_log(rng, 64, 32768), add=rng.randint(2, 33),
                        page=rng.choice([16, 32, 64, 128]), accepted=True)
        b = _log(rng, 1, 256)
        return dict(kind=kind, b=b, ctx=rng.choice([0, 0, 1000]), add=min(4096, _log(rng, 1, 4096 * 256 // b)),
                    page=rng.choice([16, 32, 64, 128]), accepted=False)
    D, heads = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 12])
    page, dt = rng.choice([16, 32, 64, 64, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "append":
        long = rng.random() < 0.4
        b = _log(rng, 1, 8 if long else 128)
        add = _log(rng, 100, 8192) if long else rng.randint(1, 33)
        while b * add * heads * D * (2 if dt == "bf16" else 4) > 4 * 8192 * 8 * 128 * 2:
            add = max(1, add // 2)
        return dict(kind=kind, dt=dt, b=b, ctx=rng.choice([0, _log(rng, 1, 4096)]), add=add, page=page, heads=heads,
                    D=D)
    b, n, ctx, group = _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 513)]), _log(rng, 1, 32768), rng.choice([1, 2, 4, 5, 8])
    most = 16 * 33 * 32 * 16384 * 128 // (1 if dt == "bf16" else 256)
    while b * (n + 8) * heads * group * (ctx + n) * D > most or b * ctx * heads * D > 64 * 8192 * 8 * 128:
        if ctx > 2048:
            ctx = ctx * 3 // 4
        elif b > 1:
            b //= 2
        elif n > 1:
            n = n * 3 // 4
        else:
            ctx = max(1, ctx // 2)
    return dict(kind=kind, dt=dt, b=b, n=n, ctx=ctx, page=page, heads=heads, group=group, D=D,
                tree=n > 1 and rng.random() < 0.7)


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["dt"] == "f32" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _contexts(case):
    """Context lengths of a batch: the longest first, the others down to half of it."""
    ctx = case["ctx"]
    return [ctx - (s * 2654435761 % 1009) * (ctx // 2) // 1009 if s else ctx for s in range(case["b"])]


def _added(case):
    """Tokens that each sequence gains: the longest first, one at least."""
    add = case["add"]
    return [1 + (s * 40503 + 7919) % 1013 * add // 1013 if s else add for s in range(case["b"])]


def _pages_of(lengths, page):
    return [-(-x // page) for x in lengths]


def _tables(held, cols, num_pages, g):
    """A block table [b, cols] with `held` pages each, drawn without order, and the pages that are left."""
    order = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((len(held), cols), dtype=torch.int32, device="cuda")
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    return table, order[at:].contiguous()


def _pow2_scale(amax):
    """The smallest power of two that brings `amax` into e4m3's range."""
    m, e = torch.frexp(amax / E4M3_MAX)
    e = torch.where(m == 0.5, e - 1, e)
    s = torch.ldexp(torch.ones_like(amax), e)
    return torch.where(amax > 0, s, torch.zeros_like(s)).clamp(SCALE_MIN, SCALE_MAX)


def _cache(num_pages, heads, page, D, g, loud):
    """Cached values [num_pages, heads, page, D] in e4m3 with a scale for each page and head: channels
    of unequal size (`loud` of them several times the others) and pages louder than others."""
    codes = torch.empty((num_pages, heads, page, D), dtype=torch.uint8, device="cuda")
    scale = torch.empty((num_pages, heads), dtype=torch.float32, device="cuda")
    gain = torch.ones((heads, 1, D), device="cuda")
    gain[:, :, torch.randperm(D, generator=g, device="cuda")[:loud]] = 4.0
    step = max(1, (1 << 26) // (heads * page * D))
    for p in range(0, num_pages, step):
        q = min(step, num_pages - p)
        x = torch.randn((q, heads, page, D), generator=g, device="cuda") * gain
        x *= torch.exp(0.5 * torch.randn((q, heads, 1, 1), generator=g, device="cuda"))
        s = _pow2_scale(x.abs().amax((2, 3)))
        codes[p:p + q] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[p:p + q] = s
    return codes, scale


def _settings(case, g):
    """temperature, top_k, top_p, min_p of each sequence."""
    b, how = case["b"], case["how"]
    kinds = {"k20": (0.6, 20, 0.95, 0.0), "nucleus": (1.0, 0, 0.9, 0.02), "plain": (0.8, 0, 1.0, 0.0),
             "greedy": (0.0, 0, 1.0, 0.0)}
    mixed = [(0.6, 20, 0.95, 0.0), (1.0, 0, 0.95, 0.0), (0.7, 50, 1.0, 0.05), (0.0, 0, 1.0, 0.0), (1.3, 0, 1.0, 0.1),
             (1.0, 0, 1.0, 0.0), (0.8, 1000, 0.8, 0.0)]
    rows = [kinds[how]] * b if how != "mixed" else [mixed[s % len(mixed)] for s in range(b)]
    t, k, p, m = zip(*rows)
    f = dict(dtype=torch.float32, device="cuda")
    return torch.tensor(t, **f), _i32(k), torch.tensor(p, **f), torch.tensor(m, **f)


def _tree_mask(b, n, seed):
    """Ancestor masks [b, n, n] of random trees: position 0 the root, a parent before its children."""
    g = torch.Generator().manual_seed(seed)
    parent = (torch.rand((b, n), generator=g).sqrt() * torch.arange(n)).long()
    mask = torch.zeros((b, n, n), dtype=torch.uint8)
    mask[:, 0, 0] = 1
    rows = torch.arange(b)
    for i in range(1, n):
        mask[:, i] = mask[rows, parent[:, i]]
        mask[:, i, i] = 1
    return mask.cuda()


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "sample":
        b, n, V = case["b"], case["n"], case["V"]
        wide = torch.randn((b, n, V + case["pad"]), generator=g, device="cuda").mul_(2.2)
        likely = torch.randint(0, V, (b, n, 40), generator=g, device="cuda")
        wide.scatter_add_(2, likely, torch.rand((b, n, 40), generator=g, device="cuda").mul_(10.0).add_(4.0))
        logits = wide.to(_dtype(case))[..., :V]
        t, k, p, m = _settings(case, g)
        return dict(kind=kind, logits=logits, uniform=torch.rand((b, n), generator=g, device="cuda"), temperature=t,
                    top_k=k, top_p=p, min_p=m)
    page, b = case["page"], case["b"]
    ctx = _contexts(case)
    if kind == "attend":
        n, heads, D = case["n"], case["heads"], case["D"]
        held = _pages_of(ctx, page)
        num_pages = sum(held) + 3
        table, _ = _tables(held, max(held), num_pages, g)
        k, ks = _cache(num_pages, heads, page, D, g, 4)
        v, vs = _cache(num_pages, heads, page, D, g, 0)
        e4 = torch.float8_e4m3fn
        f = dict(generator=g, device="cuda")
        # one projection gives queries, keys and values: the three are views of its rows
        qkv = torch.randn((b, n, (case["group"] + 2) * heads, D), **f).to(_dtype(case))
        hq = case["group"] * heads
        return dict(kind=kind, q=qkv[:, :, :hq], k_new=qkv[:, :, hq:hq + heads], v_new=qkv[:, :, hq + heads:],
                    mask=_tree_mask(b, n, seed) if case["tree"] else None, context_len=_i32(ctx), block_table=table,
                    k_cache=k.view(e4), v_cache=v.transpose(2, 3).contiguous().view(e4), k_scale=ks, v_scale=vs,
                    scale=D ** -0.5)
    add = _added(case)
    after = [c + a for c, a in zip(ctx, add)]
    held = _pages_of(ctx, page)
    cols = max(_pages_of(after, page)) + 1
    num_pages = sum(_pages_of(after, page)) + 5
    table, free = _tables(held, cols, num_pages, g)
    if kind == "slots":
        st = dict(kind=kind, context_len=_i32(ctx), block_table=table, free_pages=free, free_count=_i32([free.numel()]),
                  page=page, accepted=None, n=0, max_tokens=sum(add))
        if case["accepted"]:   # add - 1 nodes at most on a path, in a tree of twice as many
            depth, n = case["add"] - 1, 2 * case["add"]
            acc = torch.rand((b, n - 1), generator=g, device="cuda").argsort(1)[:, :depth].sort(1).values.to(torch.int32)
            ln = _i32([a - 1 for a in add])
            acc = torch.where(torch.arange(depth, device="cuda")[None] < ln[:, None], acc, torch.full_like(acc, -1))
            st.update(accepted=acc, add_len=ln, n=n, max_tokens=b * case["add"])
        else:
            st.update(add_len=_i32(add))
        return st
    # append: slots as the sequences' pages give them, rows of the new tokens in order
    heads, D = case["heads"], case["D"]
    fresh = torch.cat([table, free.new_zeros((b, 1))], 1)
    at, slots = 0, []
    for s in range(b):
        more = _pages_of(after, page)[s] - held[s]
        fresh[s, held[s]:held[s] + more] = free[at:at + more]
        at += more
        pos = torch.arange(ctx[s], after[s], device="cuda")
        slots.append(fresh[s, pos // page].to(torch.int64) * page + pos % page)
    slot = torch.cat(slots).to(torch.int32)
    k, ks = _cache(num_pages, heads, page, D, g, 4)
    v, vs = _cache(num_pages, heads, page, D, g, 0)
    e4, N = torch.float8_e4m3fn, slot.numel()
    kv = torch.randn((N, 2 * heads, D), generator=g, device="cuda") * 1.5
    kv = kv.to(_dtype(case))
    return dict(kind=kind, k_new=kv[:, :heads], v_new=kv[:, heads:], slot=slot,
                source=torch.randperm(N, generator=g, device="cuda").to(torch.int32), k_cache=k.view(e4),
                v_cache=v.transpose(2, 3).contiguous().view(e4), k_scale=ks, v_scale=vs)


# ------------------------------------------------------------------ plain forms

def _sample_plain(s):
    """In 64 bits: the sums run over a whole vocabulary, and a drawn token turns on the borders between them."""
    z = s["logits"].double()
    z = torch.where(z.isnan(), float("-inf"), z)
    t = s["temperature"].double()[:, None, None]
    top = z.amax(-1, keepdim=True)
    x = (z - top) / torch.where(t > 0, t, torch.ones_like(t))
    w = torch.exp(x)
    V = z.shape[-1]
    ranked, order = torch.sort(z, dim=-1, descending=True, stable=True)
    wr = w.gather(-1, order)
    c = wr.cumsum(-1)
    k = s["top_k"].long()[:, None, None]
    n1 = torch.where((k > 0) & (k < V), k, torch.full_like(k, V))
    z1 = c.gather(-1, (n1 - 1).expand(*z.shape[:2], 1))
    p = s["top_p"].double()[:, None, None]
    n2 = (c < p * z1).sum(-1, keepdim=True) + 1
    n2 = torch.where(p < 1, n2, torch.full_like(n2, V))
    n3 = (wr >= s["min_p"].double()[:, None, None]).sum(-1, keepdim=True)
    n = torch.minimum(torch.minimum(n1, n2), n3).clamp(min=1)
    n = torch.where(t > 0, n, torch.ones_like(n))
    keep = torch.zeros_like(w, dtype=torch.bool).scatter_(-1, order, torch.arange(V, device=z.device) < n)
    c = torch.where(keep, w, torch.zeros_like(w)).cumsum(-1)
    token = (c <= s["uniform"].double()[..., None] * c[..., -1:]).sum(-1, keepdim=True)
    lp = x.gather(-1, token) - torch.log(c[..., -1:])
    return {"token": token[..., 0].to(torch.int32), "logprob": lp[..., 0].float()}


def _slots_plain(s):
    page, table, ctx, acc = s["page"], s["block_table"], s["context_len"].long(), s["accepted"]
    add = s["add_len"].long() + (1 if acc is not None else 0)
    dev = table.device
    after = ctx + add
    had, has = (ctx + page - 1) // page, (after + page - 1) // page
    need = has - had
    before = need.cumsum(0) - need
    left = s["free_count"].long()
    ok = (need.sum() <= left) & (has.max() <= table.shape[1])
    cols = torch.arange(table.shape[1], device=dev)[None]
    fresh = (cols >= had[:, None]) & (cols < has[:, None]) & ok
    at = (left - 1 - before[:, None] - (cols - had[:, None])).clamp(0, s["free_pages"].numel() - 1)
    table = torch.where(fresh, s["free_pages"][at], table)
    start = torch.cat([add.new_zeros(1), torch.where(ok, add, torch.zeros_like(add)).cumsum(0)])
    i = torch.arange(s["max_tokens"], device=dev)
    seq = (torch.searchsorted(start, i, right=True) - 1).clamp(max=ctx.numel() - 1)
    j = i - start[seq]
    real = i < start[-1]
    pos = ctx[seq] + j
    slot = table[seq, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    none = torch.full_like(i, -1)
    if acc is not None:
        source = seq * s["n"] + torch.where(j > 0, 1 + acc[seq, (j - 1).clamp(0, acc.shape[1] - 1)].long(), torch.zeros_like(j))
    else:
        source = i
    out = dict(context_len=torch.where(ok, after, ctx), free_count=torch.where(ok, left - need.sum(), left),
               start=start, slot=torch.where(real, slot, none), position=torch.where(real, pos, none),
               source=torch.where(real, source, none), block_table=table)
    return {k: v.to(torch.int32) for k, v in out.items()}


def _append_one(new, slot, source, cache, scale, page):
    """Rows `new` [rows, heads, D] at `slot` of the cache [pages, heads, page, D]: the page's scale never falls
    while it fills, and what it held is rounded again where the scale rises."""
    x = new[source.long()].float()
    pg, off = slot.long() // page, slot.long() % page
    pages, run = torch.unique_consecutive(pg, return_inverse=True)
    first = torch.full_like(pages, page).scatter_reduce(0, run, off, "amin")
    amax = torch.zeros((pages.numel(), x.shape[1]), device=x.device).index_reduce_(0, run, x.abs().amax(-1), "amax")
    old = torch.where(first[:, None] > 0, scale[pages], torch.zeros_like(scale[pages]))
    now = torch.maximum(old, _pow2_scale(amax))
    held = cache[pages].view(torch.float8_e4m3fn).float() * (old / now)[..., None, None]
    ours = torch.arange(page, device=x.device)[None] < first[:, None]
    codes = torch.where(ours[:, None, :, None], held.to(torch.float8_e4m3fn).view(torch.uint8), cache[pages])
    new8 = (x / now[run][..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[run, :, off] = new8
    cache[pages] = codes
    scale[pages] = now


def _append_plain(s):
    page = s["k_cache"].shape[2]
    u8 = torch.uint8
    _append_one(s["k_new"], s["slot"], s["source"], s["k_cache"].view(u8), s["k_scale"], page)
    _append_one(s["v_new"], s["slot"], s["source"], s["v_cache"].view(u8).transpose(2, 3), s["v_scale"], page)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _context(codes, scale, table):
    """Cached values of a block table: [b, heads, max_pages * page, D] in fp32, from [pages, heads, page, D]."""
    x = codes[table.long()].view(torch.float8_e4m3fn).float() * scale[table.long()][..., None, None]
    b, cols, heads, page, D = x.shape
    return x.transpose(1, 2).reshape(b, heads, cols * page, D)


def _attend_plain(s):
    q, kn, vn = s["q"].float(), s["k_new"].float(), s["v_new"].float()
    b, n, hq, D = q.shape
    heads = kn.shape[2]
    u8 = torch.uint8
    k = _context(s["k_cache"].view(u8), s["k_scale"], s["block_table"])
    v = _context(s["v_cache"].view(u8).transpose(2, 3), s["v_scale"], s["block_table"])
    q = q.reshape(b, n, heads, hq // heads, D).permute(0, 2, 3, 1, 4).reshape(b, heads, -1, D) * s["scale"]
    kn, vn = kn.transpose(1, 2).contiguous(), vn.transpose(1, 2).contiguous()
    T = k.shape[2]
    seen = torch.arange(T, device=q.device)[None] < s["context_len"][:, None]
    inside = s["mask"] != 0 if s["mask"] is not None else torch.ones((n, n), dtype=torch.bool, device=q.device).tril()[None]
    inside = inside[:, None].expand(b, hq // heads, n, n).reshape(b, 1, -1, n)
    z = torch.cat([torch.matmul(q, k.transpose(2, 3).contiguous()).masked_fill(~seen[:, None, None], float("-inf")),
                   torch.matmul(q, kn.transpose(2, 3).contiguous()).masked_fill(~inside, float("-inf"))], -1)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = (torch.matmul(p[..., :T], v) + torch.matmul(p[..., T:], vn)) / total
    back = lambda t: t.reshape(b, heads, hq // heads, n, -1).permute(0, 3, 1, 2, 4).reshape(b, n, hq, -1)  # noqa: E731
    return {"out": back(o).to(s["q"].dtype), "lse": back(top + torch.log(total))[..., 0]}


# ------------------------------------------------------------------ the calls

def run(s):
    kind = s["kind"]
    if own:
        from paper_2606_03819_amd import binding
        if kind == "sample":
            token, logprob = binding.treeflash_sample(s["logits"], s["uniform"], s["temperature"], s["top_k"],
                                                      s["top_p"], s["min_p"])
            return {"token": token, "logprob": logprob}
        if kind == "slots":
            got = binding.treeflash_cache_slots(s["context_len"], s["add_len"], s["free_pages"], s["free_count"],
                                                s["block_table"], s["page"], s["max_tokens"], accepted=s["accepted"],
                                                n=s["n"])
            return {k: got[k] for k in ("context_len", "free_count", "start", "slot", "position", "source",
                                        "block_table")}
        if kind == "append":
            binding.treeflash_cache_append(s["k_new"], s["v_new"], s["slot"], s["k_cache"], s["v_cache"], s["k_scale"],
                                           s["v_scale"], source=s["source"])
            return {k: s[k] for k in ("k_cache", "v_cache", "k_scale", "v_scale")}
        out, lse = binding.treeflash_tree_attention(s["q"], s["k_new"], s["v_new"], s["mask"], s["context_len"],
                                                    s["block_table"], s["k_cache"], s["v_cache"], s["k_scale"],
                                                    s["v_scale"], s["scale"])
        return {"out": out, "lse": lse}
    return {"sample": _sample_plain, "slots": _slots_plain, "append": _append_plain, "attend": _attend_plain}[kind](s)


def work(case):
    kind = case["kind"]
    es = 4 if case.get("dt") == "f32" else 2
    b = case["b"]
    if kind == "sample":
        rows = b * case["n"]
        # one comparison, one exponential and one sum for each logit
        return {"bytes": rows * case["V"] * es + rows * 12 + b * 16, "flops": 3 * rows * case["V"]}
    if kind == "slots":
        n = sum(_added(case))
        fresh = sum(y - x for x, y in zip(_pages_of(_contexts(case), case["page"]),
                                          _pages_of([c + a for c, a in zip(_contexts(case), _added(case))], case["page"])))
        return {"bytes": 12 * n + 8 * fresh + 16 * b + (4 * n if case["accepted"] else 0), "flops": 6 * n}
    row = case["heads"] * case["D"]
    if kind == "append":
        n, ctx = sum(_added(case)), _contexts(case)
        pages = sum(y - x // case["page"] for x, y in zip(ctx, _pages_of([c + a for c, a in zip(ctx, _added(case))], case["page"])))
        return {"bytes": n * (2 * row * (es + 1) + 8) + pages * case["heads"] * 16, "flops": 6 * n * row}
    n, group = case["n"], case["group"]
    ctx = sum(_contexts(case))
    pairs = n * ctx + (b * n * (n + 1) // 2 if not case["tree"] else b * n * min(n, 6))
    return {"bytes": 2 * ctx * row + ctx // case["page"] * (case["heads"] * 8 + 4)
            + b * n * (2 * row + 2 * row * group) * es + b * n * case["heads"] * group * 4 + (b * n * n if case["tree"] else 0),
            "flops": 4 * pairs * row * group}


# ------------------------------------------------------------------ in 64 bits

def _exact_sample(s):
    """Row by row: the kept tokens as a set, their mass and the log-probability of the one that is drawn."""
    b, n, V = s["logits"].shape
    lp = torch.empty((b, n), dtype=torch.float64, device="cuda")
    for i in range(b):
        t, k, p, m = (float(s[f][i]) for f in ("temperature", "top_k", "top_p", "min_p"))
        for j in range(n):
            z = s["logits"][i, j].double().nan_to_num(nan=float("-inf"), posinf=float("inf"), neginf=float("-inf"))
            if t <= 0:
                lp[i, j] = 0.0
                continue
            x = (z - z.max()) / t
            order = torch.argsort(-x, stable=True)
            if 0 < k < V:
                order = order[:int(k)]
            mass = torch.exp(x[order])
            if p < 1:
                total = mass.sum()
                order = order[torch.cumsum(mass, 0) - mass < p * total]
            order = order[torch.exp(x[order]) >= m]
            kept = torch.sort(order).values
            c = torch.cumsum(torch.exp(x[kept]), 0)
            at = torch.searchsorted(c, s["uniform"][i, j].double() * c[-1], right=True)
            lp[i, j] = x[kept[at.clamp(max=kept.numel() - 1)]] - torch.log(c[-1])
    return {"token": None, "logprob": lp}


def _exact_attend(s):
    """Sequence by sequence and head by head, each over the tokens it holds."""
    b, n, hq, D = s["q"].shape
    heads, page = s["k_new"].shape[2], s["k_cache"].shape[2]
    out = torch.zeros((b, n, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((b, n, hq), dtype=torch.float64, device="cuda")
    chain = torch.tril(torch.ones((n, n), dtype=torch.bool, device="cuda"))
    for i in range(b):
        T = int(s["context_len"][i])
        pages = s["block_table"][i, :-(-T // page)].long()
        sees = chain if s["mask"] is None else s["mask"][i] != 0
        k8, v8 = s["k_cache"].view(torch.uint8)[pages], s["v_cache"].view(torch.uint8)[pages]
        for h in range(heads):
            k = k8[:, h].contiguous().view(torch.float8_e4m3fn).double() * s["k_scale"][pages, h].double()[:, None, None]
            v = v8[:, h].contiguous().view(torch.float8_e4m3fn).double() * s["v_scale"][pages, h].double()[:, None, None]
            k = torch.cat([k.reshape(-1, D)[:T], s["k_new"][i, :, h].double()])
            v = torch.cat([v.transpose(1, 2).reshape(-1, D)[:T], s["v_new"][i, :, h].double()])
            for a in range(h * (hq // heads), (h + 1) * (hq // heads)):
                z = s["scale"] * (s["q"][i, :, a].double() @ k.t())
                z[:, T:] = torch.where(sees, z[:, T:], float("-inf"))
                lse[i, :, a] = torch.logsumexp(z, -1)
                out[i, :, a] = torch.softmax(z, -1) @ v
    return {"out": out, "lse": lse}


def _exact_append(s):
    """Scales and codes page by page: every value is the nearest of the 8-bit values times the scale."""
    got = {}
    for name, cache in (("k", s["k_cache"].view(torch.uint8)), ("v", s["v_cache"].view(torch.uint8).transpose(2, 3))):
        page = cache.shape[2]
        values = cache.contiguous().view(torch.float8_e4m3fn).double()
        scale = s[name + "_scale"].double()
        rows = s[name + "_new"][s["source"].long()].double()
        slot = s["slot"].long()
        starts = [0] + ((slot[1:] != slot[:-1] + 1) | (slot[1:] % page == 0)).nonzero()[:, 0].add(1).tolist() + [slot.numel()]
        first = slot[torch.tensor(starts[:-1], device="cuda")].tolist()
        for lo, hi, sl in zip(starts[:-1], starts[1:], first):
            p, o = sl // page, sl % page
            x = rows[lo:hi].transpose(0, 1)
            want = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / E4M3_MAX)))
            if o:
                want = torch.maximum(want, scale[p])
                values[p, :, :o] = (values[p, :, :o] * (scale[p] / want)[:, None, None]).to(torch.float8_e4m3fn).double()
            scale[p] = want
            values[p, :, o:o + hi - lo] = (x / want[:, None, None]).to(torch.float8_e4m3fn).double()
        got[name + "_cache"] = (values if name == "k" else values.transpose(2, 3)).contiguous()
        got[name + "_scale"] = scale
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    if case["kind"] == "append":
        return _exact_append(s)
    return _exact_attend(s) if case["kind"] == "attend" else None
