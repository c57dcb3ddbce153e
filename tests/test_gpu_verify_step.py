"""The verification step beside the tree on the GPU against the 64-bit oracle: sampled tokens, slots and cached
codes exactly, attention within bounds that verify_step.check_attention derives; then the whole step as a decoding
loop makes it, eagerly and as a replayed graph."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_03819_amd import binding
from verify_step import E4, cache_np, check_attention, codes, f64, i32, make_cache, tables, tree_masks

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ sampling

def check_sample(logits, u, t=None, k=None, p=None, m=None, **kw):
    f = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt).cuda()  # noqa: E731
    f32 = torch.float32
    tt, kk, pp, mm = f(t, f32), f(k, torch.int32), f(p, f32), f(m, f32)
    tok, lp = binding.treeflash_sample(logits, u, tt, kk, pp, mm, **kw)
    torch.cuda.synchronize()
    b, n, V = logits.shape
    z, uu = f64(logits), f64(u)
    val = lambda x, s, d: d if x is None else float(x[s])  # noqa: E731
    for s in range(b):
        for i in range(n):
            want = oracle.sample_row(z[s, i], uu[s, i], val(tt, s, 1.0), int(val(kk, s, 0)), val(pp, s, 1.0), val(mm, s, 0.0))
            assert int(tok[s, i]) == want[0], (s, i, want[0])
            # one rounding to fp32 of a value and the weights' own 2^-40
            assert float(lp[s, i]) == pytest.approx(want[1], rel=2.0 ** -23, abs=2.0 ** -30)
    return tok, lp


def likely(rng, b, n, V, dt, steps=None):
    z = rng.standard_normal((b, n, V)) * 2.2
    for _ in range(min(20, V)):
        z[np.arange(b)[:, None], np.arange(n)[None], rng.integers(0, V, (b, n))] += rng.uniform(3, 12)
    if steps:
        z = np.round(z * steps) / steps   # ties
    return torch.tensor(z).to(dt).cuda()


SETTINGS = [dict(), dict(t=0.7), dict(t=0.0), dict(k=1), dict(k=20, t=0.6), dict(k=100), dict(k=2000), dict(p=0.9),
            dict(p=0.5, t=1.5), dict(m=0.05), dict(m=1.0), dict(m=2.0), dict(p=0.0), dict(k=20, p=0.95, t=0.6),
            dict(k=50, p=0.8, m=0.02, t=1.2), dict(p=0.999, m=1e-4), dict(k=-1, p=1.0, m=0.0), dict(k=500, p=0.99, t=3.0)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4096, 4099, 30011])
def test_sample_matches_the_oracle(V, dt):
    rng = np.random.default_rng(V)
    b, n = len(SETTINGS), 3
    get = lambda f, d: [s.get(f, d) for s in SETTINGS]  # noqa: E731
    for steps in (None, 4):
        print(f"V {V} {dt} steps {steps}", flush=True)
        z = likely(rng, b, n, V, dt, steps)
        u = torch.tensor(rng.random((b, n)), dtype=torch.float32).cuda()
        check_sample(z, u, get("t", 1.0), get("k", 0), get("p", 1.0), get("m", 0.0))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_sample_at_a_whole_vocabulary(dt):
    rng = np.random.default_rng(9)
    V = 151936
    sets = [dict(), dict(k=20, p=0.95, t=0.6), dict(p=0.9), dict(k=1000, p=0.8), dict(m=0.1, t=1.3), dict(k=64), dict(k=65)]
    get = lambda f, d: [s.get(f, d) for s in sets]  # noqa: E731
    z = likely(rng, len(sets), 2, V, dt)
    u = torch.tensor(rng.random((len(sets), 2)), dtype=torch.float32).cuda()
    check_sample(z, u, get("t", 1.0), get("k", 0), get("p", 1.0), get("m", 0.0))


def test_sample_masked_rows_and_values_that_are_no_numbers():
    rng = np.random.default_rng(3)
    V, inf, nan = 5000, float("inf"), float("nan")
    for dt in (torch.bfloat16, torch.float32):
        z = rng.standard_normal((10, 1, V)).astype(np.float32)
        z[0] = -inf
        z[1] = nan
        z[2, 0, rng.permutation(V)[:4990]] = -inf          # a grammar that leaves ten tokens
        z[3] = torch.finfo(dt).min                         # a mask of the type's lowest value: all alike
        z[4, 0, 7:] = torch.finfo(dt).min
        z[5, 0, [17, 400, 4000]] = inf
        z[6, 0, ::2] = nan
        z[7] = 0.0
        z[7, 0, ::3] = -0.0                                # both zeros are one value
        z[8, 0, 1:] = -inf
        z[9] *= 1e30
        zt = torch.tensor(z).to(dt).cuda()
        for u in (0.0, 0.37, 0.9999999):
            uu = torch.full((10, 1), u, device="cuda")
            for kw in (dict(), dict(k=[3] * 10), dict(p=[0.6] * 10), dict(m=[0.5] * 10), dict(t=[0.0] * 10),
                       dict(k=[700] * 10, p=[0.5] * 10, t=[0.3] * 10)):
                print(dt, u, kw, flush=True)
                check_sample(zt, uu, **kw)
    tok, lp = binding.treeflash_sample(zt[:1], torch.zeros(1, 1, device="cuda"))
    assert int(tok) == -1 and float(lp) == -inf


def test_sample_numbers_outside_their_range_and_flat_rows():
    z = torch.zeros((1, 5, 40000), device="cuda")
    u = torch.tensor([[-1.0, float("nan"), 1.0, 2.0, 0.5]], device="cuda")
    tok, _ = binding.treeflash_sample(z, u)
    assert tok.tolist() == [[0, 0, 39999, 39999, 20000]]
    for kw in (dict(k=[30000]), dict(p=[0.5]), dict(k=[30000], p=[0.25])):   # as many ties as there are tokens
        check_sample(z, u, **kw)


@pytest.mark.parametrize("spread", [0.3, 0.8, 1.5])
def test_sample_of_rows_of_little_spread(spread):
    """Thousands of tokens within a sixteenth of the border's logit."""
    rng = np.random.default_rng(17)
    V = 151936
    sets = [dict(p=0.9), dict(k=40000), dict(k=60000, p=0.5), dict(m=0.3), dict(p=0.9, m=0.25)]
    get = lambda f, d: [s.get(f, d) for s in sets]  # noqa: E731
    for dt in (torch.bfloat16, torch.float32):
        z = torch.tensor(spread * rng.standard_normal((len(sets), 2, V)), dtype=torch.float32).to(dt).cuda()
        u = torch.tensor(rng.random((len(sets), 2)), dtype=torch.float32).cuda()
        check_sample(z, u, get("t", 1.0), get("k", 0), get("p", 1.0), get("m", 0.0))


def test_sample_of_padded_and_offset_rows():
    rng = np.random.default_rng(5)
    for dt in (torch.bfloat16, torch.float32):
        wide = likely(rng, 4, 7, 3011, dt)
        wide[..., 3000:] = 1e4      # padding that would win
        wide[..., :1] = 1e4
        z = wide[..., 1:3000]       # rows that start at any element
        u = torch.tensor(rng.random((4, 7)), dtype=torch.float32).cuda()
        check_sample(z, u, [0.8] * 4, [0, 20, 0, 300], [1.0, 0.9, 0.7, 1.0])


def test_sample_of_many_rows():
    """More rows than one dimension of a launch holds; settings that are not numbers are off, or the largest logit."""
    rng = np.random.default_rng(31)
    b, n, V = 211, 191, 7
    nan = float("nan")
    z = likely(rng, b, n, V, torch.float32, 2)
    u = torch.tensor(rng.random((b, n)), dtype=torch.float32).cuda()
    f = dict(dtype=torch.float32, device="cuda")
    t = torch.full((b,), 1.0, **f)
    p, m = torch.full((b,), nan, **f), torch.full((b,), nan, **f)
    t[::3], t[1::3] = nan, float("inf")
    tok, lp = binding.treeflash_sample(z, u, t, None, p, m)
    top = z.argmax(-1).to(torch.int32)      # the first of equal ones
    assert torch.equal(tok[::3], top[::3]) and not lp[::3].any()
    # an infinite temperature makes all tokens alike: the u V-th of them
    assert torch.equal(tok[1::3], (u[1::3].double() * V).floor().to(torch.int32))
    w = torch.softmax(z[2::3].double(), -1).cumsum(-1)
    want = (w <= u[2::3].double()[..., None]).sum(-1).clamp(max=V - 1)
    assert torch.equal(tok[2::3].long(), want)


def test_sample_shares_follow_the_probabilities():
    """Random numbers on a grid give each token its share of them, to one step of the grid."""
    z = torch.tensor([3.0, 1.0, -1.0, 2.0, 0.0], device="cuda").expand(1, 4096, 5).contiguous()
    u = ((torch.arange(4096, device="cuda") + 0.5) / 4096)[None]
    tok, _ = binding.treeflash_sample(z, u)
    share = torch.bincount(tok[0].long(), minlength=5).double().cpu() / 4096
    assert torch.all((share - torch.softmax(z[0, 0].double().cpu(), 0)).abs() <= 1 / 4096)


def test_sample_without_rows_of_its_own_workspace():
    rng = np.random.default_rng(6)
    z = likely(rng, 2, 3, 20000, torch.bfloat16)
    u = torch.tensor(rng.random((2, 3)), dtype=torch.float32).cuda()
    ws = binding.alloc_workspace(binding.treeflash_sample_workspace_bytes(5, 9, 20000), z.device)
    ws.fill_(255)   # nothing that is there is read
    a = check_sample(z, u, p=[0.9, 1.0], workspace=ws)
    b = check_sample(z, u, p=[0.9, 1.0], workspace=ws)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ slots

def check_slots(ctx, add, acc, stack, count, table, n, page, max_tokens):
    want = oracle.cache_slots(ctx, add, acc, stack, count, table, n, page, max_tokens)
    t = i32(table)
    got = binding.treeflash_cache_slots(i32(ctx), i32(add), i32(stack), i32([count]), t, page, max_tokens,
                                        accepted=None if acc is None else i32(acc), n=n)
    torch.cuda.synchronize()
    assert int(got["status"]) == want["status"]
    for f in ("context_len", "start", "page_start", "slot", "position", "source", "block_table"):
        assert np.array_equal(got[f].cpu().numpy(), want[f]), f
    assert int(got["free_count"]) == want["free_count"]
    # in place
    c, fc, t2 = i32(ctx), i32([count]), i32(table)
    out = {f: torch.empty_like(v) for f, v in got.items()}
    out.update(context_len=c, free_count=fc)
    binding.treeflash_cache_slots(c, i32(add), i32(stack), fc, t2, page, max_tokens,
                                  accepted=None if acc is None else i32(acc), n=n, out=out)
    for f in got:
        assert torch.equal(out[f], got[f]), f
    return want


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("b,most", [(1, 1), (3, 40), (16, 300), (700, 9), (1500, 30), (40, 1500)])
def test_slots_match_the_oracle(b, most, page):
    rng = np.random.default_rng(b * page)
    ctx = rng.integers(0, 5 * page, b)
    ctx[:: 3] = ctx[::3] // page * page    # lengths that end with a page, zero among them
    add = rng.integers(0, most + 1, b)     # sequences that gain nothing, too
    cols = int(max(-(-(c + a) // page) for c, a in zip(ctx, add))) + 1
    table, pages, stack = tables(rng, ctx, page, cols, spare=int(sum(-(-(c + a) // page) for c, a in zip(ctx, add))) + 3)
    total = max(1, int(add.sum()))
    w = check_slots(ctx, add, None, stack, len(stack), table, 0, page, total)
    assert w["status"] == 0
    check_slots(ctx, add, None, stack, len(stack) - 2, table, most, page, total + 7)
    taken = int(w["page_start"][-1])
    assert check_slots(ctx, add, None, stack, taken, table, 0, page, total)["free_count"] == 0
    if taken > 0:
        assert check_slots(ctx, add, None, stack, taken - 1, table, 0, page, total)["status"] == 4
    if add.sum() > 1:
        assert check_slots(ctx, add, None, stack, len(stack), table, 0, page, int(add.sum()) - 1)["status"] == 2


@pytest.mark.parametrize("b,gamma,n", [(1, 1, 2), (5, 7, 33), (300, 16, 65), (1200, 16, 33)])
def test_slots_of_accepted_paths(b, gamma, n):
    rng = np.random.default_rng(b)
    page, cols = 32, 6
    ctx = rng.integers(0, 5 * page, b)
    ln = rng.integers(0, gamma + 1, b)
    acc = np.stack([np.sort(rng.permutation(max(n - 1, gamma))[:gamma]) for _ in range(b)])
    acc = np.where(np.arange(gamma) < ln[:, None], acc, -1).astype(np.int32)
    table, pages, stack = tables(rng, ctx, page, cols, spare=b + 1)
    assert check_slots(ctx, ln, acc, stack, len(stack), table, max(n, gamma + 1), page, b * (gamma + 1))["status"] == 0


def test_slots_refuse_impossible_lengths():
    table = np.arange(8, dtype=np.int32).reshape(2, 4)
    stack = np.array([8, 9, 10], dtype=np.int32)
    ok = ([10, 20], [3, 4], None, stack, 3, table, 0, 16, 20)
    assert check_slots(*ok)["status"] == 0
    for at, value, status in ((0, [-1, 20], 1), (1, [3, -4], 1), (4, -1, 1), (4, 4, 1), (6, 3, 1), (0, [10, 61], 3),
                              (1, [60, 4], 2), (1, [55, 4], 3)):
        args = list(ok)
        args[at] = value
        if status == 3:
            args[8] = 100
        assert check_slots(*args)["status"] == status, (at, value)


def test_release_gives_pages_back_and_slots_take_them_again():
    rng = np.random.default_rng(8)
    b, page, cols = 1100, 16, 6
    ctx = rng.integers(0, cols * page, b).astype(np.int32)
    table, pages, stack = tables(rng, ctx, page, cols, spare=5)
    done = (rng.random(b) < 0.4).astype(np.uint8)
    free = np.concatenate([stack, np.full(pages - len(stack), -7, np.int32)])
    c, f, fc, t = i32(ctx), i32(free), i32([len(stack)]), i32(table)
    d = torch.tensor(done).cuda()
    binding.treeflash_cache_release(d, c, t, f, fc, page)
    want = list(stack)
    for s in range(b):
        if done[s]:
            want += [int(table[s, p]) for p in range(-(-int(ctx[s]) // page))]
    assert int(fc) == len(want) and f[:len(want)].tolist() == want and np.all(f[len(want):].cpu().numpy() == -7)
    assert np.array_equal(c.cpu().numpy(), np.where(done, 0, ctx))
    binding.treeflash_cache_release(d, c, t, f, fc, page)   # they hold nothing any more
    assert int(fc) == len(want)
    out = binding.treeflash_cache_slots(c, i32(done.astype(int)), f, fc, t, page, b)
    assert int(out["status"]) == 0 and int(out["free_count"]) == len(want) - done.sum()
    assert out["slot"][:int(done.sum())].tolist() == [want[-1 - i] * page for i in range(int(done.sum()))]


def test_release_of_long_sequences_stops_at_the_stack_s_end():
    """More pages of a sequence than a wave has lanes; pages past the stack are dropped, what lies behind it stays."""
    page, cols, b = 16, 300, 3
    table = torch.arange(b * cols, dtype=torch.int32, device="cuda").view(b, cols)
    ctx = i32([page * 200 - 3, page * 299 + 1, page * cols])
    room = torch.full((1100,), -7, dtype=torch.int32, device="cuda")
    free, fc = room[:600], i32([5])
    binding.treeflash_cache_release(torch.ones((b,), dtype=torch.uint8, device="cuda"), ctx, table, free, fc, page)
    want = [-7] * 5 + list(range(200)) + list(range(cols, 2 * cols)) + list(range(2 * cols, 3 * cols))
    assert int(fc) == 600 and free.tolist() == want[:600] and (room[600:] == -7).all() and not ctx.any()


# ------------------------------------------------------------------ append

def check_append(cache, k, v, slot, source=None):
    kc, vc, ks, vs = cache_np(cache)
    R, H, D = k.shape
    want = oracle.cache_append(f64(k), f64(v), slot, source, kc, vc, ks, vs)
    binding.treeflash_cache_append(k, v, i32(slot), **cache, source=None if source is None else i32(source))
    torch.cuda.synchronize()
    for name, w in zip(("k_scale", "v_scale"), want[2:]):
        assert np.array_equal(f64(cache[name]), w), name
    for name, w in zip(("k_cache", "v_cache"), want[:2]):
        got = codes(cache[name])
        nan = np.isnan(oracle.E4M3_VALUES)
        # zeros of both signs are one value
        same = (got == w) | ((got & 127) == 0) & ((w & 127) == 0) | nan[got] & nan[w]
        assert same.all(), f"{name}: {np.argwhere(~same)[:5]}"


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_matches_the_oracle(page, D, dt):
    rng = np.random.default_rng(page + D)
    for H, lens, adds in ((1, [0], [1]), (2, [5, 0, page, 2 * page - 1], [1, page, 3, 2 * page + 5]), (3, [1, 37, 15], [16, 17, 5])):
        print(page, D, dt, H, flush=True)
        after = [x + a for x, a in zip(lens, adds)]
        table, pages, _ = tables(rng, after, page, max(-(-x // page) for x in after))
        cache = make_cache(rng, pages, H, page, D)
        slot = np.array([table[s, t // page] * page + t % page for s in range(len(lens)) for t in range(lens[s], after[s])])
        N = len(slot)
        # sizes of all kinds: some runs raise a scale, some do not, one page's values are nothing
        size = 10.0 ** rng.uniform(-3, 2, (N, 1, 1))
        size[: N // 5] = 0.0
        kv = torch.tensor(rng.standard_normal((N + 3, 2 * H, D)) * np.concatenate([size, np.ones((3, 1, 1))])).to(dt).cuda()
        check_append(cache, kv[:N, :H], kv[:N, H:], slot)
        source = rng.integers(-1, N + 5, N)      # rows twice, and rows that are none
        check_append(cache, kv[:, :H], kv[:, H:], slot, source)
        holes = np.where(rng.random(N) < 0.2, -1, slot)
        first = np.concatenate([[True], (slot[1:] != slot[:-1] + 1) | (slot[1:] % page == 0)])
        run = np.cumsum(first)
        holes = np.where([np.any(holes[run == r] < 0) for r in run], -1, slot)   # whole runs are left out
        check_append(cache, kv[:N, :H], kv[:N, H:], holes)


def test_append_of_many_tokens_at_once():
    rng = np.random.default_rng(4)
    H, page, D = 8, 64, 64
    lens, adds = [100, 0, 64], [1500, 3000, 2111]     # more rows a workgroup than one
    after = [x + a for x, a in zip(lens, adds)]
    table, pages, _ = tables(rng, after, page, max(-(-x // page) for x in after))
    cache = make_cache(rng, pages, H, page, D)
    slot = np.array([table[s, t // page] * page + t % page for s in range(3) for t in range(lens[s], after[s])])
    kv = torch.tensor(rng.standard_normal((len(slot), 2 * H, D))).to(torch.bfloat16).cuda()
    check_append(cache, kv[:, :H], kv[:, H:], slot)


def test_append_values_that_are_no_numbers_and_slots_outside():
    rng = np.random.default_rng(7)
    H, page, D = 2, 16, 64
    inf = float("inf")
    for dt in (torch.bfloat16, torch.float32):
        cache = make_cache(rng, 3, H, page, D)
        k = torch.tensor(rng.standard_normal((6, H, D))).to(dt).cuda()
        v = k.clone()
        k[0, 0, 3], k[1, 0, 4], v[2, 1, 5], v[3, 1, 6], k[4, 1, 0] = inf, float("nan"), -inf, float("nan"), torch.finfo(dt).max
        check_append(cache, k, v, np.array([18, 19, 20, 21, 22, 23]))
        check_append(cache, k, v, np.array([-1, 48, 2 ** 30, -(2 ** 31), 0, 1]))
        check_append(cache, torch.zeros_like(k), torch.zeros_like(v), np.array([32, 33, 34, 35, 36, 37]))


# ------------------------------------------------------------------ attention

def attention_case(rng, dt, b, n, Hq, H, D, page, ctx, chain=False, lens=None, spread=3):
    cols = max(1, max(-(-c // page) for c in ctx) + 1)
    table, pages, _ = tables(rng, ctx, page, cols)
    cache = make_cache(rng, pages, H, page, D, spread)
    for s, c in enumerate(ctx):   # what lies behind a sequence's tokens is NaN
        if c % page:
            p = table[s, c // page]
            cache["k_cache"].view(torch.uint8)[p, :, c % page:] = 127
            cache["v_cache"].view(torch.uint8)[p, :, :, c % page:] = 255
    qkv = torch.tensor(rng.standard_normal((b, n, Hq + 2 * H, D))).to(dt).cuda()
    mask = None if chain else torch.tensor(tree_masks(rng, b, n)).cuda()
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    args = (q, k, v, mask, i32(ctx), i32(table))
    kw, left = {}, None
    if lens is not None:
        left = (torch.full((b, n, Hq, D), 7.0, dtype=dt).cuda(), torch.full((b, n, Hq), 7.0).cuda())
        kw = dict(new_len=i32(lens), out=left[0].clone(), lse=left[1].clone())
    scale = 1.3 * D ** -0.5
    out, lse = binding.treeflash_tree_attention(*args, **cache, scale=scale, **kw)
    torch.cuda.synchronize()
    worst = check_attention(out, lse, q, k, v, mask, ctx, i32(table), cache, scale, lens, left)
    print(f"b{b} n{n} Hq{Hq} H{H} D{D} page{page} ctx{list(ctx)[:4]}: {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_matches_the_oracle(D, page, dt):
    rng = np.random.default_rng(D + page)
    for b, n, Hq, H, ctx, chain in ((1, 1, 1, 1, [0], False), (2, 1, 4, 1, [1, 333], True), (3, 5, 4, 2, [16, 0, 65], False),
                                    (1, 33, 8, 2, [300], False), (2, 17, 3, 3, [127, 129], True), (1, 9, 10, 2, [50], False),
                                    (2, 40, 8, 1, [31, 700], False), (1, 70, 5, 1, [100], True)):
        attention_case(rng, dt, b, n, Hq, H, D, page, ctx, chain)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_of_long_contexts(dt):
    rng = np.random.default_rng(12)
    attention_case(rng, dt, 2, 3, 8, 2, 128, 64, [5000, 4097])
    attention_case(rng, dt, 1, 1, 4, 1, 64, 128, [20001], chain=True)
    attention_case(rng, dt, 3, 1, 4, 1, 128, 16, [1, 3333, 17], chain=True)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_of_padded_batches(dt):
    rng = np.random.default_rng(13)
    attention_case(rng, dt, 4, 35, 8, 2, 64, 32, [0, 500, 64, 0], lens=[35, 2, 0, 1])
    attention_case(rng, dt, 3, 4, 6, 3, 128, 16, [700, 0, 5], chain=True, lens=[0, 4, 3])


def test_attention_of_a_large_tree():
    rng = np.random.default_rng(14)
    attention_case(rng, torch.bfloat16, 1, 513, 4, 1, 128, 64, [1111])
    attention_case(rng, torch.bfloat16, 2, 130, 2, 2, 64, 64, [0, 90], chain=True)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_of_many_positions_in_padded_batches(dt):
    """Several turns over the new positions, of which a row sees few, in batches that use a part of them."""
    rng = np.random.default_rng(18)
    attention_case(rng, dt, 3, 301, 2, 1, 128, 32, [0, 70, 33], lens=[301, 129, 257])
    attention_case(rng, dt, 2, 290, 6, 2, 64, 16, [9, 0], chain=True, lens=[290, 128])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_scales_of_very_different_size(dt):
    attention_case(np.random.default_rng(15), dt, 2, 5, 4, 2, 64, 16, [400, 33], spread=12)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_rows_without_anything_and_masked_nan(dt):
    rng = np.random.default_rng(16)
    b, n, Hq, H, D, page = 3, 6, 4, 2, 64, 16
    ctx = [0, 40, 0]
    table, pages, _ = tables(rng, ctx, page, 3)
    cache = make_cache(rng, pages, H, page, D)
    q = torch.tensor(rng.standard_normal((b, n, Hq, D))).to(dt).cuda()
    k = torch.tensor(rng.standard_normal((b, n, H, D))).to(dt).cuda()
    v = torch.tensor(rng.standard_normal((b, n, H, D))).to(dt).cuda()
    mask = torch.tensor(tree_masks(rng, b, n)).cuda()
    mask[:, :, 4] = 0          # nothing sees position 4, whose keys and values are not numbers
    mask[:, 4] = 0             # and it sees nothing new
    mask[0, 2] = 0             # a row of an empty context that sees nothing at all
    mask[mask != 0] = 200      # any value but 0 admits
    k[:, 4], v[:, 4] = float("nan"), float("inf")
    args = (q, k, v, mask, i32(ctx), i32(table))
    out, lse = binding.treeflash_tree_attention(*args, **cache, scale=0.2)
    kz, vz = k.clone(), v.clone()
    kz[:, 4], vz[:, 4] = 0, 0
    check_attention(out, lse, q, kz, vz, mask, ctx, i32(table), cache, 0.2)
    assert not out[0, 2].any() and torch.all(torch.isneginf(lse[0, 2])) and not out[2, 4].any()
    bad = table.copy()         # table entries that are no page: their tokens are not there
    bad[1, 0], bad[1, 2] = -1, pages
    out, lse = binding.treeflash_tree_attention(*args[:5], i32(bad), **cache, scale=0.2)
    check_attention(out, lse, q, kz, vz, mask, ctx, i32(bad), cache, 0.2)
    # lengths outside the table's
    long = [-5, 10 ** 6, 0]
    out, lse = binding.treeflash_tree_attention(q, k, v, mask, i32(long), i32(table), **cache, scale=0.2)
    check_attention(out, lse, q, kz, vz, mask, [0, 48, 0], i32(table), cache, 0.2)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_values_that_are_no_numbers_stay_with_their_rows(dt):
    """A new position whose key or value is not a number spoils the rows that attend to it, and only those."""
    rng = np.random.default_rng(20)
    b, n, Hq, H, D, page, ctx = 2, 41, 4, 2, 128, 16, [70, 0]
    table, pages, _ = tables(rng, ctx, page, 5)
    cache = make_cache(rng, pages, H, page, D)
    q, k, v = (torch.tensor(rng.standard_normal((b, n, h, D))).to(dt).cuda() for h in (Hq, H, H))
    mask = torch.tensor(tree_masks(rng, b, n)).cuda()
    kz, vz = k.clone(), v.clone()
    k[0, 3, 0, 5] = float("nan")
    v[0, 20, 1, 7], v[1, 40, 0, 9], v[1, 11, 0, 2] = float("nan"), float("-inf"), float("inf")
    out, lse = binding.treeflash_tree_attention(q, k, v, mask, i32(ctx), i32(table), **cache, scale=0.1)
    clean, clean_lse = binding.treeflash_tree_attention(q, kz, vz, mask, i32(ctx), i32(table), **cache, scale=0.1)
    sees = mask.bool()
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, :, :2] |= sees[0, :, 3, None, None]
    hit[0, :, 2:, 7] |= sees[0, :, 20, None]
    hit[1, :, :2, 9] |= sees[1, :, 40, None]
    hit[1, :, :2, 2] |= sees[1, :, 11, None]
    assert torch.equal(~torch.isfinite(out), hit)
    assert torch.equal(out[~hit], clean[~hit])
    assert torch.all(torch.isneginf(out[1, 40, :2, 9])) and torch.all(out[1, 11, :2, 2] == float("inf"))
    spoiled = sees[0, :, 3, None] & (torch.arange(Hq, device="cuda") < 2)
    assert torch.equal(torch.isnan(lse[0]), spoiled) and torch.equal(lse[1], clean_lse[1])


def test_attention_large_products():
    """Products that leave exp's range unless the largest is taken off first, of both signs."""
    rng = np.random.default_rng(17)
    for dt in (torch.bfloat16, torch.float32):
        table, pages, _ = tables(rng, [100], 16, 7)
        cache = make_cache(rng, pages, 1, 16, 64, 0)
        q = (torch.tensor(rng.standard_normal((1, 3, 2, 64))) * 60).to(dt).cuda()
        k, v = (torch.tensor(rng.standard_normal((1, 3, 1, 64))).to(dt).cuda() for _ in range(2))
        for scale in (0.5, -0.5, 0.0):
            out, lse = binding.treeflash_tree_attention(q, k, v, None, i32([100]), i32(table), **cache, scale=scale)
            check_attention(out, lse, q, k, v, None, [100], i32(table), cache, scale)


# ------------------------------------------------------------------ together

def step_state(seed):
    rng = np.random.default_rng(seed)
    b, gamma, M, B, H, Hq, D, page, V = 3, 5, 4, 15, 2, 4, 64, 16, 900
    ctx = [30, 0, 47]
    cols = 12
    table, pages, stack = tables(rng, ctx, page, cols, spare=20)
    t = dict(b=b, gamma=gamma, M=M, B=B, H=H, Hq=Hq, D=D, page=page, V=V, n=B + 1, cache=make_cache(rng, pages, H, page, D),
             ctx=i32(ctx), table=i32(table), stack=i32(stack), count=i32([len(stack)]))
    R = 1 + (gamma - 1) * M
    lp = torch.log_softmax(torch.tensor(rng.standard_normal((b, R, V)) * 2, dtype=torch.float32), -1)
    best = torch.sort(lp, dim=-1, descending=True, stable=True)
    t["cond_idx"], t["cond_lp"] = best.indices[..., :B].to(torch.int32).contiguous().cuda(), best.values[..., :B].contiguous().cuda()
    t["topk"] = torch.tensor(np.stack([[rng.permutation(V)[:M] for _ in range(gamma)] for _ in range(b)]), dtype=torch.int32).cuda()
    t["topk"][:, 0] = t["cond_idx"][:, 0, :M]       # the first depth's best nodes grow on
    t["root"] = i32(rng.integers(0, V, b))
    t["qkv"] = torch.tensor(rng.standard_normal((b, B + 1, Hq + 2 * H, D))).to(torch.bfloat16).cuda()
    t["w"] = torch.tensor(rng.standard_normal((Hq * D, V)) * 0.05, dtype=torch.float32).cuda()
    t["u"] = torch.tensor(rng.random((b, B + 1)), dtype=torch.float32).cuda()
    return t


def one_step(t):
    """Draft tree -> attention -> logits -> tokens -> walk -> slots -> cache, lengths and pages in place."""
    tree = binding.treeflash_build_tree(t["cond_idx"], t["cond_lp"], t["topk"], t["B"])
    inp = binding.treeflash_tree_attention_inputs(t["root"], tree)
    Hq, H = t["Hq"], t["H"]
    q, k, v = t["qkv"][:, :, :Hq], t["qkv"][:, :, Hq:Hq + H], t["qkv"][:, :, Hq + H:]
    att = binding.treeflash_tree_attention(q, k, v, inp["mask"], t["ctx"], t["table"], **t["cache"], scale=0.125)
    logits = (att[0].float().reshape(-1, Hq * t["D"]) @ t["w"]).reshape(t["b"], t["n"], t["V"])
    # half of the positions are made to agree with the tree, so that paths are accepted
    first = torch.full((t["b"], t["n"]), t["B"], dtype=torch.int64, device="cuda")
    first.scatter_reduce_(1, (tree["parent"] + 1).long(), torch.arange(t["B"], device="cuda").expand(t["b"], -1), "amin")
    agree = torch.cat([tree["token"], tree["token"][:, :1]], 1).gather(1, first).long()
    logits = logits + 20.0 * torch.nn.functional.one_hot(agree, t["V"]) * (t["u"] < 0.5)[..., None]
    tok, lp = binding.treeflash_sample(logits, t["u"])
    acc = binding.treeflash_accept(tree, tok, t["gamma"])
    i32e = dict(dtype=torch.int32, device="cuda")
    N = t["b"] * (t["gamma"] + 1)
    slots = dict(context_len=t["ctx"], free_count=t["count"], start=torch.empty(t["b"] + 1, **i32e),
                 page_start=torch.empty(t["b"] + 1, **i32e), slot=torch.empty(N, **i32e), position=torch.empty(N, **i32e),
                 source=torch.empty(N, **i32e), status=torch.empty(1, **i32e))
    binding.treeflash_cache_slots(t["ctx"], acc["accept_len"], t["stack"], t["count"], t["table"], t["page"], N,
                                  accepted=acc["accepted"], n=t["n"], out=slots)
    binding.treeflash_cache_append(k, v, slots["slot"], **t["cache"], source=slots["source"])
    return dict(out=att[0], lse=att[1], logits=logits, token=tok, logprob=lp, mask=inp["mask"], **acc, **slots)


def mutable(t):
    return [t["ctx"], t["table"], t["count"], *t["cache"].values()]


def test_a_decoding_loop_against_the_oracle():
    t = step_state(1)
    rng = np.random.default_rng(2)
    Hq, H = t["Hq"], t["H"]
    gained = 0
    for step in range(4):
        ctx, table, count = t["ctx"].tolist(), t["table"].cpu().numpy(), int(t["count"])
        before = {k: v.clone() for k, v in t["cache"].items()}
        t["u"] = torch.tensor(rng.random((t["b"], t["n"])), dtype=torch.float32).cuda()
        r = one_step(t)
        torch.cuda.synchronize()
        q, k, v = t["qkv"][:, :, :Hq], t["qkv"][:, :, Hq:Hq + H], t["qkv"][:, :, Hq + H:]
        check_attention(r["out"], r["lse"], q, k, v, r["mask"], ctx, i32(table), before, 0.125)
        for s in range(t["b"]):
            for i in range(t["n"]):
                assert int(r["token"][s, i]) == oracle.sample_row(f64(r["logits"][s, i]), float(t["u"][s, i]))[0]
        want = oracle.cache_slots(ctx, r["accept_len"].tolist(), r["accepted"].cpu().numpy(), t["stack"].tolist(), count, table,
                                  t["n"], t["page"], len(r["slot"]))
        assert want["status"] == int(r["status"]) == 0
        for f in ("context_len", "slot", "source", "block_table"):
            assert np.array_equal(r[f].cpu().numpy(), want[f])
        flat = lambda x: f64(x).reshape(-1, H, t["D"])  # noqa: E731
        kc, vc, ks, vs = oracle.cache_append(flat(k), flat(v), want["slot"], want["source"], *cache_np(before))
        assert np.array_equal(codes(t["cache"]["k_cache"]), kc) and np.array_equal(codes(t["cache"]["v_cache"]), vc)
        assert np.array_equal(f64(t["cache"]["k_scale"]), ks) and np.array_equal(f64(t["cache"]["v_scale"]), vs)
        gained += int(r["accept_len"].sum())
        t["qkv"] = torch.tensor(rng.standard_normal(tuple(t["qkv"].shape))).to(torch.bfloat16).cuda()
    assert gained > 4


def test_a_replayed_graph_of_the_step():
    t, e = step_state(3), step_state(3)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # warm up on a state of its own
        one_step(step_state(4))
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    start = [x.clone() for x in mutable(t)]
    with torch.cuda.graph(graph, stream=side):
        r = one_step(t)
    for x, y in zip(mutable(t), start):
        x.copy_(y)
    rng = np.random.default_rng(5)
    for replay in range(4):
        u = torch.tensor(rng.random((t["b"], t["n"])), dtype=torch.float32).cuda()
        t["u"].copy_(u)
        e["u"].copy_(u)
        graph.replay()
        torch.cuda.synchronize()
        w = one_step(e)
        torch.cuda.synchronize()
        for f in ("out", "lse", "token", "logprob", "accepted", "accept_len", "slot", "source", "start", "status"):
            assert torch.equal(r[f], w[f]), f
        for x, y in zip(mutable(t), mutable(e)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_paged_cache_of_two_layers():
    """Prompts, two decoding steps, a release and a new prompt through PagedCache, each layer against the oracle."""
    rng = np.random.default_rng(30)
    b, n, gamma, Hq, H, D, page, layers = 3, 9, 4, 4, 2, 64, 16, 2
    pc = binding.PagedCache(layers, b, n, gamma, Hq, H, D, num_pages=40, max_pages=12, page_size=page)
    ref = [cache_np(dict(k_cache=pc.k[i], v_cache=pc.v[i], k_scale=pc.k_scale[i], v_scale=pc.v_scale[i])) for i in range(layers)]
    state = dict(ctx=[0] * b, table=pc.block_table.cpu().numpy(), count=40)

    def plan(add, acc, n_rows, max_tokens):
        w = oracle.cache_slots(state["ctx"], add, acc, pc.free_pages.tolist(), state["count"], state["table"], n_rows, page, max_tokens)
        assert w["status"] == int(pc.status) == 0
        state.update(ctx=w["context_len"].tolist(), table=w["block_table"], count=w["free_count"])
        assert pc.context_len.tolist() == state["ctx"] and int(pc.free_count) == state["count"]
        assert np.array_equal(pc.block_table.cpu().numpy(), state["table"])
        return w

    def put(k, v, w):
        for i in range(layers):
            pc.append(i, k * (i + 1), v * (i + 1))
            ref[i] = oracle.cache_append(f64(k * (i + 1)).reshape(-1, H, D), f64(v * (i + 1)).reshape(-1, H, D), w["slot"],
                                         w["source"], *ref[i])
            got = cache_np(dict(k_cache=pc.k[i], v_cache=pc.v[i], k_scale=pc.k_scale[i], v_scale=pc.v_scale[i]))
            assert all(np.array_equal(x, y) for x, y in zip(got, ref[i]))

    def prompt(add):
        kv = torch.tensor(rng.standard_normal((sum(add), 2 * H, D))).to(torch.bfloat16).cuda()
        pc.extend(i32(add), sum(add) + 2)
        put(kv[:, :H], kv[:, H:], plan(add, None, 0, sum(add) + 2))

    prompt([37, 5, 70])
    for step in range(3):
        qkv = torch.tensor(rng.standard_normal((b, n, Hq + 2 * H, D))).to(torch.bfloat16).cuda()
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        mask = torch.tensor(tree_masks(rng, b, n)).cuda()
        for i in range(layers):
            out, lse = pc.attend(i, q, k, v, mask, 0.1)
            cache = dict(k_cache=pc.k[i], v_cache=pc.v[i], k_scale=pc.k_scale[i], v_scale=pc.v_scale[i])
            check_attention(out, lse, q, k, v, mask, state["ctx"], pc.block_table, cache, 0.1)
        ln = rng.integers(0, gamma + 1, b)
        acc = np.where(np.arange(gamma) < ln[:, None], np.sort(rng.permutation(n - 1)[:gamma]), -1).astype(np.int32)
        acc = np.broadcast_to(acc, (b, gamma)).copy()
        pc.advance(dict(accept_len=i32(ln), accepted=i32(acc)))
        put(k, v, plan(ln, acc, n, b * (gamma + 1)))
        if step == 1:
            held = -(-state["ctx"][1] // page)
            pc.release(torch.tensor([0, 1, 0], dtype=torch.uint8).cuda())
            state["ctx"][1] = 0
            state["count"] += held
            assert int(pc.free_count) == state["count"]
            prompt([0, 20, 0])
    pc.extend(i32([1000, 0, 0]), 2000)      # more than the table holds: nothing happens
    assert int(pc.status) == 3 and pc.context_len.tolist() == state["ctx"]
    before = [x.view(torch.uint8).clone() for x in (*pc.k, *pc.v)]
    pc.append(0, k, v)
    assert all(torch.equal(x.view(torch.uint8), y) for x, y in zip((*pc.k, *pc.v), before))
    with pytest.raises(ValueError):
        binding.PagedCache(1, 1, 1, 1, 4, 2, 80, 4, 4)


def test_calls_on_two_streams_at_once():
    rng = np.random.default_rng(18)
    z = [likely(rng, 4, 5, 20000, torch.bfloat16) for _ in range(2)]
    u = torch.tensor(rng.random((4, 5)), dtype=torch.float32).cuda()
    p = torch.full((4,), 0.9, device="cuda")
    want = [binding.treeflash_sample(x, u, top_p=p) for x in z]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = binding.treeflash_sample(z[i], u, top_p=p)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_wrong_shapes_and_types_are_refused():
    rng = np.random.default_rng(19)
    cache = make_cache(rng, 4, 2, 16, 64)
    q, k = torch.zeros(1, 3, 4, 64, device="cuda"), torch.zeros(1, 3, 2, 64, device="cuda")
    args = dict(q=q, k_new=k, v_new=k, mask=None, context_len=i32([3]), block_table=i32([[0]]), scale=1.0, **cache)
    for name, bad, err in (("q", q.half(), TypeError), ("k_new", k.bfloat16(), TypeError), ("v_new", k[:, :2], ValueError),
                           ("mask", torch.zeros(1, 3, 4, dtype=torch.uint8, device="cuda"), ValueError),
                           ("mask", torch.zeros(1, 3, 3, device="cuda"), TypeError),
                           ("k_cache", cache["v_cache"], ValueError), ("k_scale", cache["k_scale"].double(), TypeError),
                           ("context_len", torch.zeros(1, dtype=torch.int64, device="cuda"), TypeError),
                           ("context_len", torch.zeros(1, dtype=torch.int32), ValueError)):
        with pytest.raises(err):
            binding.treeflash_tree_attention(**{**args, name: bad})
    with pytest.raises(ValueError):
        binding.treeflash_sample(torch.zeros(2, 3, 10, device="cuda"), torch.zeros(2, 2, device="cuda"))
    with pytest.raises(ValueError):
        binding.treeflash_sample(torch.zeros(2, 3, 1, device="cuda").expand(2, 3, 10), torch.zeros(2, 3, device="cuda"))
    with pytest.raises(binding.TreeflashError):
        binding.treeflash_sample(torch.zeros(1, 1, 10, device="cuda").expand(2, 3, 10), torch.zeros(2, 3, device="cuda"))
    with pytest.raises(ValueError):
        binding.treeflash_cache_append(k[0], k[0, :2], i32([0]), **cache)
