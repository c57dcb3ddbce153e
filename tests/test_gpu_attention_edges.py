"""Attention over caches whose other pages hold nothing of use, and over contexts near the largest length."""
import numpy as np
import pytest
import torch

from paper_2606_03819_amd import binding
from verify_step import check_attention, i32, make_cache, tables, tree_masks

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_pages_that_no_sequence_holds(D, page, dt):
    """Neither codes nor scales of other pages count: not behind a sequence's last token, and not where a table entry
    is no page, page 0 among them."""
    rng = np.random.default_rng(D + page)
    b, n, Hq, H = 5, 3, 4, 2
    ctx = [page + 5, 3 * page - 7, 1, page, 0]
    cols = 5
    order = 1 + rng.permutation(30)                       # page 0 and most others are nobody's
    table = np.zeros((b, cols), dtype=np.int32)
    at = 0
    for s, c in enumerate(ctx):
        held = -(-c // page)
        table[s, :held] = order[at:at + held]
        table[s, held:] = rng.choice([-1, 0, 31, 32, 10 ** 9, order[-1]], cols - held)
        at += held
    table[1, 1] = -5                                      # a hole in the middle
    owned = sorted({int(table[s, p]) for s, c in enumerate(ctx) for p in range(-(-c // page)) if 0 <= table[s, p] < 32})
    clean = make_cache(rng, 32, H, page, D)
    q, k, v = (torch.tensor(rng.standard_normal((b, n, h, D))).to(dt).cuda() for h in (Hq, H, H))
    mask = torch.tensor(tree_masks(rng, b, n)).cuda()
    others = torch.ones((32,), dtype=torch.bool, device="cuda")
    others[owned] = False
    for bad in (float("nan"), float("inf"), -float("inf"), 0.0, -1.0, 3e38):
        print(D, page, dt, bad, flush=True)
        cache = {f: t.clone() for f, t in clean.items()}
        for f in ("k", "v"):
            cache[f + "_scale"][others] = bad
            cache[f + "_cache"].view(torch.uint8)[others] = 127
        out, lse = binding.treeflash_tree_attention(q, k, v, mask, i32(ctx), i32(table), **cache, scale=0.2)
        check_attention(out, lse, q, k, v, mask, ctx, i32(table), clean, 0.2)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("page", [16, 64])
def test_value_scales_at_both_ends_of_their_range(page, dt):
    """Pages whose values are nothing (the smallest scale) beside pages of the largest: the former's tokens have their
    part in the sum of weights all the same."""
    rng = np.random.default_rng(page)
    n, Hq, H, D, pages = 2, 4, 2, 64, 8
    for loud in (64, 40, 62):
        for first in (0, 1):
            cache = make_cache(rng, pages, H, page, D, 0)
            cache["v_scale"][:] = 2.0 ** loud
            quiet = torch.arange(pages, device="cuda") % 2 == first
            cache["v_scale"][quiet] = 2.0 ** -64
            cache["v_cache"].view(torch.uint8)[quiet] = 0
            table = i32([list(range(pages)), [3, 0, 2, 1, 5, 4, 6, 7]])
            ctx = [pages * page - 3, 2 * page]
            q, k = (torch.tensor(rng.standard_normal((2, n, h, D))).to(dt).cuda() for h in (Hq, H))
            v = torch.zeros_like(k)
            print(page, dt, loud, first, flush=True)
            out, lse = binding.treeflash_tree_attention(q, k, v, None, i32(ctx), table, **cache, scale=0.01)
            check_attention(out, lse, q, k, v, None, ctx, table, cache, 0.01)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("page", [16, 128])
def test_contexts_near_the_largest_length(page, dt):
    """Tables of 2^31 tokens whose entries are pages at their two ends only: the last range ends with the context."""
    rng = np.random.default_rng(page)
    n, Hq, H, D = 2, 2, 1, 64
    cols = 0x7fffff00 // page
    table = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 2
    cache = make_cache(rng, 4, H, page, D)
    q, k, v = (torch.tensor(rng.standard_normal((1, n, h, D))).to(dt).cuda() for h in (Hq, H, H))
    for ctx in (cols * page, cols * page - 7, cols * page - (1 << 25) - 5, (1 << 31) - (1 << 26) + 3):
        last = (ctx - 1) // page
        table[0, last], few = 1, page + (ctx - 1) % page + 1
        print(page, dt, ctx, flush=True)
        out, lse = binding.treeflash_tree_attention(q, k, v, None, i32([ctx]), table, **cache, scale=0.2)
        check_attention(out, lse, q, k, v, None, [few], i32([[2, 1]]), cache, 0.2)
        table[0, last] = -1


@pytest.mark.parametrize("dt", DTYPES)
def test_calls_repeat_themselves_whatever_the_workspace_holds(dt):
    rng = np.random.default_rng(11)
    for b, n, ctx in ((1, 1, [4000]), (3, 33, [1500, 0, 701]), (2, 150, [64, 900])):
        table, pages, _ = tables(rng, ctx, 64, 64)
        cache = make_cache(rng, pages, 2, 64, 128)
        q, k, v = (torch.tensor(rng.standard_normal((b, n, h, 128))).to(dt).cuda() for h in (8, 2, 2))
        args = (q, k, v, torch.tensor(tree_masks(rng, b, n)).cuda(), i32(ctx), i32(table))
        ws = binding.alloc_workspace(binding.treeflash_tree_attention_workspace_bytes(b, n, 8, 2, 128, 64, 64, dt), q.device)
        got = []
        for fill in (0, 255, 127):
            ws.fill_(fill)
            got.append(binding.treeflash_tree_attention(*args, **cache, scale=0.1, workspace=ws))
        for out, lse in got[1:]:
            assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])
