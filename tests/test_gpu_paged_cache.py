"""The paged cache's loop where not all goes at once: sequences that sit a step out, calls of another number of
positions than the cache was made for, and lists of several kinds beside a captured step."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_03819_amd import binding
from test_gpu_verify_step import check_slots
from verify_step import cache_np, check_attention, f64, i32, tables, tree_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,gamma,n", [(1, 1, 2), (6, 7, 33), (300, 16, 65), (1200, 16, 33)])
def test_slots_of_batches_of_which_some_sit_out(b, gamma, n):
    rng = np.random.default_rng(b + 1)
    page, cols = 32, 6
    ctx = rng.integers(0, 5 * page, b)
    ln = rng.integers(-1, gamma + 1, b)
    ln[:: 2] = -1
    ctx[::4] = 0
    acc = np.stack([np.sort(rng.permutation(max(n - 1, gamma))[:gamma]) for _ in range(b)])
    acc = np.where(np.arange(gamma) < ln[:, None], acc, -1).astype(np.int32)
    table, pages, stack = tables(rng, ctx, page, cols, spare=b + 1)
    rest = (stack, len(stack), table, max(n, gamma + 1), page, b * (gamma + 1))
    w = check_slots(ctx, ln, acc, *rest)
    assert w["status"] == 0 and np.array_equal(w["context_len"], ctx + ln + 1)
    assert check_slots(ctx, np.full(b, -1), acc, *rest)["free_count"] == len(stack)
    ln[b // 2] = -2
    assert check_slots(ctx, ln, acc, *rest)["status"] == 1
    ln[b // 2] = -1
    assert check_slots(ctx, ln, None, *rest)["status"] == 1


def test_released_sequences_sit_out_of_paged_steps():
    """A slot that is released gains no token and takes no page until it is filled again; eagerly and replayed."""
    rng = np.random.default_rng(40)
    b, n, gamma, Hq, H, D, page = 4, 9, 4, 4, 2, 64, 16
    pc = binding.PagedCache(1, b, n, gamma, Hq, H, D, num_pages=40, max_pages=8, page_size=page)
    kv = torch.tensor(rng.standard_normal((60, 2 * H, D))).to(torch.bfloat16).cuda()
    pc.extend(i32([17, 5, 16, 0]), 60)
    pc.append(0, kv[:, :H], kv[:, H:])
    pc.release(torch.tensor([0, 1, 0, 0], dtype=torch.uint8, device="cuda"))
    ctx, count = [17, 0, 16, 0], 40 - 3
    assert pc.context_len.tolist() == ctx and int(pc.free_count) == count
    qkv = torch.tensor(rng.standard_normal((b, n, Hq + 2 * H, D))).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    mask = torch.tensor(tree_masks(rng, b, n)).cuda()
    active = torch.tensor([1, 0, 1, 0], dtype=torch.uint8, device="cuda")
    new_len = n * active.to(torch.int32)
    walk = dict(accept_len=i32([1, 3, 0, 2]), accepted=i32([[0, 4, -1, -1], [1, 2, 3, -1], [-1] * 4, [0, 1, -1, -1]]))

    def step(which):
        out, lse = pc.attend(0, q, k, v, mask, 0.1, new_len=new_len)
        pc.advance(walk, active=which)
        pc.append(0, k, v)
        return out, lse

    def expect(which):
        acc = [[0, 4, -1, -1], [1, 2, 3, -1], [-1] * 4, [0, 1, -1, -1]]
        ln = [x if w else -1 for x, w in zip([1, 3, 0, 2], which)]
        cache = dict(k_cache=pc.k[0], v_cache=pc.v[0], k_scale=pc.k_scale[0], v_scale=pc.v_scale[0])
        w = oracle.cache_slots(pc.context_len.tolist(), ln, np.array(acc), pc.free_pages.tolist(), int(pc.free_count),
                               pc.block_table.cpu().numpy(), n, page, b * (gamma + 1))
        flat = lambda x: f64(x).reshape(-1, H, D)  # noqa: E731
        return w, oracle.cache_append(flat(k), flat(v), w["slot"], w["source"], *cache_np(cache))

    def check(want, kept):
        assert int(pc.status) == 0 and int(pc.free_count) == want["free_count"]
        assert np.array_equal(pc.context_len.cpu().numpy(), want["context_len"])
        assert np.array_equal(pc.block_table.cpu().numpy(), want["block_table"])
        got = cache_np(dict(k_cache=pc.k[0], v_cache=pc.v[0], k_scale=pc.k_scale[0], v_scale=pc.v_scale[0]))
        assert all(np.array_equal(x, y) for x, y in zip(got, kept))

    for which in (active, active.bool()):
        before = {f: [t.clone() for t in getattr(pc, f)] for f in ("k", "v", "k_scale", "v_scale")}
        old = pc.context_len.tolist(), pc.block_table.clone()
        want, kept = expect([1, 0, 1, 0])
        out, lse = step(which)
        check(want, kept)
        check_attention(out, lse, q, k, v, mask, old[0], old[1], dict(k_cache=before["k"][0], v_cache=before["v"][0],
                        k_scale=before["k_scale"][0], v_scale=before["v_scale"][0]), 0.1, new_len.tolist())
    assert pc.context_len.tolist() == [21, 0, 18, 0]

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(active)
    for who in ([1, 0, 1, 0], [0, 0, 0, 0], [1, 1, 1, 0], [0, 0, 0, 1]):
        active.copy_(torch.tensor(who, dtype=torch.uint8))
        want, kept = expect(who)
        graph.replay()
        check(want, kept)
    for bad, err in ((active.int(), TypeError), (active[:3], ValueError), (active.cpu(), ValueError), ([1, 0, 1, 0], TypeError)):
        with pytest.raises(err):
            pc.advance(walk, active=bad)


def test_status_is_the_last_call_s_on_the_gpu():
    """A captured advance replayed after an extend, and an extend after a replay, each leave their own status."""
    b, gamma, page = 2, 3, 16
    pc = binding.PagedCache(1, b, 5, gamma, 2, 1, 64, num_pages=6, max_pages=5, page_size=page)
    walk = dict(accept_len=i32([3, 2]), accepted=i32([[0, 1, 2], [0, 3, -1]]))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pc.advance(walk)
    pc.extend(i32([14, 10]), 24)
    assert int(pc.status) == 0 and int(pc.free_count) == 4
    graph.replay()
    assert int(pc.status) == 0 and pc.context_len.tolist() == [18, 13] and int(pc.free_count) == 3
    pc.extend(i32([100, 0]), 100)                       # outgrows its table
    assert int(pc.status) == 3
    graph.replay()
    assert int(pc.status) == 0 and pc.context_len.tolist() == [22, 16] and int(pc.free_count) == 3
    pc.extend(i32([42, 0]), 42)                         # to the end of a page, of the last but one page
    assert int(pc.status) == 0 and pc.context_len.tolist() == [64, 16] and int(pc.free_count) == 1
    for _ in range(3):
        graph.replay()                                  # two more pages: there is one
        assert int(pc.status) == 4 and pc.context_len.tolist() == [64, 16]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_of_other_numbers_of_positions_than_the_cache_s(dt):
    """Prompt chunks and single tokens through a cache made for trees: a smaller n can need a larger workspace."""
    rng = np.random.default_rng(41)
    b, n, Hq, H, D, page = 2, 33, 8, 2, 64, 16
    pc = binding.PagedCache(1, b, n, 4, Hq, H, D, num_pages=400, max_pages=250, page_size=page, dtype=dt)
    cache = dict(k_cache=pc.k[0], v_cache=pc.v[0], k_scale=pc.k_scale[0], v_scale=pc.v_scale[0])
    ctx = [0, 0]
    for chunk, lens in ((70, None), (1, None), (33, [33, 20]), (1, [0, 1]), (200, [200, 3]), (7, None), (33, None)):
        qkv = torch.tensor(rng.standard_normal((b, chunk, Hq + 2 * H, D))).to(dt).cuda()
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        kw, left = {}, None
        if lens is not None:
            left = (torch.full((b, chunk, Hq, D), 7.0, dtype=dt).cuda(), torch.full((b, chunk, Hq), 7.0).cuda())
            kw = dict(new_len=i32(lens), out=left[0].clone(), lse=left[1].clone())
        out, lse = pc.attend(0, q, k, v, None, 0.1, **kw)
        assert out.shape == q.shape and lse.shape == q.shape[:3]
        assert (out.data_ptr() == pc.out.data_ptr()) == (chunk == n and lens is None)
        check_attention(out, lse, q, k, v, None, ctx, pc.block_table, cache, 0.1, lens, left)
        add = lens or [chunk] * b
        pc.extend(i32(add), b * chunk, n=chunk)
        pc.append(0, k, v)
        ctx = [c + a for c, a in zip(ctx, add)]
        assert int(pc.status) == 0 and pc.context_len.tolist() == ctx
    with pytest.raises(ValueError):
        pc.attend(0, q[:1], k[:1], v[:1], None, 0.1)
    with pytest.raises(ValueError):
        pc.attend(0, q[:, :, :4].contiguous(), k, v, None, 0.1)


def test_layers_attended_to_on_two_streams_at_once():
    """Contexts in many ranges, each stream with a workspace and outputs of its own."""
    rng = np.random.default_rng(42)
    b, n, Hq, H, D, page, ctx = 2, 5, 4, 1, 128, 64, [9000, 4001]
    pc = binding.PagedCache(2, b, n, 4, Hq, H, D, num_pages=220, max_pages=150, page_size=page)
    pc.extend(i32(ctx), sum(ctx))
    for i in range(2):
        kv = torch.tensor(rng.standard_normal((sum(ctx), 2 * H, D))).to(torch.bfloat16).cuda()
        pc.append(i, kv[:, :H], kv[:, H:])
    qkv = torch.tensor(rng.standard_normal((b, n, Hq + 2 * H, D))).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    want = [[t.clone() for t in pc.attend(i, q, k, v, None, 0.1)] for i in range(2)]
    own = [dict(out=torch.empty_like(pc.out), lse=torch.empty_like(pc.lse), workspace=torch.empty_like(pc.workspace))
           for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for kw in own:
            kw["out"].zero_(), kw["lse"].zero_(), kw["workspace"].fill_(255)
        torch.cuda.synchronize()
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                pc.attend(i, q, k, v, None, 0.1, **own[i])
        torch.cuda.synchronize()
        for kw, w in zip(own, want):
            assert torch.equal(kw["out"], w[0]) and torch.equal(kw["lse"], w[1])
