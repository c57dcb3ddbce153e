"""Inputs, and comparisons with the oracle, of the verification step beside the tree (used by its GPU tests)."""
import numpy as np
import torch

import oracle
from paper_2606_03819_amd import binding

E4 = torch.float8_e4m3fn
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def f64(t):
    return t.detach().cpu().double().numpy()


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def make_cache(rng, pages, H, page, D, spread=3):
    """A cache of random values: codes and power-of-two scales of several sizes, NaN nowhere."""
    k = oracle.e4m3_encode(rng.standard_normal((pages, H, page, D)) * 100)
    v = oracle.e4m3_encode(rng.standard_normal((pages, H, D, page)) * 100)
    ks = 2.0 ** rng.integers(-7 - spread, -6, (pages, H)).astype(np.float32)
    vs = 2.0 ** rng.integers(-7 - spread, -6, (pages, H)).astype(np.float32)
    return {"k_cache": torch.tensor(k).cuda().view(E4), "v_cache": torch.tensor(v).cuda().view(E4),
            "k_scale": torch.tensor(ks, dtype=torch.float32).cuda(), "v_scale": torch.tensor(vs, dtype=torch.float32).cuda()}


def cache_np(c):
    return codes(c["k_cache"]), codes(c["v_cache"]), f64(c["k_scale"]), f64(c["v_scale"])


def tree_masks(rng, b, n):
    m = np.zeros((b, n, n), dtype=np.uint8)
    for s in range(b):
        m[s, 0, 0] = 1
        for i in range(1, n):
            m[s, i] = m[s, rng.integers(max(0, i - 6), i)]
            m[s, i, i] = 1
    return m


def check_attention(got_out, got_lse, q, k_new, v_new, mask, ctx, table, cache, scale, new_len=None, left=None):
    """Every row against the oracle.

    Bound, with w the weights, W = sum |v| w / sum w, X the largest sum |q||k| scale and N the tokens: a product q.k
    of D terms summed in fp32, and its scaling, is off by (D + 8) 2^-24 X, so w by that, 2^-20 for exp2 and its
    argument's rounding (|x| 2^-24 log2 e at |x| <= 2 X), and for bf16 by half a step of fp16, 2^-11, or 2^-25 of the
    largest weight times value, at most 448 of the largest scale, where it is below fp16's normal range; new values
    enter with weights of at least 2^-15.  Sums of N terms add N 2^-24.  All of it counts twice (numerator and
    denominator), then half a step of the output's type."""
    b, n, Hq, D = q.shape
    dt = q.dtype
    kc, vc, ks, vs = cache_np(cache)
    worst = 0.0
    for s in range(b):
        nl = n if new_len is None else int(new_len[s])
        r = oracle.tree_attention(f64(q[s]), f64(k_new[s]), f64(v_new[s]), None if mask is None else mask[s].cpu().numpy(),
                                  int(ctx[s]), table[s].cpu().numpy(), kc, vc, ks, vs, scale, nl)
        N = max(int(ctx[s]), 0) + nl
        X = r["size"][..., None]
        w = (D + 8) * 2.0 ** -24 * X + 2.0 ** -20 + 4 * X * 2.0 ** -24 + N * 2.0 ** -24
        low = 0.0
        if dt == torch.bfloat16:
            w = w + 2.0 ** -11
            low = N * 2.0 ** -25 * 448 * float(vs.max())
        tol = 2 * w * r["absv"] + low + HALF_STEP[dt] * (np.abs(r["out"]) + 2 * w * r["absv"] + low) + 1e-30
        o, ls = f64(got_out[s]), f64(got_lse[s])
        err = np.abs(o[:nl] - r["out"][:nl])
        assert np.all(err <= tol[:nl]), f"sequence {s}: out off by {np.max(err / tol[:nl]):.2f} of the bound"
        worst = max(worst, float(np.max(err / tol[:nl], initial=0.0)))
        empty = np.isneginf(r["lse"][:nl])
        assert np.array_equal(empty, np.isneginf(ls[:nl]))
        ltol = (2 * w[:nl, :, 0] + 2.0 ** -22 * np.abs(np.where(empty, 0, r["lse"][:nl])) + 2.0 ** -22)
        d = np.abs(np.where(empty, 0, ls[:nl]) - np.where(empty, 0, r["lse"][:nl]))
        assert np.all(d <= ltol), f"sequence {s}: lse off by {np.max(d / ltol):.2f} of the bound"
        if left is not None:
            assert torch.equal(got_out[s, nl:], left[0][s, nl:]) and torch.equal(got_lse[s, nl:], left[1][s, nl:])
    return worst


def tables(rng, lengths, page, cols, spare=2):
    """Block tables with pages in no order; entries behind a sequence's pages hold other pages' numbers."""
    held = [-(-x // page) for x in lengths]
    pages = sum(held) + spare
    order = rng.permutation(pages)
    t = rng.integers(0, pages, (len(lengths), cols))
    at = 0
    for s, h in enumerate(held):
        t[s, :h] = order[at:at + h]
        at += h
    return t.astype(np.int32), pages, order[at:].astype(np.int32)
