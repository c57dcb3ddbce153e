"""The verification step beside the tree, in 64 bits: sampling, cache pages and
slots, the 8-bit cache, attention over it.  Written from the definitions, one
row, token or page at a time; shares no code with the library.
"""
from __future__ import annotations

import math
from typing import Dict, Optional, Tuple

import numpy as np

__all__ = ["E4M3_VALUES", "e4m3_decode", "e4m3_encode", "sample_row", "cache_slots", "cache_append",
           "tree_attention"]


def _e4m3_table() -> np.ndarray:
    """Value of each of the 256 codes: 4 exponent bits of bias 7, 3 mantissa bits, no infinities, 0x7f NaN."""
    out = np.zeros(256)
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            out[c] = np.nan
        elif e == 0:
            out[c] = sign * m * 2.0 ** -9
        else:
            out[c] = sign * (1 + m / 8) * 2.0 ** (e - 7)
    return out


E4M3_VALUES = _e4m3_table()
_POSITIVE = E4M3_VALUES[:127]   # ascending


def e4m3_decode(codes) -> np.ndarray:
    return E4M3_VALUES[np.asarray(codes, dtype=np.uint8)]


def e4m3_encode(x) -> np.ndarray:
    """Nearest code, ties to the even one; what is larger than 448 is held to it, NaN stays NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, np.where(np.isnan(a), 0.0, a), side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def sample_row(z, u: float, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
               min_p: float = 0.0) -> Tuple[int, float, np.ndarray]:
    """(token, log-probability among the kept, kept ids in ascending order) of one row of logits."""
    z = np.asarray(z, dtype=np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    real = np.nonzero(z > -np.inf)[0]
    if len(real) == 0:
        return -1, -math.inf, real
    order = real[np.lexsort((real, -z[real]))]
    if not temperature > 0:
        return int(order[0]), 0.0, order[:1]
    top = z[order[0]]
    x = np.zeros(len(order))
    below = z[order] != top
    with np.errstate(invalid="ignore"):
        x[below] = (z[order][below] - top) / np.float64(temperature)
    w = np.exp(x)
    keep = len(order)
    if 0 < top_k < len(z):
        keep = min(keep, top_k)
    if top_p < 1:
        c = np.cumsum(w)
        keep = min(keep, int(np.sum(c[:keep] < np.float64(top_p) * c[keep - 1])) + 1)
    if min_p > 0:
        keep = min(keep, int(np.sum(w >= np.float64(min_p))))
    keep = max(keep, 1)
    ids = np.sort(order[:keep])
    rank = {int(t): r for r, t in enumerate(order[:keep])}
    wi = np.array([w[rank[int(t)]] for t in ids])
    c = np.cumsum(wi)
    u = min(u, 1 - 2.0 ** -24) if u > 0 else 0.0
    at = int(np.searchsorted(c, u * c[-1], side="right"))
    return int(ids[at]), float(x[rank[int(ids[at])]] - math.log(c[-1])), ids


def cache_slots(context_len, add_len, accepted, free_pages, free_count: int, block_table, n: int, page: int,
                max_tokens: int) -> Dict[str, object]:
    """Pages popped from the end of the stack, sequence by sequence, token by token."""
    b, cols = block_table.shape
    table, stack = block_table.copy(), list(free_pages[:max(0, min(free_count, len(free_pages)))])
    add = [int(a) + (1 if accepted is not None else 0) for a in add_len]
    none = dict(context_len=np.array(context_len), free_count=free_count, start=np.zeros(b + 1, int),
                page_start=np.zeros(b + 1, int), block_table=block_table.copy(), slot=np.full(max_tokens, -1),
                position=np.full(max_tokens, -1), source=np.full(max_tokens, -1))
    gamma = accepted.shape[1] if accepted is not None else 0
    if (free_count < 0 or free_count > len(free_pages) or min(context_len) < 0 or min(add) < 0
            or (accepted is not None and max(add_len) > gamma) or (n > 0 and max(add) > n)):
        return dict(none, status=1)
    if sum(add) > max_tokens:
        return dict(none, status=2)
    if any(c + a > cols * page for c, a in zip(context_len, add)):
        return dict(none, status=3)
    out = dict(none, start=[0], page_start=[0], slot=[], position=[], source=[])
    for s in range(b):
        taken = 0
        for j in range(add[s]):
            pos = int(context_len[s]) + j
            if pos % page == 0:
                if not stack:
                    return dict(none, status=4)
                table[s, pos // page] = stack.pop()
                taken += 1
            out["slot"].append(int(table[s, pos // page]) * page + pos % page)
            out["position"].append(pos)
            node = 0 if j == 0 or accepted is None else 1 + int(accepted[s, j - 1])
            out["source"].append(len(out["source"]) if n == 0 else s * n + (j if accepted is None else node))
        out["start"].append(len(out["slot"]))
        out["page_start"].append(out["page_start"][-1] + taken)
    for f in ("slot", "position", "source"):
        out[f] = np.array(out[f] + [-1] * (max_tokens - len(out[f])))
    return dict(out, context_len=np.array(context_len) + np.array(add), free_count=len(stack),
                start=np.array(out["start"]), page_start=np.array(out["page_start"]), block_table=table, status=0)


def _pow2(amax: float) -> float:
    """Smallest power of two s with amax <= 448 s, within 2^-64..2^64."""
    s = 2.0 ** -64
    while s < 2.0 ** 64 and amax > 448 * s:
        s *= 2
    return s


def cache_append(k_new, v_new, slot, source, k_codes, v_codes, k_scale, v_scale) -> Tuple[np.ndarray, ...]:
    """New copies of codes k [pages, H, page, D], v [pages, H, D, page] and scales after an append of rows
    [R, H, D] (fp64) to the slots, run by run."""
    k_codes, v_codes, k_scale, v_scale = (np.array(x) for x in (k_codes, v_codes, k_scale, v_scale))
    pages, H, page, D = k_codes.shape
    slot = np.asarray(slot)
    i = 0
    while i < len(slot):
        sl = int(slot[i])
        if sl < 0 or sl >= pages * page:
            i += 1
            continue
        run = 1
        while i + run < len(slot) and slot[i + run] == sl + run and (sl + run) // page == sl // page:
            run += 1
        p, o = sl // page, sl % page
        rows = [int(source[i + j]) if source is not None else i + j for j in range(run)]
        for new, codes, scale, turn in ((k_new, k_codes, k_scale, False), (v_new, v_codes, v_scale, True)):
            x = np.stack([new[r] if 0 <= r < len(new) else np.zeros((H, D)) for r in rows])   # [run, H, D]
            for h in range(H):
                held = codes[p, h].T if turn else codes[p, h]      # a view [page, D]
                a = np.abs(x[:, h])
                s = _pow2(float(np.max(np.where(np.isfinite(a), a, 0.0))))
                if o > 0:
                    s = max(s, float(scale[p, h]))
                    if s != scale[p, h]:
                        held[:o] = e4m3_encode(e4m3_decode(held[:o]) * (float(scale[p, h]) / s))
                held[o:o + run] = e4m3_encode(x[:, h] / s)
                scale[p, h] = s
        i += run
    return k_codes, v_codes, k_scale, v_scale


def tree_attention(q, k_new, v_new, mask, context_len: int, table, k_codes, v_codes, k_scale, v_scale, scale: float,
                   new_len: Optional[int] = None) -> Dict[str, np.ndarray]:
    """One sequence: q [n, Hq, D], k_new, v_new [n, H, D], mask [n, n] or None, table [max_pages].

    Besides out [n, Hq, D] and lse [n, Hq] it returns what error bounds need: `absv`, the weighted sum of |v|,
    and `size`, the largest sum of |q||k| * scale."""
    n, Hq, D = q.shape
    pages, H, page, _ = k_codes.shape
    nl = n if new_len is None else new_len
    T = min(max(context_len, 0), len(table) * page)
    toks = [t for t in range(T) if 0 <= table[t // page] < pages]
    pg = np.array([table[t // page] for t in toks], dtype=int)
    off = np.array([t % page for t in toks], dtype=int)
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    absv, size = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for h in range(H):
        kc = e4m3_decode(k_codes[pg, h, off]) * k_scale[pg, h][:, None] if toks else np.zeros((0, D))
        vc = e4m3_decode(v_codes[pg, h, :, off]) * v_scale[pg, h][:, None] if toks else np.zeros((0, D))
        for i in range(nl):
            sees = [j for j in range(nl) if (j <= i if mask is None else mask[i, j] != 0)]
            k = np.concatenate([kc, k_new[sees, h].reshape(-1, D)])
            v = np.concatenate([vc, v_new[sees, h].reshape(-1, D)])
            if len(k) == 0:
                continue
            for g in range(h * (Hq // H), (h + 1) * (Hq // H)):
                z = scale * (k @ q[i, g])
                w = np.exp(z - z.max())
                out[i, g] = w @ v / w.sum()
                absv[i, g] = w @ np.abs(v) / w.sum()
                size[i, g] = np.max(abs(scale) * (np.abs(k) @ np.abs(q[i, g])))
                lse[i, g] = z.max() + math.log(w.sum())
    return {"out": out, "lse": lse, "absv": absv, "size": size}
