"""Pins for the oracle of the verification step beside the tree: the 8-bit
format against torch's own conversion, sampling against the definition by
brute force, slots against the accepted path they come from, attention over a
cache against attention over plain arrays."""
import math

import numpy as np
import pytest
import torch

import oracle


def test_e4m3_is_torchs():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.E4M3_VALUES, every, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.6, 20000), oracle.E4M3_VALUES[:127],
                        (oracle.E4M3_VALUES[:126] + oracle.E4M3_VALUES[1:127]) / 2])   # ties too
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(oracle.e4m3_encode(x), torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert oracle.e4m3_encode([1e9, -np.inf]).tolist() == [126, 254]


@pytest.mark.parametrize("seed", range(30))
def test_sampling_by_brute_force(seed):
    rng = np.random.default_rng(seed)
    V = int(rng.integers(1, 9))
    z = rng.integers(-3, 4, V).astype(float)
    z[rng.random(V) < 0.2] = -np.inf
    t, k, p, m = float(rng.choice([0.5, 1, 2])), int(rng.integers(0, V + 2)), float(rng.choice([0.3, 0.8, 1])), float(rng.choice([0, 0.2]))
    if np.all(np.isneginf(z)):
        assert oracle.sample_row(z, 0.5)[0] == -1
        return
    ranked = sorted((i for i in range(V) if z[i] > -np.inf), key=lambda i: (-z[i], i))
    w = {i: math.exp((z[i] - max(z)) / t) for i in ranked}
    kept = ranked[:k] if 0 < k < V else list(ranked)
    if p < 1:
        total, run, cut = sum(w[i] for i in kept), 0.0, 0
        while run < p * total:
            run += w[kept[cut]]
            cut += 1
        kept = kept[:cut]
    kept = [i for i in kept if w[i] >= m] or kept[:1]
    mass = sum(w[i] for i in kept)
    seen = set()
    for u in np.linspace(0, 0.9999, 400):
        tok, lp, ids = oracle.sample_row(z, u, t, k, p, m)
        assert sorted(kept) == ids.tolist() and tok in kept
        assert lp == pytest.approx(math.log(w[tok] / mass), abs=1e-12)
        assert sum(w[i] for i in kept if i < tok) <= u * mass + 1e-9 and u * mass < sum(w[i] for i in kept if i <= tok) + 1e-9
        seen.add(tok)
    assert seen >= {i for i in kept if w[i] / mass > 0.01}


def test_slots_follow_the_accepted_path():
    table = np.array([[7, 3, -1], [9, -1, -1]], dtype=np.int32)
    acc = np.array([[2, 5, -1], [-1, -1, -1]])
    r = oracle.cache_slots([31, 16], [2, 0], acc, [4, 5, 6], 3, table, 8, 16, 10)
    assert r["status"] == 0 and r["free_count"] == 1
    assert r["slot"].tolist() == [3 * 16 + 15, 6 * 16, 6 * 16 + 1, 5 * 16] + [-1] * 6
    assert r["source"].tolist() == [0, 3, 6, 8] + [-1] * 6 and r["position"].tolist()[:4] == [31, 32, 33, 16]
    assert r["block_table"].tolist() == [[7, 3, 6], [9, 5, -1]] and r["context_len"].tolist() == [34, 17]
    assert oracle.cache_slots([31, 16], [2, 0], acc, [4, 5, 6], 1, table, 8, 16, 10)["status"] == 4
    assert oracle.cache_slots([47, 16], [2, 0], acc, [4, 5, 6], 3, table, 8, 16, 10)["status"] == 3
    assert oracle.cache_slots([31, 16], [2, 0], acc, [4, 5, 6], 3, table, 8, 16, 3)["status"] == 2
    assert oracle.cache_slots([31, 16], [4, 0], acc, [4, 5, 6], 3, table, 8, 16, 10)["status"] == 1


def test_appended_values_are_near_and_scales_never_fall():
    rng = np.random.default_rng(1)
    H, page, D = 2, 16, 8
    state = (np.zeros((3, H, page, D), np.uint8), np.zeros((3, H, D, page), np.uint8), np.zeros((3, H)), np.zeros((3, H)))
    kept_k = np.zeros((16, H, D))
    for at, size in ((0, 3), (3, 1), (4, 7), (11, 5)):
        k = rng.standard_normal((size, H, D)) * 4.0 ** at
        old = state[2][2].copy()
        state = oracle.cache_append(k, k, 2 * page + at + np.arange(size), None, *state)
        kept_k[at:at + size] = k
        assert np.all(state[2][2] >= old) and np.array_equal(state[2], state[3])
        for h in range(H):
            s, amax = state[2][2, h], np.abs(kept_k[:at + size, h]).max()
            assert amax <= 448 * s and amax > 224 * s
            got = oracle.e4m3_decode(state[0][2, h, :at + size]) * s
            # half a step, once for each time the value was rounded (at most four), and the smallest step
            assert np.all(np.abs(got - kept_k[:at + size, h]) <= 4 * (2.0 ** -4 * np.abs(kept_k[:at + size, h]) + 2.0 ** -10 * s))
            assert np.array_equal(state[0][2, h, :at + size], state[1][2, h, :, :at + size].T)
    assert not state[0][:2].any()


def test_attention_over_a_cache_is_attention_over_its_values():
    rng = np.random.default_rng(2)
    H, page, D, n, T = 2, 16, 8, 5, 37
    kc, vc = oracle.e4m3_encode(rng.standard_normal((4, H, page, D))), oracle.e4m3_encode(rng.standard_normal((4, H, D, page)))
    ks, vs = 2.0 ** rng.integers(-2, 2, (4, H)), 2.0 ** rng.integers(-2, 2, (4, H))
    q, kn, vn = rng.standard_normal((n, 4, D)), rng.standard_normal((n, H, D)), rng.standard_normal((n, H, D))
    table = np.array([2, 0, 3])
    got = oracle.tree_attention(q, kn, vn, None, T, table, kc, vc, ks, vs, 0.3)
    for h in range(4):
        k = np.array([oracle.e4m3_decode(kc[table[t // page], h // 2, t % page]) * ks[table[t // page], h // 2] for t in range(T)])
        v = np.array([oracle.e4m3_decode(vc[table[t // page], h // 2, :, t % page]) * vs[table[t // page], h // 2] for t in range(T)])
        k, v = np.concatenate([k, kn[:, h // 2]]), np.concatenate([v, vn[:, h // 2]])
        z = 0.3 * q[:, h] @ k.T
        z[:, T:] = np.where(np.tril(np.ones((n, n))) > 0, z[:, T:], -np.inf)
        p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
        assert np.allclose(got["out"][:, h], p @ v) and np.allclose(got["lse"][:, h], np.log(np.exp(z).sum(1)))
    none = oracle.tree_attention(q, kn, vn, np.zeros((n, n)), 0, table, kc, vc, ks, vs, 0.3)
    assert not none["out"].any() and np.all(np.isneginf(none["lse"]))
