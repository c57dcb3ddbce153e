"""Sampling at the ends of what its settings and steps allow, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from paper_2606_03819_amd import binding
from test_gpu_verify_step import check_sample, likely

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


def written(b, n):
    """Outputs that no sample leaves as they are."""
    return dict(token=torch.full((b, n), -7, dtype=torch.int32, device="cuda"),
                logprob=torch.full((b, n), 7.0, device="cuda"))


def crowned(kind, V):
    """Rows whose largest logits are tied, lie within a sixteenth of one another, or are all there is."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal(V).clip(-3, 3)
    if kind == "tied":
        z[[5, 9]] = 8.0
    elif kind == "tied far apart":
        z[[V - 2, 7, V // 2]] = 8.0
    elif kind == "near":
        z[[11, 3, 200, 17]] = 8.0, 7.96875, 8.0, 7.9375
    else:
        z[:] = 0.5
    return z


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("k", [0, 100, 3])
def test_no_mass_keeps_the_first_token(k, dt):
    for V in (900, 3000, 40000):
        kinds = ["tied", "tied far apart", "near", "flat"]
        z = np.stack([np.stack([crowned(kind, V)] * 2) for kind in kinds])
        zt = torch.tensor(z).to(dt).cuda()
        u = torch.tensor([[0.0, 0.97]] * len(kinds), dtype=torch.float32).cuda()
        for p in (0.0, -0.0, -1.0, -float("inf"), 1e-30, 1e-7):
            print(f"V {V} k {k} p {p} {dt}", flush=True)
            tok, lp = check_sample(zt, u, k=[k] * len(kinds), p=[p] * len(kinds), **written(len(kinds), 2))
            assert tok.tolist() == [[5, 5], [7, 7], [11, 11], [0, 0]] and lp.abs().max() < 2.0 ** -30
            check_sample(zt, u, t=[0.8, 1.0, 3.0, 0.1], k=[k] * len(kinds), p=[p] * len(kinds), m=[0.5] * len(kinds))


@pytest.mark.parametrize("dt", DTYPES)
def test_min_p_of_one_keeps_the_largest_alone(dt):
    """Largest logits at the ends of their steps of a sixteenth of T: whichever step rounding gives them, they are kept."""
    V = 5000
    temps = [1.5, 3.0, 6.0, 0.75, 0.3, 0.7, 0.1, 5.0]
    rows = np.zeros((len(temps), 24, V))
    for s, t in enumerate(temps):
        for i in range(24):
            rng = np.random.default_rng(100 * s + i)
            top = float(torch.tensor((i - 8 + 0.5) * float(np.float32(t)) / 16).to(dt))
            step = abs(top) * float(torch.finfo(dt).eps)
            rows[s, i] = top - step - rng.random(V) * t
            rows[s, i, rng.integers(0, V, 3)] = top
            rows[s, i, 40] = top - step   # and the nearest below it
    z = torch.tensor(rows).to(dt).cuda()
    u = torch.tensor(np.random.default_rng(1).random((len(temps), 24)), dtype=torch.float32).cuda()
    for kw in (dict(), dict(p=[0.9] * 8), dict(k=[300] * 8), dict(k=[300] * 8, p=[0.01] * 8)):
        print(dt, kw, flush=True)
        check_sample(z, u, temps, m=[1.0] * 8, **kw, **written(8, 24))
        check_sample(z, u, temps, m=[1.0 - 2.0 ** -24] * 8, **kw, **written(8, 24))


def test_rows_whose_slices_straddle_the_largest_distance():
    """16 z / T just above -2^20 in one slice and just below it in the others, a few units of T apart."""
    rng = np.random.default_rng(5)
    V, t = 40000, float(np.float32(1e-3))
    limit = -t * 2.0 ** 16
    z = np.full((6, 4, V), limit) - 2e-3 - rng.random((6, 4, V)) * 4e-3
    for i, above in enumerate((1e-5, 1e-4, 1e-3, 2.9e-2)):
        z[:, i, rng.integers(0, V, 3)] = limit + above
    z[5] = -z[5]                        # the other end: none of these rows is within it
    zt = torch.tensor(z, dtype=torch.float32).cuda()
    u = torch.tensor(rng.random((6, 4)), dtype=torch.float32).cuda()
    check_sample(zt, u, [t] * 6, [0, 0, 0, 500, 20000, 0], [1.0, 0.9, 1.0, 1.0, 0.7, 1.0], [0.0, 0.0, 0.01, 0.0, 0.0, 0.0])


@pytest.mark.parametrize("V,k", [(50257, 50), (64000, 50), (92544, 50), (100352, 64), (128256, 64), (30000, 64), (125000, 62)])
def test_top_k_of_more_tokens_than_the_row_has_lists(V, k):
    """As many lists of 2048 logits as k or fewer: their largest alone give no bound, so thousands of entries are joined."""
    rng = np.random.default_rng(V)
    sets = [dict(k=k), dict(k=k, p=0.95, t=0.6), dict(k=k, m=0.02), dict(k=k - 1, t=2.0)]
    get = lambda f, d: [s.get(f, d) for s in sets]  # noqa: E731
    for dt in DTYPES:
        for steps in (None, 4):
            z = likely(rng, len(sets), 2, V, dt, steps)
            u = torch.tensor(rng.random((len(sets), 2)), dtype=torch.float32).cuda()
            check_sample(z, u, get("t", 1.0), get("k", 0), get("p", 1.0), get("m", 0.0))


def test_top_k_takes_as_long_over_a_smaller_vocabulary():
    """Rows of 50 thousand logits take no longer than rows of 152 thousand do, whose lists are more than k (a third
    is allowed for: reading byte by byte takes many times as long)."""
    def microseconds(V):
        z = likely(np.random.default_rng(1), 4, 1, V, torch.bfloat16)
        u, k = torch.full((4, 1), 0.5, device="cuda"), torch.full((4,), 50, dtype=torch.int32, device="cuda")
        ws = binding.alloc_workspace(binding.treeflash_sample_workspace_bytes(4, 1, V), z.device)
        out = written(4, 1)
        call = lambda: binding.treeflash_sample(z, u, top_k=k, workspace=ws, **out)  # noqa: E731
        call()
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            for _ in range(20):
                call()
        best = 1e9
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            graph.replay()
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 50)
        return best

    long = microseconds(151936)
    for V in (50257, 64000, 100352):
        short = microseconds(V)
        print(f"top-k 50 of {V}: {short:.1f} us, of 151936: {long:.1f}", flush=True)
        assert short < long * 4 / 3
