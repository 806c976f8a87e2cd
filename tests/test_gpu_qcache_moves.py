"""Rows that move over each other in very many ranges and pieces: bit for bit as if every row had been read first, and no slower on the host than
copies of as many ranges that do not."""
import time

import numpy as np
import pytest
import torch

from tests.test_gpu_qcache_rows import arrays, bits, four_caches, full_caches

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ab():
    from paper_2504_12397_amd import binding
    return binding


@pytest.fixture(scope="module")
def ctx(ab):
    c = ab.Context(0)
    yield c
    c.close()


N = 40_000
I = np.arange(N)
ONE = np.ones(N, dtype=np.int64)
MOVES = {
    "front": np.stack([2 * I + 1, I, ONE], 1),
    "back": np.stack([I, 2 * I + 1, ONE], 1),
    "front_from_anywhere": np.stack([N + np.random.default_rng(1).permutation(N), 5 + I, ONE], 1),
    "uneven": np.stack([np.cumsum(1 + I % 3)[:N // 2] + 1, np.cumsum(np.r_[0, 1 + (I % 3)[:N // 2 - 1]]), (1 + I % 3)[:N // 2]], 1),
    "same_sources": np.stack([1 + I // 2 + N // 2, I % N, ONE], 1),
    "one_source": np.stack([np.full(N, 3), np.r_[3:3 + N], ONE], 1),
    "one_long_range": np.array([[5, 0, 2 * N - 5]]),
    "long_ranges_back": np.array([[0, 11, N], [N, N + 300, N - 300]]),
}


def moved(t, ranges):
    """What the move leaves: every source row read first."""
    src = torch.from_numpy(np.concatenate([np.arange(a, a + n) for a, _, n in ranges])).to(t.device)
    dst = torch.from_numpy(np.concatenate([np.arange(b, b + n) for _, b, n in ranges])).to(t.device)
    want = t.clone()
    want[dst] = t[src]
    return want


@pytest.mark.parametrize("kind,heads,h", [("bf16", 1, 2), ("f32", 3, 10), ("four", 2, 64), ("bf16", 4, 128)])
@pytest.mark.parametrize("name", list(MOVES))
def test_very_many_pieces(ab, ctx, name, kind, heads, h):
    ranges, rows = MOVES[name], 2 * N + 10
    c = four_caches(ab, 1, rows, heads, h, 3) if kind == "four" else full_caches(ab, 1, rows, heads, h, kind, 3)
    want = [moved(bits(t), ranges) for t in arrays(c[0])]
    for _ in range(2):
        (ab.alora_qcache_copy if kind == "four" else ab.alora_cache_copy)(ctx, c, c, ranges)
        torch.cuda.synchronize()
        for t, w in zip(arrays(c[0]), want):
            assert torch.equal(bits(t), w)
        want = [moved(w, ranges) for w in want]


@pytest.mark.parametrize("name", ["front", "back", "uneven", "same_sources"])
def test_time_on_the_host(ab, ctx, name):
    """The call's own time, at most ten times that of one with as many ranges between two pools."""
    def host(dst, src):
        best = 1e9
        for _ in range(4):
            torch.cuda.synchronize()
            t = time.perf_counter()
            ab.alora_cache_copy(ctx, dst, src, MOVES[name])
            best = min(best, time.perf_counter() - t)
        torch.cuda.synchronize()
        return best
    a, b = (full_caches(ab, 1, 2 * N + 10, 1, 2, "bf16", seed) for seed in (4, 5))
    apart, over = host(b, a), host(a, a)
    assert over <= 10 * apart, f"{1e3 * over:.2f} ms, between two pools {1e3 * apart:.2f}"


def test_arrays_that_are_staged_in_groups_of_other_sizes(ab):
    """Rows that change places, in arrays that go through a new context's workspace in groups, the second larger than the first."""
    n = 100_000
    ranges = [(0, n, n), (n, 0, n)]
    ctx = ab.Context(0)
    try:
        c = four_caches(ab, 1, 2 * n, 8, 128, 6)
        was = [t.clone() for t in arrays(c[0])]
        ab.alora_qcache_copy(ctx, c, c, ranges)
        torch.cuda.synchronize()
        for t, w in zip(arrays(c[0]), was):
            assert torch.equal(t[:n], w[n:]) and torch.equal(t[n:], w[:n])
    finally:
        ctx.close()
