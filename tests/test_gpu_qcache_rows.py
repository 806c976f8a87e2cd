"""Moving cached rows: copies between pools and over each other, rows into 4 bits and back, against numpy from the format's definition.  Copies and
codes are compared bit for bit; rows that no range names stay as they were."""
import numpy as np
import pytest
import torch

from tests import qref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ab():
    from paper_2504_12397_amd import binding
    return binding


@pytest.fixture(scope="module")
def ctx(ab):
    c = ab.Context(0)
    yield c
    c.close()


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def full_caches(ab, layers, rows, heads, h, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [ab.KVCache.from_tensors(*(torch.randn((rows, heads, h), generator=g).to(DT[dtype]).cuda() for _ in "kv")) for _ in range(layers)]


def four_caches(ab, layers, rows, heads, h, seed):
    g = torch.Generator().manual_seed(seed)
    nb = (h + 31) // 32
    def codes():
        return torch.randint(0, 256, (rows, heads, h // 2), generator=g, dtype=torch.uint8).cuda()
    def exps():
        return torch.randint(110, 140, (rows, heads, nb), generator=g, dtype=torch.uint8).cuda()
    return [ab.QCache.from_tensors(codes(), codes(), exps(), exps()) for _ in range(layers)]


def arrays(c):
    return [c.k, c.v] + ([c.k_scale, c.v_scale] if hasattr(c, "k_scale") else [])


def moved(dst, src, ranges):
    """What the copy leaves in dst: every source row read first."""
    want = dst.clone()
    for a, b, n in ranges:
        want[b:b + n] = src[a:a + n]
    return want


# ranges of every kind; the pool has 700 rows
DISJOINT = [(0, 400, 1), (3, 500, 100), (650, 650, 0), (200, 401, 37)]
FORKS = [(10, 300, 50), (10, 350, 50), (12, 400, 3)]
MANY = [(2 * i, 350 + 3 * i, 1 + i % 2) for i in range(80)]
DOWN = [(5, 0, 100), (110, 100, 200), (330, 300, 1), (340, 301, 250)]                # over each other, towards the front
UP = [(0, 7, 100), (100, 130, 200), (301, 349, 350)]                                  # towards the back
CLOSE = [(4 + 23 * i, 2 + 20 * i, 20) for i in range(30)]                             # a pool that is closed up: a little more at every sequence
SHUFFLED = [(400, 0, 120), (150, 120, 60), (600, 180, 90), (300, 270, 25), (299, 296, 3)]
SWAP = [(0, 300, 200), (300, 0, 200), (250, 250, 20)]
ROTATE = [(0, 100, 100), (100, 200, 100), (200, 0, 100), (500, 501, 150)]
ONE_OVER_ITSELF = [(100, 101, 599)]
BACK_BY_ONE = [(1, 0, 699)]


@pytest.mark.parametrize("same", [False, True], ids=["other_pool", "in_place"])
@pytest.mark.parametrize("ranges", [DISJOINT, FORKS, MANY, DOWN, UP, CLOSE, SHUFFLED, SWAP, ROTATE, ONE_OVER_ITSELF, BACK_BY_ONE, []],
                         ids=["disjoint", "forks", "many", "down", "up", "close", "shuffled", "swap", "rotate", "over_itself", "back_by_one", "none"])
@pytest.mark.parametrize("kind,layers,heads,h", [("bf16", 3, 8, 128), ("f32", 1, 5, 80), ("bf16", 40, 1, 2), ("bf16", 2, 3, 6),
                                                 ("four", 3, 8, 128), ("four", 17, 3, 34), ("four", 1, 1, 2)])
def test_copy(ab, ctx, kind, layers, heads, h, ranges, same):
    make = (lambda seed: four_caches(ab, layers, 700, heads, h, seed)) if kind == "four" else (lambda seed: full_caches(ab, layers, 700, heads, h, kind, seed))
    src = make(1)
    dst = src if same else make(2)
    want = [[moved(bits(d), bits(s), ranges) for d, s in zip(arrays(x), arrays(y))] for x, y in zip(dst, src)]
    kept = [[bits(s).clone() for s in arrays(y)] for y in src]
    (ab.alora_qcache_copy if kind == "four" else ab.alora_cache_copy)(ctx, dst, src, ranges)
    torch.cuda.synchronize()
    for l in range(layers):
        for got, w in zip(arrays(dst[l]), want[l]):
            assert torch.equal(bits(got), w), f"layer {l}"
        if not same:
            for got, w in zip(arrays(src[l]), kept[l]):
                assert torch.equal(bits(got), w), f"source of layer {l} changed"


def test_long_moves_over_each_other_again_and_again(ab, ctx):
    """Thousands of pieces in both directions, one call after the other on the same flags."""
    rows = 60000
    c = full_caches(ab, 2, rows, 8, 128, "bf16", 31)
    want = [[bits(t).clone() for t in (x.k, x.v)] for x in c]
    for ranges in ([(3, 0, 59997)], [(0, 1, 30000), (30002, 30050, 29000)], [(7 + 607 * i, 600 * i, 600) for i in range(90)],
                   [(0, 700, 59000)], [(1, 0, 59999)]):
        ab.alora_cache_copy(ctx, c, c, ranges)
        want = [[moved(t, t, ranges) for t in x] for x in want]
        for x, w in zip(c, want):
            assert torch.equal(bits(x.k), w[0]) and torch.equal(bits(x.v), w[1])


def awkward(rows, heads, h, dtype, seed):
    """Normals of every scale, exact ties and values next to them, zeros of both signs, blocks of zeros, and the largest and smallest numbers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, heads, h), generator=g) * torch.exp2(torch.randint(-30, 30, (rows, heads, 1), generator=g).float())
    ties = torch.tensor([6.0, 0.25, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 0.2499, 0.2501, 5.01, 4.99, -0.0, 0.0, 7.0])
    x[0, :, :] = ties.repeat((h + 15) // 16)[:h]
    x[1, :, :] = 1.75 * torch.randint(-1, 2, (heads, h), generator=g)            # the rule's border, at the border ...
    x[2, :, :] = x[1] * (1 + 2.0 ** -7)                                          # ... and over it
    x[3, :, :] = 0.0
    x[4, :, :] = -0.0
    x[5, :, :] = 3.0e38 * torch.sign(torch.randn((heads, h), generator=g))
    x[6, :, :] = 1.2e-38 * torch.randint(1, 9, (heads, h), generator=g).float()
    x[7, :, :] = 1.0e-36 * torch.randn((heads, h), generator=g)
    x[8, :, 0::2] = 0.0
    x[9, :, :] *= torch.exp2(torch.randint(-12, 1, (heads, h), generator=g).float())
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype,heads,h", [("bf16", 8, 128), ("f32", 4, 64), ("f32", 5, 80), ("bf16", 1, 2), ("bf16", 3, 34), ("f32", 2, 256),
                                           ("bf16", 2, 96), ("bf16", 7, 30)])
def test_store_and_load(ab, ctx, dtype, heads, h):
    rows, layers = 300, 2
    ranges = [(0, 100, 150), (150, 7, 1), (151, 250, 49), (260, 20, 33)]
    src = [ab.KVCache.from_tensors(awkward(rows, heads, h, dtype, 10 + l).cuda(), awkward(rows, heads, h, dtype, 20 + l).cuda()) for l in range(layers)]
    four = four_caches(ab, layers, 400, heads, h, 3)
    before = [[a.clone() for a in arrays(c)] for c in four]
    ab.alora_qcache_store(ctx, four, src, ranges)
    dst = full_caches(ab, layers, 350, heads, h, dtype, 4)
    had = [[a.clone() for a in arrays(c)] for c in dst]
    back = [(100, 5, 150), (7, 4, 1), (250, 200, 49), (20, 300, 33)]
    ab.alora_qcache_load(ctx, dst, four, back)
    torch.cuda.synchronize()
    for l in range(layers):
        for x, y, z, w, name in ((src[l].k, four[l].k, four[l].k_scale, dst[l].k, "k"), (src[l].v, four[l].v, four[l].v_scale, dst[l].v, "v")):
            codes, exps = qref.quantise(x.cpu().double().numpy())
            i = 0 if name == "k" else 1
            want_c, want_e, want_x = before[l][i].cpu().clone(), before[l][2 + i].cpu().clone(), had[l][i].cpu().clone()
            for (a, b, n), (_, t, _) in zip(ranges, back):
                want_c[b:b + n], want_e[b:b + n] = torch.from_numpy(codes[a:a + n]), torch.from_numpy(exps[a:a + n])
                want_x[t:t + n] = torch.from_numpy(qref.values(codes[a:a + n], exps[a:a + n])).to(DT[dtype])
            assert torch.equal(z.cpu(), want_e), name
            assert torch.equal(y.cpu(), want_c), name
            assert torch.equal(bits(w.cpu()), bits(want_x)), name


def test_not_a_number_takes_its_block_and_no_other(ab, ctx):
    x = torch.randn((4, 2, 80), generator=torch.Generator().manual_seed(5)).cuda()
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 79] = float("nan"), float("inf"), -float("inf")
    four = ab.QCache([4], 2, 80, "cuda")
    out = ab.KVCache([4], 2, 80, torch.float32, "cuda")
    ab.alora_qcache_store(ctx, four, ab.KVCache.from_tensors(x, x.clone()), [(0, 0, 4)])
    ab.alora_qcache_load(ctx, out, four, [(0, 0, 4)])
    nan = torch.isnan(out.k).cpu()
    want = torch.zeros_like(nan)
    want[0, 0, :32] = want[1, 1, 32:64] = want[2, 0, 64:] = True
    assert torch.equal(nan, want) and torch.equal(torch.isnan(out.v).cpu(), want)


def test_rows_far_into_a_pool(ab, ctx):
    """Byte offsets over 2^32 in every array."""
    rows, heads, h = 1_100_000, 16, 256                     # 9 GB of bf16 an array, 2.25 GB of codes
    k = torch.zeros((rows, heads, h), dtype=torch.bfloat16, device="cuda")
    x = torch.randn((50, heads, h), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    k[:50] = x
    full = ab.KVCache.from_tensors(k, k.clone())
    ab.alora_cache_copy(ctx, full, full, [(0, rows - 50, 50)])
    four = ab.QCache([2_200_000], heads, h, "cuda")         # 4.5 GB of codes an array
    ab.alora_qcache_store(ctx, four, full, [(rows - 50, 2_200_000 - 50, 50)])
    ab.alora_qcache_copy(ctx, four, four, [(2_200_000 - 50, 2_100_000, 50)])
    back = ab.KVCache([50], heads, h, torch.bfloat16, "cuda")
    ab.alora_qcache_load(ctx, back, four, [(2_100_000, 0, 50)])
    torch.cuda.synchronize()
    assert torch.equal(full.k[-50:], x) and torch.equal(full.v[-50:], x)
    want = torch.from_numpy(qref.values(*qref.quantise(x.cpu().double().numpy()))).to(torch.bfloat16)
    assert torch.equal(back.k.cpu(), want) and torch.equal(back.v.cpu(), want)
    assert not four.k[:2_100_000 - 1].any()


def test_another_stream_and_a_captured_call(ab, ctx):
    src, four = full_caches(ab, 2, 64, 8, 128, "bf16", 7), four_caches(ab, 2, 64, 8, 128, 8)
    dst = full_caches(ab, 2, 64, 8, 128, "bf16", 9)
    ranges = [(3, 10, 20)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ab.alora_qcache_store(ctx, four, src, ranges, stream=side)
    ab.alora_qcache_load(ctx, dst, four, [(10, 0, 20)], stream=side)
    side.synchronize()
    def want():
        return torch.from_numpy(qref.values(*qref.quantise(src[1].k[3:23].cpu().double().numpy()))).to(torch.bfloat16)
    assert torch.equal(dst[1].k[:20].cpu(), want())
    many = full_caches(ab, 1, 800, 2, 8, "bf16", 10)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ab.alora_cache_copy(ctx, src, src, [(40, 3, 20)])
        ab.alora_qcache_store(ctx, four, src, ranges)
        ab.alora_qcache_load(ctx, dst, four, [(10, 0, 20)])
        for c, over in ((src, [(0, 1, 20)]), (many, [(i, 400 + 2 * i, 1) for i in range(160)])):       # staged: refused, and the capture goes on
            with pytest.raises(ab.AloraError) as e:
                ab.alora_cache_copy(ctx, c, c, over)
            assert e.value.status == ab.ALORA_EINVAL
    for n in range(3):
        src[1].k[40:60] = torch.randn((20, 8, 128), generator=torch.Generator().manual_seed(n)).to(torch.bfloat16).cuda()
        dst[1].k.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(src[1].k[3:23], src[1].k[40:60])
        assert torch.equal(dst[1].k[:20].cpu(), want())
