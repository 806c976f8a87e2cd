"""Attention over rows of 4 bits against float64 numpy: head layouts, lengths from one token on, ragged batches, shared prefixes, masks, values that are not
numbers; the calls that run layers on such caches, against the calls on other caches and the oracle."""
import numpy as np
import pytest
import torch

from oracle import alora_oracle as orc
from paper_2504_12397_amd import workloads as wl
from tests import helpers as H
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


class Batch:
    """Sequences over contexts: sequence b has context group[b] (-1: none) of C[group[b]] rows and own[b] rows of its own, the last new[b] of which have queries."""

    def __init__(self, ab, dtype, n_q, n_kv, h, own, new, C=(), group=None, seed=1, q_scale=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.n_q, self.h, self.own, self.new, self.C = dtype, n_q, h, list(own), list(new), list(C)
        self.group = list(group) if group is not None else [-1] * len(own)
        regions = self.C + self.own
        off, at = [], 2
        for n in regions:
            off.append(at)
            at += n + 3
        self.off = off
        shape = (at, n_kv, h)
        x = [rng.standard_normal(shape) for _ in "kv"]
        self.codes = [qref.quantise(a) for a in x]
        # rows that belong to nobody hold what is not a number
        mine = np.zeros(at, dtype=bool)
        for o, n in zip(off, regions):
            mine[o:o + n] = True
        for _, e in self.codes:
            e[~mine] = 255
        nc = len(self.C)
        self.plen = [self.C[g] if g >= 0 else 0 for g in self.group]
        self.poff = [off[g] if g >= 0 else 0 for g in self.group]
        self.cu = [0] + list(np.cumsum(self.new))
        q = torch.from_numpy(rng.standard_normal((self.cu[-1], n_q * h)) * q_scale).to(DT[dtype])
        self.q = q.cuda()
        self.q64 = q.double().numpy()
        self.cache = self.make(ab)

    def make(self, ab):
        (kc, ke), (vc, ve) = self.codes
        nc = len(self.C)
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return ab.QCache.from_tensors(t(kc), t(vc), t(ke), t(ve), self.off[nc:], self.own, [p + o for p, o in zip(self.plen, self.own)],
                                      self.poff if self.C else None, self.plen if self.C else None)

    def rows(self, b):
        o = self.off[len(self.C) + b]
        return np.concatenate([np.arange(self.poff[b], self.poff[b] + self.plen[b]), np.arange(o, o + self.own[b])])

    def reference(self, b):
        at = self.rows(b)
        K, V = (qref.values(c[at], e[at]) for c, e in self.codes)
        n = len(at)
        vis = [n - self.new[b] + i + 1 for i in range(self.new[b])]
        return qref.attend(self.q64[self.cu[b]:self.cu[b + 1]], K, V, self.n_q, vis)

    def check(self, out, only=None):
        out = out.double().cpu().numpy()
        worst = 0.0
        for b in range(len(self.own)) if only is None else only:
            if self.new[b] == 0:
                continue
            ref, mag, total, spread = self.reference(b)
            tol = qref.tolerance(ref, mag, total, spread, self.h, len(self.rows(b)), self.dtype)
            err = np.abs(out[self.cu[b]:self.cu[b + 1]] - ref)
            assert np.isfinite(err).all(), f"sequence {b}: not finite"
            worst = max(worst, float((err / tol).max()))
        H.report(check="qcache_attend", worst_of_tolerance=worst)
        assert worst <= 1.0, f"{worst:.3f} of the tolerance"


SHAPES = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 4, 64), ("f32", 6, 2, 128), ("bf16", 10, 5, 80), ("f32", 3, 1, 34), ("bf16", 4, 2, 256),
          ("f32", 2, 2, 256), ("bf16", 40, 1, 96), ("bf16", 2, 2, 2), ("bf16", 18, 9, 128), ("f32", 16, 2, 8), ("bf16", 6, 3, 40)]


@pytest.mark.parametrize("dtype,n_q,n_kv,h", SHAPES)
@pytest.mark.parametrize("own,new", [([1], [1]), ([2, 31, 32, 33, 64, 65], [1, 1, 1, 1, 1, 1]), ([777], [1]), ([5, 40, 130], [5, 3, 17]), ([300, 9, 70], [0, 9, 70])],
                         ids=["one_key", "steps", "long_step", "suffixes", "whole_and_none"])
def test_shapes_and_lengths(ab, ctx, dtype, n_q, n_kv, h, own, new):
    b = Batch(ab, dtype, n_q, n_kv, h, own, new)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, n_q))


@pytest.mark.parametrize("dtype,n_q,n_kv,h", [("bf16", 8, 2, 128), ("f32", 4, 4, 64), ("bf16", 10, 5, 80), ("bf16", 32, 8, 128)])
@pytest.mark.parametrize("new", [[1] * 7, [3, 1, 20, 0, 2, 9, 1]], ids=["steps", "suffixes"])
def test_shared_contexts(ab, ctx, dtype, n_q, n_kv, h, new):
    b = Batch(ab, dtype, n_q, n_kv, h, [4, 1, 20, 6, 2, 90, 33], new, C=[257, 100], group=[0, 1, 0, 0, -1, 1, 0], seed=3)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, n_q))


def test_many_adapters_on_one_context_in_turn(ab, ctx):
    """Sequences of two contexts in turn, more of them than a workgroup takes together."""
    n = 45
    b = Batch(ab, "bf16", 8, 2, 128, [1 + i % 5 for i in range(n)], [1] * n, C=[530, 95], group=[i % 2 for i in range(n)], seed=4)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8))


@pytest.mark.parametrize("splits", [1, 3, 64])
@pytest.mark.parametrize("dtype,h", [("bf16", 128), ("f32", 64), ("bf16", 80)])
def test_number_of_parts_and_plain_kernels(ab, dtype, h, splits):
    for kernels in (0, 1):
        c = ab.Context(0)
        try:
            c.set_option("kv_splits", splits)
            c.set_option("kernels", kernels)
            b = Batch(ab, dtype, 8, 2, h, [500, 33, 129], [1, 2, 129], C=[200], group=[0, -1, 0], seed=5)
            b.check(ab.alora_qcache_attend(c, b.cache, b.q, b.cu, 8))
        finally:
            c.close()


@pytest.mark.parametrize("q_scale", [1e-6, 30.0])
def test_flat_and_peaked_scores(ab, ctx, q_scale):
    for dtype, h in (("bf16", 128), ("f32", 64)):
        b = Batch(ab, dtype, 8, 2, h, [400, 50], [1, 30], seed=6, q_scale=q_scale)
        b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8))


@pytest.mark.parametrize("e_k,e_v", [(2, 2), (20, 240), (230, 127), (100, 60), (127, 250)])
def test_exponents_of_every_size(ab, ctx, e_k, e_v):
    """Values far outside what fp16 holds: the exponents are moved, and the queries' inversely."""
    for dtype, h in (("bf16", 128), ("f32", 64), ("bf16", 80)):
        b = Batch(ab, dtype, 4, 2, h, [90, 40], [1, 7], seed=7)
        for (c, e), at in zip(b.codes, (e_k, e_v)):
            e[e != 255] = at
        s = 2.0 ** (125 - e_k) if 125 - e_k > -120 else 2.0 ** -120
        q = torch.from_numpy(np.random.default_rng(8).standard_normal(b.q64.shape) * min(s, 2.0 ** 100)).to(DT[dtype])
        b.q, b.q64 = q.cuda(), q.double().numpy()
        b.cache = b.make(ab)
        b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 4))


@pytest.mark.parametrize("e_v", [113, 114, 139, 140, 141, 90, 160])
@pytest.mark.parametrize("h", [64, 128])
def test_values_around_what_fp16_holds(ab, ctx, h, e_v):
    """Units of many columns multiply in fp16 where it holds the values: exponents on both sides of that, in all rows and in one block of one row, zeros between."""
    for everywhere in (True, False):
        b = Batch(ab, "bf16", 8, 2, h, [300, 45], [40, 45], C=[130], group=[0, -1], seed=17)
        c, e = b.codes[1]
        c[b.rows(0)[7:20]] = 0
        if everywhere:
            e[e != 255] = e_v
        else:
            e[b.rows(0)[211], 1, 1] = e_v
        b.cache = b.make(ab)
        b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8))


@pytest.mark.parametrize("dtype,n_q,n_kv,h", [("bf16", 8, 2, 128), ("f32", 4, 4, 64), ("bf16", 8, 2, 64), ("bf16", 4, 2, 256), ("bf16", 10, 5, 80)])
def test_not_a_number_reaches_the_rows_that_see_it(ab, ctx, dtype, n_q, n_kv, h):
    """A value block that is NaN at position j: the rows from j on have NaN in its channels of its heads, the others nothing."""
    b = Batch(ab, dtype, n_q, n_kv, h, [60, 70], [40, 1], seed=9)
    (kc, ke), (vc, ve) = b.codes
    clean = ab.alora_qcache_attend(ctx, b.make(ab), b.q, b.cu, n_q).clone()
    at = b.rows(0)
    ve[at[35], 0, 1] = 255                  # channels 32..63 of kv head 0, seen by rows 15..39 of sequence 0
    ke[at[50], 1, 0] = 255                  # all of kv head 1 for rows 30..39
    out = ab.alora_qcache_attend(ctx, b.make(ab), b.q, b.cu, n_q)
    G = n_q // n_kv
    want = torch.zeros((b.cu[-1], n_q, h), dtype=torch.bool)
    want[15:40, :G, 32:64] = True
    want[30:40, G:2 * G, :] = True
    got = torch.isnan(out).cpu().view(-1, n_q, h)
    assert torch.equal(got, want)
    rest = ~want
    o, c = out.cpu().double().view(-1, n_q, h), clean.cpu().double().view(-1, n_q, h)
    assert (o[rest] - c[rest]).abs().max() <= 2.0 ** -6 * c.abs().max()


def test_last_key_of_an_item_is_not_a_number(ab, ctx):
    """Loads past the end of a sequence repeat its last row: a NaN there must stay with the rows that see it."""
    b = Batch(ab, "bf16", 8, 2, 128, [37], [5], seed=10)
    (kc, ke), (vc, ve) = b.codes
    ve[b.rows(0)[36], :, :] = 255
    out = ab.alora_qcache_attend(ctx, b.make(ab), b.q, b.cu, 8)
    nan = torch.isnan(out).cpu()
    assert not nan[:4].any() and nan[4].all()


@pytest.mark.parametrize("h,n_q,n_kv", [(128, 32, 8), (64, 4, 4), (80, 10, 5)])
def test_long_sequences(ab, ctx, h, n_q, n_kv):
    b = Batch(ab, "bf16", n_q, n_kv, h, [9001, 1], [1, 1], seed=11)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, n_q))
    b = Batch(ab, "bf16", n_q, n_kv, h, [2050], [70], seed=12)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, n_q))


@pytest.mark.parametrize("dtype,h", [("bf16", 64), ("f32", 80)])
def test_more_sequences_than_compute_units(ab, ctx, dtype, h):
    """300 steps on the rows of three sequences: keys are cut in parts though there is a workgroup for every compute unit without."""
    b = Batch(ab, dtype, 8, 8, h, [2100, 1999, 2050], [1, 1, 1], seed=17)
    pick = [i % 3 for i in range(300)]
    lens = [b.own[p] for p in pick]
    cache = ab.QCache.from_tensors(b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale, [b.off[p] for p in pick], lens, lens)
    out = ab.alora_qcache_attend(ctx, cache, b.q[pick], list(range(301)), 8)
    assert torch.equal(out, out[:3][pick])
    b.check(out[:3])


def test_positions_far_into_a_pool(ab, ctx):
    """A sequence whose rows lie past byte 2^32 of the codes, read from there."""
    b = Batch(ab, "bf16", 16, 16, 256, [70], [3], seed=13)
    (kc, ke), (vc, ve) = b.codes
    at = b.rows(0)
    rows = 2_200_000
    four = ab.QCache([rows], 16, 256, "cuda")
    for dst, src in ((four.k, kc), (four.v, vc), (four.k_scale, ke), (four.v_scale, ve)):
        dst[rows - 70:] = torch.from_numpy(src[at]).cuda()
    cache = ab.QCache.from_tensors(four.k, four.v, four.k_scale, four.v_scale, [rows - 70], [70], [70])
    b.check(ab.alora_qcache_attend(ctx, cache, b.q, b.cu, 16))


def test_same_sequence_twice_and_rows_behind_stay(ab, ctx):
    b = Batch(ab, "bf16", 8, 2, 128, [100, 100], [2, 2], seed=14)
    b.cache.seq_offset[1] = b.cache.seq_offset[0]
    b.q[2:] = b.q[:2]
    out = torch.full((10, 1024), 3.0, dtype=torch.bfloat16, device="cuda")
    before = [t.clone() for t in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)]
    ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8, out=out[:4])
    torch.cuda.synchronize()
    assert torch.equal(out[:2], out[2:4]) and (out[4:] == 3.0).all()
    assert all(torch.equal(x, y) for x, y in zip(before, (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)))
    assert list(b.cache.seq_len) == [100, 100]


def test_two_contexts_at_once_and_repeated_calls_give_the_same_bits(ab):
    b = Batch(ab, "bf16", 8, 2, 128, [3000, 10, 700], [1, 1, 1], seed=15)
    c1, c2 = ab.Context(0), ab.Context(0)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    try:
        outs = []
        for _ in range(10):
            outs.append(ab.alora_qcache_attend(c1, b.cache, b.q, b.cu, 8, stream=s1))
            outs.append(ab.alora_qcache_attend(c2, b.cache, b.q, b.cu, 8, stream=s2))
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0], o) for o in outs)
    finally:
        c1.close()
        c2.close()


def test_capture_is_refused_and_goes_on(ab, ctx):
    b = Batch(ab, "bf16", 8, 2, 128, [30], [1], seed=16)
    x = torch.zeros(4, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x += 1
        with pytest.raises(ab.AloraError) as e:
            ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8, out=torch.empty_like(b.q))
        assert e.value.status == ab.ALORA_EINVAL
    x.zero_()
    for n in range(3):
        g.replay()
        b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, 8))
        assert x[0].item() == n + 1


# ---- layers on caches of 4 bits ------------------------------------------------------------------------------------
SMALL_BF16 = wl.LayerShape(d=512, n_q_heads=8, n_kv_heads=2, head_dim=128, rank=16, n_adapters=3)
SMALL_F32 = wl.LayerShape(d=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rank=8, n_adapters=2, dtype="f32")
ODD_F32 = wl.LayerShape(d=200, n_q_heads=6, n_kv_heads=3, head_dim=34, rank=5, n_adapters=2, dtype="f32")
ODD_BF16 = wl.LayerShape(d=320, n_q_heads=8, n_kv_heads=4, head_dim=80, rank=8, n_adapters=2)


def q_copy(ab, ctx, cache):
    """A cache of 4 bits with the rows and the table of a KVCache, and that KVCache with what the codes stand for."""
    n_kv, h = int(cache.k.shape[1]), int(cache.k.shape[2])
    four = ab.QCache([cache.pool_tokens], n_kv, h, "cuda")
    every = [(0, 0, cache.pool_tokens)]
    ab.alora_qcache_store(ctx, four, cache, every)
    ab.alora_qcache_load(ctx, cache, four, every)
    four.seq_offset, four.seq_capacity, four.seq_len = cache.seq_offset.copy(), cache.seq_capacity.copy(), cache.seq_len.copy()
    if cache.prefix_len is not None:
        four.prefix_offset, four.prefix_len = cache.prefix_offset.copy(), cache.prefix_len.copy()
    four._refresh()
    return four


def check_layers(ab, ctx, case, four, full, out, decode):
    """The new codes are those of the rows that the call on the other cache appends; the outputs are attention over what the codes stand for."""
    shape = case.shape
    layer = H.gpu_layer(case, shape)
    x = case.x_packed.cuda().contiguous()
    P = [int(n) for n in full.seq_len]
    if decode:
        ab.alora_decode(ctx, layer, full, x, case.k, case.adapter)
    else:
        ab.alora_prefill(ctx, layer, full, x, case.cu, case.k, case.adapter)
    ref = ab.QCache([full.pool_tokens], shape.n_kv_heads, shape.head_dim, "cuda")
    ab.alora_qcache_store(ctx, ref, full, [(0, 0, full.pool_tokens)])
    torch.cuda.synchronize()
    for name in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(ref, name), getattr(four, name)), f"{name} differs from the rows appended to a cache of the storage type"
    assert np.array_equal(four.seq_len, full.seq_len)
    K = qref.values(four.k.cpu().numpy(), four.k_scale.cpu().numpy())
    V = qref.values(four.v.cpu().numpy(), four.v_scale.cpu().numpy())
    tol, worst = H.TOL[shape.dtype], 0.0
    for b, S in enumerate(case.S):
        if S == 0:
            continue
        pos = np.arange(P[b], P[b] + S)
        q, _, _ = orc.project_qkv(case.layer, orc._normed(case.layer, H.f64(case.x_new[b]), shape.dtype), pos, case.k[b], case.adapter[b])
        q = orc.rope(q, pos, shape.n_q_heads, shape.head_dim, shape.rope_theta)
        n, plen = P[b] + S, int(four.prefix_len[b]) if four.prefix_len is not None else 0
        at = np.arange(n) + int(four.seq_offset[b]) - plen
        if plen:
            at[:plen] = np.arange(plen) + int(four.prefix_offset[b])
        want = qref.attend(q, K[at], V[at], shape.n_q_heads, list(pos + 1))[0]
        e = H.rel_err(H.f64(out[case.cu[b]:case.cu[b + 1]]), want)
        worst = max(worst, e)
        assert e <= tol, f"sequence {b}: {e:.3e}"
    H.report(check="qcache layer", err=worst, tol=tol)


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_F32, ODD_F32, ODD_BF16], ids=["bf16", "f32", "odd_f32", "odd_bf16"])
@pytest.mark.parametrize("decode", [False, True], ids=["prefill", "decode"])
def test_prefill_and_decode(ab, ctx, shape, decode):
    S = [1] * 5 if decode else [1, 40, 0, 7, 300]
    case = H.make_case(shape, [90, 0, 5, 200, 33], S, [90, 0, 2, 500, 40], [0, 1, -1, 1, 0], seed=21, prefix="random")
    full = H.gpu_cache(case)
    four = q_copy(ab, ctx, full)
    layer = H.gpu_layer(case, shape)
    x = case.x_packed.cuda().contiguous()
    out = ab.alora_qcache_decode(ctx, layer, four, x, case.k, case.adapter) if decode else ab.alora_qcache_prefill(ctx, layer, four, x, case.cu, case.k, case.adapter)
    check_layers(ab, ctx, case, four, full, out, decode)


def test_plain_kernels(ab):
    """The option that forces the kernels for any shape, on the layers' path."""
    c = ab.Context(0)
    try:
        c.set_option("kernels", 1)
        case = H.make_case(SMALL_BF16, [90, 0, 33], [3, 40, 1], [90, 0, 40], [0, 1, -1], seed=23, prefix="random")
        full = H.gpu_cache(case)
        four = q_copy(ab, c, full)
        out = ab.alora_qcache_prefill(c, H.gpu_layer(case, SMALL_BF16), four, case.x_packed.cuda().contiguous(), case.cu, case.k, case.adapter)
        check_layers(ab, c, case, four, full, out, False)
    finally:
        c.close()


@pytest.mark.parametrize("k_pow,q_pow", [(0, 0), (15, -14), (-16, 13)], ids=["as_usual", "over_fp16", "under_fp16"])
def test_keys_around_what_fp16_holds(ab, ctx, k_pow, q_pow):
    """Many rows of a sequence multiply in fp16 where it holds every key: here half of the channels' keys are far over it, or below its normal numbers, and the
    queries' the other way, so that scores are of the usual size."""
    shape = SMALL_BF16
    case = H.make_case(shape, [200, 70], [40, 33], [999, 999], [-1, -1], seed=24, prefix="random")
    channels = torch.arange(shape.head_dim) % 64 < 32       # (whole blocks, and both halves of a rotation)
    scale = torch.ones(shape.n_qkv, 1)
    scale[:shape.n_q][channels.repeat(shape.n_q_heads)] = 2.0 ** q_pow
    scale[shape.n_q:shape.n_q + shape.n_kv][channels.repeat(shape.n_kv_heads)] = 2.0 ** k_pow
    W = case.tensors["W_qkv"]
    case.tensors["W_qkv"] = (W.float() * scale).to(W.dtype)
    case.layer = H.oracle_layer(case.tensors, shape)
    for K in case.cache_K:
        K[:, channels.repeat(shape.n_kv_heads).numpy()] *= 2.0 ** k_pow
    full = H.gpu_cache(case)
    four = q_copy(ab, ctx, full)
    out = ab.alora_qcache_prefill(ctx, H.gpu_layer(case, shape), four, case.x_packed.cuda().contiguous(), case.cu, case.k, case.adapter)
    check_layers(ab, ctx, case, four, full, out, False)


@pytest.mark.parametrize("decode", [False, True], ids=["prefill", "decode"])
def test_adapters_on_shared_contexts(ab, ctx, decode):
    C, group, own = [150, 70], [0, 1, 0, -1, 0], [3, 0, 0, 9, 20]
    S = [1] * 5 if decode else [4, 9, 1, 30, 0]
    case, kv = H.contexts_case(SMALL_BF16, C, group, own, S, [150, 70, 151, 3, 999], [0, 1, 2, -1, 1], seed=22)
    full = H.contexts_cache(ab, case, kv, C, group, own)
    n = len(S)
    full.seq_offset, full.seq_capacity, full.seq_len = full.seq_offset[:n].copy(), full.seq_capacity[:n].copy(), full.seq_len[:n].copy()
    full.prefix_offset, full.prefix_len = full.prefix_offset[:n].copy(), full.prefix_len[:n].copy()
    full._refresh()
    four = q_copy(ab, ctx, full)
    layer = H.gpu_layer(case, SMALL_BF16)
    x = case.x_packed.cuda().contiguous()
    out = ab.alora_qcache_decode(ctx, layer, four, x, case.k, case.adapter) if decode else ab.alora_qcache_prefill(ctx, layer, four, x, case.cu, case.k, case.adapter)
    check_layers(ab, ctx, case, four, full, out, decode)


def test_a_conversation_as_it_is_used(ab, ctx):
    """Three layers: a base context is prefilled in bf16 and parked in 4 bits; two adapters fork its end and share the rest, are invoked, decode some tokens; one
    ends and the pool is closed up; the other goes on.  Against the same calls on bf16 caches that hold what the codes stand for, step by step."""
    shape = wl.LayerShape(d=512, n_q_heads=8, n_kv_heads=2, head_dim=128, rank=16, n_adapters=2, intermediate=1024)
    rng = wl.Rng(31)
    layers = [H.gpu_layer(wl.make_layer(shape, rng, f"L{l}"), shape) for l in range(3)]
    base = [ab.KVCache([200, 60, 60], 2, 128, torch.bfloat16, "cuda") for _ in range(3)]
    x0 = wl.make_hidden(rng, "x0", 150, shape).cuda()
    for c in base:
        c.seq_offset, c.seq_capacity, c.seq_len = c.seq_offset[:1], c.seq_capacity[:1], c.seq_len[:1]
        c._refresh()
    ab.alora_stack_prefill(ctx, layers, base, x0, [0, 150], [0], [-1])
    four = [ab.QCache([200, 60, 60], 2, 128, "cuda") for _ in range(3)]
    ab.alora_qcache_store(ctx, four, base, [(0, 0, 150)])
    # sequences 1 and 2 share rows 0..127 and have 128..149 of their own
    ab.alora_qcache_copy(ctx, four, four, [(128, 200, 22), (128, 260, 22)])

    def table(c, off, cap, length, plen):
        c.seq_offset, c.seq_capacity, c.seq_len = np.array(off, np.int64), np.array(cap, np.int32), np.array(length, np.int32)
        c.prefix_offset, c.prefix_len = np.zeros(len(off), np.int64), np.array(plen, np.int32)
        c._refresh()

    for c in four:
        table(c, [200, 260], [60, 60], [150, 150], [128, 128])

    def step(x, cu, k, a, decode):
        """The call, and the same in bf16 on what the codes stand for, layer by layer as one call."""
        full = [ab.KVCache([c.pool_tokens], 2, 128, torch.bfloat16, "cuda") for c in four]
        ab.alora_qcache_load(ctx, full, four, [(0, 0, four[0].pool_tokens)])
        for f, c in zip(full, four):
            table(f, c.seq_offset, c.seq_capacity, c.seq_len, c.prefix_len)
        if decode:
            got = ab.alora_qcache_stack_decode(ctx, layers, four, x, k, a)
            want = ab.alora_stack_decode(ctx, layers, full, x, k, a)
        else:
            got = ab.alora_qcache_stack_prefill(ctx, layers, four, x, cu, k, a)
            want = ab.alora_stack_prefill(ctx, layers, full, x, cu, k, a)
        assert np.array_equal(four[0].seq_len, full[0].seq_len) and np.array_equal(four[2].seq_len, full[0].seq_len)
        # The new rows of the call on bf16 caches are not in 4 bits, and are S of n keys; a 4-bit key or value is off by at most a sixth
        # of its size, so the hidden states of the two agree to a fraction only: a wrong row, mask or layer is of order one.
        d = (got - want).double().norm() / want.double().norm()
        assert d < 0.2, f"{float(d):.3f}"
        # layer 0 sees the same input: its new codes are those of the bf16 rows
        ref = ab.QCache([four[0].pool_tokens], 2, 128, "cuda")
        ab.alora_qcache_store(ctx, ref, full[0], [(0, 0, ref.pool_tokens)])
        for b in range(len(k)):
            lo = int(four[0].seq_offset[b]) + int(four[0].seq_len[b]) - int(four[0].prefix_len[b]) - (1 if decode else cu[b + 1] - cu[b])
            hi = int(four[0].seq_offset[b]) + int(four[0].seq_len[b]) - int(four[0].prefix_len[b])
            assert torch.equal(ref.k[lo:hi], four[0].k[lo:hi]) and torch.equal(ref.v_scale[lo:hi], four[0].v_scale[lo:hi])

    step(wl.make_hidden(rng, "x1", 9, shape).cuda(), [0, 4, 9], [150, 150], [0, 1], False)
    for t in range(3):
        step(wl.make_hidden(rng, f"y{t}", 2, shape).cuda(), None, [150, 150], [0, 1], True)
    # sequence 0 ends: the other's rows move over its region and it goes on from there
    own = int(four[0].seq_len[1]) - 128
    ab.alora_qcache_copy(ctx, four, four, [(260, 245, own)])
    for c in four:
        table(c, [245], [75], [128 + own], [128])
    for t in range(2):
        step(wl.make_hidden(rng, f"z{t}", 1, shape).cuda(), None, [150], [1], True)
