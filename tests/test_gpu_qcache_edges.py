"""Attention over rows of 4 bits and the calls that run layers on them, where they may go wrong: probabilities far below the largest, values at the lower end of the
format, codes, exponents, queries and results that begin anywhere, batches of very different numbers of rows, values that are not numbers on the layers' own path, and
stacks layer by layer."""
import numpy as np
import pytest
import torch

from oracle import alora_oracle as orc
from paper_2504_12397_amd import workloads as wl
from tests import helpers as H
from tests import qref
from tests.test_gpu_qcache_attend import Batch, check_layers, q_copy

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


# ---- numbers --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,h,rows", [("bf16", 128, 24), ("bf16", 64, 24), ("bf16", 128, 1), ("bf16", 96, 24), ("f32", 64, 24)],
                         ids=["many_rows_128", "many_rows_64", "one_row", "other_head", "f32"])
@pytest.mark.parametrize("sink", [0, 50_000], ids=["first", "in_the_middle"])
@pytest.mark.parametrize("v_sink", [0, 1])
def test_many_keys_far_below_one(ab, ctx, dtype, h, rows, sink, v_sink):
    """One key takes nearly all of the weight; 100000 others have 2^-14 to 2^-26 of it each and count together.  Their values are 1, the one key's is v_sink, so the result
    is known in closed form: small probabilities may be lost neither from the sum of values nor from the sum of probabilities."""
    n, n_kv, G = 100_000 + rows, 2, 4
    four = ab.QCache([n], n_kv, h, "cuda")
    four.v.fill_(0x22)                      # every channel 1.0
    four.k[sink, :, 0] = 7                  # channel 0 of this key is 6, all else 0
    four.v[sink] = 0x22 if v_sink else 0
    four.seq_len[0] = n
    for power in (14, 18, 21, 22, 23, 24, 26):
        q = torch.zeros((rows, n_kv * G * h), dtype=DT[dtype])
        q[:, 0::h] = power * np.log(2.0) * np.sqrt(h) / 6
        s = 6 * float(q[0, 0]) / np.sqrt(h)
        out = ab.alora_qcache_attend(ctx, four, q.cuda(), [0, rows], n_kv * G).double().cpu().numpy()
        others = np.arange(n - rows, n)[:, None] * np.exp(-s)
        ref = (v_sink + others) / (1 + others) * np.ones(out.shape)
        total = np.full(ref.shape, float(n))
        tol = qref.tolerance(ref, ref, total, np.full((rows, n_kv * G), s), h, n, dtype)
        worst = (np.abs(out - ref) / tol).max()
        assert worst <= 1.0, f"2^-{power}: {worst:.3f} of the tolerance, {out[0, 0]} for {ref[0, 0]}"


def lowest_tolerance(ref, mag, spread, h, L, dtype):
    """Values of 2^-126 and a little more: the relative part of qref.tolerance (without what fp16 loses: it does not hold such values), and what
    numbers below 2^-126 lose: sums of p v are fp32 numbers with p as small as 2^-8, each of at most 2 L + 64 additions off by half of 2^-149, and are
    divided by a sum of p of 2^-8 at least; and the stored result by half of its type's smallest number, 2^-133 or 2^-149."""
    rel = qref.tolerance(ref, mag, np.zeros_like(mag), spread, h, L, dtype) - 1e-37
    return rel + (2 * L + 64) * 2.0 ** -150 * 2.0 ** 8 + (2.0 ** -134 if dtype == "bf16" else 2.0 ** -150)


@pytest.mark.parametrize("kernels", [0, 1])
@pytest.mark.parametrize("dtype,h", [("bf16", 128), ("bf16", 64), ("bf16", 80), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 40)])
@pytest.mark.parametrize("e_v", [2, 3, 8, 30])
def test_smallest_values(ab, dtype, h, e_v, kernels):
    """Values with the lowest exponents: a result of zeros, or of the wrong sign, is outside the tolerance."""
    c = ab.Context(0)
    try:
        c.set_option("kernels", kernels)
        b = Batch(ab, dtype, 8, 2, h, [90, 40], [1, 17], seed=7)
        codes, e = b.codes[1]
        e[e != 255] = e_v
        b.cache = b.make(ab)
        out = ab.alora_qcache_attend(c, b.cache, b.q, b.cu, 8).double().cpu().numpy()
        for i in range(2):
            ref, mag, total, spread = b.reference(i)
            tol = lowest_tolerance(ref, mag, spread, h, 90, dtype)
            assert np.abs(ref).max() > 8 * tol.max(), "the tolerance would pass a result of zeros"
            worst = (np.abs(out[b.cu[i]:b.cu[i + 1]] - ref) / tol).max()
            assert worst <= 1.0, f"sequence {i}: {worst:.3f} of the tolerance"
    finally:
        c.close()


@pytest.mark.parametrize("dtype,n_q,n_kv,h", [("bf16", 32, 8, 128), ("bf16", 8, 4, 64), ("bf16", 10, 5, 80), ("f32", 8, 2, 128)])
def test_batches_of_very_different_numbers_of_rows(ab, ctx, dtype, n_q, n_kv, h):
    """One suffix of many rows beside many of a few and single tokens, some on a shared context."""
    new = [128] + [5, 1, 0, 9] * 8 + [40]
    own = [128 + 37] + [n + 3 * i for i, n in enumerate([5, 1, 2, 9] * 8)] + [40]
    b = Batch(ab, dtype, n_q, n_kv, h, own, new, C=[150], group=[i % 3 - 1 if i % 3 < 2 else 0 for i in range(len(new))], seed=41)
    b.check(ab.alora_qcache_attend(ctx, b.cache, b.q, b.cu, n_q))


# ---- where arrays begin ---------------------------------------------------------------------------------------------
def shifted(t, by):
    """The same values, `by` elements into an allocation (which begins at a multiple of 512 bytes)."""
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    out = flat[by:].view(t.shape)
    out.copy_(t)
    return out


def shift_rows(ab, c, codes, exps):
    """The cache with its codes and exponents that many bytes further on."""
    d = ab.QCache.from_tensors(shifted(c.k, codes), shifted(c.v, codes), shifted(c.k_scale, exps), shifted(c.v_scale, exps), c.seq_offset, c.seq_capacity, c.seq_len,
                               c.prefix_offset, c.prefix_len)
    return d


@pytest.mark.parametrize("codes,exps,q_at,out_at", [(4, 0, 0, 0), (8, 4, 0, 0), (1, 0, 0, 0), (16, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 4), (0, 0, 8, 8), (3, 3, 3, 3)])
@pytest.mark.parametrize("dtype,n_q,n_kv,h", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("f32", 4, 2, 64), ("bf16", 6, 3, 80), ("f32", 3, 1, 34)])
def test_attention_on_arrays_that_begin_anywhere(ab, ctx, dtype, n_q, n_kv, h, codes, exps, q_at, out_at):
    b = Batch(ab, dtype, n_q, n_kv, h, [70, 33, 150], [1, 20, 40], C=[45], group=[0, -1, 0], seed=42)
    out = shifted(torch.zeros_like(b.q), out_at)
    got = ab.alora_qcache_attend(ctx, shift_rows(ab, b.cache, codes, exps), shifted(b.q, q_at), b.cu, n_q, out=out)
    assert got.data_ptr() == out.data_ptr()
    b.check(out)


@pytest.mark.parametrize("codes,exps,out_at", [(4, 0, 0), (1, 1, 0), (0, 0, 3), (0, 0, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layers_on_arrays_that_begin_anywhere(ab, ctx, dtype, codes, exps, out_at):
    shape = LAYER[dtype]
    case = H.make_case(shape, [90, 5], [40, 1], [90, 2], [0, 1], seed=43, prefix="random")
    full = H.gpu_cache(case)
    four = shift_rows(ab, q_copy(ab, ctx, full), codes, exps)
    out = shifted(torch.zeros((41, shape.n_q), dtype=shape.torch_dtype, device="cuda"), out_at)
    ab.alora_qcache_prefill(ctx, H.gpu_layer(case, shape), four, case.x_packed.cuda().contiguous(), case.cu, case.k, case.adapter, attn_out=out)
    check_layers(ab, ctx, case, four, full, out, False)


# ---- layers ---------------------------------------------------------------------------------------------------------
LAYER = {"bf16": wl.LayerShape(d=512, n_q_heads=8, n_kv_heads=2, head_dim=128, rank=16, n_adapters=2),
         "f32": wl.LayerShape(d=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rank=8, n_adapters=2, dtype="f32")}


@pytest.mark.parametrize("dtype,n_q,n_kv,h", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("bf16", 8, 4, 80), ("f32", 4, 2, 64)])
def test_layer_rows_that_are_not_numbers(ab, ctx, dtype, n_q, n_kv, h):
    """A new row whose value overflows in one channel, one whose key does, and a cached block that is NaN: each reaches the rows that see it, in the channels it is
    in (a key: in all channels of its kv head), and no others."""
    shape = wl.LayerShape(d=320, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=h, rank=8, n_adapters=1, dtype=dtype, rmsnorm=False)
    P, S, at_v, at_k = [80, 60], [50, 30], 12, 33
    case = H.make_case(shape, P, S, [999, 999], [-1, -1], seed=44, prefix="random")
    W = case.tensors["W_qkv"]
    W[:, 3] = W[:, 5] = 0.0
    W[shape.n_q + shape.n_kv + 40, 3] = 1e30              # channel 40 of kv head 0's values
    W[shape.n_q + h + 10, 5] = 1e30                       # channel 10 of kv head 1's keys
    layer = H.gpu_layer(case, shape)
    x = case.x_packed.clone()
    x[:, [3, 5]] = 0.0
    full = H.gpu_cache(case)
    clean_cache = q_copy(ab, ctx, full)
    clean = ab.alora_qcache_prefill(ctx, layer, clean_cache, x.cuda(), case.cu, case.k, case.adapter)
    four = q_copy(ab, ctx, full)
    four.v_scale[int(four.seq_offset[1]) + 7, 1, 0] = 255
    x[at_v, 3] = x[at_k, 5] = 1e30
    out = ab.alora_qcache_prefill(ctx, layer, four, x.cuda(), case.cu, case.k, case.adapter)
    G = n_q // n_kv
    want = torch.zeros((80, n_q, h), dtype=torch.bool)
    want[at_v:50, :G, 32:64] = True
    want[at_k:50, G:2 * G, :] = True
    want[50:, G:2 * G, :32] = True
    got = torch.isnan(out).cpu().view(80, n_q, h)
    assert torch.equal(got, want)
    o, c = out.cpu().double().view(80, n_q, h), clean.cpu().double().view(80, n_q, h)
    assert (o[~want] - c[~want]).abs().max() <= 2.0 ** -6 * c.abs().max()


@pytest.mark.parametrize("k_pow,q_pow", [(0, 0), (15, -14), (-16, 13)], ids=["as_usual", "over_fp16", "under_fp16"])
def test_keys_of_smaller_heads_around_what_fp16_holds(ab, ctx, k_pow, q_pow):
    """As for heads of 128, all keys alike: far over what fp16 holds, or below its normal numbers, the queries the other way."""
    shape = wl.LayerShape(d=512, n_q_heads=8, n_kv_heads=2, head_dim=64, rank=16, n_adapters=1)
    case = H.make_case(shape, [200, 70], [40, 33], [999, 999], [-1, -1], seed=45, prefix="random")
    scale = torch.ones(shape.n_qkv, 1)
    scale[:shape.n_q] = 2.0 ** q_pow
    scale[shape.n_q:shape.n_q + shape.n_kv] = 2.0 ** k_pow
    W = case.tensors["W_qkv"]
    case.tensors["W_qkv"] = (W.float() * scale).to(W.dtype)
    case.layer = H.oracle_layer(case.tensors, shape)
    for K in case.cache_K:
        K *= 2.0 ** k_pow
    full = H.gpu_cache(case)
    four = q_copy(ab, ctx, full)
    out = ab.alora_qcache_prefill(ctx, H.gpu_layer(case, shape), four, case.x_packed.cuda().contiguous(), case.cu, case.k, case.adapter)
    check_layers(ab, ctx, case, four, full, out, False)


STACKS = {"bf16": wl.LayerShape(d=512, n_q_heads=8, n_kv_heads=2, head_dim=128, rank=16, n_adapters=2, intermediate=1024, adapt_rest=True),
          "bf16_64": wl.LayerShape(d=256, n_q_heads=4, n_kv_heads=4, head_dim=64, rank=8, n_adapters=2, intermediate=512),
          "f32": wl.LayerShape(d=256, n_q_heads=4, n_kv_heads=2, head_dim=64, rank=8, n_adapters=2, dtype="f32", intermediate=384, adapt_rest=True),
          "odd_f32": wl.LayerShape(d=200, n_q_heads=6, n_kv_heads=3, head_dim=34, rank=5, n_adapters=2, dtype="f32", intermediate=100)}


@pytest.mark.parametrize("decode", [False, True], ids=["prefill", "decode"])
@pytest.mark.parametrize("name", list(STACKS))
def test_stacks_layer_by_layer(ab, ctx, name, decode):
    """Three layers in one call are the layers one by one, bit for bit; and each of those is the call that attends alone, in the codes it stores, and the oracle's attention
    over what the codes stand for with the oracle's rest of the layer behind it, within the tolerance that the stacks on other caches are held to."""
    shape, n_layers = STACKS[name], 3
    P, S, k, a = [90, 7, 40], [1, 1, 1] if decode else [33, 1, 20], [90, 3, 999], [1, 0, -1]
    T, cu = sum(S), [0, S[0], S[0] + S[1], sum(S)]
    rng = wl.Rng(46)
    tensors = [wl.make_layer(shape, rng, f"L{l}") for l in range(n_layers)]
    layers = [H.gpu_layer(t, shape) for t in tensors]
    x = wl.make_hidden(rng, "x", T, shape).cuda()
    caps = [p + s + 4 for p, s in zip(P, S)]
    start = []
    for l in range(n_layers):
        full = ab.KVCache(caps, shape.n_kv_heads, shape.head_dim, shape.torch_dtype, "cuda")
        for b in range(3):
            full.load_prefix(b, *wl.make_random_kv(rng, f"L{l}kv{b}", P[b], shape))
        start.append(q_copy(ab, ctx, full))

    def fresh(l):
        c = start[l]
        return ab.QCache.from_tensors(c.k.clone(), c.v.clone(), c.k_scale.clone(), c.v_scale.clone(), c.seq_offset, c.seq_capacity, list(c.seq_len))

    def stack(ls, cs, x):
        return (ab.alora_qcache_stack_decode(ctx, ls, cs, x, k, a) if decode else ab.alora_qcache_stack_prefill(ctx, ls, cs, x, cu, k, a))

    def codes(c):
        return [c.k, c.v, c.k_scale, c.v_scale]

    whole = [fresh(l) for l in range(n_layers)]
    out = stack(layers, whole, x)
    tol, worst = H.TOL[shape.dtype], 0.0
    for l in range(n_layers):
        one, alone = fresh(l), fresh(l)
        y = stack([layers[l]], [one], x)
        if decode:
            ab.alora_qcache_decode(ctx, layers[l], alone, x, k, a)
        else:
            ab.alora_qcache_prefill(ctx, layers[l], alone, x, cu, k, a)
        torch.cuda.synchronize()
        for u, v, w in zip(codes(whole[l]), codes(one), codes(alone)):
            assert torch.equal(u, v) and torch.equal(u, w), f"layer {l}: codes"
        assert list(whole[l].seq_len) == list(one.seq_len) == [p + s for p, s in zip(P, S)]
        K, V = (qref.values(c.cpu().numpy(), e.cpu().numpy()) for c, e in ((one.k, one.k_scale), (one.v, one.v_scale)))
        layer = H.oracle_layer(tensors[l], shape)
        for b in range(3):
            pos = np.arange(P[b], P[b] + S[b])
            xb = H.f64(x[cu[b]:cu[b + 1]])
            q, _, _ = orc.project_qkv(layer, orc._normed(layer, xb, shape.dtype), pos, k[b], a[b])
            q = orc.rope(q, pos, shape.n_q_heads, shape.head_dim, shape.rope_theta)
            at = np.arange(P[b] + S[b]) + int(one.seq_offset[b])
            attn = qref.attend(q, K[at], V[at], shape.n_q_heads, list(pos + 1))[0]
            want = orc.layer_tail(layer, xb, attn, shape.dtype, pos, k[b], a[b])
            e = H.rel_err(H.f64(y[cu[b]:cu[b + 1]]), want)
            worst = max(worst, e)
            assert e <= tol, f"layer {l}, sequence {b}: {e:.3e}"
        x = y
    H.report(check="qcache stack", err=worst, tol=tol)
    assert torch.equal(out, x)


@pytest.mark.parametrize("h", [64, 128])
def test_option_for_probabilities_of_16_bits(ab, h):
    """qattn_fp16 = 0: a probability is rounded to 16 bits, one of 11 bits is 2^5 times as far off.  A result is stored as another number than the one next to the exact
    value where the exact value lies nearer to the middle between two numbers than the error: in proportion to the error, so in far fewer places (fp32 sums add some to both)."""
    c = ab.Context(0)
    try:
        b = Batch(ab, "bf16", 8, 2, h, [900, 300], [60, 9], C=[500], group=[0, 0], seed=47)
        off = {}
        for value in (1, 0):
            c.set_option("qattn_fp16", value)
            out = ab.alora_qcache_attend(c, b.cache, b.q, b.cu, 8)
            b.check(out)
            want = torch.cat([torch.from_numpy(b.reference(i)[0]) for i in range(2)]).to(torch.bfloat16)
            off[value] = float((out.cpu() != want).double().mean())
        H.report(check="qattn_fp16", off_11_bits=off[1], off_16_bits=off[0])
        assert off[0] < off[1] / 4
        # a value that is not a number, and values that fp16 does not hold, on this path alone
        codes, e = b.codes[1]
        e[b.rows(0)[-20], 0, 1] = 255
        nan = torch.isnan(ab.alora_qcache_attend(c, b.make(ab), b.q, b.cu, 8)).cpu().view(69, 8, h)
        want = torch.zeros_like(nan)
        want[40:60, :4, 32:64] = True
        assert torch.equal(nan, want)
        e[b.rows(0)[-20], 0, 1] = 160
        b.cache = b.make(ab)
        b.check(ab.alora_qcache_attend(c, b.cache, b.q, b.cu, 8))
        case = H.make_case(LAYER["bf16"], [200, 40], [40, 33], [200, 40], [0, 1], seed=48, prefix="random")
        full = H.gpu_cache(case)
        four = q_copy(ab, c, full)
        out = ab.alora_qcache_prefill(c, H.gpu_layer(case, LAYER["bf16"]), four, case.x_packed.cuda().contiguous(), case.cu, case.k, case.adapter)
        check_layers(ab, c, case, four, full, out, False)
    finally:
        c.close()
