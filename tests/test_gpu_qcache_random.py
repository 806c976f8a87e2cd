"""Random batches of attention over rows of 4 bits: any head layout and size, lengths, shared contexts, exponents far apart, options, against float64 numpy."""
import os

import numpy as np
import pytest

from paper_2504_12397_amd import workloads as wl
from tests import helpers as H
from tests import qref
from tests.test_gpu_qcache_attend import Batch, check_layers, q_copy

pytestmark = pytest.mark.gpu
SEEDS = range(int(os.environ.get("ALORA_RANDOM_SEEDS", "60")))


@pytest.fixture(scope="module")
def ab():
    from paper_2504_12397_amd import binding
    return binding


@pytest.mark.parametrize("seed", SEEDS)
def test_random_batch(ab, seed):
    rng = np.random.default_rng(9000 + seed)
    pick = lambda *x: x[rng.integers(len(x))]  # noqa: E731
    dtype = pick("bf16", "bf16", "f32")
    h = int(pick(64, 128, 64, 128, 2 * rng.integers(1, 129), 8 * rng.integers(1, 33)))
    n_kv, G = int(pick(1, 2, 3, 5, 8, 9, 17)), int(pick(1, 1, 2, 3, 4, 7, 16))
    B = int(rng.integers(1, 12))
    C = [int(rng.integers(1, 400)) for _ in range(rng.integers(0, 3))]
    group = [int(rng.integers(-1, len(C))) for _ in range(B)]
    most = int(pick(1, 4, 30, 90))
    new = [int(rng.integers(0, most + 1)) for _ in range(B)]
    new[int(rng.integers(B))] = most
    longest = int(pick(1, 50, 700))
    own = [n + int(rng.integers(0, longest)) if n or rng.integers(2) else int(rng.integers(1, longest + 1)) for n in new]
    own = [max(o, 1) for o in own]
    work = sum(n * (o + (C[g] if g >= 0 else 0)) for n, o, g in zip(new, own, group)) * n_kv * G * h
    if work > 6e8:                                        # (the reference is numpy)
        n_kv, G = 1, min(G, 2)
    c = ab.Context(0)
    try:
        c.set_option("kv_splits", int(pick(0, 0, 0, 1, 2, 37, 256)))
        c.set_option("qattn_fp16", int(pick(0, 1, 1)))
        c.set_option("kernels", int(pick(0, 0, 0, 0, 1)))
        print(f"seed {seed}: {dtype} {n_kv} x {G} heads of {h}, new {new} of {own} behind {C} {group}", flush=True)
        b = Batch(ab, dtype, n_kv * G, n_kv, h, own, new, C=C, group=group, seed=seed, q_scale=float(pick(0.1, 1.0, 4.0)))
        if rng.integers(2):
            for _, e in b.codes:
                live = e != 255
                e[live] = np.clip(e[live].astype(int) + rng.integers(-pick(3, 25), 4, size=int(live.sum())), 2, 200).astype(np.uint8)
            b.cache = b.make(ab)
        out = ab.alora_qcache_attend(c, b.cache, b.q, b.cu, n_kv * G).double().cpu().numpy()
        for i in range(B):
            if new[i] == 0:
                continue
            ref, mag, total, spread = b.reference(i)
            # The largest probability may be 2^-8 and they travel as up to three parts: a part below fp32's smallest normal number, 2^-126, may count as 0, which is
            # 3 * 2^-126 of a probability and 3 * 2^-118 of the largest: that many of sum |v|.  (Scores lie hundreds apart here; elsewhere this is nothing.)
            tol = qref.tolerance(ref, mag, total, spread, h, len(b.rows(i)), dtype) + 3 * 2.0 ** -118 * total
            worst = float((np.abs(out[b.cu[i]:b.cu[i + 1]] - ref) / tol).max())
            assert worst <= 1.0, f"sequence {i}: {worst:.3f} of the tolerance"
    finally:
        c.close()


@pytest.mark.parametrize("seed", [3 * s for s in range(len(SEEDS) // 3)])
def test_random_layer(ab, seed):
    """Prefill and decode on random layers: odd widths, ranks, head sizes, adapters that begin anywhere."""
    rng = np.random.default_rng(7000 + seed)
    pick = lambda *x: x[rng.integers(len(x))]  # noqa: E731
    dtype = pick("bf16", "bf16", "f32")
    h = int(pick(64, 128, 128, 2 * rng.integers(1, 129), 8 * rng.integers(1, 33)))
    n_kv, G = int(pick(1, 2, 3, 4)), int(pick(1, 2, 4, 5))
    d = int(pick(128, 256, 512, 200, 36))
    n_ad = int(rng.integers(1, 4))
    shape = wl.LayerShape(d=d, n_q_heads=n_kv * G, n_kv_heads=n_kv, head_dim=h, rank=int(pick(8, 16, 5, 32)), n_adapters=n_ad, dtype=dtype, rmsnorm=bool(rng.integers(2)))
    B = int(rng.integers(1, 7))
    decode = bool(rng.integers(3) == 0)
    P = [int(pick(0, rng.integers(0, 10), rng.integers(0, 300))) for _ in range(B)]
    S = [1] * B if decode else [int(pick(0, 1, rng.integers(1, 20), rng.integers(1, 150))) for _ in range(B)]
    k = [int(rng.integers(0, P[b] + S[b] + 2)) for b in range(B)]
    a = [int(rng.integers(-1, n_ad)) for _ in range(B)]
    if sum(S) == 0:
        S[0] = 1
    print(f"seed {seed}: {shape} decode {decode} P {P} S {S} k {k} a {a}", flush=True)
    c = ab.Context(0)
    try:
        c.set_option("qattn_fp16", int(pick(0, 1, 1)))
        case = H.make_case(shape, P, S, k, a, seed=seed, prefix="random")
        full = H.gpu_cache(case)
        four = q_copy(ab, c, full)
        x, layer = case.x_packed.cuda().contiguous(), H.gpu_layer(case, shape)
        out = ab.alora_qcache_decode(c, layer, four, x, k, a) if decode else ab.alora_qcache_prefill(c, layer, four, x, case.cu, k, a)
        check_layers(ab, c, case, four, full, out, decode)
    finally:
        c.close()
