"""Tensors that the context's GPU does not reach are refused before the library sees their addresses; pinned host memory, which it does reach, is not."""
import numpy as np
import pytest
import torch

from tests import qref

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


def test_host_tensors_are_refused(ab, ctx):
    kv, kv_cpu = (ab.KVCache([20], 2, 64, torch.float32, d) for d in ("cuda", "cpu"))
    q, q_cpu = (ab.QCache([20], 2, 64, d) for d in ("cuda", "cpu"))
    for c in (kv, kv_cpu, q, q_cpu):
        c.seq_len[0] = 5
    r = [(0, 10, 3)]
    x, x_cpu = torch.zeros(1, 256, device="cuda"), torch.zeros(1, 256)
    layer, layer_cpu = (ab.Layer({"W_qkv": torch.zeros(8 * 64, 256, device=d)}, 4, 2, 64) for d in ("cuda", "cpu"))
    bad = [lambda: ab.alora_cache_copy(ctx, kv_cpu, kv_cpu, r), lambda: ab.alora_cache_copy(ctx, kv, kv_cpu, r), lambda: ab.alora_cache_copy(ctx, kv_cpu, kv, r),
           lambda: ab.alora_cache_copy(ctx, [kv, kv_cpu], [kv, kv], r), lambda: ab.alora_cache_copy(ctx, [kv, kv], [kv, kv_cpu], r),
           lambda: ab.alora_qcache_copy(ctx, q_cpu, q_cpu, r), lambda: ab.alora_qcache_store(ctx, q, kv_cpu, r), lambda: ab.alora_qcache_store(ctx, q_cpu, kv, r),
           lambda: ab.alora_qcache_load(ctx, kv, q_cpu, r), lambda: ab.alora_qcache_load(ctx, kv_cpu, q, r),
           lambda: ab.alora_qcache_attend(ctx, q, x_cpu, [0, 1], 4), lambda: ab.alora_qcache_attend(ctx, q_cpu, x, [0, 1], 4),
           lambda: ab.alora_qcache_attend(ctx, q, x, [0, 1], 4, out=torch.zeros(1, 256)),
           lambda: ab.alora_qcache_decode(ctx, layer, q, x_cpu, [0], [-1]), lambda: ab.alora_qcache_decode(ctx, layer, q_cpu, x, [0], [-1]),
           lambda: ab.alora_qcache_decode(ctx, layer_cpu, q, x, [0], [-1]), lambda: ab.alora_qcache_decode(ctx, layer, q, x, [0], [-1], attn_out=torch.zeros(1, 256)),
           lambda: ab.alora_qcache_prefill(ctx, layer, q, x_cpu, [0, 1], [0], [-1])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert [int(c.seq_len[0]) for c in (kv, kv_cpu, q, q_cpu)] == [5] * 4
    with pytest.raises(ValueError):
        ab.KVCache.from_tensors(kv.k, kv_cpu.v)
    with pytest.raises(ValueError):
        ab.QCache.from_tensors(q.k, q.v, q.k_scale, q_cpu.v_scale)


def test_a_cache_in_pinned_memory(ab, ctx):
    """A context parked in 4 bits in the host's memory, and attended from there."""
    x = torch.randn((50, 2, 64), generator=torch.Generator().manual_seed(1))
    kv = ab.KVCache.from_tensors(x.cuda(), (x + 1).cuda())
    pin = lambda *s: torch.zeros(s, dtype=torch.uint8, pin_memory=True)  # noqa: E731
    four = ab.QCache.from_tensors(pin(60, 2, 32), pin(60, 2, 32), pin(60, 2, 2), pin(60, 2, 2), [10], [50], [50])
    ab.alora_qcache_store(ctx, four, kv, [(0, 10, 50)])
    q = torch.randn((3, 256), generator=torch.Generator().manual_seed(2))
    out = ab.alora_qcache_attend(ctx, four, q.cuda(), [0, 3], 4)
    torch.cuda.synchronize()
    codes = [qref.quantise(a.double().numpy()) for a in (x, x + 1)]
    assert np.array_equal(four.k[10:].numpy(), codes[0][0]) and np.array_equal(four.v_scale[10:].numpy(), codes[1][1])
    ref, mag, total, spread = qref.attend(q.double().numpy(), qref.values(*codes[0]), qref.values(*codes[1]), 4, [48, 49, 50])
    assert (np.abs(out.double().cpu().numpy() - ref) <= qref.tolerance(ref, mag, total, spread, 64, 50, "f32")).all()
