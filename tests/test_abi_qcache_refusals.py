"""CPU-side checks of what the calls on rows of a cache refuse beyond single bad arguments: tables of different lengths, arrays that lie over each other, sizes that no
launch or address takes, and the order in which errors are found.  Nothing is launched (validation-only context, device -1)."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.test_abi_qcache import FakeStream, GOOD, P, four, full, ranges, status, table


@pytest.fixture(scope="module")
def ab():
    from paper_2504_12397_amd import binding
    return binding


@pytest.fixture()
def v(ab):
    h = C.c_void_p()
    assert ab._lib.alora_create(C.byref(h), -1) == ab.ALORA_OK
    yield h
    ab._lib.alora_destroy(h)


# ---- tables of the binding's caches ---------------------------------------------------------------------------------
def tensors(ab, rows=20):
    t = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    return t(rows, 1, 32), t(rows, 1, 32), t(rows, 1, 2), t(rows, 1, 2)


@pytest.mark.parametrize("tables", [dict(seq_offset=[0]), dict(seq_capacity=[5, 5, 5]), dict(seq_len=[1]), dict(prefix_offset=[0], prefix_len=[0, 0]),
                                    dict(prefix_offset=[0, 0], prefix_len=[0]), dict(prefix_len=[0, 0])])
def test_tables_of_different_lengths(ab, tables):
    good = dict(seq_offset=[0, 10], seq_capacity=[5, 5], seq_len=[1, 2])
    kv = torch.zeros((20, 1, 64))
    ab.QCache.from_tensors(*tensors(ab), **good)
    ab.KVCache.from_tensors(kv, kv.clone(), **good)
    with pytest.raises(ValueError):
        ab.QCache.from_tensors(*tensors(ab), **dict(good, **tables))
    with pytest.raises(ValueError):
        ab.KVCache.from_tensors(kv, kv.clone(), **dict(good, **tables))


@pytest.mark.parametrize("change", [dict(seq_offset=np.zeros(1, np.int64)), dict(seq_capacity=np.zeros(1, np.int32)), dict(prefix_len=np.zeros(1, np.int32)),
                                    dict(prefix_offset=np.zeros(1, np.int64)), dict(seq_offset=None), dict(seq_len=None), dict(prefix_offset=None)])
def test_calls_on_tables_that_are_too_short(ab, change):
    """Tables set by hand: a call names more sequences than one of them has."""
    layer = ab.Layer({"W_qkv": torch.zeros(4 * 64, 64)}, 2, 1, 64)
    q = ab.QCache.from_tensors(*tensors(ab), seq_offset=[0, 10], seq_capacity=[5, 5], seq_len=[1, 2], prefix_offset=[0, 0], prefix_len=[0, 0])
    c = ab.Context(-1)
    try:
        def calls():
            yield lambda: ab.alora_qcache_attend(c, q, torch.zeros(2, 128), [0, 1, 2], 2, stream=FakeStream())
            yield lambda: ab.alora_qcache_decode(c, layer, q, torch.zeros(2, 64), [0, 0], [-1, -1], stream=FakeStream())
            yield lambda: ab.alora_qcache_prefill(c, layer, q, torch.zeros(2, 64), [0, 1, 2], [0, 0], [-1, -1], stream=FakeStream())
        for call in calls():
            with pytest.raises(ab.AloraError, match="validation-only"):
                call()
        for name, value in change.items():
            setattr(q, name, value)
        for call in calls():
            with pytest.raises(ValueError):
                call()
    finally:
        c.close()


def test_stacks_on_tables_of_different_lengths(ab):
    """The lengths of the first layer's cache are copied to the others after the call: they have to be as many."""
    layer = ab.Layer({"W_qkv": torch.zeros(4 * 64, 64)}, 2, 1, 64)
    c = ab.Context(-1)
    table = dict(seq_offset=[0, 10], seq_capacity=[5, 5], seq_len=[1, 2])
    try:
        for other in (dict(seq_offset=[0, 10, 15], seq_capacity=[5, 5, 5], seq_len=[1, 2, 0]), dict()):
            caches = [ab.QCache.from_tensors(*tensors(ab), **t) for t in (table, other)]
            with pytest.raises(ValueError):
                ab.alora_qcache_stack_decode(c, [layer, layer], caches, torch.zeros(2, 64), [0, 0], [-1, -1], stream=FakeStream())
    finally:
        c.close()


def test_tables_of_other_types(ab):
    q = ab.QCache.from_tensors(*tensors(ab), seq_offset=[0, 10], seq_capacity=[5, 5], seq_len=[1, 2])
    for name, bad in (("seq_offset", np.zeros(2, np.int32)), ("seq_len", np.zeros(2, np.int64)), ("seq_capacity", np.zeros(4, np.int32)[::2])):
        was = getattr(q, name)
        setattr(q, name, bad)
        with pytest.raises(ValueError):
            q._refresh()
        setattr(q, name, was)
        q._refresh()


# ---- the order in which errors are found ------------------------------------------------------------------------------
@pytest.mark.parametrize("desc,tables,want", [(dict(heads=3), dict(), "ALORA_ESHAPE"), (dict(dtype=7), dict(), "ALORA_EDTYPE"), (dict(d=0), dict(length=(50, 20)), "ALORA_ESHAPE"),
                                              (dict(), dict(length=(50, 20)), "ALORA_EINVAL")])
def test_errors_of_layers_come_first(ab, v, desc, tables, want):
    """A call with two mistakes names the one that the call on other caches names: the layer before the cache's arrays, these before the sequences."""
    desc, p = layer_desc(ab, **desc), full(ab, k=None)
    cu, zero, none = np.array([0, 1, 2], np.int32), np.zeros(2, np.int32), np.full(2, -1, np.int32)
    keep = [table(ab, p, **tables)]
    st = ab._lib.alora_prefill(v, C.byref(desc), C.byref(p), P, arg(cu), arg(zero), arg(none), 2, P, None)
    assert status(ab, st) == want
    for name in ("k", "k_scale"):
        q = four(ab)
        setattr(q, name, None)
        keep.append(table(ab, q, **tables))
        assert layer_calls(ab, v, desc, q, cu) == [want] * 2, name
        for fn in (lambda *a: ab._lib.alora_qcache_decode(v, C.byref(desc), *a), lambda *a: ab._lib.alora_qcache_stack_decode(v, C.byref(desc), 1, *a)):
            assert status(ab, fn(C.byref(q), P, arg(zero), arg(none), 2, P, None)) == want, name


def layer_desc(ab, heads=4, kv=2, h=64, dtype=1, d=64):
    return ab.LayerDesc(d, heads, kv, h, 0, 0, dtype, 128, P, None, None, None, None, None, P, 1e-5, 1e4, P, P, P, P, P)


def arg(a):
    return a.ctypes.data_as(C.POINTER(C.c_int32))


def layer_calls(ab, v, desc, cache, cu, x=P, out=P):
    B = len(cu) - 1
    cu, zero, none = np.array(cu, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    return [status(ab, ab._lib.alora_qcache_prefill(v, C.byref(desc), C.byref(cache), x, arg(cu), arg(zero), arg(none), B, out, None)),
            status(ab, ab._lib.alora_qcache_stack_prefill(v, C.byref(desc), 1, C.byref(cache), x, arg(cu), arg(zero), arg(none), B, out, None))]


# ---- sizes ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("off,poff", [(2 ** 63 - 1, 0), (2 ** 63 - 20, 0), (50, 2 ** 63 - 1), (50, 2 ** 63 - 6)])
def test_rows_whose_end_is_past_every_number(ab, v, off, poff):
    """offset + capacity and offset + prefix are over 2^63: outside the pool, not at its front."""
    q, k = four(ab), full(ab)
    tables = dict(off=(0, off), cap=(50, 50), length=(10, 20), poff=(0, poff), plen=(0, 8))
    keep = [table(ab, c, **tables) for c in (q, k)]
    cu = np.array([0, 1, 2], np.int32)
    assert status(ab, ab._lib.alora_qcache_attend(v, 1, 4, 2, 64, C.byref(q), P, arg(cu), 2, 2 * P, None)) == "ALORA_ECAPACITY"
    desc = layer_desc(ab)
    assert layer_calls(ab, v, desc, q, cu) == ["ALORA_ECAPACITY"] * 2
    zero, none = np.zeros(2, np.int32), np.full(2, -1, np.int32)
    st = ab._lib.alora_prefill(v, C.byref(desc), C.byref(k), P, arg(cu), arg(zero), arg(none), 2, P, None)
    assert status(ab, st) == "ALORA_ECAPACITY" and keep


@pytest.mark.parametrize("tokens", [2 ** 62, 2 ** 57, 2 ** 63 - 1])
def test_pools_that_no_address_reaches(ab, v, tokens):
    """pool_tokens times the bytes of a row is over 2^62."""
    lib, r = ab._lib, ranges(ab, GOOD)
    big, small, qbig, qsmall = full(ab, tokens=tokens), full(ab, 7 * P, 8 * P), four(ab, tokens=tokens), four(ab, 9 * P, 10 * P, 11 * P, 12 * P)
    for st in (lib.alora_cache_copy(v, 1, 2, 64, C.byref(big), C.byref(small), 1, r, 1, None), lib.alora_cache_copy(v, 1, 2, 64, C.byref(small), C.byref(big), 1, r, 1, None),
               lib.alora_qcache_copy(v, 2, 64, C.byref(qbig), C.byref(qsmall), 1, r, 1, None),
               lib.alora_qcache_store(v, 1, 2, 64, C.byref(qbig), C.byref(small), 1, r, 1, None),
               lib.alora_qcache_store(v, 1, 2, 64, C.byref(qsmall), C.byref(big), 1, r, 1, None),
               lib.alora_qcache_load(v, 1, 2, 64, C.byref(big), C.byref(qsmall), 1, r, 1, None)):
        assert status(ab, st) == "ALORA_ECAPACITY"
    keep = table(ab, qbig)
    cu = np.array([0, 1, 2], np.int32)
    assert status(ab, lib.alora_qcache_attend(v, 1, 4, 2, 64, C.byref(qbig), P, arg(cu), 2, 2 * P, None)) == "ALORA_ECAPACITY"
    assert layer_calls(ab, v, layer_desc(ab), qbig, cu) == ["ALORA_ECAPACITY"] * 2 and keep


# ---- arrays that lie over each other ----------------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("call", ["qcache_store", "qcache_load"])
def test_rows_and_their_codes_lie_apart(ab, v, call, side, name):
    """The rows of the storage type and those of 4 bits share no memory: codes that begin inside the rows, that end in them, and that lie right behind and right before."""
    lib, r, rows = ab._lib, ranges(ab, GOOD), 100
    row = 2 * 64 * 2                              # bytes of a row, and of its codes or exponents
    mine = 2 * 32 if "scale" not in name else 2 * 2
    def run(at):
        f, q = full(ab, 40 * P, 41 * P, rows), four(ab, tokens=rows)
        setattr(q, name, getattr(f, side) + at)
        fn = lib.alora_qcache_store if call == "qcache_store" else lib.alora_qcache_load
        a, b = (q, f) if call == "qcache_store" else (f, q)
        return status(ab, fn(v, 1, 2, 64, C.byref(a), C.byref(b), 1, r, 1, None))
    for at in (0, 64, rows * row - 64, 64 - rows * mine):
        assert run(at) == "ALORA_EINVAL", at
    for at in (rows * row, -rows * mine):
        assert run(at) == "ALORA_EHIP", at


# ---- what a launch takes ----------------------------------------------------------------------------------------------
def many(ab, T, per=2 ** 20, prefix=0):
    """A cache whose sequences have T rows in all, each all of its rows."""
    B = (T + per - 1) // per
    n = [min(per, T - b * per) for b in range(B)]
    off = [prefix + b * per for b in range(B)]
    q = four(ab, tokens=T + prefix)
    keep = table(ab, q, off=off, cap=n, length=[m + prefix for m in n], poff=[0] * B if prefix else None, plen=[prefix] * B if prefix else None)
    return q, keep, np.array([0] + list(np.cumsum(n)), np.int32)


@pytest.mark.parametrize("T,heads,kv,h,prefix,want", [
    (2 ** 22 - 1, 16, 16, 2, 0, "ALORA_EHIP"), (2 ** 22, 16, 16, 2, 0, "ALORA_EINVAL"), (2 ** 21, 64, 1, 34, 0, "ALORA_EINVAL"),      # a workgroup for each row and head
    (2 ** 21, 64, 8, 128, 0, "ALORA_EHIP"),                                                                                           # many columns a workgroup
    (2 ** 21, 64, 8, 128, 4, "ALORA_EINVAL"), (2 ** 21 - 1, 32, 8, 128, 4, "ALORA_EHIP")])                                            # two records a row and head are joined
def test_attention_of_more_rows_than_a_launch_takes(ab, v, T, heads, kv, h, prefix, want):
    q, keep, cu = many(ab, T, prefix=prefix)
    far = 2 ** 44
    assert status(ab, ab._lib.alora_qcache_attend(v, 1, heads, kv, h, C.byref(q), P, arg(cu), len(cu) - 1, far, None)) == want
    q, keep, _ = many(ab, T, prefix=prefix)
    for c in keep[2:3]:
        c[:] = prefix                             # the layers' rows are new
    desc = layer_desc(ab, heads=heads, kv=kv, h=h)
    assert layer_calls(ab, v, desc, q, cu, out=far)[0] == want


@pytest.mark.parametrize("call", ["cache_copy", "qcache_store"])
def test_more_pieces_than_a_launch_takes(ab, v, call):
    """2^24 ranges of a row each: a workgroup of 256 for every one."""
    lib, n = ab._lib, 2 ** 24
    r = np.zeros((n, 3), np.int64)
    r[:, 0] = np.arange(n)
    r[:, 1] = np.arange(n) + (n if "copy" in call else 0)
    r[:, 2] = 1
    tokens = 2 * n
    a, b = full(ab, 2 ** 40, 2 ** 41, tokens), full(ab, 2 ** 42, 2 ** 43, tokens)
    c = four(ab, 2 ** 44, 2 ** 45, 2 ** 46, 2 ** 47, tokens)
    for m, want in ((n, "ALORA_EINVAL"), (n - 1, "ALORA_EHIP")):
        p = r.ctypes.data
        st = {"cache_copy": lambda: lib.alora_cache_copy(v, 1, 1, 2, C.byref(b), C.byref(a), 1, p, m, None),
              "qcache_store": lambda: lib.alora_qcache_store(v, 1, 1, 2, C.byref(c), C.byref(a), 1, p, m, None)}[call]()
        assert status(ab, st) == want


def test_option_of_attention_over_rows_of_4_bits(ab, v):
    for value, want in ((0, ab.ALORA_OK), (1, ab.ALORA_OK), (2, ab.ALORA_EINVAL), (-1, ab.ALORA_EINVAL)):
        assert ab._lib.alora_set_option(v, b"qattn_fp16", value) == want
