"""CPU-side checks of the calls on rows of a cache: every bad argument is refused on the host, before anything is launched (through a
validation-only context, device -1), the pools' tables stay as they were, and what the tests hold the kernels to is the format's definition."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

from tests import qref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000000            # stands in for device memory: never dereferenced


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


def status(ab, st):
    return ab._lib.alora_status_string(st).decode()


def test_struct_layout_matches_header(ab):
    assert C.sizeof(ab.QCacheDesc) == 80 and C.sizeof(ab.RowRange) == 24
    text = open(os.path.join(ROOT, "include", "alora.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} alora_qcache;", text).group(1)
    names = re.findall(r"\*?(\w+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    assert names == [n for n, _ in ab.QCacheDesc._fields_]


def full(ab, k=P, v=2 * P, tokens=100):
    return ab.KVCacheDesc(k, v, tokens)


def four(ab, k=3 * P, v=4 * P, ks=5 * P, vs=6 * P, tokens=100):
    return ab.QCacheDesc(k, v, ks, vs, tokens)


def ranges(ab, r):
    return (ab.RowRange * max(1, len(r)))(*[ab.RowRange(*x) for x in r])


GOOD = [(0, 50, 10)]


@pytest.mark.parametrize("r,want", [
    ([(0, 50, -1)], "ALORA_EINVAL"), ([(-1, 50, 2)], "ALORA_ECAPACITY"), ([(0, -1, 2)], "ALORA_ECAPACITY"), ([(95, 0, 6)], "ALORA_ECAPACITY"),
    ([(0, 95, 6)], "ALORA_ECAPACITY"), ([(0, 0, 101)], "ALORA_ECAPACITY"), ([(2 ** 62, 0, 2 ** 62)], "ALORA_ECAPACITY"),
    ([(0, 2 ** 63 - 1, 5)], "ALORA_ECAPACITY"), ([(0, 50, 10), (20, 59, 5)], "ALORA_EINVAL"), ([(0, 50, 10), (30, 50, 10)], "ALORA_EINVAL"),
    (GOOD, "ALORA_EHIP"), ([(0, 50, 10), (20, 60, 5)], "ALORA_EHIP"), ([], "ALORA_OK"), ([(100, 100, 0)], "ALORA_OK"), ([(101, 0, 0)], "ALORA_ECAPACITY")])
@pytest.mark.parametrize("call", ["cache_copy", "qcache_copy", "qcache_store", "qcache_load"])
def test_ranges(ab, v, call, r, want):
    rr = ranges(ab, r)
    a, b, c, d = full(ab), full(ab, 7 * P, 8 * P), four(ab), four(ab, 9 * P, 10 * P, 11 * P, 12 * P)
    lib = ab._lib
    st = {"cache_copy": lambda: lib.alora_cache_copy(v, 1, 2, 64, C.byref(b), C.byref(a), 1, rr, len(r), None),
          "qcache_copy": lambda: lib.alora_qcache_copy(v, 2, 64, C.byref(d), C.byref(c), 1, rr, len(r), None),
          "qcache_store": lambda: lib.alora_qcache_store(v, 1, 2, 64, C.byref(c), C.byref(a), 1, rr, len(r), None),
          "qcache_load": lambda: lib.alora_qcache_load(v, 1, 2, 64, C.byref(a), C.byref(c), 1, rr, len(r), None)}[call]()
    assert status(ab, st) == want
    assert (st == 0) == (lib.alora_last_error(v) == b"")


def test_rows_that_stay_are_nothing_to_do(ab, v):
    a = full(ab)
    assert ab._lib.alora_cache_copy(v, 1, 2, 64, C.byref(a), C.byref(a), 1, ranges(ab, [(5, 5, 20)]), 1, None) == ab.ALORA_OK
    # ... and still are rows that nothing else may be written to
    st = ab._lib.alora_cache_copy(v, 1, 2, 64, C.byref(a), C.byref(a), 1, ranges(ab, [(5, 5, 20), (40, 24, 2)]), 2, None)
    assert status(ab, st) == "ALORA_EINVAL"


@pytest.mark.parametrize("over,want", [
    (dict(dtype=2), "ALORA_EDTYPE"), (dict(heads=0), "ALORA_ESHAPE"), (dict(h=3), "ALORA_ESHAPE"), (dict(h=258), "ALORA_ESHAPE"), (dict(h=0), "ALORA_ESHAPE"),
    (dict(layers=0), "ALORA_EINVAL"), (dict(n=-1), "ALORA_EINVAL"), (dict(r=None), "ALORA_EINVAL"), (dict(dst=None), "ALORA_EINVAL"), (dict(src=None), "ALORA_EINVAL")])
def test_shapes_and_nulls(ab, v, over, want):
    lib, a, b, c, d = ab._lib, full(ab), full(ab, 7 * P, 8 * P), four(ab), four(ab, 9 * P, 10 * P, 11 * P, 12 * P)
    o = dict(dtype=1, heads=2, h=64, layers=1, n=1, r=ranges(ab, GOOD), dst=True, src=True)
    o.update(over)
    def ref(x, there):
        return C.byref(x) if there else None
    calls = [lambda: lib.alora_cache_copy(v, o["dtype"], o["heads"], o["h"], ref(b, o["dst"]), ref(a, o["src"]), o["layers"], o["r"], o["n"], None),
             lambda: lib.alora_qcache_store(v, o["dtype"], o["heads"], o["h"], ref(c, o["dst"]), ref(a, o["src"]), o["layers"], o["r"], o["n"], None),
             lambda: lib.alora_qcache_load(v, o["dtype"], o["heads"], o["h"], ref(a, o["dst"]), ref(c, o["src"]), o["layers"], o["r"], o["n"], None)]
    if "dtype" not in over:
        calls.append(lambda: lib.alora_qcache_copy(v, o["heads"], o["h"], ref(d, o["dst"]), ref(c, o["src"]), o["layers"], o["r"], o["n"], None))
    for call in calls:
        assert status(ab, call()) == want
    assert lib.alora_cache_copy(None, 1, 2, 64, C.byref(b), C.byref(a), 1, o["r"], 1, None) == ab.ALORA_EINVAL


def test_pools_of_a_call(ab, v):
    lib, r = ab._lib, ranges(ab, GOOD)
    def copy(dst, src, n=1):
        return status(ab, lib.alora_cache_copy(v, 1, 2, 64, dst, src, n, r, 1, None))
    row = 2 * 64 * 2
    assert copy(C.byref(full(ab, None)), C.byref(full(ab))) == "ALORA_EINVAL"
    assert copy(C.byref(full(ab, P + row)), C.byref(full(ab))) == "ALORA_EINVAL"                # overlaps, and is not the same
    assert copy(C.byref(full(ab, P + 100 * row, 7 * P)), C.byref(full(ab))) == "ALORA_EHIP"     # right behind it
    assert copy(C.byref(full(ab, P, 7 * P)), C.byref(full(ab))) == "ALORA_EINVAL"               # the same keys, other values
    assert copy(C.byref(full(ab, tokens=90)), C.byref(full(ab))) == "ALORA_EINVAL"
    two = (ab.KVCacheDesc * 2)(full(ab), full(ab, 7 * P, 8 * P, 99))
    assert copy(two, two, 2) == "ALORA_ECAPACITY"
    assert copy(C.byref(full(ab, tokens=-1)), C.byref(full(ab, 7 * P, 8 * P))) == "ALORA_ECAPACITY"
    odd = full(ab, P + 1)
    assert status(ab, lib.alora_qcache_store(v, 1, 2, 64, C.byref(four(ab)), C.byref(odd), 1, r, 1, None)) == "ALORA_EINVAL"
    for name in ("k", "v", "k_scale", "v_scale"):
        q = four(ab)
        setattr(q, name, None)
        assert status(ab, lib.alora_qcache_load(v, 1, 2, 64, C.byref(full(ab)), C.byref(q), 1, r, 1, None)) == "ALORA_EINVAL"


def table(ab, q, off=(0, 50), cap=(50, 50), length=(10, 20), poff=None, plen=None):
    keep = [np.array(off, np.int64), np.array(cap, np.int32), np.array(length, np.int32)]
    q.seq_offset, q.seq_capacity, q.seq_len = (a.ctypes.data_as(C.POINTER(t)) for a, t in zip(keep, (C.c_int64, C.c_int32, C.c_int32)))
    if plen is not None:
        keep += [np.array(poff, np.int64), np.array(plen, np.int32)]
        q.prefix_offset, q.prefix_len = keep[3].ctypes.data_as(C.POINTER(C.c_int64)), keep[4].ctypes.data_as(C.POINTER(C.c_int32))
    return keep


@pytest.mark.parametrize("over,want", [
    (dict(), "ALORA_EHIP"), (dict(cu=[0, 0, 0]), "ALORA_OK"), (dict(dtype=9), "ALORA_EDTYPE"), (dict(n_q=5), "ALORA_ESHAPE"), (dict(n_q=0), "ALORA_ESHAPE"),
    (dict(h=7), "ALORA_ESHAPE"), (dict(B=0), "ALORA_EINVAL"), (dict(cu=[1, 2, 3]), "ALORA_EINVAL"), (dict(cu=[0, 2, 1]), "ALORA_EINVAL"), (dict(cu=[2 ** 31 - 1, -2 ** 31, 3]), "ALORA_EINVAL"),
    (dict(cu=[0, 11, 12]), "ALORA_EINVAL"), (dict(length=[-1, 20]), "ALORA_EINVAL"), (dict(length=[0, 20]), "ALORA_EINVAL"),
    (dict(cu=[0, 10, 30]), "ALORA_EHIP"), (dict(off=[-1, 50]), "ALORA_ECAPACITY"), (dict(off=[0, 51]), "ALORA_ECAPACITY"), (dict(length=[51, 20]), "ALORA_ECAPACITY"),
    (dict(poff=[0, 0], plen=[0, 15], length=[10, 20]), "ALORA_EHIP"), (dict(poff=[0, 0], plen=[0, 15], cu=[0, 1, 7]), "ALORA_EINVAL"),
    (dict(poff=[0, 90], plen=[0, 15]), "ALORA_ECAPACITY"), (dict(poff=[0, 0], plen=[-1, 0]), "ALORA_EINVAL"), (dict(poff=[0, 0], plen=[0, 21]), "ALORA_EINVAL"),
    (dict(off=[0, 0]), "ALORA_EHIP"), (dict(q=None), "ALORA_EINVAL"), (dict(out=None), "ALORA_EINVAL"), (dict(q=P + 1), "ALORA_EINVAL"),
    (dict(out=P), "ALORA_EINVAL"), (dict(out=P + 2 * 3 * 256 - 16), "ALORA_EINVAL"), (dict(out=P + 2 * 3 * 256), "ALORA_EHIP")])
def test_attend(ab, v, over, want):
    o = dict(dtype=1, n_q=4, h=64, B=2, cu=[0, 1, 3], q=P, out=2 * P)
    o.update({k: x for k, x in over.items() if k in o})
    q = four(ab)
    keep = table(ab, q, **{k: x for k, x in over.items() if k not in o})
    before = keep[2].copy()
    cu = np.array(o["cu"], np.int32)
    st = ab._lib.alora_qcache_attend(v, o["dtype"], o["n_q"], 2, o["h"], C.byref(q), o["q"], cu.ctypes.data_as(C.POINTER(C.c_int32)), o["B"], o["out"], None)
    assert status(ab, st) == want
    assert np.array_equal(keep[2], before)


def test_attend_without_its_arrays(ab, v):
    q = four(ab)
    cu = np.array([0, 1], np.int32).ctypes.data_as(C.POINTER(C.c_int32))
    def call(q, cu=cu):
        return status(ab, ab._lib.alora_qcache_attend(v, 1, 4, 2, 64, q, P, cu, 1, 2 * P, None))
    assert call(C.byref(q)) == "ALORA_EINVAL"                # no table
    keep = table(ab, q)
    assert call(C.byref(q)) == "ALORA_EHIP" and call(None) == "ALORA_EINVAL" and call(C.byref(q), None) == "ALORA_EINVAL"
    q.v_scale = None
    assert call(C.byref(q)) == "ALORA_EINVAL"
    assert keep is not None


@pytest.mark.parametrize("over,want", [
    (dict(), "ALORA_EHIP"), (dict(a=[2, 0]), "ALORA_EADAPTER"), (dict(length=[50, 20]), "ALORA_ECAPACITY"), (dict(off=[0, 40]), "ALORA_ECAPACITY"),
    (dict(d=0), "ALORA_ESHAPE"), (dict(drop="k_scale"), "ALORA_EINVAL"), (dict(poff=[0, 0], plen=[0, 12]), "ALORA_ECAPACITY"), (dict(B=0), "ALORA_EINVAL")])
def test_layers(ab, v, over, want):
    s = np.ones(2, np.float32)
    desc = ab.LayerDesc(over.get("d", 64), 4, 2, 64, 8, 2, 1, 128, P, P, P, P, P, s.ctypes.data_as(C.POINTER(C.c_float)), P, 1e-5, 1e4, P, P, P, P, P)
    q = four(ab)
    keep = table(ab, q, **{k: x for k, x in over.items() if k not in ("a", "d", "drop", "B")})
    if "drop" in over:
        setattr(q, over["drop"], None)
    p = C.POINTER(C.c_int32)
    cu, k, a = (np.array(x, np.int32) for x in ([0, 1, 2], [10, 20], over.get("a", [0, -1])))
    B, lib, before = over.get("B", 2), ab._lib, keep[2].copy()
    arg = lambda x: x.ctypes.data_as(p)  # noqa: E731
    # the rows of the second sequence's prefix (0..11) are written by the first one
    for st in (lib.alora_qcache_prefill(v, C.byref(desc), C.byref(q), P, arg(cu), arg(k), arg(a), B, P, None),
               lib.alora_qcache_decode(v, C.byref(desc), C.byref(q), P, arg(k), arg(a), B, P, None),
               lib.alora_qcache_stack_prefill(v, C.byref(desc), 1, C.byref(q), P, arg(cu), arg(k), arg(a), B, P, None),
               lib.alora_qcache_stack_decode(v, C.byref(desc), 1, C.byref(q), P, arg(k), arg(a), B, P, None)):
        assert status(ab, st) == want
    assert lib.alora_qcache_decode(None, C.byref(desc), C.byref(q), P, arg(k), arg(a), B, P, None) == ab.ALORA_EINVAL
    assert lib.alora_qcache_stack_decode(v, C.byref(desc), 0, C.byref(q), P, arg(k), arg(a), B, P, None) == ab.ALORA_EINVAL
    assert lib.alora_qcache_decode(v, C.byref(desc), None, P, arg(k), arg(a), B, P, None) == ab.ALORA_EINVAL
    assert np.array_equal(keep[2], before)


def test_binding_refuses_what_does_not_fit(ab):
    t = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(AssertionError):
        ab.QCache.from_tensors(t(4, 2, 32), t(4, 2, 32), t(4, 2, 1), t(4, 2, 1))
    q = ab.QCache([4, 3], 2, 80, "cpu", guard_rows=1)
    assert q.k.shape == (10, 2, 40) and q.v_scale.shape == (10, 2, 3) and list(q.seq_offset) == [1, 6]
    k = ab.KVCache([4], 2, 64, torch.bfloat16, "cpu")
    c = ab.Context(-1)
    try:
        with pytest.raises(ValueError):
            ab.alora_qcache_store(c, q, k, GOOD, stream=FakeStream())
        with pytest.raises(ValueError):
            ab.alora_cache_copy(c, k, [k, k], GOOD, stream=FakeStream())
        with pytest.raises(ValueError):
            ab.alora_qcache_attend(c, q, torch.zeros((3, 160)), [0, 2], 2, stream=FakeStream())
        with pytest.raises(ab.AloraError):
            ab.alora_qcache_copy(c, q, q, [(0, 20, 1)], stream=FakeStream())
        # layers of another shape or type than the first, none at all
        other = ab.QCache([4, 3], 1, 80, "cpu", guard_rows=1)
        for d, s in (([q, other], [q, q]), ([q, q], [q, other]), ([], [])):
            with pytest.raises(ValueError):
                ab.alora_qcache_copy(c, d, s, [(0, 5, 1)], stream=FakeStream())
        with pytest.raises(ValueError):
            ab.alora_cache_copy(c, [k, k], [k, ab.KVCache([4], 2, 64, torch.float32, "cpu")], [(0, 2, 1)], stream=FakeStream())
        # more sequences than the table has, queries of another type, rows that are not side by side
        for n, dtype in ((3, torch.float32), (2, torch.float16)):
            with pytest.raises(ValueError):
                ab.alora_qcache_attend(c, q, torch.zeros((n, 160), dtype=dtype), list(range(n + 1)), 2, stream=FakeStream())
        with pytest.raises(AssertionError):
            ab.KVCache.from_tensors(torch.zeros(4, 2, 128)[..., :64], torch.zeros(4, 2, 128)[..., :64])
    finally:
        c.close()


def test_binding_refuses_layers_and_rows_that_do_not_fit(ab):
    layer = ab.Layer({"W_qkv": torch.zeros(4 * 64, 64)}, 2, 1, 64)
    q = ab.QCache([4, 3], 1, 64, "cpu")
    c = ab.Context(-1)

    def call(cache=q, x=torch.zeros(2, 64), k=(0, 0), a=(-1, -1), out=None):
        ab.alora_qcache_decode(c, layer, cache, x, k, a, attn_out=out, stream=FakeStream())
    try:
        for bad in (dict(cache=ab.QCache([4, 3], 2, 64, "cpu")), dict(cache=ab.QCache([4, 3], 1, 32, "cpu")), dict(cache=ab.QCache([4], 1, 64, "cpu")),
                    dict(x=torch.zeros(1, 64)), dict(x=torch.zeros(2, 32)), dict(x=torch.zeros(2, 64, dtype=torch.bfloat16)), dict(a=(-1,)),
                    dict(out=torch.zeros(2, 64)), dict(out=torch.zeros(2, 128, dtype=torch.bfloat16))):
            with pytest.raises(ValueError):
                call(**bad)
        with pytest.raises(ValueError):
            ab.alora_qcache_prefill(c, layer, q, torch.zeros(2, 64), [0, 2], (0, 0), (-1, -1), stream=FakeStream())
        with pytest.raises(ab.AloraError, match="validation-only"):
            call()
    finally:
        c.close()


class FakeStream:
    cuda_stream = 0


# ---- the tests' own definition, on values worked by hand ------------------------------------------------------------
def test_format_by_hand():
    x = np.zeros(34)
    x[:14] = [6.0, 0.25, 0.26, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 5.01, -0.2, 0.74, -0.0, 4.9]
    x[32:] = [7.0, -0.875]
    codes, exps = qref.quantise(x)
    # amax 6 = 1.5 * 2^2: E - 127 = 0;  7 = 1.75 * 2^2: not over 1.75, so 0 too, and 7 -> 6;  -0.875 -> -1 (nearer than -0.5)
    assert list(exps) == [127, 127]
    want = [6, 0, 0.5, 1, 1, -2, 2, 4, 4, 6, -0.0, 0.5, -0.0, 4]
    assert list(qref.values(codes, exps)[:14]) == want
    assert list(qref.values(codes, exps)[32:]) == [6.0, -1.0]
    assert codes[0] == 7 | (0 << 4) and codes[2] == 2 | ((8 | 4) << 4)      # element 0 low, element 1 high; -2 is code 4 with the sign
    assert list(qref.quantise(np.array([7.01, 1.0]))[1]) == [128]
    assert list(qref.quantise(np.array([np.nan, 1.0]))[1]) == [255] and list(qref.quantise(np.array([1e-45, 0.0]))[1]) == [2]
    assert list(qref.quantise(np.array([0.0, -0.0]))[1]) == [127]
    assert list(qref.quantise(np.array([3.4e38, 0.0]))[1]) == [252]


def test_attention_by_hand():
    K = np.array([[[1.0, 0.0]], [[0.0, 1.0]]])
    V = np.array([[[2.0, 0.0]], [[0.0, 4.0]]])
    out = qref.attend(np.array([[0.0, 0.0], [np.log(3.0) * np.sqrt(2.0), 0.0]]), K, V, 1, [2, 2])[0]
    assert np.allclose(out, [[1.0, 2.0], [1.5, 1.0]])
    assert np.allclose(qref.attend(np.array([[5.0, 1.0]]), K, V, 1, [1])[0], [[2.0, 0.0]])
