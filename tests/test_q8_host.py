"""A cache held in 8 bits and eviction, on the CPU: the oracle pinned by what the definitions demand, and the argument checks
of the C calls, which return before anything is enqueued."""
import ctypes
import itertools
import math

import numpy as np
import pytest

from oracle import stepkv_oracle as O
from paper_2609_22158_gb300 import workload as wl


def _bits(rng, shape, scale=1.0):
    return wl.f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


# ------------------------------------------------------------------------------------------------ the oracle's pins
def test_e4m3_by_hand():
    assert O.e4m3_values(np.array([0, 1, 7, 8, 9, 0x38, 0x3C, 0x7E, 0x80, 0xB8])).tolist() == [
        0, 2 ** -9, 7 * 2 ** -9, 2 ** -6, 9 * 2 ** -9, 1, 1.5, 448, 0, -1]
    assert np.isnan(O.e4m3_values(np.array([0x7F, 0xFF]))).all()
    # ties to even codes: 17 lies between 16 and 18, 19 between 18 and 20; 2^-10 between 0 and 2^-9, 3 2^-10 between 2^-9 and 2^-8
    assert O.e4m3_round(np.array([17, 19, -17, 2 ** -10, 3 * 2 ** -10, 460, 1e9, -1e9])).tolist() == [
        16, 20, -16, 0, 2 ** -8, 448, 448, -448]
    assert np.isnan(O.e4m3_round(np.array([np.inf, -np.inf, np.nan]))).all()


def test_e4m3_round_is_the_nearest_of_all():
    rng = np.random.default_rng(1)
    grid = np.sort(O.e4m3_values(np.arange(127)))
    y = np.abs(rng.standard_normal(3000)) * np.exp2(rng.uniform(-12, 9, 3000))
    best = np.abs(grid[None] - y[:, None]).min(1)
    assert np.array_equal(np.abs(O.e4m3_round(y) - y), best)
    assert np.array_equal(O.e4m3_round(grid), grid)


def test_e4m3_is_torch_float8_e4m3fn():
    import torch
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(O.e4m3_values(codes.numpy()), want, equal_nan=True)


@pytest.mark.parametrize("most,k", [(448.0, 0), (448.5, 1), (447.9, 0), (224.0, -1), (224.5, 0), (1.0, -8), (0.875, -9), (0.0, -100),
                                    (2.0 ** -99, -100), (1.75 * 2.0 ** 127, 119), (3.3e38, 119)])
def test_scale_by_hand(most, k):
    assert O.q8_scale(most) == 2.0 ** k


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1.0, 1e20])
def test_written_values(scale):
    """Values fit bf16; the error is at most half a step: 2^-4 of the value, or of 2^-6 s below that; the scale is the smallest."""
    rng = np.random.default_rng(2)
    X = _bits(rng, (3, 70, 64), scale)
    v, s = O.q8_quantise(X)
    x = O.bf16_to_f64(X)
    assert np.array_equal(O.bf16_to_f64(wl.f32_to_bf16_bits(v.astype(np.float32))), v)
    rows = np.repeat(s, 32, 1)[:, :70, None]
    assert (np.abs(v - x) <= 2.0 ** -4 * np.maximum(np.abs(x), 2.0 ** -6 * rows)).all()
    for h, b in itertools.product(range(3), range(3)):
        top = np.abs(x[h, 32 * b:32 * b + 32]).max()
        assert top <= 448 * s[h, b] and top > 224 * s[h, b]
    back, s2 = O.q8_quantise(wl.f32_to_bf16_bits(v.astype(np.float32)))
    # written again: the same values (a largest value that rounds up to 448 from below keeps its scale)
    assert np.array_equal(back, v) and np.array_equal(s2, s)


@pytest.mark.parametrize("cuts", [[0, 70], [0, 1, 2, 3, 70], [0, 31, 32, 33, 64, 70], [0, 40, 70]])
def test_appending_keeps_what_is_there(cuts):
    """However rows arrive, a block's scale ends as the largest any of its pieces needed, and a value is that of all at once
    unless it was rounded twice (below 2^-6 of the scale)."""
    rng = np.random.default_rng(3)
    X = _bits(rng, (70, 64))
    X[50] = wl.f32_to_bf16_bits(O.bf16_to_f64(X[50]).astype(np.float32) * 300)
    v, s = np.zeros((70, 64)), np.zeros(3)
    for a, b in zip(cuts, cuts[1:]):
        O.q8_append(v, s, X[a:b], a)
    want, ws = O.q8_quantise(X)
    assert np.array_equal(s, ws)
    fine = np.abs(want) >= 2.0 ** -6 * np.repeat(s, 32)[:70, None]
    assert np.array_equal(v[fine], want[fine])
    assert (np.abs(v - O.bf16_to_f64(X)) <= 2.0 ** -4 * np.maximum(np.abs(O.bf16_to_f64(X)), 2.0 ** -5 * np.repeat(s, 32)[:70, None])).all()


def test_non_finite_values_are_nan_and_do_not_count():
    x = np.ones((32, 64), np.float32)
    x[3, 5], x[4, 6], x[5, 7] = np.inf, -np.inf, np.nan
    v, s = O.q8_quantise((x.view(np.uint32) >> 16).astype(np.uint16)[None])
    assert s[0, 0] == 2.0 ** -8 and np.isnan(v[0]).sum() == 3 and np.nanmax(v) == 1


def test_eviction_by_hand():
    nan = float("nan")
    #        slot  0    1    2    3    4    5    6    7
    mass = np.array([0.1, 0.9, 0.0, 0.5, 0.5, 0.2, 0.5, 0.0])
    pos = np.arange(8)
    assert O.evict_moves(mass, pos, 4, 0, 0) == ([0, 2], [4, 6])        # 1, 3, 4, 6: holes 0 and 2
    assert O.evict_moves(mass, pos, 3, 0, 0) == ([0, 2], [3, 4])        # of three equal the lower slots stay
    assert O.evict_moves(mass, pos, 4, 1, 2) == ([2, 3], [6, 7])        # 0; 6, 7 newest; then 1
    assert O.evict_moves(mass, pos[::-1], 4, 1, 2) == ([2], [7])  # 7 oldest, 0 and 1 newest; then 3 = 4 = 6: the lowest, 3
    assert O.evict_moves(mass, pos, 8, 0, 0) == ([], [])
    assert O.evict_moves(np.array([nan, -1.0, 0.0, -0.0]), pos[:4], 2, 0, 0) == ([0, 1], [2, 3])
    assert O.evict_moves(np.array([nan, nan, -np.inf, nan]), pos[:4], 2, 0, 0) == ([1], [2])
    assert O.evict_moves(np.ones(5), np.zeros(5, int), 2, 1, 1) == ([], [])  # all protected: the lower slots


# ------------------------------------------------------------------------------------------------ refusals of the C calls
@pytest.fixture(scope="module")
def lib():
    from paper_2609_22158_gb300 import binding, build
    build.build_library()
    return binding.load_library()


def _ptrs(*a):
    arr = (ctypes.c_void_p * len(a))(*a)
    return ctypes.cast(arr, ctypes.c_void_p), arr


MB = 1 << 20


class _Args:
    """Arguments that would be accepted (the pointers are never followed: every test changes one to be refused)."""

    def __init__(self, **over):
        from paper_2609_22158_gb300 import binding as B
        self.keep = []
        p = lambda k: self._arr(MB * k, MB * (k + 1))
        v = dict(n_layers=2, Hkv=2, d=128, rows=100, K=p(1), K_scale=p(3), V=p(5), V_scale=p(7), code=12800, scale=4)
        for k, x in over.items():
            if k in v:
                v[k] = self._arr(*x) if isinstance(x, tuple) else x
        self.cache = B.CQ8Cache(*v.values())
        self.x = dict(src=p(21), val=p(23), hs=12800, rs=128, T=100, idx=None, n_dev=None, n=10, row0_dev=None, rstride=0,
                      row0=0, Hq=8, nstride=0, n_cap=100, ws=1 << 28, ws_bytes=1 << 30, outs=p(25), mass=p(27), mstride=100,
                      L=2, H=2, D=128, left=50, sink=2, recent=10, pos=p(29), pstride=100, n_out=1 << 27)
        for k, x in over.items():
            if k in self.x:
                self.x[k] = self._arr(*x) if isinstance(x, tuple) else x
            else:
                assert k in v, k

    def _arr(self, *a):
        p, arr = _ptrs(*a)
        self.keep.append(arr)
        return p.value


def _write(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q8_write(ctypes.byref(a.cache), x["src"], x["val"], x["hs"], x["rs"], x["T"], x["idx"], x["n_dev"],
                               x["n"], x["row0_dev"], x["rstride"], x["row0"], None, None)


def _read(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q8_read(ctypes.byref(a.cache), x["idx"], x["n_dev"], x["n"], x["row0_dev"], x["rstride"], x["row0"],
                              x["src"], x["val"], x["hs"], x["rs"], None, None)


def _decode(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q8_decode(ctypes.byref(a.cache), x["src"], x["Hq"], x["n_dev"], x["nstride"], x["n"], x["n_cap"],
                                x["outs"], x["mass"], x["mstride"], x["ws"], x["ws_bytes"], None, None)


def _evict(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_evict(x["L"], x["src"], x["val"], x["hs"], x["H"], x["D"], x["n_dev"], x["nstride"], x["n"], x["n_cap"],
                            x["left"], x["sink"], x["recent"], x["mass"], x["mstride"], x["pos"], x["pstride"], x["n_out"],
                            x["ws"], x["ws_bytes"], None, None)


def _q8_evict(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q8_evict(ctypes.byref(a.cache), x["n_dev"], x["nstride"], x["n"], x["n_cap"], x["left"], x["sink"],
                               x["recent"], x["mass"], x["mstride"], x["pos"], x["pstride"], x["n_out"], x["ws"],
                               x["ws_bytes"], None, None)


OK, EINVAL, ENOSPACE, EUNSUPPORTED = 0, 1, 3, 4


@pytest.mark.parametrize("over,code", [
    (dict(n_layers=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(rows=0), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(d=256), EUNSUPPORTED),
    (dict(K=None), EINVAL), (dict(K_scale=None), EINVAL), (dict(V=None), EINVAL), (dict(V_scale=None), EINVAL),
    (dict(code=12799), EINVAL), (dict(code=12808), EUNSUPPORTED), (dict(scale=3), EINVAL), (dict(Hkv=65536), EUNSUPPORTED),
    (dict(rows=2 ** 30 + 1, code=2 ** 40, scale=2 ** 33), EUNSUPPORTED), (dict(K=(MB, None)), EINVAL), (dict(V_scale=(MB, None)), EINVAL),
    (dict(K=(MB, 2 * MB + 8)), EUNSUPPORTED), (dict(V=(MB + 4, 2 * MB)), EUNSUPPORTED), (dict(K_scale=(MB, 2 * MB + 2)), EUNSUPPORTED)])
def test_every_call_refuses_a_bad_cache(lib, over, code):
    for call in (_write, _read, _decode, _q8_evict):
        assert call(lib, **over) == code, call.__name__


@pytest.mark.parametrize("over,code", [
    (dict(src=None), EINVAL), (dict(val=None), EINVAL), (dict(src=(MB * 21, None)), EINVAL), (dict(val=(MB * 23, MB * 24 + 8)), EUNSUPPORTED),
    (dict(T=-1), EINVAL), (dict(n=-1), EINVAL), (dict(n=101), EINVAL), (dict(hs=-8), EINVAL), (dict(rs=-8), EINVAL),
    (dict(hs=12804), EUNSUPPORTED), (dict(rs=132), EUNSUPPORTED), (dict(n=2 ** 30 + 1, T=2 ** 31 - 1, n_dev=4096), EUNSUPPORTED),
    (dict(row0=-1), ENOSPACE), (dict(row0=91), ENOSPACE), (dict(row0=2 ** 31 - 1), ENOSPACE), (dict(row0_dev=4096, rstride=2), EINVAL),
    (dict(n=0), OK),
    (dict(K=(21 * MB, MB)), EINVAL), (dict(V=(23 * MB + 2560, MB)), EINVAL),        # the cache among the rows that are read
    (dict(K_scale=(24 * MB, 3 * MB)), EINVAL), (dict(V_scale=(MB, 8 * MB)), EINVAL),  # scales over the source, over codes
    (dict(K=(MB, MB)), EINVAL), (dict(V=(MB + 12800, 6 * MB)), EINVAL), (dict(V_scale=(3 * MB + 16, 8 * MB)), EINVAL)])
def test_write_refusals(lib, over, code):
    assert _write(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(src=None, val=None), EINVAL), (dict(src=(MB * 21, None)), EINVAL), (dict(val=(MB * 23, MB * 24 + 8)), EUNSUPPORTED),
    (dict(n=-1), EINVAL), (dict(hs=120), EINVAL), (dict(rs=120), EINVAL), (dict(rs=0), EINVAL), (dict(hs=12804), EUNSUPPORTED),
    (dict(rs=132), EUNSUPPORTED), (dict(row0=-1), EINVAL), (dict(row0=91), EINVAL), (dict(row0_dev=4096, rstride=-1), EINVAL),
    (dict(n=0), OK), (dict(n=0, src=None), OK), (dict(val=(21 * MB, 22 * MB)), EINVAL), (dict(hs=128, rs=128), EINVAL),
    (dict(src=(5 * MB, 22 * MB)), EINVAL), (dict(val=(23 * MB, 3 * MB)), EINVAL)])  # into the cache
def test_read_refusals(lib, over, code):
    assert _read(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(src=None), EINVAL), (dict(outs=None), EINVAL), (dict(ws=None), EINVAL), (dict(Hq=0), EINVAL), (dict(Hq=7), EINVAL),
    (dict(Hq=18), EUNSUPPORTED), (dict(n_cap=0), EINVAL), (dict(n_cap=101), EINVAL), (dict(n=-1), EINVAL), (dict(n=101), EINVAL),
    (dict(n_dev=4096, nstride=2), EINVAL), (dict(ws_bytes=100), ENOSPACE), (dict(ws=(1 << 28) + 16), EINVAL),
    (dict(src=(21 * MB, None)), EINVAL), (dict(src=(21 * MB, 22 * MB + 8)), EUNSUPPORTED), (dict(outs=(25 * MB + 4, 26 * MB)), EUNSUPPORTED),
    (dict(mass=(27 * MB, None)), EINVAL), (dict(mass=(27 * MB, 28 * MB + 2)), EUNSUPPORTED), (dict(mstride=99), EINVAL),
    (dict(outs=(25 * MB, 25 * MB + 4080)), EINVAL), (dict(mass=(25 * MB, 28 * MB)), EINVAL), (dict(mass=(27 * MB, 27 * MB + 400)), EINVAL)])
def test_decode_refusals(lib, over, code):
    assert _decode(lib, **over) == code


EVICT = [
    (dict(mass=None), EINVAL), (dict(pos=None), EINVAL), (dict(ws=None), EINVAL), (dict(left=0), EINVAL), (dict(left=101), EINVAL),
    (dict(sink=-1), EINVAL), (dict(recent=-1), EINVAL), (dict(sink=40, recent=11), EINVAL), (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), EINVAL),
    (dict(mstride=99), EINVAL), (dict(pstride=99), EINVAL), (dict(n=-1), EINVAL), (dict(n=101), EINVAL), (dict(n_dev=4096, nstride=-1), EINVAL),
    (dict(ws_bytes=100), ENOSPACE), (dict(ws=(1 << 28) + 128), EINVAL), (dict(mass=(27 * MB, None)), EINVAL), (dict(pos=(None, 30 * MB)), EINVAL),
    (dict(mass=(27 * MB + 2, 28 * MB)), EUNSUPPORTED), (dict(pos=(29 * MB, 30 * MB + 1)), EUNSUPPORTED), (dict(n_cap=0), EINVAL),
    (dict(mass=(29 * MB, 28 * MB)), EINVAL), (dict(pos=(29 * MB, 29 * MB + 400)), EINVAL), (dict(n_out=29 * MB + 796), EINVAL),
    (dict(n_dev=27 * MB), EINVAL), (dict(n_dev=(1 << 27) + 4, nstride=1), EINVAL)]


@pytest.mark.parametrize("over,code", EVICT)
def test_both_evictions_refuse(lib, over, code):
    assert _evict(lib, **over) == code
    assert _q8_evict(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(L=0), EINVAL), (dict(H=0), EINVAL), (dict(D=0), EINVAL), (dict(D=12), EUNSUPPORTED), (dict(D=264, hs=26400), EUNSUPPORTED),
    (dict(src=None), EINVAL), (dict(val=None), EINVAL), (dict(src=(21 * MB, None)), EINVAL), (dict(val=(23 * MB, 24 * MB + 8)), EUNSUPPORTED),
    (dict(hs=12792), EINVAL), (dict(hs=12804), EUNSUPPORTED), (dict(H=65536), EUNSUPPORTED),
    (dict(n_cap=2 ** 18 + 1, hs=2 ** 30, mstride=2 ** 30, pstride=2 ** 30), EUNSUPPORTED),
    (dict(src=(23 * MB, 22 * MB)), EINVAL), (dict(val=(27 * MB, 24 * MB)), EINVAL), (dict(n_out=21 * MB + 40), EINVAL)])
def test_evict_refusals(lib, over, code):
    assert _evict(lib, **over) == code


@pytest.mark.parametrize("over,code", [(dict(K=(5 * MB, 2 * MB)), EINVAL), (dict(K_scale=(29 * MB, 4 * MB)), EINVAL), (dict(n_cap=101), EINVAL),
                                       (dict(mass=(7 * MB, 28 * MB)), EINVAL)])
def test_q8_evict_refusals(lib, over, code):
    assert _q8_evict(lib, **over) == code


def test_workspace_sizes(lib):
    size = lib.stepkv_q8_decode_workspace_size
    for mass in (0, 1):
        assert size(32, 8, 32, 128, 8272, mass) > 0 and size(200, 8, 32, 128, 8272, mass) == size(64, 8, 32, 128, 8272, mass)
        for bad in [(0, 8, 32, 128, 10), (1, 8, 32, 96, 10), (1, 8, 32, 128, 0), (1, 8, 32, 128, 2 ** 30 + 1), (1, 8, 33, 128, 100),
                    (1, 8, 72, 128, 100), (1, 65536, 65536, 64, 10), (64, 65535, 65535, 64, 2 ** 20)]:
            assert size(*bad, mass) == 0, bad
    assert size(2, 2, 8, 64, 1000, 1) >= 4 * 2 * 8 * 1000  # every logit in 32 bits
    size = lib.stepkv_evict_workspace_size
    assert size(32, 8, 8911) > 0 and size(200, 8, 8911) == size(64, 8, 8911) and size(1, 1, 1) > 0
    for bad in [(0, 8, 10), (1, 0, 10), (1, 65536, 10), (1, 8, 0), (1, 8, 2 ** 18 + 1), (1, 1, 2 ** 31 - 1)]:
        assert size(*bad) == 0
    assert size(64, 65535, 2 ** 18) > 8 * 64 * 65535 * 2 ** 17  # a move of 8 bytes for each of n_cap / 2 rows, no count wraps


def test_header_declares_and_library_exports(lib):
    from paper_2609_22158_gb300 import binding as B
    from test_cpu_abi import HEADER
    text = open(HEADER).read()
    for name in ("stepkv_q8_write", "stepkv_q8_read", "stepkv_q8_decode", "stepkv_q8_decode_workspace_size", "stepkv_evict",
                 "stepkv_q8_evict", "stepkv_evict_workspace_size"):
        assert name + "(" in text and hasattr(lib, name) and name in B.SIGNATURES


def test_binding_refuses_host_tensors():
    import torch
    from paper_2609_22158_gb300 import binding as B
    z = torch.zeros
    f8 = torch.float8_e4m3fn
    with pytest.raises(ValueError):
        B.Q8Cache(z(1, 2, 10, 64, dtype=f8), z(1, 2, 1), z(1, 2, 10, 64, dtype=f8), z(1, 2, 1))
    with pytest.raises(TypeError):
        B.Q8Cache(z(1, 2, 10, 64), z(1, 2, 1), z(1, 2, 10, 64), z(1, 2, 1))
    with pytest.raises(ValueError):
        B.Q8Cache([], [], [], [])
    with pytest.raises(ValueError):
        B.stepkv_evict(z(1, 2, 10, 64, dtype=torch.bfloat16), z(1, 2, 10, 64, dtype=torch.bfloat16), z(1, 2, 10),
                       z(1, 2, 10, dtype=torch.int32), 10, 5)
