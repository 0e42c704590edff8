"""A cache held in 4 bits, on the CPU: the oracle's quantiser pinned by what its definition demands, and the argument
checks of the C calls, which return before anything is enqueued."""
import ctypes

import numpy as np
import pytest

from oracle import stepkv_oracle as O
from paper_2609_22158_gb300 import workload as wl


def _bits(rng, shape, scale=1.0):
    return wl.f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


# ------------------------------------------------------------------------------------------------ the oracle's pins
def test_oracle_by_hand():
    """x* = -4 (the largest magnitude): s = 4 / 8 = 0.5, codes x / 0.5 + 8 with ties to even, clamped to 15."""
    x = np.zeros(32, np.float32)
    x[:8] = [-4, 3.5, 4 - 2 ** -6, 0.25, 0.75, -0.25, -1.25, 1]
    n, s = O.q4_quantise(wl.f32_to_bf16_bits(x))
    assert s.tolist() == [0.5]
    assert n[:8].tolist() == [0, 15, 15, 8, 10, 8, 6, 10] and (n[8:] == 8).all()
    n, s = O.q4_quantise(wl.f32_to_bf16_bits(-x))  # the sign turns the scale, not the codes
    assert s.tolist() == [-0.5] and n[:8].tolist() == [0, 15, 15, 8, 10, 8, 6, 10]


def test_oracle_equal_magnitudes_take_the_positive():
    x = np.zeros(32, np.float32)
    x[3], x[9] = -2, 2
    n, s = O.q4_quantise(wl.f32_to_bf16_bits(x))
    assert s.tolist() == [-0.25] and n[9] == 0 and n[3] == 15


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 1.0, 300.0, 5000.0])
def test_oracle_properties(scale):
    """Values fit bf16; quantising them again changes nothing; the error stays within half a step, or the clamp's one and a
    quarter (the scale is rounded by at most 2^-5, so |x / s| < 8.26).  A scale below 2^-20 lies on fp16's last steps of
    2^-24 with fewer than 5 bits, so x* / s need not round to -8 there: only that values fit bf16 holds."""
    rng = np.random.default_rng(3)
    X = _bits(rng, (4000, 64), scale)
    n, s = O.q4_quantise(X)
    v = O.q4_values(n, s)
    back = wl.f32_to_bf16_bits(v.astype(np.float32))
    assert np.array_equal(O.bf16_to_f64(back), v)
    n2, s2 = O.q4_quantise(back)
    x, step = O.bf16_to_f64(X), np.abs(np.repeat(s, 32, -1))
    five, whole = step >= 2.0 ** -20, np.abs(s) >= 2.0 ** -20
    assert np.array_equal(n2[five], n[five]) and np.array_equal(s2[whole], s[whole])
    fits = five & (np.abs(x) < 7168)
    assert fits.mean() > 0.8 or scale == 1e-6
    err = np.abs(x - v)
    assert (err[fits] <= np.where(n == 15, 1.26, 0.5)[fits] * step[fits]).all()
    assert (n.reshape(4000, 2, 32).min(-1) == 0)[whole].all()


def test_oracle_limits():
    x = np.zeros((6, 32), np.float32)
    x[0, 1], x[1, 1], x[2, 1], x[3, 1], x[4, 1] = np.nan, np.inf, 3e38, 2.0 ** -30, -7168
    u = np.ascontiguousarray(x).view(np.uint32) >> 16
    n, s = O.q4_quantise(u.astype(np.uint16))
    assert np.isnan(s[0]) and np.isnan(s[1]) and (n[:2] == 8).all()
    assert s[2] == -896 and n[2, 1] == 0 and s[3] == 0 and (n[3] == 8).all() and s[4] == 896 and n[4, 1] == 0 and s[5] == 0


# ------------------------------------------------------------------------------------------------ refusals of the C calls
@pytest.fixture(scope="module")
def lib():
    from paper_2609_22158_gb300 import binding, build
    build.build_library()
    return binding.load_library()


def _ptrs(*a):
    arr = (ctypes.c_void_p * len(a))(*a)
    return ctypes.cast(arr, ctypes.c_void_p), arr


class _Args:
    """Arguments that would be accepted (the pointers are never followed: every test changes one to be refused)."""

    def __init__(self, **over):
        from paper_2609_22158_gb300 import binding as B
        base = 1 << 20
        self.keep = []
        p = lambda k: self._arr(base * k, base * (k + 1))
        v = dict(n_layers=2, Hkv=2, d=128, rows=100, K=p(1), K_scale=p(3), V=p(5), V_scale=p(7), code=6400, scale=400)
        v.update({k: x for k, x in over.items() if k in v})
        self.cache = B.CQ4Cache(*v.values())
        out = dict(v, K=p(11), K_scale=p(13), V=p(15), V_scale=p(17))
        out.update({k[4:]: x for k, x in over.items() if k.startswith("out_")})
        self.out = B.CQ4Cache(*out.values())
        self.x = dict(src=p(21), val=p(23), hs=12800, rs=128, T=100, idx=None, n_dev=None, n=10, row0_dev=None, rstride=0,
                      row0=0, Hq=8, nstride=0, n_cap=100, ws=1 << 28, ws_bytes=1 << 30, kept=1 << 27, n_kept=1 << 27, cap=50,
                      outs=p(25))
        self.x.update({k: x for k, x in over.items() if k in self.x})

    def _arr(self, *a):
        p, arr = _ptrs(*a)
        self.keep.append(arr)
        return p.value


def _write(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q4_write(ctypes.byref(a.cache), x["src"], x["val"], x["hs"], x["rs"], x["T"], x["idx"], x["n_dev"],
                               x["n"], x["row0_dev"], x["rstride"], x["row0"], None, None)


def _read(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q4_read(ctypes.byref(a.cache), x["idx"], x["n_dev"], x["n"], x["row0_dev"], x["rstride"], x["row0"],
                              x["src"], x["val"], x["hs"], x["rs"], None, None)


def _compact(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q4_compact(ctypes.byref(a.cache), x["T"], x["kept"], x["n_kept"], x["cap"], ctypes.byref(a.out), None,
                                 None, None, None, None, None)


def _decode(lib, **o):
    a = _Args(**o)
    x = a.x
    return lib.stepkv_q4_decode(ctypes.byref(a.cache), x["src"], x["Hq"], x["n_dev"], x["nstride"], x["n"], x["n_cap"],
                                x["outs"], x["ws"], x["ws_bytes"], None, None)


OK, EINVAL, ENOSPACE, EUNSUPPORTED = 0, 1, 3, 4
BAD_CACHE = [(dict(n_layers=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(rows=0), EINVAL), (dict(d=48), EUNSUPPORTED),
             (dict(d=288), EUNSUPPORTED), (dict(K=None), EINVAL), (dict(K_scale=None), EINVAL), (dict(V=None), EINVAL),
             (dict(V_scale=None), EINVAL), (dict(code=6399), EINVAL), (dict(code=6408), EUNSUPPORTED),
             (dict(scale=399), EINVAL), (dict(scale=402), EUNSUPPORTED),
             (dict(rows=2 ** 30 + 1, code=2 ** 37, scale=2 ** 33), EUNSUPPORTED), (dict(Hkv=65536), EUNSUPPORTED)]


@pytest.mark.parametrize("over,code", BAD_CACHE)
def test_every_call_refuses_a_bad_cache(lib, over, code):
    for call in (_write, _read, _compact, _decode):
        assert call(lib, **over) == code, call.__name__


def test_bad_layer_pointers(lib):
    none, off, half = _ptrs(1 << 20, None), _ptrs(1 << 20, (2 << 20) + 8), _ptrs(1 << 20, (2 << 20) + 4)
    for call in (_write, _read, _compact, _decode):
        for part, bad in (("K", off), ("K_scale", half), ("V", off), ("V_scale", half)):  # 16 bytes of codes, 8 of scales
            assert call(lib, **{part: none[0].value}) == EINVAL, (call.__name__, part)
            assert call(lib, **{part: bad[0].value}) == EUNSUPPORTED, (call.__name__, part)
    for call in (_write, _read):
        for part in ("src", "val"):
            assert call(lib, **{part: none[0].value}) == EINVAL
            assert call(lib, **{part: off[0].value}) == EUNSUPPORTED
    for part in ("src", "outs"):
        assert _decode(lib, **{part: none[0].value}) == EINVAL
        assert _decode(lib, **{part: off[0].value}) == EUNSUPPORTED


@pytest.mark.parametrize("over,code", [
    (dict(src=None), EINVAL), (dict(val=None), EINVAL), (dict(T=-1), EINVAL), (dict(n=-1), EINVAL), (dict(n=101), EINVAL),
    (dict(hs=-8), EINVAL), (dict(rs=-8), EINVAL), (dict(hs=12804), EUNSUPPORTED), (dict(rs=132), EUNSUPPORTED),
    (dict(n=2 ** 30 + 1, T=2 ** 31 - 1, n_dev=4096), EUNSUPPORTED), (dict(row0=-1), ENOSPACE), (dict(row0=91), ENOSPACE), (dict(row0=2 ** 31 - 1), ENOSPACE), (dict(row0_dev=4096, rstride=2), EINVAL),
    (dict(V=None, V_scale=None), EINVAL), (dict(n=0), OK), (dict(n=0, V=None, V_scale=None, val=None), OK)])
def test_write_refusals(lib, over, code):
    assert _write(lib, **over) == code


@pytest.mark.parametrize("over,code", [
    (dict(src=None, val=None), EINVAL), (dict(n=-1), EINVAL), (dict(hs=120), EINVAL), (dict(rs=120), EINVAL), (dict(rs=0), EINVAL),
    (dict(hs=12804), EUNSUPPORTED), (dict(rs=132), EUNSUPPORTED), (dict(row0=-1), EINVAL), (dict(row0=91), EINVAL),
    (dict(row0_dev=4096, rstride=-1), EINVAL), (dict(V=None, V_scale=None), EINVAL), (dict(n=0), OK),
    (dict(n=0, V=None, V_scale=None, val=None), OK), (dict(n=0, src=None), OK)])
def test_read_refusals(lib, over, code):
    assert _read(lib, **over) == code


def test_compact_refusals(lib):
    for over, code in [(dict(T=0), EINVAL), (dict(T=101), EINVAL), (dict(kept=None), EINVAL), (dict(n_kept=None), EINVAL),
                       (dict(cap=-1), EINVAL), (dict(cap=101), EINVAL), (dict(out_Hkv=1), EINVAL), (dict(out_n_layers=1), EINVAL),
                       (dict(out_d=64), EINVAL), (dict(out_V=None, out_V_scale=None), EINVAL), (dict(out_rows=49, out_code=6400), EINVAL)]:
        assert _compact(lib, **over) == code, over
    for part in ("K", "K_scale", "V", "V_scale"):  # a buffer of the source among the destinations
        p, keep = _ptrs(1 << 30, 1 << 31)
        assert _compact(lib, **{part: p.value, "out_" + part: p.value}) == EUNSUPPORTED, part


MB = 1 << 20


@pytest.mark.parametrize("over", [
    dict(out_K=(2 * MB, 30 * MB)),                         # layer 0 of the destination is layer 1 of the source, as
    dict(out_K_scale=(4 * MB, 30 * MB)),                   # cache.layers(0, 2) -> cache.layers(1, 3) has it
    dict(out_V=(1 * MB, 30 * MB)), dict(out_K=(30 * MB, 5 * MB)),      # keys over values, values over keys
    dict(out_K=(2 * MB - 16, 30 * MB)), dict(out_V=(6 * MB + 6400 + 2480, 30 * MB)),  # a few rows of a head
    dict(out_K_scale=(1 * MB + 64, 30 * MB)),              # scales over codes
    dict(out_K=(30 * MB, 30 * MB)), dict(out_K=(30 * MB, 31 * MB), out_V=(32 * MB, 31 * MB + 6400)),  # the same row written twice
    dict(step_in=40 * MB, step_out=40 * MB), dict(step_in=40 * MB, step_out=40 * MB + 396), dict(pos_in=40 * MB, step_out=40 * MB),
    dict(step_out=40 * MB, pos_out=40 * MB + 196), dict(pos_out=1 << 27), dict(step_out=7 * MB)])
def test_compact_refuses_destinations_that_meet_the_source(lib, over):
    """Rows move in one launch in no order: a destination that is a source as well would be read half written."""
    keep = [_ptrs(*v) for k, v in over.items() if isinstance(v, tuple)]
    caches = dict(zip((k for k, v in over.items() if isinstance(v, tuple)), (p.value for p, _ in keep)))
    a = _Args(**caches)
    x = a.x
    got = lib.stepkv_q4_compact(ctypes.byref(a.cache), x["T"], x["kept"], x["n_kept"], x["cap"], ctypes.byref(a.out),
                                over.get("step_in"), over.get("pos_in"), over.get("step_out"), over.get("pos_out"), None, None)
    assert got == EUNSUPPORTED


@pytest.mark.parametrize("call,over", [
    (_write, dict(V=(1 * MB, 2 * MB))), (_write, dict(K=(30 * MB, 30 * MB))), (_write, dict(K=(30 * MB, 30 * MB + 2 * 6400 - 16))),
    (_write, dict(V=(30 * MB, 1 * MB + 6400))), (_write, dict(V_scale=(1 * MB, 8 * MB))), (_write, dict(V_scale=(3 * MB + 1592, 8 * MB))),
    (_read, dict(val=(21 * MB, 22 * MB))),                            # keys and values to one buffer
    (_read, dict(val=(30 * MB, 22 * MB))), (_read, dict(src=(30 * MB, 30 * MB))),   # a layer's twice
    (_read, dict(src=(30 * MB, 30 * MB + 25600 + 2304))),             # the second head of layer 0
    (_read, dict(hs=128, rs=128)), (_read, dict(hs=128 * 9)), (_read, dict(hs=128, rs=136)),  # heads that overlap
    (_decode, dict(outs=(30 * MB, 30 * MB))), (_decode, dict(outs=(30 * MB, 30 * MB + 4080)))])
def test_destinations_that_overlap_are_refused(lib, call, over):
    """Two warps would write the same bytes in no order."""
    keep = {k: _ptrs(*v) for k, v in over.items() if isinstance(v, tuple)}
    assert call(lib, **{k: keep[k][0].value if k in keep else v for k, v in over.items()}) == EINVAL


@pytest.mark.parametrize("over,code", [
    (dict(src=None), EINVAL), (dict(outs=None), EINVAL), (dict(ws=None), EINVAL), (dict(Hq=0), EINVAL), (dict(Hq=7), EINVAL),
    (dict(Hq=18), EUNSUPPORTED), (dict(d=96, code=6400, scale=402), EUNSUPPORTED), (dict(n_cap=0), EINVAL), (dict(n_cap=101), EINVAL),
    (dict(n=-1), EINVAL), (dict(n=101), EINVAL), (dict(n_dev=4096, nstride=2), EINVAL), (dict(V=None, V_scale=None), EINVAL),
    (dict(ws_bytes=100), ENOSPACE), (dict(ws=(1 << 28) + 16), EINVAL)])
def test_decode_refusals(lib, over, code):
    assert _decode(lib, **over) == code


def test_workspace_size(lib):
    size = lib.stepkv_q4_decode_workspace_size
    assert size(32, 8, 32, 128, 8272) > 0 and size(0, 8, 32, 128, 8272) == 0 and size(1, 8, 32, 96, 10) == 0
    assert size(1, 8, 32, 128, 0) == 0 and size(200, 8, 32, 128, 8272) == size(64, 8, 32, 128, 8272)  # 64 layers a launch


@pytest.mark.parametrize("shape", [
    (1, 8, 32, 128, 2 ** 31 - 1), (1, 8, 32, 128, 2 ** 31 - 32), (1, 8, 32, 128, 2 ** 30 + 1), (1, 1, 1, 64, -1),  # capacities
    (1, 8, 33, 128, 100), (1, 8, 72, 128, 100), (1, 3, 8, 64, 100), (1, 65536, 65536, 64, 10),                 # heads
    (64, 65535, 65535, 64, 2 ** 20)])                                                                       # blocks of a launch
def test_workspace_size_of_what_is_refused(lib, shape):
    """0 for what the decode does not take, and no count wraps."""
    assert lib.stepkv_q4_decode_workspace_size(*shape) == 0


def test_workspace_size_of_the_largest_caches(lib):
    """A partial state is d + 4 floats for each head, group of warps (4096 at most) and pair."""
    assert lib.stepkv_q4_decode_workspace_size(1, 1, 8, 128, 2 ** 30) == (4096 + 1) * 8 * 132 * 4
    assert lib.stepkv_q4_decode_workspace_size(1, 2, 2, 64, 32) == 4 * 68 * 4


def test_header_declares_and_library_exports(lib):
    from paper_2609_22158_gb300 import binding as B
    from test_cpu_abi import HEADER
    text = open(HEADER).read()
    for name in ("stepkv_q4_write", "stepkv_q4_read", "stepkv_q4_compact", "stepkv_q4_decode", "stepkv_q4_decode_workspace_size"):
        assert name + "(" in text and hasattr(lib, name) and name in B.SIGNATURES


def test_binding_refuses_host_tensors():
    import torch
    from paper_2609_22158_gb300 import binding as B
    z = torch.zeros
    with pytest.raises(ValueError):
        B.Q4Cache(z(1, 2, 10, 64, dtype=torch.uint8), z(1, 2, 10, 4, dtype=torch.float16))
    with pytest.raises(TypeError):
        B.Q4Cache(z(1, 2, 10, 64), z(1, 2, 10, 4, dtype=torch.float16))
    with pytest.raises(ValueError):
        B.Q4Cache([], [])
