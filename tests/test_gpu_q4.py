"""GPU parity of a cache held in 4 bits against the oracle, through the public entry points.

Writing, reading back and compaction have one right answer and are compared bit for bit.  Decode attention is compared
with the oracle's over the values the codes stand for, element by element, within a bound on what 32-bit arithmetic
may lose (_decode_bound).
"""
import math

import numpy as np
import pytest

from oracle import stepkv_oracle as O
from paper_2609_22158_gb300 import workload as wl
import stepkv_testlib as TL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    from paper_2609_22158_gb300 import binding, build
    build.build_library()
    binding.load_library()
    return binding


def _bits(rng, shape, scale=1.0):
    return wl.f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


def _keys(rng, shape):
    """Keys with four channels of a head scaled by 8."""
    x = rng.standard_normal(shape)
    x[..., rng.permutation(shape[-1])[:4]] *= 8
    return wl.f32_to_bf16_bits(x.astype(np.float32))


def _pack(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def _packed(X):
    """(codes as the cache holds them, fp16 scales) of bf16 bits X, by the oracle."""
    n, s = O.q4_quantise(X)
    return _pack(n), s.astype(np.float16)


def _back_bits(X):
    """bf16 bits of the values that X's codes stand for."""
    v = O.q4_values(*O.q4_quantise(X)).astype(np.float32)
    return np.where(np.isnan(v), np.uint16(0x7FFF), wl.f32_to_bf16_bits(np.nan_to_num(v)))


def _same_bits(got, want):
    """bf16 device tensor against bits; any NaN equals any NaN, and -0 equals 0."""
    g, w = O.bf16_to_f64(TL.bits_of(got.contiguous())), O.bf16_to_f64(want)
    np.testing.assert_array_equal(g, w)


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _filled(B, K, V=None):
    """A cache with the oracle's codes of per-layer bf16 bits K, V [Hkv, rows, d]."""
    parts = []
    for X in (K, V):
        if X is not None:
            c, s = zip(*(_packed(x) for x in X))
            parts += [_dev(np.stack(c)), _dev(np.stack(s))]
    return B.Q4Cache(*parts)


def _stale(cache, rng):
    """Fills a cache with arbitrary codes and NaN scales: rows that a call must leave alone or not use."""
    import torch
    for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        if x is not None:
            x.copy_(torch.from_numpy(rng.integers(0, 256, tuple(x.shape), dtype=np.uint8)))
            s.fill_(float("nan"))
    return [None if x is None else x.clone() for x in (cache.K, cache.K_scale, cache.V, cache.V_scale)]


def _layout(x, kind):
    """Device tensors [L, Hkv, T, d] with the same values: heads in front, tokens in front, or rows with a gap."""
    import torch
    t = torch.stack([TL.bf16_dev(b) for b in x])
    if kind == "tokens":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if kind == "gaps":
        wide = torch.full((*t.shape[:2], t.shape[2] + 3, t.shape[3] + 8), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, :, :t.shape[2], :t.shape[3]] = t
        return wide[:, :, :t.shape[2], :t.shape[3]]
    return t


# ------------------------------------------------------------------------------------------------ write and read back
WRITE_CASES = [  # L, Hkv, d, T, row0, rows, layout, values
    (1, 1, 32, 1, 0, 1, "heads", True), (2, 2, 64, 5, 3, 11, "heads", True), (3, 2, 128, 33, 1, 40, "tokens", True),
    (2, 3, 96, 17, 0, 17, "gaps", True), (1, 2, 256, 9, 2, 12, "tokens", True), (2, 1, 128, 200, 7, 301, "gaps", False),
    (32, 8, 128, 1, 50, 60, "tokens", True), (70, 1, 64, 3, 1, 6, "heads", True), (1, 5, 160, 31, 0, 31, "heads", True),
    (1, 2, 64, 1000, 0, 1000, "heads", True), (2, 1, 224, 10, 1, 13, "gaps", False),
]


@pytest.mark.parametrize("L,Hkv,d,T,row0,rows,kind,values", WRITE_CASES)
def test_write_and_read_match_oracle(B, L, Hkv, d, T, row0, rows, kind, values):
    import torch
    rng = np.random.default_rng(T + d + L)
    K, V = [_keys(rng, (Hkv, T, d)) for _ in range(L)], [_bits(rng, (Hkv, T, d)) for _ in range(L)]
    cache = B.Q4Cache.allocate(L, Hkv, rows, d, values=values)
    was = _stale(cache, rng)
    Kd, Vd = _layout(K, kind), _layout(V, kind) if values else None
    st = B.stepkv_q4_write(cache, Kd, Vd, row0)
    Kb, Vb = B.stepkv_q4_read(cache, row0, T, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for X, codes, scales, back, old in ((K, cache.K, cache.K_scale, Kb, was[:2]), (V, cache.V, cache.V_scale, Vb, was[2:])):
        if codes is None:
            assert back is None
            continue
        want_c, want_s = (np.stack(w) for w in zip(*(_packed(x) for x in X)))
        np.testing.assert_array_equal(codes[:, :, row0:row0 + T].cpu().numpy(), want_c)
        np.testing.assert_array_equal(scales[:, :, row0:row0 + T].cpu().numpy(), want_s)
        for at in (slice(0, row0), slice(row0 + T, rows)):  # the other rows, bit for bit
            assert torch.equal(codes[:, :, at], old[0][:, :, at])
            assert torch.equal(scales[:, :, at].view(torch.int16), old[1][:, :, at].view(torch.int16))
        _same_bits(back, np.stack([_back_bits(x) for x in X]))


def _special_groups():
    """Groups of 32 that a quantiser can get wrong: ties of codes at every scale, both signs of the largest value, zeros,
    saturated and vanishing groups, non-finite values, bf16's own smallest numbers."""
    rng = np.random.default_rng(11)
    out = []
    for e in list(range(-26, 14)):                     # ties: every half step of a scale m 2^e of 5 bits
        for m in (16, 19, 27, 31):
            s = m * 2.0 ** (e - 4)
            x = np.zeros(32)
            x[0] = -8 * s * rng.choice([-1, 1])
            x[1:17] = (np.arange(16) - 8 + 0.5) * s    # at most 5 + 5 significant bits: those bf16 holds are exact ties
            x[17:] = rng.uniform(-8, 8, 15) * s
            out.append(x)
    for e in range(-45, 20):                           # any magnitude
        out.append(rng.standard_normal(32) * 2.0 ** e)
    for v in (0.0, -0.0, 7168, -7168, 7169, 1e5, -3e38, 2.0 ** -22, 2.0 ** -21, -2.0 ** -126, 2.0 ** -133):
        x = np.zeros(32)
        x[rng.integers(32)] = v
        out.append(x)
        x = np.full(32, v)
        x[::2] *= -1
        out.append(x)
    for v in (np.nan, np.inf, -np.inf):
        for k in (0, 7, 31):
            x = rng.standard_normal(32)
            x[k] = v
            out.append(x)
    x = rng.standard_normal(32)
    x[3], x[30] = np.inf, np.nan
    out.append(x)
    x = np.stack(out).astype(np.float32)
    nan = np.isnan(x)
    bits = wl.f32_to_bf16_bits(np.nan_to_num(x, nan=0.0, posinf=np.inf, neginf=-np.inf))
    return np.where(nan, np.uint16(0x7FC0), bits).astype(np.uint16)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_special_values(B, d):
    import torch
    g = _special_groups()
    g = np.concatenate([g, g[: -len(g) % (d // 32) or None]])[: len(g) // (d // 32) * (d // 32)]
    X = g.reshape(1, -1, d)
    cache = B.Q4Cache.allocate(1, 1, X.shape[1], d)
    st = B.stepkv_q4_write(cache, [TL.bf16_dev(X)], [TL.bf16_dev(X)], 0)
    Kb, Vb = B.stepkv_q4_read(cache, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    want_c, want_s = _packed(X)
    np.testing.assert_array_equal(cache.K_scale[0].cpu().numpy(), want_s)
    np.testing.assert_array_equal(cache.K[0].cpu().numpy(), want_c)
    assert torch.equal(cache.K, cache.V)
    _same_bits(Kb[0], _back_bits(X))
    _same_bits(Vb[0], _back_bits(X))


def test_quantising_what_was_read_changes_nothing(B):
    import torch
    rng = np.random.default_rng(4)
    cache, again = B.Q4Cache.allocate(2, 2, 90, 128), B.Q4Cache.allocate(2, 2, 90, 128)
    X = [_keys(rng, (2, 90, 128)) for _ in range(4)]
    B.stepkv_q4_write(cache, [TL.bf16_dev(x) for x in X[:2]], [TL.bf16_dev(x) for x in X[2:]], 0)
    B.stepkv_q4_write(again, *B.stepkv_q4_read(cache), 0)
    torch.cuda.synchronize()
    for name in ("K", "K_scale", "V", "V_scale"):
        assert torch.equal(getattr(cache, name), getattr(again, name)), name


@pytest.mark.parametrize("d", [64, 128])
def test_write_by_index_and_counts_on_the_device(B, d):
    """An index list with repeats and in any order; counts and first rows read on the device, one row0 per layer."""
    import torch
    rng = np.random.default_rng(d)
    L, Hkv, T, rows = 3, 2, 50, 64
    K, V = [_bits(rng, (Hkv, T, d)) for _ in range(L)], [_bits(rng, (Hkv, T, d)) for _ in range(L)]
    idx = np.array([49, 0, 7, 7, 7, 31, 2, 48, 1, 1, 30], np.int32)
    row0, n = [5, 0, 64 - 9], 9
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    was = _stale(cache, rng)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    st = B.stepkv_q4_write(cache, [TL.bf16_dev(x) for x in K], [TL.bf16_dev(x) for x in V], i32(row0), n=i32([n]), idx=_dev(idx))
    Kb, _ = B.stepkv_q4_read(cache, i32(row0), i32([n]), status=st, K=torch.zeros((L, Hkv, n + 2, d), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert st.item() == 0
    for l in range(L):
        c, s = _packed(K[l][:, idx[:n]])
        at = slice(row0[l], row0[l] + n)
        np.testing.assert_array_equal(cache.K[l, :, at].cpu().numpy(), c)
        np.testing.assert_array_equal(cache.K_scale[l, :, at].cpu().numpy(), s)
        rest = np.ones(rows, bool)
        rest[at] = False
        assert torch.equal(cache.V[l][:, rest], was[2][l][:, rest])
        _same_bits(Kb[l][:, :n], _back_bits(K[l][:, idx[:n]]))
        assert not Kb[l][:, n:].any()


@pytest.mark.parametrize("kind", ["count above", "count below", "row0 above", "row0 below", "index"])
def test_write_bad_data(B, kind):
    """What is bad is found on the device, told in the status word, and skipped: nothing else is touched."""
    import torch
    rng = np.random.default_rng(5)
    L, Hkv, d, T, rows = 2, 2, 64, 20, 30
    K = [_bits(rng, (Hkv, T, d)) for _ in range(L)]
    Kd = [TL.bf16_dev(x) for x in K]
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    was = _stale(cache, rng)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    n, row0, idx, want = i32(4), i32(3, 9), i32(0, 1, 2, 3), None
    touched = {0: (3, 7), 1: (9, 13)}
    if kind == "count above":
        n, want, touched = i32(5), B.STEPKV_ENOSPACE, {}
    elif kind == "count below":
        n, want, touched = i32(-1), B.STEPKV_EDATA, {}
    elif kind == "row0 above":
        row0, want = i32(27, 9), B.STEPKV_ENOSPACE
        del touched[0]
    elif kind == "row0 below":
        row0, want = i32(3, -1), B.STEPKV_ENOSPACE
        del touched[1]
    else:
        idx, want = i32(0, T, -1, 3), B.STEPKV_EDATA
    st = B.stepkv_q4_write(cache, Kd, Kd, row0, n=n, idx=idx)
    torch.cuda.synchronize()
    assert st.item() == want
    left = torch.ones((L, rows), dtype=torch.bool, device="cuda")
    for l, (lo, hi) in touched.items():
        rows_ok = [0, 3] if kind == "index" else range(4)
        for r in rows_ok:
            left[l, lo + r] = False
            np.testing.assert_array_equal(cache.K[l, :, lo + r].cpu().numpy(), _packed(K[l][:, r])[0])
    for l in range(L):
        for now, old in ((cache.K, was[0]), (cache.V, was[2])):
            assert torch.equal(now[l][:, left[l]], old[l][:, left[l]])
        assert cache.K_scale[l][:, left[l]].isnan().all() and not cache.K_scale[l][:, ~left[l]].isnan().any()


@pytest.mark.parametrize("kind", ["count above", "count below", "row0 above", "row0 below", "index"])
def test_read_bad_data(B, kind):
    import torch
    rng = np.random.default_rng(6)
    L, Hkv, d, rows = 2, 2, 128, 30
    K = [_bits(rng, (Hkv, rows, d)) for _ in range(L)]
    cache = _filled(B, K)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out = torch.full((L, Hkv, 4, d), 7.0, dtype=torch.bfloat16, device="cuda")
    n, row0, idx, want, good = i32(4), i32(3, 9), None, B.STEPKV_EDATA, {0: (3, range(4)), 1: (9, range(4))}
    if kind == "count above":
        n, want, good = i32(5), B.STEPKV_ENOSPACE, {}
    elif kind == "count below":
        n, good = i32(-1), {}
    elif kind == "row0 above":
        row0 = i32(27, 9)
        del good[0]
    elif kind == "row0 below":
        row0 = i32(3, -1)
        del good[1]
    else:
        idx, good = i32(0, rows, -1, 3), {0: (0, [0, 3]), 1: (0, [0, 3])}
    st = B.new_status()
    B.stepkv_q4_read(cache, row0, n, idx=idx, K=out, status=st)
    torch.cuda.synchronize()
    assert st.item() == want
    for l in range(L):
        lo, ok = good.get(l, (0, []))
        for r in range(4):
            if r in ok:
                _same_bits(out[l, :, r], _back_bits(K[l][:, lo + r]))
            else:
                assert (out[l, :, r] == 7).all()


def test_empty_writes_and_reads(B):
    import torch
    rng = np.random.default_rng(7)
    cache = B.Q4Cache.allocate(2, 2, 10, 64)
    was = _stale(cache, rng)
    X = torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    st = B.new_status()
    B.stepkv_q4_write(cache, X, X, 10, n=0, status=st)
    B.stepkv_q4_write(cache, X, X, 10, n=zero, status=st)
    B.stepkv_q4_write(cache, X[:, :, :0], X[:, :, :0], 3, status=st)
    B.stepkv_q4_write(cache, X, X, 3, idx=zero[:0], status=st)
    out = torch.full((2, 2, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.stepkv_q4_read(cache, 10, 0, K=out, status=st)
    B.stepkv_q4_read(cache, 10, zero, K=out, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and (out == 7).all()
    assert torch.equal(cache.K, was[0]) and torch.equal(cache.V, was[2])


def test_device_counts_over_no_rows(B):
    """A limit of no rows, as an empty index list or an empty block of tokens has it: a count of 0 on the device does nothing, any
    other is told."""
    import torch
    cache = B.Q4Cache.allocate(2, 2, 10, 64)
    X, idx = torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    out = torch.zeros((2, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    for n, want in ((0, 0), (3, B.STEPKV_ENOSPACE), (-1, B.STEPKV_EDATA)):
        count = torch.tensor([n], dtype=torch.int32, device="cuda")
        for call in (lambda st: B.stepkv_q4_write(cache, X, X, 0, n=count, idx=idx, status=st),
                     lambda st: B.stepkv_q4_write(cache, X[:, :, :0], X[:, :, :0], 4, n=count, status=st),
                     lambda st: B.stepkv_q4_read(cache, 0, count, K=out, status=st),
                     lambda st: B.stepkv_q4_read(cache, idx=idx, n=count, status=st)):
            st = B.new_status()
            call(st)
            torch.cuda.synchronize()
            assert st.item() == want
    assert not cache.K.any() and not cache.V.any()


def test_read_by_index_of_values_alone(B):
    import torch
    rng = np.random.default_rng(8)
    V = [_bits(rng, (3, 40, 128)) for _ in range(2)]
    cache = _filled(B, [_bits(rng, (3, 40, 128)) for _ in range(2)], V)
    idx = torch.tensor([39, 0, 5, 5, 22], dtype=torch.int32, device="cuda")
    out = _layout([np.zeros((3, 5, 128), np.uint16)] * 2, "tokens")
    B.stepkv_q4_read(cache, idx=idx, V=out)
    torch.cuda.synchronize()
    _same_bits(out, np.stack([_back_bits(v)[:, idx.cpu().numpy()] for v in V]))


# ------------------------------------------------------------------------------------------------ compaction
@pytest.mark.parametrize("order", ["lhnd", "nlhd", "hlnd", "hnld", "lnhd", "nhld"])
def test_read_into_any_order_of_axes(B, order):
    """Rows of all layers, keys and values in one buffer whose axes come in any order: nothing shares memory, so each is read
    into; a layer, a tensor or a head laid over another is refused."""
    import torch
    rng = np.random.default_rng(16)
    size = dict(l=3, h=2, n=7, d=64)
    K, V = [_bits(rng, (2, 7, 64)) for _ in range(3)], [_bits(rng, (2, 7, 64)) for _ in range(3)]
    cache, st = _filled(B, K, V), B.new_status()
    for front in (True, False):  # keys and values apart, or side by side inside each row's place
        shape = [size[a] for a in order[:3]]
        x = torch.full([2, *shape, 64] if front else [*shape, 2, 64], 7.0, dtype=torch.bfloat16, device="cuda")
        kv = x.unbind(0 if front else 3)
        Kb, Vb = (t.permute([order.index(a) for a in "lhnd"]) for t in kv)
        B.stepkv_q4_read(cache, K=Kb, V=Vb, status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
        _same_bits(Kb, np.stack([_back_bits(k) for k in K]))
        _same_bits(Vb, np.stack([_back_bits(v) for v in V]))
    one = torch.zeros((1, 2, 7, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: B.stepkv_q4_read(cache, K=Kb, V=Kb), lambda: B.stepkv_q4_read(cache, K=one.expand(3, -1, -1, -1)),
                lambda: B.stepkv_q4_read(cache, K=one.view(-1).as_strided((3, 2, 7, 64), (0, 64, 64, 1))),
                lambda: B.stepkv_q4_decode(torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda"), cache, 5,
                                           out=torch.zeros((1, 4, 64), device="cuda").expand(3, -1, -1)),
                lambda: B.stepkv_q4_write(B.Q4Cache(*(t[:1].expand(3, -1, -1, -1) for t in (cache.K, cache.K_scale, cache.V, cache.V_scale))),
                                          Kb, Vb, 0),
                lambda: B.stepkv_q4_write(B.Q4Cache(cache.K, cache.K_scale, cache.K, cache.V_scale), Kb, Vb, 0)):
        with pytest.raises(B.StepKVError):
            bad()
    shared = B.Q4Cache(*(t[:1].expand(3, -1, -1, -1) for t in (cache.K, cache.K_scale, cache.V, cache.V_scale)))
    q = _bits(rng, (4, 64))
    out = B.stepkv_q4_decode(TL.bf16_dev(q).expand(3, -1, -1), shared, 7, status=st)  # reading one cache for all is not refused
    torch.cuda.synchronize()
    for l in range(3):
        _check(out[l], q, K[0], V[0], 7, f"cache {l}")


@pytest.mark.parametrize("L,Hkv,d,T,n,values", [(1, 2, 64, 50, 13, True), (3, 2, 128, 100, 100, True), (2, 1, 32, 9, 1, True),
                                                 (2, 3, 96, 40, 39, False), (70, 2, 128, 20, 7, True), (1, 2, 256, 33, 5, True),
                                                 (2, 2, 160, 33, 20, True), (4, 8, 128, 3000, 2001, True)])
def test_compact_moves_rows_as_they_are(B, L, Hkv, d, T, n, values):
    import torch
    rng = np.random.default_rng(T + n)
    src, dst = B.Q4Cache.allocate(L, Hkv, T + 2, d, values=values), B.Q4Cache.allocate(L, Hkv, n + 5, d, values=values)
    for x in (src.K, src.V):
        if x is not None:
            x.copy_(_dev(rng.integers(0, 256, tuple(x.shape), dtype=np.uint8)))
    for s in (src.K_scale, src.V_scale):
        if s is not None:  # any bits at all: NaN payloads too
            s.copy_(_dev(rng.integers(-2 ** 15, 2 ** 15, tuple(s.shape), dtype=np.int16)).view(torch.float16))
    was = _stale(dst, rng)
    idx = np.sort(rng.permutation(T)[:n]).astype(np.int32)
    kept = _dev(np.concatenate([idx, np.full(3, -1, np.int32)]))
    step, pos = (_dev(rng.integers(0, 1000, T).astype(np.int32)) for _ in "sp")
    outs = [torch.full((n + 3,), -7, dtype=torch.int32, device="cuda") for _ in "sp"]
    st = B.stepkv_q4_compact(src, T, kept, torch.tensor([n], dtype=torch.int32, device="cuda"), n + 3, dst, step, pos, *outs)
    torch.cuda.synchronize()
    assert st.item() == 0
    at = _dev(idx).long()
    for a, b, old in zip((src.K, src.K_scale, src.V, src.V_scale), (dst.K, dst.K_scale, dst.V, dst.V_scale), was):
        if a is not None:
            bits = lambda t: t.view(torch.int16) if t.dtype == torch.float16 else t
            assert torch.equal(bits(b)[:, :, :n], bits(a)[:, :, at])
            assert torch.equal(bits(b)[:, :, n:], bits(old)[:, :, n:])
    assert torch.equal(outs[0][:n], step[at]) and torch.equal(outs[1][:n], pos[at])
    assert (outs[0][n:] == -7).all() and (outs[1][n:] == -7).all()


def test_compact_bad_data(B):
    import torch
    rng = np.random.default_rng(9)
    src, dst = _filled(B, [_bits(rng, (2, 20, 64))], [_bits(rng, (2, 20, 64))]), B.Q4Cache.allocate(1, 2, 8, 64)
    was = _stale(dst, rng)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    kept = i32(0, 20, -1, 19, 4, 5, 6, 7)
    for n in (9, -1):
        st = B.stepkv_q4_compact(src, 20, kept, i32(n), 8, dst)
        torch.cuda.synchronize()
        assert st.item() == B.STEPKV_ENOSPACE and torch.equal(dst.K, was[0])
    st = B.stepkv_q4_compact(src, 20, kept, i32(0), 8, dst)
    torch.cuda.synchronize()
    assert st.item() == 0 and torch.equal(dst.K, was[0])
    step, pos = (torch.full((8,), -7, dtype=torch.int32, device="cuda") for _ in "sp")
    st = B.stepkv_q4_compact(src, 20, kept, i32(4), 8, dst, step_id_out=step, pos_out=pos)
    torch.cuda.synchronize()
    assert st.item() == B.STEPKV_EDATA
    assert torch.equal(dst.K[:, :, [0, 3]], src.K[:, :, [0, 19]]) and torch.equal(dst.K[:, :, [1, 2, 4]], was[0][:, :, [1, 2, 4]])
    assert pos.tolist() == [0, -1, -1, 19, -7, -7, -7, -7] and step.tolist() == [-1] * 4 + [-7] * 4


@pytest.mark.parametrize("kind", ["rows of one buffer", "layers inside heads", "the next layers"])
def test_compact_between_views_of_one_buffer(B, kind):
    """Source and destination lie inside one another's strides without sharing a row."""
    import torch
    rng = np.random.default_rng(15)
    L, Hkv, d, T, n = 3, 2, 128, 40, 17
    idx = np.sort(rng.permutation(T)[:n]).astype(np.int32)

    def views(w, t):
        if kind == "rows of one buffer":      # [layer][head][row]: the first T rows, and those behind
            x = torch.zeros((L, Hkv, T + n, w), dtype=t, device="cuda")
            return x[:, :, :T], x[:, :, T:]
        if kind == "layers inside heads":     # [head][source, destination][layer][row]
            x = torch.zeros((Hkv, 2, L, T, w), dtype=t, device="cuda").transpose(0, 2)
            return x[:, 0], x[:, 1]
        x = torch.zeros((2 * L, Hkv, T, w), dtype=t, device="cuda")
        return x[:L], x[L:]

    parts = [views(64, torch.uint8), views(4, torch.float16), views(64, torch.uint8), views(4, torch.float16)]
    src, dst = (B.Q4Cache(*[p[i] for p in parts]) for i in range(2))
    for x in (src.K, src.V):
        x.copy_(_dev(rng.integers(0, 256, tuple(x.shape), dtype=np.uint8)))
    for x in (src.K_scale, src.V_scale):
        x.copy_(_dev(rng.standard_normal(tuple(x.shape)).astype(np.float16)))
    st = B.stepkv_q4_compact(src, T, _dev(idx), torch.tensor([n], dtype=torch.int32, device="cuda"), n, dst)
    torch.cuda.synchronize()
    assert st.item() == 0
    for a, b in parts:
        assert torch.equal(b[:, :, :n], a[:, :, _dev(idx).long()])


def test_compact_refuses_the_same_layers_moved_by_one(B):
    import torch
    cache = B.Q4Cache.allocate(3, 2, 20, 64)
    kept, n = torch.zeros(20, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    for src, dst in ((cache.layers(0, 2), cache.layers(1, 3)), (cache.layers(1, 3), cache.layers(0, 2)),
                     (cache.layers(0, 1), B.Q4Cache(cache.V[:1], cache.V_scale[:1], cache.K[1:2], cache.K_scale[:1]))):
        with pytest.raises(B.StepKVError):
            B.stepkv_q4_compact(src, 20, kept, n, 20, dst)
    B.stepkv_q4_compact(cache.layers(0, 1), 20, kept, n, 20, cache.layers(2, 3))  # another layer: no row in common
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ decode attention
def _decode_bound(q, K, V):
    """Per head and channel: what fp32 arithmetic may lose of out = sum_j p_j V_j / sum_j p_j.

    A logit is a sum of d products; held to 22 bits of the largest query element, and summed in fp32 in up to d / 8 steps of
    half an ulp each, it is off by at most 2^-22 scale (max|q| sum|k| + sum|q||k|) =: e (the steps' part alone would be
    d / 8 2^-24 <= 2^-20 of sum|q||k| in the worst order, of which rounding to nearest leaves less than a quarter: 2^-22).
    exp of it is off by e and by 2^-20 (an exponential of 2^-22, a weight in 22 bits, the rescalings of the maximum), and a
    weighted sum of n terms in blocks of at least 16 by (n / 16 + 64) 2^-24.  Numerator and denominator: twice that, of
    sum_j p_j |V_j|.  And a weight is a fixed-point number besides: held in two fp16 of 11 bits, the largest as 2^14, its last
    place is 2^-24 2^-14 of the largest, so that each key may be off by 2^-38 |V_j| however small its weight (a weight that
    underflows altogether is far below)."""
    G, scale = q.shape[0] // K.shape[0], 1 / math.sqrt(q.shape[1])
    qf = O.bf16_to_f64(q)
    out = np.zeros(qf.shape)
    for g in range(qf.shape[0]):
        k, v = np.abs(K[g // G]), np.abs(V[g // G])
        e = 2.0 ** -22 * scale * (np.abs(qf[g]).max() * k.sum(1) + k @ np.abs(qf[g])).max()
        x = K[g // G] @ qf[g] * scale
        p = np.exp(x - x.max())
        out[g] = (p / p.sum()) @ v * 2 * (e + 2.0 ** -20 + (len(k) / 16 + 64) * 2.0 ** -24) + 2.0 ** -38 * v.sum(0)
    return out


def _values(X):
    return O.q4_values(*O.q4_quantise(X))


def _check(got, q, K, V, n, what):
    """One cache's outputs against the oracle over its first n rows."""
    got = got.cpu().numpy().astype(np.float64)
    if n == 0:
        assert not got.any(), what
        return
    K, V = _values(K[:, :n]), _values(V[:, :n])
    err = np.abs(got - O.q4_decode_attention(q, K, V))
    bound = _decode_bound(q, K, V)
    assert (err <= bound).all(), f"{what}: off by {np.nanmax(err / bound):.3g} times the bound"


DECODE_CASES = [  # L, Hkv, G, d, n, rows, key scale
    (1, 1, 1, 64, 1, 1, 1.0), (1, 2, 4, 128, 1, 1, 1.0), (2, 2, 4, 128, 15, 15, 1.0), (1, 2, 4, 128, 16, 16, 1.0),
    (1, 2, 4, 128, 17, 40, 1.0), (1, 2, 3, 64, 31, 31, 1.0), (1, 1, 2, 64, 32, 32, 1.0), (1, 2, 8, 128, 33, 33, 1.0),
    (2, 3, 5, 128, 63, 65, 2.0), (1, 2, 6, 64, 64, 64, 1.0), (1, 2, 7, 128, 129, 130, 1.0), (3, 2, 1, 128, 1000, 1003, 1.0),
    (2, 2, 4, 64, 2049, 2100, 2.0), (1, 8, 4, 128, 8272, 8911, 1.0), (1, 2, 8, 64, 5001, 5001, 3.0), (1, 1, 5, 128, 30011, 30011, 1.0),
    (32, 8, 4, 128, 81, 90, 1.0), (12, 8, 1, 128, 700, 701, 1.0), (3, 64, 2, 64, 2000, 2000, 1.0), (66, 1, 4, 64, 50, 52, 1.0),
]


@pytest.mark.parametrize("L,Hkv,G,d,n,rows,ks", DECODE_CASES)
def test_decode_matches_oracle(B, L, Hkv, G, d, n, rows, ks):
    """Rows at or past n hold arbitrary codes and NaN scales."""
    import torch
    rng = np.random.default_rng(100 + n + d + G)
    some = min(L, 3)
    q = [_bits(rng, (Hkv * G, d), ks) for _ in range(some)]
    K, V = [_keys(rng, (Hkv, n, d)) for _ in range(some)], [_bits(rng, (Hkv, n, d)) for _ in range(some)]
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    _stale(cache, rng)
    st = B.new_status()
    stack = lambda X: [TL.bf16_dev(X[l % some]) for l in range(L)]
    B.stepkv_q4_write(cache, stack(K), stack(V), 0, status=st)
    a = B.stepkv_q4_decode(stack(q), cache, n, status=st)
    b = B.stepkv_q4_decode(torch.stack(stack(q)), cache, torch.tensor([n], dtype=torch.int32, device="cuda"), status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and isinstance(a, list) and torch.equal(torch.stack(a), b)  # the count from the device; twice the same
    for l in range(some):
        _check(a[l], q[l], K[l], V[l], n, f"layer {l}")
    if L <= 64:  # the split may cut layers alike or not, the values agree within the bound of each
        for l in range(some, L, 7):
            _check(a[l], q[l % some], K[l % some], V[l % some], n, f"layer {l}")


@pytest.mark.parametrize("L,Hkv,G,d,n", [(16, 32, 1, 128, 1), (16, 32, 4, 128, 33), (20, 32, 2, 64, 150), (33, 16, 5, 128, 500),
                                          (64, 40, 1, 64, 70), (64, 32, 8, 128, 17)])
def test_decode_more_pairs_than_ctas(B, L, Hkv, G, d, n):
    """512 to 2560 (cache, KV head) pairs of few rows, which single warps take, one count for all; then a count for each cache,
    zero among them.  Rows at or past a count hold NaN scales."""
    import torch
    rng = np.random.default_rng(L + n)
    rows = n + 3
    K, V, q = _keys(rng, (Hkv, n, d)), _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv * G, d), 2.0)
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    _stale(cache, rng)
    st = B.new_status()
    Kd, Vd = (TL.bf16_dev(x).expand(L, -1, -1, -1) for x in (K, V))
    B.stepkv_q4_write(cache, Kd, Vd, 0, status=st)
    qd = TL.bf16_dev(q).expand(L, -1, -1).contiguous()
    out = B.stepkv_q4_decode(qd, cache, n, status=st)
    counts = rng.integers(0, n + 1, L)
    counts[0], counts[L // 2], counts[-1] = n, 0, 1
    ragged = B.stepkv_q4_decode(qd, cache, _dev(counts.astype(np.int32)), status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    _check(out[0], q, K, V, n, "one count")
    bound = 2 * _dev(_decode_bound(q, _values(K), _values(V)))
    for l in range(L):  # caches that hold the same: the split cuts them differently, each within its bound of the oracle's
        assert ((out[l] - out[0]).abs() <= bound).all()
    for l in (0, L // 2, L - 1, 1, L // 3):
        _check(ragged[l], q, K, V, int(counts[l]), f"cache {l} of {counts[l]}")


FORMS = [  # L, Hkv, G, d, rows: pairs taken whole, by a CTA or a warp, and cut, with few, some and many states to join
    (1, 3, 3, 64, 500), (5, 7, 1, 128, 700), (33, 14, 2, 64, 300), (60, 9, 5, 128, 200), (31, 3, 1, 64, 2100),
    (23, 5, 3, 128, 1700), (64, 9, 1, 64, 1800), (57, 8, 1, 64, 1000), (9, 7, 4, 64, 4000), (2, 2, 2, 128, 9000),
    (66, 3, 2, 64, 2100)]


@pytest.mark.parametrize("L,Hkv,G,d,rows", FORMS)
def test_decode_forms_and_counts(B, L, Hkv, G, d, rows):
    """Caches of the same rows under one count, long, short and zero, and under counts of their own: whatever way the work is
    divided, each output is within its bound of the oracle's."""
    import torch
    rng = np.random.default_rng(L + rows)
    K, V, q = _keys(rng, (Hkv, rows, d)), _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv * G, d))
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    src = [TL.bf16_dev(x)[None].expand(L, -1, -1, -1) for x in (K, V)]
    st = B.stepkv_q4_write(cache, *src, 0)
    qd = TL.bf16_dev(q).expand(L, -1, -1).contiguous()
    own = rng.integers(0, rows + 1, L).astype(np.int32)
    own[rng.integers(0, L, 3)] = 0, rows, 1
    for counts in (rows, rows - 33, 75, 1, 0, own, np.minimum(own, 40)):
        n = _dev(np.atleast_1d(np.asarray(counts, np.int32)))
        out = torch.full((L, Hkv * G, d), 7.0, device="cuda")
        B.stepkv_q4_decode(qd, cache, n, out=out, status=st)
        torch.cuda.synchronize()
        assert st.item() == 0
        each = np.broadcast_to(counts, (L,))
        for m in sorted(set(each)) if L < 10 else sorted({each[0], each[L // 2], each[-1], each.min(), each.max()}):
            same = np.flatnonzero(each == m)
            _check(out[same[0]], q, K, V, int(m), f"{m} of {counts}, cache {same[0]}")
            if m:
                bound = 2 * _dev(_decode_bound(q, _values(K[:, :m]), _values(V[:, :m])))
                assert all(((out[l] - out[same[0]]).abs() <= bound).all() for l in same)
            else:
                assert not out[same].any()


@pytest.mark.parametrize("magnitude", [2.0 ** -9, 1.0, 2.0 ** 9])
def test_decode_keys_of_any_magnitude(B, magnitude):
    """Keys as small and as large as normal scales hold, with queries that make up for it."""
    import torch
    rng = np.random.default_rng(9)
    K, V, q = _bits(rng, (2, 300, 128), magnitude), _bits(rng, (2, 300, 128)), _bits(rng, (6, 128), 1 / magnitude)
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), 300)[0]
    torch.cuda.synchronize()
    _check(out, q, K, V, 300, "")


def _weights_bound(q, K, V, e):
    """_decode_bound's, of logits that are off by e[head] at most."""
    G, out = q.shape[0] // K.shape[0], np.zeros((q.shape[0], K.shape[2]))
    for g in range(q.shape[0]):
        x = K[g // G] @ O.bf16_to_f64(q[g]) / math.sqrt(q.shape[1])
        p, v = np.exp(x - x.max()), np.abs(V[g // G])
        out[g] = (p / p.sum()) @ v * 2 * (e[g] + 2.0 ** -20 + (len(v) / 16 + 64) * 2.0 ** -24) + 2.0 ** -38 * v.sum(0)
    return out


@pytest.mark.parametrize("G,d", [(4, 128), (6, 128), (2, 64), (8, 64)])
def test_decode_groups_do_not_round_against_each_other(B, G, d):
    """A group whose one large channel meets a zero of the query adds nothing to a logit, however large 8 s sum(q) of it is.

    The queries are whole numbers up to 15, so a group's sums are exact: the codes' products and -8 sum(q) are multiples of
    2^-10 where the largest query element is brought to [2^10, 2^11) and codes count as n 2^-17, and no operand product or sum
    reaches 2^3, so that 22 bits below the largest hold them all.  What is left is fp32's: a rounding for each group of a sum
    no larger than the groups' sizes together, and two of the factor; less than 2^-20 in all."""
    import torch
    rng = np.random.default_rng(G)
    Hkv, n = 2, 300
    k = rng.standard_normal((Hkv, n, d))
    k[..., :32] = 0
    k[..., 0] = rng.choice([-1, 1], (Hkv, n)) * rng.uniform(5000, 7000, (Hkv, n))
    qf = rng.integers(-3, 4, (Hkv * G, d)).astype(np.float32)
    qf[:, 0], qf[:, 1:32] = 0, 15
    K, V, q = wl.f32_to_bf16_bits(k.astype(np.float32)), _bits(rng, (Hkv, n, d)), wl.f32_to_bf16_bits(qf)
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0].cpu().numpy().astype(np.float64)
    Kv, Vv = _values(K), _values(V)
    groups = np.abs((Kv[:, None] * qf.reshape(Hkv, G, 1, d)).reshape(Hkv, G, n, -1, 32).sum(-1)).sum(-1).max(-1).reshape(-1)
    e = 6 * 2.0 ** -24 * groups / math.sqrt(d)
    err, bound = np.abs(out - O.q4_decode_attention(q, Kv, Vv)), _weights_bound(q, Kv, Vv, e)
    assert (err <= bound).all(), f"off by {(err / bound).max():.3g} times the bound"


@pytest.mark.parametrize("G,d", [(4, 128), (5, 128), (8, 64)])
def test_decode_one_signed_queries_and_sparse_keys(B, G, d):
    """Queries of one sign over keys with one channel a group: a group's sum of n q and its -8 sum(q) nearly cancel.  Each of the
    two and what is left is known to 22 bits of |s| 8 sum|q| (the codes that are not 8 are single), so that a logit is off by
    3 2^-22 of the sum of these over the groups at most, which is what the header states."""
    import torch
    rng = np.random.default_rng(d + G)
    Hkv, n = 2, 700
    k = np.zeros((Hkv, n, d // 32, 32))
    np.put_along_axis(k, rng.integers(0, 32, (Hkv, n, d // 32, 1)), rng.standard_normal((Hkv, n, d // 32, 1)) * 8, -1)
    qf = np.abs(rng.standard_normal((Hkv * G, d))) + 0.1
    K, V, q = wl.f32_to_bf16_bits(k.reshape(Hkv, n, d).astype(np.float32)), _bits(rng, (Hkv, n, d)), wl.f32_to_bf16_bits(qf.astype(np.float32))
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0].cpu().numpy().astype(np.float64)
    Kv, Vv = _values(K), _values(V)
    top = np.abs(Kv).reshape(Hkv, 1, n, -1, 32).max(-1)  # 8 |s|
    e = 3 * 2.0 ** -22 * (top * O.bf16_to_f64(q).reshape(Hkv, G, 1, -1, 32).sum(-1)).sum(-1).max(-1).reshape(-1) / math.sqrt(d)
    err, bound = np.abs(out - O.q4_decode_attention(q, Kv, Vv)), _weights_bound(q, Kv, Vv, e)
    assert (err <= bound).all(), f"off by {(err / bound).max():.3g} times the bound"


@pytest.mark.parametrize("magnitude", [2.0 ** -14, 2.0 ** -19])
def test_decode_keys_with_subnormal_scales(B, magnitude):
    """The scale multiplies a group's fp32 sum, so that fp16's smallest scales (exact, if of fewer bits) cost a logit nothing:
    the bound above."""
    import torch
    rng = np.random.default_rng(10)
    Hkv, G, d, n = 2, 4, 128, 300
    K, V, q = _bits(rng, (Hkv, n, d), magnitude), _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv * G, d), 1 / magnitude)
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0].cpu().numpy().astype(np.float64)
    Kv, Vv = _values(K), _values(V)
    assert (np.abs(Kv[Kv != 0]).min() < 2.0 ** -14) and (np.abs(Kv).max() > 0)
    top = np.abs(Kv).reshape(Hkv, 1, n, -1, 32).max(-1)
    e = 3 * 2.0 ** -22 * (top * np.abs(O.bf16_to_f64(q)).reshape(Hkv, G, 1, -1, 32).sum(-1)).sum(-1).max(-1).reshape(-1) / math.sqrt(d)
    err, bound = np.abs(out - O.q4_decode_attention(q, Kv, Vv)), _weights_bound(q, Kv, Vv, e)
    assert (err <= bound).all(), f"off by {(err / bound).max():.3g} times the bound"


def test_offsets_past_32_bits(B):
    """68 million rows of one head: 4.4 GB of codes.  All but the last 40 are zero keys and values, so the output is known; the
    last rows are written, read back, moved and attended where offsets need more than 32 bits."""
    import torch
    rng = np.random.default_rng(41)
    rows, n, d = 68_000_000, 40, 128
    assert rows * d // 2 > 2 ** 32
    cache = B.Q4Cache.allocate(1, 1, rows, d)
    cache.K.fill_(0x88), cache.V.fill_(0x88)  # (code 8 with scale 0: the value 0)
    K, V, q = _bits(rng, (1, n, d)), _bits(rng, (1, n, d)), _bits(rng, (4, d))
    st = B.stepkv_q4_write(cache, TL.bf16_dev(K)[None], TL.bf16_dev(V)[None], rows - n)
    Kb, Vb = B.stepkv_q4_read(cache, rows - n, n, status=st)
    by_idx, _ = B.stepkv_q4_read(cache, idx=torch.arange(rows - n, rows, dtype=torch.int32, device="cuda"), status=st)
    small = B.Q4Cache.allocate(1, 1, n, d)
    kept = torch.arange(rows - n, rows, dtype=torch.int32, device="cuda")
    B.stepkv_q4_compact(cache, rows, kept, torch.tensor([n], dtype=torch.int32, device="cuda"), n, small, status=st)
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], cache, rows, status=st)[0]
    torch.cuda.synchronize()
    assert st.item() == 0
    for got, X in ((Kb, K), (Vb, V), (by_idx, K)):
        _same_bits(got[0], _back_bits(X))
    assert torch.equal(small.K[0], cache.K[0][:, rows - n:]) and torch.equal(small.V_scale[0], cache.V_scale[0][:, rows - n:])
    k, v = _values(K)[0], _values(V)[0]
    w = np.exp(O.bf16_to_f64(q) @ k.T / math.sqrt(d))
    want = w @ v / (rows - n + w.sum(1, keepdims=True))
    # the weights of a lane are summed one after another: rows / 8 / (warps of a wave) of them at least on one GPU; half an
    # ulp each of the running sum, and the same of the values' sums
    terms = rows / 8 / 1824 + 100
    assert (np.abs(out.cpu().numpy() - want) <= 2 * terms * 2.0 ** -24 * (w @ np.abs(v)) / rows + 2.0 ** -38 * np.abs(v).sum(0)).all()


RAGGED = [  # Hkv, G, d, counts, rows
    (2, 4, 64, [8191, 0, 1, 17, 5000, 333, 0, 16, 4096, 2], 8192), (8, 4, 128, [0, 0, 0], 100), (1, 8, 128, [0, 3001], 3001),
    (8, 5, 128, [1] * 40 + [900], 900), (2, 1, 64, list(range(0, 64)), 70), (16, 2, 128, [31, 700, 32, 0, 33], 701),
    (4, 4, 128, [64] * 70 + [0, 5], 64), (8, 3, 64, [20000, 100, 100, 100], 20000),
]


@pytest.mark.parametrize("Hkv,G,d,counts,rows", RAGGED)
def test_decode_ragged_batch(B, Hkv, G, d, counts, rows):
    """A count for each cache, some of them zero, more than 64 caches among them."""
    import torch
    rng = np.random.default_rng(len(counts) + rows)
    L, top = len(counts), max(max(counts), 1)
    K, V, q = _keys(rng, (Hkv, top, d)), _bits(rng, (Hkv, top, d)), _bits(rng, (Hkv * G, d), 2.0)
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    _stale(cache, rng)
    for l, n in enumerate(counts):
        B.stepkv_q4_write(cache.layers(l, l + 1), TL.bf16_dev(K)[None], TL.bf16_dev(V)[None], 0, n=n)
    st = B.new_status()
    out = torch.full((L, Hkv * G, d), 7.0, device="cuda")
    B.stepkv_q4_decode(TL.bf16_dev(q).expand(L, -1, -1).contiguous(), cache, torch.tensor(counts, dtype=torch.int32, device="cuda"),
                       out=out, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for l in sorted({counts.index(n) for n in counts[:64]} | {L - 1}):
        _check(out[l], q, K, V, counts[l], f"cache {l}")


@pytest.mark.parametrize("G,d", [(4, 128), (6, 64)])
def test_decode_pairs_that_other_warps_take(B, G, d):
    """Ranges that run over many pairs of a block or two, of which each warp takes every fourth and passes over the others, with
    long pairs in between that all take: a warp that lost its place would skip a pair or take one twice.  Every output against
    the oracle."""
    import torch
    rng = np.random.default_rng(G)
    Hkv, rows = 40, 1700  # 64 x 40 pairs in 456 ranges
    counts = [int(x) for x in rng.choice([1, 31, 32, 33, 64], 64)]
    counts[::9] = [rows - int(x) for x in rng.integers(0, 64, len(counts[::9]))]
    K, V, q = _bits(rng, (1, rows, d)), _bits(rng, (1, rows, d)), _bits(rng, (G, d), 2.0)
    one = _filled(B, [K], [V])
    cache = B.Q4Cache(*(t.expand(64, Hkv, -1, -1).contiguous() for t in (one.K, one.K_scale, one.V, one.V_scale)))
    st, out = B.new_status(), torch.full((64, Hkv * G, d), 7.0, device="cuda")
    B.stepkv_q4_decode(TL.bf16_dev(q).repeat(64, Hkv, 1), cache, _dev(np.array(counts, np.int32)), out=out, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for n in sorted(set(counts)):
        want = O.q4_decode_attention(q, _values(K[:, :n]), _values(V[:, :n]))
        bound = _decode_bound(q, _values(K[:, :n]), _values(V[:, :n]))
        for l in (l for l in range(64) if counts[l] == n):
            err = np.abs(out[l].view(Hkv, G, d).cpu().numpy().astype(np.float64) - want)
            assert (err <= bound).all(), f"cache {l} of {n} rows: off by {(err / bound).max():.3g} times the bound"


def test_decode_bad_counts(B):
    import torch
    rng = np.random.default_rng(12)
    Hkv, G, d, rows = 2, 4, 128, 60
    K, V, q = _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv * G, d))
    cache = _filled(B, [K, K], [V, V])
    qd = TL.bf16_dev(q).expand(2, -1, -1).contiguous()
    for counts, code in (([rows + 1, 5], B.STEPKV_ENOSPACE), ([5, -3], B.STEPKV_EDATA), ([2 ** 31 - 1, 5], B.STEPKV_ENOSPACE)):
        st = B.new_status()
        out = B.stepkv_q4_decode(qd, cache, torch.tensor(counts, dtype=torch.int32, device="cuda"), status=st)
        torch.cuda.synchronize()
        assert st.item() == code
        for l, n in enumerate(counts):
            _check(out[l], q, K, V, max(0, min(n, rows)), f"counts {counts}, cache {l}")


@pytest.mark.parametrize("each", [False, True])
def test_decode_bad_counts_of_long_caches(B, each):
    """As above where the work is cut into ranges: a count above the capacity uses the capacity, a negative one none."""
    import torch
    rng = np.random.default_rng(13)
    L, Hkv, G, d, rows = 2, 2, 2, 64, 5000
    K, V, q = _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv * G, d))
    cache, qd = _filled(B, [K, K], [V, V]), TL.bf16_dev(q).expand(L, -1, -1).contiguous()
    for n, code, used in (([rows + 1, 3000], B.STEPKV_ENOSPACE, (rows, 3000)), ([2 ** 31 - 1, 0], B.STEPKV_ENOSPACE, (rows, 0)),
                          ([-1, 40], B.STEPKV_EDATA, (0, 40)), ([-2 ** 31, rows], B.STEPKV_EDATA, (0, rows))):
        st, out = B.new_status(), torch.full((L, Hkv * G, d), 7.0, device="cuda")
        B.stepkv_q4_decode(qd, cache, _dev(np.array(n if each else n[:1], np.int32)), out=out, status=st)
        torch.cuda.synchronize()
        assert st.item() == code
        for l in range(L):
            _check(out[l], q, K, V, used[l if each else 0], f"{n}, cache {l}")


@pytest.mark.parametrize("G", [3, 8])
@pytest.mark.parametrize("Hkv,d,n", [(2, 128, 60), (2, 64, 3001), (64, 128, 2000)])
@pytest.mark.parametrize("kind", ["nan key", "inf key", "nan value", "inf query", "nan query"])
def test_decode_non_finite(B, Hkv, d, n, G, kind):
    """A NaN or an infinity in a key (its group reads back as NaN) or a query makes the outputs of its heads NaN, one in a
    value row its group of channels; every other output is what it is without it."""
    import torch
    rng = np.random.default_rng(n + G)
    K, V, q = _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv * G, d))
    clean = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0]
    bad = torch.zeros((Hkv * G, d), dtype=torch.bool, device="cuda")
    h = Hkv - 1
    if kind == "nan key":
        K[h, n // 2, 9], bad[h * G:] = 0x7FC0, True
    elif kind == "inf key":
        K[h, n - 1, 40], bad[h * G:] = 0xFF80, True
    elif kind == "nan value":
        V[h, n // 2, 33], bad[h * G:, 32:64] = 0x7FC0, True
    else:
        q[h * G + 1, 5], bad[h * G + 1] = (0x7F80 if kind == "inf query" else 0x7FC0), True
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0]
    torch.cuda.synchronize()
    assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("magnitude", [2.0 ** -100, 1e-20, 1e-3, 1e3, 1e20])
def test_decode_queries_of_any_magnitude(B, magnitude):
    """Tiny queries weigh all keys alike, huge ones pick a key; one element far above the others keeps them from nothing."""
    import torch
    rng = np.random.default_rng(3)
    Hkv, G, d, n = 2, 5, 128, 200
    K, V = _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv, n, d))
    q = _bits(rng, (Hkv * G, d), magnitude)
    q[0, 3] = wl.f32_to_bf16_bits(np.float32([magnitude * 300]))[0]
    q[1] = 0
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n)[0]
    torch.cuda.synchronize()
    k, v = _values(K), _values(V)
    if magnitude <= 1e3:
        _check(out, q, K, V, n, "")
    else:  # the margin between the two largest logits is far above their rounding: the output is one value row
        for g in range(Hkv * G):
            if g != 1:
                j = int(np.argmax(k[g // G] @ O.bf16_to_f64(q[g])))
                np.testing.assert_array_equal(out[g].cpu().numpy(), v[g // G][j].astype(np.float32))


@pytest.mark.parametrize("scale", [2.0 ** -20, 2.0 ** -10, 2.0 ** 9])
def test_decode_values_of_any_magnitude(B, scale):
    """From scales on fp16's last steps to saturated values: relative to the values the bound is the same."""
    import torch
    rng = np.random.default_rng(2)
    K, V, q = _bits(rng, (2, 300, 64)), _bits(rng, (2, 300, 64), scale), _bits(rng, (8, 64))
    out = B.stepkv_q4_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), 300)[0]
    torch.cuda.synchronize()
    _check(out, q, K, V, 300, "")


def test_decode_peaked_and_flat_rows(B):
    """One key far above the rest, at the front, inside and at the end; and logits that fall or rise along the keys."""
    import torch
    rng = np.random.default_rng(1)
    d, n = 128, 700
    q = np.abs(rng.standard_normal((4, d))).astype(np.float32) + 0.5
    for at in (0, 350, 699, "falling", "rising"):
        k = (rng.standard_normal((1, n, d)) * 0.1).astype(np.float32)
        if isinstance(at, int):
            k[0, at] += 3.0
        else:
            k[0] += np.linspace(4, -4, n)[:, None] * (1 if at == "falling" else -1)
        K, V, qb = wl.f32_to_bf16_bits(k), _bits(rng, (1, n, d)), wl.f32_to_bf16_bits(q)
        out = B.stepkv_q4_decode([TL.bf16_dev(qb)], _filled(B, [K], [V]), n)[0]
        torch.cuda.synchronize()
        _check(out, qb, K, V, n, str(at))


def test_decode_agrees_with_decode_over_the_rows_read_back(B):
    """Both read the same numbers: they differ by twice what each may lose at most."""
    import torch
    rng = np.random.default_rng(21)
    L, Hkv, G, d, n = 2, 8, 4, 128, 4101
    K, V = [_keys(rng, (Hkv, n, d)) for _ in range(L)], [_bits(rng, (Hkv, n, d)) for _ in range(L)]
    q = [_bits(rng, (Hkv * G, d)) for _ in range(L)]
    cache = _filled(B, K, V)
    Kb, Vb = B.stepkv_q4_read(cache)
    qd = [TL.bf16_dev(x) for x in q]
    a, b = B.stepkv_q4_decode(qd, cache, n), B.stepkv_decode(qd, list(Kb), list(Vb), n)
    torch.cuda.synchronize()
    for l in range(L):
        err = (a[l] - b[l]).abs().cpu().numpy()
        assert (err <= 2 * _decode_bound(q[l], _values(K[l]), _values(V[l]))).all()


def test_strided_caches(B):
    """Heads and layers with room between them, as a cache preallocated for something larger has it."""
    import torch
    rng = np.random.default_rng(22)
    L, Hkv, d, rows, n = 2, 3, 128, 70, 61
    z = lambda w, t: torch.zeros((L + 1, Hkv + 2, rows + 9, w), dtype=t, device="cuda")
    big = [z(64, torch.uint8), z(4, torch.float16), z(64, torch.uint8), z(4, torch.float16)]
    cache = B.Q4Cache(*[[t[l, 1:1 + Hkv, :rows] for l in range(L)] for t in big])
    K, V = [_bits(rng, (Hkv, n, d)) for _ in range(L)], [_bits(rng, (Hkv, n, d)) for _ in range(L)]
    q = [_bits(rng, (Hkv * 2, d)) for _ in range(L)]
    st = B.stepkv_q4_write(cache, [TL.bf16_dev(x) for x in K], [TL.bf16_dev(x) for x in V], 0)
    out = B.stepkv_q4_decode([TL.bf16_dev(x) for x in q], cache, n, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for l in range(L):
        _check(out[l], q[l], K[l], V[l], n, f"layer {l}")
    for t in big:  # nothing outside the cache was written
        inside = torch.zeros_like(t, dtype=torch.bool)
        inside[:L, 1:1 + Hkv, :n] = True
        assert not t[~inside].any()


# ------------------------------------------------------------------------------------------------ streams, graphs, a run
def test_two_streams_at_once(B):
    """Calls on two streams, each with a cache and a workspace of its own."""
    import torch
    rng = np.random.default_rng(31)
    Hkv, G, d, n = 8, 4, 128, 3000
    data = [(_bits(rng, (Hkv, n, d)), _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv * G, d))) for _ in range(2)]
    caches = [B.Q4Cache.allocate(1, Hkv, n, d) for _ in range(2)]
    src = [[TL.bf16_dev(x)[None] for x in t] for t in data]
    ws = [B.q4_decode_workspace(c, Hkv * G) for c in caches]
    streams = [torch.cuda.Stream() for _ in range(2)]
    st, outs = B.new_status(), [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            B.stepkv_q4_write(caches[i], src[i][0], src[i][1], 0, status=st, stream=s)
            with torch.cuda.stream(s):
                outs[i].append(B.stepkv_q4_decode(src[i][2], caches[i], n, ws=ws[i], status=st))
    torch.cuda.synchronize()
    assert st.item() == 0
    for i, (K, V, q) in enumerate(data):
        _check(outs[i][0][0], q, K, V, n, f"stream {i}")
        assert all(torch.equal(o, outs[i][0]) for o in outs[i])


def test_captured_steps_replay_with_new_counts(B):
    """A decode step (append a token, attend) captured once: the row, the count and the data change between replays; a second
    graph over the same workspace runs in between."""
    import torch
    rng = np.random.default_rng(32)
    L, Hkv, G, d, rows, n0 = 2, 2, 4, 64, 700, 640
    K, V = [_bits(rng, (Hkv, rows, d)) for _ in range(L)], [_bits(rng, (Hkv, rows, d)) for _ in range(L)]
    q = _bits(rng, (L, Hkv * G, d))
    Kd, Vd = (torch.stack([TL.bf16_dev(x) for x in X]) for X in (K, V))
    cache = B.Q4Cache.allocate(L, Hkv, rows, d)
    st = B.stepkv_q4_write(cache, Kd, Vd, 0, n=n0)
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")
    row, count = i32(n0), i32(n0 + 1)
    tk, tv = Kd[:, :, n0:n0 + 1].clone(), Vd[:, :, n0:n0 + 1].clone()
    qd, ws = TL.bf16_dev(q), B.q4_decode_workspace(cache, Hkv * G)
    out, other = torch.zeros((L, Hkv * G, d), device="cuda"), torch.zeros((L, Hkv * G, d), device="cuda")

    def step():
        B.stepkv_q4_write(cache, tk, tv, row, status=st)
        B.stepkv_q4_decode(qd, cache, count, out=out, ws=ws, status=st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        step()
    with torch.cuda.graph(graphs[1]):
        B.stepkv_q4_decode(qd, cache, 33, out=other, ws=ws, status=st)
    got = []
    for t in range(n0, n0 + 20):
        row.fill_(t), count.fill_(t + 1)
        tk.copy_(Kd[:, :, t:t + 1]), tv.copy_(Vd[:, :, t:t + 1])
        graphs[0].replay()
        got.append(out.clone())
        graphs[1].replay()
    torch.cuda.synchronize()
    assert st.item() == 0
    for t in (0, 7, 19):
        for l in range(L):
            _check(got[t][l], q[l], K[l], V[l], n0 + t + 1, f"step {t}, layer {l}")
    for l in range(L):
        _check(other[l], q[l], K[l], V[l], 33, f"other graph, layer {l}")


def test_what_a_call_makes_belongs_to_its_stream(B):
    """Calls on a stream while the current one is busy: the status, rows and workspace that they make are neither cleared nor
    handed out again by what the current stream does late."""
    import torch
    rng = np.random.default_rng(34)
    L, Hkv, G, d, n = 1, 2, 4, 64, 600
    K, V = ([_bits(rng, (Hkv, n, d)) for _ in range(L)] for _ in range(2))
    cache = _filled(B, K, V)
    src, q = TL.bf16_dev(K[0])[None], _bits(rng, (Hkv * G, d))
    qd = TL.bf16_dev(q)[None]
    count, row0 = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (n - 7, 1))
    side = torch.cuda.Stream()
    B.stepkv_q4_decode(qd, cache, n), B.stepkv_q4_read(cache, n=count), B.stepkv_q4_write(cache, src, src, 0)
    cache = _filled(B, K, V)
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)  # some 25 ms on the current stream
    st = B.stepkv_q4_write(cache, src, src, row0, stream=side)  # a row too many
    Kb, Vb = B.stepkv_q4_read(cache, n=count, stream=side)
    out = B.stepkv_q4_decode(qd, cache, count, stream=side)
    made = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert st.item() == B.STEPKV_ENOSPACE and not made.any()
    for got, X in ((Kb, K), (Vb, V)):
        _same_bits(got[0, :, :n - 7], _back_bits(X[0])[:, :n - 7])
        assert not got[0, :, n - 7:].any()
    _check(out[0], q, K[0], V[0], n - 7, "on its own stream")


def test_rows_that_are_not_read_are_zero(B):
    """Allocated rows of an index or a first row outside the cache."""
    import torch
    rng = np.random.default_rng(35)
    K = [_bits(rng, (2, 40, 64))]
    cache, st = _filled(B, K), B.new_status()
    junk = torch.full((1, 2, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    del junk
    Kb, Vb = B.stepkv_q4_read(cache, idx=_dev(np.array([5, 40, 7], np.int32)), status=st)
    assert st.item() == B.STEPKV_EDATA and Vb is None
    _same_bits(Kb[0], np.where(np.array([1, 0, 1])[None, :, None] == 1, _back_bits(K[0])[:, [5, 0, 7]], np.uint16(0)))
    st = B.new_status()
    junk = torch.full((1, 2, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    del junk
    Kb, _ = B.stepkv_q4_read(cache, _dev(np.array([38], np.int32)), n=3, status=st)
    assert st.item() == B.STEPKV_EDATA and Kb.shape == (1, 2, 3, 64) and not Kb.any()


def test_captured_boundary(B):
    """Write by an index list, compaction and reading back in one graph, replayed with other counts, indices and data."""
    import torch
    rng = np.random.default_rng(33)
    L, Hkv, d, T = 2, 2, 64, 80
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    src = torch.zeros((L, Hkv, T, d), dtype=torch.bfloat16, device="cuda")
    cache, left = B.Q4Cache.allocate(L, Hkv, T, d), B.Q4Cache.allocate(L, Hkv, T, d)
    idx, n, kept, n_kept, st = i32(T), i32(1), i32(T), i32(1), B.new_status()
    back = torch.zeros((L, Hkv, T, d), dtype=torch.bfloat16, device="cuda")

    def boundary():
        B.stepkv_q4_write(cache, src, src, 0, n=n, idx=idx, status=st)
        B.stepkv_q4_compact(cache, T, kept, n_kept, T, left, status=st)
        B.stepkv_q4_read(left, 0, n_kept, K=back, status=st)

    boundary()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        boundary()
    for t in range(3):
        X = _bits(rng, (L, Hkv, T, d))
        a, b = int(rng.integers(2, T + 1)), int(rng.integers(1, T // 2))
        i, j = rng.integers(0, T, T).astype(np.int32), np.sort(rng.integers(0, a, T)).astype(np.int32)
        src.copy_(TL.bf16_dev(X))
        for dst, v in ((idx, i), (n, [a]), (kept, j), (n_kept, [b])):
            dst.copy_(torch.as_tensor(np.asarray(v, np.int32)))
        back.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert st.item() == 0
        _same_bits(back[:, :, :b], _back_bits(X)[:, :, i[j[:b]]])
        assert (back[:, :, b:] == 7).all()


def test_trajectory_on_a_4_bit_cache(B):
    """The operators as an agent's loop uses them: a boundary of the bf16 cache, the retained rows written in 4 bits by the
    selection's own index list, tokens appended and attended one at a time, then the next boundary on the 4-bit cache (the
    saliency layers' keys read back, scored, selected, rows moved in 4 bits) and a read of what it left."""
    import torch
    tr = wl.custom(77, L=4, Hq=8, Hkv=2, d=128, T=1500, W=32, n_steps=5, budget=wl.Budget.ratio(1, 5))
    g = TL.GpuTraj(tr)
    st = B.stepkv_compress([g.problem()], B.Params())
    rows, new = 600, 25
    cache = B.Q4Cache.allocate(4, 2, rows, 128)
    B.stepkv_q4_write(cache, g.K, g.V, 0, n=g.out.n_kept, idx=g.out.kept_idx, status=st)
    rng = np.random.default_rng(78)
    K1, V1 = [_bits(rng, (2, new, 128)) for _ in range(4)], [_bits(rng, (2, new, 128)) for _ in range(4)]
    q = [_bits(rng, (8, 128)) for _ in range(4)]
    Kd, Vd = [TL.bf16_dev(x) for x in K1], [TL.bf16_dev(x) for x in V1]
    length = g.out.n_kept.clone()  # stays on the device
    for t in range(new):
        B.stepkv_q4_write(cache, [x[:, t:t + 1] for x in Kd], [x[:, t:t + 1] for x in Vd], length, status=st)
        length += 1
    out = B.stepkv_q4_decode([TL.bf16_dev(x) for x in q], cache, length, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    n0, n = int(g.out.n_kept.item()), int(length.item())
    kept = g.out.kept_idx[:n0].cpu().numpy()
    assert n == n0 + new
    held = [(np.concatenate([tr.keys(l)[:, kept], K1[l]], 1), np.concatenate([tr.values(l)[:, kept], V1[l]], 1)) for l in range(4)]
    for l in range(4):
        _check(out[l], q[l], *held[l], n, f"layer {l}")
    # the next boundary: the last three layers' keys in bf16 for the saliency, everything else stays in 4 bits
    Ksal, _ = B.stepkv_q4_read(cache.layers(1), 0, n, K=torch.empty((3, 2, n, 128), dtype=torch.bfloat16, device="cuda"), status=st)
    Q = [_bits(rng, (8, 16, 128)) for _ in range(3)]
    sal = B.stepkv_score(list(Ksal), [TL.bf16_dev(x) for x in Q], n, status=st)
    want = np.stack([O.window_attention_saliency(_back_bits(held[l + 1][0]), Q[l]) for l in range(3)])
    TL.assert_close(sal.cpu().numpy(), want, "saliency of the keys read back")
    steps = B.StepSignals(*(torch.ones(2, device="cuda") * x for x in (1.0, 0.5, 0.1, 0.0)))
    step_id = torch.arange(n, device="cuda", dtype=torch.int32) // ((n + 1) // 2)
    prot = torch.zeros(n, dtype=torch.uint8, device="cuda")
    prot[:16] = 1
    sel = B.SelectOutputs.allocate(n, 2, n, "cuda")
    B.stepkv_select(sal.view(6, n), step_id, prot, steps, B.Params(), B.budget_count(100), sel, status=st)
    left = B.Q4Cache.allocate(4, 2, rows, 128)
    sid = torch.empty(n, dtype=torch.int32, device="cuda")
    B.stepkv_q4_compact(cache, n, sel.kept_idx, sel.n_kept, n, left, step_id_in=step_id, step_id_out=sid, status=st)
    out = B.stepkv_q4_decode([TL.bf16_dev(x) for x in q], left, sel.n_kept, status=st)
    Kb, Vb = B.stepkv_q4_read(left, 0, sel.n_kept, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and sel.n_kept.item() == 116
    kept2 = sel.kept_idx[:116].cpu().numpy()
    assert torch.equal(sid[:116], step_id[sel.kept_idx[:116].long()])
    for l in range(4):
        K, V = (x[:, kept2] for x in held[l])
        _check(out[l], q[l], K, V, 116, f"after the boundary, layer {l}")
        _same_bits(Kb[l][:, :116], _back_bits(K))
        _same_bits(Vb[l][:, :116], _back_bits(V))


def test_binding_refusals(B):
    import torch
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    cache, keys = B.Q4Cache.allocate(2, 2, 20, 64), B.Q4Cache.allocate(2, 2, 20, 64, values=False)
    X, i32 = z(2, 2, 5, 64), z(1, t=torch.int32)
    bad = [lambda: B.stepkv_q4_write(cache, X, None, 0), lambda: B.stepkv_q4_write(keys, X, X, 0),
           lambda: B.stepkv_q4_write(cache, X[:1], X[:1], 0), lambda: B.stepkv_q4_write(cache, X, z(2, 2, 6, 64), 0),
           lambda: B.stepkv_q4_write(cache, z(2, 2, 64, 5).transpose(2, 3), z(2, 2, 64, 5).transpose(2, 3), 0),
           lambda: B.stepkv_q4_write(cache, X, X, 0, n=6), lambda: B.stepkv_q4_write(cache, X, X, 0, n=-1),
           lambda: B.stepkv_q4_write(cache, X, X, z(3, t=torch.int32)), lambda: B.stepkv_q4_write(cache, X, X, 0, idx=i32.cpu()),
           lambda: B.stepkv_q4_write(cache, X.cpu(), X.cpu(), 0), lambda: B.stepkv_q4_write(cache, [X[0], X[1].cpu()], X, 0),
           lambda: B.stepkv_q4_write(cache, X, X, 0, status=i32.cpu()), lambda: B.stepkv_q4_read(keys, V=X),
           lambda: B.stepkv_q4_read(cache, 0, 6, K=X),
           lambda: B.stepkv_q4_read(cache, 0, 3, idx=z(2, t=torch.int32), K=X),
           lambda: B.stepkv_q4_compact(cache, 20, z(4, t=torch.int32), i32, 5, cache.layers(0, 2)),
           lambda: B.stepkv_q4_decode(z(2, 4, 64), keys, 5), lambda: B.stepkv_q4_decode(z(1, 4, 64), cache, 5),
           lambda: B.stepkv_q4_decode(z(2, 4, 128)[:, :, ::2], cache, 5), lambda: B.stepkv_q4_decode(z(2, 4, 64), cache, z(3, t=torch.int32)),
           lambda: B.stepkv_q4_decode(z(2, 4, 64), cache, 5, out=z(2, 4, 32, t=torch.float32)),
           lambda: B.Q4Cache(cache.K, cache.K_scale[:, :, :10]), lambda: B.Q4Cache(cache.K, cache.K_scale, cache.V)]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
    wrong_type = [lambda: B.stepkv_q4_write(cache, X.float(), X.float(), 0), lambda: B.stepkv_q4_write(cache, X, X, 0, idx=i32.long()),
                  lambda: B.stepkv_q4_decode(z(2, 4, 64, t=torch.float16), cache, 5), lambda: B.stepkv_q4_decode(z(2, 4, 64), cache, i32.long()),
                  lambda: B.Q4Cache(cache.K, cache.K_scale.float())]
    for f in wrong_type:
        with pytest.raises(TypeError):
            f()
    refused = [lambda: B.stepkv_q4_write(cache, X, X, 16), lambda: B.stepkv_q4_read(cache, 16, 5, K=X), lambda: B.stepkv_q4_read(cache, 0, 21),
               lambda: B.stepkv_q4_compact(cache, 20, z(4, t=torch.int32), i32, 4, cache.layers(0, 2)),
               lambda: B.stepkv_q4_read(cache, 0, 5, K=z(2, 2, 1, 64).expand(-1, -1, 5, -1)),
               lambda: B.stepkv_q4_decode(z(2, 18, 64), cache, 5), lambda: B.stepkv_q4_decode(z(2, 4, 64), cache, 21)]
    for f in refused:
        with pytest.raises(B.StepKVError):
            f()
    torch.cuda.synchronize()


def test_numbers_past_32_bits_are_refused(B):
    """Not cut to their lower 32 bits, which would name another row or count."""
    import torch
    cache, other = B.Q4Cache.allocate(1, 1, 20, 64), B.Q4Cache.allocate(1, 1, 20, 64)
    X, i32 = torch.ones((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(20, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    many = torch.empty((1, 1, 1, 64), dtype=torch.bfloat16, device="cuda").expand(-1, -1, 2 ** 32 + 2, -1)
    for call in (lambda: B.stepkv_q4_write(cache, X, X, 2 ** 32), lambda: B.stepkv_q4_write(cache, X, X, -2 ** 32 + 3),
                 lambda: B.stepkv_q4_write(cache, many, many, 0), lambda: B.stepkv_q4_write(cache, many, many, 0, n=2),
                 lambda: B.stepkv_q4_read(cache, 2 ** 32, 2, K=X), lambda: B.stepkv_q4_decode(q, cache, 2 ** 32 + 5),
                 lambda: B.stepkv_q4_decode(q, cache, 2 ** 32), lambda: B.q4_decode_workspace(cache, 2 ** 32 + 4),
                 lambda: B.stepkv_q4_compact(cache, 2 ** 32 + 20, i32, i32[:1], 20, other),
                 lambda: B.stepkv_q4_compact(cache, 20, i32, i32[:1], 20 - 2 ** 32, other),
                 lambda: B.Q4Cache(cache.K.expand(-1, 2 ** 32 + 1, -1, -1), cache.K_scale.expand(-1, 2 ** 32 + 1, -1, -1))):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert not cache.K.any() and not other.K.any()
