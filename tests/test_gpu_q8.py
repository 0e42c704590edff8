"""GPU parity of a cache held in 8 bits against the oracle, through the public entry points.

Writing and reading back have one right answer and are compared value for value.  Decode attention and its masses are
compared with the oracle's over the values the codes stand for, element by element, within a bound on what 32-bit
arithmetic may lose (_decode_bound, _mass_bound).
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


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _f64(t):
    """A bf16 device tensor's values."""
    return O.bf16_to_f64(TL.bits_of(t.contiguous()))


def _codes(t):
    """The values a tensor of codes stands for, without their scales."""
    import torch
    return O.e4m3_values(t.contiguous().view(torch.uint8).cpu().numpy())


def _stale(cache, rng):
    """Fills a cache with arbitrary codes and NaN scales: rows that a call must leave alone or not use."""
    import torch
    for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        x.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 256, tuple(x.shape), dtype=np.uint8)))
        s.fill_(float("nan"))
    return [x.view(torch.uint8).clone() for x in (cache.K, cache.V)]


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


def _filled(B, K, V, rows=None):
    """A cache that holds per-layer bf16 bits K, V [Hkv, n, d]."""
    Hkv, n, d = K[0].shape
    cache = B.Q8Cache.allocate(len(K), Hkv, rows or n, d)
    st = B.stepkv_q8_write(cache, [TL.bf16_dev(x) for x in K], [TL.bf16_dev(x) for x in V], 0)
    assert st.item() == 0
    return cache


# ------------------------------------------------------------------------------------------------ write and read back
WRITE_CASES = [  # L, Hkv, d, rows before, T, rows, layout
    (1, 1, 64, 0, 1, 1, "heads"), (2, 2, 64, 3, 5, 11, "heads"), (3, 2, 128, 1, 33, 40, "tokens"), (1, 2, 128, 31, 2, 64, "gaps"),
    (2, 1, 128, 7, 200, 301, "gaps"), (32, 8, 128, 50, 1, 60, "tokens"), (70, 1, 64, 40, 3, 46, "heads"), (1, 2, 64, 0, 1000, 1000, "heads"),
    (1, 5, 64, 32, 32, 64, "tokens"), (2, 2, 128, 63, 64, 127, "heads"), (1, 3, 64, 33, 31, 70, "gaps"), (1, 1, 128, 0, 32, 32, "heads")]


@pytest.mark.parametrize("L,Hkv,d,before,T,rows,kind", WRITE_CASES)
def test_write_and_read_match_oracle(B, L, Hkv, d, before, T, rows, kind):
    """Rows appended behind others, in caches of arbitrary bytes: values and scales, and every byte behind the last row."""
    import torch
    rng = np.random.default_rng(T + d + L)
    some = min(L, 3)  # layers that differ
    first = [[_keys(rng, (Hkv, max(before, 1), d)) for _ in range(some)] for _ in "kv"]
    more = [[_keys(rng, (Hkv, T, d)) for _ in range(some)], [_bits(rng, (Hkv, T, d), 40.0) for _ in range(some)]]
    all_layers = lambda x: [x[l % some] for l in range(L)]
    cache = B.Q8Cache.allocate(L, Hkv, rows, d)
    was = _stale(cache, rng)
    st = B.new_status()
    if before:
        B.stepkv_q8_write(cache, _layout(all_layers(first[0]), "heads"), _layout(all_layers(first[1]), "heads"), 0, status=st)
    B.stepkv_q8_write(cache, _layout(all_layers(more[0]), kind), _layout(all_layers(more[1]), kind), before, status=st)
    back = B.stepkv_q8_read(cache, 0, before + T, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for t, (codes, scales, old) in enumerate(((cache.K, cache.K_scale, was[0]), (cache.V, cache.V_scale, was[1]))):
        got, sc, cv = _f64(back[t]), scales.cpu().numpy().astype(np.float64), _codes(codes)
        blocks = -(-(before + T) // 32)
        for l in range(L):
            for h in range(Hkv):
                v, s = np.zeros((rows, d)), np.zeros(-(-rows // 32))
                if before:
                    O.q8_append(v, s, first[t][l % some][h], 0)
                O.q8_append(v, s, more[t][l % some][h], before)
                np.testing.assert_array_equal(got[l, h], v[:before + T])
                np.testing.assert_array_equal(sc[l, h, :blocks], s[:blocks])
                np.testing.assert_array_equal(cv[l, h, :before + T] * np.repeat(s, 32)[:before + T, None], v[:before + T])
                assert np.isnan(sc[l, h, blocks:]).all()
        assert torch.equal(codes.view(torch.uint8)[:, :, before + T:], old[:, :, before + T:])


@pytest.mark.parametrize("d", [64, 128])
def test_special_values(B, d):
    """Blocks that a quantiser can get wrong: ties at every step, values on both sides of a scale's border, zeros, subnormal and
    saturating magnitudes, single large values, infinities and NaN."""
    import torch
    rng = np.random.default_rng(11)
    blocks = []
    for e in (-130, -110, -101, -100, -90, -30, 0, 20, 100, 118, 119):
        blocks.append(rng.choice([-1, 1], (32, d)) * rng.integers(128, 256, (32, d)) * 2.0 ** (e - 7))   # every bf16 mantissa
        x = rng.standard_normal((32, d)) * 2.0 ** e
        x[5, 7] = 448 * 2.0 ** min(e, 118)
        blocks.append(x)
    for top in (448, 446, 450, 224, 225, 223):
        x = rng.integers(-400, 400, (32, d)) / 2.0
        x[np.abs(x) > top] = 0
        x[31, d - 1] = -top
        blocks.append(x)
    x = np.zeros((32, d))
    blocks += [x, -x]
    ties = np.array([(m + 0.5) * 2.0 ** k for k in range(-9, 6) for m in range(8, 16)])     # halfway between two codes
    low = np.array([(m + 0.5) * 2.0 ** -9 for m in range(0, 8)])
    x = np.resize(np.concatenate([ties, -ties, low, -low]), (32, d)).copy()
    x[0, 0] = 400
    blocks.append(x)
    for bad in (np.inf, -np.inf, np.nan):
        x = rng.standard_normal((32, d))
        x[rng.integers(0, 32, 5), rng.integers(0, d, 5)] = bad
        blocks.append(x)
    blocks.append(np.full((32, d), np.nan))
    X = np.concatenate(blocks).astype(np.float32)[None]
    bits = np.where(np.isnan(X), np.uint16(0x7FC1), (X.view(np.uint32) >> 16).astype(np.uint16))
    cache = B.Q8Cache.allocate(1, 1, X.shape[1], d)
    st = B.stepkv_q8_write(cache, [TL.bf16_dev(bits)], [TL.bf16_dev(bits ^ np.uint16(0x8000))], 0)
    Kb, Vb = B.stepkv_q8_read(cache, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    want, scales = O.q8_quantise(bits)
    np.testing.assert_array_equal(cache.K_scale.cpu().numpy()[0], scales)
    np.testing.assert_array_equal(_f64(Kb)[0], want)
    np.testing.assert_array_equal(_f64(Vb)[0], -want)


@pytest.mark.parametrize("d", [64, 128])
def test_tokens_appended_one_at_a_time(B, d):
    """A block filled row by row whose scale grows several times, by factors small and enormous."""
    import torch
    rng = np.random.default_rng(5)
    n = 70
    X = np.stack([_bits(rng, (n, d)) for _ in range(2)])
    for r, f in ((3, 2.0), (9, 2.0 ** 7), (20, 2.0 ** 12), (33, 2.0 ** 60), (40, 2.0 ** 119), (69, 2.0 ** -100)):
        X[:, r] = wl.f32_to_bf16_bits((O.bf16_to_f64(X[:, r]) * f).astype(np.float32))
    cache, st = B.Q8Cache.allocate(1, 2, n, d), B.new_status()
    row, src = torch.zeros(1, dtype=torch.int32, device="cuda"), TL.bf16_dev(X)[None]
    for r in range(n):
        row.fill_(r)
        B.stepkv_q8_write(cache, src[:, :, r:r + 1], src[:, :, r:r + 1], row, status=st)
    Kb, Vb = B.stepkv_q8_read(cache, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0
    for h in range(2):
        v, s = np.zeros((n, d)), np.zeros(3)
        for r in range(n):
            O.q8_append(v, s, X[h, r:r + 1], r)
        for got in (Kb, Vb):
            np.testing.assert_array_equal(_f64(got)[0, h], v)
        np.testing.assert_array_equal(cache.K_scale.cpu().numpy()[0, h], s)


def test_write_by_index_counts_and_rows_on_the_device(B):
    import torch
    rng = np.random.default_rng(6)
    L, Hkv, d, T, rows = 3, 2, 64, 90, 120
    X = [_bits(rng, (Hkv, T, d)) for _ in range(L)]
    lead = [_bits(rng, (Hkv, 40, d)) for _ in range(L)]
    idx = rng.integers(0, T, 50).astype(np.int32)  # in any order, some twice
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    stack = lambda x: torch.stack([TL.bf16_dev(b) for b in x])
    B.stepkv_q8_write(cache, stack(lead), stack(lead), 0, status=st)
    row0 = np.array([0, 17, 40], np.int32)
    n = torch.tensor([37], dtype=torch.int32, device="cuda")
    B.stepkv_q8_write(cache, stack(X), stack(X), _dev(row0), n=n, idx=_dev(idx), status=st)
    Kb, Vb = B.stepkv_q8_read(cache, _dev(row0), n=n, status=st)
    pick = np.array([row0[1] + 36, 3, row0[1] + 5, 3], np.int32)
    Kp, _ = B.stepkv_q8_read(cache.layers(1, 2), idx=_dev(pick), status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and not Kb[:, :, 37:].any()
    for l in range(L):
        for h in range(Hkv):
            v, s = np.zeros((rows, d)), np.zeros(4)
            O.q8_append(v, s, lead[l][h], 0)
            O.q8_append(v, s, X[l][h][idx[:37]], row0[l])
            for got in (Kb, Vb):
                np.testing.assert_array_equal(_f64(got)[l, h, :37], v[row0[l]:row0[l] + 37])
            if l == 1:
                np.testing.assert_array_equal(_f64(Kp)[0, h], v[pick])


@pytest.mark.parametrize("kind", ["count above", "count below", "row0 above", "row0 below", "index"])
def test_bad_data(B, kind):
    """Told in the status word; layers that it does not concern are written and read, the others are left as they are."""
    import torch
    rng = np.random.default_rng(7)
    L, Hkv, d, T, rows = 2, 2, 128, 40, 60
    X = [_bits(rng, (Hkv, T, d)) for _ in range(L)]
    src = torch.stack([TL.bf16_dev(x) for x in X])
    cache = B.Q8Cache.allocate(L, Hkv, rows, d)
    was = _stale(cache, rng)
    n, row0, idx = 30, [0, 0], np.arange(30, dtype=np.int32)
    code = {"count above": B.STEPKV_ENOSPACE, "count below": B.STEPKV_EDATA, "index": B.STEPKV_EDATA}.get(kind, B.STEPKV_ENOSPACE)
    if kind == "count above":
        n = 31
    elif kind == "count below":
        n = -1
    elif kind == "row0 above":
        row0[1] = 31
    elif kind == "row0 below":
        row0[1] = -1
    else:
        idx[[4, 9]] = T, -1
    st = B.stepkv_q8_write(cache, src, src, _dev(np.array(row0, np.int32)), n=_dev(np.array([n], np.int32)), idx=_dev(idx))
    torch.cuda.synchronize()
    assert st.item() == code
    written = [] if kind.startswith("count") else [0] if kind.startswith("row0") else [0, 1]
    for l in range(L):
        if l not in written:
            assert torch.equal(cache.K.view(torch.uint8)[l], was[0][l]) and cache.K_scale[l].isnan().all()
            continue
        for h in range(Hkv):
            x = O.bf16_to_f64(X[l][h][np.clip(idx, 0, T - 1)])
            if kind == "index":
                x[[4, 9]] = 0
            v, s = np.zeros((rows, d)), np.zeros(2)
            O.q8_append(v, s, x, 0)
            np.testing.assert_array_equal(_codes(cache.K)[l, h, :30] * s[0], v[:30])
    # reading
    cache = _filled(B, X, X, rows)
    back = torch.full((L, Hkv, 30, d), 7.0, dtype=torch.bfloat16, device="cuda")
    st = B.new_status()
    if kind == "index":
        idx[[4, 9]] = rows, -1
        B.stepkv_q8_read(cache, idx=_dev(idx), K=back, status=st)
    else:
        B.stepkv_q8_read(cache, _dev(np.array(row0, np.int32)), n=_dev(np.array([n], np.int32)), K=back, status=st)
    torch.cuda.synchronize()
    assert st.item() == (B.STEPKV_ENOSPACE if kind == "count above" else B.STEPKV_EDATA)
    v, _ = O.q8_quantise(X[0])
    if kind.startswith("count"):
        assert (back == 7).all()
    else:
        rest = [r for r in range(30) if kind != "index" or r not in (4, 9)]
        np.testing.assert_array_equal(_f64(back)[0][:, rest], v[:, rest])
        assert (back[0, :, [4, 9]] == 7).all() if kind == "index" else (back[1] == 7).all() or kind == "row0 above"


@pytest.mark.parametrize("row0", [31, 60, 2 ** 31 - 1, -1, -2 ** 31])
def test_rows_outside_the_cache_leave_a_layer_alone(B, row0):
    """One layer of three begins where 30 rows do not fit: its codes and scales, keys and values, and the rows read from it keep
    every byte; the others are written and read."""
    import torch
    rng = np.random.default_rng(18)
    L, Hkv, d, n, rows = 3, 2, 64, 30, 60
    X = [[_bits(rng, (Hkv, n, d)) for _ in range(L)] for _ in "kv"]
    cache = B.Q8Cache.allocate(L, Hkv, rows, d)
    was = _stale(cache, rng)
    at = np.array([0, row0, 30], np.int32)
    cache.K_scale[:, :, 0], cache.V_scale[:, :, 0] = 2.0 ** -100, 2.0 ** -100  # (of the rows before 30)
    scales = [x.clone() for x in (cache.K_scale, cache.V_scale)]
    st = B.stepkv_q8_write(cache, *[torch.stack([TL.bf16_dev(b) for b in x]) for x in X], _dev(at))
    torch.cuda.synchronize()
    assert st.item() == B.STEPKV_ENOSPACE
    back = [torch.full((L, Hkv, n, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    st = B.new_status()
    B.stepkv_q8_read(cache, _dev(at), n, K=back[0], V=back[1], status=st)
    torch.cuda.synchronize()
    assert st.item() == B.STEPKV_EDATA
    for t, (codes, scale) in enumerate(((cache.K, cache.K_scale), (cache.V, cache.V_scale))):
        assert torch.equal(codes.view(torch.uint8)[1], was[t][1]) and torch.equal(scale[1].view(torch.int32), scales[t][1].view(torch.int32))
        assert (back[t][1] == 7).all()
        assert torch.equal(codes.view(torch.uint8)[0, :, n:], was[t][0, :, n:])
        np.testing.assert_array_equal(_f64(back[t])[0], _values(X[t][0]))
        for h in range(Hkv):
            v, s = O.e4m3_values(was[t][2, h].cpu().numpy()) * 2.0 ** -100, np.array([2.0 ** -100, 0.0])
            O.q8_append(v, s, X[t][2][h], 30)
            np.testing.assert_array_equal(_f64(back[t])[2, h], v[30:])
            np.testing.assert_array_equal(scale.cpu().numpy()[2, h], s)


@pytest.mark.parametrize("order", ["lhnd", "nlhd", "hlnd", "lnhd"])
def test_read_into_any_order_of_axes(B, order):
    import torch
    rng = np.random.default_rng(8)
    L, Hkv, n, d = 3, 2, 45, 64
    X = [_bits(rng, (Hkv, n, d)) for _ in range(L)]
    cache = _filled(B, X, X)
    dims = dict(l=L, h=Hkv, n=n, d=d)
    whole = torch.full([dims[a] for a in order], 7.0, dtype=torch.bfloat16, device="cuda")
    view = whole.permute([order.index(a) for a in "lhnd"])
    _, V = B.stepkv_q8_read(cache, K=None, V=view)
    np.testing.assert_array_equal(_f64(V), np.stack([O.q8_quantise(x)[0] for x in X]))


def test_broadcast_rows(B):
    """One head's rows for all heads, one row for all tokens: strides of 0 on the side that is read."""
    import torch
    rng = np.random.default_rng(9)
    X, Y = _bits(rng, (1, 50, 64)), _bits(rng, (2, 1, 64))
    cache = B.Q8Cache.allocate(2, 2, 50, 64)
    K, V = TL.bf16_dev(X).expand(2, 2, 50, 64), TL.bf16_dev(Y).expand(2, 2, 50, 64)
    B.stepkv_q8_write(cache, K, K, 0)
    got = B.stepkv_q8_read(cache)[0]
    np.testing.assert_array_equal(_f64(got), np.broadcast_to(O.q8_quantise(X)[0], (2, 2, 50, 64)))
    B.stepkv_q8_write(cache, V, V, 0)
    got = B.stepkv_q8_read(cache)[1]
    np.testing.assert_array_equal(_f64(got), np.broadcast_to(O.q8_quantise(np.repeat(Y, 50, 1))[0], (2, 2, 50, 64)))


# ------------------------------------------------------------------------------------------------ decode
def _decode_bound(q, K, V):
    """Per head and channel: what fp32 arithmetic may lose of out = sum_j p_j V_j / sum_j p_j.

    A logit is a sum of d exact products of a query element, held to 22 bits of the head's largest, and a code, summed in fp32 in
    up to d / 16 steps of half an ulp (a tensor core's own steps truncate: an ulp): off by at most 2^-22 scale (max|q| sum|k| +
    sum|q||k|) =: e (the steps' part: d / 16 2^-23 <= 2^-20 of sum|q||k| in the worst order, of which a quarter is left where
    partial sums grow evenly: 2^-22).  exp of it is off by e and by 2^-20 (an exponential of 2^-22, a weight in 22 bits, the
    rescalings of the maximum), and a weighted sum of n terms in blocks of 32 by (n / 16 + 64) 2^-24.  Numerator and
    denominator: twice that, of sum_j p_j |V_j|.  A weight's last place is 2^-38 of the largest, so that each key may be off by
    2^-38 |V_j| however small its weight."""
    G, scale = q.shape[0] // K.shape[0], 1 / math.sqrt(q.shape[1])
    qf = O.bf16_to_f64(q)
    out = np.zeros(qf.shape)
    for g in range(qf.shape[0]):
        k, v = np.abs(K[g // G]), np.abs(V[g // G])
        e = _logit_bound(qf[g], K[g // G])
        x = K[g // G] @ qf[g] * scale
        p = np.exp(x - x.max())
        out[g] = (p / p.sum()) @ v * 2 * (e + 2.0 ** -20 + (len(k) / 16 + 64) * 2.0 ** -24) + 2.0 ** -38 * v.sum(0)
    return out


def _logit_bound(qf, K):
    k = np.abs(K)
    return (2.0 ** -22 / math.sqrt(K.shape[1]) * (np.abs(qf).max() * k.sum(1) + k @ np.abs(qf))).max()


def _mass_bound(q, K, mass):
    """Of mass + weight, weight = mean over G heads of p_j / l: a weight is off by 2 (e + 2^-20) of itself as above, and by the
    rounding of x - m, 2^-24 max|x| log2(e) of itself; sums and products of the G heads by (G + 3) 2^-24; the sum with the mass
    rounds by 2^-24 of it."""
    G, scale = q.shape[0] // K.shape[0], 1 / math.sqrt(q.shape[1])
    qf = O.bf16_to_f64(q)
    out = np.zeros(K.shape[:2])
    for g in range(qf.shape[0]):
        x = K[g // G] @ qf[g] * scale
        p = np.exp(x - x.max())
        rel = 2 * (_logit_bound(qf[g], K[g // G]) + 2.0 ** -20 + (len(x) / 16 + 64) * 2.0 ** -24) + 2.0 ** -23 * np.abs(x).max() + (G + 3) * 2.0 ** -24
        out[g // G] += p / p.sum() * rel / G
    return out + 2.0 ** -24 * (np.abs(mass) + O.attention_weights(q, K)) + 1e-37


def _values(X):
    return O.q8_quantise(X)[0]


def _check(got, q, K, V, n, what, mass=None, mass0=None):
    """One cache's outputs (and masses) against the oracle over its first n rows; K, V: values the codes stand for."""
    got = got.cpu().numpy().astype(np.float64)
    if mass is not None:
        m, m0 = mass.cpu().numpy().astype(np.float64), mass0.cpu().numpy().astype(np.float64)
        np.testing.assert_array_equal(m[:, n:], m0[:, n:])
    if n == 0:
        assert not got.any(), what
        return
    K, V = K[:, :n], V[:, :n]
    err, bound = np.abs(got - O.q4_decode_attention(q, K, V)), _decode_bound(q, K, V)
    assert (err <= bound).all(), f"{what}: off by {np.nanmax(err / bound):.3g} times the bound"
    if mass is not None:
        err, bound = np.abs(m[:, :n] - m0[:, :n] - O.attention_weights(q, K)), _mass_bound(q, K, m0[:, :n])
        assert (err <= bound).all(), f"{what}: masses off by {np.nanmax(err / bound):.3g} times the bound"


DECODE_CASES = [  # L, Hkv, G, d, n, rows, key scale
    (1, 1, 1, 64, 1, 1, 1.0), (1, 2, 4, 128, 1, 1, 1.0), (2, 2, 4, 128, 15, 15, 1.0), (1, 2, 4, 128, 16, 16, 1.0),
    (1, 2, 4, 128, 17, 40, 1.0), (1, 2, 3, 64, 31, 31, 1.0), (1, 1, 2, 64, 32, 32, 1.0), (1, 2, 8, 128, 33, 33, 1.0),
    (2, 3, 5, 128, 63, 65, 2.0), (1, 2, 6, 64, 64, 64, 1.0), (1, 2, 7, 128, 129, 130, 1.0), (3, 2, 1, 128, 1000, 1003, 1.0),
    (2, 2, 4, 64, 2049, 2100, 2.0), (1, 8, 4, 128, 8272, 8911, 1.0), (1, 2, 8, 64, 5001, 5001, 3.0), (1, 1, 5, 128, 30011, 30011, 1.0),
    (32, 8, 4, 128, 81, 90, 1.0), (12, 8, 1, 128, 700, 701, 1.0), (3, 64, 2, 64, 2000, 2000, 1.0), (66, 1, 4, 64, 50, 52, 1.0)]


@pytest.mark.parametrize("L,Hkv,G,d,n,rows,ks", DECODE_CASES)
def test_decode_matches_oracle(B, L, Hkv, G, d, n, rows, ks):
    """Rows at or past n hold arbitrary codes and NaN scales.  With masses the output is the same, bit for bit."""
    import torch
    rng = np.random.default_rng(100 + n + d + G)
    some = min(L, 3)
    q = [_bits(rng, (Hkv * G, d), ks) for _ in range(some)]
    K, V = [_keys(rng, (Hkv, n, d)) for _ in range(some)], [_bits(rng, (Hkv, n, d)) for _ in range(some)]
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    _stale(cache, rng)
    stack = lambda X: [TL.bf16_dev(X[l % some]) for l in range(L)]
    B.stepkv_q8_write(cache, stack(K), stack(V), 0, status=st)
    mass0 = torch.rand((L, Hkv, rows + 3), device="cuda")
    mass = mass0.clone()
    a = B.stepkv_q8_decode(stack(q), cache, n, status=st)
    b = B.stepkv_q8_decode(torch.stack(stack(q)), cache, torch.tensor([n], dtype=torch.int32, device="cuda"), status=st)
    c = B.stepkv_q8_decode(torch.stack(stack(q)), cache, n, mass=list(mass), status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and torch.equal(torch.stack(a), b) and torch.equal(b, c)
    Kv, Vv = [_values(x) for x in K], [_values(x) for x in V]
    for l in sorted({0, L - 1, L // 2}):
        _check(a[l], q[l % some], Kv[l % some], Vv[l % some], n, f"layer {l}", mass[l], mass0[l])


FORMS = [  # L, Hkv, G, d, rows: few pairs and many, short and long
    (1, 3, 3, 64, 500), (5, 7, 1, 128, 700), (33, 14, 2, 64, 300), (60, 9, 5, 128, 200), (31, 3, 1, 64, 2100), (23, 5, 3, 128, 1700),
    (64, 9, 1, 64, 1800), (57, 8, 1, 64, 1000), (9, 7, 4, 64, 4000), (2, 2, 2, 128, 9000), (66, 3, 2, 64, 2100), (64, 32, 8, 128, 40)]


@pytest.mark.parametrize("L,Hkv,G,d,rows", FORMS)
def test_decode_forms_and_counts(B, L, Hkv, G, d, rows):
    """Caches of the same rows under one count, long, short and zero, and under counts of their own: whatever way the work is
    divided, each output and mass is within its bound of the oracle's."""
    import torch
    rng = np.random.default_rng(L + rows)
    K, V, q = _keys(rng, (Hkv, rows, d)), _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv * G, d))
    Kv, Vv = _values(K), _values(V)
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    B.stepkv_q8_write(cache, *[TL.bf16_dev(x)[None].expand(L, -1, -1, -1) for x in (K, V)], 0, status=st)
    qd = TL.bf16_dev(q).expand(L, -1, -1).contiguous()
    own = rng.integers(0, rows + 1, L).astype(np.int32)
    own[rng.integers(0, L, 3)] = 0, rows, 1
    for counts in (rows, rows - 33, 75, 1, 0, own, np.minimum(own, 40)):
        n = _dev(np.minimum(np.atleast_1d(np.asarray(counts, np.int32)), rows))
        out, mass = torch.full((L, Hkv * G, d), 7.0, device="cuda"), torch.full((L, Hkv, rows), 0.5, device="cuda")
        B.stepkv_q8_decode(qd, cache, n, out=out, status=st)
        again = B.stepkv_q8_decode(qd, cache, n, mass=mass, status=st)
        torch.cuda.synchronize()
        assert st.item() == 0 and torch.equal(out, again)
        each = np.minimum(np.broadcast_to(counts, (L,)), rows)
        half = torch.full((Hkv, rows), 0.5)
        for m in sorted(set(each)) if L < 10 else sorted({each[0], each[L // 2], each[-1], each.min(), each.max()}):
            same = np.flatnonzero(each == m)
            _check(out[same[0]], q, Kv, Vv, int(m), f"{m} of {counts}, cache {same[0]}", mass[same[0]], half)
            if m:
                bound = 2 * _dev(_decode_bound(q, Kv[:, :m], Vv[:, :m]))
                assert all(((out[l] - out[same[0]]).abs() <= bound).all() for l in same)
                bound = 2 * _dev(_mass_bound(q, Kv[:, :m], np.full((Hkv, m), 0.5)))
                assert all(((mass[l] - mass[same[0]])[:, :m].abs() <= bound).all() for l in same)
            else:
                assert not out[same].any()


@pytest.mark.parametrize("L,Hkv,G,d,rows,some", [(64, 8, 4, 128, 1700, [1700, 33, 1, 300]), (64, 8, 8, 64, 1600, [5, 1600, 64, 65, 1, 31]),
                                                 (60, 16, 1, 64, 2000, [2000]), (64, 32, 2, 64, 1700, [1, 2, 3, 1, 200, 64, 30, 1699])])
def test_decode_batches_of_mostly_empty_caches(B, L, Hkv, G, d, rows, some):
    """More pairs than CTAs of which few have keys, where the caches might all be long: single warps take the ranges."""
    import torch
    rng = np.random.default_rng(L + rows + G)
    K, V, q = _keys(rng, (Hkv, rows, d)), _bits(rng, (Hkv, rows, d)), _bits(rng, (Hkv * G, d))
    Kv, Vv = _values(K), _values(V)
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    B.stepkv_q8_write(cache, *[TL.bf16_dev(x)[None].expand(L, -1, -1, -1) for x in (K, V)], 0, status=st)
    qd = TL.bf16_dev(q).expand(L, -1, -1).contiguous()
    n = np.zeros(L, np.int32)
    n[rng.permutation(L)[:len(some)]] = some
    for counts in (n, np.sort(n), np.sort(n)[::-1]):
        nd = _dev(counts.copy())
        mass0 = torch.rand((L, Hkv, rows), device="cuda")
        mass, out = mass0.clone(), torch.full((L, Hkv * G, d), 7.0, device="cuda")
        B.stepkv_q8_decode(qd, cache, nd, out=out, status=st)
        again = B.stepkv_q8_decode(qd, cache, nd, mass=mass, status=st)
        torch.cuda.synchronize()
        assert st.item() == 0 and torch.equal(out, again)
        for l in range(L):
            if counts[l]:
                _check(out[l], q, Kv, Vv, int(counts[l]), f"cache {l} of {counts[l]}", mass[l], mass0[l])
        empty = torch.from_numpy(counts == 0)
        assert not out[empty].any() and torch.equal(mass[empty], mass0[empty])


@pytest.mark.parametrize("magnitude", [2.0 ** -110, 2.0 ** -90, 1e-20, 1e-3, 1.0, 1e3, 1e20, 2.0 ** 90, 2.0 ** 118])
def test_decode_keys_queries_and_values_of_any_magnitude(B, magnitude):
    """Keys of any magnitude with queries that make up for it; and values of it."""
    import torch
    rng = np.random.default_rng(9)
    K, V, q = _bits(rng, (2, 300, 128), magnitude), _bits(rng, (2, 300, 128), magnitude), _bits(rng, (6, 128), 1 / magnitude)
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), 300)[0]
    torch.cuda.synchronize()
    _check(out, q, _values(K), _values(V), 300, "")


@pytest.mark.parametrize("G,d,n", [(4, 64, 1), (8, 128, 45), (3, 128, 33), (4, 128, 3000), (5, 64, 700)])
@pytest.mark.parametrize("e", [20, 24, 25, 26, 27, 28, 31, 60, 100])
def test_decode_logits_beyond_a_unit_of_32_bits(B, e, G, d, n):
    """Logits of some 2^e (the heavy keys of one head) and -2^e (of the other), whose neighbours in 32 bits are 2^(e - 23) apart:
    keys that are the same have the same logit whatever it is rounded to, and share all the weight where the others' lie 2^e
    below.  What then rounds are the weights (2^-20 relative), their sum and the weighted sum, as in _decode_bound and
    _mass_bound."""
    import torch
    rng = np.random.default_rng(19)
    half, Hkv = e // 2, 2
    heavy = np.arange(n) % 3 != 1 if n > 1 else np.ones(1, bool)
    K = np.stack([np.where(heavy, 1.0, -1.0), np.where(heavy, -1.0, -2.0)])[:, :, None] * np.full(d, 2.0 ** (e - half - int(math.log2(d)) // 2))
    q = np.tile(np.repeat(2.0 ** half * (1 + np.arange(G) / 8), d).reshape(G, d), (Hkv, 1))
    K, V, q = wl.f32_to_bf16_bits(K.astype(np.float32)), _bits(rng, (Hkv, n, d)), wl.f32_to_bf16_bits(q.astype(np.float32))
    mass, st = torch.zeros((1, Hkv, n), device="cuda"), B.new_status()
    cache = _filled(B, [K], [V])
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], cache, n, mass=mass, status=st)[0].cpu().numpy()
    torch.cuda.synchronize()
    assert st.item() == 0
    some = heavy.sum()
    for h in range(Hkv):
        v = _values(V)[h, heavy]
        bound = 2 * (2.0 ** -20 + (n / 16 + 64) * 2.0 ** -24) * np.abs(v).mean(0) + 2.0 ** -38 * np.abs(v).sum(0)
        assert (np.abs(out[h * G:(h + 1) * G] - v.mean(0)) <= bound).all()
        m = mass[0, h].cpu().numpy()
        assert (np.abs(m - heavy / some) <= (2.0 ** -19 + (n / 8 + 128 + G + 3) * 2.0 ** -24) / some).all()


def test_decode_blocks_of_different_magnitude(B):
    """Blocks whose scales differ by up to 2^40, keys and values alike."""
    import torch
    rng = np.random.default_rng(10)
    f = np.exp2(rng.integers(-20, 21, 20)).repeat(32)[:630, None]
    f2 = np.exp2(rng.integers(-20, 3, 20)).repeat(32)[:630, None]
    K = wl.f32_to_bf16_bits((rng.standard_normal((2, 630, 64)) * f2).astype(np.float32))
    V = wl.f32_to_bf16_bits((rng.standard_normal((2, 630, 64)) * f).astype(np.float32))
    q = _bits(rng, (10, 64))
    mass = torch.zeros((1, 2, 630), device="cuda")
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), 630, mass=mass)[0]
    torch.cuda.synchronize()
    _check(out, q, _values(K), _values(V), 630, "", mass[0], torch.zeros_like(mass[0]))


def test_decode_peaked_and_flat_rows(B):
    """All weight on one key, far apart from the others, and weights that are all the same."""
    import torch
    rng = np.random.default_rng(12)
    n, d = 1000, 128
    for at in (0, 31, 32, 517, 999):
        k = rng.standard_normal((1, n, d)) * 0.1
        qf = rng.standard_normal((4, d))
        k[0, at] = qf[0] * 12
        K, V, q = (wl.f32_to_bf16_bits(x.astype(np.float32)) for x in (k, rng.standard_normal((1, n, d)), qf))
        mass = torch.zeros((1, 1, n), device="cuda")
        out = B.stepkv_q8_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n, mass=mass)[0]
        _check(out, q, _values(K), _values(V), n, f"peak at {at}", mass[0], torch.zeros_like(mass[0]))
    K, V, q = np.zeros((1, n, d), np.uint16), _bits(rng, (1, n, d)), _bits(rng, (4, d))
    mass = torch.zeros((1, 1, n), device="cuda")
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n, mass=mass)[0]
    _check(out, q, _values(K), _values(V), n, "flat", mass[0], torch.zeros_like(mass[0]))


@pytest.mark.parametrize("G", [3, 8])
@pytest.mark.parametrize("Hkv,d,n", [(2, 128, 60), (2, 64, 3001), (64, 128, 700)])
@pytest.mark.parametrize("kind", ["nan key", "inf key", "nan value", "inf query", "nan query"])
def test_decode_non_finite(B, Hkv, d, n, G, kind):
    """What is not a number reaches the outputs that it enters, and no other."""
    import torch
    rng = np.random.default_rng(13)
    K, V, q = _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv, n, d)), _bits(rng, (Hkv * G, d))
    nan, inf = np.uint16(0x7FC0), np.uint16(0x7F80)
    clean = [x.copy() for x in (K, V, q)]
    bad = np.zeros((Hkv * G, d), bool)
    if kind.endswith("key"):
        K[1, n // 2, 3] = nan if kind.startswith("nan") else inf
        bad[G:2 * G] = True
    elif kind == "nan value":
        V[0, n // 3, 7] = nan
        bad[:G, 7] = True
    else:
        q[G + 1, 5] = nan if kind.startswith("nan") else inf
        bad[G + 1] = True
    mass = torch.zeros((1, Hkv, n), device="cuda")
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], _filled(B, [K], [V]), n, mass=mass)[0].cpu().numpy()
    np.testing.assert_array_equal(np.isnan(out), bad)
    Kv, Vv = _values(clean[0]), _values(clean[1])
    want, bound = O.q4_decode_attention(clean[2], Kv, Vv), _decode_bound(clean[2], Kv, Vv)
    assert (np.abs(out - want) <= bound)[~bad].all()
    m = mass[0].cpu().numpy()
    sick = np.zeros(Hkv, bool) if kind == "nan value" else np.arange(Hkv) == 1
    assert np.isnan(m[sick]).all()
    assert (np.abs(m - O.attention_weights(clean[2], Kv)) <= _mass_bound(clean[2], Kv, np.zeros((Hkv, n))))[~sick].all()


@pytest.mark.parametrize("each", [False, True])
def test_decode_bad_counts(B, each):
    import torch
    rng = np.random.default_rng(14)
    L, Hkv, G, d, rows = 3, 2, 4, 64, 100
    K, V, q = ([_bits(rng, s) for _ in range(L)] for s in ((Hkv, rows, d), (Hkv, rows, d), (Hkv * G, d)))
    cache = _filled(B, K, V)
    qd = torch.stack([TL.bf16_dev(x) for x in q])
    for bad, code in ((rows + 1, B.STEPKV_ENOSPACE), (2 ** 31 - 1, B.STEPKV_ENOSPACE), (-1, B.STEPKV_EDATA), (-2 ** 31, B.STEPKV_EDATA)):
        n = _dev(np.array([50, bad, 20] if each else [bad], np.int32))
        mass, st = torch.zeros((L, Hkv, rows), device="cuda"), B.new_status()
        out = B.stepkv_q8_decode(qd, cache, n, mass=mass, status=st)
        torch.cuda.synchronize()
        assert st.item() == code
        used = rows if bad > 0 else 0
        for l, m in enumerate([50, used, 20] if each else [used] * L):
            _check(out[l], q[l], _values(K[l]), _values(V[l]), m, f"layer {l}", mass[l], torch.zeros_like(mass[l]))


def test_strided_caches(B):
    """Layers, heads and rows of larger buffers: other strides between heads for codes and scales, layers inside heads."""
    import torch
    rng = np.random.default_rng(15)
    L, Hkv, G, d, n = 2, 3, 4, 64, 77
    K, V, q = ([_bits(rng, s) for _ in range(L)] for s in ((Hkv, n, d), (Hkv, n, d), (Hkv * G, d)))
    f8 = torch.float8_e4m3fn
    big = torch.zeros((2, Hkv, L, 90, d), dtype=f8, device="cuda")
    scales = torch.full((2, Hkv, L, 5), float("nan"), device="cuda")
    view = lambda x, t, rows: [x[t, :, l, :rows] for l in range(L)]
    cache = B.Q8Cache(view(big, 0, n), view(scales, 0, 3), view(big, 1, n), view(scales, 1, 3))
    masses = torch.zeros((Hkv, L, 100), device="cuda")
    st = B.stepkv_q8_write(cache, [TL.bf16_dev(x) for x in K], [TL.bf16_dev(x) for x in V], 0)
    out = B.stepkv_q8_decode([TL.bf16_dev(x) for x in q], cache, n, mass=masses.transpose(0, 1), status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and scales[..., 3:].isnan().all() and not big[:, :, :, n:].float().any()
    for l in range(L):
        _check(out[l], q[l], _values(K[l]), _values(V[l]), n, f"layer {l}", masses[:, l], torch.zeros((Hkv, 100)))


def test_offsets_past_32_bits(B):
    """34 million rows of one head: 4.35 GB of codes.  All but the last 40 are zero keys and values, whose logits of 0 are at
    least 30 below the others' (weights of 34e6 e^-30 < 2^-18 2^-3 together, within the bound's 2 2^-20); the last rows are
    written, read back and attended where offsets need more than 32 bits."""
    import torch
    rng = np.random.default_rng(41)
    rows, n, d = 34_000_000, 40, 128
    assert rows * d > 2 ** 32
    cache = B.Q8Cache.allocate(1, 1, rows, d)
    cache.K_scale.fill_(2.0 ** -100), cache.V_scale.fill_(2.0 ** -100)
    base = rng.standard_normal(d)
    bits = lambda x: wl.f32_to_bf16_bits(np.asarray(x, np.float32))
    q = bits(base * np.array([[1.0], [0.9], [1.1], [1.2]]))
    K, V = bits(6 * np.sign(base) + 0.5 * rng.standard_normal((1, n, d))), _bits(rng, (1, n, d))
    st = B.stepkv_q8_write(cache, [TL.bf16_dev(K)], [TL.bf16_dev(V)], rows - n)
    back, _ = B.stepkv_q8_read(cache, rows - n, n, status=st)
    mass = torch.zeros((1, 1, rows), device="cuda")
    out = B.stepkv_q8_decode([TL.bf16_dev(q)], cache, rows, mass=mass, status=st)[0]
    assert st.item() == 0
    lead = (rows - n) % 32
    v, s = np.zeros((2, 96, d)), np.full((2, 3), 2.0 ** -100)
    O.q8_append(v[0], s[0], K[0], lead)
    O.q8_append(v[1], s[1], V[0], lead)
    Kv, Vv = v[0, lead:lead + n][None], v[1, lead:lead + n][None]
    np.testing.assert_array_equal(_f64(back)[0], Kv)
    assert (Kv[0] @ O.bf16_to_f64(q).T / math.sqrt(d)).min() > 30
    m = mass[:, :, -n:]
    _check(out, q, Kv, Vv, n, "", m[0], torch.zeros_like(m[0]))
    assert mass[:, :, :-n].max() < 2.0 ** -40


def test_two_streams_at_once(B):
    import torch
    rng = np.random.default_rng(16)
    sets = []
    for i in range(2):
        K, V, q = _bits(rng, (4, 900 + i, 128)), _bits(rng, (4, 900 + i, 128)), _bits(rng, (16, 128))
        cache = _filled(B, [K], [V])
        sets.append((K, V, q, cache, torch.cuda.Stream(), B.q8_decode_workspace(cache, 16, True), torch.zeros((1, 4, 900 + i), device="cuda")))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, (K, V, q, cache, stream, ws, mass) in enumerate(sets):
            with torch.cuda.stream(stream):
                outs[i].append(B.stepkv_q8_decode([TL.bf16_dev(q)], cache, 900 + i, mass=mass, ws=ws)[0])
    torch.cuda.synchronize()
    for i, (K, V, q, cache, stream, ws, mass) in enumerate(sets):
        assert all(torch.equal(o, outs[i][0]) for o in outs[i])
        _check(outs[i][0], q, _values(K), _values(V), 900 + i, f"stream {i}")
        assert abs(mass.sum().item() / (20 * 4) - 1) < 1e-4  # (each call adds 1 a head)


def test_captured_steps_replay_with_new_counts(B):
    """Two captured steps (append a token, attend with masses) of one cache that share nothing but it, replayed in turn as it grows
    across blocks; the counts are on the device."""
    import torch
    rng = np.random.default_rng(17)
    L, Hkv, G, d, n0, steps = 2, 2, 4, 128, 25, 50
    rows = n0 + steps
    K, V = ([_bits(rng, (Hkv, rows, d)) for _ in range(L)] for _ in "kv")
    q = [_bits(rng, (Hkv * G, d)) for _ in range(L)]
    Kd, Vd = torch.stack([TL.bf16_dev(x) for x in K]), torch.stack([TL.bf16_dev(x) for x in V])
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    B.stepkv_q8_write(cache, Kd[:, :, :n0], Vd[:, :, :n0], 0, status=st)
    row, count = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in "rn")
    row.fill_(n0), count.fill_(n0)
    tk, tv = (torch.zeros((L, Hkv, 1, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    qd = torch.stack([TL.bf16_dev(x) for x in q])
    graphs, outs, masses = [], [], []
    for _ in range(2):
        out, mass, ws = torch.zeros((L, Hkv * G, d), device="cuda"), torch.zeros((L, Hkv, rows), device="cuda"), B.q8_decode_workspace(cache, Hkv * G, True)

        def step():
            B.stepkv_q8_write(cache, tk, tv, row, status=st)
            B.stepkv_q8_decode(qd, cache, count, out=out, mass=mass, ws=ws, status=st)

        tk.copy_(Kd[:, :, n0:n0 + 1]), tv.copy_(Vd[:, :, n0:n0 + 1])
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        mass.zero_()
        graphs.append(graph), outs.append(out), masses.append(mass)
    v = [[[np.zeros((rows, d)), np.zeros(-(-rows // 32))] for h in range(Hkv)] for l in range(L)]
    vv = [[[np.zeros((rows, d)), np.zeros(-(-rows // 32))] for h in range(Hkv)] for l in range(L)]
    want, bound = np.zeros((2, L, Hkv, rows)), np.zeros((2, L, Hkv, rows))
    for t in range(n0, rows):
        row.fill_(t), count.fill_(t + 1)
        tk.copy_(Kd[:, :, t:t + 1]), tv.copy_(Vd[:, :, t:t + 1])
        graphs[t & 1].replay()
        for l in range(L):
            for h in range(Hkv):
                for x, src in ((v, K), (vv, V)):
                    if t == n0:
                        O.q8_append(*x[l][h], src[l][h][:n0], 0)
                    O.q8_append(*x[l][h], src[l][h][t:t + 1], t)
        torch.cuda.synchronize()
        for l in range(L):
            Kv, Vv = (np.stack([x[l][h][0][:t + 1] for h in range(Hkv)]) for x in (v, vv))
            want[t & 1, l, :, :t + 1] += O.attention_weights(q[l], Kv)
            bound[t & 1, l, :, :t + 1] += _mass_bound(q[l], Kv, want[t & 1, l, :, :t + 1])
            if t % 7 == 0 or t == rows - 1:
                _check(outs[t & 1][l], q[l], Kv, Vv, t + 1, f"token {t}, layer {l}")
    assert st.item() == 0
    for i in range(2):
        assert (np.abs(masses[i].cpu().numpy() - want[i]) <= 1.001 * bound[i]).all()  # (a mass that is off rounds like one that is not)


def test_what_a_call_makes_belongs_to_its_stream(B):
    """Calls on a stream while the current one is busy: the status, rows and workspace that they make are neither cleared nor
    handed out again by what the current stream does late."""
    import torch
    rng = np.random.default_rng(34)
    Hkv, G, d, n = 2, 4, 64, 600
    K, V = ([_bits(rng, (Hkv, n, d))] for _ in range(2))
    cache = _filled(B, K, V)
    src, q = TL.bf16_dev(K[0])[None], _bits(rng, (Hkv * G, d))
    qd = TL.bf16_dev(q)[None]
    count, row0 = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (n - 7, 1))
    mass = torch.zeros((1, Hkv, n), device="cuda")
    side = torch.cuda.Stream()
    B.stepkv_q8_decode(qd, cache, n, mass=mass.clone()), B.stepkv_q8_read(cache, n=count), B.stepkv_q8_write(cache, src, src, 0)
    cache = _filled(B, K, V)
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)  # some 25 ms on the current stream
    st = B.stepkv_q8_write(cache, src, src, row0, stream=side)  # a row too many
    Kb, Vb = B.stepkv_q8_read(cache, n=count, stream=side)
    out = B.stepkv_q8_decode(qd, cache, count, mass=mass, stream=side)
    made = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert st.item() == B.STEPKV_ENOSPACE and not made.any()
    for got, X in ((Kb, K), (Vb, V)):
        np.testing.assert_array_equal(_f64(got[0, :, :n - 7]), _values(X[0])[:, :n - 7])
        assert not got[0, :, n - 7:].any()
    _check(out[0], q, _values(K[0]), _values(V[0]), n - 7, "on its own stream", mass[0], torch.zeros_like(mass[0]))


def test_empty_calls(B):
    import torch
    cache = B.Q8Cache.allocate(2, 2, 40, 64)
    none = torch.zeros((2, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    st = B.stepkv_q8_write(cache, none, none, 40)
    K, V = B.stepkv_q8_read(cache, 40, 0, status=st)
    assert K.shape == (2, 2, 0, 64) and V.shape == K.shape
    one = torch.ones((2, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.stepkv_q8_write(cache, one, one, 0, n=zero, status=st)
    q = torch.ones((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    mass = torch.ones((2, 2, 40), device="cuda")
    out = B.stepkv_q8_decode(q, cache, 0, mass=mass, status=st)
    assert not out.any() and (mass == 1).all() and st.item() == 0 and not cache.K.float().any()


def test_binding_refusals(B):
    import torch
    f8, bf = torch.float8_e4m3fn, torch.bfloat16
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
    K, S = z(1, 2, 40, 64, t=f8), z(1, 2, 2)
    cache = B.Q8Cache(K, S, K.clone(), S.clone())
    for bad in ((K[..., :32], S, K, S), (K, S[..., :1], K, S), (K, S, K[:, :1], S), (K, S.double(), K, S), (K.view(torch.uint8), S, K, S),
                (K, S, z(2, 2, 40, 64, t=f8), S), (z(1, 2, 40, 128, t=f8)[..., ::2], S, K, S)):
        with pytest.raises((ValueError, TypeError)):
            B.Q8Cache(*bad)
    x = z(1, 2, 5, 64, t=bf)
    for call in (lambda: B.stepkv_q8_write(cache, x, None, 0), lambda: B.stepkv_q8_write(cache, x, x[:, :1], 0),
                 lambda: B.stepkv_q8_write(cache, x.float(), x.float(), 0), lambda: B.stepkv_q8_write(cache, x, x, 0, n=6),
                 lambda: B.stepkv_q8_write(cache, x, x, 2 ** 31), lambda: B.stepkv_q8_read(cache, 0, 6, K=x, V=x),
                 lambda: B.stepkv_q8_read(cache, 0, 5, K=z(1, 2, 5, 32, t=bf)),
                 lambda: B.stepkv_q8_decode(z(1, 8, 32, t=bf), cache, 5), lambda: B.stepkv_q8_decode(z(2, 8, 64, t=bf), cache, 5),
                 lambda: B.stepkv_q8_decode(z(1, 8, 64, t=bf), cache, z(2, t=torch.int32).long()),
                 lambda: B.stepkv_q8_decode(z(1, 8, 64, t=bf), cache, z(3, t=torch.int32)),
                 lambda: B.stepkv_q8_decode(z(1, 8, 64, t=bf), cache, 5, mass=z(1, 2, 39)),
                 lambda: B.stepkv_q8_decode(z(1, 8, 64, t=bf), cache, 2 ** 33)):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: B.stepkv_q8_write(cache, x, x, 36), lambda: B.stepkv_q8_read(cache, 0, 41), lambda: B.stepkv_q8_decode(z(1, 18, 64, t=bf), cache, 5),
                 lambda: B.stepkv_q8_decode(z(1, 8, 64, t=bf), cache, 41), lambda: B.stepkv_q8_write(B.Q8Cache(K, S, K, S), x, x, 0)):
        with pytest.raises(B.StepKVError):
            call()
