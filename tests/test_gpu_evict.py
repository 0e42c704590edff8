"""GPU parity of eviction by accumulated attention against the oracle, through the public entry points.

Which rows stay, where they go, their bytes, masses and positions have one right answer, and so have the codes of an 8-bit
cache: everything is compared value for value.
"""
import numpy as np
import pytest

from oracle import stepkv_oracle as O
from paper_2609_22158_gb300 import workload as wl
import stepkv_testlib as TL
import test_gpu_q8 as Q

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


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _f64(t):
    return O.bf16_to_f64(TL.bits_of(t.contiguous()))


MASSES = ["long tail", "ties", "special", "one value"]


def _mass(rng, shape, kind):
    m = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        m = rng.integers(0, 4, shape).astype(np.float32) / 2
    elif kind == "special":
        pick = rng.integers(0, 9, shape)
        for i, v in enumerate((np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42, -1.0)):
            m[pick == i] = v
    elif kind == "one value":
        m[...] = 0.25
    return m


def _pos(rng, shape, ordered):
    """Distinct positions with gaps, ascending or in any order."""
    L, Hkv, rows = shape
    p = np.cumsum(rng.integers(1, 4, shape), -1) - 1
    if not ordered:
        p = rng.permuted(p, axis=-1)
    return p.astype(np.int32)


class _Case:
    """One call's tensors, and what they have to be afterwards."""

    def __init__(self, rng, L, Hkv, d, rows, n, keep, sink, recent, kind, ordered, width=None):
        width = width or rows
        self.L, self.Hkv, self.d, self.rows, self.keep, self.sink, self.recent = L, Hkv, d, rows, keep, sink, recent
        self.n = np.broadcast_to(n, (L,))
        self.mass, self.pos = _mass(rng, (L, Hkv, width), kind), _pos(rng, (L, Hkv, width), ordered)
        self.md, self.pd = _dev(self.mass), _dev(self.pos)
        self.moves = [[O.evict_moves(self.mass[l, h, :self.n[l]], self.pos[l, h, :self.n[l]], keep, sink, recent) for h in range(Hkv)]
                      for l in range(L)]

    def check_book(self):
        """Masses bit for bit (the NaN's too), positions, and what lies behind the rows."""
        mass, pos = self.mass.copy(), self.pos.copy()
        for l in range(self.L):
            for h in range(self.Hkv):
                to, start = self.moves[l][h]
                mass[l, h, to], pos[l, h, to] = self.mass[l, h, start], self.pos[l, h, start]
                if self.n[l] > self.keep:
                    mass[l, h, self.keep:self.n[l]] = 0
        np.testing.assert_array_equal(self.md.cpu().numpy().view(np.int32), mass.view(np.int32))
        np.testing.assert_array_equal(self.pd.cpu().numpy(), pos)

    def moved(self, X):
        """X [L, Hkv, rows, ...] after the moves."""
        X = X.copy()
        for l in range(self.L):
            for h in range(self.Hkv):
                to, start = self.moves[l][h]
                X[l, h, to] = X[l, h, start]
        return X


CASES = [  # L, Hkv, d, rows, n, keep, n_sink, n_recent
    (1, 1, 8, 2, 2, 1, 0, 0), (1, 1, 128, 1, 1, 1, 0, 0), (2, 2, 64, 33, 33, 32, 1, 2), (1, 3, 128, 40, 37, 5, 2, 3), (2, 2, 96, 100, 100, 31, 4, 8),
    (1, 2, 256, 70, 65, 64, 0, 64), (3, 2, 80, 200, 199, 198, 7, 90), (1, 4, 128, 1500, 1400, 700, 16, 100), (2, 1, 64, 4097, 4097, 1, 0, 1),
    (70, 1, 64, 50, 49, 20, 2, 2), (1, 2, 64, 2049, 2049, 2048, 4, 500), (2, 3, 128, 5000, 4999, 1024, 1024, 0), (1, 8, 128, 8911, 8911, 8272, 16, 32),
    (33, 8, 64, 90, 90, 45, 0, 0), (20, 4, 128, 3000, 2999, 1001, 4, 300), (1, 2, 8, 40000, 39999, 39990, 10, 3000), (1, 1, 8, 262144, 262144, 100001, 4, 9000),
    (2, 2, 16, 17000, 16999, 9000, 3, 700), (1, 1, 8, 60000, 60000, 30001, 100, 5000), (1, 2, 8, 50000, 49500, 400, 0, 0)]


@pytest.mark.parametrize("kind", MASSES)
@pytest.mark.parametrize("L,Hkv,d,rows,n,keep,sink,recent", CASES)
def test_evict_matches_oracle(B, L, Hkv, d, rows, n, keep, sink, recent, kind):
    """K and V bit for bit over all rows: nothing but the slots filled changes."""
    import torch
    rng = np.random.default_rng(n + keep)
    c = _Case(rng, L, Hkv, d, rows, n, keep, sink, recent, kind, ordered=kind == "ties")
    K, V = (rng.integers(0, 65536, (L, Hkv, rows, d), dtype=np.uint16) for _ in "kv")
    Kd, Vd = TL.bf16_dev(K), TL.bf16_dev(V)
    st = B.new_status()
    left = B.stepkv_evict(Kd, Vd, c.md, c.pd, n, keep, sink, recent, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and left.tolist() == [min(n, keep)]
    c.check_book()
    np.testing.assert_array_equal(TL.bits_of(Kd), c.moved(K))
    np.testing.assert_array_equal(TL.bits_of(Vd), c.moved(V))


Q8_CASES = [(1, 1, 64, 2, 2, 1, 0, 0), (1, 2, 128, 40, 37, 5, 2, 3), (2, 2, 64, 33, 33, 32, 1, 2), (1, 3, 128, 100, 99, 40, 4, 8),
            (2, 1, 64, 640, 640, 320, 16, 64), (1, 2, 128, 1500, 1401, 700, 16, 100), (70, 1, 64, 70, 69, 33, 2, 2),
            (1, 2, 64, 2049, 2049, 2048, 4, 500), (3, 2, 128, 301, 300, 299, 0, 20), (1, 1, 128, 1000, 1000, 31, 0, 10),
            (20, 4, 64, 200, 199, 77, 2, 8), (39, 2, 128, 400, 390, 300, 2, 30), (76, 1, 128, 700, 700, 352, 0, 50), (10, 8, 64, 1300, 1300, 700, 8, 100), (1, 2, 64, 17000, 16999, 6001, 16, 2000)]


@pytest.mark.parametrize("spread", [0, 3, 14])
@pytest.mark.parametrize("L,Hkv,d,rows,n,keep,sink,recent", Q8_CASES)
def test_q8_evict_matches_oracle(B, L, Hkv, d, rows, n, keep, sink, recent, spread):
    """Rows of magnitudes that differ by up to 2^spread either way, so that blocks' scales grow; NaN among them."""
    import torch
    rng = np.random.default_rng(n + keep + spread)
    c = _Case(rng, L, Hkv, d, rows, n, keep, sink, recent, "ties" if spread == 3 else "long tail", ordered=spread == 0)
    f = np.exp2(rng.integers(-spread, spread + 1, (L, Hkv, n, 1)))
    X = [wl.f32_to_bf16_bits((rng.standard_normal((L, Hkv, n, d)) * f).astype(np.float32)) for _ in "kv"]
    for x in X:
        x[rng.integers(0, L, 3), rng.integers(0, Hkv, 3), rng.integers(0, n, 3), rng.integers(0, d, 3)] = 0x7FC0
    cache, st = B.Q8Cache.allocate(L, Hkv, rows, d), B.new_status()
    B.stepkv_q8_write(cache, TL.bf16_dev(X[0]), TL.bf16_dev(X[1]), 0, status=st)
    behind = [x.view(torch.uint8)[:, :, keep:].clone() for x in (cache.K, cache.V)]
    left = B.stepkv_q8_evict(cache, c.md, c.pd, n, keep, sink, recent, status=st)
    m = min(n, keep)
    back = B.stepkv_q8_read(cache, 0, m, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and left.tolist() == [m]
    c.check_book()
    for t, (codes, scales) in enumerate(((cache.K, cache.K_scale), (cache.V, cache.V_scale))):
        assert torch.equal(codes.view(torch.uint8)[:, :, keep:], behind[t])  # what is not counted any more keeps its bytes
        sc, got = scales.cpu().numpy().astype(np.float64), _f64(back[t])
        for l in range(L):
            for h in range(Hkv):
                v, s = O.q8_quantise(X[t][l, h])
                v, s = O.q8_evict(v, s, *c.moves[l][h])
                np.testing.assert_array_equal(got[l, h], v[:m])
                np.testing.assert_array_equal(sc[l, h, :-(-m // 32)], s[:-(-m // 32)])


def test_counts_of_their_own(B):
    """A count for each layer on the device, some at or below `keep`, zero and one among them; counts out of range are told and
    leave their layers alone; n_out may be n."""
    import torch
    rng = np.random.default_rng(3)
    L, Hkv, d, rows, keep = 7, 2, 64, 130, 50
    for bad, code in ((None, 0), (rows + 1, B.STEPKV_ENOSPACE), (-1, B.STEPKV_EDATA)):
        n = np.array([0, 1, 50, 51, 130, 77, 90])
        if bad is not None:
            n[5] = bad
        used = np.where((n < 0) | (n > rows), 0, n)
        for q8 in (False, True):
            c = _Case(rng, L, Hkv, d, rows, used, keep, 4, 10, "long tail", False, width=rows + 5)
            K, V = (_bits(rng, (L, Hkv, rows, d)) for _ in "kv")
            count, st = _dev(n.astype(np.int32)), B.new_status()
            Kd, Vd = TL.bf16_dev(K), TL.bf16_dev(V)
            if q8:
                cache = B.Q8Cache.allocate(L, Hkv, rows, d)
                B.stepkv_q8_write(cache, Kd, Vd, 0, status=st)
                left = B.stepkv_q8_evict(cache, c.md, c.pd, count, keep, 4, 10, n_out=count, status=st)
            else:
                left = B.stepkv_evict(list(Kd), list(Vd), list(c.md), list(c.pd), count, keep, 4, 10, n_out=count, status=st)
            torch.cuda.synchronize()
            assert st.item() == code and left is count
            assert count.tolist() == [x if not 0 <= x <= rows else min(x, keep) for x in n.tolist()]
            c.check_book()
            if not q8:
                np.testing.assert_array_equal(TL.bits_of(Kd), c.moved(K))
                np.testing.assert_array_equal(TL.bits_of(Vd), c.moved(V))
            else:
                got = _f64(B.stepkv_q8_read(cache, status=B.new_status())[0])
                for l in range(L):
                    for h in range(Hkv):
                        v, s = O.q8_quantise(K[l, h])
                        m = min(used[l], keep)
                        np.testing.assert_array_equal(got[l, h, :m], O.q8_evict(v, s, *c.moves[l][h])[0][:m])


LENGTHS = [  # L, Hkv, d, rows, n, keep, n_sink, n_recent: every number of rows a thread holds, few rows let go and many
    (2, 2, 128, 5010, 5000, 4900, 4, 100), (2, 2, 64, 8000, 8000, 7800, 0, 32), (1, 3, 128, 8273, 8273, 8272, 4, 256), (24, 1, 64, 8911, 8911, 8272, 16, 32),
    (3, 1, 64, 10240, 10240, 10100, 16, 1000), (1, 2, 128, 10241, 10241, 10000, 0, 0), (2, 2, 64, 12000, 11999, 11900, 4, 64), (1, 2, 128, 16384, 16384, 16300, 1, 1),
    (3, 1, 64, 16385, 16385, 16300, 4, 10), (2, 1, 128, 20000, 20000, 19900, 9, 500), (1, 2, 64, 32768, 32768, 32700, 4, 32), (11, 1, 64, 32700, 32700, 30720, 4, 2000)]


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("L,Hkv,d,rows,n,keep,sink,recent", LENGTHS)
def test_heads_of_every_length(B, L, Hkv, d, rows, n, keep, sink, recent, q8):
    if q8:
        test_q8_evict_matches_oracle(B, L, Hkv, d, rows, n, keep, sink, recent, 3 if keep % 8 else 14)
    else:
        test_evict_matches_oracle(B, L, Hkv, d, rows, n, keep, sink, recent, "ties" if keep % 8 else "special")


@pytest.mark.parametrize("L,Hkv,d,n,keep", [(2, 3, 96, 1400, 700), (2, 3, 80, 1400, 650), (5, 2, 48, 1300, 700), (1, 2, 24, 2000, 999), (1, 1, 8, 3000, 1500),
                                            (1, 2, 256, 1500, 700), (1, 3, 200, 1500, 700)])
def test_many_moves_of_rows_of_any_width(B, L, Hkv, d, n, keep):
    """Rows that a warp's instruction takes 1 to 32 of, with lanes left over where their 16-byte pieces do not divide 32."""
    test_evict_matches_oracle(B, L, Hkv, d, n + 1, n, keep, 4, 50, "long tail")


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("L,Hkv,d,rows,keep,each", [
    (3, 2, 64, 1600, 700, True), (3, 2, 128, 1600, 701, False), (70, 1, 128, 4300, 2100, True), (70, 1, 128, 4250, 2100, False),
    (66, 1, 64, 1500, 733, True), (66, 1, 64, 33000, 16500, False)])
def test_many_moves_with_the_count_replaced(B, L, Hkv, d, rows, keep, each, q8):
    """Calls that move rows by a launch of their own, more than 64 layers (two of either launch, which share the workspace) among
    them; n_out is n, one for all or one each, of which some are zero, at `keep` or out of range."""
    import torch
    rng = np.random.default_rng(L + rows + each)
    d = 8 if rows > 30000 and not q8 else d
    n = rng.integers(rows // 2, rows + 1, L) if each else np.array([rows - 3])
    code = 0
    if each:
        n[:2] = keep, rows
        n[-1] = rows + 1
        code = B.STEPKV_ENOSPACE
        if L > 3:
            n[[5, 40, 64]] = 0, keep + 1, rows
    used = np.broadcast_to(np.where(n > rows, 0, n), (L,))
    c = _Case(rng, L, Hkv, d, rows, used, keep, 4, 30, "long tail", False)
    few = 3  # caches that differ
    if q8:
        X = [_bits(rng, (few, Hkv, rows, d)) for _ in "kv"]
        for x in X:
            x[:, :, rng.integers(0, rows, rows // 50)] += 5 << 7  # rows 32 times as large
    else:
        X = [rng.integers(0, 65536, (few, Hkv, rows, d), dtype=np.uint16) for _ in "kv"]
    Kd, Vd = (TL.bf16_dev(x)[[l % few for l in range(L)]] for x in X)
    count, st = _dev(n.astype(np.int32)), B.new_status()
    if q8:
        cache = B.Q8Cache.allocate(L, Hkv, rows, d)
        B.stepkv_q8_write(cache, Kd, Vd, 0, status=st)
        B.stepkv_q8_evict(cache, c.md, c.pd, count, keep, 4, 30, n_out=count, status=st)
        got = B.stepkv_q8_read(cache)
    else:
        B.stepkv_evict(Kd, Vd, c.md, c.pd, count, keep, 4, 30, n_out=count, status=st)
        got = (Kd, Vd)
    torch.cuda.synchronize()
    assert st.item() == code
    assert count.tolist() == [x if x > rows else min(x, keep) for x in n.tolist()]
    c.check_book()
    want = [O.q8_quantise(x) for x in X] if q8 else None
    for l in sorted({0, 1, 2, 5, 40, 63, 64, L - 1} & set(range(L))) if q8 else range(L):
        for t in range(2):
            for h in range(Hkv):
                to, start = c.moves[l][h]
                if q8:
                    m = min(int(used[l]), keep)
                    v, s = want[t][0][l % few, h], want[t][1][l % few, h]
                    np.testing.assert_array_equal(_f64(got[t][l, h])[:m], O.q8_evict(v, s, to, start)[0][:m])
                else:
                    x = X[t][l % few, h].copy()
                    x[to] = x[start]
                    np.testing.assert_array_equal(TL.bits_of(got[t][l, h].contiguous()), x)


@pytest.mark.parametrize("L", [3, 130])
def test_one_count_on_the_device_for_all(B, L):
    """130 layers take three launches, which all read the one count before it is replaced."""
    import torch
    rng = np.random.default_rng(4)
    Hkv, d, rows, n, keep = 2, 8, 90, 81, 40
    c = _Case(rng, L, Hkv, d, rows, n, keep, 3, 7, "ties", True)
    K = rng.integers(0, 65536, (L, Hkv, rows, d), dtype=np.uint16)
    Kd, Vd = TL.bf16_dev(K), TL.bf16_dev(K)
    count, st = _dev(np.array([n], np.int32)), B.new_status()
    B.stepkv_evict(Kd, Vd, c.md, c.pd, count, keep, 3, 7, n_out=count, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and count.item() == keep
    c.check_book()
    np.testing.assert_array_equal(TL.bits_of(Kd), c.moved(K))


def test_strided_tensors(B):
    """Heads of larger buffers, layers inside heads, masses and positions of other widths."""
    import torch
    rng = np.random.default_rng(5)
    L, Hkv, d, rows, n, keep = 2, 3, 64, 60, 55, 20
    c = _Case(rng, L, Hkv, d, rows, n, keep, 2, 5, "long tail", False)
    K = rng.integers(0, 65536, (L, Hkv, rows, d), dtype=np.uint16)
    big = torch.full((2, Hkv, L, rows + 7, d), 3.0, dtype=torch.bfloat16, device="cuda")
    views = [[big[t, :, l, :rows] for l in range(L)] for t in range(2)]
    for l in range(L):
        for t in range(2):
            views[t][l].copy_(TL.bf16_dev(K[l]))
    mass, pos = torch.full((Hkv, L, 70), 9.0, device="cuda"), torch.full((Hkv, L, 81), 9, dtype=torch.int32, device="cuda")
    mass[:, :, :rows], pos[:, :, :rows] = c.md.transpose(0, 1), c.pd.transpose(0, 1)
    st = B.new_status()
    B.stepkv_evict(*views, mass.transpose(0, 1), pos.transpose(0, 1), n, keep, 2, 5, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and (mass[:, :, rows:] == 9).all() and (pos[:, :, rows:] == 9).all() and (big[:, :, :, rows:] == 3).all()
    c.md, c.pd = mass[:, :, :rows].transpose(0, 1).contiguous(), pos[:, :, :rows].transpose(0, 1).contiguous()
    c.check_book()
    for t in range(2):
        for l in range(L):
            np.testing.assert_array_equal(TL.bits_of(views[t][l].contiguous()), c.moved(K)[l])


def test_positions_at_the_ends_of_32_bits(B):
    import torch
    lo, hi = -2 ** 31, 2 ** 31 - 1
    for pos, sink, recent in (([hi, hi - 1, lo, 0, 5, hi - 2], 0, 2), ([lo, lo + 1, lo + 2, lo + 3, lo + 4, lo + 5], 0, 2),
                              ([3, 1, 2, hi, 0, lo], 2, 1), ([7] * 6, 0, 1), ([lo] * 6, 1, 0), ([hi] * 6, 3, 0)):
        mass = np.array([0.1, 0.2, 0.9, 0.8, 0.7, 0.3], np.float32)
        K = torch.arange(6 * 8, dtype=torch.float32).reshape(1, 1, 6, 8).cuda().bfloat16()
        V, md, pd = K.clone(), _dev(mass)[None, None], _dev(np.array(pos, np.int32))[None, None]
        B.stepkv_evict(K, V, md, pd, 6, 3, sink, recent)
        to, start = O.evict_moves(mass, np.array(pos, np.int64), 3, sink, recent)
        want = np.array(pos)
        want[to] = want[start]
        np.testing.assert_array_equal(pd[0, 0].cpu().numpy()[:3], want[:3])
        assert (K[0, 0, :3, 0] / 8).tolist() == [dict(zip(to, start)).get(j, j) for j in range(3)]


@pytest.mark.parametrize("rows", [20000, 70000])
def test_long_capacities_and_short_counts(B, rows):
    """What is launched goes by the capacity (here several CTAs a head), what is done by the counts on the device."""
    import torch
    rng = np.random.default_rng(8)
    L, Hkv, d, keep = 5, 1, 8, 32
    n = np.array([33, 5, rows, 2000, 0])
    c = _Case(rng, L, Hkv, d, rows, n, keep, 2, 9, "special", False)
    K = rng.integers(0, 65536, (L, Hkv, rows, d), dtype=np.uint16)
    Kd, Vd = TL.bf16_dev(K), TL.bf16_dev(K)
    count, st = _dev(n.astype(np.int32)), B.new_status()
    left = B.stepkv_evict(Kd, Vd, c.md, c.pd, count, keep, 2, 9, status=st)
    torch.cuda.synchronize()
    assert st.item() == 0 and left.tolist() == np.minimum(n, keep).tolist()
    c.check_book()
    np.testing.assert_array_equal(TL.bits_of(Kd), c.moved(K))
    np.testing.assert_array_equal(TL.bits_of(Vd), c.moved(K))


@pytest.mark.parametrize("q8", [False, True])
def test_caches_with_room_for_more_rows_than_are_ranked(B, q8):
    """Heads of 300000 rows with short counts, given on the host and on the device; counts above 262144 are refused or told, and
    leave their layers alone."""
    import torch
    rng = np.random.default_rng(9)
    L, Hkv, d, rows, keep, limit = 3, 1, 64 if q8 else 8, 300000, 1000, B.EVICT_MAX_ROWS
    K = _bits(rng, (L, Hkv, rows, d))
    for n in (np.full(L, 1777), np.array([1500, 900, 1234]), np.array([limit + 1, 1300, rows])):
        used = np.where(n > limit, 0, n)
        c = _Case(rng, L, Hkv, d, rows, used, keep, 4, 40, "long tail", False)
        Kd, Vd, st = TL.bf16_dev(K), TL.bf16_dev(K), B.new_status()
        if q8:
            front = (B.Q8Cache.allocate(L, Hkv, rows, d),)
            B.stepkv_q8_write(front[0], Kd, Vd, 0, n=2000, status=st)
        else:
            front = (Kd, Vd)
        call = B.stepkv_q8_evict if q8 else B.stepkv_evict
        with pytest.raises(B.StepKVError):
            call(*front, c.md, c.pd, limit + 1, keep, 4, 40)
        ws = B.evict_workspace(c.md)
        left = call(*front, c.md, c.pd, int(n[0]) if n[0] == n[1] else _dev(n.astype(np.int32)), keep, 4, 40, ws=ws, status=st)
        torch.cuda.synchronize()
        assert st.item() == (B.STEPKV_ENOSPACE if n.max() > limit else 0)
        assert left.tolist() == ([keep] if n[0] == n[1] else [0 if x > limit else min(x, keep) for x in n.tolist()])
        c.check_book()
        got = _f64(B.stepkv_q8_read(front[0], 0, keep)[0]) if q8 else O.bf16_to_f64(TL.bits_of(Kd))
        for l in range(L):
            to, start = c.moves[l][0]
            if q8:
                v, s = O.q8_quantise(K[l, 0, :2000])
                np.testing.assert_array_equal(got[l, 0], O.q8_evict(v, s, to, start)[0][:keep])
            else:
                x = K[l, 0].copy()
                x[to] = x[start]
                np.testing.assert_array_equal(got[l, 0], O.bf16_to_f64(x))


def test_two_streams_at_once(B):
    import torch
    rng = np.random.default_rng(6)
    L, Hkv, d, rows, keep = 4, 8, 64, 3000, 1000
    cases = [_Case(rng, L, Hkv, d, rows, rows, keep, 4, 100, "long tail", False) for _ in range(2)]
    K = [rng.integers(0, 65536, (L, Hkv, rows, d), dtype=np.uint16) for _ in range(2)]
    dev = [(TL.bf16_dev(k), TL.bf16_dev(k)) for k in K]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [B.stepkv_evict(*dev[i], cases[i].md, cases[i].pd, rows, keep, 4, 100, stream=streams[i]) for i in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        assert outs[i].tolist() == [keep]
        cases[i].check_book()
        np.testing.assert_array_equal(TL.bits_of(dev[i][0]), cases[i].moved(K[i]))


def _attended(rng, steps, L, Hkv, G, d):
    return [(_bits(rng, (L, Hkv, 1, d)), _bits(rng, (L, Hkv, 1, d)), _bits(rng, (L, Hkv * G, d), 2.0)) for _ in range(steps)]


@pytest.mark.parametrize("q8", [True, False])
@pytest.mark.parametrize("captured", [False, True])
def test_decoding_at_a_budget(B, q8, captured):
    """The operators as they are used together: a prompt brought to its budget, then tokens appended, attended with their weights
    accumulated, and one row of each head evicted, eagerly or as one captured step replayed, in 8 bits and in bf16.  The
    oracle follows the device's masses (a sum's last bits decide between rows that are near one another), and all else is its
    own."""
    import torch
    rng = np.random.default_rng(7)
    L, Hkv, G, d, prompt, keep, sink, recent, steps = 2, 2, 4, 64, 70, 60, 4, 20, 12
    rows = prompt + 1
    X = [_bits(rng, (L, Hkv, prompt, d)) for _ in "kv"]
    tokens = _attended(rng, steps, L, Hkv, G, d)
    mass = torch.rand((L, Hkv, rows), device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda").expand(L, Hkv, rows).contiguous()
    n, row, st = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(3))
    n.fill_(prompt)
    tk, tv = (torch.zeros((L, Hkv, 1, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    q, out = torch.zeros((L, Hkv * G, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((L, Hkv * G, d), device="cuda")
    now = torch.full((L, Hkv, 1), prompt, dtype=torch.int32, device="cuda")
    if q8:
        cache = B.Q8Cache.allocate(L, Hkv, rows, d)
        B.stepkv_q8_write(cache, TL.bf16_dev(X[0]), TL.bf16_dev(X[1]), 0, status=st)
        ws = B.q8_decode_workspace(cache, Hkv * G, True)
    else:
        K, V = (torch.zeros((L, Hkv, rows, d), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        K[:, :, :prompt], V[:, :, :prompt] = TL.bf16_dev(X[0]), TL.bf16_dev(X[1])
        ws = torch.zeros(B.load_library().stepkv_decode_h2o_workspace_size(L, Hkv, Hkv * G, d, rows) + 512, dtype=torch.uint8, device="cuda")
    ews, masses = B.evict_workspace(mass), torch.zeros_like(mass)

    def evict():
        masses.copy_(mass)  # (what the oracle decides by)
        if q8:
            B.stepkv_q8_evict(cache, mass, pos, n, keep, sink, recent, n_out=n, ws=ews, status=st)
        else:
            B.stepkv_evict(K, V, mass, pos, n, keep, sink, recent, n_out=n, ws=ews, status=st)

    def step():
        at = n.long().expand(L, Hkv, 1)
        pos.scatter_(2, at, now)
        if q8:
            B.stepkv_q8_write(cache, tk, tv, n, status=st)
        else:
            K.scatter_(2, at[..., None].expand(-1, -1, -1, d), tk), V.scatter_(2, at[..., None].expand(-1, -1, -1, d), tv)
        n.add_(1)
        now.add_(1)
        if q8:
            B.stepkv_q8_decode(q, cache, n, out=out, mass=mass, ws=ws, status=st)
        else:
            B.stepkv_decode_h2o(list(q), list(K), list(V), n, list(mass), out=list(out), ws=ws, status=st)
        evict()

    # the oracle's side
    v = [[[np.zeros((rows, d)) for _ in range(Hkv)] for _ in range(L)] for _ in "kv"]
    s = [[[np.zeros(-(-rows // 32)) for _ in range(Hkv)] for _ in range(L)] for _ in "kv"]
    at = [[np.arange(rows) for _ in range(Hkv)] for _ in range(L)]

    def append(t, l, h, x, r):
        if q8:
            O.q8_append(v[t][l][h], s[t][l][h], x, r)
        else:
            v[t][l][h][r:r + len(x)] = O.bf16_to_f64(x)

    def follow(m):
        for l in range(L):
            for h in range(Hkv):
                to, start = O.evict_moves(masses[l, h, :m].cpu().numpy(), at[l][h][:m], keep, sink, recent)
                at[l][h][to] = at[l][h][start]
                for t in range(2):
                    if q8:
                        v[t][l][h], s[t][l][h] = O.q8_evict(v[t][l][h], s[t][l][h], to, start)
                    else:
                        v[t][l][h][to] = v[t][l][h][start]

    for t in range(2):
        for l in range(L):
            for h in range(Hkv):
                append(t, l, h, X[t][l, h], 0)
    evict()
    torch.cuda.synchronize()
    follow(prompt)
    assert n.item() == keep
    graph = None
    if captured:
        saved = [x.clone() for x in (n, now, mass, pos)]
        state = [x.clone() for x in ((cache.K.view(torch.uint8), cache.V.view(torch.uint8), cache.K_scale, cache.V_scale) if q8 else (K, V))]
        step()  # an ordinary call before capturing
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for x, w in zip((n, now, mass, pos), saved):
            x.copy_(w)
        for x, w in zip((cache.K.view(torch.uint8), cache.V.view(torch.uint8), cache.K_scale, cache.V_scale) if q8 else (K, V), state):
            x.copy_(w)
    for i, (k, val, qq) in enumerate(tokens):
        tk.copy_(TL.bf16_dev(k)), tv.copy_(TL.bf16_dev(val)), q.copy_(TL.bf16_dev(qq))
        before = mass.clone()
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert st.item() == 0 and n.item() == keep
        for l in range(L):
            for h in range(Hkv):
                append(0, l, h, k[l, h], keep)
                append(1, l, h, val[l, h], keep)
                at[l][h][keep] = prompt + i
            Kv, Vv = (np.stack([v[t][l][h][:keep + 1] for h in range(Hkv)]) for t in range(2))
            want, weights = O.q4_decode_attention(qq[l], Kv, Vv), O.attention_weights(qq[l], Kv)
            got, was, now_ = (x[l].cpu().numpy().astype(np.float64) for x in (out, before, masses))
            if q8:
                assert (np.abs(got - want) <= Q._decode_bound(qq[l], Kv, Vv)).all()
                assert (np.abs((now_ - was)[:, :keep + 1] - weights) <= Q._mass_bound(qq[l], Kv, was[:, :keep + 1])).all()
            else:  # as the decode and its masses are tested: 2e-3, of the terms' magnitude where they cancel
                assert (np.abs(got - want) <= 2e-3 * np.maximum(np.abs(want), 1e-3 * O.q4_decode_attention(qq[l], Kv, np.abs(Vv)))).all()
                assert (np.abs((now_ - was)[:, :keep + 1] - weights) <= 2e-3 * weights + 2.0 ** -22 * (was[:, :keep + 1] + 1)).all()
        follow(keep + 1)
        for l in range(L):
            for h in range(Hkv):
                np.testing.assert_array_equal(pos[l, h, :keep].cpu().numpy(), at[l][h][:keep])
    got = B.stepkv_q8_read(cache, 0, keep) if q8 else (K[:, :, :keep], V[:, :, :keep])
    for t in range(2):
        for l in range(L):
            for h in range(Hkv):
                np.testing.assert_array_equal(_f64(got[t])[l, h], v[t][l][h][:keep])
    assert (mass[:, :, keep:prompt] == 0).all()


def test_binding_refusals(B):
    import torch
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")
    K, mass, pos = z(1, 2, 40, 64, t=torch.bfloat16), z(1, 2, 40), z(1, 2, 40, t=torch.int32)
    V = K.clone()
    good = dict(K=K, V=V, mass=mass, pos=pos, n=40, keep=20)
    for bad in (dict(V=V[:, :1]), dict(V=z(1, 2, 40, 64)), dict(K=K[..., ::2], V=V[..., ::2]), dict(mass=z(1, 2, 39)), dict(mass=z(2, 2, 40)),
                dict(mass=pos), dict(pos=mass), dict(pos=pos[..., :10]), dict(n=2 ** 31), dict(n=z(3, t=torch.int32)), dict(n=z(1)),
                dict(keep=2 ** 32 + 1), dict(n_sink=2 ** 40), dict(n_out=z(2, t=torch.int32)), dict(n_out=z(1)), dict(pos=pos.cpu()),
                dict(mass=mass.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises((ValueError, TypeError)):
            B.stepkv_evict(**{**good, **bad})
    for bad in (dict(keep=0), dict(keep=41), dict(n=41), dict(n=-1), dict(n_sink=15, n_recent=6), dict(n_recent=-1), dict(V=K),
                dict(ws=z(256, t=torch.uint8))):
        with pytest.raises(B.StepKVError):
            B.stepkv_evict(**{**good, **bad})
