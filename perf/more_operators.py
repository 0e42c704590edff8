"""A cache held in 8 bits, and eviction by accumulated attention, as cases that can be timed and compared.

The cache keeps e4m3 codes, and per head and block of 32 rows (tokens) one scale s = 2^k, k in -100 .. 119 the smallest
with max |x| <= 448 2^k over the finite values of the block's rows; a code stands for code * s, infinities and NaN for
NaN.  Rows are appended: a block that holds rows already keeps them, s becomes the larger of its own and what the new rows
need, and the codes that stay are rounded to it.

Eviction leaves `keep` of a head's rows: first those with a position below n_sink or among the n_recent newest
(position > newest - n_recent), then those of the largest accumulated attention (NaN last), ties to the lower slot.  The
i-th slot below `keep` that goes is filled from the i-th slot at or above it that stays.

A case is one pass: "write" appends rows and reads them back, "read" reads rows back to bf16, "decode" is one query
token's attention over the cache (with `mass`, adding each key's weight to its accumulated attention), "evict" is one
eviction from a cache in bf16, "q8_evict" from one in 8 bits, read back afterwards.  With `own` set a pass makes the
library's calls, else it computes the same in elementary torch operations.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 32
F8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------ the cases
def _write(name, L, Hkv, d, n, T, row0, rows, outliers=4):
    """n rows to row0 of a cache of `rows` rows: n new tokens as the projections leave them, [token][head][d] (T = 0),
    or the n retained of T slots of a bf16 cache."""
    c = dict(op="write", L=L, Hkv=Hkv, d=d, n=n, T=T, row0=row0, rows=rows, outliers=outliers)
    return dict(c, name=name) if name else c


def _read(name, L, Hkv, d, n, row0, rows, values, outliers=4):
    """Rows row0 .. row0 + n of every head, keys alone or keys and values."""
    c = dict(op="read", L=L, Hkv=Hkv, d=d, n=n, row0=row0, rows=rows, values=values, outliers=outliers)
    return dict(c, name=name) if name else c


def _decode(name, L, Hq, Hkv, d, n, rows, ragged=0, mass=False, outliers=4):
    """L caches of `rows` rows, n of them in use (ragged > 0: a count for each cache, 0 to n, drawn from that seed);
    the counts are read on the device."""
    c = dict(op="decode", L=L, Hq=Hq, Hkv=Hkv, d=d, n=n, rows=rows, ragged=ragged, mass=mass, outliers=outliers)
    return dict(c, name=name) if name else c


def _evict(name, op, L, Hkv, d, n, keep, n_sink, n_recent, ordered, outliers=4):
    """n rows down to `keep`, in the order they came (ordered) or as earlier evictions left them."""
    c = dict(op=op, L=L, Hkv=Hkv, d=d, n=n, keep=keep, n_sink=n_sink, n_recent=n_recent, ordered=ordered, outliers=outliers)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded token's keys and values, appended to every layer inside a block: latency
        _write("write_token", 32, 8, 128, 1, 0, 8272, 8911),
        # a whole Observation appended after its prefill, an odd number of tokens
        _write("write_observation", 32, 8, 128, 639, 0, 8272, 8911),
        # a cache read back whole for a prefill, 64 layers of the fixed 4096 budget
        _read("read_cache", 64, 8, 128, 4240, 0, 4999, True),
        # one decoded token, one layer, as an agent's model runs it: latency
        _decode("decode_layer", 1, 32, 8, 128, 8272, 8911),
        # a serving batch of small-model trajectories of different lengths, one of them empty
        _decode("decode_ragged", 24, 8, 2, 64, 8191, 8192, ragged=3),
        # a long cache of 64 layers, 5 query heads per KV head: the largest call
        _decode("decode_64_layers", 64, 40, 8, 128, 16417, 16500),
        # one layer's token whose weights are accumulated for the next eviction
        _decode("mass_layer", 1, 32, 8, 128, 8272, 8911, mass=True),
        # the same over all layers in one call
        _decode("mass_32_layers", 32, 32, 8, 128, 8272, 8911, mass=True),
        # a cache at its budget after one more token: each head lets one row go
        _evict("evict_token", "evict", 32, 8, 128, 8273, 8272, 16, 2048, False),
        # the end of a long prefill: the budget's worth of the prompt is kept
        _evict("evict_prompt", "evict", 32, 8, 128, 32768, 8272, 16, 2048, True),
        # a serving batch of small-model trajectories at their budget, in 8 bits
        _evict("q8_evict_token", "q8_evict", 24, 2, 64, 2049, 2048, 4, 500, False),
        # an Observation was appended to an 8-bit cache: back to the budget
        _evict("q8_evict_boundary", "q8_evict", 32, 8, 128, 8911, 8272, 16, 2048, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "decode", "decode", "decode", "mass", "mass", "evict", "evict", "q8_evict", "q8_evict"])
    L = rng.choice([1, 2, 4, 16, 32])
    outliers = rng.choice([0, 4])
    Hkv, d = rng.choice([(2, 64), (8, 128), (8, 128), (8, 64), (16, 128)])
    if op in ("write", "read"):
        n = _log_int(rng, 1, min(8911 * 32 * 8 // (L * Hkv), 30000))
        row0 = rng.randint(0, 4000)
        if op == "write":
            T = rng.choice([0, 0, n + _log_int(rng, 1, 2 * n + 10)])
            return _write("", L, Hkv, d, n, T, row0, row0 + n + rng.randint(0, 700), outliers)
        return _read("", L, Hkv, d, n, row0, row0 + n + rng.randint(0, 700), rng.random() < 0.6, outliers)
    if op in ("evict", "q8_evict"):
        n = _log_int(rng, 2, 32768 * 32 * 8 // max(32 * 8, L * Hkv) if op == "evict" else min(32768, 16384 * 32 * 8 // (L * Hkv)))
        keep = max(1, n - 1 if rng.random() < 0.3 else n - _log_int(rng, 1, n - 1))
        n_sink = rng.randint(0, min(16, keep))
        return _evict("", op, L, Hkv, d, n, keep, n_sink, rng.randint(0, (keep - n_sink) // 2), rng.random() < 0.4, outliers)
    Hq, Hkv, d = rng.choice([(8, 2, 64), (32, 8, 128), (32, 8, 128), (40, 8, 128), (16, 8, 64), (16, 16, 128), (64, 8, 128), (6, 1, 64)])
    n = _log_int(rng, 1, 32768 if L < 16 else 16384)
    return _decode("", L, Hq, Hkv, d, n, n + rng.randint(0, 1500), rng.choice([0, 0, rng.randint(1, 999)]), op == "mass", outliers)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _keys(gen, outliers, *shape):
    """Keys [..., rows, d]; with outliers, that many channels per head scaled by 8."""
    k = _randn(gen, *shape)
    if outliers:
        order = torch.rand((*shape[:-2], 1, shape[-1]), generator=gen, device=DEV).argsort(-1)
        k *= torch.where(order < outliers, 8.0, 1.0).to(torch.bfloat16)
    return k


def _tokens(x):
    """[L, Hkv, n, d] laid out as projections leave it: [L][n][Hkv][d]."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def _retained(seed, n, T):
    """n of T slots, ascending."""
    return sorted(random.Random(int(seed)).sample(range(T), n))


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _blocks(rows):
    return (rows + BLOCK - 1) // BLOCK


def _filled_cache(c, rows, used, gen):
    """A cache whose first `used` rows are written."""
    L, Hkv, d = c["L"], c["Hkv"], c["d"]
    z = lambda w, t: torch.zeros((L, Hkv, *w), dtype=t, device=DEV)
    cache = dict(K=z((rows, d), F8), K_scale=z((_blocks(rows),), torch.float32), V=z((rows, d), F8),
                 V_scale=z((_blocks(rows),), torch.float32))
    if used:
        for l in range(L):  # layer by layer: the 32-bit copies of a large cache are several times its size
            one = {k: x[l:l + 1] for k, x in cache.items()}
            _append(one["K"], one["K_scale"], 0, _keys(gen, c["outliers"], 1, Hkv, used, d))
            _append(one["V"], one["V_scale"], 0, _randn(gen, 1, Hkv, used, d))
    return cache


def _counts(c):
    if not c["ragged"]:
        return [c["n"]]
    r = random.Random(c["ragged"])
    n = [c["n"]] + [min(c["n"], _log_int(r, 1, c["n"] + 1)) for _ in range(c["L"] - 1)]
    return n[:2] + [0] * (c["L"] > 2) + n[3:]


def _book(c, gen):
    """Accumulated attention and positions of a head's rows, as one int32 tensor [2, L, Hkv, n]: a few rows have most of the
    weight, the newest none yet.  Not ordered: rows stand up to some hundred slots from their place in time."""
    shape = (c["L"], c["Hkv"], c["n"])
    mass = torch.exp(2.0 * torch.randn(shape, generator=gen, device=DEV))
    mass[..., -max(1, c["n"] // 50):] = 0.0
    pos = torch.arange(c["n"], device=DEV).expand(shape)
    if not c["ordered"]:
        pos = (pos + 200.0 * torch.rand(shape, generator=gen, device=DEV)).argsort(-1)
    return torch.stack([mass.view(torch.int32), pos.to(torch.int32)])


def prepare(case, seed):
    c, gen = case, _gen(seed)
    L, Hkv, d, n = c["L"], c["Hkv"], c["d"], c["n"]
    s = dict(case=c)
    bf16 = lambda rows: torch.zeros((L, Hkv, rows, d), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "write":
        T = c["T"] or n
        s["cache"] = _filled_cache(c, c["rows"], c["row0"], gen)
        s["K"], s["V"] = _keys(gen, c["outliers"], L, Hkv, T, d), _randn(gen, L, Hkv, T, d)
        if not c["T"]:
            s["K"], s["V"] = _tokens(s["K"]), _tokens(s["V"])
        s["idx"] = _int32(_retained(seed, n, T)) if c["T"] else None
        s["row0"], s["n"] = _int32([c["row0"]]), _int32([n])
        lead = c["row0"] % BLOCK
        s["K_back"], s["V_back"] = bf16(lead + n), bf16(lead + n)
    elif c["op"] == "read":
        s["cache"] = _filled_cache(c, c["rows"], c["rows"], gen)
        s["K_back"], s["V_back"] = bf16(n), bf16(n) if c["values"] else None
    elif c["op"] == "decode":
        s["cache"] = _filled_cache(c, c["rows"], c["rows"], gen)
        s["q"] = _randn(gen, L, c["Hq"], d)
        s["n"] = _int32(_counts(c))
        s["out"] = torch.zeros((L, c["Hq"], d), dtype=torch.float32, device=DEV)
        if c["mass"]:
            s["mass0"] = torch.rand((L, Hkv, c["rows"]), generator=gen, device=DEV) / n
            s["mass"] = torch.zeros_like(s["mass0"])
    else:
        if c["op"] == "evict":
            s["K"] = torch.stack([_keys(gen, c["outliers"], Hkv, n, d) for _ in range(L)])
            s["V"] = torch.stack([_randn(gen, Hkv, n, d) for _ in range(L)])
        else:
            s["cache"] = _filled_cache(c, n, n, gen)
            s["K_back"], s["V_back"] = bf16(c["keep"]), bf16(c["keep"])
        s["book0"] = _book(c, gen)
        s["book"] = torch.zeros_like(s["book0"])
        s["mass"], s["pos"] = s["book"][0].view(torch.float32), s["book"][1]
        s["n"], s["n_out"] = _int32([n]), _int32([0])
    if own:  # the handles, workspace and status word that a program keeps
        from paper_2609_22158_gb300 import binding as B
        if "cache" in s:
            s["cache"] = B.Q8Cache(**s["cache"])
        if c["op"] == "decode":
            s["ws"] = B.q8_decode_workspace(s["cache"], c["Hq"], mass=c["mass"])
        elif "book" in s:
            s["ws"] = B.evict_workspace(s["mass"])
        s["status"] = B.new_status()
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _scale_of(most):
    """2^k for the largest magnitude of a block."""
    m, e = torch.frexp(most)
    k = torch.where(most == 0, -100, e - 9 + (m > 0.875)).clamp(-100, 119)
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)


def _codes(x, s):
    """fp32 values over scales (broadcast) as e4m3, what is not finite as NaN."""
    return torch.where(x.isfinite(), x / s, float("nan")).clamp(-448, 448).to(F8)


def _spread(scale, row0, n):
    """The scales [..., blocks] of rows row0 .. row0 + n, as [..., n, 1]."""
    b0 = row0 // BLOCK
    s = scale[..., b0:_blocks(row0 + n)].repeat_interleave(BLOCK, -1)
    return s[..., row0 - b0 * BLOCK:row0 - b0 * BLOCK + n, None]


def _values(codes, scale, row0, n):
    """fp32 values of rows row0 .. row0 + n."""
    return codes[:, :, row0:row0 + n].float() * _spread(scale, row0, n)


def _append(codes, scale, row0, x):
    """Rows x [L, Hkv, n, d] to row0 of the cache."""
    n, b0 = x.shape[2], row0 // BLOCK
    lead = row0 - b0 * BLOCK
    x = x.float()
    new = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    new = torch.nn.functional.pad(new, (lead, -(lead + n) % BLOCK)).unflatten(-1, (-1, BLOCK)).amax(-1)
    s = _scale_of(new)
    if lead:
        s[..., 0] = torch.maximum(s[..., 0], scale[..., b0])
        x = torch.cat([_values(codes, scale, b0 * BLOCK, lead), x], 2)
    codes[:, :, b0 * BLOCK:row0 + n].copy_(_codes(x, _spread(s, 0, lead + n)))
    scale[..., b0:b0 + s.shape[-1]].copy_(s)


def _plain_write(s):
    c, cache = s["case"], s["cache"]
    pick = lambda x: x if s["idx"] is None else x[:, :, s["idx"]]
    _append(cache["K"], cache["K_scale"], c["row0"], pick(s["K"]))
    _append(cache["V"], cache["V_scale"], c["row0"], pick(s["V"]))
    lead = c["row0"] % BLOCK
    at = c["row0"] - lead, lead + c["n"]
    return dict(K=_values(cache["K"], cache["K_scale"], *at).bfloat16(), V=_values(cache["V"], cache["V_scale"], *at).bfloat16())


def _plain_read(s):
    c, cache = s["case"], s["cache"]
    out = dict(K=_values(cache["K"], cache["K_scale"], c["row0"], c["n"]).bfloat16())
    if c["values"]:
        out["V"] = _values(cache["V"], cache["V_scale"], c["row0"], c["n"]).bfloat16()
    return out


def _plain_decode(s):
    c, cache, n = s["case"], s["cache"], s["n"]
    L, Hkv, d, rows = c["L"], c["Hkv"], c["d"], c["n"]
    q = s["q"].float().view(L, Hkv, -1, d)
    x = q @ _values(cache["K"], cache["K_scale"], 0, rows).transpose(2, 3) / math.sqrt(d)
    seen = torch.arange(rows, device=DEV) < n.view(-1, 1, 1, 1)
    x = torch.where(seen, x, float("-inf"))
    p = torch.where(seen, torch.exp(x - x.amax(-1, keepdim=True)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p @ _values(cache["V"], cache["V_scale"], 0, rows)) / total
    out = dict(out=torch.where(total > 0, o, 0.0).view(L, -1, d))
    if c["mass"]:
        s["mass"].copy_(s["mass0"])
        s["mass"][:, :, :rows] += torch.where(total > 0, p / total, 0.0).mean(2)
        out["mass"] = s["mass"]
    return out


def _moves(s):
    """Which slot each of the first `keep` rows comes from: [L, Hkv, keep]."""
    c = s["case"]
    n, keep, mass, pos = c["n"], c["keep"], s["mass"], s["pos"]
    bits = mass.view(torch.int32).long()
    rank = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)  # in the order of the numbers
    rank = torch.where(mass.isnan(), -1 << 32, torch.where(mass == 0, 0, rank))
    safe = (pos < c["n_sink"]) | (pos > pos.amax(-1, keepdim=True) - c["n_recent"])
    rank = torch.where(safe, 1 << 32, rank)
    slot = torch.arange(n, device=DEV)
    order = (rank * (1 << 20) - slot).argsort(-1, descending=True)
    stays = torch.zeros_like(safe).scatter_(-1, order[..., :keep], True)
    before = stays.cumsum(-1) - stays.long()  # retained slots below
    low = before[..., keep:keep + 1] if keep < n else stays.sum(-1, keepdim=True)
    # sources by their rank, the others out of the way
    at = torch.where(stays & (slot >= keep), before - low, n)
    source = torch.zeros((*at.shape[:-1], n + 1), dtype=torch.long, device=DEV).scatter_(-1, at, slot.expand(at.shape))
    gone = slot - before  # holes below
    return torch.where(stays, slot, source.gather(-1, gone.clamp(max=n)))[..., :keep]


def _plain_book(s, move):
    keep = s["case"]["keep"]
    s["mass"][..., :keep] = s["mass"].gather(-1, move)
    s["pos"][..., :keep] = s["pos"].gather(-1, move)
    s["mass"][..., keep:] = 0.0
    s["n_out"].copy_(s["n"].clamp(max=keep))
    return dict(mass=s["mass"], pos=s["pos"][..., :keep], n=s["n_out"])


def _plain_evict(s):
    c, keep = s["case"], s["case"]["keep"]
    s["book"].copy_(s["book0"])
    move = _moves(s)
    rows = move[..., None].expand(-1, -1, -1, c["d"])
    s["K"][:, :, :keep] = s["K"].gather(2, rows)
    s["V"][:, :, :keep] = s["V"].gather(2, rows)
    return dict(_plain_book(s, move), K=s["K"][:, :, :keep], V=s["V"][:, :, :keep])


def _refill(codes, scale, move):
    """The first rows of the cache := the rows `move` names, those that stay keeping their block's scale or a larger one."""
    keep, n, d = move.shape[-1], codes.shape[2], codes.shape[3]
    x = _values(codes, scale, 0, n).gather(2, move[..., None].expand(-1, -1, -1, d))
    moved = move != torch.arange(keep, device=DEV)
    most = torch.where(moved, torch.where(x.isnan(), 0.0, x.abs()).amax(-1), 0.0)
    most = torch.nn.functional.pad(most, (0, -keep % BLOCK)).unflatten(-1, (-1, BLOCK)).amax(-1)
    s = torch.maximum(scale[..., :_blocks(keep)], _scale_of(most))
    codes[:, :, :keep].copy_(_codes(x, _spread(s, 0, keep)))
    scale[..., :_blocks(keep)].copy_(s)
    return _values(codes, scale, 0, keep).bfloat16()


def _plain_q8_evict(s):
    cache = s["cache"]
    s["book"].copy_(s["book0"])
    move = _moves(s)
    K = _refill(cache["K"], cache["K_scale"], move)
    V = _refill(cache["V"], cache["V_scale"], move)
    return dict(_plain_book(s, move), K=K, V=V)


# ------------------------------------------------------------------------------------------------ one pass
def _own_pass(s):
    from paper_2609_22158_gb300 import binding as B
    c, status = s["case"], s["status"]
    if c["op"] == "write":
        lead = c["row0"] % BLOCK
        B.stepkv_q8_write(s["cache"], s["K"], s["V"], s["row0"], n=s["n"], idx=s["idx"], status=status)
        B.stepkv_q8_read(s["cache"], c["row0"] - lead, lead + c["n"], K=s["K_back"], V=s["V_back"], status=status)
        return dict(K=s["K_back"], V=s["V_back"])
    if c["op"] == "read":
        B.stepkv_q8_read(s["cache"], c["row0"], c["n"], K=s["K_back"], V=s["V_back"], status=status)
        return dict(K=s["K_back"], V=s["V_back"]) if c["values"] else dict(K=s["K_back"])
    if c["op"] == "decode":
        if not c["mass"]:
            B.stepkv_q8_decode(s["q"], s["cache"], s["n"], out=s["out"], ws=s["ws"], status=status)
            return dict(out=s["out"])
        s["mass"].copy_(s["mass0"])
        B.stepkv_q8_decode(s["q"], s["cache"], s["n"], out=s["out"], mass=s["mass"], ws=s["ws"], status=status)
        return dict(out=s["out"], mass=s["mass"])
    s["book"].copy_(s["book0"])  # (the same rows go in every pass: the slots they leave are filled with what they hold already)
    how = dict(n_sink=c["n_sink"], n_recent=c["n_recent"], n_out=s["n_out"], ws=s["ws"], status=status)
    keep = c["keep"]
    if c["op"] == "evict":
        B.stepkv_evict(s["K"], s["V"], s["mass"], s["pos"], s["n"], keep, **how)
        out = dict(K=s["K"][:, :, :keep], V=s["V"][:, :, :keep])
    else:
        B.stepkv_q8_evict(s["cache"], s["mass"], s["pos"], s["n"], keep, **how)
        B.stepkv_q8_read(s["cache"], 0, keep, K=s["K_back"], V=s["V_back"], status=status)
        out = dict(K=s["K_back"], V=s["V_back"])
    return dict(out, mass=s["mass"], pos=s["pos"][..., :keep], n=s["n_out"])


def run(state):
    if own:
        return _own_pass(state)
    return globals()["_plain_" + state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ what it takes
def _moved(c):
    """Rows a head moves, about: the newest, and of the others the share of those at or above `keep` that stay."""
    n, keep, S, R = c["n"], c["keep"], c["n_sink"], c["n_recent"]
    if n <= keep:
        return 0
    late = min(R, n - keep)
    return min(keep, late + (keep - S - R) * (n - keep - late) / max(1, n - S - R))


def work(c):
    """Each input once, each output once: rows in bf16 (2 d bytes) and in 8 bits (d, and 4 a block)."""
    L, Hkv, d, n = c["L"], c["Hkv"], c["d"], c["n"]
    wide, narrow = 2 * d, d + 4 / BLOCK
    if c["op"] == "write":
        return dict(bytes=2 * L * Hkv * n * (wide + narrow + wide) + (4 * n if c["T"] else 0), flops=0)
    if c["op"] == "read":
        return dict(bytes=(2 if c["values"] else 1) * L * Hkv * n * (narrow + wide), flops=0)
    if c["op"] == "decode":
        rows = sum(_counts(c)) * (1 if c["ragged"] else L)
        return dict(bytes=Hkv * rows * (2 * narrow + 8 * c["mass"]) + L * c["Hq"] * d * 6, flops=4 * rows * c["Hq"] * d)
    book = 8 * n + 4 * (n - c["keep"])
    if c["op"] == "evict":
        return dict(bytes=L * Hkv * (book + _moved(c) * (8 + 4 * wide)), flops=0)
    return dict(bytes=L * Hkv * (book + _moved(c) * (8 + 4 * narrow) + 2 * c["keep"] * (narrow + wide)), flops=0)


# ------------------------------------------------------------------------------------------------ 64-bit values
def _step64(most):
    """The scale of a block from its largest magnitude, in 64 bits."""
    k = torch.ceil(torch.log2(most.clamp_min(1e-300) / 448.0))
    k = k + (most > 448.0 * torch.exp2(k)).double() - (most <= 448.0 * torch.exp2(k - 1)).double()
    return torch.exp2(k.clamp(-100, 119))


def _nearest64(v, s):
    """The multiples of s that e4m3 holds, nearest to v, ties to the even one."""
    y = v / s
    grid = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(y / grid) * grid).clamp(-448, 448) * s


def _values64(codes, scale, rows):
    """fp64 values of one layer's rows (a list of row numbers)."""
    bits = codes.view(torch.uint8)[:, rows].long()
    e, m = bits >> 3 & 15, (bits & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2((e - 10).double()))
    v = torch.where(bits & 127 == 127, float("nan"), torch.where(bits >= 128, -v, v))
    return v * scale[:, torch.div(rows, BLOCK, rounding_mode="floor")].double()[..., None]


def _written64(codes, scale, x, row0):
    """What one layer's rows hold from the start of row0's block on, after rows x were written to row0."""
    lead, n = row0 % BLOCK, x.shape[1]
    out = torch.cat([_values64(codes, scale, torch.arange(row0 - lead, row0, device=DEV)), x.double()], 1)
    for at in range(0, lead + n, BLOCK):
        part = out[:, at:at + BLOCK]
        s = _step64(part[:, lead if at == 0 else 0:].abs().amax((1, 2)))
        if lead and at == 0:
            s = torch.maximum(s, scale[:, row0 // BLOCK].double())
        out[:, at:at + BLOCK] = _nearest64(part, s[:, None, None])
    return out


def _evicted(c, mass, pos):
    """One head: (slots filled, slots they are filled from) by sorting in the order of the definition."""
    newest = int(pos.max())
    m, p = mass.double().tolist(), pos.tolist()
    safe = [x < c["n_sink"] or x > newest - c["n_recent"] for x in p]
    order = sorted(range(c["n"]), key=lambda j: (not safe[j], math.isnan(m[j]), 0.0 if safe[j] or math.isnan(m[j]) else -m[j], j))
    kept = set(order[:c["keep"]])
    holes = [j for j in range(c["keep"]) if j not in kept]
    return holes, [j for j in range(c["keep"], c["n"]) if j in kept]


def exact(case, seed):
    c, s = case, prepare(case, int(seed))
    L, Hkv = c["L"], c["Hkv"]
    cache = s.get("cache")
    if own and cache is not None:
        cache = dict(K=cache.K, K_scale=cache.K_scale, V=cache.V, V_scale=cache.V_scale)
    if c["op"] == "write":
        if L * Hkv * c["n"] > 2e7 / 8:
            return None
        rows = slice(None) if s["idx"] is None else s["idx"]
        return {k: torch.stack([_written64(cache[k][l], cache[k + "_scale"][l], s[k][l][:, rows], c["row0"]) for l in range(L)])
                for k in ("K", "V")}
    if c["op"] == "read":
        rows = torch.arange(c["row0"], c["row0"] + c["n"], device=DEV)
        return {k: torch.stack([_values64(a, b, rows) for a, b in zip(cache[k], cache[k + "_scale"])])
                for k in ("K", "V")[:1 + c["values"]]}
    if c["op"] == "decode":
        G = c["Hq"] // Hkv
        counts = s["n"].tolist() * (1 if c["ragged"] else L)
        out = torch.zeros((L, c["Hq"], c["d"]), dtype=torch.float64, device=DEV)
        mass = s["mass0"].double() if c["mass"] else None
        for l, n in enumerate(counts):
            if n:
                k, v = (_values64(cache[x][l], cache[x + "_scale"][l], torch.arange(n, device=DEV)) for x in ("K", "V"))
                p = torch.softmax(s["q"][l].double().view(Hkv, G, -1) @ k.transpose(1, 2) / math.sqrt(c["d"]), -1)
                out[l] = (p @ v).reshape(c["Hq"], -1)
                if c["mass"]:
                    mass[l, :, :n] += p.sum(1) / G
        return dict(out=out, mass=mass) if c["mass"] else dict(out=out)
    if L * Hkv * c["n"] > 3e6:
        return None
    keep = c["keep"]
    mass, pos = s["book0"][0].view(torch.float32), s["book0"][1]
    new_mass = mass.double().clone()
    whole = {}
    for k in ("K", "V"):
        if c["op"] == "evict":
            whole[k] = s[k].double()
        else:
            at = torch.arange(c["n"], device=DEV)
            whole[k] = torch.stack([_values64(a, b, at) for a, b in zip(cache[k], cache[k + "_scale"])])
    out = {k: whole[k][:, :, :keep].clone() for k in whole}
    for l in range(L):
        for h in range(Hkv):
            to, start = _evicted(c, mass[l, h].cpu(), pos[l, h].cpu())
            new_mass[l, h, to] = mass[l, h, start].double()
            for k in out:
                x = out[k][l, h]
                x[to] = whole[k][l, h, start]
                if c["op"] == "q8_evict":
                    s_old = cache[k + "_scale"][l, h].double()
                    most = torch.zeros(_blocks(keep), dtype=torch.float64, device=DEV)
                    if to:
                        where = torch.tensor(to, device=DEV) // BLOCK
                        most.scatter_reduce_(0, where, x[to].abs().amax(-1), "amax")
                    s_new = torch.maximum(s_old[:_blocks(keep)], _step64(most))
                    x.copy_(_nearest64(x, s_new.repeat_interleave(BLOCK)[:keep, None]))
    new_mass[..., keep:] = 0
    return dict(out, mass=new_mass, pos=None, n=None)
