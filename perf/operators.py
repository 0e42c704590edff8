"""The operators of a cache held in 4 bits, as cases that can be timed and compared.

The cache keeps, per row (one token of one KV head) and group of 32 channels, one fp16 scale s of 5 significant bits
and 32 codes n in 0..15; a code stands for s (n - 8).  For a group x with maximum M and minimum m:
    x* = M if M >= -m else m,   s = fp16(-x* / 8 to 5 significant bits), |s| <= 896,
    n = 8 + clamp(rint(x / s), -8, 7), and 8 where s = 0.
Byte b of a row's codes holds channel 2b in its low half and channel 2b + 1 in its high half.

A case is one pass: "write" quantises rows into the cache and reads them back, "read" reads rows back to bf16,
"compact" gathers the retained rows in 4 bits and reads them back (as the next Observation's prefill does), "decode"
is one query token's attention over the cache.  With `own` set a pass makes the library's calls, else it computes the
same in elementary torch operations.
"""
import math
import random

import torch

own = False

DEV = "cuda"
GROUP = 32
N_PROMPT = 16  # protected prompt slots of a trajectory


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


def _compact(name, L, Hkv, d, n, T, outliers=4):
    """The n retained of T slots."""
    c = dict(op="compact", L=L, Hkv=Hkv, d=d, n=n, T=T, outliers=outliers)
    return dict(c, name=name) if name else c


def _decode(name, L, Hq, Hkv, d, n, rows, ragged=0, outliers=4):
    """L caches of `rows` rows, n of them in use (ragged > 0: a count for each cache, 0 to n, drawn from that seed);
    the counts are read on the device."""
    c = dict(op="decode", L=L, Hq=Hq, Hkv=Hkv, d=d, n=n, rows=rows, ragged=ragged, outliers=outliers)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoded token's keys and values, appended to every layer of a compacted cache: latency
        _write("write_token", 32, 8, 128, 1, 0, 8272, 8911),
        # a whole Observation appended after its prefill, an odd number of tokens
        _write("write_observation", 32, 8, 128, 639, 0, 8272, 8911),
        # the first boundary of a long trajectory: the retained rows of the bf16 cache go into 4 bits
        _write("write_kept", 32, 8, 128, 8272, 32768, 0, 8911),
        # the saliency layers' keys in bf16, as the scoring of a boundary reads them
        _read("read_keys", 3, 8, 128, 8911, 0, 8911, False),
        # a cache read back whole for a prefill, 64 layers of the fixed 4096 budget
        _read("read_cache", 64, 8, 128, 4240, 0, 4999, True),
        # a boundary of a short episode on a small model
        _compact("compact_short", 1, 2, 64, 548, 2048),
        # a boundary of the incremental loop, read back for the next Observation's prefill
        _compact("compact_boundary", 32, 8, 128, 8272, 8911),
        # one decoded token, one layer, as an agent's model runs it: latency
        _decode("decode_layer", 1, 32, 8, 128, 8272, 8911),
        # the same over all layers in one call
        _decode("decode_32_layers", 32, 32, 8, 128, 8272, 8911),
        # a long cache of 64 layers, 5 query heads per KV head: the largest call
        _decode("decode_64_layers", 64, 40, 8, 128, 16417, 16500),
        # a serving batch of small-model trajectories of different lengths, one of them empty
        _decode("decode_ragged", 24, 8, 2, 64, 8191, 8192, ragged=3),
        # the first tokens after a boundary with a small budget: many short lists of rows
        _decode("decode_short", 32, 32, 8, 128, 81, 211),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "compact", "decode", "decode", "decode", "decode"])
    L = rng.choice([1, 2, 4, 16, 32])
    outliers = rng.choice([0, 4])
    if op != "decode":
        Hkv, d = rng.choice([(2, 64), (8, 128), (8, 128), (8, 64), (16, 128)])
        most = 8911 * 32 * 8 // (L * Hkv)  # rows a head, of the largest listed case
        n = _log_int(rng, 1, min(most, 30000))
        if op == "write":
            T = rng.choice([0, n + _log_int(rng, 1, 2 * n + 10)])
            row0 = rng.randint(0, 4000)
            return _write("", L, Hkv, d, n, T, row0, row0 + n + rng.randint(0, 700), outliers)
        if op == "read":
            row0 = rng.randint(0, 1000)
            return _read("", L, Hkv, d, n, row0, row0 + n + rng.randint(0, 700), rng.random() < 0.6, outliers)
        return _compact("", L, Hkv, d, n, n + _log_int(rng, 1, n + 10), outliers)
    Hq, Hkv, d = rng.choice([(8, 2, 64), (32, 8, 128), (32, 8, 128), (40, 8, 128), (16, 8, 64), (16, 16, 128), (64, 8, 128)])
    n = _log_int(rng, 1, 32768 if L < 16 else 16384)
    return _decode("", L, Hq, Hkv, d, n, n + rng.randint(0, 1500), rng.choice([0, 0, rng.randint(1, 999)]), outliers)


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
    """n of T slots, ascending: the prompt, the newest, and others in between."""
    r = random.Random(int(seed))
    ends = min(n // 2, N_PROMPT)
    return list(range(ends)) + sorted(r.sample(range(ends, T - ends), n - 2 * ends)) + list(range(T - ends, T))


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _empty_cache(c, rows):
    codes = [torch.zeros((c["L"], c["Hkv"], rows, c["d"] // 2), dtype=torch.uint8, device=DEV) for _ in "kv"]
    scales = [torch.zeros((c["L"], c["Hkv"], rows, c["d"] // GROUP), dtype=torch.float16, device=DEV) for _ in "kv"]
    return dict(K=codes[0], K_scale=scales[0], V=codes[1], V_scale=scales[1])


def _filled_cache(c, rows, gen):
    L, Hkv, d = c["L"], c["Hkv"], c["d"]
    keys = [_quantised(_keys(gen, c["outliers"], Hkv, rows, d)) for _ in range(L)]
    values = [_quantised(_randn(gen, Hkv, rows, d)) for _ in range(L)]
    K, K_scale, V, V_scale = (torch.stack(x) for x in (*zip(*keys), *zip(*values)))
    return dict(K=K, K_scale=K_scale, V=V, V_scale=V_scale)


def _counts(c):
    if not c["ragged"]:
        return [c["n"]]
    r = random.Random(c["ragged"])
    n = [c["n"]] + [min(c["n"], _log_int(r, 1, c["n"] + 1)) for _ in range(c["L"] - 1)]
    return n[:2] + [0] * (c["L"] > 2) + n[3:]


def prepare(case, seed):
    c, gen = case, _gen(seed)
    L, Hkv, d, n = c["L"], c["Hkv"], c["d"], c["n"]
    s = dict(case=c)
    bf16 = lambda: torch.zeros((L, Hkv, n, d), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "write":
        T = c["T"] or n
        s["cache"] = _empty_cache(c, c["rows"])
        s["K"], s["V"] = _keys(gen, c["outliers"], L, Hkv, T, d), _randn(gen, L, Hkv, T, d)
        if not c["T"]:
            s["K"], s["V"] = _tokens(s["K"]), _tokens(s["V"])
        s["idx"] = _int32(_retained(seed, n, T)) if c["T"] else None
        s["row0"], s["n"] = _int32([c["row0"]]), _int32([n])
        s["K_back"], s["V_back"] = bf16(), bf16()
    elif c["op"] == "read":
        s["cache"] = _filled_cache(c, c["rows"], gen)
        s["K_back"], s["V_back"] = bf16(), bf16() if c["values"] else None
    elif c["op"] == "compact":
        s["cache"], s["dst"] = _filled_cache(c, c["T"], gen), _empty_cache(c, n)
        s["idx"], s["n"] = _int32(_retained(seed, n, c["T"])), _int32([n])
        s["step_id"] = torch.randint(0, 40, (c["T"],), generator=gen, device=DEV, dtype=torch.int32).sort().values
        s["pos"] = torch.arange(c["T"], dtype=torch.int32, device=DEV) * 2 + 5
        s["step_out"], s["pos_out"] = (torch.zeros(n, dtype=torch.int32, device=DEV) for _ in "sp")
        s["K_back"], s["V_back"] = bf16(), bf16()
    else:
        s["cache"] = _filled_cache(c, c["rows"], gen)
        s["q"] = _randn(gen, L, c["Hq"], d)
        s["n"] = _int32(_counts(c))
        s["out"] = torch.zeros((L, c["Hq"], d), dtype=torch.float32, device=DEV)
    if own:  # the handles, workspace and status word that a program keeps
        from paper_2609_22158_gb300 import binding as B
        for name in ("cache", "dst"):
            if name in s:
                s[name] = B.Q4Cache(**s[name])
        if c["op"] == "decode":
            s["ws"] = B.q4_decode_workspace(s["cache"], c["Hq"])
        s["status"] = B.new_status()
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _quantised(x):
    """[..., d] -> codes [..., d / 2] uint8, scales [..., d / 32] fp16."""
    g = x.float().unflatten(-1, (-1, GROUP))
    hi, lo = g.amax(-1), g.amin(-1)
    bits = (-torch.where(hi >= -lo, hi, lo) / 8).view(torch.int32)
    bits = bits + 0x3FFFF + (bits >> 19 & 1) & ~0x7FFFF  # 4 of the 23 explicit bits, ties to even
    s = bits.view(torch.float32).clamp(-896, 896).half()
    step = s.float()[..., None]
    code = torch.where(step == 0, 0.0, torch.round(g / step).clamp(-8, 7)) + 8
    code = code.to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, s


def _values(codes, scales):
    """fp32 values [..., d]."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8
    return (n.unflatten(-1, (-1, GROUP)) * scales.float()[..., None]).flatten(-2)


def _plain_write(s):
    c, cache = s["case"], s["cache"]
    rows = slice(c["row0"], c["row0"] + c["n"])
    back = {}
    pick = lambda x: x if s["idx"] is None else x[:, :, s["idx"]]
    kc, ks = cache["K"][:, :, rows], cache["K_scale"][:, :, rows]
    vc, vs = cache["V"][:, :, rows], cache["V_scale"][:, :, rows]
    codes, scales = _quantised(pick(s["K"]))
    kc.copy_(codes), ks.copy_(scales)
    codes, scales = _quantised(pick(s["V"]))
    vc.copy_(codes), vs.copy_(scales)
    return dict(K=_values(kc, ks).bfloat16(), V=_values(vc, vs).bfloat16())


def _plain_read(s):
    c, cache = s["case"], s["cache"]
    rows = slice(c["row0"], c["row0"] + c["n"])
    out = dict(K=_values(cache["K"][:, :, rows], cache["K_scale"][:, :, rows]).bfloat16())
    if c["values"]:
        out["V"] = _values(cache["V"][:, :, rows], cache["V_scale"][:, :, rows]).bfloat16()
    return out


def _plain_compact(s):
    cache, dst, idx = s["cache"], s["dst"], s["idx"]
    torch.index_select(cache["K"], 2, idx, out=dst["K"])
    torch.index_select(cache["K_scale"], 2, idx, out=dst["K_scale"])
    torch.index_select(cache["V"], 2, idx, out=dst["V"])
    torch.index_select(cache["V_scale"], 2, idx, out=dst["V_scale"])
    return dict(K=_values(dst["K"], dst["K_scale"]).bfloat16(), V=_values(dst["V"], dst["V_scale"]).bfloat16(),
                step_id=s["step_id"][idx], pos=s["pos"][idx])


def _plain_decode(s):
    c, cache, n = s["case"], s["cache"], s["n"]
    L, Hkv, d, rows = c["L"], c["Hkv"], c["d"], c["n"]
    q = s["q"].float().view(L, Hkv, -1, d)
    x = q @ _values(cache["K"][:, :, :rows], cache["K_scale"][:, :, :rows]).transpose(2, 3) / math.sqrt(d)
    seen = torch.arange(rows, device=DEV) < n.view(-1, 1, 1, 1)
    x = torch.where(seen, x, float("-inf"))
    p = torch.where(seen, torch.exp(x - x.amax(-1, keepdim=True)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p @ _values(cache["V"][:, :, :rows], cache["V_scale"][:, :, :rows])) / total
    return dict(out=torch.where(total > 0, o, 0.0).view(L, -1, d))


# ------------------------------------------------------------------------------------------------ one pass
def _own_pass(s):
    from paper_2609_22158_gb300 import binding as B
    c, status = s["case"], s["status"]
    if c["op"] == "write":
        B.stepkv_q4_write(s["cache"], s["K"], s["V"], s["row0"], n=s["n"], idx=s["idx"], status=status)
        B.stepkv_q4_read(s["cache"], s["row0"], s["n"], K=s["K_back"], V=s["V_back"], status=status)
        return dict(K=s["K_back"], V=s["V_back"])
    if c["op"] == "read":
        B.stepkv_q4_read(s["cache"], c["row0"], c["n"], K=s["K_back"], V=s["V_back"], status=status)
        return dict(K=s["K_back"], V=s["V_back"]) if c["values"] else dict(K=s["K_back"])
    if c["op"] == "compact":
        B.stepkv_q4_compact(s["cache"], c["T"], s["idx"], s["n"], c["n"], s["dst"], step_id_in=s["step_id"],
                            pos_in=s["pos"], step_id_out=s["step_out"], pos_out=s["pos_out"], status=status)
        B.stepkv_q4_read(s["dst"], 0, s["n"], K=s["K_back"], V=s["V_back"], status=status)
        return dict(K=s["K_back"], V=s["V_back"], step_id=s["step_out"], pos=s["pos_out"])
    B.stepkv_q4_decode(s["q"], s["cache"], s["n"], out=s["out"], ws=s["ws"], status=status)
    return dict(out=s["out"])


def run(state):
    if own:
        return _own_pass(state)
    return globals()["_plain_" + state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ what it takes
def work(c):
    """Each input once, each output once: rows in bf16 (2 d bytes) and in 4 bits (d / 2 + d / 16)."""
    L, Hkv, d, n = c["L"], c["Hkv"], c["d"], c["n"]
    wide, narrow = 2 * d, d // 2 + d // 16
    if c["op"] == "write":
        by = 2 * L * Hkv * n * (wide + narrow + wide) + (4 * n if c["T"] else 0)
        return dict(bytes=by, flops=0)
    if c["op"] == "read":
        return dict(bytes=(2 if c["values"] else 1) * L * Hkv * n * (narrow + wide), flops=0)
    if c["op"] == "compact":
        return dict(bytes=2 * L * Hkv * n * (narrow + narrow + wide) + 20 * n, flops=0)
    rows = sum(_counts(c)) * (1 if c["ragged"] else L)
    return dict(bytes=2 * Hkv * rows * narrow + L * c["Hq"] * d * 6, flops=4 * rows * c["Hq"] * d)


# ------------------------------------------------------------------------------------------------ 64-bit values
def _values64(packed, s):
    """fp64 values of one layer's codes [..., d / 2] and scales [..., d / 32], nibble by nibble."""
    x = torch.empty((*packed.shape[:-1], packed.shape[-1] * 2), dtype=torch.float64, device=DEV)
    x[..., 0::2] = (packed % 16).double()
    x[..., 1::2] = torch.div(packed, 16, rounding_mode="floor").double()
    return (x - 8) * s.double().repeat_interleave(GROUP, -1)


def _nearest64(x):
    """fp64 [..., d]: the values that the codes of rows x stand for, from the definition."""
    v = x.double().unflatten(-1, (-1, GROUP))
    most = v.abs().amax(-1)
    t = torch.where(v.amax(-1) == most, -most, most) / 8
    unit = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(1e-300))) - 4)
    s = (torch.round(t / unit) * unit).clamp(-896, 896).to(torch.float16).double()[..., None]
    return torch.where(s == 0, 0.0, torch.round(v / torch.where(s == 0, 1.0, s)).clamp(-8, 7) * s).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, int(seed))
    cache = s["cache"]
    if c["op"] == "write":
        rows = slice(None) if s["idx"] is None else s["idx"]
        return {k: torch.stack([_nearest64(x[:, rows]) for x in s[k]]) for k in ("K", "V")}
    if c["op"] == "read":
        at = slice(c["row0"], c["row0"] + c["n"])
        return {k: torch.stack([_values64(a[:, at], b[:, at]) for a, b in zip(cache[k], cache[k + "_scale"])])
                for k in ("K", "V")[:1 + c["values"]]}
    if c["op"] == "compact":
        got = {k: torch.stack([_values64(a[:, s["idx"]], b[:, s["idx"]]) for a, b in zip(cache[k], cache[k + "_scale"])])
               for k in ("K", "V")}
        return dict(got, step_id=None, pos=None)
    G = c["Hq"] // c["Hkv"]
    counts = s["n"].tolist() * (1 if c["ragged"] else c["L"])
    out = torch.zeros((c["L"], c["Hq"], c["d"]), dtype=torch.float64, device=DEV)
    for l, n in enumerate(counts):
        if n:
            k, v = (_values64(cache[x][l][:, :n], cache[x + "_scale"][l][:, :n]) for x in ("K", "V"))
            p = torch.softmax(s["q"][l].double().view(c["Hkv"], G, -1) @ k.transpose(1, 2) / math.sqrt(c["d"]), -1)
            out[l] = (p @ v).reshape(c["Hq"], -1)
    return dict(out=out)
