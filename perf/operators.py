"""Serving operators for timing: attention over packed prompts, rows into and out of a 4-bit K/V cache, decoding over it.

A serving engine calls them together: the prompts of a batch lie back to back and attend (`packed`), their keys and values
go into the cache (`store`), each new token goes in too and attends to it (`decode`), and the cached rows of a
conversation come back in 16 bits when its next prompt arrives (`load`, then `packed` with more keys than queries).

`run` computes them from elementary torch operations in 32 bits, or with `own` set through the library's entry points.
A cached row is D values in blocks of 32: 4-bit codes of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4 and 6 (the low nibble is
the even element) under one power of two per block, held as a byte with bias 127.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
MOST_COST = 4.7e10     # bytes, or FLOPs over 50: what the largest listed case has
MOST_ROWS = 1 << 15    # of a drawn store or load


def _packed(name, Hq, Hkv, D, q_lens, k_lens="", causal=True, dtype="bf16", padding=0):
    """Packed sequences; `k_lens` empty: as many keys as queries.  `padding`: rows behind the last sequence."""
    return {"name": name, "op": "packed", "Hq": Hq, "Hkv": Hkv, "D": D, "q_lens": q_lens, "k_lens": k_lens, "causal": causal,
            "dtype": dtype, "padding": padding}


def _rows(name, op, T, B, Hkv, S, D, dtype="bf16", skipped=0):
    """T rows of a cache of B sequences of at most S; `skipped`: of how many rows one is padding (0: none)."""
    return {"name": name, "op": op, "T": T, "B": B, "Hkv": Hkv, "S": S, "D": D, "dtype": dtype, "skipped": skipped}


def _decode(name, Hq, Hkv, Sq, S, D, lens, dtype="bf16", seq_major=False):
    return {"name": name, "op": "decode", "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "S": S, "D": D, "lens": lens, "dtype": dtype,
            "seq_major": seq_major}


def listed():
    return [
        # two or three users' short prompts that arrive together: latency
        _packed("packed_few", 32, 8, 128, "77 1 203"),
        # texts of all lengths through an encoder, no mask
        _packed("packed_encoder_d64", 16, 16, 64, "512 37 480 129 256 1 390 64 511 333 200 18 450 97 301 512", causal=False, dtype="f16"),
        # a step of a busy engine: prompts from a line to a few pages
        _packed("packed_batch", 32, 8, 128, "1003 64 2777 350 1 511 1290 96 2048 700 129 1811 33 415", padding=100),
        # the next turns of conversations, their earlier turns in the cache: fewer queries than keys
        _packed("packed_turns", 64, 8, 128, "300 128 17 512 64 1 700 250", "4396 2048 6017 1512 8100 333 700 3250"),
        # long documents, many query heads
        _packed("packed_long", 64, 8, 128, "8192 5001 7003 2049"),
        # a decoding step's new row of every sequence
        _rows("store_step", "store", 32, 32, 8, 8192, 128),
        # the rows of a batch of prompts, a row in sixteen of it padding
        _rows("store_prompts", "store", 16384, 8, 8, 8192, 128, skipped=16),
        # a conversation's earlier turns, and many of them
        _rows("load_turn", "load", 700, 4, 8, 4096, 128, dtype="f16"),
        _rows("load_turns", "load", 32768, 8, 8, 16384, 128),
        # generation: a lone request
        _decode("decode_one", 32, 8, 1, 4099, 128, "4099"),
        # a full batch against 16k caches
        _decode("decode_full", 32, 8, 1, 16384, 128, "16384 16384 16384 16384 16384 16384 16384 16384"),
        # four positions at once (speculative), caches between empty and full, sequence-major
        _decode("decode_ragged_d64", 16, 4, 4, 16384, 64, "16384 5 777 12001 0 3333 8192 40 15000 1 9999 2500 6144 128 4097 11111",
                dtype="f16", seq_major=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(lens):
    return " ".join(str(x) for x in lens)


def draw(rng):
    op = rng.choice(["packed", "packed", "decode", "decode", "store", "load"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    group, Hkv = rng.choice([1, 1, 4, 4, 7, 8]), rng.choice([1, 2, 4, 8])
    if op == "packed":
        D, n = rng.choice([64, 64, 128, 128, 128, 80, 96, 192, 256]), _log(rng, 1, 40)
        longest = _log(rng, 8, 8192)
        q = [rng.choice([_log(rng, 1, longest), longest, rng.randint(1, longest)]) for _ in range(n)]
        k = [x + rng.choice([0, _log(rng, 1, 4096)]) for x in q] if rng.random() < 0.3 else []
        case = _packed("", Hkv * group, Hkv, D, _text(q), _text(k), rng.random() < 0.75, dtype, rng.choice([0, 0, rng.randint(1, 300)]))
        while _cost(case) > MOST_COST:
            q, k = q[: (len(q) + 1) // 2], k[: (len(k) + 1) // 2]
            if len(q) == 1:
                q, k = [max(1, q[0] // 2)], [max(1, x // 2) for x in k]
            case.update(q_lens=_text(q), k_lens=_text(k))
    elif op == "decode":
        D, B, S = rng.choice([64, 128, 128, 128, 96, 32, 256]), _log(rng, 1, 48), _log(rng, 32, 65536)
        while B * Hkv * S * D > 1 << 28:
            S //= 2
        lens = [S] * B if rng.random() < 0.4 else [rng.choice([S, rng.randint(1, S), _log(rng, 1, S)]) for _ in range(B)]
        Sq = rng.choice([1, 1, 1, 2, 4])
        case = _decode("", Hkv * group, Hkv, Sq, S, D, _text(lens), dtype, rng.random() < 0.5)
    else:
        D, B, T = rng.choice([64, 128, 128, 128, 96, 32, 256]), _log(rng, 1, 32), _log(rng, 1, MOST_ROWS)
        S = max(64, -(-T // B) + rng.randint(0, 500))
        case = _rows("", op, T, B, Hkv, S, D, dtype, rng.choice([0, 0, 5]))
    del case["name"]
    return case


def _lens(text):
    return [int(x) for x in text.split()]


def _packed_lens(case):
    q = _lens(case["q_lens"])
    return q, _lens(case["k_lens"]) if case["k_lens"] else q


def _pairs(Sq, Sk, causal):
    """(query, key) pairs that the mask leaves; the queries are the last Sq of Sk positions."""
    if not causal:
        return Sq * Sk
    seen = min(Sq, Sk)  # queries that see a key: the last of them sees Sk
    return seen * Sk - seen * (seen - 1) // 2


def work(case):
    c = case
    D = c["D"]
    if c["op"] == "packed":
        q, k = _packed_lens(c)
        return {"bytes": float((2 * c["Hq"] * sum(q) + 2 * c["Hkv"] * sum(k)) * D * 2 + c["Hq"] * sum(q) * 4),
                "flops": 4.0 * D * c["Hq"] * sum(_pairs(x, y, c["causal"]) for x, y in zip(q, k))}
    row = D / 2 + D / BLOCK  # of a cache, in bytes
    if c["op"] == "decode":
        lens = _lens(c["lens"])
        n_q = len(lens) * c["Hq"] * c["Sq"]
        return {"bytes": 2 * c["Hkv"] * sum(lens) * row + n_q * (4 * D + 4),
                "flops": 4.0 * D * c["Hq"] * sum(_pairs(c["Sq"], x, True) for x in lens)}
    values = 2.0 * (c["T"] - (c["T"] // c["skipped"] if c["skipped"] else 0)) * c["Hkv"]  # rows of a head
    # a stored row is read in 16 bits and written in 4; it comes back in 16 to be looked at
    return {"bytes": values * (2 * D + row) * (2 if c["op"] == "store" else 1), "flops": values * D * 4}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---- inputs ----

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _key_rows(gen, *shape):
    """Keys as models have them: a few channels much larger than the rest."""
    x = _normal(gen, *shape)
    x[..., torch.randperm(shape[-1], generator=gen, device="cuda")[: max(1, shape[-1] // 32)]] *= 4.0
    return x


def _offsets(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _scale_bytes(D):
    """A block's scale is a byte; rows of them are padded to 2, 4 or 8."""
    return 2 if D <= 64 else 4 if D <= 128 else 8


def _cache_of(x):
    """Codes and scales of rows [..., D], as a cache holds them."""
    D = x.shape[-1]
    value, power = _quantised(x, 252)
    mag = torch.tensor(MAGNITUDES, device="cuda")
    code = torch.bucketize(value.abs(), mag).to(torch.uint8) + 8 * (value < 0)
    code = code.view(*x.shape[:-1], D // 2, 2)
    scales = torch.full((*x.shape[:-1], _scale_bytes(D)), 127, dtype=torch.uint8, device="cuda")
    scales[..., : D // BLOCK] = (power + 127).squeeze(-1).to(torch.uint8)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scales


def _cache(gen, c, B):
    """K and V caches [B][Hkv][S]; sequence-major in memory where the case says so."""
    shape = (B, c["S"], c["Hkv"], c["D"]) if c.get("seq_major") else (B, c["Hkv"], c["S"], c["D"])
    out = []
    for make in (_key_rows, _normal):
        codes, scales = zip(*(_cache_of(make(gen, *shape[1:])) for _ in range(B)))  # a sequence at a time: in 32 bits it is eight times as large
        codes, scales = torch.stack(codes), torch.stack(scales)
        out += [t.transpose(1, 2) if c.get("seq_major") else t for t in (codes, scales)]
    return out


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) + 414)
    dtype = DTYPES[c["dtype"]]
    D, Hkv = c["D"], c["Hkv"]
    c["scale"] = 1.0 / math.sqrt(D)
    if c["op"] == "packed":
        q_lens, k_lens = _packed_lens(c)
        Tq, Tk = sum(q_lens) + c["padding"], sum(k_lens) + c["padding"]
        c["q"] = _normal(gen, Tq, c["Hq"], D).to(dtype)
        c["k"], c["v"] = _key_rows(gen, Tk, Hkv, D).to(dtype), _normal(gen, Tk, Hkv, D).to(dtype)
        c["cu_q"] = _offsets(q_lens)
        c["cu_k"] = _offsets(k_lens)
        c["o"] = torch.zeros((Tq, c["Hq"], D), device="cuda", dtype=dtype)
        c["lse"] = torch.zeros((c["Hq"], Tq), device="cuda", dtype=torch.float32)
        return c
    if c["op"] == "decode":
        lens = _lens(c["lens"])
        B = len(lens)
        c["cache"] = _cache(gen, c, B)
        c["lens_t"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        c["q"] = _normal(gen, B, c["Hq"], c["Sq"], D).to(dtype)
        c["o"] = torch.empty((B, c["Hq"], c["Sq"], D), device="cuda", dtype=dtype)
        c["lse"] = torch.empty((B, c["Hq"], c["Sq"]), device="cuda", dtype=torch.float32)
        if own:
            from paper_2604_14825_amd import binding as nb
            c["ws"] = torch.empty(nb.decode_kv4_workspace_bytes(B, c["Hq"], Hkv, c["Sq"], c["S"], D), device="cuda", dtype=torch.uint8)
            c["handle"] = nb.KV4Cache(*c["cache"])
        return c
    T, B, S = c["T"], c["B"], c["S"]
    # the rows of a batch: every sequence's next ones, in the order of the batch
    start = torch.randint(0, S - -(-T // B) + 1, (B,), generator=gen, device="cuda")
    t = torch.arange(T, device="cuda")
    per = -(-T // B)
    slots = (t // per) * S + start[t // per] + t % per
    if c["skipped"]:
        slots[c["skipped"] - 1 :: c["skipped"]] = -1
    c["slots"] = slots.to(torch.int32)
    c["k_out"] = torch.zeros((T, Hkv, D), device="cuda", dtype=dtype)
    c["v_out"] = torch.zeros((T, Hkv, D), device="cuda", dtype=dtype)
    if c["op"] == "store":
        c["k"], c["v"] = _key_rows(gen, T, Hkv, D).to(dtype), _normal(gen, T, Hkv, D).to(dtype)
        width = _scale_bytes(D)
        c["cache"] = [torch.full((B, Hkv, S, n), fill, device="cuda", dtype=torch.uint8) for n, fill in ((D // 2, 0), (width, 127)) * 2]
    else:
        c["cache"] = _cache(gen, c, B)
    if own:
        from paper_2604_14825_amd import binding as nb
        c["handle"] = nb.KV4Cache(*c["cache"])
    return c


# ---- the plain forms ----

def _quantised(x, most):
    """The codes' signed magnitudes, and the powers of their blocks [..., 1], of rows in 32 bits."""
    b = x.float().view(*x.shape[:-1], -1, BLOCK)
    mantissa, power = torch.frexp(b.abs().amax(-1, keepdim=True))  # mantissa in [0.5, 1)
    power = (power - 3 + (mantissa >= 0.875)).clamp(-126, most - 127)
    y = torch.ldexp(b, -power)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.where(y < 0, -a, a).view(x.shape), power


def _values(codes, scales, D):
    """Rows of a cache, in 32 bits."""
    low_high = torch.stack([codes & 15, codes >> 4], -1).view(*codes.shape[:-1], D).long()
    table = torch.tensor(MAGNITUDES + tuple(-x for x in MAGNITUDES), device="cuda")
    power = scales[..., : D // BLOCK].float() - 127
    return table[low_high] * torch.exp2(power).repeat_interleave(BLOCK, -1)


def _attend(q, k, v, scale, mask):
    """q [..., R, D], k and v [..., S, D], mask (true where a key is seen) broadcast over [..., R, S]; all in 32 bits."""
    s = torch.matmul(q, k.transpose(-1, -2)) * scale
    if mask is not None:
        s = s.masked_fill(~mask, -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3.0e38)  # a row that sees nothing: every exponential below is 0
    p = torch.exp(s - top)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / l.clamp(min=1e-30)
    return o, torch.where(l > 0, torch.log(l) + top, -math.inf).squeeze(-1)


def _plain_packed(c):
    q_lens, k_lens = _packed_lens(c)
    Hq, Hkv, D, g = c["Hq"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    o, lse = torch.zeros_like(c["o"]), torch.zeros_like(c["lse"])
    q0 = k0 = 0
    for Sq, Sk in zip(q_lens, k_lens):
        q = c["q"][q0 : q0 + Sq].float().permute(1, 0, 2).reshape(Hkv, g * Sq, D)
        k, v = (c[n][k0 : k0 + Sk].float().permute(1, 0, 2).contiguous() for n in ("k", "v"))
        mask = None
        if c["causal"]:
            mask = torch.arange(Sk, device="cuda") <= torch.arange(Sq, device="cuda")[:, None] + (Sk - Sq)
            mask = mask.repeat(g, 1)
        x, y = _attend(q, k, v, c["scale"], mask)
        o[q0 : q0 + Sq] = x.view(Hq, Sq, D).permute(1, 0, 2).to(o.dtype)
        lse[:, q0 : q0 + Sq] = y.view(Hq, Sq)
        q0, k0 = q0 + Sq, k0 + Sk
    return {"o": o, "lse": lse}


def _plain_decode(c):
    B, Hq, Sq, D = c["q"].shape
    Hkv, S, g = c["Hkv"], c["S"], Hq // c["Hkv"]
    kc, ks, vc, vs = c["cache"]
    last = c["lens_t"].view(B, 1, 1, 1) - Sq + torch.arange(Sq, device="cuda").repeat(g).view(1, 1, g * Sq, 1)
    mask = torch.arange(S, device="cuda") <= last
    o, lse = _attend(c["q"].float().reshape(B, Hkv, g * Sq, D), _values(kc, ks, D).contiguous(), _values(vc, vs, D), c["scale"], mask)
    return {"o": o.view(B, Hq, Sq, D).to(c["o"].dtype), "lse": lse.view(B, Hq, Sq)}


def _plain_store(c):
    stored = (c["slots"] >= 0).view(-1, 1, 1)
    out = {}
    for n in ("k", "v"):
        value, power = _quantised(c[n], 140 if c["dtype"] == "f16" else 252)
        value = torch.ldexp(value.view(*value.shape[:-1], -1, BLOCK), power).view(value.shape)
        out[n] = torch.where(stored, value, 0.0).to(c[n].dtype)
    return out


def _plain_load(c):
    S, D = c["S"], c["D"]
    stored = (c["slots"] >= 0).view(-1, 1, 1)
    slot = c["slots"].clamp(min=0).long()
    kc, ks, vc, vs = c["cache"]
    at = lambda t: t[slot // S, :, slot % S]
    return {n: torch.where(stored, _values(at(codes), at(scales), D), 0.0).to(c[n + "_out"].dtype) for n, codes, scales in (("k", kc, ks), ("v", vc, vs))}


def run(state):
    c = state
    if not own:
        return {"packed": _plain_packed, "decode": _plain_decode, "store": _plain_store, "load": _plain_load}[c["op"]](c)
    from paper_2604_14825_amd import binding as nb
    if c["op"] == "packed":
        nb.naut_attn_fwd_packed(c["q"], c["k"], c["v"], c["o"], c["lse"], c["cu_q"], c["cu_k"], c["causal"], c["scale"])
        return {"o": c["o"], "lse": c["lse"]}
    if c["op"] == "decode":
        nb.naut_attn_decode_kv4(c["q"], c["o"], c["lse"], c["handle"], c["lens_t"], True, c["scale"], c["ws"])
        return {"o": c["o"], "lse": c["lse"]}
    if c["op"] == "store":
        nb.naut_kv4_store(c["k"], c["v"], c["handle"], c["slots"])
    nb.naut_kv4_load(c["k_out"], c["v_out"], c["handle"], c["slots"])  # what was stored comes back as the values it stands for
    return {"k": c["k_out"], "v": c["v_out"]}


# ---- the definitions in 64 bits ----

def _exact_rows(x, most):
    """Every value on the grid of its block: by comparison with the halves between neighbours, ties to the even code."""
    b = x.double().reshape(*x.shape[:-1], -1, BLOCK)
    power = torch.frexp(b.abs().amax(-1, keepdim=True) / 7.0)[1].clamp(-126, most - 127)  # the least with max / 2^power < 7
    a = b.abs() * torch.exp2(-power.double())
    code = sum(((a >= t) if i % 2 else (a > t)).long() for i, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    y = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")[code] * torch.exp2(power.double())
    return (y * torch.sign(b)).reshape(x.shape)


def _exact_cached(codes, scales, D):
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
    out = torch.empty((*codes.shape[:-1], D), dtype=torch.float64, device="cuda")
    for i, nibble in enumerate((codes.int() % 16, codes.int() // 16)):
        out[..., i::2] = torch.where(nibble < 8, 1.0, -1.0).double() * grid[(nibble % 8).long()]
    for i in range(D // BLOCK):
        out[..., i * BLOCK : (i + 1) * BLOCK] *= torch.pow(2.0, scales[..., i : i + 1].double() - 127.0)
    return out


def _exact_head(q, k, v, scale, causal):
    """One head [Sq, D] against [Sk, D]."""
    Sq, Sk = q.shape[0], k.shape[0]
    if Sk == 0:
        return torch.zeros_like(q), q.new_full((Sq,), -math.inf)
    s = (q @ k.t()) * scale
    if causal:
        s = torch.tril(torch.ones_like(s), Sk - Sq).log() + s
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse > -math.inf, lse, 0.0)[:, None])
    return p @ v, lse


def exact(case, seed):
    c = prepare(case, seed)
    D = c["D"]
    if c["op"] == "packed":
        q_lens, k_lens = _packed_lens(c)
        g = c["Hq"] // c["Hkv"]
        o, lse = c["o"].double(), c["lse"].double()
        a = b = 0
        for Sq, Sk in zip(q_lens, k_lens):
            for h in range(c["Hq"]):
                o[a : a + Sq, h], lse[h, a : a + Sq] = _exact_head(
                    c["q"][a : a + Sq, h].double(), c["k"][b : b + Sk, h // g].double(), c["v"][b : b + Sk, h // g].double(), c["scale"], c["causal"])
            a, b = a + Sq, b + Sk
        return {"o": o, "lse": lse}
    if c["op"] == "decode":
        g = c["Hq"] // c["Hkv"]
        o, lse = torch.empty_like(c["o"], dtype=torch.float64), torch.empty_like(c["lse"], dtype=torch.float64)
        kc, ks, vc, vs = c["cache"]
        for b, n in enumerate(_lens(c["lens"])):
            k, v = _exact_cached(kc[b, :, :n], ks[b, :, :n], D), _exact_cached(vc[b, :, :n], vs[b, :, :n], D)
            for h in range(c["Hq"]):
                o[b, h], lse[b, h] = _exact_head(c["q"][b, h].double(), k[h // g], v[h // g], c["scale"], True)
        return {"o": o, "lse": lse}
    kept = (c["slots"] >= 0).double().view(-1, 1, 1)
    if c["op"] == "store":
        return {n: _exact_rows(c[n], 140 if c["dtype"] == "f16" else 252) * kept for n in ("k", "v")}
    kc, ks, vc, vs = c["cache"]
    at = c["slots"].clamp(min=0).long()
    b, s = at // c["S"], at % c["S"]
    return {n: _exact_cached(codes[b, :, s], scales[b, :, s], D) * kept for n, codes, scales in (("k", kc, ks), ("v", vc, vs))}
