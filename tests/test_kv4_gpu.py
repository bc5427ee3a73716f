"""The 4-bit cache: codes and scales bit for bit, rows read back exactly, decode-time attention over it against plain 64-bit
attention on the values that it holds, and packed prompts, stores, decode steps and loads together."""
import math

import numpy as np
import pytest
import torch

from paper_2604_14825_amd import binding as nb

import serving_util as su

pytestmark = pytest.mark.gpu


def new_cache(B, Hkv, S, D, seq_major=False, fill=0xFF):
    """A cache of bytes that would show if they were read: scale 255 is not a number."""
    n = nb.kv4_scale_bytes(D)
    shape = lambda w: (B, S, Hkv, w) if seq_major else (B, Hkv, S, w)
    make = lambda w: torch.full(shape(w), fill, dtype=torch.uint8, device="cuda")
    ts = [make(D // 2), make(n), make(D // 2), make(n)]
    return nb.KV4Cache(*(t.transpose(1, 2) if seq_major else t for t in ts))


def slots_of(x):
    return torch.tensor(np.asarray(x).astype(np.int32), device="cuda")


def wide_rows(T, H, D, dtype, seed):
    """Rows of every magnitude: blocks of their own power, ties, zeros, the type's largest and its subnormals."""
    rng = np.random.default_rng(seed)
    lo, hi = (-22, 13) if dtype == "f16" else (-130, 122)
    x = rng.standard_normal((T, H, D // 32, 32)) * 2.0 ** rng.integers(lo, hi, (T, H, D // 32, 1))
    grid = rng.choice(np.concatenate([su.MAGNITUDES, su.HALVES, [7.0, 6.5, 7.5]]), (T, H, D // 32, 32)) * rng.choice([-1, 1], (T, H, D // 32, 32))
    pick = rng.integers(0, 8, (T, H, D // 32, 1))
    x = np.where(pick == 0, grid * 2.0 ** rng.integers(lo + 10, hi - 3, (T, H, D // 32, 1)), x)
    x = np.where(pick == 1, 0.0, x)
    top = 65504.0 if dtype == "f16" else float(torch.finfo(torch.bfloat16).max)
    x = np.where((pick == 2) & (rng.integers(0, 16, x.shape) == 0), top, x)
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -126
    x = np.where(pick == 3, rng.integers(-9, 10, x.shape) * tiny, x)
    x = np.clip(x, -top, top)
    return torch.tensor(x.reshape(T, H, D)).to(su.TORCH[dtype]).cuda()


def held(cache):
    """The values of K and V [B,Hkv,S,D] (garbage where nothing was stored)."""
    kc, ks, vc, vs = (t.cpu().numpy() for t in cache.tensors)
    return su.decode(kc, ks, cache.D), su.decode(vc, vs, cache.D)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("seq_major", [False, True])
def test_store_bit_for_bit(dtype, D, seq_major):
    B, Hkv, S, T = 3, 2, 50, 77
    print("store", dtype, D, seq_major, flush=True)
    cache = new_cache(B, Hkv, S, D, seq_major, fill=0xA5)
    rng = np.random.default_rng(D)
    slots = rng.permutation(B * S)[:T]
    slots[5] = -1
    slots[9] = B * S          # beyond the cache
    slots[10] = 0x7fffffff
    slots[11] = -0x80000000
    k, v = wide_rows(T, Hkv, D, dtype, 1), wide_rows(T, Hkv, D, dtype, 2)
    nb.naut_kv4_store(k, v, cache, slots_of(slots))
    torch.cuda.synchronize()
    got = [t.cpu().numpy() for t in cache.tensors]
    want = [np.full(t.shape, 0xA5, np.uint8) for t in got]
    for i, x in enumerate((k, v)):
        codes, scales = su.encode(x.double().cpu().numpy(), dtype)
        for t, s in enumerate(slots):
            if 0 <= s < B * S:
                want[2 * i][s // S, :, s % S] = codes[t]
                want[2 * i + 1][s // S, :, s % S, : D // 32] = scales[t]
    for name, g, w in zip(("K codes", "K scales", "V codes", "V scales"), got, want):
        assert np.array_equal(g, w), "%s: %d bytes differ, first at %s: %x for %x" % (name, (g != w).sum(), np.argwhere(g != w)[0], g[g != w][0], w[g != w][0])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [32, 96, 128, 256])
def test_load_gives_the_values_and_leaves_skipped_rows(dtype, D):
    """Every code under every scale that the type holds exactly; a position read twice; rows with slots outside the cache."""
    rng = np.random.default_rng(3)
    B, Hkv, S = 2, 2, 128
    cache = new_cache(B, Hkv, S, D)
    lo, hi = (104, 140) if dtype == "f16" else (1, 252)
    for t in cache.tensors[0::2]:
        t.copy_(torch.tensor(rng.integers(0, 256, t.shape), dtype=torch.uint8))
    for t in cache.tensors[1::2]:
        t.copy_(torch.tensor(rng.integers(lo, hi + 1, t.shape), dtype=torch.uint8))
    slots = np.concatenate([rng.integers(0, B * S, 300), [3, 3, -1, B * S, -77]])
    big = torch.full((305, Hkv, 2 * D), 7.0, dtype=su.TORCH[dtype], device="cuda")
    k, v = big[..., :D], big[..., D:]
    nb.naut_kv4_load(k, v, cache, slots_of(slots))
    torch.cuda.synchronize()
    for x, want in zip((k, v), held(cache)):
        got = x.double().cpu().numpy()
        assert (got[302:] == 7.0).all()
        w = want[slots[:302] // S, :, slots[:302] % S]
        exact = torch.tensor(w).to(su.TORCH[dtype]).double().numpy()  # f16: below 2^-24 the values round
        assert np.array_equal(got[:302], exact), (np.abs(got[:302] - exact).max(), np.argwhere(got[:302] != exact)[0])


def test_load_of_scales_beyond_f16_stays_finite():
    cache = new_cache(1, 1, 4, 64, fill=0x77)   # codes 7: magnitude 6
    for t in cache.tensors[1::2]:
        t[0, 0, :, :] = torch.tensor([[140, 140], [141, 200], [254, 254], [1, 103]], dtype=torch.uint8, device="cuda")
    k, v = torch.empty((4, 1, 64), device="cuda", dtype=torch.float16), torch.empty((4, 1, 64), device="cuda", dtype=torch.float16)
    nb.naut_kv4_load(k, v, cache, slots_of([0, 1, 2, 3]))
    assert (k[:3] == 49152.0).all() and (v[:3] == 49152.0).all()
    assert (k[3, 0, :32] == 0).all() and (k[3, 0, 32:] == 6 * 2.0 ** -24).all()


def test_load_of_scales_beyond_those_that_a_store_writes():
    """bf16: what the type holds is exact up to the last scale that is a number, the rest infinite; 252 is the last where all is finite."""
    cache = new_cache(1, 1, 3, 32)
    for t in cache.tensors[0::2]:
        t[0, 0, :, :] = torch.tensor([0x10 * (2 * i + 1) + 2 * i for i in range(8)] * 2, dtype=torch.uint8, device="cuda")
    for t in cache.tensors[1::2]:
        t[0, 0, :, 0] = torch.tensor([252, 253, 254], dtype=torch.uint8, device="cuda")
    k, v = (torch.empty((3, 1, 32), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    nb.naut_kv4_load(k, v, cache, slots_of([0, 1, 2]))
    codes = np.array(list(range(16)) * 2)
    signed = np.where(codes < 8, 1.0, -1.0) * su.MAGNITUDES[codes & 7]
    for i, byte in enumerate((252, 253, 254)):
        want = signed * 2.0 ** (byte - 127)
        want = np.where(np.abs(want) < 2.0 ** 128, want, np.copysign(np.inf, want))
        assert np.isfinite(want).all() == (byte == 252)
        for x in (k, v):
            assert np.array_equal(x[i, 0].double().cpu().numpy(), want), byte


@pytest.mark.parametrize("D", [64, 128, 256])
def test_f16_decode_takes_the_values_that_a_load_gives(D):
    """A cache stored from bf16 with scales above and below what f16 holds: decode in f16 is attention over its rows loaded in f16."""
    gen = torch.Generator(device="cuda").manual_seed(19)
    S, n = 300, 257
    k, v = (torch.randn((S, 2, D), device="cuda", generator=gen) for _ in range(2))
    k[:, :, 32:64] *= 1e-8
    v[::7] *= 2.0 ** 16     # scales of 2^14 and more
    v[:, :, :32] *= 1e-8
    cache = new_cache(1, 2, S, D)
    every = slots_of(np.arange(S))
    nb.naut_kv4_store(k.to(torch.bfloat16), v.to(torch.bfloat16), cache, every)
    assert (cache.tensors[3][..., : D // 32] > 140).any()
    k16, v16 = (torch.empty((S, 2, D), device="cuda", dtype=torch.float16) for _ in range(2))
    nb.naut_kv4_load(k16, v16, cache, every)
    q = torch.randn((1, 4, 1, D), device="cuda", generator=gen).to(torch.float16)
    o, lse = torch.empty((1, 4, 1, D), device="cuda"), torch.empty((1, 4, 1), device="cuda")
    ws = torch.empty(nb.decode_kv4_workspace_bytes(1, 4, 2, 1, S, D), dtype=torch.uint8, device="cuda")
    nb.naut_attn_decode_kv4(q, o, lse, cache, slots_of([n]), True, D ** -0.5, ws)
    torch.cuda.synchronize()
    qn, kn, vn = (x.double().cpu().numpy() for x in (q, k16, v16))
    for h in range(4):
        ref = su.reference(qn[0, h], kn[:n, h // 2], vn[:n, h // 2], D ** -0.5, True)
        su.check(o[0, h].double().cpu().numpy(), lse[0, h].double().cpu().numpy(), ref, "f16", "f32", n, "head %d" % h)


def filled(B, Hkv, S, D, lens, dtype, seq_major=False, seed=0, magnify=1.0):
    """A cache whose first lens[b] positions hold rows, the rest garbage that is not a number."""
    cache = new_cache(B, Hkv, S, D, seq_major)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    slots = np.concatenate([b * S + np.arange(n) for b, n in enumerate(lens)] + [[-1]])
    k, v = (torch.randn((len(slots), Hkv, D), device="cuda", generator=gen) for _ in range(2))
    nb.naut_kv4_store((k * magnify).to(su.TORCH[dtype]), v.to(su.TORCH[dtype]), cache, slots_of(slots))
    return cache


def reference(q, cache, lens, scale, causal):
    q = q.double().cpu().numpy()
    k, v = held(cache)
    B, Hq, Sq, D = q.shape
    g = Hq // cache.Hkv
    out = [np.zeros_like(q), np.zeros(q.shape[:3]), np.zeros_like(q), np.zeros(q.shape[:3])]
    for b in range(B):
        for h in range(Hq):
            for x, y in zip(out, su.reference(q[b, h], k[b, h // g, : lens[b]], v[b, h // g, : lens[b]], scale, causal)):
                x[b, h] = y
    return out


def run(Hq, Hkv, Sq, S, D, lens, causal=True, dtype="bf16", out="bf16", seq_major=False, given=True, seed=0, magnify=1.0, layout=False):
    what = "decode kv4 Hq %d Hkv %d Sq %d S %d D %d lens %s causal %d %s->%s seq_major %d" % (
        Hq, Hkv, Sq, S, D, lens if len(lens) < 20 else len(lens), causal, dtype, out, seq_major)
    print(what, flush=True)
    B = len(lens)
    cache = filled(B, Hkv, S, D, lens, dtype, seq_major, seed, magnify)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = torch.randn((B, Hq, Sq, D), device="cuda", generator=gen).to(su.TORCH[dtype])
    o = torch.full((B, Hq, Sq, D), float("nan"), device="cuda", dtype=su.TORCH[out])
    if layout:  # [B,Sq,Hq,D] with room between the rows
        q = torch.empty((B, Sq, Hq, D + 8), device="cuda", dtype=q.dtype)[..., :D].transpose(1, 2).copy_(q)
        o = torch.full((B, Sq, Hq, D + 8), 7.0, device="cuda", dtype=o.dtype)[..., :D].transpose(1, 2)
    lse = torch.full((B, Hq, Sq), float("nan"), device="cuda")
    ws = torch.full((nb.decode_kv4_workspace_bytes(B, Hq, Hkv, Sq, S, D),), 0xFF, dtype=torch.uint8, device="cuda")
    scale = 1 / math.sqrt(D)
    nb.naut_attn_decode_kv4(q, o, lse, cache, slots_of(lens) if given else None, causal, scale, ws)
    torch.cuda.synchronize()
    su.check(o.double().cpu().numpy(), lse.double().cpu().numpy(), reference(q, cache, lens, scale, causal), dtype, out, max(max(lens), 1), what)
    return o, lse


EDGES = [1, 31, 32, 33, 0, 64, 127, 129, 200, 16, 15, 17]


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_at_the_edges_of_blocks(D, causal):
    run(4, 2, 1, 200, D, EDGES, causal)
    run(4, 2, 3, 203, D, EDGES, causal, seed=1)   # causal: rows that see nothing where there are fewer keys than queries


@pytest.mark.parametrize("Hq,Hkv,Sq", [(1, 1, 1), (8, 8, 1), (16, 1, 1), (17, 1, 1), (7, 1, 3), (32, 1, 1), (40, 1, 1), (8, 2, 5), (24, 2, 3), (6, 3, 16), (4, 2, 33)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_query_rows(Hq, Hkv, Sq, D):
    run(Hq, Hkv, Sq, 300, D, [300, 77, 40, 2], seed=2)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_types_and_layouts(D, dtype, out):
    run(8, 2, 2, 500, D, [500, 123], True, dtype, out, seq_major=True, layout=True, seed=3)


@pytest.mark.parametrize("D,S,B", [(128, 20000, 1), (128, 5000, 9), (64, 40001, 2), (256, 9000, 3), (96, 12345, 2)])
def test_long_caches(D, S, B):
    rng = np.random.default_rng(S)
    run(8, 2, 1, S, D, [S] + [int(x) for x in rng.integers(1, S, B - 1)], seed=4)
    run(8, 2, 1, S, D, [S] * B, given=False, seed=4)


@pytest.mark.parametrize("B", [63, 64, 65, 200, 1100])
def test_many_sequences(B):
    """64 to a lane each, more than the splits that the plan aims at."""
    rng = np.random.default_rng(B)
    run(2, 1, 1, 150, 64, [int(x) for x in rng.integers(0, 151, B)], seed=5)


def test_one_long_sequence_among_short_ones():
    run(8, 2, 1, 30000, 128, [3, 30000, 0, 17, 1, 2900], seed=6)
    run(6, 3, 1, 30000, 64, [30000] + [5] * 40, seed=6)     # three K/V heads: a number of splits that eight does not divide
    run(10, 5, 2, 12000, 128, [12000, 300, 11000], seed=6)


def test_more_sequences_than_fill_the_chip():
    """And too long for a part each: the mean is cut in halves."""
    rng = np.random.default_rng(300)
    run(2, 1, 1, 3000, 64, [int(x) for x in rng.integers(0, 3001, 300)], seed=14)
    run(4, 4, 1, 2500, 128, [2500] * 70, seed=14)


@pytest.mark.parametrize("B", [255, 256, 257, 1025])
def test_many_unlike_sequences(B):
    """The plan of many: empty ones, one that is cut into many parts, few or none that are cut."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in np.where(rng.random(B) < 0.5, 0, rng.integers(1, 100, B))]
    H = 1 if B > 1000 else 3
    run(H, H, 1, 2080, 32, lens, seed=15)
    lens[0], lens[B // 2], lens[-1] = 2080, 2000, 2079
    run(2 * H, H, 1, 2080, 64, lens, seed=15)
    run(3, 1, 2, 4200, 32, lens, False, "f16", "f32", seed=15)
    run(2, 1, 1, 2080, 32, [0] * B, seed=15)


@pytest.mark.parametrize("B,Hkv,S", [(63, 8, 3000), (40, 8, 2500), (300, 1, 2240), (400, 1, 2240), (1025, 2, 2100), (3, 1, 30000), (70, 3, 2600), (5, 300, 600)])
def test_partials_stay_in_the_workspace(B, Hkv, S):
    """Sequences that are all split, nearly all, and few of many: nothing is written behind the workspace, whose bytes are not a number."""
    lens = [S] * B if B < 1000 else [S if b % 16 == 0 else 3 for b in range(B)]
    print("partials", B, Hkv, S, flush=True)
    D = 32
    cache = filled(B, Hkv, S, D, lens, "bf16", seed=17)
    q = torch.randn((B, Hkv, 1, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(18)).to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((B, Hkv, 1), device="cuda")
    n = nb.decode_kv4_workspace_bytes(B, Hkv, Hkv, 1, S, D)
    room = torch.full((n + (1 << 22),), 0xFF, dtype=torch.uint8, device="cuda")
    nb.naut_attn_decode_kv4(q, o, lse, cache, slots_of(lens), True, 0.2, room[:n])
    torch.cuda.synchronize()
    assert (room[n:] == 0xFF).all()
    some = sorted(set(range(0, B, max(1, B // 40))) | {B - 1})
    k, v = (su.decode(c[some].cpu().numpy(), s[some].cpu().numpy(), D) for c, s in (cache.tensors[:2], cache.tensors[2:]))
    qn, on, ln = q[some].double().cpu().numpy(), o[some].double().cpu().numpy(), lse[some].double().cpu().numpy()
    for i, b in enumerate(some):
        for h in sorted({0, Hkv // 2, Hkv - 1}):
            ref = su.reference(qn[i, h], k[i, h, : lens[b]], v[i, h, : lens[b]], 0.2, True)
            su.check(on[i, h], ln[i, h], ref, "bf16", "bf16", S, "sequence %d head %d" % (b, h))


def test_a_plan_in_a_captured_call_follows_the_lengths():
    B, S = 300, 2200
    cache = filled(B, 2, S, 64, [S] * B, "bf16")
    gen = torch.Generator(device="cuda").manual_seed(16)
    q = torch.randn((B, 4, 1, 64), device="cuda", generator=gen).to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((B, 4, 1), device="cuda")
    ws = torch.empty(nb.decode_kv4_workspace_bytes(B, 4, 2, 1, S, 64), dtype=torch.uint8, device="cuda")
    lens = slots_of([S] * B)
    call = lambda: nb.naut_attn_decode_kv4(q, o, lse, cache, lens, True, 0.125, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    rng = np.random.default_rng(16)
    for these in ([7] * B, [0] * (B - 1) + [S], [int(x) for x in rng.integers(0, S + 1, B)], [S] * B):
        lens.copy_(slots_of(these))
        ws.fill_(0xFF)
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = o.clone(), lse.clone()
        ws.zero_()
        o.fill_(7.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, o) and torch.equal(got_lse, lse)
        su.check(o.double().cpu().numpy(), lse.double().cpu().numpy(), reference(q, cache, these, 0.125, True), "bf16", "bf16", S, "replayed plan")


@pytest.mark.parametrize("D", [64, 128, 256])
def test_maxima_that_move(D):
    run(8, 2, 2, 900, D, [900, 411], seed=7, magnify=8.0)
    run(8, 2, 2, 900, D, [900, 411], True, "f16", "f16", seed=7, magnify=8.0)


def test_scale_zero_is_the_mean():
    cache = filled(1, 1, 100, 64, [70], "bf16")
    q = torch.randn((1, 1, 1, 64), device="cuda").to(torch.bfloat16)
    o, lse = torch.empty((1, 1, 1, 64), device="cuda", dtype=torch.float32), torch.empty((1, 1, 1), device="cuda")
    ws = torch.empty(nb.decode_kv4_workspace_bytes(1, 1, 1, 1, 100, 64), dtype=torch.uint8, device="cuda")
    nb.naut_attn_decode_kv4(q, o, lse, cache, slots_of([70]), True, 0.0, ws)
    want = held(cache)[1][0, 0, :70].mean(0)
    assert np.abs(o[0, 0, 0].double().cpu().numpy() - want).max() <= 70 * 2.0 ** -24 * 6 and abs(float(lse) - math.log(70)) < 1e-5


def test_lengths_outside_the_cache_count_as_its_ends():
    cache = filled(3, 1, 100, 64, [100, 100, 100], "bf16")
    q = torch.randn((3, 2, 1, 64), device="cuda").to(torch.bfloat16)
    ws = torch.empty(nb.decode_kv4_workspace_bytes(3, 2, 1, 1, 100, 64), dtype=torch.uint8, device="cuda")
    got = []
    for lens in ([-5, 101, 0x7fffffff], [0, 100, 100]):
        o, lse = torch.empty_like(q), torch.empty((3, 2, 1), device="cuda")
        nb.naut_attn_decode_kv4(q, o, lse, cache, slots_of(lens), True, 0.125, ws)
        torch.cuda.synchronize()
        got.append((o, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert (got[0][0][0] == 0).all() and torch.isneginf(got[0][1][0]).all()


def test_calls_repeat_bit_for_bit_and_on_another_stream():
    a, la = run(16, 4, 1, 3000, 128, [3000, 1234, 5], seed=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b, lb = run(16, 4, 1, 3000, 128, [3000, 1234, 5], seed=8)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_two_captured_calls_share_a_workspace_in_turn_and_follow_the_lengths():
    B, Hq, Hkv, S, D = 3, 8, 2, 2000, 128
    cache = filled(B, Hkv, S, D, [S] * B, "bf16", seed=9)
    gen = torch.Generator(device="cuda").manual_seed(10)
    qs = [torch.randn((B, Hq, 1, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2)]
    os = [torch.empty_like(q) for q in qs]
    lens = slots_of([S, 1, 700])
    ws = torch.empty(nb.decode_kv4_workspace_bytes(B, Hq, Hkv, 1, S, D), dtype=torch.uint8, device="cuda")
    call = lambda i: nb.naut_attn_decode_kv4(qs[i], os[i], None, cache, lens, True, 0.09, ws)
    call(0)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i)
    for now in ([S, 1, 700], [1, 1, 1], [0, S, S - 1], [64, 500, 31], [S, 1, 700]):
        lens.copy_(slots_of(now))
        ws.fill_(0xFF)
        for i in (0, 1):
            os[i].fill_(7.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in os]
        for i in (0, 1):
            call(i)
            torch.cuda.synchronize()
            assert torch.equal(got[i], os[i]), (now, i)
            ref = reference(qs[i], cache, now, 0.09, True)
            su.check(os[i].double().cpu().numpy(), None, ref, "bf16", "bf16", S, str(now))


@pytest.mark.parametrize("B,S", [(1, 1), (7, 1), (3, 31), (300, 2)])
def test_the_smallest_caches(B, S):
    for D in (32, 128, 256):
        run(4, 2, 1, S, D, [S] * B, seed=21)
        run(4, 2, 3, S, D, [b % (S + 1) for b in range(B)], seed=21)


def test_a_captured_step_follows_slots_and_lengths():
    """One graph of a step of generation: new rows into the cache, attention over it, the rows back; slots and lengths change between replays,
    a finished sequence's slot is skipped, and eager work runs in between."""
    B, Hq, Hkv, S, D = 4, 8, 2, 700, 128
    lens0 = [600, 1, 33, 0]
    cache = filled(B, Hkv, S, D, lens0, "bf16", seed=22)
    gen = torch.Generator(device="cuda").manual_seed(23)
    rows = lambda H: torch.randn((B, H, D), device="cuda", generator=gen).to(torch.bfloat16)
    q, k, v = rows(Hq), rows(Hkv), rows(Hkv)
    o, lse = torch.empty((B, Hq, 1, D), device="cuda", dtype=torch.bfloat16), torch.empty((B, Hq, 1), device="cuda")
    k_back, v_back = torch.empty_like(k), torch.empty_like(v)
    slots, lens = slots_of([-1] * B), slots_of(lens0)
    ws = torch.empty(nb.decode_kv4_workspace_bytes(B, Hq, Hkv, 1, S, D), dtype=torch.uint8, device="cuda")

    def step():
        nb.naut_kv4_store(k, v, cache, slots)
        nb.naut_attn_decode_kv4(q.unsqueeze(2), o, lse, cache, lens, True, 0.09, ws)
        nb.naut_kv4_load(k_back, v_back, cache, slots)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    have = list(lens0)
    for turn in range(5):
        runs = [b != turn for b in range(B)]  # one sequence sits out
        slots.copy_(slots_of([b * S + have[b] if runs[b] else -1 for b in range(B)]))
        have = [n + r for n, r in zip(have, runs)]
        lens.copy_(slots_of(have))
        for x, H in ((q, Hq), (k, Hkv), (v, Hkv)):
            x.copy_(rows(H))
        k_back.fill_(7.0)
        v_back.fill_(7.0)
        before = [t.clone() for t in cache.tensors]
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            for i, x in enumerate((k, v)):
                codes, scales = su.encode(x[b].double().cpu().numpy(), "bf16")
                for j, new in ((2 * i, codes), (2 * i + 1, scales)):
                    if runs[b]:
                        before[j][b, :, have[b] - 1, : new.shape[-1]] = torch.tensor(new, device="cuda")
                    assert torch.equal(cache.tensors[j][b], before[j][b]), (turn, b)
        values = held(cache)
        for b in range(B):
            for x, want in zip((k_back, v_back), values):
                got = x[b].double().cpu().numpy()
                assert np.array_equal(got, want[b, :, have[b] - 1]) if runs[b] else (got == 7.0).all()
        su.check(o.double().cpu().numpy(), lse.double().cpu().numpy(), reference(q.unsqueeze(2), cache, have, 0.09, True), "bf16", "bf16", S, "turn %d" % turn)


def test_a_cache_past_4_gib():
    """Offsets that pass 32 bits: far-apart positions, and the last sequences of a large cache."""
    B, Hkv, S, D, step = 2, 1, 1100, 64, 1 << 22
    codes = [torch.empty(B * S * step, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((B, Hkv, S, 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    kc, vc = (torch.as_strided(c, (B, Hkv, S, D // 2), (S * step, S * step, step, 1)) for c in codes)
    cache = nb.KV4Cache(kc, scales[0], vc, scales[1])
    gen = torch.Generator(device="cuda").manual_seed(11)
    rows = [torch.randn((B * S, Hkv, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2)]
    slots = slots_of(np.arange(B * S))
    nb.naut_kv4_store(*rows, cache, slots)
    back = [torch.empty_like(r) for r in rows]
    nb.naut_kv4_load(*back, cache, slots)
    q = torch.randn((B, 4, 1, D), device="cuda", generator=gen).to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((B, 4, 1), device="cuda")
    ws = torch.empty(nb.decode_kv4_workspace_bytes(B, 4, Hkv, 1, S, D), dtype=torch.uint8, device="cuda")
    nb.naut_attn_decode_kv4(q, o, lse, cache, None, True, 0.125, ws)
    torch.cuda.synchronize()
    k, v = held(cache)
    for x, want in zip(back, (k, v)):
        assert np.array_equal(x.double().cpu().numpy(), want.transpose(0, 2, 1, 3).reshape(B * S, Hkv, D))
    su.check(o.double().cpu().numpy(), lse.double().cpu().numpy(), reference(q, cache, [S] * B, 0.125, True), "bf16", "bf16", S, "far rows")


@pytest.mark.parametrize("D", [64, 128])
def test_a_conversation(D):
    """Prompts attend packed and go into the cache; tokens are stored and decoded; the next turn's prompt attends to the rows
    that come back from the cache and to its own."""
    Hq, Hkv, S, dtype = 8, 2, 400, torch.bfloat16
    lens = [150, 1, 77]
    B, T, scale = len(lens), sum(lens), 1 / math.sqrt(D)
    gen = torch.Generator(device="cuda").manual_seed(12)
    rows = lambda n, H: torch.randn((n, H, D), device="cuda", generator=gen).to(dtype)
    cu = lambda x: slots_of(np.concatenate([[0], np.cumsum(x)]))
    cache = new_cache(B, Hkv, S, D)

    q, k, v = rows(T, Hq), rows(T, Hkv), rows(T, Hkv)
    o, lse = torch.empty_like(q), torch.empty((Hq, T), device="cuda")
    nb.naut_attn_fwd_packed(q, k, v, o, lse, cu(lens), cu(lens), True, scale)
    nb.naut_kv4_store(k, v, cache, slots_of(np.concatenate([b * S + np.arange(n) for b, n in enumerate(lens)])))
    kn, vn = k.double().cpu().numpy(), v.double().cpu().numpy()
    at = 0
    for b, n in enumerate(lens):
        ref = [np.stack(x, 1) for x in zip(*(su.reference(q[at : at + n, h].double().cpu().numpy(), kn[at : at + n, h // 4], vn[at : at + n, h // 4], scale, True) for h in range(Hq)))]
        su.check(o[at : at + n].double().cpu().numpy(), lse[:, at : at + n].T.double().cpu().numpy(), ref, "bf16", "bf16", n, "prompt %d" % b)
        at += n

    ws = torch.empty(nb.decode_kv4_workspace_bytes(B, Hq, Hkv, 1, S, D), dtype=torch.uint8, device="cuda")
    have = list(lens)
    for step in range(3):
        kt, vt, qt = rows(B, Hkv), rows(B, Hkv), rows(B, Hq)
        nb.naut_kv4_store(kt, vt, cache, slots_of([b * S + n for b, n in enumerate(have)]))
        have = [n + 1 for n in have]
        ot, lt = torch.empty_like(qt), torch.empty((B, Hq, 1), device="cuda")
        nb.naut_attn_decode_kv4(qt.unsqueeze(2), ot.unsqueeze(2), lt, cache, slots_of(have), True, scale, ws)
        ref = reference(qt.unsqueeze(2), cache, have, scale, True)
        su.check(ot.unsqueeze(2).double().cpu().numpy(), lt.double().cpu().numpy(), ref, "bf16", "bf16", max(have), "step %d" % step)

    more = [20, 33, 0]
    now = [n + m for n, m in zip(have, more)]
    q2, k2, v2 = rows(sum(more), Hq), rows(sum(now), Hkv), rows(sum(now), Hkv)
    slots = np.concatenate([np.concatenate([b * S + np.arange(n), np.full(m, -1)]) for b, (n, m) in enumerate(zip(have, more))])
    new = torch.tensor(slots < 0, device="cuda")
    own_k = k2[new].clone()
    nb.naut_kv4_load(k2, v2, cache, slots_of(slots))
    o2, lse2 = torch.empty_like(q2), torch.empty((Hq, sum(more)), device="cuda")
    nb.naut_attn_fwd_packed(q2, k2, v2, o2, lse2, cu(more), cu(now), True, scale)
    torch.cuda.synchronize()
    assert torch.equal(k2[new], own_k)
    held_k, held_v = held(cache)
    kn, vn, a, c = k2.double().cpu().numpy(), v2.double().cpu().numpy(), 0, 0
    for b in range(B):
        assert np.array_equal(kn[c : c + have[b]], held_k[b, :, : have[b]].transpose(1, 0, 2)) and np.array_equal(vn[c : c + have[b]], held_v[b, :, : have[b]].transpose(1, 0, 2))
        for h in range(Hq):
            ref = su.reference(q2[a : a + more[b], h].double().cpu().numpy(), kn[c : c + now[b], h // 4], vn[c : c + now[b], h // 4], scale, True)
            su.check(o2[a : a + more[b], h].double().cpu().numpy(), lse2[h, a : a + more[b]].double().cpu().numpy(), ref, "bf16", "bf16", now[b], "turn %d" % b)
        a, c = a + more[b], c + now[b]
