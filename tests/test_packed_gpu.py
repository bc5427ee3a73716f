"""naut_attn_fwd_packed against plain 64-bit attention of every sequence: lengths, masks, head dimensions, strides; what lies
outside the sequences; offsets that make no sense; replays of a captured call that follow the lengths."""
import math

import numpy as np
import pytest
import torch

from paper_2604_14825_amd import binding as nb

import serving_util as su

pytestmark = pytest.mark.gpu


def offsets(lens, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32), device="cuda")


def reference(q, k, v, q_lens, k_lens, scale, causal, first=0):
    """Over the rows of the sequences alone: o [T,Hq,D], lse [Hq,T], A, G as the checks want them."""
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    Hq, g = q.shape[1], q.shape[1] // k.shape[1]
    out = [np.zeros_like(q), np.zeros(q.shape[:2]), np.zeros_like(q), np.zeros(q.shape[:2])]
    a = b = first
    for Sq, Sk in zip(q_lens, k_lens):
        for h in range(Hq):
            for x, y in zip(out, su.reference(q[a : a + Sq, h], k[b : b + Sk, h // g], v[b : b + Sk, h // g], scale, causal)):
                x[a : a + Sq, h] = y
        a, b = a + Sq, b + Sk
    return out


def run(q_lens, k_lens, Hq, Hkv, D, causal, dtype="bf16", out="bf16", pad=0, first=0, layout="dense", seed=0, magnify=1.0):
    k_lens = q_lens if k_lens is None else k_lens
    what = "packed q %s k %s Hq %d Hkv %d D %d causal %d %s->%s pad %d first %d %s" % (
        q_lens if len(q_lens) < 20 else len(q_lens), k_lens if len(k_lens) < 20 else len(k_lens), Hq, Hkv, D, causal, dtype, out, pad, first, layout)
    print(what, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    Tq, Tk = first + sum(q_lens) + pad, first + sum(k_lens) + pad

    def rows(T, H, factor=1.0, kind=dtype):
        if layout == "heads":     # head-major memory
            x = torch.empty((H, T, D), device="cuda", dtype=su.TORCH[kind]).transpose(0, 1)
        elif layout == "fused":   # rows of a wider tensor
            x = torch.empty((T, H, D + 24), device="cuda", dtype=su.TORCH[kind])[..., 8 : 8 + D]
        else:
            x = torch.empty((T, H, D), device="cuda", dtype=su.TORCH[kind])
        return x.copy_(torch.randn((T, H, D), device="cuda", generator=gen) * factor)

    q, k, v = rows(Tq, Hq, magnify), rows(Tk, Hkv), rows(Tk, Hkv)
    ref = reference(q, k, v, q_lens, k_lens, 1 / math.sqrt(D), causal, first)
    o, lse = rows(Tq, Hq, 0.0, out).fill_(7.0), torch.full((Hq, Tq), 7.0, device="cuda")
    for x in (k, v):  # what belongs to no sequence
        x[:first] = float("nan")
        x[first + sum(k_lens) :] = float("nan")
    cu_q = offsets(q_lens, first)
    nb.naut_attn_fwd_packed(q, k, v, o, lse, cu_q, cu_q if k_lens is q_lens else offsets(k_lens, first), causal, 1 / math.sqrt(D))
    torch.cuda.synchronize()
    inside = slice(first, first + sum(q_lens))
    on, ln = o.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (np.delete(on, np.r_[inside], 0) == 7.0).all() and (np.delete(ln, np.r_[inside], 1) == 7.0).all(), what + ": rows of no sequence"
    su.check(on[inside], ln.T[inside], (ref[0][inside], ref[1][inside], ref[2][inside], ref[3][inside]), dtype, out, max(list(k_lens) + [1]), what)
    return o, lse


EDGES = [1, 0, 31, 32, 33, 127, 128, 129, 2, 255, 257, 64, 0]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_at_the_edges_of_tiles(D, causal):
    run(EDGES, None, 4, 2, D, causal)


@pytest.mark.parametrize("D", [8, 40, 72, 80, 88, 96, 104, 136, 192, 200, 248])
def test_head_dimensions(D):
    run([70, 1, 161, 33], None, 2, 1, D, True, "bf16" if D % 16 else "f16", "bf16" if D % 16 else "f16", pad=3)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("D", [64, 80, 96, 128, 192, 256])
def test_types(D, dtype, out):
    run([200, 5, 77], None, 6, 2, D, True, dtype, out, seed=1)


@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (8, 1), (12, 4), (14, 2), (16, 8), (7, 7), (40, 8)])
def test_head_counts(heads):
    run([130, 31, 64, 300], None, heads[0], heads[1], 64, True, seed=2)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_more_keys_than_queries(D):
    run([1, 5, 128, 33, 200, 64], [300, 5, 129, 700, 1100, 65], 4, 1, D, True, seed=3)
    run([1, 5, 128, 33, 200, 64], [300, 9, 1, 700, 31, 0], 4, 1, D, False, seed=3)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_that_see_nothing(D):
    """Fewer keys than queries under the mask, no keys at all: o = 0, lse = -inf, beside ordinary rows and tiles."""
    run([200, 40, 300, 129, 5, 260], [60, 0, 299, 1, 5, 3], 4, 2, D, True, seed=4)
    run([40, 3, 1], [0, 0, 0], 2, 2, D, False, seed=4)
    run([40, 3, 1], [0, 0, 0], 2, 2, D, True, "f16", "f32", seed=4)


@pytest.mark.parametrize("layout", ["heads", "fused"])
@pytest.mark.parametrize("D", [64, 72, 128, 192])
def test_strides_and_offsets_that_do_not_start_at_zero(layout, D):
    run([100, 1, 190], None, 4, 2, D, True, pad=40, first=37, layout=layout, seed=5)


@pytest.mark.parametrize("n", [63, 64, 65, 255, 257, 700])
def test_many_sequences(n):
    """One sequence to a lane, four lots of 64 kept in registers, more than that."""
    rng = np.random.default_rng(n)
    run([int(x) for x in rng.integers(0, 6, n - 1)] + [140], None, 8, 4, 64, True, seed=6)
    run([int(x) for x in rng.integers(0, 200, n)] if n < 100 else [1] * (n - 2) + [300, 129], None, 2, 1, 128, True, seed=6)


@pytest.mark.parametrize("n,first", [(512, 0), (513, 11), (1031, 0), (4097, 5)])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (8, 8, 128), (5, 1, 256)])
def test_more_sequences_than_are_looked_at(n, first, Hq, Hkv, D):
    """Where a work-group searches for its sequence: runs of empty ones, one of several tiles at either end and in between."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in np.where(rng.random(n) < 0.5, 0, rng.integers(1, 5, n))]
    lens[n // 2 : n // 2 + 130] = [0] * 130
    lens[0], lens[n // 3], lens[-1] = 200, 333, 129
    k_lens = [x + int(y) if x else int(y) for x, y in zip(lens, rng.integers(0, 3, n))]
    run(lens, k_lens, Hq, Hkv, D, True, first=first, pad=9, seed=13)
    run([0] * (n - 1) + [70], None, Hq, Hkv, D, False, seed=13)


@pytest.mark.parametrize("n", [31, 32, 64, 65, 255, 256, 257])
@pytest.mark.parametrize("behind", [0, 150])
def test_orders_of_tiles(n, behind):
    """By level, one or more lots of 64 sequences in registers, and by sequence."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 90, n)]
    lens[n // 2] = 400
    run(lens, [x + int(y) for x, y in zip(lens, rng.integers(0, behind + 1, n))], 4, 2, 64, True, seed=14)


@pytest.mark.parametrize("n", [33, 64, 65, 127, 128, 129, 130])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (16, 8, 128), (5, 1, 256)])
def test_counted_sequences(n, Hq, Hkv, D):
    """Up to 128 sequences their tiles are counted, beyond that numbered: empty ones, one row each, several tiles at either end and
    where a lane's lot of 64 changes, fewer keys than queries."""
    rng = np.random.default_rng(n)
    run([1] * n, None, Hq, Hkv, D, True, seed=16)
    run([0] * (n - 1) + [140], None, Hq, Hkv, D, False, seed=16)
    lens = [int(x) for x in rng.integers(0, 6, n)]
    for i in (0, 31, 32, 62, 63, 64, n - 1):
        lens[min(i, n - 1)] = int(rng.integers(60, 290))
    run(lens, [int(x) for x in np.maximum(0, np.array(lens) + rng.integers(-2, 3, n))], Hq, Hkv, D, True, first=7, pad=5, seed=16)


@pytest.mark.parametrize("n", [2, 3, 30, 31, 64, 65, 256])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (16, 8, 128), (3, 3, 256)])
def test_orders_of_tiles_without_a_mask(n, Hq, Hkv, D):
    """By level all tiles of a sequence go together: of unlike lengths, with keys only, queries only, fewer keys than queries."""
    rng = np.random.default_rng(n)
    top = 900 if n < 10 else 300 if n < 40 else 40
    lens = [int(x) for x in rng.integers(1, top, n)]
    keys = [int(x) for x in rng.integers(0, top, n) + np.where(rng.random(n) < 0.3, 2 * top, 0)]
    lens[-1], keys[0] = 3 * top, 0
    run(lens, lens, Hq, Hkv, D, False, seed=17)
    run(lens, keys, Hq, Hkv, D, False, first=3, pad=2, seed=17)
    run([0] + lens[1:], [5] + [x + 2 * top for x in lens[1:]], Hq, Hkv, D, False, seed=17)   # the rule of more keys than queries


@pytest.mark.parametrize("D", [64, 128, 256])
def test_maxima_that_move(D):
    run([600, 129], None, 4, 4, D, True, seed=7, magnify=6.0)
    run([600, 129], None, 4, 4, D, True, "f16", "f16", seed=7, magnify=6.0)


@pytest.mark.parametrize("variant", ["w4q32", "w4q32g2", "w8q32", "bm128g4", "w4q64", "bm128"])
@pytest.mark.parametrize("D", [64, 80, 128, 192, 256])
def test_every_form(variant, D, monkeypatch):
    """Each kernel that a launch may choose, on edges of its tiles, rows that see nothing, and moving maxima."""
    monkeypatch.setenv("NAUT_ATTN_VARIANT", variant)
    run([1, 0, 63, 64, 65, 127, 129, 255, 257, 30], None, 6, 2, D, True, pad=5, seed=13)
    run([40, 200, 3, 129], [700, 513, 1, 0], 4, 4, D, False, "f16", "f16", seed=13)
    run([200, 40, 300, 129, 5, 260], [60, 0, 299, 1, 900, 3], 8, 1, D, True, seed=13, layout="heads")
    run([600, 129], None, 4, 2, D, True, seed=13, magnify=6.0)


@pytest.mark.parametrize("D,Hq,Hkv,lens", [(128, 32, 8, [1500, 40, 700]), (128, 16, 16, [4100]), (64, 8, 8, [2300, 2000, 1]), (256, 4, 1, [1800, 900]),
                                           (128, 5, 5, [2600, 2100]), (64, 33, 11, [1000, 600])])
@pytest.mark.parametrize("causal", [True, False])
def test_long_sequences(D, Hq, Hkv, lens, causal):
    run(lens, None, Hq, Hkv, D, causal, seed=8)


def test_scale_zero_is_the_mean():
    gen = torch.Generator(device="cuda").manual_seed(15)
    q, k, v = (torch.randn((90, 2, 64), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    o, lse = torch.empty((90, 2, 64), device="cuda"), torch.empty((2, 90), device="cuda")
    nb.naut_attn_fwd_packed(q, k, v, o, lse, offsets([30, 60]), offsets([30, 60]), True, np.float32(0.0))
    for first, n in ((0, 30), (30, 60)):
        want = v[first : first + n].double().cumsum(0).cpu().numpy() / np.arange(1, n + 1)[:, None, None]
        got = o[first : first + n].double().cpu().numpy()
        assert np.abs(got - want).max() <= 64 * 2.0 ** -24 * 4  # P is 1 in every place: only the sums round
        assert np.abs(lse[:, first : first + n].double().cpu().numpy() - np.log(np.arange(1, n + 1))).max() < 1e-5


def test_no_rows():
    z = torch.zeros((0, 4, 64), device="cuda", dtype=torch.bfloat16)
    x = torch.full((5, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb.naut_attn_fwd_packed(z, z, z, z, None, none, none, True, 0.1)                     # no sequence, no row
    nb.naut_attn_fwd_packed(x, x, x, o := x.clone(), None, none, none, True, 0.1)        # rows, but no sequence
    nb.naut_attn_fwd_packed(z, x, x, z, None, offsets([0, 0]), offsets([2, 3]), False, 0.1)
    nb.naut_attn_fwd_packed(x, z, z, p := x.clone(), None, offsets([5]), offsets([0]), False, 0.1)  # no keys anywhere
    torch.cuda.synchronize()
    assert (o == 7.0).all() and (p == 0.0).all()


def test_offsets_that_make_no_sense_are_empty_sequences():
    """Falling, negative, or beyond the tensors: nothing of that sequence is read or written, the others stand."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = (torch.randn((300, 2, 64), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    whole = reference(q[:100], k[:100], v[:100], [100], [100], 0.125, True)
    many = [0, 300] * 500 + [0]  # falling every other time: 500 sequences in the same place, more tiles than a launch has
    for cu_q, cu_k, left in [(many, many, 300), ([0, 100, 90], [0, 100, 200], 100), ([0, 100, 301], [0, 100, 200], 100), ([0, 100, 200], [0, 100, 1 << 30], 100),
                             ([0, 100, -5], [0, 100, 200], 100), ([0, 100, 200], [0, 100, 50], 100), ([-7, -3], [0, 10], 0),
                             ([0, 100, 0x7fffffff], [0, 100, 0x7fffffff], 100)]:
        print(cu_q[:4], cu_k[:4], flush=True)
        o, lse = torch.full_like(q, 7.0), torch.full((2, 300), 7.0, device="cuda")
        as_t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        nb.naut_attn_fwd_packed(q, k, v, o, lse, as_t(cu_q), as_t(cu_k), True, 0.125)
        torch.cuda.synchronize()
        assert (o[left:] == 7.0).all() and (lse[:, left:] == 7.0).all()
        if left == 100:
            su.check(o[:100].double().cpu().numpy(), lse[:, :100].T.double().cpu().numpy(), [whole[0], whole[1], whole[2], whole[3]], "bf16", "bf16", 100, "first sequence")


@pytest.mark.parametrize("variant", ["", "w4q32", "w8q32", "bm128g4"])
@pytest.mark.parametrize("turns,length,causal", [(1, 3000, True), (15, 400, True), (15, 400, False), (30, 130, True), (60, 300, False), (500, 300, True)])
def test_sequences_that_share_rows_are_right_or_left_out(turns, length, causal, variant, monkeypatch):
    """Offsets that rise and fall in turn give sequences in the same place, with more tiles than the grid has, whichever order
    the tiles go in: every row of them is the sequence's result or was not touched, and no other row is written."""
    monkeypatch.setenv("NAUT_ATTN_VARIANT", variant)
    print("shared rows", turns, length, causal, variant, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(18)
    guard = 37
    q, k, v = (torch.randn((length + guard, 2, 64), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    ref = reference(q[:length], k[:length], v[:length], [length], [length], 0.125, causal)
    cu = torch.tensor([0, length] * (turns + 1), dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full((2, length + guard), 7.0, device="cuda")
    nb.naut_attn_fwd_packed(q, k, v, o, lse, cu, cu, causal, 0.125)
    torch.cuda.synchronize()
    on, ln = o.double().cpu().numpy(), lse.T.double().cpu().numpy()
    assert (on[length:] == 7.0).all() and (ln[length:] == 7.0).all()
    left = (on[:length] == 7.0).all(2)
    assert ((ln[:length] == 7.0) == left).all()
    on, ln = np.where(left[..., None], ref[0], on[:length]), np.where(left, ref[1], ln[:length])
    su.check(on, ln, ref, "bf16", "bf16", length, "shared rows")
    assert not left.all()


@pytest.mark.parametrize("variant", ["w4q32", "w4q32g2", "w8q32", "bm128g4"])
@pytest.mark.parametrize("D,causal,far", [(128, True, 8200), (128, False, 4100), (80, True, 8200), (64, False, 16500)])
def test_a_sequence_is_as_exact_beside_long_ones(D, causal, far, variant, monkeypatch):
    """Keys of which a few are much larger move the reference maximum: how far it may lag is a matter of the sequence's own length,
    and so the same kernel gives the same bits whatever else is in the batch."""
    monkeypatch.setenv("NAUT_ATTN_VARIANT", variant)
    print("beside long ones", D, causal, variant, flush=True)
    lens, Hq, Hkv = [300, 1000, 77], 2 if D == 64 else 8, 2 if D == 64 else 8
    gen = torch.Generator(device="cuda").manual_seed(20)
    T, more = sum(lens), [far] * (4 if D == 64 else 3)
    q, k, v = (torch.randn((T + sum(more), H, D), device="cuda", generator=gen) for H in (Hq, Hkv, Hkv))
    k = torch.where(torch.rand((T + sum(more), Hkv, 1), device="cuda", generator=gen) < 1 / 256, 6 * k, k)
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    out = []
    for ls in (lens, lens + more):
        n = sum(ls)
        o, lse = torch.full((n, Hq, D), 7.0, device="cuda"), torch.full((Hq, n), 7.0, device="cuda")
        nb.naut_attn_fwd_packed(q[:n], k[:n], v[:n], o, lse, offsets(ls), offsets(ls), causal, D ** -0.5)
        torch.cuda.synchronize()
        out.append((o[:T], lse[:, :T]))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_as_many_sequences_as_a_call_takes():
    """2^20 of them, of one row or none (O is V and lse the score) but for one: a grid of three axes."""
    n, D = 1 << 20, 8
    rng = np.random.default_rng(21)
    lens = (rng.random(n) < 0.3).astype(np.int64)
    lens[n // 2] = 300
    gen = torch.Generator(device="cuda").manual_seed(21)
    T = int(lens.sum())
    print("sequences", n, "rows", T, flush=True)
    q, k, v = (torch.randn((T + 5, 2, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    o, lse = torch.full((T + 5, 2, D), 7.0, device="cuda"), torch.full((2, T + 5), 7.0, device="cuda")
    cu = offsets(lens)
    nb.naut_attn_fwd_packed(q, k, v, o, lse, cu, cu, True, 0.25)
    torch.cuda.synchronize()
    assert (o[T:] == 7.0).all() and (lse[:, T:] == 7.0).all()
    a = int(lens[: n // 2].sum())
    one = torch.ones(T, dtype=torch.bool, device="cuda")
    one[a : a + 300] = False
    assert torch.equal(o[:T][one], v[:T][one].float())
    score = (q.double() * k.double()).sum(-1)[:T][one] * 0.25
    assert float((lse.T[:T][one].double() - score).abs().max()) <= 8 * 2.0 ** -24 * 40 * 0.25 + 4 * 2.0 ** -23 * 12  # su.check's, |q.k| <= 40
    ref = reference(q[a : a + 300], k[a : a + 300], v[a : a + 300], [300], [300], 0.25, True)
    su.check(o[a : a + 300].double().cpu().numpy(), lse[:, a : a + 300].T.double().cpu().numpy(), ref, "bf16", "f32", 300, "the long one")


@pytest.mark.parametrize("D", [64, 128, 256])
def test_without_lse(D):
    gen = torch.Generator(device="cuda").manual_seed(22)
    q, k, v = (torch.randn((300, 4, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3))
    cu_q, cu_k = offsets([100, 40, 160]), offsets([100, 3, 197])   # the second with rows that see nothing
    out = []
    for lse in (torch.empty((4, 300), device="cuda"), None):
        o = torch.empty_like(q)
        nb.naut_attn_fwd_packed(q, k, v, o, lse, cu_q, cu_k, True, 0.1)
        out.append(o)
    torch.cuda.synchronize()
    assert torch.equal(*out)


def test_calls_repeat_bit_for_bit_and_on_another_stream():
    a, la = run([333, 1, 90], None, 8, 2, 128, True, seed=10)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b, lb = run([333, 1, 90], None, 8, 2, 128, True, seed=10)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("variant,D,stride", [("", 64, 1 << 22), ("", 64, 1 << 23), ("w4q32", 128, 1 << 23), ("w4q32g2", 128, 1 << 22), ("w4q32g2", 128, 1 << 23),
                                              ("w8q32", 128, 1 << 23), ("w8q32", 64, 1 << 23), ("bm128g4", 128, 1 << 23), ("w4q32", 256, 1 << 23), ("w8q32", 256, 1 << 23)])
def test_rows_beyond_2_31_bytes(variant, D, stride, monkeypatch):
    """Offsets that pass 32 bits: rows 8 and 16 MiB apart, the most that a call takes, so that the last sequence lies past 4 GiB."""
    monkeypatch.setenv("NAUT_ATTN_VARIANT", variant)
    T, H = 700, 2
    gen = torch.Generator(device="cuda").manual_seed(11)
    base = torch.empty(T * stride, device="cuda", dtype=torch.bfloat16)
    wide = lambda at: torch.as_strided(base, (T, H, D), (stride, D, 1), at)
    q, k, v, o = (wide(at) for at in (0, 1024, 2048, 4096))
    for x in (q, k, v):
        x.copy_(torch.randn((T, H, D), device="cuda", generator=gen))
    o.fill_(7.0)
    lse = torch.empty((H, T), device="cuda")
    lens = [90, 610]
    print("far rows", variant, D, stride, flush=True)
    nb.naut_attn_fwd_packed(q, k, v, o, lse, offsets(lens), offsets(lens), True, 0.125)
    torch.cuda.synchronize()
    ref = reference(q.contiguous(), k.contiguous(), v.contiguous(), lens, lens, 0.125, True)
    su.check(o.double().cpu().numpy(), lse.T.double().cpu().numpy(), ref, "bf16", "bf16", 610, "far rows")


def test_a_captured_call_follows_the_lengths():
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, v = (torch.randn((500, H, 128), device="cuda", generator=gen).to(torch.bfloat16) for H in (8, 2, 2))
    o, lse = torch.empty_like(q), torch.empty((8, 500), device="cuda")
    call = lambda: nb.naut_attn_fwd_packed(q, k, v, o, lse, cu4, cu4, True, 0.09)
    cu4 = offsets([100, 100, 100, 200])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([100, 100, 100, 200], [1, 498, 0, 1], [0, 0, 0, 500], [130, 7, 260, 3], [100, 100, 100, 200]):
        cu4.copy_(offsets(lens))
        q.copy_(torch.randn(q.shape, device="cuda", generator=gen))
        o.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = o.clone(), lse.clone()
        o.fill_(7.0)
        lse.fill_(7.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, o) and torch.equal(got_lse, lse), lens
        n = sum(lens)
        ref = reference(q[:n], k[:n], v[:n], lens, lens, 0.09, True)
        su.check(o[:n].double().cpu().numpy(), lse[:, :n].T.double().cpu().numpy(), ref, "bf16", "bf16", 500, str(lens))
