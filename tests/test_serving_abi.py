"""Refusals of the packed and 4-bit cache entry points: all of them on the host, before any HIP call (no GPU here), and the
reference encoder that the GPU tests go by."""
import ctypes

import numpy as np
import pytest

from paper_2604_14825_amd import binding as nb

import serving_util as su

A = 0x10000  # a fake, 16-byte aligned, never dereferenced device address
BF, F16, F32 = nb.NAUT_BF16, nb.NAUT_F16, nb.NAUT_F32


def packed(q=A, k=A, v=A, o=A, lse=A, cu_q=A, cu_k=A, n=2, Tq=100, Tk=100, Hq=4, Hkv=2, D=64, scale=0.1, types=(BF, BF), st=None):
    s = nb.NautStrides(*st) if st else None
    return nb.lib().naut_attn_fwd_packed(q, k, v, o, lse, cu_q, cu_k, n, Tq, Tk, Hq, Hkv, D, 1, scale, None, *types, ctypes.byref(s) if s else None)


GOOD = (0, 64, 256, 0, 64, 128, 0, 64, 128, 0, 64, 256)


def but(i, x):
    return GOOD[:i] + (x,) + GOOD[i + 1 :]


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), nb.NAUT_ERR_NULL), (dict(k=None), nb.NAUT_ERR_NULL), (dict(v=None), nb.NAUT_ERR_NULL), (dict(o=None), nb.NAUT_ERR_NULL),
    (dict(cu_q=None), nb.NAUT_ERR_NULL), (dict(cu_k=None), nb.NAUT_ERR_NULL),
    (dict(n=-1), nb.NAUT_ERR_SHAPE), (dict(Tq=-1), nb.NAUT_ERR_SHAPE), (dict(Tk=-1), nb.NAUT_ERR_SHAPE), (dict(Hq=0), nb.NAUT_ERR_SHAPE),
    (dict(Hq=5), nb.NAUT_ERR_SHAPE), (dict(D=0), nb.NAUT_ERR_SHAPE), (dict(scale=float("nan")), nb.NAUT_ERR_SHAPE),
    (dict(scale=float("inf")), nb.NAUT_ERR_SHAPE), (dict(scale=-0.5), nb.NAUT_ERR_UNSUPPORTED), (dict(D=100), nb.NAUT_ERR_UNSUPPORTED),
    (dict(D=264), nb.NAUT_ERR_UNSUPPORTED), (dict(types=(F32, F32)), nb.NAUT_ERR_UNSUPPORTED), (dict(types=(BF, F16)), nb.NAUT_ERR_UNSUPPORTED),
    (dict(Tq=(1 << 30) + 1), nb.NAUT_ERR_UNSUPPORTED), (dict(n=(1 << 20) + 1), nb.NAUT_ERR_UNSUPPORTED),
    (dict(Tk=(1 << 30) - 1023, Hq=1, Hkv=1), nb.NAUT_ERR_UNSUPPORTED), (dict(Tq=(1 << 29) - 511), nb.NAUT_ERR_UNSUPPORTED),
    (dict(Tq=1 << 30, Hq=512, Hkv=512), nb.NAUT_ERR_UNSUPPORTED), (dict(Hq=2048, Hkv=1), nb.NAUT_ERR_UNSUPPORTED), (dict(Hq=1 << 16, Hkv=1 << 16), nb.NAUT_ERR_UNSUPPORTED),
    (dict(Tk=1 << 29, Hq=8, Hkv=2), nb.NAUT_ERR_UNSUPPORTED),
    (dict(q=A + 8), nb.NAUT_ERR_ALIGN), (dict(v=A + 2), nb.NAUT_ERR_ALIGN), (dict(o=A + 4), nb.NAUT_ERR_ALIGN), (dict(lse=A + 2), nb.NAUT_ERR_ALIGN),
    (dict(cu_q=A + 2), nb.NAUT_ERR_ALIGN), (dict(cu_k=A + 1), nb.NAUT_ERR_ALIGN),
    (dict(st=but(2, 260)), nb.NAUT_ERR_ALIGN), (dict(st=but(5, -128)), nb.NAUT_ERR_ALIGN), (dict(st=but(7, 4)), nb.NAUT_ERR_ALIGN),
    (dict(st=but(10, 0)), nb.NAUT_ERR_ALIGN), (dict(st=but(11, 258)), nb.NAUT_ERR_ALIGN), (dict(st=but(5, 56)), nb.NAUT_ERR_SHAPE),
    (dict(st=but(11, 60)), nb.NAUT_ERR_SHAPE), (dict(st=but(8, 1 << 24)), nb.NAUT_ERR_UNSUPPORTED),
])
def test_packed_refusals(kw, code):
    assert packed(**kw) == code
    assert nb.last_error_string()


def test_packed_without_rows_is_done_at_once():
    assert packed(n=0, cu_q=None, cu_k=None) == nb.NAUT_OK
    assert packed(Tq=0, q=None, o=None) == nb.NAUT_OK
    assert packed(Tq=0, Tk=0, q=None, k=None, v=None, o=None) == nb.NAUT_OK


def cache(B=2, Hkv=2, S=100, D=64, codes=A, scales=A, v_codes=A, v_scales=A, c=None, s=None):
    half, row = D // 2, max(2, nb.kv4_scale_bytes(D))
    c = c or (Hkv * S * half, S * half, half)
    s = s or (Hkv * S * row, S * row, row)
    return nb.NautKv4Cache(codes, scales, v_codes, v_scales, *c, *s, B, Hkv, S, D)


BAD_CACHES = [
    (dict(codes=None), nb.NAUT_ERR_NULL), (dict(scales=None), nb.NAUT_ERR_NULL), (dict(v_codes=None), nb.NAUT_ERR_NULL), (dict(v_scales=None), nb.NAUT_ERR_NULL),
    (dict(B=0), nb.NAUT_ERR_SHAPE), (dict(S=-1), nb.NAUT_ERR_SHAPE), (dict(Hkv=0), nb.NAUT_ERR_SHAPE), (dict(D=0), nb.NAUT_ERR_SHAPE),
    (dict(D=48), nb.NAUT_ERR_UNSUPPORTED), (dict(D=288), nb.NAUT_ERR_UNSUPPORTED), (dict(B=1 << 16, S=1 << 16), nb.NAUT_ERR_UNSUPPORTED),
    (dict(codes=A + 8), nb.NAUT_ERR_ALIGN), (dict(v_codes=A + 4), nb.NAUT_ERR_ALIGN), (dict(c=(6400, 3200, 40)), nb.NAUT_ERR_ALIGN),
    (dict(c=(6400, -3200, 32)), nb.NAUT_ERR_ALIGN), (dict(scales=A + 1), nb.NAUT_ERR_ALIGN), (dict(D=128, scales=A + 2), nb.NAUT_ERR_ALIGN),
    (dict(s=(400, 200, 3)), nb.NAUT_ERR_ALIGN), (dict(D=128, s=(800, 400, 6)), nb.NAUT_ERR_ALIGN), (dict(c=(6400, 3200, 16)), nb.NAUT_ERR_SHAPE),
    (dict(s=(400, 200, 0)), nb.NAUT_ERR_SHAPE), (dict(c=(6400, 3200, 1 << 24)), nb.NAUT_ERR_UNSUPPORTED), (dict(s=(400, 200, 1 << 24)), nb.NAUT_ERR_UNSUPPORTED),
]


def store(c, k=A, v=A, slots=A, T=10, dtype=BF, st=None, f="naut_kv4_store"):
    s = nb.NautStrides(*st) if st else None
    return getattr(nb.lib(), f)(k, v, ctypes.byref(c) if c else None, slots, T, dtype, ctypes.byref(s) if s else None, None)


def decode(c, q=A, o=A, lse=A, lens=A, Hq=4, Sq=1, scale=0.1, ws=A, room=1 << 30, types=(BF, BF), st=None):
    s = nb.NautStrides(*st) if st else None
    return nb.lib().naut_attn_decode_kv4(q, o, lse, ctypes.byref(c) if c else None, lens, Hq, Sq, 1, scale, ws, room, None, *types, ctypes.byref(s) if s else None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches_are_refused_everywhere(kw, code):
    c = cache(**kw)
    assert store(c) == code and nb.last_error_string()
    assert store(c, f="naut_kv4_load") == code
    assert decode(c) == code


def test_row_refusals():
    for f in ("naut_kv4_store", "naut_kv4_load"):
        c = cache()
        call = lambda **kw: store(c, f=f, **kw)
        assert store(None, f=f) == nb.NAUT_ERR_NULL
        assert call(k=None) == call(v=None) == call(slots=None) == nb.NAUT_ERR_NULL
        assert call(T=-1) == nb.NAUT_ERR_SHAPE
        assert call(T=0, k=None, v=None, slots=None) == nb.NAUT_OK
        assert call(dtype=F32) == nb.NAUT_ERR_UNSUPPORTED
        assert call(k=A + 8) == call(slots=A + 2) == nb.NAUT_ERR_ALIGN
        row = lambda k_h, k_s, v_h, v_s: (0, 0, 0, 0, k_h, k_s, 0, v_h, v_s, 0, 0, 0)
        assert call(st=row(64, 132, 64, 128)) == call(st=row(64, 128, -64, 128)) == nb.NAUT_ERR_ALIGN
        assert call(T=(1 << 30) + 1) == nb.NAUT_ERR_UNSUPPORTED
        assert store(cache(Hkv=1 << 12), f=f, T=1 << 30) == nb.NAUT_ERR_UNSUPPORTED              # more work-groups than a grid has
    assert store(cache(), f="naut_kv4_load", st=row(0, 128, 64, 128)) == nb.NAUT_ERR_ALIGN     # rows written to the same place
    assert store(cache(), f="naut_kv4_load", st=row(64, 56, 64, 128)) == nb.NAUT_ERR_SHAPE
    for c in (cache(c=(6400, 0, 32)), cache(c=(0, 3200, 32)), cache(s=(400, 0, 2)), cache(s=(0, 200, 2))):
        assert store(c) == nb.NAUT_ERR_SHAPE                                                    # heads that share their bytes
    assert store(cache(B=1, Hkv=1, c=(0, 0, 32), s=(0, 0, 2)), T=0) == nb.NAUT_OK


def test_decode_refusals():
    c = cache(B=2, Hkv=2, S=5000, D=128)
    need = nb.decode_kv4_workspace_bytes(2, 4, 2, 1, 5000, 128)
    assert need > 0 and need % 16 == 0
    assert decode(None) == nb.NAUT_ERR_NULL
    for kw in (dict(q=None), dict(o=None), dict(ws=None)):
        assert decode(c, **kw) == nb.NAUT_ERR_NULL, kw
    for kw in (dict(Hq=0), dict(Hq=3), dict(Sq=0), dict(scale=float("inf")), dict(room=need - 1)):
        assert decode(c, **kw) == nb.NAUT_ERR_SHAPE, kw
    for kw in (dict(scale=-1.0), dict(types=(F32, F32)), dict(types=(F16, BF)), dict(Sq=1 << 30), dict(Hq=1 << 27)):
        assert decode(c, **kw) == nb.NAUT_ERR_UNSUPPORTED, kw
    for kw in (dict(q=A + 8), dict(o=A + 8), dict(ws=A + 8), dict(lse=A + 2), dict(lens=A + 2)):
        assert decode(c, **kw) == nb.NAUT_ERR_ALIGN, kw
    good = (512, 128, 128, 0, 0, 0, 0, 0, 0, 512, 128, 128)
    at = lambda i, x: good[:i] + (x,) + good[i + 1 :]
    assert decode(c, st=at(2, 132)) == decode(c, st=at(1, -8)) == decode(c, st=at(9, 0)) == decode(c, st=at(11, 130)) == nb.NAUT_ERR_ALIGN
    assert decode(c, st=at(2, 120)) == decode(c, st=at(11, 124)) == nb.NAUT_ERR_SHAPE
    assert decode(c, st=at(2, 1 << 24)) == nb.NAUT_ERR_UNSUPPORTED


def test_sizes():
    assert [nb.kv4_scale_bytes(D) for D in (0, 16, 32, 64, 96, 128, 160, 256, 288)] == [0, 0, 2, 2, 4, 4, 8, 8, 0]
    w = nb.decode_kv4_workspace_bytes
    assert w(1, 8, 3, 1, 100, 128) == w(1, 8, 2, 1, 100, 100) == w(0, 8, 2, 1, 100, 128) == w(1, 8, 2, 1, 1 << 31 - 1, 128) * 0 == 0
    assert w(1, 8, 2, 1, 100, 128) > 0 and w(1, 32, 8, 1, 1 << 20, 128) < 64 << 20   # the partials do not grow with the cache


def test_workspace_where_the_positions_pass_32_bits():
    w = nb.decode_kv4_workspace_bytes
    assert w(1, 8, 2, 1, (1 << 31) - 1, 128) > 0 and w(2, 8, 2, 1, 1 << 30, 128) == 0 and w(65023, 8, 2, 1, 33025, 128) > 0
    assert w(65023, 8, 2, 1, 33027, 128) == 0    # 2^31 + 30973 positions
    assert w(65024, 8, 2, 1, 64, 128) == 0       # more sequences than a grid has with the parts of the split ones


def test_the_partials_do_not_grow_with_the_sequences():
    """Sequences of one part have no partial result; what is left is the plan, a few words each."""
    w = nb.decode_kv4_workspace_bytes
    for Hq, Hkv, Sq, S, D in ((32, 8, 1, 2304, 128), (8, 1, 1, 2304, 64), (64, 8, 4, 4096, 256), (3, 3, 1, 5000, 96)):
        assert w(8192, Hq, Hkv, Sq, S, D) - w(1024, Hq, Hkv, Sq, S, D) <= 64 * (8192 - 1024)
        assert w(60000, Hq, Hkv, Sq, S, D) - w(1024, Hq, Hkv, Sq, S, D) <= 64 * (60000 - 1024)


def test_reference_encoder():
    """By hand: ties to the even code, saturation at the type's end, the power that keeps the largest from rounding past 6."""
    x = np.zeros((1, 32))
    x[0, :8] = [6.0, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, -5.0]
    codes, scales = su.encode(x, "bf16")
    assert scales[0, 0] == 127
    assert list(codes[0, :4]) == [7 + 16 * 0, 2 + 16 * 10, 4 + 16 * 4, 6 + 16 * 14]
    assert np.array_equal(su.decode(codes, scales, 32)[0, :8], [6, 0, 1, -1, 2, 2, 4, -4])
    for top, byte, value in ((6.99, 127, 6), (7.0, 128, 8), (4.0, 127, 4), (3.49, 126, 3), (3.5, 127, 4)):
        x[0] = 0
        x[0, 5] = top
        codes, scales = su.encode(x, "bf16")
        assert scales[0, 0] == byte and su.decode(codes, scales, 32)[0, 5] == value, top
    x[0, 5] = 65504.0
    codes, scales = su.encode(x, "f16")
    assert scales[0, 0] == 140 and su.decode(codes, scales, 32)[0, 5] == 49152.0
    x[0, 5] = 0
    assert su.encode(x, "bf16")[1][0, 0] == 1
