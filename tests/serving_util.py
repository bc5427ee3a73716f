"""Shared by the tests of packed prompts and of the 4-bit cache: plain 64-bit references, and the error that a correct kernel can have.

With u half a step of the 16-bit type relative to the value (2^-8 bf16, 2^-11 f16), w the weights and A = sum_j w_j |v_j|:
every P is rounded to 16 bits (<= u A in the numerator), the divisor may be the sum of the rounded or of the unrounded P
(<= u |o|), and a 16-bit O is rounded once (<= u |o|).  In fp32 a score of D products is off by at most D 2^-24 G, G = scale *
sum_d |q_d k_d|, which moves every weight by that much relative (twice: numerator and divisor), an exponential or a repair
factor by a few 2^-23, and a sum of n terms by n 2^-24; lse sees the same without the 16-bit roundings."""
import numpy as np
import torch

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def reference(q, k, v, scale, causal):
    """One head: q [Sq,D], k and v [Sk,D] in float64 -> o, lse, A, G (largest of the row)."""
    Sq, Sk = q.shape[0], k.shape[0]
    if Sk == 0:
        z = np.zeros_like(q)
        return z, np.full(Sq, -np.inf), z, np.zeros(Sq)
    s = q @ k.T * scale
    seen = np.ones((Sq, Sk), bool)
    if causal:
        seen = np.arange(Sk)[None] <= np.arange(Sq)[:, None] + Sk - Sq
    s = np.where(seen, s, -np.inf)
    top = np.maximum(s.max(1, keepdims=True), -1e300)
    p = np.exp(s - top)
    l = p.sum(1, keepdims=True)
    w = p / np.where(l > 0, l, 1.0)
    with np.errstate(divide="ignore"):
        lse = np.where(l[:, 0] > 0, np.log(l[:, 0]) + top[:, 0], -np.inf)
    return w @ v, lse, w @ np.abs(v), (np.abs(q) @ np.abs(k).T * scale).max(1)


def check(o, lse, ref, dtype, out, n, what):
    """o [..,D], lse [..] against reference()'s four arrays of the same leading shape; n: terms of the longest sum."""
    ro, rl, A, G = ref
    D = o.shape[-1]
    u = HALF_STEP[dtype]
    f32 = D * 2.0 ** -24 * G + n * 2.0 ** -24 + 8 * 2.0 ** -23
    tol = u * A + u * np.abs(ro) * (1 if out == "f32" else 2) + 2 * f32[..., None] * A
    if out == "f16":
        tol = tol + 2.0 ** -25  # half a step of the subnormals
    assert np.isfinite(o).all(), what + ": O not finite"
    bad = np.abs(o - ro) > tol * (1 + 2.0 ** -6) + 1e-30  # second-order terms
    assert not bad.any(), "%s: O off by %.3e, allowed %.3e, at %s (%d places)" % (
        what, np.abs(o - ro)[bad].max(), tol[bad].max(), np.argwhere(bad)[0], bad.sum())
    if lse is not None:
        none = np.isneginf(rl)
        assert (np.isneginf(lse) == none).all(), what + ": lse of rows that see nothing"
        d = np.abs(np.where(none, 0, lse) - np.where(none, 0, rl))[~none]
        limit = (f32 + 4 * 2.0 ** -23 * (1 + np.abs(np.where(none, 0, rl))))[~none]
        assert (d <= limit).all(), "%s: lse off by %.3e" % (what, d.max())
    return float(np.abs(o - ro).max()) if o.size else 0.0


# ---- the 4-bit format ----
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALVES = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])  # between neighbours; the even code takes a tie


def encode(x, dtype):
    """Rows [..,D] in float64 -> code bytes [..,D/2], scale bytes [..,D/32]."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    a = np.abs(b)
    e = np.frexp(a.max(-1, keepdims=True) / 7.0)[1]           # the least with max / 2^e < 7
    e = np.where(a.max(-1, keepdims=True) == 0, -126, e)
    byte = np.clip(e + 127, 1, 140 if dtype == "f16" else 252)
    y = a / 2.0 ** (byte - 127.0)
    code = np.zeros(b.shape, np.int64)
    for i, t in enumerate(HALVES):
        code += (y >= t) if i % 2 else (y > t)
    code = (code + 8 * np.signbit(b)).reshape(x.shape)
    return (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8), byte[..., 0].astype(np.uint8)


def decode(codes, scales, D):
    """The values that code bytes [..,D/2] and scale bytes [..,>=D/32] stand for."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D)
    return np.where(c < 8, 1.0, -1.0) * MAGNITUDES[c & 7] * np.repeat(2.0 ** (scales[..., : D // 32].astype(np.float64) - 127), 32, -1)
