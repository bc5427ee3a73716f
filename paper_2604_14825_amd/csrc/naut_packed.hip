// naut_packed.hip -- naut_attn_fwd_packed: argument checks and dispatch.  The kernels are those of naut_attn_kernels.h and
// naut_attn_pipe.h in their PACKED form, instantiated in naut_packed_inst.hip.
#include "naut_packed_launch.h"

namespace naut_k {

#define NAUT_EXTERN(IN, OUT)                                                      \
    extern template int launch_packed<64, IN, OUT>(PackedParams, int, hipStream_t);   \
    extern template int launch_packed<80, IN, OUT>(PackedParams, int, hipStream_t);   \
    extern template int launch_packed<96, IN, OUT>(PackedParams, int, hipStream_t);   \
    extern template int launch_packed<128, IN, OUT>(PackedParams, int, hipStream_t);  \
    extern template int launch_packed<192, IN, OUT>(PackedParams, int, hipStream_t);  \
    extern template int launch_packed<256, IN, OUT>(PackedParams, int, hipStream_t);
NAUT_EXTERN(NAUT_BF16, NAUT_BF16)
NAUT_EXTERN(NAUT_BF16, NAUT_F32)
NAUT_EXTERN(NAUT_F16, NAUT_F16)
NAUT_EXTERN(NAUT_F16, NAUT_F32)
#undef NAUT_EXTERN

}  // namespace naut_k

extern "C" int naut_attn_fwd_packed(const void* q, const void* k, const void* v, void* o, float* lse, const int* cu_q,
                                    const int* cu_k, int n, int Tq, int Tk, int Hq, int Hkv, int D, int causal, float scale,
                                    void* stream, int in_dtype, int out_dtype, const naut_strides* st)
{
    using namespace naut;
    using namespace naut_k;
    if (n < 0 || Tq < 0 || Tk < 0 || Hq <= 0 || Hkv <= 0 || D <= 0)
        return fail(NAUT_ERR_SHAPE, "n, Tq and Tk must not be negative, Hq, Hkv and D must be positive");
    if ((Tq > 0 && (!q || !o)) || (Tk > 0 && (!k || !v)))
        return fail(NAUT_ERR_NULL, "q, k, v and o must be non-NULL device pointers");
    if (n > 0 && (!cu_q || !cu_k))
        return fail(NAUT_ERR_NULL, "cu_q and cu_k must be non-NULL device pointers");
    if (Hq % Hkv != 0)
        return fail(NAUT_ERR_SHAPE, "Hq must be a multiple of Hkv");
    if (!std::isfinite(scale))
        return fail(NAUT_ERR_SHAPE, "scale must be finite");
    if (scale < 0.f)
        return fail(NAUT_ERR_UNSUPPORTED, "negative scale is not supported");
    if (D % 8 != 0 || D > 256)
        return fail(NAUT_ERR_UNSUPPORTED, "D must be a multiple of 8, at most 256");
    if ((in_dtype != NAUT_BF16 && in_dtype != NAUT_F16) || (out_dtype != in_dtype && out_dtype != NAUT_F32))
        return fail(NAUT_ERR_UNSUPPORTED, "supported dtypes: q/k/v bf16 or f16; o of the same type or f32");
    const int g = Hq / Hkv;
    constexpr long long most = (1 << 30) - 1024;  // a position of a tile plus the keys before it fits 32 bits, those behind the last one too
    if (g > 1024 || Hkv > 65535 || (long long)Tq * g > most || (long long)Tk * g > most || n > 1 << 20)
        return fail(NAUT_ERR_UNSUPPORTED, "at most 2^20 sequences, 65535 K/V heads, Hq/Hkv 1024, Tq and Tk times Hq/Hkv 2^30 - 1024");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15u)
        return fail(NAUT_ERR_ALIGN, "q, k, v and o must be 16-byte aligned");
    if (((uintptr_t)lse | (uintptr_t)cu_q | (uintptr_t)cu_k) & 3u)
        return fail(NAUT_ERR_ALIGN, "lse, cu_q and cu_k must be 4-byte aligned");
    naut_strides cs = {};  // contiguous [T][H][D]
    cs.q_h = cs.k_h = cs.v_h = cs.o_h = D;
    cs.q_s = cs.o_s = (long long)Hq * D;
    cs.k_s = cs.v_s = (long long)Hkv * D;
    if (!st)
        st = &cs;
    const long long in_strides[6] = {st->q_h, st->q_s, st->k_h, st->k_s, st->v_h, st->v_s};
    for (long long x : in_strides)
        if (x < 0 || x % 8 != 0)
            return fail(NAUT_ERR_ALIGN, "q/k/v strides must be non-negative multiples of 8 elements (16 bytes)");
    if (st->o_h <= 0 || st->o_s <= 0 || st->o_h % 4 != 0 || st->o_s % 4 != 0)
        return fail(NAUT_ERR_ALIGN, "o strides must be positive multiples of 4 elements");
    if (st->q_s < D || st->k_s < D || st->v_s < D || st->o_s < D)
        return fail(NAUT_ERR_SHAPE, "a sequence stride is smaller than D: rows would overlap");
    const long long max_rs = 1LL << 23;  // elements: keeps 64 rows of byte offsets inside 32 bits
    if (st->q_s > max_rs || st->k_s > max_rs || st->v_s > max_rs || st->o_s > max_rs)
        return fail(NAUT_ERR_UNSUPPORTED, "sequence stride too large");
    if (n == 0 || Tq == 0)
        return NAUT_OK;  // no rows

    const int out_b = out_dtype == NAUT_F32 ? 4 : 2;
    PackedParams p = {};
    p.q = q;
    p.k = k;
    p.v = v;
    p.o = o;
    p.lse = lse;
    p.B = 1;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.cu_q = cu_q;
    p.cu_k = cu_k;
    p.n = n;
    p.Tq = Tq;
    p.Tk = Tk;
    p.g = g;
    p.g_inv = ((1u << 22) + (unsigned)g - 1) / (unsigned)g;
    const float c = scale * 1.4426950408889634f;
    p.c = c > 0.f ? c : 1e-30f;  // as in naut_attn_fwd_strided
    p.q_hs = st->q_h * 2;
    p.q_rs = (int)(st->q_s * 2);
    p.k_hs = st->k_h * 2;
    p.k_rs = (int)(st->k_s * 2);
    p.v_hs = st->v_h * 2;
    p.v_rs = (int)(st->v_s * 2);
    p.o_hs = st->o_h * out_b;
    p.o_rs = (int)(st->o_s * out_b);
    p.cpr = D / 8;
    hipStream_t hs = (hipStream_t)stream;
    const int DK = compiled_width(D);
#define NAUT_DISPATCH(IN, OUT)                                        \
    if (in_dtype == IN && out_dtype == OUT)                           \
        switch (DK) {                                                 \
        case 64: return launch_packed<64, IN, OUT>(p, causal, hs);    \
        case 80: return launch_packed<80, IN, OUT>(p, causal, hs);    \
        case 96: return launch_packed<96, IN, OUT>(p, causal, hs);    \
        case 128: return launch_packed<128, IN, OUT>(p, causal, hs);  \
        case 192: return launch_packed<192, IN, OUT>(p, causal, hs);  \
        default: return launch_packed<256, IN, OUT>(p, causal, hs);   \
        }
    NAUT_DISPATCH(NAUT_BF16, NAUT_BF16)
    NAUT_DISPATCH(NAUT_BF16, NAUT_F32)
    NAUT_DISPATCH(NAUT_F16, NAUT_F16)
    NAUT_DISPATCH(NAUT_F16, NAUT_F32)
#undef NAUT_DISPATCH
    return fail(NAUT_ERR_UNSUPPORTED, "no kernel for this (D, dtype) combination");
}
