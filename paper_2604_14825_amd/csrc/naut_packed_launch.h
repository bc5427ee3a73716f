// naut_packed_launch.h -- the launch of a packed call: which kernel, and the grid (included by naut_packed.hip, which only
// declares the instantiations, and by naut_packed_inst.hip, which defines them).
#ifndef NAUT_PACKED_LAUNCH_H
#define NAUT_PACKED_LAUNCH_H
#include "naut_attn_kernels.h"

namespace naut_k {

// Tiles of `bm` rows: n sequences of Tq positions in all have at most this many for each K/V head, whatever their lengths.
inline long long packed_tiles(const PackedParams& p, int bm)
{
    const long long rows = (long long)p.Tq * p.g, tiles = (rows + (long long)(bm - 1) * p.n) / bm;
    return tiles < rows ? tiles : rows;
}

// What a packed launch runs, D the compiled width: kernel 2 on 4 x 32 rows (V_W4Q32, one or two key groups), on 8 x 32 (V_W8Q32;
// D <= 64: on 4 x 64), or, D > 128, kernel 1 on eight wavefronts (V_W8Q32) or four (V_W4Q32).
inline int packed_form(const PackedParams& p, int D, int causal, int* groups)
{
    int named = named_variant(groups);
    if (named == V_UNKNOWN)
        return V_UNKNOWN;
    if (named == V_W4Q32 || named == V_W8Q32)
        return named;
    *groups = 1;
    return V_W4Q32;
}

template <int D, int DT_IN, int DT_OUT>
int launch_packed(PackedParams p, int causal, hipStream_t stream)
{
    const int mean = (int)(((long long)(p.Tk > p.Tq ? p.Tk : p.Tq) + p.n - 1) / p.n);
    p.p_limit = long_loops(mean, (long long)p.n * p.Hq, D, causal) ? In<DT_IN>::P_LIMIT : 24.0f;  // as in launch(), for a sequence of mean length
    int groups;
    const int form = packed_form(p, D, causal, &groups);
    if (form == V_UNKNOWN)
        return fail(NAUT_ERR_UNSUPPORTED, "NAUT_ATTN_VARIANT names no kernel variant (w8q32, w4q64, w4q32, w4q32g2, bm128, bm128g1, bm128g2 or bm128g4)");
    const int bm = form == V_W8Q32 ? BM2 : BM;
    p.pos_per_tile = bm % p.g == 0 ? bm / p.g : 0;
    long long level = ((long long)(p.Tk > p.Tq ? p.Tk : p.Tq) * p.g / p.n + bm - 1) / bm * 8;  // eight times the mean
    for (int& end : p.class_of) {
        end = (int)(level < 1 ? 1 : level < 0x7fffffff ? level : 0x7fffffff);
        level /= 2;
    }
    const long long tiles = packed_tiles(p, bm), y = tiles < 1 << 15 ? tiles : 1 << 15;
    if ((tiles + y - 1) / y > 65535 || tiles * p.Hkv > 0x7fffffffLL)
        return fail(NAUT_ERR_UNSUPPORTED, "the heads times the query tiles exceed the grid limits");
    const dim3 grid((unsigned)p.Hkv, (unsigned)y, (unsigned)((tiles + y - 1) / y));
#define NAUT_LAUNCH(THREADS, KERNEL, ...)                                                                                    \
    do {                                                                                                                     \
        if (causal)                                                                                                          \
            hipLaunchKernelGGL((KERNEL<D, DT_IN, DT_OUT, true, __VA_ARGS__, true>), grid, dim3(THREADS), 0, stream, p);      \
        else                                                                                                                 \
            hipLaunchKernelGGL((KERNEL<D, DT_IN, DT_OUT, false, __VA_ARGS__, true>), grid, dim3(THREADS), 0, stream, p);     \
    } while (0)
    if constexpr (D > 128) {
        if (form == V_W8Q32)
            NAUT_LAUNCH(512, naut_fwd_kernel_bm128, 8, 1);
        else
            NAUT_LAUNCH(256, naut_fwd_kernel_bm128, 4, 1);
    } else if (form == V_W8Q32) {
        if constexpr (D <= 64)
            NAUT_LAUNCH(256, naut_fwd_kernel_pipe, 2, 4, 1);
        else
            NAUT_LAUNCH(512, naut_fwd_kernel_pipe, 1, 8, 1);
    } else if (groups == 2) {
        NAUT_LAUNCH(512, naut_fwd_kernel_pipe, 1, 4, 2);
    } else {
        NAUT_LAUNCH(256, naut_fwd_kernel_pipe, 1, 4, 1);
    }
#undef NAUT_LAUNCH
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return fail_launch(e);
    return NAUT_OK;
}

}  // namespace naut_k

#endif  // NAUT_PACKED_LAUNCH_H
