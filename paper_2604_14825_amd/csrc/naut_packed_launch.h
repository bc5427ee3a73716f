// naut_packed_launch.h -- the launch of a packed call: which kernel, and the grid (included by naut_packed.hip, which only
// declares the instantiations, and by naut_packed_inst.hip, which defines them).
#ifndef NAUT_PACKED_LAUNCH_H
#define NAUT_PACKED_LAUNCH_H
#include "naut_attn_kernels.h"

namespace naut_k {

// Work-groups of tiles of `bm` queries: n sequences of Tq rows in all have at most this many tiles, whatever their lengths.
inline long long packed_grid(const PackedParams& p, int bm)
{
    const long long tiles = ((long long)p.Tq + (long long)(bm - 1) * p.n) / bm;
    return (tiles < p.Tq ? tiles : p.Tq) * p.Hq;
}

template <int D, int DT_IN, int DT_OUT>
int launch_packed(PackedParams p, int causal, hipStream_t stream)
{
    const int mean = (int)(((long long)(p.Tk > p.Tq ? p.Tk : p.Tq) + p.n - 1) / p.n);
    p.p_limit = long_loops(mean, (long long)p.n * p.Hq, D, causal) ? In<DT_IN>::P_LIMIT : 24.0f;  // as in launch(), for a sequence of mean length
    const long long nblocks = packed_grid(p, BM);
    if (nblocks > 0x7fffffffLL)
        return fail(NAUT_ERR_UNSUPPORTED, "Hq times the query tiles exceeds the 1-D grid limit");
    const dim3 grid((unsigned)nblocks);
    if constexpr (D > 128) {
        if (causal)
            hipLaunchKernelGGL((naut_fwd_kernel_bm128<D, DT_IN, DT_OUT, true, 4, 1, true>), grid, dim3(256), 0, stream, p);
        else
            hipLaunchKernelGGL((naut_fwd_kernel_bm128<D, DT_IN, DT_OUT, false, 4, 1, true>), grid, dim3(256), 0, stream, p);
    } else {
        if (causal)
            hipLaunchKernelGGL((naut_fwd_kernel_pipe<D, DT_IN, DT_OUT, true, 1, 4, 1, true>), grid, dim3(256), 0, stream, p);
        else
            hipLaunchKernelGGL((naut_fwd_kernel_pipe<D, DT_IN, DT_OUT, false, 1, 4, 1, true>), grid, dim3(256), 0, stream, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return fail_launch(e);
    return NAUT_OK;
}

}  // namespace naut_k

#endif  // NAUT_PACKED_LAUNCH_H
