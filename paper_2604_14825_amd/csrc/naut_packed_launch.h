// naut_packed_launch.h -- the launch of a packed call: which kernel, and the grid (included by naut_packed.hip, which only
// declares the instantiations, and by naut_packed_inst.hip, which defines them).
#ifndef NAUT_PACKED_LAUNCH_H
#define NAUT_PACKED_LAUNCH_H
#include "naut_attn_kernels.h"

namespace naut_k {

// Three keys for two queries or more: new turns of conversations that are cached.
inline bool packed_more_keys(const PackedParams& p) { return 2LL * p.Tk >= 3LL * p.Tq; }

// Tiles of `bm` rows: n sequences of Tq positions in all have at most this many for each K/V head, whatever their lengths.
inline long long packed_tiles(const PackedParams& p, int bm)
{
    const long long rows = (long long)p.Tq * p.g, tiles = (rows + (long long)(bm - 1) * p.n) / bm;
    if (!p.by_level)
        return rows / bm + p.n;  // the numbers of packed_tile_by_sequence, enough for those of packed_tile_by_count
    return tiles < rows ? tiles : rows;
}

// What a packed launch runs, D the compiled width: kernel 2 on 4 x 32 rows (V_W4Q32) with one or two key groups, on 8 x 32
// (V_W8Q32; D <= 64: on 4 x 64), kernel 1 on 2 x 32 with four key groups (V_BM128), or, D > 128, kernel 1 on eight wavefronts
// (V_W8Q32) or four (V_W4Q32).  NAUT_ATTN_VARIANT names one as in the rectangular launch (w4q32, w4q32g2, w8q32 or w4q64,
// bm128g4); a name without a packed form chooses nothing.
//   The host knows the totals and the number of sequences, not the lengths, so the rule goes by means: tiles of 128 rows (at
// most), keys per sequence, keys per query.  Fitted to timings of every form in turn over 2914 batches, with the tiles in an earlier
// order.  On the present kernels, 2725 batches (1 to 256 sequences, eight pairs of head counts, D = 64, 96 and 128, equal, even and
// log-even lengths, as many keys as queries or up to 8000 more; time over that of the best form): the rule 1.013 on average, 1.19 at the
// 99th percentile, 1.55 at most; 4 x 32 alone 1.074, 1.55 and 1.66.  It goes by time alone: the key groups that the rectangular rule keeps because
// they make O more exact (see key_groups) are not kept (error of O up to 1.17 times the rectangular call's, with outlier keys 1.57).
//   With few tiles the longest loop is what a launch takes, and key groups cut it: up to one tile on every second CU four
// (1 to 8 heads' prompts of 1000 keys, D = 64 1.2, D = 128 1.1), then two.  Where there are several times as many keys as
// queries (new turns of long conversations) loops are longer and more unlike, and groups pay up to five rounds of tiles (500 to 900
// tiles, 6 to 15 keys a query 1.08 to 1.27; as many keys as queries 0.8); eight prompts of 1 to 700 behind 333 to 8100
// keys, 64/8 heads 149 -> 136 us.
//   256-row tiles read K and V half as often: long loops on full chips (64/8 heads, two of 8192, D = 128 1856 -> 1827 us, eight of 8192, 32/8
// heads, D = 64 2164 -> 2043); D > 128 wherever they fill the chip (16/4 heads, D = 256, 6 of 100 to 4096 466 -> 374).
inline int packed_form(const PackedParams& p, int D, int causal, int* groups)
{
    const int named = named_variant(groups);
    const bool has4 = named == V_BM128 && *groups == 4 && D <= 128;
    if (named == V_UNKNOWN || named == V_W8Q32 || named == V_W4Q32 || has4)
        return named;
    *groups = 1;
    if (named == V_W4Q64 && D <= 64)
        return V_W8Q32;
    const long long w = packed_tiles(p, BM) * p.Hkv, w2 = packed_tiles(p, BM2) * p.Hkv;
    if (D > 128)
        return w <= 512 ? V_W4Q32 : V_W8Q32;
    const int keys = p.Tk / p.n;
    const bool more_keys = packed_more_keys(p);
    if (more_keys ? w <= (D <= 64 ? 256 : 160) && keys >= 200 : w <= 128 && keys >= 400) {
        *groups = 4;
        return V_BM128;
    }
    // keys per query, in quarters, from a half to one and a half of 850 tiles
    const long long ratio = p.Tk / p.Tq, most = 850 * (ratio < 2 ? 2 : ratio < 6 ? ratio : 6) / 4;
    if (more_keys ? w <= most && keys >= 200 : D <= 64 ? w <= 400 && keys >= 600 : w <= 256 && keys >= 500) {
        *groups = 2;
        return V_W4Q32;
    }
    const int loop = causal ? keys / 2 : keys;
    if (D <= 64 ? w2 >= 512 && loop >= (causal ? 3000 : 1000) : w2 >= 480 && loop >= (causal ? 2500 : 2000))
        return V_W8Q32;
    return V_W4Q32;
}

template <int D, int DT_IN, int DT_OUT>
int launch_packed(PackedParams p, int causal, hipStream_t stream)
{
    const int mean = (int)(((long long)(p.Tk > p.Tq ? p.Tk : p.Tq) + p.n - 1) / p.n);
    // As in launch(), for a sequence of mean length; shorter ones beside long ones keep the limit of short loops, as their O would be
    // less exact for the company (error of O against 64 bits beside six sequences of 16384, D = 128, over that without them: 1000
    // keys, some of them outliers 1.42, 300 and 1000 keys at three times the usual scale 1.15 and 1.19).
    p.p_limit = long_loops(mean, (long long)p.n * p.Hq, D, causal) ? In<DT_IN>::P_LIMIT : P_LIMIT_SHORT;
    p.long_from = long_length(D, causal);
    p.by_level = p.n > 1 && p.n < (packed_more_keys(p) ? PACKED_BY_LEVEL + 1 : 32);  // both sides' times are at packed_tile
    int groups;
    const int form = packed_form(p, D, causal, &groups);
    if (form == V_W4Q32 && groups == 2 && D <= 128 && (p.k_rs > p.v_rs ? p.k_rs : p.v_rs) > 8 << 20)
        groups = 1;  // two key groups step over twice the rows at a time: farther apart, they pass the 32 bits of an offset
    if (form == V_UNKNOWN)
        return fail(NAUT_ERR_UNSUPPORTED, "NAUT_ATTN_VARIANT names no kernel variant (w8q32, w4q64, w4q32, w4q32g2, bm128, bm128g1, bm128g2 or bm128g4)");
    const int bm = form == V_W8Q32 ? BM2 : form == V_BM128 ? BM / 2 : BM;
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
    // One kernel for both masks: no mask is one that leaves every key.  (Its own instantiation takes as long again to compile, a quarter of
    // the library, and is faster by 0.3 us a round of work-groups: 32/8 heads, D = 128, 64 of 1 to 4 7.2 us for 7.6, 200 of 1 to 64 39.4
    // for 40.8, 128 of 1 to 200 72.4 for 74.6, 200 of 1 to 1000 1248 for 1245, 6 of 500 to 4096 827 for 829.)
    p.all_keys = !causal;
#define NAUT_LAUNCH(THREADS, KERNEL, ...) \
    hipLaunchKernelGGL((KERNEL<D, DT_IN, DT_OUT, true, __VA_ARGS__, true>), grid, dim3(THREADS), 0, stream, p)
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
    } else if (form == V_BM128) {
        NAUT_LAUNCH(512, naut_fwd_kernel_bm128, 2, 4);
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
