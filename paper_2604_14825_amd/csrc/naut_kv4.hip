// naut_kv4.hip -- a key/value cache in 4 bits for gfx950 (MI355X): rows into it, rows out of it, decode-time attention over it.
//
// The format is OCP MXFP4: blocks of 32 values, E2M1 codes under one power of two.  gfx950 converts between such codes and
// 16-bit values with the block's power in one instruction per pair, and a code times its power is exact in bf16, so the
// attention runs on the cache's values as they are, on the 16-bit matrix instructions.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "naut_attn.h"
#include "naut_common.h"

namespace {

using namespace naut;

constexpr int MX = 32;  // values per block

// The value of a scale byte as the conversions take it (its exponent field).
__device__ __forceinline__ float mx_scale(int byte) { return __builtin_bit_cast(float, byte << 23); }

// Pairs of values: code byte I of `word` times `scale`, and back.
template <int DT>
struct Mx;
template <>
struct Mx<NAUT_BF16> {
    typedef bf16x2_t pair;
    static constexpr int MOST = 252;  // 6 * 2^125 is finite, 4 * 2^126 is not
    template <int I>
    static __device__ __forceinline__ int decode(int word, float scale)
    {
        return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((unsigned)word, scale, I));
    }
    template <int I>
    static __device__ __forceinline__ int encode(int old, int two, float scale)
    {
        return (int)__builtin_amdgcn_cvt_scalef32_pk_fp4_bf16((unsigned)old, __builtin_bit_cast(pair, two), scale, I);
    }
    static __device__ __forceinline__ float high(int two) { return __builtin_bit_cast(float, two & (int)0xffff0000); }
    static __device__ __forceinline__ float low(int two) { return __builtin_bit_cast(float, two << 16); }
    static __device__ __forceinline__ int scale_of(int byte) { return byte; }  // (none above MOST, by the format of the header)
    static __device__ __forceinline__ f32x4_t mfma(i32x4_t a, i32x4_t b, f32x4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
};
template <>
struct Mx<NAUT_F16> {
    typedef f16x2_t pair;
    static constexpr int MOST = 140;  // 6 * 2^13 = 49152
    template <int I>
    static __device__ __forceinline__ int decode(int word, float scale)
    {
        return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4((unsigned)word, scale, I));
    }
    template <int I>
    static __device__ __forceinline__ int encode(int old, int two, float scale)
    {
        return (int)__builtin_amdgcn_cvt_scalef32_pk_fp4_f16((unsigned)old, __builtin_bit_cast(pair, two), scale, I);
    }
    static __device__ __forceinline__ float high(int two) { return (float)__builtin_bit_cast(pair, two).y; }
    static __device__ __forceinline__ float low(int two) { return (float)__builtin_bit_cast(pair, two).x; }
    static __device__ __forceinline__ int scale_of(int byte) { return byte < MOST ? byte : MOST; }  // no value becomes infinite
    static __device__ __forceinline__ f32x4_t mfma(i32x4_t a, i32x4_t b, f32x4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
};

// ---- rows into and out of the cache ----------------------------------------------------------------------------------

struct RowParams {
    unsigned char *codes[2], *scales[2];  // K, V
    unsigned char* rows[2];               // 16-bit rows
    long long hs[2], rs[2];               // their head and row strides, in bytes
    const int* slots;
    long long c_b, c_h, c_s, s_b, s_h, s_s;
    int T, Hkv, S;
    unsigned slots_of_all;                // B * S
    unsigned s_inv;                       // floor((2^32 - 1) / S)
    int oct;                              // eights of values per row
    int per;                              // rows that a work-group takes at a time = 256 / oct
};

// A thread takes eight values, four neighbours a block: 16 bytes of a row, 4 bytes of codes.  A work-group takes some
// rows of one head: rows that follow each other in the cache, as a prompt's do, are one piece of memory there, and the
// work-groups of a position's heads are neighbours.  Bound by memory; a thread has two rows on their way at once, since one at a
// time (slot, then codes, then the store) is bound by their latency.  32768 rows of 8 heads, D = 128, out of a cache: one
// row, all heads of a position in a work-group 56.0 us; one head 50.4; two rows 35.7 (4.8 TB/s), four 42.5, eight 40.1; two
// with loads from a stand-in address in place of the branches 1.2 times as long.
constexpr int KV_ROWS = 2;
struct RowPlace {
    unsigned char *codes, *scale, *row;
    bool ok;
};
__device__ __forceinline__ void row_places(const RowParams& p, RowPlace (&r)[KV_ROWS])
{
    const int kv = blockIdx.y, tid = threadIdx.x, tl = tid / p.oct, o = tid % p.oct;
    const int hd = blockIdx.x % p.Hkv, t0 = blockIdx.x / p.Hkv * (p.per * KV_ROWS) + tl;
    unsigned slot[KV_ROWS];
#pragma unroll
    for (int i = 0; i < KV_ROWS; ++i) {
        const int t = t0 + i * p.per;
        slot[i] = tl < p.per && t < p.T ? (unsigned)p.slots[t] : ~0u;
    }
#pragma unroll
    for (int i = 0; i < KV_ROWS; ++i) {
        r[i].ok = slot[i] < p.slots_of_all;       // (a negative slot is beyond them)
        unsigned b = __umulhi(slot[i], p.s_inv);  // the quotient, or one less
        unsigned s = slot[i] - b * p.S;
        if (s >= (unsigned)p.S) {
            ++b;
            s -= p.S;
        }
        r[i].codes = p.codes[kv] + b * p.c_b + hd * p.c_h + s * p.c_s + o * 4;  // not used unless ok
        r[i].scale = p.scales[kv] + b * p.s_b + hd * p.s_h + s * p.s_s + (o >> 2);
        r[i].row = p.rows[kv] + (long long)(t0 + i * p.per) * p.rs[kv] + hd * p.hs[kv] + o * 16;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void naut_kv4_store_kernel(const RowParams p)
{
    using X = Mx<DT>;
    RowPlace r[KV_ROWS];
    row_places(p, r);
    i32x4_t w[KV_ROWS];
#pragma unroll
    for (int n = 0; n < KV_ROWS; ++n) {
        w[n] = i32x4_t{0, 0, 0, 0};
        if (r[n].ok)
            w[n] = *(const i32x4_t*)r[n].row;
    }
#pragma unroll
    for (int n = 0; n < KV_ROWS; ++n) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a = fmaxf(a, fmaxf(fabsf(X::low(w[n][i])), fabsf(X::high(w[n][i]))));
        // the largest of the block: four neighbouring lanes have its values (D is a multiple of 32)
        a = fmaxf(a, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), 0xb1, 0xf, 0xf, true)));  // lane ^ 1
        a = fmaxf(a, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), 0x4e, 0xf, 0xf, true)));  // lane ^ 2
        // a = m 2^e, 1 <= m < 2: the power is e - 2, one more from m = 1.75 on, where a quarter carries into the exponent
        int byte = ((__builtin_bit_cast(int, a) + 0x00200000) >> 23) - 2;
        byte = byte < 1 ? 1 : byte < X::MOST ? byte : X::MOST;
        const float scale = mx_scale(byte);
        int codes = X::template encode<0>(0, w[n][0], scale);
        codes = X::template encode<1>(codes, w[n][1], scale);
        codes = X::template encode<2>(codes, w[n][2], scale);
        codes = X::template encode<3>(codes, w[n][3], scale);
        if (r[n].ok) {
            *(int*)r[n].codes = codes;
            if ((threadIdx.x & 3) == 0)
                *r[n].scale = (unsigned char)byte;
        }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void naut_kv4_load_kernel(const RowParams p)
{
    using X = Mx<DT>;
    RowPlace r[KV_ROWS];
    row_places(p, r);
    int codes[KV_ROWS], byte[KV_ROWS];
#pragma unroll
    for (int n = 0; n < KV_ROWS; ++n) {
        codes[n] = byte[n] = 0;
        if (r[n].ok) {
            codes[n] = *(const int*)r[n].codes;
            byte[n] = *r[n].scale;
        }
    }
#pragma unroll
    for (int n = 0; n < KV_ROWS; ++n) {
        const float scale = mx_scale(X::scale_of(byte[n]));
        if (r[n].ok)
            *(i32x4_t*)r[n].row = i32x4_t{X::template decode<0>(codes[n], scale), X::template decode<1>(codes[n], scale),
                                          X::template decode<2>(codes[n], scale), X::template decode<3>(codes[n], scale)};
    }
}

int check_cache(const naut_kv4_cache* c)
{
    if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales)
        return fail(NAUT_ERR_NULL, "the cache and its four pointers must be non-NULL");
    if (c->B <= 0 || c->Hkv <= 0 || c->S <= 0 || c->D <= 0)
        return fail(NAUT_ERR_SHAPE, "the cache's B, Hkv, S and D must be positive");
    if (c->D % MX != 0 || c->D > 256)
        return fail(NAUT_ERR_UNSUPPORTED, "the cache's D must be a multiple of 32, at most 256");
    if ((long long)c->B * c->S > 0x7fffffffLL)
        return fail(NAUT_ERR_UNSUPPORTED, "the cache's B*S exceeds 2^31 - 1");
    if (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) & 15u || c->c_b < 0 || c->c_h < 0 || (c->c_b | c->c_h | c->c_s) % 16 != 0)
        return fail(NAUT_ERR_ALIGN, "codes must be 16-byte aligned, their strides non-negative multiples of 16 bytes");
    const int row = naut_kv4_scale_bytes(c->D);
    if (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) % row != 0 || c->s_b < 0 || c->s_h < 0 || (c->s_b | c->s_h | c->s_s) % row != 0)
        return fail(NAUT_ERR_ALIGN, "scales and their strides must be aligned to naut_kv4_scale_bytes(), the strides non-negative");
    if (c->c_s < c->D / 2 || c->s_s < row)
        return fail(NAUT_ERR_SHAPE, "a position's stride is smaller than its row: rows would overlap");
    if (c->c_s > 1LL << 23 || c->s_s > 1LL << 23)
        return fail(NAUT_ERR_UNSUPPORTED, "position stride too large");
    return NAUT_OK;
}

// Arguments of a store (writes the cache) or a load (writes the rows).
int rows_of(const void* k, const void* v, const naut_kv4_cache* c, const int* slots, int T, int dtype, const naut_strides* st,
            bool load, RowParams* p)
{
    const int rc = check_cache(c);
    if (rc != NAUT_OK)
        return rc;
    if (T < 0)
        return fail(NAUT_ERR_SHAPE, "T must not be negative");
    if (T > 0 && (!k || !v || !slots))
        return fail(NAUT_ERR_NULL, "k, v and slots must be non-NULL device pointers");
    if (dtype != NAUT_BF16 && dtype != NAUT_F16)
        return fail(NAUT_ERR_UNSUPPORTED, "k and v must be bf16 or f16");
    if (((uintptr_t)k | (uintptr_t)v) & 15u)
        return fail(NAUT_ERR_ALIGN, "k and v must be 16-byte aligned");
    if ((uintptr_t)slots & 3u)
        return fail(NAUT_ERR_ALIGN, "slots must be 4-byte aligned");
    naut_strides cs = {};
    cs.k_h = cs.v_h = c->D;
    cs.k_s = cs.v_s = (long long)c->Hkv * c->D;
    if (!st)
        st = &cs;
    const long long strides[4] = {st->k_h, st->k_s, st->v_h, st->v_s};
    for (long long x : strides)
        if (x < 0 || x % 8 != 0 || (load && x == 0))
            return fail(NAUT_ERR_ALIGN, "k/v strides must be multiples of 8 elements (16 bytes), not negative (load: positive)");
    // a store needs every row's bytes to itself
    if (!load && ((c->Hkv > 1 && (c->c_h == 0 || c->s_h == 0)) || (c->B > 1 && (c->c_b == 0 || c->s_b == 0))))
        return fail(NAUT_ERR_SHAPE, "a cache that is stored to cannot have heads or sequences in the same place (stride 0)");
    if (load && (st->k_s < c->D || st->v_s < c->D))
        return fail(NAUT_ERR_SHAPE, "a sequence stride is smaller than D: rows would overlap");
    if (T > 1 << 30 || ((long long)T / (2048 / c->D) + 1) * c->Hkv > 1 << 23)  // 2^31 threads
        return fail(NAUT_ERR_UNSUPPORTED, "too many rows for one call");
    p->codes[0] = (unsigned char*)c->k_codes;
    p->codes[1] = (unsigned char*)c->v_codes;
    p->scales[0] = (unsigned char*)c->k_scales;
    p->scales[1] = (unsigned char*)c->v_scales;
    p->rows[0] = (unsigned char*)k;
    p->rows[1] = (unsigned char*)v;
    p->hs[0] = st->k_h * 2;
    p->hs[1] = st->v_h * 2;
    p->rs[0] = st->k_s * 2;
    p->rs[1] = st->v_s * 2;
    p->slots = slots;
    p->c_b = c->c_b;
    p->c_h = c->c_h;
    p->c_s = c->c_s;
    p->s_b = c->s_b;
    p->s_h = c->s_h;
    p->s_s = c->s_s;
    p->T = T;
    p->Hkv = c->Hkv;
    p->S = c->S;
    p->slots_of_all = (unsigned)c->B * (unsigned)c->S;
    p->s_inv = 0xffffffffu / (unsigned)c->S;
    p->oct = c->D / 8;
    p->per = 256 / p->oct;
    return NAUT_OK;
}

int launched()
{
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? fail_launch(e) : NAUT_OK;
}

// ---- decode-time attention over the cache ----------------------------------------------------------------------------
//
// Bound by reading the cache once: 2 (D/2 + D/32) bytes a key and K/V head.  A wavefront takes blocks of 32 keys, in two key
// tiles of 16, against tiles of 16 query rows (the R = Hq/Hkv * Sq rows that share a K/V head): S^T = K Q^T and O^T += V^T P^T
// on the 16x16x32 matrix instructions, the softmax in between as in the 16-bit kernels, lane-local but for the sum and the
// maximum over the four lane groups of 16.
//   K goes from memory into registers: a lane's 16 bytes of codes are one block of 32 values of one key, four conversions make
// eight of them an A operand, and Q is loaded in the order that this gives the contraction.  V's codes come in the same
// way, are converted, and pass through the wavefront's own LDS as 16-bit rows to be read transposed.
constexpr int KV_SHIFT = 5, KV_BLK = 1 << KV_SHIFT;  // keys per block
constexpr int KV_FINER = 2;     // how much finer it cuts more sequences than fill the chip
constexpr int KV_TARGET = 256;  // work-groups that the plan aims at: one to a CU, of eight wavefronts
constexpr int KV_PLANNED = 256; // sequences from which on a kernel of its own makes the plan (see naut_decode_kv4_plan_kernel)
constexpr int MRG_WAVES = 4;

struct Kv4Params {
    const void* q;
    void* o;
    float* lse;
    const unsigned char *codes[2], *scales[2];  // K, V
    long long c_b, c_h, c_s, s_b, s_h, s_s;
    const int* lens;
    float* ws;        // partial O [nparts][rows][D], then m [nparts][rows], l [nparts][rows], then {first place, splits} [B] or the plan
    int B, Hq, Hkv, Sq, S;
    int R;            // query rows per (sequence, K/V head)
    int rows;         // of a chunk of them, a multiple of 16
    int nchunks;
    int aim;          // splits of all sequences together that fill the chip
    int P;            // and at most: KV_FINER aim + B, or B where every sequence is one split (the grid)
    int slots;        // places for partials, per K/V head and chunk: only parts of a sequence that is split have one, at most 4 aim
    int least;        // blocks per split, at least
    int merges;       // sequences that the merge looks at: B, or, with a plan, those that are split: at most KV_FINER aim
    int planned;
    int causal;
    float c;          // scale * log2(e), > 0
    int out_f32;
    long long q_bs, q_hs, o_bs, o_hs;
    int q_rs, o_rs;
    int nb;           // blocks of 32 values in a row = D / 32
};

__device__ __forceinline__ int kv4_len(const Kv4Params& p, int b)
{
    const int n = p.lens ? p.lens[b] : p.S;
    return n < 0 ? 0 : n < p.S ? n : p.S;
}

struct Kv4Split {
    int b, split, nsplit, slot;  // sequence, its split, its splits, the place of this one's partial (several splits)
    int len, begin, end;         // keys, blocks

    __device__ __forceinline__ void cut()  // from split, nsplit and len
    {
        const int all = ((len - 1) >> KV_SHIFT) + 1, each = (all + nsplit - 1) / nsplit;
        begin = split * each < all ? split * each : all;
        end = begin + each < all ? begin + each : all;
    }
};

// The plan as its kernel leaves it: splits P, each {sequence or -1, split and splits << 16, the place of its partial, keys}, then
// merges, each {sequence or -1, the place of its first partial, splits, 0}.  (A sequence has at most KV_FINER aim + 1 splits.)
__device__ __forceinline__ i32x4_t* kv4_plan_of(const Kv4Params& p, int D)
{
    return (i32x4_t*)(p.ws + (size_t)p.Hkv * p.nchunks * p.slots * p.rows * (D + 2));
}

// Parts of a sequence of n blocks (-1: there is no sequence), rcp = 1 / L.  Need not be the exact quotient: its blocks are dealt out
// evenly over whatever it is.
__device__ __forceinline__ int kv4_parts(int n, float rcp)
{
    const int m = (int)__builtin_fmaf((float)n, rcp, 0.9999f);
    return n < 0 ? 0 : m < 1 ? 1 : m;
}

// How every sequence is cut: into equal parts of about L blocks (an empty one is one part); count(L) gives the parts of all.
//   L is the mean, total / aim, where that makes no more than `aim` parts, as it does for lengths that are alike; or up to twice
// the mean if that keeps them to `aim`, found by halving to a sixteenth (a further round of work-groups costs more than longer parts,
// a longer search more than the shorter parts give); or, with many sequences or one that is most of the batch, half the mean
// (at most 2 aim + B parts).  A sequence of m > 1 parts has more than (m - 1) L blocks, at least m L / 2, so that the parts of those
// that are split are at most 2 total / L, 4 aim.  32/8 heads, D = 128, us with L = total / max(aim, B) always, the mean, half and a quarter of it: one of
// 30000 among 47 of 100 keys 115 / 17.5 / 18.1 / 22.1, 100 of 1 to 8192 103 / 108 / 98 / 91, 64 of 5000 60.5 / 64.1 / 63.9 / 68.1.
template <typename Count>
__device__ __forceinline__ int kv4_part_blocks(const Kv4Params& p, int total, Count&& count)
{
    int L = (total + p.aim - 1) / p.aim;
    L = L > p.least ? L : p.least;
    if (count(L) <= p.aim)
        return L;
    if (count(2 * L) <= p.aim) {
        int lo = L, hi = 2 * L;
        while (hi - lo > (lo >> 4) + 1) {
            const int mid = (lo + hi) >> 1;
            if (count(mid) <= p.aim)
                hi = mid;
            else
                lo = mid;
        }
        return hi;
    }
    L = (total + p.aim * KV_FINER - 1) / (p.aim * KV_FINER);
    return L > p.least ? L : p.least;
}

// Which part of which sequence split x is.  Without a plan every work-group finds it by itself, 64 sequences at a time, one to a lane.
template <int D>
__device__ __forceinline__ bool kv4_split(const Kv4Params& p, int x, int lane, Kv4Split* out)
{
    if (x >= p.P)
        return false;  // the grid is rounded up to eights
    if (p.P == p.B) {  // short caches, or many: a part each
        out->b = x;
        out->split = 0;
        out->nsplit = 1;
        out->slot = 0;
        out->len = __builtin_amdgcn_readfirstlane(kv4_len(p, x));
        out->cut();
        return true;
    }
    if (p.planned) {
        const i32x4_t e = kv4_plan_of(p, D)[x];
        out->b = __builtin_amdgcn_readfirstlane(e.x);
        const int y = __builtin_amdgcn_readfirstlane(e.y);
        out->split = y & 0xffff;
        out->nsplit = y >> 16;
        out->slot = __builtin_amdgcn_readfirstlane(e.z);
        out->len = __builtin_amdgcn_readfirstlane(e.w);
        if (out->b < 0)
            return false;
        out->cut();
        return true;
    }
    const int nch = (p.B + 63) >> 6;
    auto blocks = [&](int c) { return c * 64 + lane < p.B ? ((kv4_len(p, c * 64 + lane) - 1) >> KV_SHIFT) + 1 : -1; };
    const int mine = blocks(0);  // the first 64's, kept
    auto of = [&](int c) { return c == 0 ? mine : blocks(c); };
    int total = 0;
    for (int c = 0; c < nch; ++c)
        total += of(c) > 0 ? of(c) : 0;
    total = wave_sum(total);
    const int L = kv4_part_blocks(p, total, [&](int L) {
        const float rcp = __builtin_amdgcn_rcpf((float)L);
        int sum = kv4_parts(mine, rcp);
        for (int c = 1; c < nch; ++c)
            sum += kv4_parts(blocks(c), rcp);
        return wave_sum(sum);
    });
    const float rcp = __builtin_amdgcn_rcpf((float)L);
    int before = 0, slots_before = 0;
    for (int c = 0; c < nch; ++c) {
        const int m = kv4_parts(of(c), rcp);
        int sum[2] = {m, m > 1 ? m : 0};
        wave_scan(sum);
        const int incl = sum[0] + before;
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(incl > x);
        if (mask == 0) {
            before = __builtin_amdgcn_readlane(incl, 63);
            slots_before += __builtin_amdgcn_readlane(sum[1], 63);
            continue;
        }
        const int src = __builtin_ctzll(mask);
        out->b = c * 64 + src;
        out->nsplit = __builtin_amdgcn_readlane(m, src);
        out->split = x - (__builtin_amdgcn_readlane(incl, src) - out->nsplit);
        out->slot = slots_before + __builtin_amdgcn_readlane(sum[1], src) - out->nsplit + out->split;  // (one part: not used)
        out->len = __builtin_amdgcn_readfirstlane(kv4_len(p, out->b));
        out->cut();
        return true;
    }
    return false;
}

// The plan of many sequences, by one work-group: found by every work-group of the split kernel it takes time that grows with the
// square of the sequences.  The merge gets the sequences that are split, of which there are at most KV_FINER aim.  32/8 heads,
// D = 128, lengths of 1 to 2304, us without and with this kernel: 128 sequences 38.9 / 40.0, 256 77 / 69, 1024 406 / 244, 8192 13700 / 1850;
// 8/1 heads, 1 to 30 keys: 128 12.9 / 15.6, 256 13.1 / 15.2, 512 21.6 / 16.0.
constexpr int PLAN_THREADS = 1024;
template <int D>
__global__ __launch_bounds__(PLAN_THREADS) void naut_decode_kv4_plan_kernel(const Kv4Params p)
{
    constexpr int NW = PLAN_THREADS / 64;
    __shared__ int sums[2][2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int turn = 0;  // two sets of sums in turn: one barrier each
    // sums over the wavefronts before this one, and over all
    auto over_waves = [&](int x, int y, int* x_before, int* y_before, int* x_all, int* y_all) {
        turn ^= 1;
        if (lane == 0) {
            sums[turn][0][wave] = x;
            sums[turn][1][wave] = y;
        }
        __syncthreads();
        *x_before = *y_before = *x_all = *y_all = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int a = sums[turn][0][w], b = sums[turn][1][w];
            *x_before += w < wave ? a : 0;
            *y_before += w < wave ? b : 0;
            *x_all += a;
            *y_all += b;
        }
    };
    auto len_of = [&](int b) { return b < p.B ? kv4_len(p, b) : -KV_BLK; };
    auto blocks = [&](int len) { return ((len - 1) >> KV_SHIFT) + 1; };  // (no sequence: -1)
    static_assert(((-KV_BLK - 1) >> KV_SHIFT) + 1 == -1);
    auto all_of = [&](int x) {
        int a, b, c, d;
        over_waves(wave_sum(x), 0, &a, &b, &c, &d);
        return __builtin_amdgcn_readfirstlane(c);
    };
    int total = 0;
    for (int b = tid; b < p.B; b += PLAN_THREADS)
        total += blocks(len_of(b));
    total = all_of(total);
    const int L = kv4_part_blocks(p, total, [&](int L) {
        const float rcp = __builtin_amdgcn_rcpf((float)L);
        int sum = 0;
        for (int b = tid; b < p.B; b += PLAN_THREADS)
            sum += kv4_parts(blocks(len_of(b)), rcp);
        return all_of(sum);
    });
    const float rcp = __builtin_amdgcn_rcpf((float)L);
    i32x4_t* const plan = kv4_plan_of(p, D);
    int parts = 0, merges = 0;  // of the sequences so far; merges: sequences that are split, and their parts << 16 (at most 4 aim <= 1024)
    for (int b0 = 0; b0 < p.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid, len = len_of(b), m = kv4_parts(blocks(len), rcp), s = m > 1 ? m << 16 | 1 : 0;
        const int m_incl = wave_scan(m), s_incl = wave_scan(s);
        int mb, sb, ma, sa;
        over_waves(__builtin_amdgcn_readlane(m_incl, 63), __builtin_amdgcn_readlane(s_incl, 63), &mb, &sb, &ma, &sa);
        const int first = parts + mb + m_incl - m, at = merges + sb + s_incl - s, slot = at >> 16;
        if (m > 0 && first < p.P)
            plan[first] = i32x4_t{b, m << 16, slot, len};
        if (s != 0 && (at & 0xffff) < p.merges)
            plan[p.P + (at & 0xffff)] = i32x4_t{b, slot, m, 0};
        // the other parts of a sequence, by the wavefront
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(s != 0); left != 0; left &= left - 1) {
            const int src = __builtin_ctzll(left);
            const int first_s = __builtin_amdgcn_readlane(first, src), m_s = __builtin_amdgcn_readlane(m, src);
            const int slot_s = __builtin_amdgcn_readlane(slot, src), len_s = __builtin_amdgcn_readlane(len, src);
            for (int i = 1 + lane; i < m_s; i += 64)
                if (first_s + i < p.P)
                    plan[first_s + i] = i32x4_t{b0 + wave * 64 + src, m_s << 16 | i, slot_s + i, len_s};
        }
        parts += __builtin_amdgcn_readfirstlane(ma);
        merges += __builtin_amdgcn_readfirstlane(sa);
    }
    for (int x = parts + tid; x < p.P; x += PLAN_THREADS)
        plan[x] = i32x4_t{-1, 0, 0, 0};
    for (int x = (merges & 0xffff) + tid; x < p.merges; x += PLAN_THREADS)
        plan[p.P + x] = i32x4_t{-1, 0, 0, 0};
}

// A row of O (four values at d) and, from one thread, of lse: row r of (sequence b, K/V head hk).
template <int DT>
__device__ __forceinline__ void kv4_store_o(const Kv4Params& p, int b, int hk, int r, int d, f32x4_t o)
{
    const int head = hk * (p.Hq / p.Hkv) + r / p.Sq, pos = r % p.Sq;
    unsigned char* const row = (unsigned char*)p.o + b * p.o_bs + head * p.o_hs + (long long)pos * p.o_rs;
    if (d >= p.nb * MX)
        return;  // padding columns of a narrower head
    if (p.out_f32)
        *(f32x4_t*)(row + d * 4) = o;
    else
        *(i32x2_t*)(row + d * 2) = i32x2_t{In<DT>::pack2(o.x, o.y), In<DT>::pack2(o.z, o.w)};
}
__device__ __forceinline__ void kv4_store_lse(const Kv4Params& p, int b, int hk, int r, float m, float l)
{
    if (p.lse != nullptr)  // log2(0) = -inf: a row that saw nothing
        p.lse[((size_t)b * p.Hkv + hk) * p.R + r] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// maximum and sum over the four lane groups of 16
__device__ __forceinline__ float group_max(float x)
{
    float a = x, b = x;
    asm volatile(NAUT_NOP_SHORT "v_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return half_max(fmaxf(a, b));
}
__device__ __forceinline__ float group_sum(float x)
{
    float a = x, b = x;
    asm volatile(NAUT_NOP_SHORT "v_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    a += b;
    b = a;
    asm volatile(NAUT_NOP_SHORT "v_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return a + b;
}

// Bytes between V's rows in LDS.  A transposed read takes 32 bytes of each of 16 rows, a write 16 bytes of each of eight: with
// 32 bytes of padding both go to different banks, and every address is one register plus a constant.
constexpr int v4_row(int D) { return D * 2 + 32; }

// Wavefronts of a split kernel.
constexpr int kv4_waves(int D, int RT) { return D == 256 && RT == 2 ? 4 : 8; }

template <int D, int DT, int RT>
__global__ __launch_bounds__(kv4_waves(D, RT) * 64) void naut_decode_kv4_kernel(const Kv4Params p)
{
    using X = Mx<DT>;
    constexpr int NW = kv4_waves(D, RT);
    // A lane's codes of a block: 16 bytes, one block of 32 values, of one key at a time.  At D >= 128 the four lane groups hold
    // the blocks of the same 16 keys (SETS = 2 of them to a block of keys), at D = 64 two groups those of either key tile.
    constexpr int SETS = D == 64 ? 1 : 2;
    constexpr int KW = D == 64 ? 4 : D / 32;  // words of codes, and MFMAs, per set
    constexpr int DT16 = D / 16;           // 16-row tiles of O^T
    constexpr int VROW = v4_row(D), VB = KV_BLK * VROW;  // a block of V in LDS
    constexpr int OB = RT * 16 * D * 4;    // a wavefront's O
    constexpr int REGION = VB > OB ? VB : OB;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * REGION];
    __shared__ float ml_lds[NW][2][RT * 16];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    // Work-groups are dealt to the XCDs by linear id mod 8.  Eight splits of every chunk and K/V head are neighbours, so that a
    // split of all of them is on one XCD, whose L2 serves the chunks from one read and the heads of a sequence-major cache from
    // whole lines; a number of splits that eight does not divide would leave XCDs idle, and goes one by one.  The splits that
    // no sequence has come last either way: ahead of others they would make room for two work-groups on one CU
    // and none on another (8 caches of 16384 keys 27.5 us for 37.2).
    const int eight = p.aim & 7 ? 0 : 3, y = blockIdx.x >> eight, x_of = (blockIdx.y << eight) + (blockIdx.x & ((1 << eight) - 1));
    const int chunk = p.nchunks == 1 ? 0 : y / p.Hkv, hk = y - chunk * p.Hkv;
    Kv4Split sp;
    if (!kv4_split<D>(p, x_of, lane, &sp))
        return;
    const int b = sp.b, len = sp.len;
    const int g = p.Hq / p.Hkv;
    const int row0 = chunk * p.rows;
    const float c = p.c;
    const unsigned char* const cg[2] = {p.codes[0] + b * p.c_b + hk * p.c_h, p.codes[1] + b * p.c_b + hk * p.c_h};
    const unsigned char* const sg[2] = {p.scales[0] + b * p.s_b + hk * p.s_h, p.scales[1] + b * p.s_b + hk * p.s_h};

    const int key_of = D == 64 ? 16 * (g4 >> 1) + l16 : l16;  // the key of set 0, in the block
    // Word ks holds the values dim(ks) .. + 8 of the key's row, which is the contraction order of MFMA ks.
    auto dim = [&](int ks) { return D == 64 ? 32 * (g4 & 1) + 8 * ks : 32 * (4 * (ks >> 2) + g4) + 8 * (ks & 3); };
    // the block of a lane's chunk j (D = 256 has two), a real one also where the head is narrower
    auto blk_of = [&](int j) {
        const int x = D == 64 ? g4 & 1 : 4 * j + g4;
        return x < p.nb ? x : p.nb - 1;
    };
    constexpr int CH = D == 256 ? 2 : 1;   // chunks per lane and key

    // D = 64: one copy of Q for each key tile, zero in the lanes that hold the other's keys (twice the MFMAs, half the loads)
    constexpr int QT = D == 64 ? 2 : 1;
    i32x4_t qf[RT][QT][KW];
    int lim[RT];  // last key that the lane's row sees
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = row0 + rt * 16 + l16, r = row < p.R ? row : p.R - 1;
        const unsigned char* const qr = (const unsigned char*)p.q + b * p.q_bs + (hk * g + r / p.Sq) * p.q_hs + (long long)(r % p.Sq) * p.q_rs;
        lim[rt] = p.causal ? len - p.Sq + r % p.Sq : len - 1;
#pragma unroll
        for (int ks = 0; ks < KW; ++ks) {
            const i32x4_t x = dim(ks) < p.nb * MX ? *(const i32x4_t*)(qr + dim(ks) * 2) : i32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < QT; ++t)
                qf[rt][t][ks] = QT == 1 || g4 >> 1 == t ? x : i32x4_t{0, 0, 0, 0};
        }
    }

    // Codes of the lane's keys of a block, of K or of V.  The next block's are requested into the same registers as soon as this
    // block's have been converted.
    struct Block {
        int w[SETS][KW];
    };
    const int c_s = (int)p.c_s, s_s = (int)p.s_s;
    auto load = [&](Block& x, int kv, int blk) {
        const int left = len - 1 - blk * KV_BLK;  // the ragged last block reads its last key again
        const unsigned char* const cb = cg[kv] + (long long)blk * (KV_BLK * (long long)c_s);
#pragma unroll
        for (int t = 0; t < SETS; ++t) {
            int key = t * 16 + key_of;
            key = key < left ? key : left;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const i32x4_t y = *(const i32x4_t*)(cb + (unsigned)(key * c_s + blk_of(j) * 16));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x.w[t][4 * j + i] = y[i];
            }
        }
    };
    // The scales of a block's 32 keys of K and of V, a key's row of them to a lane (K's in the lower half of the lanes): one load
    // that touches every line once.  (A byte to a lane straight from memory is four loads, and where the rows of heads lie side by
    // side they cost as much as the codes: 8 sequence-major caches of 16384 keys, 8 heads, D = 128 37.2 us for 28.4.)  Each
    // lane then fetches the words of its keys.
    int sw[CH];
    const unsigned char* const sl = lane < 32 ? sg[0] : sg[1];
    auto load_scales = [&](int blk) {
        const int left = len - 1 - blk * KV_BLK, key = (lane & 31) < left ? lane & 31 : left;
        const unsigned char* const at = sl + (long long)(blk * KV_BLK + key) * s_s;
        if constexpr (D == 64) {
            sw[0] = *(const unsigned short*)at;
        } else if constexpr (D == 128) {
            sw[0] = *(const int*)at;
        } else {
            const i32x2_t y = *(const i32x2_t*)at;
            sw[0] = y.x;
            sw[CH - 1] = y.y;
        }
    };
    float sc[2][SETS][CH];  // of K, V
    auto spread_scales = [&](int kv) {
#pragma unroll
        for (int t = 0; t < SETS; ++t)
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int row = __builtin_amdgcn_ds_bpermute((kv * 32 + t * 16 + key_of) * 4, sw[j]);
                sc[kv][t][j] = mx_scale(X::scale_of(row >> ((blk_of(j) & 3) * 8) & 0xff));
            }
    };
    // eight values of word ks
    auto values = [&](const Block& x, int kv, int t, int ks) -> i32x4_t {
        const float s = sc[kv][t][CH == 1 ? 0 : ks >> 2];
        const int w = x.w[t][ks];
        return i32x4_t{X::template decode<0>(w, s), X::template decode<1>(w, s), X::template decode<2>(w, s), X::template decode<3>(w, s)};
    };

    // where the lane writes its values of V's key, and reads keys 4 g4 .. 4 g4 + 3 of 16 columns transposed
    unsigned char* const v_write = smem + wave * REGION + key_of * VROW + dim(0) * 2;
    const unsigned char* const v_read = smem + wave * REGION + (4 * g4 + (l16 >> 2)) * VROW + (l16 & 3) * 8;
    f32x4_t oacc[RT][DT16];
    float m_run[RT], l_run[RT];  // reference maximum (log2 units, the lowest value there is at first), the lane's share of the sum
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int dt = 0; dt < DT16; ++dt)
            oacc[rt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m_run[rt] = -FLT_MAX;
        l_run[rt] = 0.f;
    }

    Block kx, vx;
    int blk = sp.begin + wave;
    if (blk < sp.end) {
        load_scales(blk);
        load(kx, 0, blk);
        load(vx, 1, blk);
    }
    for (; blk < sp.end; blk += NW) {
        const int nxt = blk + NW < sp.end ? blk + NW : blk;  // the last one's loads are for nobody, and cost less than a branch
        spread_scales(0);
        f32x4_t s[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            s[rt][0] = s[rt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < SETS; ++t)
#pragma unroll
            for (int ks = 0; ks < KW; ++ks) {
                const i32x4_t kf = values(kx, 0, t, ks);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int u = 0; u < QT; ++u)
                        s[rt][t + u] = X::mfma(kf, qf[rt][u][ks], s[rt][t + u]);
            }
        spread_scales(1);
        load_scales(nxt);
        load(kx, 0, nxt);
        // V to LDS, as rows of 16-bit values
#pragma unroll
        for (int t = 0; t < SETS; ++t)
#pragma unroll
            for (int ks = 0; ks < KW; ++ks)
                *(i32x4_t*)(v_write + t * 16 * VROW + (ks >> 2) * 256 + (ks & 3) * 16) = values(vx, 1, t, ks);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        load(vx, 1, nxt);
        const int key0 = blk * KV_BLK;
        i32x4_t pb[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (key0 + KV_BLK - 1 > len - p.Sq || key0 + KV_BLK > len) {  // some row's limit may fall inside the block
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[rt][t][r] = key0 + 16 * t + 4 * g4 + r > lim[rt] ? -INFINITY : s[rt][t][r];
            }
            float mx = s[rt][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                mx = fmaxf(mx, s[rt][i >> 2][i & 3]);
            if (__builtin_amdgcn_ballot_w64(mx * c > m_run[rt]) != 0) {  // the largest P of a row stays exactly 1
                const float m_new = fmaxf(m_run[rt], group_max(mx) * c);
                const float alpha = __builtin_amdgcn_exp2f(m_run[rt] - m_new);
                m_run[rt] = m_new;
                l_run[rt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT16; ++dt)
                    oacc[rt][dt] *= alpha;
            }
            float e[8], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][i >> 2][i & 3], c, -m_run[rt]));
                sum += e[i];
            }
            l_run[rt] += sum;
            pb[rt] = i32x4_t{In<DT>::pack2(e[0], e[1]), In<DT>::pack2(e[2], e[3]), In<DT>::pack2(e[4], e[5]), In<DT>::pack2(e[6], e[7])};
        }
        // A lane's eight keys of P are 4 g4 + {0..3} of either key tile: so are those of the V^T fragments.
#pragma unroll
        for (int dt = 0; dt < DT16; ++dt) {
            const i16x4_t r0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((NAUT_LDS i16x4_t*)(v_read + dt * 32));
            const i16x4_t r1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((NAUT_LDS i16x4_t*)(v_read + dt * 32 + 16 * VROW));
            const i32x2_t lo = __builtin_bit_cast(i32x2_t, r0), hi = __builtin_bit_cast(i32x2_t, r1);
            const i32x4_t vf = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                oacc[rt][dt] = X::mfma(vf, pb[rt], oacc[rt][dt]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // the next block's writes stay behind these reads
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }

    // ---- the wavefronts' partials, merged through LDS (each in its own, now idle, region) ----
    constexpr int Q4 = D / 4;
    auto piece = [&](int w, int r, int q4) { return (f32x4_t*)(smem + w * REGION) + r * Q4 + (q4 ^ (r & 7)); };
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int dt = 0; dt < DT16; ++dt)
            *piece(wave, rt * 16 + l16, 4 * dt + g4) = oacc[rt][dt];
        const float l = group_sum(l_run[rt]);
        if (g4 == 0) {
            ml_lds[wave][0][rt * 16 + l16] = m_run[rt];
            ml_lds[wave][1][rt * 16 + l16] = l;
        }
    }
    __syncthreads();
    const int rows = p.R - row0 < p.rows ? p.R - row0 : p.rows;
    const int part = (hk * p.nchunks + chunk) * p.slots + sp.slot;  // not used by a sequence of one part
    const size_t nparts = (size_t)p.Hkv * p.nchunks * p.slots;
    float* const ws_m = p.ws + nparts * p.rows * D;
    float* const ws_l = ws_m + nparts * p.rows;
    if (sp.split == 0 && chunk == 0 && hk == 0 && tid == 0 && p.P > p.B && !p.planned) {  // for the merge
        int* const at = (int*)(ws_l + nparts * p.rows) + 2 * b;
        at[0] = sp.slot;
        at[1] = sp.nsplit;
    }
    for (int x = tid; x < rows * Q4; x += NW * 64) {
        const int r = x / Q4, q4 = x % Q4;
        float m = -FLT_MAX, l = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w)
            m = fmaxf(m, ml_lds[w][0][r]);
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml_lds[w][0][r] - m);
            l += f * ml_lds[w][1][r];
            acc += *piece(w, r, q4) * f;
        }
        if (sp.nsplit == 1) {
            kv4_store_o<DT>(p, b, hk, row0 + r, 4 * q4, acc * (l > 0.f ? 1.0f / l : 0.f));
            if (q4 == 0)
                kv4_store_lse(p, b, hk, row0 + r, m, l);
        } else {
            *(f32x4_t*)(p.ws + ((size_t)part * p.rows + r) * D + 4 * q4) = acc;
            if (q4 == 0) {
                ws_m[(size_t)part * p.rows + r] = m;
                ws_l[(size_t)part * p.rows + r] = l;
            }
        }
    }
}

// One work-group per query row: the splits of its sequence, where there are several.  Wavefront w takes splits w, w + 4, ..., up
// to eight of them at a time; lanes run over D.
template <int D, int DT>
__global__ __launch_bounds__(MRG_WAVES * 64) void naut_decode_kv4_merge_kernel(const Kv4Params p)
{
    constexpr int EPT = D / 64;
    typedef float fe_t __attribute__((ext_vector_type(EPT)));
    __shared__ float red_m[MRG_WAVES], red_l[MRG_WAVES];
    __shared__ __attribute__((aligned(16))) float red_o[MRG_WAVES][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x, hk = blockIdx.y;
    const int chunk = row / p.rows, r = row % p.rows;
    const size_t nparts = (size_t)p.Hkv * p.nchunks * p.slots;
    const float* ws_m = p.ws + nparts * p.rows * D;
    const float* ws_l = ws_m + nparts * p.rows;
    int b = blockIdx.z, first, nsplit;
    if (p.planned) {
        const i32x4_t e = kv4_plan_of(p, D)[p.P + b];
        b = e.x;
        first = e.y;
        nsplit = e.z;
    } else {
        const int* const at = (const int*)(ws_l + nparts * p.rows) + 2 * b;
        first = at[0];
        nsplit = at[1];
    }
    if (nsplit <= 1)
        return;  // stored already, or no sequence
    const size_t part0 = (size_t)(hk * p.nchunks + chunk) * p.slots + first;
    ws_m += part0 * p.rows + r;
    ws_l += part0 * p.rows + r;
    const float* const ws_o = p.ws + (part0 * p.rows + r) * D;
    fe_t acc = (fe_t)(0.f);
    float M = -FLT_MAX, L = 0.f;
    auto gather = [&](auto BC) {
        constexpr int BATCH = decltype(BC)::value;
        for (int s0 = wave; s0 < nsplit; s0 += MRG_WAVES * BATCH) {
            float m[BATCH], l[BATCH];
            fe_t x[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int s = s0 + u * MRG_WAVES;
                const size_t sc = s < nsplit ? s : s0;  // past the end: repeats a split, not added
                m[u] = ws_m[sc * p.rows];
                l[u] = ws_l[sc * p.rows];
                x[u] = *(const fe_t*)(ws_o + sc * p.rows * D + lane * EPT);
            }
            float m_new = M;
#pragma unroll
            for (int u = 0; u < BATCH; ++u)
                m_new = fmaxf(m_new, m[u]);
            const float alpha = __builtin_amdgcn_exp2f(M - m_new);
            M = m_new;
            L *= alpha;
            acc *= alpha;
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const float f = s0 + u * MRG_WAVES < nsplit ? __builtin_amdgcn_exp2f(m[u] - M) : 0.f;
                L += f * l[u];
                acc += f * x[u];
            }
        }
    };
    if (nsplit <= MRG_WAVES)
        gather(std::integral_constant<int, 1>{});
    else if (nsplit <= 2 * MRG_WAVES)
        gather(std::integral_constant<int, 2>{});
    else
        gather(std::integral_constant<int, 8>{});
    *(fe_t*)&red_o[wave][lane * EPT] = acc;
    if (lane == 0) {
        red_m[wave] = M;
        red_l[wave] = L;
    }
    __syncthreads();
    if (wave != 0 || lane >= D / 4)
        return;
    float m = -FLT_MAX, l = 0.f;
#pragma unroll
    for (int w = 0; w < MRG_WAVES; ++w)
        m = fmaxf(m, red_m[w]);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < MRG_WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(red_m[w] - m);
        l += f * red_l[w];
        o += *(const f32x4_t*)&red_o[w][4 * lane] * f;
    }
    kv4_store_o<DT>(p, b, hk, row, 4 * lane, o * (l > 0.f ? 1.0f / l : 0.f));
    if (lane == 0)
        kv4_store_lse(p, b, hk, row, m, l);
}

constexpr int kv4_width(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Fills in what the sizes decide: R, rows, nchunks, P, slots, least, and the workspace.
bool kv4_plan(int B, int Hq, int Hkv, int Sq, int S, int D, Kv4Params* p, size_t* bytes)
{
    const long long R = (long long)(Hq / Hkv) * Sq;
    const int rows = R <= 16 ? 16 : 32;
    const long long nchunks = (R + rows - 1) / rows;
    if (R > 0x7fffffffLL / 4 || nchunks > 65535 || Hkv > 65535 || B > 65535 - KV_FINER * KV_TARGET || nchunks * Hkv > 1 << 22)  // 2^31 threads
        return false;
    const long long nblk = (S + KV_BLK - 1LL) / KV_BLK;
    const long long least = kv4_waves(kv4_width(D), rows / 16);  // a block for every wavefront
    const long long aim = KV_TARGET / (Hkv * nchunks) > 1 ? KV_TARGET / (Hkv * nchunks) : 1;
    // A part each, and so no merge: where a whole cache is two blocks for every wavefront, or eight and there are enough of them
    // (what a merge costs, 4 us, is what the longest can be behind the others).
    const bool one = nblk <= 2 * least || (B >= aim && nblk <= 8 * least);
    const long long P = one ? B : aim * KV_FINER + B;
    p->R = (int)R;
    p->rows = rows;
    p->nchunks = (int)nchunks;
    p->aim = (int)aim;
    p->P = (int)P;
    p->slots = (int)(P < 4 * aim ? P : 4 * aim);  // P: a few sequences
    p->least = (int)least;
    p->planned = P > B && B >= KV_PLANNED;
    p->merges = p->planned && B > KV_FINER * aim ? (int)aim * KV_FINER : B;
    const size_t ints = p->planned ? ((size_t)P + p->merges) * 4 : (size_t)B * 2;
    *bytes = P > B ? ((size_t)Hkv * nchunks * p->slots * rows * (kv4_width(D) + 2) * sizeof(float) + ints * sizeof(int) + 15) / 16 * 16 : 16;
    return true;
}

template <int D, int DT>
int launch_kv4(const Kv4Params& p, hipStream_t stream)
{
    if (p.planned) {
        hipLaunchKernelGGL((naut_decode_kv4_plan_kernel<D>), dim3(1), dim3(PLAN_THREADS), 0, stream, p);
        const int rc = launched();
        if (rc != NAUT_OK)
            return rc;
    }
    const unsigned eight = p.aim & 7 ? 1 : 8;
    const dim3 grid((unsigned)(p.Hkv * p.nchunks) * eight, ((unsigned)p.P + eight - 1) / eight);
    if (p.rows == 16)
        hipLaunchKernelGGL((naut_decode_kv4_kernel<D, DT, 1>), grid, dim3(kv4_waves(D, 1) * 64), 0, stream, p);
    else
        hipLaunchKernelGGL((naut_decode_kv4_kernel<D, DT, 2>), grid, dim3(kv4_waves(D, 2) * 64), 0, stream, p);
    const int rc = launched();
    if (rc != NAUT_OK || p.P <= p.B)  // one split each
        return rc;
    hipLaunchKernelGGL((naut_decode_kv4_merge_kernel<D, DT>), dim3((unsigned)p.R, (unsigned)p.Hkv, (unsigned)p.merges), dim3(MRG_WAVES * 64), 0, stream, p);
    return launched();
}

}  // namespace

extern "C" {

int naut_kv4_scale_bytes(int D) { return D <= 0 || D % MX != 0 || D > 256 ? 0 : D <= 64 ? 2 : D <= 128 ? 4 : 8; }

int naut_kv4_store(const void* k, const void* v, const naut_kv4_cache* cache, const int* slots, int T, int in_dtype,
                   const naut_strides* st, void* stream)
{
    RowParams p;
    const int rc = rows_of(k, v, cache, slots, T, in_dtype, st, false, &p);
    if (rc != NAUT_OK || T == 0)
        return rc;
    const int rows = p.per * KV_ROWS;
    const dim3 grid((unsigned)((T + rows - 1) / rows * p.Hkv), 2);
    if (in_dtype == NAUT_BF16)
        hipLaunchKernelGGL((naut_kv4_store_kernel<NAUT_BF16>), grid, dim3(256), 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL((naut_kv4_store_kernel<NAUT_F16>), grid, dim3(256), 0, (hipStream_t)stream, p);
    return launched();
}

int naut_kv4_load(void* k, void* v, const naut_kv4_cache* cache, const int* slots, int T, int out_dtype,
                  const naut_strides* st, void* stream)
{
    RowParams p;
    const int rc = rows_of(k, v, cache, slots, T, out_dtype, st, true, &p);
    if (rc != NAUT_OK || T == 0)
        return rc;
    const int rows = p.per * KV_ROWS;
    const dim3 grid((unsigned)((T + rows - 1) / rows * p.Hkv), 2);
    if (out_dtype == NAUT_BF16)
        hipLaunchKernelGGL((naut_kv4_load_kernel<NAUT_BF16>), grid, dim3(256), 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL((naut_kv4_load_kernel<NAUT_F16>), grid, dim3(256), 0, (hipStream_t)stream, p);
    return launched();
}

size_t naut_attn_decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int Sq, int S, int D)
{
    Kv4Params p;
    size_t bytes;
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || S <= 0 || Hq % Hkv != 0 || naut_kv4_scale_bytes(D) == 0 ||
        (long long)B * S > 0x7fffffffLL || !kv4_plan(B, Hq, Hkv, Sq, S, D, &p, &bytes))
        return 0;
    return bytes;
}

int naut_attn_decode_kv4(const void* q, void* o, float* lse, const naut_kv4_cache* cache, const int* lens, int Hq, int Sq,
                         int causal, float scale, void* workspace, size_t workspace_bytes, void* stream, int in_dtype,
                         int out_dtype, const naut_strides* st)
{
    const int rc = check_cache(cache);
    if (rc != NAUT_OK)
        return rc;
    if (!q || !o)
        return fail(NAUT_ERR_NULL, "q and o must be non-NULL device pointers");
    const int B = cache->B, Hkv = cache->Hkv, S = cache->S, D = cache->D;
    if (Hq <= 0 || Sq <= 0)
        return fail(NAUT_ERR_SHAPE, "Hq and Sq must be positive");
    if (Hq % Hkv != 0)
        return fail(NAUT_ERR_SHAPE, "Hq must be a multiple of the cache's Hkv");
    if (!std::isfinite(scale))
        return fail(NAUT_ERR_SHAPE, "scale must be finite");
    if (scale < 0.f)
        return fail(NAUT_ERR_UNSUPPORTED, "negative scale is not supported");
    if ((in_dtype != NAUT_BF16 && in_dtype != NAUT_F16) || (out_dtype != in_dtype && out_dtype != NAUT_F32))
        return fail(NAUT_ERR_UNSUPPORTED, "supported dtypes: q bf16 or f16; o of the same type or f32");
    Kv4Params p = {};
    size_t bytes;
    if (!kv4_plan(B, Hq, Hkv, Sq, S, D, &p, &bytes))
        return fail(NAUT_ERR_UNSUPPORTED, "shape exceeds the grid limits");
    if (((uintptr_t)q | (uintptr_t)o | (uintptr_t)workspace) & 15u)
        return fail(NAUT_ERR_ALIGN, "q, o and workspace must be 16-byte aligned");
    if (((uintptr_t)lse | (uintptr_t)lens) & 3u)
        return fail(NAUT_ERR_ALIGN, "lse and lens must be 4-byte aligned");
    if (!workspace)
        return fail(NAUT_ERR_NULL, "workspace must be a non-NULL device pointer");
    if (workspace_bytes < bytes)
        return fail(NAUT_ERR_SHAPE, "workspace is smaller than naut_attn_decode_kv4_workspace_bytes()");
    naut_strides cs = {};  // contiguous [B][Hq][Sq][D]
    cs.q_s = cs.o_s = D;
    cs.q_h = cs.o_h = (long long)Sq * D;
    cs.q_b = cs.o_b = (long long)Hq * Sq * D;
    if (!st)
        st = &cs;
    const long long in_strides[3] = {st->q_b, st->q_h, st->q_s};
    for (long long x : in_strides)
        if (x < 0 || x % 8 != 0)
            return fail(NAUT_ERR_ALIGN, "q strides must be non-negative multiples of 8 elements (16 bytes)");
    if (st->o_b <= 0 || st->o_h <= 0 || st->o_s <= 0 || st->o_b % 4 != 0 || st->o_h % 4 != 0 || st->o_s % 4 != 0)
        return fail(NAUT_ERR_ALIGN, "o strides must be positive multiples of 4 elements");
    if (st->q_s < D || st->o_s < D)
        return fail(NAUT_ERR_SHAPE, "a sequence stride is smaller than D: rows would overlap");
    const long long max_rs = 1LL << 23;
    if (st->q_s > max_rs || st->o_s > max_rs)
        return fail(NAUT_ERR_UNSUPPORTED, "sequence stride too large");

    const int out_b = out_dtype == NAUT_F32 ? 4 : 2;
    p.q = q;
    p.o = o;
    p.lse = lse;
    p.codes[0] = (const unsigned char*)cache->k_codes;
    p.codes[1] = (const unsigned char*)cache->v_codes;
    p.scales[0] = (const unsigned char*)cache->k_scales;
    p.scales[1] = (const unsigned char*)cache->v_scales;
    p.c_b = cache->c_b;
    p.c_h = cache->c_h;
    p.c_s = cache->c_s;
    p.s_b = cache->s_b;
    p.s_h = cache->s_h;
    p.s_s = cache->s_s;
    p.lens = lens;
    p.ws = (float*)workspace;
    p.B = B;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.Sq = Sq;
    p.S = S;
    p.causal = causal ? 1 : 0;
    const float c = scale * 1.4426950408889634f;
    p.c = c > 0.f ? c : 1.0e-30f;  // scale == 0: every score becomes (almost exactly) 0, the softmax uniform
    p.out_f32 = out_dtype == NAUT_F32;
    p.q_bs = st->q_b * 2;
    p.q_hs = st->q_h * 2;
    p.q_rs = (int)(st->q_s * 2);
    p.o_bs = st->o_b * out_b;
    p.o_hs = st->o_h * out_b;
    p.o_rs = (int)(st->o_s * out_b);
    p.nb = D / MX;
    hipStream_t hs = (hipStream_t)stream;
    const bool bf = in_dtype == NAUT_BF16;
    switch (kv4_width(D)) {
    case 64: return bf ? launch_kv4<64, NAUT_BF16>(p, hs) : launch_kv4<64, NAUT_F16>(p, hs);
    case 128: return bf ? launch_kv4<128, NAUT_BF16>(p, hs) : launch_kv4<128, NAUT_F16>(p, hs);
    default: return bf ? launch_kv4<256, NAUT_BF16>(p, hs) : launch_kv4<256, NAUT_F16>(p, hs);
    }
}

}  // extern "C"
