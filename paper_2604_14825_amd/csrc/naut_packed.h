// naut_packed.h -- packed sequences: the launch parameters of naut_attn_fwd_packed, and which tile a work-group takes.
//
// The sequences of a batch lie back to back in memory and only the GPU knows their lengths (cu_q and cu_k, offsets of
// n + 1 entries each), so that the host needs no copy of them and a captured launch follows them.  The grid is an upper
// bound, and every work-group finds its own tile: a few reductions over the sequences, one to a lane, before its first load.
#ifndef NAUT_PACKED_H
#define NAUT_PACKED_H

namespace naut_k {

struct PackedParams : Params {  // batch strides, S and the counts of tiles are not used
    const int* cu_q;
    const int* cu_k;
    int n;        // sequences
    int Tq, Tk;   // rows of q and o, and of k and v: no offset reaches beyond them
};

template <bool PACKED>
using ParamsOf = std::conditional_t<PACKED, PackedParams, Params>;

struct PackedTile {
    int qt, hq;      // query tile of its sequence (-1: no tile is left for this work-group), query head
    int q0, k0;      // the sequence's first row of q and of k
    int Sq, Sk;
};

// Offsets that do not rise, or that leave the tensors, make an empty sequence: no address comes from them.
struct PackedSeq {
    int q0, k0, Sq, Sk;
};
__device__ __forceinline__ PackedSeq packed_seq(const PackedParams& p, int b)
{
    const int q0 = p.cu_q[b], q1 = p.cu_q[b + 1], k0 = p.cu_k[b], k1 = p.cu_k[b + 1];
    const bool ok = q0 >= 0 && q1 >= q0 && q1 <= p.Tq && k0 >= 0 && k1 >= k0 && k1 <= p.Tk;
    return {q0, k0, ok ? q1 - q0 : 0, ok ? k1 - k0 : 0};
}

// Tile `bid` of a launch over the n sequences, in tiles of BM queries.  The order is that of one long causal sequence,
// heaviest first: the last tile of a sequence has the level ceil(Sk / BM) (at least its number of tiles), those before it
// one less each, and all tiles of a level come before the next.  F(L), the tiles at level L or above, is a sum over the
// sequences; tile i is at the largest L with F(L) > i, found by halving.  Work-groups are dealt to the XCDs by block id
// mod 8: where eight divides the query heads, an XCD keeps to an eighth of them, which share their K/V heads' rows in its L2.
template <int BM>
__device__ __forceinline__ PackedTile packed_tile(const PackedParams& p, int bid, int lane)
{
    PackedTile t;
    int i;
    if (p.Hq & 7) {
        i = bid / p.Hq;
        t.hq = bid % p.Hq;
    } else {
        const int hpx = p.Hq >> 3, s = bid >> 3;
        i = s / hpx;
        t.hq = (bid & 7) * hpx + s % hpx;
    }
    const int nch = (p.n + 63) >> 6;  // 64 sequences at a time
    constexpr int KEPT = 4;           // chunks that stay in registers; later ones are read again for every sum
    int nqt[KEPT], top[KEPT];
    auto load = [&](int c, int& tiles, int& level) {
        tiles = level = 0;
        if (c * 64 + lane < p.n) {
            const PackedSeq s = packed_seq(p, c * 64 + lane);
            tiles = (s.Sq + BM - 1) / BM;
            const int keys = (s.Sk + BM - 1) / BM;
            level = tiles > keys ? tiles : keys;
        }
    };
    int most = 0;
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
        nqt[c] = top[c] = 0;
        if (c < nch)
            load(c, nqt[c], top[c]);
        most = most > top[c] ? most : top[c];
    }
    for (int c = KEPT; c < nch; ++c) {
        int a, b;
        load(c, a, b);
        most = most > b ? most : b;
    }
    auto at_or_above = [&](int L) {
        auto part = [&](int tiles, int level) {
            const int x = level - L + 1;
            return x < 0 ? 0 : x < tiles ? x : tiles;
        };
        int sum = 0;
#pragma unroll
        for (int c = 0; c < KEPT; ++c)
            sum += part(nqt[c], top[c]);
        for (int c = KEPT; c < nch; ++c) {
            int a, b;
            load(c, a, b);
            sum += part(a, b);
        }
        return wave_sum(sum);
    };
    t.qt = -1;
    if (at_or_above(1) <= i)
        return t;
    int lo = 1, hi = 1;
    while (__builtin_amdgcn_ballot_w64(most > hi) != 0)  // the highest level, within a factor of two
        hi *= 2;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at_or_above(mid) > i)
            lo = mid;
        else
            hi = mid - 1;
    }
    int rank = i - at_or_above(lo + 1);  // among the sequences that have a tile at this level
    for (int c = 0; c < nch; ++c) {
        int a, b;
        if (c < KEPT) {
            a = c == 0 ? nqt[0] : c == 1 ? nqt[1] : c == 2 ? nqt[2] : nqt[3];
            b = c == 0 ? top[0] : c == 1 ? top[1] : c == 2 ? top[2] : top[3];
        } else {
            load(c, a, b);
        }
        const bool has = b >= lo && b - a < lo;
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(has);
        const int count = __builtin_popcountll(mask);
        if (rank >= count) {
            rank -= count;
            continue;
        }
        const int before = (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
        const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(has && before == rank));
        t.qt = __builtin_amdgcn_readlane(a, src) - 1 - (__builtin_amdgcn_readlane(b, src) - lo);
        const PackedSeq s = packed_seq(p, c * 64 + src);
        t.q0 = __builtin_amdgcn_readfirstlane(s.q0);
        t.k0 = __builtin_amdgcn_readfirstlane(s.k0);
        t.Sq = __builtin_amdgcn_readfirstlane(s.Sq);
        t.Sk = __builtin_amdgcn_readfirstlane(s.Sk);
        break;
    }
    return t;
}

// Rows that see no key: O is 0 and lse is -inf.  Rows first .. first + count of the packed tensors, by a whole work-group.
template <int OUTB>
__device__ __forceinline__ void packed_empty_rows(const PackedParams& p, int hq, int first, int count, int tid, int threads)
{
    const int pieces = p.cpr * 2;  // four values each
    unsigned char* const o = (unsigned char*)p.o + (long long)first * p.o_rs + hq * p.o_hs;
    for (int x = tid; x < count * pieces; x += threads) {
        unsigned char* const at = o + (long long)(x / pieces) * p.o_rs + x % pieces * (4 * OUTB);
        if constexpr (OUTB == 2)
            *(i32x2_t*)at = i32x2_t{0, 0};
        else
            *(f32x4_t*)at = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    if (p.lse != nullptr)
        for (int x = tid; x < count; x += threads)
            p.lse[(size_t)hq * p.Tq + first + x] = -INFINITY;
}

}  // namespace naut_k

#endif  // NAUT_PACKED_H
