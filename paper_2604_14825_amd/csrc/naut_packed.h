// naut_packed.h -- packed sequences: the launch parameters of naut_attn_fwd_packed, and which tile a work-group takes.
//
// The sequences of a batch lie back to back in memory and only the GPU knows their lengths (cu_q and cu_k, offsets of
// n + 1 entries each), so that the host needs no copy of them and a captured launch follows them.  The grid is an upper
// bound, and every work-group finds its own tile before its first load.
#ifndef NAUT_PACKED_H
#define NAUT_PACKED_H

namespace naut_k {

constexpr int PACKED_BY_LEVEL = 256;
constexpr int PACKED_COUNTED = 128;

struct PackedParams : Params {  // batch strides, S and the counts of tiles are not used
    const int* cu_q;
    const int* cu_k;
    int n;        // sequences
    int Tq, Tk;   // rows of q and o, and of k and v: no offset reaches beyond them
    int g;        // query heads per K/V head, at most 1024
    unsigned g_inv;  // ceil(2^22 / g)
    int pos_per_tile;  // positions of a tile where they are whole, otherwise 0
    int all_keys;      // no mask: every query sees every key, as if Sk - 1 keys came before the first one's own
    int long_from;     // keys from which on a sequence may have p_limit, shorter ones P_LIMIT_SHORT
    int by_level;      // the tiles go by level, not by sequence (see packed_tile; at most PACKED_BY_LEVEL sequences)
    int class_of[6];   // levels at which a class of tiles ends, falling
};

template <bool PACKED>
using ParamsOf = std::conditional_t<PACKED, PackedParams, Params>;

// The rows of a tile are (position, query head) pairs of one K/V head, the heads of a position next to each other: row r of a
// sequence is position r / g of head hk g + r % g.  Sequences that fill no tile of their own waste g times fewer rows than
// with a tile per head, and the rows of a tile end at nearly the same key (64/8 heads, 8 sequences of 1 to 700 new positions
// behind 333 to 8100 keys, D = 128: 126 tiles for 152).
struct PackedTile {
    int qt, hk;      // tile of its sequence's rows (-1: no tile is left for this work-group), K/V head
    int q0, k0;      // the sequence's first row of q and of k
    int Sq, Sk;
    int rows;        // Sq * g
    int ahead;       // keys before the first query's own
    int pos0, head0; // position and head (of the g) of the tile's first row
    int pos_end;     // the position behind its last row's
};

// Position and head (of the g) of the row x of a tile whose first row is position `pos` of head `head`; x + head < 1280 (BM + g),
// for which the product is exact: (x + head) g < 2^22.
struct PackedRow {
    int pos, head;
};
__device__ __forceinline__ PackedRow packed_row(const PackedParams& p, int pos, int head, int x)
{
    const unsigned y = (unsigned)(x + head), d = y * p.g_inv >> 22;
    return {pos + (int)d, (int)(y - d * (unsigned)p.g)};
}

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

// Tile i by sequence, each from its last one.  Up to PACKED_COUNTED sequences: by their tiles' sums, so that the numbers that no
// tile has come last.  Between others they would take places on the chip that a tile of its last round needs (32/8 heads, D = 128,
// 64 sequences of 1 to 4, as many work-groups with a tile as fit at once: 7.4 us, numbered as below 10.7; 128 of 1 to 16 14.4 / 17.7, of
// 1 to 200 61.9 / 63.7).  The sums of 256 sequences cost as much as they give (256 of 1 to 200 139 for 136, of 1 to 16 27.5 for 28.8).
template <int BM>
__device__ __forceinline__ void packed_tile_by_count(const PackedParams& p, int lane, int i, PackedTile& t)
{
    constexpr int KEPT = PACKED_COUNTED / 64;
    PackedSeq s[KEPT];
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
        s[c] = {0, 0, 0, 0};
        if (c * 64 + lane < p.n)
            s[c] = packed_seq(p, c * 64 + lane);
    }
    int before = 0;
#pragma unroll
    for (int c = 0; c < KEPT; ++c)
        if (c * 64 < p.n) {
            const int incl = before + wave_scan((s[c].Sq * p.g + BM - 1) / BM);
            const unsigned long long mask = __builtin_amdgcn_ballot_w64(incl > i);
            if (mask != 0) {
                const int src = __builtin_ctzll(mask);
                t.q0 = __builtin_amdgcn_readlane(s[c].q0, src);
                t.k0 = __builtin_amdgcn_readlane(s[c].k0, src);
                t.Sq = __builtin_amdgcn_readlane(s[c].Sq, src);
                t.Sk = __builtin_amdgcn_readlane(s[c].Sk, src);
                t.rows = t.Sq * p.g;
                t.qt = __builtin_amdgcn_readlane(incl, src) - 1 - i;
                if (t.qt < 0 || (long long)t.qt * BM >= t.rows)
                    t.qt = -1;  // offsets that fall: sequences that overlap, and a sum that need not fit 32 bits
                return;
            }
            before = __builtin_amdgcn_readlane(incl, 63);
        }
}

// More sequences: sequence b's tiles have the numbers from floor(cu_q[b] g / BM) + b on, which
// are enough of them without a sum over the sequences before; the sequence of a number is found 64 probes at a time.
template <int BM>
__device__ __forceinline__ int packed_number(const PackedParams& p, int b)
{
    const int q0 = p.cu_q[b];
    return (q0 < 0 ? 0 : q0 < p.Tq ? q0 : p.Tq) * p.g / BM + b;
}
template <int BM>
__device__ __forceinline__ void packed_tile_by_sequence(const PackedParams& p, int lane, int i, PackedTile& t)
{
    int lo = 0, hi = p.n;  // the sequence is lo or later, and before hi
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, b = lo + step * (lane + 1);
        const unsigned long long beyond = __builtin_amdgcn_ballot_w64(b >= hi || packed_number<BM>(p, b) > i);  // (lane 63's b is not before hi)
        lo += step * __builtin_ctzll(beyond);
        hi = hi < lo + step ? hi : lo + step;
    }
    const PackedSeq s = packed_seq(p, lo);
    t.q0 = __builtin_amdgcn_readfirstlane(s.q0);
    t.k0 = __builtin_amdgcn_readfirstlane(s.k0);
    t.Sq = __builtin_amdgcn_readfirstlane(s.Sq);
    t.Sk = __builtin_amdgcn_readfirstlane(s.Sk);
    t.rows = t.Sq * p.g;
    const int tiles = (t.rows + BM - 1) / BM, at = i - __builtin_amdgcn_readfirstlane(packed_number<BM>(p, lo));
    t.qt = at >= 0 && at < tiles ? tiles - 1 - at : -1;
}

// The work-group's tile, of BM rows.  Tiles go by sequence, or, with few sequences, by level: heavy ones come first then, as in one
// long causal sequence, and none is left to run behind the others, but a work-group looks at every sequence and those of a sequence
// are apart, which its K and V in the L2s tell.  32/8 heads, D = 128, us by level and by sequence: 16 of 1 to 2000 152 / 157, 24 of
// 50 to 1000 (12/12 heads, D = 64) 33.3 / 36.2, 32 of 1 to 512 47.7 / 45.7, 128 of 1 to 1000 583 / 556, 256 of 1 to 64 55.7 / 49.7, 64 of 1
// to 4 7.9 / 7.4; new turns of 1 to 100 behind up to 1500 keys, 64/8 heads, 64 of them 100 / 109, 100 190 / 196, 256 430 / 434.
//   By level: the last tile of a sequence has the level ceil(Sk g / BM) (at least its number of tiles), those before it one
// less each, as their loops end sooner.  Without the mask a sequence's loops are alike, and all of its tiles have its level (as with the
// mask they would leave the first tiles of long sequences to run behind the others: 6 of 1 to 1646 78.8 us for 88.9, 14 of 1 to 4785,
// 16/16 heads, D = 64 128 for 154).  The tiles go by classes of levels, each half as high as the one before (8, 4, 2, 1, 1/2 and 1/4 of
// the mean level, which the host knows, and the rest).  Inside a class they go by sequence and fall.  F(L), the tiles at level L or
// above, is a sum over the sequences, one to a lane; those of all classes are formed at once, so that the steps of one sum hide the
// latency of another's.  The exact order by levels, found by halving, took every work-group about 1 us longer (14 prompts 172 us for 163).
//   Work-groups are dealt to the XCDs by linear id mod 8: where eight divides the K/V heads, which are the grid's
// first axis, an XCD keeps to an eighth of them, whose rows stay in its L2.
template <int BM>
__device__ __forceinline__ PackedTile packed_tile(const PackedParams& p, int lane)
{
    PackedTile t;
    const int x = blockIdx.x, i = (int)(blockIdx.y + blockIdx.z * gridDim.y);
    t.hk = p.Hkv & 7 ? x : (x & 7) * (p.Hkv >> 3) + (x >> 3);
    t.qt = -1;
    if (!p.by_level) {
        if (p.n <= PACKED_COUNTED)
            packed_tile_by_count<BM>(p, lane, i, t);
        else
            packed_tile_by_sequence<BM>(p, lane, i, t);
        return t;
    }
    const int nch = (p.n + 63) >> 6;  // 64 sequences at a time
    constexpr int KEPT = PACKED_BY_LEVEL / 64;
    constexpr int NC = 7;             // classes
    PackedSeq first = {0, 0, 0, 0};   // of the first 64, for their sequences' own numbers
    int nqt[KEPT], top[KEPT];
    const bool alike = p.all_keys != 0;  // the tiles of a sequence
    auto load = [&](int c, int& tiles, int& level) {
        tiles = level = 0;
        if (c * 64 + lane < p.n) {
            const PackedSeq s = packed_seq(p, c * 64 + lane);
            tiles = (s.Sq * p.g + BM - 1) / BM;
            const int keys = (s.Sk * p.g + BM - 1) / BM;
            const int least = alike ? 1 : tiles;
            level = least > keys ? least : keys;
            if (c == 0)
                first = s;
        }
    };
    // a sequence's tiles at level L or above
    auto part = [&](int tiles, int level, int L) {
        const int y = level - L + 1, m = alike ? tiles : y;
        return y <= 0 ? 0 : m < tiles ? m : tiles;
    };
    int sum[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k)
        sum[k] = 0;
    auto add = [&](int tiles, int level) {
#pragma unroll
        for (int k = 0; k < NC - 1; ++k)
            sum[k] += part(tiles, level, p.class_of[k]);
        sum[NC - 1] += tiles;
    };
#pragma unroll
    for (int c = 0; c < KEPT; ++c) {
        nqt[c] = top[c] = 0;
        if (c < nch) {
            load(c, nqt[c], top[c]);
            add(nqt[c], top[c]);
        }
    }
    wave_scan(sum);
    int from = 0, lower = 1, upper = 0x7fffffff;  // tiles before the class, its lowest level and that of the class before
    bool found = false;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
        const int end = __builtin_amdgcn_readlane(sum[k], 63);
        if (!found && i >= end) {
            from = end;
            if (k < NC - 1)
                upper = p.class_of[k];
        } else if (!found) {
            found = true;
            lower = k < NC - 1 ? p.class_of[k] : 1;
        }
    }
    if (!found)
        return t;  // the grid is an upper bound
    int rank = i - from;
    auto pick = [&](int c, int tiles, int level) {
        const int before = upper == 0x7fffffff ? 0 : part(tiles, level, upper);
        const int m = part(tiles, level, lower) - before;
        const int incl = wave_scan(m);
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(incl > rank);
        if (mask == 0) {
            rank -= __builtin_amdgcn_readlane(incl, 63);
            return false;
        }
        const int src = __builtin_ctzll(mask);
        t.qt = __builtin_amdgcn_readlane(tiles - 1 - before + incl - m, src) - rank;
        if (c == 0) {
            t.q0 = __builtin_amdgcn_readlane(first.q0, src);
            t.k0 = __builtin_amdgcn_readlane(first.k0, src);
            t.Sq = __builtin_amdgcn_readlane(first.Sq, src);
            t.Sk = __builtin_amdgcn_readlane(first.Sk, src);
        } else {
            const PackedSeq s = packed_seq(p, c * 64 + src);
            t.q0 = __builtin_amdgcn_readfirstlane(s.q0);
            t.k0 = __builtin_amdgcn_readfirstlane(s.k0);
            t.Sq = __builtin_amdgcn_readfirstlane(s.Sq);
            t.Sk = __builtin_amdgcn_readfirstlane(s.Sk);
        }
        t.rows = t.Sq * p.g;
        // Offsets that fall can give sequences that overlap, more tiles than the sums above hold, and so a tile that is none.
        if (t.qt < 0 || (long long)t.qt * BM >= t.rows)
            t.qt = -1;
        return true;
    };
#pragma unroll
    for (int c = 0; c < KEPT; ++c)
        if (c < nch && pick(c, nqt[c], top[c]))
            return t;
    return t;
}

// O of packed prompts is stored past the caches: short sequences write half of what a launch moves, and K and V stay in the L2s
// (32/8 heads, D = 128, causal, 64 sequences of 256 103.1 -> 90.8 us, 16 of 1024 183 -> 167, 8 of 2048 287 -> 280; the 14 prompts of 1
// to 2777 169.3 -> 168.2).  (Q loaded past them is slower, 113 us: a row's pieces come by several instructions.)
template <bool PACKED, typename V>
__device__ __forceinline__ void store_o(unsigned char* at, V x)
{
    typedef V __attribute__((aligned(8))) V8;  // O rows of 16-bit values are 8-byte aligned, not more
    if constexpr (PACKED)
        __builtin_nontemporal_store(x, (V8*)at);
    else
        *(V8*)at = x;
}

// Rows that see no key: O is 0 and lse is -inf.  Rows first .. first + count of a tile's sequence, by a whole work-group.
template <int OUTB>
__device__ __forceinline__ void packed_empty_rows(const PackedParams& p, const PackedTile& t, int first, int count, int tid, int threads)
{
    const int pieces = p.cpr * 2;  // four values each
    for (int x = tid; x < count * pieces; x += threads) {
        const int r = first + x / pieces;
        unsigned char* const at = (unsigned char*)p.o + (long long)(t.q0 + r / p.g) * p.o_rs + (t.hk * p.g + r % p.g) * p.o_hs + x % pieces * (4 * OUTB);
        if constexpr (OUTB == 2)
            *(i32x2_t*)at = i32x2_t{0, 0};
        else
            *(f32x4_t*)at = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (p.lse != nullptr && x % pieces == 0)
            p.lse[(size_t)(t.hk * p.g + r % p.g) * p.Tq + t.q0 + r / p.g] = -INFINITY;
    }
}

// The work-group's tile of BM rows with where it starts and ends; false: there is none for it, or one whose rows see nothing, done here.
template <int BM, int OUTB>
__device__ __forceinline__ bool packed_start(const PackedParams& p, int lane, int tid, int threads, PackedTile& t)
{
    t = packed_tile<BM>(p, lane);
    if (t.qt < 0)
        return false;
    const int first = t.qt * BM, count = t.rows - first < BM ? t.rows - first : BM;
    t.ahead = p.all_keys ? t.Sk - 1 : t.Sk - t.Sq;
    t.pos0 = p.pos_per_tile ? t.qt * p.pos_per_tile : first / p.g;
    t.head0 = first - t.pos0 * p.g;
    t.pos_end = packed_row(p, t.pos0, t.head0, count - 1).pos + 1;
    if (t.Sk == 0 || t.pos_end + t.ahead <= 0) {
        packed_empty_rows<OUTB>(p, t, first, count, tid, threads);
        return false;
    }
    return true;
}

}  // namespace naut_k

#endif  // NAUT_PACKED_H
