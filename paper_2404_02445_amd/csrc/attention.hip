// Attention of decoder-style models (gfx950): causal attention over packed prompts, and attention of newly
// drafted tokens over a paged cache.  One pass over the keys with the running maximum and sum of the softmax.
//
// Tiles.  A wave owns 32 query rows.  Scores come out transposed, S^T = K Q^T on the 32x32 MFMA (key fragment
// first): a lane holds one query (lane % 32) and, in register i, key 8 (i / 4) + 4 (lane / 32) + i % 4 of a 32-key
// tile, so a row's maximum and sum are in-lane but for one exchange with lane ^ 32, the statistics are one
// register per lane, and the weights are already in the layout of the second product's B operand, O^T = V^T P^T
// -- the k index of an MFMA may run over the keys in any order that both operands share, so P never leaves the
// registers.  V^T fragments come from row-major V in LDS by transposing reads (bf16) or element reads (float32).
//
// Keys and values stream to LDS with 16-byte direct loads, two stages (K, K, V, V); a row of LDS is the head's dims, a power
// of two of 16-byte chunks, chunk c of row r at place c ^ f(r) (swizzle()), which keeps both the fragment reads
// of K (32 rows, one chunk) and those of V (four rows, 64 bytes) off each other's banks.
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef const __attribute__((address_space(1))) void* gptr_t;

// what absent keys and values are read from
__device__ __attribute__((aligned(16))) const unsigned int kZeros[4] = {0u, 0u, 0u, 0u};

constexpr int kRsrcWord3 = 0x00020000;       // raw buffer, 32-bit data format
constexpr unsigned kOOB = 0x80000000u;       // a lane offset past every resource: reads zeros

// One 16-byte chunk per lane from base + voff into place `lane` of the 1 KB block at dst; zeros where voff is kOOB.
__device__ __forceinline__ void load_lds(const unsigned char* base, lds_ptr_t dst, unsigned voff) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), static_cast<short>(0),
                                                                      0x7fffffff, kRsrcWord3);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, 0, 0, 0);
}

constexpr float kNoMax = -3.40282347e38f;    // running maximum of a row that has seen no key

struct AttnParams {
    const unsigned char *q, *k, *v;
    unsigned char* out;
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;   // bytes
    const int32_t* offsets;          // null: n_seq sequences of max_rows rows
    int n_seq, max_rows;             // rows (tokens) of a sequence at most
    int64_t tokens;
    int heads, kv_heads, group;
    float c;                         // scale * log2(e): weights are powers of two
    // cache
    const int32_t *table, *len;
    int64_t table_stride, pages;
    int max_pages, shift, max_len;
    const uint64_t* mask;
    int mask_words;
    // over a cache: whether blocks take equal shares of all key stages (else one unit each), the least share,
    // partial sums [2 blocks][rows of a tile][head_dim] and their statistics, row tiles of a (sequence, key head)
    int split, least;
    float *part, *stat;
    int row_tiles;
};

constexpr int pow2_up(int v) { int p = 1; while (p < v) p *= 2; return p; }

template <typename T, int D> struct Geo {
    static constexpr int ES = sizeof(T), EPC = 16 / ES;
    static constexpr int CH = D / EPC;           // chunks of a row
    static constexpr int RS = pow2_up(CH);       // chunk places of a row in LDS
    static constexpr int RB = RS * 16;           // bytes of a row in LDS
    static constexpr int KG = CH / 2 % 4 == 0 ? 4 : CH / 2 % 3 == 0 ? 3 : 2;   // K fragments read together
    static_assert(CH / 2 % KG == 0, "whole groups");
};

// Chunk c of row r sits at place c ^ swizzle(r): linear in the bits of r.
template <int RS> __host__ __device__ constexpr int swizzle(int r) {
    if (RS >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    if (RS == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return (r >> 2) & 3;
}

template <int OFF> __device__ __forceinline__ u32x4 lds_read16(unsigned addr) {
    static_assert(OFF >= 0 && OFF < 65536, "ds offset");
    u32x4 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF> __device__ __forceinline__ u32x2 lds_read_tr(unsigned addr) {
    static_assert(OFF >= 0 && OFF < 65536, "ds offset");
    u32x2 v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF> __device__ __forceinline__ unsigned lds_read4(unsigned addr) {
    static_assert(OFF >= 0 && OFF < 65536, "ds offset");
    unsigned v;
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
// until at most N of this wave's LDS reads are still in flight (they complete in order)
template <int N = 0> __device__ __forceinline__ void lds_wait() {
    static_assert(N >= 0 && N <= 15, "lgkmcnt range");
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N) : "memory");
}
template <typename V> __device__ __forceinline__ void pin(V& v) { asm volatile("" : "+v"(v)); }

template <int N, typename F, int I = 0> __device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, F, I + 1>(static_cast<F&&>(f));
    }
}

// the bits of the elements of a word that are infinite or NaN
template <int ES> __device__ __forceinline__ unsigned not_finite(unsigned w) {
    if constexpr (ES == 4) return (w & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
    const unsigned t = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return (t >> 15) * 0xffffu;
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// a sequence's rows [start, start + rows) of the packed tensors
__device__ __forceinline__ void rows_of(const AttnParams& p, int s, int64_t& start, int& rows) {
    if (!p.offsets) {
        start = static_cast<int64_t>(s) * p.max_rows;
        rows = p.max_rows;
        return;
    }
    const int64_t lo = min(max(static_cast<int64_t>(p.offsets[s]), int64_t(0)), p.tokens);
    const int64_t hi = min(static_cast<int64_t>(p.offsets[s + 1]), p.tokens);
    start = lo;
    rows = static_cast<int>(min(max(hi - lo, int64_t(0)), static_cast<int64_t>(p.max_rows)));
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) v += __shfl_xor(v, i, 64);
    return v;
}

// A sequence over the cache: its drafted rows, tokens before them and in all, and its work -- a unit is a tile of BM
// query rows of one key head, of nt key stages (one, empty, where there is nothing to see).
struct SeqShape {
    int64_t start;
    int rows, past, total, nt, units;
};
template <int KT, int BM> __device__ __forceinline__ SeqShape seq_shape(const AttnParams& p, int s) {
    SeqShape q;
    rows_of(p, s, q.start, q.rows);
    q.past = min(max(p.len[s], 0), p.max_len);
    q.total = min(q.past + min(q.rows, p.max_len - q.past), p.max_pages << p.shift);
    q.nt = max(1, (q.total + KT - 1) / KT);
    q.units = (q.rows * p.group + BM - 1) / BM * p.kv_heads;
    return q;
}
// Stages of all sequences, which come one sequence after the other, in it one unit after the other.
template <int KT, int BM> __device__ __forceinline__ int all_stages(const AttnParams& p, int lane) {
    int n = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        const SeqShape q = seq_shape<KT, BM>(p, min(s0 + lane, p.n_seq - 1));
        n += wave_sum(s0 + lane < p.n_seq ? q.nt * q.units : 0);
    }
    return n;
}
// the sequence that stage g < all_stages is in, and its first stage
template <int KT, int BM> __device__ __forceinline__ void find_stage(const AttnParams& p, int lane, int g, int& s, int& base) {
    base = 0;
    for (int s0 = 0;; s0 += 64) {
        const SeqShape q = seq_shape<KT, BM>(p, min(s0 + lane, p.n_seq - 1));
        const int n = s0 + lane < p.n_seq ? q.nt * q.units : 0;
        int upto = n;
#pragma unroll
        for (int i = 1; i < 64; i *= 2) {
            const int v = __shfl_up(upto, i, 64);
            if (lane >= i) upto += v;
        }
        const uint64_t past_g = __ballot(base + upto > g);
        if (past_g) {
            const int at = static_cast<int>(__builtin_ctzll(past_g));
            s = s0 + at;
            base += __shfl(upto - n, at, 64);
            s = __builtin_amdgcn_readfirstlane(s);
            base = __builtin_amdgcn_readfirstlane(base);
            return;
        }
        base += __shfl(upto, 63, 64);
    }
}

// The item-th tile of BM rows: within each 64 sequences, the tiles furthest along their sequence -- the causal
// ones with most keys -- first, so that the long ones start early and the short ones fill the end.
template <int BM> __device__ __forceinline__ bool pick_tile(const AttnParams& p, int item, int lane, int& s, int& tile) {
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        int64_t start;
        int rows = 0;
        if (s0 + lane < p.n_seq) rows_of(p, s0 + lane, start, rows);
        const int nt = (rows + BM - 1) / BM, all = wave_sum(nt);
        if (item >= all) {
            item -= all;
            continue;
        }
        // the level of the item: at least `above` tiles lie higher, sum of (nt - level) over the taller sequences
        int lo = 0, hi = (p.max_rows + BM - 1) / BM, above = 0;      // tiles at or past lo: > item; at or past hi: <= item
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2, n = wave_sum(max(nt - mid, 0));
            if (n > item) lo = mid; else hi = mid, above = n;
        }
        const uint64_t have = __ballot(nt > lo);
        const int rank = item - above;
        const uint64_t below = have & ((uint64_t(1) << lane) - 1);
        const uint64_t hit = __ballot(((have >> lane) & 1) && __popcll(below) == rank);
        s = __builtin_amdgcn_readfirstlane(s0 + static_cast<int>(__builtin_ctzll(hit)));
        tile = __builtin_amdgcn_readfirstlane(lo);
        return true;
    }
    return false;
}

// WR waves take 32 RT rows each, WK waves share a row tile and take every WK-th 32-key tile.
template <typename T, int D, int WR, int WK, int RT, int SUBS, bool PAGED>
__global__ __launch_bounds__(WR * WK * 64, 2) void attention_kernel(const AttnParams p) {
    using G = Geo<T, D>;
    constexpr int ES = G::ES, CH = G::CH, RS = G::RS, RB = G::RB, DT = D / 32;
    constexpr int NW = WR * WK;
    constexpr int BM = WR * RT * 32;                 // rows of a block
    constexpr int KT = 32 * SUBS * WK;               // keys of a stage
    constexpr int TILE = KT * RB;                    // bytes of K (or V) in a stage
    constexpr int NBLK = TILE / 1024, LPW = (NBLK + NW - 1) / NW;
    constexpr int MERGE = WK > 1 ? WK * BM * (D + 4) * 4 + WK * BM * 8 : 0;
    constexpr int LDS = 4 * TILE > MERGE ? 4 * TILE : MERGE;
    constexpr bool OWN = WR == 1 && WK > 1;          // a wave loads the very keys it works on: no barrier a stage
    static_assert(TILE % 1024 == 0 && (!OWN || LPW * (64 / RS) == 32), "whole load blocks");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave % WR, wk = wave / WR;
    const int lr = lane & 31, lh = lane >> 5;

    // --- what this block does ------------------------------------------------------------------
    // Over a cache: stages [g, gend) of the sequences' stages one after the other, so that ragged lengths leave no
    // block with more than another; units cut by a share's end are joined by attention_join_kernel.
    int g = 0, gend = 0, base = 0, s = 0;
    SeqShape sq{};
    if constexpr (PAGED) {
        if (p.split) {
            const int all = all_stages<KT, BM>(p, lane), per = max(p.least, static_cast<int>((all + gridDim.x - 1) / gridDim.x));
            if (static_cast<int64_t>(blockIdx.x) * per >= all) return;
            g = blockIdx.x * per;
            gend = min(all, g + per);
            find_stage<KT, BM>(p, lane, g, s, base);
            sq = seq_shape<KT, BM>(p, s);
        } else {
            const int units = p.kv_heads * p.row_tiles;
            s = blockIdx.x / units;
            sq = seq_shape<KT, BM>(p, s);
            const int unit = blockIdx.x - s * units;
            if (unit >= sq.units) return;
            g = unit * sq.nt;
            gend = g + sq.nt;
        }
    }
    for (;;) {
    int64_t start;
    int rows, kvh, head = 0, tile, past = 0, total, key0 = 0, key1, slot = 0, took = 0;
    bool whole = true;                                // no other block has keys of these rows
    if constexpr (PAGED) {
        start = sq.start;
        rows = sq.rows;
        past = sq.past;                               // tokens before the first query's
        total = sq.total;
        const int row_tiles = sq.units / p.kv_heads, unit = (g - base) / sq.nt, t0 = g - base - unit * sq.nt;
        kvh = unit / row_tiles;
        tile = unit - kvh * row_tiles;
        took = min(sq.nt - t0, gend - g);
        key0 = t0 * KT;
        key1 = min(total, key0 + took * KT);
        whole = took == sq.nt;
        slot = 2 * blockIdx.x + (t0 == 0);
    } else {
        // key heads fastest: the XCDs take blocks round-robin, so the query heads of a key head meet in one L2
        const int hi = blockIdx.x % p.heads, gi = hi / p.kv_heads;
        kvh = hi - gi * p.kv_heads;
        head = kvh * p.group + gi;
        if (!pick_tile<BM>(p, blockIdx.x / p.heads, lane, s, tile)) return;
        rows_of(p, s, start, rows);
        total = rows;
        key1 = min(total, (tile + 1) * BM);
    }
    const int group = PAGED ? p.group : 1;
    const int nrow = rows * group;                    // query rows: tokens, times the heads of a group over a cache
    const int row0 = tile * BM;

    // --- rows of this wave ---------------------------------------------------------------------
    int qtok[RT];                                     // the row's token within the sequence
    u32x4 qf[RT][CH / 2];
    const unsigned char* qrow[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + (wr * RT + r) * 32 + lr, nrow - 1);
        qtok[r] = row / group;
        const int h = PAGED ? kvh * group + (row - qtok[r] * group) : head;
        qrow[r] = p.q + (start + qtok[r]) * p.q_ts + h * p.q_hs;
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) qf[r][i] = *reinterpret_cast<const u32x4*>(qrow[r] + (2 * i + lh) * 16);
    }

    // --- loads -----------------------------------------------------------------------------------
    // Block b of a stage is rows b * 64 / RS ..; lane l fills place l % RS of row (b * 64 + l) / RS.  Wave w
    // loads blocks w LPW .. of K and of V.  A block's rows lie in one page unless pages are smaller than it.
    constexpr int RPB = 64 / RS;                      // rows of a load block
    const unsigned char* const kbase = p.k + (PAGED ? 0 : start * p.k_ts + kvh * p.k_hs);
    const unsigned char* const vbase = p.v + (PAGED ? 0 : start * p.v_ts + kvh * p.v_hs);
    const int lrow = lane / RS;                       // this lane's row in a block
    auto chunk = [&](int b) __attribute__((always_inline)) { return (lane % RS) ^ swizzle<RS>(b * RPB + lrow); };
    const int32_t* const pages = PAGED ? p.table + s * p.table_stride : nullptr;
    // The pages of a stage's blocks, one a lane (-1: absent), are read a stage before its loads go out.
    const bool small = PAGED && (1 << p.shift) < RPB;
    auto pages_of = [&](int k0) __attribute__((always_inline)) -> int {
        if constexpr (!PAGED) return 0;
        const int key = k0 + lane * RPB;
        int page = 0;
        if (lane < NBLK && key < key1 && !small) page = pages[key >> p.shift];
        return static_cast<unsigned>(page) < static_cast<unsigned>(p.pages) ? page : -1;
    };
    auto issue = [&](int k0, int buf, int pgs) __attribute__((always_inline)) {
        const lds_ptr_t dst = (lds_ptr_t)(lds + buf * TILE);
#pragma unroll
        for (int j = 0; j < LPW; ++j) {
            const int b = wave * LPW + j;
            if (NBLK % NW != 0 && b >= NBLK) continue;
            const int ch = chunk(b), key = k0 + b * RPB;             // first key of the block
            unsigned char __attribute__((address_space(3)))* const kd = (unsigned char __attribute__((address_space(3)))*)dst + b * 1024;
            bool in = (key + lrow < key1) & (ch < CH);
            if constexpr (PAGED) {
                if (!small) {
                    const int page = __builtin_amdgcn_readlane(pgs, b);
                    const int64_t at = (((static_cast<int64_t>(max(page, 0)) * p.kv_heads + kvh) << p.shift) + (key & ((1 << p.shift) - 1))) * (D * ES);
                    const unsigned vo = in & (page >= 0) ? static_cast<unsigned>(lrow * (D * ES) + ch * 16) : kOOB;
                    load_lds(kbase + at, (lds_ptr_t)kd, vo);
                    load_lds(vbase + at, (lds_ptr_t)(kd + 2 * TILE), vo);
                } else {
                    const int page = in ? pages[(key + lrow) >> p.shift] : -1;
                    const unsigned char *ks = reinterpret_cast<const unsigned char*>(kZeros), *vs = ks;
                    if (page >= 0 && page < p.pages) {
                        const int64_t off = (((static_cast<int64_t>(page) * p.kv_heads + kvh) << p.shift) + ((key + lrow) & ((1 << p.shift) - 1))) *
                                                (D * ES) + ch * 16;
                        ks = kbase + off;
                        vs = vbase + off;
                    }
                    __builtin_amdgcn_global_load_lds((gptr_t)ks, (lds_ptr_t)kd, 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((gptr_t)vs, (lds_ptr_t)(kd + 2 * TILE), 16, 0, 0);
                }
            } else {
                const int row = b * RPB + lrow;
                load_lds(kbase + k0 * p.k_ts, (lds_ptr_t)kd, in ? static_cast<unsigned>(row * static_cast<int>(p.k_ts)) + ch * 16 : kOOB);
                load_lds(vbase + k0 * p.v_ts, (lds_ptr_t)(kd + 2 * TILE), in ? static_cast<unsigned>(row * static_cast<int>(p.v_ts)) + ch * 16 : kOOB);
            }
        }
    };

    // --- state -----------------------------------------------------------------------------------
    f32x16 o[RT][DT];
    float m[RT], l[RT];                               // maximum (times c) so far; this lane's share of the sum
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = kNoMax;
        l[r] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[r][d][i] = 0.0f;
    }
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_ptr_t)lds));
    // K fragment: row lr, chunk 2 st + lh;  V fragment (bf16): row 4 lh + (lane % 16) / 4 of eight, dims 16 ((lane / 16) % 2)
    // + 4 (lane % 4) of 32; (float32): row 4 lh, dim lr of 32
    const unsigned ka = lds0 + static_cast<unsigned>(lr * RB + ((lh ^ swizzle<RS>(lr)) << 4));
    unsigned va;
    if constexpr (ES == 2) {
        const int row = 4 * lh + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        va = lds0 + static_cast<unsigned>(2 * TILE + row * RB + ((ch ^ swizzle<RS>(row)) << 4) + (lane & 1) * 8);
    } else {
        const int row = 4 * lh, ch = lr >> 2;
        va = lds0 + static_cast<unsigned>(2 * TILE + row * RB + ((ch ^ swizzle<RS>(row)) << 4) + (lr & 3) * 4);
    }

    // visible keys of a row among 64 from k0 on, one bit each
    auto visible = [&](int r, int k0) -> uint64_t {
        const int own = total - past;                 // drafted tokens within bounds
        auto ones = [](int n) -> uint64_t { return n <= 0 ? 0 : n >= 64 ? ~uint64_t(0) : (uint64_t(1) << n) - 1; };
        if (!PAGED || !p.mask) return ones(min(past + qtok[r] + 1, key1) - k0);
        const uint64_t* mrow = p.mask + (start + qtok[r]) * p.mask_words;
        const int j0 = k0 - past;
        uint64_t bits;
        if (j0 >= 0) {
            const int w = j0 >> 6, sh = j0 & 63;
            const uint64_t lo = w < p.mask_words ? mrow[w] : 0, hi = w + 1 < p.mask_words ? mrow[w + 1] : 0;
            bits = (sh ? (lo >> sh) | (hi << (64 - sh)) : lo) & ones(own - j0);
        } else {
            bits = ones(-j0) | (-j0 < 64 ? (mrow[0] & ones(own)) << -j0 : 0);
        }
        return bits & ones(key1 - k0);
    };

    bool marred = false;                              // infinities or NaN among the values were left out
    uint64_t ok = 0;                                  // blocks of the stage at hand whose page is there
    // one 32-key tile: scores, weights and products; `cut`: some row may not see some key
    auto tile32 = [&](int buf, auto sub, int k0, auto cut) __attribute__((always_inline)) {
        const int st0 = buf * TILE + (WK > 1 ? wk * 32 * RB : 0);
        f32x16 sc[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[r][i] = 0.0f;
        constexpr int KG = G::KG, NKG = CH / 2 / KG;      // K fragments of a group, groups
        u32x4 kf[2][KG];
        auto read_k = [&](auto g) __attribute__((always_inline)) {
            static_for<KG>([&](auto e) __attribute__((always_inline)) {
                constexpr int slot = g % 2, st = g * KG + e, el = e;
                kf[slot][el] = lds_read16<sub * 32 * RB>((ka + st0) ^ (st << 5));
            });
        };
        read_k(std::integral_constant<int, 0>{});
        static_for<NKG>([&](auto g) __attribute__((always_inline)) {
            constexpr int slot = g % 2;
            if constexpr (g + 1 < NKG) {
                read_k(std::integral_constant<int, g + 1>{});
                lds_wait<KG>();
            } else {
                lds_wait();
            }
            static_for<KG>([&](auto e) __attribute__((always_inline)) {
                constexpr int st = g * KG + e, el = e;
                pin(kf[slot][el]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if constexpr (ES == 2)
                        sc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[slot][el]),
                                                                        __builtin_bit_cast(bf16x8, qf[r][st]), sc[r], 0, 0, 0);
                    else
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            sc[r] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[slot][el][c]), __uint_as_float(qf[r][st][c]), sc[r],
                                                                         0, 0, 0);
                }
            });
        });
        uint64_t vis[RT];
        if constexpr (cut) {
            // keys of absent pages
            uint64_t held = ~uint64_t(0);
            if constexpr (PAGED) {
                if (small) {
                    const int key = k0 + lane, page = lane < 32 && key < key1 ? pages[key >> p.shift] : -1;
                    held = __ballot(static_cast<unsigned>(page) < static_cast<unsigned>(p.pages));
                } else {
                    constexpr int NB = 32 / RPB;
                    const int b0 = (WK > 1 ? wk * 32 : sub * 32) / RPB;
                    held = 0;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        if ((ok >> (b0 + b)) & 1) held |= ((uint64_t(1) << RPB) - 1) << (b * RPB);
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                vis[r] = visible(r, k0) & held;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((vis[r] >> (8 * (i / 4) + 4 * lh + i % 4)) & 1)) sc[r][i] = -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float mx = sc[r][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[r][i]);
            mx = fmaxf(mx, other_half(mx)) * p.c;
            const float mn = fmaxf(m[r], mx), f = __builtin_amdgcn_exp2f(m[r] - mn);
            m[r] = mn;
            l[r] *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[r][d][i] *= f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[r][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r][i], p.c, -mn));
                l[r] += sc[r][i];
            }
        }
        // O^T += V^T P^T
        constexpr int STEPS = ES == 2 ? 2 : 4;        // groups of registers whose V fragments are read together
        static_for<STEPS>([&](auto u) __attribute__((always_inline)) {
            bf16x8 pf[RT];
            if constexpr (ES == 2)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) pf[r][i] = static_cast<__bf16>(sc[r][8 * u + i]);
            u32x4 vf[DT];
            if constexpr (ES == 2) {
                static_for<DT>([&](auto d) __attribute__((always_inline)) {
                    const u32x2 lo = lds_read_tr<(sub * 32 + u * 16) * RB>((va + st0) ^ (d << 6));
                    const u32x2 hi = lds_read_tr<(sub * 32 + u * 16 + 8) * RB>((va + st0) ^ ((d << 6) | (swizzle<RS>(8) << 4)));
                    vf[d] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                });
            } else {
                static_for<DT>([&](auto d) __attribute__((always_inline)) {
                    static_for<4>([&](auto e) __attribute__((always_inline)) {
                        constexpr int row = 8 * u + e, el = e;
                        vf[d][el] = lds_read4<(sub * 32 + row) * RB>((va + st0) ^ ((d << 7) ^ (swizzle<RS>(row) << 4)));
                    });
                });
            }
            lds_wait();
#pragma unroll
            for (int d = 0; d < DT; ++d) pin(vf[d]);
            // Where a row does not see every key, an infinity or NaN among the values must not meet its zero weight:
            // it is left out here and added where it is seen at the end.
            if constexpr (cut) {
                unsigned bad = 0;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad |= not_finite<ES>(vf[d][e]);
                if (__any(bad != 0)) {
                    marred = true;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) vf[d][e] &= ~not_finite<ES>(vf[d][e]);
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if constexpr (ES == 2)
                        o[r][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[d]), pf[r], o[r][d], 0, 0, 0);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[r][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(vf[d][e]), sc[r][4 * u + e], o[r][d], 0, 0, 0);
                }
        });
    };

    // a stage that every row sees whole: the 32-key tiles of this wave together
    unsigned kr[ES == 2 ? CH / 2 : 1], vr[ES == 2 ? 2 * DT : 1];
    if constexpr (ES == 2) {
        static_for<CH / 2>([&](auto st) __attribute__((always_inline)) { kr[st] = ((ka + (WK > 1 ? wk * 32 * RB : 0)) ^ (st << 5)); });
        static_for<DT>([&](auto d) __attribute__((always_inline)) {
            vr[2 * d] = (va + (WK > 1 ? wk * 32 * RB : 0)) ^ (d << 6);
            vr[2 * d + 1] = vr[2 * d] ^ (swizzle<RS>(8) << 4);
        });
    }
    auto full = [&](auto buf) __attribute__((always_inline)) {
        constexpr int B0 = buf * TILE;
        constexpr int KG = G::KG, NKG = SUBS * (CH / 2) / KG;     // K fragments of a group, groups
        f32x16 sc[SUBS][RT];
#pragma unroll
        for (int t = 0; t < SUBS; ++t)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][r][i] = 0.0f;
        u32x4 kf[2][KG];
        auto read_k = [&](auto g) __attribute__((always_inline)) {
            static_for<KG>([&](auto e) __attribute__((always_inline)) {
                constexpr int st = (g * KG + e) % (CH / 2), sub = (g * KG + e) / (CH / 2), slot = g % 2;
                kf[slot][e] = lds_read16<B0 + sub * 32 * RB>(kr[st]);
            });
        };
        read_k(std::integral_constant<int, 0>{});
        static_for<NKG>([&](auto g) __attribute__((always_inline)) {
            constexpr int slot = g % 2;
            if constexpr (g + 1 < NKG) {
                read_k(std::integral_constant<int, g + 1>{});
                lds_wait<KG>();
            } else {
                lds_wait();
            }
            static_for<KG>([&](auto e) __attribute__((always_inline)) {
                constexpr int st = (g * KG + e) % (CH / 2), sub = (g * KG + e) / (CH / 2);
                pin(kf[slot][e]);
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    sc[sub][r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[slot][e]),
                                                                         __builtin_bit_cast(bf16x8, qf[r][st]), sc[sub][r], 0, 0, 0);
            });
        });
        // the first values on their way under the softmax
        constexpr int NVG = 2 * SUBS;
        u32x2 vf[2][2 * DT];
        auto read_v = [&](auto g) __attribute__((always_inline)) {
            static_for<DT>([&](auto d) __attribute__((always_inline)) {
                constexpr int slot = g % 2, off = B0 + (g / 2 * 32 + g % 2 * 16) * RB;
                vf[slot][2 * d] = lds_read_tr<off>(vr[2 * d]);
                vf[slot][2 * d + 1] = lds_read_tr<off + 8 * RB>(vr[2 * d + 1]);
            });
        };
        read_v(std::integral_constant<int, 0>{});
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float mx = sc[0][r][0];
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, sc[t][r][i]), sc[t][r][i + 1]);
            mx = fmaxf(mx, other_half(mx)) * p.c;
            // The maximum in use may lag by up to 8 (weights stay below 2^8): rescaling is rare.
            if (__any(mx > m[r] + 8.0f)) {
                const float mn = fmaxf(m[r], mx), f = __builtin_amdgcn_exp2f(m[r] - mn);
                m[r] = mn;
                l[r] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[r][d][i] *= f;
            }
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[t][r][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][r][i], p.c, -m[r]));
                    sum[i & 1] += sc[t][r][i];
                }
            l[r] += sum[0] + sum[1];
        }
        static_for<NVG>([&](auto g) __attribute__((always_inline)) {
            constexpr int slot = g % 2;
            if constexpr (g + 1 < NVG) {
                read_v(std::integral_constant<int, g + 1>{});
                lds_wait<2 * DT>();
            } else {
                lds_wait();
            }
            bf16x8 pf[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[r][i] = static_cast<__bf16>(sc[g / 2][r][8 * (g % 2) + i]);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                pin(vf[slot][2 * d]);
                pin(vf[slot][2 * d + 1]);
                const u32x4 w = {vf[slot][2 * d][0], vf[slot][2 * d][1], vf[slot][2 * d + 1][0], vf[slot][2 * d + 1][1]};
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    o[r][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf[r], o[r][d], 0, 0, 0);
            }
        });
    };

    // --- the keys ----------------------------------------------------------------------------------
    // rows of this wave, all of them past the last visible key of the tile: nothing to do (causal)
    const int wave_end = PAGED ? key1 : min(key1, row0 + (wr + 1) * RT * 32);
    // Stages that every row of the block sees whole come first; from an absent page on, every stage is looked at
    // key by key.
    constexpr uint64_t ALL = NBLK >= 64 ? ~uint64_t(0) : (uint64_t(1) << NBLK) - 1;
    const int seen = PAGED ? min(past, key1) : row0 + 1;
    const int full_end = seen > key0 && !small ? key0 + (seen - key0) / KT * KT : key0;
    int pgs = 0;
    auto stage = [&](int k0, int buf) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (!OWN) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int next = pgs;
        if (k0 + KT < key1) issue(k0 + KT, buf ^ 1, next);
        if constexpr (PAGED) pgs = pages_of(k0 + 2 * KT);
        return next;
    };
    int k0 = key0, buf = 0;
    if (key0 < key1) {
        pgs = pages_of(key0);
        issue(key0, 0, pgs);
        ok = PAGED ? __ballot(pgs >= 0) & ALL : ALL;
        pgs = pages_of(key0 + KT);
    }
    // compute of a stage is done: what the next one holds
    auto advance = [&](int next) __attribute__((always_inline)) {
        if constexpr (PAGED) ok = __ballot(next >= 0) & ALL;
        k0 += KT;
        buf ^= 1;
    };
    if constexpr (ES == 2) {
        while (k0 < full_end && ok == ALL) {
            int next = stage(k0, 0);
            full(std::integral_constant<int, 0>{});
            advance(next);
            if (k0 >= full_end || ok != ALL) break;
            next = stage(k0, 1);
            full(std::integral_constant<int, 1>{});
            advance(next);
        }
    } else {
        while (k0 < full_end && ok == ALL) {
            const int next = stage(k0, buf);
            static_for<SUBS>([&](auto sub) __attribute__((always_inline)) {
                tile32(buf, sub, k0 + (WK > 1 ? wk * 32 : 0) + sub * 32, std::false_type{});
            });
            advance(next);
        }
    }
    const int looked_at = k0;                         // keys from here on: one by one
    while (k0 < key1) {
        const int next = stage(k0, buf);
        static_for<SUBS>([&](auto sub) __attribute__((always_inline)) {
            const int k = k0 + (WK > 1 ? wk * 32 : 0) + sub * 32;
            if (k < wave_end) tile32(buf, sub, k, std::true_type{});
        });
        advance(next);
    }

    // what was left out, where it is seen (a weight is positive: the sum becomes infinite or NaN itself)
    if (marred) {
        for (int key = looked_at; key < wave_end; ++key) {
            const unsigned char* vrow;
            if constexpr (PAGED) {
                const int page = pages[key >> p.shift];
                if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.pages)) continue;
                vrow = vbase + (((static_cast<int64_t>(page) * p.kv_heads + kvh) << p.shift) + (key & ((1 << p.shift) - 1))) * (D * ES);
            } else {
                vrow = vbase + key * p.v_ts;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (!(visible(r, key) & 1)) continue;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned* src = reinterpret_cast<const unsigned*>(vrow + (d * 32 + 8 * i + 4 * lh) * ES);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned w = ES == 2 ? (e & 1 ? src[e / 2] & 0xffff0000u : src[e / 2] << 16) : src[e];
                            if (not_finite<4>(w)) o[r][d][4 * i + e] += __uint_as_float(w);
                        }
                    }
            }
        }
    }

    // --- results -----------------------------------------------------------------------------------
#pragma unroll
    for (int r = 0; r < RT; ++r) l[r] += other_half(l[r]);
    if constexpr (WK == 1) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = row0 + (wr * RT + r) * 32 + lr;
            if (row >= nrow) continue;
            const int h = PAGED ? kvh * group + (row - qtok[r] * group) : head;
            if (whole) {
                const float inv = l[r] != 0.0f ? 1.0f / l[r] : 0.0f;
                unsigned char* dst = p.out + (start + qtok[r]) * p.o_ts + h * p.o_hs;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 v = {o[r][d][4 * i] * inv, o[r][d][4 * i + 1] * inv, o[r][d][4 * i + 2] * inv, o[r][d][4 * i + 3] * inv};
                        const int dim = d * 32 + 8 * i + 4 * lh;
                        if constexpr (ES == 2)
                            *reinterpret_cast<bf16x4*>(dst + dim * 2) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                        else
                            *reinterpret_cast<f32x4*>(dst + dim * 4) = v;
                    }
            } else {
                const int64_t at = static_cast<int64_t>(slot) * BM + (row - row0);
                if (lh == 0) {
                    p.stat[2 * at] = m[r];
                    p.stat[2 * at + 1] = l[r];
                }
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(p.part + at * D + d * 32 + 8 * i + 4 * lh) =
                            f32x4{o[r][d][4 * i], o[r][d][4 * i + 1], o[r][d][4 * i + 2], o[r][d][4 * i + 3]};
            }
        }
    } else {
        // the waves of a row tile meet in LDS
        static_assert(RT == 1 || WK == 1, "one row tile a wave");
        constexpr int LD = D + 4;
        __syncthreads();                              // the last stage has been read
        float* const os = reinterpret_cast<float*>(lds);
        float* const ms = os + WK * BM * LD;
        {
            const int row = wr * 32 + lr;
            float* dst = os + (wk * BM + row) * LD + 4 * lh;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(dst + d * 32 + 8 * i) = f32x4{o[0][d][4 * i], o[0][d][4 * i + 1], o[0][d][4 * i + 2], o[0][d][4 * i + 3]};
            if (lh == 0) {
                ms[(wk * BM + row) * 2] = m[0];
                ms[(wk * BM + row) * 2 + 1] = l[0];
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < BM * (D / 4); i += NW * 64) {
            const int rr = i / (D / 4), dim = (i - rr * (D / 4)) * 4, row = row0 + rr;
            if (row >= nrow) continue;
            float top = kNoMax, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WK; ++w) top = fmaxf(top, ms[(w * BM + rr) * 2]);
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float f = __builtin_amdgcn_exp2f(ms[(w * BM + rr) * 2] - top);
                sum += ms[(w * BM + rr) * 2 + 1] * f;
                acc += *reinterpret_cast<const f32x4*>(os + (w * BM + rr) * LD + dim) * f;
            }
            const int tok = row / group, h = PAGED ? kvh * group + (row - tok * group) : head;
            if (whole) {
                const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
                unsigned char* dst = p.out + (start + tok) * p.o_ts + h * p.o_hs;
                acc *= inv;
                if constexpr (ES == 2)
                    *reinterpret_cast<bf16x4*>(dst + dim * 2) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
                else
                    *reinterpret_cast<f32x4*>(dst + dim * 4) = acc;
            } else {
                const int64_t at = static_cast<int64_t>(slot) * BM + rr;
                if (dim == 0) {
                    p.stat[2 * at] = top;
                    p.stat[2 * at + 1] = sum;
                }
                *reinterpret_cast<f32x4*>(p.part + at * D + dim) = acc;
            }
        }
    }
    if constexpr (!PAGED) {
        return;
    } else {
        g += took;
        if (g >= gend) return;
        while (g - base >= sq.units * sq.nt) {        // (stages are left, so there is a sequence with some)
            base += sq.units * sq.nt;
            sq = seq_shape<KT, BM>(p, ++s);
        }
        __syncthreads();                              // LDS is free again
    }
    }
}

// Partial sums of the units that attention_kernel's blocks cut, in block order; the block whose share of stages holds
// a cut unit's end joins it.
template <typename T, int D, int KT, int BM>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnParams p) {
    const int lane = threadIdx.x & 63;
    const int all = all_stages<KT, BM>(p, lane), per = max(p.least, static_cast<int>((all + gridDim.x - 1) / gridDim.x));
    if (blockIdx.x == 0 || static_cast<int64_t>(blockIdx.x) * per >= all) return;
    const int g = blockIdx.x * per;
    int s, base;
    find_stage<KT, BM>(p, lane, g, s, base);
    const SeqShape sq = seq_shape<KT, BM>(p, s);
    const int unit = (g - base) / sq.nt, t0 = g - base - unit * sq.nt;
    if (t0 == 0 || g - t0 + sq.nt > g + per) return;
    const int first = (g - t0) / per, parts = blockIdx.x - first + 1;      // slot 2 first + 1, then 2 (first + i)
    const int row_tiles = sq.units / p.kv_heads, kvh = unit / row_tiles, row0 = (unit - kvh * row_tiles) * BM;
    const int nrow = min(BM, sq.rows * p.group - row0);
    for (int i = threadIdx.x; i < nrow * (D / 4); i += 256) {
        const int rr = i / (D / 4), dim = (i - rr * (D / 4)) * 4;
        auto at = [&](int k) { return static_cast<int64_t>(2 * (first + k) + (k == 0)) * BM + rr; };
        float top = kNoMax, sum = 0.0f;
        for (int k = 0; k < parts; ++k) top = fmaxf(top, p.stat[2 * at(k)]);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < parts; ++k) {
            const float f = __builtin_amdgcn_exp2f(p.stat[2 * at(k)] - top);
            sum += p.stat[2 * at(k) + 1] * f;
            acc += *reinterpret_cast<const f32x4*>(p.part + at(k) * D + dim) * f;
        }
        acc *= sum != 0.0f ? 1.0f / sum : 0.0f;
        const int row = row0 + rr, tok = row / p.group, h = kvh * p.group + (row - tok * p.group);
        unsigned char* dst = p.out + (sq.start + tok) * p.o_ts + h * p.o_hs;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<bf16x4*>(dst + dim * 2) = bf16x4{(__bf16)acc[0], (__bf16)acc[1], (__bf16)acc[2], (__bf16)acc[3]};
        else
            *reinterpret_cast<f32x4*>(dst + dim * 4) = acc;
    }
}

void set_rows(AttnParams& p, int es, const mopar_rows* q, const mopar_rows* out) {
    p.q = static_cast<const unsigned char*>(q->data);
    p.q_ts = q->token_stride * es;
    p.q_hs = q->head_stride * es;
    p.out = static_cast<unsigned char*>(out->data);
    p.o_ts = out->token_stride * es;
    p.o_hs = out->head_stride * es;
}

template <typename F> hipError_t by_type(int dtype, int d, F&& go) {
    auto dims = [&](auto t) {
        switch (d) {
            case 32: return go(t, std::integral_constant<int, 32>{});
            case 64: return go(t, std::integral_constant<int, 64>{});
            case 96: return go(t, std::integral_constant<int, 96>{});
            default: return go(t, std::integral_constant<int, 128>{});
        }
    };
    return dtype == MOPAR_BF16 ? dims(__bf16{}) : dims(float{});
}

// How a call over a cache runs: the rows of a tile by the query rows of a key head, the keys of a stage, and
// whether the blocks take equal shares of the stages.
struct CachePlan {
    int bm, kt, row_tiles, split, blocks;
    int64_t slots_bytes;
};
constexpr int kLeastStages = 2;
CachePlan cache_plan(const mopar_attention& a, int n_seq, int max_q, int max_len) {
    CachePlan c{};
    const bool half = a.dtype == MOPAR_BF16;
    const int64_t rows = static_cast<int64_t>(max_q) * (a.heads / a.kv_heads);
    c.bm = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    c.kt = c.bm == 32 ? (half ? 128 : 64) : c.bm == 64 ? 64 : half ? 64 : 32;
    c.row_tiles = static_cast<int>((rows + c.bm - 1) / c.bm);
    const int64_t units = static_cast<int64_t>(n_seq) * a.kv_heads * c.row_tiles, nt = (max_len + c.kt - 1) / c.kt;
    c.split = nt > 2 * kLeastStages;
    const int64_t blocks = c.split ? std::min<int64_t>(512, units * nt) : units;
    c.blocks = static_cast<int>(std::min<int64_t>(blocks, int64_t(1) << 30));
    c.slots_bytes = c.split ? int64_t(2) * c.blocks * c.bm * (a.head_dim + 2) * 4 : 0;
    return c;
}

}  // namespace

// stages of a call over a cache at most (they are counted in 32 bits)
bool attention_cache_fits(const mopar_attention& a, int n_seq, int max_q, int max_len) {
    const CachePlan c = cache_plan(a, n_seq, max_q, max_len);
    const double stages = static_cast<double>(n_seq) * a.kv_heads * c.row_tiles * ((max_len + static_cast<double>(c.kt) - 1) / c.kt);
    return stages < 1073741824.0;
}

hipError_t launch_attention_prompt(const mopar_attention& a, int64_t tokens, int n_seq, const int32_t* offsets, int max_len,
                                   const mopar_rows* q, const mopar_rows* k, const mopar_rows* v, const mopar_rows* out,
                                   hipStream_t s) {
    if (tokens == 0 || n_seq == 0 || max_len == 0) return hipSuccess;
    const int es = static_cast<int>(dtype_size(a.dtype));
    AttnParams p{};
    set_rows(p, es, q, out);
    p.k = static_cast<const unsigned char*>(k->data);
    p.k_ts = k->token_stride * es;
    p.k_hs = k->head_stride * es;
    p.v = static_cast<const unsigned char*>(v->data);
    p.v_ts = v->token_stride * es;
    p.v_hs = v->head_stride * es;
    p.offsets = offsets;
    p.n_seq = n_seq;
    p.max_rows = max_len;
    p.tokens = tokens;
    p.heads = a.heads;
    p.kv_heads = a.kv_heads;
    p.group = a.heads / a.kv_heads;
    p.c = a.scale * 1.44269504088896341f;
    // tiles of 128 rows: no more than the tokens fill and one more a sequence
    const int64_t items = std::min<int64_t>(tokens / 128 + n_seq, static_cast<int64_t>(n_seq) * ((max_len + 127) / 128));
    if (items * a.heads >= (int64_t(1) << 31)) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(items * a.heads));
    return by_type(a.dtype, a.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        launch_kernel((attention_kernel<T, d, 4, 1, 1, sizeof(T) == 2 ? 2 : 1, false>), grid, dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

size_t attention_cache_ws_bytes(const mopar_attention& a, const mopar_cache& c, int64_t, int max_q, int max_len) {
    return static_cast<size_t>(cache_plan(a, c.n_seq, max_q, max_len).slots_bytes);
}

hipError_t launch_attention_cache(const mopar_attention& a, const mopar_cache& c, int64_t tokens, const int32_t* offsets,
                                  int max_q, const int32_t* len, int max_len, const uint64_t* mask, int mask_words,
                                  const mopar_rows* q, const mopar_rows* out, void* ws, hipStream_t s) {
    if (tokens == 0 || c.n_seq == 0 || max_q == 0) return hipSuccess;
    const int es = static_cast<int>(dtype_size(a.dtype));
    AttnParams p{};
    set_rows(p, es, q, out);
    p.k = static_cast<const unsigned char*>(c.k);
    p.v = static_cast<const unsigned char*>(c.v);
    p.offsets = offsets;
    p.n_seq = c.n_seq;
    p.max_rows = max_q;
    p.tokens = tokens;
    p.heads = a.heads;
    p.kv_heads = a.kv_heads;
    p.group = a.heads / a.kv_heads;
    p.c = a.scale * 1.44269504088896341f;
    p.table = c.table_dev;
    p.len = len;
    p.table_stride = c.table_stride;
    p.pages = c.pages;
    p.max_pages = c.max_pages;
    p.shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));
    p.max_len = max_len;
    p.mask = mask;
    p.mask_words = mask_words;
    const CachePlan cp = cache_plan(a, c.n_seq, max_q, max_len);
    p.row_tiles = cp.row_tiles;
    p.split = cp.split;
    p.least = kLeastStages;
    p.part = static_cast<float*>(ws);
    if (cp.split) p.stat = p.part + int64_t(2) * cp.blocks * cp.bm * a.head_dim;
    const dim3 grid(static_cast<unsigned>(cp.blocks));
    return by_type(a.dtype, a.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr bool H = sizeof(T) == 2;
        auto go = [&](auto kernel, auto join, int threads) {
            launch_kernel(kernel, grid, dim3(threads), 0, s, p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || !cp.split) return e;
            launch_kernel(join, grid, dim3(256), 0, s, p);
            return hipGetLastError();
        };
        if (cp.bm == 32)
            return go(attention_kernel<T, d, 1, H ? 4 : 2, 1, 1, true>, attention_join_kernel<T, d, H ? 128 : 64, 32>, H ? 256 : 128);
        if (cp.bm == 64) return go(attention_kernel<T, d, 2, 2, 1, 1, true>, attention_join_kernel<T, d, 64, 64>, 256);
        return go(attention_kernel<T, d, 4, 1, 1, H ? 2 : 1, true>, attention_join_kernel<T, d, H ? 64 : 32, 128>, 256);
    });
}

}  // namespace mopar
