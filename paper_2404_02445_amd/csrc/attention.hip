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
// Keys and values stream through a ring of stages in LDS (all K, then all V) by 16-byte direct loads; a row of LDS is the
// head's dims, a power of two of 16-byte chunks, chunk c of row r at place c ^ f(r) (swizzle()), which keeps both the
// fragment reads of K (32 rows, one chunk) and those of V (four rows, 64 bytes) off each other's banks.
//
// Softmax.  Weights are 2^(s c - m), c = scale log2(e), with m at most 8 below the row's running maximum (they stay under
// 2^8, far from overflow in float32 and in bf16's exponent), so the accumulators are rescaled only where a maximum rises by
// more.  Sums are taken in float32 before the weights are rounded to bf16 for the second product: that rounding (2^-8
// relative, at most) is the one that the matrix instruction's operand needs.
//
// Stages that every row of a block sees whole run without masks, their tiles together and LDS reads ahead of the MFMAs
// (`full`, bf16); the others -- the causal edge, the drafts' own keys, the last keys, absent pages -- run tile by tile with
// a mask (`tile32`).  float32 has its MFMAs at a tenth of bf16's rate and runs on tile32 alone.
//
// Measured, with what bounds it (32 heads of 128 on 8 key heads in bf16; copies reach 5.0 TB/s here, large bf16 products 1450
// TFLOP/s):
//   8192 causal tokens: 530 to 560 us on different cards, 980 to 1040 TFLOP/s.  Matrix units busy 51 % of the time, vector
//     instructions active 46 %: two waves a SIMD (the registers of 32 rows x 128 dims) hide each other's softmax only in part.
//     Deeper LDS prefetch, 32-key stages and products issued a stage ahead of the softmax did not help.
//   16 prompts of 20 to 1100 tokens: 138 to 145 us.  Their bytes are 48 us of copying, their products 80 us at the rate above;
//     the rest is the edges of tiles and, in each short tile, the time to its first keys.
//   64 single tokens over 100 to 4096 cached ones: 122 to 126 us, 4.3 to 4.4 TB/s: memory.
//   16 trees of 20 to 48 over 1000 to 8000: 118 us, 17 us of it the join.  Neither memory (2.9 TB/s) nor the matrix units (19 %
//     busy): waves wait half of their time, one block a CU with a barrier a stage, of whose eight waves three to six have rows.
//   One float32 token over 16400, 12 heads of 64: 38 to 40 us, 2.6 TB/s: a wave's float32 products for 32 rows of which one
//     counts (12 us) behind its loads, and the join (7 us).
// What costs more than its work:
//   Pages whose rows of a key head do not fill 1 KB of LDS (fewer than 4 tokens of 128 bf16 dims, 16 of 32): every stage is
//     masked and looks its pages up key by key.  64 single tokens over 2000: 107 us in pages of 4 or 16, 232 in pages of 1 or 2.
//   max_len far past the sequences: it alone decides whether blocks share.  64 single tokens over 200: 16 us with a max_len of
//     201, 21 with 4096.
//   Thousands of short sequences: each block looks all of them up, 64 at a time.  Prompts of 32 tokens: 512 in 99 us, 4096 in
//     1270; single tokens over 60: 37 and 274.
//   Many new tokens without a mask over a cache: each row meets all the new keys, masked.  2048 over nothing 145 us, where as
//     a prompt they take 52.
// Scalar registers do not suffice over a cache: 15 to 67 are kept in lanes of vector registers, and some forms have a few bytes of
// scratch for that; no vector register is spilled.
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

// what absent keys and values are read from
__device__ __attribute__((aligned(16))) const unsigned int kZeros[4] = {0u, 0u, 0u, 0u};

constexpr int kRsrcWord3 = 0x00020000;       // raw buffer, 32-bit data format
constexpr unsigned kOOB = 0x80000000u;       // a lane offset past every resource: reads zeros

// Direct loads into LDS, to the byte address dst (the same in every lane), in inline asm so that the compiler does not take
// every later read of LDS for a reader of theirs (it would wait for all loads in flight).  They have no result in registers.
// What they write is read after begin(): a count of the loads in flight and a barrier, which the compiler moves no access
// of memory across.  m0, which they write, is in no other use (the compiler warns that it is a reserved register).
// Wait states: one after a write of m0, five after a vector instruction (a readlane) wrote a scalar register of a resource.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ u32x4 resource(const unsigned char* base) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    return u32x4{static_cast<unsigned>(a), static_cast<unsigned>(a >> 32) & 0xffffu, 0x7fffffffu, kRsrcWord3};
}
// Two 16-byte chunks per lane, from k + kofs and v + vofs into place `lane` of the 1 KB blocks at kdst and vdst; zeros where an
// offset is kOOB.
__device__ __forceinline__ void load_lds(const unsigned char* k, unsigned kdst, unsigned kofs, const unsigned char* v, unsigned vdst, unsigned vofs) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
                 "s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                 ::"s"(kdst), "v"(kofs), "s"(resource(k)), "s"(vdst), "v"(vofs), "s"(resource(v))
                 : "memory", "m0");
}
// ... from the lane's own addresses
__device__ __forceinline__ void load_lds(const unsigned char* k, unsigned kdst, const unsigned char* v, unsigned vdst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\t"
                 "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, off"
                 ::"s"(kdst), "v"(k), "s"(vdst), "v"(v)
                 : "memory", "m0");
}
// One word per lane from its own address into word `lane` of dst.
__device__ __forceinline__ void load_lds(const int32_t* src, unsigned dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(dst), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

constexpr float kNoMax = -3.40282347e38f;    // running maximum of a row that has seen no key

// A unit that several blocks had keys of: its partial sums are slot 2 first + 1, then 2 (first + i), i < parts.
struct CutUnit {
    int parts, first, rows, row0, kvh, reserved;
    int64_t start;
};

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
    int shift, max_len;              // max_len: at most the slots of the table, at most 2^30
    const uint64_t* mask;
    int mask_words;
    int side;                        // over prompts: log2 of the query heads of a tile
    // over a cache: whether blocks take equal shares of all key stages (else one unit each), partial sums
    // [2 blocks][rows of a tile][head_dim] and their statistics, row tiles of a (sequence, key head)
    int split;
    float *part, *stat;
    CutUnit* cuts;                   // a block's: the unit that it ends and did not begin (parts 0: none)
    int row_tiles;
};

// The kernel's arguments, read again: what is needed once in a while is not kept in scalar registers.
typedef const __attribute__((address_space(4))) AttnParams* ArgsPtr;
__device__ __forceinline__ ArgsPtr args_again() {
    ArgsPtr a = (ArgsPtr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
}

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

// LDS fragment reads.  Those of the masked tiles wait within their asm; of the whole stages the compiler knows each (lds_get16,
// lds_get_tr), and waits for it where its value is used.  A read whose wait stands elsewhere would leave its registers to the
// allocator before they are written, so there are none.
template <int N, int OFF> __device__ __forceinline__ void lds_read16(u32x4 (&v)[N], const unsigned (&a)[N]) {
    static_assert(OFF >= 0 && OFF < 65536 && N >= 2 && N <= 4, "ds offset");
    if constexpr (N == 4)
        asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\tds_read_b128 %2, %6 offset:%8\n\t"
                     "ds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
                     : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(OFF)
                     : "memory");
    else if constexpr (N == 3)
        asm volatile("ds_read_b128 %0, %3 offset:%6\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_b128 %2, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2])
                     : "v"(a[0]), "v"(a[1]), "v"(a[2]), "n"(OFF)
                     : "memory");
    else
        asm volatile("ds_read_b128 %0, %2 offset:%4\n\tds_read_b128 %1, %3 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1])
                     : "v"(a[0]), "v"(a[1]), "n"(OFF)
                     : "memory");
}
// two transposing reads: lanes 4 i .. 4 i + 3 of 16 read 4 x 4 elements of a row each, lane i gets column i of the four rows
template <int OFF0, int OFF1> __device__ __forceinline__ void lds_read_tr(u32x2& v0, u32x2& v1, unsigned a0, unsigned a1) {
    static_assert(OFF0 >= 0 && OFF0 < 65536 && OFF1 >= 0 && OFF1 < 65536, "ds offset");
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%4\n\tds_read_b64_tr_b16 %1, %3 offset:%5\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(v0), "=&v"(v1)
                 : "v"(a0), "v"(a1), "n"(OFF0), "n"(OFF1)
                 : "memory");
}
template <int O0, int O1, int O2, int O3> __device__ __forceinline__ void lds_read4(u32x4& v, const unsigned (&a)[4]) {
    static_assert(O0 >= 0 && O3 < 65536, "ds offset");
    unsigned w0, w1, w2, w3;
    asm volatile("ds_read_b32 %0, %4 offset:%8\n\tds_read_b32 %1, %5 offset:%9\n\tds_read_b32 %2, %6 offset:%10\n\t"
                 "ds_read_b32 %3, %7 offset:%11\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(w0), "=&v"(w1), "=&v"(w2), "=&v"(w3)
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(O0), "n"(O1), "n"(O2), "n"(O3)
                 : "memory");
    v = u32x4{w0, w1, w2, w3};
}
__device__ __forceinline__ unsigned lds_read_word(unsigned a) {
    unsigned v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(a) : "memory");
    return v;
}
template <int OFF> __device__ __forceinline__ u32x4 lds_get16(unsigned addr) {
    return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)(addr + OFF);
}
template <int OFF> __device__ __forceinline__ bf16x4 lds_get_tr(unsigned addr) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4*)(uintptr_t)(addr + OFF));
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

// the same in every lane: kept in scalar registers, and branches on it are scalar ones (a resource in vector registers
// would cost a loop over the lanes at each load)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<unsigned>(uniform(static_cast<int>(v >> 32)))) << 32 |
                                static_cast<unsigned>(uniform(static_cast<int>(v))));
}

// within rows of 16 lanes by DPP moves (partners 1 and 2 apart, the mirrored half row, the mirrored row), then the rows
__device__ __forceinline__ int wave_sum(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false);
    return (__builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16)) +
           (__builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48));
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
    q.total = q.past + min(q.rows, p.max_len - q.past);
    q.nt = max(1, (q.total + KT - 1) / KT);
    q.units = (q.rows * p.group + BM - 1) / BM * p.kv_heads;
    return q;
}
// ... of a sequence that every lane asks for
template <int KT, int BM> __device__ __forceinline__ SeqShape seq_shape_of_block(const AttnParams& p, int s) {
    SeqShape q = seq_shape<KT, BM>(p, uniform(s));
    q.start = uniform(q.start);
    q.rows = uniform(q.rows), q.past = uniform(q.past), q.total = uniform(q.total), q.nt = uniform(q.nt), q.units = uniform(q.units);
    return q;
}

// All sequences' stages, one sequence after the other and in it one unit after the other, cut into equal shares for
// the blocks of a grid: this block's share [g, gend), the sequence that it starts in and that one's first stage.
// False: no share.
struct Share {
    int per, g, gend, s, base;
};
template <int KT, int BM> __device__ __forceinline__ bool take_share(const AttnParams& p, int lane, Share& sh) {
    auto stages = [&](int s) {
        const SeqShape q = seq_shape<KT, BM>(p, min(s, p.n_seq - 1));
        return s < p.n_seq ? q.nt * q.units : 0;
    };
    const int head = stages(lane);                     // the first 64 sequences are looked up once
    int all = wave_sum(head);
    for (int s0 = 64; s0 < p.n_seq; s0 += 64) all += wave_sum(stages(s0 + lane));
    sh.per = static_cast<int>((all + gridDim.x - 1) / gridDim.x);
    if (static_cast<int64_t>(blockIdx.x) * sh.per >= all) return false;
    sh.g = blockIdx.x * sh.per;
    sh.gend = min(all, sh.g + sh.per);
    for (int s0 = 0, base = 0;; s0 += 64) {
        const int n = s0 == 0 ? head : stages(s0 + lane);
        int upto = n;
#pragma unroll
        for (int i = 1; i < 64; i *= 2) {
            const int v = __shfl_up(upto, i, 64);
            if (lane >= i) upto += v;
        }
        const uint64_t past_g = __ballot(base + upto > sh.g);
        if (past_g) {                                  // (g < all: some chunk has it)
            const int at = static_cast<int>(__builtin_ctzll(past_g));
            sh.s = __builtin_amdgcn_readfirstlane(s0 + at);
            sh.base = __builtin_amdgcn_readfirstlane(base + __shfl(upto - n, at, 64));
            return true;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
}

// The item-th tile of 2^sh tokens: within each 64 sequences, the tiles furthest along their sequence -- the causal
// ones with most keys -- first, so that the long ones start early and the short ones fill the end.  With its
// sequence's rows.
__device__ __forceinline__ bool pick_tile(const AttnParams& p, int sh, int item, int lane, int& tile, int64_t& start, int& rows) {
    for (int s0 = 0; s0 < p.n_seq; s0 += 64) {
        int64_t first = 0;
        int n = 0;
        if (s0 + lane < p.n_seq) rows_of(p, s0 + lane, first, n);
        const int nt = (n + (1 << sh) - 1) >> sh, all = wave_sum(nt);
        if (item >= all) {
            item -= all;
            continue;
        }
        // the level of the item: at least `above` tiles lie higher, sum of (nt - level) over the taller sequences
        int lo = 0, hi = (p.max_rows + (1 << sh) - 1) >> sh, above = 0;      // tiles at or past lo: > item; at or past hi: <= item
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2, higher = wave_sum(max(nt - mid, 0));
            if (higher > item) lo = mid; else hi = mid, above = higher;
        }
        const uint64_t have = __ballot(nt > lo);
        const int rank = item - above;
        const uint64_t below = have & ((uint64_t(1) << lane) - 1);
        const uint64_t hit = __ballot(((have >> lane) & 1) && __popcll(below) == rank);
        const int at = uniform(static_cast<int>(__builtin_ctzll(hit)));
        tile = uniform(lo);
        start = static_cast<int64_t>(static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(first >> 32), at))) << 32 |
                                     static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(first), at)));
        rows = __builtin_amdgcn_readlane(n, at);
        return true;
    }
    return false;
}

// A block of WR waves takes WR tiles of 32 rows.  The keys come in stages of KT through a ring of NS stages in LDS: while
// one is worked on, NS - 1 (a single wave: all NS, each stage's place being filled again as soon as it is done) are on
// their way.  A block of one wave needs no barrier.
template <typename T, int D, int WR, int SUBS, int NS, bool PAGED>
__global__ __launch_bounds__(WR * 64, 2) void attention_kernel(const AttnParams p) {
    using G = Geo<T, D>;
    constexpr int ES = G::ES, CH = G::CH, RS = G::RS, RB = G::RB, DT = D / 32, KG = G::KG;
    constexpr int BM = WR * 32;                      // rows of a block
    constexpr int KT = 32 * SUBS;                    // keys of a stage
    constexpr int TILE = KT * RB;                    // bytes of K (or V) in a stage
    constexpr int NBLK = TILE / 1024, LPW = (NBLK + WR - 1) / WR;
    constexpr int RPB = 64 / RS;                     // rows of a load block
    constexpr bool OWN = WR == 1;
    static_assert(TILE % 1024 == 0 && NBLK <= 64 && NS >= 2 && (NS & (NS - 1)) == 0, "stages");
    static_assert(PAGED || NS == 2, "the loop over prompts knows its two stages at compile time");
    static_assert((NS - 1) * (2 * LPW + 1) <= 63, "vmcnt range");
    constexpr int AHEAD = OWN ? NS : NS - 1;         // stages on their way when one is begun
    constexpr int RING = 2 * NS * TILE;              // then, over a cache, each wave's pages of four stages
    __shared__ __attribute__((aligned(1024))) unsigned char lds[RING + (PAGED ? WR * 1024 : 0)];
    static_assert(AHEAD <= 3, "places for the pages");
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_ptr_t)lds));

    const int lane = threadIdx.x & 63, wave = OWN ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 31, lh = lane >> 5;

    // --- what this block does ------------------------------------------------------------------
    // Over a cache: stages [g, gend) of the sequences' stages one after the other, so that ragged lengths leave no
    // block with more than another; units cut by a share's end are joined by attention_join_kernel.
    int per = 0, g = 0, gend = 0, base = 0, s = 0;
    SeqShape sq{};
    if constexpr (PAGED) {
        if (p.split) {
            Share sh;
            const bool any = take_share<KT, BM>(p, lane, sh);
            if (threadIdx.x == 0) p.cuts[blockIdx.x].parts = 0;       // (set below where this block ends a cut unit)
            if (!any) return;
            per = sh.per;
            g = sh.g;
            gend = sh.gend;
            s = sh.s;
            base = sh.base;
            sq = seq_shape_of_block<KT, BM>(p, s);
        } else {
            const int units = p.kv_heads * p.row_tiles;
            s = blockIdx.x / units;
            sq = seq_shape_of_block<KT, BM>(p, s);
            const int unit = blockIdx.x - s * units;
            if (unit >= sq.units) return;
            g = unit * sq.nt;
            gend = g + sq.nt;
        }
    }
    for (;;) {
        int64_t start;
        int rows, kvh, head = 0, tile, row0, wave0, past = 0, total, key0 = 0, key1, slot = 0, took = 0;
        bool whole = true;                            // no other block has keys of these rows
        if constexpr (PAGED) {
            start = sq.start;
            rows = sq.rows;
            past = sq.past;                           // tokens before the first query's
            total = sq.total;
            const int row_tiles = sq.units / p.kv_heads, unit = (g - base) / sq.nt, t0 = g - base - unit * sq.nt;
            kvh = unit / row_tiles;
            tile = unit - kvh * row_tiles;
            row0 = tile * BM;
            wave0 = row0 + wave * 32;
            took = min(sq.nt - t0, gend - g);
            key0 = t0 * KT;
            key1 = min(total, key0 + took * KT);
            whole = took == sq.nt;
            slot = 2 * blockIdx.x + (t0 == 0);
            if (t0 > 0 && t0 + took == sq.nt && threadIdx.x == 0) {
                const int first = (g - t0) / per;
                args_again()->cuts[blockIdx.x] =
                    CutUnit{static_cast<int>(blockIdx.x) - first + 1, first, min(BM, rows * p.group - row0), row0, kvh, 0, start};
            }
        } else {
            // a tile is 2^side heads of a key head by BM >> side tokens, a wave 32 tokens of one head.  Key heads fastest: the
            // XCDs take blocks round-robin, so the query heads of a key head meet in one L2
            const int sets = p.heads >> p.side, hi = blockIdx.x % sets, gi = hi / p.kv_heads;
            kvh = hi - gi * p.kv_heads;
            head = kvh * p.group + (gi << p.side) + (wave & ((1 << p.side) - 1));
            constexpr int kShift = __builtin_ctz(BM);
            if (!pick_tile(p, kShift - p.side, blockIdx.x / sets, lane, tile, start, rows)) return;
            total = rows;
            row0 = tile << (kShift - p.side);
            wave0 = row0 + (wave >> p.side) * 32;
            key1 = min(total, row0 + (BM >> p.side));
        }
        const int group = PAGED ? p.group : 1;
        const int nrow = rows * group;                // query rows: tokens, times the heads of a group over a cache

        // --- this wave's rows: row lr of its 32 (past the last: that one again, never stored) ------------
        const int row = min(wave0 + lr, nrow - 1);
        const int qtok = PAGED ? row / group : row;   // the row's token within the sequence
        const int qhead = PAGED ? kvh * group + (row - qtok * group) : head;
        u32x4 qf[CH / 2];
        {
            const ArgsPtr ar = args_again();
            const unsigned char* q = ar->q + (start + qtok) * ar->q_ts + qhead * ar->q_hs + lh * 16;
#pragma unroll
            for (int i = 0; i < CH / 2; ++i) qf[i] = *reinterpret_cast<const u32x4*>(q + i * 32);
        }

        // --- loads -----------------------------------------------------------------------------------
        // Block b of a stage is rows b RPB ..; lane l fills place l % RS of row b RPB + l / RS.  Wave w loads blocks
        // w LPW .. of K and of V.  A block's rows lie in one page unless pages are smaller than it (`small`).
        const int64_t page_bytes = (static_cast<int64_t>(p.kv_heads) << p.shift) * (D * ES);
        const int64_t in_page = (static_cast<int64_t>(kvh) << p.shift) * (D * ES);     // of this head
        const unsigned char* const kbase = p.k + (PAGED ? in_page : start * p.k_ts + kvh * p.k_hs);
        const unsigned char* const vbase = p.v + (PAGED ? in_page : start * p.v_ts + kvh * p.v_hs);
        const int lrow = lane / RS;
        const int32_t* const pages = PAGED ? p.table + s * p.table_stride : nullptr;
        const int page_mask = (1 << p.shift) - 1;
        const bool small = PAGED && page_mask + 1 < RPB;
        auto page_at = [&](unsigned page, int key) __attribute__((always_inline)) {    // byte offset of a key's row
            return static_cast<int64_t>(page) * page_bytes + (key & page_mask) * (D * ES);
        };
        // The pages of a stage's blocks, one a lane.  They go to LDS as the keys do, AHEAD stages before the stage's own
        // loads: a plain load carried round the loop would make the compiler wait for every load in flight.  From the
        // first absent page on (bad_from), keys are looked at one by one.
        int bad_from = small ? key0 : 0x7fffffff;
        auto page_of = [&](int k0) __attribute__((always_inline)) {    // (lanes past the stage or the keys: the last key's)
            return pages + (min(k0 + min(lane, NBLK - 1) * RPB, key1 - 1) >> p.shift);
        };
        auto send_pages = [&](int k0) __attribute__((always_inline)) {
            if constexpr (PAGED)
                load_lds(page_of(k0), lds0 + RING + wave * 1024 + (k0 / KT & 3) * 256);
        };
        auto sent_pages = [&](int k0) __attribute__((always_inline)) -> int {
            if constexpr (!PAGED) return 0;
            return lds_read_word(lds0 + RING + wave * 1024 + (k0 / KT & 3) * 256 + lane * 4);
        };
        auto look_at = [&](int pgs, int k0) __attribute__((always_inline)) {
            if constexpr (PAGED)
                if (__any(static_cast<unsigned>(pgs) >= static_cast<unsigned>(p.pages))) bad_from = min(bad_from, k0);
        };
        auto issue = [&](int k0, int at, int pgs) __attribute__((always_inline)) {
            const unsigned place = lds0 + at * TILE;
            if (PAGED && small) {
                for (int j = 0; j < LPW; ++j) {
                    const int b = wave * LPW + j;
                    if (NBLK % WR != 0 && b >= NBLK) break;
                    const int rrow = b * RPB + lrow, ch = (lane % RS) ^ swizzle<RS>(rrow), key = k0 + rrow;
                    const unsigned page = key < key1 && ch < CH ? pages[key >> p.shift] : ~0u;
                    const unsigned char *ks = reinterpret_cast<const unsigned char*>(kZeros), *vs = ks;
                    if (page < static_cast<unsigned>(p.pages)) {
                        const int64_t off = page_at(page, key) + ch * 16;
                        ks = kbase + off;
                        vs = vbase + off;
                    }
                    load_lds(ks, place + b * 1024, vs, place + NS * TILE + b * 1024);
                }
                return;
            }
            // Over a cache lane b works out where block b starts.  Rows past the last key and absent pages (page 0
            // stands for them) load what is there: keys looked at one by one leave it out.
            unsigned lo = 0, hi = 0;
            if constexpr (PAGED) {
                const unsigned page = static_cast<unsigned>(pgs) < static_cast<unsigned>(p.pages) ? pgs : 0;
                const uint64_t off = page_at(page, k0 + lane * RPB);
                lo = static_cast<unsigned>(off), hi = static_cast<unsigned>(off >> 32);
            }
#pragma unroll
            for (int j = 0; j < LPW; ++j) {
                const int b = wave * LPW + j;
                if (NBLK % WR != 0 && b >= NBLK) continue;
                const int rrow = b * RPB + lrow, ch = (lane % RS) ^ swizzle<RS>(rrow);
                const unsigned kd = place + b * 1024, vd = place + NS * TILE + b * 1024;
                if constexpr (PAGED) {
                    const int64_t off = static_cast<int64_t>(__builtin_amdgcn_readlane(lo, b)) |
                                        static_cast<int64_t>(__builtin_amdgcn_readlane(hi, b)) << 32;
                    const unsigned vo = CH == RS || ch < CH ? static_cast<unsigned>(lrow * (D * ES) + ch * 16) : kOOB;
                    load_lds(kbase + off, kd, vo, vbase + off, vd, vo);
                } else {
                    const bool in = (k0 + rrow < key1) & (ch < CH);
                    load_lds(kbase + k0 * p.k_ts, kd, in ? static_cast<unsigned>(rrow * static_cast<int>(p.k_ts)) + ch * 16 : kOOB,
                             vbase + k0 * p.v_ts, vd, in ? static_cast<unsigned>(rrow * static_cast<int>(p.v_ts)) + ch * 16 : kOOB);
                }
            }
        };

        // --- state -----------------------------------------------------------------------------------
        f32x16 o[DT];
        float m = kNoMax, l = 0.0f;                   // maximum (times c) in use; this lane's share of the sum
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
        // K fragment: row lr, chunk 2 st + lh;  V fragment (bf16): row 4 lh + (lane % 16) / 4 of eight, dims 16 ((lane / 16) % 2)
        // + 4 (lane % 4) of 32; (float32): row 4 lh, dim lr of 32
        const unsigned ka = lds0 + static_cast<unsigned>(lr * RB + ((lh ^ swizzle<RS>(lr)) << 4));
        unsigned va;
        if constexpr (ES == 2) {
            const int vrow = 4 * lh + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            va = lds0 + static_cast<unsigned>(NS * TILE + vrow * RB + ((ch ^ swizzle<RS>(vrow)) << 4) + (lane & 1) * 8);
        } else {
            const int vrow = 4 * lh, ch = lr >> 2;
            va = lds0 + static_cast<unsigned>(NS * TILE + vrow * RB + ((ch ^ swizzle<RS>(vrow)) << 4) + (lr & 3) * 4);
        }

        // visible keys of this lane's row among 64 from k0 on, one bit each
        auto visible = [&](int k0) -> uint64_t {
            auto ones = [](int n) -> uint64_t { return n <= 0 ? 0 : n >= 64 ? ~uint64_t(0) : (uint64_t(1) << n) - 1; };
            const ArgsPtr ar = args_again();
            const uint64_t* mrow = PAGED ? ar->mask : nullptr;
            if (!mrow) return ones(min(past + qtok + 1, key1) - k0);
            const int words = ar->mask_words;
            mrow += (start + qtok) * words;
            const int j0 = k0 - past, own = total - past;       // drafted tokens within bounds
            uint64_t bits;
            if (j0 >= 0) {
                const int w = j0 >> 6, sh = j0 & 63;
                uint64_t lo = w < words ? mrow[w] : 0, hi = w + 1 < words ? mrow[w + 1] : 0;
                pin(lo);                              // (waited for here on every path, and so nowhere in the loop)
                pin(hi);
                bits = (sh ? (lo >> sh) | (hi << (64 - sh)) : lo) & ones(own - j0);
            } else {
                uint64_t lo = mrow[0];
                pin(lo);
                bits = ones(-j0) | (-j0 < 64 ? (lo & ones(own)) << -j0 : 0);
            }
            return bits & ones(key1 - k0);
        };

        bool marred = false;                          // infinities or NaN among the values were left out
        int looked_at = key1;                         // keys from here on may have been looked at one by one
        // The maximum in use may lag by up to 8 (weights stay below 2^8), so that rescaling is rare.
        auto keep_max = [&](float mx) __attribute__((always_inline)) {
            if (__any(mx > m + 8.0f)) {
                const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
            }
        };
        // one 32-key tile, st0 bytes into the ring; `cut`: some row may not see some key
        auto tile32 = [&](int st0, int k0, bool cut) __attribute__((always_inline)) {
            f32x16 sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
            constexpr int NKG = CH / 2 / KG;          // groups of K fragments
            static_for<NKG>([&](auto gr) __attribute__((always_inline)) {
                u32x4 kf[KG];
                unsigned a[KG];
#pragma unroll
                for (int e = 0; e < KG; ++e) a[e] = (ka + st0) ^ ((gr * KG + e) << 5);
                lds_read16<KG, 0>(kf, a);
#pragma unroll
                for (int e = 0; e < KG; ++e) {
                    if constexpr (ES == 2)
                        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[e]), __builtin_bit_cast(bf16x8, qf[gr * KG + e]),
                                                                     sc, 0, 0, 0);
                    else
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            sc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e][c]), __uint_as_float(qf[gr * KG + e][c]), sc, 0, 0, 0);
                }
            });
            if (cut) {
                looked_at = min(looked_at, k0);
                uint64_t vis = visible(k0);
                if constexpr (PAGED)
                    if (k0 + 32 > bad_from) {         // keys of absent pages
                        const int key = k0 + lane;
                        unsigned page = lane < 32 && key < key1 ? pages[key >> p.shift] : ~0u;
                        pin(page);
                        vis &= __ballot(page < static_cast<unsigned>(p.pages));
                    }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((vis >> (8 * (i / 4) + 4 * lh + i % 4)) & 1)) sc[i] = -INFINITY;
            }
            float mx = sc[0];
#pragma unroll
            for (int i = 1; i < 15; i += 2) mx = fmaxf(fmaxf(mx, sc[i]), sc[i + 1]);
            mx = fmaxf(mx, sc[15]);
            mx = fmaxf(mx, other_half(mx)) * p.c;
            keep_max(mx);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], p.c, -m));
                l += sc[i];
            }
            // O^T += V^T P^T
            constexpr int STEPS = ES == 2 ? 2 : 4;    // groups of registers whose V fragments are read together
            static_for<STEPS>([&](auto u) __attribute__((always_inline)) {
                bf16x8 pf;
                if constexpr (ES == 2)
#pragma unroll
                    for (int i = 0; i < 8; ++i) pf[i] = static_cast<__bf16>(sc[8 * u + i]);
                u32x4 vf[DT];
                static_for<DT>([&](auto d) __attribute__((always_inline)) {
                    if constexpr (ES == 2) {
                        constexpr int R0 = u * 16 * RB;
                        u32x2 lo, hi;
                        lds_read_tr<R0, R0 + 8 * RB>(lo, hi, (va + st0) ^ (d << 6), (va + st0) ^ ((d << 6) | (swizzle<RS>(8) << 4)));
                        vf[d] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                    } else {
                        constexpr int R0 = 8 * u;
                        unsigned a[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = (va + st0) ^ ((d << 7) ^ (swizzle<RS>(8 * u + e) << 4));
                        lds_read4<R0 * RB, (R0 + 1) * RB, (R0 + 2) * RB, (R0 + 3) * RB>(vf[d], a);
                    }
                });
                // Where a row does not see every key, an infinity or NaN among the values must not meet its zero weight:
                // it is left out here and put back where it is seen at the end.
                if (cut) {
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
                for (int d = 0; d < DT; ++d) {
                    if constexpr (ES == 2)
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[d]), pf, o[d], 0, 0, 0);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(vf[d][e]), sc[4 * u + e], o[d], 0, 0, 0);
                }
            });
        };

        // a stage that every row sees whole (bf16): its 32-key tiles together.  `at` is its place in the ring, a
        // compile-time constant over prompts (folded into the reads' offsets).
        unsigned kr[ES == 2 && !PAGED ? CH / 2 : 1], vr[ES == 2 && !PAGED ? 2 * DT : 1];
        if constexpr (ES == 2 && !PAGED) {
            static_for<CH / 2>([&](auto st) __attribute__((always_inline)) { kr[st] = ka ^ (st << 5); });
            static_for<DT>([&](auto d) __attribute__((always_inline)) {
                vr[2 * d] = va ^ (d << 6);
                vr[2 * d + 1] = vr[2 * d] ^ (swizzle<RS>(8) << 4);
            });
        }
        auto full = [&](auto at) __attribute__((always_inline)) {
            constexpr int B0 = [] { if constexpr (PAGED) return 0; else return decltype(at)::value * TILE; }();
            unsigned kd = 0, vd = 0;                  // the reads' bases in this stage
            if constexpr (PAGED) kd = ka + at * TILE, vd = va + at * TILE;
            constexpr int NKG = SUBS * (CH / 2) / KG; // groups of K fragments
            f32x16 sc[SUBS];
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = 0.0f;
            u32x4 kf[2][KG];
            auto read_k = [&](auto gr) __attribute__((always_inline)) {
                static_for<KG>([&](auto e) __attribute__((always_inline)) {
                    constexpr int st = (gr * KG + e) % (CH / 2), sub = (gr * KG + e) / (CH / 2), half = gr % 2;
                    kf[half][e] = lds_get16<B0 + sub * 32 * RB>(PAGED ? kd ^ (st << 5) : kr[PAGED ? 0 : st]);
                });
            };
            read_k(std::integral_constant<int, 0>{});
            static_for<NKG>([&](auto gr) __attribute__((always_inline)) {
                constexpr int half = gr % 2;
                if constexpr (gr + 1 < NKG) read_k(std::integral_constant<int, gr + 1>{});
                __builtin_amdgcn_sched_barrier(0);    // (the next group's reads before this one's products)
                static_for<KG>([&](auto e) __attribute__((always_inline)) {
                    constexpr int st = (gr * KG + e) % (CH / 2), sub = (gr * KG + e) / (CH / 2);
                    sc[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[half][e]), __builtin_bit_cast(bf16x8, qf[st]),
                                                                      sc[sub], 0, 0, 0);
                });
            });
            // the first values on their way under the softmax
            constexpr int NVG = 2 * SUBS;
            bf16x4 vf[2][2 * DT];
            auto read_v = [&](auto gr) __attribute__((always_inline)) {
                static_for<DT>([&](auto d) __attribute__((always_inline)) {
                    constexpr int half = gr % 2, off = B0 + gr * 16 * RB;
                    vf[half][2 * d] = lds_get_tr<off>(PAGED ? vd ^ (d << 6) : vr[PAGED ? 0 : 2 * d]);
                    vf[half][2 * d + 1] = lds_get_tr<off + 8 * RB>(PAGED ? vd ^ ((d << 6) | (swizzle<RS>(8) << 4)) : vr[PAGED ? 0 : 2 * d + 1]);
                });
            };
            read_v(std::integral_constant<int, 0>{});
            float mx = sc[0][0];
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, sc[t][i]), sc[t][i + 1]);
            mx = fmaxf(mx, other_half(mx)) * p.c;
            keep_max(mx);
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < SUBS; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], p.c, -m));
                    sum[i & 1] += sc[t][i];
                }
            l += sum[0] + sum[1];
            static_for<NVG>([&](auto gr) __attribute__((always_inline)) {
                constexpr int half = gr % 2;
                if constexpr (gr + 1 < NVG) read_v(std::integral_constant<int, gr + 1>{});
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 pf;
#pragma unroll
                for (int i = 0; i < 8; ++i) pf[i] = static_cast<__bf16>(sc[gr / 2][8 * (gr % 2) + i]);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const bf16x8 w = __builtin_shufflevector(vf[half][2 * d], vf[half][2 * d + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, pf, o[d], 0, 0, 0);
                }
            });
        };

        // --- the keys ----------------------------------------------------------------------------------
        // Of this wave's rows: the keys that all of them see, and the end of those that any sees.
        const int all_see = PAGED ? past : wave0 + 1;
        const int wave_end = PAGED ? (wave0 < nrow ? key1 : key0) : min(key1, wave0 + 32);
        int k0 = key0, at = 0;                        // the stage at hand and its place
        int first[AHEAD];                             // pages of the first stages
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) first[i] = PAGED && key0 < key1 ? *page_of(key0 + i * KT) : 0;
        if (!PAGED) issue(0, 0, 0);
        // the queries are waited for here, or the compiler would do it, for every load in flight, in the loop
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) pin(qf[i]);
        if (PAGED && key0 < key1) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                look_at(first[i], key0 + i * KT);
                send_pages(key0 + (i + AHEAD) * KT);
                if (key0 + i * KT < key1) issue(key0 + i * KT, i, first[i]);
            }
        }
        // stage k0 + AHEAD KT to its place; its pages were sent before the loads of stage k0, which are done
        auto ahead = [&]() __attribute__((always_inline)) {
            const int now = sent_pages(k0 + AHEAD * KT);
            send_pages(k0 + 2 * AHEAD * KT);
            if (k0 + AHEAD * KT < key1) {
                look_at(now, k0 + AHEAD * KT);
                issue(k0 + AHEAD * KT, (at + AHEAD) & (NS - 1), now);
            }
        };
        // the stage at hand has arrived once only the loads of the AHEAD - 1 after it (or later ones) are on their way
        auto begin = [&]() __attribute__((always_inline)) {
            if (AHEAD > 1 && k0 + (AHEAD - 1) * KT < key1)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NBLK % WR == 0 ? (AHEAD - 1) * (2 * LPW + PAGED) : 0) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if constexpr (!OWN) {
                __builtin_amdgcn_s_barrier();         // for every wave, and none works on the stage before any more
                asm volatile("" ::: "memory");
                ahead();
            }
        };
        auto end = [&]() __attribute__((always_inline)) {
            if constexpr (OWN) ahead();
            k0 += KT;
            at = (at + 1) & (NS - 1);
        };
        // stages that every row of the block sees whole, then (from an absent page on at the latest) the others
        if constexpr (ES == 2) {
            const int seen = PAGED ? min(past, key1) : row0 + 1;
            const int full_end = key0 + max(seen - key0, 0) / KT * KT;
            if constexpr (!PAGED) {
                while (k0 < full_end) {
                    begin();
                    full(std::integral_constant<int, 0>{});
                    end();
                    if (k0 < full_end) {
                        begin();
                        full(std::integral_constant<int, 1>{});
                        end();
                    }
                }
            } else {
                while (k0 < full_end && k0 + KT <= bad_from) {
                    begin();
                    if (OWN || k0 < wave_end) full(at);
                    end();
                }
            }
        }
        while (k0 < key1) {
            begin();
            for (int k = k0; k < min(k0 + KT, wave_end); k += 32)
                tile32(at * TILE + (k - k0) * RB, k, k + 32 > min(min(all_see, key1), bad_from));
            end();
        }

        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // no load into LDS outlives the unit (the pages sent last)

        // --- results -----------------------------------------------------------------------------------
        l += other_half(l);
        const ArgsPtr ar = args_again();
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;
        unsigned char* const dst = ar->out + (start + qtok) * ar->o_ts + qhead * ar->o_hs;
        const int64_t to = static_cast<int64_t>(slot) * BM + wave * 32 + lr;
        float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};     // 0 where the results are finite, else NaN
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) zero[i & 3] = __builtin_fmaf(o[d][i], 0.0f, zero[i & 3]);
        const bool off = __any((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.0f && l * 0.0f == 0.0f);   // results off, their sum is not
        if (wave0 + lr < nrow) {
            if (whole) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 v = {o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv};
                        const int dim = d * 32 + 8 * i + 4 * lh;
                        if constexpr (ES == 2)
                            *reinterpret_cast<bf16x4*>(dst + dim * 2) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                        else
                            *reinterpret_cast<f32x4*>(dst + dim * 4) = v;
                    }
            } else {
                if (lh == 0) {
                    ar->stat[2 * to] = m;
                    ar->stat[2 * to + 1] = l;
                }
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(ar->part + to * D + d * 32 + 8 * i + 4 * lh) =
                            f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            }
        }
        // An infinity or NaN among the values reaches every row that sees it, whatever its weight.  The products lose that
        // where a weight has become 0 (and makes NaN of an infinity) and where values were left out, so the visible values
        // that are not finite are added up alone, and where there are any their sum is the result.
        if (marred || off) {
            int ln = lane;                            // (nothing of this is worked out before the loops: registers)
            pin(ln);
#pragma unroll 1
            for (int d = 0; d < DT; ++d) {
                float sum[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
                bool all_nan = false;
#pragma unroll 1
                for (int k = off ? key0 : looked_at; k < wave_end && !all_nan; k += 64) {
                    auto value = [&](int key) __attribute__((always_inline)) -> const u32x4* {      // its 32 dims; null on an absent page
                        if constexpr (PAGED) {
                            const unsigned page = pages[key >> p.shift];
                            return page < static_cast<unsigned>(p.pages) ? reinterpret_cast<const u32x4*>(vbase + page_at(page, key) + d * 32 * ES) : nullptr;
                        } else {
                            return reinterpret_cast<const u32x4*>(vbase + key * p.v_ts + d * 32 * ES);
                        }
                    };
                    bool has = false;                 // a lane looks at a key
                    if (k + ln < wave_end) {
                        const u32x4* v = value(k + ln);
                        for (int i = 0; v && i < 2 * ES; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) has |= not_finite<ES>(v[i][e]) != 0;
                    }
                    for (uint64_t keys = __ballot(has); keys && !all_nan; keys &= keys - 1) {
                        const int key = k + static_cast<int>(__builtin_ctzll(keys));
                        const unsigned char* v = reinterpret_cast<const unsigned char*>(value(key));
                        all_nan = true;
                        const bool sees = visible(key) & 1;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int dim = 8 * (i / 4) + 4 * (ln >> 5) + i % 4;
                            const unsigned w = ES == 2 ? static_cast<unsigned>(*reinterpret_cast<const uint16_t*>(v + dim * 2)) << 16
                                                       : *reinterpret_cast<const unsigned*>(v + dim * ES);
                            if (sees && not_finite<4>(w)) sum[i] += __uint_as_float(w);
                            all_nan &= sum[i] != sum[i];
                        }
                        all_nan = __all(all_nan);
                    }
                }
                if (wave0 + lr < nrow)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (sum[i] == 0.0f) continue;
                        const int dim = d * 32 + 8 * (i / 4) + 4 * (ln >> 5) + i % 4;
                        if (whole)
                            reinterpret_cast<typename std::conditional<ES == 2, __bf16, float>::type*>(dst)[dim] = sum[i] * inv;
                        else
                            ar->part[to * D + dim] = sum[i];
                    }
            }
        }
        if constexpr (!PAGED) {
            return;
        } else {
            g += took;
            if (g >= gend) return;
            while (g - base >= sq.units * sq.nt) {    // (stages are left, so there is a sequence with some)
                base += sq.units * sq.nt;
                sq = seq_shape_of_block<KT, BM>(p, ++s);
            }
            if constexpr (!OWN) __syncthreads();      // every wave is done with the ring
        }
    }
}

// Partial sums of the units that attention_kernel's blocks cut, in block order: a wave takes a row, its lanes the
// parts' statistics, then D / 64 dims each (two for D = 32, half of the wave).
template <typename T, int D, int BM>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnParams p) {
    const CutUnit u = p.cuts[blockIdx.x];
    const int lane = threadIdx.x & 63;
    constexpr int PER = D >= 64 ? D / 64 + (D % 64 != 0) : 1, LANES = D / PER;      // dims a lane, lanes
    typedef float fv __attribute__((ext_vector_type(PER)));
    auto at = [&](int k) { return static_cast<int64_t>(2 * (u.first + k) + (k == 0)) * BM; };
    if (u.parts == 0) return;
    // `many` loads in flight: 16, or four where there are no more parts (a tree's tile of a sequence)
    auto join = [&](auto many) __attribute__((always_inline)) {
        for (int rr = blockIdx.y * 4 + (threadIdx.x >> 6); rr < u.rows; rr += gridDim.y * 4) {
            float top = kNoMax, sum = 0.0f;
            for (int k0 = 0; k0 < u.parts; k0 += 64)
                top = fmaxf(top, k0 + lane < u.parts ? p.stat[2 * (at(k0 + lane) + rr)] : kNoMax);
#pragma unroll
            for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i, 64));
            float acc[PER] = {};
            for (int k0 = 0; k0 < u.parts; k0 += 64) {
                float f = 0.0f;                           // this lane's part: its weight
                if (k0 + lane < u.parts) {
                    // (not 0: a part's infinity counts whatever its weight)
                    f = fmaxf(__builtin_amdgcn_exp2f(p.stat[2 * (at(k0 + lane) + rr)] - top), 0x1p-126f);
                    sum += p.stat[2 * (at(k0 + lane) + rr) + 1] * f;
                }
                const int n = min(64, u.parts - k0);
                for (int k = 0; k < n; k += many) {
                    fv v[many];
#pragma unroll
                    for (int i = 0; i < many; ++i)           // (past the last part: that one again, with weight 0)
                        if (lane < LANES) v[i] = *reinterpret_cast<const fv*>(p.part + (at(min(k0 + k + i, u.parts - 1)) + rr) * D + lane * PER);
#pragma unroll
                    for (int i = 0; i < many; ++i) {
                        const float w = __shfl(f, min(k + i, 63), 64);
#pragma unroll
                        for (int e = 0; e < PER; ++e) acc[e] += k + i < n ? v[i][e] * w : 0.0f;
                    }
                }
            }
#pragma unroll
            for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i, 64);
            const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            const int row = u.row0 + rr, tok = row / p.group, h = u.kvh * p.group + (row - tok * p.group);
            T* dst = reinterpret_cast<T*>(p.out + (u.start + tok) * p.o_ts + h * p.o_hs);
            if (lane < LANES)
#pragma unroll
                for (int e = 0; e < PER; ++e) dst[lane * PER + e] = static_cast<T>(acc[e] * inv);
        }
    };
    if (u.parts <= 4) join(std::integral_constant<int, 4>{}); else join(std::integral_constant<int, 16>{});
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
    int64_t units, nt;                 // (sequence, key head, row tile) triples at most, stages of each at most
    int64_t shared_bytes;              // the workspace of equal shares
};
// Stages in a block's ring: two, and four in 64-row blocks where they fill 64 KB (head dims of 256 bytes).  16 sequences of
// 4.5k tokens, 32 heads of 128 on 8, bf16: 16 drafted tokens 97 -> 92 us with four (of 64 dims: 53 -> 54), 48 (256-row
// blocks) 142 us with either.
constexpr int ring_of(int wr, int stage_bytes) { return wr == 2 && stage_bytes == 16384 ? 4 : 2; }
// Tiles hold a key head's query rows where 256 do, so that its keys are read once; small ones where few rows leave most of
// a tile idle.  The same sequences: single tokens 122 us in tiles of 32 rows and 131 of 64; 16 drafted tokens (64 rows) 92 us
// in 64 and 94 in 128; 32 (128 rows) 154 us in 64, 115 in 128, 110 in 256, so there are none of 128.
int tile_rows(int64_t rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 256; }
// Stages that equal shares must save to be taken: see plan_of.
int join_stages(const mopar_attention& a) { return a.dtype == MOPAR_BF16 ? 9 : 4; }
// Its tiles alone: n_seq below 2^31, at most 2^16 key heads and 2^15 row tiles, so the units fit 64 bits.
CachePlan tiles_of(const mopar_attention& a, int n_seq, int64_t rows, int max_len) {
    CachePlan c{};
    c.bm = tile_rows(rows);
    // 64 keys a stage in the large tiles in bf16: 32 of them cost 6 % (two tiles' scores for one rescale); float32 has not
    // the registers
    c.kt = a.dtype == MOPAR_BF16 && c.bm == 256 ? 64 : 32;
    c.row_tiles = static_cast<int>((rows + c.bm - 1) / c.bm);
    c.units = static_cast<int64_t>(n_seq) * a.kv_heads * c.row_tiles;
    c.nt = (static_cast<int64_t>(max_len) + c.kt - 1) / c.kt;
    return c;
}
// The whole plan, of tiles that attention_cache_fits has let pass.
CachePlan plan_of(const mopar_attention& a, int n_seq, int64_t rows, int max_len) {
    CachePlan c = tiles_of(a, n_seq, rows, max_len);
    // blocks that the card holds at once, by LDS and two waves a SIMD
    const int stage = 2 * c.kt * (a.head_dim > 64 ? 128 : a.head_dim) * static_cast<int>(dtype_size(a.dtype));
    const int64_t slots = 256 * std::min(256 / c.bm, 160 * 1024 / (ring_of(c.bm / 32, stage) * stage + c.bm / 32 * 1024));
    const int64_t units = c.units, nt = c.nt;
    // Equal shares, with partial sums and a second launch to join them, where they save more stages on the longest path
    // than the join costs: about 9 of bf16 (1 to 2 us each), 4 of float32 (3 us).  64 single tokens over 600: 42 us in
    // shares, 34 with a unit a block; 8 over 200: 14 and 13, over 400: 16 and 20; a float32 one over 100: 16 and 16,
    // over 200: 16 and 25; 16 drafts of 20 to 48 over 200 to 800: 47 and 34.
    const int64_t saved = nt * ((units + slots - 1) / slots) - (nt * units + slots - 1) / slots;
    c.split = saved > join_stages(a);
    c.blocks = static_cast<int>(std::min<int64_t>(c.split ? std::min(slots, units * nt) : units, int64_t(1) << 30));
    c.shared_bytes = std::min(slots, units * nt) * (int64_t(2) * c.bm * (a.head_dim + 2) * 4 + static_cast<int64_t>(sizeof(CutUnit)));
    return c;
}
int64_t query_rows(const mopar_attention& a, int max_q) { return static_cast<int64_t>(max_q) * (a.heads / a.kv_heads); }

}  // namespace

// A grid of a tile a block holds its threads, and stages are counted in 32 bits.
bool attention_cache_fits(const mopar_attention& a, int n_seq, int max_q, int max_len) {
    const CachePlan c = tiles_of(a, n_seq, query_rows(a, max_q), max_len);
    return c.units < 1 << 22 && c.units * c.nt < 1 << 30;
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
    p.max_rows = static_cast<int>(std::min<int64_t>(max_len, tokens));
    p.tokens = tokens;
    p.heads = a.heads;
    p.kv_heads = a.kv_heads;
    p.group = a.heads / a.kv_heads;
    p.c = a.scale * 1.44269504088896341f;
    // As many heads of a key head to a tile as its four waves take: the causal edge then meets every wave alike, and the
    // heads share their keys' loads.  16 prompts of 20 to 1100 tokens, 4 heads a key head: 151 -> 141 us (against one head
    // by 128 tokens), of 20 to 400 38 -> 31 us, one of 8192 the same.
    p.side = p.group % 4 == 0 ? 2 : p.group % 2 == 0 ? 1 : 0;
    const dim3 grid(static_cast<unsigned>(prompt_tiles(tokens, n_seq, max_len, 128 >> p.side) * (a.heads >> p.side)));
    return by_type(a.dtype, a.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        launch_kernel((attention_kernel<T, d, 4, sizeof(T) == 2 ? 2 : 1, 2, false>), grid, dim3(256), 0, s, p);
        return hipGetLastError();
    });
}

// What this call or one of fewer sequences, drafted tokens or keys may take (a smaller call may share where this one does
// not): none where there are no more stages than a join costs.
size_t attention_cache_ws_bytes(const mopar_attention& a, const mopar_cache& c, int64_t, int max_q, int max_len) {
    if ((static_cast<int64_t>(max_len) + 31) / 32 <= join_stages(a)) return 0;
    const int64_t rows = query_rows(a, max_q);
    int64_t most = plan_of(a, c.n_seq, rows, max_len).shared_bytes;
    for (int64_t r : {32, 64}) most = std::max(most, plan_of(a, c.n_seq, std::min(rows, r), max_len).shared_bytes);
    return static_cast<size_t>(most);
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
    p.shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));
    p.max_len = cache_limit(c, max_len);
    p.mask = mask;
    p.mask_words = mask_words;
    const CachePlan cp = plan_of(a, c.n_seq, query_rows(a, max_q), max_len);
    p.row_tiles = cp.row_tiles;
    p.split = cp.split;
    p.part = static_cast<float*>(ws);
    if (cp.split) {
        p.stat = p.part + int64_t(2) * cp.blocks * cp.bm * a.head_dim;
        p.cuts = reinterpret_cast<CutUnit*>(p.stat + int64_t(2) * cp.blocks * cp.bm * 2);
    }
    const dim3 grid(static_cast<unsigned>(cp.blocks));
    return by_type(a.dtype, a.head_dim, [&](auto t, auto d) {
        using T = decltype(t);
        auto go = [&](auto kernel, auto join, int threads) {
            launch_kernel(kernel, grid, dim3(threads), 0, s, p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess || !cp.split) return e;
            launch_kernel(join, dim3(grid.x, cp.bm / 8), dim3(256), 0, s, p);
            return hipGetLastError();
        };
        auto of = [&](auto wr) {
            constexpr int WR = wr, SUBS = sizeof(T) == 2 && WR == 8 ? 2 : 1, STAGE = 2 * 32 * SUBS * Geo<T, d>::RB;
            return go(attention_kernel<T, d, WR, SUBS, ring_of(WR, STAGE), true>, attention_join_kernel<T, d, WR * 32>, WR * 64);
        };
        if (cp.bm == 32) return of(std::integral_constant<int, 1>{});
        if (cp.bm == 64) return of(std::integral_constant<int, 2>{});
        return of(std::integral_constant<int, 8>{});
    });
}

}  // namespace mopar
