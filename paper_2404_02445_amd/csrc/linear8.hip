// Products of 8-bit rows (gfx950): out[m][n] = (sum_k x[m][k] w[n][k]) sx[m] sw[n] + bias[n].
//
// Sums are int32 and exact, so the order and the cut of a sum are free: tiles, the waves' share of a stage and the
// blocks' share of a sum change no bit of a result.
//
// Operands come straight to LDS, 128 bytes of k a row and stage, eight rows (1 KB) a load instruction, whole lines where rows
// start at multiples of 128 bytes.  The weight fragment is the MFMA's first operand: a lane ends up with four neighbouring columns of
// one row.  Chunks past the sum read zeros; a chunk that the sum ends in is cut in the fragments of x.  Rows that start off 128-byte
// lines (by 16): 8192 x 4096 by 14336 columns 395 -> 410 us, 64 x 14336 by 4096 15.4 -> 21.1, 128 x 14336 by 4096 20.2 -> 29.4.
#pragma clang diagnostic ignored "-Winline-asm"      // (m0, which the loads into LDS take, is in no other use)
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

constexpr int kRsrcWord3 = 0x00020000;       // raw buffer, 32-bit data format
constexpr unsigned kOOB = 0x80000000u;       // a lane offset past every resource: reads zeros
constexpr int kCUs = 256;

struct Linear8Params {
    const int8_t *x, *w;
    const float *sx, *sw;
    const void* bias;
    void* out;
    int* partial;                // [splits][m][n], with splits > 1
    int64_t m, n, xs, ws, os;
    int k, splits;
    int mt, nt, total, per_xcd;  // tiles, those of all shares, and an XCD's
    int nk;                      // 128-byte steps of a wave's share, or of the sum
    // linear8_pair_kernel: tiles a block, and the divisors of the tiles' order
    int chunk;
    FastDiv div_group, div_last;
};

// Direct loads into LDS are inline asm, so that the compiler does not take every later read of LDS for a reader of theirs (it would
// wait for all loads in flight); they have no result in registers.  What they write is read after a counted wait and a
// barrier.  (Five wait states between a vector instruction's write of a scalar register and its use as a resource or offset.)
// in a scalar register (a step that the compiler knows is none that a load takes)
__device__ __forceinline__ unsigned opaque(unsigned v) {
    v = __builtin_amdgcn_readfirstlane(v);
    asm volatile("" : "+s"(v));
    return v;
}
__device__ __forceinline__ void load_lds(u32x4 rsrc, unsigned dst, unsigned voff, unsigned soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(opaque(dst)), "v"(voff), "s"(rsrc), "s"(opaque(soff))
                 : "memory", "m0");
}
__device__ __forceinline__ u32x4 resource(const int8_t* base) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);          // (the same in every lane)
    const unsigned lo = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(a)), hi = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(a >> 32));
    return u32x4{lo, hi & 0xffffu, 0x7fffffffu, kRsrcWord3};
}

// the first n bytes of a chunk (n < 16; none with n <= 0)
__device__ __forceinline__ u32x4 first_bytes(u32x4 v, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = n - 4 * i;
        v[i] &= b >= 4 ? 0xffffffffu : b <= 0 ? 0u : (1u << (8 * b)) - 1u;
    }
    return v;
}

template <typename T> __device__ __forceinline__ void load4(const T* p, int n, float (&v)[4]) {
    if (sizeof(T) == 4 && n >= 4) {
        f32x4 r;
        __builtin_memcpy(&r, __builtin_assume_aligned(p, 4), 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? static_cast<float>(p[i]) : 0.0f;
}
template <typename T> __device__ __forceinline__ void store4(T* p, int n, const float (&v)[4]) {
    if (n >= 4) {
        if constexpr (sizeof(T) == 2) {
            const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            __builtin_memcpy(__builtin_assume_aligned(p, 2), &o, 8);
        } else {
            const f32x4 o = {v[0], v[1], v[2], v[3]};
            __builtin_memcpy(__builtin_assume_aligned(p, 4), &o, 16);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) p[i] = static_cast<T>(v[i]);
}

__device__ __forceinline__ void store4(int* p, int n, const i32x4& v) {
    if (n >= 4) {
        __builtin_memcpy(__builtin_assume_aligned(p, 4), &v, 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) p[i] = v[i];
}

// Tile t of all: its share of the sum, and its place.  The eight XCDs take blocks round-robin: each gets a run of
// tiles, eight m tiles of one n tile after the other, so that the blocks it runs together share rows in its L2.
struct Place { int m0, n0, split; };
__device__ __forceinline__ bool place_of(const Linear8Params& p, int bm, int bn, Place& at) {
    const int t = static_cast<int>(blockIdx.x & 7) * p.per_xcd + static_cast<int>(blockIdx.x >> 3);
    if (static_cast<int>(blockIdx.x >> 3) >= p.per_xcd || t >= p.total) return false;
    const int tiles = p.mt * p.nt;
    at.split = t / tiles;
    const int in = t - at.split * tiles, group = in / (8 * p.nt), within = in - group * 8 * p.nt;
    const int gm = min(8, p.mt - group * 8), n = within / gm;
    at.n0 = n * bn;
    at.m0 = (group * 8 + (within - n * gm)) * bm;
    return true;
}

// ---------------------------------------------------------------------------
// Large products: 256 x 256 or 128 x 128 tiles on v_mfma_i32_32x32x32_i8, eight waves in two groups that take turns on
// the matrix units.
//
// Waves 0-3 (one a SIMD) own the upper half of the tile's rows, waves 4-7 the lower, each TILE / 2 x TILE / 4 results.
// A step of k is 128 bytes; with 256 x 256 tiles it is worked in two phases, the upper (A0) and the lower half (A1) of the wave's
// rows against all its columns.  A phase is a memory step (fragment reads, loads of later steps) and an MFMA step, with a
// barrier behind each, and the second group runs one step behind the first: while one wave of a SIMD multiplies, the other
// reads and loads.  256: two stages of 64 KB in LDS; A0 and the columns' halves (B) are read in the first phase and loaded again,
// for the step after next, in the second; A1 the other way round.  128: one phase, four stages of 32 KB, loads three steps
// ahead.  At the end of a memory step eight later loads stay in flight.  8192 x 4096 by 14336 columns take 395 to 410 us, 2.4 POP/s of
// the card's 5 (a library product 2.3); the matrix units are busy 68 % of the cycles, the rest is the steps' barriers and the tiles' ends.
//
// A block runs up to kPairTiles tiles, and the loads go on into the next one during the last steps of a tile.  The scales of a
// tile come to LDS with its first step, into the wave's own space, where its results turn at the end so that a store covers
// whole rows of the wave's part.
// ---------------------------------------------------------------------------
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
constexpr int kPairTiles = 4;

// the lane, worked out anew from here on: what a loop needs rarely is not kept in registers across it
__device__ __forceinline__ int lane_again(int lane) {
    asm volatile("" : "+v"(lane));
    return lane;
}
// one word a lane from its own address into word `lane` of dst
__device__ __forceinline__ void load_lds_word(const float* src, unsigned dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(opaque(dst)), "v"(src) : "memory", "m0");
}

template <int N, typename F, int I = 0> __device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, F, I + 1>(static_cast<F&&>(f));
    }
}

// WHOLE: every row of results is whole 16-byte groups on 16-byte addresses
template <typename T, int TILE, bool WHOLE>
__global__ __launch_bounds__(512, 2) void linear8_pair_kernel(const Linear8Params p) {
    constexpr int TM = TILE / 2, TN = TILE / 4;          // a wave's part
    constexpr int IA = TM / 32, NJ = TN / 32;            // its 32 x 32 tiles
    constexpr int HALVES = TILE / 128;                   // 128-row halves of an operand's stage
    constexpr unsigned HALF = 16384, STAGE = 2 * HALVES * HALF, RING = 131072;   // a stage holds A0 (A1) B0 (B1)
    constexpr unsigned OWN = 4096;                       // a wave's space: scales, then results
    __shared__ __attribute__((aligned(1024))) unsigned char lds[RING + 8 * OWN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3, lrow = lane & 31, lhalf = lane >> 5;
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<size_t>((lds_ptr_t)(&lds[0])));

    // --- the block's tiles: number first + 32 j of its XCD's run ---------------------------------
    const int t_lo = static_cast<int>(blockIdx.x & 7) * p.per_xcd, t_end = min(p.per_xcd, p.total - t_lo);
    const int li = static_cast<int>(blockIdx.x >> 3);
    int t_next = (li >> 5) * 32 * p.chunk + (li & 31);
    const int t_last = min(t_end, ((li >> 5) + 1) * 32 * p.chunk);
    struct Tile { int64_t m0, n0; };
    auto take = [&](Tile& tl) __attribute__((always_inline)) -> bool {
        if (t_next >= t_last) return false;
        const unsigned t = static_cast<unsigned>(t_lo + t_next);
        t_next += 32;
        const unsigned group = p.div_group.div(t), within = t - group * static_cast<unsigned>(8 * p.nt);
        const bool last = static_cast<int>(group) == (p.mt - 1) / 8;
        const unsigned gm = last ? static_cast<unsigned>(p.mt) - group * 8 : 8;
        const unsigned nti = last ? p.div_last.div(within) : within / 8;
        tl.n0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(nti))) * TILE;
        tl.m0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(group * 8 + (within - nti * gm)))) * TILE;
        return true;
    };
    Tile cur, ahead;
    if (!take(cur)) return;                              // (the whole block, before any barrier)
    ahead = cur;
    bool live = true;                                    // the loads still have a tile

    // --- operand loads -----------------------------------------------------------------------------
    // A half is 16 blocks of 1 KB (8 rows x 128 bytes); wave w loads blocks w and w + 8.  Chunk c of row r sits at place
    // c ^ (r % 8) ^ (bit 4 of r), which keeps the 32-row fragment reads off each other's banks.  Row r of A half i is tile row
    // TM (r / 64) + 64 i + r % 64, row r of B half j tile column TN (r / 32) + 32 j + r % 32.
    const int nk = p.nk, ktail = (p.k & 127) ? nk - 1 : nk;      // nk >= 2 (256) or 3 (128): see the launcher
    u32x4 va = {}, vb = {};                              // element 2 half + slot
    const int8_t *xb = nullptr, *wb = nullptr;           // of the tile that loads are at
    int ikt = 0;
    unsigned koff = 0, dst = lds0 + static_cast<unsigned>(wave) * 1024u;
    auto offsets = [&]() __attribute__((always_inline)) {
        xb = p.x + ahead.m0 * p.xs, wb = p.w + ahead.n0 * p.ws;
        const int mleft = static_cast<int>(min<int64_t>(p.m - 1 - ahead.m0, TILE - 1)), nleft = static_cast<int>(min<int64_t>(p.n - 1 - ahead.n0, TILE - 1));
        const int ln = lane_again(lane), cl = (ln & 7) ^ (ln >> 3) ^ ((wave >> 1) & 1);
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int r = (wave + 8 * s) * 8 + (ln >> 3);
                const int m = min((r >> 6) * TM + h * 64 + (r & 63), mleft), n = min((r >> 5) * TN + h * 32 + (r & 31), nleft);
                va[2 * h + s] = static_cast<unsigned>(m) * static_cast<unsigned>(p.xs) + static_cast<unsigned>(cl * 16);
                vb[2 * h + s] = static_cast<unsigned>(n) * static_cast<unsigned>(p.ws) + static_cast<unsigned>(cl * 16);
            }
    };
    auto load_a = [&](auto h) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) load_lds(resource(xb), dst + h * HALF + s * 8192, va[2 * h + s], koff);
    };
    auto load_b = [&](auto h) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) load_lds(resource(wb), dst + (HALVES + h) * HALF + s * 8192, vb[2 * h + s], koff);
    };
    // the loads go on to the next step: of the same tile, or the first of the block's next one
    unsigned ring = 0;
    auto load_next = [&]() __attribute__((always_inline)) {
        ring = (ring + STAGE) & (RING - 1);
        dst = lds0 + ring + static_cast<unsigned>(wave) * 1024u;
        koff += 128;
        ++ikt;
        if (ikt == nk) {
            ikt = 0;
            koff = 0;
            live = live && take(ahead);
            if (live) {
                offsets();
            } else {
                va = vb = u32x4{kOOB, kOOB, kOOB, kOOB};
            }
        } else if (ikt == ktail) {                       // chunks past the sum
            const int ln = lane_again(lane), cl = (ln & 7) ^ (ln >> 3) ^ ((wave >> 1) & 1);
            const unsigned past = ikt * 128 + cl * 16 >= p.k ? kOOB : 0u;
            va |= past, vb |= past;
        }
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, HALVES - 1>;
    offsets();
    if constexpr (TILE == 256) {                         // step 0, and step 1 but for A1
        load_b(I0{}), load_b(I1{}), load_a(I0{}), load_a(I1{});
        load_next();
        load_b(I0{}), load_b(I1{}), load_a(I0{});
    } else {                                             // steps 0, 1 and 2
#pragma unroll
        for (int u = 0; u < 3; ++u) {
            if (u) load_next();
            load_b(I0{}), load_a(I0{});
        }
    }
    // the scales of the wave's rows and columns to its own space: TM row scales, then at 512 TN column scales
    constexpr int SCALES = (TM + 63) / 64 + 1;
    const unsigned own = RING + static_cast<unsigned>(wave) * OWN;
    auto load_scales = [&]() __attribute__((always_inline)) {
        const int ln = lane_again(lane);
#pragma unroll
        for (int i = 0; i < SCALES - 1; ++i)
            load_lds_word(p.sx + min<int64_t>(cur.m0 + wm * TM + i * 64 + ln, p.m - 1), lds0 + own + i * 256);
        load_lds_word(p.sw + min<int64_t>(cur.n0 + wn * TN + ln, p.n - 1), lds0 + own + 512);
    };

    // --- fragments: lane's 16 bytes of 32 of k, row l % 32 of a 32-row tile, chunk 2 kk + l / 32 -----
    unsigned fa[4], fb[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const unsigned f = lds0 + (lrow >> 3) * 1024 + (lrow & 7) * 128 + (((2 * kk + lhalf) ^ (lrow & 7) ^ (lrow >> 4)) << 4);
        fa[kk] = f + wm * 8192;
        fb[kk] = f + wn * 4096;
    }
    u32x4 af[2][4], bf[NJ][4];
    i32x16 acc[HALVES][2][NJ];                           // [A half][row tile][column tile]
    unsigned roff = 0;                                   // the stage that fragments come from
    bool stored = false;                                 // a tile's stores, of a known number, are behind
    constexpr int STORES = WHOLE ? IA * NJ * (sizeof(T) == 4 ? 4 : 2) : 0;
    const int cut = p.k & 15 ? p.k >> 7 : -1;            // the step that a chunk is cut in
    int kt = 0;
    // The end of a memory step, whose reads are there: wait for the loads that the next memory step reads, the eight issued since staying in
    // flight (in a tile's first step the scales' loads and the stores of the tile before lie between them).  Then the MFMAs.
    auto mfma_step = [&](auto i, auto first) __attribute__((always_inline)) {
        if constexpr (decltype(first)::value) {
            if (WHOLE && stored)
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(8 + SCALES + STORES) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(8 + SCALES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        }
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (kt == cut) {
            const int left = p.k - kt * 128 - (lane_again(lane) >> 5) * 16;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int a = 0; a < 2; ++a) af[a][kk] = first_bytes(af[a][kk], left - kk * 32);
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    acc[i][a][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, bf[j][kk]), __builtin_bit_cast(i32x4, af[a][kk]),
                                                                         acc[i][a][j], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The reads and loads of a memory step, and the wait for the reads, in one piece of assembly: the compiler would not let
    // the reads go ahead of the loads' issue, which holds a wave for some 50 cycles each.
    auto step = [&](auto first) __attribute__((always_inline)) {
        unsigned a[4], b[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) a[kk] = fa[kk] + roff, b[kk] = fb[kk] + roff;
        if constexpr (TILE == 256) {
            const u32x4 rx1 = resource(xb);              // A1 of the step that load_next leaves
            const unsigned dst1 = dst + HALF, koff1 = opaque(koff), v0 = va[2 * HALVES - 2], v1 = va[2 * HALVES - 1];
            load_next();
            asm volatile(
                "ds_read_b128 %0, %16 offset:32768\n\tds_read_b128 %8, %20\n\tds_read_b128 %4, %16 offset:49152\n\tds_read_b128 %12, %20 offset:4096\n\t"
                "ds_read_b128 %1, %17 offset:32768\n\tds_read_b128 %9, %21\n\tds_read_b128 %5, %17 offset:49152\n\tds_read_b128 %13, %21 offset:4096\n\t"
                "ds_read_b128 %2, %18 offset:32768\n\tds_read_b128 %10, %22\n\tds_read_b128 %6, %18 offset:49152\n\tds_read_b128 %14, %22 offset:4096\n\t"
                "ds_read_b128 %3, %19 offset:32768\n\tds_read_b128 %11, %23\n\tds_read_b128 %7, %19 offset:49152\n\tds_read_b128 %15, %23 offset:4096\n\t"
                "s_mov_b32 m0, %24\n\ts_nop 0\n\tbuffer_load_dwordx4 %25, %27, %28 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %26, %27, %28 offen lds\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(bf[0][0]), "=&v"(bf[0][1]), "=&v"(bf[0][2]), "=&v"(bf[0][3]), "=&v"(bf[NJ - 1][0]), "=&v"(bf[NJ - 1][1]), "=&v"(bf[NJ - 1][2]),
                  "=&v"(bf[NJ - 1][3]), "=&v"(af[0][0]), "=&v"(af[0][1]), "=&v"(af[0][2]), "=&v"(af[0][3]), "=&v"(af[1][0]), "=&v"(af[1][1]),
                  "=&v"(af[1][2]), "=&v"(af[1][3])
                : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "s"(opaque(dst1)), "v"(v0), "v"(v1), "s"(rx1), "s"(koff1)
                : "memory", "m0", "scc");
            if constexpr (decltype(first)::value) load_scales();
            mfma_step(I0{}, first);
            const unsigned ko = opaque(koff);
            asm volatile(
                "ds_read_b128 %0, %8 offset:16384\n\tds_read_b128 %4, %8 offset:20480\n\tds_read_b128 %1, %9 offset:16384\n\tds_read_b128 %5, %9 offset:20480\n\t"
                "ds_read_b128 %2, %10 offset:16384\n\tds_read_b128 %6, %10 offset:20480\n\tds_read_b128 %3, %11 offset:16384\n\tds_read_b128 %7, %11 offset:20480\n\t"
                "s_add_u32 m0, %12, 32768\n\ts_nop 0\n\tbuffer_load_dwordx4 %13, %20, %21 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %14, %20, %21 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %15, %20, %21 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %16, %20, %21 offen lds\n\t"
                "s_mov_b32 m0, %12\n\ts_nop 0\n\tbuffer_load_dwordx4 %17, %19, %21 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %18, %19, %21 offen lds\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(af[0][0]), "=&v"(af[0][1]), "=&v"(af[0][2]), "=&v"(af[0][3]), "=&v"(af[1][0]), "=&v"(af[1][1]), "=&v"(af[1][2]), "=&v"(af[1][3])
                : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "s"(opaque(dst)), "v"(vb[0]), "v"(vb[1]), "v"(vb[2 * HALVES - 2]), "v"(vb[2 * HALVES - 1]), "v"(va[0]),
                  "v"(va[1]), "s"(resource(xb)), "s"(resource(wb)), "s"(ko)
                : "memory", "m0", "scc");
            roff ^= STAGE;
            mfma_step(I1{}, first);
        } else {
            load_next();
            const unsigned ko = opaque(koff);
            asm volatile(
                "ds_read_b128 %0, %12 offset:16384\n\tds_read_b128 %4, %16\n\tds_read_b128 %8, %16 offset:4096\n\t"
                "ds_read_b128 %1, %13 offset:16384\n\tds_read_b128 %5, %17\n\tds_read_b128 %9, %17 offset:4096\n\t"
                "ds_read_b128 %2, %14 offset:16384\n\tds_read_b128 %6, %18\n\tds_read_b128 %10, %18 offset:4096\n\t"
                "ds_read_b128 %3, %15 offset:16384\n\tds_read_b128 %7, %19\n\tds_read_b128 %11, %19 offset:4096\n\t"
                "s_add_u32 m0, %20, 16384\n\ts_nop 0\n\tbuffer_load_dwordx4 %21, %26, %27 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %22, %26, %27 offen lds\n\t"
                "s_mov_b32 m0, %20\n\ts_nop 0\n\tbuffer_load_dwordx4 %23, %25, %27 offen lds\n\t"
                "s_add_u32 m0, m0, 8192\n\ts_nop 0\n\tbuffer_load_dwordx4 %24, %25, %27 offen lds\n\t"
                "s_waitcnt lgkmcnt(0)"
                : "=&v"(bf[0][0]), "=&v"(bf[0][1]), "=&v"(bf[0][2]), "=&v"(bf[0][3]), "=&v"(af[0][0]), "=&v"(af[0][1]), "=&v"(af[0][2]), "=&v"(af[0][3]),
                  "=&v"(af[1][0]), "=&v"(af[1][1]), "=&v"(af[1][2]), "=&v"(af[1][3])
                : "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "s"(opaque(dst)), "v"(vb[0]), "v"(vb[1]), "v"(va[0]),
                  "v"(va[1]), "s"(resource(xb)), "s"(resource(wb)), "s"(ko)
                : "memory", "m0", "scc");
            if constexpr (decltype(first)::value) load_scales();
            roff = (roff + STAGE) & (RING - 1);
            mfma_step(I0{}, first);
        }
    };
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");     // what the first phase of step 0 reads
    __builtin_amdgcn_s_barrier();
    if (wave >= 4) __builtin_amdgcn_s_barrier();         // the second group runs one step behind
    asm volatile("" ::: "memory");
    for (;;) {
#pragma unroll
        for (int i = 0; i < HALVES; ++i)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][a][j][e] = 0;
        kt = 0;
        step(std::true_type{});
        for (kt = 1; kt < nk; ++kt) step(std::false_type{});
        // --- results: rows m0 + TM wm + 32 ia + l % 32, columns n0 + TN wn + 32 j + 8 g + 4 (l / 32) .. + 3 ------
        const int64_t mb = cur.m0 + wm * TM, nb = cur.n0 + wn * TN;
        const int ln = lane_again(lane), lrow = ln & 31, lhalf = ln >> 5;
        float sx[IA];
        f32x4 sw[NJ][4], bias[NJ][4];
#pragma unroll
        for (int ia = 0; ia < IA; ++ia) sx[ia] = *reinterpret_cast<const float*>(lds + own + (ia * 32 + lrow) * 4);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = j * 32 + g * 8 + lhalf * 4;
                sw[j][g] = *reinterpret_cast<const f32x4*>(lds + own + 512 + n * 4);
                bias[j][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (p.bias) {
                    float b[4];
                    load4(static_cast<const T*>(p.bias) + min(nb + n, p.n), static_cast<int>(max<int64_t>(min<int64_t>(p.n - nb - n, 4), 0)), b);
                    bias[j][g] = f32x4{b[0], b[1], b[2], b[3]};
                }
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // results turn in the wave's space, 32 rows at a time: CPR 16-byte chunks a row, chunk c of row r at place c ^ (r % CPR)
        constexpr int CPR = sizeof(T) == 4 ? 8 : TN * 2 / 16, ROWS = 64 / CPR, PASSES = sizeof(T) == 4 ? NJ : 1;
        constexpr int CC = 16 / sizeof(T);               // columns of a chunk
        const int sc = ln & (CPR - 1), sr = ln / CPR;
        const int64_t left_m = p.m - mb;
        const auto rs = __builtin_amdgcn_make_buffer_rsrc(static_cast<T*>(p.out) + mb * p.os + nb, static_cast<short>(0), 0x7fffffff, kRsrcWord3);
        static_for<IA>([&](auto ia) __attribute__((always_inline)) {
            static_for<PASSES>([&](auto pass) __attribute__((always_inline)) {
#pragma unroll
                for (int j = sizeof(T) == 4 ? pass : 0; j < (sizeof(T) == 4 ? pass + 1 : NJ); ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = static_cast<float>(acc[ia / 2][ia % 2][j][4 * g + e]) * sx[ia] * sw[j][g][e] + bias[j][g][e];
                        if constexpr (sizeof(T) == 4) {
                            const int c = 2 * g + lhalf;
                            *reinterpret_cast<f32x4*>(lds + own + (lrow * CPR + (c ^ (lrow & (CPR - 1)))) * 16) = v;
                        } else {
                            const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                            const int c = 4 * j + g;
                            *reinterpret_cast<bf16x4*>(lds + own + (lrow * CPR + (c ^ (lrow & (CPR - 1)))) * 16 + lhalf * 8) = o;
                        }
                    }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                const int col = pass * 32 + sc * CC;
                const int some = static_cast<int>(max<int64_t>(min<int64_t>(p.n - nb - col, CC), 0));
#pragma unroll
                for (int i = 0; i < 32 / ROWS; ++i) {
                    const int r = sr + i * ROWS, row = ia * 32 + r;
                    const u32x4 w = *reinterpret_cast<const u32x4*>(lds + own + (r * CPR + (sc ^ (r & (CPR - 1)))) * 16);
                    if constexpr (WHOLE) {               // what is not stored gets an offset past the results: every lane issues the same stores
                        const unsigned off = row < left_m && some == CC ? static_cast<unsigned>(row) * static_cast<unsigned>(p.os * sizeof(T)) + col * sizeof(T) : kOOB;
                        __builtin_amdgcn_raw_buffer_store_b128(w, rs, static_cast<int>(off), 0, 0);
                    } else if (row < left_m) {
                        T* const q = static_cast<T*>(p.out) + (mb + row) * p.os + nb + col;
                        if (some == CC) {
                            __builtin_memcpy(__builtin_assume_aligned(q, sizeof(T)), &w, 16);
                        } else {
#pragma unroll
                            for (int e = 0; e < CC; ++e)
                                if (e < some) {
                                    if constexpr (sizeof(T) == 4)
                                        reinterpret_cast<unsigned*>(q)[e] = w[e];
                                    else
                                        reinterpret_cast<unsigned short*>(q)[e] = static_cast<unsigned short>(w[e / 2] >> (16 * (e & 1)));
                                }
                        }
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            });
        });
        stored = WHOLE;
        if (!live) break;                                // (the loads have at least begun the next tile)
        cur = ahead;
    }
    if (wave < 4) __builtin_amdgcn_s_barrier();          // the second group's last step
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no load into LDS outlives the block
}

// ---------------------------------------------------------------------------
// Few tiles: a block of W waves takes 16 FM rows by 16 FN columns, and its waves share out the sum: what counts is that the
// operands are asked for early and in whole lines, and that no wave waits for another.  Each wave has a ring of NS stages of its
// own, 128 bytes of k of all the tile's rows and columns; the waves' sums meet in LDS at the end.  XL: 8-row loads of x a
// stage (rows past them are never stored).
//
// Up to 16 rows the weight's bytes bound it (1 x 4096 by 4096 columns 4.3 us, 5.8 with other weights in every call, by 28672 23.2: 5.1
// TB/s).  Past them about 3 us (launch, first loads, the waves' sums) and what a CU takes in by direct loads, 70 to 90 GB/s for all that its
// tiles read: by 4096 columns, sums of 4096 and 14336, 32 rows 5.3 and 12.5 us, 64 rows 6.7 and 15.4, 128 rows 7.9 and 20.2, 192 rows 9.5 and 24.4.
// Operands straight into registers took 38 us for 23 there, and 64 x 64 tiles of waves in step with each other 13.3 us for 8.5 at 128 x 4096.
// ---------------------------------------------------------------------------
template <typename T, int FM, int XL, int FN, int W, int NS>
__global__ __launch_bounds__(W * 64) void linear8_wave_kernel(const Linear8Params p) {
    constexpr int STAGE = (FM + FN) * 2048, L = XL + 2 * FN, RING = NS * STAGE;
    static_assert(FM * FN * 1024 <= RING && W * RING <= 163840, "the sums take the place of the rings");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[W * RING];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place at;
    if (!place_of(p, 16 * FM, 16 * FN, at)) return;                       // (the whole block)
    const int lo = (at.split * W + wave) * p.nk * 128, hi = min(p.k, lo + p.nk * 128);   // the wave's part of the sum
    const int nk = hi > lo ? (hi - lo + 127) >> 7 : 0;
    // loads: row l / 8 of eight, chunk (l % 8) ^ row
    const u32x4 rx = resource(p.x + at.m0 * p.xs + lo), rw = resource(p.w + at.n0 * p.ws + lo);
    const int cl = (lane & 7) ^ (lane >> 3);
    unsigned ox[XL], ow[2 * FN];
#pragma unroll
    for (int i = 0; i < XL; ++i) ox[i] = static_cast<unsigned>(min<int64_t>(i * 8 + (lane >> 3), p.m - 1 - at.m0)) * static_cast<unsigned>(p.xs) + cl * 16;
#pragma unroll
    for (int i = 0; i < 2 * FN; ++i)
        ow[i] = static_cast<unsigned>(min<int64_t>(i * 8 + (lane >> 3), p.n - 1 - at.n0)) * static_cast<unsigned>(p.ws) + cl * 16;
    const unsigned mine = static_cast<unsigned>(reinterpret_cast<size_t>((lds_ptr_t)(&lds[0]))) + wave * RING;
    unsigned slot = 0;
    auto load_stage = [&](int kt) __attribute__((always_inline)) {
        const unsigned past = kt >= nk || kt * 128 + cl * 16 >= hi - lo ? kOOB : 0u;
#pragma unroll
        for (int i = 0; i < 2 * FN; ++i) load_lds(rw, mine + slot + (FM * 2 + i) * 1024, ow[i] | past, kt * 128);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_lds(rx, mine + slot + i * 1024, ox[i] | past, kt * 128);
        slot = slot + STAGE == RING ? 0 : slot + STAGE;
    };
    i32x4 acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
    if (nk > 0) {
#pragma unroll
        for (int i = 0; i < NS; ++i) load_stage(i);
    }
    const int cut = (hi - lo) & 15 ? (hi - lo) >> 7 : -1;                 // the step that a chunk is cut in
    unsigned from = 0;
    for (int kt = 0; kt < nk; ++kt) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * L) : "memory");
        const unsigned char* const st = lds + wave * RING + from;
        from = from + STAGE == RING ? 0 : from + STAGE;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int c = 4 * kk + (lane >> 4), place = (c ^ (lane & 7)) * 16, r = (lane & 15) * 128;
            u32x4 xf[FM], wf[FN];
#pragma unroll
            for (int b = 0; b < FN; ++b) wf[b] = *reinterpret_cast<const u32x4*>(st + (FM + b) * 2048 + r + place);
#pragma unroll
            for (int a = 0; a < FM; ++a) xf[a] = *reinterpret_cast<const u32x4*>(st + a * 2048 + r + place);
            if (kt == cut) {
#pragma unroll
                for (int a = 0; a < FM; ++a) xf[a] = first_bytes(xf[a], hi - lo - kt * 128 - c * 16);
            }
#pragma unroll
            for (int a = 0; a < FM; ++a)
#pragma unroll
                for (int b = 0; b < FN; ++b)
                    acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[b]), __builtin_bit_cast(i32x4, xf[a]), acc[a][b], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                 // the stage is read: it can be loaded again
        load_stage(kt + NS);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                       // no load into LDS outlives the loop
    __syncthreads();
    i32x4* const sums = reinterpret_cast<i32x4*>(lds);                     // [W][FM][FN][64]
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) sums[((wave * FM + a) * FN + b) * 64 + lane] = acc[a][b];
    __syncthreads();
    for (int t = threadIdx.x; t < FM * FN * 64; t += W * 64) {
        const int l = t & 63, b = (t >> 6) % FN, a = (t >> 6) / FN;
        const int64_t m = at.m0 + a * 16 + (l & 15), n = at.n0 + b * 16 + (l >> 4) * 4;
        const int some = static_cast<int>(min<int64_t>(p.n - n, 4));
        if (m >= p.m || some <= 0) continue;
        i32x4 s = sums[t];
#pragma unroll
        for (int w = 1; w < W; ++w) s += sums[w * FM * FN * 64 + t];
        if (p.splits > 1) {
            store4(p.partial + (at.split * p.m + m) * p.n + n, some, s);
            continue;
        }
        float sw[4], bias[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4];
        load4(p.sw + n, some, sw);
        if (p.bias) load4(static_cast<const T*>(p.bias) + n, some, bias);
        const float sx = p.sx[m];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(s[i]) * sx * sw[i] + bias[i];
        store4(static_cast<T*>(p.out) + m * p.os + n, some, v);
    }
}

// The shares of a sum added up: a thread takes four columns of a row.  Bound by its launch (2 us), as the partial sums fit the caches.
template <typename T>
__global__ __launch_bounds__(256) void linear8_join_kernel(const Linear8Params p) {
    const int64_t groups = (p.n + 3) / 4, t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t m = t / groups, n = (t - m * groups) * 4;
    if (m >= p.m) return;
    const int some = static_cast<int>(min<int64_t>(p.n - n, 4));
    i32x4 sum = {0, 0, 0, 0};
    const int* q = p.partial + m * p.n + n;
    if (some >= 4) {
        for (int s = 0; s < p.splits; ++s, q += p.m * p.n) {
            i32x4 part;
            __builtin_memcpy(&part, __builtin_assume_aligned(q, 4), 16);
            sum += part;
        }
    } else {
        for (int s = 0; s < p.splits; ++s, q += p.m * p.n)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += i < some ? q[i] : 0;
    }
    float sw[4], bias[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4];
    load4(p.sw + n, some, sw);
    if (p.bias) load4(static_cast<const T*>(p.bias) + n, some, bias);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(sum[i]) * p.sx[m] * sw[i] + bias[i];
    store4(static_cast<T*>(p.out) + m * p.os + n, some, v);
}

}  // namespace

// Tile edge of linear8_pair_kernel for a product, 0 where linear8_wave_kernel runs it: its tiles have to fill the CUs.  Sums of
// 4096 in us: 128 tiles take 31.2 for 96 rows by 28672 columns (224 tiles), the others 41.7, 22.0 and 28.1 for 512 by 6144 (192 tiles), 20.8 and
// 16.4 for 192 by 6144 (96); 256 tiles 60.5 for 512 by 28672 (224 tiles), 128 tiles 87.8.  64 rows by 28672: 30.6 and 30.9.
// Sums up to 256, of fewer steps than the 128 tiles load ahead, go to the other form whatever their tiles: it shares out a sum among waves of which most
// then have none, and stores 8 bytes a lane.  8192 by 4096 in bf16, sums of 16 to 256 75 to 79 us (13 to 14 for the results' bytes),
// sums of 272 24 in 256 tiles and 82 in the others; 1024 by 4096, 256 and 272, 12.0 and 7.5.
static int pair_tile(int64_t m, int64_t n, int k) {
    if (k <= 256 || m <= 64) return 0;
    const int64_t tiles = (m + 255) / 256 * ((n + 255) / 256), rounds = (tiles + kCUs - 1) / kCUs;
    const int64_t small = (m + 127) / 128 * ((n + 127) / 128), srounds = (small + kCUs - 1) / kCUs;
    if (rounds == 1 ? tiles >= 140 : tiles * 10 >= rounds * kCUs * 6) return 256;
    return small >= 140 && small * 10 >= srounds * kCUs * 6 ? 128 : 0;
}

constexpr int kLongShare = 512 << 10, kShortShare = 128 << 10;     // operand bytes of a tile: shared out from here, and down to here
constexpr int kMostSplits = 8;

// Partial sums of blocks that fill the CUs once; a size that does not fall as a product grows.
size_t linear8_ws_bytes(int64_t m, int64_t n, int k) {
    if (k < kLongShare / 128 || m == 0 || n == 0) return 0;
    constexpr int64_t most = int64_t(kCUs) * 64 * 64;               // results of all blocks
    return static_cast<size_t>(m >= most / n ? most : std::min(most, m * n * kMostSplits)) * 4;
}

// Few rows: the fewest rows and columns a block that leave no CU two of them; more stages where a CU has one block.  In us, sums of 4096: one row
// by 28672 columns 23.2 with two stages, 24.2 with four, 1 x 14336 by 4096 14.7 and 12.0; 32 rows by 4096, 6144 and 28672 5.8, 8.2 and 34.9
// in blocks of 32 x 16, 6.5, 7.1 and 27.7 in 32 x 32.  64 rows by 4096: 32 x 32 7.3, 64 x 32 8.5, 64 x 64 10.5; 128 rows 11.7, 8.5, 10.5;
// 192 rows by 4096 (192 blocks of 64 x 64) 10.6 with eight waves, 13.6 with four, by 6144 (288) 19.1 and 16.8.
// Shares of a sum: 64 x 14336 by 1024 columns 13.1 whole, 11.0 in four, 1 x 28672 by 512 12.8 and 8.9; below kLongShare the join costs
// more than it gives (64 x 4096 by 1024 6.9 and 8.9, 1 x 14336 by 1024 8.2 and 8.3).
Linear8Plan linear8_plan(int64_t m, int64_t n, int k, size_t ws_bytes) {
    auto tiles = [&](int bm, int bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); };
    Linear8Plan plan{64, 64, 4, 1, 1};
    if (const int pair = pair_tile(m, n, k)) {
        plan = {pair, pair, 0, 0, 1};
    } else if (m <= 16 && n <= 1 << 25) {
        plan = {m <= 8 ? 8 : 16, 16, 4, tiles(16, 16) <= kCUs ? 4 : 2, 1};
    } else if (m <= 32 && n <= 1 << 25) {
        plan = tiles(32, 16) <= kCUs ? Linear8Plan{32, 16, 4, 3, 1} : Linear8Plan{32, 32, 4, 2, 1};
    } else if (tiles(32, 32) <= kCUs) {
        plan = {32, 32, 8, 2, 1};
    } else if (tiles(64, 32) <= kCUs) {
        plan = {64, 32, 8, 1, 1};
    } else if (tiles(64, 64) <= kCUs) {
        plan = {64, 64, 8, 1, 1};
    }
    const int64_t blocks = tiles(plan.bm, plan.bn), bytes = int64_t(plan.bm + plan.bn) * k;
    if (plan.waves && blocks <= kCUs / 2 && bytes >= kLongShare) {
        const int64_t fit = static_cast<int64_t>(ws_bytes / 4) / (m * n);
        plan.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kCUs / blocks, bytes / kShortShare, kMostSplits, fit})));
    }
    return plan;
}

hipError_t launch_linear8(int dtype, int64_t m, int64_t n, int k, const mopar_rows8& x, const mopar_rows8& w, const void* bias,
                          const mopar_matrix& out, void* ws, const Linear8Plan& plan, hipStream_t s) {
    const int tile_m = plan.bm == 8 ? 16 : plan.bm;
    Linear8Params p{};
    p.x = x.q, p.w = w.q, p.sx = x.scale, p.sw = w.scale;
    p.bias = bias;
    p.out = out.data;
    p.partial = static_cast<int*>(ws);
    p.m = m, p.n = n, p.k = k;
    p.xs = x.stride, p.ws = w.stride, p.os = out.stride;
    p.splits = plan.splits;
    p.mt = static_cast<int>((m + tile_m - 1) / tile_m);
    p.nt = static_cast<int>((n + plan.bn - 1) / plan.bn);
    p.total = p.mt * p.nt * p.splits;
    p.per_xcd = (p.total + 7) / 8;
    const int steps = (k + 127) / 128, waves = std::max(plan.waves, 1) * plan.splits;
    p.nk = (steps + waves - 1) / waves;
    auto pair = [&](auto t, auto tile) {
        using T = decltype(t);
        constexpr int TILE = decltype(tile)::value;
        p.div_group = FastDiv(static_cast<unsigned>(8 * p.nt));
        p.div_last = FastDiv(static_cast<unsigned>(p.mt - (p.mt - 1) / 8 * 8));
        p.chunk = std::min((p.per_xcd + 31) / 32, kPairTiles);
        const int per = 32 * p.chunk;
        const dim3 blocks(static_cast<unsigned>((p.per_xcd + per - 1) / per * 32 * 8));
        // (the results of a tile are addressed with 32 bits there)
        const int64_t es = sizeof(T);
        if (n * es % 16 == 0 && p.os * es % 16 == 0 && reinterpret_cast<uintptr_t>(p.out) % 16 == 0 && p.os * es < (int64_t(1) << 23))
            launch_kernel((linear8_pair_kernel<T, TILE, true>), blocks, dim3(512), 0, s, p);
        else
            launch_kernel((linear8_pair_kernel<T, TILE, false>), blocks, dim3(512), 0, s, p);
        return hipGetLastError();
    };
    auto go = [&](auto t) {
        using T = decltype(t);
        using std::integral_constant;
        if (!plan.waves) return plan.bm == 256 ? pair(t, integral_constant<int, 256>{}) : pair(t, integral_constant<int, 128>{});
        bool found = false;
        auto form = [&](auto bm, auto bn, auto wv, auto st) {
            constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value, W = decltype(wv)::value, NS = decltype(st)::value;
            if (plan.bm != BM || plan.bn != BN || plan.waves != W || plan.stages != NS) return;
            found = true;
            launch_kernel((linear8_wave_kernel<T, (BM + 15) / 16, BM / 8, BN / 16, W, NS>), dim3(static_cast<unsigned>(p.per_xcd) * 8), dim3(W * 64), 0, s, p);
        };
        integral_constant<int, 1> one;
        integral_constant<int, 2> two;
        integral_constant<int, 3> three;
        integral_constant<int, 4> four;
        integral_constant<int, 8> eight;
        integral_constant<int, 16> r16;
        integral_constant<int, 32> r32;
        integral_constant<int, 64> r64;
        form(eight, r16, four, two), form(eight, r16, four, four), form(r16, r16, four, two), form(r16, r16, four, four);
        form(r32, r16, four, three), form(r32, r32, four, two), form(r32, r32, eight, two);
        form(r64, r32, eight, one), form(r64, r64, eight, one), form(r64, r64, four, one);
        if (!found) return hipErrorInvalidValue;
        if (p.splits > 1) {
            const int64_t threads = m * ((n + 3) / 4);
            launch_kernel(linear8_join_kernel<T>, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s, p);
        }
        return hipGetLastError();
    };
    return dtype == MOPAR_BF16 ? go(__bf16{}) : go(float{});
}

}  // namespace mopar
