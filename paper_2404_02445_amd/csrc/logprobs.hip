// What logits say (gfx950): log probabilities of given tokens, their ranks, the entropy and the most likely alternatives.
//
// One pass over a row.  With z = scale (x - m) log2(e) and m a running maximum, S = sum 2^z and U = sum z 2^z give
//   ln sum exp = scale m + ln S,   entropy = ln 2 (log2 S - U / S);
// a lane keeps its own m and rescales S and U where it rises: 2^d S and 2^d (U + d S) for a rise of -d.
//
// The alternatives: the pass over a row also notes the largest logit of each piece of it, 64 elements or more.  The top-th largest of
// those is at most the top-th largest logit, so only the few pieces that reach it are looked at again.  There, keys that order as
// (logit, lowest index first) -- the float's bits made ascending in the upper word, the index's complement in the lower, so that
// no two are equal -- wait in LDS behind the largest that the wave has met until there are 16, and then every key's place is the
// number of larger ones.  In the end the waves' keys, and the blocks', find their places in the same way.
//
// What bounds it, measured (a copy reaches 5.16 TB/s): 2048 x 128000 in bf16, 524 MB, 98 us without alternatives (memory; some ten
// vector instructions a logit, of which the exponential counts four, keep the ALUs at two thirds), 119 with five (124 between other
// calls), 129 with 20: the pieces that are looked at again, when nothing is left to be streamed.  64 registers, for eight waves a
// SIMD: with 72 the 2048 blocks took two rounds of the card and 147 us.  (That bound holds in every form; those with alternatives keep three vector
// registers in scratch memory and 28 scalar ones in lanes for it, though few rows never have eight waves on a SIMD.)  257 x 32003 in float32 10.6 us: one row more than CUs (256
// rows 9.3).  4 x 128000 with 20 alternatives 14.4 us: two launches, two loads in a row, and six barriers.
// Tried without gain: keeping the list up to date along the row by bitonic sorts across lanes (4 x 128000 16.7, 2048 x 128000 138 us
// with five), by insertions one at a time (17.4, 145), loads a step ahead (168).
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.40282347e38f, kInf = __builtin_inff();
constexpr int kLogprobSplits = 32;                   // blocks that share a row at most
constexpr int kLogprobBlocks = 256;                  // blocks in all where rows are shared out

// A block's part of a row, or a row's: statistics, and the list that follows it in memory.
struct Part {
    float m, s, u;
    int rank;
};

struct LogprobParams {
    const unsigned char* x;
    int64_t stride;                                  // elements
    int vocab, top, splits, share;                   // share: elements of a block, a multiple of 64
    int fine, span, pieces;                          // the lanes (4 or 2) whose elements are a piece, or 0: so many steps of a wave; pieces of all waves
    float c, scale;                                  // scale log2(e), scale
    const int32_t* token;
    float *logprob, *entropy, *top_logprob;
    int32_t *rank, *top_id;
    Part* parts;                                     // [rows][splits]
    uint64_t* keys;                                  // [rows][splits][top]
};

__device__ __forceinline__ uint64_t key_of(float x, int at) {
    const unsigned b = __float_as_uint(x + 0.0f);    // (-0 as 0)
    const unsigned up = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
    return static_cast<uint64_t>(up) << 32 | (0xffffffffu - static_cast<unsigned>(at));
}
__device__ __forceinline__ float key_value(uint64_t k) {
    const unsigned up = static_cast<unsigned>(k >> 32);
    return __uint_as_float(up ^ (up >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int key_at(uint64_t k) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(k)); }

// The value of lane ^ D, without LDS: quads, halves of rows of 16, rows, halves of the wave.
template <int D> __device__ __forceinline__ unsigned xor_lane(unsigned v) {
    if constexpr (D == 1) return __builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true);                 // quad_perm 1 0 3 2
    if constexpr (D == 2) return __builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true);                 // quad_perm 2 3 0 1
    if constexpr (D == 3) return __builtin_amdgcn_mov_dpp(v, 0x1b, 0xf, 0xf, true);                 // quad_perm 3 2 1 0
    if constexpr (D == 4) return xor_lane<3>(xor_lane<7>(v));
    if constexpr (D == 7) return __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true);                // row_half_mirror
    if constexpr (D == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);                // row_ror:8
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);                        // odd rows of one with even rows of the other
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    if constexpr (D == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int D> __device__ __forceinline__ float xor_lane(float v) { return __uint_as_float(xor_lane<D>(__float_as_uint(v))); }
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }
// what the wave's lanes wrote to LDS is read by others of them
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// The place of k among n keys in LDS, from a multiple of 16 bytes on: how many are larger.  (Two keys a read.)
__device__ __forceinline__ int place_of(uint64_t k, const uint64_t* keys, int n) {
    int place = 0;
    const ulonglong2* const two = reinterpret_cast<const ulonglong2*>(keys);
#pragma unroll 8
    for (int j = 0; j < n / 2; ++j) {
        const ulonglong2 q = two[j];
        place += (q.x > k) + (q.y > k);
    }
    if (n & 1) place += keys[n - 1] > k;
    return place;
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, xor_lane<1>(v)), v = fmaxf(v, xor_lane<2>(v)), v = fmaxf(v, xor_lane<4>(v));
    return v = fmaxf(v, xor_lane<8>(v)), v = fmaxf(v, xor_lane<16>(v)), fmaxf(v, xor_lane<32>(v));
}
// The top-th largest of the lanes' values (no NaN).
__device__ __forceinline__ float nth_largest(float v, int top) {
    int larger = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) larger += lane_value(v, j) > v;
    float least = larger < top ? v : kInf;
    least = fminf(least, xor_lane<1>(least)), least = fminf(least, xor_lane<2>(least)), least = fminf(least, xor_lane<4>(least));
    least = fminf(least, xor_lane<8>(least)), least = fminf(least, xor_lane<16>(least)), least = fminf(least, xor_lane<32>(least));
    return least;
}

// z of a logit: scale log2(e) x less that of the maximum m.  The product of m is rounded, but to the same float everywhere, so
// that cancels; where it is large (and the rounding more than a part of an exponent), the difference goes first.
__device__ __forceinline__ bool large(float mc) { return !(fabsf(mc) < 65536.0f); }
__device__ __forceinline__ float exponent(float x, float m, float c) {
    const float mc = m * c;
    return large(mc) ? (x - m) * c : __builtin_fmaf(x, c, -mc);
}
// ... of a maximum m less that of a larger one, as their sums have them: how far sums rise; 2^-1000 and less is 0
__device__ __forceinline__ float rise(float m, float n, float c) {
#pragma clang fp contract(off)                       // (the products are rounded before they are subtracted, as in the sums)
    const float mc = m * c, nc = n * c;
    float d = mc - nc;
    if (large(mc)) d += __builtin_fmaf(m, c, -mc);
    if (large(nc)) d -= __builtin_fmaf(n, c, -nc);
    return fmaxf(fabsf(mc) < kInf && fabsf(nc) < kInf ? d : (m - n) * c, -1000.0f);
}
// Two sums with their maxima.
__device__ __forceinline__ void join(float& m, float& s, float& u, float m2, float s2, float u2, float c) {
    const float n = fmaxf(m, m2), d = rise(m, n, c), d2 = rise(m2, n, c);
    const float f = __builtin_amdgcn_exp2f(d), f2 = __builtin_amdgcn_exp2f(d2);
    u = f * (u + d * s) + f2 * (u2 + d2 * s2);
    s = f * s + f2 * s2;
    m = n;
}
// ... of the wave's lanes
__device__ __forceinline__ void join_lanes(float& m, float& s, float& u, int& rank, float c) {
    auto with = [&](auto d) __attribute__((always_inline)) {
        constexpr int D = decltype(d)::value;
        join(m, s, u, xor_lane<D>(m), xor_lane<D>(s), xor_lane<D>(u), c);
        rank += static_cast<int>(xor_lane<D>(static_cast<unsigned>(rank)));
    };
    using std::integral_constant;
    with(integral_constant<int, 32>{}), with(integral_constant<int, 16>{}), with(integral_constant<int, 8>{});
    with(integral_constant<int, 4>{}), with(integral_constant<int, 2>{}), with(integral_constant<int, 1>{});
}

// a row's results from its statistics and list (a key a lane)
__device__ __forceinline__ void finish(const LogprobParams& p, int64_t row, float xt, bool known, float m, float s, float u, int rank, uint64_t key,
                                       int lane) {
    const float log2s = __builtin_log2f(s);
    const bool nothing = s == 0.0f;                  // every logit is -infinity
    auto logprob = [&](float x) {
        const float z = exponent(x, m, p.c);
        // (z past float32, where the logarithm is nothing beside it: halves, whose difference is not)
        return nothing ? -kInf : z == -kInf ? (0.5f * x - 0.5f * m) * p.scale * 2.0f - log2s : (z - log2s) * 0.693147181f;
    };
    if (lane == 0) {
        p.logprob[row] = known ? logprob(xt) : -kInf;
        if (p.entropy) p.entropy[row] = nothing ? 0.0f : (log2s - u / s) * 0.693147181f;
        if (p.rank) p.rank[row] = known ? rank : p.vocab;
    }
    if (lane < p.top) {
        p.top_id[row * p.top + lane] = key ? key_at(key) : -1;
        p.top_logprob[row * p.top + lane] = key ? logprob(key_value(key)) : __builtin_nanf("");
    }
}

template <typename T> __device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
    if (n >= 8) {
        if constexpr (sizeof(T) == 2) {
            u32x4 r;
            __builtin_memcpy(&r, __builtin_assume_aligned(p, 2), 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(r[i] << 16), v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        } else {
            f32x4 r[2];
            __builtin_memcpy(&r, __builtin_assume_aligned(p, 4), 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r[i / 4][i % 4];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? static_cast<float>(p[i]) : -kInf;
    }
}

// One block of W waves a part of a row.  A wave's step is two groups of 512 elements, eight a lane.
template <typename T, bool TOP, int W>
__global__ __launch_bounds__(W * 64, 8) void logprob_kernel(const LogprobParams p) {
    constexpr int GROUPS = 2, STEP = W * 512 * GROUPS;
    __shared__ __attribute__((aligned(16))) uint64_t lists[W][128];               // a wave's list of at most top keys in descending order, and what waits behind it
    __shared__ __attribute__((aligned(16))) float pieces[W * 64];    // the largest logits of the waves' pieces
    __shared__ uint64_t best[64];
    __shared__ int remain;
    __shared__ Part sums[W];
    __shared__ unsigned least_piece;
    __shared__ unsigned long long bar;               // the highest of the waves' last keys: what is below it is in no list of the row
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / p.splits;
    const int split = blockIdx.x % p.splits;
    const int lo = split * p.share, hi = min(p.vocab, lo + p.share);
    const T* const x = reinterpret_cast<const T*>(p.x) + row * p.stride;
    const int tok = p.token[row];
    const bool known = tok >= 0 && tok < p.vocab;
    const float xt = known ? static_cast<float>(x[tok]) : kInf;
    const float c = p.c;
    if constexpr (TOP) {
        if (threadIdx.x == 0) bar = 0, remain = 0, least_piece = 0xffffffffu;
        if (threadIdx.x < 64) best[threadIdx.x] = 0;
        pieces[threadIdx.x] = -kInf;
        __syncthreads();
    }

    float m = kLowest, mc = kLowest, s = 0.0f, u = 0.0f;
    bool far = true;                                 // m times c is large
    int rank = 0;                                    // of the wave
    float v[GROUPS][8];
    auto load = [&](int at0) __attribute__((always_inline)) {
        const int at = at0 + lane * 8;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int n = hi - at - g * 512;
            load8(x + (n > 0 ? at + g * 512 : lo), n, v[g]);
        }
    };
    const int first = lo + wave * 512 * GROUPS;
    float piece_most = -kInf;
    int in_piece = 0, piece = 0, loaded = first;
    for (int at0 = first; at0 < hi; at0 += STEP) {
        load(at0);
        loaded = at0;
        float most = v[0][0], least = v[0][0];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, v[g][i]), least = fminf(least, v[g][i]);
        if (most > m) {
            const float d = rise(m, most, c), f = __builtin_amdgcn_exp2f(d);
            u = f * (u + d * s);
            s *= f;
            m = most;
            mc = m * c;
            far = large(mc);
        }
        if (__any(far || !(least * c > -1e30f))) {   // (weights of 0 times what is left of infinities would be NaN)
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = far ? (v[g][i] - m) * c : __builtin_fmaf(v[g][i], c, -mc), e = __builtin_amdgcn_exp2f(z);
                    s += e;
                    u = __builtin_fmaf(e, fmaxf(z, -200.0f), u);
                }
        } else {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = __builtin_fmaf(v[g][i], c, -mc), e = __builtin_amdgcn_exp2f(z);
                    s += e;
                    u = __builtin_fmaf(e, z, u);
                }
        }
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i) rank += __popcll(__ballot(v[g][i] > xt));
        if constexpr (TOP) {
            piece_most = fmaxf(piece_most, most);    // (fmaxf drops NaN)
            if (p.fine) {
                if (at0 + STEP < hi) continue;
                piece_most = fmaxf(piece_most, xor_lane<1>(piece_most));
                if (p.fine == 4) piece_most = fmaxf(piece_most, xor_lane<2>(piece_most));
                if ((lane & (p.fine - 1)) == 0) pieces[threadIdx.x / p.fine] = piece_most;
            } else if (++in_piece == p.span || at0 + STEP >= hi) {
                const float w = wave_max(piece_most);
                if (lane == 0) pieces[piece * W + wave] = w;
                piece_most = -kInf;
                in_piece = 0;
                ++piece;
            }
        }
    }
    if constexpr (TOP) {
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < p.pieces) {              // the top-th largest piece, -infinity where there are not so many
            const float mine = pieces[threadIdx.x];
            int larger = 0;
            for (int j = 0; j < p.pieces; j += 4) {                  // (W divides them: a multiple of four)
                const f32x4 q = *reinterpret_cast<const f32x4*>(pieces + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) larger += q[i] > mine;
            }
            if (larger < p.top) atomicMin(&least_piece, p.top > p.pieces ? 0x007fffffu : static_cast<unsigned>(key_of(mine, -1) >> 32));
        }
        __syncthreads();
    }
    // what joins the list has to be larger than last_x, or equal with an index below last_at; floor: the largest key known to end a list
    uint64_t* const list = lists[wave];
    float last_x = -kInf;
    int last_at = 0x7fffffff;
    uint64_t floor = 0;
    auto raise = [&](uint64_t k) __attribute__((always_inline)) {
        if (k <= floor) return;
        floor = k;
        const float w = key_value(k);
        if (w > last_x || (w == last_x && key_at(k) < last_at)) last_x = w, last_at = key_at(k);
    };
    int kept = 0, held = 0;                          // keys in the list; with those that wait
    auto take = [&]() __attribute__((always_inline)) {
        wave_sync();
        const uint64_t k0 = lane < held ? list[lane] : 0, k1 = lane + 64 < held ? list[lane + 64] : 0;
        const int p0 = place_of(k0, list, held), p1 = held > 64 ? place_of(k1, list, held) : 64;
        wave_sync();
        if (lane < held && p0 < p.top) list[p0] = k0;
        if (lane + 64 < held && p1 < p.top) list[p1] = k1;
        kept = held = min(held, p.top);
        wave_sync();
        if (kept == p.top) raise(list[p.top - 1]);
    };
    if constexpr (TOP) {
        last_x = key_value(static_cast<uint64_t>(least_piece) << 32);
        const bool reach = p.fine ? pieces[threadIdx.x / p.fine] >= last_x : lane < piece && pieces[lane * W + wave] >= last_x;
        const uint64_t reached = __ballot(reach);
        for (uint64_t todo = p.fine ? reached != 0 : reached; todo; todo &= todo - 1) {
            const int e = __builtin_ctzll(todo);
            for (int st = e * p.span; st < (e + 1) * p.span; ++st) {
                const int at0 = first + st * STEP;
                if (at0 >= hi) break;
                if (at0 != loaded) {
                    load(at0);
                    loaded = at0;
                }
                raise(__hip_atomic_load(&bar, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
                const int at = at0 + lane * 8;
                if (kept == 0 && last_x == -kInf) {  // the top-th largest of the lanes' maxima bounds the list, too
                    float most = -kInf;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                        for (int i = 0; i < 8; ++i) most = fmaxf(most, v[g][i]);
                    const float w = nth_largest(hi > at ? most : -kInf, p.top);
                    if (w > last_x) last_x = w;      // (last_at is as it was: equal ones join)
                }
                const uint64_t before = floor;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (!__any(v[g][i] >= last_x)) continue;
                        const int a = at + g * 512 + i;
                        auto joins = [&]() __attribute__((always_inline)) { return a < hi && (v[g][i] > last_x || (v[g][i] == last_x && a < last_at)); };
                        uint64_t in = __ballot(joins());
                        if (held + __popcll(in) > kept + 64) {
                            take();
                            in = __ballot(joins());
                        }
                        if ((in >> lane) & 1) list[held + __popcll(in & ((uint64_t(1) << lane) - 1))] = key_of(v[g][i], a);
                        held += __popcll(in);
                    }
                if (held > 32 && held >= kept + 16) take();
                if (floor > before && lane == 0) atomicMax(&bar, static_cast<unsigned long long>(floor));
            }
        }
        if (held > 64) take();                       // (fewer need no order among themselves)
    }
    int none = 0;
    join_lanes(m, s, u, none, c);
    if (lane == 0) sums[wave] = Part{m, s, u, rank};
    if constexpr (TOP) {
        // what is left of the waves' lists above the highest of their last keys, together, and its places
        wave_sync();
        if (lane == 0 && floor) atomicMax(&bar, static_cast<unsigned long long>(floor));
        const uint64_t k = lane < held ? list[lane] : 0;
        __syncthreads();
        const uint64_t in = __ballot(k != 0 && k >= bar);
        int at = 0;
        if (lane == 0 && in) at = atomicAdd(&remain, __popcll(in));
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(in & ((uint64_t(1) << lane) - 1));
        uint64_t* const all = lists[0];              // (64 keys of each wave at most)
        if ((in >> lane) & 1) all[at] = k;
        __syncthreads();
        const int n = remain;
        if (wave * 64 < n) {
            const int t = threadIdx.x;
            const uint64_t mine = t < n ? all[t] : 0;
            const int place = place_of(mine, all, n);
            if (t < n && place < p.top) best[place] = mine;
        }
    }
    __syncthreads();
    if (wave) return;
    const Part mine = lane < W ? sums[lane] : Part{kLowest, 0.0f, 0.0f, 0};
    m = mine.m, s = mine.s, u = mine.u, rank = mine.rank;
    join_lanes(m, s, u, rank, c);
    if (p.splits == 1) return finish(p, row, xt, known, m, s, u, rank, TOP ? best[lane] : 0, lane);
    const int64_t part = row * p.splits + split;
    if (lane == 0) p.parts[part] = Part{m, s, u, rank};
    if (lane < p.top) p.keys[part * p.top + lane] = best[lane];
}

// The parts of a row joined by a block.  The top-th largest of the first keys of all parts, 64 or a few more, bounds the row's list closely; what
// is not below it finds its place.
template <typename T>
__global__ __launch_bounds__(256) void logprob_join_kernel(const LogprobParams p) {
    __shared__ __attribute__((aligned(16))) uint64_t all[kLogprobSplits * 64];
    __shared__ uint64_t best[64];
    __shared__ unsigned long long bar;
    __shared__ int remain;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    const int tok = p.token[row];
    const uint64_t* const keys = p.keys + row * p.splits * p.top;
    const int total = p.splits * p.top;
    if (total) {
        const int each = min((64 + p.splits - 1) / p.splits, p.top), firsts = each * p.splits;      // (at most 64 + 32; top or more where there are)
        uint64_t k[kLogprobSplits * 64 / 256];
#pragma unroll
        for (int i = 0; i < kLogprobSplits * 64 / 256; ++i) k[i] = i * 256 + tid < total ? keys[i * 256 + tid] : 0;
        uint64_t first = 0;
        if (tid < firsts) all[tid] = first = keys[tid / each * p.top + tid % each];
        if (tid == 0) bar = 0, remain = 0;
        if (tid < 64) best[tid] = 0;
        __syncthreads();
        if (first && place_of(first, all, firsts) == p.top - 1) bar = first;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLogprobSplits * 64 / 256; ++i) {
            const uint64_t in = __ballot(k[i] != 0 && k[i] >= bar);
            if (!in) continue;
            int at = 0;
            if (lane == 0) at = atomicAdd(&remain, __popcll(in));
            at = __builtin_amdgcn_readfirstlane(at) + __popcll(in & ((uint64_t(1) << lane) - 1));
            if ((in >> lane) & 1) all[at] = k[i];
        }
        __syncthreads();
        const int n = remain;
        for (int t = tid; t < n; t += 256) {
            const uint64_t mine = all[t];
            const int place = place_of(mine, all, n);
            if (place < p.top) best[place] = mine;
        }
        __syncthreads();
    }
    if (tid >= 64) return;
    const bool known = tok >= 0 && tok < p.vocab;
    const float xt = known ? static_cast<float>(reinterpret_cast<const T*>(p.x)[row * p.stride + tok]) : kInf;
    const Part q = lane < p.splits ? p.parts[row * p.splits + lane] : Part{kLowest, 0.0f, 0.0f, 0};
    float m = q.m, s = q.s, u = q.u;
    int rank = q.rank;
    join_lanes(m, s, u, rank, p.c);
    finish(p, row, xt, known, m, s, u, rank, total ? best[lane] : 0, lane);
}

}  // namespace

// Blocks that share a row.  Few rows leave most CUs idle: with 20 alternatives of 128000 4 rows take 23.2 us whole and 14.4 shared out, 64
// rows 26.1 and 21.1, 128 rows 27.3 and 27.2 (without alternatives 16.7 and 14.0), 4 x 32000 14.1 either way, 64 x 32000 14.9 and 16.6: so up to 32
// rows are, in pieces of 4096 elements and more, and up to 128 long ones.
int logprob_splits(int64_t rows, int vocab) {
    if (rows > (vocab >= 65536 ? 128 : 32)) return 1;
    const int64_t idle = kLogprobBlocks / std::max<int64_t>(rows, 1);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({idle, (vocab + 4095) / 4096, kLogprobSplits})));
}

// The waves of a block.  One share of a row: four (4 x 128000 14.4 us, by eight 14.8), of long rows, of which each CU has one share, eight up to 8192
// elements and 16 past them (16 x 128000 17.1 by four, 15.0 by eight, 16.5 by 16, 32 rows 21.6, 17.9, 17.6).  Whole rows: four
// where they fill the card many times; 16 hold two rows a CU, so past 512 rows eight; and eight past 256 rows of up to 32768 elements, or up to 8192,
// where a wave of 16 has two steps and less.  Both sides of each border, bf16 without alternatives, us:
//   four and eight   1000 x 32000 20.6 and 19.4, 1024 20.7 and 19.7, 1200 22.9 and 24.9, 1500 25.6 and 28.1;
//                    1000 x 128000 51.8 and 45.4, 1024 52.4 and 45.7, 1200 67.7 and 65.9, 1500 77.1 and 79.9
//   eight and 16     512 x 128000 35.9 and 30.2, 513 38.2 and 39.9; 512 x 32003 11.9 and 13.3, 513 x 32000 13.2 and 15.4
//                    300 x 32003 11.3 and 12.8, 33000 11.3 and 12.4, 40000 12.5 and 12.7, 64000 17.0 and 16.8, 128000 34.1 and 27.7
//                    100 x 8000 4.8 and 5.1, 8200 5.3 and 5.4, 32000 8.9 and 7.7; 200 x 8000 5.3 and 5.3, 32000 9.2 and 8.1
// (so the borders at 1024 rows and 32768 elements lie somewhat low: up to 14 and 10 % for what is just past them).
static int logprob_waves(int64_t rows, int vocab, int splits, int share) {
    if (splits > 1) return rows <= 8 || vocab < 65536 ? 4 : share <= 8192 ? 8 : 16;
    if (rows >= 1024) return 4;
    return rows > 512 || vocab <= (rows > 256 ? 32768 : 8192) ? 8 : 16;
}

// (of as many rows as share at all: a size that does not fall as rows grow)
size_t logprob_ws_bytes(int64_t rows, int vocab, int top) {
    const int64_t splits = std::min<int64_t>((vocab + 4095) / 4096, kLogprobSplits);
    const int64_t parts = splits < 2 ? 0 : std::min<int64_t>(std::min<int64_t>(rows, 32) * splits, kLogprobBlocks);
    return static_cast<size_t>(parts) * (sizeof(Part) + 8 * static_cast<size_t>(top));
}

hipError_t launch_token_logprobs(const LogprobJob& j, int splits, void* ws, hipStream_t s) {
    LogprobParams p{};
    p.x = static_cast<const unsigned char*>(j.logits.data);
    p.stride = j.logits.stride;
    p.vocab = j.vocab;
    p.top = j.top;
    p.splits = splits;
    p.share = ((j.vocab + splits - 1) / splits + 63) / 64 * 64;
    p.c = j.scale * 1.44269504f;
    p.scale = j.scale;
    p.token = j.token;
    p.logprob = j.logprob, p.entropy = j.entropy, p.rank = j.rank;
    p.top_logprob = j.top_logprob, p.top_id = j.top_id;
    p.parts = static_cast<Part*>(ws);
    p.keys = reinterpret_cast<uint64_t*>(p.parts + j.rows * splits);
    const dim3 grid(static_cast<unsigned>(j.rows * splits));
    auto go = [&](auto t, auto w) {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        // pieces: of four or two lanes where a wave takes few steps, else of whole steps, at most 64 of a wave
        const int steps = (p.share + W * 1024 - 1) / (W * 1024);
        p.fine = steps > 4 ? 0 : j.top <= W * 8 ? 4 : 2;
        p.span = p.fine ? steps : (steps + 63) / 64;
        p.pieces = p.fine ? W * 64 / p.fine : (steps + p.span - 1) / p.span * W;
        if (j.top)
            launch_kernel((logprob_kernel<T, true, W>), grid, dim3(W * 64), 0, s, p);
        else
            launch_kernel((logprob_kernel<T, false, W>), grid, dim3(W * 64), 0, s, p);
        if (splits > 1) launch_kernel(logprob_join_kernel<T>, dim3(static_cast<unsigned>(j.rows)), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    auto types = [&](auto w) { return j.dtype == MOPAR_BF16 ? go(__bf16{}, w) : go(float{}, w); };
    switch (logprob_waves(j.rows, j.vocab, splits, p.share)) {
    case 4: return types(std::integral_constant<int, 4>{});
    case 8: return types(std::integral_constant<int, 8>{});
    default: return types(std::integral_constant<int, 16>{});
    }
}

}  // namespace mopar
