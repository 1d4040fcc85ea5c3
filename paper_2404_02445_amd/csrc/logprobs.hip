// What logits say (gfx950): log probabilities of given tokens, their ranks, the entropy and the most likely alternatives.
//
// One pass over a row.  With z = scale (x - m) log2(e) and m a running maximum, S = sum 2^z and U = sum z 2^z give
//   ln sum exp = scale m + ln S,   entropy = ln 2 (log2 S - U / S);
// a lane keeps its own m and rescales S and U where it rises: 2^d S and 2^d (U + d S) for a rise of -d.
//
// The alternatives are kept by each wave as a sorted list, one entry a lane, of keys that order as (logit, lowest index
// first): the float's bits made ascending in the upper word, the index's complement in the lower.  What may belong to the list is
// collected in LDS, 64 at a time, sorted across the lanes and merged; the list's last key keeps out nearly all of a row.
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.40282347e38f, kInf = __builtin_inff();
constexpr int kWaves = 4;                            // of a block
constexpr int kLogprobSplits = 32;                   // blocks that share a row at most

// A block's part of a row, or a row's: statistics, and the list that follows it in memory.
struct Part {
    float m, s, u;
    int rank;
};

struct LogprobParams {
    const unsigned char* x;
    int64_t stride;                                  // elements
    int vocab, top, splits, share;                   // share: elements of a block, a multiple of 512
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

__device__ __forceinline__ uint64_t other_lane(uint64_t k, int lane) {
    const int lo = __builtin_amdgcn_ds_bpermute(lane * 4, static_cast<int>(k)), hi = __builtin_amdgcn_ds_bpermute(lane * 4, static_cast<int>(k >> 32));
    return static_cast<uint64_t>(static_cast<unsigned>(hi)) << 32 | static_cast<unsigned>(lo);
}
// the larger or smaller of the lane's key and that of lane ^ d
__device__ __forceinline__ uint64_t choose(uint64_t k, int lane, int d, bool larger) {
    const uint64_t o = other_lane(k, lane ^ d);
    return (k > o) == larger ? k : o;
}
// 64 keys in descending order over the lanes
__device__ __forceinline__ uint64_t sorted(uint64_t k, int lane) {
#pragma unroll
    for (int n = 2; n <= 64; n *= 2)
#pragma unroll
        for (int d = n / 2; d; d /= 2) k = choose(k, lane, d, ((lane & n) == 0) == ((lane & d) == 0));
    return k;
}
// the 64 largest of two descending lists, descending
__device__ __forceinline__ uint64_t merged(uint64_t a, uint64_t b, int lane) {
    const uint64_t o = other_lane(b, 63 - lane);
    uint64_t k = a > o ? a : o;
#pragma unroll
    for (int d = 32; d; d /= 2) k = choose(k, lane, d, (lane & d) == 0);
    return k;
}

__device__ __forceinline__ void join(float& m, float& s, float& u, float m2, float s2, float u2, float c) {
    const float n = fmaxf(m, m2), d = fmaxf((m - n) * c, -1000.0f), d2 = fmaxf((m2 - n) * c, -1000.0f);
    const float f = __builtin_amdgcn_exp2f(d), f2 = __builtin_amdgcn_exp2f(d2);
    u = f * (u + d * s) + f2 * (u2 + d2 * s2);
    s = f * s + f2 * s2;
    m = n;
}

// a row's results from its statistics and list (a key a lane)
__device__ __forceinline__ void finish(const LogprobParams& p, int64_t row, float xt, bool known, float m, float s, float u, int rank, uint64_t key,
                                       int lane) {
    const float log2s = __builtin_log2f(s);
    const bool nothing = s == 0.0f;                  // every logit is -infinity
    auto logprob = [&](float x) { return nothing ? -kInf : (x - m) * p.scale - log2s * 0.693147181f; };
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

// One block a part of a row: a wave's step is 512 elements, eight a lane.
template <typename T, bool TOP>
__global__ __launch_bounds__(kWaves * 64) void logprob_kernel(const LogprobParams p) {
    __shared__ uint64_t found[kWaves][64];
    __shared__ uint64_t lists[kWaves][64];
    __shared__ Part sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / p.splits;
    const int split = blockIdx.x % p.splits;
    const int lo = split * p.share, hi = min(p.vocab, lo + p.share);
    const T* const x = reinterpret_cast<const T*>(p.x) + row * p.stride;
    const int tok = p.token[row];
    const bool known = tok >= 0 && tok < p.vocab;
    const float xt = known ? static_cast<float>(x[tok]) : kInf;
    const float c = p.c;

    float m = kLowest, s = 0.0f, u = 0.0f;
    int rank = 0;
    uint64_t list = 0, last = 0;                     // the wave's list; the key that what joins it has to pass
    int waiting = 0;                                 // keys in found
    auto take = [&]() __attribute__((always_inline)) {
        const uint64_t k = lane < waiting ? found[wave][lane] : 0;
        list = merged(list, sorted(k, lane), lane);
        last = other_lane(list, p.top - 1);
        waiting = 0;
    };
    for (int at = lo + wave * 512 + lane * 8; at - lane * 8 < hi; at += kWaves * 512) {      // (the same trips in every lane)
        float v[8];
        const int n = hi - at;
        load8(x + min(at, hi - 1), n, v);
        if (n <= 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = -kInf;
        }
        float most = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) most = fmaxf(most, v[i]);
        if (most > m) {
            const float d = fmaxf((m - most) * c, -1000.0f), f = __builtin_amdgcn_exp2f(d);
            u = f * (u + d * s);
            s *= f;
            m = most;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = (v[i] - m) * c, e = __builtin_amdgcn_exp2f(z);
            s += e;
            u = __builtin_fmaf(e, fmaxf(z, -200.0f), u);       // (0 where the weight is 0; NaN through e)
            rank += v[i] > xt;
        }
        if constexpr (TOP) {
            if (__any(most >= key_value(last) || last == 0)) {
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const float xi = i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : i == 3 ? v[3] : i == 4 ? v[4] : i == 5 ? v[5] : i == 6 ? v[6] : v[7];
                    const uint64_t k = key_of(xi, at + i);
                    const bool real = i < n && xi == xi;
                    uint64_t in = __ballot(real && k > last);
                    if (in == 0) continue;
                    if (waiting + __popcll(in) > 64) {
                        take();
                        in = __ballot(real && k > last);
                        if (in == 0) continue;
                    }
                    if (real && k > last) found[wave][waiting + __popcll(in & ((uint64_t(1) << lane) - 1))] = k;
                    waiting += __popcll(in);
                }
            }
        }
    }
    if constexpr (TOP) {
        if (waiting) take();
        lists[wave][lane] = list;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        join(m, s, u, __shfl_xor(m, o), __shfl_xor(s, o), __shfl_xor(u, o), c);
        rank += __shfl_xor(rank, o);
    }
    if (lane == 0) sums[wave] = Part{m, s, u, rank};
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        join(m, s, u, sums[w].m, sums[w].s, sums[w].u, c);
        rank += sums[w].rank;
        if constexpr (TOP) list = merged(list, lists[w][lane], lane);
    }
    if (p.splits == 1) return finish(p, row, xt, known, m, s, u, rank, list, lane);
    const int64_t part = row * p.splits + split;
    if (lane == 0) p.parts[part] = Part{m, s, u, rank};
    if (lane < p.top) p.keys[part * p.top + lane] = list;
}

// The parts of a row joined by a wave.
template <typename T>
__global__ __launch_bounds__(64) void logprob_join_kernel(const LogprobParams p) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int tok = p.token[row];
    const bool known = tok >= 0 && tok < p.vocab;
    const float xt = known ? static_cast<float>(reinterpret_cast<const T*>(p.x)[row * p.stride + tok]) : kInf;
    float m = kLowest, s = 0.0f, u = 0.0f;
    int rank = 0;
    if (lane < p.splits) {
        const Part q = p.parts[row * p.splits + lane];
        m = q.m, s = q.s, u = q.u, rank = q.rank;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        join(m, s, u, __shfl_xor(m, o), __shfl_xor(s, o), __shfl_xor(u, o), p.c);
        rank += __shfl_xor(rank, o);
    }
    uint64_t list = 0;
    if (p.top)
        for (int i = 0; i < p.splits; ++i) {
            const uint64_t k = lane < p.top ? p.keys[(row * p.splits + i) * p.top + lane] : 0;
            list = merged(list, k, lane);
        }
    finish(p, row, xt, known, m, s, u, rank, list, lane);
}

}  // namespace

// Blocks that share a row: while the rows alone leave CUs idle, shares of 4096 elements and more.
int logprob_splits(int64_t rows, int vocab) {
    const int64_t idle = 1024 / std::max<int64_t>(rows, 1);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({idle, vocab / 4096, kLogprobSplits})));
}

// (of as many rows as share at all: a size that does not fall as rows grow)
size_t logprob_ws_bytes(int64_t rows, int vocab, int top) {
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(vocab / 4096, kLogprobSplits));
    const int64_t parts = std::min<int64_t>(rows * splits, 1024);
    return static_cast<size_t>(parts) * (sizeof(Part) + 8 * static_cast<size_t>(top));
}

hipError_t launch_token_logprobs(const LogprobJob& j, int splits, void* ws, hipStream_t s) {
    LogprobParams p{};
    p.x = static_cast<const unsigned char*>(j.logits.data);
    p.stride = j.logits.stride;
    p.vocab = j.vocab;
    p.top = j.top;
    p.splits = splits;
    p.share = static_cast<int>((static_cast<int64_t>(j.vocab) + 512 * splits - 1) / (512 * splits) * 512);
    p.c = j.scale * 1.44269504f;
    p.scale = j.scale;
    p.token = j.token;
    p.logprob = j.logprob, p.entropy = j.entropy, p.rank = j.rank;
    p.top_logprob = j.top_logprob, p.top_id = j.top_id;
    p.parts = static_cast<Part*>(ws);
    p.keys = reinterpret_cast<uint64_t*>(p.parts + j.rows * splits);
    const dim3 grid(static_cast<unsigned>(j.rows * splits)), block(kWaves * 64);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (j.top)
            launch_kernel((logprob_kernel<T, true>), grid, block, 0, s, p);
        else
            launch_kernel((logprob_kernel<T, false>), grid, block, 0, s, p);
        if (splits > 1) launch_kernel(logprob_join_kernel<T>, dim3(static_cast<unsigned>(j.rows)), dim3(64), 0, s, p);
        return hipGetLastError();
    };
    return j.dtype == MOPAR_BF16 ? go(__bf16{}) : go(float{});
}

}  // namespace mopar
