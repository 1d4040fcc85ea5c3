// Products of 8-bit rows (gfx950): out[m][n] = (sum_k x[m][k] w[n][k]) sx[m] sw[n] + bias[n].
//
// Sums are int32 and exact, so the order and the cut of a sum are free: tiles, the waves' share of a stage and the
// blocks' share of a sum change no bit of a result.
//
// linear8_kernel: a BM x BN tile of results by WM x WN waves on v_mfma_i32_16x16x64_i8, the weight fragment first: a lane ends
// up with four neighbouring columns of one row.  Operands come straight to LDS, 128 bytes of k a row and stage, eight
// rows (1 KB) a load instruction; chunk c of row r sits at place c ^ (r % 8), which keeps the fragment reads (16 rows, one
// chunk each) off each other's banks.  Chunks past the sum read zeros; a chunk that the sum ends in is cut in
// the fragments of x.
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
constexpr size_t kMostPartial = size_t(64) << 20;
constexpr int kMostSplits = 16;

struct Linear8Params {
    const int8_t *x, *w;
    const float *sx, *sw;
    const void* bias;
    void* out;
    int* partial;                // [splits][m][n], with splits > 1
    int64_t m, n, xs, ws, os;
    int k, splits;
    int mt, nt, total, per_xcd;  // tiles, those of all shares, and an XCD's
    int nk;                      // 128-byte steps of a share
};

// Direct loads into LDS are inline asm, so that the compiler does not take every later read of LDS for a reader of theirs (it would
// wait for all loads in flight); they have no result in registers.  What they write is read after a counted wait and a
// barrier.  (Five wait states between a vector instruction's write of a scalar register and its use as a resource or offset.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(u32x4 rsrc, unsigned dst, unsigned voff, unsigned soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(dst), "v"(voff), "s"(rsrc), "s"(soff)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ u32x4 resource(const int8_t* base) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    return u32x4{static_cast<unsigned>(a), static_cast<unsigned>(a >> 32) & 0xffffu, 0x7fffffffu, kRsrcWord3};
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

template <typename T, int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(WM * WN * 64) void linear8_kernel(const Linear8Params p) {
    constexpr int W = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    constexpr int STAGE = (BM + BN) * 128, L = (BM + BN) / 8 / W;          // bytes; loads a wave and stage
    static_assert((BM + BN) / 8 % W == 0 && BM / 8 % W == 0, "a wave's loads are all of x or all of w");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NS * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    Place at;
    if (!place_of(p, BM, BN, at)) return;                                 // (the whole block)
    const int k_lo = at.split * p.nk * 128, nk = min(p.nk, (p.k - k_lo + 127) / 128);   // (at least 1: see the launcher)

    // this wave's loads: 1 KB blocks wave, wave + W, ... of the stage's rows, x before w; lane l chunk (l % 8) ^ row
    const u32x4 rx = resource(p.x + at.m0 * p.xs + k_lo), rw = resource(p.w + at.n0 * p.ws + k_lo);
    const int cl = (lane & 7) ^ (lane >> 3);
    unsigned off[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int r = (wave + W * i) * 8 + (lane >> 3);
        const bool of_x = i < BM / 8 / W;
        const int row = of_x ? static_cast<int>(min<int64_t>(r, p.m - 1 - at.m0)) : static_cast<int>(min<int64_t>(r - BM, p.n - 1 - at.n0));
        off[i] = static_cast<unsigned>(row) * static_cast<unsigned>(of_x ? p.xs : p.ws) + static_cast<unsigned>(cl * 16);
    }
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<size_t>((lds_ptr_t)(&lds[0])));
    unsigned slot = 0;
    auto load_stage = [&](int kt) __attribute__((always_inline)) {
        const bool past = kt >= nk || k_lo + kt * 128 + cl * 16 >= p.k;
#pragma unroll
        for (int i = 0; i < L; ++i)
            load_lds(i < BM / 8 / W ? rx : rw, lds0 + slot * STAGE + (wave + W * i) * 1024, past ? kOOB : off[i], kt * 128);
        slot = slot + 1 == NS ? 0 : slot + 1;
    };
    i32x4 acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) load_stage(i);
    unsigned from = 0;
    const int cut = p.k & 15 ? (p.k - k_lo) >> 7 : -1;                    // the step that a chunk is cut in
    for (int kt = 0; kt < nk; ++kt) {
        // this wave's loads of the stage are there, and its reads of the one before; then everyone's
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * L) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load_stage(kt + NS - 1);
        const unsigned char* const st = lds + from * STAGE;
        from = from + 1 == NS ? 0 : from + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int c = 4 * kk + (lane >> 4), place = (c ^ (lane & 7)) * 16, r = lane & 15;
            u32x4 xf[FM], wf[FN];
#pragma unroll
            for (int a = 0; a < FM; ++a) xf[a] = *reinterpret_cast<const u32x4*>(st + (wm * TM + a * 16 + r) * 128 + place);
#pragma unroll
            for (int b = 0; b < FN; ++b) wf[b] = *reinterpret_cast<const u32x4*>(st + (BM + wn * TN + b * 16 + r) * 128 + place);
            if (kt == cut) {
#pragma unroll
                for (int a = 0; a < FM; ++a) xf[a] = first_bytes(xf[a], p.k - k_lo - kt * 128 - c * 16);
            }
#pragma unroll
            for (int a = 0; a < FM; ++a)
#pragma unroll
                for (int b = 0; b < FN; ++b)
                    acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[b]), __builtin_bit_cast(i32x4, xf[a]), acc[a][b], 0, 0, 0);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                       // no load into LDS outlives the block
#pragma unroll
    for (int a = 0; a < FM; ++a) {
        const int64_t m = at.m0 + wm * TM + a * 16 + (lane & 15);
        if (m >= p.m) continue;
        const float sx = p.sx[m];
#pragma unroll
        for (int b = 0; b < FN; ++b) {
            const int64_t n = at.n0 + wn * TN + b * 16 + (lane >> 4) * 4;
            const int some = static_cast<int>(min<int64_t>(p.n - n, 4));
            if (some <= 0) continue;
            if (p.splits > 1) {
                int* const q = p.partial + (at.split * p.m + m) * p.n + n;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < some) q[i] = acc[a][b][i];
                continue;
            }
            float sw[4], bias[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4];
            load4(p.sw + n, some, sw);
            if (p.bias) load4(static_cast<const T*>(p.bias) + n, some, bias);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(acc[a][b][i]) * sx * sw[i] + bias[i];
            store4(static_cast<T*>(p.out) + m * p.os + n, some, v);
        }
    }
}

// The shares of a sum added up: a thread takes four columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void linear8_join_kernel(const Linear8Params p) {
    const int64_t groups = (p.n + 3) / 4, t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t m = t / groups, n = (t - m * groups) * 4;
    if (m >= p.m) return;
    const int some = static_cast<int>(min<int64_t>(p.n - n, 4));
    int sum[4] = {0, 0, 0, 0};
    for (int s = 0; s < p.splits; ++s) {
        const int* const q = p.partial + (s * p.m + m) * p.n + n;
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

// The most that shares of any smaller product may take, too.
size_t linear8_ws_bytes(int64_t m, int64_t n, int k) {
    const size_t splits = static_cast<size_t>(std::min((k + 127) / 128, kMostSplits));
    if (splits < 2 || m == 0 || n == 0) return 0;
    const size_t all = static_cast<size_t>(m) * static_cast<size_t>(n);                     // (less than 2^36: see the entry points)
    return std::min(kMostPartial, all * splits * 4);
}

Linear8Plan linear8_plan(int64_t m, int64_t n, int k, size_t ws_bytes) {
    Linear8Plan plan{64, 64, 1};
    const int64_t tiles = (m + plan.bm - 1) / plan.bm * ((n + plan.bn - 1) / plan.bn), steps = (k + 127) / 128;
    const size_t all = static_cast<size_t>(m) * static_cast<size_t>(n) * 4;
    int64_t splits = std::min<int64_t>({2 * kCUs / tiles, steps / 4, kMostSplits, static_cast<int64_t>(std::min(ws_bytes, kMostPartial) / all)});
    splits = std::max<int64_t>(splits, 1);
    const int64_t nk = (steps + splits - 1) / splits;
    plan.splits = static_cast<int>((steps + nk - 1) / nk);      // no share without a step
    return plan;
}

hipError_t launch_linear8(int dtype, int64_t m, int64_t n, int k, const mopar_rows8& x, const mopar_rows8& w, const void* bias,
                          const mopar_matrix& out, void* ws, const Linear8Plan& plan, hipStream_t s) {
    Linear8Params p{};
    p.x = x.q, p.w = w.q, p.sx = x.scale, p.sw = w.scale;
    p.bias = bias;
    p.out = out.data;
    p.partial = static_cast<int*>(ws);
    p.m = m, p.n = n, p.k = k;
    p.xs = x.stride, p.ws = w.stride, p.os = out.stride;
    p.splits = plan.splits;
    p.mt = static_cast<int>((m + plan.bm - 1) / plan.bm);
    p.nt = static_cast<int>((n + plan.bn - 1) / plan.bn);
    p.total = p.mt * p.nt * p.splits;
    p.per_xcd = (p.total + 7) / 8;
    p.nk = ((k + 127) / 128 + p.splits - 1) / p.splits;
    const dim3 grid(static_cast<unsigned>(p.per_xcd) * 8);
    auto go = [&](auto t) {
        using T = decltype(t);
        launch_kernel((linear8_kernel<T, 64, 64, 2, 2, 3>), grid, dim3(256), 0, s, p);
        if (p.splits > 1) {
            const int64_t threads = m * ((n + 3) / 4);
            launch_kernel(linear8_join_kernel<T>, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s, p);
        }
        return hipGetLastError();
    };
    return dtype == MOPAR_BF16 ? go(__bf16{}) : go(float{});
}

}  // namespace mopar
