// Root mean square norm of the residual stream and rows to 8 bits, plain or gated (gfx950).
//
// A row's 8-bit steps are 127 p / a, a = max |p|, rounded to the nearest integer: p = h weight for the norm (its
// factor r is the same for the whole row and goes into the scale alone), x, or activation(gate) x.  So the sum of squares and the
// maximum come from one pass, and a row is read once, kept in registers and written once; rows past 32768 elements are read
// again for the second pass.
//
// The steps are those of 64-bit arithmetic.  In float32 127 p / a is off by a few 2^-24 of itself, which decides
// nothing unless it lies within that of the middle between two steps: those values (one in ten thousand) are worked out
// again in float64.  So that a is exact too, the values within float32's error of the largest are reduced a second
// time in float64; bf16 norms need neither, their products of two 8-bit mantissas are exact in float32.
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

enum { NORM = 3 };                                   // beside mopar_gate's kinds

// Eight elements from p on, of which n exist (any address that elements may have: the hardware takes unaligned vectors).
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
        for (int i = 0; i < 8; ++i) v[i] = i < n ? static_cast<float>(p[i]) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        if constexpr (sizeof(T) == 2) {
            const bf16x8 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3], (__bf16)v[4], (__bf16)v[5], (__bf16)v[6], (__bf16)v[7]};
            __builtin_memcpy(__builtin_assume_aligned(p, 2), &o, 16);
        } else {
            const f32x4 o[2] = {{v[0], v[1], v[2], v[3]}, {v[4], v[5], v[6], v[7]}};
            __builtin_memcpy(__builtin_assume_aligned(p, 4), &o, 32);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = static_cast<T>(v[i]);
    }
}

// e^v for v <= 88: v log2(e) as a rounded product and its remainder, 2^ of each; off by at most 2 half steps of float32.
__device__ __forceinline__ float exp_(float v) {
    constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f;          // their sum: log2(e)
    const float hi = v * kLog2e, lo = __builtin_fmaf(v, kLog2e, -hi) + v * kLog2eLow;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fmaf(e, lo * 0.693147181f, e);
}

// activation(g) in float32
template <int KIND> __device__ __forceinline__ float activation(float g) {
    if constexpr (KIND == MOPAR_GATE_SILU) return g * __builtin_amdgcn_rcpf(1.0f + exp_(fminf(fmaxf(-g, -104.0f), 88.0f)));
    return 0.5f * g * erfcf(g * -0.707106781f);
}
// The bound of p's relative error in float32, in units of 2^-24.  A product of two elements: 1.  SiLU: the exponential 4, the
// sum 1, the reciprocal 2, products 2.  GELU: erfc itself 16, products 3, and the rounding of its argument z > 0, of which it
// changes by 2 z^2 + 2 parts in one.
template <int KIND> __device__ __forceinline__ float bound_of(float g) {
    if constexpr (KIND == NORM) return 1.0f;
    if constexpr (KIND == MOPAR_GATE_SILU) return 10.0f;
    const float z = fminf(g, 0.0f);
    return 24.0f + 3.0f * z * z;
}
template <int KIND> __device__ __forceinline__ double value64(double v, double w) {
    if constexpr (KIND == MOPAR_GATE_SILU) return w / (1.0 + exp(-w)) * v;
    if constexpr (KIND == MOPAR_GATE_GELU) return 0.5 * w * erfc(w * -0.70710678118654752) * v;
    return v * w;
}
constexpr float kHalfStep = 6.0e-8f;                 // 2^-24, and the roundings of the bounds

struct RowsParams {
    const unsigned char *x, *residual, *gate, *weight;
    unsigned char *total, *out;
    int8_t* q;
    float* scale;
    int64_t tokens, xs, rs, gs, ts, os, qs;     // strides in elements
    int width, chunks;                          // chunks of eight elements
    float eps, inv_width;
};

template <int TPR> struct RowSum {              // TPR threads of a row: reductions over them
    __device__ static float all(float v, bool sum, float* lds) {
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const float w = __shfl_xor(v, o);
            v = sum ? v + w : fmaxf(v, w);
        }
        if constexpr (TPR > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
            __syncthreads();
            v = lds[0];
#pragma unroll
            for (int i = 1; i < TPR / 64; ++i) v = sum ? v + lds[i] : fmaxf(v, lds[i]);
        }
        return v;
    }
    __device__ static double top(double v, double* lds) {
#pragma unroll
        for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
        if constexpr (TPR > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
            __syncthreads();
            v = lds[0];
#pragma unroll
            for (int i = 1; i < TPR / 64; ++i) v = fmax(v, lds[i]);
        }
        return v;
    }
};

// TPR threads take a row, CH chunks each (0: any number, read twice); a block takes the rows of 256 threads, or one.
template <typename T, int KIND, int TPR, int CH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rows8_kernel(const RowsParams p) {
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    constexpr bool EXACT = KIND == MOPAR_GATE_NONE || (KIND == NORM && sizeof(T) == 2);      // p is exact in float32
    __shared__ double lds[16];
    float* const ldsf = reinterpret_cast<float*>(lds);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (THREADS / TPR) + threadIdx.x / TPR;
    const int me = threadIdx.x % TPR;
    if (row >= p.tokens) return;                                   // (whole waves, and whole blocks where rows take several)
    const T* const x = reinterpret_cast<const T*>(p.x) + row * p.xs;
    const T* const res = p.residual ? reinterpret_cast<const T*>(p.residual) + row * p.rs : nullptr;
    const T* const other = KIND == NORM ? reinterpret_cast<const T*>(p.weight) : reinterpret_cast<const T*>(p.gate) + row * p.gs;
    T* const total = p.total ? reinterpret_cast<T*>(p.total) + row * p.ts : nullptr;
    T* const out = p.out ? reinterpret_cast<T*>(p.out) + row * p.os : nullptr;

    float squares = 0.0f, top = 0.0f;       // top: what the row's largest |p| is at least
    bool odd = false;                       // an infinity or NaN among the p
    // p of chunk c; the first time, total is stored and the row's sums go on
    auto read = [&](int c, float (&f)[8], bool first) __attribute__((always_inline)) {
        const int at = c * 8, n = p.width - at;
        float w[8];
        if (KIND == NORM && !first && total) {
            load8<T>(total + at, n, f);
        } else {
            load8(x + at, n, f);
            if (KIND == NORM && res) {
                float r[8];
                load8(res + at, n, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(static_cast<T>(f[i] + r[i]));
                if (total) store8(total + at, n, f);
            }
        }
        if constexpr (KIND != MOPAR_GATE_NONE) load8(other + at, n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (KIND == NORM) {
                if (first) squares = __builtin_fmaf(f[i], f[i], squares);
                f[i] *= w[i];
            } else if constexpr (KIND != MOPAR_GATE_NONE) {
                f[i] *= activation<KIND>(w[i]);
            }
            if (first) {
                const float a = fabsf(f[i]);
                odd |= !(a < __builtin_inff());
                top = fmaxf(top, EXACT ? a : a - a * (bound_of<KIND>(w[i]) * kHalfStep));
            }
        }
    };
    // p of element at in float64; read again, as few are
    auto exact = [&](int at) __attribute__((always_inline)) -> double {
        float h = static_cast<float>(total ? total[at] : x[at]);
        if (KIND == NORM && res && !total) h = static_cast<float>(static_cast<T>(h + static_cast<float>(res[at])));
        return value64<KIND>(h, static_cast<float>(other[at]));
    };
    constexpr int KEPT = CH > 0 ? CH : 1;
    float f[KEPT][8];
    if constexpr (CH > 0) {
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (me + k * TPR < p.chunks) read(me + k * TPR, f[k], true);
    } else {
        for (int c = me; c < p.chunks; c += TPR) read(c, f[0], true);
    }
    // the thread's chunks again
    auto each = [&](auto&& g) __attribute__((always_inline)) {
        if constexpr (CH > 0) {
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (me + k * TPR < p.chunks) g(me + k * TPR, f[k]);
        } else {
            for (int c = me; c < p.chunks; c += TPR) {
                read(c, f[0], false);
                g(c, f[0]);
            }
        }
    };
    float r = 1.0f;
    if constexpr (KIND == NORM) r = 1.0f / __builtin_sqrtf(RowSum<TPR>::all(squares, true, ldsf) * p.inv_width + p.eps);
    bool finite = false;
    double top64 = 0.0;
    if (p.q) {
        top = RowSum<TPR>::all(odd ? __builtin_inff() : top, false, ldsf);
        finite = top < __builtin_inff();
        top64 = top;
        if constexpr (!EXACT) {
            double mine = 0.0;
            if (finite && top > 0.0f)
                each([&](int c, const float (&a)[8]) __attribute__((always_inline)) {
                    float w[8];
                    if constexpr (KIND == MOPAR_GATE_GELU) load8(other + c * 8, p.width - c * 8, w);
                    unsigned near = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        near |= fabsf(a[i]) * (1.0f + bound_of<KIND>(w[i]) * kHalfStep) >= top ? 1u << i : 0u;
                    for (; near; near &= near - 1) mine = fmax(mine, fabs(exact(c * 8 + __builtin_ctz(near))));
                });
            top64 = RowSum<TPR>::top(mine, lds);
        }
        if (me == 0) p.scale[row] = finite ? static_cast<float>(top64 * static_cast<double>(r) / 127.0) : __builtin_nanf("");
    }
    const bool some = finite && top64 > 0.0, tiny = top64 < 1e-30;     // (127 / a within float32)
    const float inv = some && !tiny ? static_cast<float>(127.0 / top64) : 0.0f;
    int8_t* const q = p.q ? p.q + row * p.qs : nullptr;
    each([&](int c, const float (&a)[8]) __attribute__((always_inline)) {
        const int at = c * 8, n = p.width - at;
        uint64_t steps = 0;
        if (q && some) {
            float w[8];
            if constexpr (KIND == MOPAR_GATE_GELU) load8(other + at, n, w);
            unsigned near = 0, s[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // off by the bound of p, and 2 half steps of 127 / a and of the product
                const float t = a[i] * inv, step = __builtin_rintf(t);
                const float off = EXACT ? 127.0f * 3.0f * kHalfStep : fabsf(t) * ((bound_of<KIND>(w[i]) + 3.0f) * kHalfStep) + 1e-6f;
                near |= fabsf(t - step) > 0.5f - off ? 1u << i : 0u;
                s[i / 4] |= (static_cast<unsigned>(static_cast<int>(step)) & 255u) << (8 * (i & 3));
            }
            steps = static_cast<uint64_t>(s[1]) << 32 | s[0];
            for (near = tiny ? 255u : near; near; near &= near - 1) {
                const int i = __builtin_ctz(near);
                if (i >= n) break;
                double v;
                if constexpr (KIND == MOPAR_GATE_NONE)
                    v = static_cast<float>(x[at + i]);
                else
                    v = exact(at + i);
                const uint64_t step = static_cast<uint64_t>(static_cast<int64_t>(rint(v * 127.0 / top64))) & 255u;
                steps = (steps & ~(uint64_t(255) << (8 * i))) | step << (8 * i);
            }
        }
        if (out) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = a[i] * r;
            store8(out + at, n, o);
        }
        if (!q) return;
        if (n >= 8) {
            *reinterpret_cast<uint64_t*>(q + at) = steps;
        } else {
            for (int i = 0; i < n; ++i) q[at + i] = static_cast<int8_t>(steps >> (8 * i));
        }
    });
}

template <typename T, int KIND> hipError_t launch(const RowsParams& p, hipStream_t s) {
    auto go = [&](auto tpr, auto ch) {
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value, THREADS = TPR > 256 ? TPR : 256, PER = THREADS / TPR;
        launch_kernel((rows8_kernel<T, KIND, TPR, CH>), dim3(static_cast<unsigned>((p.tokens + PER - 1) / PER)), dim3(THREADS), 0, s, p);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (p.chunks <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (p.chunks <= 256) return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    if (p.chunks <= 512) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (p.chunks <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if (p.chunks <= 4096) return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    return go(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}

}  // namespace

hipError_t launch_rows8(const RowsJob& j, hipStream_t s) {
    RowsParams p{};
    auto bytes = [](const void* q) { return static_cast<const unsigned char*>(q); };
    p.x = bytes(j.x.data), p.xs = j.x.stride;
    p.residual = bytes(j.residual.data), p.rs = j.residual.stride;
    p.gate = bytes(j.gate.data), p.gs = j.gate.stride;
    p.weight = bytes(j.weight);
    p.total = static_cast<unsigned char*>(j.total.data), p.ts = j.total.stride;
    p.out = static_cast<unsigned char*>(j.out.data), p.os = j.out.stride;
    p.q = j.out8.q, p.qs = j.out8.stride, p.scale = j.out8.scale;
    p.tokens = j.tokens;
    p.width = j.width;
    p.chunks = (j.width + 7) / 8;
    p.eps = j.eps;
    p.inv_width = static_cast<float>(1.0 / j.width);
    auto kinds = [&](auto t) {
        using T = decltype(t);
        if (j.weight) return launch<T, NORM>(p, s);
        if (j.act == MOPAR_GATE_SILU) return launch<T, MOPAR_GATE_SILU>(p, s);
        if (j.act == MOPAR_GATE_GELU) return launch<T, MOPAR_GATE_GELU>(p, s);
        return launch<T, MOPAR_GATE_NONE>(p, s);
    };
    return j.dtype == MOPAR_BF16 ? kinds(__bf16{}) : kinds(float{});
}

}  // namespace mopar
