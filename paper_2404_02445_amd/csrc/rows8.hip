// Root mean square norm of the residual stream and rows to 8 bits, plain or gated (gfx950).
//
// A row's 8-bit steps are 127 p / a, a = max |p|, rounded to the nearest integer: p = h weight for the norm (its
// factor r is the same for the whole row and goes into the scale alone), x, or activation(gate) x.  So the sum of squares and the
// maximum come from one pass, and a row is read once, kept in registers and written once; rows past 32768 elements, four chunks of eight for each
// of 1024 threads, are read (and gated) again for the second pass: 300 x 40000 by SiLU 42 us, of a floor of 12.
//
// The steps are those of 64-bit arithmetic.  In float32 127 p / a is off by a part that is known (value()), which decides nothing
// unless the value lies within it of the middle between two steps: those, one in some thousands, are worked out again in float64 (a row
// that float32 knows too little of, as one of gates all far below zero, altogether).  So that a is exact too, the values within float32's
// error of the largest are worked out in float64 first; bf16 norms and plain rows need not, their p is exact in float32.  Rows whose largest
// p float32 does not hold, or holds with few bits (below 1e-30), are worked out in float64 altogether, from what is read again.
//
// Bound by memory from some hundred rows on: bf16 norms with a residual, to 8 bits, of 16384 x 4096 take 89 us (5.3 TB/s, a large copy
// 5.2), 65536 x 256 25 us, float32 4096 x 4096 53; rows of 4096 x 14336 39 us plain, 70 by SiLU (4.2 TB/s), 76 by GELU, whose
// vector instructions (some 50 a value in all) are active 80 % of the time.  Few rows wait for their loads and one reduction: 8 x 8192 4.0 us, 64 x 14336 by SiLU 7.1.  Rows that
// start between 16-byte places cost nothing (4001 x 11007 by GELU 59 us, 11008 on such places 58).
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mopar {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

enum { NORM = 3 };                                   // beside mopar_gate's kinds

// Eight elements from p on, of which n exist (any address that elements may have: the hardware takes unaligned vectors).  The last, short chunk of a row
// is cut from the row's last eight elements, `wide` where it has so many: element by element, rows of 11007 gated by
// GELU took 77 us for 61 at 4001.
template <typename T> __device__ __forceinline__ void load8(const T* p, int n, bool wide, float (&v)[8]) {
    if (n >= 8 || wide) {
        const int back = n < 8 ? 8 - n : 0;
        if constexpr (sizeof(T) == 2) {
            u32x4 r;
            __builtin_memcpy(&r, __builtin_assume_aligned(p - back, 2), 16);
            if (back) {
                uint64_t lo = static_cast<uint64_t>(r[1]) << 32 | r[0], hi = static_cast<uint64_t>(r[3]) << 32 | r[2];
                const int by = 16 * back;
                lo = by < 64 ? lo >> by | hi << (64 - by) : hi >> (by - 64);
                hi = by < 64 ? hi >> by : 0;
                r = u32x4{static_cast<unsigned>(lo), static_cast<unsigned>(lo >> 32), static_cast<unsigned>(hi), static_cast<unsigned>(hi >> 32)};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(r[i] << 16), v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        } else {
            f32x4 r[2];
            __builtin_memcpy(&r, __builtin_assume_aligned(p - back, 4), 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = r[i / 4][i % 4];
            if (back) {
#pragma unroll
                for (int by = 1; by < 8; by *= 2)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = back & by ? (i + by < 8 ? v[i + by < 8 ? i + by : 7] : 0.0f) : v[i];
            }
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

// e^v for v <= 88: v log2(e) as a rounded product and its remainder, 2^ of each; off by at most 4 half steps of float32.
__device__ __forceinline__ float exp_(float v) {
    constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f;          // their sum: log2(e)
    const float hi = v * kLog2e, lo = __builtin_fmaf(v, kLog2e, -hi) + v * kLog2eLow;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fmaf(e, lo * 0.693147181f, e);
}
// (1 + erf(g / sqrt 2)) / 2, erf by formula 7.1.26 of Abramowitz and Stegun's Handbook of Mathematical Functions, off by at most
// 1.5e-7 / 2, and by float32's roundings: of t (3 half steps, where the polynomial in t changes by at most 1.1 of itself), its five
// steps, e^(-g^2 / 2) and their product, of at most 1/2.  The factors 1 / sqrt 2 and 1 / 2 are in the constants.
__device__ __forceinline__ float phi_(float g) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(g), 0.231641889f, 1.0f));
    const float poly = t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
    const float tail = poly * __builtin_amdgcn_exp2f(g * g * -0.72134752f);
    return g < 0.0f ? tail : 1.0f - tail;
}

constexpr float kHalfStep = 6.0e-8f;                 // 2^-24, and the roundings of the bounds
// p in float32.  How far it may be off follows (in far_of()) from the row's largest |p| and its largest reach.
template <int KIND> __device__ __forceinline__ float value(float v, float w, float& reach) {
    if constexpr (KIND == NORM) {
        return v * w;
    } else if constexpr (KIND == MOPAR_GATE_SILU) {
        const float g = __builtin_fmaf(w, 0.0f, fmaxf(w, -88.0f));      // (infinities and NaN give NaN)
        reach = fabsf(v);
        return g * __builtin_amdgcn_rcpf(1.0f + exp_(-fminf(g, 104.0f))) * v;
    } else if constexpr (KIND == MOPAR_GATE_GELU) {
        const float g = __builtin_fmaf(w, 0.0f, fmaxf(w, -15.0f));
        const float gv = g * v;                                         // (first: g phi(g) of a subnormal gate may be no float32)
        reach = fabsf(gv);
        return gv * phi_(g);
    } else {
        return v;
    }
}
// A product of two elements: half a step.  SiLU: exponential 4 half steps, sum 1, reciprocal 2, products 3, and 1.1e-36 |x| where the
// reciprocal underflows (from g = -126 ln 2 on, where g e^g is 1.03e-36), or g is below -88.  GELU: erf 1.5e-7 + 20 half steps (1.35e-6 in all) and 12 more of the sum
// and the products, all times |g x| / 2; g below -15 leaves less than that.
template <int KIND> __device__ __forceinline__ float far_of(float top, float reach) {
    if constexpr (KIND == NORM) return top * kHalfStep;
    if constexpr (KIND == MOPAR_GATE_SILU) return top * (10.0f * kHalfStep) + reach * 1.1e-36f;
    return reach * (0.5f * (1.35e-6f + 12.0f * kHalfStep));
}
// (a call of its own: with its registers the kernels of 14336 columns gated by GELU took 127 us for 84)
template <int KIND> __device__ __attribute__((noinline)) double value64(double v, double w) {
    if constexpr (KIND == MOPAR_GATE_SILU) return w / (1.0 + exp(-w)) * v;
    // (1 + erf as it stands where it loses nothing: values of the top's own gate are ratios of x, ties among them, and go as this formula rounds)
    if constexpr (KIND == MOPAR_GATE_GELU) {
        const double z = w * 0.70710678118654752;
        return 0.5 * w * (w >= 0.0 ? 1.0 + erf(z) : erfc(-z)) * v;
    }
    return v * w;
}

struct RowsParams {
    const unsigned char *x, *residual, *gate, *weight;
    unsigned char *total, *out;
    int8_t* q;
    float* scale;
    int64_t first, tokens;                      // rows of this launch: first .. tokens - 1
    int64_t xs, rs, gs, ts, os, qs;             // strides in elements
    int width, chunks;                          // chunks of eight elements
    float eps, inv_width;
};

// The value of lane ^ D.
template <int D> __device__ __forceinline__ unsigned xor_lane(unsigned v) {
    if constexpr (D == 1) return __builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true);                 // quad_perm 1 0 3 2
    if constexpr (D == 2) return __builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true);                 // quad_perm 2 3 0 1
    if constexpr (D == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);   // 7 - i, then 3 - i
    if constexpr (D == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);                // row_ror:8
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);                        // odd rows of one with even rows of the other
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
}
template <int D> __device__ __forceinline__ float xor_lane(float v) { return __uint_as_float(xor_lane<D>(__float_as_uint(v))); }
template <int D> __device__ __forceinline__ double xor_lane(double v) {
    const uint64_t k = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, static_cast<uint64_t>(xor_lane<D>(static_cast<unsigned>(k >> 32))) << 32 | xor_lane<D>(static_cast<unsigned>(k)));
}
// v >= 0 of all the TPR threads of a row (0: of the block), combined by f, a sum or a maximum; each value of a block has its own lds[16]
template <int TPR, typename V, typename F> __device__ __forceinline__ V over_row(V v, F f, V* lds) {
    if constexpr (TPR != 32) v = f(v, xor_lane<32>(v));
    v = f(v, xor_lane<16>(v)), v = f(v, xor_lane<8>(v)), v = f(v, xor_lane<4>(v)), v = f(v, xor_lane<2>(v)), v = f(v, xor_lane<1>(v));
    if constexpr (TPR == 0) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (threadIdx.x & 15) < blockDim.x / 64 ? lds[threadIdx.x & 15] : V(0);
        v = f(v, xor_lane<8>(v)), v = f(v, xor_lane<4>(v)), v = f(v, xor_lane<2>(v)), v = f(v, xor_lane<1>(v));
    }
    return v;
}

// TPR threads take a row and a block the rows of 256 threads, or a block (TPR 0, up to 1024 threads) takes one; CH chunks a thread (0: any
// number, read twice).
template <typename T, int KIND, int TPR, int CH>
__global__ __launch_bounds__(TPR ? 256 : 1024) void rows8_kernel(const RowsParams p) {
    constexpr bool EXACT = KIND == MOPAR_GATE_NONE || (KIND == NORM && sizeof(T) == 2);      // p is exact in float32 (within its range)
    __shared__ double lds64[16];
    __shared__ float lds[3][16];
    const int many = TPR ? TPR : static_cast<int>(blockDim.x);
    const int64_t row = p.first + (TPR ? static_cast<int64_t>(blockIdx.x) * (256 / (TPR ? TPR : 1)) + threadIdx.x / many : blockIdx.x);
    const int me = TPR ? threadIdx.x % many : threadIdx.x;
    if (row >= p.tokens) return;                     // (lanes of one row stay together: none is missed by others, and no barrier by rows of several waves)
    const T* const x = reinterpret_cast<const T*>(p.x) + row * p.xs;
    const T* const res = p.residual ? reinterpret_cast<const T*>(p.residual) + row * p.rs : nullptr;
    const T* const other = KIND == NORM ? reinterpret_cast<const T*>(p.weight) : reinterpret_cast<const T*>(p.gate) + row * p.gs;
    T* const total = p.total ? reinterpret_cast<T*>(p.total) + row * p.ts : nullptr;
    T* const out = p.out ? reinterpret_cast<T*>(p.out) + row * p.os : nullptr;

    float squares = 0.0f, reach = 0.0f;
    unsigned top_bits = 0;                           // of the row's largest |p|; infinities and NaN are above all others
    // x of chunk c, the norm's h; the first time, total is stored
    const bool wide = p.width >= 8;
    auto load = [&](int c, float (&f)[8], bool first) __attribute__((always_inline)) {
        const int at = c * 8, n = p.width - at;
        if (KIND == NORM && !first && total) {
            load8<T>(total + at, n, false, f);
        } else {
            load8(x + at, n, wide, f);
            if (KIND == NORM && res) {
                float r[8];
                load8(res + at, n, wide, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(static_cast<T>(f[i] + r[i]));
                if (total) store8(total + at, n, f);
            }
        }
    };
    // p of chunk c; the first time, the row's sums go on
    auto read = [&](int c, float (&f)[8], bool first) __attribute__((always_inline)) {
        float w[8];
        load(c, f, first);
        if constexpr (KIND != MOPAR_GATE_NONE) load8(other + c * 8, p.width - c * 8, wide, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (KIND == NORM && first) squares = __builtin_fmaf(f[i], f[i], squares);
            float its = 0.0f;
            f[i] = value<KIND>(f[i], w[i], its);
            if (first) {
                top_bits = max(top_bits, __float_as_uint(f[i]) & 0x7fffffffu);
                reach = fmaxf(reach, its);
            }
        }
    };
    // p of element at in float64; read again, as few are
    auto exact = [&](int at) __attribute__((always_inline)) -> double {
        float h = static_cast<float>(total ? total[at] : x[at]);
        if constexpr (KIND == MOPAR_GATE_NONE) return h;
        if (KIND == NORM && res && !total) h = static_cast<float>(static_cast<T>(h + static_cast<float>(res[at])));
        return value64<KIND>(h, static_cast<float>(other[at]));
    };
    constexpr int KEPT = CH > 0 ? CH : 1;
    float f[KEPT][8];
    if constexpr (CH > 0) {
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (me + k * many < p.chunks) read(me + k * many, f[k], true);
    } else {
        for (int c = me; c < p.chunks; c += many) read(c, f[0], true);
    }
    auto place = [&](int bit) { return (me + (bit >> 3) * many) * 8 + (bit & 7); };      // of element bit % 8 of the thread's chunk bit / 8
    auto most = [](float a, float b) { return fmaxf(a, b); };
    float r = 1.0f;
    if constexpr (KIND == NORM) {
        squares = over_row<TPR>(squares, [](float a, float b) { return a + b; }, lds[0]);
        r = 1.0f / __builtin_sqrtf(squares * p.inv_width + p.eps);
    }
    float top = 0.0f, far = 0.0f;                    // far: how far a p of the row may be off
    double top64 = 0.0;
    bool finite = false;
    if (p.q) {
        const float mine = __uint_as_float(min(top_bits, 0x7f800000u));        // (NaN counts as infinity)
        top = over_row<TPR>(mine, most, lds[1]);
        finite = top < __builtin_inff();
        top64 = top;
        // (the norm's products past float32's range, few bits of them, or none; a row without squares, too, is one of zeros: to read such again
        // took 16384 x 4096 of them from 87 us to 104)
        const bool few = KIND == NORM && !(finite && top >= 1e-30f) && (top > 0.0f || squares > 0.0f);
        if (!EXACT || __builtin_expect(few, false)) {
            if constexpr (KIND != NORM) reach = over_row<TPR>(reach, most, lds[2]);
            far = far_of<KIND>(top, reach);
            // the row's largest in float64 is among those that float32 has within twice that of its largest, `bar` and more; among all where
            // float32 has none (a product past its range, or an infinity or NaN of the row), or few bits of it, or lost them all
            float bar = top + far > 0.0f ? top - 2.0f * far : __builtin_inff();
            if (__builtin_expect(!finite, false)) bar = -1.0f;
            if constexpr (KIND != NORM) {
                if (__builtin_expect(top < 1e-30f, false)) {
                    bar = reach > 0.0f ? -1.0f : __builtin_inff();
                    // (GELU's reach is a product, too: its rows of zeros are read again, 4096 x 14336 of them 72 us for 61)
                    if (KIND == MOPAR_GATE_GELU && reach == 0.0f)
                        for (int c = me; c < p.chunks; c += many) {
                            auto largest = [&](const T* factor) __attribute__((always_inline)) {
                                float a[8], m = 0.0f;
                                load8(factor + c * 8, p.width - c * 8, wide, a);
#pragma unroll
                                for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(a[i]));
                                return m;
                            };
                            if (largest(x) > 0.0f && largest(other) > 0.0f) bar = -1.0f;
                        }
                }
            }
            uint64_t best = 0;                       // |p| as its bits: infinities and NaN are above all others
            auto with = [&](double v) __attribute__((always_inline)) { best = max(best, __builtin_bit_cast(uint64_t, v) & ~(uint64_t(1) << 63)); };
            if (!few && !(mine < bar)) {
                if constexpr (CH > 0) {
                    uint64_t near = 0;
#pragma unroll
                    for (int k = 0; k < CH; ++k)
                        if (me + k * many < p.chunks)
#pragma unroll
                            for (int i = 0; i < 8; ++i) near |= !(fabsf(f[k][i]) < bar) ? uint64_t(1) << (8 * k + i) : 0u;
                    for (; near; near &= near - 1) {
                        const int at = place(__builtin_ctzll(near));
                        if (at < p.width) with(exact(at));
                    }
                } else {
                    for (int c = me; c < p.chunks; c += many) {
                        read(c, f[0], false);
                        for (int i = 0; i < min(8, p.width - c * 8); ++i)
                            if (!(fabsf(f[0][i]) < bar)) with(exact(c * 8 + i));
                    }
                }
            }
            if (KIND == NORM && __builtin_expect(few, false))
                for (int c = me; c < p.chunks; c += many) {
                    float h[8], w[8];
                    load(c, h, false);
                    load8(other + c * 8, p.width - c * 8, wide, w);
                    for (int i = 0; i < 8; ++i) with(static_cast<double>(h[i]) * static_cast<double>(w[i]));
                }
            best = min(best, uint64_t(0x7ff) << 52);     // (NaN counts as infinity)
            top64 = over_row<TPR>(__builtin_bit_cast(double, best), [](double a, double b) { return fmax(a, b); }, lds64);
            finite = top64 < __builtin_inf();
        }
        if (me == 0) p.scale[row] = !finite ? __builtin_nanf("") : top64 > 0.0 ? static_cast<float>(top64 * static_cast<double>(r) / 127.0) : 0.0f;   // (r may be infinite)
    }
    // (a row whose a or 127 / a is past float32, or that float32 knows too little of, has all of its steps worked out in float64)
    const bool some = finite && top64 > 0.0, rough = top64 < 1e-30 || !(top < __builtin_inff());
    const float inv = some && !rough ? static_cast<float>(127.0 / top64) : 0.0f;
    const float middle = rough ? -1.0f : 0.5f - (far * inv * 1.01f + 127.0f * 3.0f * kHalfStep);   // how far a sure step may be from its value
    int8_t* const q = p.q ? p.q + row * p.qs : nullptr;
    auto right = [&](int at) __attribute__((always_inline)) { return static_cast<int8_t>(rint(exact(at) * 127.0 / top64)); };
    // the steps of chunk c to its place; those that are not sure are marked
    auto store_steps = [&](int c, const float (&a)[8]) __attribute__((always_inline)) -> unsigned {
        const int at = c * 8, n = p.width - at;
        uint64_t steps = 0;
        unsigned near = 0;
        if (some) {
            // 1.5 * 2^23 added: rounded to whole numbers, halves to even, with the step in the low bits
            float m[8], apart = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = a[i] * inv;
                m[i] = t + 12582912.0f;
                apart = fmaxf(apart, fabsf(t - (m[i] - 12582912.0f)));
            }
            auto low = [&](int i) { return __float_as_uint(m[i]); };
            const unsigned s0 = __builtin_amdgcn_perm(low(1), low(0), 0x0c0c0400), s1 = __builtin_amdgcn_perm(low(3), low(2), 0x04000c0c);
            const unsigned s2 = __builtin_amdgcn_perm(low(5), low(4), 0x0c0c0400), s3 = __builtin_amdgcn_perm(low(7), low(6), 0x04000c0c);
            steps = static_cast<uint64_t>(s2 | s3) << 32 | (s0 | s1);
            if (apart > middle) {
#pragma unroll
                for (int i = 0; i < 8; ++i) near |= !(fabsf(a[i] * inv - (m[i] - 12582912.0f)) <= middle) ? 1u << i : 0u;
                if (n < 8) near &= (1u << n) - 1;
            }
        }
        if (n >= 8) {
            *reinterpret_cast<uint64_t*>(q + at) = steps;
        } else {
            for (int i = 0; i < n; ++i) q[at + i] = static_cast<int8_t>(steps >> (8 * i));
        }
        return near;
    };
    // (h w may have passed float32's range where h r w does not; what it has lost below 2^-149 is counted where r makes it more than 2^-126)
    const bool far_out = KIND == NORM && (top_bits >= 0x7f800000u || !(r <= 16777216.0f));
    auto store_out = [&](int c, const float (&a)[8]) __attribute__((always_inline)) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = a[i] * r;
        if (__builtin_expect(far_out, false)) {
            float h[8], w[8];
            int again = c;
            asm volatile("" : "+v"(again));          // (addresses worked out anew, not kept in registers since the first time)
            load(again, h, false);
            load8(other + again * 8, p.width - again * 8, wide, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)              // fractions times fractions, and the exponents at the end
                o[i] = ldexpf(__builtin_amdgcn_frexp_mantf(h[i]) * __builtin_amdgcn_frexp_mantf(w[i]) * __builtin_amdgcn_frexp_mantf(r),
                              __builtin_amdgcn_frexp_expf(h[i]) + __builtin_amdgcn_frexp_expf(w[i]) + __builtin_amdgcn_frexp_expf(r));
        }
        store8(out + c * 8, p.width - c * 8, o);
    };
    // (out may be what the exact values are read from: it is stored after them)
    if constexpr (CH > 0) {
        if (q) {
            uint64_t near = 0;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (me + k * many < p.chunks) near |= static_cast<uint64_t>(store_steps(me + k * many, f[k])) << (8 * k);
            for (; near; near &= near - 1) {
                const int at = place(__builtin_ctzll(near));
                q[at] = right(at);
            }
        }
        if (out)
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (me + k * many < p.chunks) store_out(me + k * many, f[k]);
    } else {
        for (int c = me; c < p.chunks; c += many) {
            read(c, f[0], false);
            if (q)
                for (unsigned near = store_steps(c, f[0]); near; near &= near - 1) {
                    const int at = c * 8 + __builtin_ctz(near);
                    q[at] = right(at);
                }
            if (out) store_out(c, f[0]);
        }
    }
}

template <typename T, int KIND> hipError_t launch(const RowsParams& p, hipStream_t s) {
    auto go = [&](auto kernel, int threads, int per) {   // a launch takes less than 2^32 threads
        RowsParams part = p;
        for (constexpr int64_t kBlocks = 1 << 21; part.first < p.tokens; part.first += kBlocks * per) {
            const int64_t blocks = std::min(kBlocks, (p.tokens - part.first + per - 1) / per);
            launch_kernel(kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, s, part);
        }
        return hipGetLastError();
    };
    auto rows = [&](auto tpr, auto ch) {                 // several rows a block
        constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value;
        return go(rows8_kernel<T, KIND, TPR, CH>, 256, 256 / TPR);
    };
    auto row = [&](auto ch) {                            // a row a block, its waves in fours, one a SIMD (4096 x 14336 by SiLU 86 us with 14 waves, 74 with 16)
        constexpr int CH = decltype(ch)::value;
        return go(rows8_kernel<T, KIND, 0, CH>, CH ? 256 * ((p.chunks + 256 * CH - 1) / (256 * (CH ? CH : 1))) : 1024, 1);
    };
    using std::integral_constant;
    integral_constant<int, 1> one;
    integral_constant<int, 2> two;
    integral_constant<int, 4> four;
    integral_constant<int, 32> t32;
    integral_constant<int, 64> t64;
    // Threads by the row's length, so that each has 1 to 4 chunks, kept in registers: 32 threads for 256 columns 24 us at 65536 rows, 64
    // (half of them idle) 39.  Where the rows leave most of the card idle, a row's loads go out at once from as many threads as
    // it has chunks: 8 x 8192 4.0 us, 256 threads 6.5; norms of 64 x 2048 3.6, a wave a row 6.3; 64 x 14336 by SiLU 7.1 with two a thread, 7.8 with four.
    if (p.chunks > 64 && p.chunks <= 2048 && p.tokens <= 512) return p.chunks <= 1024 ? row(one) : row(two);
    if (p.chunks <= 32) return rows(t32, one);
    if (p.chunks <= 64) return rows(t64, one);
    if (p.chunks <= 128) return rows(t64, two);
    // (past 1024 columns a wave a row holds its loads for long: 16384 x 2048 norms 49.5 us, 43.3 in blocks of 256 threads, a chunk each, 8192 x 2048 in
    // float32 by SiLU 35.8 and 31.6; bf16 rows to 8 bits, which have two loads a value at most, 41.9 and 48.1 by SiLU)
    if constexpr (KIND != NORM && sizeof(T) == 2) {
        if (p.chunks <= 256) return rows(t64, four);
    }
    if constexpr (KIND == NORM) {
        // two a thread hide the loads of the others best: 4096 x 14336 80 us, four 86
        if (p.chunks <= 2048) return row(two);
    } else if (p.chunks <= 4096) {
        // the fewest idle threads, then the fewest threads: 4096 x 11008 by GELU 72, 60 and 66 us with 2, 3 and 4 a thread, x 14336 86, 84, 76
        // (float32, whose chunks are two loads: the most threads, x 14336 by SiLU 98, 99 and 103)
        auto room = [&](int ch) { const int by = (p.chunks + 256 * ch - 1) / (256 * ch); return by <= 4 ? by * ch : 1 << 20; };
        const int same = sizeof(T) == 4;
        if (room(2) < room(3) + same && room(2) < room(4) + same) return row(two);
        if (room(3) < room(4) + same) return row(integral_constant<int, 3>{});
        return row(four);
    }
    if (p.chunks <= 4096) return row(four);
    return row(integral_constant<int, 0>{});
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
