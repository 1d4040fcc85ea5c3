// Rotary positions and the paged cache's writes (gfx950): turning the heads of packed token rows, the
// same on the way into the cache, and moving the accepted tokens of a drafted tree.  All three read and
// write each byte once and are bound by HBM, or by a launch when there are few tokens.  Measured (a copy reaches 5.0 TB/s
// here): 16384 tokens of 40 heads of 128 in bf16 turned in 73 us, 4.6 TB/s; 22k tokens of 32 + 8 + 8 heads turned and
// stored in 119 us, 4.55 TB/s; eight tokens in 5 us, a launch and two loads in a row; up to five kept
// tokens of four sequences in 5 us, up to eight of 32 in 16 layers (22 MB) in 11 us: a path's entries one after the other (see keep_kernel).
//
// Rotation.  Pair j of a token at position p turns by p w_j.  The host keeps w_j / 2 pi as a 64-bit
// fraction of a turn, so p times it, wrapped to 64 bits, is the angle modulo a turn: range reduction by one
// integer product, off by the fraction's error (2^-64 turns) times p: 2^-33 turns for any int32 position.  Its top 32
// bits (the others: below 2^-32 turns) give the quadrant and an angle of at most pi/4, 2^29 units of 2^-32 turns, which
// float32 rounds by at most 16: 2^-28 turns.  Its sine and cosine are their Taylor polynomials (degree 9 and 10: the
// next terms are below 2e-9).
#include <algorithm>

#include "internal.h"

namespace mopar {

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int EPC = 16 / static_cast<int>(sizeof(T));   // elements of a 16-byte chunk

template <typename T> __device__ __forceinline__ void unpack(const u32x4& r, float (&v)[EPC<T>]) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    }
}
template <typename T> __device__ __forceinline__ u32x4 pack(const float (&v)[EPC<T>]) {
    u32x4 r;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __bf16 lo = static_cast<__bf16>(v[2 * i]), hi = static_cast<__bf16>(v[2 * i + 1]);
            r[i] = static_cast<unsigned>(__builtin_bit_cast(unsigned short, lo)) |
                   static_cast<unsigned>(__builtin_bit_cast(unsigned short, hi)) << 16;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
    }
    return r;
}

// m times the cosine and sine of `pos` times the fraction w of a turn
__device__ __forceinline__ void turn_of(int pos, uint64_t w, float m, float& c, float& s) {
    const unsigned hi = static_cast<unsigned>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * w) >> 32);
    const unsigned quad = (hi + 0x20000000u) >> 30;                       // nearest quarter turn, 0..3 (4 wraps)
    const float x = static_cast<float>(static_cast<int>(hi - (quad << 30))) * 1.46291807926715969e-9f;   // 2 pi / 2^32
    const float z = x * x;
    const float sp = x + x * z * (-1.6666666666666666e-1f + z * (8.3333333333333333e-3f + z * (-1.9841269841269841e-4f + z * 2.7557319223985893e-6f)));
    const float cp = 1.0f + z * (-0.5f + z * (4.1666666666666664e-2f + z * (-1.3888888888888889e-3f +
                                              z * (2.4801587301587302e-5f + z * -2.7557319223985888e-7f))));
    const bool swap = quad & 1;
    const float cc = swap ? sp : cp, ss = swap ? cp : sp;
    c = ((quad + 1) & 2) ? -m * cc : m * cc;                              // cos: + - - + over the quadrants
    s = (quad & 2) ? -m * ss : m * ss;
}

struct RowView {
    unsigned char* data;
    int64_t ts, hs;      // bytes
};

struct RotaryParams {
    RotaryTable tab;
    const int32_t* pos;  // null: row t at position t mod period
    int period;
    int units;           // units of a head: what one thread turns (see rotary_kernel)
    int rot_units;       // of them, the first that turn
    int heads, turned;   // query heads (all heads without a cache); of them, the first that turn
    int groups;          // threads that share a token's heads
    int64_t tokens;
    RowView x, y;
    // cache
    RowView k, v;
    unsigned char *kc, *vc;
    const int32_t *table, *seq, *slot;
    int64_t table_stride, pages;
    int kv_heads, shift, max_pages, n_seq;
};

// One thread turns one unit of a token in every groups-th head: the pair's angles are worked out once and
// serve all of its heads.  Units: with pairs (j, j + r/2) whose halves are whole 16-byte chunks, a chunk of
// each half (MODE 0); with pairs of neighbours, one chunk (MODE 1; pairs past rot_dim pass); with halves
// off the chunk, one pair, element by element (MODE 2).  The units after rot_units pass unchanged: a chunk
// each (MODE 0) or an element (MODE 2).  Units of neighbouring threads are neighbours in memory.
// CACHE: heads are the queries, then the keys (turned into their page) and the values (copied into it).
template <typename T, int MODE, bool CACHE>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryParams p) {
    constexpr int N = MODE == 2 ? 1 : MODE == 1 ? EPC<T> / 2 : EPC<T>;   // pairs of a unit
    constexpr int ES = sizeof(T);
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int per_token = p.units * p.groups;
    const int64_t t = id / per_token;
    if (t >= p.tokens) return;
    const int rem = static_cast<int>(id - t * per_token), g = rem / p.units, u = rem - g * p.units;
    const bool turns = u < p.rot_units;
    const int half = p.tab.rot / 2;
    // byte offsets of the unit's two parts within a head
    const int a = MODE == 0 ? (turns ? u * 16 : (u + p.rot_units) * 16) : MODE == 1 ? u * 16 : (turns ? u : u + half) * ES;
    const int b = a + half * ES;

    float c[N], s[N];
    const bool with_angles = !CACHE || p.tab.rot > 0;
    if (turns && with_angles) {
        const int pos = p.pos ? p.pos[t] : static_cast<int>(t % p.period);
        const int j0 = MODE == 1 ? u * N : MODE == 0 ? u * N : u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            turn_of(pos, p.tab.w[min(j0 + i, 127)], p.tab.m, c[i], s[i]);
            if (MODE == 1 && j0 + i >= half) c[i] = 1.0f, s[i] = 0.0f;
        }
    }
    // the row's place in the cache: byte offset of head 0 in both pools, or -1
    int64_t place = -1, head_bytes = 0;
    if constexpr (CACHE) {
        const int sq = p.seq[t], sl = p.slot[t];
        head_bytes = (static_cast<int64_t>(p.tab.d) * ES) << p.shift;
        if (sq >= 0 && sq < p.n_seq && sl >= 0 && (sl >> p.shift) < p.max_pages) {
            const int page = p.table[sq * p.table_stride + (sl >> p.shift)];
            if (page >= 0 && page < p.pages)
                place = static_cast<int64_t>(page) * p.kv_heads * head_bytes + static_cast<int64_t>(sl & ((1 << p.shift) - 1)) * (p.tab.d * ES);
        }
    }
    const int total = CACHE ? p.heads + 2 * p.kv_heads : p.heads;
    for (int h = g; h < total; h += p.groups) {
        const unsigned char* src;
        unsigned char* dst;
        bool turn = turns;
        if (!CACHE || h < p.heads) {
            turn = turns && h < p.turned;
            src = p.x.data + t * p.x.ts + h * p.x.hs;
            dst = p.y.data + t * p.y.ts + h * p.y.hs;
        } else {
            if (place < 0) continue;
            const bool val = h >= p.heads + p.kv_heads;
            const int kh = h - p.heads - (val ? p.kv_heads : 0);
            src = val ? p.v.data + t * p.v.ts + kh * p.v.hs : p.k.data + t * p.k.ts + kh * p.k.hs;
            dst = (val ? p.vc : p.kc) + place + kh * head_bytes;
            turn = turns && !val && with_angles;
        }
        if constexpr (MODE == 2) {
            const T x = *reinterpret_cast<const T*>(src + a);
            if (!turns) {
                *reinterpret_cast<T*>(dst + a) = x;
                continue;
            }
            const T y = *reinterpret_cast<const T*>(src + b);
            const float xf = static_cast<float>(x), yf = static_cast<float>(y);
            *reinterpret_cast<T*>(dst + a) = turn ? static_cast<T>(xf * c[0] - yf * s[0]) : x;
            *reinterpret_cast<T*>(dst + b) = turn ? static_cast<T>(yf * c[0] + xf * s[0]) : y;
        } else if constexpr (MODE == 1) {
            const u32x4 r = *reinterpret_cast<const u32x4*>(src + a);
            if (!turn) {
                *reinterpret_cast<u32x4*>(dst + a) = r;
                continue;
            }
            float v[EPC<T>], o[EPC<T>];
            unpack<T>(r, v);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                o[2 * i] = v[2 * i] * c[i] - v[2 * i + 1] * s[i];
                o[2 * i + 1] = v[2 * i + 1] * c[i] + v[2 * i] * s[i];
                if ((u * N + i) >= half) o[2 * i] = v[2 * i], o[2 * i + 1] = v[2 * i + 1];   // passes, NaN and all
            }
            *reinterpret_cast<u32x4*>(dst + a) = pack<T>(o);
        } else {
            const u32x4 ra = *reinterpret_cast<const u32x4*>(src + a);
            if (!turns) {
                *reinterpret_cast<u32x4*>(dst + a) = ra;
                continue;
            }
            const u32x4 rb = *reinterpret_cast<const u32x4*>(src + b);
            if (!turn) {
                *reinterpret_cast<u32x4*>(dst + a) = ra;
                *reinterpret_cast<u32x4*>(dst + b) = rb;
                continue;
            }
            float x[EPC<T>], y[EPC<T>], ox[EPC<T>], oy[EPC<T>];
            unpack<T>(ra, x);
            unpack<T>(rb, y);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ox[i] = x[i] * c[i] - y[i] * s[i];
                oy[i] = y[i] * c[i] + x[i] * s[i];
            }
            *reinterpret_cast<u32x4*>(dst + a) = pack<T>(ox);
            *reinterpret_cast<u32x4*>(dst + b) = pack<T>(oy);
        }
    }
}

RowView view(const mopar_rows* r, int es) {
    return r ? RowView{static_cast<unsigned char*>(r->data), r->token_stride * es, r->head_stride * es} : RowView{};
}

template <typename T, bool CACHE>
hipError_t rotary_launch(RotaryParams& p, hipStream_t s) {
    const int epc = EPC<T>, d = p.tab.d, rot = p.tab.rot;
    int mode = p.tab.interleaved ? 1 : (rot / 2) % epc == 0 ? 0 : 2;
    if (mode == 0) {
        p.rot_units = rot / 2 / epc;
        p.units = p.rot_units + (d - rot) / epc;
    } else if (mode == 1) {
        p.rot_units = (rot + epc - 1) / epc;
        p.units = d / epc;
    } else {
        p.rot_units = rot / 2;
        p.units = rot / 2 + (d - rot);
    }
    const int total = CACHE ? p.heads + 2 * p.kv_heads : p.heads;
    // Threads that share a token's heads: eight heads a thread, so that an angle serves eight (22k tokens stored: 119 us,
    // 147 with a head a thread), fewer while the threads would not fill the card (eight tokens: 7.4 us with eight, 5.0)
    const int64_t base = p.tokens * p.units;
    int64_t groups = (total + 7) / 8;
    while (groups < total && base * groups < 256 * 1024) groups = std::min<int64_t>(total, groups * 2);
    p.groups = static_cast<int>(groups);
    const int64_t blocks = (base * groups + 255) / 256;
    if (blocks >= kMaxThreads / 256) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<unsigned>(blocks));
    if (mode == 0)
        launch_kernel((rotary_kernel<T, 0, CACHE>), grid, dim3(256), 0, s, p);
    else if (mode == 1)
        launch_kernel((rotary_kernel<T, 1, CACHE>), grid, dim3(256), 0, s, p);
    else
        launch_kernel((rotary_kernel<T, 2, CACHE>), grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The accepted path of a drafted tree: a thread carries one 16-byte column of the rows of one sequence, layer
// and pool, and moves its path entries in order, up to eight rows before they are stored.  Entry i lands in slot i
// after the sequence and comes from slot path[i] >= i: a slot is never written before an entry that
// comes from it has been read, whatever the path holds.
// What bounds it is not the bytes: the tests of an entry, its source page and its destination page are branches, and each of
// those words is waited for before the next load, with the row that the entry before has sent for.  Eight entries are up to
// 32 loads in a row.
// ---------------------------------------------------------------------------
struct KeepParams {
    unsigned char *k, *v;
    int64_t layer_bytes, pages, table_stride, entries;
    const int32_t *table, *len, *offsets, *path;
    int layers, kv_heads, row_bytes, shift, max_pages, n_seq, max_path;
    int cols, col_blocks;      // 16-byte columns of a token in both pools, blocks of 256 of them
};

__global__ __launch_bounds__(256) void keep_kernel(const KeepParams p) {
    const int cb = blockIdx.x % p.col_blocks, rest = blockIdx.x / p.col_blocks, s = rest % p.n_seq, layer = rest / p.n_seq;
    const int64_t lo = p.offsets[s], hi = p.offsets[s + 1];
    if (lo < 0 || hi > p.entries || hi <= lo) return;
    const int n = static_cast<int>(min(hi - lo, static_cast<int64_t>(p.max_path)));
    const int len = p.len[s];
    if (len < 0) return;
    const int col = cb * 256 + threadIdx.x;
    if (col >= p.cols) return;
    const int per_head = p.row_bytes / 16, half = p.cols / 2;
    const int c = col < half ? col : col - half, head = c / per_head, part = c - head * per_head;
    unsigned char* const pool = (col < half ? p.k : p.v) + layer * p.layer_bytes;
    const int64_t head_bytes = static_cast<int64_t>(p.row_bytes) << p.shift;
    const int32_t* const row = p.table + s * p.table_stride;
    auto at = [&](int64_t slot) -> unsigned char* {
        const int64_t pg = slot >> p.shift;
        if (pg >= p.max_pages) return nullptr;
        const int page = row[pg];
        if (page < 0 || page >= p.pages) return nullptr;
        return pool + (page * static_cast<int64_t>(p.kv_heads) + head) * head_bytes +
               static_cast<int64_t>(slot & ((1 << p.shift) - 1)) * p.row_bytes + part * 16;
    };
    for (int i0 = 0; i0 < n; i0 += 8) {
        u32x4 r[8];
        unsigned char* dst[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dst[i] = nullptr;
            if (i0 + i >= n) continue;
            const int from = p.path[lo + i0 + i];
            if (from <= i0 + i) continue;                 // in place already, or no path
            const unsigned char* src = at(static_cast<int64_t>(len) + from);
            if (!src) continue;
            dst[i] = at(static_cast<int64_t>(len) + i0 + i);
            if (dst[i]) r[i] = *reinterpret_cast<const u32x4*>(src);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (dst[i]) *reinterpret_cast<u32x4*>(dst[i]) = r[i];
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryTable& tab, int dtype, int64_t tokens, int heads, int turned, const int32_t* pos,
                         int period, const mopar_rows* x, const mopar_rows* y, hipStream_t s) {
    if (tokens == 0 || heads == 0) return hipSuccess;
    const int es = static_cast<int>(dtype_size(dtype));
    RotaryParams p{};
    p.tab = tab;
    p.pos = pos;
    p.period = period;
    p.heads = heads;
    p.turned = turned;
    p.tokens = tokens;
    p.x = view(x, es);
    p.y = view(y, es);
    return dtype == MOPAR_BF16 ? rotary_launch<__bf16, false>(p, s) : rotary_launch<float, false>(p, s);
}

hipError_t launch_cache_append(const mopar_cache& c, const RotaryTable* tab, int64_t tokens, int heads, const int32_t* pos,
                               const int32_t* seq, const int32_t* slot, const mopar_rows* q, const mopar_rows* q_out,
                               const mopar_rows* k, const mopar_rows* v, hipStream_t s) {
    if (tokens == 0) return hipSuccess;
    const int es = static_cast<int>(dtype_size(c.dtype));
    RotaryParams p{};
    if (tab) p.tab = *tab;
    p.tab.d = c.head_dim;
    p.pos = pos;
    p.period = 1;
    p.heads = heads;
    p.turned = heads;
    p.tokens = tokens;
    p.x = view(q, es);
    p.y = view(q_out, es);
    p.k = view(k, es);
    p.v = view(v, es);
    p.kc = static_cast<unsigned char*>(c.k);
    p.vc = static_cast<unsigned char*>(c.v);
    p.table = c.table_dev;
    p.seq = seq;
    p.slot = slot;
    p.table_stride = c.table_stride;
    p.pages = c.pages;
    p.kv_heads = c.kv_heads;
    p.shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));
    p.max_pages = c.max_pages;
    p.n_seq = c.n_seq;
    return c.dtype == MOPAR_BF16 ? rotary_launch<__bf16, true>(p, s) : rotary_launch<float, true>(p, s);
}

hipError_t launch_cache_keep(const mopar_cache& c, int layers, int64_t layer_stride, const int32_t* len, const int32_t* offsets,
                             int64_t entries, const int32_t* path, int max_path, hipStream_t s) {
    if (c.n_seq == 0 || layers == 0 || entries == 0 || max_path == 0) return hipSuccess;
    const int es = static_cast<int>(dtype_size(c.dtype));
    KeepParams p{};
    p.k = static_cast<unsigned char*>(c.k);
    p.v = static_cast<unsigned char*>(c.v);
    p.layer_bytes = layers > 1 ? layer_stride * es : 0;
    p.pages = c.pages;
    p.table_stride = c.table_stride;
    p.entries = entries;
    p.table = c.table_dev;
    p.len = len;
    p.offsets = offsets;
    p.path = path;
    p.layers = layers;
    p.kv_heads = c.kv_heads;
    p.row_bytes = c.head_dim * es;
    p.shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));
    p.max_pages = c.max_pages;
    p.n_seq = c.n_seq;
    p.max_path = max_path;
    p.cols = 2 * c.kv_heads * p.row_bytes / 16;
    p.col_blocks = (p.cols + 255) / 256;
    const int64_t blocks = static_cast<int64_t>(p.col_blocks) * c.n_seq * layers;
    launch_kernel(keep_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace mopar
