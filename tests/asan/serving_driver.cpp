// Host-side checks of decoding with a paged cache under AddressSanitizer and UndefinedBehaviorSanitizer: the
// argument checks and the sizing of workspaces, over the whole range of every size that a caller passes.  Offsets, lengths
// and positions are null, which every entry point refuses after its sizes, so nothing is launched.  Exit status 0 when every
// call returned what was expected.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>

#include "../../include/mopar.h"

static int failures = 0;
#define CHECK(cond)                                                                  \
    do {                                                                             \
        if (!(cond)) {                                                               \
            std::fprintf(stderr, "check failed: %s (line %d)\n", #cond, __LINE__);   \
            ++failures;                                                              \
        }                                                                            \
    } while (0)

static void* const A = reinterpret_cast<void*>(0x10000);

static mopar_cache cache_of(int32_t n_seq, int32_t kv_heads, int32_t head_dim, int32_t dtype) {
    mopar_cache c{};
    c.dtype = dtype;
    c.kv_heads = kv_heads;
    c.head_dim = head_dim;
    c.page_tokens = 16;
    c.pages = 100;
    c.k = A;
    c.v = A;
    c.table_dev = static_cast<const int32_t*>(A);
    c.table_stride = 1 << 26;
    c.max_pages = 1 << 26;
    c.n_seq = n_seq;
    return c;
}

// A model of one operator over b sequences of n rows of f elements.
static int create(mopar_op op, int32_t dtype, int64_t b, int64_t n, int64_t f_in, int64_t f_out) {
    mopar_tensor_desc t[2] = {{dtype, 3, {b, n, f_in, 0}}, {dtype, 3, {b, n, f_out, 0}}};
    op.in0 = 0;
    op.in1 = -1;
    op.out = 1;
    mopar_model_desc d{};
    d.dtype = dtype;
    d.n_tensors = 2;
    d.tensors = t;
    d.n_ops = 1;
    d.ops = &op;
    d.n_layers = 1;
    d.input = 0;
    d.output = 1;
    static unsigned char weights[16];
    mopar_model_t m = nullptr;
    const int rc = mopar_model_create(&d, weights, sizeof weights, &m);
    CHECK((rc == MOPAR_OK) == (m != nullptr));
    if (m) {
        mopar_layer_profile p;
        CHECK(mopar_model_profile(m, &p) == MOPAR_OK);
    }
    mopar_model_destroy(m);
    return rc;
}

int main() {
    const int32_t most = 2147483647;
    const mopar_rows rows{A, 1 << 20, 128};
    // the largest sizes that pass the checks one by one
    for (int32_t dtype : {MOPAR_F32, MOPAR_BF16})
        for (int32_t d : {32, 64, 96, 128})
            for (int32_t kv : {1, 65536})
                for (int32_t heads : {kv, 65536})
                    for (int32_t n_seq : {0, 1, 1 << 20, most})
                        for (int32_t max_q : {0, 1, 1 << 4, (1 << 20) - 1, most})
                            for (int32_t max_len : {1, 1 << 30, most}) {
                                const mopar_attention a{dtype, heads, kv, d, 0.1f, 0};
                                const mopar_cache c = cache_of(n_seq, kv, d, dtype);
                                size_t n = 0;
                                const int rc = mopar_attention_cache_workspace_bytes(&a, &c, most, max_q, max_len, &n);
                                CHECK(rc == MOPAR_OK || rc == MOPAR_E_UNSUPPORTED);
                                if (n_seq == most && max_q == (1 << 4) && heads == kv) CHECK(rc == MOPAR_E_UNSUPPORTED);
                                CHECK(mopar_attention_cache(&a, &c, most, nullptr, max_q, nullptr, max_len, nullptr, 0, &rows, &rows, A, n,
                                                            nullptr) == (rc != MOPAR_OK ? rc : n_seq && max_q ? MOPAR_E_ARG : MOPAR_OK));
                            }
    // the two operators in a model, of sizes whose products pass 64 bits
    mopar_op rot_op{}, att_op{};
    rot_op.kind = MOPAR_OP_ROTARY;
    rot_op.heads = 1;
    rot_op.rotary.head_dim = rot_op.rotary.rot_dim = 64;
    rot_op.rotary.base = 10000;
    att_op.kind = MOPAR_OP_CAUSAL_ATTENTION;
    att_op.heads = att_op.kv_heads = 1;
    att_op.head_dim = 64;
    att_op.scale = 0.125f;
    const int64_t sizes[] = {1, 7, 1 << 20, (int64_t(1) << 30) - 1, int64_t(1) << 31, int64_t(1) << 33, int64_t(1) << 47, int64_t(1) << 62};
    for (int32_t dtype : {MOPAR_F32, MOPAR_BF16})
        for (int64_t b : sizes)
            for (int64_t n : sizes) {
                const bool small = b <= 7 && n <= 7, large = b > 1 << 20 && n > 1 << 20;
                const int r = create(rot_op, dtype, b, n, 64, 64), a = create(att_op, dtype, b, n, 192, 64);
                CHECK(r == MOPAR_OK || r == MOPAR_E_UNSUPPORTED);
                CHECK(a == MOPAR_OK || a == MOPAR_E_UNSUPPORTED);
                if (small) CHECK(r == MOPAR_OK && a == MOPAR_OK);
                if (large) CHECK(r == MOPAR_E_UNSUPPORTED && a == MOPAR_E_UNSUPPORTED);
                CHECK(create(rot_op, dtype, b, n, int64_t(1) << 62, int64_t(1) << 62) == MOPAR_E_UNSUPPORTED);
            }
    for (int64_t h : {1, 65536, 2147483647}) {
        att_op.heads = att_op.kv_heads = static_cast<int32_t>(h);
        CHECK(create(att_op, MOPAR_F32, 1, 4, 3 * h * 64, h * 64) != MOPAR_OK || h == 1 || h == 65536);
        rot_op.heads = static_cast<int32_t>(h);
        create(rot_op, MOPAR_F32, 1, 4, h * 64, h * 64);
    }
    // random sizes, small and near the ends of their types
    std::mt19937_64 rng(11);
    auto pick32 = [&]() -> int32_t {
        const int sh = static_cast<int>(rng() % 32);
        const int32_t v = static_cast<int32_t>(rng() >> 33) >> sh;
        return rng() % 8 == 0 ? -v : v;
    };
    auto pick64 = [&]() -> int64_t {
        const int sh = static_cast<int>(rng() % 64);
        const int64_t v = static_cast<int64_t>(rng() >> 1) >> sh;
        return rng() % 8 == 0 ? -v : rng() % 2 ? v / 8 * 8 : v;
    };
    const mopar_rotary_desc rd{0, 0, 128, 128, 1e4, 1, 0, 0, 0, 0};
    mopar_rotary_t rot = nullptr;
    CHECK(mopar_rotary_create(&rd, &rot) == MOPAR_OK);
    for (int i = 0; i < 200000; ++i) {
        const int32_t dtype = static_cast<int32_t>(rng() % 2), dims[4] = {32, 64, 96, 128};
        mopar_cache c = cache_of(pick32(), pick32(), rng() % 4 ? 128 : pick32(), dtype);
        c.page_tokens = 1 << (rng() % 14);
        c.pages = pick64();
        c.max_pages = pick32();
        c.table_stride = rng() % 2 ? c.max_pages : pick64();
        const int32_t kv = rng() % 2 ? c.kv_heads : pick32(), heads = rng() % 2 ? kv : pick32();
        const mopar_attention a{dtype, heads, kv, dims[rng() % 4], 0.1f, 0};
        const int64_t tokens = rng() % 2 ? pick32() : pick64();
        const int32_t max_q = pick32(), max_len = pick32(), n_seq = pick32();
        const mopar_rows x{A, pick64(), pick64()}, y{A, pick64(), pick64()};
        size_t n = 0;
        const int rc = mopar_attention_cache_workspace_bytes(&a, &c, tokens, max_q, max_len, &n);
        const bool nothing = tokens == 0 || c.n_seq == 0 || max_q == 0;
        const int rc2 = mopar_attention_cache(&a, &c, tokens, nullptr, max_q, nullptr, max_len, nullptr, 0, &x, &y, A, n, nullptr);
        CHECK(rc2 == (rc != MOPAR_OK ? rc : nothing ? MOPAR_OK : MOPAR_E_ARG));
        CHECK(mopar_attention_prompt(&a, tokens, n_seq, nullptr, max_len, &x, &x, &x, &y, nullptr) != MOPAR_OK || tokens == 0 ||
              n_seq == 0 || max_len == 0);
        CHECK(mopar_cache_append(&c, rot, tokens, heads, nullptr, nullptr, nullptr, &x, &y, &x, &x, nullptr) != MOPAR_OK || tokens == 0);
        const int64_t entries = pick64(), stride = pick64();
        const int32_t layers = pick32();
        CHECK(mopar_cache_keep(&c, layers, stride, nullptr, nullptr, entries, nullptr, max_q, nullptr) != MOPAR_OK || c.n_seq == 0 ||
              layers == 0 || entries == 0 || max_q == 0);
        // rows: a bad second output, so that every check of the first runs and none launches
        const mopar_rows none{nullptr, 0, 0};
        CHECK(mopar_rotary_apply(rot, dtype, tokens, heads, static_cast<const int32_t*>(A), &x, &none, nullptr) != MOPAR_OK || tokens == 0 ||
              heads == 0);
        CHECK(mopar_rotary_apply(rot, dtype, tokens, heads, nullptr, &x, &y, nullptr) != MOPAR_OK || tokens == 0 || heads == 0);
        mopar_rotary_desc d{pick32() & 3, pick32() & 3, static_cast<int32_t>(rng() % 300), static_cast<int32_t>(rng() % 300), 1.0 + rng() % 1000000,
                            1.0 + rng() % 100, static_cast<double>(rng() % 100000), 0, 0, static_cast<double>(rng() % 3)};
        mopar_rotary_t r = nullptr;
        CHECK((mopar_rotary_create(&d, &r) == MOPAR_OK) == (r != nullptr));
        mopar_rotary_destroy(r);
    }
    mopar_rotary_destroy(rot);
    std::printf("%d failed checks\n", failures);
    return failures != 0;
}
