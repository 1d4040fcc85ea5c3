// Host-side checks of a decoder's steps in 8 bits under AddressSanitizer and UndefinedBehaviorSanitizer: the argument checks, the
// sizes of workspaces and the plans of products, over the whole range of every size that a caller passes.  Each call lacks a
// pointer that its entry point checks last, so nothing is launched.  Exit status 0 when every call returned what was expected.
#include <cstdint>
#include <cstdio>
#include <random>

#include "../../paper_2404_02445_amd/csrc/internal.h"

static int failures = 0;
#define CHECK(cond)                                                                  \
    do {                                                                             \
        if (!(cond)) {                                                               \
            std::fprintf(stderr, "check failed: %s (line %d)\n", #cond, __LINE__);   \
            ++failures;                                                              \
        }                                                                            \
    } while (0)

int main() {
    void* const A = reinterpret_cast<void*>(0x10000);
    std::mt19937_64 rng(5);
    auto pick64 = [&]() -> int64_t {
        const int64_t edges[] = {0, 1, -1, 2147483647, 2147483648LL, INT64_MAX, INT64_MIN, 1 << 23, 1 << 24, int64_t(1) << 46};
        switch (rng() % 4) {
        case 0: return edges[rng() % 10];
        case 1: return static_cast<int64_t>(rng());
        default: return static_cast<int64_t>(rng() >> (1 + rng() % 63));
        }
    };
    auto pick32 = [&]() -> int32_t {
        const int32_t edges[] = {0, 1, -1, 2147483647, INT32_MIN, 131071, 131072, 1 << 24, (1 << 28) - 1, 64};
        switch (rng() % 4) {
        case 0: return edges[rng() % 10];
        case 1: return static_cast<int32_t>(rng());
        default: return static_cast<int32_t>((rng() & 0x7fffffff) >> (rng() % 31));
        }
    };
    for (int i = 0; i < 300000; ++i) {
        const int32_t dtype = rng() % 8 ? static_cast<int32_t>(rng() % 2) : pick32(), width = pick32();
        const int64_t tokens = pick64(), n_out = pick64();
        const mopar_matrix x{A, pick64()}, y{A, pick64()}, none{nullptr, 0};
        const mopar_rows8 q{static_cast<int8_t*>(A), rng() % 2 ? (pick64() & 0x7ffff0) : pick64(), static_cast<float*>(A)};
        const mopar_rows8 unscaled{q.q, q.stride, nullptr};
        CHECK(mopar_rms_norm(dtype, tokens, width, &x, &y, &y, A, 1e-5f, &x, &unscaled, nullptr) != MOPAR_OK || tokens == 0);
        CHECK(mopar_rms_norm(dtype, tokens, width, &x, nullptr, nullptr, nullptr, 1e-5f, &y, &q, nullptr) != MOPAR_OK || tokens == 0);
        CHECK(mopar_quantize_rows(dtype, tokens, width, &x, &y, 1 + static_cast<int32_t>(rng() % 2), &unscaled, nullptr) != MOPAR_OK || tokens == 0);
        CHECK(mopar_quantize_rows(dtype, tokens, width, &x, nullptr, pick32() | 1, &q, nullptr) == (dtype >> 1 ? MOPAR_E_DTYPE : tokens < 0 ? MOPAR_E_ARG
              : tokens >> 31 ? MOPAR_E_UNSUPPORTED : MOPAR_E_ARG));
        size_t bytes = 0;
        const int rc = mopar_linear8_workspace_bytes(tokens, n_out, width, &bytes);
        const int rc2 = mopar_linear8(rng() % 2, tokens, n_out, width, &q, &q, nullptr, &none, A, bytes, nullptr);
        CHECK(rc == MOPAR_OK ? rc2 != MOPAR_OK || tokens == 0 || n_out == 0 : rc2 == rc);
        if (rc == MOPAR_OK && tokens > 0 && n_out > 0) {
            for (size_t ws : {size_t(0), bytes, bytes * 2}) {
                const mopar::Linear8Plan plan = mopar::linear8_plan(tokens, n_out, width, ws);
                const int64_t m = (tokens + plan.bm - 1) / plan.bm, n = (n_out + plan.bn - 1) / plan.bn;
                CHECK(plan.splits >= 1 && m * n * plan.splits < (int64_t(1) << 23));
                CHECK(plan.splits == 1 || static_cast<size_t>(tokens * n_out * plan.splits) * 4 <= ws);
                CHECK(m * n * plan.splits * (plan.waves ? plan.waves : 8) * 64 < (int64_t(1) << 32));
            }
        }
        const int32_t top = rng() % 4 ? static_cast<int32_t>(rng() % 70) : pick32();
        size_t log_bytes = 0;
        const int rc3 = mopar_token_logprobs_workspace_bytes(tokens, width, top, &log_bytes);
        const int rc4 = mopar_token_logprobs(rng() % 2, tokens, width, &x, 1.0f, static_cast<int32_t*>(A), top, nullptr, nullptr, nullptr, nullptr, nullptr, A,
                                             log_bytes, nullptr);
        CHECK(rc3 == MOPAR_OK ? rc4 != MOPAR_OK || tokens == 0 : rc4 == rc3);
        if (rc3 == MOPAR_OK && tokens > 0) {
            const int splits = mopar::logprob_splits(tokens, width);
            CHECK(splits >= 1 && (splits == 1 || static_cast<size_t>(tokens) * splits * 8 * top <= log_bytes));
        }
    }
    std::printf("%d failed checks\n", failures);
    return failures != 0;
}
