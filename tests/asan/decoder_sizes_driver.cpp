// Sizes of a decoder's steps in 8 bits, with the sanitizers on.  Without arguments: what a log probability's launch writes to its
// workspace, against the workspace's size.  With "plan": for each line "tokens n_out width" of the input the form of its product with a workspace
// of the size asked for, "rows columns waves stages shares"; with "forms": every form that any size reaches, shares as 1 or 2.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <set>
#include <tuple>

#include "../../paper_2404_02445_amd/csrc/internal.h"

static int check_logprob_sizes() {
    int failures = 0;
    for (int64_t rows = 1; rows <= 140; ++rows)
        for (int32_t base : {64, 1000, 4096, 8192, 12288, 32768, 61440, 65536, 69632, 126976, 131072, 135168, 1 << 20, (1 << 28) - 4097})
            for (int32_t d : {-4096, -4095, -65, -1, 0, 1, 64, 4095, 4096}) {
                const int32_t vocab = base + d;
                if (vocab < 64) continue;
                for (int32_t top : {0, 1, 20, 64}) {
                    size_t bytes = 0;
                    if (mopar_token_logprobs_workspace_bytes(rows, vocab, top, &bytes) != MOPAR_OK) return 1000;
                    const int splits = mopar::logprob_splits(rows, vocab);
                    // a part: its maximum, two sums and a count, four bytes each, and its keys of eight
                    if (splits < 1 || (splits > 1 && static_cast<size_t>(rows) * splits * (16 + 8 * static_cast<size_t>(top)) > bytes)) {
                        std::printf("rows %lld vocab %d top %d: %d shares, %zu bytes\n", static_cast<long long>(rows), vocab, top, splits, bytes);
                        ++failures;
                    }
                }
            }
    return failures;
}

static mopar::Linear8Plan plan_of(int64_t m, int64_t n, int k) { return mopar::linear8_plan(m, n, k, mopar::linear8_ws_bytes(m, n, k)); }

int main(int argc, char** argv) {
    if (argc > 1 && std::strcmp(argv[1], "plan") == 0) {
        long long m, n;
        int k;
        while (std::scanf("%lld %lld %d", &m, &n, &k) == 3) {
            const mopar::Linear8Plan p = plan_of(m, n, k);
            std::printf("%d %d %d %d %d\n", p.bm, p.bn, p.waves, p.stages, p.splits);
        }
        return 0;
    }
    if (argc > 1 && std::strcmp(argv[1], "forms") == 0) {
        std::set<std::tuple<int, int, int, int, int>> forms;
        for (int64_t m = 1; m < 100000; m += 1 + m / 9)
            for (int64_t n = 1; n < 300000; n += 1 + n / 9)
                for (int k : {1, 128, 129, 256, 257, 512, 1000, 4096, 5000, 8192, 11000, 16384, 22000, 40000, 131071}) {
                    const mopar::Linear8Plan p = plan_of(m, n, k);
                    forms.insert({p.bm, p.bn, p.waves, p.stages, p.splits > 1 ? 2 : 1});
                }
        for (const auto& [bm, bn, waves, stages, shares] : forms) std::printf("%d %d %d %d %d\n", bm, bn, waves, stages, shares);
        return 0;
    }
    const int failures = check_logprob_sizes();
    std::printf("%d failed checks\n", failures);
    return failures != 0;
}
