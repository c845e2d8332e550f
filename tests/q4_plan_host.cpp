// Workspace of the 4-bit product over batches around its panels (no GPU), built
// and run by test_q4_plan_host.py: every batch is planned, and a batch of several
// panels takes the workspace of its largest one.
#include <algorithm>
#include <cstdio>

#include "../paper_2607_12969_amd/csrc/lrc_internal.h"

using namespace lrc;

int main() {
    int bad = 0;
    const int64_t panel = 1 << 20;
    for (int prec : {P32, P16, PB16})
        for (int64_t n : {32, 200, 1024})
            for (int64_t k : {0, 7}) {
                const Q4Weights w{nullptr, nullptr, 48, n, 32, P16, nullptr, nullptr, nullptr, k, P16};
                const void* X = reinterpret_cast<const void*>((uintptr_t)0x10000);
                auto bytes = [&](int64_t b) { return q4_apply_workspace_bytes(w, X, n, b, prec); };
                const size_t whole = bytes(panel);
                for (int64_t count : {1, 2, 3, 5})
                    for (int64_t more : {0, 1, 3, 9, 1000}) {
                        const int64_t b = count * panel + more;
                        const size_t got = bytes(b), want = more ? std::max(whole, bytes(more)) : whole;
                        if (got != want) {
                            ++bad;
                            std::printf("prec %d n %lld k %lld batch %lld: %zu, want %zu\n", prec, (long long)n, (long long)k,
                                        (long long)b, got, want);
                        }
                    }
            }
    return bad != 0;
}
