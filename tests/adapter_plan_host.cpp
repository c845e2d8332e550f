// Workspace of the adapters' gradient (no GPU), built and run by test_adapter_plan_host.py: places for
// the partial sums of every run of an adapter with several, however the rows are shared out, and no more than that needs.
#include <algorithm>
#include <cstdio>
#include <random>

#include "../paper_2607_12969_amd/csrc/lrc_internal.h"

using namespace lrc;

static constexpr int64_t kRun = 512;      // rows of a run

int main() {
    int bad = 0;
    std::mt19937 rng(1);
    for (int64_t rows : {1, 65, 512, 513, 1024, 1025, 1026, 4096, 5000, 65536})
        for (int64_t count : {1, 2, 7, 64, 1000}) {
            const int64_t n = 128, m = 64, k = 16;
            AdapterGradArgs a{};
            a.rows = rows;
            a.count = count;
            a.m = m;
            a.n = n;
            a.k = k;
            a.lddy = m;
            a.ldx = n;
            a.prec = P32;
            int out;
            const size_t without = adapter_grad_workspace_bytes(a);
            a.dA = &out;
            const int64_t slots = (int64_t)(adapter_grad_workspace_bytes(a) - without) / (n * k * 4);
            auto used = [&](int64_t left, auto&& share) {      // runs of the adapters that have several
                int64_t runs = 0;
                for (int64_t q = 0; q < count && left > 0; ++q) {
                    const int64_t r = std::min(left, share(q, left));
                    if (r > kRun) runs += (r + kRun - 1) / kRun;
                    left -= r;
                }
                return runs;
            };
            int64_t most = 0;
            for (int64_t first = 1; first <= 4096; first += 1)        // 513 rows each, the first (of odd sizes) before them
                most = std::max(most, used(rows, [&](int64_t q, int64_t) { return q ? kRun + 1 : first; }));
            for (int64_t first = 0; first < count; ++first)           // 513 rows each, the rest in one
                most = std::max(most, used(rows, [&](int64_t q, int64_t left) { return q < first ? kRun + 1 : left; }));
            for (int trial = 0; trial < 2000; ++trial)
                most = std::max(most, used(rows, [&](int64_t, int64_t left) { return 1 + (int64_t)(rng() % left); }));
            if (slots < most || slots > std::max<int64_t>(1, most)) {
                ++bad;
                std::printf("rows %lld count %lld: %lld places, %lld used\n", (long long)rows, (long long)count, (long long)slots,
                            (long long)most);
            }
        }
    return bad != 0;
}
