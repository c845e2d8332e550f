// An exception inside an output-head call (no GPU), built and run by
// test_exception_host.py: the runtime's hipGetDevice is replaced by one that throws
// as a failing allocation does.
#include <cstdio>
#include <cstring>
#include <new>

#include "../paper_2607_12969_amd/csrc/lrc_internal.h"
#include "../include/lrc.h"

extern "C" hipError_t hipGetDevice(int*) { throw std::bad_alloc(); }

int main() {
    auto at = [](uintptr_t i) { return reinterpret_cast<void*>(i << 24); };
    float* f[4] = {(float*)at(3), (float*)at(4), (float*)at(5), (float*)at(6)};
    int64_t* ids = (int64_t*)at(2);
    int bad = 0;
    auto expect = [&](const char* what, int rc) {
        if (rc == LRC_ENOMEM && !std::strcmp(lrc_last_error(), "out of memory")) return;
        ++bad;
        std::printf("%s: %d %s\n", what, rc, lrc_last_error());
    };
    auto stale = [&] { (void)lrc_sample(at(1), 10, -1, 10, LRC_FP32, f[0], nullptr, nullptr, nullptr, nullptr, ids); };
    stale();
    expect("sample", lrc_sample(at(1), 10, 4, 10, LRC_FP32, f[0], nullptr, nullptr, nullptr, nullptr, ids));
    stale();
    expect("distill", lrc_distill(at(1), 10, 4, 10, LRC_FP32, ids, f[0], 2, LRC_FP32, nullptr, nullptr, 1.0, f[1], f[2], f[3], 10));
    stale();
    expect("backward", lrc_distill_backward(at(1), 10, 4, 10, LRC_FP32, ids, f[0], 2, LRC_FP32, nullptr, nullptr, 1.0, f[1],
                                            nullptr, f[3], 10));
    stale();
    expect("quantize", lrc_q4_quantize(at(1), 64, 4, 64, 32, LRC_FP32, at(2), at(3), LRC_FP16, nullptr, nullptr));
    stale();
    expect("apply", lrc_q4_apply(at(1), at(2), LRC_FP16, 32, nullptr, nullptr, nullptr, 0, 0, at(3), 64, at(4), 8, 8, 64, 2,
                                 LRC_FP16, LRC_FP16));
    return bad != 0;
}
