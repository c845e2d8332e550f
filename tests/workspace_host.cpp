// The grow-only workspace and graph capture (no GPU), built and run by
// test_workspace_host.py.  The runtime's calls that it makes are replaced by ones
// that count: a buffer taken under capture stays until the workspace is released.
#include <cstdio>
#include <cstdlib>
#include <set>
#include <utility>

#include "../paper_2607_12969_amd/csrc/lrc_internal.h"

namespace {
std::set<void*> live;
int syncs = 0, bad = 0;
bool capturing = false;
hipStreamCaptureMode mode = hipStreamCaptureModeGlobal;
}  // namespace

extern "C" {
hipError_t hipMalloc(void** p, size_t bytes) {
    if (capturing && mode != hipStreamCaptureModeRelaxed) return hipErrorStreamCaptureUnsupported;
    *p = std::malloc(bytes);
    live.insert(*p);
    return hipSuccess;
}
hipError_t hipFree(void* p) {
    live.erase(p);
    std::free(p);
    return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) {
    ++syncs;
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
    *s = capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode* m) {
    std::swap(*m, mode);
    return hipSuccess;
}
}

#define EXPECT(x)                                        \
    do {                                                 \
        if (!(x)) {                                      \
            ++bad;                                       \
            std::printf("line %d: %s\n", __LINE__, #x);  \
        }                                                \
    } while (0)

int main() {
    const hipStream_t st = reinterpret_cast<hipStream_t>((uintptr_t)0x10000);
    lrc::Workspace ws;
    auto call = [&](size_t bytes) -> void* {
        ws.reset();
        return ws.reserve(bytes, st) == hipSuccess ? ws.take(bytes) : nullptr;
    };
    // without a capture a larger call frees the smaller buffer
    void* a = call(1000);
    EXPECT(a && live.count(ws.base));
    void* b = call(100000);
    EXPECT(b && live.size() == 1 && syncs == 1);
    // a captured call's buffer outlives larger calls
    capturing = true;
    void* held = call(5000);
    capturing = false;
    EXPECT(held == ws.base);
    EXPECT(call(1 << 20) && live.size() == 2 && live.count(held));
    EXPECT(call(1 << 22) && live.size() == 2 && live.count(held));     // that one held nothing
    // under capture a larger call gets memory, and neither waits nor frees
    const int s = syncs;
    capturing = true;
    EXPECT(call(1 << 24) && syncs == s && live.size() == 3 && mode == hipStreamCaptureModeGlobal);
    held = call(1 << 24);
    capturing = false;
    EXPECT(held == ws.base && call(1 << 26) && live.size() == 4 && live.count(held));
    // the null stream takes no capture
    lrc::Workspace other;
    EXPECT(other.reserve(1000, nullptr) == hipSuccess && !other.captured);
    EXPECT(live.size() == 5);
    other.release();
    ws.release();
    EXPECT(live.empty());
    return bad != 0;
}
