// What the operators around the step share on the host (skew_ops.h).
#include "skew_ops.h"

#include <atomic>
#include <cstdarg>
#include <cstdio>

namespace skew {

namespace {
thread_local char g_ops_error[512];
constexpr int kDevices = 64;
std::atomic<int> g_sms[kDevices];  // 0: not asked yet
}

int ops_fail(int code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_ops_error, sizeof g_ops_error, fmt, ap);
    va_end(ap);
    return code;
}

int ops_sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < kDevices && (sms = g_sms[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < kDevices) g_sms[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

}  // namespace skew

extern "C" const char *skew_ops_last_error(void) { return skew::g_ops_error; }
