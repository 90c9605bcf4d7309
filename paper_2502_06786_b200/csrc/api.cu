// Entry points that launch nothing: version and status strings.
#include "common.cuh"

extern "C" int matq_version(void) { return 100; }

extern "C" const char* matq_status_string(int status) {
    switch (status) {
        case MATQ_OK: return "ok";
        case MATQ_ERR_INVALID_ARG: return "invalid argument";
        case MATQ_ERR_UNSUPPORTED: return "unsupported bit-width";
        case MATQ_ERR_SHAPE: return "unsupported shape";
        case MATQ_ERR_ALIGNMENT: return "pointer not 16-byte aligned";
        case MATQ_ERR_WORKSPACE: return "workspace missing or too small";
        case MATQ_ERR_CUDA: return "CUDA runtime error";
        case MATQ_ERR_NONFINITE: return "non-finite weight";
        case MATQ_ERR_CAPACITY: return "overflow list capacity exceeded";
        case MATQ_ERR_TIMEOUT: return "device-side wait timed out";
        case MATQ_ERR_PAGE: return "page, position or sequence bounds out of range";
        default: return "unknown status";
    }
}

// Tests of the error paths (matq_serving_test_stall): process-wide, read when a call builds its launch.
static std::atomic<int> g_serving_stall{0};

extern "C" int matq_serving_test_stall(int on) { return g_serving_stall.exchange(on ? 1 : 0); }

namespace matq {
namespace tc {
bool test_stall() { return g_serving_stall.load(std::memory_order_relaxed) != 0; }
}  // namespace tc
}  // namespace matq
