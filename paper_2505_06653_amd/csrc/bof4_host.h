// bof4_host.h - what the host sides of all entry points share: the error record of the calling thread, the events of
// bof4_time_next_call, checks of arguments, the codebook in the form the kernels take.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstdio>

#include "bof4.h"
#include "bof4_device.h"

namespace bof4 {

inline thread_local char g_err[256] = "";
inline thread_local int g_hip_err = 0;
// Caller-owned events to be recorded around the main kernel of the next call (bof4_time_next_call).
inline thread_local hipEvent_t g_ev_start = nullptr, g_ev_stop = nullptr;
inline void timing_begin(hipStream_t s) {
    if (g_ev_start) (void)hipEventRecord(g_ev_start, s);
}
inline void timing_end(hipStream_t s) {
    if (g_ev_stop) (void)hipEventRecord(g_ev_stop, s);
    g_ev_start = nullptr;
    g_ev_stop = nullptr;
}

inline int fail(int code, const char* msg) {
    snprintf(g_err, sizeof(g_err), "%s", msg);
    return code;
}
inline int fail_hip(hipError_t e, const char* where) {
    g_hip_err = (int)e;
    snprintf(g_err, sizeof(g_err), "%s: %s", where, hipGetErrorString(e));
    return BOF4_ERR_HIP;
}
#define HIP_TRY(expr)                                  \
    do {                                               \
        hipError_t e_ = (expr);                        \
        if (e_ != hipSuccess) return fail_hip(e_, #expr); \
    } while (0)

inline bool valid_block(uint32_t b) { return b == 32 || b == 64 || b == 128 || b == 256; }
inline bool valid_codebook(const double* cb) {
    if (!cb) return false;
    for (int l = 0; l < 16; ++l)
        if (!std::isfinite(cb[l])) return false;
    for (int l = 1; l < 16; ++l)
        if (!(cb[l] > cb[l - 1])) return false;
    return true;
}
inline bool valid_type(uint32_t t) { return t == BOF4_F32 || t == BOF4_BF16; }
inline size_t type_bytes(uint32_t t) { return t == BOF4_BF16 ? 2 : 4; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline void make_thresholds(const double* cb, float* thr) {
    for (int k = 0; k < 15; ++k) {
        double mid = (cb[k] + cb[k + 1]) * 0.5;
        float f = (float)mid;  // round to nearest
        if ((double)f > mid) f = std::nextafterf(f, -INFINITY);
        thr[k] = f;
    }
}
inline CodebookArgs make_codebook_args(const double* cb) {
    CodebookArgs a;
    make_thresholds(cb, a.thr);
    a.thr[15] = INFINITY;
    for (int l = 0; l < 16; ++l) {
        a.lv32[l] = (float)cb[l];
        a.cb64[l] = cb[l];
    }
    return a;
}

}  // namespace bof4
