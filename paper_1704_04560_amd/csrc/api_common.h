// What the files of the C ABI (api.hip, api_ops.hip) share: the calling thread's error message and
// the checks of caller pointers.
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

#include "mtx.h"

namespace mtx {

// Keep the message for mtx_last_error() and return `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* what);

#define HIP_TRY(expr, what)                        \
    do {                                           \
        hipError_t _e = (expr);                    \
        if (_e != hipSuccess) return hip_fail(_e, what); \
    } while (0)

constexpr size_t kAlign = 256;

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool overlap(const void* a, size_t abytes, const void* b, size_t bbytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + bbytes && y < x + abytes;
}

inline bool being_captured(hipStream_t s)
{
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    const bool yes = hipStreamIsCapturing(s, &cap) == hipSuccess && cap != hipStreamCaptureStatusNone;
    (void)hipGetLastError();
    return yes;
}

// Wait for what was enqueued on a stream.  Calls on a stream that is being captured have not run,
// and waiting for them would end the capture; so would waiting for any other stream while one is
// captured, unless the thread's calls are declared apart from captures (relaxed).
inline void finish_stream(hipStream_t s)
{
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    const bool relaxed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
    if (!being_captured(s)) (void)hipStreamSynchronize(s);
    if (relaxed) (void)hipThreadExchangeStreamCaptureMode(&mode);
    (void)hipGetLastError();
}

}  // namespace mtx
