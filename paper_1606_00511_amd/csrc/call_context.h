// What the contexts whose calls work on rows share on the host: the last error,
// the checks of arrays, and the order of calls that use one workspace on
// several streams.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>

#include "hf.h"

namespace hfk {

constexpr int64_t MAX_LD = (int64_t)1 << 22;  // in-tile offsets are 32 bits

struct CallContext {
  hipStream_t stream = nullptr;
  // The calls so far that no graph captured are on `work` (if pending), or
  // `work` waits for them.
  bool pending = false;
  hipStream_t work = nullptr;
  hipEvent_t last = nullptr;       // their end, for another stream to wait for
  std::string err;
};

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

inline int fail(CallContext* c, int code, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
inline int fail(CallContext* c, int code, const char* fmt, ...) {
  if (c) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    c->err = buf;
  }
  return code;
}

#define HIP_TRY(ctx, expr)                                                     \
  do {                                                                         \
    hipError_t e_ = (expr);                                                    \
    if (e_ != hipSuccess)                                                      \
      return fail(ctx, HF_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// a rows x D array of elements of es bytes, rows ld elements apart
inline int check_mat(CallContext* c, const void* p, int64_t ld, int64_t cols, int es, int64_t rows,
              const char* what) {
  if (rows == 0) return HF_OK;
  if (!p) return fail(c, HF_EINVAL, "%s is NULL", what);
  if ((uintptr_t)p % es) return fail(c, HF_EINVAL, "%s is not aligned to its elements", what);
  if (ld < cols || ld > ((int64_t)1 << 31))
    return fail(c, HF_EINVAL, "rows of %s are %lld elements apart, %lld wide", what,
                (long long)ld, (long long)cols);
  return HF_OK;
}

// an output over an input, which is read after parts of the output are written
inline int check_apart(CallContext* c, const void* in, const char* in_name, const void* out,
                const char* out_name, int64_t rows) {
  if (rows > 0 && out && in == out)
    return fail(c, HF_EINVAL, "%s is %s: not in place", out_name, in_name);
  return HF_OK;
}

// Puts the context's stream behind the calls so far, with which it shares the
// workspace, for a call or ahead of one.  While the stream is captured nothing
// is done: a wait would go into the graph, and the caller orders what is
// captured.  The first call after that, if it is not captured itself, gets
// here with work still on the stream of before.
inline int follow(CallContext* c, bool call) {
  if (c->pending && c->work == c->stream) return HF_OK;
  hipStreamCaptureStatus to = hipStreamCaptureStatusNone, from = to;
  HIP_TRY(c, hipStreamIsCapturing(c->stream, &to));
  if (to != hipStreamCaptureStatusNone) return HF_OK;
  if (c->pending) {
    HIP_TRY(c, hipStreamIsCapturing(c->work, &from));
    if (from != hipStreamCaptureStatusNone)
      return !call ? HF_OK
                   : fail(c, HF_EHIP, "the stream of the calls before this one is being captured");
    if (!c->last) HIP_TRY(c, hipEventCreateWithFlags(&c->last, hipEventDisableTiming));
    HIP_TRY(c, hipEventRecord(c->last, c->work));
    HIP_TRY(c, hipStreamWaitEvent(c->stream, c->last, 0));
  }
  c->work = c->stream;
  c->pending = true;
  return HF_OK;
}

}  // namespace hfk
