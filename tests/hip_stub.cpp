// Stands in for the HIP runtime where there is no GPU: it runs nothing, keeps a
// log of the launches, events and waits that libhf.so asks for, and reports
// streams as capturing, or calls as failed, where a test says so.  Loaded with
// RTLD_GLOBAL ahead of the library, whose HIP calls then come here.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <map>
#include <set>
#include <string>

namespace {
std::string text;
std::map<const void*, std::string> names;
std::set<const void*> capturing;
std::string failing;                 // the call that fails next, once

void say(const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  text += buf;
}
bool fails(const char* call) {
  if (failing != call) return false;
  failing.clear();
  return true;
}
}  // namespace

extern "C" {

const char* stub_log() { return text.c_str(); }
void stub_clear() { text.clear(); }
void stub_capture(void* stream, int on) {
  if (on) capturing.insert(stream);
  else capturing.erase(stream);
}
void stub_fail(const char* call) { failing = call; }

void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*,
                           void*, void*, int*) {
  names[f] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void**) {}

hipError_t hipExtLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t, hipStream_t s,
                              hipEvent_t, hipEvent_t, int) {
  say("launch %s %u %u %u %u %u %u %p\n", names[f].c_str(), g.x, g.y, g.z, b.x, b.y, b.z,
      (void*)s);
  return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* out) {
  if (fails("hipStreamIsCapturing")) return hipErrorUnknown;
  *out = capturing.count(s) ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
  if (fails("hipEventCreateWithFlags")) return hipErrorUnknown;
  static size_t n = 0x1000;
  *e = (hipEvent_t)(n += 16);
  return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
  if (fails("hipEventRecord")) return hipErrorUnknown;
  say("record %p %p\n", (void*)e, (void*)s);
  return hipSuccess;
}
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t e, unsigned) {
  if (fails("hipStreamWaitEvent")) return hipErrorUnknown;
  say("wait %p %p\n", (void*)e, (void*)s);
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t s) {
  say("sync %p\n", (void*)s);
  return hipSuccess;
}
hipError_t hipDeviceSynchronize() {
  say("syncall\n");
  return hipSuccess;
}
hipError_t hipMemcpy(void* dst, const void*, size_t n, hipMemcpyKind kind) {
  if (kind == hipMemcpyDeviceToHost) memset(dst, 0, n);
  return hipSuccess;
}
hipError_t hipMemset(void*, int, size_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error of the stub"; }

}  // extern "C"
