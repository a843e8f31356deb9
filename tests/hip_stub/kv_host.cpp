// The runtime and the launches behind kv_api.cpp on a machine without a GPU: memory is the
// host's, copies are done at once, launches keep their arguments.  Every call notes the device
// that was current.
#include <cstdlib>
#include <cstring>

#include "../../paper_2607_18253_amd/csrc/kv_device.h"

namespace {
int current = 0;
int calls[2] = {};  // of each device
hipError_t note() {
  ++calls[current];
  return hipSuccess;
}
lar::KvAttendArgs attend{};
lar::KvCopyArgs copy{};
}  // namespace

const char* hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipGetDevice(int* d) {
  *d = current;
  return hipSuccess;
}
hipError_t hipSetDevice(int d) {
  if (d < 0 || d > 1) return hipErrorInvalidValue;
  current = d;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
  *v = 256;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t n) {
  *p = std::malloc(n);
  return note();
}
hipError_t hipFree(void* p) {
  std::free(p);
  return note();
}
hipError_t hipHostMalloc(void** p, size_t n, unsigned) {
  *p = std::malloc(n);
  return note();
}
hipError_t hipHostFree(void* p) {
  std::free(p);
  return note();
}
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
  *e = nullptr;
  return note();
}
hipError_t hipEventDestroy(hipEvent_t) { return note(); }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return note(); }
hipError_t hipEventSynchronize(hipEvent_t) { return note(); }
hipError_t hipMemset(void* p, int x, size_t n) {
  std::memset(p, x, n);
  return note();
}
hipError_t hipMemsetAsync(void* p, int x, size_t n, hipStream_t) { return hipMemset(p, x, n); }
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) {
  std::memcpy(to, from, n);
  return note();
}
hipError_t hipStreamSynchronize(hipStream_t) { return note(); }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = hipStreamCaptureStatusNone;
  return note();
}

namespace lar {
hipError_t launch_kv_append(const KvCopyArgs& a, hipStream_t) {
  copy = a;
  return note();
}
hipError_t launch_kv_read(const KvCopyArgs& a, hipStream_t) {
  copy = a;
  return note();
}
hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t) {
  attend = a;
  return note();
}
}  // namespace lar

extern "C" {
void stub_use(int device) { current = device; }
int stub_device() { return current; }
// The number of the plan that the last launch was made for, and that of the device's plan.
uint64_t stub_attend_plan() { return attend.plan.id; }
uint64_t stub_copy_plan() { return copy.plan.id; }
uint64_t stub_device_plan() { return *attend.plan.now; }
// The plan that the last launches have on the device, as numbers; what a count is past `room` is
// not written.  0: tokens (seq, pos), 1: narrow stretches, 2: wide ones, 3 and 4: where the runs
// of each start, 5: joins, each in the order of its fields.
int stub_plan(int what, int32_t* to, int room) {
  const void* p = nullptr;
  int n = 0;
  if (what == 0) p = copy.tok, n = 2 * copy.n_tok;
  if (what == 1) p = attend.narrow, n = attend.n_narrow ? attend.narrow_at[attend.n_narrow] * 10 : 0;
  if (what == 2) p = attend.wide, n = attend.n_wide ? attend.wide_at[attend.n_wide] * 10 : 0;
  if (what == 3) p = attend.narrow_at, n = attend.n_narrow ? attend.n_narrow + 1 : 0;
  if (what == 4) p = attend.wide_at, n = attend.n_wide ? attend.n_wide + 1 : 0;
  if (what == 5) p = attend.join, n = attend.n_join * 8;
  if (n) std::memcpy(to, p, sizeof(int32_t) * (n < room ? n : room));
  return n;
}
// Calls made while a device was current, since the last time.
int stub_calls(int device) {
  const int n = calls[device];
  calls[device] = 0;
  return n;
}
}
