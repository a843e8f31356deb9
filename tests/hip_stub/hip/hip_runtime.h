// A stand-in for the HIP runtime, as far as the host side of the paged cache calls it, for
// tests on a machine without a GPU: two devices whose memory is the host's (kv_host.cpp).
#ifndef LAR_TEST_HIP_RUNTIME_H
#define LAR_TEST_HIP_RUNTIME_H

#include <cstddef>
#include <cstdint>

struct float4 {
  float x, y, z, w;
};
typedef struct ihipStream* hipStream_t;
typedef struct ihipEvent* hipEvent_t;
enum hipError_t { hipSuccess = 0, hipErrorInvalidValue = 1 };
enum hipDeviceAttribute_t { hipDeviceAttributeMultiprocessorCount };
enum hipMemcpyKind { hipMemcpyHostToDevice, hipMemcpyDeviceToHost };
enum hipStreamCaptureStatus { hipStreamCaptureStatusNone, hipStreamCaptureStatusActive };
constexpr unsigned hipHostMallocDefault = 0, hipEventDisableTiming = 2;

const char* hipGetErrorString(hipError_t);
hipError_t hipGetDevice(int*);
hipError_t hipSetDevice(int);
hipError_t hipDeviceGetAttribute(int*, hipDeviceAttribute_t, int);
hipError_t hipMalloc(void**, size_t);
hipError_t hipFree(void*);
hipError_t hipHostMalloc(void**, size_t, unsigned);
hipError_t hipHostFree(void*);
hipError_t hipEventCreateWithFlags(hipEvent_t*, unsigned);
hipError_t hipEventDestroy(hipEvent_t);
hipError_t hipEventRecord(hipEvent_t, hipStream_t);
hipError_t hipEventSynchronize(hipEvent_t);
hipError_t hipMemset(void*, int, size_t);
hipError_t hipMemsetAsync(void*, int, size_t, hipStream_t);
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t);
hipError_t hipStreamSynchronize(hipStream_t);
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus*);

#endif  // LAR_TEST_HIP_RUNTIME_H
