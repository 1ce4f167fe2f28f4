// Stands in for the HIP runtime where salt_serve.cpp is built for the host by itself (tests/test_serve_host.py): device
// memory is malloc's, streams and events are addresses, nothing runs.  A stream can be said to be under
// capture; a memory call then fails and spoils the capture, as it does on a device.  Nothing in here uses operator new.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

typedef struct fake_stream* hipStream_t;
typedef struct fake_event* hipEvent_t;
enum hipError_t { hipSuccess = 0, hipErrorOutOfMemory = 2, hipErrorStreamCaptureUnsupported = 900 };
enum hipStreamCaptureStatus { hipStreamCaptureStatusNone = 0, hipStreamCaptureStatusActive = 1, hipStreamCaptureStatusInvalidated = 2 };
enum hipMemcpyKind { hipMemcpyHostToDevice = 1 };
enum { hipHostMallocDefault = 0, hipEventDisableTiming = 2 };

namespace fake {
inline hipStream_t capturing = nullptr;
inline bool spoiled = false;
inline long live = 0;                       // allocations and events not yet freed
inline hipError_t memory_call() {
  if (!capturing) return hipSuccess;
  spoiled = true;
  return hipErrorStreamCaptureUnsupported;
}
inline hipError_t get(void** p, size_t n) {
  *p = nullptr;
  if (memory_call() != hipSuccess) return hipErrorStreamCaptureUnsupported;
  *p = malloc(n ? n : 1);
  live += *p != nullptr;
  return *p ? hipSuccess : hipErrorOutOfMemory;
}
inline hipError_t put(void* p) {
  live -= p != nullptr;
  free(p);
  return hipSuccess;
}
}  // namespace fake

inline hipError_t hipGetLastError() { return hipSuccess; }
inline hipError_t hipSetDevice(int) { return hipSuccess; }
inline hipError_t hipDeviceSynchronize() { return fake::memory_call(); }
inline hipError_t hipMalloc(void** p, size_t n) { return fake::get(p, n); }
inline hipError_t hipHostMalloc(void** p, size_t n, unsigned) { return fake::get(p, n); }
inline hipError_t hipFree(void* p) { return fake::put(p); }
inline hipError_t hipHostFree(void* p) { return fake::put(p); }
inline hipError_t hipMemset(void* p, int v, size_t n) {
  memset(p, v, n);
  return fake::memory_call();
}
inline hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind, hipStream_t) {
  memcpy(d, s, n);
  return hipSuccess;
}
inline hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* st) {
  *st = s && s == fake::capturing ? (fake::spoiled ? hipStreamCaptureStatusInvalidated : hipStreamCaptureStatusActive)
                                  : hipStreamCaptureStatusNone;
  return hipSuccess;
}
inline hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
inline hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) {
  *e = (hipEvent_t)malloc(1);
  fake::live += *e != nullptr;
  return *e ? hipSuccess : hipErrorOutOfMemory;
}
inline hipError_t hipEventDestroy(hipEvent_t e) { return fake::put(e); }
inline hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
inline hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
