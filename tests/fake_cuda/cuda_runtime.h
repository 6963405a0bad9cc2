// The part of the CUDA runtime that the library's scratch pool calls, on host memory, for tests without a GPU. Streams are
// small integers, kernels do not exist; every allocation, release and wait is counted.
#pragma once

#include <cstdio>
#include <cstdlib>
#include <map>
#include <set>

using cudaError_t = int;
constexpr cudaError_t cudaSuccess = 0, cudaErrorMemoryAllocation = 2, cudaErrorNotReady = 600, cudaErrorStreamCaptureUnsupported = 900;
using cudaStream_t = struct FakeStream*;
using cudaEvent_t = struct FakeEvent*;
enum cudaStreamCaptureStatus { cudaStreamCaptureStatusNone = 0, cudaStreamCaptureStatusActive = 1 };
constexpr unsigned cudaEventDisableTiming = 2;

namespace fake {
inline std::set<cudaStream_t> capturing;
inline std::map<void*, size_t> live;      // allocations that have not been freed
inline int mallocs = 0, frees = 0, syncs = 0, bad = 0;
inline bool events_ready = true;
inline cudaError_t last = cudaSuccess;
inline cudaError_t set(cudaError_t e) {
  if (e != cudaSuccess) last = e;
  return e;
}
}  // namespace fake

inline cudaError_t cudaGetLastError() {
  const cudaError_t e = fake::last;
  fake::last = cudaSuccess;
  return e;
}
inline cudaError_t cudaMalloc(void** p, size_t bytes) {
  if (!fake::capturing.empty()) return fake::set(cudaErrorStreamCaptureUnsupported);
  ++fake::mallocs;
  *p = std::malloc(16);
  fake::live[*p] = bytes;
  return cudaSuccess;
}
inline cudaError_t cudaFree(void* p) {
  ++fake::frees;
  if (!fake::live.erase(p)) ++fake::bad;
  return cudaSuccess;   // (the address is not given back, so that no later allocation has it)
}
inline cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus* out) {
  *out = fake::capturing.count(s) ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
inline cudaError_t cudaStreamSynchronize(cudaStream_t s) {
  ++fake::syncs;
  if (fake::capturing.count(s)) {
    ++fake::bad;   // ends the capture in an error
    return fake::set(cudaErrorStreamCaptureUnsupported);
  }
  return cudaSuccess;
}
inline cudaError_t cudaDeviceSynchronize() { return fake::capturing.empty() ? cudaSuccess : fake::set(cudaErrorStreamCaptureUnsupported); }
inline cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) {
  *e = reinterpret_cast<cudaEvent_t>(std::malloc(1));
  return cudaSuccess;
}
inline cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
inline cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
inline cudaError_t cudaEventQuery(cudaEvent_t) { return fake::events_ready ? cudaSuccess : fake::set(cudaErrorNotReady); }
inline cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
