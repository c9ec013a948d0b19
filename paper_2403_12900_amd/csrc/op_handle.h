// What the operator handles of the C ABI (drafted trees, 4-bit caches) have in
// common: workspace, stream, device, sticky errors and the device check flag.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>
#include <new>
#include <string>

#include "device_common.h"
#include "../../include/sprout.h"

namespace spr {
// The calling thread's last error message (spr_last_error).
spr_status set_error(spr_status s, const std::string& msg);
void clear_error();
}  // namespace spr

namespace sprk {

// Operator workspace: partials of attention (or verification's sums), then
// attention's counters (zero between launches).
constexpr size_t kOpPartBytes = size_t{32} << 20;
constexpr int kOpCounters = 65536;
constexpr size_t kOpWorkspaceBytes = kOpPartBytes + kOpCounters * sizeof(int32_t);

// A bit of the device check flag beside those of device_common.h: a fork's fresh
// block that another of its forks copies from.
constexpr int kErrFresh = 16;

struct OpHandle {
  char* ws = nullptr;
  hipStream_t st = nullptr;
  int dev = 0, n_cu = 1;
  spr_status sticky = SPR_OK;
  std::string sticky_msg;
  int* err_host = nullptr;  // device check flag in mapped pinned host memory
  int* err_dev = nullptr;
  ~OpHandle() {
    if (err_host != nullptr) (void)hipHostFree(err_host);
  }
  float* part() const { return reinterpret_cast<float*>(ws); }
  int32_t* counters() const { return reinterpret_cast<int32_t*>(ws + kOpPartBytes); }
};

// Makes the handle's device current for the call.
struct DeviceGuard {
  int before = -1;
  hipError_t e;
  explicit DeviceGuard(int dev) {
    e = hipGetDevice(&before);
    if (e == hipSuccess && before != dev) e = hipSetDevice(dev);
    else before = -1;
  }
  ~DeviceGuard() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

inline spr_status bad_arg(const char* msg) { return spr::set_error(SPR_ERR_INVALID_ARG, msg); }

inline spr_status hip_failed(OpHandle* o, const char* what, hipError_t e) {
  const std::string msg = std::string(what) + ": " + hipGetErrorString(e);
  if (o != nullptr) {
    o->sticky = SPR_ERR_HIP;
    o->sticky_msg = "an earlier HIP error left the handle unusable; release it (" + msg + ")";
  }
  return spr::set_error(SPR_ERR_HIP, msg);
}

inline spr_status check_handle(OpHandle* o) {
  if (o == nullptr) return bad_arg("operator handle is null");
  if (o->sticky == SPR_OK) {
    const int bits = *reinterpret_cast<volatile int*>(o->err_host);
    if (bits != 0) {
      o->sticky = SPR_ERR_DEVICE_CHECK;
      o->sticky_msg = "a device check failed on an earlier call:";
      if (bits & kErrTokenRange) o->sticky_msg += " a drafted token outside [0, vocab);";
      if (bits & kErrLogits) o->sticky_msg += " a logits row with a NaN or no finite maximum;";
      if (bits & kErrBlockId) o->sticky_msg += " a block id outside the pool;";
      if (bits & kErrPath) o->sticky_msg += " a malformed path of tree nodes;";
      if (bits & kErrFresh) o->sticky_msg += " a fork's fresh block that holds positions already;";
      o->sticky_msg += " release the handle";
    }
  }
  return o->sticky == SPR_OK ? SPR_OK : spr::set_error(o->sticky, o->sticky_msg);
}

// No exception crosses the ABI (a failed host allocation is the only source).
template <class F>
spr_status guarded(F f) {
  try {
    spr::clear_error();
    return f();
  } catch (const std::exception&) {
    return SPR_ERR_HIP;
  }
}

// A handle of type T in the caller's workspace, on the current device.  what:
// the entry point's name, for messages.
template <class T>
spr_status init_handle(const char* what, void* dev_ws, size_t ws_bytes, void* hip_stream, T** out) {
  return guarded([&]() -> spr_status {
    const std::string w = what;
    if (out == nullptr) return bad_arg((w + ": out must not be null").c_str());
    *out = nullptr;
    if (dev_ws == nullptr || (reinterpret_cast<uintptr_t>(dev_ws) & 255) != 0)
      return spr::set_error(SPR_ERR_WORKSPACE, w + ": workspace must be a non-null, 256-byte aligned device pointer");
    if (ws_bytes < kOpWorkspaceBytes)
      return spr::set_error(SPR_ERR_WORKSPACE, w + ": workspace has " + std::to_string(ws_bytes) + " bytes, " +
                                                   std::to_string(kOpWorkspaceBytes) + " needed");
    T* o = new (std::nothrow) T();
    if (o == nullptr) return SPR_ERR_HIP;
    o->ws = static_cast<char*>(dev_ws);
    o->st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = hipGetDevice(&o->dev);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&o->n_cu, hipDeviceAttributeMultiprocessorCount, o->dev);
    if (e == hipSuccess) e = hipHostMalloc(reinterpret_cast<void**>(&o->err_host), sizeof(int), hipHostMallocMapped);
    if (e == hipSuccess) {
      *o->err_host = 0;
      e = hipHostGetDevicePointer(reinterpret_cast<void**>(&o->err_dev), o->err_host, 0);
    }
    if (e == hipSuccess) e = hipMemsetAsync(o->ws + kOpPartBytes, 0, kOpCounters * sizeof(int32_t), o->st);
    if (e == hipSuccess) e = hipStreamSynchronize(o->st);
    if (e != hipSuccess) {
      delete o;
      return hip_failed(nullptr, what, e);
    }
    *out = o;
    return SPR_OK;
  });
}

}  // namespace sprk
