// Host-side checks shared by the C ABI layers (rrs_api.cpp, rrs_kv_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <memory>
#include <new>

#include "rrs.h"

namespace rrs {

inline bool is_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline rrs_status from_hip(hipError_t e) { return e == hipSuccess ? RRS_OK : RRS_ERR_HIP; }

// A device is present and is a gfx950.
rrs_status check_device();

// RRS_DEBUG (rrs_api.cpp): whether it is set, and the checks on device data under it.
bool debug_enabled();
rrs_status debug_fetch(void* host, const void* dev, size_t bytes, void* stream);
// The same into memory of its own; RRS_ERR_HIP where there is none (no exception leaves a C call).
template <typename T>
rrs_status debug_fetch_new(std::unique_ptr<T[]>* h, const void* dev, size_t count, void* stream) {
  h->reset(new (std::nothrow) T[count]);
  return *h ? debug_fetch(h->get(), dev, count * sizeof(T), stream) : RRS_ERR_HIP;
}
rrs_status debug_check_finite_f16(const void* p, size_t count, const char* what, void* stream);

}  // namespace rrs
