// What the host sides of the operators share: checks of arguments and errors of HIP.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "onebitlamb.h"

namespace obm {

inline int elem_size(int dtype) { return dtype == OB_F32 ? 4 : 2; }
inline bool off_element(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_size(dtype) != 0; }
inline bool off(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }
inline bool any_dtype(int d) { return d == OB_F32 || d == OB_F16 || d == OB_BF16; }

template <class Ctx>
bool hip_ok(Ctx* ctx, hipError_t e, const char* what) {
  if (e == hipSuccess) return true;
  try {
    ctx->hip_err = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return false;
}

inline bool on_device(int device) {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && dev == device;
}

// A kernel may ask for more than 64 KB of LDS once it has been told.
template <class K>
hipError_t allow_lds(K* kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

}  // namespace obm
