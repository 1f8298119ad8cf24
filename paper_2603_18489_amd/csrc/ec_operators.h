// What the entry points of the operators around a step have in common.
#pragma once
#include <string>

#include "ec_internal.h"

namespace ec {

inline int op_fail(int code, const char* msg) {
  set_global_error(msg);
  return code;
}
// what the launches left behind
inline int op_done(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EC_OK;
  try {
    set_global_error((std::string(what) + ": " + hipGetErrorString(e)).c_str());
  } catch (...) {
    set_global_error(what);
  }
  return EC_ERR_HIP;
}
inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
inline bool plain_type(int32_t t) { return t == EC_T_F32 || t == EC_T_BF16; }
inline size_t type_bytes(int32_t t) { return t == EC_T_F32 ? 4 : 2; }

}  // namespace ec
