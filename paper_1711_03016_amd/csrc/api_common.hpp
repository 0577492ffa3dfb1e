// What the files of the C ABI share: the message of the last failure, and the
// checks and address arithmetic of their arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <string>

#include "dlvm.h"

namespace dlvm {
namespace api {

inline thread_local std::string g_last_error;

inline dlvm_status fail(dlvm_status code, const std::string& msg) {
  g_last_error = msg;
  return code;
}

inline dlvm_status hip_fail(hipError_t e, const char* where) {
  return fail(DLVM_ERR_HIP, std::string(where) + ": " + hipGetErrorString(e));
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline size_t elem_size(int dtype) { return dtype == DLVM_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool valid_dtype(int32_t d) { return d == DLVM_F32 || d == DLVM_BF16; }
inline bool valid_act(int32_t a) { return a >= DLVM_ACT_NONE && a <= DLVM_ACT_RELU; }

// Address arithmetic on integers: a dry run (plan description) uses null bases.
template <typename T> T* at(const void* base, size_t off) {
  return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(base) + off);
}

}  // namespace api
}  // namespace dlvm
