// Checks of arguments shared by the operators' C entry points.
#pragma once

#include <cstdint>
#include <stdexcept>
#include <string>

#include "../../include/dycl_tokens.h"
#include "abi.hpp"

namespace dycl {
namespace checks {

struct Bad : std::runtime_error {
  using std::runtime_error::runtime_error;
};

// throws (mapped to DYCL_E_INVALID) unless ok
inline void need(bool ok, const char* op, const char* what) {
  if (!ok) throw Bad(std::string(op) + ": " + what);
}

inline bool at(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align == 0; }

inline bool type_ok(int t) { return t == DYCL_BF16 || t == DYCL_F32; }

inline size_t size_of(int t) { return t == DYCL_F32 ? 4 : 2; }

constexpr int64_t kMaxRows = int64_t(1) << 31, kMaxPitch = int64_t(1) << 40;

inline bool pitch_ok(int64_t ld, int64_t width) { return ld >= width && ld < kMaxPitch; }

}  // namespace checks
}  // namespace dycl
