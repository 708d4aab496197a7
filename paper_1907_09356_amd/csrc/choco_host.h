// What the host sides of choco_train.h's operators share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "choco_train.h"
#include "choco_types.h"

namespace choco {

inline thread_local int g_last_hip_error = 0;

#define TRY_HIP(expr)                        \
  do {                                       \
    const hipError_t e_ = (expr);            \
    if (e_ != hipSuccess) {                  \
      choco::g_last_hip_error = (int)e_;     \
      return CHOCO_E_HIP;                    \
    }                                        \
  } while (0)

constexpr int64_t kMaxIndex = (int64_t)1 << 31;
constexpr int64_t kMaxExtent = (int64_t)1 << 60;   // entries of any array, strides included

inline int type_bytes(int type) { return type == CHOCO_F32 ? 4 : type == CHOCO_BF16 || type == CHOCO_F16 ? 2 : 0; }
inline bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
// A grid's first dimension holds less than 2^32 threads.
inline bool launch_fits(double blocks, int threads) { return blocks * threads < 4294967296.0; }
inline uint32_t blocks_of(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

// calls FN.operator()<T>() for the C++ type of a CHOCO_F32 / BF16 / F16
template <class Fn>
void with_type(int type, Fn&& fn) {
  if (type == CHOCO_F32) fn(float{});
  else if (type == CHOCO_BF16) fn(bf16_t{});
  else fn(f16_t{});
}

// A kernel's leave to take more than 64 KB of LDS at launch, asked for once on each device; `done`: where it has been.
inline hipError_t allow_lds(const void* kernel, size_t bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  if (const hipError_t e = hipGetDevice(&device)) return e;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  if (const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)) return e;
  if (device < 64) done.fetch_or(bit, std::memory_order_relaxed);
  return hipSuccess;
}

// Parts of a workspace, one behind the other on multiples of 256 bytes.
struct Parts {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) / 256 * 256;
    return here;
  }
};

}  // namespace choco
