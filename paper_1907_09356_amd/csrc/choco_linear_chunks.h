// Launches of linear attention's chunks, each type's compiled on its own.
#pragma once

#include <atomic>
#include <type_traits>

#include "choco_host.h"
#include "choco_linear.h"

namespace choco {

inline int slices_of(int dim, int slice = kLinearSlice) { return (dim + slice - 1) / slice; }
inline int64_t rows_of(const choco_linear_config& c) { return c.batch * c.heads; }
// Columns of a result that a workgroup takes: 16 a wave, four waves where that is enough, else eight (but four where eight's columns
// leave no room in LDS).
inline int slice_of(const choco_linear_config& c, int da, int dc) { return dc <= 64 || (c.type == CHOCO_F32 && da > 128) ? 64 : 128; }
inline int rows_held(int da) { return da <= 64 ? 64 : da <= 128 ? 128 : 256; }      // rows of a state that a workgroup has registers for

// A pass (MODE: kStates, kResult, kOfStates, kOfPairs) over all segments.
template <class In, int MODE>
int run_chunks(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P, LinearChunks C);

#ifdef CHOCO_LINEAR_TYPE
template <class In, int DA, int WAVES, int MODE, int WAY>
int launch_chunks(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P, const LinearChunks& C) {
  const size_t lds = sizeof(ChunkShared<In, DA, WAVES>);
  const auto kernel = k_linear_chunks<In, DA, WAVES, MODE, WAY>;
  if (lds > 65536) {
    static std::atomic<uint64_t> done{0};
    TRY_HIP(allow_lds((const void*)kernel, lds, done));
  }
  kernel<<<dim3(C.blocks), 64 * WAVES, lds, (hipStream_t)c.stream>>>(A, P, C);
  TRY_HIP(hipGetLastError());
  return CHOCO_OK;
}
template <class In, int MODE>
int run_chunks(const choco_linear_config& c, const LinearArgs& A, const LinearPass& P, LinearChunks C) {
  const int slice = slice_of(c, P.da, P.dc);
  C.slices = slices_of(P.dc, slice);
  C.blocks = (uint32_t)((rows_of(c) * C.segments + 7) / 8 * 8 * C.slices);
  const auto with_way = [&](auto dim, auto waves, auto way) -> int {
    constexpr int DA = decltype(dim)::value, WAVES = decltype(waves)::value;
    if constexpr (WAVES == 8 && DA > 128 && std::is_same_v<In, float>) return CHOCO_E_UNSUPPORTED;     // (slice_of does not say so)
    else return launch_chunks<In, DA, WAVES, MODE, decltype(way)::value>(c, A, P, C);
  };
  const auto with_waves = [&](auto dim, auto waves) -> int {
    if (C.way == kParts) return with_way(dim, waves, std::integral_constant<int, kParts>{});
    if (C.way == kWords) return with_way(dim, waves, std::integral_constant<int, kWords>{});
    return with_way(dim, waves, std::integral_constant<int, kEntries>{});
  };
  const auto with_dim = [&](auto dim) -> int {
    if (slice == 64) return with_waves(dim, std::integral_constant<int, 4>{});
    return with_waves(dim, std::integral_constant<int, 8>{});
  };
  if (rows_held(P.da) == 64) return with_dim(std::integral_constant<int, 64>{});
  if (rows_held(P.da) == 128) return with_dim(std::integral_constant<int, 128>{});
  return with_dim(std::integral_constant<int, 256>{});
}


template int run_chunks<CHOCO_LINEAR_TYPE, kStates>(const choco_linear_config&, const LinearArgs&, const LinearPass&, LinearChunks);
template int run_chunks<CHOCO_LINEAR_TYPE, kResult>(const choco_linear_config&, const LinearArgs&, const LinearPass&, LinearChunks);
template int run_chunks<CHOCO_LINEAR_TYPE, kOfStates>(const choco_linear_config&, const LinearArgs&, const LinearPass&, LinearChunks);
template int run_chunks<CHOCO_LINEAR_TYPE, kOfPairs>(const choco_linear_config&, const LinearArgs&, const LinearPass&, LinearChunks);
#endif

}  // namespace choco
