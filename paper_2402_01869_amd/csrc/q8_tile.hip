// Tile kernel of the 8-bit cache: the query rows of a recomputation chunk against their sequence's quantised keys, on the matrix cores.
//
// The expansion of a code, with its scale, to bf16 is exact (q8.h), so the tile is the bf16 pools' (tile32_body.h, head_dim 256
// tile16_body.h): the same steps and the same arithmetic on the same numbers.  What differs is how a tile gets into LDS (q8_stage.h).
// Rows that see fewer than 64 keys do not run here: the weights are rounded to bf16 (2^-9 each).
//
// Bound by the matrix pipe's issue and, on long chunks, by the power cap, as the bf16 kernel: converting a tile's codes once for its 256 (128)
// rows is hidden between the products.  208 registers, two waves a SIMD, leave the 96 that a wave of the slim row kernel has beside them.
// Measured alone, e4m3 / integers (two more instructions a pair of codes), TFLOP/s: 16 chunks of 2048 on 16384 keys, 32 heads of 128, 1120 / 1035;
// 8 of 512 on 1024..4096, 64 heads over 8, 1020 / 975, 40 heads 835 / 785; 8 of 2048 on 8192, 16 heads of 256, 955 / 887; 8 of 1024 on 4096, 32
// heads of 64, 835 / 780.
#include <algorithm>

#include "tile16_body.h"

namespace ic {

namespace {

using q8::kE4m3;
using q8::kInt8;

template <int D, int FMT>
struct Impl8 {
  static constexpr int kThreads = tile32::G32<D>::kThreads;
  static constexpr int kLdsBytes = tile32::tile32_lds_bytes<D>();
  static __device__ __forceinline__ void body(const AttnParams& p, const TileItem& it, int th, uint16_t* lds) {
    tile32::tile32_body<D, FMT>(p, it, th, lds);
  }
};
template <int FMT>
struct Impl8<tile16::kDim, FMT> {
  static constexpr int kThreads = tile16::kThreads;
  static constexpr int kLdsBytes = tile16::kLdsBytes;
  static __device__ __forceinline__ void body(const AttnParams& p, const TileItem& it, int th, uint16_t* lds) {
    tile16::tile16_body<FMT>(p, it, th, lds);
  }
};

// Workgroups (of one XCD where each has its queue) that hand out every item in one round.
__host__ __device__ inline uint32_t q8_tile_round(const AttnParams& p) {
  const uint32_t n_th = (uint32_t)p.num_heads >> p.tile_g_shift;
  return (uint32_t)p.n_tile_items * (n_th < 8u ? n_th : (n_th + 7u) / 8u);
}

// Persistent: a queue of tile items per XCD, the head groups x mod 8 in head-major order, so that the tiles of one (sequence,
// head group), which read the same keys, run on one L2 at the same time; fewer than 8 head groups: one shared queue (as the bf16
// pools' persistent kernel).  The first round goes by index.
template <int D, int FMT>
__global__ __launch_bounds__((Impl8<D, FMT>::kThreads), 2) __attribute__((amdgpu_num_vgpr(104))) void q8_tile_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(1024))) uint16_t lds[Impl8<D, FMT>::kLdsBytes / 2];
  __shared__ int s_next;
  if (p.tile_first) __builtin_amdgcn_s_setprio(3);
  const uint32_t H = (uint32_t)p.num_heads >> p.tile_g_shift;  // head groups
  const bool per_xcd = H >= 8;
  const uint32_t x = blockIdx.x & 7u;
  const uint32_t n_all = (uint32_t)p.n_tile_items * (per_xcd ? (H - x + 7u) / 8u : H);
  const uint32_t round = per_xcd ? gridDim.x / 8u : gridDim.x;
  const bool queued = q8_tile_round(p) > round;  // the same for every XCD
  uint32_t idx = per_xcd ? blockIdx.x / 8u : blockIdx.x;
  while (idx < n_all) {
    const uint32_t hsel = idx / (uint32_t)p.n_tile_items;
    const uint32_t item = per_xcd ? idx - hsel * (uint32_t)p.n_tile_items : idx / H;
    const TileItem it = p.tile_items[item];
    Impl8<D, FMT>::body(p, it, (int)(per_xcd ? x + 8u * hsel : idx - item * H), lds);
    idx = queued ? queue_pull(&p.counters[per_xcd ? x : (uint32_t)kCtrTileShared], round, &s_next) : n_all;
  }
  if (queued) queue_leave(p.counters, 0, 8, kCtrTileShared, kCtrTileLeft);
}

}  // namespace

// slots is rounded down to a multiple of 8 so that every XCD gets the same number of workgroups.
hipError_t launch_q8_tile(const AttnParams& p, int head_dim, int dtype, int slots, hipStream_t st) {
  if (p.n_tile_items <= 0) return hipSuccess;
  if (!p.counters || slots < 8 || (dtype != kE4m3 && dtype != kInt8)) return hipErrorInvalidValue;
  const bool per_xcd = (p.num_heads >> p.tile_g_shift) >= 8;
  const dim3 g(per_xcd ? 8u * std::min((uint32_t)slots / 8u, q8_tile_round(p)) : std::min((uint32_t)(slots - slots % 8), q8_tile_round(p)));
#define IC_Q8_TILE(DD)                                                                                                      \
  case DD:                                                                                                                  \
    if (dtype == kE4m3) hipLaunchKernelGGL((q8_tile_kernel<DD, kE4m3>), g, dim3(Impl8<DD, kE4m3>::kThreads), 0, st, p);      \
    else hipLaunchKernelGGL((q8_tile_kernel<DD, kInt8>), g, dim3(Impl8<DD, kInt8>::kThreads), 0, st, p);                     \
    break;
  switch (head_dim) {
    IC_Q8_TILE(64)
    IC_Q8_TILE(128)
    IC_Q8_TILE(256)
    default: return hipErrorInvalidValue;
  }
#undef IC_Q8_TILE
  return hipGetLastError();
}

}  // namespace ic
