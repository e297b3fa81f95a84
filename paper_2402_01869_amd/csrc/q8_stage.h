// How a wave of the tile kernels brings its 8 keys of a 64-key tile of an 8-bit cache into LDS: codes to registers, a step ahead of where they
// are needed, then as bf16 numbers, scale and all, into the places that a bf16 pool's copies would have put them.  A code is
// converted once for all rows of the workgroup (256, or 128 at head_dim 256).
// Lane i has key i / 8 of the wave's and 16 codes (8 at head_dim 64) of every 128 dims.
#pragma once

#include "q8.h"

namespace ic {
namespace q8 {

template <int D>
struct Codes {
  static constexpr int kLoads = D / 128 > 0 ? D / 128 : 1;
  static constexpr int kWords = D >= 128 ? 4 : 2;  // dwords of a load
  uint32_t c[kLoads][kWords];
  uint32_t ks, vs;  // scale bytes of the key and (vs, also for keys) of the value
};

template <int D, int FMT>
struct Stager {
  const char* pool;      // base of the pool
  uint32_t block_bytes;
  uint32_t code_at[2];   // this lane's codes of K and of V, and
  uint32_t scale_at;     // ... its key's scale byte, inside a block
  uint32_t lds_at;       // this lane's first 16 bytes among the wave's 8 keys of a staged tile

  // key: the lane's key inside its block, spread: what the tile kernel permutes the 16-byte chunks of that key by
  __device__ __forceinline__ Stager(const AttnParams& p, int kvh, int Hk, int lane, int key, int spread) {
    pool = (const char*)p.pool;
    block_bytes = p.block_bytes;
    const uint32_t part = lane & 7;
#pragma unroll
    for (int i = 0; i < 2; ++i) code_at[i] = (uint32_t)((i * Hk + kvh) * kBlockSize + key) * D + part * (4 * Codes<D>::kWords);
    scale_at = 2u * Hk * kBlockSize * D + (uint32_t)kvh * 2u * kBlockSize + key;
    if constexpr (D >= 128) lds_at = (part >> 2) * 1024 + (lane >> 3) * 128 + (((part & 3) * 2) ^ spread) * 16;
    else lds_at = (lane >> 3) * 128 + (part ^ spread) * 16;
  }
  template <int KV>
  __device__ __forceinline__ void load(Codes<D>& s, int id) const {
    const char* b = pool + (uint64_t)(uint32_t)id * block_bytes;
#pragma unroll
    for (int j = 0; j < Codes<D>::kLoads; ++j) {
      if constexpr (D >= 128) {
        const u32x4 x = *(const u32x4*)(b + code_at[KV] + 128 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) s.c[j][i] = x[i];
      } else {
        const u32x2 x = *(const u32x2*)(b + code_at[KV]);
        s.c[j][0] = x[0];
        s.c[j][1] = x[1];
      }
    }
    if constexpr (KV == 0) s.ks = ((const uint8_t*)b)[scale_at];
    s.vs = ((const uint8_t*)b)[scale_at + kBlockSize];
  }
  // What the codes are multiplied by.  A token whose key or value is a NaN vector gets a key of NaN and a value of 0 (its codes): its score
  // makes NaN of every row that sees it, and 0 * NaN does not reach the others.
  template <int KV>
  static __device__ __forceinline__ float factor(const Codes<D>& s) {
    if constexpr (KV == 0) return __builtin_bit_cast(float, s.ks == 255u || s.vs == 255u ? 0x7fc00000u : s.ks << 23);
    else return __builtin_bit_cast(float, s.vs == 255u ? 0u : s.vs << 23);
  }
  // Piece K of kPieces of the store: 16 bytes of LDS (8 numbers).
  static constexpr int kPieces = D / 64;
  template <int K>
  __device__ __forceinline__ void store(const Codes<D>& s, float f, uint32_t base) const {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    constexpr int j = K / 2, w = 2 * (K % 2);
    const u32x4 o = {two_values<FMT, false>(s.c[j][w], f), two_values<FMT, true>(s.c[j][w], f), two_values<FMT, false>(s.c[j][w + 1], f),
                     two_values<FMT, true>(s.c[j][w + 1], f)};
    *(lds_u32x4*)(uintptr_t)(base + 2048u * j + (K % 2 ? lds_at ^ 16u : lds_at)) = o;
  }
};

}  // namespace q8
}  // namespace ic
