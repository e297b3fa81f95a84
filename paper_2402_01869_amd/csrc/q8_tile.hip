// Tile kernel of the 8-bit cache: the query rows of a recomputation chunk against their sequence's quantised keys, on the matrix cores
// (v_mfma_f32_32x32x16_bf16, fp32 accumulation).
//
// One workgroup = one TileItem x one head group: up to tile_rows(D) rows = query rows x heads of the group, a wave per 32 rows.  A tile of
// 64 keys is loaded as codes (16 bytes a lane), expanded to bf16 with its scales on the way into LDS, and shared by all waves:
// a code is converted once for 256 rows.  The expansion is exact (q8.h), so the rest is attention over a bf16 tile:
//   - S^T = K Q^T, A operand = 32 keys x 16 dims from LDS, B operand = the wave's Q^T in registers.  Every lane owns one query column and
//     16 of 32 keys.
//   - O^T += V^T P^T: the scores' registers, as bf16 weights, are the B operand; V^T comes from LDS by transpose loads.
//   - Running maximum and sum per column; the sum counts the weights as rounded to bf16 (2^-9 each: rows of fewer than 64 keys do
//     not run here), so the result stays a convex combination of the values.
// A vector of NaN (scale byte 255): the key of a token whose key or value is NaN is staged as NaN and its value as 0.  Every row that sees the
// token gets NaN by its score, and no other row does (0 * NaN would be NaN in rows that do not see it).
#include "q8.h"
#include "tile_body.h"

namespace ic {

namespace {

using namespace tilep;
using q8::kE4m3;
using q8::kInt8;

template <int D>
struct T8 {
  static constexpr int kWaves = tile_rows(D) / 32;
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kChunkRow = D / 16;                 // 16-code pieces of a key
  static constexpr int kPieces = kTileK * kChunkRow;       // ... of a tile of K, or of V
  static constexpr int kPer = 2 * kPieces / kThreads;      // pieces per thread
  static constexpr int kBuf = kTileK * (TG<D>::kKStride + TG<D>::kVStride);  // bf16 of a staged tile
  static_assert(2 * kPieces % kThreads == 0 && kPieces % 64 == 0, "whole waves take K or V");
};

template <int D>
struct Codes {
  u32x4 c[T8<D>::kPer];
  uint32_t ks[T8<D>::kPer], vs[T8<D>::kPer];
};

// Piece u of the tile: K for u < kPieces, V behind; key and part of the key.
template <int D>
__device__ __forceinline__ void fetch(Codes<D>& s, const char* pool, uint64_t block_bytes, const int (&ids)[4], int kvh, int Hk, int tid) {
  using T = T8<D>;
#pragma unroll
  for (int j = 0; j < T::kPer; ++j) {
    const int u = tid + T::kThreads * j;
    const bool is_v = u >= T::kPieces;
    const int uu = is_v ? u - T::kPieces : u;
    const int key = uu / T::kChunkRow, part = uu % T::kChunkRow;
    const int bsel = __builtin_amdgcn_readfirstlane(key / kBlockSize);  // a wave's pieces are of one block
    const char* base = pool + (uint64_t)(uint32_t)ids[bsel] * block_bytes;
    s.c[j] = *(const u32x4*)(base + (uint32_t)(((is_v ? Hk : 0) + kvh) * kBlockSize + key % kBlockSize) * D + part * 16);
    const uint8_t* sp = (const uint8_t*)base + 2u * Hk * kBlockSize * D + (uint32_t)kvh * 2u * kBlockSize + key % kBlockSize;
    s.ks[j] = sp[0];
    s.vs[j] = sp[kBlockSize];
  }
}

// Codes -> bf16 rows in LDS.  V of keys >= n_valid is zeroed (dead slots may hold anything).
template <int D, int FMT>
__device__ __forceinline__ void stage(const Codes<D>& s, uint16_t* ks, uint16_t* vs, int tid, int n_valid) {
  using T = T8<D>;
#pragma unroll
  for (int j = 0; j < T::kPer; ++j) {
    const int u = tid + T::kThreads * j;
    const bool is_v = __builtin_amdgcn_readfirstlane(u >= T::kPieces);
    const int uu = is_v ? u - T::kPieces : u;
    const int key = uu / T::kChunkRow, part = uu % T::kChunkRow;
    const bool bad = s.ks[j] == 255u || s.vs[j] == 255u;
    const float scale = __builtin_bit_cast(float, (is_v ? s.vs[j] : s.ks[j]) << 23);
    const bool fill = bad || (is_v && key >= n_valid);
    const uint32_t with = is_v ? 0u : q8::kNanBf16x2;
    u32x4 o[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = q8::two_values<FMT, false>(s.c[j][i], scale), b = q8::two_values<FMT, true>(s.c[j][i], scale);
      o[i / 2][2 * (i % 2)] = fill ? with : a;
      o[i / 2][2 * (i % 2) + 1] = fill ? with : b;
    }
    uint16_t* dst = is_v ? vs + key * TG<D>::kVStride + part * 16 : ks + key * TG<D>::kKStride + part * 16;
    *(u32x4*)dst = o[0];
    *(u32x4*)(dst + 8) = o[1];
  }
}

// One 64-key tile for one wave.  mask: the tile straddles the wave's diagonal, or ends behind the item's last key.
template <int D>
__device__ __forceinline__ void wave_step(const uint16_t* ks, const uint16_t* vs, const bf16x8 (&q)[TG<D>::kQSteps], f32x16 (&acc)[TG<D>::kDTiles],
                                          float& m, float& l, int kt, int pos, int col, int hl, float sc, bool mask) {
  using G = TG<D>;
  f32x16 s[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
  {
    const uint16_t* kp0 = ks + col * G::kKStride + 8 * hl;
    const uint16_t* kp1 = kp0 + 32 * G::kKStride;
#pragma unroll
    for (int k = 0; k < G::kQSteps; ++k) {
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kp0 + 16 * k), q[k], s[0], 0, 0, 0);
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kp1 + 16 * k), q[k], s[1], 0, 0, 0);
    }
  }
  if (mask) {  // wave-uniform; the empty asm keeps this a branch
    asm volatile("" ::: "memory");
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kt + 32 * tt + 8 * (i / 4) + 4 * hl + (i % 4);
        s[tt][i] = key > pos ? -__builtin_inff() : s[tt][i];
      }
  }
  float top = -__builtin_inff();
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, s[tt][i]);
  top *= sc;
  if (__builtin_amdgcn_ballot_w64(top > m + kLazyLog2) != 0) {
    top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    const float m_new = top > m + kLazyLog2 ? top : m;  // the same in both lanes of a column
    const float was = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= was;
#pragma unroll
    for (int dt = 0; dt < G::kDTiles; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[dt][i] *= was;
  }
  float sum = 0.f;
  bf16x8 pw[4];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i], sc, -m));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tt][i + 1], sc, -m));
      const bf16x2 pr = {(__bf16)p0, (__bf16)p1};
      sum += (float)pr[0] + (float)pr[1];
      pw[2 * tt + i / 8][i % 8] = pr[0];
      pw[2 * tt + i / 8][i % 8 + 1] = pr[1];
    }
  l += sum;
  const int lane = col + 32 * hl;
#pragma unroll
  for (int ksp = 0; ksp < 4; ++ksp)
#pragma unroll
    for (int dt = 0; dt < G::kDTiles; ++dt)
      acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_vt_operand<D>(vs, 32 * dt, ksp, lane), pw[ksp], acc[dt], 0, 0, 0);
}

template <int D, int FMT>
__device__ __forceinline__ void q8_tile_body(const AttnParams& p, const TileItem& it, int th, uint16_t* lds) {
  using G = TG<D>;
  using T = T8<D>;
  const int H = p.num_heads, Hk = p.num_kv_heads;
  const int gs = p.tile_g_shift;
  const int head0 = th << gs;
  const int kvh = head0 / p.group;
  const int n_rows_t = it.n_rows << gs;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hl = lane >> 5;
  const int r = 32 * w + col, r_eff = min(r, n_rows_t - 1);  // dead rows mirror the last live one
  const int pos = it.pos0 + (r_eff >> gs);                   // last key the row sees
  const int wave_lo = it.pos0 + min((32 * w) >> gs, it.n_rows - 1), wave_hi = it.pos0 + min((32 * w + 31) >> gs, it.n_rows - 1);
  bf16x8 q[G::kQSteps];
  {
    const uint16_t* qp = p.q + ((int64_t)(it.qrow0 + (r_eff >> gs)) * H + head0 + (r_eff & ((1 << gs) - 1))) * D + 8 * hl;
#pragma unroll
    for (int k = 0; k < G::kQSteps; ++k) q[k] = *(const bf16x8*)(qp + 16 * k);
  }
  f32x16 acc[G::kDTiles];
#pragma unroll
  for (int dt = 0; dt < G::kDTiles; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
  float m = kNegBig, l = 0.f;

  typedef __attribute__((address_space(4))) const int32_t const_i32;
  const_i32* bt = (const_i32*)(p.bt_flat + p.bt_off[it.seq]);
  const int last_blk = (it.k_end - 1) / kBlockSize;  // last table entry this item may touch
  const int n_tiles = (it.k_end - it.k_begin + kTileK - 1) / kTileK;
  const float sc = p.scale_log2e;
  const char* pool = (const char*)p.pool;
  // Tiles past the item's end re-read its last block and are never staged.
  const auto fetch_tile = [&](Codes<D>& s, int t) __attribute__((always_inline)) {
    int ids[4];
    const int b0 = (it.k_begin + t * kTileK) / kBlockSize;
#pragma unroll
    for (int i = 0; i < 4; ++i) ids[i] = bt[min(b0 + i, last_blk)];
    fetch<D>(s, pool, p.block_bytes, ids, kvh, Hk, tid);
  };
  // Two buffers in LDS, one tile in registers: step t computes on buffer t % 2, puts tile t + 1 into the other one and loads tile t + 2.
  Codes<D> s;
  fetch_tile(s, 0);
  stage<D, FMT>(s, lds, lds + kTileK * G::kKStride, tid, it.k_end - it.k_begin);
  fetch_tile(s, 1);
  __syncthreads();
  for (int t = 0; t < n_tiles; ++t) {
    const int kt = it.k_begin + t * kTileK;
    const uint16_t* ks = lds + (t & 1) * T::kBuf;
    uint16_t* nks = lds + ((t + 1) & 1) * T::kBuf;
    if (kt <= wave_hi) wave_step<D>(ks, ks + kTileK * G::kKStride, q, acc, m, l, kt, min(pos, it.k_end - 1), col, hl, sc, kt + kTileK - 1 > min(wave_lo, it.k_end - 1));
    if (t + 1 < n_tiles) {
      stage<D, FMT>(s, nks, nks + kTileK * G::kKStride, tid, it.k_end - (kt + kTileK));
      fetch_tile(s, t + 2);
    }
    __syncthreads();
  }

  // lane: O^T[d][col], d = 32 dt + 8 (i / 4) + 4 hl + i % 4
  l += __shfl_xor(l, 32);
  if (r < n_rows_t) {
    const int qr = r >> gs, head = head0 + (r & ((1 << gs) - 1));
    if (it.slot0 < 0) {
      const float inv = 1.0f / l;
      uint16_t* op = p.out + ((int64_t)(it.qrow0 + qr) * H + head) * D;
#pragma unroll
      for (int dt = 0; dt < G::kDTiles; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          bf16x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[dt][4 * g + e] * inv);  // round to nearest even
          *(bf16x4*)(op + 32 * dt + 8 * g + 4 * hl) = o;
        }
    } else {
      const int64_t ps = (int64_t)(it.slot0 + qr * it.nparts) * H + head;
      float* op = p.part_o + ps * D;
#pragma unroll
      for (int dt = 0; dt < G::kDTiles; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f32x4*)(op + 32 * dt + 8 * g + 4 * hl) = (f32x4){acc[dt][4 * g], acc[dt][4 * g + 1], acc[dt][4 * g + 2], acc[dt][4 * g + 3]};
      if (hl == 0) {
        p.part_ml[ps * 2] = m;
        p.part_ml[ps * 2 + 1] = l;
      }
    }
  }
}

template <int D, int FMT>
__global__ __launch_bounds__(T8<D>::kThreads, D <= 128 ? 2 : 1) void q8_tile_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[2 * T8<D>::kBuf];
  const uint32_t n_th = (uint32_t)p.num_heads >> p.tile_g_shift;  // head groups, each served by one workgroup per item
  const uint32_t item = blockIdx.x / n_th;
  const TileItem it = p.tile_items[item];
  q8_tile_body<D, FMT>(p, it, (int)(blockIdx.x - item * n_th), lds);
}

}  // namespace

hipError_t launch_q8_tile(const AttnParams& p, int head_dim, int dtype, hipStream_t st) {
  if (p.n_tile_items <= 0) return hipSuccess;
  const uint64_t grid = (uint64_t)p.n_tile_items * (uint64_t)(p.num_heads >> p.tile_g_shift);
  if (grid > 0x7fffffffull || (dtype != kE4m3 && dtype != kInt8)) return hipErrorInvalidValue;
  const dim3 g((uint32_t)grid);
#define IC_Q8_TILE(DD)                                                                                             \
  case DD:                                                                                                         \
    if (dtype == kE4m3) hipLaunchKernelGGL((q8_tile_kernel<DD, kE4m3>), g, dim3(T8<DD>::kThreads), 0, st, p);       \
    else hipLaunchKernelGGL((q8_tile_kernel<DD, kInt8>), g, dim3(T8<DD>::kThreads), 0, st, p);                      \
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
