// Row kernel of the 8-bit cache: query rows that are few for their keys.  Decode rows of every pool (Section 4.2: one query token,
// every cached vector read once), short chunks, and the rows of a fresh chunk that see fewer than 64 keys.
//
// One workgroup = one row item (up to 16 columns: consecutive query rows of a sequence x the query heads of a K/V head) x one K/V head,
// 4 waves, wave w the item's 32-key tiles w, w + 4, ...  HBM-bound: a byte of the cache is read once and meets all columns.
// Codes become MFMA operands in registers; nothing is staged:
//   - S^T = K Q^T (16x16x32): a lane's A operand is 8 numbers of one key.  It loads 16 bytes of the key, two operands; which dims
//     an operand's 8 places are does not matter as long as Q^T has the same, so Q is loaded in that order.  The accumulator
//     then has 4 keys of one column in a lane, for each of the tile's two blocks.
//   - Codes are exact in bf16 and the scale of a key is a power of two, so it multiplies the key's score in fp32, and the
//     weight of the key's value, instead of the codes: 16 products a tile and lane instead of one per number.
//   - O^T += V^T P^T: a lane's 8 weights ARE the B operand if its A operand has the same 8 keys: a lane loads its dims of those
//     8 keys (D / 16 bytes each), and the bytes of two keys are paired by v_perm on their way to bf16.  Rows of V^T are
//     dims in the order that falls out: row n of product (w, b) is dim n * D / 16 + 4 w + b.
//   - Weights go in as two bf16 numbers (16 bits of significand; the rounding of one, 2^-9, would show in rows of a few keys): the
//     matrix pipe has the time.  The normaliser is the fp32 sum of the unrounded weights, what is lost is 2^-17 of a weight.
// Keys a column does not see: score -inf, weight 0, and 0 for the scale of their value, which may be infinite (NaN vectors); codes
// behind the item's last key are cleared, they may be anything (0 * NaN).
#include "merge_body.h"
#include "q8.h"

namespace ic {

namespace {

using namespace q8;

constexpr int kWaves = 4;
constexpr int kKeys = 32;  // of a wave's tile: two blocks
constexpr int kCols = 16;
constexpr float kNegBig = -1.0e30f;
constexpr float kLazyLog2 = 8.0f;  // slack of the running maximum, in log2 units: below it nothing is rescaled

template <int D>
struct R8 {
  static constexpr int kKL = D / 64;     // 16-byte loads of a key block per lane; MFMA steps of Q K^T are twice as many
  static constexpr int kVW = D / 64;     // dwords of a key's value per lane
  static constexpr int kDT = D / 16;     // products of V^T P^T
  static constexpr int kSlice = kCols * D + 2 * kCols;  // floats of one wave's result in LDS
};

template <int N> struct Words { typedef __attribute__((ext_vector_type(N))) uint32_t type; };
template <> struct Words<1> { typedef uint32_t type; };

template <int D>
struct Tile {
  u32x4 k[2][R8<D>::kKL];
  uint32_t ks[2];
  uint32_t v[8][R8<D>::kVW];
  uint32_t vs[2];
};

// Where a lane reads in a block: 16 g bytes into key n (K), dims of n of key 4 g (V), scale bytes of keys 4 g ..+3.
struct Place {
  const char* pool;      // base of the pool
  uint64_t block_bytes;
  uint32_t k_at, v_at, ks_at;  // offsets inside a block
};

template <int D>
__device__ __forceinline__ void load_k(Tile<D>& t, const Place& at, int id0, int id1) {
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const char* base = at.pool + (uint64_t)(uint32_t)(b ? id1 : id0) * at.block_bytes;
#pragma unroll
    for (int j = 0; j < R8<D>::kKL; ++j) t.k[b][j] = __builtin_nontemporal_load((const u32x4*)(base + at.k_at + 64 * j));
    t.ks[b] = *(const uint32_t*)(base + at.ks_at);
  }
}
template <int D>
__device__ __forceinline__ void load_v(Tile<D>& t, const Place& at, int id0, int id1) {
  typedef typename Words<R8<D>::kVW>::type words;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const char* base = at.pool + (uint64_t)(uint32_t)(b ? id1 : id0) * at.block_bytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const words x = __builtin_nontemporal_load((const words*)(base + at.v_at + i * D));
      if constexpr (R8<D>::kVW == 1) t.v[4 * b + i][0] = x;
      else
#pragma unroll
        for (int e = 0; e < R8<D>::kVW; ++e) t.v[4 * b + i][e] = x[e];
    }
    t.vs[b] = *(const uint32_t*)(base + at.ks_at + kBlockSize);
  }
}

// Byte B of two keys' words as a pair of bf16.
template <int FMT, int B>
__device__ __forceinline__ uint32_t pair_of(uint32_t first, uint32_t second) {
  if constexpr (FMT == kE4m3) {
    return two_codes<FMT, (B & 1) != 0>(__builtin_amdgcn_perm(second, first, B < 2 ? 0x05010400u : 0x07030602u));
  } else {
    const float a = (float)(int)(int8_t)(first >> (8 * B)), b = (float)(int)(int8_t)(second >> (8 * B));
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
  }
}

template <int FMT, int B, int D>
__device__ __forceinline__ bf16x8 value_operand(const Tile<D>& t, int w) {
  const u32x4 x = {pair_of<FMT, B>(t.v[0][w], t.v[1][w]), pair_of<FMT, B>(t.v[2][w], t.v[3][w]), pair_of<FMT, B>(t.v[4][w], t.v[5][w]),
                   pair_of<FMT, B>(t.v[6][w], t.v[7][w])};
  return __builtin_bit_cast(bf16x8, x);
}

__device__ __forceinline__ f32x4 mfma(const bf16x8 a, const bf16x8 b, const f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// kMerge: split decode rows are merged by their last partition, else by the merge kernel.
template <int D, int FMT, bool kMerge>
__global__ __launch_bounds__(64 * kWaves, D <= 128 ? 3 : 2) void q8_rows_kernel(AttnParams p) {
  using R = R8<D>;
  __shared__ __attribute__((aligned(16))) float lds[kWaves * R::kSlice];
  __shared__ int s_last;
  const uint32_t item_idx = blockIdx.x / (uint32_t)p.row_units;
  const int unit = (int)(blockIdx.x - item_idx * (uint32_t)p.row_units);
  const RowItem it = p.row_items[p.group_first + item_idx];
  const int n_rows = it.pad[0], pos0 = it.pad[1], nparts = it.pad[2];
  const int H = p.num_heads, Hk = p.num_kv_heads, G = p.group;
  const int subs = p.row_units / Hk;             // units of a K/V head: more than one where a group has more than 16 heads
  const int kvh = unit / subs, first = (unit - kvh * subs) * kCols;
  const int head0 = kvh * G + first, heads = min(kCols, G - first);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int cols = n_rows * heads;               // columns that are rows of the result, <= 16
  const int col = min(n, cols - 1);              // the others mirror the last one
  const int row = col / heads, head = head0 + (col - row * heads);
  const int limit = min(pos0 + row + 1, it.k_end);  // keys the column sees are below
  const int least = min(pos0 + 1, it.k_end);        // ... and every column's are at least these

  bf16x8 q[2 * R::kKL];
  {
    const uint16_t* qp = p.q + ((int64_t)(it.qrow + row) * H + head) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < R::kKL; ++j) {
      q[2 * j] = *(const bf16x8*)(qp + 64 * j);
      q[2 * j + 1] = *(const bf16x8*)(qp + 64 * j + 8);
    }
  }
  f32x4 o[R::kDT];
#pragma unroll
  for (int i = 0; i < R::kDT; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = kNegBig, l = 0.f;

  typedef __attribute__((address_space(4))) const int32_t const_i32;
  const_i32* bt = (const_i32*)(p.bt_flat + p.bt_off[it.seq]);
  const int last_blk = (it.k_end - 1) / kBlockSize;
  const int n_tiles = (it.k_end - it.k_begin + kKeys - 1) / kKeys;
  const float sc = p.scale_log2e;
  Place at;
  at.pool = (const char*)p.pool;
  at.block_bytes = p.block_bytes;
  at.k_at = (uint32_t)(kvh * kBlockSize + n) * D + 16u * g;
  at.v_at = (uint32_t)((Hk + kvh) * kBlockSize + 4 * g) * D + (uint32_t)n * (D / 16);
  at.ks_at = 2u * Hk * kBlockSize * D + (uint32_t)kvh * 2u * kBlockSize + 4u * g;

  Tile<D> t;
  const auto block0 = [&](int tile) { return bt[it.k_begin / kBlockSize + 2 * tile]; };
  const auto block1 = [&](int tile) { return bt[min(it.k_begin / kBlockSize + 2 * tile + 1, last_blk)]; };

  const auto step = [&](auto more_tag, int tile) __attribute__((always_inline)) {
    constexpr bool kMore = decltype(more_tag)::value;
    const int kt = it.k_begin + tile * kKeys;
    int id0 = 0, id1 = 0;
    if constexpr (kMore) {
      id0 = block0(tile + kWaves);
      id1 = block1(tile + kWaves);
    }
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int j = 0; j < R::kKL; ++j)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t x = t.k[b][j][2 * half], y = t.k[b][j][2 * half + 1];
          const u32x4 a = {two_codes<FMT, false>(x), two_codes<FMT, true>(x), two_codes<FMT, false>(y), two_codes<FMT, true>(y)};
          s[b] = mfma(__builtin_bit_cast(bf16x8, a), q[2 * j + half], s[b]);
        }
    float x[8], vf[8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[4 * b] = s[b][0] * (scale_of<0>(t.ks[b]) * sc);
      x[4 * b + 1] = s[b][1] * (scale_of<1>(t.ks[b]) * sc);
      x[4 * b + 2] = s[b][2] * (scale_of<2>(t.ks[b]) * sc);
      x[4 * b + 3] = s[b][3] * (scale_of<3>(t.ks[b]) * sc);
      vf[4 * b] = scale_of<0>(t.vs[b]);
      vf[4 * b + 1] = scale_of<1>(t.vs[b]);
      vf[4 * b + 2] = scale_of<2>(t.vs[b]);
      vf[4 * b + 3] = scale_of<3>(t.vs[b]);
    }
    if constexpr (kMore) load_k<D>(t, at, id0, id1);
    if (kt + kKeys > least) {  // wave-uniform
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = kt + 16 * (i / 4) + 4 * g + i % 4;
        x[i] = key < limit ? x[i] : -__builtin_inff();
        vf[i] = key < limit ? vf[i] : 0.f;
#pragma unroll
        for (int e = 0; e < R::kVW; ++e) t.v[i][e] = key < it.k_end ? t.v[i][e] : 0u;
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = __builtin_fmaxf(top, x[i]);
    // the running maximum moves, and the sums with it, only when some score is over it by more than kLazyLog2
    if (__builtin_amdgcn_ballot_w64(top > m + kLazyLog2) != 0) {
      top = __builtin_fmaxf(top, __shfl_xor(top, 16));
      top = __builtin_fmaxf(top, __shfl_xor(top, 32));
      const float m_new = top > m + kLazyLog2 ? top : m;  // the same in the four lanes of a column
      const float was = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= was;
#pragma unroll
      for (int i = 0; i < R::kDT; ++i) o[i] *= was;
    }
    u32x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(x[i] - m), p1 = __builtin_amdgcn_exp2f(x[i + 1] - m);
      l += p0 + p1;
      const float a = p0 * vf[i], b = p1 * vf[i + 1];
      const bf16x2 h = {(__bf16)a, (__bf16)b};
      const uint32_t hb = __builtin_bit_cast(uint32_t, h);
      const bf16x2 r = {(__bf16)(a - __builtin_bit_cast(float, hb << 16)), (__bf16)(b - __builtin_bit_cast(float, hb & 0xffff0000u))};
      hi[i / 2] = hb;
      lo[i / 2] = __builtin_bit_cast(uint32_t, r);
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
#pragma unroll
    for (int e = 0; e < R::kVW; ++e) {
      const bf16x8 a0 = value_operand<FMT, 0, D>(t, e), a1 = value_operand<FMT, 1, D>(t, e);
      const bf16x8 a2 = value_operand<FMT, 2, D>(t, e), a3 = value_operand<FMT, 3, D>(t, e);
      o[4 * e] = mfma(a0, ph, o[4 * e]);
      o[4 * e + 1] = mfma(a1, ph, o[4 * e + 1]);
      o[4 * e + 2] = mfma(a2, ph, o[4 * e + 2]);
      o[4 * e + 3] = mfma(a3, ph, o[4 * e + 3]);
      o[4 * e] = mfma(a0, pl, o[4 * e]);
      o[4 * e + 1] = mfma(a1, pl, o[4 * e + 1]);
      o[4 * e + 2] = mfma(a2, pl, o[4 * e + 2]);
      o[4 * e + 3] = mfma(a3, pl, o[4 * e + 3]);
    }
    if constexpr (kMore) load_v<D>(t, at, id0, id1);
  };

  if (w < n_tiles) {
    const int id0 = block0(w), id1 = block1(w);
    load_k<D>(t, at, id0, id1);
    load_v<D>(t, at, id0, id1);
    int tile = w;
    for (; tile + kWaves < n_tiles; tile += kWaves) step(std::true_type{}, tile);
    step(std::false_type{}, tile);
  }

  // ---- the waves' results meet in LDS: O^T as [column][dim], then (m, l) of every column
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  float* const mine = lds + w * R::kSlice;
  if (n < cols) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < R::kVW; ++e)
        *(f32x4*)(mine + n * D + (4 * g + r) * (D / 16) + 4 * e) = (f32x4){o[4 * e][r], o[4 * e + 1][r], o[4 * e + 2][r], o[4 * e + 3][r]};
    if (g == 0) {
      mine[kCols * D + 2 * n] = m;
      mine[kCols * D + 2 * n + 1] = l;
    }
  }
  __syncthreads();
  for (int idx = tid; idx < cols * D; idx += 64 * kWaves) {
    const int c = idx / D, d = idx % D;
    float M = kNegBig;
#pragma unroll
    for (int ww = 0; ww < kWaves; ++ww) M = __builtin_fmaxf(M, lds[ww * R::kSlice + kCols * D + 2 * c]);
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int ww = 0; ww < kWaves; ++ww) {
      const float* sl = lds + ww * R::kSlice;
      const float wgt = __builtin_amdgcn_exp2f(sl[kCols * D + 2 * c] - M);
      L = __builtin_fmaf(sl[kCols * D + 2 * c + 1], wgt, L);
      O = __builtin_fmaf(sl[c * D + d], wgt, O);
    }
    const int r = c / heads, h = head0 + (c - r * heads);
    if (it.slot < 0) {
      const __bf16 v = (__bf16)(O / L);  // round to nearest even
      p.out[((int64_t)(it.qrow + r) * H + h) * D + d] = __builtin_bit_cast(uint16_t, v);
    } else {
      const int64_t ps = (int64_t)(it.slot + r * nparts) * H + h;
      mergep::store_shared(&p.part_o[ps * D + d], O);
      if (d == 0) {
        mergep::store_shared(&p.part_ml[ps * 2], M);
        mergep::store_shared(&p.part_ml[ps * 2 + 1], L);
      }
    }
  }
  if constexpr (kMerge) {
    if (it.slot >= 0 && nparts == 0) mergep::finish_split<D, 4>(p, it.slot, unit, head0, heads, &s_last);
  }
}

template <int D, int FMT>
void launch(const AttnParams& p, dim3 grid, hipStream_t st) {
  const dim3 b(64 * kWaves);
  if (p.split_units > 0) hipLaunchKernelGGL((q8_rows_kernel<D, FMT, true>), grid, b, 0, st, p);
  else hipLaunchKernelGGL((q8_rows_kernel<D, FMT, false>), grid, b, 0, st, p);
}

}  // namespace

hipError_t launch_q8_rows(const AttnParams& p, int head_dim, int dtype, hipStream_t st) {
  const int n_items = p.n_row_items - p.group_first;
  if (n_items <= 0) return hipSuccess;
  if (p.row_units < p.num_kv_heads || p.row_units % p.num_kv_heads != 0 || p.row_units / p.num_kv_heads * kCols < p.group) return hipErrorInvalidValue;
  const uint64_t grid = (uint64_t)n_items * (uint64_t)p.row_units;
  if (grid > 0x7fffffffull) return hipErrorInvalidValue;
  const dim3 g((uint32_t)grid);
  if (dtype != kE4m3 && dtype != kInt8) return hipErrorInvalidValue;
  const bool e4m3 = dtype == kE4m3;
  switch (head_dim) {
    case 64: e4m3 ? launch<64, kE4m3>(p, g, st) : launch<64, kInt8>(p, g, st); break;
    case 128: e4m3 ? launch<128, kE4m3>(p, g, st) : launch<128, kInt8>(p, g, st); break;
    case 256: e4m3 ? launch<256, kE4m3>(p, g, st) : launch<256, kInt8>(p, g, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ic
