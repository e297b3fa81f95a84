// An 8-bit pool's way in and out: kv_write_span quantises the rows that a chunk or a decode token has just computed as it writes them
// through the block table, kv_read_span reads cached positions back as bf16 rows (of a bf16 pool: as they are).
//
// Both are byte movement: 2 Hkv (2 D + D + 1) bytes a token.  One lane has 8 numbers of a vector, 16 bytes of bf16 and 8 of codes, so that
// what a wave loads or stores of the bf16 rows with one instruction is contiguous; a vector is D / 8 adjacent lanes, whose largest
// magnitude is found by exchanges inside the group.  A lane does that for 4 consecutive rows, all asked for at once: waves start at
// some 3.2 a ns, which at 1.5 KiB each (one row) is 4.9 TB/s.  Measured, e4m3, 40 heads of 128: 17143 rows read back 109 us with
// one row a lane, 102 with two, 95 with four (5.6 TB/s), 98 with eight; 16 numbers a lane and one row, 98; 8320 rows (256 MB)
// written 42 -> 41 us, read back 42 -> 41 (16 numbers a lane: 57).
#include <algorithm>

#include "q8.h"

namespace ic {

namespace {

using namespace q8;

constexpr int kThreads = 64;  // one-wave workgroups, as for the block moves
constexpr int kRows = 4;  // consecutive rows of a lane

// The largest magnitude of 8 bf16 numbers, as their bits without the sign: for finite numbers, infinities and NaN alike a
// larger number is a larger magnitude, and everything from 0x7f80 on is infinite or NaN.
__device__ __forceinline__ uint32_t largest_bits(const u32x4 a) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max(a[i] & 0x7fffu, a[i] >> 16 & 0x7fffu));
  return m;
}
template <int kCtrl>
__device__ __forceinline__ uint32_t with_dpp(uint32_t m) {
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, kCtrl, 0xf, 0xf, true));
}
// ... of 8, 16 or 32 adjacent lanes, in all of them.
template <int kLanes>
__device__ __forceinline__ uint32_t largest_of_group(uint32_t m) {
  m = with_dpp<0xb1>(m);   // lane ^ 1
  m = with_dpp<0x4e>(m);   // lane ^ 2
  m = with_dpp<0x141>(m);  // 7 - lane of 8
  if constexpr (kLanes >= 16) m = with_dpp<0x140>(m);  // 15 - lane of 16
  if constexpr (kLanes >= 32) m = max(m, (uint32_t)__shfl_xor((int)m, 16));
  return m;
}

// Scale byte of a vector whose largest magnitude has these bf16 bits.  a = (1 + f / 128) 2^E; top = 1.75 * 2^8 or (1 + 126 / 128) * 2^6, so e is
// E - 8 (6), one more where f is over 96 (126).  A subnormal a counts as E = -127, below every exponent kept.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  if (bits >= 0x7f80u) return 255u;
  const int E = (int)(bits >> 7), f = (int)(bits & 127u);  // E with its bias of 127
  const int b = FMT == kE4m3 ? E - 8 + (f > 96) : E - 6 + (f > 126);
  return (uint32_t)max(b, 27);
}

// The largest numbers under the largest scale round to 2^128, which bf16 does not hold: e4m3, e = 120, from 248 * 2^120 on (codes of 256), integers,
// e = 122, from 63.5 * 2^122 on (codes of 64).  They are lowered to the bf16 number below those, which rounds to the code below.  (As
// they came they would be read as infinity, and weight 0 times infinity is NaN: a row that does not see the key would have it too.)
template <int FMT>
constexpr uint32_t kLastScale = FMT == kE4m3 ? 247u : 249u;
template <int FMT>
__device__ __forceinline__ uint32_t kept_finite(uint32_t x) {
  constexpr uint32_t kMost = FMT == kE4m3 ? 0x7f77u : 0x7f7du;
  return (x & 0x80008000u) | min(x & 0x7fffu, kMost) | min(x >> 16 & 0x7fffu, kMost) << 16;
}

// Four numbers (two pairs of bf16) as codes; scale = 2^e, inv = 2^-e.
template <int FMT>
__device__ __forceinline__ uint32_t four_codes(uint32_t x, uint32_t y, float scale, float inv) {
  if constexpr (FMT == kE4m3) {
    s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, x), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, y), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  } else {
    // x / 2^e + 1.5 * 2^23 rounds to a whole number, ties to even, whose low byte is the code's
    constexpr float kWhole = 12582912.0f;
    const uint32_t c0 = __builtin_bit_cast(uint32_t, __builtin_fmaf(__builtin_bit_cast(float, x << 16), inv, kWhole));
    const uint32_t c1 = __builtin_bit_cast(uint32_t, __builtin_fmaf(__builtin_bit_cast(float, x & 0xffff0000u), inv, kWhole));
    const uint32_t c2 = __builtin_bit_cast(uint32_t, __builtin_fmaf(__builtin_bit_cast(float, y << 16), inv, kWhole));
    const uint32_t c3 = __builtin_bit_cast(uint32_t, __builtin_fmaf(__builtin_bit_cast(float, y & 0xffff0000u), inv, kWhole));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(c3, c2, 0x0c0c0400u), __builtin_amdgcn_perm(c1, c0, 0x0c0c0400u), 0x05040100u);
  }
}

// What a lane has: 8 numbers of the same head's key or value of rows row .. row + kRows - 1.
template <int D>
struct Piece {
  static constexpr uint32_t kLanes = D / 8;  // of a vector
  uint32_t row, kv, head, part;
  __device__ __forceinline__ explicit Piece(uint32_t num_heads) {
    const uint64_t idx = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const uint32_t per_row = 2u * num_heads * kLanes;
    const uint64_t r = idx / per_row;
    row = (uint32_t)r * kRows;
    const uint32_t rem = (uint32_t)(idx - r * per_row);
    const uint32_t vec = rem / kLanes;
    part = rem % kLanes;
    kv = vec >= num_heads;
    head = vec - (kv ? num_heads : 0u);
  }
  // byte offset of the lane's 8 numbers of row + u among the rows of k_new, v_new, k_out or v_out
  __device__ __forceinline__ uint64_t row_at(uint32_t num_heads, int u) const { return (((uint64_t)(row + u) * num_heads + head) * D + part * 8u) * 2u; }
  __device__ __forceinline__ uint32_t code_at(uint32_t num_heads, uint32_t slot) const {
    return ((kv * num_heads + head) * kBlockSize + slot) * D + part * 8u;
  }
  __device__ __forceinline__ uint32_t scale_at(uint32_t num_heads, uint32_t slot) const {
    return 2u * num_heads * kBlockSize * D + (head * 2u + kv) * kBlockSize + slot;
  }
};

template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void q8_write_kernel(char* __restrict__ pool, uint64_t block_bytes, const char* __restrict__ k_new,
                                                           const char* __restrict__ v_new, const int32_t* __restrict__ dst, uint32_t rows,
                                                           uint32_t num_heads) {
  const Piece<D> at(num_heads);
  int32_t d[kRows];
  u32x4 a[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const bool live = at.row + u < rows;  // the lanes of a vector have the same rows
    d[u] = live ? dst[at.row + u] : -1;
    a[u] = (u32x4){0u, 0u, 0u, 0u};
    // (loaded beside the destination, not after it: the row is there whoever owns it)
    if (live) a[u] = __builtin_nontemporal_load((const u32x4*)((at.kv ? v_new : k_new) + at.row_at(num_heads, u)));
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const uint32_t sb = scale_byte<FMT>(largest_of_group<(int)Piece<D>::kLanes>(largest_bits(a[u])));
    if (d[u] < 0) continue;
    uint32_t x[4] = {a[u][0], a[u][1], a[u][2], a[u][3]};
    if (sb == kLastScale<FMT>) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = kept_finite<FMT>(x[i]);
    }
    const float scale = __builtin_bit_cast(float, sb << 23), inv = __builtin_bit_cast(float, (254u - sb) << 23);
    u32x2 c = {four_codes<FMT>(x[0], x[1], scale, inv), four_codes<FMT>(x[2], x[3], scale, inv)};
    if (sb == 255u) c = (u32x2){0u, 0u};
    const uint32_t blk = (uint32_t)d[u] / (uint32_t)kBlockSize, slot = (uint32_t)d[u] % (uint32_t)kBlockSize;
    char* base = pool + blk * block_bytes;
    *(u32x2*)(base + at.code_at(num_heads, slot)) = c;
    if (at.part == 0) base[at.scale_at(num_heads, slot)] = (char)sb;
  }
}

template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void q8_read_kernel(const char* __restrict__ pool, uint64_t block_bytes, char* __restrict__ k_out,
                                                          char* __restrict__ v_out, const int32_t* __restrict__ src, uint32_t rows,
                                                          uint32_t num_heads) {
  const Piece<D> at(num_heads);
  int32_t d[kRows];
  u32x2 c[kRows];
  uint32_t sb[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) d[u] = at.row + u < rows ? src[at.row + u] : -1;
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    if (d[u] < 0) continue;
    const uint32_t blk = (uint32_t)d[u] / (uint32_t)kBlockSize, slot = (uint32_t)d[u] % (uint32_t)kBlockSize;
    const char* base = pool + blk * block_bytes;
    c[u] = __builtin_nontemporal_load((const u32x2*)(base + at.code_at(num_heads, slot)));
    sb[u] = (uint8_t)base[at.scale_at(num_heads, slot)];
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    if (d[u] < 0) continue;
    const bool bad = sb[u] == 255u;
    const float scale = __builtin_bit_cast(float, bad ? 0x3f800000u : sb[u] << 23);
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o[2 * i] = bad ? kNanBf16x2 : two_values<FMT, false>(c[u][i], scale);
      o[2 * i + 1] = bad ? kNanBf16x2 : two_values<FMT, true>(c[u][i], scale);
    }
    __builtin_nontemporal_store(o, (u32x4*)((at.kv ? v_out : k_out) + at.row_at(num_heads, u)));
  }
}

// The rows of a bf16 pool, 16 bytes a lane: the append the other way round.
template <int D>
__global__ __launch_bounds__(kThreads) void kv_gather_kernel(const char* __restrict__ pool, char* __restrict__ k_out, char* __restrict__ v_out,
                                                            const int32_t* __restrict__ src, uint32_t rows, uint32_t num_heads) {
  constexpr uint32_t kChunksPerHead = D / 8;
  const uint32_t per_plane = num_heads * kChunksPerHead;
  const uint64_t idx = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  const uint64_t row = idx / (2u * per_plane);
  if (row >= rows) return;
  const uint32_t rem = (uint32_t)(idx - row * (2u * per_plane));
  const uint32_t kv = rem / per_plane, c = rem - kv * per_plane;
  const uint32_t h = c / kChunksPerHead, cc = c % kChunksPerHead;
  const int32_t d = src[row];
  if (d < 0) return;
  const uint32_t blk = (uint32_t)d / (uint32_t)kBlockSize, slot = (uint32_t)d % (uint32_t)kBlockSize;
  const char* from = pool + ((((uint64_t)blk * 2u + kv) * num_heads + h) * kBlockSize + slot) * (D * 2) + cc * 16u;
  char* out = (kv ? v_out : k_out) + (row * per_plane + c) * 16u;
  __builtin_nontemporal_store(__builtin_nontemporal_load((const u32x4*)from), (u32x4*)out);
}

template <int D>
hipError_t move_rows(void* pool, size_t block_bytes, int dtype, bool write, void* k_rows, void* v_rows, const int32_t* dev_rows, int32_t rows, int heads,
                     hipStream_t st) {
  // 8 numbers a lane, of one row (bf16 pools) or of a set of kRows (8-bit pools)
  const uint64_t set = dtype == IC_DTYPE_BF16 ? 1 : kRows, lanes = 2u * (uint64_t)heads * (uint64_t)(D / 8);
  const uint64_t most = (kMaxLaunchThreads / lanes - 1) * set;  // rows of a launch; -1: whole workgroups
  for (uint64_t r = 0; r < (uint64_t)rows; r += most) {
    const uint32_t n = (uint32_t)std::min<uint64_t>(most, (uint64_t)rows - r), h = (uint32_t)heads;
    const dim3 g((uint32_t)(((n + set - 1) / set * lanes + kThreads - 1) / kThreads)), b(kThreads);
    char *k = (char*)k_rows + r * lanes * 8, *v = (char*)v_rows + r * lanes * 8;
    const int32_t* at = dev_rows + r;
    if (dtype == IC_DTYPE_BF16) hipLaunchKernelGGL(kv_gather_kernel<D>, g, b, 0, st, (const char*)pool, k, v, at, n, h);
    else if (dtype == kE4m3 && write) hipLaunchKernelGGL((q8_write_kernel<D, kE4m3>), g, b, 0, st, (char*)pool, block_bytes, k, v, at, n, h);
    else if (dtype == kE4m3) hipLaunchKernelGGL((q8_read_kernel<D, kE4m3>), g, b, 0, st, (const char*)pool, block_bytes, k, v, at, n, h);
    else if (write) hipLaunchKernelGGL((q8_write_kernel<D, kInt8>), g, b, 0, st, (char*)pool, block_bytes, k, v, at, n, h);
    else hipLaunchKernelGGL((q8_read_kernel<D, kInt8>), g, b, 0, st, (const char*)pool, block_bytes, k, v, at, n, h);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t move_any(void* pool, size_t block_bytes, int dtype, bool write, void* k, void* v, const int32_t* dev_rows, int32_t rows, int heads,
                    int head_dim, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  switch (head_dim) {
    case 64: return move_rows<64>(pool, block_bytes, dtype, write, k, v, dev_rows, rows, heads, st);
    case 128: return move_rows<128>(pool, block_bytes, dtype, write, k, v, dev_rows, rows, heads, st);
    case 256: return move_rows<256>(pool, block_bytes, dtype, write, k, v, dev_rows, rows, heads, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_q8_write(void* pool, size_t block_bytes, int dtype, const void* k_new, const void* v_new, const int32_t* dev_dst, int32_t rows,
                           int num_heads, int head_dim, hipStream_t st) {
  if (dtype != kE4m3 && dtype != kInt8) return hipErrorInvalidValue;
  return move_any(pool, block_bytes, dtype, true, (void*)k_new, (void*)v_new, dev_dst, rows, num_heads, head_dim, st);
}

hipError_t launch_read(const void* pool, size_t block_bytes, int dtype, void* k_out, void* v_out, const int32_t* dev_src, int32_t rows,
                       int num_heads, int head_dim, hipStream_t st) {
  return move_any((void*)pool, block_bytes, dtype, false, k_out, v_out, dev_src, rows, num_heads, head_dim, st);
}

}  // namespace ic
