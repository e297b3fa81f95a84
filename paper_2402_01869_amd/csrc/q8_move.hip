// An 8-bit pool's way in and out: kv_write_span quantises the rows that a chunk or a decode token has just computed as it writes them
// through the block table, kv_read_span reads cached positions back as bf16 rows (of a bf16 pool: as they are).
//
// Both are byte movement: 2 Hkv (2 D + D + 1) bytes a token.  One lane has 16 numbers of a vector: two 16-byte pieces of bf16, one of
// codes; a vector is D / 16 adjacent lanes, whose largest magnitude is found by exchanges inside the group.
#include "q8.h"

namespace ic {

namespace {

using namespace q8;

constexpr int kThreads = 64;  // one-wave workgroups, as for the block moves

// The largest magnitude of 16 bf16 numbers, as their bits without the sign: for finite numbers, infinities and NaN alike a
// larger number is a larger magnitude, and everything from 0x7f80 on is infinite or NaN.
__device__ __forceinline__ uint32_t largest_bits(const u32x4 a, const u32x4 b) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = a[i] & 0x7fff7fffu, y = b[i] & 0x7fff7fffu;
    m = max(max(m, max(x & 0xffffu, x >> 16)), max(y & 0xffffu, y >> 16));
  }
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

// What a lane has: 16 numbers of one vector.
template <int D>
struct Piece {
  static constexpr uint32_t kLanes = D / 16;  // of a vector
  uint32_t row, kv, head, part;
  bool live;
  __device__ __forceinline__ Piece(uint32_t rows, uint32_t num_heads) {
    const uint64_t idx = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    const uint32_t per_row = 2u * num_heads * kLanes;
    const uint64_t r = idx / per_row;
    live = r < rows;
    row = (uint32_t)r;
    const uint32_t rem = (uint32_t)(idx - r * per_row);
    const uint32_t vec = rem / kLanes;
    part = rem % kLanes;
    kv = vec >= num_heads;
    head = vec - (kv ? num_heads : 0u);
  }
  // byte offset of the lane's 16 numbers among the new rows
  __device__ __forceinline__ uint64_t row_at(uint32_t num_heads) const { return (((uint64_t)row * num_heads + head) * D + part * 16u) * 2u; }
  __device__ __forceinline__ uint32_t code_at(uint32_t num_heads, uint32_t slot) const {
    return ((kv * num_heads + head) * kBlockSize + slot) * D + part * 16u;
  }
  __device__ __forceinline__ uint32_t scale_at(uint32_t num_heads, uint32_t slot) const {
    return 2u * num_heads * kBlockSize * D + (head * 2u + kv) * kBlockSize + slot;
  }
};

template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void q8_write_kernel(char* __restrict__ pool, uint64_t block_bytes, const char* __restrict__ k_new,
                                                           const char* __restrict__ v_new, const int32_t* __restrict__ dst, uint32_t rows,
                                                           uint32_t num_heads) {
  const Piece<D> at(rows, num_heads);
  const int32_t d = at.live ? dst[at.row] : -1;
  u32x4 a = {}, b = {};
  if (d >= 0) {  // the lanes of a vector have the same d
    const char* src = (at.kv ? v_new : k_new) + at.row_at(num_heads);
    a = __builtin_nontemporal_load((const u32x4*)src);
    b = __builtin_nontemporal_load((const u32x4*)(src + 16));
  }
  uint32_t m = largest_bits(a, b);
#pragma unroll
  for (int x = 1; x < (int)Piece<D>::kLanes; x *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, x));
  if (d < 0) return;
  const uint32_t sb = scale_byte<FMT>(m);
  const float scale = __builtin_bit_cast(float, sb << 23), inv = __builtin_bit_cast(float, (254u - sb) << 23);
  u32x4 c;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    c[i] = four_codes<FMT>(a[2 * i], a[2 * i + 1], scale, inv);
    c[2 + i] = four_codes<FMT>(b[2 * i], b[2 * i + 1], scale, inv);
  }
  if (sb == 255u) c = (u32x4){0u, 0u, 0u, 0u};
  const uint32_t blk = (uint32_t)d / (uint32_t)kBlockSize, slot = (uint32_t)d % (uint32_t)kBlockSize;
  char* base = pool + blk * block_bytes;
  *(u32x4*)(base + at.code_at(num_heads, slot)) = c;
  if (at.part == 0) base[at.scale_at(num_heads, slot)] = (char)sb;
}

template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void q8_read_kernel(const char* __restrict__ pool, uint64_t block_bytes, char* __restrict__ k_out,
                                                          char* __restrict__ v_out, const int32_t* __restrict__ src, uint32_t rows,
                                                          uint32_t num_heads) {
  const Piece<D> at(rows, num_heads);
  if (!at.live) return;
  const int32_t d = src[at.row];
  if (d < 0) return;
  const uint32_t blk = (uint32_t)d / (uint32_t)kBlockSize, slot = (uint32_t)d % (uint32_t)kBlockSize;
  const char* base = pool + blk * block_bytes;
  const u32x4 c = __builtin_nontemporal_load((const u32x4*)(base + at.code_at(num_heads, slot)));
  const uint32_t sb = (uint8_t)base[at.scale_at(num_heads, slot)];
  const bool bad = sb == 255u;
  const float scale = __builtin_bit_cast(float, bad ? 0x3f800000u : sb << 23);
  u32x4 o[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[i / 2][2 * (i % 2)] = bad ? kNanBf16x2 : two_values<FMT, false>(c[i], scale);
    o[i / 2][2 * (i % 2) + 1] = bad ? kNanBf16x2 : two_values<FMT, true>(c[i], scale);
  }
  char* out = (at.kv ? v_out : k_out) + at.row_at(num_heads);
  __builtin_nontemporal_store(o[0], (u32x4*)out);
  __builtin_nontemporal_store(o[1], (u32x4*)(out + 16));
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
hipError_t move_rows(void* pool, size_t block_bytes, int dtype, bool write, void* k, void* v, const int32_t* dev_rows, int32_t rows, int heads,
                     hipStream_t st) {
  const int numbers = dtype == IC_DTYPE_BF16 ? 8 : 16;  // of a vector in one lane
  const uint64_t lanes = (uint64_t)rows * 2u * (uint64_t)heads * (uint64_t)(D / numbers);
  const uint64_t grid = (lanes + kThreads - 1) / kThreads;
  if (grid > 0x7fffffffull) return hipErrorInvalidValue;
  const dim3 g((uint32_t)grid), b(kThreads);
  const uint32_t n = (uint32_t)rows, h = (uint32_t)heads;
  if (dtype == IC_DTYPE_BF16) hipLaunchKernelGGL(kv_gather_kernel<D>, g, b, 0, st, (const char*)pool, (char*)k, (char*)v, dev_rows, n, h);
  else if (dtype == kE4m3 && write) hipLaunchKernelGGL((q8_write_kernel<D, kE4m3>), g, b, 0, st, (char*)pool, block_bytes, (const char*)k, (const char*)v, dev_rows, n, h);
  else if (dtype == kE4m3) hipLaunchKernelGGL((q8_read_kernel<D, kE4m3>), g, b, 0, st, (const char*)pool, block_bytes, (char*)k, (char*)v, dev_rows, n, h);
  else if (write) hipLaunchKernelGGL((q8_write_kernel<D, kInt8>), g, b, 0, st, (char*)pool, block_bytes, (const char*)k, (const char*)v, dev_rows, n, h);
  else hipLaunchKernelGGL((q8_read_kernel<D, kInt8>), g, b, 0, st, (const char*)pool, block_bytes, (char*)k, (char*)v, dev_rows, n, h);
  return hipGetLastError();
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
