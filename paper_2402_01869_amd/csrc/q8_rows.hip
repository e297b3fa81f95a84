// Row kernel of the 8-bit cache: query rows that are few for their keys.  Decode rows of every pool (Section 4.2: one query token,
// every cached vector read once), short chunks, and the rows of a fresh chunk that see fewer than 64 keys.
//
// Measured, GB/s of cached bytes, e4m3 / integers: 128 rows of 256..4096, 40 heads of 128, 6690 / 6630; 256 rows of 512..2048, 16 heads of 256, 6390 / 6370;
// 128 rows, 32 heads of 64, 6530 / 6430; 64 heads over 8, 5850 / 5460.  Vector ALU 30 % (integers 45 %) and matrix pipe 9 % busy, no LDS
// conflicts, 1.02 times the bytes fetched.  Beside the tile kernel, one workgroup a CU, the wait for memory is exposed: 4000 to 5000.
//
// One workgroup = one row item (up to 16 columns: consecutive query rows of a sequence x the query heads of a K/V head) x one K/V head,
// 4 waves, wave w the item's 32-key tiles w, w + 4, ...; of items of few keys that are many, each wave has one (row_long).  HBM-bound: a byte of the
// cache is read once per item and meets all its columns.  The 16-column parts of a larger group, and the items of a span, read it once each: 256 rows of
// 256..4096 keys, 16 heads over 1 37 us, 24 and 32 over 1 64.
// Every wave copies its tiles from the pool straight into a ring of its own in LDS (no registers, no barrier), a tile ahead, and codes
// become MFMA operands in registers:
//   - S^T = K Q^T (16x16x32): a lane's A operand is 8 numbers of one key.  It reads 16 bytes of the key, two operands; which dims
//     an operand's 8 places are does not matter as long as Q^T has the same, so Q is loaded in that order.  The accumulator
//     then has 4 keys of one column in a lane, for each of the tile's two blocks.
//   - Codes are exact in bf16 and scales are powers of two.  An e4m3 key's scale goes into its converts, where it costs nothing; an
//     integer key's multiplies its score in fp32, a value's the value's weight: 8 products a tile and lane instead of one per number.
//   - O^T += V^T P^T: a lane's 8 weights ARE the B operand if its A operand has the same 8 keys: a lane loads its dims of those
//     8 keys (D / 16 bytes each), and the bytes of two keys are paired by v_perm on their way to bf16.  Rows of V^T are
//     dims in the order that falls out: row n of product (w, b) is dim n * D / 16 + 4 w + b.
//   - Weights go in as two bf16 numbers (16 bits of significand; the rounding of one, 2^-9, would show in rows of a few keys): the
//     matrix pipe has the time.  The normaliser is the fp32 sum of the unrounded weights, what is lost is 2^-17 of a weight.
//     Items of up to 8 columns (kPair: decode rows of groups of up to 8 heads) have their first numbers in columns 0..7 and
//     the second ones in 8..15: half the products, and one sum across lanes at the end.  Beside the tile kernel: 128 rows and 8
//     chunks, 40 heads, 573 -> 568 us; by itself, int8, 8 rows of 1000..3000 keys, 32 heads of 64, 21.2 -> 20.2 us, 200 of 600..1200,
//     40 heads of 128, 293 -> 289.
// Keys a column does not see: score -inf, weight 0, and 0 for the scale of their value, which may be infinite (NaN vectors); codes
// behind the item's last key are cleared, they may be anything (0 * NaN).
#include <algorithm>
#include <mutex>

#include "merge_body.h"
#include "q8.h"

namespace ic {

namespace {

using namespace q8;

constexpr int kWaves = 4;
constexpr int kKeys = 32;  // of a wave's tile: two blocks
constexpr int kCols = 16;
constexpr uint32_t kGridItems = 32768;  // work items (or fours of those that a wave has alone) in y, the rest of them in z
constexpr float kNegBig = -1.0e30f;
// Slack of the running maximum, in log2 units: below it nothing is rescaled.  A weight is then at most two to that power, and times the largest
// scale (2^120, integers 2^122) has to stay finite, in bf16 too: infinity would make NaN of the dimensions whose codes are 0.
template <int FMT>
constexpr float kLazyLog2 = FMT == kE4m3 ? 7.0f : 5.0f;

// A wave's ring of stages in LDS: 32 keys as they lie in the cache, K of the two blocks, V of the two blocks, their scale bytes.
template <int D>
struct R8 {
  static constexpr int kKL = D / 64;                    // 16-byte reads of a key block per lane; MFMA steps of Q K^T are twice as many
  static constexpr int kVW = D / 64;                    // dwords of a key's value per lane
  static constexpr int kDT = D / 16;                    // products of V^T P^T
  static constexpr int kTile = kBlockSize * D;          // bytes of a block's K or V
  static constexpr int kCopiesV = 2 * (kTile / 1024), kCopiesK = kCopiesV + 2;  // loads of a stage: 1 KiB each, and two of scale bytes
  static constexpr int kCopies = kCopiesK + kCopiesV;
  static constexpr int kStage = 4 * kTile + 512;
  // head_dim 256: one stage, whose keys are copied anew as soon as they are read, then its values.  Two stages (33 KiB a wave) let one
  // workgroup on a CU, and nothing covers its beginning and end.  head_dim 64: two stages and four workgroups on a CU; three and two
  // were slower (256 rows of 500..1000 keys, 32 heads, 147 -> 131 us, of 30..60 18.0 -> 14.1).  head_dim 128: with one stage and four workgroups
  // rows of 30..60 keys take 10 % less, long ones 2 to 8 % longer.
  static constexpr int kStages = D == 256 ? 1 : 2;
  static constexpr int kWaveLds = kStages * kStage;
  static constexpr int kSlice = kWaveLds / 4;           // floats of one wave's LDS: at the end its result
  static_assert((kCols * D + 2 * kCols) * 4 <= kWaveLds, "a wave's result takes the place of its ring");
};

// Chunks of 16 bytes of a block's K or V are permuted on their way into LDS, so that what is read together lies in all 64 banks.  K: lane (n, g)
// reads chunk 4 j + g of key n, 16 keys at the same chunk: the chunk is exchanged by the key.  V: lane (n, g) reads D / 16 bytes at n of key
// 4 g + i: rows four apart at the same place, so rows are exchanged by the key's upper bits.
template <int D>
__device__ __forceinline__ uint32_t swap_k(uint32_t key) {
  if constexpr (D == 64) return ((key >> 2) & 1) * 2 ^ (key >> 3) * 3;
  else if constexpr (D == 128) return key >> 1;
  else return key;
}
template <int D>
__device__ __forceinline__ uint32_t swap_v(uint32_t key) {  // on the chunk's number in the block
  if constexpr (D == 64) return (key >> 2) << 2;
  else if constexpr (D == 128) return ((key >> 2) & 1) << 3;
  else return 0;
}

template <int N> struct Words { typedef __attribute__((ext_vector_type(N))) uint32_t type; };
template <> struct Words<1> { typedef uint32_t type; };

// A block's K or V (1, 2 or 4 KiB) to LDS address at, 16 bytes a lane and KiB; off[i]: what the lane fetches of KiB i.  The offset of an
// instruction counts on both sides.  As assembly: the compiler would make every LDS read wait for all such copies in flight.  (clang
// warns that m0 is a reserved register; what it would put there it has to know to be overwritten.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int N>
__device__ __forceinline__ void copy_block(const char* base, const uint32_t (&off)[N], uint32_t at) {
  if constexpr (N == 1)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1 nt" ::"s"(at), "s"(base), "v"(off[0]) : "memory", "m0");
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1 nt\n\tglobal_load_lds_dwordx4 %3, %1 offset:0x400 nt" ::"s"(at),
                 "s"(base), "v"(off[0]), "v"(off[1])
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1 nt\n\tglobal_load_lds_dwordx4 %3, %1 offset:0x400 nt\n\t"
                 "global_load_lds_dwordx4 %4, %1 offset:0x800 nt\n\tglobal_load_lds_dwordx4 %5, %1 offset:0xc00 nt" ::"s"(at),
                 "s"(base), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3])
                 : "memory", "m0");
}
// 4 bytes a lane.
__device__ __forceinline__ void copy_scales(const char* base, uint32_t lane_off, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %2, %1" ::"s"(at), "s"(base), "v"(lane_off) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int kPending>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPending) : "memory");
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

template <int FMT, int B, int W>
__device__ __forceinline__ bf16x8 value_operand(const uint32_t (&v)[8][W], int w) {
  const u32x4 x = {pair_of<FMT, B>(v[0][w], v[1][w]), pair_of<FMT, B>(v[2][w], v[3][w]), pair_of<FMT, B>(v[4][w], v[5][w]),
                   pair_of<FMT, B>(v[6][w], v[7][w])};
  return __builtin_bit_cast(bf16x8, x);
}

__device__ __forceinline__ f32x4 mfma(const bf16x8 a, const bf16x8 b, const f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// What the lane 8 on among 16 has.
__device__ __forceinline__ float across(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x128, 0xf, 0xf, true));
}

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
// As mergep::store_shared.
__device__ __forceinline__ void store_two(float* a, float x, float y) {
  __hip_atomic_store((uint64_t*)a, __builtin_bit_cast(uint64_t, (mergep::f32x2){x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// End of a partition of a split decode row: as mergep::finish_split (the workgroup that finds the others' partial results there merges
// them, in an order that does not depend on who is last), but with all 256 threads.  The row's heads x D values are few for one head, and a
// thread that reads all partitions of its own waits for memory once per batch of them: here a thread has four values of every
// sets-th partition, and the sets meet in LDS.
template <int D>
__device__ __forceinline__ void finish_row(const AttnParams& p, int slot, int unit, int head0, int heads, float* lds, int* s_last) {
  using mergep::f32x2;
  const int mi = p.slot_merge[slot];
  const MergeItem mg = p.merge_items[mi];
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's partial results have reached the memory that all share
  __syncthreads();
  if (threadIdx.x == 0) {
    int32_t* const arrived = p.arrived + (int64_t)mi * p.split_units + unit;
    const int before = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == mg.nparts - 1) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *s_last = before;
  }
  __syncthreads();
  if (*s_last != mg.nparts - 1) return;  // the same for the whole workgroup
  constexpr int kBatch = 4, kThreads = 64 * kWaves;
  const int quads = heads * (D / 4);  // pieces of four values, at least 16
  const int sets = quads >= kThreads ? 1 : kThreads / quads;
  const uint32_t row_elems = (uint32_t)p.num_heads * D;
  for (int q0 = 0; q0 < quads; q0 += kThreads) {
    const int set = quads >= kThreads ? 0 : (int)threadIdx.x / quads, quad = quads >= kThreads ? q0 + (int)threadIdx.x : (int)threadIdx.x - set * quads;
    float M = kNegBig, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    const bool live = set < sets && quad < quads;
    const uint32_t e = (uint32_t)head0 * D + 4u * min(quad, quads - 1);
    if (live) {
      const float* po = p.part_o + (int64_t)mg.slot0 * row_elems + e;
      const float* pm = p.part_ml + ((int64_t)mg.slot0 * p.num_heads + e / D) * 2;
      for (int k0 = set; k0 < mg.nparts; k0 += kBatch * sets) {
        f32x4 o[kBatch];
        f32x2 ml[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int64_t part = min(k0 + k * sets, mg.nparts - 1);
          ml[k] = mergep::load_shared(pm + part * p.num_heads * 2);
          const f32x2 a = mergep::load_shared(po + part * row_elems), b = mergep::load_shared(po + part * row_elems + 2);
          o[k] = (f32x4){a[0], a[1], b[0], b[1]};
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          if (k0 + k * sets >= mg.nparts) break;
          const float m_new = __builtin_fmaxf(M, ml[k][0]);
          const float was = __builtin_amdgcn_exp2f(M - m_new), wgt = __builtin_amdgcn_exp2f(ml[k][0] - m_new);
          M = m_new;
          L = __builtin_fmaf(ml[k][1], wgt, L * was);
#pragma unroll
          for (int i = 0; i < 4; ++i) O[i] = __builtin_fmaf(o[k][i], wgt, O[i] * was);
        }
      }
    }
    if (sets > 1) {  // (then one round: the sets' (O, M, L) of a piece, six floats)
      float* const mine = lds + 6 * (set * quads + quad);
      if (live) {
        *(f32x2*)mine = (f32x2){O[0], O[1]};
        *(f32x2*)(mine + 2) = (f32x2){O[2], O[3]};
        *(f32x2*)(mine + 4) = (f32x2){M, L};
      }
      __syncthreads();
      if (live && set == 0)
        for (int k = 1; k < sets; ++k) {
          const float* const other = lds + 6 * (k * quads + quad);
          const float m_new = __builtin_fmaxf(M, other[4]);
          const float was = __builtin_amdgcn_exp2f(M - m_new), wgt = __builtin_amdgcn_exp2f(other[4] - m_new);
          M = m_new;
          L = __builtin_fmaf(other[5], wgt, L * was);
#pragma unroll
          for (int i = 0; i < 4; ++i) O[i] = __builtin_fmaf(other[i], wgt, O[i] * was);
        }
    }
    if (live && set == 0) {
      bf16x4 out;
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = (__bf16)(O[i] / L);  // round to nearest even
      *(bf16x4*)(p.out + (int64_t)mg.qrow * row_elems + e) = out;
    }
  }
}

// kMerge: split decode rows are merged by their last partition, else by the merge kernel.
// kSlim: Q^T stays in LDS behind the rings, which takes 16 registers less.
// kPair: the item has at most 8 columns; lanes n and n + 8 share one.
// kAlone: the wave has an item of its own (whole rows of few keys), no partner, and meets no barrier.
template <int D, int FMT, bool kMerge, bool kSlim, bool kPair, bool kAlone>
__device__ __forceinline__ void rows_body(const AttnParams& p, float* lds, int* s_last, uint32_t item_idx) {
  using R = R8<D>;
  constexpr int kTeam = kAlone ? 1 : kWaves;                  // waves that share an item
  constexpr int kRing = kAlone && kSlim ? R::kStages - 1 : R::kStages;  // (Q^T takes the last stage)
  const int unit = (int)blockIdx.x;
  const RowItem it = p.row_items[item_idx];
  const int n_rows = it.pad[0], pos0 = it.pad[1], nparts = it.pad[2];
  const int H = p.num_heads, Hk = p.num_kv_heads, G = p.group;
  const int subs = p.row_subs;                   // units of a K/V head: more than one where a group has more than 16 heads
  const int kvh = subs == 1 ? unit : unit / subs, first = (unit - kvh * subs) * kCols;
  const int head0 = kvh * G + first, heads = min(kCols, G - first);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int cols = n_rows * heads;               // columns that are rows of the result, <= 16
  const int col = min(kPair ? n & 7 : n, cols - 1);  // the others mirror the last one
  const auto row_of = [&](int c) { return n_rows == 1 ? 0 : c * p.row_recip >> 16; };  // c / heads (several rows: all heads of the group)
  const int row = row_of(col), head = head0 + (col - row * heads);
  const int limit = min(pos0 + row + 1, it.k_end);  // keys the column sees are below
  const int least = min(pos0 + 1, it.k_end);        // ... and every column's are at least these

  bf16x8 q[2 * R::kKL];
  typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
  lds_bf16x8* const q_lds = (lds_bf16x8*)(kAlone ? lds + w * R::kSlice + kRing * (R::kStage / 4) : lds + kWaves * R::kSlice) + lane;  // operand i of the lane at q_lds[64 i]
  {
    const uint16_t* qp = p.q + ((int64_t)(it.qrow + row) * H + head) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < R::kKL; ++j) {
      q[2 * j] = *(const bf16x8*)(qp + 64 * j);
      q[2 * j + 1] = *(const bf16x8*)(qp + 64 * j + 8);
    }
  }
  const bool upper = (n & 8) != 0;
  const float take = upper ? -1.0f : 0.0f;
  f32x4 o[R::kDT];
#pragma unroll
  for (int i = 0; i < R::kDT; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = kNegBig, l = 0.f;

  typedef __attribute__((address_space(4))) const int32_t const_i32;
  const_i32* bt = (const_i32*)(p.bt_flat + p.bt_off[it.seq]);
  const int last_blk = (it.k_end - 1) / kBlockSize;
  const int n_tiles = (it.k_end - it.k_begin + kKeys - 1) / kKeys;
  const float sc = p.scale_log2e;
  const int first_tile = kAlone ? 0 : w;
  const int n_mine = (n_tiles - first_tile + kTeam - 1) / kTeam;  // tiles of this wave

  // ---- copies: lane i fills chunk i of every KiB of a stage
  typedef __attribute__((address_space(3))) const char lds_char;
  lds_char* const ring = (lds_char*)lds + w * R::kWaveLds;
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  constexpr int kCh = D / 16, kParts = R::kTile / 1024;  // chunks of a key; KiB of a block's K or V
  // What this lane fetches of a block's K and V, KiB i: chunk 64 i + lane exchanged by its key 64 i / kCh + lane / kCh.
  uint32_t k_off = (uint32_t)kvh * R::kTile + (lane ^ swap_k<D>(lane / kCh)) * 16u;
  uint32_t v_off = (uint32_t)(Hk + kvh) * R::kTile + (lane ^ swap_v<D>(lane / kCh)) * 16u;
  uint32_t s_off = 2u * Hk * R::kTile + (uint32_t)kvh * 2u * kBlockSize + 4u * (lane & 7);
  const char* const pool = (const char*)p.pool;
  const uint32_t block_bytes = p.block_bytes;
  const auto fetch = [&](auto k_tag, auto v_tag, int id0, int id1, uint32_t at) __attribute__((always_inline)) {
    constexpr bool kDoK = decltype(k_tag)::value, kDoV = decltype(v_tag)::value;
    if constexpr (kSlim) asm volatile("" : "+v"(k_off), "+v"(v_off));  // what is derived from them is worked out here, not kept
    const char* const base[2] = {pool + (uint64_t)(uint32_t)id0 * block_bytes, pool + (uint64_t)(uint32_t)id1 * block_bytes};
    uint32_t k[kParts], v[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      k[i] = k_off ^ swap_k<D>(64 * i / kCh) * 16u;
      v[i] = v_off ^ swap_v<D>(64 * i / kCh) * 16u;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if constexpr (kDoK) {
        copy_block(base[b], k, at + b * R::kTile);
        copy_scales(base[b], s_off, at + 4 * R::kTile + 256 * b);
      }
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if constexpr (kDoV) copy_block(base[b], v, at + (2 + b) * R::kTile);
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};

  // ---- reads
  uint32_t k_at = (uint32_t)n * D + ((uint32_t)g ^ swap_k<D>(n)) * 16u;  // chunk 4 j + g of key n: ^ 64 j
  // value of key 4 g + i at its D / 16 bytes n; rows 4 g .. 4 g + 3 are exchanged alike, so key i is ^ i rows
  uint32_t v_at = (((uint32_t)(4 * g) * kCh) ^ swap_v<D>(4 * g)) * 16u + (uint32_t)n * (D / 16);

  // keys_read: called when the stage's keys and scale bytes are in registers; values_there: when its values are wanted.
  const auto step = [&](int tile, uint32_t at, auto keys_read, auto values_there) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) const uint32_t lds_u32;
    typedef __attribute__((address_space(3))) const uint8_t lds_u8;
    typedef typename Words<R::kVW>::type words;
    typedef __attribute__((address_space(3))) const words lds_words;
    lds_char* const stage = ring + at;
    if constexpr (kSlim) asm volatile("" : "+v"(k_at), "+v"(v_at));
    int ln = lane;
    if constexpr (kSlim) {
      ln = threadIdx.x & 63;
      asm volatile("" : "+v"(ln));
    }
    const uint32_t vs_at = ln >> 4 << 2, ks_at = FMT == kE4m3 ? ln & 15 : vs_at;
    const int kt = it.k_begin + tile * kKeys;
    uint32_t ksc[2], vsc[2];  // scale bytes: of keys 4 g ..+3; e4m3 keys: of key n, for the converts
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if constexpr (FMT == kE4m3) ksc[b] = *(lds_u8*)(stage + 4 * R::kTile + 256 * b + ks_at);
      else ksc[b] = *(lds_u32*)(stage + 4 * R::kTile + 256 * b + ks_at);
      vsc[b] = *(lds_u32*)(stage + 4 * R::kTile + 256 * b + kBlockSize + vs_at);
    }
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int j = 0; j < R::kKL; ++j)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const u32x4 c = *(lds_u32x4*)(stage + b * R::kTile + (k_at ^ 64u * j));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t x = c[2 * half], y = c[2 * half + 1];
          const float f = __builtin_bit_cast(float, ksc[b] << 23);
          const u32x4 a = FMT == kE4m3 ? (u32x4){two_values<FMT, false>(x, f), two_values<FMT, true>(x, f), two_values<FMT, false>(y, f), two_values<FMT, true>(y, f)}
                                       : (u32x4){two_codes<FMT, false>(x), two_codes<FMT, true>(x), two_codes<FMT, false>(y), two_codes<FMT, true>(y)};
          s[b] = mfma(__builtin_bit_cast(bf16x8, a), kSlim ? *(q_lds + 64 * (2 * j + half)) : q[2 * j + half], s[b]);
        }
      }
    keys_read();
    uint32_t v[8][R::kVW];
    if constexpr (kSlim) __builtin_amdgcn_sched_barrier(0);
    const auto read_v = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const words x = *(lds_words*)(stage + (2 + i / 4) * R::kTile + (v_at ^ (uint32_t)(i % 4 * D)));
        if constexpr (R::kVW == 1) v[i][0] = x;
        else
#pragma unroll
          for (int e = 0; e < R::kVW; ++e) v[i][e] = x[e];
      }
    };
    const bool partly = kt + kKeys > least;  // some column does not see all keys; wave-uniform
    const auto clear_v = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < R::kVW; ++e) v[i][e] = kt + 16 * (i / 4) + 4 * g + i % 4 < it.k_end ? v[i][e] : 0u;
    };
    if constexpr (R::kStages > 1) read_v();
    float x[8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[4 * b] = FMT == kE4m3 ? s[b][0] : s[b][0] * scale_of<0>(ksc[b]);
      x[4 * b + 1] = FMT == kE4m3 ? s[b][1] : s[b][1] * scale_of<1>(ksc[b]);
      x[4 * b + 2] = FMT == kE4m3 ? s[b][2] : s[b][2] * scale_of<2>(ksc[b]);
      x[4 * b + 3] = FMT == kE4m3 ? s[b][3] : s[b][3] * scale_of<3>(ksc[b]);
    }
    if (partly) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = kt + 16 * (i / 4) + 4 * g + i % 4;
        x[i] = key < limit ? x[i] : -__builtin_inff();
        vsc[i / 4] = key < limit ? vsc[i / 4] : vsc[i / 4] & ~(0xffu << 8 * (i % 4));  // a scale of 0
      }
      if constexpr (R::kStages > 1) clear_v();
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = __builtin_fmaxf(top, x[i]);
    top *= sc;
    // the running maximum moves, and the sums with it, only when some score is over it by more than the slack
    if (__builtin_amdgcn_ballot_w64(top > m + kLazyLog2<FMT>) != 0) {
      top = __builtin_fmaxf(top, __shfl_xor(top, 16));
      top = __builtin_fmaxf(top, __shfl_xor(top, 32));
      const float m_new = top > m + kLazyLog2<FMT> ? top : m;  // the same in the four lanes of a column
      const float was = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= was;
#pragma unroll
      for (int i = 0; i < R::kDT; ++i) o[i] *= was;
    }
    u32x4 hi, lo = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], sc, -m)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i + 1], sc, -m));
      l += p0 + p1;
      const uint32_t vb = vsc[i / 4];
      const float a = p0 * (i % 4 == 0 ? scale_of<0>(vb) : scale_of<2>(vb)), b = p1 * (i % 4 == 0 ? scale_of<1>(vb) : scale_of<3>(vb));
      const bf16x2 h = {(__bf16)a, (__bf16)b};
      uint32_t hb = __builtin_bit_cast(uint32_t, h);
      asm("" : "+v"(hb));  // the halves are taken from the pair, not rounded again
      if constexpr (kPair) {
        // lanes 0..7 take 0 off and round as before, the upper ones are left with the second number
        const bf16x2 r = {(__bf16)__builtin_fmaf(take, __builtin_bit_cast(float, hb << 16), a),
                          (__bf16)__builtin_fmaf(take, __builtin_bit_cast(float, hb & 0xffff0000u), b)};
        hi[i / 2] = __builtin_bit_cast(uint32_t, r);
      } else {
        const bf16x2 r = {(__bf16)(a - __builtin_bit_cast(float, hb << 16)), (__bf16)(b - __builtin_bit_cast(float, hb & 0xffff0000u))};
        hi[i / 2] = hb;
        lo[i / 2] = __builtin_bit_cast(uint32_t, r);
      }
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
    if constexpr (R::kStages == 1) {
      values_there();
      read_v();
      if (partly) {
        asm volatile("" ::: "memory");
        clear_v();
      }
    }
#pragma unroll
    for (int e = 0; e < R::kVW; ++e) {
      const bf16x8 a0 = value_operand<FMT, 0>(v, e), a1 = value_operand<FMT, 1>(v, e);
      const bf16x8 a2 = value_operand<FMT, 2>(v, e), a3 = value_operand<FMT, 3>(v, e);
      o[4 * e] = mfma(a0, ph, o[4 * e]);
      o[4 * e + 1] = mfma(a1, ph, o[4 * e + 1]);
      o[4 * e + 2] = mfma(a2, ph, o[4 * e + 2]);
      o[4 * e + 3] = mfma(a3, ph, o[4 * e + 3]);
      if constexpr (!kPair) {
        o[4 * e] = mfma(a0, pl, o[4 * e]);
        o[4 * e + 1] = mfma(a1, pl, o[4 * e + 1]);
        o[4 * e + 2] = mfma(a2, pl, o[4 * e + 2]);
        o[4 * e + 3] = mfma(a3, pl, o[4 * e + 3]);
      }
    }
  };

  // Q and the first tiles are asked for together; from the wait for Q on, no load but copies is in flight.
  const int blk0 = it.k_begin / kBlockSize + 2 * first_tile;
  const auto block = [&](int i, int b) { return bt[min(blk0 + 2 * kTeam * i + b, last_blk)]; };  // of this wave's tile i
  for (int i = 0; i < kRing && i < n_mine; ++i) fetch(yes, yes, block(i, 0), block(i, 1), ring_at + i * R::kStage);
  // Ids of the tile that is asked for next, loaded an iteration ahead (waited for where they are used: 8 rows of 1000..8000 keys, 64 heads
  // over 8, plan and 4 layers 102 -> 100 us; 128 rows beside 8 chunks, 40 heads, 582 -> 575).
  int id0 = block(kRing, 0), id1 = block(kRing, 1);
#pragma unroll
  for (int j = 0; j < 2 * R::kKL; ++j) asm volatile("" ::"v"(q[j]));
  if constexpr (kSlim) {
    if (kAlone || w == 0)
#pragma unroll
      for (int i = 0; i < 2 * R::kKL; ++i) q_lds[64 * i] = q[i];
    if constexpr (kAlone) asm volatile("" ::: "memory");  // a wave's LDS operations stay in order
    else __syncthreads();
  }
  if constexpr (R::kStages > 1) {
    uint32_t at = 0;
    for (int i = 0; i < n_mine; ++i) {
      // the copies of the tile behind this one stay in flight
      if (kRing == 1 || i == n_mine - 1) wait_copies<0>();
      else wait_copies<R::kCopies>();
      step(first_tile + kTeam * i, at, [] {}, [] {});
      if (i + kRing < n_mine) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage has been read
        fetch(yes, yes, id0, id1, ring_at + at);
        id0 = block(i + 1 + kRing, 0);
        id1 = block(i + 1 + kRing, 1);
      }
      at = at + R::kStage == (uint32_t)(kRing * R::kStage) ? 0u : at + R::kStage;
    }
  } else {
    for (int i = 0; i < n_mine; ++i) {
      const bool more = i + 1 < n_mine;
      wait_copies<R::kCopiesV>();  // the values behind the keys stay in flight
      step(
          first_tile + kTeam * i, 0u,
          [&]() __attribute__((always_inline)) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) fetch(yes, no, id0, id1, ring_at);
          },
          [&]() __attribute__((always_inline)) {
            if (more) wait_copies<R::kCopiesK>();
            else wait_copies<0>();
          });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) fetch(no, yes, id0, id1, ring_at);
      id0 = block(i + 2, 0);
      id1 = block(i + 2, 1);
    }
  }

  // ---- the waves' results meet in LDS (alone: change their lanes there): O^T as [column][dim], then (m, l) of every column
  int tid_e = threadIdx.x;
  asm volatile("" : "+v"(tid_e));  // lane numbers worked out again, not kept across the loop
  const int ne = tid_e & 15, ge = (tid_e >> 4) & 3;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if constexpr (kPair) {
#pragma unroll
    for (int i = 0; i < R::kDT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[i][r] += across(o[i][r]);
  }
  float* const mine = lds + w * R::kSlice;
  if (ne < cols) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < R::kVW; ++e)
        *(f32x4*)(mine + ne * D + (4 * ge + r) * (D / 16) + 4 * e) = (f32x4){o[4 * e][r], o[4 * e + 1][r], o[4 * e + 2][r], o[4 * e + 3][r]};
    if (ge == 0) {
      mine[kCols * D + 2 * ne] = m;
      mine[kCols * D + 2 * ne + 1] = l;
    }
  }
  if constexpr (kAlone) asm volatile("" ::: "memory");
  else __syncthreads();
  const float* const all = kAlone ? mine : lds;
  for (int idx = kAlone ? tid_e & 63 : tid_e; idx < cols * (D / 4); idx += 64 * kTeam) {
    const int c = idx / (D / 4), d = 4 * (idx % (D / 4));
    float M = kNegBig;
#pragma unroll
    for (int ww = 0; ww < kTeam; ++ww) M = __builtin_fmaxf(M, all[ww * R::kSlice + kCols * D + 2 * c]);
    float L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < kTeam; ++ww) {
      const float* sl = all + ww * R::kSlice;
      const float wgt = __builtin_amdgcn_exp2f(sl[kCols * D + 2 * c] - M);
      L = __builtin_fmaf(sl[kCols * D + 2 * c + 1], wgt, L);
      const f32x4 x = *(const f32x4*)(sl + c * D + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) O[i] = __builtin_fmaf(x[i], wgt, O[i]);
    }
    const int r = row_of(c), h = head0 + (c - r * heads);
    if (kAlone || it.slot < 0) {
      bf16x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (__bf16)(O[i] / L);  // round to nearest even
      *(bf16x4*)(p.out + ((int64_t)(it.qrow + r) * H + h) * D + d) = v;
    } else {
      const int64_t ps = (int64_t)(it.slot + r * nparts) * H + h;
      store_two(&p.part_o[ps * D + d], O[0], O[1]);
      store_two(&p.part_o[ps * D + d + 2], O[2], O[3]);
      if (d == 0) store_two(&p.part_ml[ps * 2], M, L);
    }
  }
  if constexpr (kMerge && !kAlone) {
    if (it.slot >= 0 && nparts == 0) finish_row<D>(p, it.slot, unit, head0, heads, lds, s_last);
  }
}

// Work items [0, row_long) have a workgroup each, of the others every wave has one.
template <int D, int FMT, bool kMerge, bool kSlim>
__device__ __forceinline__ void rows_any(const AttnParams& p, float* lds, int* s_last) {
  const uint32_t y = blockIdx.z * kGridItems + blockIdx.y, n_items = (uint32_t)p.n_row_items, n_long = (uint32_t)p.row_long;
  const int heads = p.row_subs == 1 ? p.group : kCols;  // (the last part of a larger group may have fewer)
  if (y < n_long) {
    if (p.row_items[y].pad[0] * heads <= 8) rows_body<D, FMT, kMerge, kSlim, true, false>(p, lds, s_last, y);
    else rows_body<D, FMT, kMerge, kSlim, false, false>(p, lds, s_last, y);
  } else {
    const uint32_t item = n_long + (y - n_long) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= n_items) return;
    if (p.row_items[item].pad[0] * heads <= 8) rows_body<D, FMT, kMerge, kSlim, true, true>(p, lds, s_last, item);
    else rows_body<D, FMT, kMerge, kSlim, false, true>(p, lds, s_last, item);
  }
}

template <int D, int FMT, bool kMerge>
__global__ __launch_bounds__(64 * kWaves, 2) void q8_rows_kernel(AttnParams p) {
  __shared__ __attribute__((aligned(1024))) float lds[kWaves * R8<D>::kSlice];
  __shared__ int s_last;
  rows_any<D, FMT, kMerge, false>(p, lds, &s_last);
}

// The build that runs beside the tile kernel (208 registers, two waves a SIMD): at most 96 registers, one of its waves a SIMD.  LDS is asked
// for at launch, so that the compiler's register budget follows the launch bounds (5 waves a SIMD).  Split rows are the merge kernel's.
template <int D>
constexpr int slim_lds_bytes() {
  return kWaves * R8<D>::kWaveLds + 2 * R8<D>::kKL * 1024;  // the rings, then Q^T
}
template <int D, int FMT>
__global__ __launch_bounds__(64 * kWaves, 5) void q8_rows_slim_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) float slim_lds[];
  if (!p.tile_first) __builtin_amdgcn_s_setprio(3);
  rows_any<D, FMT, false, true>(p, slim_lds, nullptr);
}

template <int D, int FMT>
hipError_t launch(const AttnParams& p, dim3 grid, bool slim, hipStream_t st) {
  const dim3 b(64 * kWaves);
  if constexpr (D <= 128) {
    if (slim) {
      // more than 64 KiB of launch-time LDS has to be asked for, once per device
      static std::mutex mu;
      static bool asked[64] = {};
      int dev = 0;
      if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
      {
        std::lock_guard<std::mutex> lock(mu);
        if (!asked[dev]) {
          const hipError_t e = hipFuncSetAttribute((const void*)q8_rows_slim_kernel<D, FMT>, hipFuncAttributeMaxDynamicSharedMemorySize, slim_lds_bytes<D>());
          if (e != hipSuccess) return e;
          asked[dev] = true;
        }
      }
      hipLaunchKernelGGL((q8_rows_slim_kernel<D, FMT>), grid, b, slim_lds_bytes<D>(), st, p);
      return hipGetLastError();
    }
  }
  if (slim) return hipErrorInvalidValue;
  if (p.split_units > 0) hipLaunchKernelGGL((q8_rows_kernel<D, FMT, true>), grid, b, 0, st, p);
  else hipLaunchKernelGGL((q8_rows_kernel<D, FMT, false>), grid, b, 0, st, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_rows(const AttnParams& p, int head_dim, int dtype, bool slim, hipStream_t st) {
  if (p.n_row_items <= 0) return hipSuccess;
  if (p.row_subs < 1 || p.row_subs * kCols < p.group || p.row_units != p.num_kv_heads * p.row_subs || p.row_units > 65535 || p.group_first != 0 || p.row_long < 0 || p.row_long > p.n_row_items ||
      (dtype != kE4m3 && dtype != kInt8))
    return hipErrorInvalidValue;
  const uint32_t n = (uint32_t)(p.row_long + (p.n_row_items - p.row_long + kWaves - 1) / kWaves);
  const dim3 g((uint32_t)p.row_units, std::min(n, kGridItems), (n + kGridItems - 1) / kGridItems);
  if (g.z > 65535) return hipErrorInvalidValue;
  const bool e4m3 = dtype == kE4m3;
  switch (head_dim) {
    case 64: return e4m3 ? launch<64, kE4m3>(p, g, slim, st) : launch<64, kInt8>(p, g, slim, st);
    case 128: return e4m3 ? launch<128, kE4m3>(p, g, slim, st) : launch<128, kInt8>(p, g, slim, st);
    case 256: return e4m3 ? launch<256, kE4m3>(p, g, slim, st) : launch<256, kInt8>(p, g, slim, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ic
