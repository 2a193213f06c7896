// Attention of a few new tokens over a KV cache (one token, a drafted chain or tree), dense or paged, in its
// own type or quantised, over all of it or over listed blocks.
//
// The queries of all heads of a KV group and of all new tokens are the rows that one key serves: R = T * G of
// them.  A wave takes kTile keys at a time and 16 NC of those rows (NC = 1 or 2; RW waves share the tiles):
//   S^T = K Q^T      keys x rows, 16x16 matrix instructions: a lane holds one row's logits, of every fourth group of
//                    four keys
//   softmax          one reference exponent and one sum per row in registers
//   O^T += V^T P^T   the probabilities are already laid out as the second product's operand; V is read
//                    transposed from LDS (ds_read_b64_tr)
// Bound by reading K and V (4 R flops for a value read).  Waves share nothing until their keys are done: each copies
// its own tiles asynchronously into its own part of the LDS, kStages of them in flight, and waits for nobody; at the
// end the workgroup's waves add up their rows.  The keys of a sequence are cut over workgroups so that the chip is
// full; the pieces' results are merged by a second kernel.
//
// Measured: 8 sequences of 2048 bf16 keys, 67 MB, 16 us (4.3 TB/s; more where they come from memory and not from the
// last-level cache) and 4 to merge; 4 paged e4m3 caches of up to 32768 keys, 225 MB, 50 to 57 us (4.1 TB/s; 3 to 8 of them
// until the first tiles are there); 64 rows over 16384 bf16 keys 23.5 us, four tiles a wave, so that the way to the first
// tile, its code still to be fetched, and the end are half of it; 256 rows over 2 x 7839 8-bit keys 46 us, a wave and
// tile of 32 rows being about 510 vector instructions and 48 matrix instructions: those issue in 60 % of the time, these
// take 20, and the rest is the way through the LDS and the barriers.
#include <algorithm>
#include <cmath>

#include "cache.h"
#include "tiles.h"

namespace {

using namespace kvc::cache;
using kvc::tiles::kLn2;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr int kAhead = 512;         // keys whose places a wave looks up at once
constexpr float kNegBig = -3.0e38f;  // reference of a row that has seen nothing yet: finite, and below what logits come to

struct AttendParams {
  View c;
  const char* q;
  char* out;
  float* lse;
  float* part_o;   // workspace [Hkv][pieces][T * G][D]
  float2* part_ml;  // workspace [Hkv][pieces][T * G]
  int2* cuts;       // workspace [64]: first piece and number of pieces of each sequence, where they are dealt by length
  const uint64_t* mask;
  const int32_t* n_new;
  const int32_t* blocks;
  int64_t q_stride[3], out_stride[3];  // elements
  int64_t mask_stride;
  int Hq, G, T, n_list, unit, mask_words, q_dtype;
  int pieces;     // of all sequences together, per KV head
  int n_split;    // pieces of each sequence; 0: they are dealt by length
  int row_tiles;  // workgroups that share a piece
  int once;       // the keys pass the caches by
  float scale_log2;
};

template <int FORMAT_, int D_>
struct Fmt {
  static constexpr int FORMAT = FORMAT_, D = D_;
  static constexpr bool kQuant = quantised(FORMAT);
  static constexpr int kBits = format_bits(FORMAT);
  static constexpr int kRow = D * kBits / 8;       // bytes of a row
  static constexpr int kChunks = kRow / 16;        // 16-byte chunks of a row
  // Keys of a tile: 32 are one step of the second product; transposed reads of 4-bit values bring 64 at a time.
  static constexpr int kTile = kBits == 32 ? 16 : kBits == 4 ? 64 : 32;
  static constexpr int kSub = kTile / 16;          // groups of 16 keys
  static constexpr int kTileBytes = kTile * kRow;
  static constexpr int kLoads = kTileBytes / 1024;  // wave instructions that copy a tile of K (or V)
  static constexpr int kParam = kQuant ? (FORMAT == KVCRUSH_I4 ? 2 : 1) : 0;  // floats beside a row
  static constexpr int kParamLoads = kParam * 2 * kTile / 64;                 // of 4 bytes a lane
  static constexpr int kStage = 2 * kTileBytes + kParamLoads * 256;
  // Eight waves where LDS and registers have room for them: two to a SIMD, so that one's matrix instructions run beside
  // the other's arithmetic.  RW of them share a tile.
  static constexpr int lds(int waves, int RW) { return waves / RW * stages(RW) * kStage + waves * kAhead * 4; }
  // Groups of waves that share tiles meet at a barrier for every second one where there is room for two pairs (256 rows over
  // 2 x 7839 8-bit keys: a barrier a tile 53.5 us, every second 48.5, every fourth 48.9).
  static constexpr int stages(int RW) { return RW > 1 && 8 / RW * 4 * kStage + 8 * kAhead * 4 <= kvc::kLdsPerWorkgroup ? 4 : 2; }
  static constexpr int waves(int NC, int RW) {
    return (NC == 2 && kBits == 4) || lds(8, RW) > kvc::kLdsPerWorkgroup ? 4 : 8;
  }
  static constexpr int kSteps = D / 32;            // matrix steps of 32 values along D (16-bit operands)
  static constexpr int kDTiles = D / 16;
  static constexpr int kVTerms = FORMAT == KVCRUSH_F16 ? 2 : 1;  // bfloat16 values that one of V is the sum of
  static_assert(kTileBytes % 1024 == 0, "whole wave instructions");

  // XOR on a 16-byte chunk's place in its 256-byte line of the tile's image, by the line's number.  Two reads must find
  // their pieces in different banks: K's, one chunk of 16 neighbouring rows; V's, transposed, 8 values (4-bit: 16) of
  // 4 values' width of rows that differ in bits 0, 1, 2 (8-bit: and 4; 4-bit: 4 and 5).
  __device__ static int swizzle(int line) {
    const int l0 = line & 1, l1 = (line >> 1) & 1, l2 = (line >> 2) & 1, l3 = (line >> 3) & 1;
    if constexpr (kBits == 32) return kRow == 512 ? (line >> 1) & 15 : line & 15;
    if constexpr (kBits == 16) return kRow == 256 ? ((line & 7) << 1) | l3 : ((line & 3) << 1) | l2;
    if constexpr (kBits == 8) return kRow == 128 ? l0 | (l1 << 1) | ((l2 ^ l3) << 2) : l0 | ((l1 ^ l2) << 1);
    return kRow == 64 ? (l0 ^ l2) | ((l1 ^ l3) << 1) : l0 ^ l1;
  }
  __device__ static int chunk_at(int row, int chunk) {  // byte offset in the image
    const int q = row * kChunks + chunk, line = q >> 4;
    return (line << 8) | (((q & 15) ^ swizzle(line)) << 4);
  }
  // The row and chunk whose bytes lie at physical chunk `p` of the image.
  __device__ static void chunk_of(int p, int& row, int& chunk) {
    const int line = p >> 4, q = line * 16 + ((p & 15) ^ swizzle(line));
    row = q / kChunks;
    chunk = q % kChunks;
  }
};

// C += A B^T for one step of 32 values along the inner axis; operands are bfloat16 or halves.
template <int FORMAT>
__device__ __forceinline__ void mma(f32x4& c, const u32x4& a, const u32x4& b) {
  if constexpr (FORMAT == KVCRUSH_BF16)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x2 read_tr16(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}
__device__ __forceinline__ u32x2 read_tr8(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p));
}
__device__ __forceinline__ u32x2 read_tr4(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) i32x2*)p));
}

// The largest of the four lanes of a row (lane, lane ^ 16, lane ^ 32, lane ^ 48), and their sum.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A float without what lies below its eighth bit.
__device__ __forceinline__ float first8(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// Keys: register r of group u of lane group g = lane / 16 holds key 16 u + 4 g + r; element e of a step of 32 keys is
// register e % 4 of group e / 4.
__device__ __forceinline__ int step_key(int g, int e) { return 16 * (e >> 2) + 4 * g + (e & 3); }

// K's operands for 16 keys: all matrix steps.  A lane takes 16-byte chunks 4 j + g of its key's row (the order of the
// inner axis is free; the queries follow it).
template <class F>
__device__ __forceinline__ void k_frags(const char* tile, int lane, int u, u32x4 (&f)[F::kBits == 32 ? F::D / 16 : F::kSteps]) {
  const int row = 16 * u + (lane & 15), g = lane >> 4;
  if constexpr (F::kBits >= 16) {
#pragma unroll
    for (int j = 0; j < F::kChunks / 4; ++j) f[j] = *(const u32x4*)(tile + F::chunk_at(row, 4 * j + g));
  } else if constexpr (F::kBits == 8) {
#pragma unroll
    for (int j = 0; j < F::kChunks / 4; ++j) {
      const u32x4 w = *(const u32x4*)(tile + F::chunk_at(row, 4 * j + g));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x2 a = codes4_to_f16<F::FORMAT, true>(w[2 * i]), b = codes4_to_f16<F::FORMAT, true>(w[2 * i + 1]);
        f[2 * j + i] = u32x4{a[0], a[1], b[0], b[1]};
      }
    }
  } else if constexpr (F::kChunks == 4) {
    const u32x4 w = *(const u32x4*)(tile + F::chunk_at(row, g));
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = codes8_to_small_f16(w[i]);
  } else {
    const u32x2 w = *(const u32x2*)(tile + F::chunk_at(row, g >> 1) + (g & 1) * 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = codes8_to_small_f16(w[i]);
  }
}
// First value of the eight (four of a 32-bit type) that this lane's step t of the inner axis has.
template <class F>
__device__ __forceinline__ int step_value(int g, int t) {
  if constexpr (F::kBits == 32) return (4 * t + g) * 4;
  if constexpr (F::kBits == 16) return (4 * t + g) * 8;
  if constexpr (F::kBits == 8) return (4 * (t >> 1) + g) * 16 + (t & 1) * 8;
  return F::kChunks == 4 ? g * 32 + t * 8 : g * 16 + t * 8;
}

// V^T's operand of 16 values (tile dt) x 32 keys (step ks) as bfloat16: lane = value, its eight keys step_key(g, e).
// A half is the sum of two, exactly: its first eight bits and the three that are left.
template <class F>
__device__ __forceinline__ void v_frag(const char* tile, int lane, int dt, int ks, u32x4 (&f)[F::kVTerms]) {
  const int g = lane >> 4, i = lane & 15;
  if constexpr (F::kBits == 16) {
    const int row = 32 * ks + 4 * g + (i >> 2), chunk = dt * 2 + ((i & 3) >> 1), off = (i & 1) * 8;
    const u32x2 a = read_tr16(tile + F::chunk_at(row, chunk) + off), b = read_tr16(tile + F::chunk_at(row + 16, chunk) + off);
    f[0] = u32x4{a[0], a[1], b[0], b[1]};
    if constexpr (F::FORMAT == KVCRUSH_F16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x2 h = as_f16x2(f[0][j]);
        const float x = (float)h[0], y = (float)h[1];
        f[0][j] = upper2(x, y);
        f[1][j] = upper2(x - first8(x), y - first8(y));
      }
    }
  } else {
    static_assert(F::kBits == 8, "");
    const int row = 32 * ks + step_key(g, i >> 1);
    const u32x2 w = read_tr8(tile + F::chunk_at(row, dt) + (i & 1) * 8);
    const u32x2 a = codes4_to_bf16<F::FORMAT>(w[0]), b = codes4_to_bf16<F::FORMAT>(w[1]);
    f[0] = u32x4{a[0], a[1], b[0], b[1]};
  }
}
// 4-bit codes of 64 keys: one word a step.  codes8_to_bf16's order is undone by the order of the rows.
template <class F>
__device__ __forceinline__ u32x2 v_codes4(const char* tile, int lane, int dt) {
  const int g = lane >> 4, i = lane & 15, j = i & 7;
  const int row = 32 * (i >> 3) + step_key(g, (j >> 1) + 4 * (j & 1));
  return read_tr4(tile + F::chunk_at(row, dt >> 1) + (dt & 1) * 8);
}

// Position of a key slot, and whether there is a token (without branches, so that many are looked up at a time).
struct Slots {
  const int32_t* list;  // this query's blocks, or null
  int n, unit, L;
  __device__ bool position(int slot, int& pos) const {
    pos = slot;
    if (!list) return slot < n;
    const int e = min(slot, n - 1) / unit, blk = list[e], before = list[max(e - 1, 0)];
    const bool there = (slot < n) & (blk >= 0) & ((e == 0) | (blk > before)) & (blk <= (L - 1) / unit);
    pos = (there ? blk : 0) * unit + (slot - e * unit);
    return there & (pos < L);
  }
};

// The slots of query t (without lists: of every query), n of whose sequence's T new tokens are real.
__device__ __forceinline__ Slots key_slots(const AttendParams& p, int b, int h, int t, int n) {
  Slots s;
  s.L = p.c.length(b);
  s.list = p.blocks ? p.blocks + ((size_t)(b * p.c.Hkv + h) * p.T + t) * p.n_list : nullptr;
  s.unit = p.unit;
  s.n = p.blocks ? (t < n ? p.n_list * p.unit : 0) : n > 0 ? s.L : 0;
  return s;
}

// Asynchronous copies into LDS, 16 or 4 bytes a lane to `dst` + 16 or 4 x lane (dst uniform).  Written out, so that the
// compiler does not wait for all of them before each LDS read that follows; whoever reads waits with wait_copies and
// whoever overwrites what was read, with wait_reads.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// ONCE: past the caches (kOnceBytes).
template <bool ONCE>
__device__ __forceinline__ void copy16(const char* from, uint32_t dst) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "m0", "memory");
}
template <bool ONCE>
__device__ __forceinline__ void copy16(const char* base, uint32_t off, uint32_t dst) {  // base uniform
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(off), "s"(base) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(off), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void copy4(const char* from, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop
template <int LEFT>
__device__ __forceinline__ void wait_copies() {  // until at most LEFT of this wave's are under way
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LEFT) : "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Sums of several waves, then of several pieces are added up as these fractions of themselves: eight, and kMaxSplit, of the
// largest numbers that fp32 has stay below it.
constexpr int kMaxSplit = 256;
constexpr float kWaveRoom = 0x1p-4f, kPieceRoom = 0x1p-9f;
// 2^x for x <= 0, the factor of what a row has seen; never 0, so that an infinity stays one.
__device__ __forceinline__ float factor(float x) { return fmaxf(__builtin_amdgcn_exp2f(x), 0x1p-149f); }

// Four values of a row, from its sums: out = sum / room / total, lse = m + log2 total.
__device__ __forceinline__ void store_result(const AttendParams& p, int b, int head, int t, int e, float m, float total, f32x4 sum, float room) {
  if (p.lse && e == 0)
    p.lse[((size_t)b * p.Hq + head) * p.T + t] = total == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(total)) * kLn2;
  const float inv = 1.0f / room / total;
  float x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = total == 0.0f ? 0.0f : sum[i] * inv;
  const size_t at = (size_t)b * p.out_stride[0] + (size_t)head * p.out_stride[1] + (size_t)t * p.out_stride[2] + e;
  if (p.q_dtype == KVCRUSH_F32)
    *(f32x4*)(p.out + at * 4) = f32x4{x[0], x[1], x[2], x[3]};
  else if (p.q_dtype == KVCRUSH_BF16)
    *(u32x2*)(p.out + at * 2) = u32x2{pack2<KVCRUSH_BF16>(x[0], x[1]), pack2<KVCRUSH_BF16>(x[2], x[3])};
  else
    *(u32x2*)(p.out + at * 2) = u32x2{pack2<KVCRUSH_F16>(x[0], x[1]), pack2<KVCRUSH_F16>(x[2], x[3])};
}

// Some rows over the key slots from `first` to `last`, key by key and without the matrix cores: for what they get wrong.  A
// value that is not finite must reach the rows that see its key, as it is, and no others (0 x NaN; an infinity times the
// terms of a weight, some of them 0, is NaN), and the product of a very large one with a weight above 1 is not finite.  Here
// a row's weights add up to less than 1.  Rare, so written to be short: with an infinity among the keys, 8 sequences of 2048
// bf16 keys take 40 us, 64 rows over 16384 keys 340, 256 rows over 2 x 7839 1.5 ms.
constexpr int kTogether = 4;
template <int D>
struct Sums {
  float m[kTogether], l[kTogether], sum[kTogether][8];  // sum: values 8 (lane % (D / 8)) .. + 7
};
template <int FORMAT, int D>
__device__ __forceinline__ Sums<D> key_by_key(int b, int h, int t_list, int n, const int (&rows)[kTogether], int first, int last) {
  // (the kernel's arguments once more from where they were: kept in registers for this, they cost every call)
  auto at = (const __attribute__((address_space(4))) AttendParams*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  const AttendParams p = *(const AttendParams*)at;
  constexpr int kLanes = D / 8, kKeys = KVC_WAVE / kLanes;  // lanes of a key, keys of a load
  const int lane = kvc::lane_id(), chunk = lane % kLanes, first_new = p.c.length(b) - n;
  const Slots slots = key_slots(p, b, h, t_list, n);
  last = min(last, slots.n);
  const size_t base = p.c.base(b, h), step = p.c.step();
  const float scale = fmaxf(p.scale_log2, 0x1p-149f), room = (float)(33 - __builtin_clz(max(last - first, 1)));
  Sums<D> y;
  float q[kTogether][8];
  int t_of[kTogether];
#pragma unroll
  for (int r = 0; r < kTogether; ++r) {
    const int t = p.blocks ? t_list : rows[r] / p.G, head = h * p.G + (p.blocks ? rows[r] : rows[r] - t * p.G);
    const char* from = p.q + ((size_t)b * p.q_stride[0] + (size_t)head * p.q_stride[1] + (size_t)t * p.q_stride[2] + chunk * 8) * (format_bits(p.q_dtype) / 8);
    if (p.q_dtype == KVCRUSH_F32)
      load8<KVCRUSH_F32>(from, q[r]);
    else if (p.q_dtype == KVCRUSH_BF16)
      load8<KVCRUSH_BF16>(from, q[r]);
    else
      load8<KVCRUSH_F16>(from, q[r]);
    t_of[r] = t;
    y.m[r] = kNegBig;
    y.l[r] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) y.sum[r][j] = 0.0f;
  }
#pragma unroll 1
  for (int k0 = first; k0 < last; k0 += KVC_WAVE) {
    int pos;
    const bool there = slots.position(k0 + lane, pos) & (k0 + lane < last);
    const int draft = pos - first_new, token = p.c.token(b, there ? pos : 0);
    float x[kTogether] = {};
#pragma unroll 4
    for (int i = 0; i < kLanes; ++i) {
      float k[8];
      row_values<FORMAT>(p.c.k, p.c.k_param, base + (size_t)__shfl(token, i * kKeys + lane / kLanes) * step, D, chunk * 8, k);
#pragma unroll
      for (int r = 0; r < kTogether; ++r) {
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) part = __builtin_fmaf(q[r][j], k[j], part);
#pragma unroll
        for (int off = 1; off < kLanes; off *= 2) part += __shfl_xor(part, off);
        part = __shfl(part, lane % kKeys * kLanes);
        x[r] = i == lane / kKeys ? part : x[r];
      }
    }
    float weight[kTogether];
    uint64_t seen[kTogether];
#pragma unroll
    for (int r = 0; r < kTogether; ++r) {
      const uint64_t* words = p.mask ? p.mask + (size_t)b * p.mask_stride + (size_t)t_of[r] * p.mask_words : nullptr;
      const bool see = there & (draft < 0 || (words ? (words[min(max(draft >> 6, 0), p.mask_words - 1)] >> (draft & 63)) & 1 : draft <= t_of[r]));
      const float v = see ? x[r] * scale : -__builtin_inff(), mn = fmaxf(y.m[r], kvc::wave_max(v) + room), a = factor(y.m[r] - mn);
      y.m[r] = mn;
      weight[r] = v - mn > -__builtin_inff() ? factor(v - mn) : __builtin_amdgcn_exp2f(v - mn);  // (0, NaN as they are)
      y.l[r] = y.l[r] * a + weight[r];
      seen[r] = __ballot(see);
#pragma unroll
      for (int j = 0; j < 8; ++j) y.sum[r][j] *= a;
    }
#pragma unroll 4
    for (int i = 0; i < kLanes; ++i) {
      const int key = i * kKeys + lane / kLanes;
      float v[8];
      row_values<FORMAT>(p.c.v, p.c.v_param, base + (size_t)__shfl(token, key) * step, D, chunk * 8, v);
#pragma unroll
      for (int r = 0; r < kTogether; ++r) {
        const float w = __shfl(weight[r], key);
        const bool it = (seen[r] >> key) & 1;
#pragma unroll
        for (int j = 0; j < 8; ++j) y.sum[r][j] = it ? __builtin_fmaf(w, v[j], y.sum[r][j]) : y.sum[r][j];
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kTogether; ++r) {
    y.l[r] = kvc::wave_sum(y.l[r]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int off = kLanes; off < KVC_WAVE; off *= 2) y.sum[r][j] += __shfl_xor(y.sum[r][j], off);
  }
  return y;
}

// The cut of the sequences' keys into p.pieces pieces of `size` steps of `step` keys, in order of the sequences, each with
// one piece at least: the smallest size (but for a sixteenth) with which they suffice.  Whole waves; B <= 64.
struct Deal {
  int size;         // steps of a piece
  int first, n;     // of sequence `lane`
  int total;
};
__device__ __forceinline__ Deal deal(const AttendParams& p, int step) {
  const int lane = kvc::lane_id();
  const int steps = lane < p.c.B ? (p.c.length(lane) + step - 1) / step : 0;
  auto sum = [](int v) { return (int)kvc::wave_reduce((uint32_t)v, 0u, [](uint32_t a, uint32_t b) { return a + b; }); };
  Deal d;
  d.size = max((sum(steps) + p.pieces - 1) / p.pieces, 1);
  for (;; d.size += max(d.size >> 4, 1)) {
    d.n = lane < p.c.B ? max((steps + d.size - 1) / d.size, 1) : 0;
    d.total = sum(d.n);
    if (d.total <= p.pieces) break;  // (pieces >= B: with one piece each at the latest)
  }
  int end = d.n;
#pragma unroll
  for (int off = 1; off < KVC_WAVE; off *= 2) {
    const int o = __shfl_up(end, off);
    if (lane >= off) end += o;
  }
  d.first = end - d.n;
  return d;
}

// RW: waves that share a tile, each with 16 NC rows of its own.  One: the waves are on their own, and nobody waits for
// another's copies.  More: they copy a share each and meet at a barrier every kMeet tiles, so that many rows cost one
// reading of the keys.
template <class F, int NC, int RW>
__global__ __launch_bounds__(F::waves(NC, RW) * KVC_WAVE) void attend_kernel(AttendParams p) {
  constexpr int kWaves = F::waves(NC, RW), kGroups = kWaves / RW, kStages = F::stages(RW);
  constexpr int D = F::D, FORMAT = F::FORMAT, kTile = F::kTile, U = F::kSub;
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int tid = threadIdx.x, lane = kvc::lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / KVC_WAVE);
  const int g = lane >> 4, col = lane & 15, key_group = wave / RW, row_wave = wave % RW;
  // Workgroups with numbers 8 apart run on one chiplet, one after the other: the row tiles of a piece, which read the same
  // keys, are put there side by side.
  const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3, row_tile = place % p.row_tiles;
  const int group = place / p.row_tiles * 8 + xcd, h = group / p.pieces, piece = group - h * p.pieces;
  if (h >= p.c.Hkv) return;
  int b, split, n_split, piece_tiles = 0;  // this piece of the n_split of sequence b
  if (p.n_split > 0) {
    n_split = p.n_split;
    b = piece / n_split;
    split = piece - b * n_split;
  } else {
    const Deal d = deal(p, F::kTile * kGroups);
    if (piece >= d.total) return;
    b = 63 - __builtin_clzll(__ballot(lane < p.c.B && d.first <= piece));
    split = piece - __builtin_amdgcn_readlane(d.first, b);
    n_split = __builtin_amdgcn_readlane(d.n, b);
    piece_tiles = d.size * kGroups;
    if (blockIdx.x == 0 && tid < p.c.B) p.cuts[tid] = make_int2(d.first, d.n);
  }
  const int L = p.c.length(b), n = new_tokens(p.n_new, b, p.T, L);
  // with lists, a query's G heads are the rows
  constexpr int kRows = 16 * NC * RW;
  const int tiles_of_query = (p.G + kRows - 1) / kRows;
  const int t_list = p.blocks ? row_tile / tiles_of_query : 0;
  const int row0 = (p.blocks ? row_tile % tiles_of_query : row_tile) * kRows;
  const int rows = p.blocks ? p.G : p.G * p.T;

  const Slots slots = key_slots(p, b, h, t_list, n);

  // this wave's (or its group's) tiles: a contiguous piece of the workgroup's
  const int tiles = (slots.n + kTile - 1) / kTile, per_wg = piece_tiles > 0 ? piece_tiles : (tiles + n_split - 1) / n_split;
  const int wg0 = min(split * per_wg, tiles), wg1 = min(wg0 + per_wg, tiles);
  const int per_group = (wg1 - wg0 + kGroups - 1) / kGroups;
  const int tile0 = __builtin_amdgcn_readfirstlane(min(wg0 + key_group * per_group, wg1));
  const int tile1 = __builtin_amdgcn_readfirstlane(min(tile0 + per_group, wg1));

  // ---- copies of tiles into this group's stages
  char* own = lds_all + key_group * (kStages * F::kStage);
  const uint32_t own_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)own);
  // token of each slot (a table of each wave's own); bit 31: the slot has to be looked at
  int* places = (int*)(lds_all + kGroups * kStages * F::kStage) + wave * kAhead;
  const size_t row_base = p.c.base(b, h), row_step = p.c.step();
  const bool lookup = p.c.table || p.blocks;
  const int first_new = L - n;
  uint32_t looks = 0;  // bit i % 32: tile tile0 + i has such slots (lookups only)
  // A tile is 2 kLoads pieces of 1 KiB, K's and behind them V's; wave row_wave of a group copies pieces row_wave,
  // row_wave + RW, ..  in_tile: this lane's bytes of a piece, in a tile whose rows lie one behind the other.
  constexpr int kOwn = 2 * F::kLoads / RW;
  static_assert(2 * F::kLoads % RW == 0, "the waves of a group copy alike");
  constexpr int kOffsets = F::kLoads / RW > 0 ? F::kLoads / RW : 1;  // (K's pieces and V's lie alike)
  uint32_t in_tile[kOffsets];
#pragma unroll
  for (int j = 0; j < kOffsets; ++j) {
    int row, chunk;
    F::chunk_of((j * RW + row_wave) % F::kLoads * 64 + lane, row, chunk);
    in_tile[j] = row * F::kRow + chunk * 16;
  }
  constexpr int kCopies = kOwn + F::kParamLoads;
  constexpr int kMeet = kStages / 2;  // tiles from one barrier to the next (RW > 1)
  auto issue = [&](int tile) {
    const int k0 = tile * kTile, i = tile - tile0, ahead = (i * kTile) & (kAhead - 1);
    const uint32_t stage = own_at + (i % kStages) * F::kStage, dst = stage + row_wave * 1024;
    if (lookup && ahead == 0) {
      // (branches only around the loops, so that a loop's loads are all on their way before the first is used)
      constexpr int kEach = kAhead / KVC_WAVE;
      int at[kEach];
      uint32_t marked = 0;
#pragma unroll
      for (int x = 0; x < kEach; ++x) at[x] = k0 + x * KVC_WAVE + lane;
      if (slots.list) {
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
          int pos;
          const bool there = slots.position(at[x], pos);
          if (!there || pos >= first_new) marked |= 1u << x;
          at[x] = there ? pos : 0;
        }
      } else {
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
          if (at[x] >= first_new) marked |= 1u << x;
          at[x] = at[x] < L ? at[x] : 0;
        }
      }
      if (p.c.table) {
#pragma unroll
        for (int x = 0; x < kEach; ++x) at[x] = p.c.paged_token(b, at[x]);
      }
#pragma unroll
      for (int x = 0; x < kEach; ++x)
        places[x * KVC_WAVE + lane] = at[x] | ((marked >> x) & 1 ? (int)0x80000000 : 0);
      kvc::wave_fence();
    }
    auto copy = [&](auto as) {
      constexpr bool ONCE = decltype(as)::value;
      if (!lookup && k0 + kTile <= L) {
        const size_t from = (row_base + k0) * F::kRow;
        const char *k = kvc::tiles::wave_uniform(p.c.k + from), *v = kvc::tiles::wave_uniform(p.c.v + from);
#pragma unroll
        for (int j = 0; j < kOwn; ++j) copy16<ONCE>(j * RW + row_wave < F::kLoads ? k : v, in_tile[j % kOffsets], dst + j * RW * 1024);
      } else {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
          const uint32_t at = in_tile[j % kOffsets];
          const int row = at / F::kRow;
          const int tok = lookup ? places[ahead + row] & 0x7FFFFFFF : min(k0 + row, L - 1);
          const size_t from = (row_base + (size_t)tok * row_step) * F::kRow + at % F::kRow;
          copy16<ONCE>((j * RW + row_wave < F::kLoads ? p.c.k : p.c.v) + from, dst + j * RW * 1024);
        }
      }
    };
    if (RW == 1 && p.once)
      copy(std::true_type{});
    else
      copy(std::false_type{});
    if constexpr (F::kQuant) {
      // (all of them by every wave of a group: the same bytes to the same place, and equal numbers of copies to wait for)
#pragma unroll
      for (int j = 0; j < F::kParamLoads; ++j) {
        // [parameter][K, V][key] floats
        const int e = j * 64 + lane, key = e % kTile, which = (e / kTile) & 1, par = e / (2 * kTile);
        const int tok = lookup ? places[ahead + key] & 0x7FFFFFFF : min(k0 + key, L - 1);
        const float* src = which ? p.c.v_param : p.c.k_param;
        copy4((const char*)(src + (row_base + (size_t)tok * row_step) * F::kParam + par), stage + 2 * F::kTileBytes + j * 256);
      }
    }
    if (lookup) {
      const bool look = __ballot(places[ahead + (lane & (kTile - 1))] < 0) != 0;
      looks = (looks & ~(1u << (i & 31))) | (look ? 1u << (i & 31) : 0u);
    }
  };
#pragma unroll
  for (int i = 0; i < (RW > 1 ? kMeet : kStages); ++i)
    if (tile0 + i < tile1) issue(tile0 + i);

  // ---- this lane's rows, and the queries as the first product's other operand
  constexpr int kQRegs = F::kBits == 32 ? D / 16 : F::kSteps;
  int t_of[NC];
  u32x4 qf[NC][kQRegs];
  float col_scale[NC], q_sum[NC];  // logit = (products) * col_scale; q_sum: the lowest value's factor
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int rr = min(row0 + (row_wave * NC + c) * 16 + col, rows - 1);
    const int t = p.blocks ? t_list : rr / p.G, head = h * p.G + (p.blocks ? rr : rr - t * p.G);
    t_of[c] = t;
    const char* q = p.q + ((size_t)b * p.q_stride[0] + (size_t)head * p.q_stride[1] + (size_t)t * p.q_stride[2]) * (format_bits(p.q_dtype) / 8);
    col_scale[c] = fmaxf(p.scale_log2, 0x1p-149f);  // (never zero: what a row does not see is -infinity times this)
    q_sum[c] = 0.0f;
    if constexpr (!F::kQuant) {
#pragma unroll
      for (int j = 0; j < kQRegs; ++j) qf[c][j] = *(const u32x4*)(q + step_value<F>(g, j) * (F::kBits / 8));
    } else {
      // Halves for every type of query: a row is scaled by the power of two that brings its largest value to
      // 2^14 .. 2^15, so that a bfloat16 value loses nothing unless it is 2^-29 of the largest.  K's codes come times 2^-14
      // (kCodeFactor), so that products with large keys stay below fp32's largest.
      float x[F::kSteps][8];
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) {
        const int d = step_value<F>(g, s);
        if (p.q_dtype == KVCRUSH_BF16)
          load8<KVCRUSH_BF16>(q + d * 2, x[s]);
        else
          load8<KVCRUSH_F16>(q + d * 2, x[s]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          top = max(top, __float_as_uint(x[s][i]) & 0x7FFFFFFFu);
          q_sum[c] += x[s][i];
        }
      }
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      q_sum[c] = row_sum(q_sum[c]);
      const int up = min(141 - (int)(top >> 23), 126);  // >= -114
      const float by = __builtin_amdgcn_ldexpf(1.0f, up);
      q_sum[c] *= by * kCodeFactor;
      col_scale[c] = fminf(fmaxf(__builtin_amdgcn_ldexpf(p.scale_log2, 14 - up), 0x1p-149f), 0x1p127f);
      constexpr int kOrder[2][8] = {{0, 1, 2, 3, 4, 5, 6, 7}, {0, 4, 1, 5, 2, 6, 3, 7}};
      constexpr int o = FORMAT == KVCRUSH_I4 ? 1 : 0;
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          qf[c][s][i] = pack2<KVCRUSH_F16>(x[s][kOrder[o][2 * i]] * by, x[s][kOrder[o][2 * i + 1]] * by);
    }
  }

  f32x4 o[NC][F::kDTiles];
  // Reference exponent m (base 2) of a row: o, l and z are sums of 2^(logit - m).  It need not be the largest logit: it is
  // raised, and the sums brought to it, only where a probability would pass 2^8, so that few tiles pay for it.
  float m[NC], l[NC], z[NC];  // l: sum of this lane's keys; z: sum of probability x lowest value
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNegBig;
    l[c] = z[c] = 0.0f;
#pragma unroll
    for (int d = 0; d < F::kDTiles; ++d) o[c][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // The two waves of a SIMD (wave, wave + 4) leave a barrier together: one goes ahead, so that its matrix instructions run
  // beside the other's arithmetic (256 rows of 8-bit keys 48.9 -> 48.2 us, 64 of bfloat16 27.4 -> 27.2).
  if (RW > 1 && wave >= 4) __builtin_amdgcn_s_setprio(2);
  for (int turn = 0; turn < (RW > 1 ? per_group : tile1 - tile0); ++turn) {
    const int tile = tile0 + turn, k0 = tile * kTile;
    if constexpr (RW > 1) {
      // behind the barrier the group's copies of the next kMeet tiles are all done, and so are its reads of those before
      if (turn % kMeet == 0) {
        wait_copies<0>();
        wait_reads();
        __syncthreads();
        for (int i = kMeet; i < kStages; ++i)
          if (tile + i < tile1) issue(tile + i);
      }
      if (tile >= tile1) continue;  // (the last group may have a tile less)
    } else {
      if (turn > 0) {
        wait_reads();  // (of the stage that is filled again)
        if (tile + kStages - 1 < tile1) issue(tile + kStages - 1);
      }
      if (tile + 1 < tile1)
        wait_copies<kCopies>();
      else
        wait_copies<0>();
    }
    const char* kt = own + turn % kStages * F::kStage;
    const char* vt = kt + F::kTileBytes;
    const float* kp = (const float*)(kt + 2 * F::kTileBytes);  // [parameter][K, V][key]
    const float* vp = kp + kTile;
    const bool look = lookup ? (looks >> (turn & 31)) & 1 : k0 + kTile > first_new;

    // ---- logits, but for the row's factor
    f32x4 s[NC][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      u32x4 kf[kQRegs];
      k_frags<F>(kt, lane, u, kf);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kQRegs; ++j) {
          if constexpr (F::kBits == 32) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[j][i]), __uint_as_float(qf[c][j][i]), acc, 0, 0, 0);
          } else {
            mma<FORMAT>(acc, kf[j], qf[c][j]);
          }
        }
        s[c][u] = acc;
      }
    }
    if constexpr (F::kQuant) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const f32x4 scale = *(const f32x4*)(kp + 16 * u + 4 * g);
        f32x4 low = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (FORMAT == KVCRUSH_I4) low = *(const f32x4*)(kp + 2 * kTile + 16 * u + 4 * g);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[c][u][r] = FORMAT == KVCRUSH_I4 ? __builtin_fmaf(s[c][u][r], scale[r], low[r] * q_sum[c]) : s[c][u][r] * scale[r];
      }
    }
    f32x4 v_scale[U], v_low[U];
    if constexpr (F::kQuant) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v_scale[u] = *(const f32x4*)(vp + 16 * u + 4 * g);
        if constexpr (FORMAT == KVCRUSH_I4) v_low[u] = *(const f32x4*)(vp + 2 * kTile + 16 * u + 4 * g);
      }
    }
    uint32_t seen[NC] = {};  // bit 4 u + r: this row sees the key (where it is looked at)
    if (look) {
      // Which keys of the tile are there, and which rows see those of them that are new: bit k is key k.
      int pos;
      const uint64_t there = __ballot(slots.position(k0 + (lane & (kTile - 1)), pos)) & (~0ull >> (64 - kTile));
      const int draft = pos - first_new;  // of key `lane`: number of the new token, negative for an older one
      const uint64_t old = __ballot(draft < 0);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint64_t* words = p.mask ? p.mask + (size_t)b * p.mask_stride + (size_t)t_of[c] * p.mask_words : nullptr;
        const int last = p.mask_words - 1;
        uint64_t see = 0;
        if (!slots.list) {  // the tile's new tokens are neighbours
          const int d0 = k0 - first_new, up = max(-d0, 0), from = max(d0, 0);  // key `up` is new token `from`
          if (words) {
            const int w = from >> 6, s0 = from & 63;
            const uint64_t a = words[min(w, last)], next = words[min(w + 1, last)];
            see = (a >> s0) | ((next << 1) << (63 - s0));
          } else {
            const int most = t_of[c] - from;
            see = most < 0 ? 0 : most >= 63 ? ~0ull : (2ull << most) - 1;
          }
          see = up >= 64 ? 0 : see << up;
        } else {  // all rows are heads of one query: each lane asks for its key
          see = __ballot(words ? (words[min(max(draft >> 6, 0), last)] >> (draft & 63)) & 1 : draft <= t_list);
        }
        see = t_of[c] < n ? (see | old) & there : 0;
#pragma unroll
        for (int u = 0; u < U; ++u) seen[c] |= (uint32_t)(see >> (16 * u + 4 * g) & 15) << (4 * u);
        // (a logit that the row does not see may be anything)
#pragma unroll
        for (int i = 0; i < 4 * U; ++i) s[c][i / 4][i % 4] = (seen[c] >> i) & 1 ? s[c][i / 4][i % 4] : -__builtin_inff();
      }
    }

    // ---- probabilities, times V's scale
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float most = s[c][0][0];
#pragma unroll
      for (int i = 1; i < 4 * U; ++i) most = fmaxf(most, s[c][i / 4][i % 4]);
      most *= col_scale[c];
      if (__ballot(most - m[c] > 8.0f) != 0) {
        const float mn = fmaxf(m[c], row_max(most)), a = __builtin_amdgcn_exp2f(m[c] - mn);
        m[c] = mn;
        l[c] *= a;
        if constexpr (FORMAT == KVCRUSH_I4) z[c] *= a;
#pragma unroll
        for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[c][d][r] *= a;
      }
      f32x4 pr[U];
#pragma unroll
      for (int i = 0; i < 4 * U; ++i) {
        pr[i / 4][i % 4] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][i / 4][i % 4], col_scale[c], -m[c]));
        l[c] += pr[i / 4][i % 4];
        if constexpr (F::kQuant)
          s[c][i / 4][i % 4] = pr[i / 4][i % 4] * v_scale[i / 4][i % 4];
        else
          s[c][i / 4][i % 4] = pr[i / 4][i % 4];
      }
      if constexpr (F::kQuant) {
        if (look) {
          asm volatile("");  // (a branch, not selections that every tile would pay for)
#pragma unroll
          for (int i = 0; i < 4 * U; ++i) {
            const bool it = (seen[c] >> i) & 1;
            s[c][i / 4][i % 4] = it ? s[c][i / 4][i % 4] : 0.0f;
            if constexpr (FORMAT == KVCRUSH_I4) z[c] = it ? __builtin_fmaf(pr[i / 4][i % 4], v_low[i / 4][i % 4], z[c]) : z[c];
          }
        } else if constexpr (FORMAT == KVCRUSH_I4) {
#pragma unroll
          for (int i = 0; i < 4 * U; ++i) z[c] = __builtin_fmaf(pr[i / 4][i % 4], v_low[i / 4][i % 4], z[c]);
        }
      }
    }
    // ---- values
    if constexpr (F::kBits == 32) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int d = 0; d < F::kDTiles; ++d) {
          const int e = d * 16 + col;  // value
          const float v = *(const float*)(vt + F::chunk_at(4 * g + r, e >> 2) + (e & 3) * 4);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[c][0][r], o[c][d], 0, 0, 0);
        }
      }
    } else {
      // A weight is the sum of bfloat16 values, whatever its size: its rounding, that of what is left, and what is left then.
      // (Halves end at 2^-24.)  Three are the weight, exactly; with two, off by 2^-18 of it, 8-bit values make do (256 rows
      // over 2 x 7839 keys 49 us, with three 55).  4-bit ones do not: the codes' sum and the lowest values' cancel.
      constexpr int kTerms = F::kBits == 8 ? 2 : 3;
      u32x4 w[NC][U / 2][kTerms];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) {
          float x = s[c][i / 2][2 * (i % 2)], y = s[c][i / 2][2 * (i % 2) + 1];
          // (values from here on: otherwise the compiler may round the product behind x in one step for a term and in two
          // for what it left)
          asm("" : "+v"(x), "+v"(y));
#pragma unroll
          for (int j = 0; j < kTerms; ++j) {
            const uint32_t both = pack2<KVCRUSH_BF16>(x, y);
            w[c][i / 4][j][i % 4] = both;
            x -= __uint_as_float(both << 16);
            y -= __uint_as_float(both & 0xFFFF0000u);
          }
        }
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d) {
        u32x2 codes;
        if constexpr (F::kBits == 4) codes = v_codes4<F>(vt, lane, d);
#pragma unroll
        for (int ks = 0; ks < U / 2; ++ks) {
          u32x4 vf[F::kVTerms];
          if constexpr (F::kBits == 4)
            vf[0] = codes8_to_bf16(codes[ks]);
          else
            v_frag<F>(vt, lane, d, ks, vf);
          // (what is left of both is below 2^-25 of the product)
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < F::kVTerms; ++i)
#pragma unroll
              for (int j = 0; i + j < kTerms; ++j) mma<KVCRUSH_BF16>(o[c][d], vf[i], w[c][ks][j]);
        }
      }
    }
  }

  // ---- the waves' rows are brought to one reference and added up
  constexpr int kPitch = D + 4;
  float2* ml = (float2*)lds_all;                                    // [waves][NC][16]
  float* sums = (float*)(lds_all + kWaves * NC * 128);              // [waves][16][kPitch]
  uint64_t bad = 0;  // bit 16 c + col: a row of this wave whose sums are not finite
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] = row_sum(l[c]);
    if constexpr (FORMAT == KVCRUSH_I4) z[c] = row_sum(z[c]);
    float check = 0.0f;  // NaN as soon as one value is not finite
#pragma unroll
    for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (FORMAT == KVCRUSH_I4) o[c][d][r] += z[c];
        check = __builtin_fmaf(o[c][d][r], 0.0f, check);
      }
    if (t_of[c] >= n) {  // padding: it sees nothing
      l[c] = 0.0f;
      m[c] = kNegBig;
    }
    const bool stored = row0 + (row_wave * NC + c) * 16 + col < rows && t_of[c] < n;
    const uint64_t rows_of = __ballot(check != 0.0f && stored);
    bad |= ((rows_of | rows_of >> 16 | rows_of >> 32 | rows_of >> 48) & 0xFFFF) << (16 * c);
  }
  // The rows whose sums are not finite are done again.  (Nothing is asked of the values in the loop above: a test of each
  // tile would cost every call.)
#pragma unroll 1
  while (bad != 0) {
    int at[kTogether], of[kTogether];  // which of the wave's rows, and of all
#pragma unroll
    for (int i = 0; i < kTogether; ++i) {
      at[i] = bad != 0 ? __builtin_ctzll(bad) : at[0];
      of[i] = row0 + row_wave * NC * 16 + at[i];
      bad &= bad - 1;
    }
    const Sums<D> y = key_by_key<FORMAT, D>(b, h, t_list, n, of, tile0 * kTile, tile1 * kTile);
#pragma unroll
    for (int i = 0; i < kTogether; ++i) {
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float even = __shfl(y.sum[i][r], 2 * d + (g >> 1)), odd = __shfl(y.sum[i][4 + r], 2 * d + (g >> 1));
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c][d][r] = 16 * c + col == at[i] ? (g & 1 ? odd : even) : o[c][d][r];
        }
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        l[c] = 16 * c + col == at[i] ? y.l[i] : l[c];
        m[c] = 16 * c + col == at[i] ? y.m[i] : m[c];
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (g == 0) ml[(wave * NC + c) * 16 + col] = make_float2(m[c], l[c]);
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float top = kNegBig;
#pragma unroll
    for (int x = 0; x < kGroups; ++x) top = fmaxf(top, ml[((x * RW + row_wave) * NC + c) * 16 + col].x);
    const float a = factor(m[c] - top);
    if (c > 0) __syncthreads();
#pragma unroll
    for (int d = 0; d < F::kDTiles; ++d)
      *(f32x4*)(sums + (wave * 16 + col) * kPitch + d * 16 + 4 * g) = o[c][d] * kWaveRoom * a;
    __syncthreads();
    // four values a thread
    for (int i = tid; i < RW * 16 * (D / 4); i += kWaves * KVC_WAVE) {
      const int of = i / (16 * (D / 4)), row = i / (D / 4) % 16, e = i % (D / 4) * 4;  // (of: the row wave)
      const int r = row0 + (of * NC + c) * 16 + row;
      if (r >= rows) break;  // (rows ascend with i)
      const int t = p.blocks ? t_list : r / p.G, head = h * p.G + (p.blocks ? r : r - t * p.G);
      float most = kNegBig, total = 0.0f;
#pragma unroll
      for (int x = 0; x < kGroups; ++x) most = fmaxf(most, ml[((x * RW + of) * NC + c) * 16 + row].x);
      f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int x = 0; x < kGroups; ++x) {
        const float2 y = ml[((x * RW + of) * NC + c) * 16 + row];
        total += y.y * __builtin_amdgcn_exp2f(y.x - most);
        sum += *(const f32x4*)(sums + ((x * RW + of) * 16 + row) * kPitch + e);
      }
      if (n_split > 1) {
        const size_t at = ((size_t)h * p.pieces + piece) * (p.T * p.G) + t * p.G + (head - h * p.G);
        if (e == 0) p.part_ml[at] = make_float2(most, total);
        *(f32x4*)(p.part_o + at * D + e) = sum;
      } else {
        store_result(p, b, head, t, e, most, total, sum, kWaveRoom);
      }
    }
  }
}

// The pieces of a row (query t of a head): D / 4 lanes of four values.  Few rows: the pieces are dealt to the 256 / (D / 4)
// such groups of a workgroup.  ALONE: each group has a row.
template <int D, bool ALONE>
__global__ __launch_bounds__(256) void attend_merge_kernel(AttendParams p) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ f32x4 sums[ALONE ? 1 : kGroups][kLanes];
  __shared__ float2 mls[ALONE ? 1 : kGroups];
  const int group = threadIdx.x / kLanes, e = threadIdx.x % kLanes * 4;
  const int row = ALONE ? blockIdx.x * kGroups + group : blockIdx.x, part = ALONE ? 0 : group;  // row = (b * Hq + head) * T + t
  if (ALONE && row >= p.c.B * p.Hq * p.T) return;
  const int t = row % p.T, head = row / p.T % p.Hq, b = row / p.T / p.Hq, h = head / p.G;
  int first, n = p.n_split;
  if (n > 0) {
    first = b * n;
  } else {
    first = p.cuts[b].x;
    n = p.cuts[b].y;
    if (n == 1) return;  // (there already; uniform where there is a barrier below)
  }
  const size_t pitch = p.T * p.G, at = ((size_t)h * p.pieces + first) * pitch + t * p.G + (head - h * p.G);
  float m = kNegBig, total = 0.0f;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = part; i < n; i += ALONE ? 1 : kGroups) {
    const float2 x = p.part_ml[at + i * pitch];
    const f32x4 y = *(const f32x4*)(p.part_o + (at + i * pitch) * D + e);
    const float mn = fmaxf(m, x.x), a = factor(m - mn), c = factor(x.x - mn);
    m = mn;
    total = total * a + x.y * c;
    sum = sum * a + y * kPieceRoom * c;
  }
  if constexpr (!ALONE) {
    sums[part][e / 4] = sum;
    if (e == 0) mls[part] = make_float2(m, total);
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int i = 1; i < kGroups; ++i) {
      const float2 x = mls[i];
      const f32x4 y = sums[i][e / 4];
      const float mn = fmaxf(m, x.x), a = factor(m - mn), c = factor(x.x - mn);
      m = mn;
      total = total * a + x.y * c;
      sum = sum * a + y * c;
    }
  }
  store_result(p, b, head, t, e, m, total, sum, kWaveRoom * kPieceRoom);
}

// ------------------------------------------------------------------------------------ host
struct Plan {
  int G, NC, RW, row_tiles, n_split, pieces;  // n_split 0: dealt by length
  int most_pieces;                            // that any length up to this one has
  long long rows;  // B * Hq * T
};

// Keys that one workgroup reads each, and that are more than half of the last-level cache's 256 MB holds, pass the caches
// by: nothing of them is left there for the next step.  (225 MB: 61 -> 55 us; 67 MB, which do stay: 18.6 -> 20.0.  Where
// row tiles or queries share keys, 6 % slower.)
constexpr long long kOnceBytes = 128ll << 20;
constexpr long long kUnits = 256;  // compute units of the chip

kvcrush_status make_plan(const kvcrush_cache* c, const kvcrush_attend_args* a, Plan& plan) {
  kvcrush_status st = check(c);
  if (st != KVCRUSH_OK) return st;
  if (!a || a->Hq < 1 || a->Hq % c->Hkv != 0 || a->T < 1 || !is_dtype(a->dtype)) return KVCRUSH_ERR_INVALID_ARG;
  if (quantised(c->format) ? a->dtype == KVCRUSH_F32 : a->dtype != c->format) return KVCRUSH_ERR_INVALID_ARG;
  if (!(a->softmax_scale >= 0.0f) || a->softmax_scale > 1.0e6f) return KVCRUSH_ERR_INVALID_ARG;
  if (a->mask_stride < 0) return KVCRUSH_ERR_INVALID_ARG;
  if (a->blocks && (a->n_list < 1 || a->unit < 1)) return KVCRUSH_ERR_INVALID_ARG;
  if (a->T > 1024 || (long long)c->B * a->Hq * a->T > (1 << 22) || (long long)c->B * c->Hkv > 65535) return KVCRUSH_ERR_UNSUPPORTED;
  if (a->blocks && (long long)a->n_list * a->unit >= (1 << 30)) return KVCRUSH_ERR_UNSUPPORTED;
  plan.G = a->Hq / c->Hkv;
  plan.rows = (long long)c->B * a->Hq * a->T;
  const long long r = a->blocks ? plan.G : (long long)plan.G * a->T;
  // Rows of a workgroup: 16 or 32 if they are no more; otherwise 64 or 128 that share their tiles, whichever leaves fewer
  // places empty (128 if both leave as many: the keys are read half as often).
  plan.NC = r > 16 ? 2 : 1;
  plan.RW = r <= 32 ? 1 : (r + 127) / 128 * 2 > (r + 63) / 64 ? 2 : 4;
  const int rows = 16 * plan.NC * plan.RW;
  const long long tiles = (r + rows - 1) / rows * (a->blocks ? a->T : 1);
  plan.row_tiles = (int)tiles;
  const long long keys = a->blocks ? std::min<long long>((long long)a->n_list * a->unit, c->capacity) : c->S;
  // One workgroup to a compute unit: as many pieces as leave the fewest keys to the unit that has most, fewer where that
  // gains nothing.
  const long long base = (long long)c->Hkv * tiles;
  int step = 256;  // keys that a workgroup's waves take at a time: no piece is smaller
  with_format(c->format, [&](auto fmt) {
    using F128 = Fmt<decltype(fmt)::value, 128>;
    using F64 = Fmt<decltype(fmt)::value, 64>;
    step = c->D == 128 ? F128::kTile * F128::waves(plan.NC, plan.RW) / plan.RW : F64::kTile * F64::waves(plan.NC, plan.RW) / plan.RW;
    return KVCRUSH_OK;
  });
  const long long most = std::max(1ll, std::min<long long>((keys + step - 1) / step, kMaxSplit));
  // Time of n pieces a sequence, in us as measured at both ends: 4 for a workgroup and 1.5 for each tile of its waves, in
  // rounds of one workgroup to a compute unit; 5 to merge pieces (3.5 on the chip, and the host launches for 3.4 as well).
  // 2 sequences of 160 keys in one piece each take 10.4, in two 14.2; 8 of 2048 in one 32, in four 18.6.
  const long long workgroups = base * c->B, steps = (keys + step - 1) / step;
  const long long n_end = std::min(most, 2 * kUnits / workgroups + 1);
  double least = 0.0;
  plan.n_split = 1;
  for (long long n = 1; n <= n_end; ++n) {
    const double us = (double)((workgroups * n + kUnits - 1) / kUnits) * (4.0 + 1.5 * (double)((steps + n - 1) / n)) + (n > 1 ? 5.0 : 0.0);
    if (n > 1 && us >= 0.97 * least) continue;
    least = us;
    plan.n_split = (int)n;
  }
  plan.pieces = c->B * plan.n_split;
  if (plan.n_split > 1 && c->lengths && !a->blocks && c->B > 1 && c->B <= KVC_WAVE) {
    plan.n_split = 0;
    plan.pieces = (int)std::max<long long>(c->B, std::min(kUnits / base, n_end * c->B));
  }
  plan.most_pieces = (int)(n_end * c->B);
  return KVCRUSH_OK;
}

constexpr size_t kCutBytes = KVC_WAVE * sizeof(int2);
// The scratch memory is that of the most pieces, so that a longer sequence never needs less than a shorter one.
bool merged(const Plan& p) { return p.most_pieces > p.pieces || p.n_split != 1; }
long long part_rows(const kvcrush_cache* c, const kvcrush_attend_args* a, const Plan& p) {
  return (long long)a->Hq * a->T * p.most_pieces;
}
size_t ml_bytes(long long rows) { return kvc::align_up((size_t)rows * sizeof(float2), 256); }
size_t plan_bytes(const kvcrush_cache* c, const kvcrush_attend_args* a, const Plan& p) {
  if (!merged(p)) return 0;
  const long long rows = part_rows(c, a, p);
  return kCutBytes + ml_bytes(rows) + (size_t)rows * c->D * sizeof(float);
}

template <class F, int NC, int RW>
kvcrush_status launch_attend(const AttendParams& p, hipStream_t stream) {
  constexpr int kWaves = F::waves(NC, RW);
  constexpr int kLoop = F::lds(kWaves, RW), kEnd = kWaves * (NC * 128 + 16 * (F::D + 4) * 4);
  constexpr int kLds = kLoop > kEnd ? kLoop : kEnd;
  static_assert(kLds <= kvc::kLdsPerWorkgroup, "LDS of a workgroup");
  kvcrush_status st = kvc::allow_large_lds<attend_kernel<F, NC, RW>>(0);
  if (st != KVCRUSH_OK) return st;
  const dim3 grid((unsigned)((p.c.Hkv * p.pieces + 7) / 8 * 8) * p.row_tiles);
  st = kvc::launch(attend_kernel<F, NC, RW>, grid, dim3(kWaves * KVC_WAVE), kLds, stream, p);
  if (st != KVCRUSH_OK || p.n_split == 1) return st;
  // With eight workgroups to a compute unit or more, each row's lanes merge its pieces alone, unless those are many (4096
  // rows of 8 pieces: 7.2 -> 5.1 us).
  const int rows = p.c.B * p.Hq * p.T, groups = 1024 / F::D;
  if (rows >= 8 * kUnits && p.pieces <= 16 * p.c.B)
    return kvc::launch(attend_merge_kernel<F::D, true>, dim3((unsigned)((rows + groups - 1) / groups)), dim3(256), 0, stream, p);
  return kvc::launch(attend_merge_kernel<F::D, false>, dim3((unsigned)rows), dim3(256), 0, stream, p);
}

template <class F>
kvcrush_status launch_rows(const AttendParams& p, const Plan& plan, hipStream_t stream) {
  if (plan.NC == 1) return launch_attend<F, 1, 1>(p, stream);
  return plan.RW == 1 ? launch_attend<F, 2, 1>(p, stream) : plan.RW == 2 ? launch_attend<F, 2, 2>(p, stream) : launch_attend<F, 2, 4>(p, stream);
}

}  // namespace

extern "C" size_t kvcrush_attend_workspace(const kvcrush_cache* cache, const kvcrush_attend_args* args) {
  Plan plan;
  return make_plan(cache, args, plan) == KVCRUSH_OK ? plan_bytes(cache, args, plan) : 0;
}

extern "C" kvcrush_status kvcrush_attend(const kvcrush_cache* cache, const kvcrush_attend_args* args, const void* q,
                                         void* out, float* lse, void* workspace, size_t workspace_bytes,
                                         void* hip_stream) {
  Plan plan;
  kvcrush_status st = make_plan(cache, args, plan);
  if (st != KVCRUSH_OK) return st;
  if (!q || !out || !kvc::aligned16(q) || !kvc::aligned16(out) || (lse && !kvc::aligned16(lse))) return KVCRUSH_ERR_INVALID_ARG;
  AttendParams p;
  const int D = cache->D, elem = format_bits(args->dtype) / 8;
  if (!strides_ok(args->q_stride, args->Hq, args->T, D, elem, 0, p.q_stride) ||
      !strides_ok(args->out_stride, args->Hq, args->T, D, elem, D, p.out_stride))
    return KVCRUSH_ERR_INVALID_ARG;
  const size_t need = plan_bytes(cache, args, plan);
  if (need > 0 && (!workspace || !kvc::aligned16(workspace) || workspace_bytes < need)) return KVCRUSH_ERR_WORKSPACE;
  p.c = view(cache);
  p.q = (const char*)q;
  p.out = (char*)out;
  p.lse = lse;
  p.cuts = (int2*)workspace;
  p.part_ml = (float2*)((char*)workspace + kCutBytes);
  p.part_o = need > 0 ? (float*)((char*)p.part_ml + ml_bytes(part_rows(cache, args, plan))) : nullptr;
  p.mask = args->mask;
  p.mask_stride = args->mask_stride;
  p.mask_words = (args->T + 63) / 64;
  p.n_new = args->n_new;
  p.blocks = args->blocks;
  p.n_list = args->blocks ? args->n_list : 0;
  p.unit = args->blocks ? args->unit : 1;
  p.Hq = args->Hq;
  p.G = plan.G;
  p.T = args->T;
  p.n_split = plan.n_split;
  p.row_tiles = plan.row_tiles;
  p.pieces = plan.pieces;
  p.once = plan.row_tiles == 1 && !args->blocks &&
           2ll * cache->B * cache->Hkv * cache->S * D * format_bits(cache->format) / 8 >= kOnceBytes;
  p.q_dtype = args->dtype;
  p.scale_log2 = (float)(1.4426950408889634 *
                         (args->softmax_scale != 0.0f ? (double)args->softmax_scale : 1.0 / sqrt((double)D)));
  hipStream_t stream = (hipStream_t)hip_stream;
  return with_format(cache->format, [&](auto fmt) -> kvcrush_status {
    constexpr int FMT = decltype(fmt)::value;
    return D == 128 ? launch_rows<Fmt<FMT, 128>>(p, plan, stream) : launch_rows<Fmt<FMT, 64>>(p, plan, stream);
  });
}
