// Attention of a few new tokens over a KV cache (one token, a drafted chain or tree), dense or paged, in its
// own type or quantised, over all of it or over listed blocks.
//
// The queries of all heads of a KV group and of all new tokens are the rows that one key serves: R = T * G of
// them.  A wave takes 32 keys at a time and 32 or 64 of those rows (NC = 1, 2):
//   S^T = K Q^T      keys x rows, 32x32 matrix instructions: a lane holds one row's logits of 16 keys
//   softmax          running maximum and sum per row in registers
//   O^T += V^T P^T   the probabilities are already laid out as the second product's operand; V is read
//                    transposed from LDS (ds_read_b64_tr)
// Waves share nothing until their keys are done: each copies its own tiles into its own part of the LDS, and
// the workgroup's waves merge their rows at the end.  The keys of a sequence are cut over workgroups so that the
// chip is full; the pieces' results are merged by a second kernel.
#include <algorithm>
#include <cmath>

#include "cache.h"
#include "tiles.h"

namespace {

using namespace kvc::cache;
using kvc::tiles::f32x16;
using kvc::tiles::kLn2;
using kvc::tiles::kNegBig;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr float kMasked = -3.0e38f;  // below every running maximum (>= kNegBig) by more than any exponent
constexpr int kTile = 32;            // keys of a tile
constexpr int kAhead = 1024;         // keys whose places a wave looks up at once

struct AttendParams {
  View c;
  const char* q;
  char* out;
  float* lse;
  float* part_o;   // workspace [B * Hkv * rows][n_split][D], rows = G * T
  float2* part_ml;  // workspace [B * Hkv * rows][n_split]
  const uint64_t* mask;
  const int32_t* n_new;
  const int32_t* blocks;
  int64_t q_stride[3], out_stride[3];  // elements
  int64_t mask_stride;
  int Hq, G, T, n_split, n_list, unit, mask_words, q_dtype;
  float scale_log2;
};

template <int FORMAT_, int D_>
struct Fmt {
  static constexpr int FORMAT = FORMAT_, D = D_;
  static constexpr bool kQuant = quantised(FORMAT);
  static constexpr int kBits = format_bits(FORMAT);
  static constexpr int kRow = D * kBits / 8;       // bytes of a row
  static constexpr int kChunks = kRow / 16;        // 16-byte chunks of a row
  static constexpr int kTileBytes = kTile * kRow;
  static constexpr int kLoads = kTileBytes / 1024;  // wave instructions that copy a tile
  static constexpr int kParam = kQuant ? (FORMAT == KVCRUSH_I4 ? 2 : 1) : 0;  // floats beside a row
  static constexpr int kParamBytes = 2 * kTile * 4 * kParam;                  // K's, then V's, of a tile
  static constexpr int kStage = 2 * kTileBytes + kParamBytes;
  static constexpr int kWaves = kRow == 512 ? 2 : 4;
  static constexpr int kSteps = D / 16;            // matrix steps of 16 values along D (16-bit operands)
  static constexpr int kDTiles = D / 32;
  static_assert(kTileBytes % 1024 == 0, "whole wave instructions");

  // XOR on a 16-byte chunk's place in its 256-byte line.  K is read one chunk a lane, neighbouring lanes
  // neighbouring rows; V in pieces of 16 values x 4, 8 or 16 rows (transposed), which must not share banks.
  __device__ static int k_xor(int line) { return line & 15; }
  __device__ static int v_xor(int line) {
    if constexpr (kBits == 32) return kRow == 512 ? ((line >> 3) & 1) << 3 : ((line >> 2) & 1) << 3;
    if constexpr (kBits == 16) return kRow == 256 ? ((line & 3) << 2) | ((line >> 2) & 3) : (line & 1) << 2;
    if constexpr (kBits == 8) return kRow == 128 ? ((line & 1) | ((line >> 1) & 2)) << 1 : ((line >> 1) & 1) << 1;
    return kRow == 64 ? (line >> 1) & 3 : (line & 1) | ((line & 2) << 2);
  }
  template <bool V>
  __device__ static int chunk_at(int row, int chunk) {  // byte offset in the tile's image
    const int q = row * kChunks + chunk, line = q >> 4;
    return (line << 8) | (((q & 15) ^ (V ? v_xor(line) : k_xor(line))) << 4);
  }
  // The row and chunk whose bytes lie at physical chunk `p` of the image.
  template <bool V>
  __device__ static void chunk_of(int p, int& row, int& chunk) {
    const int line = p >> 4, q = line * 16 + ((p & 15) ^ (V ? v_xor(line) : k_xor(line)));
    row = q / kChunks;
    chunk = q % kChunks;
  }
};

// C += A B^T for one step of 16 values along the inner axis; operands are halves unless the cache is bfloat16.
template <int FORMAT>
__device__ __forceinline__ void mma16(f32x16& c, const u32x4& a, const u32x4& b) {
  if constexpr (FORMAT == KVCRUSH_BF16)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
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

__device__ __forceinline__ int acc_key(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// K fragments of the 32 keys for 16-byte chunk j of this lane's half of a row: kSub matrix steps.
template <class F>
struct KFrag {
  static constexpr int kSub = F::kBits == 32 ? 1 : 16 / F::kBits;  // steps that one chunk feeds
  u32x4 f[kSub];
  __device__ __forceinline__ void load(const char* tile, int lane, int j) {
    const u32x4 w = *(const u32x4*)(tile + F::template chunk_at<false>(lane & 31, (lane >> 5) * (F::kChunks / 2) + j));
    if constexpr (F::kBits >= 16) {
      f[0] = w;
    } else if constexpr (F::kBits == 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x2 a = codes4_to_f16<F::FORMAT>(w[2 * i]), b = codes4_to_f16<F::FORMAT>(w[2 * i + 1]);
        f[i] = u32x4{a[0], a[1], b[0], b[1]};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = codes8_to_f16(w[i]);
    }
  }
};

// V^T fragment: lane = value d (of 32) of tile dt, the eight keys acc_key(8 * step + e, half) in order.
template <class F>
__device__ __forceinline__ u32x4 v_frag(const char* tile, int lane, int dt, int step) {
  const int half = lane >> 5, group = (lane >> 4) & 1, i = lane & 15;
  if constexpr (F::kBits == 16) {
    const int row = 16 * step + 4 * half + (i >> 2), chunk = dt * 4 + group * 2 + ((i & 3) >> 1), off = (i & 1) * 8;
    const u32x2 a = read_tr16(tile + F::template chunk_at<true>(row, chunk) + off);
    const u32x2 b = read_tr16(tile + F::template chunk_at<true>(row + 8, chunk) + off);
    return u32x4{a[0], a[1], b[0], b[1]};
  } else {
    static_assert(F::kBits == 8, "");
    const int row = acc_key(8 * step + (i >> 1), half);
    const u32x2 w = read_tr8(tile + F::template chunk_at<true>(row, dt * 2 + group) + (i & 1) * 8);
    const u32x2 a = codes4_to_f16<F::FORMAT>(w[0]), b = codes4_to_f16<F::FORMAT>(w[1]);
    return u32x4{a[0], a[1], b[0], b[1]};
  }
}
// Both steps' fragments of 4-bit codes: one read.  codes8_to_f16's order is undone by the order of the rows.
template <class F>
__device__ __forceinline__ u32x2 v_codes4(const char* tile, int lane, int dt) {
  const int half = lane >> 5, group = (lane >> 4) & 1, i = lane & 15, j = i & 7;
  const int row = acc_key((i & 8) + (j < 4 ? 2 * j : 2 * j - 7), half);
  return read_tr4(tile + F::template chunk_at<true>(row, dt) + group * 8);
}

template <int FORMAT>
__device__ __forceinline__ bool all_finite(uint32_t w) {  // the values in one word
  if constexpr (FORMAT == KVCRUSH_F32) return (w & 0x7F800000u) != 0x7F800000u;
  if constexpr (FORMAT == KVCRUSH_BF16) return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u;
  if constexpr (FORMAT == KVCRUSH_F16) return (w & 0x7C00u) != 0x7C00u && (w & 0x7C000000u) != 0x7C000000u;
  w &= 0x7F7F7F7Fu;  // e4m3: 0x7F is NaN
  return (w & 255u) != 127u && ((w >> 8) & 255u) != 127u && ((w >> 16) & 255u) != 127u && (w >> 24) != 127u;
}
// Value d of row `key` of V's tile, as it enters the second product.
template <class F>
__device__ __forceinline__ float tile_value(const char* tile, int key, int d) {
  const int at = d * F::kBits / 8;
  const char* p = tile + F::template chunk_at<true>(key, at >> 4) + (at & 15);
  if constexpr (F::FORMAT == KVCRUSH_F32) return *(const float*)p;
  if constexpr (F::FORMAT == KVCRUSH_BF16) return __uint_as_float((uint32_t) * (const uint16_t*)p << 16);
  if constexpr (F::FORMAT == KVCRUSH_F16) return (float)*(const _Float16*)p;
  const u32x2 h = codes4_to_f16<F::FORMAT>(*(const uint8_t*)p);
  return (float)as_f16x2(h[0])[0];
}

// What a query sees of one key slot: position and whether the slot exists.
struct Slots {
  const int32_t* list;  // this query's blocks, or null
  int n, unit, L;
  __device__ bool position(int slot, int& pos) const {
    pos = slot;
    if (slot >= n) return false;
    if (list) {
      const int e = slot / unit, blk = list[e];
      if (blk < 0 || (e > 0 && blk <= list[e - 1]) || blk > (L - 1) / unit) return false;
      pos = blk * unit + (slot - e * unit);
    }
    return pos < L;
  }
};

template <class F, int NC>
__global__ __launch_bounds__(F::kWaves * KVC_WAVE) void attend_kernel(AttendParams p) {
  constexpr int D = F::D, FORMAT = F::FORMAT;
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  const int tid = threadIdx.x, lane = kvc::lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / KVC_WAVE);
  const int half = lane >> 5, col = lane & 31;
  const int split = blockIdx.x, bh = blockIdx.z, b = bh / p.c.Hkv, h = bh % p.c.Hkv;
  const int L = p.c.length(b), n = new_tokens(p.n_new, b, p.T, L);
  const int t_list = p.blocks ? (int)blockIdx.y : 0;           // with lists: the query, whose G heads are the rows
  const int row0 = p.blocks ? 0 : (int)blockIdx.y * 32 * NC;
  const int rows = p.blocks ? p.G : p.G * p.T;

  Slots slots;
  slots.list = p.blocks ? p.blocks + ((size_t)bh * p.T + t_list) * p.n_list : nullptr;
  slots.unit = p.blocks ? p.unit : 1;
  slots.n = p.blocks ? (t_list < n ? p.n_list * p.unit : 0) : n > 0 ? L : 0;
  slots.L = L;

  // this lane's rows
  int t_of[NC];
  const char* q_row[NC];
  bool live[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int r = row0 + c * 32 + col;
    live[c] = r < rows;
    const int rr = live[c] ? r : rows - 1;
    const int t = p.blocks ? t_list : rr / p.G, g = p.blocks ? rr : rr - t * p.G;
    t_of[c] = t;
    const int elem = format_bits(p.q_dtype) / 8;
    q_row[c] = p.q + ((size_t)b * p.q_stride[0] + (size_t)(h * p.G + g) * p.q_stride[1] + (size_t)t * p.q_stride[2]) * elem;
  }

  // queries as the first product's other operand: in the order of the K fragments
  constexpr int kQRegs = F::kBits == 32 ? D / 8 : F::kSteps;
  u32x4 qf[NC][kQRegs];
  float col_scale[NC], q_sum[NC];  // logit = (products) * col_scale; q_sum: the lowest value's factor
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    col_scale[c] = p.scale_log2;
    q_sum[c] = 0.0f;
    if constexpr (!F::kQuant) {
#pragma unroll
      for (int j = 0; j < kQRegs; ++j) qf[c][j] = *(const u32x4*)(q_row[c] + (half * kQRegs + j) * 16);
    } else {
      // Halves for every type of query: a row is scaled by the power of two that brings its largest value to
      // 2^14 .. 2^15, so that a bfloat16 value loses nothing unless it is 2^-29 of the largest.
      float x[F::kSteps][8];
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) {
        const int d = half * (D / 2) + s * 8;
        if (p.q_dtype == KVCRUSH_BF16)
          load8<KVCRUSH_BF16>(q_row[c] + d * 2, x[s]);
        else
          load8<KVCRUSH_F16>(q_row[c] + d * 2, x[s]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          top = max(top, __float_as_uint(x[s][i]) & 0x7FFFFFFFu);
          q_sum[c] += x[s][i];
        }
      }
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      q_sum[c] += __shfl_xor(q_sum[c], 32);
      const int up = min(141 - (int)(top >> 23), 126);  // >= -114
      const float by = __builtin_amdgcn_ldexpf(1.0f, up);
      q_sum[c] *= by;
      col_scale[c] = p.scale_log2 * __builtin_amdgcn_ldexpf(1.0f, -up);
      constexpr int kOrder[2][8] = {{0, 1, 2, 3, 4, 5, 6, 7}, {0, 4, 1, 5, 2, 6, 3, 7}};
      constexpr int o = FORMAT == KVCRUSH_I4 ? 1 : 0;
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          qf[c][s][i] = pack2<KVCRUSH_F16>(x[s][kOrder[o][2 * i]] * by, x[s][kOrder[o][2 * i + 1]] * by);
    }
  }

  f32x16 o[NC][F::kDTiles];
  float m[NC], l[NC], z[NC];  // running maximum (base 2), sum of this half's keys, sum of probability x lowest value
  float unit[NC];             // quantised: what o is to be multiplied with
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNegBig;
    l[c] = z[c] = unit[c] = 0.0f;
#pragma unroll
    for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[c][d][r] = 0.0f;
  }

  // this wave's tiles: a contiguous piece of the workgroup's
  const int tiles = (slots.n + kTile - 1) / kTile, per_wg = (tiles + p.n_split - 1) / p.n_split;
  const int wg0 = min(split * per_wg, tiles), wg1 = min(wg0 + per_wg, tiles);
  const int per_wave = (wg1 - wg0 + F::kWaves - 1) / F::kWaves;
  const int tile0 = min(wg0 + wave * per_wave, wg1), tile1 = min(tile0 + per_wave, wg1);

  char* stage = lds_all + wave * (F::kStage + kAhead * 4);
  int* places = (int*)(stage + F::kStage);  // token of each slot; bit 31: the slot has to be looked at
  const size_t row_base = p.c.base(b, h), row_step = p.c.step();
  const bool lookup = p.c.table || p.blocks;
  const int first_new = L - n;

  for (int tile = tile0; tile < tile1; ++tile) {
    const int k0 = tile * kTile, ahead = (tile - tile0) & (kAhead / kTile - 1);
    if (lookup && ahead == 0) {
      const int end = min(kAhead, (tile1 - tile) * kTile);
      for (int i = lane; i < end; i += KVC_WAVE) {
        int pos;
        const bool there = slots.position(k0 + i, pos);
        const int at = p.c.token(b, there ? pos : 0);
        places[i] = at | (!there || pos >= first_new ? (int)0x80000000 : 0);
      }
      kvc::wave_fence();
    }
    // ---- the tile's rows, their parameters
    auto row_of = [&](int key) -> size_t {
      const int tok = lookup ? places[ahead * kTile + key] & 0x7FFFFFFF : min(k0 + key, L - 1);
      return row_base + (size_t)tok * row_step;
    };
#pragma unroll
    for (int j = 0; j < F::kLoads; ++j) {
      int row, chunk;
      F::template chunk_of<false>(j * 64 + lane, row, chunk);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p.c.k + row_of(row) * F::kRow + chunk * 16),
                                       (__attribute__((address_space(3))) void*)(stage + j * 1024), 16, 0, 0);
      F::template chunk_of<true>(j * 64 + lane, row, chunk);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p.c.v + row_of(row) * F::kRow + chunk * 16),
                                       (__attribute__((address_space(3))) void*)(stage + F::kTileBytes + j * 1024), 16, 0, 0);
    }
    if constexpr (F::kQuant) {
      const float* src = half ? p.c.v_param : p.c.k_param;
      float* dst = (float*)(stage + 2 * F::kTileBytes) + half * kTile * F::kParam;
      const size_t row = row_of(col);
#pragma unroll
      for (int i = 0; i < F::kParam; ++i) dst[i * kTile + col] = src[row * F::kParam + i];
    }
    bool look = lookup ? __ballot(places[ahead * kTile + col] < 0) != 0 : k0 + kTile > first_new;
    kvc::tiles::wait_async_loads();
    kvc::wave_fence();
    const char *kt = stage, *vt = stage + F::kTileBytes;
    const float* kp = (const float*)(stage + 2 * F::kTileBytes);
    const float* vp = kp + kTile * F::kParam;

    // ---- logits
    f32x16 s[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[c][r] = 0.0f;
    constexpr int kSub = KFrag<F>::kSub;
#pragma unroll
    for (int j = 0; j < F::kChunks / 2; ++j) {
      KFrag<F> kf;
      kf.load(kt, lane, j);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if constexpr (F::kBits == 32) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.f[0][i]), __uint_as_float(qf[c][j][i]), s[c], 0, 0, 0);
        } else {
#pragma unroll
          for (int i = 0; i < kSub; ++i) mma16<FORMAT>(s[c], kf.f[i], qf[c][j * kSub + i]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = acc_key(r, half);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float x = s[c][r];
        if constexpr (FORMAT == KVCRUSH_I4)
          x = __builtin_fmaf(x, kp[key], kp[kTile + key] * q_sum[c]);
        else if constexpr (F::kQuant)
          x *= kp[key];
        s[c][r] = x * col_scale[c];
      }
    }
    uint32_t seen[NC];  // bit r: this row sees the key of register r
#pragma unroll
    for (int c = 0; c < NC; ++c) seen[c] = 0xFFFFu;
    if (look) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint64_t* words = p.mask ? p.mask + (size_t)b * p.mask_stride + (size_t)t_of[c] * p.mask_words : nullptr;
        for (int r = 0; r < 16; ++r) {
          int pos;
          bool see = slots.position(k0 + acc_key(r, half), pos) && t_of[c] < n;
          const int draft = pos - first_new;
          if (see && draft >= 0) see = words ? (words[draft >> 6] >> (draft & 63)) & 1 : draft <= t_of[c];
          if (!see) seen[c] &= ~(1u << r);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!((seen[c] >> r) & 1)) s[c][r] = kMasked;
      }
    }

    // ---- running maximum; the sums so far are brought to it
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float t = s[c][0];
#pragma unroll
      for (int r = 1; r < 16; ++r) t = fmaxf(t, s[c][r]);
      t = fmaxf(t, __shfl_xor(t, 32));
      const float mn = fmaxf(m[c], t), a = __builtin_amdgcn_exp2f(m[c] - mn);
      m[c] = mn;
      l[c] *= a;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[c][r] = __builtin_amdgcn_exp2f(s[c][r] - mn);
        l[c] += s[c][r];
      }
      float down = a;
      if constexpr (F::kQuant) {
        // what multiplies the codes: probability x scale, as a share of the largest such product of this row so far
        if constexpr (FORMAT == KVCRUSH_I4) z[c] *= a;
        float top = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = acc_key(r, half);
          const bool see = (seen[c] >> r) & 1;
          if constexpr (FORMAT == KVCRUSH_I4) z[c] = see ? __builtin_fmaf(s[c][r], vp[kTile + key], z[c]) : z[c];
          s[c][r] = see ? s[c][r] * vp[key] : 0.0f;
          top = fmaxf(top, s[c][r]);  // (a NaN is passed over)
        }
        top = fmaxf(top, __shfl_xor(top, 32));
        const float before = unit[c] * a;
        unit[c] = fmaxf(before, top);
        const float inv = unit[c] > 0.0f ? 1.0f / unit[c] : 0.0f;
        down = before * inv;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[c][r] *= inv;
      }
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][d][r] *= down;
    }
    if constexpr (FORMAT != KVCRUSH_I8 && FORMAT != KVCRUSH_I4) {
      if (look) {
        // A value that is not finite must not reach the rows that do not see its key (0 x NaN): such keys are
        // added one by one, to the rows that do, and taken out of the tile.
        uint32_t bad = 0;
#pragma unroll
        for (int j = 0; j < F::kLoads; ++j) {
          const u32x4 w = *(const u32x4*)(vt + j * 1024 + lane * 16);
          bool odd = false;
#pragma unroll
          for (int i = 0; i < 4; ++i) odd = odd || !all_finite<FORMAT>(w[i]);
          int row, chunk;
          F::template chunk_of<true>(j * 64 + lane, row, chunk);
          if (odd) bad |= 1u << row;
        }
        bad = kvc::wave_reduce(bad, 0u, [](uint32_t x, uint32_t y) { return x | y; });
        if (bad) {
          for (uint32_t left = bad; left; left &= left - 1) {
            const int key = __builtin_ctz(left), reg = (key & 3) + 4 * (key >> 3), from = col + 32 * ((key >> 2) & 1);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              float x = 0.0f;
#pragma unroll
              for (int r = 0; r < 16; ++r) x = r == reg ? s[c][r] : x;
              x = __shfl(x, from);
              if (__shfl((int)((seen[c] >> reg) & 1), from)) {
#pragma unroll
                for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
                  for (int r = 0; r < 16; ++r)
                    o[c][d][r] += x * tile_value<F>(vt, key, d * 32 + acc_key(r, half));
              }
            }
          }
          kvc::wave_fence();
#pragma unroll
          for (int j = 0; j < F::kLoads; ++j) {
            int row, chunk;
            F::template chunk_of<true>(j * 64 + lane, row, chunk);
            if ((bad >> row) & 1) *(u32x4*)(stage + F::kTileBytes + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
          }
          kvc::wave_fence();
        }
      }
    }

    // ---- values
    if constexpr (F::kBits == 32) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
#pragma unroll
        for (int d = 0; d < F::kDTiles; ++d) {
          const int e = d * 32 + col;  // value
          const float v = *(const float*)(vt + F::template chunk_at<true>(acc_key(r, half), e >> 2) + (e & 3) * 4);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[c][r], o[c][d], 0, 0, 0);
        }
      }
    } else {
      // a probability is the sum of two 16-bit values: its rounding and what that left
      constexpr int P = FORMAT == KVCRUSH_BF16 ? KVCRUSH_BF16 : KVCRUSH_F16;
      u32x4 hi[NC][2], lo[NC][2];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = s[c][8 * st + 2 * i], y = s[c][8 * st + 2 * i + 1];
            // (values from here on: otherwise the compiler may round the product behind x to 16 bits in one step for
            // `hi` and in two for what `hi` left)
            asm("" : "+v"(x), "+v"(y));
            const uint32_t w = pack2<P>(x, y);
            float xh, yh;
            if constexpr (P == KVCRUSH_BF16) {
              xh = __uint_as_float(w << 16);
              yh = __uint_as_float(w & 0xFFFF0000u);
            } else {
              const f16x2 f = as_f16x2(w);
              xh = (float)f[0];
              yh = (float)f[1];
            }
            hi[c][st][i] = w;
            lo[c][st][i] = pack2<P>(x - xh, y - yh);
          }
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d) {
        u32x2 codes;
        if constexpr (F::kBits == 4) codes = v_codes4<F>(vt, lane, d);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          u32x4 vf;
          if constexpr (F::kBits == 4)
            vf = codes8_to_f16(codes[st]);
          else
            vf = v_frag<F>(vt, lane, d, st);
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            mma16<FORMAT>(o[c][d], vf, hi[c][st]);
            mma16<FORMAT>(o[c][d], vf, lo[c][st]);
          }
        }
      }
    }
    kvc::wave_fence();  // the stage's last reads come before its next copies
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // ---- the waves' rows are brought to one maximum and added up
  float* ml = (float*)lds_all;                                     // [waves][NC][32][2]
  float* sums = (float*)(lds_all + F::kWaves * NC * 256);          // [waves / 2][64 lanes][16 D / 32 + 1]
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 32);
    if (t_of[c] >= n) {  // padding: it sees nothing
      l[c] = 0.0f;
      m[c] = kNegBig;
    }
    if constexpr (FORMAT == KVCRUSH_I4) z[c] += __shfl_xor(z[c], 32);
    if constexpr (F::kQuant) {
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if constexpr (FORMAT == KVCRUSH_I4)
            o[c][d][r] = __builtin_fmaf(o[c][d][r], unit[c], z[c]);
          else
            o[c][d][r] *= unit[c];
        }
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (half == 0) *(float2*)(ml + ((wave * NC + c) * 32 + col) * 2) = make_float2(m[c], l[c]);
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float mt = kNegBig, lt = 0.0f;
#pragma unroll
    for (int w = 0; w < F::kWaves; ++w) mt = fmaxf(mt, ml[((w * NC + c) * 32 + col) * 2]);
#pragma unroll
    for (int w = 0; w < F::kWaves; ++w) {
      const float2 x = *(const float2*)(ml + ((w * NC + c) * 32 + col) * 2);
      lt += x.y * __builtin_amdgcn_exp2f(x.x - mt);
    }
    const float a = __builtin_amdgcn_exp2f(m[c] - mt);
    l[c] = lt;
    m[c] = mt;
    constexpr int kPer = 16 * F::kDTiles;
#pragma unroll
    for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[c][d][r] *= a;
    for (int left = F::kWaves / 2; left > 0; left /= 2) {  // waves left .. 2 left - 1 hand theirs to 0 .. left - 1
      __syncthreads();
      if (wave >= left && wave < 2 * left) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) sums[((wave - left) * kPer + i) * 64 + lane] = o[c][i / 16][i % 16];
      }
      __syncthreads();
      if (wave < left) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[c][i / 16][i % 16] += sums[(wave * kPer + i) * 64 + lane];
      }
    }
  }
  if (wave != 0) return;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    if (!live[c]) continue;
    const int r = row0 + c * 32 + col, t = t_of[c], g = p.blocks ? r : r - t * p.G;
    if (p.n_split > 1) {
      const size_t at = (((size_t)bh * p.G + g) * p.T + t) * p.n_split + split;
      if (half == 0) p.part_ml[at] = make_float2(m[c], l[c]);
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(float4*)(p.part_o + at * D + d * 32 + 8 * q + 4 * half) =
              make_float4(o[c][d][4 * q], o[c][d][4 * q + 1], o[c][d][4 * q + 2], o[c][d][4 * q + 3]);
    } else {
      const float inv = l[c] > 0.0f || l[c] != l[c] ? 1.0f / l[c] : 0.0f;
      const int head = h * p.G + g;
      if (p.lse && half == 0)
        p.lse[((size_t)b * p.Hq + head) * p.T + t] = l[c] == 0.0f ? -__builtin_inff() : (m[c] + __builtin_amdgcn_logf(l[c])) * kLn2;
      const size_t at = (size_t)b * p.out_stride[0] + (size_t)head * p.out_stride[1] + (size_t)t * p.out_stride[2];
#pragma unroll
      for (int d = 0; d < F::kDTiles; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const size_t e = at + d * 32 + 8 * q + 4 * half;
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = l[c] == 0.0f ? 0.0f : o[c][d][4 * q + i] * inv;
          if (FORMAT == KVCRUSH_F32)
            *(float4*)(p.out + e * 4) = make_float4(x[0], x[1], x[2], x[3]);
          else if (p.q_dtype == KVCRUSH_BF16)
            *(u32x2*)(p.out + e * 2) = u32x2{pack2<KVCRUSH_BF16>(x[0], x[1]), pack2<KVCRUSH_BF16>(x[2], x[3])};
          else
            *(u32x2*)(p.out + e * 2) = u32x2{pack2<KVCRUSH_F16>(x[0], x[1]), pack2<KVCRUSH_F16>(x[2], x[3])};
        }
    }
  }
}

// The pieces of a row (query t of head hq): D / 4 lanes, four values each.
template <int D>
__global__ __launch_bounds__(256) void attend_merge_kernel(AttendParams p) {
  constexpr int kLanes = D / 4;
  const long long row = (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;  // (b * Hq + head) * T + t
  if (row >= (long long)p.c.B * p.Hq * p.T) return;
  const int e = threadIdx.x % kLanes * 4;
  const float2* ml = p.part_ml + row * p.n_split;
  float m = kNegBig;
  for (int i = 0; i < p.n_split; ++i) m = fmaxf(m, ml[i].x);
  float l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i = 0; i < p.n_split; ++i) {
    const float2 x = ml[i];
    const float a = __builtin_amdgcn_exp2f(x.x - m);
    const float4 y = *(const float4*)(p.part_o + (row * p.n_split + i) * D + e);
    l += x.y * a;
    o.x += y.x * a, o.y += y.y * a, o.z += y.z * a, o.w += y.w * a;
  }
  const int t = (int)(row % p.T), head = (int)(row / p.T % p.Hq), b = (int)(row / p.T / p.Hq);
  if (p.lse && e == 0) p.lse[row] = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (l == 0.0f) o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const size_t at = (size_t)b * p.out_stride[0] + (size_t)head * p.out_stride[1] + (size_t)t * p.out_stride[2] + e;
  if (p.q_dtype == KVCRUSH_F32)
    *(float4*)(p.out + at * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else if (p.q_dtype == KVCRUSH_BF16)
    *(u32x2*)(p.out + at * 2) = u32x2{pack2<KVCRUSH_BF16>(o.x * inv, o.y * inv), pack2<KVCRUSH_BF16>(o.z * inv, o.w * inv)};
  else
    *(u32x2*)(p.out + at * 2) = u32x2{pack2<KVCRUSH_F16>(o.x * inv, o.y * inv), pack2<KVCRUSH_F16>(o.z * inv, o.w * inv)};
}

// ------------------------------------------------------------------------------------ host
struct Plan {
  int G, NC, row_tiles, n_split;
  long long rows;  // B * Hq * T
};

constexpr int kMaxSplit = 128;

kvcrush_status make_plan(const kvcrush_cache* c, const kvcrush_attend_args* a, Plan& plan) {
  kvcrush_status st = check(c);
  if (st != KVCRUSH_OK) return st;
  if (!a || a->Hq < 1 || a->Hq % c->Hkv != 0 || a->T < 1 || !is_dtype(a->dtype)) return KVCRUSH_ERR_INVALID_ARG;
  if (quantised(c->format) ? a->dtype == KVCRUSH_F32 : a->dtype != c->format) return KVCRUSH_ERR_INVALID_ARG;
  if (!(a->softmax_scale >= 0.0f) || a->softmax_scale > 1.0e6f) return KVCRUSH_ERR_INVALID_ARG;
  if (a->mask_stride < 0) return KVCRUSH_ERR_INVALID_ARG;
  if (a->blocks && (a->n_list < 1 || a->unit < 1)) return KVCRUSH_ERR_INVALID_ARG;
  if (a->T > 1024 || (long long)c->B * c->Hkv > 65535 || c->capacity > (1 << 30)) return KVCRUSH_ERR_UNSUPPORTED;
  if (a->blocks && (long long)a->n_list * a->unit >= (1 << 30)) return KVCRUSH_ERR_UNSUPPORTED;
  plan.G = a->Hq / c->Hkv;
  plan.rows = (long long)c->B * a->Hq * a->T;
  const long long r = a->blocks ? plan.G : (long long)plan.G * a->T;
  plan.NC = r > 32 ? 2 : 1;
  const long long tiles = (r + 32 * plan.NC - 1) / (32 * plan.NC);
  if (tiles > 1 && a->blocks) plan.NC = 2;
  const long long y = a->blocks ? a->T : tiles;
  if (y > 65535 || (a->blocks && tiles > 1)) return KVCRUSH_ERR_UNSUPPORTED;
  plan.row_tiles = (int)y;
  const long long keys = a->blocks ? std::min<long long>((long long)a->n_list * a->unit, c->capacity) : c->S;
  const long long base = (long long)c->B * c->Hkv * y;
  long long split = (512 + base - 1) / base;
  split = std::min(split, (keys + 255) / 256);
  plan.n_split = (int)std::max(1ll, std::min<long long>(split, kMaxSplit));
  return KVCRUSH_OK;
}

size_t ml_bytes(const Plan& p) { return kvc::align_up((size_t)p.rows * p.n_split * sizeof(float2), 256); }
size_t plan_bytes(const Plan& p, int D) {
  return p.n_split == 1 ? 0 : ml_bytes(p) + (size_t)p.rows * p.n_split * D * sizeof(float);
}

template <class F, int NC>
kvcrush_status launch_attend(const AttendParams& p, int row_tiles, hipStream_t stream) {
  constexpr int kLoop = F::kWaves * (F::kStage + kAhead * 4);
  constexpr int kEnd = F::kWaves * NC * 256 + F::kWaves / 2 * F::kDTiles * 16 * 256;
  constexpr int kLds = kLoop > kEnd ? kLoop : kEnd;
  static_assert(kLds <= kvc::kLdsPerWorkgroup, "LDS of a workgroup");
  kvcrush_status st = kvc::allow_large_lds<attend_kernel<F, NC>>(0);
  if (st != KVCRUSH_OK) return st;
  return kvc::launch(attend_kernel<F, NC>, dim3(p.n_split, row_tiles, p.c.B * p.c.Hkv), dim3(F::kWaves * KVC_WAVE), kLds, stream, p);
}

}  // namespace

extern "C" size_t kvcrush_attend_workspace(const kvcrush_cache* cache, const kvcrush_attend_args* args) {
  Plan plan;
  return make_plan(cache, args, plan) == KVCRUSH_OK ? plan_bytes(plan, cache->D) : 0;
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
  const size_t need = plan_bytes(plan, D);
  if (need > 0 && (!workspace || !kvc::aligned16(workspace) || workspace_bytes < need)) return KVCRUSH_ERR_WORKSPACE;
  p.c = view(cache);
  p.q = (const char*)q;
  p.out = (char*)out;
  p.lse = lse;
  p.part_ml = (float2*)workspace;
  p.part_o = need > 0 ? (float*)((char*)workspace + ml_bytes(plan)) : nullptr;
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
  p.q_dtype = args->dtype;
  p.scale_log2 = (float)(1.4426950408889634 *
                         (args->softmax_scale != 0.0f ? (double)args->softmax_scale : 1.0 / sqrt((double)D)));
  hipStream_t stream = (hipStream_t)hip_stream;
  st = with_format(cache->format, [&](auto fmt) -> kvcrush_status {
    constexpr int FMT = decltype(fmt)::value;
    if (D == 128)
      return plan.NC == 2 ? launch_attend<Fmt<FMT, 128>, 2>(p, plan.row_tiles, stream)
                          : launch_attend<Fmt<FMT, 128>, 1>(p, plan.row_tiles, stream);
    return plan.NC == 2 ? launch_attend<Fmt<FMT, 64>, 2>(p, plan.row_tiles, stream)
                        : launch_attend<Fmt<FMT, 64>, 1>(p, plan.row_tiles, stream);
  });
  if (st != KVCRUSH_OK || plan.n_split == 1) return st;
  const int per = 256 / (D / 4);
  const dim3 grid((unsigned)((plan.rows + per - 1) / per));
  return D == 128 ? kvc::launch(attend_merge_kernel<128>, grid, dim3(256), 0, stream, p)
                  : kvc::launch(attend_merge_kernel<64>, grid, dim3(256), 0, stream, p);
}
