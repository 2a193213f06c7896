// The KV cache as the kernels that use it see it: addresses of rows, element formats (not part of the ABI).
#pragma once
#include "common.h"

namespace kvc {
namespace cache {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMostTokens = 1 << 29;  // of a sequence: grids stay below 2^32 threads
constexpr float kTiny = 0x1p-100f;  // rows (ranges) below this are stored as zero: 448 / a stays finite above it

__host__ __device__ constexpr int format_bits(int format) {
  return format == KVCRUSH_F32 ? 32 : format <= KVCRUSH_F16 ? 16 : format == KVCRUSH_I4 ? 4 : 8;
}
__host__ __device__ constexpr bool quantised(int format) { return format >= KVCRUSH_E4M3; }

// Where the cache's rows are.  A row's number counts rows of D values from the start of k (and v), and
// parameters (pairs with I4) from the start of k_param.
struct View {
  char* k;
  char* v;
  float* k_param;
  float* v_param;
  const int32_t* lengths;
  const int32_t* table;  // null: dense
  int B, Hkv, S, capacity, block_size, block_shift, n_blocks, table_width;  // block_shift: log2 of a power of two, else -1

  __device__ int length(int b) const { return lengths ? min(max(lengths[b], 0), S) : S; }
  // Token `pos` of sequence b as the pool or the sequence counts tokens (a block outside the pool is pulled into it).
  __device__ int token(int b, int pos) const { return table ? paged_token(b, pos) : pos; }
  __device__ int paged_token(int b, int pos) const {
    const int of = block_shift >= 0 ? pos >> block_shift : pos / block_size;
    const int block = min(max(table[(size_t)b * table_width + of], 0), n_blocks - 1);
    return block * block_size + (pos - of * block_size);
  }
  // Row of KV head h = base(b, h) + token * step().
  __device__ size_t base(int b, int h) const { return table ? (size_t)h : ((size_t)b * Hkv + h) * capacity; }
  __device__ size_t step() const { return table ? (size_t)Hkv : 1; }
};

// Real ones of the T new tokens of sequence b.
__device__ __forceinline__ int new_tokens(const int32_t* n_new, int b, int T, int length) {
  const int most = min(T, length);
  return n_new ? min(max(n_new[b], 0), most) : most;
}

inline bool is_dtype(int t) { return t == KVCRUSH_F32 || t == KVCRUSH_BF16 || t == KVCRUSH_F16; }

// The caller's description, checked.
inline kvcrush_status check(const kvcrush_cache* c) {
  if (!c || c->B < 1 || c->Hkv < 1 || c->S < 0 || c->D < 1 || c->capacity < 1 || c->S > c->capacity) return KVCRUSH_ERR_INVALID_ARG;
  if (c->format < KVCRUSH_F32 || c->format > KVCRUSH_I4) return KVCRUSH_ERR_INVALID_ARG;
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return KVCRUSH_ERR_INVALID_ARG;
  if (quantised(c->format) && (!c->k_param || !c->v_param || !aligned16(c->k_param) || !aligned16(c->v_param)))
    return KVCRUSH_ERR_INVALID_ARG;
  if (c->block_table) {
    if (c->block_size < 1 || c->n_blocks < 1 || c->capacity % c->block_size != 0) return KVCRUSH_ERR_INVALID_ARG;
    if ((long long)c->n_blocks * c->block_size > 0x7FFFFFFFll) return KVCRUSH_ERR_UNSUPPORTED;
  }
  if ((c->D != 64 && c->D != 128) || c->capacity > kMostTokens) return KVCRUSH_ERR_UNSUPPORTED;
  return KVCRUSH_OK;
}

inline View view(const kvcrush_cache* c) {
  View w;
  w.k = (char*)c->k;
  w.v = (char*)c->v;
  w.k_param = c->k_param;
  w.v_param = c->v_param;
  w.lengths = c->lengths;
  w.table = c->block_table;
  w.B = c->B;
  w.Hkv = c->Hkv;
  w.S = c->S;
  w.capacity = c->capacity;
  w.block_size = c->block_table ? c->block_size : 1;
  w.block_shift = (w.block_size & (w.block_size - 1)) == 0 ? __builtin_ctz(w.block_size) : -1;
  w.n_blocks = c->block_table ? c->n_blocks : 1;
  w.table_width = c->block_table ? c->capacity / c->block_size : 0;
  return w;
}

// Strides {sequence, head, token} in elements: null or all zero is the packed layout of [B, H, T, D].  `least`: 0 for
// what is only read (one row may stand for several), D for an output.
inline bool strides_ok(const int64_t* s, int H, int T, int D, int bytes, int64_t least, int64_t (&out)[3]) {
  if (!s || (s[0] == 0 && s[1] == 0 && s[2] == 0)) {
    out[0] = (int64_t)H * T * D, out[1] = (int64_t)T * D, out[2] = D;
    return true;
  }
  for (int i = 0; i < 3; ++i) {
    if (s[i] < least || s[i] > ((int64_t)1 << 40) || (s[i] * bytes) % 16 != 0) return false;
    out[i] = s[i];
  }
  return true;
}

// ------------------------------------------------------------------ elements
// (a function: __builtin_bit_cast of a vector's element takes the vector's first one, whichever is named)
__device__ __forceinline__ f16x2 as_f16x2(uint32_t w) { return __builtin_bit_cast(f16x2, w); }

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const char* at) {
  return ONCE ? __builtin_nontemporal_load((const u32x4*)at) : *(const u32x4*)at;
}
template <bool ONCE>
__device__ __forceinline__ void store16(char* at, const u32x4& v) {
  if (ONCE)
    __builtin_nontemporal_store(v, (u32x4*)at);
  else
    *(u32x4*)at = v;
}

template <int DTYPE, bool ONCE = false>
__device__ __forceinline__ void load8(const char* at, float (&x)[8]) {  // eight values, 16 or 32 bytes
  if constexpr (DTYPE == KVCRUSH_F32) {
    const u32x4 a = load16<ONCE>(at), b = load16<ONCE>(at + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(a[i]), x[4 + i] = __uint_as_float(b[i]);
  } else {
    const u32x4 a = load16<ONCE>(at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DTYPE == KVCRUSH_BF16) {
        x[2 * i] = __uint_as_float(a[i] << 16);
        x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
      } else {
        const f16x2 h = as_f16x2(a[i]);
        x[2 * i] = (float)h[0];
        x[2 * i + 1] = (float)h[1];
      }
    }
  }
}

// Two values rounded to a 16-bit type (nearest, ties to even).
template <int DTYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DTYPE == KVCRUSH_BF16) {
    const f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
  } else {
    const f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
  }
}

template <int DTYPE, bool ONCE = false>
__device__ __forceinline__ void store8(char* at, const float (&x)[8]) {
  if constexpr (DTYPE == KVCRUSH_F32) {
    store16<ONCE>(at, u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])});
    store16<ONCE>(at + 16, u32x4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])});
  } else {
    store16<ONCE>(at, u32x4{pack2<DTYPE>(x[0], x[1]), pack2<DTYPE>(x[2], x[3]), pack2<DTYPE>(x[4], x[5]), pack2<DTYPE>(x[6], x[7])});
  }
}

// Four 8-bit codes as halves, exactly; SMALL: times kCodeFactor.  Integers: code + 128 behind the exponent of 1024, less 1152.
constexpr float kCodeFactor = 0x1p-14f;
template <int FORMAT, bool SMALL = false>
__device__ __forceinline__ u32x2 codes4_to_f16(uint32_t w) {
  constexpr float kBy = SMALL ? kCodeFactor : 1.0f;
  if constexpr (FORMAT == KVCRUSH_E4M3) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, kBy, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, kBy, true))};
  } else {
    w ^= 0x80808080u;
    const f16x2 by = {(_Float16)kBy, (_Float16)kBy}, off = {(_Float16)(-1152.0f * kBy), (_Float16)(-1152.0f * kBy)};
    const f16x2 lo = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)), by, off);
    const f16x2 hi = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)), by, off);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}
// Two floats' upper halves: as bfloat16, cut off below their eighth bit (exact where there is nothing below).
__device__ __forceinline__ uint32_t upper2(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
// Four 8-bit codes as bfloat16, exactly.
template <int FORMAT>
__device__ __forceinline__ u32x2 codes4_to_bf16(uint32_t w) {
  if constexpr (FORMAT == KVCRUSH_E4M3) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
  } else {
    auto code = [&](int i) { return (float)(int)(int8_t)(w >> (8 * i)); };
    return u32x2{upper2(code(0), code(1)), upper2(code(2), code(3))};
  }
}
// Eight 4-bit codes as bfloat16, exactly, in the order 0 2 4 6 1 3 5 7.  (As an 8-bit float of 3 mantissa bits, a byte
// below 16 stands for itself times 2^-9.)
__device__ __forceinline__ u32x4 codes8_to_bf16(uint32_t w) {
  const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, true))};
}
// Eight 4-bit codes times kCodeFactor as halves, exactly, in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ u32x4 codes8_to_small_f16(uint32_t w) {
  const f16x2 by = {(_Float16)kCodeFactor, (_Float16)kCodeFactor}, off = {(_Float16)(-1024.0f * kCodeFactor), (_Float16)(-1024.0f * kCodeFactor)};
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, ((w >> (4 * i)) & 0x000F000Fu) | 0x64006400u), by, off));
  return r;
}

// Values d .. d + 7 of a cached row (d a multiple of 8) as fp32, its parameters applied.
template <int FORMAT>
__device__ __forceinline__ void row_values(const char* rows, const float* params, size_t row, int D, int d, float (&x)[8]) {
  if constexpr (!quantised(FORMAT)) {
    load8<FORMAT>(rows + (row * D + d) * (format_bits(FORMAT) / 8), x);
  } else if constexpr (FORMAT == KVCRUSH_I4) {
    const uint32_t w = *(const uint32_t*)(rows + (row * D + d) / 2);
    const f32x2 p = *(const f32x2*)(params + row * 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(p[0], (float)((w >> (4 * i)) & 15u), p[1]);
  } else {
    const u32x2 w = *(const u32x2*)(rows + row * D + d);
    const float s = params[row];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2 h = codes4_to_f16<FORMAT>(w[i]);
      const f16x2 a = as_f16x2(h[0]), b = as_f16x2(h[1]);
      x[4 * i] = (float)a[0] * s;
      x[4 * i + 1] = (float)a[1] * s;
      x[4 * i + 2] = (float)b[0] * s;
      x[4 * i + 3] = (float)b[1] * s;
    }
  }
}

// A call with a run-time type as one with a constant.
template <class F>
kvcrush_status with_dtype(int dtype, F f) {
  switch (dtype) {
    case KVCRUSH_F32: return f(std::integral_constant<int, KVCRUSH_F32>{});
    case KVCRUSH_BF16: return f(std::integral_constant<int, KVCRUSH_BF16>{});
    default: return f(std::integral_constant<int, KVCRUSH_F16>{});
  }
}
template <class F>
kvcrush_status with_format(int format, F f) {
  switch (format) {
    case KVCRUSH_E4M3: return f(std::integral_constant<int, KVCRUSH_E4M3>{});
    case KVCRUSH_I8: return f(std::integral_constant<int, KVCRUSH_I8>{});
    case KVCRUSH_I4: return f(std::integral_constant<int, KVCRUSH_I4>{});
    default: return with_dtype(format, f);
  }
}

}  // namespace cache
}  // namespace kvc
