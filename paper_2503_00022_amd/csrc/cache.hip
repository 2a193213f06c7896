// Rows of a KV cache in 8 or 4 bits: quantised as they are written, read back as values.
//
// Both directions are bound by the bytes they move (a value of 2 or 4 bytes on one side, 1 or 1/2 on the
// other).  Eight neighbouring values of a row belong to one lane, so that a row is D / 8 = 8 or 16 lanes
// whose extremes are combined by DPP moves, a wave moves four or eight rows with one 16-byte load a lane,
// and kRows of those are in flight together (one where there are few rows: a single token's 128 rows take 2.9 us,
// a launch's latency).  The side in values is used once and passes the caches by: 8 x 8192 tokens of 8 heads into a
// paged e4m3 cache 90 -> 73 us (5.6 TB/s), four e4m3 caches of up to 7839 tokens back 40 -> 26 (6.1 TB/s, part of the codes
// from the last-level cache).
#include <algorithm>

#include "cache.h"

namespace {

using namespace kvc::cache;

constexpr int kThreads = 256;
constexpr int kRows = 4;  // rows of a lane in flight together

// `v` of the LANES (8 or 16) neighbouring lanes of a row, combined.
template <int LANES, class Op>
__device__ __forceinline__ float row_reduce(float v, Op op) {
  auto step = [&](int moved) { v = op(v, __int_as_float(moved)); };
  step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true));   // quad_perm [1, 0, 3, 2]
  step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true));   // quad_perm [2, 3, 0, 1]
  step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));  // row_half_mirror
  if constexpr (LANES == 16) step(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true));  // row_mirror
  return v;
}

// Quantises this lane's eight values of a row and stores codes and parameters (header: kvcrush_format).
template <int FORMAT, int D>
__device__ __forceinline__ void store_row(const float (&x)[8], char* rows, float* params, size_t row, int col) {
  constexpr int kLanes = D / 8;
  // the largest magnitude as an integer: unlike fmaxf, it does not lose a NaN
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = __float_as_uint(row_reduce<kLanes>(__uint_as_float(top), [](float a, float b) {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
  }));
  const float a = __uint_as_float(top);
  const float nan = __uint_as_float(0x7FC00000u);
  if constexpr (FORMAT == KVCRUSH_I4) {
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]);
    lo = row_reduce<kLanes>(lo, [](float p, float q) { return fminf(p, q); });
    hi = row_reduce<kLanes>(hi, [](float p, float q) { return fmaxf(p, q); });
    const float d = hi - lo;
    const bool bad = top >= 0x7F800000u || !(d < __builtin_inff()), flat = d < kTiny;
    const float inv = flat || bad ? 0.0f : 15.0f / d;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = bad ? 0.0f : (x[i] - lo) * inv;
      w |= (uint32_t)__builtin_rintf(y) << (4 * i);
    }
    *(uint32_t*)(rows + row * (D / 2) + col * 4) = w;
    if (col == 0) *(f32x2*)(params + row * 2) = f32x2{bad ? nan : flat ? 0.0f : d / 15.0f, bad ? nan : lo};
  } else {
    constexpr float kTop = FORMAT == KVCRUSH_E4M3 ? 448.0f : 127.0f;
    const bool bad = top >= 0x7F800000u, zero = a < kTiny;
    const float inv = zero || bad ? 0.0f : kTop / a;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = bad ? 0.0f : x[i] * inv;
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (FORMAT == KVCRUSH_E4M3) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], p, true);
      } else {
        w[i] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i] |= ((uint32_t)(int)__builtin_rintf(y[4 * i + j]) & 255u) << (8 * j);
      }
    }
    *(u32x2*)(rows + row * D + col * 8) = w;
    if (col == 0) params[row] = bad ? nan : zero ? 0.0f : a / kTop;
  }
}

struct WriteParams {
  View c;
  const char* src[2];    // k_new, v_new
  int64_t stride[2][3];  // elements: sequence, head, token
  const int32_t* n_new;
  int T;
};

// Grid: x = groups of new tokens, y = KV head, z = 2 * sequence + (0: K, 1: V).
template <int DTYPE, int FORMAT, int D, int ROWS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(WriteParams p) {
  constexpr int kLanes = D / 8, kGroup = kThreads / kLanes;  // rows of one pass of the workgroup
  const int b = blockIdx.z >> 1, which = blockIdx.z & 1, h = blockIdx.y;
  const int col = threadIdx.x % kLanes, r = threadIdx.x / kLanes;
  const int L = p.c.length(b), n = new_tokens(p.n_new, b, p.T, L);
  const int t0 = blockIdx.x * (kGroup * ROWS) + r;
  const char* src = p.src[which] + ((size_t)b * p.stride[which][0] + (size_t)h * p.stride[which][1] + col * 8) * (format_bits(DTYPE) / 8);
  char* rows = which ? p.c.v : p.c.k;
  float* params = which ? p.c.v_param : p.c.k_param;
  const size_t base = p.c.base(b, h), step = p.c.step();
  float x[ROWS][8];
  int token[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int t = t0 + u * kGroup;
    if (t < n) {
      load8<DTYPE, (ROWS > 1)>(src + (size_t)t * p.stride[which][2] * (format_bits(DTYPE) / 8), x[u]);
      token[u] = p.c.token(b, L - n + t);
    }
  }
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    if (t0 + u * kGroup < n) {  // (the same for all lanes of a row)
      const size_t row = base + (size_t)token[u] * step;
      if constexpr (quantised(FORMAT))
        store_row<FORMAT, D>(x[u], rows, params, row, col);
      else
        store8<FORMAT>(rows + (row * D + col * 8) * (format_bits(FORMAT) / 8), x[u]);
    }
  }
}

struct ReadParams {
  View c;
  char* dst[2];
  const int32_t* idx;
  int n;
};

template <int DTYPE, int FORMAT, int D, int ROWS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(ReadParams p) {
  constexpr int kLanes = D / 8, kGroup = kThreads / kLanes;
  const int b = blockIdx.z >> 1, which = blockIdx.z & 1, h = blockIdx.y;
  const int col = threadIdx.x % kLanes, r = threadIdx.x / kLanes;
  const int L = p.c.length(b);
  const int end = p.idx ? (L > 0 ? p.n : 0) : min(p.n, L);
  const int j0 = blockIdx.x * (kGroup * ROWS) + r;
  const char* rows = which ? p.c.v : p.c.k;
  const float* params = which ? p.c.v_param : p.c.k_param;
  const size_t base = p.c.base(b, h), step = p.c.step();
  float x[ROWS][8];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int j = j0 + u * kGroup;
    if (j < end) {
      const int pos = p.idx ? min(max(p.idx[(size_t)b * p.n + j], 0), L - 1) : j;
      row_values<FORMAT>(rows, params, base + (size_t)p.c.token(b, pos) * step, D, col * 8, x[u]);
    }
  }
  char* dst = p.dst[which] + ((((size_t)b * p.c.Hkv + h) * p.n) * D + col * 8) * (format_bits(DTYPE) / 8);
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    const int j = j0 + u * kGroup;
    if (j < end) store8<DTYPE, (ROWS > 1)>(dst + (size_t)j * D * (format_bits(DTYPE) / 8), x[u]);
  }
}

// K and V of B sequences along z, rows along x.
bool grid_for(const kvcrush_cache* c, int rows_per_wg, int n, dim3& grid) {
  if (c->B > 32767 || c->Hkv > 65535) return false;
  grid = dim3((unsigned)(((long long)n + rows_per_wg - 1) / rows_per_wg), (unsigned)c->Hkv, (unsigned)(2 * c->B));
  return true;
}

}  // namespace

extern "C" kvcrush_status kvcrush_cache_write(const kvcrush_cache* cache, int32_t T, int32_t dtype, const void* k_new,
                                              const void* v_new, const int64_t* k_stride, const int64_t* v_stride,
                                              const int32_t* n_new, void* hip_stream) {
  kvcrush_status st = check(cache);
  if (st != KVCRUSH_OK) return st;
  if (T < 0 || !is_dtype(dtype)) return KVCRUSH_ERR_INVALID_ARG;
  if (!quantised(cache->format) && dtype != cache->format) return KVCRUSH_ERR_INVALID_ARG;
  if (T == 0 || cache->S == 0) return KVCRUSH_OK;  // (no token is new)
  if (!k_new || !v_new || !kvc::aligned16(k_new) || !kvc::aligned16(v_new)) return KVCRUSH_ERR_INVALID_ARG;
  WriteParams p;
  p.c = view(cache);
  p.src[0] = (const char*)k_new;
  p.src[1] = (const char*)v_new;
  if (!strides_ok(k_stride, cache->Hkv, T, cache->D, format_bits(dtype) / 8, 0, p.stride[0]) ||
      !strides_ok(v_stride, cache->Hkv, T, cache->D, format_bits(dtype) / 8, 0, p.stride[1]))
    return KVCRUSH_ERR_INVALID_ARG;
  p.n_new = n_new;
  p.T = T;
  const int group = kThreads / (cache->D / 8);
  dim3 grid;
  const int most = std::min(T, cache->S);  // (no sequence has more new tokens)
  const bool few = most <= group;
  if (!grid_for(cache, group * (few ? 1 : kRows), most, grid)) return KVCRUSH_ERR_UNSUPPORTED;
  return with_dtype(dtype, [&](auto dt) {
    return with_format(cache->format, [&](auto fmt) -> kvcrush_status {
      constexpr int DT = decltype(dt)::value, FMT = decltype(fmt)::value;
      if constexpr (quantised(FMT) || DT == FMT) {
        hipStream_t stream = (hipStream_t)hip_stream;
        if (cache->D == 128)
          return few ? kvc::launch(cache_write_kernel<DT, FMT, 128, 1>, grid, dim3(kThreads), 0, stream, p)
                     : kvc::launch(cache_write_kernel<DT, FMT, 128, kRows>, grid, dim3(kThreads), 0, stream, p);
        return few ? kvc::launch(cache_write_kernel<DT, FMT, 64, 1>, grid, dim3(kThreads), 0, stream, p)
                   : kvc::launch(cache_write_kernel<DT, FMT, 64, kRows>, grid, dim3(kThreads), 0, stream, p);
      } else {
        return KVCRUSH_ERR_INVALID_ARG;
      }
    });
  });
}

extern "C" kvcrush_status kvcrush_cache_read(const kvcrush_cache* cache, int32_t n, const int32_t* idx, int32_t dtype,
                                             void* k_out, void* v_out, void* hip_stream) {
  kvcrush_status st = check(cache);
  if (st != KVCRUSH_OK) return st;
  if (n < 0 || (!idx && n > cache->capacity) || !is_dtype(dtype)) return KVCRUSH_ERR_INVALID_ARG;
  if (!quantised(cache->format) && dtype != cache->format) return KVCRUSH_ERR_INVALID_ARG;
  if (n == 0) return KVCRUSH_OK;
  if (n > kMostTokens) return KVCRUSH_ERR_UNSUPPORTED;
  if (!k_out || !v_out || !kvc::aligned16(k_out) || !kvc::aligned16(v_out)) return KVCRUSH_ERR_INVALID_ARG;
  ReadParams p;
  p.c = view(cache);
  p.dst[0] = (char*)k_out;
  p.dst[1] = (char*)v_out;
  p.idx = idx;
  p.n = n;
  const int group = kThreads / (cache->D / 8);
  dim3 grid;
  const bool few = n <= group;
  if (!grid_for(cache, group * (few ? 1 : kRows), n, grid)) return KVCRUSH_ERR_UNSUPPORTED;
  return with_dtype(dtype, [&](auto dt) {
    return with_format(cache->format, [&](auto fmt) -> kvcrush_status {
      constexpr int DT = decltype(dt)::value, FMT = decltype(fmt)::value;
      if constexpr (quantised(FMT) || DT == FMT) {
        hipStream_t stream = (hipStream_t)hip_stream;
        if (cache->D == 128)
          return few ? kvc::launch(cache_read_kernel<DT, FMT, 128, 1>, grid, dim3(kThreads), 0, stream, p)
                     : kvc::launch(cache_read_kernel<DT, FMT, 128, kRows>, grid, dim3(kThreads), 0, stream, p);
        return few ? kvc::launch(cache_read_kernel<DT, FMT, 64, 1>, grid, dim3(kThreads), 0, stream, p)
                   : kvc::launch(cache_read_kernel<DT, FMT, 64, kRows>, grid, dim3(kThreads), 0, stream, p);
      } else {
        return KVCRUSH_ERR_INVALID_ARG;
      }
    });
  });
}
