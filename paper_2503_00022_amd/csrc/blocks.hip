// Which blocks of a cache a query attends to: 8-bit bounds of each block's keys, kept as the cache grows, and the
// choice of the best blocks by them.
//
// A block's score for a query is sum_d max(q_d lo_d, q_d hi_d), an upper bound of its keys' products (of a box around them,
// as J. Tang et al. choose pages by in "Query-Aware Sparsity for Efficient Long-Context LLM Inference", 2024), with q, lo and
// hi in 8 bits: an integer below 2^24, so that it is the same in whatever order it is summed, on the matrix cores as
// 2 D products of [min(q, 0), max(q, 0)] with [lo, hi].  Choosing reads 2 D + 4 bytes per block and KV head where
// attending to the block reads 2 unit rows.  All three kernels are latency at one token: 3.9, 5.3 and 7.0 us for 2048 blocks
// of 8 KV heads.  (Scores and choice in one workgroup a query: 34 us, a compute unit alone reads the bounds too slowly.)
#include <algorithm>

#include "cache.h"

namespace {

using namespace kvc::cache;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ------------------------------------------------------------------------------------------------ bounds
struct BoundsParams {
  View c;
  const int32_t* n_new;
  int8_t* bounds;
  float* scales;
  int unit, T, n_blocks;  // n_blocks: of the capacity
};

constexpr int kBoundWaves = 4;
constexpr int kMostBounds = 1 << 25;  // blocks of a sequence: a grid's axis stays below 2^32 threads

// A wave takes one block: D / 8 lanes a row, 64 / (D / 8) rows at a time.
template <int FORMAT, int D>
__global__ __launch_bounds__(kBoundWaves * KVC_WAVE) void block_bounds_kernel(BoundsParams p) {
  constexpr int kLanes = D / 8, kRows = KVC_WAVE / kLanes;
  const int lane = kvc::lane_id(), wave = threadIdx.x / KVC_WAVE, col = lane % kLanes, sub = lane / kLanes;
  const int b = blockIdx.y / p.c.Hkv, h = blockIdx.y % p.c.Hkv;
  const int L = p.c.length(b), n = p.T == 0 ? L : new_tokens(p.n_new, b, p.T, L);
  if (n == 0) return;
  const int block = (L - n) / p.unit + blockIdx.x * kBoundWaves + wave;
  if (block > (L - 1) / p.unit) return;
  const int first = block * p.unit, end = min(first + p.unit, L);
  const size_t base = p.c.base(b, h), step = p.c.step();
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) lo[i] = __builtin_inff(), hi[i] = -__builtin_inff();
#pragma unroll 4
  for (int pos = first + sub; pos < end; pos += kRows) {
    float x[8];
    row_values<FORMAT>(p.c.k, p.c.k_param, base + (size_t)p.c.token(b, pos) * step, D, col * 8, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = fminf(lo[i], x[i]), hi[i] = fmaxf(hi[i], x[i]);
  }
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int off = kLanes; off < KVC_WAVE; off *= 2) {
      lo[i] = fminf(lo[i], __shfl_xor(lo[i], off));
      hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], off));
    }
    a = fmaxf(a, fmaxf(fabsf(lo[i]), fabsf(hi[i])));
  }
  a = kvc::wave_max(a);
  const bool zero = a < kTiny;
  const float inv = zero ? 0.0f : 127.0f / a;
  const size_t at = (size_t)blockIdx.y * p.n_blocks + block;
  if (sub < 2) {
    u32x2 w = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = (sub ? hi[i] : lo[i]) * inv;
      w[i / 4] |= ((uint32_t)(int)__builtin_rintf(x) & 255u) << (8 * (i % 4));
    }
    *(u32x2*)(p.bounds + (at * 2 + sub) * D + col * 8) = w;
  }
  if (lane == 0) p.scales[at] = zero ? 0.0f : a / 127.0f;
}

// ------------------------------------------------------------------------------------------------ scores
struct SelectParams {
  View c;
  const char* q;
  const int8_t* bounds;
  const float* scales;
  float* scores;  // workspace [B * Hkv * T][n_stride]
  int32_t* blocks;
  const int32_t* n_new;
  int64_t q_stride[3];
  int Hq, G, T, unit, n_blocks, n_stride, n_select, n_sink, n_recent;
};

constexpr int kScoreWaves = 4;
constexpr int kScoreBlocks = 32;  // blocks of a wave at a time

// Rows of the matrix product: up to 32 heads of the group; columns: 32 blocks, so that a lane has one block's scores
// for half the heads.
template <int DTYPE, int D>
__global__ __launch_bounds__(kScoreWaves * KVC_WAVE) void block_scores_kernel(SelectParams p) {
  constexpr int kPairs = D / 32;  // 16-byte chunks of lo (and of hi) that a lane half has
  __shared__ float head_scale[kScoreWaves][32];
  const int lane = kvc::lane_id(), wave = threadIdx.x / KVC_WAVE, half = lane >> 5, col = lane & 31;
  const int bh = blockIdx.z, b = bh / p.c.Hkv, h = bh % p.c.Hkv, t = blockIdx.y;
  const int L = p.c.length(b), n = new_tokens(p.n_new, b, p.T, L);
  if (t >= n) return;
  const int nb = (L + p.unit - 1) / p.unit;
  const int block0 = (blockIdx.x * kScoreWaves + wave) * kScoreBlocks;
  if (block0 >= nb) return;  // (no barrier below: the waves are on their own)
  const int block = min(block0 + col, nb - 1);
  const size_t at = (size_t)bh * p.n_blocks + block;
  const char* rows = (const char*)p.bounds + at * 2 * D;
  i32x4 bound[2 * kPairs];
#pragma unroll
  for (int s = 0; s < kPairs; ++s) {
    bound[s] = *(const i32x4*)(rows + (2 * s + half) * 16);
    bound[kPairs + s] = *(const i32x4*)(rows + D + (2 * s + half) * 16);
  }
  const float block_scale = p.scales[at];
  float best = -__builtin_inff();
  for (int g0 = 0; g0 < p.G; g0 += 32) {
    const int g = min(g0 + col, p.G - 1);
    const char* q = p.q + ((size_t)b * p.q_stride[0] + (size_t)(h * p.G + g) * p.q_stride[1] + (size_t)t * p.q_stride[2]) * (format_bits(DTYPE) / 8);
    float x[kPairs][16];
    float a = 0.0f;
#pragma unroll
    for (int s = 0; s < kPairs; ++s) {
      float y[8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        load8<DTYPE>(q + ((2 * s + half) * 16 + k * 8) * (format_bits(DTYPE) / 8), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[s][k * 8 + i] = y[i], a = fmaxf(a, fabsf(y[i]));
      }
    }
    a = fmaxf(a, __shfl_xor(a, 32));
    const bool zero = a < kTiny;
    const float inv = zero ? 0.0f : 127.0f / a;
    i32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0;
#pragma unroll
    for (int s = 0; s < kPairs; ++s) {
      i32x4 neg = {0, 0, 0, 0}, pos = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = (int)__builtin_rintf(x[s][i] * inv);
        neg[i / 4] |= (int)(((uint32_t)min(c, 0) & 255u) << (8 * (i % 4)));
        pos[i / 4] |= (int)(((uint32_t)max(c, 0) & 255u) << (8 * (i % 4)));
      }
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(neg, bound[s], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(pos, bound[kPairs + s], acc, 0, 0, 0);
    }
    kvc::wave_fence();
    if (half == 0) head_scale[wave][col] = zero ? 0.0f : a / 127.0f;
    kvc::wave_fence();
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int head = 8 * (r >> 2) + 4 * half + (r & 3);
      const float v = ((float)acc[r] * block_scale) * head_scale[wave][head];
      best = g0 + head < p.G ? fmaxf(best, v) : best;
    }
  }
  best = fmaxf(best, __shfl_xor(best, 32));
  if (half == 0 && block0 + col < nb) p.scores[((size_t)bh * p.T + t) * p.n_stride + block0 + col] = best;
}

// ------------------------------------------------------------------------------------------------ choice
// Order-preserving integer of a score.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kMaxBlocks = 32768;

// One workgroup per (sequence, KV head, query).  The n-th largest key is found eight bits at a time, from the first
// bit in which the keys differ; equal keys go to the lower block.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void block_choose_kernel(SelectParams p) {
  constexpr int kWaves = THREADS / KVC_WAVE;
  extern __shared__ uint32_t keys[];  // [nb], then two counts per 64 keys
  __shared__ uint32_t bins[256], found[4], red[2][kWaves];
  const int tid = threadIdx.x, lane = kvc::lane_id(), wave = tid / KVC_WAVE;
  const int row = blockIdx.x, t = row % p.T, bh = row / p.T, b = bh / p.c.Hkv;
  int32_t* out = p.blocks + (size_t)row * p.n_select;
  const int L = p.c.length(b), n = new_tokens(p.n_new, b, p.T, L);
  const int nb = t < n ? (L + p.unit - 1) / p.unit : 0;
  const int want = min(p.n_select, nb);
  for (int i = want + tid; i < p.n_select; i += THREADS) out[i] = -1;
  if (nb == want) {  // all of them (uniform)
    for (int i = tid; i < nb; i += THREADS) out[i] = i;
    return;
  }
  uint32_t* counts = keys + ((nb + 63) & ~63);
  const float* scores = p.scores + (size_t)row * p.n_stride;
  uint32_t lo = ~0u, hi = 0;
  constexpr int kAhead = 4;  // loads of a lane under way together
  for (int i0 = tid; i0 < nb; i0 += kAhead * THREADS) {
    float x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = scores[min(i0 + u * THREADS, nb - 1)];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u * THREADS;
      if (i >= nb) break;
      const bool forced = i < p.n_sink || i >= nb - p.n_recent;
      const uint32_t k = forced ? ~0u : min(order_key(x[u]), ~0u - 1);
      keys[i] = k;
      if (!forced) lo = min(lo, k), hi = max(hi, k);
    }
  }
  lo = kvc::wave_min(lo);
  hi = ~kvc::wave_min(~hi);
  if (lane == 0) red[0][wave] = lo, red[1][wave] = hi;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) lo = min(lo, red[0][w]), hi = max(hi, red[1][w]);
  int need = want - (p.n_sink + p.n_recent);  // of the others (nb > n_select >= n_sink + n_recent: no block is in both ends)
  // the need-th largest of them: `prefix` is its bits above `shift`
  uint32_t prefix = lo;
  int shift = lo == hi ? 0 : 32 - __builtin_clz(lo ^ hi);
  if (need == 0) {
    prefix = ~0u;  // (none of the others reaches it)
    shift = 0;
  }
  while (shift > 0) {
    const int next = max(shift - 8, 0), width = shift - next;
    for (int i = tid; i < 256; i += THREADS) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < nb; i += THREADS) {
      const uint32_t k = keys[i];
      const bool same = shift == 32 || (k >> shift) == (prefix >> shift);
      if (same && k != ~0u) atomicAdd(&bins[(k >> next) & ((1u << width) - 1)], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // from the top: four bins a lane, lane 0 the highest
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = bins[255 - 4 * lane - i], sum += c[i];
      uint32_t incl = sum;
      for (int off = 1; off < KVC_WAVE; off *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)incl, off);
        if (lane >= off) incl += o;
      }
      uint32_t above = incl - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < (uint32_t)need && above + c[i] >= (uint32_t)need) {
          found[0] = 255 - 4 * lane - i;
          found[1] = above;
          found[2] = c[i];
        }
        above += c[i];
      }
    }
    __syncthreads();
    const uint32_t digit = found[0], above = found[1], inside = found[2];
    prefix = (shift == 32 ? 0u : prefix >> shift << shift) | digit << next;
    need -= (int)above;
    shift = next;
    __syncthreads();
    if ((uint32_t)need == inside) break;  // all that share the prefix are taken
  }
  // taken: keys above the prefix's range, and the first `need` inside it
  const int chunks = (nb + 63) / 64;
  for (int c = wave; c < chunks; c += kWaves) {
    const int i = c * 64 + lane;
    const uint32_t k = i < nb ? keys[i] : 0;
    const bool inside = i < nb && (k >> shift) == (prefix >> shift) && k != ~0u, above = i < nb && (k >> shift) > (prefix >> shift);
    const bool forced = i < nb && k == ~0u;
    const uint64_t in = __ballot(inside), up = __ballot(above || forced);
    if (lane == 0) counts[2 * c] = __popcll(up), counts[2 * c + 1] = __popcll(in);
  }
  __syncthreads();
  if (wave == 0) {  // counts become the taken blocks, and the blocks inside the range, before each chunk
    uint32_t taken = 0, inside = 0;
    for (int c0 = 0; c0 < chunks; c0 += KVC_WAVE) {
      const int c = c0 + lane;
      const uint32_t up = c < chunks ? counts[2 * c] : 0, in = c < chunks ? counts[2 * c + 1] : 0;
      uint32_t si = in;
      for (int off = 1; off < KVC_WAVE; off *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)si, off);
        if (lane >= off) si += o;
      }
      const uint32_t before = inside + si - in;
      const uint32_t here = up + (before < (uint32_t)need ? min(in, (uint32_t)need - before) : 0u);
      uint32_t st = here;
      for (int off = 1; off < KVC_WAVE; off *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)st, off);
        if (lane >= off) st += o;
      }
      if (c < chunks) counts[2 * c] = taken + st - here, counts[2 * c + 1] = before;
      inside += (uint32_t)__shfl((int)si, KVC_WAVE - 1);
      taken += (uint32_t)__shfl((int)st, KVC_WAVE - 1);
    }
  }
  __syncthreads();
  for (int c = wave; c < chunks; c += kWaves) {
    const int i = c * 64 + lane;
    const uint32_t k = i < nb ? keys[i] : 0;
    const bool forced = i < nb && k == ~0u;
    const bool inside = i < nb && (k >> shift) == (prefix >> shift) && !forced, above = i < nb && (k >> shift) > (prefix >> shift);
    const uint64_t lt = kvc::lanemask_lt();
    const uint32_t before = counts[2 * c + 1] + (uint32_t)__popcll(__ballot(inside) & lt);
    const bool take = forced || above || (inside && before < (uint32_t)need);
    const uint64_t all = __ballot(take);
    const uint32_t at = counts[2 * c] + (uint32_t)__popcll(all & lt);
    if (take && at < (uint32_t)want) out[at] = i;
  }
}

kvcrush_status select_ok(const kvcrush_cache* c, const kvcrush_attend_args* a, int unit, int n_select) {
  kvcrush_status st = check(c);
  if (st != KVCRUSH_OK) return st;
  if (!a || a->Hq < 1 || a->Hq % c->Hkv != 0 || a->T < 1 || !is_dtype(a->dtype) || unit < 1 || n_select < 1)
    return KVCRUSH_ERR_INVALID_ARG;
  if (a->T > 1024 || a->Hq / c->Hkv > 1024 || (long long)c->B * c->Hkv > 65535 || (long long)c->B * c->Hkv * a->T > (1 << 21))
    return KVCRUSH_ERR_UNSUPPORTED;
  if (((long long)c->S + unit - 1) / unit > kMaxBlocks || n_select > kMaxBlocks) return KVCRUSH_ERR_UNSUPPORTED;
  return KVCRUSH_OK;
}

int blocks_of(int tokens, int unit) { return (int)(((long long)tokens + unit - 1) / unit); }

size_t scores_bytes(const kvcrush_cache* c, const kvcrush_attend_args* a, int unit) {
  return (size_t)c->B * c->Hkv * a->T * kvc::align_up((size_t)blocks_of(c->S, unit), 64) * sizeof(float);
}

}  // namespace

extern "C" kvcrush_status kvcrush_block_bounds(const kvcrush_cache* cache, int32_t unit, int32_t T, const int32_t* n_new,
                                               int8_t* bounds, float* scales, void* hip_stream) {
  kvcrush_status st = check(cache);
  if (st != KVCRUSH_OK) return st;
  if (unit < 1 || T < 0) return KVCRUSH_ERR_INVALID_ARG;
  if (unit > 1024 || (long long)cache->B * cache->Hkv > 65535 || blocks_of(cache->capacity, unit) > kMostBounds)
    return KVCRUSH_ERR_UNSUPPORTED;
  if (!bounds || !scales || !kvc::aligned16(bounds) || !kvc::aligned16(scales)) return KVCRUSH_ERR_INVALID_ARG;
  if (cache->S == 0) return KVCRUSH_OK;
  BoundsParams p;
  p.c = view(cache);
  p.n_new = n_new;
  p.bounds = bounds;
  p.scales = scales;
  p.unit = unit;
  p.T = T;
  p.n_blocks = blocks_of(cache->capacity, unit);
  const int all = blocks_of(cache->S, unit);
  const int most = T == 0 ? all : (int)std::min<long long>(all, (long long)(T - 1) / unit + 2);
  const dim3 grid((most + kBoundWaves - 1) / kBoundWaves, cache->B * cache->Hkv);
  return with_format(cache->format, [&](auto fmt) {
    constexpr int FMT = decltype(fmt)::value;
    hipStream_t stream = (hipStream_t)hip_stream;
    return cache->D == 128 ? kvc::launch(block_bounds_kernel<FMT, 128>, grid, dim3(kBoundWaves * KVC_WAVE), 0, stream, p)
                           : kvc::launch(block_bounds_kernel<FMT, 64>, grid, dim3(kBoundWaves * KVC_WAVE), 0, stream, p);
  });
}

extern "C" size_t kvcrush_block_select_workspace(const kvcrush_cache* cache, const kvcrush_attend_args* args, int32_t unit,
                                                 int32_t n_select) {
  return select_ok(cache, args, unit, n_select) == KVCRUSH_OK ? scores_bytes(cache, args, unit) : 0;
}

extern "C" kvcrush_status kvcrush_block_select(const kvcrush_cache* cache, const kvcrush_attend_args* args, int32_t unit,
                                               int32_t n_select, int32_t n_sink, int32_t n_recent, const void* q,
                                               const int8_t* bounds, const float* scales, int32_t* blocks, void* workspace,
                                               size_t workspace_bytes, void* hip_stream) {
  kvcrush_status st = select_ok(cache, args, unit, n_select);
  if (st != KVCRUSH_OK) return st;
  if (n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > n_select) return KVCRUSH_ERR_INVALID_ARG;
  if (!q || !bounds || !scales || !blocks || !kvc::aligned16(q) || !kvc::aligned16(bounds) || !kvc::aligned16(scales) ||
      !kvc::aligned16(blocks))
    return KVCRUSH_ERR_INVALID_ARG;
  SelectParams p;
  if (!strides_ok(args->q_stride, args->Hq, args->T, cache->D, format_bits(args->dtype) / 8, 0, p.q_stride))
    return KVCRUSH_ERR_INVALID_ARG;
  const size_t need = scores_bytes(cache, args, unit);
  if (need > 0 && (!workspace || !kvc::aligned16(workspace) || workspace_bytes < need)) return KVCRUSH_ERR_WORKSPACE;
  p.c = view(cache);
  p.q = (const char*)q;
  p.bounds = bounds;
  p.scales = scales;
  p.scores = (float*)workspace;
  p.blocks = blocks;
  p.n_new = args->n_new;
  p.Hq = args->Hq;
  p.G = args->Hq / cache->Hkv;
  p.T = args->T;
  p.unit = unit;
  p.n_blocks = blocks_of(cache->capacity, unit);
  const int nb = blocks_of(cache->S, unit);
  p.n_stride = (int)kvc::align_up((size_t)nb, 64);
  p.n_select = n_select;
  p.n_sink = n_sink;
  p.n_recent = n_recent;
  hipStream_t stream = (hipStream_t)hip_stream;
  if (nb > n_select) {  // (otherwise all blocks are taken)
    const dim3 grid((nb + kScoreWaves * kScoreBlocks - 1) / (kScoreWaves * kScoreBlocks), args->T, cache->B * cache->Hkv);
    st = with_dtype(args->dtype, [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      return cache->D == 128 ? kvc::launch(block_scores_kernel<DT, 128>, grid, dim3(kScoreWaves * KVC_WAVE), 0, stream, p)
                             : kvc::launch(block_scores_kernel<DT, 64>, grid, dim3(kScoreWaves * KVC_WAVE), 0, stream, p);
    });
    if (st != KVCRUSH_OK) return st;
  }
  const size_t lds = ((size_t)p.n_stride + 2 * (p.n_stride / 64)) * sizeof(uint32_t);
  const dim3 grid((unsigned)((size_t)cache->B * cache->Hkv * args->T));
  if (nb <= 1024) return kvc::launch(block_choose_kernel<256>, grid, dim3(256), lds, stream, p);
  st = kvc::allow_large_lds<block_choose_kernel<1024>>(2048);
  return st != KVCRUSH_OK ? st : kvc::launch(block_choose_kernel<1024>, grid, dim3(1024), lds, stream, p);
}
