// Operators on prefix caches: conversion to and from 4 bits, eviction of
// tokens, and plain forms of the attention over either format and of the
// attention weight that cached tokens gather.
#include <math.h>

#include <algorithm>

#include "rosa_device.h"
#include "rosa_internal.h"

namespace rosa {

// ------------------------------------------------------------------ to 4 bits and back
// A block of 32 elements x: a = max |x|, e = the least integer with
// a <= 7 2^e (a normal a = 1.m 2^E: E - 2 where 1.m <= 1.75, else E - 1),
// code = x / 2^e rounded to the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} (ties to the
// even code).  7 2^e and not 6 2^e: magnitudes in (6, 7] round to 6 anyway,
// and of the borders between 6 and 8 (every one there is) 7 gives normal
// data the least error (relative 0.1119; 6: 0.1154, 8: 0.1150).
//
// A thread takes 8 elements (16 or 32 bytes in, 4 bytes of codes out, both
// contiguous over a wave), four threads a block.  One pass, memory bound: 32 bf16 caches of 512 to 1280
// tokens (644 MB each way) take 137 us, and 131 back: 4.7 and 4.9 TB/s where a copy reaches 5.0.
template <typename T>
__global__ void __launch_bounds__(256) kv_quantize_kernel(KvJobs jobs, int L, int nkv, int hd) {
  const KvJob &j = jobs.j[blockIdx.y];
  const T *src = reinterpret_cast<const T *>(blockIdx.z ? j.sv : j.sk);
  uint8_t *dst = reinterpret_cast<uint8_t *>(blockIdx.z ? j.dv : j.dk);
  const size_t n8 = (size_t)L * j.P * nkv * (hd / 8);     // a multiple of 4: a block's threads end together
  uint8_t *scales = dst + kv4_code_bytes(L, j.P, nkv, hd);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += (size_t)gridDim.x * 256) {
    uint32_t x[8];                                        // fp32 bits
    if constexpr (sizeof(T) == 2) {
      const uint4 w = reinterpret_cast<const uint4 *>(src)[i];
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) { x[2 * q] = ww[q] << 16; x[2 * q + 1] = ww[q] & 0xffff0000u; }
    } else {
      const uint4 w0 = reinterpret_cast<const uint4 *>(src)[2 * i], w1 = reinterpret_cast<const uint4 *>(src)[2 * i + 1];
      x[0] = w0.x; x[1] = w0.y; x[2] = w0.z; x[3] = w0.w; x[4] = w1.x; x[5] = w1.y; x[6] = w1.z; x[7] = w1.w;
    }
    uint32_t a = 0;                                       // magnitudes order as their bits, NaN above all
#pragma unroll
    for (int q = 0; q < 8; ++q) a = max(a, x[q] & 0x7fffffffu);
    a = max(a, (uint32_t)__shfl_xor((int)a, 1, 64));
    a = max(a, (uint32_t)__shfl_xor((int)a, 2, 64));
    const bool finite = a < 0x7f800000u;
    const int E = (int)(a >> 23) - 127;
    const int e = min(125, max(-125, (a & 0x7fffffu) <= 0x600000u ? E - 2 : E - 1));
    const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    uint32_t c = 0;
    if (finite) {
      // the conversion divides by the scale, rounds half to even and saturates
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x[4]), __uint_as_float(x[5]), scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(x[6]), __uint_as_float(x[7]), scale, 3);
    }
    reinterpret_cast<uint32_t *>(dst)[i] = c;
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = finite ? (uint8_t)(e + 127) : 255;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) kv_expand_kernel(KvJobs jobs, int L, int nkv, int hd) {
  const KvJob &j = jobs.j[blockIdx.y];
  const uint8_t *src = reinterpret_cast<const uint8_t *>(blockIdx.z ? j.sv : j.sk);
  T *dst = reinterpret_cast<T *>(blockIdx.z ? j.dv : j.dk);
  const size_t n8 = (size_t)L * j.P * nkv * (hd / 8);
  const uint8_t *scales = src + kv4_code_bytes(L, j.P, nkv, hd);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += (size_t)gridDim.x * 256) {
    const bf16x8 v = kv4_bf16x8(reinterpret_cast<const uint32_t *>(src)[i], kv4_scale(scales[i >> 2]));
    if constexpr (sizeof(T) == 2) {
      reinterpret_cast<uint4 *>(dst)[i] = __builtin_bit_cast(uint4, v);
    } else {
      float4 f0 = make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
      float4 f1 = make_float4((float)v[4], (float)v[5], (float)v[6], (float)v[7]);
      reinterpret_cast<float4 *>(dst)[2 * i] = f0;
      reinterpret_cast<float4 *>(dst)[2 * i + 1] = f1;
    }
  }
}

// Blocks of 256 threads along x for the largest of the jobs' unit counts.
static int grid_x(size_t most_units, int most_blocks) {
  return (int)std::min<size_t>((most_units + 255) / 256, (size_t)most_blocks);
}

static size_t most_units8(const KvJobs &jobs, int n, int L, int nkv, int hd) {
  int P = 0;
  for (int i = 0; i < n; ++i) P = std::max(P, jobs.j[i].P);
  return (size_t)L * P * nkv * (hd / 8);
}

hipError_t launch_kv_quantize(const KvJobs &jobs, int n, int L, int nkv, int hd, bool bf16_mode, hipStream_t s) {
  const size_t u = most_units8(jobs, n, L, nkv, hd);
  if (n <= 0 || u == 0) return hipSuccess;
  dim3 grid(grid_x(u, 4096), n, 2);
  if (bf16_mode) hipLaunchKernelGGL(kv_quantize_kernel<bf16>, grid, dim3(256), 0, s, jobs, L, nkv, hd);
  else hipLaunchKernelGGL(kv_quantize_kernel<float>, grid, dim3(256), 0, s, jobs, L, nkv, hd);
  return hipGetLastError();
}

hipError_t launch_kv_expand(const KvJobs &jobs, int n, int L, int nkv, int hd, bool bf16_mode, hipStream_t s) {
  const size_t u = most_units8(jobs, n, L, nkv, hd);
  if (n <= 0 || u == 0) return hipSuccess;
  dim3 grid(grid_x(u, 4096), n, 2);
  if (bf16_mode) hipLaunchKernelGGL(kv_expand_kernel<bf16>, grid, dim3(256), 0, s, jobs, L, nkv, hd);
  else hipLaunchKernelGGL(kv_expand_kernel<float>, grid, dim3(256), 0, s, jobs, L, nkv, hd);
  return hipGetLastError();
}

// ------------------------------------------------------------------ eviction
// A mass as an unsigned whole number of the same order: NaN 0, below -infinity; -0 as +0.
__device__ __forceinline__ uint32_t mass_key(float m) {
  uint32_t u = __float_as_uint(m);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One block per (layer, KV head) row of a job: the `want` = keep - first - last
// largest of its unprotected masses.  Four passes over the row find the key T of
// the want-th largest, eight bits at a time (histogram of the keys that share
// the bits found so far; the digit by a sum over the larger ones across the block); a last pass lists the
// protected tokens, the keys above T and the first ties at T, in order.  The row is read from memory once,
// but for what lies behind its first kSelectRow tokens.  Latency bounds it: 18 rows of 816 tokens take
// 9 us, 576 of 512 to 1280 tokens 14.
constexpr int kSelectRow = 12288;
__global__ void __launch_bounds__(1024) kv_select_kernel(KvEvictJobs jobs, int rows) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t sh[2];
  __shared__ uint32_t wsum[2][16];
  extern __shared__ float near[];            // the row's first kSelectRow masses
  const KvEvictJob &j = jobs.j[blockIdx.y];
  const int row = blockIdx.x, P = j.P, keep = j.keep;
  if (keep == 0) return;
  const float *mass = j.mass + (size_t)row * P;
  int32_t *kept = j.kept + (size_t)row * keep;
  float *kmass = j.kept_mass ? j.kept_mass + (size_t)row * keep : nullptr;
  const int lo = j.first, hi = P - j.last;
  const uint32_t want = (uint32_t)(keep - j.first - j.last);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nt = blockDim.x, nw = nt >> 6;
  for (int i = tid; i < min(P, kSelectRow); i += nt) near[i] = mass[i];
  __syncthreads();
  auto at_row = [&](int i) { return i < kSelectRow ? near[i] : mass[i]; };
  uint32_t T = 0, left = want;               // bits found; how many of the keys that share them are wanted
  if (want > 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t above = shift == 24 ? 0u : ~0u << (shift + 8);
      for (int i0 = lo + tid; i0 < hi; i0 += 4 * nt) {
        uint32_t k[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) k[x] = mass_key(at_row(min(i0 + x * nt, hi - 1)));
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (i0 + x * nt < hi && (k[x] & above) == T) atomicAdd(&hist[(k[x] >> shift) & 255], 1u);
      }
      __syncthreads();
      // thread d: the keys of digits d and above; exactly one d has `left` of them but not above it
      const uint32_t own = tid < 256 ? hist[tid] : 0;
      uint32_t sum = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_down(sum, o, 64);
        if (lane + o < 64) sum += v;
      }
      if (lane == 0) wsum[0][wave] = sum;
      __syncthreads();
      for (int w = wave + 1; w < 4; ++w) sum += wsum[0][w];
      if (tid < 256 && sum >= left && sum - own < left) {
        sh[0] = T | (uint32_t)tid << shift;
        sh[1] = left - (sum - own);
      }
      __syncthreads();
      T = sh[0];
      left = sh[1];
      __syncthreads();
    }
  // `left` of the keys equal to T are kept: those of the lowest indices.  A wave takes a run of the row: it
  // counts, and with the runs before it counted it knows where its own tokens go.
  const int run = ((P + nw - 1) / nw + 63) & ~63, r0 = wave * run, r1 = min(P, r0 + run);
  auto look = [&](int i, float &m, bool &sure, bool &tie) {
    m = at_row(min(i, P - 1));
    const uint32_t k = mass_key(m);
    const bool safe = i < lo || i >= hi, cand = !safe && want > 0;
    sure = i < r1 && (safe || (cand && k > T));
    tie = i < r1 && cand && k == T;
  };
  uint32_t ties = 0, out = 0;
  for (int i0 = r0; i0 < r1; i0 += 256) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      float m;
      bool sure, tie;
      look(i0 + 64 * x + lane, m, sure, tie);
      out += (uint32_t)__popcll(__ballot(sure));
      ties += (uint32_t)__popcll(__ballot(tie));
    }
  }
  if (lane == 0) { wsum[0][wave] = ties; wsum[1][wave] = out; }
  __syncthreads();
  ties = out = 0;
  for (int w = 0; w < wave; ++w) { ties += wsum[0][w]; out += wsum[1][w]; }
  out += min(ties, left);
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = r0; i0 < r1; i0 += 256) {
    float m[4];
    bool sure[4], tie[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) look(i0 + 64 * x + lane, m[x], sure[x], tie[x]);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const uint64_t tb = __ballot(tie[x]);
      const bool take = sure[x] || (tie[x] && ties + (uint32_t)__popcll(tb & below) < left);
      const uint64_t kb = __ballot(take);
      if (take) {
        const uint32_t at = out + (uint32_t)__popcll(kb & below);
        kept[at] = i0 + 64 * x + lane;
        if (kmass) kmass[at] = m[x];
      }
      ties += (uint32_t)__popcll(tb);
      out += (uint32_t)__popcll(kb);
    }
  }
}

// The kept tokens' rows (K and V): 16-byte pieces, `pieces` of them a row; at the copy's rate (half of 32 caches,
// 513 MB read and written: 93 us).  Rows of the
// caches are [L][tokens][nkv]; destination row r = (layer keep + i) nkv + head.
__global__ void __launch_bounds__(256) kv_gather_kernel(KvEvictJobs jobs, int L, int nkv, int pieces) {
  const KvEvictJob &j = jobs.j[blockIdx.y];
  const uint4 *src = reinterpret_cast<const uint4 *>(blockIdx.z ? j.sv : j.sk);
  uint4 *dst = reinterpret_cast<uint4 *>(blockIdx.z ? j.dv : j.dk);
  const size_t n = (size_t)L * j.keep * nkv * pieces;
  for (size_t u = (size_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (size_t)gridDim.x * 256) {
    const size_t r = u / pieces;
    const int p = (int)(u - r * pieces);
    const size_t t = r / nkv;                  // layer keep + i
    const int h = (int)(r - t * nkv);
    const size_t l = t / j.keep, i = t - l * j.keep;
    const size_t tok = (size_t)j.kept[(l * nkv + h) * j.keep + i];
    dst[u] = src[((l * j.P + tok) * nkv + h) * pieces + p];
  }
}

// The scale bytes of 4-bit caches, `groups` a row.
__global__ void __launch_bounds__(256) kv_gather_scales_kernel(KvEvictJobs jobs, int L, int nkv, int hd) {
  const KvEvictJob &j = jobs.j[blockIdx.y];
  const int groups = hd / kKvGroup;
  const uint8_t *src = reinterpret_cast<const uint8_t *>(blockIdx.z ? j.sv : j.sk) + kv4_code_bytes(L, j.P, nkv, hd);
  uint8_t *dst = reinterpret_cast<uint8_t *>(blockIdx.z ? j.dv : j.dk) + kv4_code_bytes(L, j.keep, nkv, hd);
  const size_t n = (size_t)L * j.keep * nkv * groups;
  for (size_t u = (size_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (size_t)gridDim.x * 256) {
    const size_t r = u / groups;
    const int p = (int)(u - r * groups);
    const size_t t = r / nkv;
    const int h = (int)(r - t * nkv);
    const size_t l = t / j.keep, i = t - l * j.keep;
    const size_t tok = (size_t)j.kept[(l * nkv + h) * j.keep + i];
    dst[u] = src[((l * j.P + tok) * nkv + h) * groups + p];
  }
}

hipError_t launch_kv_evict(const KvEvictJobs &jobs, int n, int L, int nkv, int hd, int esz, bool fp4, hipStream_t s) {
  int most = 0;
  for (int i = 0; i < n; ++i) most = std::max(most, jobs.j[i].keep);
  if (n <= 0 || most == 0) return hipSuccess;
  int longest = 0;
  for (int i = 0; i < n; ++i) longest = std::max(longest, jobs.j[i].P);
  // Rows of few tokens want many blocks a CU, long ones many loads in flight a row: 256 and 1024 threads take
  // 14 and 20 us over 576 rows of 512 to 1280 tokens, 637 and 287 over 4 rows of 131072 (the latter before the last pass was
  // dealt to the waves in runs: 178 now).
  hipLaunchKernelGGL(kv_select_kernel, dim3(L * nkv, n), dim3(longest <= 4096 ? 256 : 1024),
                     std::min(longest, kSelectRow) * sizeof(float), s, jobs, L * nkv);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pieces = (fp4 ? hd / 2 : hd * esz) / 16;
  const size_t rows = (size_t)L * most * nkv;
  hipLaunchKernelGGL(kv_gather_kernel, dim3(grid_x(rows * pieces, 4096), n, 2), dim3(256), 0, s, jobs, L, nkv, pieces);
  e = hipGetLastError();
  if (e != hipSuccess || !fp4) return e;
  hipLaunchKernelGGL(kv_gather_scales_kernel, dim3(grid_x(rows * (hd / kKvGroup), 1024), n, 2), dim3(256), 0, s, jobs, L,
                     nkv, hd);
  return hipGetLastError();
}

// ------------------------------------------------------------------ plain attention, either format
// 16 consecutive elements of a row in fp32.
template <typename T>
__device__ __forceinline__ void load16(const T *p, float (&f)[16]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x8 v = reinterpret_cast<const bf16x8 *>(p)[h];
#pragma unroll
      for (int q = 0; q < 8; ++q) f[8 * h + q] = (float)v[q];
    }
  } else {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const float4 v = reinterpret_cast<const float4 *>(p)[h];
      f[4 * h] = v.x; f[4 * h + 1] = v.y; f[4 * h + 2] = v.z; f[4 * h + 3] = v.w;
    }
  }
}
// Elements 16 c .. 16 c + 15 of row `row` of a cache (rows of HD elements).
template <int HD, typename T, bool FP4>
__device__ __forceinline__ void load16_cache(const void *cache, size_t code_bytes, size_t row, int c, float (&f)[16]) {
  if constexpr (FP4) {
    const uint8_t *b = reinterpret_cast<const uint8_t *>(cache);
    const uint2 w = *reinterpret_cast<const uint2 *>(b + row * (HD / 2) + c * 8);
    const float s = kv4_scale(b[code_bytes + row * (HD / kKvGroup) + (c >> 1)]);
    const bf16x8 v0 = kv4_bf16x8(w.x, s), v1 = kv4_bf16x8(w.y, s);
#pragma unroll
    for (int q = 0; q < 8; ++q) { f[q] = (float)v0[q]; f[8 + q] = (float)v1[q]; }
  } else {
    load16(reinterpret_cast<const T *>(cache) + row * HD + c * 16, f);
  }
}
template <int LG>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = 1; o < LG; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// fp32 mode.  A block takes four query rows, its four waves different keys.  LG = HD / 16 lanes hold a key (16
// elements each), so 64 / LG keys are under way at once in a wave, read once for the four rows; each lane group
// has a softmax of its own for each (running maximum, sum, weighted values); the groups join at the end, then the
// waves through LDS, in order.  Vector units and the latency of K and V bound it: 40 requests of 512 to 768
// tokens under 16 or 50, 8 heads of 256: 450 us over caches of either format (860 over fp32 ones with a wave a row and
// no key shared); one token over 816: 87.
template <int HD, bool FP4>
__global__ void __launch_bounds__(256) kv_attention_rows_kernel(KvAttnArgs ka) {
  constexpr int LG = HD / 16, NG = 64 / LG, RW = 4;
  __shared__ float so[4][RW][HD], sm[4][RW], sl[4][RW];
  const AttnArgs &a = ka.a;
  const AttnItem it = a.items[blockIdx.x];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, q0 = blockIdx.y * RW;
  if (q0 >= it.nq) return;
  const int G = a.nq / a.nkv, c = lane % LG, g = lane / LG;
  const float *qkv = reinterpret_cast<const float *>(a.qkv);
  float q[RW][16], acc[RW][16] = {}, m[RW], l[RW];
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const int qrow = it.q0 + min(q0 + r, it.nq - 1);
    load16(qkv + ((size_t)it.tok_off + qrow / G) * a.ldqkv + (size_t)(it.kvh * G + qrow % G) * HD + c * 16, q[r]);
    m[r] = -INFINITY;
    l[r] = 0.f;
  }
  const size_t codes = kv4_code_bytes(ka.L, it.P, a.nkv, HD);
  const float scale = 1.0f / sqrtf((float)HD);
  for (int k0 = it.kbeg + wave * NG; k0 < it.kend; k0 += 4 * NG) {
    const int key = k0 + g;
    const bool on = key < it.kend;
    const int kk = on ? key : it.kend - 1;
    float kf[16], vf[16];
    if (kk < it.P) {
      const size_t r = ((size_t)a.layer * it.P + kk) * a.nkv + it.kvh;
      load16_cache<HD, float, FP4>(it.pk, codes, r, c, kf);
      load16_cache<HD, float, FP4>(it.pv, codes, r, c, vf);
    } else {
      const float *p = qkv + ((size_t)it.tok_off + kk - it.P) * a.ldqkv + (size_t)(a.nq + it.kvh) * HD + c * 16;
      load16(p, kf);
      load16(p + (size_t)a.nkv * HD, vf);
    }
#pragma unroll
    for (int r = 0; r < RW; ++r) {
      float dot = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) dot = fmaf(q[r][e], kf[e], dot);
      dot = group_sum<LG>(dot) * scale;
      if (!on || dot == -INFINITY) continue;                // a weight of 0
      const float mn = fmaxf(m[r], dot), al = expf(m[r] - mn), p = expf(dot - mn);
      l[r] = l[r] * al + p;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[r][e] = acc[r][e] * al + p * vf[e];
      m[r] = mn;
    }
  }
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    float mx = m[r];
#pragma unroll
    for (int o = LG; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    const bool any = l[r] > 0.f || l[r] != l[r];            // a group without keys adds nothing
    const float w = any ? expf(m[r] - mx) : 0.f;
    float ls = l[r] * w;
#pragma unroll
    for (int o = LG; o < 64; o <<= 1) ls += __shfl_xor(ls, o, 64);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = any ? acc[r][e] * w : 0.f;
#pragma unroll
      for (int o = LG; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
      if (g == 0) so[wave][r][c * 16 + e] = v;
    }
    if (lane == 0) { sm[wave][r] = mx; sl[wave][r] = ls; }
  }
  __syncthreads();
  // a wave a row
  if (q0 + wave >= it.nq) return;
  const int qrow = it.q0 + q0 + wave, qg = it.kvh * G + qrow % G;
  const size_t row = (size_t)it.tok_off + qrow / G;
  float mx = -INFINITY, f[4], L = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm[w][wave]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float x = sl[w][wave];
    f[w] = x > 0.f || x != x ? expf(sm[w][wave] - mx) : 0.f;
    L += x * f[w];
  }
  const float inv = 1.0f / L;
  float *out = reinterpret_cast<float *>(a.o);
  for (int e = lane; e < HD; e += 64) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v += so[w][wave][e] * f[w];
    const size_t col = (size_t)qg * HD + e;
    out[a.o_rows > 0 ? kb32_offset(a.o_rows, row, col) : row * a.ldo + col] = v * inv;   // row-major, or kb32
  }
  if (a.lse && lane == 0) a.lse[row * a.nq + qg] = mx + logf(L);
}

template <int HD>
static void launch_rows(const KvAttnArgs &a, dim3 grid, hipStream_t s) {
  if (a.fp4) hipLaunchKernelGGL((kv_attention_rows_kernel<HD, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_attention_rows_kernel<HD, false>), grid, dim3(256), 0, s, a);
}

hipError_t launch_kv_attention_rows(const KvAttnArgs &a, hipStream_t s) {
  if (a.a.n_items <= 0) return hipSuccess;
  dim3 grid(a.a.n_items, kAttnQB / 4);
  switch (a.a.hd) {
    case 32: launch_rows<32>(a, grid, s); break;
    case 64: launch_rows<64>(a, grid, s); break;
    case 128: launch_rows<128>(a, grid, s); break;
    case 256: launch_rows<256>(a, grid, s); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace rosa
