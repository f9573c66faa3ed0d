// Attention weight of cached tokens on the matrix cores (gfx950), one layer:
//   mass_j = sum over the KV head's query rows r of exp(q_r . k_j / sqrt(hd) - lse_r).
//
// S = Q K^T in 32 x 32 tiles with a key to each lane: the sum over query rows is then a sum over a lane's
// registers.  The keys stay, the queries pass: a wave holds KT tiles of 32 keys in registers (a 4-bit
// cache's turned to bf16 there, exactly, once for all queries, so both formats share the products), and the
// block's queries come by through a ring in LDS.  A block's waves take WK different groups of keys and 4 / WK
// different tiles of queries; each key's sum is made by one block in a fixed order (no atomics).
// 256 requests of 512 to 1280 cached tokens, 16 or 50 action tokens x 8 heads, head_dim 256: 54 us over
// a bf16 cache (a key at a time on the vector units: 2220), 45 us over a 4-bit one; one request's 816
// tokens under 50: 9 (385).  In the fp32 mode the products are fp32 ones, a key tile fills the registers:
// 60 us over 40 requests of 512 to 768 tokens under 16 or 50, 59 over the one of 816 under 50 (380).
// Bounds (bf16, 256 requests): the products take 14 us of the matrix cores, K 24 us of HBM.
#include <math.h>

#include <type_traits>

#include "rosa_device.h"
#include "rosa_internal.h"

namespace rosa {

// 64 floats, each lane's from its own byte offset behind a uniform base, to lds + 4 lane
__device__ __forceinline__ void dma_256(const float *base, uint32_t off, uint32_t lds) {
  const uint64_t b = (uint64_t)(size_t)base;
  const uint64_t ub = ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32) |
                      (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(ub), "s"(lds) : "memory", "m0");
#pragma clang diagnostic pop
}

// 16 bytes of a row, an operand: 8 bf16 or (four products of 2 elements each) 4 fp32
template <typename T> struct MassOperand { typedef bf16x8 type; };
template <> struct MassOperand<float> { typedef f32x4 type; };
__device__ __forceinline__ f32x16 mass_product(bf16x8 q, bf16x8 k, f32x16 s) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k, s, 0, 0, 0); }
__device__ __forceinline__ f32x16 mass_product(f32x4 q, f32x4 k, f32x16 s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q[e], k[e], s, 0, 0, 0);
  return s;
}

// A lane's half of a cached row (HD / 2 elements) in the model's type, in the order of its operands: operand i is the
// row's chunk of 16 bytes 2 i + half, of a 4-bit cache the chunk i of the row's half (whole blocks, or half of one).
template <int HD, typename T, bool FP4>
__device__ __forceinline__ void read_key(const KvMassArgs &a, const MassItem &it, int key, int half,
                                         typename MassOperand<T>::type (&k)[HD * (int)sizeof(T) / 32]) {
  const size_t row = ((size_t)a.layer * it.P + key) * a.nkv + it.kvh;
  if constexpr (!FP4) {
    const uint8_t *p = reinterpret_cast<const uint8_t *>(it.pk) + row * HD * sizeof(T) + half * 16;
#pragma unroll
    for (int i = 0; i < HD * (int)sizeof(T) / 32; ++i) k[i] = *reinterpret_cast<const typename MassOperand<T>::type *>(p + 32 * i);
    return;
  } else {
  constexpr int NW = HD / 16, NB = HD >= 64 ? HD / 64 : 1;      // code words, blocks
  const uint8_t *p = reinterpret_cast<const uint8_t *>(it.pk) + row * (HD / 2) + half * (HD / 4);
  const uint8_t *sp = reinterpret_cast<const uint8_t *>(it.pk) + kv4_code_bytes(a.L, it.P, a.nkv, HD) + row * (HD / 32) +
                      (HD >= 64 ? half * NB : 0);
  uint32_t w[NW];
  if constexpr (NW == 2) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < NW / 4; ++j) {
      const uint4 v = reinterpret_cast<const uint4 *>(p)[j];
      w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
    }
  }
  uint8_t s[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) s[j] = sp[j];
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const bf16x8 v = kv4_bf16x8(w[i], kv4_scale(s[i / 4]));
    if constexpr (sizeof(T) == 2) {
      k[i] = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) k[2 * i + e / 4][e % 4] = (float)v[e];
    }
  }
  }
}

template <int HD, typename T, int KT, int WK>
struct MassTile {
  static constexpr int ROWB = HD * (int)sizeof(T), CPR = ROWB / 16, TILEB = 32 * ROWB, NF = CPR / 2;
  static constexpr int WR = 4 / WK, KEYS = 32 * KT * WK;
  static constexpr int STAGEB = WR * TILEB, UNITS = STAGEB / 1024;      // a stage of the ring: WR query tiles
  static constexpr int DEPTH = 65536 / STAGEB < 4 ? 65536 / STAGEB : 4;
  static constexpr int LSE = DEPTH * STAGEB;                            // then 64 lse words a stage and wave
  static constexpr int LDSB = LSE + DEPTH * 4 * 256;
  static_assert(DEPTH >= 2 && LDSB <= 81920, "two blocks a CU");
};

template <int HD, typename E, int KT, int WK, bool FP4>
__global__ void __launch_bounds__(256, 2) kv_mass_kernel(KvMassArgs a) {
  using T = MassTile<HD, E, KT, WK>;
  typedef typename MassOperand<E>::type operand;
  constexpr int ROWB = T::ROWB, CPR = T::CPR, NF = T::NF, WR = T::WR, DEPTH = T::DEPTH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDSB];
  // Neighbouring items read the same queries: blocks of one XCD (every eighth) take a run of items.
  const int per = a.n_items >> 3, b = blockIdx.x;
  const MassItem it = a.items[b < 8 * per ? (b & 7) * per + (b >> 3) : b];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int col = lane & 31, half = lane >> 5, kg = wave % WK, rg = wave / WK;
  const int G = a.nq / a.nkv, R = it.H * G, n = (R + 32 * WR - 1) / (32 * WR);
  const float rG = 1.0f / (float)G;
  const E *qkv = reinterpret_cast<const E *>(a.qkv);
  const uint32_t lds0 = lds_u32(smem);

  // The queries of stage t (rows past the last: the last one), whole rows side by side, chunk c of row r at
  // c ^ swz(r), and the lse of the wave's own tile.  Row x of the stage: its token and head from their first
  // ones (tok0, head0); a quotient by G in fp32, exact below 2^20.
  constexpr int NU = (T::UNITS + 3) / 4;
  auto row_of = [&](int x, int h0, int last, int &tok, int &head) {
    x = min(h0 + x, last);
    tok = (int)(((float)x + 0.5f) * rG);
    head = x - tok * G;
  };
  auto unit_row = [&](int j) { return (wave + 4 * j) * (64 / CPR) + lane / CPR; };
  auto unit_col = [&](int r) { return ((lane % CPR) ^ at::swz(r, CPR)) * (16 / (int)sizeof(E)); };
  // Where G divides a stage its rows lie the same way in each: lane offsets made once.
  const bool even = (32 * WR) % G == 0;
  uint32_t qoff[NU], loff;
  {
    int tok, head;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      row_of(unit_row(j), 0, 32 * WR, tok, head);
      qoff[j] = (uint32_t)(tok * a.ldqkv + head * HD + unit_col(unit_row(j))) * (uint32_t)sizeof(E);
    }
    row_of(rg * 32 + col, 0, 32 * WR, tok, head);
    loff = (uint32_t)(tok * a.nq + head) * 4;
  }
  auto fetch = [&](int t) {
    const int base = t * 32 * WR, tok0 = base / G;
    const uint32_t st = lds0 + (uint32_t)(t % DEPTH * T::STAGEB), lst = lds0 + (uint32_t)(T::LSE + (t % DEPTH * 4 + wave) * 256);
    const E *q = qkv + (size_t)(it.tok_off + tok0) * a.ldqkv + (size_t)it.kvh * G * HD;
    const float *l = a.lse + (size_t)(it.tok_off + tok0) * a.nq + it.kvh * G;
    if (even && base + 32 * WR <= R) {
#pragma unroll
      for (int j = 0; j < NU; ++j)
        if (T::UNITS % 4 == 0 || wave + 4 * j < T::UNITS) dma_1k_s(q, qoff[j], st + (wave + 4 * j) * 1024);
      dma_256(l, loff, lst);
      return;
    }
    const int h0 = base - tok0 * G, last = R - 1 - tok0 * G;
    int tok, head;
#pragma unroll
    for (int j = 0; j < NU; ++j) {
      if (T::UNITS % 4 && wave + 4 * j >= T::UNITS) continue;
      row_of(unit_row(j), h0, last, tok, head);
      dma_1k(q + (size_t)tok * a.ldqkv + head * HD + unit_col(unit_row(j)), st + (wave + 4 * j) * 1024);
    }
    row_of(rg * 32 + col, h0, last, tok, head);
    dma_256(l, (uint32_t)(tok * a.nq + head) * 4, lst);
  };
#pragma unroll
  for (int t = 0; t < DEPTH - 1; ++t)
    if (t < n) fetch(t);

  const bool active = kg * KT * 32 < it.nk;
  operand k[KT][NF];
  if (active)
#pragma unroll
    for (int x = 0; x < KT; ++x) read_key<HD, E, FP4>(a, it, it.k0 + min((kg * KT + x) * 32 + col, it.nk - 1), half, k[x]);
  __builtin_amdgcn_s_waitcnt(at::waitcnt_vm(0));      // the keys, here: no wait for them is left to the loop

  const float sl2 = 1.4426950408889634f / sqrtf((float)HD);
  float sum[KT] = {};
  for (int t = 0; t < n; ++t) {
    // stage t has landed (DEPTH - 2 behind it may not have: as many copies a wave, at least one); then it is in LDS
    // for every wave, and every wave is done with stage t - 1, whose place the next takes
    if (t + DEPTH - 1 > n || T::UNITS % 4) __builtin_amdgcn_s_waitcnt(at::waitcnt_vm(0));
    else __builtin_amdgcn_s_waitcnt(at::waitcnt_vm((DEPTH - 2) * (T::UNITS / 4 + 1)));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + DEPTH - 1 < n) fetch(t + DEPTH - 1);
    const int base = (t * WR + rg) * 32;
    if (!active || base >= R) continue;
    const uint32_t q0 = lds0 + (uint32_t)(t % DEPTH * T::STAGEB + rg * T::TILEB + col * ROWB) +
                        (uint32_t)(((FP4 ? NF * half : half) ^ at::swz(col, CPR)) << 4);
    constexpr int RA = KT == 2 || NF < 6 ? (NF < 4 ? NF : 4) : 6;            // operands are read RA - 1 ahead
    auto qfrag = [&](int i) {
      return *reinterpret_cast<const __attribute__((address_space(3))) operand *>(lds_ptr(q0 ^ (uint32_t)(i << (FP4 ? 4 : 5))));
    };
    operand q[RA];
#pragma unroll
    for (int i = 0; i < RA - 1; ++i) q[i] = qfrag(i);
    // register r: query row (r / 4) 8 + 4 half + r % 4 of the tile
    const uint32_t l0 = lds0 + (uint32_t)(T::LSE + (t % DEPTH * 4 + wave) * 256 + half * 16);
    f32x4 l[4];
    f32x16 s[KT] = {};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      if (i + RA - 1 < NF) q[(i + RA - 1) % RA] = qfrag(i + RA - 1);
      else if (i + RA - 1 - NF < 4) l[i + RA - 1 - NF] = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(lds_ptr(l0 + (i + RA - 1 - NF) * 32));
#pragma unroll
      for (int x = 0; x < KT; ++x) s[x] = mass_product(q[i % RA], k[x][i], s[x]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = RA - 1; j < 4; ++j) l[j] = *reinterpret_cast<const __attribute__((address_space(3))) f32x4 *>(lds_ptr(l0 + j * 32));
    auto add = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        const f32x4 lj = l[j4] * -1.4426950408889634f;
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          float w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            w[j] = __builtin_amdgcn_exp2f(fmaf(s[x][4 * j4 + j], sl2, lj[j]));
            if (!whole.value) w[j] = base + j4 * 8 + half * 4 + j < R ? w[j] : 0.f;
          }
          sum[x] += (w[0] + w[1]) + (w[2] + w[3]);
        }
      }
    };
    if (base + 32 <= R) add(std::true_type{});
    else add(std::false_type{});
  }
  float *m = it.mass + ((size_t)a.layer * a.nkv + it.kvh) * it.P + it.k0;
#pragma unroll
  for (int x = 0; x < KT; ++x) sum[x] += __shfl_xor(sum[x], 32, 64);
  if constexpr (WR > 1) {                       // the query groups' sums, in order
    float *red = reinterpret_cast<float *>(smem);
    __syncthreads();
    if (half == 0)
#pragma unroll
      for (int x = 0; x < KT; ++x) red[rg * T::KEYS + (kg * KT + x) * 32 + col] = sum[x];
    __syncthreads();
    for (int j = threadIdx.x; j < it.nk; j += 256) {
      float v = red[j];
#pragma unroll
      for (int r = 1; r < WR; ++r) v += red[r * T::KEYS + j];
      m[j] = a.accumulate ? m[j] + v : v;
    }
  } else {
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const int j = (kg * KT + x) * 32 + col;
      if (half == 0 && j < it.nk) m[j] = a.accumulate ? m[j] + sum[x] : sum[x];
    }
  }
}

template <int HD, typename E, int KT, int WK>
static void launch_mass(const KvMassArgs &a, hipStream_t s) {
  if (a.fp4) hipLaunchKernelGGL((kv_mass_kernel<HD, E, KT, WK, true>), dim3(a.n_items), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_mass_kernel<HD, E, KT, WK, false>), dim3(a.n_items), dim3(256), 0, s, a);
}

template <int HD>
static hipError_t launch_mass_keys(const KvMassArgs &a, bool bf16_mode, hipStream_t s) {
  static_assert(MassTile<HD, bf16, 2, 4>::KEYS == kMassLarge && MassTile<HD, bf16, 1, 2>::KEYS == kMassSmall &&
                    MassTile<HD, float, 1, 4>::KEYS == kMassFloat, "item sizes");
  if (!bf16_mode && a.keys == kMassFloat) launch_mass<HD, float, 1, 4>(a, s);
  else if (bf16_mode && a.keys == kMassLarge) launch_mass<HD, bf16, 2, 4>(a, s);
  else if (bf16_mode && a.keys == kMassSmall) launch_mass<HD, bf16, 1, 2>(a, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

// Keys a block takes.  Large blocks read the queries from LDS once for two tiles of keys and from memory once for 256
// keys; but a set of fewer than one of them for each CU is done sooner in small ones.
int kv_mass_keys(bool bf16_mode, int64_t large_blocks) {
  return !bf16_mode ? kMassFloat : large_blocks >= 256 ? kMassLarge : kMassSmall;
}

hipError_t launch_kv_mass(const KvMassArgs &a, bool bf16_mode, hipStream_t s) {
  if (a.n_items <= 0) return hipSuccess;
  switch (a.hd) {
    case 32: return launch_mass_keys<32>(a, bf16_mode, s);
    case 64: return launch_mass_keys<64>(a, bf16_mode, s);
    case 128: return launch_mass_keys<128>(a, bf16_mode, s);
    case 256: return launch_mass_keys<256>(a, bf16_mode, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace rosa
