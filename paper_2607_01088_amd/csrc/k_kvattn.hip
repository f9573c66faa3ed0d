// Ragged attention of action tokens over 4-bit prefix caches and their own bf16
// keys and values (gfx950 MFMA), one layer.
//
// Work items, blocks and lists are those of the bf16 attention kernel: an
// item is (request, KV head, up to 128 NG query rows, key range), four waves own
// NG groups of 32 query rows each, S^T = K Q^T and O^T += V^T P^T with 32 x 32 MFMA tiles,
// each lane one query column.  What differs is where K and V come from.
//
// K: the matrix cores read the codes themselves.  v_mfma_scale_f32_32x32x64_f8f6f4
// takes a 4-bit operand whose lane holds 32 consecutive elements (16 bytes) of a row
// and their scale byte: exactly a block of the cache.  The other operand, Q in bf16, is
// split into three terms of 6 bits (e2m1's wider sibling e2m3: 4 significant bits
// near the top of a block) on scales 2^e, 2^(e-4), 2^(e-9), e the least with
// max|q| <= 7.5 2^e over 32 elements: q is then a multiple of 2^(e-12) and exact, unless it has
// bits below that; so off by at most 2^(e-13) <= 2^-14.9 of the block's
// largest magnitude, well below what rounding q to bf16 lost.  Three products with 6-bit operands at
// 9.5 PFLOP/s (measured, 4 x 6 bit) cost 3/4 of one in bf16 (2.3 PFLOP/s), and no
// instruction is spent on turning K to bf16.
// V: its scales run along head_dim, across the product's summed index, so it is
// turned to bf16 (exact): every thread converts one block of the next tile into
// LDS, from where the transposed reads feed the MFMAs.
// The request's own keys and values (bf16, at the end of the key range) run
// through the same loop with bf16 products.
// 256 requests of 512 to 1280 cached tokens, 16 or 50 action tokens x 8 heads, head_dim 256: 98 us (the matrix
// cores alone 24, the memory 28; the kernel over a bf16 cache 105), 512 of 1024 to 2048 under 50: 380 (125, 90; 445).
// Two waves a SIMD wait for each other's phases: neither the loads nor the score products hold it (leaving
// either out saves 4 to 6%), P V is a quarter; an item's own keys, queries and results take 14 us, the split 6.
#include <math.h>

#include <type_traits>

#include "rosa_device.h"
#include "rosa_internal.h"

namespace rosa {

typedef __attribute__((ext_vector_type(32))) __bf16 bf16x32;
typedef __attribute__((ext_vector_type(32))) float f32x32;
typedef __attribute__((ext_vector_type(6))) uint32_t u32x6;
typedef __attribute__((ext_vector_type(6))) int i32x6;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// A tile's rows in global memory: a uniform base (scalar registers) plus a per-lane byte offset.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t tile_rsrc(const uint8_t *base) {
  const uint64_t b = (uint64_t)(size_t)base;
  const uint64_t u = ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  return __builtin_amdgcn_make_buffer_rsrc((void *)(size_t)u, 0, -1, 0x00027000);
}

// Every wave's LDS accesses so far are done before any wave goes on.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// This wave's loads and copies have landed.
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(at::waitcnt_vm(0));
  asm volatile("" ::: "memory");
}

template <int HD, int NG>
struct Kv4Tile {
  static constexpr int ROWB = HD * 2, CPR = ROWB / 16;     // bf16 row: bytes, 16-byte chunks
  static constexpr int TILEB = 32 * ROWB;                  // 32 bf16 rows
  static constexpr int K4ROW = HD / 2, CK = HD / 32;       // code row: bytes, 16-byte chunks (blocks)
  static constexpr int K4TILE = 32 * K4ROW;
  static constexpr int NCH = HD >= 64 ? HD / 64 : 1;       // 64-wide products over head_dim
  // LDS: V tiles (bf16) 2, own keys' K tiles (bf16) 2, K code tiles 3
  static constexpr int AOFF = 2 * TILEB, KOFF = 4 * TILEB, RINGB = KOFF + 3 * K4TILE;
  static constexpr int STGB = 4 * NG * 32 * 2 * HD;        // output staging
  static constexpr int LDSB = RINGB > STGB ? RINGB : STGB;
  static_assert(LDSB >= 4 * TILEB + 512, "a tile a wave and their sums");
  // chunk swizzle of code rows: the 16 rows that a 16-lane group reads at one chunk fall in
  // distinct 16-byte columns of the 256-byte bank row
  static constexpr int SHIFT = K4ROW == 128 ? 1 : K4ROW == 64 ? 2 : K4ROW == 32 ? 3 : 4;
  __device__ static int ksw(int row) { return (row >> SHIFT) & (CK - 1); }
};

// Conversions of 32 elements on scale s to 6 bits and back.  In assembly for the early clobber:
// they write their first result registers before they have read every source register, and the
// builtins let the compiler put the result onto a source.
__device__ __forceinline__ u32x6 to_fp6(const bf16x32 &v, float s) {
  u32x6 t;
  asm volatile("v_cvt_scalef32_pk32_fp6_bf16 %0, %1, %2" : "=&v"(t) : "v"(v), "v"(s));
  return t;
}
// element 2 i from a, 2 i + 1 from b
__device__ __forceinline__ u32x6 to_fp6(const f32x16 &a, const f32x16 &b, float s) {
  u32x6 t;
  asm volatile("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3" : "=&v"(t) : "v"(a), "v"(b), "v"(s));
  return t;
}
__device__ __forceinline__ f32x32 from_fp6(const u32x6 &t, float s) {
  f32x32 v;
  asm volatile("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2" : "=&v"(v) : "v"(t), "v"(s));
  return v;
}

// 32 consecutive query elements as three 6-bit terms; returns the first one's scale byte (the
// others' are 4 and 9 less), 255 where an element is not finite (every product with the first
// term is then NaN).
__device__ __forceinline__ uint32_t split_query(const bf16x8 (&q)[4], u32x6 (&t)[3]) {
  f32x16 r[2];                               // even and odd elements
  bf16x32 b;
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    b[i] = q[i / 8][i % 8];
    r[i & 1][i >> 1] = (float)b[i];
    a = max(a, __float_as_uint((float)b[i]) & 0x7fffffffu);
  }
  const int E = (int)(a >> 23) - 127;
  const int e = min(125, max(-115, (a & 0x7fffffu) <= 0x700000u ? E - 2 : E - 1));
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float s = __uint_as_float((uint32_t)(e + 127 - (k == 0 ? 0 : k == 1 ? 4 : 9)) << 23);
    t[k] = k == 0 ? to_fp6(b, s) : to_fp6(r[0], r[1], s);
    if (k == 2) break;
    const f32x32 v = from_fp6(t[k], s);
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i & 1][i >> 1] -= v[i];     // exact: a multiple of the element's last bit
  }
  return a >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
}

// ------------------------------------------------------------------ few rows
// An item of at most 16 query rows (an action token or two): memory and latency are all it costs, so its four
// waves take different keys, tile by tile in turn, with no barrier between them.  16 x 16 tiles, a
// lane one query row (lane & 15): S^T = K Q^T with 128-wide products of codes that come straight from the cache
// into registers (lane group g, lane >> 4: block 4 c + g of keys lane & 15 and 16 more), O^T += V^T P^T with V
// turned to bf16 through a tile of LDS that is the wave's own.  The loads of a wave's next tile or
// two are always on their way; the waves' O are joined in order at the end.
// One token x 8 heads over 816 keys: 11 us with the join (14 as an ordinary item, three of its waves idle); over
// 60 and 131 thousand, head_dim 128: 27 (57), of which the codes take 11 at a copy's rate.
constexpr int kFewRows = 16;

template <int HD>
__device__ __forceinline__ void kv4_few_rows(const KvAttnArgs &ka, const AttnItem &it, uint8_t *smem, float sl2) {
  constexpr int ROWB = HD * 2, CPR = ROWB / 16, TILEB = 32 * ROWB, K4ROW = HD / 2, CK = HD / 32;
  constexpr int NP = HD > 128 ? HD / 128 : 1;              // 128-wide products
  constexpr int NB = CK > 2 ? CK / 2 : 1;                  // V blocks a lane turns to bf16
  constexpr int NT = HD / 16;
  const AttnArgs &a = ka.a;
  const int G = a.nq / a.nkv;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, r = lane & 15, g = lane >> 4;
  const uint32_t lds0 = lds_u32(smem), tile0 = lds0 + (uint32_t)(wave * TILEB);
  const __attribute__((address_space(1))) bf16 *qkv = (const __attribute__((address_space(1))) bf16 *)(a.qkv);

  const int x = it.q0 + min(r, it.nq - 1), head = it.kvh * G + x % G;
  const size_t tok = (size_t)(it.tok_off + x / G);
  const __attribute__((address_space(1))) bf16 *qp = qkv + tok * a.ldqkv + (size_t)head * HD;
  const int pn = max(0, min(it.kend, it.P) - it.kbeg), np = (pn + 31) >> 5;
  const int ab = max(it.kbeg, it.P), an = max(0, it.kend - ab), na = (an + 31) >> 5;

  f32x4 o[NT];
  float mb = 3e38f, l = 0.f;                               // as in the kernel below
#pragma unroll
  for (int n = 0; n < NT; ++n) o[n] = f32x4{};

  // Rows of V in LDS: chunk c of row k at c ^ swz(k).  The transposed reads: rows 4 g + (lane & 15) / 4 and 16
  // more, 8 bytes each of a tile's 32.
  uint32_t vbase;
  {
    const int k = 4 * g + (r >> 2);
    vbase = tile0 + (uint32_t)(k * ROWB + ((((r >> 1) & 1) ^ at::swz(k, CPR)) << 4) + 8 * (r & 1));
  }
  // Scores (s[h] register j: key 16 h + 4 g + j, masked from n_keys on) to weights, and their V rows, which are
  // in LDS, onto O.
  auto accumulate = [&](f32x4 (&s)[2], int n_keys) __attribute__((always_inline)) {
    if (n_keys < 32) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (16 * h + 4 * g + j >= n_keys) s[h][j] = -INFINITY;
    }
    float tmax = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) tmax = fmaxf(tmax, s[i / 4][i % 4]);
    if (__ballot(fmaf(tmax, sl2, mb) > 32.0f)) {
      float tm = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
      const bool up = fmaf(tm, sl2, mb) > 32.0f;           // the groups of a query agree
      const float nb = up ? -tm * sl2 : mb, f = up ? __builtin_amdgcn_exp2f(nb - mb) : 1.0f;
      mb = nb;
      l *= f;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] *= f;
    }
    asm volatile("" ::: "memory");                         // V rows written, then read (LDS keeps a wave's order)
    // Weights in two bf16 terms (16 significant bits, not 8): a product more for each V operand, which the loads
    // of the next tile cover.
    bf16x8 p, p2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float w = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], sl2, mb));
      l += w;
      p[i] = (bf16)w;
      p2[i] = (bf16)(w - (float)p[i]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t v = vbase ^ (uint32_t)(n << 5);
      const bf16x8 f = lds_tr_pair(lds_ptr(v), lds_ptr(v) + 16 * ROWB);
      o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p, o[n], 0, 0, 0);
      o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p2, o[n], 0, 0, 0);
    }
  };

  if (wave < np) {
    u32x6 q6[NP][3];
    uint32_t qs[NP];
#pragma unroll
    for (int c = 0; c < NP; ++c) {
      const int b = 4 * c + g;
      bf16x8 q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q[j] = *(const __attribute__((address_space(1))) bf16x8 *)(qp + 32 * (b < CK ? b : 0) + 8 * j);
        if (b >= CK) q[j] = bf16x8{};                      // a product is 128 wide
      }
      qs[c] = split_query(q, q6[c]);
    }
    // A tile: codes and scales of its keys, and of the V blocks that this lane turns to bf16 (rows and blocks dealt
    // so that 16 lanes write distinct 16-byte columns)
    auto vblock = [&](int j, int &row, int &blk) __attribute__((always_inline)) {
      if constexpr (HD == 256) { blk = (lane & 3) | ((lane >> 2) & 4); row = (((lane >> 2) & 3) << 2) | (lane >> 5) | ((j & 1) << 1) | ((j >> 1) << 4); }
      else if constexpr (HD == 128) { blk = lane & 3; row = (((lane >> 2) & 3) << 2) | (lane >> 4) | (j << 4); }
      else { blk = lane % CK; row = (lane / CK) & 31; }
    };
    const uint32_t rowb = (uint32_t)a.nkv * K4ROW, srow = (uint32_t)a.nkv * CK;
    const size_t r0 = ((size_t)a.layer * it.P + it.kbeg) * a.nkv + it.kvh, codes = kv4_code_bytes(ka.L, it.P, a.nkv, HD);
    typedef const __attribute__((address_space(1))) uint8_t g_u8;
    g_u8 *pk = (g_u8 *)(size_t)it.pk, *pv = (g_u8 *)(size_t)it.pv;
    struct Tile {
      i32x4 k[2][NP], v[NB];
      uint32_t ks[2][NP], vs[NB];
    };
    auto load = [&](Tile &x, int f) __attribute__((always_inline)) {
      g_u8 *kc = pk + (r0 + (size_t)f * a.nkv) * K4ROW, *vc = pv + (r0 + (size_t)f * a.nkv) * K4ROW;
      g_u8 *kz = pk + codes + (r0 + (size_t)f * a.nkv) * CK, *vz = pv + codes + (r0 + (size_t)f * a.nkv) * CK;
      const int last = pn - 1 - f;                         // rows past the last: the last one
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < NP; ++c) {
          const uint32_t row = (uint32_t)min(16 * h + r, last), b = (uint32_t)(4 * c + g < CK ? 4 * c + g : 0);
          x.k[h][c] = *(const __attribute__((address_space(1))) i32x4 *)(kc + (row * rowb + b * 16));
          x.ks[h][c] = kz[row * srow + b];
        }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        int row, blk;
        vblock(j, row, blk);
        row = min(row, last);
        x.v[j] = *(const __attribute__((address_space(1))) i32x4 *)(vc + ((uint32_t)row * rowb + (uint32_t)blk * 16));
        x.vs[j] = vz[(uint32_t)row * srow + (uint32_t)blk];
      }
    };
    // tile t, which x holds; then the wave's DEEP-next tile leaves for x (past the last tile that one again).
    // Two tiles on their way at head_dim 256 take registers that the other items' key loop, in the same kernel, needs.
    constexpr int DEEP = HD == 256 ? 1 : 2;
    auto step = [&](Tile &x, int t) __attribute__((always_inline)) {
      f32x4 s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h] = f32x4{};
#pragma unroll
        for (int c = 0; c < NP; ++c) {
          i32x4 kk = x.k[h][c];
          if (CK < 4 && g >= CK) kk = i32x4{};
          const i32x8 kf = __builtin_shufflevector(kk, kk, 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
          for (int x3 = 0; x3 < 3; ++x3) {
            const i32x6 q = __builtin_bit_cast(i32x6, q6[c][x3]);
            const i32x8 qf = __builtin_shufflevector(q, q, 0, 1, 2, 3, 4, 5, -1, -1);
            s[h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qf, s[h], 4, 2, 0, x.ks[h][c], 0, qs[c] - (x3 == 0 ? 0 : x3 == 1 ? 4 : 9));
          }
        }
      }
      if (32 * CK >= 64 || lane < 32 * CK)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          int row, blk;
          vblock(j, row, blk);
          const uint32_t d = tile0 + (uint32_t)(row * ROWB + (((4 * blk) ^ at::swz(row, CPR)) << 4));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<__attribute__((address_space(3))) bf16x8 *>((__attribute__((address_space(3))) uint8_t *)(size_t)(d ^ (i << 4))) =
                kv4_bf16x8((uint32_t)x.v[j][i], kv4_scale((uint8_t)x.vs[j]));
        }
      load(x, 32 * min(t + 4 * DEEP, np - 1));
      accumulate(s, pn - 32 * t);
    };
    Tile x0;
    load(x0, 32 * wave);
    int t = wave;
    if constexpr (DEEP == 1) {
      for (; t < np; t += 4) step(x0, t);
    } else {
      Tile x1;
      load(x1, 32 * min(wave + 4, np - 1));
      const int cnt = (np - wave + 3) >> 2;
      for (int i = 0; i < cnt >> 1; ++i, t += 8) {         // (no exit between the steps: the compiler would wait for both tiles)
        step(x0, t);
        step(x1, t + 4);
      }
      if (cnt & 1) step(x0, t);
    }
  }
  // the request's own keys, tiles np, np + 1, .. of the item
  for (int u = (wave - np) & 3; u < na; u += 4) {
    const int last = an - 1 - 32 * u;
    const __attribute__((address_space(1))) bf16 *ap = qkv + (size_t)(it.tok_off + ab - it.P + 32 * u) * a.ldqkv;
    const int kcol = (a.nq + it.kvh) * HD, vcol = (a.nq + a.nkv + it.kvh) * HD;
    f32x4 s[2] = {};
#pragma unroll
    for (int c = 0; c < HD / 32; ++c) {
      const bf16x8 q = *(const __attribute__((address_space(1))) bf16x8 *)(qp + 32 * c + 8 * g);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 kf = *(const __attribute__((address_space(1))) bf16x8 *)(ap + (size_t)min(16 * h + r, last) * a.ldqkv + kcol + 32 * c + 8 * g);
        s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q, s[h], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 32 * CPR / 64; ++i) {
      const int row = (i * 64 + lane) / CPR, c = lane % CPR;
      const i32x4 w = *(const __attribute__((address_space(1))) i32x4 *)(ap + (size_t)min(row, last) * a.ldqkv + vcol + c * 8);
      *reinterpret_cast<__attribute__((address_space(3))) i32x4 *>((__attribute__((address_space(3))) uint8_t *)(size_t)(tile0 + row * ROWB + ((c ^ at::swz(row, CPR)) << 4))) = w;
    }
    accumulate(s, last + 1);
  }

  // ---- the waves' results through LDS: o[n] as it lies, reference and sum behind them
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  lds_barrier();
  f32x4 *so = reinterpret_cast<f32x4 *>(smem);
  float2 *sml = reinterpret_cast<float2 *>(smem + 4 * TILEB);
#pragma unroll
  for (int n = 0; n < NT; ++n) so[(wave * NT + n) * 64 + lane] = o[n];
  if (g == 0) sml[wave * 16 + r] = make_float2(-mb, l);
  __syncthreads();
  float m = sml[r].x, f[4], L = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) m = fmaxf(m, sml[w * 16 + r].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = exp2f(sml[w * 16 + r].x - m);
    L += f[w] * sml[w * 16 + r].y;
  }
  if (r < it.nq) {
    const float inv = 1.0f / L;
    for (int n = wave; n < NT; n += 4) {
      f32x4 y = {};
#pragma unroll
      for (int w = 0; w < 4; ++w) y += so[(w * NT + n) * 64 + lane] * f[w];
      const int col = 16 * n + 4 * g;
      if (it.slot >= 0) {
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.part_o) + ((size_t)it.slot * kAttnQB + r) * HD + col) = y;
      } else {
        const size_t oc = (size_t)head * HD + col;
        const bf16x4 b = {(bf16)(y[0] * inv), (bf16)(y[1] * inv), (bf16)(y[2] * inv), (bf16)(y[3] * inv)};
        *reinterpret_cast<bf16x4 *>(reinterpret_cast<bf16 *>(a.o) + (a.o_rows > 0 ? kb32_offset(a.o_rows, tok, oc) : tok * a.ldo + oc)) = b;
      }
    }
    if (wave == 0 && g == 0) {
      if (it.slot >= 0) *reinterpret_cast<float2 *>(a.part_ml + ((size_t)it.slot * kAttnQB + r) * 2) = make_float2(m, L);
      else if (a.lse) a.lse[tok * a.nq + head] = (m + log2f(L)) * 0.6931471805599453f;
    }
  }
  lds_barrier();
}

template <int HD, int NG>
__global__ void __launch_bounds__(256, 2) kv4_attention_kernel(KvAttnArgs ka) {
  using T = Kv4Tile<HD, NG>;
  constexpr int NS = HD / 16, NT = HD / 32, CPR = T::CPR, ROWB = T::ROWB, TILEB = T::TILEB, CK = T::CK, NCH = T::NCH;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDSB];
  const AttnArgs &a = ka.a;
  if (a.ordered[blockIdx.x].nq <= 0) return;
  const int G = a.nq / a.nkv;
  const bf16 *qkv = reinterpret_cast<const bf16 *>(a.qkv);
  const uint32_t lds0 = lds_u32(smem);
  const float sl2 = 1.4426950408889634f / sqrtf((float)HD);   // log2(e) / sqrt(hd)

  for (int e = blockIdx.x; e >= 0;) {
  AttnItem it;
  {
    const uint32_t *src = reinterpret_cast<const uint32_t *>(a.ordered + e);
    uint32_t w[sizeof(AttnItem) / 4];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(AttnItem) / 4); ++i) w[i] = __builtin_amdgcn_readfirstlane(src[i]);
    __builtin_memcpy(&it, w, sizeof(AttnItem));
  }
  e = it.next;
  if (it.nq <= kFewRows) {
    kv4_few_rows<HD>(ka, it, smem, sl2);
    continue;
  }
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));      // per-lane addresses are not kept across items
  const int lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;
  const bool active = 32 * wave < it.nq;      // a wave without rows only helps with the copies

  // Key range in tiles of 32 keys: np prefix tiles, then na of the request's own keys.  Tile 0 of
  // each starts at the range's first key and gives its first pv0 (av0) keys; the others follow
  // without a gap and end at the range's end, so tile 0's remaining rows are tile 1's
  // first ones (masked here).  A range of fewer than 32 keys is one tile whose lanes past
  // the end read its last row.  So every tile is a uniform base plus per-lane offsets fixed for the item.
  const int pe = min(it.kend, it.P), ab = max(it.kbeg, it.P);
  const int pn = max(0, pe - it.kbeg), np = (pn + 31) >> 5, pv0 = pn - 32 * (np - 1);
  const int an = max(0, it.kend - ab), na = (an + 31) >> 5, av0 = an - 32 * (na - 1);
  auto atile = [&](int u) { return ab - it.P + (u == 0 ? 0 : 32 * (u - 1) + av0); };

  const uint32_t rowb = (uint32_t)a.nkv * T::K4ROW, srow = (uint32_t)a.nkv * CK;
  const size_t r0 = ((size_t)a.layer * it.P + it.kbeg) * a.nkv + it.kvh, codes = kv4_code_bytes(ka.L, it.P, a.nkv, HD);
  // the next tile to fetch: its codes and scales
  const uint8_t *kc = reinterpret_cast<const uint8_t *>(it.pk) + r0 * T::K4ROW;
  const uint8_t *vc = reinterpret_cast<const uint8_t *>(it.pv) + r0 * T::K4ROW;
  const uint8_t *ks = reinterpret_cast<const uint8_t *>(it.pk) + codes + r0 * CK;
  const uint8_t *vs = reinterpret_cast<const uint8_t *>(it.pv) + codes + r0 * CK;

  // ---- copies
  // K codes of prefix tile t into ring stage t % 3: 1 KB a wave (head_dim 32: half of one)
  constexpr bool K4HALF = T::K4TILE < 1024;
  const bool k4on = 1024 * wave < T::K4TILE;
  uint32_t koff;
  {
    const int p = wave * 64 + (K4HALF ? lane & 31 : lane), row = p / CK, c = (p % CK) ^ T::ksw(row);
    koff = (uint32_t)min(row, pn - 1) * rowb + c * 16;
  }
  // own keys: one bf16 tile (K or V columns) into LDS at dst
  auto copy_own = [&](int u, int col, uint32_t dst) __attribute__((always_inline)) {
    constexpr int UNITS = TILEB / 1024, RPU = 1024 / ROWB;
    int ln = lane;
    asm volatile("" : "+v"(ln));             // recomputed at each use, not held through the key loop
#pragma unroll
    for (int j = 0; j < (UNITS + 3) / 4; ++j) {
      if (4 * j + wave >= UNITS) continue;
      const int row = (4 * j + wave) * RPU + ln / CPR, c = (ln % CPR) ^ at::swz(row, CPR);
      const int key = atile(u) + min(row, an - 1);
      dma_1k(qkv + (size_t)(it.tok_off + key) * a.ldqkv + col + c * 8, dst + (4 * j + wave) * 1024);
    }
  };
  const int kcol = (a.nq + it.kvh) * HD, vcol = (a.nq + a.nkv + it.kvh) * HD;
  auto vstage = [&](int t) { return lds0 + (uint32_t)((t & 1) * TILEB); };
  auto astage = [&](int t) { return lds0 + (uint32_t)(T::AOFF + (t & 1) * TILEB); };

  // V: this thread's block (vrow, vblk) of a tile, held from its load to its conversion one step
  // later.  Lanes are dealt so that the 16 of a group write distinct 16-byte columns.
  auto vblock = [&](int &vrow, int &vblk) __attribute__((always_inline)) {
    int ln = lane;
    asm volatile("" : "+v"(ln));             // made at each use, not held through the key loop
    if constexpr (HD == 256) {
      vblk = (ln & 3) | ((ln >> 2) & 4);
      vrow = (((ln >> 2) & 3) << 2) | (ln >> 5) | ((wave & 1) << 1) | ((wave >> 1) << 4);
    } else if constexpr (HD == 128) {
      vblk = ln & 3;
      vrow = (((ln >> 2) & 3) << 2) | (ln >> 4) | ((wave & 1) << 4);
    } else {
      vblk = ln % CK;
      vrow = (ln / CK) & 31;
    }
  };
  uint32_t voff;                             // a block's scale lies at 1/16 of its code offset
  {
    int vrow, vblk;
    vblock(vrow, vblk);
    voff = (uint32_t)min(vrow, pn - 1) * rowb + vblk * 16;
  }
  i32x4 vreg = {};
  uint32_t vscale = 0;
  const bool von = 64 * wave < HD;            // waves that convert (head_dim 32: half of one)
  // bf16 of the block's words 0 .. 3, one at a time, into the V tile at dst
  auto v_dst = [&](uint32_t dst) __attribute__((always_inline)) -> uint32_t {
    int vrow, vblk;
    vblock(vrow, vblk);
    return dst + (uint32_t)(vrow * ROWB + (((4 * vblk) ^ at::swz(vrow, CPR)) << 4));
  };
  auto write_v = [&](uint32_t d, int i) __attribute__((always_inline)) {
    if (!von || (HD == 32 && half)) return;
    *reinterpret_cast<__attribute__((address_space(3))) bf16x8 *>((__attribute__((address_space(3))) uint8_t *)(size_t)(d ^ (i << 4))) =
        kv4_bf16x8((uint32_t)vreg[i], kv4_scale((uint8_t)vscale));
  };
  // K scale bytes of this lane's row (lane & 31): of its half's blocks, NCH half + c in byte c
  uint32_t ksv = 0;
  // Prefix tile t on its way: K codes to ring stage t % 3, V and the scales to registers.  Tiles are
  // fetched in order; past the last one it is fetched again, into what nothing reads, so that no
  // branch (whose joined registers would have to be waited for) stands in the key loop.
  uint32_t kring = lds0 + T::KOFF + wave * 1024;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    if (k4on && !(K4HALF && half)) dma_1k_s(kc, koff, kring);
    if (von) {
      vreg = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(tile_rsrc(vc), voff, 0, 0));
      uint32_t vo = voff;
      asm volatile("" : "+v"(vo));
      vscale = __builtin_amdgcn_raw_buffer_load_b8(tile_rsrc(vs), vo >> 4, 0, 0);
    }
    const rsrc_t p = tile_rsrc(ks);
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const uint32_t ksoff = (uint32_t)min(ln & 31, pn - 1) * srow + (CK > 1 ? (uint32_t)(ln >> 5) * NCH : 0u);
    if constexpr (CK == 8) ksv = __builtin_amdgcn_raw_buffer_load_b32(p, ksoff, 0, 0);
    else if constexpr (CK == 4) ksv = __builtin_amdgcn_raw_buffer_load_b16(p, ksoff, 0, 0);
    else ksv = __builtin_amdgcn_raw_buffer_load_b8(p, ksoff, 0, 0);
    kring = kring + T::K4TILE >= lds0 + T::KOFF + 3 * T::K4TILE ? kring - 2 * T::K4TILE : kring + T::K4TILE;
    const uint32_t rows = t + 1 >= np ? 0 : t == 0 ? pv0 : 32;
    kc += rows * rowb; vc += rows * rowb; ks += rows * srow; vs += rows * srow;
  };
  // ---- LDS operand addresses
  const int krow = lane & 31;
  // code chunk NCH half + c of the lane's row: base ^ 16 c (rows and stages are multiples of the
  // swizzled bits' span)
  const uint32_t k4base = lds0 + T::KOFF + krow * T::K4ROW + (CK == 1 ? 0 : (((NCH * half) ^ T::ksw(krow)) << 4));
  // own-key K chunk HD >= 64: 8 c + 4 half + j (a lane's elements 32 consecutive, as in the codes),
  // HD 32: 2 j + half
  const uint32_t abase = (uint32_t)(krow * ROWB + (((HD == 32 ? half : 4 * half) ^ at::swz(krow, CPR)) << 4));
  const int src16 = lane & 15, g16 = (lane >> 4) & 1;
  // source row 4 half + src16 / 4 (the pair's second 8 rows further: the swizzle's bit 1 turned)
  uint32_t vbase;
  {
    const int r = half * 4 + (src16 >> 2), sw = at::swz(r, CPR);
    const int cl = (2 * g16 + ((src16 >> 1) & 1)) ^ (sw & 3);
    vbase = (uint32_t)(r * ROWB + 16 * cl + 8 * (src16 & 1)) ^ ((uint32_t)(sw >> 2) << 6);
  }

  // ---- queries
  auto query = [&](int g) __attribute__((always_inline)) -> const bf16 * {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int loc = 32 * (wave + 4 * g) + (ln & 31);
    const int qrow = it.q0 + (loc < it.nq ? loc : 0);   // rows past the item's: its first (never stored)
    return qkv + (size_t)(it.tok_off + qrow / G) * a.ldqkv + (size_t)(it.kvh * G + qrow % G) * HD;
  };

  f32x16 o[NG][NT];
  // negative reference of the row's weights in log2 units (3e38: none yet), their sum
  float mb[NG], l_run[NG];
  // (behind the queries' conversion, volatile too: both at once need more registers than there are)
  auto clear = [&]() __attribute__((always_inline)) {
    float z;
    asm volatile("v_mov_b32 %0, 0" : "=v"(z));
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      mb[g] = 3e38f;
      l_run[g] = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[g][n][r] = z;
    }
  };

  // Softmax of one tile of scores (register r: key (r/4)*8 + 4 half + r%4) into P^T.
  // Weights are 2^(s sl2 + mb) against a reference that is the first tile's maximum and
  // moves (with O and the sum rescaled) only when a score exceeds it by 2^32 in weight: weights
  // and sums stay far from overflow, and the accumulators are left alone nearly always.
  // Keys of the tile from index n_keys on are masked.
  auto softmax = [&](f32x16 (&s)[NG], bf16x8 (&pp)[NG][2], int n_keys) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (n_keys < 32) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((r >> 2) * 8 + half * 4 + (r & 3) >= n_keys) s[g][r] = -INFINITY;
      }
      float tmax = fmaxf(s[g][0], s[g][1]);
#pragma unroll
      for (int r = 2; r < 16; ++r) tmax = fmaxf(tmax, s[g][r]);
      if (__ballot(fmaf(tmax, sl2, mb[g]) > 32.0f)) {     // also every first tile
        const float tm = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
        const bool up = fmaf(tm, sl2, mb[g]) > 32.0f;     // the halves of a query agree
        const float nb = up ? -tm * sl2 : mb[g];
        const float f = up ? __builtin_amdgcn_exp2f(nb - mb[g]) : 1.0f;
        mb[g] = nb;
        l_run[g] *= f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[g][n][r] *= f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[g][r] = __builtin_amdgcn_exp2f(fmaf(s[g][r], sl2, mb[g]));
      float ps = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
          bf16x2 p2;
          p2[0] = (bf16)s[g][8 * h + 2 * q];
          p2[1] = (bf16)s[g][8 * h + 2 * q + 1];
          ps += s[g][8 * h + 2 * q] + s[g][8 * h + 2 * q + 1];
          w[q] = __builtin_bit_cast(uint32_t, p2);
        }
        pp[g][h] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      }
      l_run[g] += ps;
    }
  };
  // O^T += V^T P^T over the V tile at vst
  auto pv_acc = [&](uint32_t vst, const bf16x8 (&pp)[NG][2]) __attribute__((always_inline)) {
    const uint32_t v0 = vst + vbase;
    auto vfrag = [&](int j) __attribute__((always_inline)) -> bf16x8 {
      const int kk = j / NT, n = j % NT, c = (n / 4) * 256 + kk * 16 * ROWB;
      uint32_t v = v0;
      if (HD == 256) asm volatile("" : "+v"(v));   // addresses made at each use: registers are short
      v ^= (uint32_t)(64 * (n % 4));
      return lds_tr_pair(lds_ptr(v) + c, lds_ptr(v ^ 32u) + c + 8 * ROWB);
    };
    constexpr int NJ = 2 * NT;
    bf16x8 fr[3];
    fr[0] = vfrag(0);
    fr[1] = vfrag(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (j + 2 < NJ) fr[(j + 2) % 3] = vfrag(j + 2);
#pragma unroll
      for (int g = 0; g < NG; ++g) o[g][j % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[j % 3], pp[g][j / NT], o[g][j % NT], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- prologue: the first tiles' copies, then the queries
  if (np > 0) {
    fetch(0);
  } else {
    copy_own(0, kcol, astage(0));
    copy_own(0, vcol, vstage(0));
  }
  if (np == 0) {
    clear();
  } else {
    u32x6 q6[NG][NCH][3];
    uint32_t qs[NG] = {};                   // byte c: the scale of product c's block, first term
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const bf16 *qp = query(g);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        bf16x8 q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          q[j] = *reinterpret_cast<const bf16x8 *>(qp + 32 * c + (HD == 32 ? 0 : 32 * NCH * half) + 8 * j);
          if (HD == 32 && half) q[j] = bf16x8{};        // a product is 64 wide
        }
        qs[g] |= split_query(q, q6[g][c]) << (8 * c);
      }
    }
    clear();
    wait_loads();
    {
      const uint32_t d = v_dst(vstage(0));
#pragma unroll
      for (int i = 0; i < 4; ++i) write_v(d, i);
    }
    uint32_t ksc = ksv;
    fetch(1);
    uint32_t kst = k4base;                  // the lane's row in the tile's ring stage
    auto key_loop = [&](auto act) __attribute__((always_inline)) {
    for (int t = 0; t < np; ++t) {
      lds_barrier();                        // tile t is in LDS; every wave is done with tile t - 1
      wait_loads();                         // K codes, V and scales of tile t + 1
      // Runs in the shadow of the last score products, where registers are free: V of tile t + 1 to
      // the other stage (behind the last tile to the own-key stage that is still free), then the
      // next copies.
      uint32_t d = 0, ksn = 0;
      auto next = [&](int c) __attribute__((always_inline)) {
        constexpr int C0 = NCH > 1 ? NCH - 2 : 0;
        if (c == C0) d = v_dst(t + 1 < np ? vstage(t + 1) : astage(t));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c == C0 + (NCH > 1 ? i / 2 : 0)) write_v(d, i);
        if (c < NCH - 1) return;
        ksn = ksv;
        fetch(t + 2);
      };
      f32x16 s[NG];
      bf16x8 pp[NG][2];
      if constexpr (act.value) {
        auto kfrag = [&](int c) __attribute__((always_inline)) -> i32x4 {
          const i32x4 k = *reinterpret_cast<const __attribute__((address_space(3))) i32x4 *>(lds_ptr(kst ^ (uint32_t)(16 * c)));
          return HD == 32 && half ? i32x4{} : k;
        };
        i32x4 kr[2];                        // codes are read one product ahead
        kr[0] = kfrag(0);
        if (NCH > 1) kr[1] = kfrag(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const i32x4 k = kr[c & 1];
          const i32x8 kf = __builtin_shufflevector(k, k, 0, 1, 2, 3, -1, -1, -1, -1);   // a 4-bit operand is 4 registers
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            auto term = [&](auto kk) __attribute__((always_inline)) {
              constexpr int K = decltype(kk)::value;
              const i32x6 x = __builtin_bit_cast(i32x6, q6[g][c][K]);
              const i32x8 qf = __builtin_shufflevector(x, x, 0, 1, 2, 3, 4, 5, -1, -1);
              uint32_t sc = qs[g];          // the terms' scales are 4 and 9 below the first's
              if (K > 0) asm volatile("" : "+v"(sc));
              sc -= K == 0 ? 0u : K == 1 ? 0x04040404u : 0x09090909u;
              const f32x16 acc = c == 0 && K == 0 ? f32x16{} : s[g];
              if (c == 0) s[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kf, qf, acc, 4, 2, 0, ksc, 0, sc);
              if (c == 1) s[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kf, qf, acc, 4, 2, 1, ksc, 1, sc);
              if (c == 2) s[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kf, qf, acc, 4, 2, 2, ksc, 2, sc);
              if (c == 3) s[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kf, qf, acc, 4, 2, 3, ksc, 3, sc);
            };
            term(std::integral_constant<int, 0>{});
            term(std::integral_constant<int, 1>{});
            term(std::integral_constant<int, 2>{});
          }
          if (c + 2 < NCH) kr[c & 1] = kfrag(c + 2);
          next(c);
          __builtin_amdgcn_sched_barrier(0);
        }
        softmax(s, pp, t == 0 ? pv0 : 32);
      }
      else {
#pragma unroll
        for (int c = 0; c < NCH; ++c) next(c);
      }
      if (t + 1 == np && na > 0) {
        copy_own(0, kcol, astage(t + 1));
        copy_own(0, vcol, vstage(t + 1));
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (act.value) pv_acc(vstage(t), pp);
      ksc = ksn;
      kst = (t + 1) % 3 == 0 ? kst - 2 * T::K4TILE : kst + T::K4TILE;
    }
    };
    if (active) key_loop(std::true_type{});
    else key_loop(std::false_type{});
  }
  // ---- the request's own keys
  if (na > 0) {
    bf16x8 qf[NG][NS];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const bf16 *qp = query(g);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        // fragment i: elements 64 (i / 4) + 32 half + 8 (i % 4) (HD 32: 16 i + 8 half)
        const int at = HD == 32 ? 16 * i + 8 * half : 64 * (i / 4) + 32 * half + 8 * (i % 4);
        qf[g][i] = *reinterpret_cast<const bf16x8 *>(qp + at);
      }
    }
    auto own_loop = [&](auto act) __attribute__((always_inline)) {
    for (int u = 0; u < na; ++u) {
      const int t = np + u;
      wait_loads();
      lds_barrier();
      f32x16 s[NG];
      bf16x8 pp[NG][2];
      if constexpr (act.value) {
        const uint32_t ab0 = astage(t) + abase;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const uint32_t x = (uint32_t)((HD == 32 ? 2 * i : 8 * (i / 4) + i % 4) << 4);
          const bf16x8 kf = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8 *>(lds_ptr(ab0 ^ x));
#pragma unroll
          for (int g = 0; g < NG; ++g)
            s[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[g][i], i == 0 ? f32x16{} : s[g], 0, 0, 0);
        }
        softmax(s, pp, u == 0 ? av0 : 32);
      }
      if (u + 1 < na) {
        copy_own(u + 1, kcol, astage(t + 1));
        copy_own(u + 1, vcol, vstage(t + 1));
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (act.value) pv_acc(vstage(t), pp);
    }
    };
    if (active) own_loop(std::true_type{});
    else own_loop(std::false_type{});
  }
  wait_loads();
  lds_barrier();                          // every wave is done with the rings

  // ---- results.  Lane: query (lane & 31) of the group; register r of tile n: element
  // 32 n + (r/4)*8 + 4 half + r%4.
  constexpr int CPRO = HD / 8;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    const float l = l_run[g] + __shfl_xor(l_run[g], 32, 64);
    const int loc = 32 * (wave + 4 * g) + (lane & 31);
    if (loc >= it.nq) continue;
    const float m2 = -mb[g];                              // log2 units
    if (it.slot >= 0) {
      const size_t pr = (size_t)it.slot * kAttnQB + loc;
      float *po = reinterpret_cast<float *>(a.part_o) + pr * HD + 4 * half;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4 *>(po + 32 * n + 8 * q) =
              make_float4(o[g][n][4 * q], o[g][n][4 * q + 1], o[g][n][4 * q + 2], o[g][n][4 * q + 3]);
      if (half == 0) *reinterpret_cast<float2 *>(a.part_ml + pr * 2) = make_float2(m2, l);
      continue;
    }
    const int qrow = it.q0 + loc;
    if (a.lse && half == 0)
      a.lse[(size_t)(it.tok_off + qrow / G) * a.nq + it.kvh * G + qrow % G] = (m2 + log2f(l)) * 0.6931471805599453f;
    // through LDS, so that whole 16-byte chunks of rows go out side by side
    const float inv = 1.0f / l;
    uint8_t *stg = smem + (wave * NG + g) * (32 * 2 * HD);
    const int q = lane & 31;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        bf16x4 v;
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = (bf16)(o[g][n][rg * 4 + x] * inv);
        const int c = (4 * n + rg) ^ (q & (CPRO - 1));
        *reinterpret_cast<bf16x4 *>(stg + q * 2 * HD + c * 16 + half * 8) = v;
      }
  }
  if (it.slot < 0) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's staging writes are done
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int base = 32 * (wave + 4 * g);
      if (base >= it.nq) continue;
      const uint8_t *stg = smem + (wave * NG + g) * (32 * 2 * HD);
      constexpr int RPI = 64 / CPRO;
#pragma unroll
      for (int i = 0; i < 32 / RPI; ++i) {
        const int r = i * RPI + lane / CPRO, c = lane % CPRO;
        if (base + r < it.nq) {
          const uint4 v = *reinterpret_cast<const uint4 *>(stg + r * 2 * HD + ((c ^ (r & (CPRO - 1))) * 16));
          const int qrow = it.q0 + base + r;
          const size_t orow = (size_t)(it.tok_off + qrow / G), ocol = (size_t)(it.kvh * G + qrow % G) * HD + c * 8;
          bf16 *dst = reinterpret_cast<bf16 *>(a.o) + (a.o_rows > 0 ? kb32_offset(a.o_rows, orow, ocol) : orow * a.ldo + ocol);
          *reinterpret_cast<uint4 *>(dst) = v;
        }
      }
    }
  }
  lds_barrier();                          // the staging reads are done before the next item's copies
  }
}

hipError_t launch_kv4_attention(const KvAttnArgs &ka, hipStream_t s) {
  const AttnArgs &a = ka.a;
  if (a.n_blocks <= 0) return hipSuccess;
  dim3 grid(a.n_blocks);
  switch (a.hd) {
    case 32: hipLaunchKernelGGL((kv4_attention_kernel<32, attn_groups_per_wave(32)>), grid, dim3(256), 0, s, ka); break;
    case 64: hipLaunchKernelGGL((kv4_attention_kernel<64, attn_groups_per_wave(64)>), grid, dim3(256), 0, s, ka); break;
    case 128: hipLaunchKernelGGL((kv4_attention_kernel<128, attn_groups_per_wave(128)>), grid, dim3(256), 0, s, ka); break;
    case 256: hipLaunchKernelGGL((kv4_attention_kernel<256, attn_groups_per_wave(256)>), grid, dim3(256), 0, s, ka); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ joining split items
// o = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c over a group's slots c, slots in order, eight in flight.  LG =
// head_dim / 4 lanes hold a query row (four elements each).  A group of few rows has many slots (one long request: 64):
// there a block's waves take every fourth slot of the same rows and are joined in order.
template <int HD>
__global__ void __launch_bounds__(256) kv4_merge_kernel(const AttnGroup *__restrict__ groups, KvAttnArgs ka) {
  __shared__ float sacc[4][64][4], sml[4][64];
  const AttnArgs &a = ka.a;
  const AttnGroup gr = groups[blockIdx.y];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int nw = gr.nq <= kAttnQB / 4 ? 4 : 1;             // waves a row
  constexpr int LG = HD / 4, RW = 64 / LG;                 // lanes a row, rows a wave
  const int G = a.nq / a.nkv, e0 = 4 * (lane & (LG - 1));
  const int qloc = (nw == 4 ? blockIdx.x : blockIdx.x * 4 + wave) * RW + lane / LG;
  if (qloc >= gr.nq) return;
  const float *po = reinterpret_cast<const float *>(a.part_o);
  const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
  // a lane's share of the slots' maxima
  float mx = -INFINITY;
  for (int c = lane & (LG - 1); c < gr.n; c += LG) mx = fmaxf(mx, ml[(size_t)(gr.first_slot + c) * kAttnQB + qloc].x);
  if constexpr (LG == 64) {
    mx = wave_max(mx);
  } else {
#pragma unroll
    for (int o = 1; o < LG; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  }
  constexpr int CH = 8;
  float L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int c0 = nw == 4 ? wave : 0; c0 < gr.n; c0 += nw * CH) {
    float2 p[CH];
    float4 v[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const bool live = c0 + nw * c < gr.n;
      const size_t r = (size_t)(gr.first_slot + (live ? c0 + nw * c : 0)) * kAttnQB + qloc;
      p[c] = live ? ml[r] : make_float2(-INFINITY, 0.f);
      v[c] = live ? *reinterpret_cast<const float4 *>(po + r * HD + e0) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const float w = exp2f(p[c].x - mx);
      if (c0 + nw * c >= gr.n) break;
      L += w * p[c].y;
      acc[0] += w * v[c].x; acc[1] += w * v[c].y; acc[2] += w * v[c].z; acc[3] += w * v[c].w;
    }
  }
  if (nw == 4) {                                           // the whole block
#pragma unroll
    for (int j = 0; j < 4; ++j) sacc[wave][lane][j] = acc[j];
    sml[wave][lane] = L;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < 4; ++w) {
      L += sml[w][lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += sacc[w][lane][j];
    }
  }
  const int qrow = gr.q0 + qloc;
  const size_t orow = (size_t)gr.tok_off + qrow / G;
  const int qg = gr.kvh * G + qrow % G;
  if (a.lse && e0 == 0) a.lse[orow * a.nq + qg] = (mx + log2f(L)) * 0.6931471805599453f;
  const float inv = 1.0f / L;
  const size_t col = (size_t)qg * HD + e0;
  bf16x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (bf16)(acc[j] * inv);
  *reinterpret_cast<bf16x4 *>(reinterpret_cast<bf16 *>(a.o) + (a.o_rows > 0 ? kb32_offset(a.o_rows, orow, col) : orow * a.ldo + col)) = r;
}

hipError_t launch_kv4_merge(const AttnGroup *groups, int n_groups, const KvAttnArgs &a, hipStream_t s) {
  if (n_groups <= 0) return hipSuccess;
  const dim3 grid(kAttnQB / 4 * a.a.hd / 256, n_groups);
  switch (a.a.hd) {
    case 32: hipLaunchKernelGGL(kv4_merge_kernel<32>, grid, dim3(256), 0, s, groups, a); break;
    case 64: hipLaunchKernelGGL(kv4_merge_kernel<64>, grid, dim3(256), 0, s, groups, a); break;
    case 128: hipLaunchKernelGGL(kv4_merge_kernel<128>, grid, dim3(256), 0, s, groups, a); break;
    case 256: hipLaunchKernelGGL(kv4_merge_kernel<256>, grid, dim3(256), 0, s, groups, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kv_attention(const KvAttnArgs &ka, const AttnGroup *groups, int n_groups, bool bf16_mode, hipStream_t s) {
  if (!bf16_mode) return launch_kv_attention_rows(ka, s);
  const AttnArgs &a = ka.a;
  if (ka.fp4) {
    const hipError_t e = launch_kv4_attention(ka, s);
    return e != hipSuccess ? e : launch_kv4_merge(groups, n_groups, ka, s);
  }
  const hipError_t e = launch_attention(a, true, s);
  if (e != hipSuccess) return e;
  // with the log-sum-exp split items leave their parts in fp32
  return a.lse ? launch_kv4_merge(groups, n_groups, ka, s)
               : launch_attn_merge(groups, n_groups, a.part_o, a.part_ml, a.o, a.ldo, a.nq, a.nkv, a.hd, true, s, a.o_rows);
}

}  // namespace rosa
