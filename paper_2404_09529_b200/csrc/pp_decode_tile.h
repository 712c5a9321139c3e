// Pieces of the generation step that the kernels over contiguous caches and over pages share: 16 keys of a warp against
// 8 query heads on mma.m16n8k16, with the online softmax between the two products.
#ifndef PREPACK_B200_PP_DECODE_TILE_H_
#define PREPACK_B200_PP_DECODE_TILE_H_

#include <cuda_bf16.h>

#include <cfloat>
#include <cstdint>

namespace pp {
namespace {

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 transpose of 16-bit elements across the warp
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Read once, so not kept in L1. And, like all tensors here, not through the read-only path: this kernel may have started before
// the one in front of it has written them (the rows it appends to the caches, the new token).
__device__ __forceinline__ uint4 load16(const __nv_bfloat16* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Fragments of one 16-key step of a warp. Lane = 4 g + t. K: rows g and g + 8, 16-byte pieces t, t + 4, ...
// of a row. V: rows 2t, 2t + 1, 2t + 8, 2t + 9, the 16-byte piece g of a row (and, at D = 128, piece g + 8).
template <int D>
struct StepK { uint4 r[2][D / 32]; };
template <int D>
struct StepV { uint4 r[4][D / 64]; };

// A maximum over nothing. Finite, so that a score of -inf (a key with an infinite element) weighs nothing beside it.
constexpr float kNoScore = -FLT_MAX;

// The rows past the last real one are copies of it, whose weight is 0: no part of O, not as 0 times an infinity either.
template <int D>
__device__ __forceinline__ void clear_past(StepV<D>& f, int n_real, int t) {
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (2 * t + (x & 1) + 8 * (x >> 1) >= n_real) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) f.r[x][i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

template <int D>
struct Softmax {
  float m[2] = {kNoScore, kNoScore};      // running maximum of query heads 2t and 2t + 1 (all lanes of equal t agree)
  float l[2] = {0.f, 0.f};                // this thread's keys' share of the running sum
  float acc[D / 16][4];                   // O^T: product j, rows d (see pv), columns = heads 2t, 2t + 1
};

// Online softmax over the 16 keys (those at or past n_real are hidden); leaves P in c. scale: of heads 2t and 2t + 1, the factor
// to log2 units in it.
template <int D>
__device__ __forceinline__ void softmax_step(Softmax<D>& s, float (&c)[4], const float (&scale)[2], int n_real, int g) {
#pragma unroll
  for (int x = 0; x < 4; ++x) c[x] = g + 8 * (x >> 1) < n_real ? c[x] * scale[x & 1] : -INFINITY;
  float mx[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    mx[h] = fmaxf(c[h], c[2 + h]);
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], o));
  }
  if (__any_sync(0xffffffffu, mx[0] > s.m[0] || mx[1] > s.m[1])) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float m_new = fmaxf(s.m[h], mx[h]);
      const float alpha = ex2(s.m[h] - m_new);           // 0 on the first step
      s.m[h] = m_new;
      s.l[h] *= alpha;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) { s.acc[j][h] *= alpha; s.acc[j][2 + h] *= alpha; }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    c[h] = ex2(c[h] - s.m[h]);
    c[2 + h] = ex2(c[2 + h] - s.m[h]);
    s.l[h] += c[h] + c[2 + h];
  }
}

// (a, b) cut to bf16, a in the low half.
__device__ __forceinline__ uint32_t truncate_bf16x2(float a, float b) {
  uint32_t y;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(b), "f"(a));
  return y;
}

// O^T += V^T P. Product j: row g is d = 8g + j, row g + 8 is d = 64 + 8g + j (D = 128) or 8g + 4 + j (D = 64).
template <int D>
__device__ __forceinline__ void pv(Softmax<D>& s, const StepV<D>& f, const float (&p)[4]) {
  // P in three parts of 8 bits, cut and not rounded, so that none is negative, and none of a weight above 0 (which is at least
  // 2^-126) is 0: an infinite value then gives an infinity and not a NaN, a finite one up to 2^-125 of itself too much.
  uint32_t b[3][2];
  float r[4] = {p[0], p[1], p[2], p[3]};
  uint32_t least[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) least[x] = (p[2 * x] > 0.f ? 0x0080u : 0u) | (p[2 * x + 1] > 0.f ? 0x00800000u : 0u);
#pragma unroll
  for (int part = 0; part < 3; ++part)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t cut = truncate_bf16x2(r[2 * x], r[2 * x + 1]);
      const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&cut);
      const __nv_bfloat162 w = part == 0 ? v : __hmax2_nan(v, *reinterpret_cast<const __nv_bfloat162*>(&least[x]));
      b[part][x] = transpose8x8(*reinterpret_cast<const uint32_t*>(&w));
      const float2 back = __bfloat1622float2(v);
      r[2 * x] -= back.x;
      r[2 * x + 1] -= back.y;
    }
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    uint32_t a[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {      // a0: row g, keys 2t, 2t + 1; a1: row g + 8; a2, a3: the same for keys 2t + 8, 2t + 9
      const int e = (D == 128) ? j : j + 4 * (x & 1), piece = (D == 128) ? (x & 1) : 0;
      const uint32_t k0 = word_of(f.r[2 * (x >> 1)][piece], e >> 1), k1 = word_of(f.r[2 * (x >> 1) + 1][piece], e >> 1);
      a[x] = __byte_perm(k0, k1, (e & 1) ? 0x7632 : 0x5410);
    }
#pragma unroll
    for (int part = 2; part >= 0; --part) mma16816(s.acc[j], a[0], a[1], a[2], a[3], b[part][0], b[part][1]);
  }
}

}  // namespace
}  // namespace pp

#endif  // PREPACK_B200_PP_DECODE_TILE_H_
