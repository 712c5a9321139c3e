// A KV cache in pages: rows appended to it (append_kernel), one generation step over it (paged_decode_kernel,
// paged_combine_kernel), and what a step in which prompts share pages needs around the attention of the shared rows
// (shared_plan_kernel; the attention itself is in pp_paged_shared.cu).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "pp_decode_tile.h"
#include "pp_device_once.h"
#include "pp_paged.h"

namespace pp {
namespace {

__device__ __forceinline__ void note_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}

// cos and sin of position * theta_j: the angle in double, reduced to [-pi, pi] as in the prefill kernels, which makes the rotated
// keys those of the prefill bit for bit.
__device__ __forceinline__ void angle(int position, double inv_freq, float& cs, float& sn) {
  const double ang = (double)position * inv_freq;
  const double n = rint(ang * 0.15915494309189535);
  double red = fma(-n, 6.283185307179586, ang);
  red = fma(-n, 2.4492935982947064e-16, red);
  sincosf((float)red, &sn, &cs);
}
__device__ __forceinline__ float turn_lo(float a, float b, float cs, float sn) { return __fmaf_rn(a, cs, -__fmul_rn(b, sn)); }
__device__ __forceinline__ float turn_hi(float a, float b, float cs, float sn) { return __fmaf_rn(b, cs, __fmul_rn(a, sn)); }

__device__ __forceinline__ float2 unpack_bf16(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ uint32_t round_bf16(float lo, float hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&x);
}
// Four numbers as e4m3 bytes, to nearest; what is beyond the largest (448) becomes it, a NaN stays one.
__device__ __forceinline__ uint32_t round_e4m3(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// ------------------------------------------------------------------------------------------
// Rows into pages
// ------------------------------------------------------------------------------------------
// A copy with a rotation in it, bound by HBM: a CTA takes as many rows as make 4096 elements of K (one 8 + 8 element pair of
// pieces per thread, two pieces of V), finds where they go, and has all of its loads under way before it needs the angles,
// which are computed once for all heads of a row.
constexpr int kAppendThreads = 256;
constexpr int kAppendMaxRows = 16;

struct AppendArgs {
  PagedCacheArgs c;
  const int32_t *prompt, *position;
  const __nv_bfloat16 *k_new, *v_new;
  int64_t k_stride, v_stride, n_rows;
  int32_t n_prompts, n_kv_heads, rows_per_cta;
  bool rotate;
  int32_t* status;
  RopeAngles angles;
};

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kAppendThreads)
append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kHalf = D / 2, kSize = kE4m3 ? 1 : 2;
  constexpr int kKUnits = kHalf / 8, kVUnits = D / 8;       // per head: pieces of 8 + 8 elements, pieces of 8 elements
  __shared__ int32_t s_pos[kAppendMaxRows];
  __shared__ int64_t s_to[kAppendMaxRows];                  // byte offset of the row (head 0) in either pool, -1: not written
  __shared__ float s_cos[kAppendMaxRows][kHalf], s_sin[kAppendMaxRows][kHalf];
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_cta;
  const int rows = (int)min((int64_t)a.rows_per_cta, a.n_rows - row0);
  pdl_launch_dependents();
  pdl_wait();
  if (tid < rows) {
    const int prompt = a.prompt[row0 + tid];
    int64_t to = -1;
    int pos = 0;
    if (prompt >= 0) {
      pos = a.position[row0 + tid];
      if (prompt >= a.n_prompts) note_status(a.status, PP_PAGED_BAD_PROMPT);
      else if (pos < 0 || (pos >> a.c.page_shift) >= a.c.table_stride) note_status(a.status, PP_PAGED_BAD_POSITION);
      else {
        const int page = a.c.table[(int64_t)prompt * a.c.table_stride + (pos >> a.c.page_shift)];
        if ((unsigned)page >= (unsigned)a.c.n_pages) note_status(a.status, PP_PAGED_BAD_PAGE);
        else to = (int64_t)page * a.c.page_stride + (int64_t)(pos & ((1 << a.c.page_shift) - 1)) * a.c.row_stride;
      }
    }
    s_pos[tid] = pos;
    s_to[tid] = to;
  }
  __syncthreads();
  const int k_units = a.n_kv_heads * kKUnits, v_units = a.n_kv_heads * kVUnits;
  const int trips = (rows * k_units + kAppendThreads - 1) / kAppendThreads;
  for (int trip = 0; trip < trips; ++trip) {
    const int u = trip * kAppendThreads + tid;
    // K: elements 8c .. and D/2 + 8c ..; V: the same number of pieces, two per thread
    const int r = u / k_units, w = u - r * k_units, head = w / kKUnits, c = w - head * kKUnits;
    const bool k_here = r < rows && s_to[r] >= 0;
    uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo, v[2] = {lo, lo};
    int vr[2], vw[2];
    bool v_here[2];
    if (k_here) {
      const __nv_bfloat16* p = a.k_new + (row0 + r) * a.k_stride + head * D + 8 * c;
      lo = load16(p);
      hi = load16(p + kHalf);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int n = trip * 2 * kAppendThreads + 2 * tid + x;      // (a thread's two pieces stand next to one another)
      vr[x] = n / v_units;
      vw[x] = n - vr[x] * v_units;
      v_here[x] = vr[x] < rows && s_to[vr[x]] >= 0;
      if (v_here[x]) v[x] = load16(a.v_new + (row0 + vr[x]) * a.v_stride + 8 * vw[x]);
    }
    if (trip == 0) {
      if (a.rotate) {
        for (int n = tid; n < rows * kHalf; n += kAppendThreads) {
          const int ar = n / kHalf, j = n - ar * kHalf;
          float cs, sn;
          angle(s_pos[ar], a.angles.inv_freq[j], cs, sn);
          s_cos[ar][j] = cs;
          s_sin[ar][j] = sn;
        }
      }
      __syncthreads();
    }
    if (k_here) {
      char* to = a.c.k_pages + s_to[r] + (int64_t)head * a.c.head_stride + 8 * c * kSize;
      if (a.rotate || kE4m3) {
        float x[8], y[8];
        const uint32_t lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 l2 = unpack_bf16(lw[e]), h2 = unpack_bf16(hw[e]);
          x[2 * e] = l2.x; x[2 * e + 1] = l2.y;
          y[2 * e] = h2.x; y[2 * e + 1] = h2.y;
        }
        if (a.rotate) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float cs = s_cos[r][8 * c + e], sn = s_sin[r][8 * c + e], p = x[e], q = y[e];
            x[e] = turn_lo(p, q, cs, sn);
            y[e] = turn_hi(p, q, cs, sn);
          }
        }
        if constexpr (kE4m3) {
          const float scale = a.c.k_scale[head];
#pragma unroll
          for (int e = 0; e < 8; ++e) { x[e] = __fdiv_rn(x[e], scale); y[e] = __fdiv_rn(y[e], scale); }
          *reinterpret_cast<uint2*>(to) = make_uint2(round_e4m3(x[0], x[1], x[2], x[3]), round_e4m3(x[4], x[5], x[6], x[7]));
          *reinterpret_cast<uint2*>(to + kHalf) = make_uint2(round_e4m3(y[0], y[1], y[2], y[3]), round_e4m3(y[4], y[5], y[6], y[7]));
        } else {
          lo = make_uint4(round_bf16(x[0], x[1]), round_bf16(x[2], x[3]), round_bf16(x[4], x[5]), round_bf16(x[6], x[7]));
          hi = make_uint4(round_bf16(y[0], y[1]), round_bf16(y[2], y[3]), round_bf16(y[4], y[5]), round_bf16(y[6], y[7]));
        }
      }
      if constexpr (!kE4m3) {
        *reinterpret_cast<uint4*>(to) = lo;
        *reinterpret_cast<uint4*>(to + kHalf * kSize) = hi;
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (!v_here[x]) continue;
      const int vh = vw[x] / kVUnits, vc = vw[x] - vh * kVUnits;
      char* to = a.c.v_pages + s_to[vr[x]] + (int64_t)vh * a.c.head_stride + 8 * vc * kSize;
      if constexpr (kE4m3) {
        const float scale = a.c.v_scale[vh];
        const uint32_t w4[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
        float e[8];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const float2 f = unpack_bf16(w4[n]);
          e[2 * n] = __fdiv_rn(f.x, scale);
          e[2 * n + 1] = __fdiv_rn(f.y, scale);
        }
        *reinterpret_cast<uint2*>(to) = make_uint2(round_e4m3(e[0], e[1], e[2], e[3]), round_e4m3(e[4], e[5], e[6], e[7]));
      } else {
        *reinterpret_cast<uint4*>(to) = v[x];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// One generation step
// ------------------------------------------------------------------------------------------
// Work: a prompt's rows are cut into chunks of equal size, a whole number of 64-row blocks, such that all prompts together
// make about kChunksWanted (chunk, KV head) pieces; persistent CTAs take them in turn. The lengths live on the device, so every
// CTA sums them itself (one or two loads per thread, two passes of the block), and the grid and the room for partial results
// depend on k and the heads alone: sum of ceil(blocks_i / C) <= kChunksWanted / Hkv + k with C the block count that
// divides all blocks into kChunksWanted / Hkv.
constexpr int kPagedThreads = 128;
constexpr int kPagedWarps = kPagedThreads / 32;
constexpr int kMaxGroup = 8;            // query heads per KV head: the N of the tensor-core product
constexpr int kStepKeys = 16;           // keys per warp and step
constexpr int kBlockKeys = kStepKeys * kPagedWarps;
constexpr int kChunksWanted = kSms * 3 * 4;

struct PagedArgs {
  PagedCacheArgs c;
  const int32_t* lengths;
  const int32_t* own_start;             // rows before it are read by the kernel of the shared rows; null: none are
  const __nv_bfloat16 *q_new, *k_new, *v_new;
  int64_t q_stride, k_stride, v_stride;
  __nv_bfloat16* o;
  int32_t* chunk_ptr;                   // [k + 1], left by CTA 0 for the kernel that joins the chunks
  float2* part_ml;                      // [chunk][Hq]
  float* part_o;                        // [chunk][Hq][D]
  int32_t n_prompts, n_q_heads, n_kv_heads, group, chunks_wanted;
  float scale_log2;
  int32_t* status;
  RopeAngles angles;
};

// Rows that the pages hold for prompt i before the step; -1 for a row of no prompt, and for a length that its table row has no room for.
__device__ __forceinline__ int checked_length(const PagedCacheArgs& c, const int32_t* lengths, int i, bool fresh, int32_t* status) {
  const int len = lengths[i];
  const int64_t room = (int64_t)c.table_stride << c.page_shift;
  if (len + (int64_t)fresh > room) {
    note_status(status, PP_PAGED_BAD_LENGTH);
    return -1;
  }
  return max(len, -1);
}

// Sum over the block's threads; every thread gets it. (Two barriers.)
template <int kThreads>
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* s_warp) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = x;
  __syncthreads();
  int64_t sum = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) sum += s_warp[w];
  __syncthreads();
  return sum;
}
// Exclusive prefix sum over the block's threads.
template <int kThreads>
__device__ __forceinline__ int64_t block_prefix(int64_t x, int64_t* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 31) s_warp[warp] = sum;
  __syncthreads();
  int64_t before = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w)
    if (w < warp) before += s_warp[w];
  __syncthreads();
  return before + sum - x;
}

// Blocks per chunk; s_ptr[0 .. k]: first chunk of every prompt. A prompt without rows of its own has one chunk all the same, in
// which its output is written; a row of no prompt has none.
__device__ __forceinline__ int cut_into_chunks(const PagedArgs& a, int32_t* s_ptr, int64_t* s_warp) {
  const int k = a.n_prompts, tid = threadIdx.x;
  const bool fresh = a.k_new != nullptr;
  const int each = (k + kPagedThreads - 1) / kPagedThreads, i0 = min(tid * each, k), i1 = min(i0 + each, k);
  int32_t* status = blockIdx.x == 0 ? a.status : nullptr;
  int64_t blocks = 0;
  for (int i = i0; i < i1; ++i) {
    const int len = checked_length(a.c, a.lengths, i, fresh, status);
    const int n = len < 0 ? -1 : (len - (a.own_start ? a.own_start[i] : 0) + kBlockKeys - 1) / kBlockKeys;
    s_ptr[i] = n;
    blocks += max(n, 0);
  }
  const int64_t total = block_sum<kPagedThreads>(blocks, s_warp);
  const int chunk_blocks = (int)max((total + a.chunks_wanted - 1) / a.chunks_wanted, (int64_t)1);
  int64_t mine = 0;
  for (int i = i0; i < i1; ++i) {
    const int n = s_ptr[i];
    const int chunks = n < 0 ? 0 : max((n + chunk_blocks - 1) / chunk_blocks, 1);
    s_ptr[i] = chunks;
    mine += chunks;
  }
  int at = (int)block_prefix<kPagedThreads>(mine, s_warp);
  for (int i = i0; i < i1; ++i) {
    const int chunks = s_ptr[i];
    s_ptr[i] = at;
    at += chunks;
  }
  if (tid == kPagedThreads - 1) s_ptr[k] = at;
  __syncthreads();
  return chunk_blocks;
}

// 16 keys of a warp in e4m3: K rows g and g + 8, 16-byte pieces t, t + 4 of a row (D = 64: piece t); V rows 2t, 2t + 1, 2t + 8,
// 2t + 9, the g-th eighth of a row. The numbers are multiplied as f16, which holds every e4m3 number.
template <int D>
struct StepK8 { uint4 r[2][D / 64]; };
template <int D>
struct StepV8 { uint32_t r[4][D / 32]; };

__device__ __forceinline__ void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The two e4m3 numbers in the lower (upper) half of a word as f16, in the same order.
__device__ __forceinline__ uint32_t f16_of_e4m3_lo(uint32_t x) {
  uint32_t y;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t f16_of_e4m3_hi(uint32_t x) {
  uint32_t y;
  asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(y) : "r"(x));
  return y;
}

// What differs between pages of bf16 and of e4m3: how a step's rows are loaded and multiplied.
template <int D, bool kE4m3>
struct Rows;

template <int D>
struct Rows<D, false> {
  using K = StepK<D>;
  using V = StepV<D>;
  // Row pitch of the queries in shared memory, in 16-bit elements: rows 64 bytes apart modulo 128 serve the 8 lanes of a
  // 16-byte access without conflicts
  static constexpr int kPitch = D + 32;
  static constexpr int kQ = D / 32;                   // 16-byte pieces of a query that a thread meets
  static constexpr float kWeight = 1.f;
  static __device__ __forceinline__ void load_k(K& f, const char* p, int64_t row_stride, int g, int t) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        f.r[x][i] = load16(reinterpret_cast<const __nv_bfloat16*>(p + (g + 8 * x) * row_stride) + 8 * t + 32 * i);
  }
  static __device__ __forceinline__ void load_v(V& f, const char* p, int64_t row_stride, int g, int t) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        f.r[x][i] = load16(reinterpret_cast<const __nv_bfloat16*>(p + (2 * t + (x & 1) + 8 * (x >> 1)) * row_stride) + 8 * g + 64 * i);
  }
  // the new token's rows, from shared memory, as a step with one real key
  static __device__ __forceinline__ void one_row(K& fk, V& fv, const uint8_t* k_row, const uint8_t* v_row, int g, int t) {
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      fk.r[0][i] = g == 0 ? *reinterpret_cast<const uint4*>(k_row + 16 * t + 64 * i) : none;
      fk.r[1][i] = none;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < D / 64; ++i) fv.r[x][i] = x == 0 && t == 0 ? *reinterpret_cast<const uint4*>(v_row + 16 * g + 128 * i) : none;
  }
  // piece i of query `row` that this thread's K pieces meet
  static __device__ __forceinline__ uint4 q_piece(const uint16_t* q, int t, int i) { return *reinterpret_cast<const uint4*>(q + 8 * t + 32 * i); }
  static __device__ __forceinline__ void scores(float (&c)[4], const K& f, const uint4 (&q)[kQ], const uint16_t* q_low, int t) {
    c[0] = c[1] = c[2] = c[3] = 0.f;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const uint4 l = q_piece(q_low, t, i);
      mma16816(c, f.r[0][i].x, f.r[1][i].x, f.r[0][i].y, f.r[1][i].y, l.x, l.y);
      mma16816(c, f.r[0][i].z, f.r[1][i].z, f.r[0][i].w, f.r[1][i].w, l.z, l.w);
    }
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      mma16816(c, f.r[0][i].x, f.r[1][i].x, f.r[0][i].y, f.r[1][i].y, q[i].x, q[i].y);
      mma16816(c, f.r[0][i].z, f.r[1][i].z, f.r[0][i].w, f.r[1][i].w, q[i].z, q[i].w);
    }
  }
  static __device__ __forceinline__ void clear(V& f, int n_real, int t) { clear_past<D>(f, n_real, t); }
  static __device__ __forceinline__ void product(Softmax<D>& s, const V& f, const float (&p)[4]) { pv<D>(s, f, p); }
  // element of O that acc[j][0], acc[j][1] (x = 0) and acc[j][2], acc[j][3] (x = 1) stand for
  static __device__ __forceinline__ int element(int j, int x, int g) { return D == 128 ? 64 * x + 8 * g + j : 8 * g + 4 * x + j; }
  // the two 16-bit parts of a pair of query elements
  static __device__ __forceinline__ uint32_t high(float a, float b) { return round_bf16(a, b); }
  static __device__ __forceinline__ uint32_t low(float a, float b, uint32_t h) {
    const float2 f = unpack_bf16(h);
    // (an infinite element has no lower part)
    return round_bf16(isfinite(f.x) ? a - f.x : 0.f, isfinite(f.y) ? b - f.y : 0.f);
  }
};

template <int D>
struct Rows<D, true> {
  using K = StepK8<D>;
  using V = StepV8<D>;
  static constexpr int kPitch = D + 8;                // rows 16 bytes apart modulo 128, pieces of a thread 32
  static constexpr int kQ = D / 32;
  // Weights are at most 1 and multiplied in two f16 parts, which end at 2^-24: times 2^15 they reach down to 2^-39 of the
  // largest, so that the sum of 2^17 of the smallest is still below 2^-22 of it.
  static constexpr float kWeight = 32768.f;
  static __device__ __forceinline__ void load_k(K& f, const char* p, int64_t row_stride, int g, int t) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        f.r[x][i] = load16(reinterpret_cast<const __nv_bfloat16*>(p + (g + 8 * x) * row_stride + 16 * t + 64 * i));
  }
  static __device__ __forceinline__ void load_v(V& f, const char* p, int64_t row_stride, int g, int t) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const char* row = p + (2 * t + (x & 1) + 8 * (x >> 1)) * row_stride + (D / 8) * g;
      if constexpr (D == 128)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(f.r[x][0]), "=r"(f.r[x][1]), "=r"(f.r[x][2]), "=r"(f.r[x][3]) : "l"(row));
      else
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(f.r[x][0]), "=r"(f.r[x][1]) : "l"(row));
    }
  }
  static __device__ __forceinline__ void one_row(K& fk, V& fv, const uint8_t* k_row, const uint8_t* v_row, int g, int t) {
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      fk.r[0][i] = g == 0 ? *reinterpret_cast<const uint4*>(k_row + 16 * t + 64 * i) : none;
      fk.r[1][i] = none;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        fv.r[x][i] = x == 0 && t == 0 ? *reinterpret_cast<const uint32_t*>(v_row + (D / 8) * g + 4 * i) : 0u;
  }
  static __device__ __forceinline__ uint4 q_piece(const uint16_t* q, int t, int i) {
    return *reinterpret_cast<const uint4*>(q + 16 * t + 64 * (i >> 1) + 8 * (i & 1));
  }
  static __device__ __forceinline__ void scores(float (&c)[4], const K& f, const uint4 (&q)[kQ], const uint16_t* q_low, int t) {
    c[0] = c[1] = c[2] = c[3] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {        // four elements of a row in each word of the piece
        const uint32_t r0 = word_of(f.r[0][i], w), r1 = word_of(f.r[1][i], w);
        const uint32_t a0 = f16_of_e4m3_lo(r0), a1 = f16_of_e4m3_lo(r1), a2 = f16_of_e4m3_hi(r0), a3 = f16_of_e4m3_hi(r1);
        const uint4 h = q[2 * i + (w >> 1)], l = q_piece(q_low, t, 2 * i + (w >> 1));
        mma16816_f16(c, a0, a1, a2, a3, (w & 1) ? l.z : l.x, (w & 1) ? l.w : l.y);
        mma16816_f16(c, a0, a1, a2, a3, (w & 1) ? h.z : h.x, (w & 1) ? h.w : h.y);
      }
  }
  static __device__ __forceinline__ void clear(V& f, int n_real, int t) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (2 * t + (x & 1) + 8 * (x >> 1) >= n_real) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) f.r[x][i] = 0u;
      }
  }
  // O^T += V^T P. Product j: row g is d = (D / 8) g + 2j, row g + 8 the element after it.
  static __device__ __forceinline__ void product(Softmax<D>& s, const V& f, const float (&p)[4]) {
    uint32_t b[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float p0 = p[2 * x] * kWeight, p1 = p[2 * x + 1] * kWeight;
      const __half2 h = __floats2half2_rn(p0, p1);
      const float2 back = __half22float2(h);
      const __half2 l = __floats2half2_rn(p0 - back.x, p1 - back.y);
      b[0][x] = transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
      b[1][x] = transpose8x8(*reinterpret_cast<const uint32_t*>(&l));
    }
#pragma unroll
    for (int w = 0; w < D / 32; ++w)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int j = 2 * w + y;
        const uint32_t k0 = __byte_perm(f.r[0][w], f.r[1][w], y ? 0x7362 : 0x5140), k1 = __byte_perm(f.r[2][w], f.r[3][w], y ? 0x7362 : 0x5140);
        const uint32_t a0 = f16_of_e4m3_lo(k0), a1 = f16_of_e4m3_hi(k0), a2 = f16_of_e4m3_lo(k1), a3 = f16_of_e4m3_hi(k1);
        mma16816_f16(s.acc[j], a0, a1, a2, a3, b[1][0], b[1][1]);
        mma16816_f16(s.acc[j], a0, a1, a2, a3, b[0][0], b[0][1]);
      }
  }
  static __device__ __forceinline__ int element(int j, int x, int g) { return (D / 8) * g + 2 * j + x; }
  static __device__ __forceinline__ uint32_t high(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t low(float a, float b, uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    const __half2 l = __floats2half2_rn(isfinite(f.x) ? a - f.x : 0.f, isfinite(f.y) ? b - f.y : 0.f);
    return *reinterpret_cast<const uint32_t*>(&l);
  }
};

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kPagedThreads, D == 128 ? 3 : 4)
paged_decode_kernel(const __grid_constant__ PagedArgs a) {
  using R = Rows<D, kE4m3>;
  constexpr int kHalf = D / 2, kSize = kE4m3 ? 1 : 2;
  extern __shared__ int32_t s_ptr[];                                       // [k + 1]
  __shared__ int64_t s_warp[kPagedWarps];
  __shared__ float s_cos[kHalf], s_sin[kHalf];
  __shared__ __align__(16) uint16_t s_q[2][kMaxGroup][R::kPitch];          // rotated queries, upper and lower part
  __shared__ __align__(16) uint8_t s_new[2][D * kSize];                    // the new token's rows of the pages
  __shared__ float s_scale[kMaxGroup];                                     // to scaled log2 units
  __shared__ float s_m[kPagedWarps][kMaxGroup], s_l[kPagedWarps][kMaxGroup];
  __shared__ float s_o[kPagedWarps][kMaxGroup][D];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const bool fresh = a.k_new != nullptr;
  pdl_wait();                           // lengths, table, pages: all may come from the kernel before
  pdl_launch_dependents();
  const int chunk_blocks = cut_into_chunks(a, s_ptr, s_warp);
  const int n_chunks_all = s_ptr[a.n_prompts];
  if (blockIdx.x == 0)
    for (int i = tid; i <= a.n_prompts; i += kPagedThreads) a.chunk_ptr[i] = s_ptr[i];

  const int64_t n_work = (int64_t)n_chunks_all * a.n_kv_heads;
  for (int64_t work = blockIdx.x; work < n_work; work += gridDim.x) {
    const int chunk = (int)(work / a.n_kv_heads), kvh = (int)(work - (int64_t)chunk * a.n_kv_heads);
    int lo = 0, hi = a.n_prompts - 1;   // last prompt whose first chunk is <= chunk (the prompts without any come before it)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_ptr[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    const int i = lo, c0 = s_ptr[i], n_chunks = s_ptr[i + 1] - c0, len = a.lengths[i];
    const int start = a.own_start ? a.own_start[i] : 0;
    const int64_t chunk_keys = (int64_t)chunk_blocks * kBlockKeys;
    const int key0 = (int)min(start + (chunk - c0) * chunk_keys, (int64_t)len), key_end = (int)min(key0 + chunk_keys, (int64_t)len);
    const bool last_chunk = chunk - c0 == n_chunks - 1;
    const int32_t* table = a.c.table + (int64_t)i * a.c.table_stride;
    const int64_t head_at = (int64_t)kvh * a.c.head_stride;
    // Pages of this warp's steps (key0 + 16 * (warp + 4n)), 32 at a time, one per lane.
    const int first = key0 + kStepKeys * warp;
    auto page_ids = [&](int n0) {
      const int64_t key = first + (int64_t)(n0 + lane) * kBlockKeys;
      int id = 0;
      if (key < key_end) {
        id = table[key >> a.c.page_shift];
        if ((unsigned)id >= (unsigned)a.c.n_pages) {
          note_status(a.status, PP_PAGED_BAD_PAGE);
          id = 0;
        }
      }
      return id;
    };
    int ids = page_ids(0), ids_next = 0;
    const int row_mask = (1 << a.c.page_shift) - 1;
    auto offset = [&](int n, int key) {
      return (int64_t)__shfl_sync(0xffffffffu, ids, n & 31) * a.c.page_stride + head_at + (int64_t)(key & row_mask) * a.c.row_stride;
    };

    // queries of the group and the new key, four (j, j + D/2) pairs at a time, zeros for absent heads
    constexpr int kUnits = kHalf / 4, kRotUnits = (kMaxGroup + 1) * kUnits, kTrips = (kRotUnits + kPagedThreads - 1) / kPagedThreads;
    uint2 lo2[kTrips], hi2[kTrips];
#pragma unroll
    for (int x = 0; x < kTrips; ++x) {
      const int u = tid + x * kPagedThreads, h = u / kUnits, j = 4 * (u - h * kUnits);
      lo2[x] = hi2[x] = make_uint2(0u, 0u);
      if (h < a.group || (h == kMaxGroup && last_chunk && fresh)) {
        const __nv_bfloat16* src = h == kMaxGroup ? a.k_new + (int64_t)i * a.k_stride + kvh * D
                                                  : a.q_new + (int64_t)i * a.q_stride + (kvh * a.group + h) * D;
        lo2[x] = *reinterpret_cast<const uint2*>(src + j);
        hi2[x] = *reinterpret_cast<const uint2*>(src + j + kHalf);
      }
    }
    uint2 v_mine = make_uint2(0u, 0u);
    const bool v_here = last_chunk && fresh && tid < D / 4;
    if (v_here) v_mine = *reinterpret_cast<const uint2*>(a.v_new + (int64_t)i * a.v_stride + kvh * D + 4 * tid);
    typename R::K fk;
    typename R::V fv;
    int key = first, n = 0;
    if (key < key_end) {
      const int64_t at = offset(0, key);
      R::load_k(fk, a.c.k_pages + at, a.c.row_stride, g, t);
      R::load_v(fv, a.c.v_pages + at, a.c.row_stride, g, t);
    }
    if (tid < kHalf) angle(fresh ? len : max(len - 1, 0), a.angles.inv_freq[tid], s_cos[tid], s_sin[tid]);
    __syncthreads();
    const float k_scale = kE4m3 ? a.c.k_scale[kvh] : 1.f, v_scale = kE4m3 ? a.c.v_scale[kvh] : 1.f;
#pragma unroll
    for (int x = 0; x < kTrips; ++x) {
      const int u = tid + x * kPagedThreads, h = u / kUnits, j = 4 * (u - h * kUnits);
      float p[4], y[4];
      {
        const float2 p0 = unpack_bf16(lo2[x].x), p1 = unpack_bf16(lo2[x].y), y0 = unpack_bf16(hi2[x].x), y1 = unpack_bf16(hi2[x].y);
        p[0] = p0.x; p[1] = p0.y; p[2] = p1.x; p[3] = p1.y;
        y[0] = y0.x; y[1] = y0.y; y[2] = y1.x; y[3] = y1.y;
      }
      int shift = 0;
      if constexpr (kE4m3) {
        // f16 has 5 exponent bits: a query is brought to below 2 by a power of two, which goes into its factor
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(p[e]), fabsf(y[e])));
#pragma unroll
        for (int o = kUnits / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (top > 0.f && top < INFINITY) shift = ilogbf(top) + 1;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float cs = s_cos[j + e], sn = s_sin[j + e], pe = p[e], ye = y[e];
        p[e] = turn_lo(pe, ye, cs, sn);
        y[e] = turn_hi(pe, ye, cs, sn);
      }
      if (h < kMaxGroup) {
        if constexpr (kE4m3) {
#pragma unroll
          for (int e = 0; e < 4; ++e) { p[e] = scalbnf(p[e], -shift); y[e] = scalbnf(y[e], -shift); }
        }
        if (j == 0) s_scale[h] = scalbnf(a.scale_log2 * k_scale, shift);
        const uint32_t ph[2] = {R::high(p[0], p[1]), R::high(p[2], p[3])}, yh[2] = {R::high(y[0], y[1]), R::high(y[2], y[3])};
        *reinterpret_cast<uint2*>(&s_q[0][h][j]) = make_uint2(ph[0], ph[1]);
        *reinterpret_cast<uint2*>(&s_q[0][h][j + kHalf]) = make_uint2(yh[0], yh[1]);
        *reinterpret_cast<uint2*>(&s_q[1][h][j]) = make_uint2(R::low(p[0], p[1], ph[0]), R::low(p[2], p[3], ph[1]));
        *reinterpret_cast<uint2*>(&s_q[1][h][j + kHalf]) = make_uint2(R::low(y[0], y[1], yh[0]), R::low(y[2], y[3], yh[1]));
      } else if (h == kMaxGroup) {
        if constexpr (kE4m3) {
#pragma unroll
          for (int e = 0; e < 4; ++e) { p[e] = __fdiv_rn(p[e], k_scale); y[e] = __fdiv_rn(y[e], k_scale); }
          *reinterpret_cast<uint32_t*>(&s_new[0][j]) = round_e4m3(p[0], p[1], p[2], p[3]);
          *reinterpret_cast<uint32_t*>(&s_new[0][j + kHalf]) = round_e4m3(y[0], y[1], y[2], y[3]);
        } else {
          *reinterpret_cast<uint2*>(&s_new[0][2 * j]) = make_uint2(round_bf16(p[0], p[1]), round_bf16(p[2], p[3]));
          *reinterpret_cast<uint2*>(&s_new[0][2 * (j + kHalf)]) = make_uint2(round_bf16(y[0], y[1]), round_bf16(y[2], y[3]));
        }
      }
    }
    if (v_here) {
      if constexpr (kE4m3) {
        const float2 x = unpack_bf16(v_mine.x), y = unpack_bf16(v_mine.y);
        *reinterpret_cast<uint32_t*>(&s_new[1][4 * tid]) = round_e4m3(__fdiv_rn(x.x, v_scale), __fdiv_rn(x.y, v_scale), __fdiv_rn(y.x, v_scale), __fdiv_rn(y.y, v_scale));
      } else {
        *reinterpret_cast<uint2*>(&s_new[1][8 * tid]) = v_mine;
      }
    }
    __syncthreads();
    uint4 q[R::kQ];
#pragma unroll
    for (int x = 0; x < R::kQ; ++x) q[x] = R::q_piece(s_q[0][g], t, x);
    const uint16_t* q_low = s_q[1][g];
    const float scale[2] = {s_scale[2 * t], s_scale[2 * t + 1]};

    Softmax<D> s;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int x = 0; x < 4; ++x) s.acc[j][x] = 0.f;
    float c[4];
    // K of the next step is loaded as soon as the scores of this one are there, V after its product.
    while (key < key_end) {
      R::scores(c, fk, q, q_low, t);
      const int next = key + kBlockKeys;
      const bool more = next < key_end;
      int64_t at = 0;
      if (more) {
        ++n;
        if ((n & 31) == 16) ids_next = page_ids((n & ~31) + 32);
        if ((n & 31) == 0) ids = ids_next;
        at = offset(n, next);
        R::load_k(fk, a.c.k_pages + at, a.c.row_stride, g, t);
      }
      softmax_step<D>(s, c, scale, key_end - key, g);
      if (key_end - key < kStepKeys) R::clear(fv, key_end - key, t);
      R::product(s, fv, c);
      if (more) R::load_v(fv, a.c.v_pages + at, a.c.row_stride, g, t);
      key = next;
    }
    if (last_chunk && fresh && warp == 0) {        // the new token, and its rows of the pages
      R::one_row(fk, fv, s_new[0], s_new[1], g, t);
      R::scores(c, fk, q, q_low, t);
      softmax_step<D>(s, c, scale, 1, g);
      R::product(s, fv, c);
      const int page = table[len >> a.c.page_shift];
      if ((unsigned)page < (unsigned)a.c.n_pages) {
        const int64_t at = (int64_t)page * a.c.page_stride + head_at + (int64_t)(len & row_mask) * a.c.row_stride;
        if (lane < D * kSize / 16) {
          *reinterpret_cast<uint4*>(a.c.k_pages + at + 16 * lane) = *reinterpret_cast<const uint4*>(&s_new[0][16 * lane]);
          *reinterpret_cast<uint4*>(a.c.v_pages + at + 16 * lane) = *reinterpret_cast<const uint4*>(&s_new[1][16 * lane]);
        }
      } else if (lane == 0) {
        note_status(a.status, PP_PAGED_BAD_PAGE);
      }
    }
    // merge the four warps (one without keys has m = kNoScore, l = 0)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float l = s.l[h];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      const int head = 2 * t + h;
      if (head < a.group) {
        if (g == 0) { s_m[warp][head] = s.m[h]; s_l[warp][head] = l; }
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x) s_o[warp][head][R::element(j, x, g)] = s.acc[j][2 * x + h];
      }
    }
    __syncthreads();
    const float out_scale = v_scale / R::kWeight;
    for (int u = tid; u < a.group * D; u += kPagedThreads) {
      const int h = u / D, d = u - h * D;
      float mm = s_m[0][h];
#pragma unroll
      for (int w = 1; w < kPagedWarps; ++w) mm = fmaxf(mm, s_m[w][h]);
      float ll = 0.f, oo = 0.f;
#pragma unroll
      for (int w = 0; w < kPagedWarps; ++w) {
        const float f = ex2(s_m[w][h] - mm);
        ll += s_l[w][h] * f;
        oo += s_o[w][h][d] * f;
      }
      oo *= out_scale;
      const int head = kvh * a.group + h;
      if (n_chunks == 1 && !a.own_start) {
        // (a row that attends to nothing is 0; one all of whose scores are -inf is a NaN)
        a.o[((int64_t)i * a.n_q_heads + head) * D + d] = __float2bfloat16_rn(len + (int)fresh > 0 ? oo / ll : 0.f);
      } else {
        const int64_t at = (int64_t)chunk * a.n_q_heads + head;
        if (d == 0) a.part_ml[at] = make_float2(mm, ll);
        a.part_o[at * D + d] = oo;
      }
    }
    __syncthreads();
  }
}

// Joins the parts of every (prompt, query head): the chunks of the prompt's own rows and, with a plan, the pieces of the
// shared ones. kAcross = false: one warp for a head, four heads in a CTA. true: four warps for a head, for few (prompt,
// head) pairs, of which one may have hundreds of parts.
template <int D, bool kAcross>
__global__ void __launch_bounds__(kPagedThreads)
paged_combine_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ SharedPlan plan) {
  constexpr int E = D / 32;             // consecutive elements per lane
  __shared__ float s_m[kPagedWarps], s_l[kPagedWarps], s_o[kPagedWarps][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = blockIdx.x, head = kAcross ? blockIdx.y : blockIdx.y * kPagedWarps + warp;
  const bool fresh = a.k_new != nullptr;
  pdl_wait();                           // the partial results come from the kernels before this one
  pdl_launch_dependents();
  if (!kAcross && head >= a.n_q_heads) return;
  const int c0 = a.chunk_ptr[i], n_own = a.chunk_ptr[i + 1] - c0;
  if (n_own == 0 || (n_own == 1 && !a.own_start)) return;      // a row of no prompt; one whose O is complete
  const int len = a.lengths[i];
  const float2* ml_own = a.part_ml + (int64_t)c0 * a.n_q_heads + head;
  const float* o_own = a.part_o + ((int64_t)c0 * a.n_q_heads + head) * D;
  const float2* ml_shared = nullptr;
  const float* o_shared = nullptr;
  int n_shared = 0;
  if (a.own_start) {
    const int gr = plan.group_of[i], tiles = gr >= 0 ? plan.key_tiles[gr] : 0;
    if (tiles > 0) {
      const int first = plan.group_ptr[gr], rows = (plan.group_ptr[gr + 1] - first) * a.group;
      const int kvh = head / a.group, row = (i - first) * a.group + head - kvh * a.group, rt = row / kSharedTileRows;
      const int64_t per = units_per_piece(*plan.units, plan.n_ctas);
      const int64_t u0 = plan.unit_start[gr] + ((int64_t)kvh * ((rows + kSharedTileRows - 1) / kSharedTileRows) + rt) * tiles;
      const int p0 = (int)(u0 / per);
      n_shared = (int)((u0 + tiles - 1) / per) - p0 + 1;
      const int64_t at = (int64_t)p0 * kSharedTileRows + ((int64_t)(first - plan.group_ptr[0]) * a.n_kv_heads * a.group) + (int64_t)kvh * rows + row;
      ml_shared = plan.ml + at;
      o_shared = plan.o + at * D;
    }
  }
  float mm = kNoScore, ll = 0.f, oo[E];
#pragma unroll
  for (int e = 0; e < E; ++e) oo[e] = 0.f;
  const int n_all = n_own + n_shared, step = kAcross ? kPagedWarps : 1;
  for (int base = kAcross ? warp : 0; base < n_all; base += 32 * step) {      // 32 parts at a time: one (m, l) per lane
    const int n = min(32, (n_all - base + step - 1) / step), mine = base + lane * step;
    float2 ml = make_float2(kNoScore, 0.f);
    if (lane < n) ml = mine < n_own ? ml_own[(int64_t)mine * a.n_q_heads] : ml_shared[(int64_t)(mine - n_own) * kSharedTileRows];
    float m_new = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m_new = fmaxf(m_new, __shfl_xor_sync(0xffffffffu, m_new, o));
    m_new = fmaxf(mm, m_new);
    const float alpha = ex2(mm - m_new), f = ex2(ml.x - m_new);
    mm = m_new;
    float l = ml.y * f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    ll = ll * alpha + l;
#pragma unroll
    for (int e = 0; e < E; ++e) oo[e] *= alpha;
#pragma unroll 8
    for (int c = 0; c < n; ++c) {
      const float fc = __shfl_sync(0xffffffffu, f, c);
      const int part = base + c * step;
      const float* src = (part < n_own ? o_own + (int64_t)part * a.n_q_heads * D : o_shared + (int64_t)(part - n_own) * kSharedTileRows * D) + E * lane;
      float p[E];
      if constexpr (E == 4) {
        const float4 x = *reinterpret_cast<const float4*>(src);
        p[0] = x.x; p[1] = x.y; p[2] = x.z; p[3] = x.w;
      } else {
        const float2 x = *reinterpret_cast<const float2*>(src);
        p[0] = x.x; p[1] = x.y;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) oo[e] += p[e] * fc;
    }
  }
  if constexpr (kAcross) {
    if (lane == 0) { s_m[warp] = mm; s_l[warp] = ll; }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][E * lane + e] = oo[e];
    __syncthreads();
    if (warp != 0) return;
    mm = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    ll = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) oo[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedWarps; ++w) {
      const float f = ex2(s_m[w] - mm);
      ll += s_l[w] * f;
#pragma unroll
      for (int e = 0; e < E; ++e) oo[e] += s_o[w][E * lane + e] * f;
    }
  }
  uint32_t r[E / 2];
  const bool none = len + (int)fresh <= 0;
#pragma unroll
  for (int e = 0; e < E / 2; ++e) r[e] = none ? 0u : round_bf16(oo[2 * e] / ll, oo[2 * e + 1] / ll);
  __nv_bfloat16* dst = a.o + ((int64_t)i * a.n_q_heads + head) * D + E * lane;
  if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(r[0], r[1]);
  else *reinterpret_cast<uint32_t*>(dst) = r[0];
}

// ------------------------------------------------------------------------------------------
// Plan of a step with shared rows
// ------------------------------------------------------------------------------------------
// CTA i < k rotates the queries of prompt i into the rows that the tensor cores read. The last CTA lays the work out: how many
// rows each group really shares (no more than its shortest prompt has, whole pages), and the line of units.
constexpr int kPlanThreads = 512;
struct PlanArgs {
  PagedArgs a;
  SharedPlan plan;
  const int32_t* shared_len;
};

template <int D>
__global__ void __launch_bounds__(kPlanThreads)
shared_plan_kernel(const __grid_constant__ PlanArgs p) {
  const PagedArgs& a = p.a;
  const SharedPlan& plan = p.plan;
  const int tid = threadIdx.x, k = a.n_prompts;
  const bool fresh = a.k_new != nullptr;
  pdl_wait();
  pdl_launch_dependents();
  if ((int)blockIdx.x < k) {
    constexpr int kHalf = D / 2, kUnits = kHalf / 4;
    __shared__ float s_cos[kHalf], s_sin[kHalf];
    const int i = blockIdx.x, len = a.lengths[i];
    if (len < 0) return;                // (its rows of the tiles hold what they held: nothing of them is read)
    if (tid < kHalf) angle(fresh ? len : max(len - 1, 0), a.angles.inv_freq[tid], s_cos[tid], s_sin[tid]);
    __syncthreads();
    for (int u = tid; u < a.n_q_heads * kUnits; u += kPlanThreads) {
      const int h = u / kUnits, j = 4 * (u - h * kUnits), kvh = h / a.group;
      const __nv_bfloat16* src = a.q_new + (int64_t)i * a.q_stride + (int64_t)h * D + j;
      __nv_bfloat16* dst = plan.q_rot + (((int64_t)kvh * k + i) * a.group + h - kvh * a.group) * D + j;
      const uint2 lo = *reinterpret_cast<const uint2*>(src), hi = *reinterpret_cast<const uint2*>(src + kHalf);
      const float2 p0 = unpack_bf16(lo.x), p1 = unpack_bf16(lo.y), y0 = unpack_bf16(hi.x), y1 = unpack_bf16(hi.y);
      const float x[4] = {p0.x, p0.y, p1.x, p1.y}, y[4] = {y0.x, y0.y, y1.x, y1.y};
      float rx[4], ry[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        rx[e] = turn_lo(x[e], y[e], s_cos[j + e], s_sin[j + e]);
        ry[e] = turn_hi(x[e], y[e], s_cos[j + e], s_sin[j + e]);
      }
      *reinterpret_cast<uint2*>(dst) = make_uint2(round_bf16(rx[0], rx[1]), round_bf16(rx[2], rx[3]));
      *reinterpret_cast<uint2*>(dst + kHalf) = make_uint2(round_bf16(ry[0], ry[1]), round_bf16(ry[2], ry[3]));
    }
    return;
  }
  extern __shared__ int32_t s_plan[];   // group_ptr [n_groups + 1], the rows shared [n_groups], the first prompt of each group
  __shared__ int64_t s_warp[kPlanThreads / 32];
  __shared__ int s_bad;
  const int n = plan.n_groups;
  int32_t *s_ptr = s_plan, *s_rows = s_plan + n + 1, *s_lead = s_rows + n;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int g = tid; g <= n; g += kPlanThreads) {
    const int at = plan.group_ptr[g], before = g ? plan.group_ptr[g - 1] : 0;
    if (at < before || at < 0 || at > k) s_bad = 1;
    s_ptr[g] = at;
    if (g < n) {
      s_rows[g] = max(p.shared_len[g], 0);
      s_lead[g] = k;
    }
  }
  __syncthreads();
  const bool bad = s_bad != 0;
  if (bad && tid == 0) note_status(a.status, PP_PAGED_BAD_GROUPS);
  auto group_of = [&](int i) {
    if (bad || i < s_ptr[0] || i >= s_ptr[n]) return -1;
    int lo = 0, hi = n - 1;             // last group that begins at or before i (the empty ones come before it)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_ptr[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
  };
  for (int i = tid; i < k; i += kPlanThreads) {
    const int g = group_of(i), len = checked_length(a.c, a.lengths, i, fresh, nullptr);
    plan.group_of[i] = g;
    if (g >= 0 && len >= 0) {
      atomicMin(&s_rows[g], len);
      atomicMin(&s_lead[g], i);
    }
  }
  __syncthreads();
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int each = (n + kPlanThreads - 1) / kPlanThreads, g0 = min(tid * each, n), g1 = min(g0 + each, n);
  int64_t units = 0;
  for (int g = g0; g < g1; ++g) {
    const int prompts = bad ? 0 : s_ptr[g + 1] - s_ptr[g];
    const int rows = prompts > 0 && s_lead[g] < k ? s_rows[g] & ~page_mask : 0;      // (a group may be all rows of no prompt)
    s_rows[g] = rows;
    const int tiles = (rows + kSharedTileKeys - 1) / kSharedTileKeys;
    units += (int64_t)tiles * ((prompts * a.group + kSharedTileRows - 1) / kSharedTileRows) * a.n_kv_heads;
  }
  int64_t at = block_prefix<kPlanThreads>(units, s_warp);
  for (int g = g0; g < g1; ++g) {
    const int prompts = bad ? 0 : s_ptr[g + 1] - s_ptr[g], tiles = (s_rows[g] + kSharedTileKeys - 1) / kSharedTileKeys;
    plan.unit_start[g] = at;
    plan.key_tiles[g] = tiles;
    plan.shared_rows[g] = s_rows[g];
    plan.lead[g] = s_lead[g];
    at += (int64_t)tiles * ((prompts * a.group + kSharedTileRows - 1) / kSharedTileRows) * a.n_kv_heads;
  }
  if (tid == kPlanThreads - 1) {        // (the last thread's share ends the line, also where it is empty)
    plan.unit_start[n] = at;
    *plan.units = at;
  }
  __syncthreads();
  for (int i = tid; i < k; i += kPlanThreads) {
    const int g = group_of(i);
    plan.own_start[i] = g >= 0 && a.lengths[i] >= 0 ? s_rows[g] : 0;
  }
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------
int check_paged_device() {
  static thread_local int cached_dev = -1, cached = PP_OK;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return note_cuda_error((int)e, "cudaGetDevice");
  if (dev != cached_dev) {
    int major = 0;
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e != cudaSuccess) return note_cuda_error((int)e, "compute capability");
    cached = major == 10 ? PP_OK : PP_ERR_UNSUPPORTED;
    cached_dev = dev;
  }
  return cached;
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_heads(const pp_attn_params* p, bool queries) {
  if (!p || p->n_kv_heads < 1 || (queries && p->n_q_heads < 1)) return PP_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return PP_ERR_UNSUPPORTED;
  if (p->n_kv_heads > 65535) return PP_ERR_UNSUPPORTED;
  if (queries) {
    if (p->n_q_heads % p->n_kv_heads != 0 || p->n_q_heads / p->n_kv_heads > kMaxGroup || p->n_q_heads > 65535) return PP_ERR_UNSUPPORTED;
    if (p->softmax_scale < 0.f || !(p->softmax_scale <= 3.4e38f)) return PP_ERR_INVALID_ARG;
  }
  if (!(p->rope_base > 0.f)) return PP_ERR_INVALID_ARG;
  return PP_OK;
}

int check_cache(const pp_attn_params& p, const pp_paged_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table) return PP_ERR_INVALID_ARG;
  if (c->type != PP_CACHE_BF16 && c->type != PP_CACHE_E4M3) return PP_ERR_UNSUPPORTED;
  if (c->type == PP_CACHE_E4M3 && (!c->k_scale || !c->v_scale)) return PP_ERR_INVALID_ARG;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return PP_ERR_UNSUPPORTED;
  if (c->n_pages < 1 || c->table_stride < 1) return PP_ERR_INVALID_ARG;
  if ((int64_t)c->table_stride * c->page_size > (int64_t(1) << 30)) return PP_ERR_UNSUPPORTED;     // rows are counted in 32 bits
  const int64_t piece = c->type == PP_CACHE_E4M3 ? 16 : 8;
  for (int64_t s : {c->page_stride, c->head_stride, c->row_stride}) {
    if (s < p.head_dim) return PP_ERR_INVALID_ARG;
    if (s % piece != 0) return PP_ERR_ALIGNMENT;
    if (s > (int64_t(1) << 38)) return PP_ERR_UNSUPPORTED;
  }
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16)) return PP_ERR_ALIGNMENT;
  if (!aligned(c->page_table, 4) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return PP_ERR_ALIGNMENT;
  return PP_OK;
}

// A row stride as given (0: dense) in elements, or an error.
int row_stride(int64_t given, int64_t dense, int64_t* out) {
  *out = given ? given : dense;
  if (*out < dense) return PP_ERR_INVALID_ARG;
  return *out % 8 ? PP_ERR_ALIGNMENT : PP_OK;
}

template <int D, bool kE4m3>
cudaError_t launch_paged_decode(const PagedArgs& a, int grid, size_t smem, cudaStream_t s) {
  static DeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(paged_decode_kernel<D, kE4m3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxPagedPrompts + 1) * (int)sizeof(int32_t));
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  return launch_dependent(paged_decode_kernel<D, kE4m3>, dim3(grid), dim3(kPagedThreads), smem, s, a);
}

template <int D>
cudaError_t launch_plan(const PlanArgs& p, cudaStream_t s) {
  static DeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(shared_plan_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kMaxPagedPrompts + 1) * (int)sizeof(int32_t));
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  return launch_dependent(shared_plan_kernel<D>, dim3(p.a.n_prompts + 1), dim3(kPlanThreads), (3 * (size_t)p.plan.n_groups + 1) * sizeof(int32_t), s, p);
}

int decode_step(const pp_attn_params* params, const pp_paged_cache* cache, const int32_t* lengths, int32_t k, const int32_t* group_ptr,
                const int32_t* shared_len, int32_t n_groups, const void* q_new, int64_t q_stride, const void* k_new, int64_t k_stride,
                const void* v_new, int64_t v_stride, void* o, void* workspace, size_t workspace_bytes, int32_t* device_status, void* stream) {
  int st = check_heads(params, true);
  if (st != PP_OK) return st;
  if (params->flags != 0) return PP_ERR_INVALID_ARG;
  if ((st = check_cache(*params, cache)) != PP_OK) return st;
  if (!lengths || k < 1 || !q_new || !o || !workspace || (k_new == nullptr) != (v_new == nullptr)) return PP_ERR_INVALID_ARG;
  if (n_groups > k) return PP_ERR_INVALID_ARG;
  if (n_groups > 0 && cache->type != PP_CACHE_BF16) return PP_ERR_UNSUPPORTED;
  if (k > kMaxPagedPrompts) return PP_ERR_TOO_LARGE;
  PagedArgs a;
  const int64_t d = params->head_dim;
  if ((st = row_stride(q_stride, params->n_q_heads * d, &a.q_stride)) != PP_OK) return st;
  if ((st = row_stride(k_stride, params->n_kv_heads * d, &a.k_stride)) != PP_OK) return st;
  if ((st = row_stride(v_stride, params->n_kv_heads * d, &a.v_stride)) != PP_OK) return st;
  if (!aligned(q_new, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(o, 16) || !aligned(workspace, 256) || !aligned(lengths, 4) ||
      !aligned(group_ptr, 4) || !aligned(shared_len, 4) || !aligned(device_status, 4))
    return PP_ERR_ALIGNMENT;
  const PagedWorkspace L = paged_workspace(*params, k, n_groups);
  if (workspace_bytes < L.total) return PP_ERR_BUFFER_TOO_SMALL;
  if ((st = check_paged_device()) != PP_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  a.c = paged_cache_args(*cache);
  a.lengths = lengths;
  a.own_start = n_groups > 0 ? reinterpret_cast<const int32_t*>(ws + L.own_start) : nullptr;
  a.q_new = static_cast<const __nv_bfloat16*>(q_new);
  a.k_new = static_cast<const __nv_bfloat16*>(k_new);
  a.v_new = static_cast<const __nv_bfloat16*>(v_new);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.chunk_ptr = reinterpret_cast<int32_t*>(ws + L.chunk_ptr);
  a.part_ml = reinterpret_cast<float2*>(ws + L.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + L.part_o);
  a.n_prompts = k;
  a.n_q_heads = params->n_q_heads;
  a.n_kv_heads = params->n_kv_heads;
  a.group = params->n_q_heads / params->n_kv_heads;
  a.chunks_wanted = L.chunks_wanted;
  const float scale = params->softmax_scale > 0.f ? params->softmax_scale : 1.0f / sqrtf((float)params->head_dim);
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = device_status;
  a.angles = rope_angles(params->rope_base, params->head_dim);
  SharedPlan plan = {};
  if (n_groups > 0) {
    plan.units = reinterpret_cast<int64_t*>(ws + L.units);
    plan.unit_start = reinterpret_cast<int64_t*>(ws + L.unit_start);
    plan.key_tiles = reinterpret_cast<int32_t*>(ws + L.key_tiles);
    plan.shared_rows = reinterpret_cast<int32_t*>(ws + L.shared_rows);
    plan.lead = reinterpret_cast<int32_t*>(ws + L.lead);
    plan.own_start = reinterpret_cast<int32_t*>(ws + L.own_start);
    plan.group_of = reinterpret_cast<int32_t*>(ws + L.group_of);
    plan.q_rot = reinterpret_cast<__nv_bfloat16*>(ws + L.q_rot);
    plan.ml = reinterpret_cast<float2*>(ws + L.shared_ml);
    plan.o = reinterpret_cast<float*>(ws + L.shared_o);
    plan.group_ptr = group_ptr;
    plan.n_groups = n_groups;
    plan.n_ctas = kSms;
    PlanArgs p{a, plan, shared_len};
    const cudaError_t e = d == 128 ? launch_plan<128>(p, s) : launch_plan<64>(p, s);
    if (e != cudaSuccess) return note_cuda_error((int)e, "plan kernel launch");
    if ((st = launch_shared_attention(*params, a.c, plan, k, a.scale_log2, device_status, s)) != PP_OK) return st;
  }
  // three CTAs per SM (four at D = 64), or as many as there can be chunks
  const int64_t most_blocks = std::max<int64_t>(((int64_t)cache->table_stride * cache->page_size + kBlockKeys - 1) / kBlockKeys, 1);
  const int64_t most = std::min<int64_t>((int64_t)k * most_blocks, (int64_t)L.chunks_wanted + k) * params->n_kv_heads;
  const int grid = (int)std::min<int64_t>(most, kSms * (d == 128 ? 3 : 4));
  const size_t smem = ((size_t)k + 1) * sizeof(int32_t);
  const bool e4m3 = cache->type == PP_CACHE_E4M3;
  cudaError_t e = d == 128 ? (e4m3 ? launch_paged_decode<128, true>(a, grid, smem, s) : launch_paged_decode<128, false>(a, grid, smem, s))
                           : (e4m3 ? launch_paged_decode<64, true>(a, grid, smem, s) : launch_paged_decode<64, false>(a, grid, smem, s));
  if (e != cudaSuccess) return note_cuda_error((int)e, "paged generation step launch");
  if (n_groups == 0 && most_blocks == 1) return PP_OK;         // no prompt can have two chunks
  // four warps for a head as long as all of them run at once
  if ((int64_t)k * params->n_q_heads <= kSms * 16) {
    const dim3 heads((unsigned)k, (unsigned)params->n_q_heads);
    e = d == 128 ? launch_dependent(paged_combine_kernel<128, true>, heads, dim3(kPagedThreads), 0, s, a, plan)
                 : launch_dependent(paged_combine_kernel<64, true>, heads, dim3(kPagedThreads), 0, s, a, plan);
  } else {
    const dim3 heads((unsigned)k, (unsigned)((params->n_q_heads + kPagedWarps - 1) / kPagedWarps));
    e = d == 128 ? launch_dependent(paged_combine_kernel<128, false>, heads, dim3(kPagedThreads), 0, s, a, plan)
                 : launch_dependent(paged_combine_kernel<64, false>, heads, dim3(kPagedThreads), 0, s, a, plan);
  }
  return e == cudaSuccess ? PP_OK : note_cuda_error((int)e, "paged combine launch");
}

}  // namespace

RopeAngles rope_angles(float base, int32_t head_dim) {
  RopeAngles r;
  for (int j = 0; j < 64; ++j) r.inv_freq[j] = j < head_dim / 2 ? pow((double)base, -2.0 * j / (double)head_dim) : 0.0;
  return r;
}

PagedWorkspace paged_workspace(const pp_attn_params& p, int32_t k, int32_t n_groups) {
  PagedWorkspace L = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) & ~size_t(255);
    return here;
  };
  L.chunks_wanted = std::max(kChunksWanted / p.n_kv_heads, 1);
  const size_t parts = ((size_t)L.chunks_wanted + k) * p.n_q_heads;
  L.chunk_ptr = take(((size_t)k + 1) * sizeof(int32_t));
  L.part_ml = take(parts * sizeof(float2));
  L.part_o = take(parts * p.head_dim * sizeof(float));
  if (n_groups > 0) {
    L.units = take(sizeof(int64_t));
    L.unit_start = take(((size_t)n_groups + 1) * sizeof(int64_t));
    L.key_tiles = take((size_t)n_groups * sizeof(int32_t));
    L.shared_rows = take((size_t)n_groups * sizeof(int32_t));
    L.lead = take((size_t)n_groups * sizeof(int32_t));
    L.own_start = take((size_t)k * sizeof(int32_t));
    L.group_of = take((size_t)k * sizeof(int32_t));
    L.q_rot = take((size_t)k * p.n_q_heads * p.head_dim * sizeof(__nv_bfloat16));
    const size_t rows = (size_t)kSms * kSharedTileRows + (size_t)k * p.n_q_heads;
    L.shared_ml = take(rows * sizeof(float2));
    L.shared_o = take(rows * p.head_dim * sizeof(float));
  }
  L.total = at;
  return L;
}

}  // namespace pp

extern "C" int pp_paged_append(const pp_attn_params* params, const pp_paged_cache* cache, const int32_t* prompt, const int32_t* position,
                               int64_t n_rows, int32_t n_prompts, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                               int32_t* device_status, void* stream) {
  int st = pp::check_heads(params, false);
  if (st != PP_OK) return st;
  if (params->flags & ~PP_FLAG_SKIP_ROPE) return PP_ERR_INVALID_ARG;
  if ((st = pp::check_cache(*params, cache)) != PP_OK) return st;
  if (n_rows < 0 || n_prompts < 1) return PP_ERR_INVALID_ARG;
  if (n_rows > 0 && (!prompt || !position || !k_new || !v_new)) return PP_ERR_INVALID_ARG;
  pp::AppendArgs a;
  const int64_t dense = (int64_t)params->n_kv_heads * params->head_dim;
  if ((st = pp::row_stride(k_stride, dense, &a.k_stride)) != PP_OK) return st;
  if ((st = pp::row_stride(v_stride, dense, &a.v_stride)) != PP_OK) return st;
  if (!pp::aligned(k_new, 16) || !pp::aligned(v_new, 16) || !pp::aligned(prompt, 4) || !pp::aligned(position, 4) || !pp::aligned(device_status, 4))
    return PP_ERR_ALIGNMENT;
  if (n_rows == 0) return PP_OK;
  a.rows_per_cta = (int32_t)std::min<int64_t>(std::max<int64_t>(4096 / dense, 1), pp::kAppendMaxRows);
  const int64_t grid = (n_rows + a.rows_per_cta - 1) / a.rows_per_cta;
  if (grid > INT32_MAX) return PP_ERR_UNSUPPORTED;
  if ((st = pp::check_paged_device()) != PP_OK) return st;
  a.c = pp::paged_cache_args(*cache);
  a.prompt = prompt;
  a.position = position;
  a.k_new = static_cast<const __nv_bfloat16*>(k_new);
  a.v_new = static_cast<const __nv_bfloat16*>(v_new);
  a.n_rows = n_rows;
  a.n_prompts = n_prompts;
  a.n_kv_heads = params->n_kv_heads;
  a.rotate = !(params->flags & PP_FLAG_SKIP_ROPE);
  a.status = device_status;
  a.angles = pp::rope_angles(params->rope_base, params->head_dim);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool e4m3 = cache->type == PP_CACHE_E4M3;
  auto launch = [&](auto kernel) { return pp::launch_dependent(kernel, dim3((unsigned)grid), dim3(pp::kAppendThreads), 0, s, a); };
  const cudaError_t e = params->head_dim == 128 ? (e4m3 ? launch(pp::append_kernel<128, true>) : launch(pp::append_kernel<128, false>))
                                                : (e4m3 ? launch(pp::append_kernel<64, true>) : launch(pp::append_kernel<64, false>));
  return e == cudaSuccess ? PP_OK : pp::note_cuda_error((int)e, "append kernel launch");
}

extern "C" size_t pp_paged_decode_workspace_bytes(const pp_attn_params* params, int32_t k, int32_t n_groups) {
  if (pp::check_heads(params, true) != PP_OK || k < 1 || k > pp::kMaxPagedPrompts || n_groups < 0 || n_groups > k) return 0;
  return pp::paged_workspace(*params, k, n_groups).total;
}

extern "C" int pp_paged_decode_step(const pp_attn_params* params, const pp_paged_cache* cache, const int32_t* lengths, int32_t k,
                                    const void* q_new, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new,
                                    int64_t v_stride, void* o, void* workspace, size_t workspace_bytes, int32_t* device_status, void* stream) {
  return pp::decode_step(params, cache, lengths, k, nullptr, nullptr, 0, q_new, q_stride, k_new, k_stride, v_new, v_stride, o, workspace,
                         workspace_bytes, device_status, stream);
}

extern "C" int pp_paged_decode_shared(const pp_attn_params* params, const pp_paged_cache* cache, const int32_t* lengths, int32_t k,
                                      const int32_t* group_ptr, const int32_t* shared_len, int32_t n_groups, const void* q_new, int64_t q_stride,
                                      const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, void* o, void* workspace,
                                      size_t workspace_bytes, int32_t* device_status, void* stream) {
  if (!group_ptr || !shared_len || n_groups < 1) return PP_ERR_INVALID_ARG;
  return pp::decode_step(params, cache, lengths, k, group_ptr, shared_len, n_groups, q_new, q_stride, k_new, k_stride, v_new, v_stride, o, workspace,
                         workspace_bytes, device_status, stream);
}
