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
#include "pp_tcgen05.h"

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
// Those of four neighbouring elements, one after another: the code of a sine is long, and instructions have to be fetched too.
__device__ __forceinline__ void angles4(int position, const double* inv_freq, float (&cs)[4], float (&sn)[4]) {
#pragma unroll 1
  for (int e = 0; e < 4; ++e) {
    float c, s;
    angle(position, inv_freq[e], c, s);
    cs[0] = cs[1]; cs[1] = cs[2]; cs[2] = cs[3]; cs[3] = c;
    sn[0] = sn[1]; sn[1] = sn[2]; sn[2] = sn[3]; sn[3] = s;
  }
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
// A copy with a rotation in it, bound by HBM: a CTA takes as many rows (or heads of one) as make 2048 elements of K. A thread has one pair of 8-element
// pieces of K (c and D/2 + c) and two pieces of V of the same row, so that all it needs is that row's prompt and position:
// its loads, the page's number and the angles (once for all heads of a row, through shared memory) are then under way together.
// 17 554 rows of 32 heads of 128 take 89 us (6.5 TB/s; 114 with the row's place found first and handed round), 44 k short rows of
// 8 heads of 64 into 8 bits 33 us (4.1 TB/s, was 55), where instructions count: 430 a thread, a quarter of them for the angle, and as
// many for the conversions.
constexpr int kAppendThreads = 128;
constexpr int kAppendElements = 16 * kAppendThreads;        // of K in a CTA: several rows, or some heads of one
constexpr int kAppendMaxRows = 16;

struct AppendArgs {
  PagedCacheArgs c;
  const int32_t *prompt, *position;
  const __nv_bfloat16 *k_new, *v_new;
  int64_t k_stride, v_stride, n_rows;
  int32_t n_prompts, n_kv_heads, rows_per_cta, heads_per_cta;
  bool rotate;
  int32_t* status;
  RopeAngles angles;
};

__device__ __forceinline__ void widen8(const uint4& x, float (&f)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 y = unpack_bf16(w[e]);
    f[2 * e] = y.x;
    f[2 * e + 1] = y.y;
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&f)[8]) {
  return make_uint4(round_bf16(f[0], f[1]), round_bf16(f[2], f[3]), round_bf16(f[4], f[5]), round_bf16(f[6], f[7]));
}
__device__ __forceinline__ uint2 narrow8(const float (&f)[8], float per_scale) {
  return make_uint2(round_e4m3(f[0] * per_scale, f[1] * per_scale, f[2] * per_scale, f[3] * per_scale),
                    round_e4m3(f[4] * per_scale, f[5] * per_scale, f[6] * per_scale, f[7] * per_scale));
}

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kAppendThreads, kE4m3 ? 8 : 10)
append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kHalf = D / 2, kSize = kE4m3 ? 1 : 2, kUnits = kHalf / 8;      // pairs of pieces per head
  __shared__ __align__(16) float s_cos[kAppendMaxRows][kHalf], s_sin[kAppendMaxRows][kHalf];
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_cta;
  const int rows = (int)min((int64_t)a.rows_per_cta, a.n_rows - row0), head0 = blockIdx.y * a.heads_per_cta;
  const int units = min(a.heads_per_cta, a.n_kv_heads - head0) * kUnits;
  pdl_launch_dependents();
  pdl_wait();
  for (int u0 = 0; u0 < rows * units; u0 += kAppendThreads) {
    const int u = u0 + tid, r = u / units, w = u - r * units + head0 * kUnits, head = w / kUnits, c = 8 * (w - head * kUnits);
    int prompt = -1, pos = 0;
    if (r < rows) {
      prompt = a.prompt[row0 + r];
      pos = a.position[row0 + r];
    }
    if (prompt >= a.n_prompts) {
      if (w == 0) note_status(a.status, PP_PAGED_BAD_PROMPT);
      prompt = -1;
    }
    if (prompt >= 0 && (pos < 0 || (pos >> a.c.page_shift) >= a.c.table_stride)) {
      if (w == 0) note_status(a.status, PP_PAGED_BAD_POSITION);
      prompt = -1;
    }
    int page = 0;
    uint4 lo, hi, v[2];
    if (prompt >= 0) {
      page = a.c.table[(int64_t)prompt * a.c.table_stride + (pos >> a.c.page_shift)];
      const __nv_bfloat16 *k = a.k_new + (row0 + r) * a.k_stride + head * D + c, *vs = a.v_new + (row0 + r) * a.v_stride + 16 * w;
      lo = load16(k);
      hi = load16(k + kHalf);
      v[0] = load16(vs);
      v[1] = load16(vs + 8);
    }
    if (u0 == 0) {
      if (a.rotate) {
        for (int n = tid; n < rows * kHalf; n += kAppendThreads) {
          const int ar = n / kHalf, j = n - ar * kHalf;
          angle(a.position[row0 + ar], a.angles.inv_freq[j], s_cos[ar][j], s_sin[ar][j]);
        }
      }
      __syncthreads();
    }
    if (prompt < 0) continue;
    if ((unsigned)page >= (unsigned)a.c.n_pages) {
      if (w == 0) note_status(a.status, PP_PAGED_BAD_PAGE);
      continue;
    }
    const int64_t to = (int64_t)page * a.c.page_stride + (int64_t)(pos & ((1 << a.c.page_shift) - 1)) * a.c.row_stride;
    const int v_head = 16 * w / D, v_at = 16 * w - v_head * D;
    char *k_to = a.c.k_pages + to + (int64_t)head * a.c.head_stride + c * kSize, *v_to = a.c.v_pages + to + (int64_t)v_head * a.c.head_stride + v_at * kSize;
    if (a.rotate || kE4m3) {
      float x[8], y[8];
      widen8(lo, x);
      widen8(hi, y);
      if (a.rotate) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const float4 c4 = *reinterpret_cast<const float4*>(&s_cos[r][c + e]), s4 = *reinterpret_cast<const float4*>(&s_sin[r][c + e]);
          const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float p = x[e + n], q = y[e + n];
            x[e + n] = turn_lo(p, q, cs[n], sn[n]);
            y[e + n] = turn_hi(p, q, cs[n], sn[n]);
          }
        }
      }
      if constexpr (kE4m3) {
        const float per_scale = __frcp_rn(a.c.k_scale[head]);
        *reinterpret_cast<uint2*>(k_to) = narrow8(x, per_scale);
        *reinterpret_cast<uint2*>(k_to + kHalf) = narrow8(y, per_scale);
      } else {
        lo = narrow8(x);
        hi = narrow8(y);
      }
    }
    if constexpr (kE4m3) {
      const float per_scale = __frcp_rn(a.c.v_scale[v_head]);
      float x[8], y[8];
      widen8(v[0], x);
      widen8(v[1], y);
      const uint2 p = narrow8(x, per_scale), q = narrow8(y, per_scale);
      *reinterpret_cast<uint4*>(v_to) = make_uint4(p.x, p.y, q.x, q.y);
    } else {
      *reinterpret_cast<uint4*>(k_to) = lo;
      *reinterpret_cast<uint4*>(k_to + kHalf * kSize) = hi;
      *reinterpret_cast<uint4*>(v_to) = v[0];
      *reinterpret_cast<uint4*>(v_to + 16) = v[1];
    }
  }
}

// ------------------------------------------------------------------------------------------
// One generation step
// ------------------------------------------------------------------------------------------
// Bound: HBM, every row of K and V is read once. The work is a line of units of 8 KB (16, 32 or 64 rows of K and V of one KV
// head), ordered by (prompt, KV head, rows), and cut into equal pieces, one for each warp that the GPU holds: all warps read the
// same number of bytes whatever the lengths are. A warp works on its own from there on. Its rows arrive by TMA in a ring of
// two units in shared memory, whose loads run ahead over the ends of items. Six warps (seven over 8-bit pages, which take more
// instructions a byte) keep up to 96 KB of an SM under way, which is all that HBM takes: with twelve, the loads queued up and SMs
// were served so unevenly that of 148 equal shares the last ended 20 % after the mean. A piece that is a whole item (prompt, KV head) leaves O at once; of an item that is cut the parts (m, l, o) are joined by
// paged_combine_kernel.
// The arithmetic is that of the step over contiguous caches (pp_decode.cu): mma.m16n8k16 with 16 keys as rows and the query heads
// of a KV head as the 8 columns, absent heads 0. Over bf16 pages a query and a weight each reach it as the sum of two
// 16-bit numbers: HBM leaves the tensor cores idle, and scores and O are then exact to 2^-16, far below O's last rounding of 2^-8.
// The lengths live on the device: every CTA sums them itself, and the grid and the room for parts depend on neither them nor k.
constexpr int kMaxGroup = 8;            // query heads per KV head: the N of the tensor-core product
constexpr int kMostStepWarps = 7, kMostPieces = kSms * kMostStepWarps;
constexpr int kHalfUnit = 4096;         // bytes of K, and of V, in a unit
constexpr int kScratch = 2304;          // per warp: queries, the new token's rows, O on its way out
constexpr int kCombineThreads = 256;
// The running maximum of a row moves only when a score exceeds it by more than 2^kLazyLog2: until then no lane has to ask the
// others (three exchanges for each of two heads). Sums are at most 2^kLazyLog2 as large, which costs fp32 nothing.
constexpr float kLazyLog2 = 4.f;
enum WaitCode { kWaitRows = 41 };

struct PagedArgs {
  PagedCacheArgs c;
  const int32_t* lengths;
  const int2* own;                      // .x: rows before it are read by the kernel of the shared rows; null: none are
  const __nv_bfloat16 *q_new, *k_new, *v_new;
  int64_t q_stride, k_stride, v_stride;
  __nv_bfloat16* o;
  int4* cut;                            // [pieces]: of the item that begins in a piece and ends in another: prompt, KV head, pieces; 0 pieces: none
  float2* part_ml;                      // [2 pieces][group]
  float* part_o;                        // [2 pieces][group][D]
  int32_t n_prompts, n_q_heads, n_kv_heads, group;
  float scale_log2;
  int32_t* status;
  uint32_t wait_limit;                  // in units of 1024 ns
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

// Exclusive prefix sum over the block's threads, and the sum of all. (Two barriers.)
template <int kThreads>
__device__ __forceinline__ int64_t block_prefix(int64_t x, int64_t* s_warp, int64_t& total) {
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
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s_warp[w];
    total += s_warp[w];
  }
  __syncthreads();
  return before + sum - x;
}

// A box of a page: 16 rows of one head. Coordinates: column (0), row of the page, chunk of 64 columns (0: all of them), head, page.
// Every lane whose `issue` is set loads its own; beyond the last page: zeros.
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row, int head, int page, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %6, 0;\n"
      "@q cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%7, %3, %7, %4, %5}], [%2];\n}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(row), "r"(head), "r"(page), "r"(issue), "r"(0) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 shared8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}

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

// What differs between pages of bf16 and of e4m3: where a row's 16-byte pieces stand in shared memory, and how 16 keys are
// multiplied. Lane = 4 g + t. A: 16 keys (g, g + 8) by 16 elements, or 16 elements of O (`element`) by 16 keys. q: D / 8 words of a
// thread for the upper part of the queries, as many for the lower one.
template <int D, bool kE4m3>
struct Rows;

template <int D>
struct Rows<D, false> {
  static constexpr int kWarps = 6;
  static constexpr int kRowBytes = 2 * D, kSteps = kHalfUnit / (16 * kRowBytes);      // steps of 16 keys in a unit
  static constexpr float kWeight = 1.f;
  static constexpr bool kLowPart = true;
  // A step's box, as TMA leaves it: chunks of 64 elements one behind the other, rows of 128 bytes, the 16-byte pieces of 8 rows
  // swizzled so that one of each row fill all banks once.
  static constexpr int kStepBytes = 16 * kRowBytes, kChunkBytes = 2048;
  static __device__ __forceinline__ int row_of(int at) { return (D == 128 ? 0 : (at >> 11) * 16) + ((at >> 7) & 15); }   // of byte `at` of a unit
  static __device__ __forceinline__ void load_q(uint32_t (&q)[D / 8], uint32_t row_at, int t) {
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q[2 * kk + x]) : "r"(row_at + 32 * kk + 16 * x + 4 * t) : "memory");
  }
  static __device__ __forceinline__ void mma_scores(float (&c)[4], const uint32_t (*a)[4], const uint32_t (&qh)[D / 8], const uint32_t (&ql)[D / 8]) {
    // four chains of products instead of one: each waits for the one before it
    float p[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x) p[x][0] = p[x][1] = p[x][2] = p[x][3] = 0.f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      mma16816(p[kk & 1], a[kk][0], a[kk][1], a[kk][2], a[kk][3], qh[2 * kk], qh[2 * kk + 1]);
      mma16816(p[2 + (kk & 1)], a[kk][0], a[kk][1], a[kk][2], a[kk][3], ql[2 * kk], ql[2 * kk + 1]);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) c[x] = (p[0][x] + p[1][x]) + (p[2][x] + p[3][x]);
  }
  // scores of the 16 rows that begin at `at`
  static __device__ __forceinline__ void scores(float (&c)[4], uint32_t at, const uint32_t (&qh)[D / 8], const uint32_t (&ql)[D / 8], int lane) {
    uint32_t a[D / 16][4];
    const uint32_t from = at + ((lane & 7) + (lane & 8)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) ldmatrix4(a[kk], (from ^ ((kk & 3) << 5)) + (kk >> 2) * kChunkBytes);
    mma_scores(c, a, qh, ql);
  }
  // a row of its own, as the first of 16
  static __device__ __forceinline__ void scores_one(float (&c)[4], uint32_t at, const uint32_t (&qh)[D / 8], const uint32_t (&ql)[D / 8], int g, int t) {
    uint32_t a[D / 16][4];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      uint32_t x, y;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at + 32 * kk + 4 * t) : "memory");
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(y) : "r"(at + 32 * kk + 16 + 4 * t) : "memory");
      a[kk][0] = g == 0 ? x : 0u;
      a[kk][1] = 0u;
      a[kk][2] = g == 0 ? y : 0u;
      a[kk][3] = 0u;
    }
    mma_scores(c, a, qh, ql);
  }
  // P in two parts of 8 bits, the first cut and not rounded, so that neither is negative, and none of a weight above 0 (which is
  // at least 2^-126) is 0: an infinite value then gives an infinity and not a NaN, a finite one up to 2^-125 of itself too much.
  struct Weights { uint32_t b[2][2]; };
  static __device__ __forceinline__ Weights weights(const float (&p)[4]) {
    Weights w;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float p0 = p[2 * x], p1 = p[2 * x + 1];
      const uint32_t cut = truncate_bf16x2(p0, p1), least = (p0 > 0.f ? 0x0080u : 0u) | (p1 > 0.f ? 0x00800000u : 0u);
      const float2 back = unpack_bf16(cut);
      const uint32_t rest = round_bf16(p0 - back.x, p1 - back.y);
      const __nv_bfloat162 low = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&rest), *reinterpret_cast<const __nv_bfloat162*>(&least));
      w.b[0][x] = transpose8x8(cut);
      w.b[1][x] = transpose8x8(*reinterpret_cast<const uint32_t*>(&low));
    }
    return w;
  }
  static __device__ __forceinline__ void add(float (&acc)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const Weights& w) {
    mma16816(acc, a0, a1, a2, a3, w.b[1][0], w.b[1][1]);
    mma16816(acc, a0, a1, a2, a3, w.b[0][0], w.b[0][1]);
  }
  static __device__ __forceinline__ void product(float (&acc)[D / 16][4], uint32_t at, const float (&p)[4], int lane) {
    const Weights w = weights(p);
    const uint32_t from = at + ((lane & 7) + ((lane >> 1) & 8)) * 128 + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      uint32_t a[4];
      ldmatrix4_trans(a, (from ^ ((j & 3) << 5)) + (j >> 2) * kChunkBytes);
      add(acc[j], a[0], a[1], a[2], a[3], w);
    }
  }
  static __device__ __forceinline__ void product_one(float (&acc)[D / 16][4], uint32_t at, const float (&p)[4], int g, int t) {
    const Weights w = weights(p);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      uint16_t x, y;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at + 2 * (16 * j + g)) : "memory");
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(at + 2 * (16 * j + g + 8)) : "memory");
      add(acc[j], t == 0 ? x : 0u, t == 0 ? y : 0u, 0u, 0u, w);
    }
  }
  // element of O that acc[j][0], acc[j][1] (x = 0) and acc[j][2], acc[j][3] (x = 1) stand for
  static __device__ __forceinline__ int element(int j, int x, int g) { return 16 * j + 8 * x + g; }
  // and at place (D / 8) g + 2 j + x of a part, so that those of a lane stand together
  static __device__ __forceinline__ int element_at(int place) {
    const int g = place / (D / 8), r = place % (D / 8);
    return 16 * (r >> 1) + 8 * (r & 1) + g;
  }
  static __device__ __forceinline__ int place_of(int element) { return (D / 8) * (element & 7) + (element >> 4) * 2 + ((element >> 3) & 1); }
  // O of the eight heads as rows of bf16, heads 2t and 2t + 1 times f0 and f1 (transposed, a lane holds pairs of elements of one head)
  static __device__ __forceinline__ void leave(const float (&acc)[D / 16][4], float f0, float f1, uint32_t at, int g, int t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t w = transpose8x8(round_bf16(acc[j][2 * x] * f0, acc[j][2 * x + 1] * f1));
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + 2 * (g * D + 16 * j + 8 * x + 2 * t)), "r"(w) : "memory");
      }
  }
  // the two 16-bit parts of a pair of query elements
  static __device__ __forceinline__ uint32_t high(float a, float b) { return round_bf16(a, b); }
  static __device__ __forceinline__ uint32_t low(float a, float b, uint32_t h) {
    const float2 f = unpack_bf16(h);
    // (an infinite element has no lower part)
    return round_bf16(isfinite(f.x) ? a - f.x : 0.f, isfinite(f.y) ? b - f.y : 0.f);
  }
};

// e4m3 numbers are multiplied as f16, which holds all of them: K rows g and g + 8, 16-byte pieces 2t, 2t + 1 of a row (D = 64: piece t);
// V rows 2t, 2t + 1, 2t + 8, 2t + 9, the g-th eighth of a row.
template <int D>
struct Rows<D, true> {
  static constexpr int kWarps = 7;
  static constexpr int kRowBytes = D, kSteps = kHalfUnit / (16 * kRowBytes);
  // Queries and weights are rounded to f16 once: 11 bits, 2^-12 of each, against the 2^-8 of O's last rounding and keys of 4 bits.
  // Weights are at most 2^kLazyLog2; times 2^11 those down to 2^-25 of the largest have all of their bits, and what the sum of 2^17
  // of the smallest loses is below 2^-18 of it.
  static constexpr bool kLowPart = false;
  static constexpr float kWeight = 2048.f;
  // A step's box, as TMA leaves it: rows of 128 (64) bytes, whose 16-byte pieces are swizzled.
  static constexpr int kStepBytes = 16 * kRowBytes;
  static __device__ __forceinline__ uint32_t place(int row, int piece) { return row * D + ((piece ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4); }
  static __device__ __forceinline__ int row_of(int at) { return at / D; }
  static __device__ __forceinline__ void load_q(uint32_t (&q)[D / 8], uint32_t row_at, int t) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {                // words 8 (piece) + 2 (word of the piece) + pair
      const uint4 x = shared16(row_at + D / 2 * t + 16 * i);
      q[4 * i] = x.x; q[4 * i + 1] = x.y; q[4 * i + 2] = x.z; q[4 * i + 3] = x.w;
    }
  }
  static __device__ __forceinline__ void mma_scores(float (&c)[4], const uint4 (&r0)[D / 64], const uint4 (&r1)[D / 64], const uint32_t (&q)[D / 8]) {
    float p[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) p[x][0] = p[x][1] = p[x][2] = p[x][3] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {                   // four elements of a row in each word of the piece
        const uint32_t x0 = word_of(r0[i], w), x1 = word_of(r1[i], w);
        const uint32_t a0 = f16_of_e4m3_lo(x0), a1 = f16_of_e4m3_lo(x1), a2 = f16_of_e4m3_hi(x0), a3 = f16_of_e4m3_hi(x1);
        mma16816_f16(p[w & 1], a0, a1, a2, a3, q[8 * i + 2 * w], q[8 * i + 2 * w + 1]);
      }
#pragma unroll
    for (int x = 0; x < 4; ++x) c[x] = p[0][x] + p[1][x];
  }
  static __device__ __forceinline__ void scores(float (&c)[4], uint32_t at, const uint32_t (&q)[D / 8], const uint32_t (&)[D / 8], int lane) {
    uint4 r0[D / 64], r1[D / 64];
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      r0[i] = shared16(at + place(g, D / 64 * t + i));
      r1[i] = shared16(at + place(g + 8, D / 64 * t + i));
    }
    mma_scores(c, r0, r1, q);
  }
  static __device__ __forceinline__ void scores_one(float (&c)[4], uint32_t at, const uint32_t (&q)[D / 8], const uint32_t (&)[D / 8], int g, int t) {
    uint4 r0[D / 64], r1[D / 64];
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint4 x = shared16(at + 16 * (D / 64 * t + i));
      r0[i] = g == 0 ? x : none;
      r1[i] = none;
    }
    mma_scores(c, r0, r1, q);
  }
  struct Weights { uint32_t b[2]; };
  static __device__ __forceinline__ Weights weights(const float (&p)[4]) {
    Weights w;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const __half2 h = __floats2half2_rn(p[2 * x] * kWeight, p[2 * x + 1] * kWeight);
      w.b[x] = transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
    }
    return w;
  }
  // O^T += V^T P. Product j: row g is d = (D / 8) g + 2j, row g + 8 the element after it. r: words w of the four rows.
  static __device__ __forceinline__ void add(float (&acc)[D / 16][4], int w, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, const Weights& p) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t k0 = __byte_perm(r0, r1, y ? 0x7362 : 0x5140), k1 = __byte_perm(r2, r3, y ? 0x7362 : 0x5140);
      const uint32_t a0 = f16_of_e4m3_lo(k0), a1 = f16_of_e4m3_hi(k0), a2 = f16_of_e4m3_lo(k1), a3 = f16_of_e4m3_hi(k1);
      mma16816_f16(acc[2 * w + y], a0, a1, a2, a3, p.b[0], p.b[1]);
    }
  }
  static __device__ __forceinline__ void product(float (&acc)[D / 16][4], uint32_t at, const float (&p)[4], int lane) {
    const Weights w = weights(p);
    const int g = lane >> 2, t = lane & 3;
    uint4 r[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int row = 2 * t + (x & 1) + 8 * (x >> 1);
      if constexpr (D == 128) {
        r[x] = shared16(at + place(row, g));
      } else {
        const uint2 y = shared8(at + place(row, g >> 1) + 8 * (g & 1));
        r[x] = make_uint4(y.x, y.y, 0u, 0u);
      }
    }
#pragma unroll
    for (int n = 0; n < D / 32; ++n) add(acc, n, word_of(r[0], n), word_of(r[1], n), word_of(r[2], n), word_of(r[3], n), w);
  }
  static __device__ __forceinline__ void product_one(float (&acc)[D / 16][4], uint32_t at, const float (&p)[4], int g, int t) {
    const Weights w = weights(p);
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
      uint32_t x;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at + (D / 8) * g + 4 * n) : "memory");
      add(acc, n, t == 0 ? x : 0u, 0u, 0u, 0u, w);
    }
  }
  static __device__ __forceinline__ int element(int j, int x, int g) { return (D / 8) * g + 2 * j + x; }
  static __device__ __forceinline__ int element_at(int place) { return place; }
  static __device__ __forceinline__ void leave(const float (&acc)[D / 16][4], float f0, float f1, uint32_t at, int g, int t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w = round_bf16(acc[j][h] * (h ? f1 : f0), acc[j][2 + h] * (h ? f1 : f0));
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + 2 * ((2 * t + h) * D + (D / 8) * g + 2 * j)), "r"(w) : "memory");
      }
  }
  static __device__ __forceinline__ uint32_t high(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t low(float, float, uint32_t) { return 0u; }
};

// A warp's place on the line: the part of an item (prompt i, KV head kvh) that lies in its piece. An item takes kItemUnits of the line
// more than it has units: what its beginning and end cost its warp. With 1, 2, 3, 4 and 6 (seven warps; us a step): 256 prompts behind
// 8192 shared rows -, 128, 124, 122, 122; 256 prompts of two lengths, 240 k rows, 32 / 8 heads -, 166, 168, 169, 168, in e4m3 -, 101, 92,
// 94, 98; 64 prompts on 32 heads -, 55.8, 56.6, 57.8, 59.0.
constexpr int kItemUnits = 3;
struct Place {
  int64_t left;                         // of the piece, from here on
  int i, kvh;
  int len, start;                       // rows of the prompt, first row that is read here
  int units;                            // of an item of this prompt
  int off, n;                           // units off .. off + n - 1 of the item
  int used;                             // of the piece by this part
  int next_len, next_start;             // of prompt i + 1, on their way
};

template <int kUnitRows>
struct Line {
  const PagedArgs& a;
  bool fresh;
  __device__ __forceinline__ int units(int len, int start) const { return max((len - start + kUnitRows - 1) / kUnitRows, 1); }
  __device__ __forceinline__ void read(int i, int& len, int& start) const {
    len = -1;
    start = 0;
    if (i < a.n_prompts) {
      len = checked_length(a.c, a.lengths, i, fresh, nullptr);
      if (a.own) start = a.own[i].x;
    }
  }
  __device__ __forceinline__ int64_t line_units(int len, int start) const { return (int64_t)(units(len, start) + kItemUnits) * a.n_kv_heads; }
  // `at`: place within the item
  __device__ __forceinline__ void enter_item(Place& p, int at) const {
    p.used = (int)min((int64_t)(p.units + kItemUnits - at), p.left);
    p.off = max(at - kItemUnits, 0);
    p.n = max(at + p.used - kItemUnits, 0) - p.off;
  }
  // `p` at prompt i (a prompt, not an idle row), `at` within what its items take of the line.
  __device__ __forceinline__ void enter(Place& p, int64_t at) const {
    p.units = units(p.len, p.start);
    const int item = p.units + kItemUnits;
    p.kvh = (int)(at / item);
    enter_item(p, (int)(at - (int64_t)p.kvh * item));
    read(p.i + 1, p.next_len, p.next_start);
  }
  __device__ __forceinline__ void advance(Place& p) const {
    p.left -= p.used;
    if (p.left <= 0) {
      p.n = 0;
      return;
    }
    if (++p.kvh < a.n_kv_heads) return enter_item(p, 0);
    do {                                // (there is one: the piece is not at its end)
      ++p.i;
      p.len = p.next_len;
      p.start = p.next_start;
      if (p.len < 0) read(p.i + 1, p.next_len, p.next_start);
    } while (p.len < 0);
    enter(p, 0);
  }
};

template <int D, bool kE4m3>
__global__ void __launch_bounds__(32 * Rows<D, kE4m3>::kWarps, 1)
paged_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PagedArgs a,
                    const __grid_constant__ SharedPlan plan) {
  using R = Rows<D, kE4m3>;
  constexpr int kWarps = R::kWarps, kThreads = 32 * kWarps, kPieces = kSms * kWarps;
  constexpr int kSteps = R::kSteps, kUnitRows = 16 * kSteps, kHalf = D / 2, kSize = kE4m3 ? 1 : 2;
  constexpr int kLanesPerHead = kHalf / 4, kHeadsAtOnce = 32 / kLanesPerHead;       // queries: four (j, j + D/2) pairs a lane
  constexpr int kQPitch = 2 * D + 16;                                               // bytes
  static_assert(kMaxGroup * kQPitch <= kScratch && kMaxGroup * D * 2 <= kScratch && 4 * D <= kScratch, "scratch");
  extern __shared__ __align__(1024) uint8_t s_dyn[];
  __shared__ int64_t s_warp[kWarps], s_before[kThreads];
  __shared__ uint64_t s_bar[kWarps][4];                 // K of two units, V of two units
  __shared__ int s_abort;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, g = lane >> 2, t = lane & 3;
  const Line<kUnitRows> line{a, a.k_new != nullptr};
  const bool fresh = line.fresh;
  const uint32_t bars = smem_u32(s_bar[warp]);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) mbar_init(bars + 8 * i, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const WaitCtx wctx{smem_u32(&s_abort), a.wait_limit, a.status};
  pdl_wait();                           // lengths, table, pages: all may come from the kernel before
  pdl_launch_dependents();

  // ---- the line, and this warp's piece of it
  const int each = (a.n_prompts + kThreads - 1) / kThreads;
  int64_t mine = 0, total;
  for (int i = tid * each; i < min((tid + 1) * each, a.n_prompts); ++i) {
    const int len = checked_length(a.c, a.lengths, i, fresh, blockIdx.x == 0 ? a.status : nullptr);
    if (len >= 0) mine += line.line_units(len, a.own ? a.own[i].x : 0);
  }
  s_before[tid] = block_prefix<kThreads>(mine, s_warp, total);
  __syncthreads();
  const int64_t per = (total + kPieces - 1) / kPieces;
  const int piece = warp * kSms + blockIdx.x;               // few units: a warp on each SM first
  const int64_t u0 = piece * per;
  Place c;                              // where the arithmetic is
  c.left = min(per, total - u0);
  if (lane == 0) a.cut[piece] = make_int4(0, 0, 0, 0);
  if (c.left <= 0) return;
  {
    int lo = 0;                         // last thread whose prompts begin at or before u0 (those without units come before it)
    for (int w = 0; w < kWarps; ++w) lo += __popc(__ballot_sync(0xffffffffu, s_before[32 * w + lane] <= u0));
    --lo;
    int64_t at = u0 - s_before[lo];
    c.i = lo * each;
    for (;; ++c.i) {
      line.read(c.i, c.len, c.start);
      const int64_t here = c.len < 0 ? 0 : line.line_units(c.len, c.start);
      if (at < here) break;
      at -= here;
    }
    line.enter(c, at);
    if (c.n == 0) line.advance(c);      // a piece that ends before the item's first unit leaves it to the next
    if (c.n == 0) return;
  }

  // ---- loads, which run ahead
  const uint32_t aligned = (smem_u32(s_dyn) + 1023u) & ~1023u;
  const uint32_t ring = aligned + warp * (4 * kHalfUnit);                           // K of two units, V of two units
  uint8_t* scratch_p = s_dyn + (aligned - smem_u32(s_dyn)) + kWarps * (4 * kHalfUnit) + warp * kScratch;
  const uint32_t scratch = smem_u32(scratch_p), issue = elect_one(), lane_issue = lane < kSteps ? 1u : 0u;
  const int row_mask = (1 << a.c.page_shift) - 1;
  Place f = c;                          // where the copies are: unit f_at of the part f
  int f_at = 0, f_batch = -1, ids = 0, ids_prompt = -1;
  // Pages of the steps of an item, 32 at a time, one per lane; the next head of a prompt starts with the same ones.
  auto pages_of = [&](int batch) {
    if (ids_prompt == f.i && f_batch == batch) return;
    f_batch = batch;
    ids_prompt = f.i;
    const int64_t row = f.start + ((int64_t)batch * 32 + lane) * 16;
    ids = 0;
    if (row < f.len) {
      ids = a.c.table[(int64_t)f.i * a.c.table_stride + (row >> a.c.page_shift)];
      if ((unsigned)ids >= (unsigned)a.c.n_pages) {
        note_status(a.status, PP_PAGED_BAD_PAGE);
        ids = 0;
      }
    }
  };
  uint32_t stage_f = 0;                 // stage that the next unit goes to
  auto load_half = [&](int v) {         // a lane for each step of the unit
    const int unit = f.off + f_at, step = unit * kSteps + lane, row = f.start + step * 16;
    pages_of(unit * kSteps >> 5);
    const int id = __shfl_sync(0xffffffffu, ids, step & 31);
    const uint32_t bar = bars + 8 * (2 * v + stage_f), to = ring + (2 * v + stage_f) * kHalfUnit;
    mbar_expect_tx(bar, kHalfUnit, issue);
    __syncwarp();
    load_rows(to + lane * R::kStepBytes, v ? &map_v : &map_k, bar, row & row_mask, f.kvh, row < f.len ? id : a.c.n_pages, lane_issue);
  };
  auto load_k = [&]() {                 // (f.n = 0: nothing is left)
    if (f.n > 0) load_half(0);
  };
  auto load_v = [&]() {                 // and on to the next unit
    if (f.n == 0) return;
    load_half(1);
    stage_f ^= 1;
    if (++f_at == f.n) {
      line.advance(f);
      f_at = 0;
    }
  };
  load_k();
  load_v();
  load_k();
  load_v();

  uint32_t stage = 0, phase = 0;
  int angles_of = -1;
  float cs[4], sn[4];                   // of this lane's four pairs, at the position of prompt angles_of
  const int j0 = 4 * (lane % kLanesPerHead);
  // A wait gave up: loads of this warp may still be in flight. They get time to land before shared memory is handed back.
  auto settle = [&]() {
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 100000ull) {}
  };
  // What a part of an item needs beside its rows: four (j, j + D/2) pairs of the lane's heads, and of the new token.
  struct Raw { uint2 lo[kMaxGroup / kHeadsAtOnce], hi[kMaxGroup / kHeadsAtOnce], new_lo, new_hi, new_v; };
  auto ends_item = [&](const Place& p) { return p.off + p.n == p.units; };
  auto fetch = [&](Raw& r, const Place& p) {
    const __nv_bfloat16* q_row = a.q_new + (int64_t)p.i * a.q_stride + (int64_t)p.kvh * a.group * D;
#pragma unroll
    for (int x = 0; x < kMaxGroup / kHeadsAtOnce; ++x) {
      const int h = x * kHeadsAtOnce + lane / kLanesPerHead;
      r.lo[x] = r.hi[x] = make_uint2(0u, 0u);
      if (h < a.group) {
        r.lo[x] = *reinterpret_cast<const uint2*>(q_row + h * D + j0);
        r.hi[x] = *reinterpret_cast<const uint2*>(q_row + h * D + j0 + kHalf);
      }
    }
    if (fresh && ends_item(p)) {
      const __nv_bfloat16* k_row = a.k_new + (int64_t)p.i * a.k_stride + p.kvh * D;
      r.new_lo = *reinterpret_cast<const uint2*>(k_row + j0);
      r.new_hi = *reinterpret_cast<const uint2*>(k_row + j0 + kHalf);
      r.new_v = *reinterpret_cast<const uint2*>(a.v_new + (int64_t)p.i * a.v_stride + p.kvh * D + 4 * (lane % (D / 4)));
    }
  };
  Raw raw, raw_next;
  fetch(raw_next, c);
  while (true) {
    // ---- a part of an item; the queries of the next one are on their way meanwhile
    const bool begins = c.off == 0, ends = ends_item(c), new_row = ends && fresh;
    raw = raw_next;
    Place next = c;
    line.advance(next);
    if (next.n > 0) fetch(raw_next, next);
    // (m, l) and o over the rows that the prompt shares, where this part is the item's first
    float m[2] = {kNoScore, kNoScore}, l[2] = {0.f, 0.f}, acc[D / 16][4];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    if (begins && c.start > 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = 2 * t + h;
        if (head >= a.group) continue;
        const int64_t at = (int64_t)c.i * a.n_q_heads + c.kvh * a.group + head;
        const float2 ml = plan.row_ml[at];
        m[h] = ml.x;
        l[h] = g == 0 ? ml.y : 0.f;
        const float4* from = reinterpret_cast<const float4*>(plan.row_o + at * D + (D / 8) * g);
#pragma unroll
        for (int j = 0; j < D / 16; j += 2) {
          const float4 x = from[j >> 1];
          acc[j][h] = x.x; acc[j][2 + h] = x.y;
          acc[j + 1][h] = x.z; acc[j + 1][2 + h] = x.w;
        }
      }
    }
    if (angles_of != c.i) {
      angles_of = c.i;
      angles4(fresh ? c.len : max(c.len - 1, 0), a.angles.inv_freq + j0, cs, sn);
    }
    auto turn = [&](uint2 lo, uint2 hi, float (&p)[4], float (&y)[4]) {
      const float2 p0 = unpack_bf16(lo.x), p1 = unpack_bf16(lo.y), y0 = unpack_bf16(hi.x), y1 = unpack_bf16(hi.y);
      const float x[4] = {p0.x, p0.y, p1.x, p1.y}, z[4] = {y0.x, y0.y, y1.x, y1.y};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = turn_lo(x[e], z[e], cs[e], sn[e]);
        y[e] = turn_hi(x[e], z[e], cs[e], sn[e]);
      }
    };
    const float k_scale = kE4m3 ? a.c.k_scale[c.kvh] : 1.f, v_scale = kE4m3 ? a.c.v_scale[c.kvh] : 1.f;
    uint32_t qh[D / 8], ql[D / 8];
    float scale[2] = {a.scale_log2, a.scale_log2};
    // the upper parts through the scratch memory, then the lower ones, which wait in `raw`
#pragma unroll
    for (int x = 0; x < kMaxGroup / kHeadsAtOnce; ++x) {
      if (x * kHeadsAtOnce >= a.group) break;
      const int h = x * kHeadsAtOnce + lane / kLanesPerHead;
      float p[4], y[4];
      turn(raw.lo[x], raw.hi[x], p, y);
      if constexpr (kE4m3) {
        // f16 has 5 exponent bits: a query is brought to below 2 by a power of two (of up to 2^120: the rest f16 has room
        // for), which goes into its factor
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(p[e]), fabsf(y[e])));
#pragma unroll
        for (int o = kLanesPerHead / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int shift = min(max((int)(__float_as_uint(top) >> 23) - 127, -120), 120);
        const float down = __uint_as_float((uint32_t)(127 - shift) << 23), factor = a.scale_log2 * k_scale * __uint_as_float((uint32_t)(127 + shift) << 23);
#pragma unroll
        for (int e = 0; e < 4; ++e) { p[e] *= down; y[e] *= down; }
#pragma unroll
        for (int z = 0; z < 2; ++z) {       // heads 2t and 2t + 1 are this lane's columns
          const float other = __shfl_sync(0xffffffffu, factor, ((2 * t + z) % kHeadsAtOnce) * kLanesPerHead);
          if ((2 * t + z) / kHeadsAtOnce == x) scale[z] = other;
        }
      }
      const uint32_t w[4] = {R::high(p[0], p[1]), R::high(p[2], p[3]), R::high(y[0], y[1]), R::high(y[2], y[3])};
      *reinterpret_cast<uint2*>(scratch_p + h * kQPitch + 2 * j0) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2*>(scratch_p + h * kQPitch + 2 * (j0 + kHalf)) = make_uint2(w[2], w[3]);
      raw.lo[x] = make_uint2(R::low(p[0], p[1], w[0]), R::low(p[2], p[3], w[1]));
      raw.hi[x] = make_uint2(R::low(y[0], y[1], w[2]), R::low(y[2], y[3], w[3]));
    }
    __syncwarp();
    R::load_q(qh, scratch + g * kQPitch, t);
    __syncwarp();
    if constexpr (R::kLowPart) {
#pragma unroll
      for (int x = 0; x < kMaxGroup / kHeadsAtOnce; ++x) {
        if (x * kHeadsAtOnce >= a.group) break;
        const int h = x * kHeadsAtOnce + lane / kLanesPerHead;
        *reinterpret_cast<uint2*>(scratch_p + h * kQPitch + 2 * j0) = raw.lo[x];
        *reinterpret_cast<uint2*>(scratch_p + h * kQPitch + 2 * (j0 + kHalf)) = raw.hi[x];
      }
      __syncwarp();
      R::load_q(ql, scratch + g * kQPitch, t);
      __syncwarp();
    }
    if (g >= a.group) {                 // absent heads
#pragma unroll
      for (int x = 0; x < D / 8; ++x) qh[x] = ql[x] = 0u;
    }

    // ---- the rows
    // Weights of the scores in s (rows at or past n_real are hidden), with O, l and m brought to the new maximum.
    auto soften = [&](auto& s, int n_real) {
      constexpr int kN = sizeof(s) / sizeof(s[0]);
      if (n_real < 16 * kN) {
#pragma unroll
        for (int x = 0; x < kN; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (16 * x + g + 8 * (y >> 1) >= n_real) s[x][y] = -INFINITY;
      }
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < kN; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) mx[y & 1] = fmaxf(mx[y & 1], s[x][y]);
      mx[0] *= scale[0];
      mx[1] *= scale[1];
      if (__any_sync(0xffffffffu, mx[0] > m[0] + kLazyLog2 || mx[1] > m[1] + kLazyLog2)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], o));
          const float m_new = fmaxf(m[h], mx[h]), alpha = ex2(m[h] - m_new);         // 0 on the first step
          m[h] = m_new;
          l[h] *= alpha;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) { acc[j][h] *= alpha; acc[j][2 + h] *= alpha; }
        }
      }
#pragma unroll
      for (int x = 0; x < kN; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          s[x][y] = ex2(__fmaf_rn(s[x][y], scale[y & 1], -m[y & 1]));
          l[y & 1] += s[x][y];
        }
    };
    int row0 = c.start + c.off * kUnitRows;
    for (int n = 0; n < c.n; ++n, row0 += kUnitRows) {
      float s[kSteps][4];
      const uint32_t k_at = ring + stage * kHalfUnit, v_at = k_at + 2 * kHalfUnit;
      if (!mbar_wait_issuer<kWaitRows>(bars + 8 * stage, phase, wctx)) return settle();
#pragma unroll
      for (int x = 0; x < kSteps; ++x) R::scores(s[x], k_at + x * R::kStepBytes, qh, ql, lane);
      __syncwarp();
      load_k();
      const int n_real = c.len - row0;
      soften(s, n_real);
      if (!mbar_wait_issuer<kWaitRows>(bars + 16 + 8 * stage, phase, wctx)) return settle();
      if (n_real < kUnitRows) {
        // The rows past the last one are of no part of O, not as 0 times what they hold either.
        for (int at = 16 * lane; at < kHalfUnit; at += 16 * 32)
          if (R::row_of(at) >= n_real) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v_at + at), "r"(0) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
#pragma unroll
      for (int x = 0; x < kSteps; ++x) R::product(acc, v_at + x * R::kStepBytes, s[x], lane);
      __syncwarp();
      load_v();
      stage ^= 1;
      phase ^= stage ^ 1;               // (after every second unit)
    }
    if (new_row) {                      // the new token, and its rows of the pages
      float p[4], y[4];
      turn(raw.new_lo, raw.new_hi, p, y);
      const float2 v0 = unpack_bf16(raw.new_v.x), v1 = unpack_bf16(raw.new_v.y);
      if constexpr (kE4m3) {
        const float per_k = __frcp_rn(k_scale), per_v = __frcp_rn(v_scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) { p[e] *= per_k; y[e] *= per_k; }
        if (lane < kLanesPerHead) {
          *reinterpret_cast<uint32_t*>(scratch_p + j0) = round_e4m3(p[0], p[1], p[2], p[3]);
          *reinterpret_cast<uint32_t*>(scratch_p + j0 + kHalf) = round_e4m3(y[0], y[1], y[2], y[3]);
        }
        if (lane < D / 4)
          *reinterpret_cast<uint32_t*>(scratch_p + D + 4 * lane) =
              round_e4m3(v0.x * per_v, v0.y * per_v, v1.x * per_v, v1.y * per_v);
      } else {
        if (lane < kLanesPerHead) {
          *reinterpret_cast<uint2*>(scratch_p + 2 * j0) = make_uint2(round_bf16(p[0], p[1]), round_bf16(p[2], p[3]));
          *reinterpret_cast<uint2*>(scratch_p + 2 * (j0 + kHalf)) = make_uint2(round_bf16(y[0], y[1]), round_bf16(y[2], y[3]));
        }
        if (lane < D / 4) *reinterpret_cast<uint2*>(scratch_p + 2 * D + 8 * lane) = raw.new_v;
      }
      __syncwarp();
      float s[1][4];
      R::scores_one(s[0], scratch, qh, ql, g, t);
      soften(s, 1);
      R::product_one(acc, scratch + D * kSize, s[0], g, t);
      const int page = a.c.table[(int64_t)c.i * a.c.table_stride + (c.len >> a.c.page_shift)];
      if ((unsigned)page < (unsigned)a.c.n_pages) {
        const int64_t to = (int64_t)page * a.c.page_stride + (int64_t)c.kvh * a.c.head_stride + (int64_t)(c.len & row_mask) * a.c.row_stride;
        if (lane < R::kRowBytes / 16) {
          *reinterpret_cast<uint4*>(a.c.k_pages + to + 16 * lane) = shared16(scratch + 16 * lane);
          *reinterpret_cast<uint4*>(a.c.v_pages + to + 16 * lane) = shared16(scratch + D * kSize + 16 * lane);
        }
      } else if (lane == 0) {
        note_status(a.status, PP_PAGED_BAD_PAGE);
      }
      __syncwarp();
    }

    // ---- out
    const float out_scale = v_scale / R::kWeight;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
    if (begins && ends) {
      // (a row that attends to nothing is 0; one all of whose scores are -inf is a NaN)
      const bool none = c.len + (int)fresh <= 0;
      R::leave(acc, none ? 0.f : out_scale / l[0], none ? 0.f : out_scale / l[1], scratch, g, t);
      __syncwarp();
      __nv_bfloat16* to = a.o + ((int64_t)c.i * a.n_q_heads + c.kvh * a.group) * D;
      for (int x = lane; x < a.group * D / 8; x += 32) *reinterpret_cast<uint4*>(to + 8 * x) = shared16(scratch + 16 * x);
      __syncwarp();
    } else {
      const int64_t slot = 2 * (int64_t)piece + (begins ? 1 : 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = 2 * t + h;
        if (head >= a.group) continue;
        if (g == 0) a.part_ml[slot * a.group + head] = make_float2(m[h], l[h]);
        float* to = a.part_o + (slot * a.group + head) * D + (D / 8) * g;
#pragma unroll
        for (int j = 0; j < D / 16; j += 4)       // (whole sectors: 32 bytes a store)
          asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                       ::"l"(to + 2 * j), "f"(acc[j][h] * out_scale), "f"(acc[j][2 + h] * out_scale), "f"(acc[j + 1][h] * out_scale),
                         "f"(acc[j + 1][2 + h] * out_scale), "f"(acc[j + 2][h] * out_scale), "f"(acc[j + 2][2 + h] * out_scale),
                         "f"(acc[j + 3][h] * out_scale), "f"(acc[j + 3][2 + h] * out_scale) : "memory");
      }
      if (begins && lane == 0)          // the pieces over which the item goes on: units behind this one's end
        a.cut[piece] = make_int4(c.i, c.kvh, 1 + (int)((c.units - c.n + per - 1) / per), 0);
    }
    if (next.n == 0) return;
    c = next;
  }
}

// The parts of one query head, (m, l) and D floats each, joined by one warp: parts first, first + step, ... of n; `at` says where a part lies.
template <int D>
struct Joined {
  static constexpr int E = D / 32;      // consecutive elements per lane
  float m, l, o[E];
};
template <int D, int kAtOnce, class At>
__device__ __forceinline__ Joined<D> join_parts(int first, int step, int n, const float2* mls, const float* os, int lane, const At& at) {
  constexpr int E = D / 32;
  Joined<D> s{kNoScore, 0.f, {}};
  for (int base = first; base < n; base += kAtOnce * step) {
    float2 ml[kAtOnce];
    float p[kAtOnce][E];
#pragma unroll
    for (int c = 0; c < kAtOnce; ++c) {               // (all of these loads are under way together)
      ml[c] = make_float2(kNoScore, 0.f);
#pragma unroll
      for (int e = 0; e < E; ++e) p[c][e] = 0.f;
      if (base + c * step >= n) continue;
      const int64_t from = at(base + c * step);
      ml[c] = mls[from];
      const float* src = os + from * D + E * lane;
      if constexpr (E == 4) {
        const float4 x = *reinterpret_cast<const float4*>(src);
        p[c][0] = x.x; p[c][1] = x.y; p[c][2] = x.z; p[c][3] = x.w;
      } else {
        const float2 x = *reinterpret_cast<const float2*>(src);
        p[c][0] = x.x; p[c][1] = x.y;
      }
    }
    float m_new = s.m;
#pragma unroll
    for (int c = 0; c < kAtOnce; ++c) m_new = fmaxf(m_new, ml[c].x);
    const float alpha = ex2(s.m - m_new);
    s.m = m_new;
    s.l *= alpha;
#pragma unroll
    for (int e = 0; e < E; ++e) s.o[e] *= alpha;
#pragma unroll
    for (int c = 0; c < kAtOnce; ++c) {
      if (ml[c].y == 0.f) continue;     // (a part that took no keys may have left no O)
      const float f = ex2(ml[c].x - m_new);
      s.l += ml[c].y * f;
#pragma unroll
      for (int e = 0; e < E; ++e) s.o[e] += p[c][e] * f;
    }
  }
  return s;
}
// What the warps of a CTA have joined of one head, as one: `leave` gets m, l and o of every place, a thread for each. (Ends with a barrier.)
template <int D, int kWarps>
struct JoinSpace { float m[kWarps], l[kWarps], o[kWarps][D]; };
template <int D, int kWarps, class Leave>
__device__ __forceinline__ void join_warps(const Joined<D>& s, JoinSpace<D, kWarps>& space, const Leave& leave) {
  constexpr int E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) {
    space.m[warp] = s.m;
    space.l[warp] = s.l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) space.o[warp][E * lane + e] = s.o[e];
  __syncthreads();
  if (threadIdx.x < D) {
    float m = space.m[0], l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmaxf(m, space.m[w]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = space.l[w] == 0.f ? 0.f : ex2(space.m[w] - m);
      l += space.l[w] * f;
      o += space.o[w][threadIdx.x] * f;
    }
    leave(m, l, o, (int)threadIdx.x);
  }
  __syncthreads();
}

// Joins the parts of the items that are cut. kAcross: a CTA for a query head and a piece in which such an item may begin (the others
// leave at once), where a CTA for each runs at once. Otherwise a warp for each, neighbouring warps for neighbouring pieces; an item in
// many parts (one prompt alone may have a hundred) is the work of the whole CTA here too. (Whole steps in the first form and in the
// second: ten prompts, 32 heads, 11.1 and 11.8 us; 240 k rows on 32 / 8 heads 161 and 159.)
template <int D, class R, bool kAcross>
__global__ void __launch_bounds__(kCombineThreads)
paged_combine_kernel(const __grid_constant__ PagedArgs a, int n_pieces) {
  constexpr int E = D / 32, kWarps = kCombineThreads / 32, kManyParts = 16;
  __shared__ JoinSpace<D, kWarps> space;
  __shared__ int4 s_cut[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();                           // the parts come from the kernels before this one
  pdl_launch_dependents();
  const int h = blockIdx.y, piece0 = kAcross ? blockIdx.x : blockIdx.x * kWarps, piece = kAcross ? piece0 : piece0 + warp;
  const int4 cut = piece < n_pieces ? a.cut[piece] : make_int4(0, 0, 0, 0);
  auto leave = [&](const int4& c, const Joined<D>& s) {         // (an item that is cut has rows)
    __nv_bfloat16* to = a.o + ((int64_t)c.x * a.n_q_heads + c.y * a.group + h) * D;
#pragma unroll
    for (int e = 0; e < E; ++e) to[R::element_at(E * lane + e)] = __float2bfloat16_rn(s.o[e] / s.l);
  };
  auto at = [&](int first) { return [first, h, group = a.group](int part) { return (2 * (int64_t)first + (part == 0 ? 1 : 2 * part)) * group + h; }; };
  auto together = [&](const int4& c, int first) {
    join_warps<D, kWarps>(join_parts<D, 4>(warp, kWarps, c.z, a.part_ml, a.part_o, lane, at(first)), space, [&](float, float l, float o, int place) {
      a.o[((int64_t)c.x * a.n_q_heads + c.y * a.group + h) * D + R::element_at(place)] = __float2bfloat16_rn(o / l);
    });
  };
  if constexpr (kAcross) {
    if (cut.z > 0) together(cut, piece);
  } else {
    const bool many = cut.z > kManyParts;
    if (cut.z > 0 && !many) leave(cut, join_parts<D, 8>(0, 1, cut.z, a.part_ml, a.part_o, lane, at(piece)));
    if (!__syncthreads_or(many)) return;
    if (lane == 0) s_cut[warp] = many ? cut : make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int w = 0; w < kWarps; ++w)
      if (s_cut[w].z > 0) together(s_cut[w], piece0 + w);
  }
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
    if (g >= 0 && len >= 0) {
      atomicMin(&s_rows[g], len);
      atomicMin(&s_lead[g], i);
    }
  }
  __syncthreads();
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int each = (n + kPlanThreads - 1) / kPlanThreads, g0 = min(tid * each, n), g1 = min(g0 + each, n);
  int64_t units = 0, parts = 0;
  for (int g = g0; g < g1; ++g) {
    const int prompts = bad ? 0 : s_ptr[g + 1] - s_ptr[g];
    const int rows = prompts > 0 && s_lead[g] < k ? s_rows[g] & ~page_mask : 0;      // (a group may be all rows of no prompt)
    s_rows[g] = rows;
    const int tiles = (rows + kSharedTileKeys - 1) / kSharedTileKeys;
    units += (int64_t)tiles * ((prompts * a.group + kSharedTileRows - 1) / kSharedTileRows) * a.n_kv_heads;
    parts += (int64_t)shared_part_rows(prompts * a.group) * a.n_kv_heads;
  }
  int64_t all, none, at = block_prefix<kPlanThreads>(units, s_warp, all), part = block_prefix<kPlanThreads>(parts, s_warp, none);
  for (int g = g0; g < g1; ++g) {
    const int prompts = bad ? 0 : s_ptr[g + 1] - s_ptr[g];
    SharedGroup x;
    x.unit_start = at;
    x.part_start = part;
    x.key_tiles = (s_rows[g] + kSharedTileKeys - 1) / kSharedTileKeys;
    x.shared_rows = s_rows[g];
    x.lead = s_lead[g];
    x.first = s_ptr[g];
    x.query_rows = prompts * a.group;
    plan.groups[g] = x;
    at += (int64_t)x.key_tiles * ((x.query_rows + kSharedTileRows - 1) / kSharedTileRows) * a.n_kv_heads;
    part += (int64_t)shared_part_rows(x.query_rows) * a.n_kv_heads;
  }
  if (tid == 0) *plan.units = all;
  __syncthreads();
  for (int i = tid; i < k; i += kPlanThreads) {
    const int g = group_of(i);
    plan.prompts[i] = make_int2(g >= 0 && a.lengths[i] >= 0 ? s_rows[g] : 0, g);
  }
}

// The parts of every query head over the shared rows, from the CTAs of the attention kernel, become one: a warp for each head of each
// prompt, or, of few, a CTA (kAcross). The step over the prompts' own rows goes on from there, and finds the elements in its order.
template <int D, bool kAcross>
__global__ void __launch_bounds__(kCombineThreads)
shared_join_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ SharedPlan plan) {
  using R = Rows<D, false>;
  constexpr int E = D / 32, kWarps = kCombineThreads / 32;
  __shared__ JoinSpace<D, kAcross ? kWarps : 1> space;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = kAcross ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kWarps + warp;
  pdl_wait();
  pdl_launch_dependents();
  if (row >= (int64_t)a.n_prompts * a.n_q_heads) return;
  const int i = (int)(row / a.n_q_heads), head = (int)(row - (int64_t)i * a.n_q_heads), kvh = head / a.group;
  const int2 own = plan.prompts[i];
  const int64_t per = units_per_piece(*plan.units, plan.n_ctas);
  if (own.x == 0) return;               // nothing shared
  const SharedGroup gr = plan.groups[own.y];
  const int r = (i - gr.first) * a.group + head - kvh * a.group, rt = r / kSharedTileRows;
  const int64_t u0 = gr.unit_start + ((int64_t)kvh * ((gr.query_rows + kSharedTileRows - 1) / kSharedTileRows) + rt) * gr.key_tiles;
  const int p0 = (int)(u0 / per), n = (int)((u0 + gr.key_tiles - 1) / per) - p0 + 1;
  // (an item of few rows has two parts in each piece, see pp_paged.h)
  const int item_rows = min(gr.query_rows - rt * kSharedTileRows, kSharedTileRows), sides = item_rows <= kSharedTileRows / 2 ? 2 : 1;
  const int64_t at = (int64_t)p0 * kSharedTileRows + gr.part_start + (int64_t)kvh * shared_part_rows(gr.query_rows) + r;
  auto part_row = [&](int part) { return at + (int64_t)(sides == 2 ? part >> 1 : part) * kSharedTileRows + (sides == 2 && (part & 1) ? item_rows : 0); };
  float* to = plan.row_o + row * D;
  if constexpr (kAcross) {
    join_warps<D, kWarps>(join_parts<D, 4>(warp, kWarps, n * sides, plan.ml, plan.o, lane, part_row), space, [&](float m, float l, float o, int element) {
      if (element == 0) plan.row_ml[row] = make_float2(m, l);
      to[R::place_of(element)] = o;
    });
  } else {
    const Joined<D> s = join_parts<D, 4>(0, 1, n * sides, plan.ml, plan.o, lane, part_row);
    if (lane == 0) plan.row_ml[row] = make_float2(s.m, s.l);
#pragma unroll
    for (int e = 0; e < E; ++e) to[R::place_of(E * lane + e)] = s.o[e];
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

// 5-D map (column, row, chunk of 128 bytes, head, page) over a pool of pages; box = 16 rows of one head.
bool page_map(CUtensorMap* map, const void* pages, const PagedArgs& a, int d, bool e4m3) {
  EncodeFn enc = get_encode_fn();
  if (!enc) return false;
  const int size = e4m3 ? 1 : 2, columns = std::min(d, 128 / size);
  const cuuint64_t dims[5] = {(cuuint64_t)columns, (cuuint64_t)1 << a.c.page_shift, (cuuint64_t)(d / columns), (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.c.n_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)a.c.row_stride, 128u, (cuuint64_t)a.c.head_stride, (cuuint64_t)a.c.page_stride};
  const cuuint32_t box[5] = {(cuuint32_t)columns, 16u, (cuuint32_t)(d / columns), 1u, 1u}, ones[5] = {1u, 1u, 1u, 1u, 1u};
  return enc(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(pages), dims, strides, box, ones,
             CU_TENSOR_MAP_INTERLEAVE_NONE, columns * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kE4m3>
cudaError_t launch_paged_decode(const PagedArgs& a, const SharedPlan& plan, cudaStream_t s) {
  constexpr int kWarps = Rows<D, kE4m3>::kWarps, kSmem = 1024 + kWarps * (4 * kHalfUnit + kScratch);     // rings on 1024-byte boundaries
  static DeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(paged_decode_kernel<D, kE4m3>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  CUtensorMap mk, mv;
  if (!page_map(&mk, a.c.k_pages, a, D, kE4m3) || !page_map(&mv, a.c.v_pages, a, D, kE4m3)) return cudaErrorInvalidValue;
  e = launch_dependent(paged_decode_kernel<D, kE4m3>, dim3(kSms), dim3(32 * kWarps), (size_t)kSmem, s, mk, mv, a, plan);
  if (e != cudaSuccess) return e;
  constexpr int kPieces = kSms * kWarps, kJoiners = kCombineThreads / 32;
  using R = Rows<D, kE4m3>;
  if (kPieces * a.group <= 8 * kSms) return launch_dependent(paged_combine_kernel<D, R, true>, dim3(kPieces, a.group), dim3(kCombineThreads), 0, s, a, kPieces);
  return launch_dependent(paged_combine_kernel<D, R, false>, dim3((kPieces + kJoiners - 1) / kJoiners, a.group), dim3(kCombineThreads), 0, s, a, kPieces);
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
  a.own = n_groups > 0 ? reinterpret_cast<const int2*>(ws + L.prompts) : nullptr;
  a.q_new = static_cast<const __nv_bfloat16*>(q_new);
  a.k_new = static_cast<const __nv_bfloat16*>(k_new);
  a.v_new = static_cast<const __nv_bfloat16*>(v_new);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.cut = reinterpret_cast<int4*>(ws + L.cut);
  a.part_ml = reinterpret_cast<float2*>(ws + L.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + L.part_o);
  a.n_prompts = k;
  a.n_q_heads = params->n_q_heads;
  a.n_kv_heads = params->n_kv_heads;
  a.group = params->n_q_heads / params->n_kv_heads;
  const float scale = params->softmax_scale > 0.f ? params->softmax_scale : 1.0f / sqrtf((float)params->head_dim);
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = device_status;
  a.wait_limit = (uint32_t)std::min<unsigned long long>(wait_limit_ns() >> 10, 0x7fffffffu);
  a.angles = rope_angles(params->rope_base, params->head_dim);
  SharedPlan plan = {};
  if (n_groups > 0) {
    plan.units = reinterpret_cast<int64_t*>(ws + L.units);
    plan.groups = reinterpret_cast<SharedGroup*>(ws + L.groups);
    plan.prompts = reinterpret_cast<int2*>(ws + L.prompts);
    plan.q_rot = reinterpret_cast<__nv_bfloat16*>(ws + L.q_rot);
    plan.ml = reinterpret_cast<float2*>(ws + L.shared_ml);
    plan.o = reinterpret_cast<float*>(ws + L.shared_o);
    plan.row_ml = reinterpret_cast<float2*>(ws + L.row_ml);
    plan.row_o = reinterpret_cast<float*>(ws + L.row_o);
    plan.group_ptr = group_ptr;
    plan.n_groups = n_groups;
    plan.n_ctas = kSms;
    PlanArgs p{a, plan, shared_len};
    const cudaError_t e = d == 128 ? launch_plan<128>(p, s) : launch_plan<64>(p, s);
    if (e != cudaSuccess) return note_cuda_error((int)e, "plan kernel launch");
    if ((st = launch_shared_attention(*params, a.c, plan, k, a.scale_log2, device_status, s)) != PP_OK) return st;
    const int64_t heads = (int64_t)k * params->n_q_heads;
    const bool across = heads <= 8 * kSms;          // as long as a CTA for each runs at once
    const dim3 blocks((unsigned)(across ? heads : (heads + kCombineThreads / 32 - 1) / (kCombineThreads / 32)));
    auto join = [&](auto kernel) { return launch_dependent(kernel, blocks, dim3(kCombineThreads), 0, s, a, plan); };
    const cudaError_t joined = d == 128 ? (across ? join(shared_join_kernel<128, true>) : join(shared_join_kernel<128, false>))
                                        : (across ? join(shared_join_kernel<64, true>) : join(shared_join_kernel<64, false>));
    if (joined != cudaSuccess) return note_cuda_error((int)joined, "join kernel launch");
  }
  const bool e4m3 = cache->type == PP_CACHE_E4M3;
  const cudaError_t e = d == 128 ? (e4m3 ? launch_paged_decode<128, true>(a, plan, s) : launch_paged_decode<128, false>(a, plan, s))
                                 : (e4m3 ? launch_paged_decode<64, true>(a, plan, s) : launch_paged_decode<64, false>(a, plan, s));
  return e == cudaSuccess ? PP_OK : note_cuda_error((int)e, "paged generation step launch");
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
  const size_t parts = 2 * (size_t)kMostPieces * (p.n_q_heads / p.n_kv_heads);
  L.cut = take((size_t)kMostPieces * sizeof(int4));
  L.part_ml = take(parts * sizeof(float2));
  L.part_o = take(parts * p.head_dim * sizeof(float));
  if (n_groups > 0) {
    L.units = take(sizeof(int64_t));
    L.groups = take((size_t)n_groups * sizeof(SharedGroup));
    L.prompts = take((size_t)k * sizeof(int2));
    L.q_rot = take((size_t)k * p.n_q_heads * p.head_dim * sizeof(__nv_bfloat16));
    const size_t rows = (size_t)kSms * kSharedTileRows + 2 * (size_t)k * p.n_q_heads;
    L.shared_ml = take(rows * sizeof(float2));
    L.shared_o = take(rows * p.head_dim * sizeof(float));
    L.row_ml = take((size_t)k * p.n_q_heads * sizeof(float2));
    L.row_o = take((size_t)k * p.n_q_heads * p.head_dim * sizeof(float));
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
  a.rows_per_cta = (int32_t)std::min<int64_t>(std::max<int64_t>(pp::kAppendElements / dense, 1), pp::kAppendMaxRows);
  // The heads of one long row are shared out to several CTAs only while the GPU has room for all of them at once: each needs the row's
  // angles. (64 rows of 32 heads of 128: 3.2 -> 2.5 us; 17 554 of them 89 -> 94.)
  a.heads_per_cta = std::min(params->n_kv_heads, pp::kAppendElements / params->head_dim);
  if (n_rows * ((params->n_kv_heads + a.heads_per_cta - 1) / a.heads_per_cta) > 8 * pp::kSms) a.heads_per_cta = params->n_kv_heads;
  const int32_t head_blocks = (params->n_kv_heads + a.heads_per_cta - 1) / a.heads_per_cta;
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
  auto launch = [&](auto kernel) { return pp::launch_dependent(kernel, dim3((unsigned)grid, (unsigned)head_blocks), dim3(pp::kAppendThreads), 0, s, a); };
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
