// A KV cache in pages: rows appended to it (append_kernel), one generation step over it (paged_decode_kernel,
// paged_combine_kernel), and what a step in which prompts share pages needs around the attention of the shared rows
// (shared_plan_kernel; the attention itself is in pp_paged_shared.cu).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
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
// A copy with a rotation in it, bound by HBM: a CTA takes as many rows (or heads of one) as make 2048 elements of K. A thread has one
// pair of 8-element pieces of K (c and D/2 + c) and two pieces of V of the same row, so that all it needs is that row's prompt and
// position: its loads, the page's number and the angles (once for all heads of a row, through shared memory) are then under way together.
// 17 554 rows of 32 heads of 128 take 90 to 92 us (6.2 to 6.4 TB/s; 114 us with the row's place found first and handed round), 44 k short
// rows of 8 heads of 64 into 8 bits 33 us (4.1 TB/s, was 55), where instructions count: 430 a thread, a quarter of them for the angle, and
// as many for the conversions.
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
  pdl_wait();
  pdl_launch_dependents();              // (not before the wait: a step reads ahead what lies two kernels back, see below)
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
// Two kernels, and a third for what the second one cuts:
//   step_prepare_kernel   a CTA for each prompt: rotates its queries, rotates and appends the new token. (With shared rows a further
//                         CTA lays their work out, see below.)
//   paged_decode_kernel   attention over the rows, the appended one like any other
//   paged_combine_kernel  joins the parts of items that were cut (with shared rows shared_join_kernel does, and those over shared rows)
// Bound: HBM, every row of K and V is read once. The work is a line of units of 8 KB (16, 32 or 64 rows of K and V of one KV
// head), ordered by (prompt, KV head, rows), and cut into equal pieces, one for each warp that the GPU holds: all warps read the
// same number of bytes whatever the lengths are. A warp works on its own from there on. Its rows arrive by TMA in a ring of
// two units in shared memory, whose loads run ahead over the ends of items. Six warps (seven over 8-bit pages, which take more
// instructions a byte) keep up to 96 KB of an SM under way, which is all that HBM takes: with twelve, the loads queued up and SMs
// were served so unevenly that of 148 equal shares the last ended 20 % after the mean. A piece that is a whole item (prompt, KV head)
// leaves O at once. What an item costs beside its rows is the latency of one warp: with the queries rotated there, and the new token a
// step of its own, 4700 cycles, a unit 1800 (prepared apart: 64 prompts on 32 heads 57.8 -> 56.9 us, 64 prompts behind one document
// of 32 700 rows 59 -> 55, 16 samples of one prompt 25.9 -> 23.7; ten prompts on one layer 11.4 -> 12.1).
// The arithmetic is that of the step over contiguous caches (pp_decode.cu): mma.m16n8k16 with 16 keys as rows and the query heads
// of a KV head as the 8 columns, absent heads 0. Over bf16 pages a query and a weight each reach it as the sum of two
// 16-bit numbers: HBM leaves the tensor cores idle, and scores and O are then exact to 2^-16, far below O's last rounding of 2^-8.
// The lengths live on the device: every CTA sums them itself, and the grid and the room for parts depend on neither them nor k.
// (It does so before its wait for the kernel in front, which, like all kernels of this file and pp_paged_shared.cu, lets the next one start
// only after its own wait: what that one waited for is there then. Not through L1, which may hold what it was before.)
constexpr int kMaxGroup = 8;            // query heads per KV head: the N of the tensor-core product
constexpr int kMostStepWarps = 7, kMostPieces = kSms * kMostStepWarps;
constexpr int kHalfUnit = 4096;         // bytes of K, and of V, in a unit
constexpr int kScratch = 2048;          // per warp: O on its way out
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
  int2* items;                          // with shared rows: of every item (prompt, KV head) the piece in which it begins and its parts, 0: one,
                                        // which lies in row_ml, row_o [prompt][head]
  float2* row_ml;
  float* row_o;
  int4* cut;                            // [pieces]: of the item that begins in a piece and ends in another: prompt, KV head, pieces; 0 pieces: none
  uint32_t* q;                          // queries as the products take them: [prompt][head][t][parts][D / 8] words, see Rows
  float* q_factor;                      // [prompt][head] over 8-bit pages: from a product with them to scaled log2 units
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
  const int len = __ldcg(lengths + i);
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
  static constexpr int kParts = 2;                    // 16-bit parts of a query
  // which thread t takes the pair of elements (e, e + 1) of a query, and as which of its D / 8 words
  static __device__ __forceinline__ int word_thread(int e) { return (e >> 1) & 3; }
  static __device__ __forceinline__ int word_index(int e) { return (e >> 4) * 2 + ((e >> 3) & 1); }
  // A step's box, as TMA leaves it: chunks of 64 elements one behind the other, rows of 128 bytes, the 16-byte pieces of 8 rows
  // swizzled so that one of each row fill all banks once.
  static constexpr int kStepBytes = 16 * kRowBytes, kChunkBytes = 2048;
  static __device__ __forceinline__ int row_of(int at) { return (D == 128 ? 0 : (at >> 11) * 16) + ((at >> 7) & 15); }   // of byte `at` of a unit
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
  // element of O that acc[j][0], acc[j][1] (x = 0) and acc[j][2], acc[j][3] (x = 1) stand for
  static __device__ __forceinline__ int element(int j, int x, int g) { return 16 * j + 8 * x + g; }
  // and at place (D / 8) g + 2 j + x of a part, so that those of a lane stand together
  static __device__ __forceinline__ int element_at(int place) {
    const int g = place / (D / 8), r = place % (D / 8);
    return 16 * (r >> 1) + 8 * (r & 1) + g;
  }
  // O of the eight heads as rows of bf16, heads 2t and 2t + 1 times f0 and f1 (transposed, a lane holds pairs of elements of one head)
  static __device__ __forceinline__ void leave(const float (&acc)[D / 16][4], float f0, float f1, float, uint32_t at, int g, int t) {
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
  static constexpr int kParts = 1;
  static __device__ __forceinline__ int word_thread(int e) { return e / (D / 4); }
  static __device__ __forceinline__ int word_index(int e) { return e % (D / 4) / 2; }
  static constexpr float kWeight = 2048.f;
  // A step's box, as TMA leaves it: rows of 128 (64) bytes, whose 16-byte pieces are swizzled.
  static constexpr int kStepBytes = 16 * kRowBytes;
  static __device__ __forceinline__ uint32_t place(int row, int piece) { return row * D + ((piece ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4); }
  static __device__ __forceinline__ int row_of(int at) { return at / D; }
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
  static __device__ __forceinline__ int element(int j, int x, int g) { return (D / 8) * g + 2 * j + x; }
  static __device__ __forceinline__ int element_at(int place) { return place; }
  static __device__ __forceinline__ void leave(const float (&acc)[D / 16][4], float f0, float f1, float v_scale, uint32_t at, int g, int t) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w = round_bf16(acc[j][h] * (h ? f1 : f0) * v_scale, acc[j][2 + h] * (h ? f1 : f0) * v_scale);
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
// more than it has units: what its beginning and end cost its warp. (1, 2, 3 over 242 k rows of 256 prompts on 8 KV heads: 167.5, 160.6,
// 160.0 us; over 8-bit pages 95.4, 90.4, 91.7; 192 prompts with about 160 rows of their own each: 184, 167.7, 167.8.)
constexpr int kItemUnits = 2;
struct Place {
  int64_t left;                         // of the piece, from here on
  int i, kvh;
  int len, start;                       // rows of the prompt, the new one among them; first row that is read here
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
      if (len >= 0) len += fresh;
      if (a.own) start = __ldcg(&a.own[i].x);
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
paged_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ PagedArgs a) {
  using R = Rows<D, kE4m3>;
  constexpr int kWarps = R::kWarps, kThreads = 32 * kWarps, kPieces = kSms * kWarps;
  constexpr int kSteps = R::kSteps, kUnitRows = 16 * kSteps, kWords = R::kParts * D / 8;
  static_assert(kMaxGroup * D * 2 <= kScratch, "scratch");
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
  // ---- the line, and this warp's piece of it
  const int each = (a.n_prompts + kThreads - 1) / kThreads;
  int64_t mine = 0, total;
  for (int i = tid * each; i < min((tid + 1) * each, a.n_prompts); ++i) {
    const int len = checked_length(a.c, a.lengths, i, fresh, blockIdx.x == 0 ? a.status : nullptr);
    if (len >= 0) mine += line.line_units(len + fresh, a.own ? __ldcg(&a.own[i].x) : 0);
  }
  s_before[tid] = block_prefix<kThreads>(mine, s_warp, total);
  __syncthreads();
  const int64_t per = (total + kPieces - 1) / kPieces;
  const int piece = warp * kSms + blockIdx.x;               // few units: a warp on each SM first
  const int64_t u0 = piece * per;
  Place c;                              // where the arithmetic is
  c.left = min(per, total - u0);
  if (lane == 0) a.cut[piece] = make_int4(0, 0, 0, 0);
  if (c.left <= 0) return pdl_wait();
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
    if (c.n == 0) return pdl_wait();
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
      ids = __ldcg(a.c.table + (int64_t)f.i * a.c.table_stride + (row >> a.c.page_shift));
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
  // Rows that were there before the step need not wait for it to be prepared.
  int loaded = 0;
  for (; loaded < 2 && f.n > 0 && f.start + (f.off + f_at + 1) * kUnitRows <= f.len - (int)fresh; ++loaded) {
    load_k();
    load_v();
  }
  // The queries and the appended rows. With shared rows they are there: the kernel in front has waited for them, and nothing of its own
  // is looked at here. So this one begins on every SM that has done its share of that.
  if (!a.items) {
    pdl_wait();
    pdl_launch_dependents();
  }
  for (; loaded < 2; ++loaded) {
    load_k();
    load_v();
  }

  uint32_t stage = 0, phase = 0;
  // A wait gave up: loads of this warp may still be in flight. They get time to land before shared memory is handed back. (And the
  // end of this kernel still says that those in front of it have ended.)
  auto settle = [&]() {
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 100000ull) {}
    pdl_wait();
  };
  // The queries of an item, of head g (zeros for absent heads), and of heads 2t and 2t + 1 the factor of their scores.
  struct Queries { uint32_t w[kWords]; float factor[2]; };
  auto fetch = [&](Queries& q, const Place& p) {
    const int64_t head = (int64_t)p.i * a.n_q_heads + p.kvh * a.group;
    const uint4* from = reinterpret_cast<const uint4*>(a.q + (head + g) * (4 * kWords) + t * kWords);
#pragma unroll
    for (int x = 0; x < kWords / 4; ++x) {
      const uint4 w = g < a.group ? __ldcg(from + x) : make_uint4(0u, 0u, 0u, 0u);
      q.w[4 * x] = w.x; q.w[4 * x + 1] = w.y; q.w[4 * x + 2] = w.z; q.w[4 * x + 3] = w.w;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) q.factor[h] = kE4m3 && 2 * t + h < a.group ? __ldcg(a.q_factor + head + 2 * t + h) : a.scale_log2;
  };
  Queries next_q;
  fetch(next_q, c);
  while (true) {
    // ---- a part of an item; the queries of the next one are on their way meanwhile
    const bool begins = c.off == 0, ends = c.off + c.n == c.units;
    uint32_t qh[D / 8], ql[D / 8];
#pragma unroll
    for (int x = 0; x < D / 8; ++x) {
      qh[x] = next_q.w[x];
      ql[x] = R::kParts == 2 ? next_q.w[(R::kParts - 1) * (D / 8) + x] : 0u;
    }
    const float scale[2] = {next_q.factor[0], next_q.factor[1]};
    Place next = c;
    line.advance(next);
    if (next.n > 0) fetch(next_q, next);
    float m[2] = {kNoScore, kNoScore}, l[2] = {0.f, 0.f}, acc[D / 16][4];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

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
    // ---- out
    // (Products with the scale of the values come last: divided by a sum of weights it may have no bits left in fp32.)
    const float v_scale = kE4m3 ? a.c.v_scale[c.kvh] : 1.f;
    auto part = [&](float x) { return kE4m3 ? x * (1.f / R::kWeight) * v_scale : x; };
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
    if (begins && ends && !a.items) {
      // (a row that attends to nothing is 0; one all of whose scores are -inf is a NaN)
      const bool none = c.len == 0;
      R::leave(acc, none ? 0.f : 1.f / (l[0] * R::kWeight), none ? 0.f : 1.f / (l[1] * R::kWeight), v_scale, scratch, g, t);
      __syncwarp();
      __nv_bfloat16* to = a.o + ((int64_t)c.i * a.n_q_heads + c.kvh * a.group) * D;
      for (int x = lane; x < a.group * D / 8; x += 32) *reinterpret_cast<uint4*>(to + 8 * x) = shared16(scratch + 16 * x);
      __syncwarp();
    } else {
      const bool whole = begins && ends;
      const int64_t item = (int64_t)c.i * a.n_kv_heads + c.kvh, to_row = (whole ? item : 2 * (int64_t)piece + (begins ? 1 : 0)) * a.group;
      float2* to_ml = (whole ? a.row_ml : a.part_ml) + to_row;
      float* to_o = (whole ? a.row_o : a.part_o) + to_row * D;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = 2 * t + h;
        if (head >= a.group) continue;
        if (g == 0) to_ml[head] = make_float2(m[h], l[h]);
        float* to = to_o + head * D + (D / 8) * g;
#pragma unroll
        for (int j = 0; j < D / 16; j += 4)       // (whole sectors: 32 bytes a store)
          asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                       ::"l"(to + 2 * j), "f"(part(acc[j][h])), "f"(part(acc[j][2 + h])), "f"(part(acc[j + 1][h])), "f"(part(acc[j + 1][2 + h])),
                         "f"(part(acc[j + 2][h])), "f"(part(acc[j + 2][2 + h])), "f"(part(acc[j + 3][h])), "f"(part(acc[j + 3][2 + h])) : "memory");
      }
      if (begins && lane == 0) {        // the pieces over which the item goes on: units behind this one's end
        const int parts = whole ? 0 : 1 + (int)((c.units - c.n + per - 1) / per);
        if (a.items) a.items[item] = make_int2(piece, parts);
        else a.cut[piece] = make_int4(c.i, c.kvh, parts, 0);
      }
    }
    if (next.n == 0) return pdl_wait();     // (the kernel after this one counts on all in front of it)
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
      ml[c] = __ldcg(mls + from);
      const float* src = os + from * D + E * lane;
      if constexpr (E == 4) {
        const float4 x = __ldcg(reinterpret_cast<const float4*>(src));
        p[c][0] = x.x; p[c][1] = x.y; p[c][2] = x.z; p[c][3] = x.w;
      } else {
        const float2 x = __ldcg(reinterpret_cast<const float2*>(src));
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
template <int D>
__device__ __forceinline__ Joined<D> join_two(const Joined<D>& x, const Joined<D>& y) {
  const float m = fmaxf(x.m, y.m), f = x.l == 0.f ? 0.f : ex2(x.m - m), g = y.l == 0.f ? 0.f : ex2(y.m - m);
  Joined<D> s{m, x.l * f + y.l * g, {}};
#pragma unroll
  for (int e = 0; e < Joined<D>::E; ++e) s.o[e] = x.o[e] * f + y.o[e] * g;
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
// What a step prepares
// ------------------------------------------------------------------------------------------
// CTAs (i < k, part): prompt i's queries, rotated, in the order of the words that the products take (and, with shared rows, as rows for the
// tensor cores of their kernel); its new token's key, rotated, and value, into its pages. With shared rows the last CTA lays their
// work out: how many rows each group really shares (no more than its shortest prompt has, whole pages), and the line of units.
constexpr int kPrepareThreads = 256;
struct PrepareArgs {
  PagedArgs a;
  SharedPlan plan;
  const int32_t* shared_len;
};

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kPrepareThreads)
step_prepare_kernel(const __grid_constant__ PrepareArgs p) {
  using R = Rows<D, kE4m3>;
  const PagedArgs& a = p.a;
  const SharedPlan& plan = p.plan;
  const int tid = threadIdx.x, k = a.n_prompts;
  const bool fresh = a.k_new != nullptr;
  pdl_wait();
  pdl_launch_dependents();
  if ((int)blockIdx.x < k) {
    constexpr int kHalf = D / 2, kUnits = kHalf / 4, kSize = kE4m3 ? 1 : 2;      // units: four (j, j + D/2) pairs of a head
    __shared__ __align__(16) float s_cos[kHalf], s_sin[kHalf];
    const int i = blockIdx.x, len = checked_length(a.c, a.lengths, i, fresh, nullptr);
    if (len < 0) return;                // (what its rows of the workspace hold is not read)
    int64_t to = -1;                    // byte offset of the new row
    if (fresh) {
      const int page = a.c.table[(int64_t)i * a.c.table_stride + (len >> a.c.page_shift)];
      if ((unsigned)page < (unsigned)a.c.n_pages) to = (int64_t)page * a.c.page_stride + (int64_t)(len & ((1 << a.c.page_shift) - 1)) * a.c.row_stride;
      else if (tid == 0) note_status(a.status, PP_PAGED_BAD_PAGE);
    }
    const __nv_bfloat16 *q = a.q_new + (int64_t)i * a.q_stride, *kn = a.k_new + (int64_t)i * a.k_stride, *vn = a.v_new + (int64_t)i * a.v_stride;
    const int q_units = a.n_q_heads * kUnits, units = q_units + (to >= 0 ? a.n_kv_heads * kUnits : 0);
    for (int u0 = blockIdx.y * kPrepareThreads; u0 < units || u0 == (int)blockIdx.y * kPrepareThreads; u0 += gridDim.y * kPrepareThreads) {    // queries, then keys
      const int u = u0 + tid, h = u / kUnits, j = 4 * (u - h * kUnits), kvh = h < a.n_q_heads ? h / a.group : h - a.n_q_heads;
      uint2 lo = make_uint2(0u, 0u), hi = lo;
      if (u < units) {
        const __nv_bfloat16* src = u < q_units ? q + (int64_t)h * D : kn + (int64_t)kvh * D;
        lo = *reinterpret_cast<const uint2*>(src + j);
        hi = *reinterpret_cast<const uint2*>(src + j + kHalf);
      }
      if (u0 == (int)blockIdx.y * kPrepareThreads) {
        if (tid < kHalf) angle(fresh ? len : max(len - 1, 0), a.angles.inv_freq[tid], s_cos[tid], s_sin[tid]);
        __syncthreads();
      }
      const float2 p0 = unpack_bf16(lo.x), p1 = unpack_bf16(lo.y), y0 = unpack_bf16(hi.x), y1 = unpack_bf16(hi.y);
      const float4 cs = *reinterpret_cast<const float4*>(&s_cos[j]), sn = *reinterpret_cast<const float4*>(&s_sin[j]);
      float x[4] = {turn_lo(p0.x, y0.x, cs.x, sn.x), turn_lo(p0.y, y0.y, cs.y, sn.y), turn_lo(p1.x, y1.x, cs.z, sn.z), turn_lo(p1.y, y1.y, cs.w, sn.w)};
      float y[4] = {turn_hi(p0.x, y0.x, cs.x, sn.x), turn_hi(p0.y, y0.y, cs.y, sn.y), turn_hi(p1.x, y1.x, cs.z, sn.z), turn_hi(p1.y, y1.y, cs.w, sn.w)};
      int shift = 0;
      if constexpr (kE4m3) {
        // f16 has 5 exponent bits: a query is brought to below 2 by a power of two (of up to 2^120: the rest f16 has room
        // for), which goes into its factor. (The lanes of a head are neighbours.)
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(x[e]), fabsf(y[e])));
#pragma unroll
        for (int o = kUnits / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        shift = min(max((int)(__float_as_uint(top) >> 23) - 127, -120), 120);
      }
      if (u >= units) continue;
      if (u < q_units) {
        if constexpr (kE4m3) {
          const float down = __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
          for (int e = 0; e < 4; ++e) { x[e] *= down; y[e] *= down; }
          // The factor stays a normal number: hidden rows are -inf before it is applied, and -inf times 0 would be a NaN. (A query of zeros
          // over keys of a scale below 7e-9 had a factor of 0. One of 2^-126 brings every sum of products to below 2^-109 too.)
          if (j == 0) {
            const double factor = (double)a.scale_log2 * a.c.k_scale[kvh] * __uint_as_float((uint32_t)(127 + shift) << 23);
            a.q_factor[(int64_t)i * a.n_q_heads + h] = (float)fmin(fmax(factor, (double)FLT_MIN), (double)FLT_MAX);
          }
        }
        uint32_t* words = a.q + ((int64_t)i * a.n_q_heads + h) * (R::kParts * D / 2);
        const uint32_t high[4] = {R::high(x[0], x[1]), R::high(x[2], x[3]), R::high(y[0], y[1]), R::high(y[2], y[3])};
        const uint32_t low[4] = {R::low(x[0], x[1], high[0]), R::low(x[2], x[3], high[1]), R::low(y[0], y[1], high[2]), R::low(y[2], y[3], high[3])};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int e = j + (n & 1) * 2 + (n >> 1) * kHalf;
          uint32_t* word = words + R::word_thread(e) * (R::kParts * D / 8) + R::word_index(e);
          word[0] = high[n];
          if constexpr (R::kParts == 2) word[D / 8] = low[n];
        }
        if (plan.n_groups > 0) {
          __nv_bfloat16* row = plan.q_rot + (((int64_t)kvh * k + i) * a.group + h - kvh * a.group) * D + j;
          *reinterpret_cast<uint2*>(row) = make_uint2(high[0], high[1]);
          *reinterpret_cast<uint2*>(row + kHalf) = make_uint2(high[2], high[3]);
          row += (int64_t)k * a.n_q_heads * D;
          *reinterpret_cast<uint2*>(row) = make_uint2(low[0], low[1]);
          *reinterpret_cast<uint2*>(row + kHalf) = make_uint2(low[2], low[3]);
        }
      } else {
        char* row = a.c.k_pages + to + (int64_t)kvh * a.c.head_stride + j * kSize;
        if constexpr (kE4m3) {
          const float per = __frcp_rn(a.c.k_scale[kvh]);
          *reinterpret_cast<uint32_t*>(row) = round_e4m3(x[0] * per, x[1] * per, x[2] * per, x[3] * per);
          *reinterpret_cast<uint32_t*>(row + kHalf) = round_e4m3(y[0] * per, y[1] * per, y[2] * per, y[3] * per);
        } else {
          *reinterpret_cast<uint2*>(row) = make_uint2(round_bf16(x[0], x[1]), round_bf16(x[2], x[3]));
          *reinterpret_cast<uint2*>(row + D) = make_uint2(round_bf16(y[0], y[1]), round_bf16(y[2], y[3]));
        }
      }
    }
    if (to < 0) return;
    for (int u = blockIdx.y * kPrepareThreads + tid; u < a.n_kv_heads * (D / 8); u += gridDim.y * kPrepareThreads) {
      const int h = u / (D / 8), c = 8 * (u - h * (D / 8));
      const uint4 v = load16(vn + (int64_t)h * D + c);
      char* row = a.c.v_pages + to + (int64_t)h * a.c.head_stride + c * kSize;
      if constexpr (kE4m3) {
        float x[8];
        widen8(v, x);
        *reinterpret_cast<uint2*>(row) = narrow8(x, __frcp_rn(a.c.v_scale[h]));
      } else {
        *reinterpret_cast<uint4*>(row) = v;
      }
    }
    return;
  }
  if (blockIdx.y > 0) return;
  extern __shared__ int32_t s_plan[];   // group_ptr [n_groups + 1], the rows shared [n_groups], the first prompt of each group
  __shared__ int64_t s_warp[kPrepareThreads / 32];
  __shared__ int s_bad, s_wide;
  const int n = plan.n_groups;
  int32_t *s_ptr = s_plan, *s_rows = s_plan + n + 1, *s_lead = s_rows + n;
  if (tid == 0) s_bad = s_wide = 0;
  __syncthreads();
  for (int g = tid; g <= n; g += kPrepareThreads) {
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
  for (int i = tid; i < k; i += kPrepareThreads) {
    const int g = group_of(i), len = checked_length(a.c, a.lengths, i, fresh, nullptr);
    if (g >= 0 && len >= 0) {
      atomicMin(&s_rows[g], len);
      atomicMin(&s_lead[g], i);
    }
  }
  __syncthreads();
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int each = (n + kPrepareThreads - 1) / kPrepareThreads, g0 = min(tid * each, n), g1 = min(g0 + each, n);
  int64_t units = 0, parts = 0;
  for (int g = g0; g < g1; ++g) {
    const int prompts = bad ? 0 : s_ptr[g + 1] - s_ptr[g];
    const int rows = prompts > 0 && s_lead[g] < k ? s_rows[g] & ~page_mask : 0;      // (a group may be all rows of no prompt)
    s_rows[g] = rows;
    if (rows > 0 && prompts * a.group > kSharedTileRows / 2) s_wide = 1;
    const int tiles = (rows + kSharedTileKeys - 1) / kSharedTileKeys;
    units += (int64_t)tiles * ((prompts * a.group + kSharedTileRows - 1) / kSharedTileRows) * a.n_kv_heads;
    parts += (int64_t)shared_part_rows(prompts * a.group) * a.n_kv_heads;
  }
  int64_t all, none, at = block_prefix<kPrepareThreads>(units, s_warp, all), part = block_prefix<kPrepareThreads>(parts, s_warp, none);
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
  if (tid == 0) {
    plan.units[0] = all;
    plan.units[1] = s_wide;
  }
  __syncthreads();
  for (int i = tid; i < k; i += kPrepareThreads) {
    const int g = group_of(i);
    plan.prompts[i] = make_int2(g >= 0 && a.lengths[i] >= 0 ? s_rows[g] : 0, g);
  }
}

// With shared rows: joins the parts of every query head, those over the rows that its prompt shares, from the CTAs of their kernel, and
// those over its own. A warp for each head of each prompt, or, of few, a CTA (kAcross).
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
  const int i = (int)(row / a.n_q_heads), head = (int)(row - (int64_t)i * a.n_q_heads), kvh = head / a.group, h = head - kvh * a.group;
  const bool fresh = a.k_new != nullptr;
  const int len = checked_length(a.c, a.lengths, i, fresh, nullptr);
  const int2 own = __ldcg(plan.prompts + i), item = __ldcg(a.items + (int64_t)i * a.n_kv_heads + kvh);
  const int64_t per = units_per_piece(__ldcg(plan.units), plan.n_ctas);
  if (len < 0) return;
  // (a row that attends to nothing is 0; one all of whose scores are -inf is a NaN)
  const bool none = len + (int)fresh == 0;
  __nv_bfloat16* to = a.o + row * D;
  auto own_row = [&](int part) { return (2 * (int64_t)item.x + (part == 0 ? 1 : 2 * part)) * a.group + h; };
  auto whole_row = [&](int) { return row; };
  int n = 0, item_rows = 0, sides = 1;
  int64_t at = 0;
  if (own.x > 0) {
    const SharedGroup gr = plan.groups[own.y];
    const int r = (i - gr.first) * a.group + h, rt = r / kSharedTileRows;
    const int64_t u0 = gr.unit_start + ((int64_t)kvh * ((gr.query_rows + kSharedTileRows - 1) / kSharedTileRows) + rt) * gr.key_tiles;
    const int p0 = (int)(u0 / per);
    n = (int)((u0 + gr.key_tiles - 1) / per) - p0 + 1;
    // (an item of few rows has two parts in each piece, see pp_paged.h)
    item_rows = min(gr.query_rows - rt * kSharedTileRows, kSharedTileRows);
    sides = item_rows <= kSharedTileRows / 2 ? 2 : 1;
    at = (int64_t)p0 * kSharedTileRows + gr.part_start + (int64_t)kvh * shared_part_rows(gr.query_rows) + r;
  }
  auto shared_row = [&](int part) { return at + (int64_t)(sides == 2 ? part >> 1 : part) * kSharedTileRows + (sides == 2 && (part & 1) ? item_rows : 0); };
  const int first = kAcross ? warp : 0, step = kAcross ? kWarps : 1;
  Joined<D> s = item.y > 0 ? join_parts<D, 4>(first, step, item.y, a.part_ml, a.part_o, lane, own_row)
                           : join_parts<D, 1>(first, step, 1, a.row_ml, a.row_o, lane, whole_row);
  if (n > 0) s = join_two(s, join_parts<D, 4>(first, step, n * sides, plan.ml, plan.o, lane, shared_row));
  if constexpr (kAcross) {
    join_warps<D, kWarps>(s, space, [&](float, float l, float o, int place) { to[R::element_at(place)] = __float2bfloat16_rn(none ? 0.f : o / l); });
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) to[R::element_at(E * lane + e)] = __float2bfloat16_rn(none ? 0.f : s.o[e] / s.l);
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
cudaError_t launch_paged_decode(const PagedArgs& a, cudaStream_t s) {
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
  e = launch_dependent(paged_decode_kernel<D, kE4m3>, dim3(kSms), dim3(32 * kWarps), (size_t)kSmem, s, mk, mv, a);
  if (e != cudaSuccess || a.items) return e;          // (with shared rows another kernel joins the parts)
  constexpr int kPieces = kSms * kWarps, kJoiners = kCombineThreads / 32;
  using R = Rows<D, kE4m3>;
  if (kPieces * a.group <= 8 * kSms) return launch_dependent(paged_combine_kernel<D, R, true>, dim3(kPieces, a.group), dim3(kCombineThreads), 0, s, a, kPieces);
  return launch_dependent(paged_combine_kernel<D, R, false>, dim3((kPieces + kJoiners - 1) / kJoiners, a.group), dim3(kCombineThreads), 0, s, a, kPieces);
}

template <int D, bool kE4m3>
cudaError_t launch_prepare(const PrepareArgs& p, cudaStream_t s) {
  static DeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(step_prepare_kernel<D, kE4m3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kMaxPagedPrompts + 1) * (int)sizeof(int32_t));
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  const int n = p.plan.n_groups;
  // a thread for each four pairs of a head, as long as all CTAs run at once
  const int64_t units = ((int64_t)p.a.n_q_heads + p.a.n_kv_heads) * (D / 8);
  const int parts = (int)std::min<int64_t>((units + kPrepareThreads - 1) / kPrepareThreads, std::max(8 * kSms / p.a.n_prompts, 1));
  return launch_dependent(step_prepare_kernel<D, kE4m3>, dim3(p.a.n_prompts + (n > 0), parts), dim3(kPrepareThreads), n > 0 ? (3 * (size_t)n + 1) * sizeof(int32_t) : 0, s, p);
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
  a.items = n_groups > 0 ? reinterpret_cast<int2*>(ws + L.items) : nullptr;
  a.row_ml = reinterpret_cast<float2*>(ws + L.row_ml);
  a.row_o = reinterpret_cast<float*>(ws + L.row_o);
  a.q = reinterpret_cast<uint32_t*>(ws + L.q);
  a.q_factor = reinterpret_cast<float*>(ws + L.q_factor);
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
    plan.group_ptr = group_ptr;
    plan.n_groups = n_groups;
    plan.n_ctas = kSms;
  }
  const bool e4m3 = cache->type == PP_CACHE_E4M3;
  const PrepareArgs p{a, plan, shared_len};
  const cudaError_t prepared = d == 128 ? (e4m3 ? launch_prepare<128, true>(p, s) : launch_prepare<128, false>(p, s))
                                        : (e4m3 ? launch_prepare<64, true>(p, s) : launch_prepare<64, false>(p, s));
  if (prepared != cudaSuccess) return note_cuda_error((int)prepared, "step preparation launch");
  if (n_groups > 0) {
    if ((st = launch_shared_attention(*params, a.c, plan, k, a.scale_log2, device_status, s)) != PP_OK) return st;
  }
  cudaError_t e = d == 128 ? (e4m3 ? launch_paged_decode<128, true>(a, s) : launch_paged_decode<128, false>(a, s))
                           : (e4m3 ? launch_paged_decode<64, true>(a, s) : launch_paged_decode<64, false>(a, s));
  if (e == cudaSuccess && n_groups > 0) {
    const int64_t heads = (int64_t)k * params->n_q_heads;
    const bool across = heads <= 8 * kSms;          // as long as a CTA for each runs at once
    const dim3 blocks((unsigned)(across ? heads : (heads + kCombineThreads / 32 - 1) / (kCombineThreads / 32)));
    auto join = [&](auto kernel) { return launch_dependent(kernel, blocks, dim3(kCombineThreads), 0, s, a, plan); };
    e = d == 128 ? (across ? join(shared_join_kernel<128, true>) : join(shared_join_kernel<128, false>))
                 : (across ? join(shared_join_kernel<64, true>) : join(shared_join_kernel<64, false>));
  }
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
  L.q = take((size_t)k * p.n_q_heads * p.head_dim * sizeof(uint32_t));
  L.q_factor = take((size_t)k * p.n_q_heads * sizeof(float));
  L.part_ml = take(parts * sizeof(float2));
  L.part_o = take(parts * p.head_dim * sizeof(float));
  if (n_groups > 0) {
    L.units = take(2 * sizeof(int64_t));
    L.groups = take((size_t)n_groups * sizeof(SharedGroup));
    L.prompts = take((size_t)k * sizeof(int2));
    L.q_rot = take(2 * (size_t)k * p.n_q_heads * p.head_dim * sizeof(__nv_bfloat16));
    const size_t rows = (size_t)kSms * kSharedTileRows + 2 * (size_t)k * p.n_q_heads;
    L.shared_ml = take(rows * sizeof(float2));
    L.shared_o = take(rows * p.head_dim * sizeof(float));
    L.items = take((size_t)k * p.n_kv_heads * sizeof(int2));
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
