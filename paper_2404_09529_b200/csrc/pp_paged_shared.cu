// Attention of the rows that the prompts of a group share, for sm_100a: for every (group, KV head) the queries of all prompts of
// the group, `group` heads each, are the rows of tensor-core tiles that meet the shared keys once:
//   m, l, o[D] of every query over the shared rows,   s = q' . k scale,  o = sum_j 2^(s_j - m) v_j,  l = sum_j 2^(s_j - m)
// unnormalised, to be joined with the prompt's own rows by the kernel after. Nothing is masked but the end of the last tile.
//
// Read once per group the rows cost (samples of a prompt) x less HBM traffic; what bounds is HBM for groups of up to about
// 128 queries per KV head, and the exponentials and products beyond. Work is cut into one equal piece for each CTA of a
// line of (row tile pair, key tile) units (pp_paged.h), so that CTAs finish together whatever the groups are like.
//   warp 0       finds the pieces, TMA-loads the K / V tiles of 128 keys into one ring; a lane per page (and 64 columns)
//   warp 1       issues tcgen05.mma: S_t = Q_t K^T into TMEM, O_t += P_t V with P_t read from TMEM, for the two row tiles t
//   warps 2-3    TMA-load Q of tile 0 / 1, as two bf16 numbers, which the products add up: one alone moves O by as much as its last
//                rounding does (against 64 bits, O's last rounding being 1.7e-3 of it: 16 samples of a prompt of 2000 rows 2.7e-3 with
//                one, 2.1e-3 with two, 22.0 and 22.3 us; 24 prompts of 8 samples 2.6e-3 and 2.1e-3, 178 and 193; 64 prompts behind 32 700
//                rows, heads of 64, 2.9e-3 and 2.3e-3, 52.4 and 52.8; 256 prompts behind 8200 rows 2.9e-3 and 2.3e-3, 113 and 120).
//                P is one bf16 number: two would double the conversions of the softmax, which bounds, and P V.
//   warps 4-7    softmax of tile 0, a thread per row: no row is split between threads, so nothing is exchanged
//   warps 8-11   the same for tile 1
// A tile's softmax runs while the other tile's products do. An item of at most 128 rows has no second row tile: the two then take its
// key tiles in turn, each with an O of its own, so that there are two chains of product, softmax and product here too. The pages of a
// tile that the group does not share are loaded from beyond the last page, which TMA fills with zeros.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>

#include "pp_device_once.h"
#include "pp_paged.h"
#include "pp_tcgen05.h"

namespace pp {
namespace {

constexpr int BM = 128, BN = kSharedTileKeys;
constexpr int kSharedThreads = 384;
constexpr uint32_t kTmemCols = 512;
constexpr int kRegsSoftmax = 208, kRegsOther = 80;      // 384 threads start with 168: 256 * 208 + 128 * 80 <= 384 * 168
constexpr uint32_t kRing = 3;                           // pieces in flight between warp 0 and their readers
constexpr int kRingInts = 8;
// The running maximum of a row moves only when a score exceeds it by more than 2^8: the sums are then at most 2^8 as large,
// which costs fp32 and bf16 nothing, and O is rarely rescaled.
constexpr float kLazyLog2 = 8.f;

template <int D> struct SharedCfg {
  static constexpr int kQBytes = BM * D * 2, kTileBytes = BN * D * 2;
  static constexpr int kMiscBytes = 1024;
  // Tile t's part x of Q lies at (2 t + x) kQBytes, and behind the queries the ring. Both parts of both tiles leave it three stages with
  // heads of 128. Where no group has more than 128 queries for a KV head, nothing needs the second tile's room, and it has five (24 prompts
  // of 8 samples, 32 heads of 128: 190 to 194 us with five, 204 with three).
  static constexpr int kSlots = D == 128 ? 7 : 14;
  static constexpr int kStages = D == 128 ? 5 : 10, kWideStages = D == 128 ? 3 : 10;
  static __device__ __forceinline__ uint32_t q_at(uint32_t t, uint32_t part) { return (2u * t + part) * (uint32_t)kQBytes; }
  static __device__ __forceinline__ uint32_t stage_of(uint32_t tile, bool wide) { return kStages == kWideStages || !wide ? tile % kStages : tile % kWideStages; }
  static __device__ __forceinline__ uint32_t turn_of(uint32_t tile, bool wide) { return kStages == kWideStages || !wide ? tile / kStages : tile / kWideStages; }
  static constexpr int kSmemBytes = kMiscBytes + 1024 + kSlots * kTileBytes;     // tiles on 1024-byte boundaries
  static_assert(kQBytes == kTileBytes && 4 + kWideStages <= kSlots && (D == 64 ? 4 : 2) + kStages <= kSlots, "shared memory");
};
static_assert(SharedCfg<128>::kSmemBytes <= 227 * 1024 && SharedCfg<64>::kSmemBytes <= 227 * 1024, "shared memory");

struct SharedArgs {
  SharedPlan plan;
  const int32_t* table;
  int32_t table_stride, page_shift, n_pages;
  int32_t n_kv_heads, group;
  float scale_log2;
  int32_t* status;
  uint32_t wait_limit;                  // in units of 1024 ns
};

enum WaitCode { kWaitItemFull = 21, kWaitItemEmpty, kWaitQFull, kWaitQEmpty, kWaitKvFull, kWaitKvEmpty, kWaitS, kWaitP, kWaitOFull, kWaitOEmpty };

// Coordinates: column (0), row of the page, chunk of 64 columns, head, page. Every lane whose `issue` is set loads its own box.
__device__ __forceinline__ void load_page(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row, int chunk, int head, int page, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %7, 0;\n"
      "@q cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%8, %3, %4, %5, %6}], [%2];\n}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(row), "r"(chunk), "r"(head), "r"(page), "r"(issue), "r"(0)
      : "memory");
}
// Coordinates: column (0), row, chunk (0), head (those of the lower parts behind those of the upper ones).
__device__ __forceinline__ void load_queries(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row, int head, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %5, 0;\n"
      "@q cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%6, %3, %6, %4}], [%2];\n}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(row), "r"(head), "r"(issue), "r"(0)
      : "memory");
}

template <int D>
__global__ void __launch_bounds__(kSharedThreads, 1)
shared_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const __grid_constant__ SharedArgs args) {
  using Cfg = SharedCfg<D>;
  constexpr uint32_t NS = Cfg::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t s_misc = smem_u32(smem_raw);
  const uint32_t s_q = (s_misc + Cfg::kMiscBytes + 1023u) & ~1023u;
  const uint32_t bar_item_full = s_misc, bar_item_empty = s_misc + 32;      // [kRing] each
  const uint32_t bar_q_full = s_misc + 64, bar_q_empty = s_misc + 80;       // [2] each, and so on
  const uint32_t bar_s_full = s_misc + 96, bar_p_full = s_misc + 112;
  const uint32_t bar_o_full = s_misc + 128, bar_o_empty = s_misc + 144;
  const uint32_t bar_kv_full = s_misc + 160, bar_kv_empty = s_misc + 256;   // [NS] each
  static_assert(NS <= 12 && kRing <= 4, "barrier slots");
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(smem_raw + 352);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem_raw + 356);
  volatile int* s_ring = reinterpret_cast<volatile int*>(smem_raw + 384);   // [kRing][kRingInts]
  const int warp = uniform((int)(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const WaitCtx wctx{s_misc + 356u, args.wait_limit, args.status};

  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < kRing; ++i) {
      mbar_init(bar_item_full + 8 * i, 1);
      mbar_init(bar_item_empty + 8 * i, 1 + 2 + 8);             // the issuer, two loaders, a lane of each softmax warp
    }
    for (uint32_t t = 0; t < 2; ++t) {
      mbar_init(bar_q_full + 8 * t, 1);
      mbar_init(bar_q_empty + 8 * t, 1);
      mbar_init(bar_s_full + 8 * t, 1);
      mbar_init(bar_p_full + 8 * t, BM);
      mbar_init(bar_o_full + 8 * t, 1);
      mbar_init(bar_o_empty + 8 * t, BM);
    }
    for (uint32_t s = 0; s < NS; ++s) {
      mbar_init(bar_kv_full + 8 * s, 1);
      mbar_init(bar_kv_empty + 8 * s, 1);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(s_tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = (uint32_t)uniform((int)*s_tmem_base);
  pdl_wait();                           // the plan, the rotated queries and the pages
  pdl_launch_dependents();
  // of the whole launch: some group has more than 128 queries for a KV head
  const bool wide = warp < 4 && args.plan.units[1] != 0;
  const uint32_t s_kv = s_q + (D == 64 || wide ? 4u : 2u) * Cfg::kQBytes;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 0) {
      // ---------------------------------------------------------------- pieces, K / V tiles
      const SharedPlan& plan = args.plan;
      const uint32_t issue = elect_one();
      const int64_t units = *plan.units, per = units_per_piece(units, plan.n_ctas);
      const int64_t u_end = min((int64_t)(blockIdx.x + 1) * per, units);
      const int page_rows = 1 << args.page_shift;
      // a lane's box: page `mine` of the tile, columns 64 * chunk ..
      constexpr int kChunks = D / 64;
      const int box_rows = min(page_rows, BN), boxes = BN / box_rows * kChunks;
      const int mine = lane / kChunks, chunk = lane - mine * kChunks;
      const uint32_t lane_issue = lane < boxes ? 1u : 0u;
      const uint32_t lane_dst = (uint32_t)(chunk * BN + mine * box_rows) * 128u;
      uint32_t it_n = 0, stage = 0, phase = 0;
      bool ok = true;
      for (int64_t u = (int64_t)blockIdx.x * per;; ) {
        const uint32_t ring = it_n % kRing;
        volatile int* e = s_ring + ring * kRingInts;
        if (!(ok = mbar_wait_issuer<kWaitItemEmpty>(bar_item_empty + 8 * ring, ((it_n / kRing) & 1u) ^ 1u, wctx))) break;
        if (u >= u_end) {
          if (issue) {
            e[0] = -1;
            mbar_arrive(bar_item_full + 8 * ring);
          }
          break;
        }
        // last group that begins at or before u (those without units come before it), 32 candidates at a time
        int gr = 0;
        for (int size = plan.n_groups; size > 1;) {
          const int step = (size + 31) >> 5, at = gr + lane * step;
          const bool before = lane * step < size && plan.groups[at].unit_start <= u;
          gr += (__popc(__ballot_sync(0xffffffffu, before)) - 1) * step;
          size = min(step, plan.n_groups - gr);
        }
        const SharedGroup g = plan.groups[gr];
        const int tiles = g.key_tiles, rows = g.query_rows, row_tiles = (rows + kSharedTileRows - 1) / kSharedTileRows;
        const int64_t within = u - g.unit_start;
        const int item = (int)(within / tiles), tile0 = (int)(within - (int64_t)item * tiles);
        const int kv_head = item / row_tiles, rt = item - kv_head * row_tiles;
        const int n = (int)min((int64_t)(tiles - tile0), u_end - u);
        const int rows_here = min(rows - rt * kSharedTileRows, kSharedTileRows), shared = g.shared_rows;
        const int64_t out = (int64_t)blockIdx.x * kSharedTileRows + g.part_start + (int64_t)kv_head * shared_part_rows(rows) + rt * kSharedTileRows;
        if (issue) {
          e[0] = n;
          e[1] = rows_here;
          e[2] = g.first * args.group + rt * kSharedTileRows;
          e[3] = kv_head;
          e[4] = min(shared - (tile0 + n - 1) * BN, BN);       // keys of the piece's last tile
          e[5] = (int)(uint32_t)out;
          e[6] = (int)(out >> 32);
          mbar_arrive(bar_item_full + 8 * ring);
        }
        const int32_t* table = args.table + (int64_t)g.lead * args.table_stride;
        auto page_of = [&](int tile) {            // page of this lane's box; beyond the last one: zeros
          const int key = tile * BN + mine * box_rows;
          if (!lane_issue || tile >= tile0 + n || key >= shared) return args.n_pages;
          const int id = table[key >> args.page_shift];
          if ((unsigned)id < (unsigned)args.n_pages) return id;
          if (args.status) atomicCAS(args.status, 0, PP_PAGED_BAD_PAGE);
          return args.n_pages;
        };
        int page = page_of(tile0);
        for (int j = 0; ok && j < n; ++j) {
          const int page_next = page_of(tile0 + j + 1);
          const int row = (tile0 + j) * BN & (page_rows - 1);   // (pages longer than a tile)
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const uint32_t full = bar_kv_full + 8 * stage;
            if (!(ok = mbar_wait_issuer<kWaitKvEmpty>(bar_kv_empty + 8 * stage, phase ^ 1u, wctx))) break;
            mbar_expect_tx(full, Cfg::kTileBytes, issue);
            __syncwarp();
            load_page(s_kv + stage * Cfg::kTileBytes + lane_dst, part ? &map_v : &map_k, full, row, chunk, kv_head, page, lane_issue);
            if (++stage == (wide ? (uint32_t)Cfg::kWideStages : NS)) { stage = 0; phase ^= 1u; }
          }
          page = page_next;
        }
        if (!ok) break;
        u += n;
        ++it_n;
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- products
      constexpr uint32_t idesc_qk = instr_desc(BN, false), idesc_pv = instr_desc(D, true);
      const uint32_t q_lo = desc_lo(s_q, 0), k_lo = desc_lo(s_kv, 0), v_lo = desc_lo(s_kv, BN * 128);
      const uint32_t issue = elect_one();
      uint32_t it_n = 0, kv = 0, count[2] = {0, 0};       // kv: K and V tiles of the items before (K of tile j: kv + 2j)
      int n = 0;
      bool split = false, ok = true;
      auto wait_kv = [&](uint32_t at) { return mbar_wait_issuer<kWaitKvFull>(bar_kv_full + 8 * Cfg::stage_of(at, wide), Cfg::turn_of(at, wide) & 1u, wctx); };
      // The scores are what a tile's softmax waits for: their commit comes first, the one that gives the stages back after it.
      auto issue_qk = [&](int t, int j) {
        const uint32_t s = Cfg::stage_of(kv + 2u * (uint32_t)j, wide);
        tc_fence_after();
        const uint32_t b = k_lo + s * (Cfg::kTileBytes >> 4);
#pragma unroll 1
        for (uint32_t part = 0; part < 2; ++part) {
          const uint32_t a = q_lo + (Cfg::q_at(split ? 0u : (uint32_t)t, part) >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_ss(tmem_base + 128u * t, a + (uint32_t)(kk >> 2) * ((BM * 128) >> 4) + (uint32_t)(kk & 3) * 2,
                   b + (uint32_t)(kk >> 2) * ((BN * 128) >> 4) + (uint32_t)(kk & 3) * 2, idesc_qk, kk > 0 || part > 0 ? 1u : 0u, issue);
        }
        tc_commit(bar_s_full + 8 * t, issue);
        if (t == 1 || split) tc_commit(bar_kv_empty + 8 * s, issue);
        if (j + 1 == n) {
          tc_commit(bar_q_empty + (split ? 0 : 8 * t), issue);
          if (split) tc_commit(bar_q_empty + 8, issue);       // (a phase for each item, also where tile 1 has no queries of its own)
        }
      };
      // O_t (+)= P_t V_j, then the tile's next scores, those of key tile `next`. The next K is waited for first where it has been there
      // for long (heads of 64, unless the item is split). Otherwise it may be the one that is loaded last: the product goes first, and
      // so does what gives V's stage back (256 prompts behind 8200 rows, heads of 128: 124.7 -> 118.7 us).
      auto step = [&](int t, int j, bool first, int next) -> bool {
        if (first && !mbar_wait_issuer<kWaitOEmpty>(bar_o_empty + 8 * t, (it_n & 1u) ^ 1u, wctx)) return false;
        const uint32_t vc = kv + 2u * (uint32_t)j + 1u, s = Cfg::stage_of(vc, wide), kc = kv + 2u * (uint32_t)next;
        if (!wait_kv(vc)) return false;
        if (D == 64 && !split && next < n && !wait_kv(kc)) return false;
        if (!mbar_wait_issuer<kWaitP>(bar_p_full + 8 * t, count[t] & 1u, wctx)) return false;
        tc_fence_after();
        const uint32_t d = tmem_base + 256u + (uint32_t)(D * t), a = tmem_base + 128u * t, b = v_lo + s * (Cfg::kTileBytes >> 4);
#pragma unroll
        for (int kk = 0; kk < BN / 16; ++kk)
          mma_ts(d, a + kk * 8, b + (uint32_t)kk * ((16 * 128) >> 4), idesc_pv, kk > 0 || !first ? 1u : 0u, issue);
        ++count[t];
        if (next < n) {
          if (split || (D == 128 && t == 1)) tc_commit(bar_kv_empty + 8 * s, issue);
          if ((D == 128 || split) && !wait_kv(kc)) return false;
          issue_qk(t, next);
          if (D == 64 && !split && t == 1) tc_commit(bar_kv_empty + 8 * s, issue);
        } else {
          if (t == 1 || split) tc_commit(bar_kv_empty + 8 * s, issue);
          tc_commit(bar_o_full + 8 * t, issue);
        }
        return true;
      };
      while (ok) {
        const uint32_t ring = it_n % kRing;
        if (!mbar_wait_issuer<kWaitItemFull>(bar_item_full + 8 * ring, (it_n / kRing) & 1u, wctx)) break;
        const volatile int* e = s_ring + ring * kRingInts;
        n = uniform(e[0]);
        split = uniform(e[1]) <= BM;
        if (issue) mbar_arrive(bar_item_empty + 8 * ring);
        if (n < 0) break;
        if (!(ok = mbar_wait_issuer<kWaitQFull>(bar_q_full, it_n & 1u, wctx) && mbar_wait_issuer<kWaitQFull>(bar_q_full + 8, it_n & 1u, wctx) &&
                   wait_kv(kv)))
          break;
        issue_qk(0, 0);
        if (!split) {
          issue_qk(1, 0);
          for (int j = 0; ok && j < n; ++j) ok = step(0, j, j == 0, j + 1) && step(1, j, j == 0, j + 1);
        } else {
          if (n > 1) {
            if (!(ok = wait_kv(kv + 2u))) break;
            issue_qk(1, 1);
          }
          for (int j = 0; ok && j < n; ++j) ok = step(j & 1, j, j < 2, j + 2);
          if (ok && n == 1) {
            // Tile 1 has nothing, but keeps its barriers in step, one phase for each item; all of its softmax threads must have seen
            // the phase before.
            if (!(ok = mbar_wait_issuer<kWaitOEmpty>(bar_o_empty + 8, (it_n & 1u) ^ 1u, wctx))) break;
            if (issue) mbar_arrive(bar_o_full + 8);
          }
        }
        if (!ok) break;
        kv += 2u * (uint32_t)n;
        ++it_n;
      }
    } else {
      // ---------------------------------------------------------------- queries of tile t
      const int t = warp - 2;
      const uint32_t issue = elect_one();
      for (uint32_t it_n = 0;; ++it_n) {
        const uint32_t ring = it_n % kRing;
        if (!mbar_wait_issuer<kWaitItemFull>(bar_item_full + 8 * ring, (it_n / kRing) & 1u, wctx)) break;
        const volatile int* e = s_ring + ring * kRingInts;
        const int n = uniform(e[0]), rows = uniform(e[1]), q_row = uniform(e[2]), kv_head = uniform(e[3]);
        if (issue) mbar_arrive(bar_item_empty + 8 * ring);
        if (n < 0) break;
        if (!mbar_wait_issuer<kWaitQEmpty>(bar_q_empty + 8 * t, (it_n & 1u) ^ 1u, wctx)) break;
        if (t == 0 || rows > BM) {
          mbar_expect_tx(bar_q_full + 8 * t, 2 * Cfg::kQBytes, issue);
          for (uint32_t part = 0; part < 2; ++part)
            load_queries(s_q + Cfg::q_at((uint32_t)t, part), &map_q, bar_q_full + 8 * t, q_row + BM * t, (int)part * args.n_kv_heads + kv_head, issue);
        } else if (issue) {
          mbar_arrive(bar_q_full + 8 * t);
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax of tile t
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int t = (warp - 4) >> 2, quad = warp & 3, row = 32 * quad + lane;
    const uint32_t lane_at = (uint32_t)(32 * quad) << 16;
    const uint32_t tm_s = tmem_base + 128u * t + lane_at, tm_o = tmem_base + 256u + (uint32_t)(D * t) + lane_at;
    const float c_scale = args.scale_log2;
    const uint64_t c2 = pack_f2(__float_as_uint(c_scale), __float_as_uint(c_scale));
    uint32_t count = 0;
    for (uint32_t it_n = 0;; ++it_n) {
      const uint32_t ring = it_n % kRing;
      if (!mbar_wait_warp<kWaitItemFull>(bar_item_full + 8 * ring, (it_n / kRing) & 1u, wctx)) break;
      const volatile int* e = s_ring + ring * kRingInts;
      const int n = uniform(e[0]), item_rows = uniform(e[1]), last_keys = uniform(e[4]);
      const bool split = item_rows <= BM;
      const int rows = split ? item_rows : item_rows - BM * t;            // of this tile
      const int64_t out = (int64_t)((uint64_t)(uint32_t)uniform(e[5]) | ((uint64_t)(uint32_t)uniform(e[6]) << 32)) + (split ? item_rows : BM) * t;
      if (lane == 0) mbar_arrive(bar_item_empty + 8 * ring);
      if (n < 0) break;
      float m_run = -INFINITY, neg_m = 0.f;
      uint64_t sum_a = 0ull, sum_b = 0ull;
      bool ok = true;
      const bool idle = 32 * quad >= rows;        // a warp without rows leaves its P as it is: no other row reads it
      const int first = split ? t : 0, each = split ? 2 : 1;
      for (int j = first; j < n; j += each) {
        if (!(ok = mbar_wait_warp<kWaitS>(bar_s_full + 8 * t, count & 1u, wctx))) break;
        if (idle) {
          mbar_arrive(bar_p_full + 8 * t);
          ++count;
          continue;
        }
        tc_fence_after();
        uint32_t v[BN];
#pragma unroll
        for (int ch = 0; ch < BN / 32; ++ch) tmem_ld32(tm_s + 32 * ch, *reinterpret_cast<uint32_t(*)[32]>(&v[32 * ch]));
        tc_wait_ld();
        if (j + 1 == n && last_keys < BN) {
#pragma unroll
          for (int i = 0; i < BN; ++i) v[i] = i < last_keys ? v[i] : 0xff800000u;      // -inf
        }
        const float m_tile = fmaxf(max64(*reinterpret_cast<uint32_t(*)[64]>(&v[0])), max64(*reinterpret_cast<uint32_t(*)[64]>(&v[64]))) * c_scale;
        const float m_new = m_tile > m_run + kLazyLog2 ? m_tile : m_run;
        const bool rescale = m_new != m_run && m_run != -INFINITY;
        if (j != first && __any_sync(0xffffffffu, rescale)) {
          // (these scores are there, so the product before them, P V of the tile before, is done)
          const float alpha = rescale ? fast_exp2(m_run - m_new) : 1.f;
#pragma unroll 1
          for (int ch = 0; ch < D / 16; ++ch) {
            uint32_t ov[16];
            tmem_ld16(tm_o + ch * 16, ov);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * alpha);
            tmem_st16(tm_o + ch * 16, ov);
          }
          const uint64_t alpha2 = pack_f2(__float_as_uint(alpha), __float_as_uint(alpha));
          sum_a = mul_f2(sum_a, alpha2);
          sum_b = mul_f2(sum_b, alpha2);
        }
        m_run = m_new;
        neg_m = m_run == -INFINITY ? 0.f : -m_run;
        const uint64_t negm2 = pack_f2(__float_as_uint(neg_m), __float_as_uint(neg_m));
#pragma unroll
        for (int ch = 0; ch < BN / 32; ++ch) {
          uint32_t pk[16];
          exp_chunk(&v[32 * ch], c2, negm2, sum_a, sum_b, pk);
          tmem_st16(tm_s + 16 * ch, pk);
        }
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(bar_p_full + 8 * t);
        ++count;
      }
      if (!ok) break;
      if (!mbar_wait_warp<kWaitOFull>(bar_o_full + 8 * t, it_n & 1u, wctx)) break;
      if (!idle) {
        tc_fence_after();
        const bool any = first < n;               // (a tile that took no keys leaves l = 0, and its O is not looked at)
        if (row < rows) args.plan.ml[out + row] = make_float2(fmaxf(m_run, -FLT_MAX), sum_f2x2(sum_a, sum_b));
        float* dst = args.plan.o + (out + row) * D;
        if (any) {
          uint32_t ov[D];
#pragma unroll
          for (int ch = 0; ch < D / 32; ++ch) tmem_ld32(tm_o + 32 * ch, *reinterpret_cast<uint32_t(*)[32]>(&ov[32 * ch]));
          tc_wait_ld();
          if (row < rows) {
            // whole sectors, 32 bytes a store, in the order of the parts over own rows: element 16 j + 8 x + g at (D / 8) g + 2 j + x
#pragma unroll
            for (int to = 0; to < D; to += 8) {
              const int g = to / (D / 8), j = to % (D / 8) / 2;
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                           ::"l"(dst + to), "r"(ov[16 * j + g]), "r"(ov[16 * j + 8 + g]), "r"(ov[16 * j + 16 + g]), "r"(ov[16 * j + 24 + g]),
                             "r"(ov[16 * j + 32 + g]), "r"(ov[16 * j + 40 + g]), "r"(ov[16 * j + 48 + g]), "r"(ov[16 * j + 56 + g]) : "memory");
            }
          }
        }
        tc_fence_before();
      }
      mbar_arrive(bar_o_empty + 8 * t);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*s_abort) {
    if (threadIdx.x == 0 && args.status) atomicCAS(args.status, 0, *s_abort);
    // A wait gave up: loads and products of this CTA may still be in flight. They get time to land before shared
    // memory and TMEM are handed back.
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 100000ull) {}
    __syncthreads();
  }
  if (warp == 0) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

int encode(CUtensorMap* map, const void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeFn enc = get_encode_fn();
  if (!enc) return note_cuda_error(-1, "cuTensorMapEncodeTiled entry point not found");
  const cuuint32_t ones[5] = {1u, 1u, 1u, 1u, 1u};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(ptr), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? PP_OK : note_cuda_error((int)r, "cuTensorMapEncodeTiled");
}

template <int D>
int launch(const pp_attn_params& p, const PagedCacheArgs& c, const SharedArgs& a, int32_t k, cudaStream_t stream) {
  using Cfg = SharedCfg<D>;
  CUtensorMap mq, mk, mv;
  const cuuint64_t q_rows = (cuuint64_t)k * (cuuint64_t)a.group;
  const cuuint64_t q_dims[4] = {64u, q_rows, D / 64, 2 * (cuuint64_t)p.n_kv_heads}, q_strides[3] = {D * 2, 128u, q_rows * D * 2};
  const cuuint32_t q_box[4] = {64u, BM, D / 64, 1u};
  const cuuint64_t page_rows = (cuuint64_t)1 << c.page_shift;
  const cuuint64_t dims[5] = {64u, page_rows, D / 64, (cuuint64_t)p.n_kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)c.row_stride, 128u, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride};
  const cuuint32_t box[5] = {64u, (cuuint32_t)std::min<cuuint64_t>(page_rows, BN), 1u, 1u, 1u};
  int st;
  if ((st = encode(&mq, a.plan.q_rot, 4, q_dims, q_strides, q_box)) != PP_OK) return st;
  if ((st = encode(&mk, c.k_pages, 5, dims, strides, box)) != PP_OK) return st;
  if ((st = encode(&mv, c.v_pages, 5, dims, strides, box)) != PP_OK) return st;
  static DeviceOnce configured;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return note_cuda_error((int)e, "cudaGetDevice");
  if (!configured.done(dev)) {
    e = cudaFuncSetAttribute(shared_attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes);
    if (e != cudaSuccess) return note_cuda_error((int)e, "cudaFuncSetAttribute(smem)");
    configured.mark(dev);
  }
  e = launch_dependent(shared_attention_kernel<D>, dim3((unsigned)a.plan.n_ctas), dim3(kSharedThreads), (size_t)Cfg::kSmemBytes, stream, mq, mk, mv, a);
  return e == cudaSuccess ? PP_OK : note_cuda_error((int)e, "shared attention launch");
}

}  // namespace

int launch_shared_attention(const pp_attn_params& p, const PagedCacheArgs& c, const SharedPlan& plan, int32_t k, float scale_log2,
                            int32_t* status, cudaStream_t stream) {
  SharedArgs a;
  a.plan = plan;
  a.table = c.table;
  a.table_stride = c.table_stride;
  a.page_shift = c.page_shift;
  a.n_pages = c.n_pages;
  a.n_kv_heads = p.n_kv_heads;
  a.group = p.n_q_heads / p.n_kv_heads;
  a.scale_log2 = scale_log2;
  a.status = status;
  a.wait_limit = (uint32_t)std::min<unsigned long long>(wait_limit_ns() >> 10, 0x7fffffffu);
  return p.head_dim == 128 ? launch<128>(p, c, a, k, stream) : launch<64>(p, c, a, k, stream);
}

}  // namespace pp
