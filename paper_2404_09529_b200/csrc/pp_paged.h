// What the translation units of the paged cache share: the cache as the kernels see it, the workspace of the generation
// step, and the plan of a step in which prompts share pages.
#ifndef PREPACK_B200_PP_PAGED_H_
#define PREPACK_B200_PP_PAGED_H_

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "pp_internal.h"

namespace pp {

constexpr int kMaxPagedPrompts = 8192;   // and groups, of which the block that lays the shared work out holds three numbers each in shared memory
constexpr int kSharedTileRows = 256;     // query rows of a work item of the shared rows: two tiles of 128
constexpr int kSharedTileKeys = 128;

struct PagedCacheArgs {
  char *k_pages, *v_pages;
  const float *k_scale, *v_scale;
  const int32_t* table;
  int64_t page_stride, head_stride, row_stride;   // bytes
  int32_t n_pages, page_shift, table_stride;
};
inline PagedCacheArgs paged_cache_args(const pp_paged_cache& c) {
  PagedCacheArgs a;
  const int64_t size = c.type == PP_CACHE_E4M3 ? 1 : 2;
  a.k_pages = static_cast<char*>(c.k_pages);
  a.v_pages = static_cast<char*>(c.v_pages);
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.table = c.page_table;
  a.page_stride = c.page_stride * size;
  a.head_stride = c.head_stride * size;
  a.row_stride = c.row_stride * size;
  a.n_pages = c.n_pages;
  a.page_shift = 0;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.table_stride = c.table_stride;
  return a;
}

struct RopeAngles {
  double inv_freq[64];                  // theta_j = base^(-2j/D), computed in double on the host
};
RopeAngles rope_angles(float base, int32_t head_dim);

// Parts of results: (m, l), m in scaled log2 units, and the unnormalised sum of D floats for a query head.
// Own rows: pp_paged.cu. Shared rows (a kernel over kSharedTileRows x kSharedTileKeys tiles): the work is a line of
// units, one tile of keys against one tile of rows each, ordered by (group, KV head, row tile, key tile), and cut into equal
// pieces, one for each CTA. CTA c's part of an item (group, KV head, row tile) lies at rows c * kSharedTileRows + (part rows of all
// items before it) of the arrays: pieces and items both only ascend, and an item has at most kSharedTileRows part rows, one for each of
// its rows, or two where it has so few rows that both tiles of the kernel work on them (first all those of one, then of the other).
struct PagedWorkspace {
  size_t cut;                           // int4 for each piece of the line of own rows
  size_t q, q_factor;                   // the queries as the products take them
  size_t part_ml, part_o;               // float2, float[D]
  // with shared rows only
  size_t units;                         // int64 [2]: units in all; whether some group has more than half a row tile of queries
  size_t groups;                        // SharedGroup [n_groups]
  size_t prompts;                       // int2 [k]: first row that the prompt reads on its own, its group (-1: none)
  size_t q_rot;                         // bf16 [upper, lower part][Hkv][k * group][D]
  size_t shared_ml, shared_o;           // float2, float[D]: parts
  size_t items, row_ml, row_o;          // int2 [k][Hkv]; float2, float[D] [k][Hq]: of items that are not cut
  size_t total;
};
PagedWorkspace paged_workspace(const pp_attn_params& p, int32_t k, int32_t n_groups);

// A group, as the plan leaves it: what a kernel needs to know of it is one load away.
struct alignas(16) SharedGroup {
  int64_t unit_start, part_start;       // units and part rows before the group's
  int32_t key_tiles;                    // of the shared rows
  int32_t shared_rows;                  // rows of pages read for the group
  int32_t lead;                         // the prompt whose row of the page table stands for the group's
  int32_t first, query_rows;            // first prompt; query rows per KV head
  int32_t pad[3];
};
// The plan of the shared rows as the kernels find it in the workspace.
struct SharedPlan {
  int64_t* units;
  SharedGroup* groups;
  int2* prompts;
  __nv_bfloat16* q_rot;
  float2* ml;
  float* o;
  const int32_t* group_ptr;
  int32_t n_groups, n_ctas;             // n_ctas: pieces that the line of units is cut into
};

int launch_shared_attention(const pp_attn_params& p, const PagedCacheArgs& c, const SharedPlan& plan, int32_t k, float scale_log2,
                            int32_t* status, cudaStream_t stream);

#ifdef __CUDACC__
// Units of each piece.
__device__ __forceinline__ int64_t units_per_piece(int64_t units, int32_t n_ctas) { return (units + n_ctas - 1) / n_ctas; }
// Part rows of a group and KV head with so many query rows.
__device__ __forceinline__ int shared_part_rows(int rows) {
  const int last = rows % kSharedTileRows;
  return rows + (last <= kSharedTileRows / 2 ? last : 0);
}
#endif

}  // namespace pp

#endif  // PREPACK_B200_PP_PAGED_H_
