// Internal declarations of the paged cache: how kernels see it, and what the entry points launch.
#pragma once
#include "common.h"

namespace scalekv {

constexpr int kPageRowsMin = 16, kPageRowsMax = 256;  // powers of two
// Exponents of an e4m3 row's scale.  The least keeps every value (2^-9 the least code) a normal fp32 / bf16 number, the
// most is what the largest fp32 value needs.
constexpr int kScaleMin = -117, kScaleMax = 120;

// Element types: scalekv_dtype.
constexpr int kTypeF32 = 0, kTypeBf16 = 1, kTypeE4m3 = 2;

// Strides in bytes.  Row r of sequence s, KV head h: base + table[s * width + (r >> page_shift)] * page + h * head +
// (r & (page_rows - 1)) * row bytes; its scale byte likewise with the scales' strides and one byte a row.
struct PagesView {
  unsigned char *k, *v;
  uint8_t *k_scale, *v_scale;  // NULL unless the type is e4m3
  const int32_t *table, *len;
  long long page, head, scale_page, scale_head;
  int width, page_shift, n_page, n_kv_head;
  int type;
};
// Row i (of sequence s unless they are packed), head h: p + s * seq + h * head + i * row; i in [0, n_row).
struct RowsView {
  unsigned char* p;
  long long seq, head, row;
  int n_row;
};
// The new tokens of a sequence: `count` (at most max_new) rows from row `first` on.
struct ChunkView {
  int max_new;
  const int32_t *first, *count;
};
struct MaskView {
  int causal, window, n_sink;  // window 0: none
};

// What is read from device memory is brought into range here, so that no value of it leads out of a buffer: a page that
// is not in the pool reads as zeros and is not written, a length ends with the table, rows outside a tensor are skipped.
__device__ __forceinline__ int pages_len(const PagesView& c, int seq) {
  return min(max(c.len[seq], 0), c.width << c.page_shift);
}
__device__ __forceinline__ int chunk_count(const ChunkView& c, int seq) {
  return c.count ? min(max(c.count[seq], 0), c.max_new) : c.max_new;
}
__device__ __forceinline__ int chunk_first(const ChunkView& c, int seq) { return c.first ? c.first[seq] : 0; }

// rows of [n_seq, KV heads, max_new] -> pages
hipError_t launch_pages_write(int dtype, int d, int n_seq, const PagesView& pages, const RowsView& k, const RowsView& v,
                              const ChunkView& chunk, hipStream_t stream);
// rows [0, n_row) or idx [n_seq, n_head, n_row] of the pages -> dense caches
hipError_t launch_pages_read(int dtype, int d, int n_seq, int n_head, const PagesView& pages, const int32_t* idx, int n_row,
                             KvView k_dst, KvView v_dst, hipStream_t stream);

// How scalekv_pages_attend cuts its work.  A workgroup has query rows (token, query head) of one KV head, so that they
// share its rows of the cache.
struct PagesPlan {
  int row_waves;     // waves of a workgroup that split its query rows; the others split the keys of a tile
  int row_tiles;     // tiles of 16 query rows to a wave
  int target;        // workgroups that the keys are to be cut for, where that takes more than the rows do; 0: never
  int min_tiles;     // tiles that a workgroup has at least, where keys are cut
  int n_wg;          // workgroups of the launch: as many as there may be
  int rows() const { return 16 * row_waves * row_tiles; }
};
PagesPlan pages_plan(int dtype, int d, int n_seq, int n_head, const PagesView& pages, int max_new, const MaskView& mask);
// Workspace: the sums of every workgroup's rows, {offset, sum of weights} of each, {first workgroup, cuts} of each sequence.
inline size_t pages_partial_rows(int group, int max_new, const PagesPlan& plan) {
  const long long unit_rows = (long long)group * max_new;
  return (size_t)plan.n_wg * (size_t)(unit_rows < plan.rows() ? unit_rows : plan.rows());
}
inline size_t pages_partial_bytes(int n_seq, int d, int group, int max_new, const PagesPlan& plan) {
  if (plan.target == 0) return 0;
  return pages_partial_rows(group, max_new, plan) * (size_t)(d + 2) * sizeof(float) + (size_t)n_seq * 2 * sizeof(int);
}
hipError_t launch_pages_attend(int dtype, int d, int n_seq, int n_head, const PagesView& pages, const RowsView& q,
                               const RowsView& out, const ChunkView& chunk, const MaskView& mask, float sm_scale,
                               const PagesPlan& plan, void* ws, hipStream_t stream);

}  // namespace scalekv
