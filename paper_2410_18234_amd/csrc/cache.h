// The paged 8-bit cache of keys and values: geometry, code conversions and the kernels' arguments.
//
// A page holds `page_size` tokens of every head in units of 16 tokens.  Keys of a unit are [d / 16][16 tokens]
// [16 of d], values [d][16 tokens], so that the lane of a matrix product that owns a token (keys) or an element of
// d (values) finds 16 bytes of it together, whatever the page size.  A value is code * 2^exp with one exponent for
// a page and head; e4m3 keeps its relative precision under a power of two, so a page whose exponent grows loses
// only what falls below its smallest code.
#pragma once

#include "common.h"
#include "mdss.h"

namespace mdss {

constexpr int kCacheMinExp = -40, kCacheMaxExp = 40;
constexpr int kRowNoPage = 64;

struct CacheView {
  uint8_t *k, *v;
  int8_t *k_exp, *v_exp;
  int layers, heads, d, page_shift;  // page_size = 1 << page_shift
  int64_t pages;
  __host__ __device__ int page_size() const { return 1 << page_shift; }
  __host__ __device__ int64_t region() const { return ((int64_t)heads * d) << page_shift; }  // bytes of k of a page
};

// The ragged new tokens of S sequences: tokens starts[s] .. starts[s + 1] - 1 (NULL: T / S each), the last of
// lengths[s] cached ones; page j of sequence s is table[s * width + j].
struct CacheRows {
  const int32_t *starts, *table, *lengths;
  int64_t T, width;
  int S;
};

hipError_t launch_cache_append(const CacheView& c, int layer, const void* key, const void* value, int dtype,
                               int64_t key_st, int64_t key_sh, int64_t val_st, int64_t val_sh, const CacheRows& rows,
                               int32_t* row_status, hipStream_t st);
size_t workspace_bytes_cache_fork(int64_t pages, int64_t rows);
hipError_t launch_cache_fork(const CacheView& c, const int32_t* table, const int32_t* lengths, int64_t S,
                             int64_t width, const int32_t* refs, const int32_t* parent, const int32_t* keep,
                             const int32_t* grow, int64_t S_out, int32_t* table_out, int32_t* lengths_out,
                             int32_t* refs_out, int32_t* row_status, void* workspace, hipStream_t st);
size_t workspace_bytes_cache_compact(int64_t pages);
hipError_t launch_cache_compact(const CacheView& c, const int32_t* table, const int32_t* lengths, int64_t S,
                                int64_t width, const int32_t* refs, int32_t* table_out, int32_t* refs_out,
                                int32_t* used, void* workspace, hipStream_t st);
hipError_t launch_cache_copy(const CacheView& c, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t st);
size_t workspace_bytes_attention(const CacheView& c, int64_t T, int64_t S, int64_t width, int64_t heads_q,
                                 int64_t max_new, int64_t max_length, bool uniform);
hipError_t launch_cache_attention(const CacheView& c, int layer, const void* q, int dtype, int64_t heads_q,
                                  int64_t q_st, int64_t q_sh, const CacheRows& rows, float scale, int64_t max_new,
                                  int64_t max_length, void* out, float* lse, void* workspace, hipStream_t st);
size_t workspace_bytes_beam(int64_t B, int64_t W, int64_t V, int64_t n);
hipError_t launch_beam_select(const void* logits, int dtype, int64_t row_stride, const float* scores,
                              const uint8_t* done, int64_t B, int64_t W, int64_t V, int64_t n, int32_t eos,
                              int32_t* parent, int32_t* token, float* score, uint8_t* done_out, int32_t* row_status,
                              void* workspace, hipStream_t st);
hipError_t launch_beam_reorder(const void* state, const int32_t* parent, int64_t B, int64_t W, int64_t n,
                               int64_t row_bytes, void* out, hipStream_t st);

// ---------------------------------------------------------------- device helpers
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Sequence of the slot `slot`, where sequence s owns the slots from first(s) = floor(starts[s] * num / den) + extra
// * s on: the largest s with first(s) <= slot (first is monotone in s).  The wave reads 64 candidates a step, so
// 4096 sequences take two dependent loads.
__device__ __forceinline__ int slot_sequence(const int32_t* starts, int S, int64_t slot, int num, int den, int extra,
                                             int lane) {
  int lo = 0, n = S;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int s = lo + lane * step;
    const bool le = s < lo + n && (int64_t)starts[s] * num / den + (int64_t)extra * s <= slot;
    const int hits = __popcll(__ballot(le));  // lane 0 always hits
    const int at = hits > 0 ? hits - 1 : 0;
    lo += at * step;
    n = min(step, n - at * step);
  }
  return lo;
}
__device__ __forceinline__ int64_t slot_first(const int32_t* starts, int s, int num, int den, int extra) {
  return (int64_t)starts[s] * num / den + (int64_t)extra * s;
}

}  // namespace mdss
