// The paged int8 KV cache on the device: where a token lies, and the batch that writes, reads or attends.
#pragma once

#include "common.h"
#include "kv_plan.h"

namespace lrqat {

// Codes [pages][heads][page tokens][d], scales [pages][heads][page tokens / scale tokens].  A scale is never
// below kKvMinScale, so that a block of zeros needs no case of its own anywhere.
constexpr float kKvMinScale = 0x1p-100f;

constexpr int64_t kMaxThreads = int64_t(UINT32_MAX);  // of a grid

struct KvCache {
  int8_t* code[2];   // K, V
  float* scale[2];
  int64_t pages;
  int heads, d;
  int lpage, lscale;  // log2 of the tokens of a page and of a scale block
};

// Tokens of a batch: sequence i has rows first[i] .. first[i + 1] - 1 of the batch's tensors, at the positions
// that follow its cached[i] earlier tokens.  The kernels check what they read of it: rows past the batch,
// positions past the table and page numbers outside the cache hold nothing.
struct KvBatch {
  const int32_t* first;
  const int32_t* cached;
  const int32_t* table;  // [seqs][width]
  int64_t tokens;
  int seqs, width;
  int max_new, max_cached;
};

struct KvSeq {
  int64_t row0;      // first row of the batch
  int64_t c0, end;   // positions of the new tokens: c0 .. end - 1
};

// Sequence s of the batch, cut to the batch's rows; c0 = end where it has none.
__device__ __forceinline__ KvSeq kv_seq(const KvBatch& b, int s) {
  const int64_t f0 = b.first[s], f1 = min(int64_t(b.first[s + 1]), b.tokens);
  KvSeq q;
  q.row0 = f0;
  q.c0 = b.cached[s];
  const bool ok = f0 >= 0 && f1 > f0 && q.c0 >= 0;
  q.end = ok ? q.c0 + min(f1 - f0, int64_t(b.max_new)) : q.c0;
  return q;
}

// The table's entry for a position of sequence s (any of its entries where the position is outside the table), and
// whether it names a page.
__device__ __forceinline__ int32_t kv_entry(const KvCache& c, const KvBatch& b, int s, int64_t pos) {
  return b.table[int64_t(s) * b.width + min(max(pos >> c.lpage, int64_t(0)), int64_t(b.width) - 1)];
}
__device__ __forceinline__ bool kv_inside(const KvCache& c, const KvBatch& b, int32_t entry, int64_t pos) {
  return entry >= 0 && entry < c.pages && pos >= 0 && pos >> c.lpage < b.width;
}
// Page of a position, or -1.
__device__ __forceinline__ int64_t kv_page(const KvCache& c, const KvBatch& b, int s, int64_t pos) {
  const int32_t e = kv_entry(c, b, s, pos);
  return kv_inside(c, b, e, pos) ? e : -1;
}

// First code of a token's row, and index of its scale.
__device__ __forceinline__ int64_t kv_row(const KvCache& c, int64_t page, int head, int64_t pos) {
  return (((page * c.heads + head) << c.lpage) + (pos & ((int64_t(1) << c.lpage) - 1))) * c.d;
}
__device__ __forceinline__ int64_t kv_scale(const KvCache& c, int64_t page, int head, int64_t pos) {
  const int l = c.lpage - c.lscale;
  return ((page * c.heads + head) << l) + ((pos >> c.lscale) & ((int64_t(1) << l) - 1));
}

struct KvWriteArgs {
  KvCache c;
  KvBatch b;
  const void* x[2];   // K, V: token rows of heads x d values, bf16 or float
  int64_t stride[2];  // elements from one token to the next
};
struct KvReadArgs {
  KvCache c;
  KvBatch b;
  void* x[2];
  int64_t stride[2];
};
// Whether one launch holds the batch (the host checks).
bool kv_fits(const KvCache& c, const KvBatch& b, bool write);
hipError_t launch_kv_write(bool bf16, const KvWriteArgs& a, hipStream_t st);
hipError_t launch_kv_read(bool bf16, const KvReadArgs& a, hipStream_t st);

// Attention over the cache (kv_attention.hip).
struct KvAttnArgs {
  KvCache c;
  KvBatch b;
  const uint16_t* q;   // [tokens][hq][d] bf16, q_stride elements between tokens
  int64_t q_stride;
  uint16_t* o;
  int64_t o_stride;
  int hq, group;       // query heads, and those that share a key/value head
  float qk;            // the score's scale times log2(e)
  int causal;
  int chunk, nsplit;   // keys of a split (a multiple of 64), and splits of the longest sequence
  uint32_t tiles;      // row tiles of a sequence and key/value head
  float* part_o;       // [nsplit][tokens][hq][d] where nsplit > 1
  float* part_ml;      // [nsplit][tokens][hq][2]: maximum of the weights' exponents, denominator
};
bool kv_attention_fits(const KvCache& c, const KvBatch& b, int hq, const KvAttnPlan& p);
hipError_t launch_kv_attention(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t st);

}  // namespace lrqat
