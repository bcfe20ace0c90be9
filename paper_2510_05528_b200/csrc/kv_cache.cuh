// A paged cache of keys and values as int8 rows with a scale each, seen from a kernel: where a sequence's positions lie, and which rows of the
// packed arrays are whose.  Nothing that a table or an offset holds is trusted: what it names outside of the arrays is neither read nor
// written, and raises a status word.
#pragma once
#include "kv_order.h"
#include "rows_io.cuh"

namespace kv {

struct Cache {
  int8_t *k, *v;
  float *ks, *vs;
  int64_t page, head, slot;                 // strides of the values, in elements
  int64_t spage, shead, sslot;              // strides of the scales
  uint32_t n_pages, page_size;
  uint32_t mul; int shift;                  // p / page_size = p mul >> shift for p < 2^31
  int heads;
};
struct Batch {
  const int32_t *pages, *lengths, *starts;
  int64_t ld;
  int n, max_pages;
  int64_t rows;                             // rows of the packed arrays
  int64_t capacity;                         // positions that a table holds
};

// a / b of numbers that are not negative: in 32 bits where they fit (a 64-bit division is a hundred instructions or so, and a call of 10 us has ten of them
// one behind the other)
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  if (((uint64_t)a | (uint64_t)b) >> 32 == 0) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}

// what a sequence is made of: n new rows from row `first` on, the last n of `length` positions
struct Seq { int first, n, length; };
__device__ __forceinline__ Seq sequence(const Batch& b, int at, bool& bad) {
  Seq s;
  s.first = b.starts[at];
  const int64_t n = (int64_t)b.starts[at + 1] - s.first;
  s.length = max(b.lengths[at], 0);
  bad = s.first < 0 || n < 0 || s.first + n > b.rows || s.length > b.capacity;
  s.n = bad ? 0 : (int)n;
  return s;
}
__device__ __forceinline__ void report(int32_t* status) {
  atomicAdd(&status[ST_KV_REFUSED], 1);
  status[ST_LAST_ERR] = ARMOR_ERR_INVALID_ARG;
}

// The sequence of row t, by a whole warp (t may differ between lanes): 32 offsets are compared at a time.  -1: before the first
// one's rows or behind the last one's.
__device__ __forceinline__ int sequence_of(const Batch& b, int64_t t) {
  const int lane = threadIdx.x & 31;
  int mine = -2;
  for (;;) {
    const unsigned open = __ballot_sync(0xffffffffu, mine == -2);
    if (!open) return mine;
    const int64_t row = __shfl_sync(0xffffffffu, t, __ffs(open) - 1);
    // how many of starts[1 .. n] are at most `row`: the sequence that holds it
    int lo = 0, hi = b.n;                   // the count lies in [lo, hi]
    while (hi > lo) {
      const int step = (hi - lo + 31) >> 5;
      const int i = lo + (lane + 1) * step; // starts[i] is looked at: the count is at least i where it is at most `row`
      const bool at_most = i <= hi && b.starts[i] <= row;
      const int c = __popc(__ballot_sync(0xffffffffu, at_most));
      lo += c * step;
      if (step == 1) break;
      hi = min(hi, lo + step - 1);
    }
    const int64_t first = lo < b.n ? b.starts[lo] : 0, last = lo < b.n ? b.starts[lo + 1] : 0;
    const int found = lo < b.n && (lo > 0 || row >= first) ? lo : -1;
    if (mine == -2 && (t == row || (found >= 0 && t >= first && t < last))) mine = found;
  }
}

// Page and slot of position p of sequence `at`; false where the table has none
__device__ __forceinline__ bool place(const Cache& c, const Batch& b, int at, uint32_t p, uint32_t& page, uint32_t& slot) {
  const uint32_t i = quotient(p, c.mul, c.shift);
  slot = p - i * c.page_size;
  if (i >= (uint32_t)b.max_pages) return false;
  page = (uint32_t)b.pages[(int64_t)at * b.ld + i];
  return page < c.n_pages;
}

// The scale that a position's contribution is measured with, sv itself for all that matter.  A row of zeros may have any: 2^-60, so that neither its own
// weight, which the sum of the weights needs, nor the others' contributions fall below what fp32 holds.  Scales below 2^-100 count as that (their values
// are below 1e-28).  A scale that is no number stays what it is.
__device__ __forceinline__ float measure(float sv) { return sv == 0.f ? 8.6736174e-19f : (sv < 7.8886091e-31f ? 7.8886091e-31f : sv); }

// A row's weights are 2^(t - m), m its largest t so far less RAISED, and they are rounded to fp16.  So the largest is 2^RAISED, or 2^(RAISED + LAZY) = 2^15
// before m moves, and one is off by half of fp16's smallest step, 2^-25 or 2^-32 of the largest, at most where it is small.  (With RAISED 0 weights below
// 2^-25 of the largest were zeros in O, but not in l: with one position far above 131,071 others, 2^-9 of the output was missing.)  l takes the
// weights unrounded, in fp32, and without the 2^RAISED, which rides on the inverse scales and comes out of O with 1 / l: 2^15 of scales of 2^-100
// over all positions would come near the end of fp32's range.
constexpr float RAISED = 7.f, LOWERED = 0.0078125f;   // 2^-RAISED
constexpr float LAZY = 8.f;                 // m moves when the largest t is above m + RAISED by this much (log2)

}  // namespace kv

// kv_attend_few.cu, kv_attend_tcgen05.cu
struct KvAttend {
  kv::Cache c;
  kv::Batch b;
  const void* q; int64_t q_row, q_head;
  void* o; int64_t o_row, o_head;
  int group, dim;
  int dtype;
  int64_t window;                           // 0: none
  int64_t max_chunk;                        // rows of a sequence expected; 0: not known
  float scale;                              // of the scores, times log2 e
  int aligned;                              // rows of q and o start on 16-byte boundaries
};
// sequences of up to `limit` rows (a token and a head of the group each)
armor_status launch_kv_attend_few(armor_ctx* c, const KvAttend& a, int64_t limit, cudaStream_t s);
// sequences of more
armor_status launch_kv_attend_tile(armor_ctx* c, const KvAttend& a, int64_t limit, cudaStream_t s);
constexpr int64_t KV_FEW_ROWS = 32;
