// Keys and values on their way into a paged cache and out of it, and the C entry points of the cache's calls.
//
// In: a row x (one token, one head, keys or values) becomes q = round(127 x / a), s = a / 127, a = max |x| (rows_io.cuh has the exact
// rounding).  Out: q s in fp32, rounded once to the output's type.  Both are bound by HBM: in, an element is read once and one byte
// written; out, the reverse.  A warp has some tokens and some heads of each.  Its lanes look up the places of all its tokens at once, then
// take the rows, dim / 8 lanes and eight elements each, so that a row's bytes go out whole and its maximum needs three or four
// shuffles and no barrier; UNROLL rows of a lane are under way together (out: UNROLL_OUT; with four there 12.6 us for 10.8).
//
// With a search for every row, 8,188 tokens of 8 heads of 128 took 63 us in and out; so 29, in 18.2 (51 MB, 2.8 TB/s) and out 10.8
// (4.7 TB/s).  What is left of long calls: 16 sequences of 8,000 go in at 3.7 TB/s (issue slots half taken; rows asked for ahead of the search,
// fewer registers or more tokens a warp change 5 % either way) and out at 4.5, reads and writes mixed; of short ones: the chain of
// loads, from the table to the page to the row.
#include <algorithm>

#include "kv_cache.cuh"

namespace {

using namespace rows;
using namespace kv;

constexpr int THREADS = 128, UNROLL = 4, UNROLL_OUT = 2, WARPS_RESIDENT = 32, MOST_TOKENS = 4;

struct Packed {                             // rows [n][heads][dim] of keys and of values
  const void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
};
struct Split { int tokens, heads, head_groups; };      // of a warp; groups of heads

// What a warp has: tokens first .. first + n - 1, heads head .. head + heads - 1; lane u knows where token u lies.
// found: 0: nowhere (a row of no sequence); 1: at `at` (its scale at `scale`) of head 0; 2: refused; 3: padding
struct Share {
  int64_t first; int n, head, heads;
  int64_t at, scale; int found;
  __device__ __forceinline__ Share(const Cache& c, const Batch& b, const Split& s, int32_t* status) {
    const int64_t w = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5), group = w % s.head_groups;
    const int lane = threadIdx.x & 31;
    first = w / s.head_groups * s.tokens;
    n = (int)max((int64_t)0, min((int64_t)s.tokens, b.rows - first));
    head = (int)group * s.heads;
    heads = min(s.heads, c.heads - head);
    at = scale = 0;
    found = 0;
    if (n < 1) return;
    const int64_t row = first + min(lane, n - 1);
    const int seq = sequence_of(b, row);
    if (seq < 0 || lane >= n) return;
    bool bad;
    const Seq q = sequence(b, seq, bad);
    const int64_t off = row - q.first, p = (int64_t)q.length - q.n + off;
    uint32_t page = 0, slot = 0;
    if (bad || off < 0 || off >= q.n) found = 2;
    else if (p < 0) found = 3;
    else found = place(c, b, seq, (uint32_t)p, page, slot) ? 1 : 2;
    if (found == 2 && head == 0) report(status);
    if (found == 1) {
      at = page * c.page + slot * c.slot;
      scale = page * c.spage + slot * c.sslot;
    }
  }
};

// How the lanes stand: DIM / 8 to a row, the first half of the warp's rows keys and the second values, or by turns (DIM 64: two heads)
template <int DIM>
struct Lane {
  static constexpr int LANES = DIM / 8, HEADS = 16 / LANES;               // of a row; heads at once
  int e, values, head;
  __device__ __forceinline__ Lane() {
    const int r = (threadIdx.x & 31) / LANES;
    e = (threadIdx.x % LANES) * 8;
    values = r & 1;
    head = r >> 1;
  }
};

template <int DIM>
__device__ __forceinline__ unsigned row_top(unsigned v) {
#pragma unroll
  for (int o = DIM / 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

template <typename T, int DIM, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
kv_write_kernel(const Cache c, const Batch b, const Packed x, const Split split, int32_t* status) {
  grid_begin();
  using L = Lane<DIM>;
  const L lane;
  const Share s(c, b, split, status);
  const int64_t x_head = lane.values ? x.v_head : x.k_head, x_row = lane.values ? x.v_row : x.k_row;
  const T* const from = static_cast<const T*>(lane.values ? x.v : x.k) + s.first * x_row + (s.head + lane.head) * x_head;
  int8_t* const to = (lane.values ? c.v : c.k) + (s.head + lane.head) * c.head + lane.e;
  float* const to_scale = (lane.values ? c.vs : c.ks) + (s.head + lane.head) * c.shead;
  for (int t = 0; t < s.n; ++t) {
    const int64_t at = __shfl_sync(0xffffffffu, s.at, t), scale = __shfl_sync(0xffffffffu, s.scale, t);
    if (__shfl_sync(0xffffffffu, s.found, t) != 1) continue;
    for (int h = 0; h < s.heads; h += UNROLL * L::HEADS) {
      Raw8<T> raw[UNROLL];
      unsigned top[UNROLL], own = 0;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int head = h + u * L::HEADS;
        raw[u] = head + lane.head < s.heads ? row_load<ALIGNED>(from + t * x_row + head * x_head, lane.e, DIM) : raw_zero<T>();
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        top[u] = row_top<DIM>(raw_top(raw[u]));
        if (threadIdx.x % UNROLL == u) own = top[u];
      }
      // a row's scale and inverse by one of its lanes, four rows at once
      const RowScale mine = row_scale<sizeof(T) == 2>(own);
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        RowScale r;
        r.pre = __shfl_sync(0xffffffffu, mine.pre, u, L::LANES);
        r.inv = __shfl_sync(0xffffffffu, mine.inv, u, L::LANES);
        r.top = __shfl_sync(0xffffffffu, mine.top, u, L::LANES);
        r.edge = __shfl_sync(0xffffffffu, mine.edge, u, L::LANES);
        const int head = h + u * L::HEADS;
        if (head + lane.head >= s.heads) continue;
        float v[8];
        raw_get(raw[u], v);
        *reinterpret_cast<uint2*>(to + at + head * c.head) = row_round8<sizeof(T) == 2>(v, r);
        if (lane.e == 8 * u) to_scale[scale + head * c.shead] = mine.s;
      }
    }
  }
}

// (positions that have no page, and padding, read as zeros; rows of no sequence are left as they are)
template <typename T, int DIM, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
kv_read_kernel(const Cache c, const Batch b, const Packed y, const Split split, int32_t* status) {
  grid_begin();
  using L = Lane<DIM>;
  const L lane;
  const Share s(c, b, split, status);
  const int64_t y_head = lane.values ? y.v_head : y.k_head, y_row = lane.values ? y.v_row : y.k_row;
  T* const to = const_cast<T*>(static_cast<const T*>(lane.values ? y.v : y.k)) + s.first * y_row + (s.head + lane.head) * y_head;
  const int8_t* const from = (lane.values ? c.v : c.k) + (s.head + lane.head) * c.head + lane.e;
  const float* const from_scale = (lane.values ? c.vs : c.ks) + (s.head + lane.head) * c.shead;
  for (int t = 0; t < s.n; ++t) {
    const int64_t at = __shfl_sync(0xffffffffu, s.at, t), at_scale = __shfl_sync(0xffffffffu, s.scale, t);
    const int found = __shfl_sync(0xffffffffu, s.found, t);
    if (!found) continue;
    for (int h = 0; h < s.heads; h += UNROLL_OUT * L::HEADS) {
      uint2 q[UNROLL_OUT];
      float scale[UNROLL_OUT];
#pragma unroll
      for (int u = 0; u < UNROLL_OUT; ++u) {
        const int head = h + u * L::HEADS;
        q[u] = make_uint2(0u, 0u);
        scale[u] = 0.f;
        if (found == 1 && head + lane.head < s.heads) {
          q[u] = *reinterpret_cast<const uint2*>(from + at + head * c.head);
          scale[u] = from_scale[at_scale + head * c.shead];
        }
      }
#pragma unroll
      for (int u = 0; u < UNROLL_OUT; ++u) {
        const int head = h + u * L::HEADS;
        if (head + lane.head >= s.heads) continue;
        // a byte in the last place of 2^23 + (byte + 128), less 2^23 + 128: the number, exactly, without the conversions' few units
        const uint32_t w[2] = {q[u].x ^ 0x80808080u, q[u].y ^ 0x80808080u};
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          v[k] = (__uint_as_float(__byte_perm(w[k >> 2], 0x4b000000u, 0x7440 + (k & 3))) - 8388736.f) * scale[u];
        row_store<ALIGNED>(to + t * y_row + head * y_head, lane.e, DIM, v);
      }
    }
  }
}

template <typename F>
armor_status by_row_type(int32_t dtype, F&& f) {
  if (dtype == ARMOR_DTYPE_F32) return f(float());
  return dtype == ARMOR_DTYPE_BF16 ? f(__nv_bfloat16()) : f(__half());
}

constexpr int64_t MOST = 0x7fffffff, MOST_POSITIONS = MOST + 1 - 4096;      // (a step that begins in a sequence ends below 2^31)

template <typename... P>
bool on_boundary(size_t bytes, P... p) { return ((reinterpret_cast<uintptr_t>(p) % bytes == 0) && ...); }

armor_status check_cache(const armor_kv_cache* g) {
  if (!g) return ARMOR_ERR_INVALID_ARG;
  if (g->n_pages < 1 || g->page_size < 1 || g->kv_heads < 1 || g->head_dim < 1) return ARMOR_ERR_SHAPE;
  if (g->head_dim != 64 && g->head_dim != 128) return ARMOR_ERR_UNSUPPORTED;
  if (g->n_pages > MOST || g->page_size > MOST || g->kv_heads > 65535) return ARMOR_ERR_TOO_LARGE;
  if (g->slot_stride < g->head_dim || g->page_stride < g->head_dim || g->head_stride < g->head_dim || g->scale_page_stride < 1 ||
      g->scale_head_stride < 1 || g->scale_slot_stride < 1)
    return ARMOR_ERR_SHAPE;
  if (g->page_stride % 16 || g->head_stride % 16 || g->slot_stride % 16 || !on_boundary(16, g->k, g->v) || !on_boundary(4, g->k_scale, g->v_scale))
    return ARMOR_ERR_SHAPE;
  return g->k && g->v && g->k_scale && g->v_scale ? ARMOR_OK : ARMOR_ERR_INVALID_ARG;
}
armor_status check_batch(const armor_kv_batch* g, int64_t rows) {
  if (!g || g->n_seqs < 0 || rows < 0) return ARMOR_ERR_INVALID_ARG;
  if (g->max_pages < 0 || g->ld_pages < g->max_pages) return ARMOR_ERR_SHAPE;
  if (g->n_seqs > MOST || g->max_pages > MOST || rows > MOST) return ARMOR_ERR_TOO_LARGE;
  if (g->n_seqs == 0 || rows == 0) return ARMOR_OK;       // (nothing is read)
  if (!g->lengths || !g->starts || (g->max_pages > 0 && !g->pages)) return ARMOR_ERR_INVALID_ARG;
  return on_boundary(4, g->lengths, g->starts, g->pages) ? ARMOR_OK : ARMOR_ERR_SHAPE;
}
Cache view(const armor_kv_cache* g) {
  Cache c;
  c.k = g->k; c.v = g->v; c.ks = g->k_scale; c.vs = g->v_scale;
  c.page = g->page_stride; c.head = g->head_stride; c.slot = g->slot_stride;
  c.spage = g->scale_page_stride; c.shead = g->scale_head_stride; c.sslot = g->scale_slot_stride;
  c.n_pages = (uint32_t)g->n_pages; c.page_size = (uint32_t)g->page_size; c.heads = (int)g->kv_heads;
  divisor(c.page_size, c.mul, c.shift);
  return c;
}
Batch view(const armor_kv_batch* g, const armor_kv_cache* c, int64_t rows) {
  Batch b;
  b.pages = g->pages; b.lengths = g->lengths; b.starts = g->starts; b.ld = g->ld_pages;
  b.n = (int)g->n_seqs; b.max_pages = (int)g->max_pages; b.rows = rows;
  b.capacity = std::min(g->max_pages * c->page_size, MOST_POSITIONS);
  return b;
}

enum { WRITE, READ };
template <int WHAT>
armor_status move_rows(armor_ctx* c, const armor_kv_cache* cache, const armor_kv_batch* batch, const armor_kv_rows* g, armor_stream_t stream) {
  armor_status st = check_cache(cache);
  if (st != ARMOR_OK) return st;
  if (!g) return ARMOR_ERR_INVALID_ARG;
  if ((st = check_batch(batch, g->n_rows)) != ARMOR_OK) return st;
  const int es = rows_dtype_bytes(g->dtype);
  if (!es) return ARMOR_ERR_UNSUPPORTED;
  if (g->n_rows > 0 && batch->n_seqs > 0 && !on_boundary(es, g->k, g->v)) return ARMOR_ERR_SHAPE;
  // (what is written must not overlap; what is read may: heads may share a row)
  const int64_t least = WHAT == READ ? cache->head_dim : 0;
  if (g->k_row_stride < least || g->k_head_stride < least || g->v_row_stride < least || g->v_head_stride < least) return ARMOR_ERR_SHAPE;
  if (!c) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows == 0 || batch->n_seqs == 0) return ARMOR_OK;
  if (!g->k || !g->v) return ARMOR_ERR_INVALID_ARG;
  const Cache cv = view(cache);
  const Batch bv = view(batch, cache, g->n_rows);
  const Packed x{g->k, g->v, g->k_row_stride, g->k_head_stride, g->v_row_stride, g->v_head_stride};
  const bool al = aligned16(g->k, g->k_row_stride, es) && aligned16(g->v, g->v_row_stride, es) && g->k_head_stride * es % 16 == 0 &&
                  g->v_head_stride * es % 16 == 0;
  // As many warps as the SMs hold: with few tokens some heads of one to a warp, with many several tokens and all heads, whose search and places are
  // paid for once.
  const int64_t heads = cache->kv_heads, items = 2 * g->n_rows * heads, resident = (int64_t)c->n_sm * WARPS_RESIDENT;
  const int64_t batch_heads = (WHAT == READ ? UNROLL_OUT : UNROLL) * 16 / (cache->head_dim / 8);        // heads under way at once
  Split split;
  split.tokens = (int)std::min<int64_t>(MOST_TOKENS, std::max<int64_t>(1, g->n_rows / resident));
  const int64_t groups = std::min((heads + batch_heads - 1) / batch_heads, std::max<int64_t>(1, resident / g->n_rows));
  split.heads = (int)((heads + groups - 1) / groups);
  split.head_groups = (int)((heads + split.heads - 1) / split.heads);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int64_t warps = (g->n_rows + split.tokens - 1) / split.tokens * split.head_groups, blocks = (warps + THREADS / 32 - 1) / (THREADS / 32);
  if (blocks > MOST) return ARMOR_ERR_TOO_LARGE;
  KTimer kt(c, ARMOR_KC_FORWARD, (double)items * (double)(cache->head_dim * (es + 1) + 4), s);
  st = by_row_type(g->dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid((unsigned)blocks), block(THREADS);
    auto go = [&](auto dim) {
      constexpr int DIM = decltype(dim)::value;
      if (WHAT == WRITE) {
        if (al) launch_dependent(kv_write_kernel<T, DIM, true>, grid, block, 0, s, cv, bv, x, split, c->status);
        else launch_dependent(kv_write_kernel<T, DIM, false>, grid, block, 0, s, cv, bv, x, split, c->status);
      } else {
        if (al) launch_dependent(kv_read_kernel<T, DIM, true>, grid, block, 0, s, cv, bv, x, split, c->status);
        else launch_dependent(kv_read_kernel<T, DIM, false>, grid, block, 0, s, cv, bv, x, split, c->status);
      }
    };
    if (cache->head_dim == 64) go(std::integral_constant<int, 64>());
    else go(std::integral_constant<int, 128>());
    return ARMOR_OK;
  });
  c->launches++;
  return finish_call(c);
}

}  // namespace

// (sizes and types are looked at before the context)
extern "C" armor_status armor_kv_write(armor_ctx* c, const armor_kv_cache* cache, const armor_kv_batch* batch, const armor_kv_rows* rows,
                                       armor_stream_t stream) {
  return move_rows<WRITE>(c, cache, batch, rows, stream);
}

extern "C" armor_status armor_kv_read(armor_ctx* c, const armor_kv_cache* cache, const armor_kv_batch* batch, const armor_kv_rows* rows,
                                      armor_stream_t stream) {
  return move_rows<READ>(c, cache, batch, rows, stream);
}

extern "C" armor_status armor_kv_attend(armor_ctx* c, const armor_kv_cache* cache, const armor_kv_batch* batch, const armor_kv_attend_args* g,
                                        armor_stream_t stream) {
  armor_status st = check_cache(cache);
  if (st != ARMOR_OK) return st;
  if (!g) return ARMOR_ERR_INVALID_ARG;
  if ((st = check_batch(batch, g->n_rows)) != ARMOR_OK) return st;
  if (g->dtype != ARMOR_DTYPE_BF16 && g->dtype != ARMOR_DTYPE_F16) return ARMOR_ERR_UNSUPPORTED;
  if (g->heads < 1 || g->heads % cache->kv_heads) return ARMOR_ERR_SHAPE;
  if (g->q_row_stride < 0 || g->q_head_stride < 0 || g->o_row_stride < cache->head_dim || g->o_head_stride < cache->head_dim) return ARMOR_ERR_SHAPE;
  if (g->window < 0 || g->max_chunk < 0 || !(g->scale >= 0.f) || g->scale > 1e30f) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows > 0 && batch->n_seqs > 0 && !on_boundary(2, g->q, g->o)) return ARMOR_ERR_SHAPE;
  if (g->n_rows > 0 && g->heads / cache->kv_heads > MOST_POSITIONS / g->n_rows) return ARMOR_ERR_TOO_LARGE;
  if (!c) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows == 0 || batch->n_seqs == 0) return ARMOR_OK;
  if (!g->q || !g->o) return ARMOR_ERR_INVALID_ARG;
  KvAttend a;
  a.c = view(cache);
  a.b = view(batch, cache, g->n_rows);
  a.q = g->q; a.q_row = g->q_row_stride; a.q_head = g->q_head_stride;
  a.o = g->o; a.o_row = g->o_row_stride; a.o_head = g->o_head_stride;
  a.group = (int)(g->heads / cache->kv_heads); a.dim = (int)cache->head_dim; a.dtype = g->dtype;
  a.window = g->window; a.max_chunk = std::min(g->max_chunk, g->n_rows);
  a.scale = g->scale * 1.4426950408889634f;
  a.aligned = aligned16(a.q, a.q_row, 2) && aligned16(a.o, a.o_row, 2) && a.q_head % 8 == 0 && a.o_head % 8 == 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // Which kernels: the one for few rows a sequence reads keys and values once for every 16 of them, the other one once for 256, of which a few cost what all
  // do.  (16 sequences of 4,003, 8 key heads: 25 rows each 73 us and 86, 40 rows 102 and 86; 64 of 8,000: 32 rows 432 and 489, 48 rows 644 and
  // 499.)  Where the host cannot tell (lengths are on the device), both run, each on its sequences.
  const int64_t chunk = a.max_chunk ? a.max_chunk : (a.b.n == 1 ? g->n_rows : 0), rows = chunk * a.group;
  if (chunk ? rows <= KV_FEW_ROWS : g->n_rows <= batch->n_seqs && a.group <= KV_FEW_ROWS) st = launch_kv_attend_few(c, a, MOST, s);
  else if (a.b.n == 1 || a.group > KV_FEW_ROWS) st = launch_kv_attend_tile(c, a, 0, s);
  else {
    st = launch_kv_attend_tile(c, a, KV_FEW_ROWS, s);
    if (st == ARMOR_OK) st = launch_kv_attend_few(c, a, KV_FEW_ROWS, s);
  }
  if (st != ARMOR_OK) return st;
  return finish_call(c);
}
