// Keys and values on their way into a paged cache and out of it, and the C entry points of the cache's calls.
//
// In: a row x (one token, one head, keys or values) becomes q = round(127 x / a), s = a / 127, a = max |x| (rows_io.cuh has the exact
// rounding).  Out: q s in fp32, rounded once to the output's type.  Both are bound by HBM: in, an element is read once and one byte
// written; out, the reverse.  A row is taken by dim / 8 lanes, eight elements each, so that its bytes go out whole and its maximum needs
// three or four shuffles and no barrier; a lane has ITEMS rows under way.
#include "kv_cache.cuh"

namespace {

using namespace rows;
using namespace kv;

constexpr int THREADS = 256, ITEMS = 4;

struct Packed {                             // rows [n][heads][dim] of keys and of values
  const void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
};

// Item i: keys (even) or values (odd) of head i / 2 % heads in row i / 2 / heads.
struct Item { int64_t row; int head, values; };
__device__ __forceinline__ Item item(int64_t i, int heads) {
  Item r;
  r.values = (int)(i & 1);
  const uint64_t u = (uint64_t)i >> 1;
  r.row = u < (1ull << 32) ? (uint32_t)u / (uint32_t)heads : (int64_t)(u / (uint32_t)heads);
  r.head = (int)(u - (uint64_t)r.row * heads);
  return r;
}

template <int DIM>
__device__ __forceinline__ unsigned row_top(unsigned v) {
#pragma unroll
  for (int o = DIM / 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Position and place of the rows that a lane has under way.  place 0: nothing to do; 1: found; 2: a position with no page; 3: padding
template <int DIM>
struct Rows {
  Item it[ITEMS];
  uint32_t page[ITEMS], slot[ITEMS];
  int found[ITEMS];
  __device__ __forceinline__ void find(const Cache& c, const Batch& b, int64_t n_items, int32_t* status) {
    constexpr int LANES = DIM / 8, PER = THREADS / LANES;
    const int64_t i0 = (int64_t)blockIdx.x * (PER * ITEMS) + threadIdx.x / LANES;
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
      const int64_t i = i0 + u * PER;
      it[u] = item(i < n_items ? i : 0, c.heads);
      found[u] = 0;
      const int at = sequence_of(b, it[u].row);
      if (i < n_items && at >= 0) {
        bool bad;
        const Seq s = sequence(b, at, bad);
        const int64_t off = it[u].row - s.first, p = (int64_t)s.length - s.n + off;
        if (bad || off < 0 || off >= s.n) found[u] = 2;
        else if (p < 0) found[u] = 3;
        else found[u] = place(c, b, at, (uint32_t)p, page[u], slot[u]) ? 1 : 2;
        if (found[u] == 2 && threadIdx.x % LANES == 0) report(status);
      }
    }
  }
};

template <typename T, int DIM, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
kv_write_kernel(const Cache c, const Batch b, const Packed x, int64_t n_items, int32_t* status) {
  grid_begin();
  const int e = (threadIdx.x % (DIM / 8)) * 8;
  Rows<DIM> r;
  r.find(c, b, n_items, status);
  Raw8<T> raw[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const Item& it = r.it[u];
    const T* const at = it.values ? static_cast<const T*>(x.v) + it.row * x.v_row + it.head * x.v_head
                                  : static_cast<const T*>(x.k) + it.row * x.k_row + it.head * x.k_head;
    raw[u] = r.found[u] == 1 ? row_load<ALIGNED>(at, e, DIM) : raw_zero<T>();
  }
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const RowScale s = row_scale<sizeof(T) == 2>(row_top<DIM>(raw_top(raw[u])));
    if (r.found[u] != 1) continue;
    float v[8];
    raw_get(raw[u], v);
    const Item& it = r.it[u];
    *reinterpret_cast<uint2*>((it.values ? c.v : c.k) + r.page[u] * c.page + it.head * c.head + r.slot[u] * c.slot + e) = row_round8<sizeof(T) == 2>(v, s);
    if (e == 0) (it.values ? c.vs : c.ks)[r.page[u] * c.spage + it.head * c.shead + r.slot[u] * c.sslot] = s.s;
  }
}

// (positions that have no page, and padding, read as zeros; rows behind the last sequence are left as they are)
template <typename T, int DIM, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
kv_read_kernel(const Cache c, const Batch b, const Packed y, int64_t n_items, int32_t* status) {
  grid_begin();
  const int e = (threadIdx.x % (DIM / 8)) * 8;
  Rows<DIM> r;
  r.find(c, b, n_items, status);
  uint2 q[ITEMS];
  float s[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const Item& it = r.it[u];
    q[u] = make_uint2(0u, 0u);
    s[u] = 0.f;
    if (r.found[u] == 1) {
      q[u] = *reinterpret_cast<const uint2*>((it.values ? c.v : c.k) + r.page[u] * c.page + it.head * c.head + r.slot[u] * c.slot + e);
      s[u] = (it.values ? c.vs : c.ks)[r.page[u] * c.spage + it.head * c.shead + r.slot[u] * c.sslot];
    }
  }
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    if (!r.found[u]) continue;
    const Item& it = r.it[u];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)((i < 4 ? q[u].x : q[u].y) >> (8 * (i & 3))) * s[u];
    T* const at = const_cast<T*>(it.values ? static_cast<const T*>(y.v) + it.row * y.v_row + it.head * y.v_head
                                           : static_cast<const T*>(y.k) + it.row * y.k_row + it.head * y.k_head);
    row_store<ALIGNED>(at, e, DIM, v);
  }
}

template <typename F>
armor_status by_row_type(int32_t dtype, F&& f) {
  if (dtype == ARMOR_DTYPE_F32) return f(float());
  return dtype == ARMOR_DTYPE_BF16 ? f(__nv_bfloat16()) : f(__half());
}

constexpr int64_t MOST = 0x7fffffff;

armor_status check_cache(const armor_kv_cache* g) {
  if (!g) return ARMOR_ERR_INVALID_ARG;
  if (g->n_pages < 1 || g->page_size < 1 || g->kv_heads < 1 || g->head_dim < 1) return ARMOR_ERR_SHAPE;
  if (g->head_dim != 64 && g->head_dim != 128) return ARMOR_ERR_UNSUPPORTED;
  if (g->n_pages > MOST || g->page_size > MOST || g->kv_heads > 65535) return ARMOR_ERR_TOO_LARGE;
  if (g->slot_stride < g->head_dim || g->page_stride < g->head_dim || g->head_stride < g->head_dim || g->scale_page_stride < 1 ||
      g->scale_head_stride < 1 || g->scale_slot_stride < 1)
    return ARMOR_ERR_SHAPE;
  if (g->page_stride % 16 || g->head_stride % 16 || g->slot_stride % 16 || reinterpret_cast<uintptr_t>(g->k) % 16 || reinterpret_cast<uintptr_t>(g->v) % 16)
    return ARMOR_ERR_SHAPE;
  return g->k && g->v && g->k_scale && g->v_scale ? ARMOR_OK : ARMOR_ERR_INVALID_ARG;
}
armor_status check_batch(const armor_kv_batch* g, int64_t rows) {
  if (!g || g->n_seqs < 0 || rows < 0) return ARMOR_ERR_INVALID_ARG;
  if (g->max_pages < 0 || g->ld_pages < g->max_pages) return ARMOR_ERR_SHAPE;
  if (g->n_seqs > MOST || g->max_pages > MOST || rows > MOST) return ARMOR_ERR_TOO_LARGE;
  if (g->n_seqs > 0 && rows > 0 && (!g->lengths || !g->starts || (g->max_pages > 0 && !g->pages))) return ARMOR_ERR_INVALID_ARG;
  return ARMOR_OK;
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
Batch view(const armor_kv_batch* g, int64_t rows) {
  Batch b;
  b.pages = g->pages; b.lengths = g->lengths; b.starts = g->starts; b.ld = g->ld_pages;
  b.n = (int)g->n_seqs; b.max_pages = (int)g->max_pages; b.rows = rows;
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
  // (what is written must not overlap; what is read may: heads may share a row)
  const int64_t least = WHAT == READ ? cache->head_dim : 0;
  if (g->k_row_stride < least || g->k_head_stride < least || g->v_row_stride < least || g->v_head_stride < least) return ARMOR_ERR_SHAPE;
  if (!c) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows == 0 || batch->n_seqs == 0) return ARMOR_OK;
  if (!g->k || !g->v) return ARMOR_ERR_INVALID_ARG;
  const Cache cv = view(cache);
  const Batch bv = view(batch, g->n_rows);
  const Packed x{g->k, g->v, g->k_row_stride, g->k_head_stride, g->v_row_stride, g->v_head_stride};
  const bool al = aligned16(g->k, g->k_row_stride, es) && aligned16(g->v, g->v_row_stride, es) && g->k_head_stride * es % 16 == 0 &&
                  g->v_head_stride * es % 16 == 0;
  const int64_t items = 2 * g->n_rows * cache->kv_heads;
  const int64_t per = THREADS / (cache->head_dim / 8) * ITEMS;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = (items + per - 1) / per;
  if (blocks > MOST) return ARMOR_ERR_TOO_LARGE;
  KTimer kt(c, ARMOR_KC_FORWARD, (double)items * (double)(cache->head_dim * (es + 1) + 4), s);
  st = by_row_type(g->dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid((unsigned)blocks), block(THREADS);
    auto go = [&](auto dim) {
      constexpr int DIM = decltype(dim)::value;
      if (WHAT == WRITE) {
        if (al) launch_dependent(kv_write_kernel<T, DIM, true>, grid, block, 0, s, cv, bv, x, items, c->status);
        else launch_dependent(kv_write_kernel<T, DIM, false>, grid, block, 0, s, cv, bv, x, items, c->status);
      } else {
        if (al) launch_dependent(kv_read_kernel<T, DIM, true>, grid, block, 0, s, cv, bv, x, items, c->status);
        else launch_dependent(kv_read_kernel<T, DIM, false>, grid, block, 0, s, cv, bv, x, items, c->status);
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
  if (g->n_rows * (g->heads / cache->kv_heads) > MOST) return ARMOR_ERR_TOO_LARGE;
  if (!c) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows == 0 || batch->n_seqs == 0) return ARMOR_OK;
  if (!g->q || !g->o) return ARMOR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(g->q) % 2 || reinterpret_cast<uintptr_t>(g->o) % 2) return ARMOR_ERR_SHAPE;
  KvAttend a;
  a.c = view(cache);
  a.b = view(batch, g->n_rows);
  a.q = g->q; a.q_row = g->q_row_stride; a.q_head = g->q_head_stride;
  a.o = g->o; a.o_row = g->o_row_stride; a.o_head = g->o_head_stride;
  a.group = (int)(g->heads / cache->kv_heads); a.dim = (int)cache->head_dim; a.dtype = g->dtype;
  a.window = g->window; a.max_chunk = g->max_chunk;
  a.scale = g->scale * 1.4426950408889634f;
  a.aligned = aligned16(a.q, a.q_row, 2) && aligned16(a.o, a.o_row, 2) && a.q_head % 8 == 0 && a.o_head % 8 == 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // Which kernels: the one for few rows a sequence reads keys and values once for every KV_FEW_ROWS of them, the other one once for 256.  Where
  // the host cannot tell (lengths are on the device), both run, each on its sequences.
  const int64_t chunk = g->max_chunk ? g->max_chunk : (a.b.n == 1 ? g->n_rows : 0), rows = chunk * a.group;
  if (chunk ? rows <= KV_FEW_ROWS : g->n_rows <= batch->n_seqs && a.group <= KV_FEW_ROWS) st = launch_kv_attend_few(c, a, MOST, s);
  else if (a.b.n == 1 || a.group > KV_FEW_ROWS) st = launch_kv_attend_tile(c, a, 0, s);
  else {
    st = launch_kv_attend_tile(c, a, KV_FEW_ROWS, s);
    if (st == ARMOR_OK) st = launch_kv_attend_few(c, a, KV_FEW_ROWS, s);
  }
  if (st != ARMOR_OK) return st;
  return finish_call(c);
}
