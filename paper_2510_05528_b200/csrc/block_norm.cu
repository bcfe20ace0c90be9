// What lies between the last linear layer of a block of a transformer and the first of the next one, norms by the root mean square:
//   u = y / rms(y) (.) w_post   (or y)          rms(v)^2 = mean(v^2) + eps
//   h = a x + gate (.) u                        x: the residual stream, a: its scale, gate: a row for every rows_per_gate rows
//   n = h / rms(h) (.) w_pre                    what the next block reads, in 16 or 32 bits, or int8 with a scale for the row
// and the gradient.  Sums, the stream and the norms are held in fp32; h, n, dx and dy are rounded once, as they are stored (n is that of
// the unrounded h).
//
// Bound by HBM: two reads and two writes an element forward, four and two backward.  A CTA takes a row, which stays in
// registers from its loads to its stores.  Backward, with g = dn (.) w_pre and bars for divided by rms:
//   dh' = dh + (g - hbar mean(g hbar)) / rms(h)      dx = a dh'      e = gate (.) dh'      f = e (.) w_post
//   dy = (f - ybar mean(f ybar)) / rms(y)   (or e)
//   dw_pre = sum_t dn hbar      dw_post = sum_t e ybar      dgate = sum over the row's rows of dh' u
// The sums over rows: a CTA takes consecutive rows and adds into shared memory, where an element of the row has one owner, so no order
// is left to chance; the CTAs' sums are added in order by a second kernel, in fp64.  A gate's rows may end inside a CTA's: the CTA
// keeps two sums for the gates at its ends, and writes one that lies within its rows at once.
#include "rows_io.cuh"

namespace {

using namespace rows;

// rows [lo(b), lo(b + 1)) of CTA b of `ctas`
__host__ __device__ __forceinline__ int64_t rows_lo(int64_t b, int64_t rows, int64_t ctas) { return b * rows / ctas; }
__device__ __forceinline__ int64_t rows_owner(int64_t r, int64_t rows, int64_t ctas) { return ((r + 1) * ctas - 1) / rows; }

struct NormP {
  int64_t rows, d, ldx, ldy, ldh, ldn, ldq, ldg, per_gate;
  const void *x, *y;
  void *h, *n;
  int8_t* q;
  float* q_scale;
  const float *w_post, *w_pre, *gate;
  float a, eps;
  int post, pre;
};

// TS: type of the stream (x, h), TB: of the branch (y, n)
template <typename TS, typename TB, bool ALIGNED, int CHUNKS>
__global__ void __launch_bounds__(CHUNKS == 1 ? 1024 : CHUNKS * 128)
block_norm_kernel(const NormP p) {
  grid_begin();
  __shared__ float red[3][2][32];
  const int64_t row = blockIdx.x, d = p.d;
  const float inv_d = 1.f / (float)d;
  const TS* const x = static_cast<const TS*>(p.x) + row * p.ldx;
  const TB* const y = p.y ? static_cast<const TB*>(p.y) + row * p.ldy : nullptr;
  const float* const gate = p.gate ? p.gate + row / p.per_gate * p.ldg : nullptr;
  float h[CHUNKS][8];
  float r1 = 1.f;
  Raw8<TS> xr[CHUNKS];
  Raw8<TB> yr[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    xr[c] = e < d ? row_load<ALIGNED>(x, e, d) : raw_zero<TS>();
    yr[c] = y && e < d ? row_load<ALIGNED>(y, e, d) : raw_zero<TB>();
  }
  if (p.post) {
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      float v[8];
      raw_get(yr[c], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] = fmaf(v[i], v[i], s[0]);
    }
    cta_sums(s, red[0]);
    r1 = rsqrtf(s[0] * inv_d + p.eps);
  }
  float s[1] = {0.f};
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    float v[8], xv[8];
    raw_get(yr[c], v);
    raw_get(xr[c], xv);
    if (p.w_post) {
      float w[8];
      raw_get(e < d ? row_load<ALIGNED>(p.w_post, e, d) : raw_zero<float>(), w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (gate) {
      float w[8];
      raw_get(e < d ? row_load<ALIGNED>(gate, e, d) : raw_zero<float>(), w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[c][i] = fmaf(r1, v[i], p.a * xv[i]);
      s[0] = fmaf(h[c][i], h[c][i], s[0]);
    }
    if (p.h && e < d) row_store<ALIGNED>(static_cast<TS*>(p.h) + row * p.ldh, e, d, h[c]);
  }
  if (!p.n && !p.q) return;
  float r2 = 1.f;
  if (p.pre) {
    cta_sums(s, red[1]);
    r2 = rsqrtf(s[0] * inv_d + p.eps);
  }
  unsigned top = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    float w[8];
    if (p.w_pre) raw_get(e < d ? row_load<ALIGNED>(p.w_pre, e, d) : raw_zero<float>(), w);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[c][i] *= p.w_pre ? r2 * w[i] : r2;
    if (p.n && e < d) row_store<ALIGNED>(static_cast<TB*>(p.n) + row * p.ldn, e, d, h[c]);
    if (p.q) top = max(top, abs_bits8(h[c]));
  }
  if (!p.q) return;
  const RowScale r = row_scale(cta_max(top, red[2]));
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    if (e < d) *reinterpret_cast<uint2*>(p.q + row * p.ldq + e) = row_round8(h[c], r);
  }
  if (threadIdx.x == 0) p.q_scale[row] = r.s;
}

struct GradP {
  int64_t rows, d, ldh, ldy, lddh, lddn, lddx, lddy, ldg, per_gate, n_gates;
  const void *h, *y, *dh, *dn;
  void *dx, *dy;
  const float *w_post, *w_pre, *gate;
  float *dw_post, *dw_pre, *dgate;     // null: not wanted
  float* part;                         // [sums][ctas][d]: dw_pre, dw_post, the gate at either end
  float a, eps;
  int post, pre, ctas;
};
// where the CTAs' sums of a parameter lie
__host__ __device__ __forceinline__ int part_pre(const GradP&) { return 0; }
__host__ __device__ __forceinline__ int part_post(const GradP& p) { return p.dw_pre ? 1 : 0; }
__host__ __device__ __forceinline__ int part_gate(const GradP& p) { return part_post(p) + (p.dw_post ? 1 : 0); }

template <typename TS, typename TB, bool ALIGNED, int CHUNKS>
__global__ void __launch_bounds__(1024)
block_norm_grad_kernel(const GradP p) {
  grid_begin();
  extern __shared__ __align__(16) float sums[];            // [dw_pre, dw_post, dgate as wanted][d rounded up to 8]
  __shared__ float red[2][2][3][32];
  const int64_t d = p.d, dp = (d + 7) / 8 * 8;
  const float inv_d = 1.f / (float)d;
  float* const s_pre = sums;
  float* const s_post = sums + (p.dw_pre ? dp : 0);
  float* const s_gate = s_post + (p.dw_post ? dp : 0);
  const int64_t r_lo = rows_lo(blockIdx.x, p.rows, p.ctas), r_hi = rows_lo(blockIdx.x + 1, p.rows, p.ctas);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
      if (e < d) f(c, e);
    }
  };
  auto zero = [&](float* at) {
    each([&](int, int64_t e) {
#pragma unroll
      for (int i = 0; i < 8; ++i) at[e + i] = 0.f;
    });
  };
  // the elements of `at` to a row of d floats
  auto spill = [&](const float* at, float* out) {
    each([&](int, int64_t e) {
      for (int i = 0; i < 8 && e + i < d; ++i) out[e + i] = at[e + i];
    });
  };
  if (p.dw_pre) zero(s_pre);
  if (p.dw_post) zero(s_post);
  if (p.dgate) zero(s_gate);
  const int64_t g_first = p.dgate ? r_lo / p.per_gate : 0;
  auto gate_done = [&](int64_t g) {
    // alone with the gate's rows: its gradient; else a sum for the CTA's first or its last gate
    const int64_t g0 = g * p.per_gate, g1 = g0 + p.per_gate < p.rows ? g0 + p.per_gate : p.rows;
    float* const out = r_lo <= g0 && g1 <= r_hi ? p.dgate + g * d
                                                : p.part + ((int64_t)(part_gate(p) + (g == g_first ? 0 : 1)) * p.ctas + blockIdx.x) * d;
    spill(s_gate, out);
  };
  for (int64_t row = r_lo; row < r_hi; ++row) {
    float (*const buf)[3][32] = red[row & 1];
    const TS* const hrow = p.h ? static_cast<const TS*>(p.h) + row * p.ldh : nullptr;
    const TB* const yrow = p.y ? static_cast<const TB*>(p.y) + row * p.ldy : nullptr;
    const TS* const dhrow = p.dh ? static_cast<const TS*>(p.dh) + row * p.lddh : nullptr;
    const TB* const dnrow = p.dn ? static_cast<const TB*>(p.dn) + row * p.lddn : nullptr;
    const float* const gate = p.gate ? p.gate + row / p.per_gate * p.ldg : nullptr;
    Raw8<TS> hr[CHUNKS], dhr[CHUNKS];
    Raw8<TB> yr[CHUNKS], dnr[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
      hr[c] = hrow && e < d ? row_load<ALIGNED>(hrow, e, d) : raw_zero<TS>();
      dhr[c] = dhrow && e < d ? row_load<ALIGNED>(dhrow, e, d) : raw_zero<TS>();
      yr[c] = yrow && e < d ? row_load<ALIGNED>(yrow, e, d) : raw_zero<TB>();
      dnr[c] = dnrow && e < d ? row_load<ALIGNED>(dnrow, e, d) : raw_zero<TB>();
    }
    // h.h, (dn w_pre).h, y.y
    float s[3] = {0.f, 0.f, 0.f};
    float r1 = 1.f, r2 = 1.f, m2 = 0.f;
    if (p.pre || p.post) {
      each([&](int c, int64_t e) {
        float hv[8], gv[8], yv[8];
        raw_get(hr[c], hv); raw_get(dnr[c], gv); raw_get(yr[c], yv);
        if (p.w_pre) {
          float w[8];
          raw_get(row_load<ALIGNED>(p.w_pre, e, d), w);
#pragma unroll
          for (int i = 0; i < 8; ++i) gv[i] *= w[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] = fmaf(hv[i], hv[i], s[0]);
          s[1] = fmaf(gv[i], hv[i], s[1]);
          s[2] = fmaf(yv[i], yv[i], s[2]);
        }
      });
      cta_sums(s, buf[0]);
      if (p.pre) {
        r2 = rsqrtf(s[0] * inv_d + p.eps);
        m2 = s[1] * inv_d * r2 * r2;                        // mean(g hbar) / rms(h)
      }
      if (p.post) r1 = rsqrtf(s[2] * inv_d + p.eps);
    }
    float f[CHUNKS][8];                                     // dh', then e, then f
    float sf[1] = {0.f};
    each([&](int c, int64_t e) {
      float hv[8], nv[8], dv[8], yv[8], w[8];
      raw_get(hr[c], hv); raw_get(dnr[c], nv); raw_get(dhr[c], dv); raw_get(yr[c], yv);
      if (p.w_pre) raw_get(row_load<ALIGNED>(p.w_pre, e, d), w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float g = p.w_pre ? nv[i] * w[i] : nv[i];
        f[c][i] = dv[i] + (p.pre ? r2 * (g - hv[i] * m2) : g);
      }
      if (p.dw_pre) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_pre[e + i] = fmaf(nv[i], hv[i] * r2, s_pre[e + i]);
      }
      if (p.dx) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = p.a * f[c][i];
        row_store<ALIGNED>(static_cast<TS*>(p.dx) + row * p.lddx, e, d, o);
      }
      float wp[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { wp[i] = 1.f; yv[i] *= r1; }
      if (p.w_post) raw_get(row_load<ALIGNED>(p.w_post, e, d), wp);
      if (p.dgate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_gate[e + i] = fmaf(f[c][i], yv[i] * wp[i], s_gate[e + i]);
      }
      if (gate) {
        raw_get(row_load<ALIGNED>(gate, e, d), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[c][i] *= w[i];
      }
      if (p.dw_post) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_post[e + i] = fmaf(f[c][i], yv[i], s_post[e + i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[c][i] *= wp[i];
        sf[0] = fmaf(f[c][i], yv[i], sf[0]);
      }
    });
    if (p.dy) {
      float m1 = 0.f;
      if (p.post) {
        cta_sums(sf, buf[1]);
        m1 = sf[0] * inv_d * r1;                            // mean(f ybar) / rms(y)
      }
      each([&](int c, int64_t e) {
        float yv[8], o[8];
        raw_get(yr[c], yv);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = p.post ? r1 * (f[c][i] - yv[i] * m1) : f[c][i];
        row_store<ALIGNED>(static_cast<TB*>(p.dy) + row * p.lddy, e, d, o);
      });
    }
    if (p.dgate && (row + 1 == r_hi || (row + 1) % p.per_gate == 0)) {
      gate_done(row / p.per_gate);
      zero(s_gate);
    }
  }
  if (p.dw_pre) spill(s_pre, p.part + ((int64_t)part_pre(p) * p.ctas + blockIdx.x) * d);
  if (p.dw_post) spill(s_post, p.part + ((int64_t)part_post(p) * p.ctas + blockIdx.x) * d);
}

// The CTAs' sums added up in order: blockIdx.y = 0, 1: the weights' gradients, from 2 on: the gates'.  32 columns x 8 lanes of CTAs.
__global__ void __launch_bounds__(256)
block_norm_grad_sums_kernel(const GradP p) {
  grid_begin();
  __shared__ double add[8][32];
  const int64_t col = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int lane = threadIdx.x >> 5;
  for (int64_t y = blockIdx.y; y < 2 + (p.dgate ? p.n_gates : 0); y += gridDim.y) {
    int64_t b0 = 0, b1 = p.ctas;
    float* out;
    const float* part;
    int64_t gate = -1;
    if (y == 0) { out = p.dw_pre; part = p.part + (int64_t)part_pre(p) * p.ctas * p.d; }
    else if (y == 1) { out = p.dw_post; part = p.part + (int64_t)part_post(p) * p.ctas * p.d; }
    else {
      gate = y - 2;
      out = p.dgate + gate * p.d;
      part = p.part + (int64_t)part_gate(p) * p.ctas * p.d;
      const int64_t g0 = gate * p.per_gate, g1 = g0 + p.per_gate < p.rows ? g0 + p.per_gate : p.rows;
      if (g0 >= p.rows) b1 = 0;                             // no rows of its own
      else {
        b0 = rows_owner(g0, p.rows, p.ctas);
        b1 = rows_owner(g1 - 1, p.rows, p.ctas) + 1;
        if (b1 == b0 + 1) continue;                         // the CTA has written it
      }
    }
    if (!out) continue;
    double t = 0.0;
    if (col < p.d)
      for (int64_t b = b0 + lane; b < b1; b += 8) {
        // a gate that is not the CTA's first lies in the CTA's second sum
        const bool second = gate >= 0 && rows_lo(b, p.rows, p.ctas) / p.per_gate != gate;
        t += (double)part[((second ? p.ctas : 0) + b) * p.d + col];
      }
    __syncthreads();
    add[lane][threadIdx.x & 31] = t;
    __syncthreads();
    if (lane == 0 && col < p.d) {
#pragma unroll
      for (int k = 1; k < 8; ++k) t += add[k][threadIdx.x & 31];
      out[col] = (float)t;
    }
  }
}

template <typename TS, typename TB, bool ALIGNED>
void launch_norm(const NormP& p, int64_t rows, cudaStream_t s) {
  const int64_t units = (p.d + 7) / 8;
  auto threads = [&](int chunks) { return dim3((unsigned)(((units + chunks - 1) / chunks + 31) / 32 * 32)); };
  const dim3 grid((unsigned)rows);
  if (units <= 128 || (rows <= 148 && units <= 1024)) launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 1>, grid, threads(1), 0, s, p);
  else if (units <= 512) launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 2>, grid, threads(2), 0, s, p);
  else launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 4>, grid, threads(4), 0, s, p);
}
template <typename TS, typename TB, bool ALIGNED>
armor_status launch_grad(armor_ctx* c, const GradP& p, cudaStream_t s) {
  const int64_t units = (p.d + 7) / 8;
  const int n_sums = (p.dw_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.dgate ? 1 : 0);
  const size_t smem = (size_t)n_sums * (size_t)units * 8 * sizeof(float);
  auto threads = [&](int chunks) { return dim3((unsigned)(((units + chunks - 1) / chunks + 31) / 32 * 32)); };
  if (units <= 1024) {
    static PerDeviceOnce attr;
    if (ensure_dynamic_smem(attr, c->device, block_norm_grad_kernel<TS, TB, ALIGNED, 1>, 98304) != ARMOR_OK) return ARMOR_ERR_CUDA;
    launch_dependent(block_norm_grad_kernel<TS, TB, ALIGNED, 1>, dim3((unsigned)p.ctas), threads(1), smem, s, p);
  } else {
    static PerDeviceOnce attr;
    if (ensure_dynamic_smem(attr, c->device, block_norm_grad_kernel<TS, TB, ALIGNED, 2>, 196608) != ARMOR_OK) return ARMOR_ERR_CUDA;
    launch_dependent(block_norm_grad_kernel<TS, TB, ALIGNED, 2>, dim3((unsigned)p.ctas), threads(2), smem, s, p);
  }
  c->launches++;
  if (n_sums) {
    const int64_t sets = 2 + (p.dgate ? p.n_gates : 0);
    launch_dependent(block_norm_grad_sums_kernel, dim3((unsigned)((p.d + 31) / 32), (unsigned)(sets < 64 ? sets : 64)), dim3(256), 0, s, p);
    c->launches++;
  }
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}

// TS and TB of the two dtypes, as arguments of f
template <typename F>
armor_status by_types(int32_t stream, int32_t branch, F&& f) {
  if (stream == ARMOR_DTYPE_F32) {
    if (branch == ARMOR_DTYPE_F32) return f(float(), float());
    if (branch == ARMOR_DTYPE_BF16) return f(float(), __nv_bfloat16());
    return f(float(), __half());
  }
  return stream == ARMOR_DTYPE_BF16 ? f(__nv_bfloat16(), __nv_bfloat16()) : f(__half(), __half());
}

bool row_ok(const void* p, int64_t ld, int64_t d) { return !p || ld >= d; }

// what both directions ask of their sizes and types
armor_status check_norm(int64_t rows, int64_t d, int32_t stream, int32_t branch, const void* gate, int64_t per_gate, int64_t n_gates,
                        int64_t ldg, float eps) {
  if (rows < 0 || !(eps >= 0.f)) return ARMOR_ERR_INVALID_ARG;
  if (d < 1) return ARMOR_ERR_SHAPE;
  if (d > ARMOR_BLOCK_NORM_MAX_COLS || rows > 0x7fffffff) return ARMOR_ERR_TOO_LARGE;
  if (!rows_dtype_bytes(stream) || !rows_dtype_bytes(branch)) return ARMOR_ERR_UNSUPPORTED;
  if (stream != branch && stream != ARMOR_DTYPE_F32) return ARMOR_ERR_UNSUPPORTED;
  if (gate && (per_gate < 1 || n_gates < 1 || ldg < d || (rows > 0 && n_gates - 1 < (rows - 1) / per_gate))) return ARMOR_ERR_SHAPE;
  return ARMOR_OK;
}

}  // namespace

// (sizes and types are looked at before the context)
extern "C" armor_status armor_block_norm(armor_ctx* c, const armor_block_norm_args* g, armor_stream_t stream) {
  if (!g) return ARMOR_ERR_INVALID_ARG;
  armor_status st = check_norm(g->n_rows, g->d, g->stream_dtype, g->branch_dtype, g->gate, g->rows_per_gate, g->n_gates, g->ld_gate, g->eps);
  if (st != ARMOR_OK) return st;
  if (g->n_rows > 0 && !g->y && (g->gate || g->post)) return ARMOR_ERR_INVALID_ARG;
  if ((g->w_post && !g->post) || (g->w_pre && !g->pre)) return ARMOR_ERR_INVALID_ARG;
  if (!row_ok(g->x, g->ldx, g->d) || !row_ok(g->y, g->ldy, g->d) || !row_ok(g->h, g->ldh, g->d) || !row_ok(g->n, g->ldn, g->d)) return ARMOR_ERR_SHAPE;
  if (g->q && (!rows::aligned16(g->q, g->ldq, 1) || g->ldq < g->d)) return ARMOR_ERR_SHAPE;
  if (!c || (g->q == nullptr) != (g->q_scale == nullptr)) return ARMOR_ERR_INVALID_ARG;
  if (g->n_rows == 0) return ARMOR_OK;
  if (!g->x || (!g->h && !g->n && !g->q)) return ARMOR_ERR_INVALID_ARG;
  NormP p{};
  p.rows = g->n_rows; p.d = g->d; p.ldx = g->ldx; p.ldy = g->ldy; p.ldh = g->ldh; p.ldn = g->ldn; p.ldq = g->ldq;
  p.ldg = g->ld_gate; p.per_gate = g->gate ? g->rows_per_gate : 1;
  p.x = g->x; p.y = g->y; p.h = g->h; p.n = g->n; p.q = g->q; p.q_scale = g->q_scale;
  p.w_post = g->w_post; p.w_pre = g->w_pre; p.gate = g->gate;
  p.a = g->residual_scale; p.eps = g->eps; p.post = g->post != 0; p.pre = g->pre != 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int es = rows_dtype_bytes(g->stream_dtype), eb = rows_dtype_bytes(g->branch_dtype);
  const bool al = rows::aligned16(p.x, p.ldx, es) && (!p.y || rows::aligned16(p.y, p.ldy, eb)) && (!p.h || rows::aligned16(p.h, p.ldh, es)) &&
                  (!p.n || rows::aligned16(p.n, p.ldn, eb)) && (!p.gate || rows::aligned16(p.gate, p.ldg, 4)) && rows::aligned16(p.w_post, 0, 4) &&
                  rows::aligned16(p.w_pre, 0, 4);
  KTimer kt(c, ARMOR_KC_FORWARD, (double)p.rows * (double)p.d * (es + (p.y ? eb : 0) + (p.h ? es : 0) + (p.n ? eb : 0) + (p.q ? 1 : 0)), s);
  by_types(g->stream_dtype, g->branch_dtype, [&](auto ts, auto tb) {
    using TS = decltype(ts);
    using TB = decltype(tb);
    if (al) launch_norm<TS, TB, true>(p, p.rows, s);
    else launch_norm<TS, TB, false>(p, p.rows, s);
    return ARMOR_OK;
  });
  c->launches++;
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}

extern "C" armor_status armor_block_norm_backward(armor_ctx* c, const armor_block_norm_grad_args* g, armor_stream_t stream) {
  if (!g) return ARMOR_ERR_INVALID_ARG;
  armor_status st = check_norm(g->n_rows, g->d, g->stream_dtype, g->branch_dtype, g->gate, g->rows_per_gate, g->n_gates, g->ld_gate, g->eps);
  if (st != ARMOR_OK) return st;
  if ((g->w_post && !g->post) || (g->w_pre && !g->pre)) return ARMOR_ERR_INVALID_ARG;
  if ((g->dw_post && !g->post) || (g->dw_pre && !g->pre) || (g->dgate && !g->gate)) return ARMOR_ERR_INVALID_ARG;
  if (!row_ok(g->h, g->ldh, g->d) || !row_ok(g->y, g->ldy, g->d) || !row_ok(g->dh, g->lddh, g->d) || !row_ok(g->dn, g->lddn, g->d) ||
      !row_ok(g->dx, g->lddx, g->d) || !row_ok(g->dy, g->lddy, g->d)) return ARMOR_ERR_SHAPE;
  if (!c) return ARMOR_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (g->n_rows == 0) {                                     // sums over no rows
    if (g->dw_post) ARMOR_CUDA_OK(cudaMemsetAsync(g->dw_post, 0, (size_t)g->d * 4, s));
    if (g->dw_pre) ARMOR_CUDA_OK(cudaMemsetAsync(g->dw_pre, 0, (size_t)g->d * 4, s));
    if (g->dgate) ARMOR_CUDA_OK(cudaMemsetAsync(g->dgate, 0, (size_t)g->n_gates * (size_t)g->d * 4, s));
    return ARMOR_OK;
  }
  if ((!g->dh && !g->dn) || (!g->dx && !g->dy && !g->dw_pre && !g->dw_post && !g->dgate)) return ARMOR_ERR_INVALID_ARG;
  if (!g->h && g->pre) return ARMOR_ERR_INVALID_ARG;
  if (!g->y && (g->post || g->dgate)) return ARMOR_ERR_INVALID_ARG;
  GradP p{};
  p.rows = g->n_rows; p.d = g->d; p.ldh = g->ldh; p.ldy = g->ldy; p.lddh = g->lddh; p.lddn = g->lddn; p.lddx = g->lddx; p.lddy = g->lddy;
  p.ldg = g->ld_gate; p.per_gate = g->gate ? g->rows_per_gate : 1; p.n_gates = g->gate ? g->n_gates : 0;
  p.h = g->pre ? g->h : nullptr; p.y = g->post || g->dgate ? g->y : nullptr; p.dh = g->dh; p.dn = g->dn; p.dx = g->dx; p.dy = g->dy;
  p.w_post = g->w_post; p.w_pre = g->w_pre; p.gate = g->gate;
  p.dw_post = g->dw_post; p.dw_pre = g->dw_pre; p.dgate = g->dgate;
  p.part = c->T; p.a = g->residual_scale; p.eps = g->eps; p.post = g->post != 0; p.pre = g->pre != 0;
  // Two CTAs an SM, fewer where the workspace has no room for their sums
  const int64_t sums = (p.dw_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.dgate ? 2 : 0);
  int64_t ctas = 2 * c->n_sm;
  if (ctas > p.rows) ctas = p.rows;
  if (sums && ctas > ws_scratch_bytes(c) / (sums * p.d * 4)) ctas = ws_scratch_bytes(c) / (sums * p.d * 4);
  if (ctas < 1) return ARMOR_ERR_WORKSPACE;
  p.ctas = (int)ctas;
  const int es = rows_dtype_bytes(g->stream_dtype), eb = rows_dtype_bytes(g->branch_dtype);
  const bool al = rows::aligned16(p.h, p.ldh, es) && rows::aligned16(p.y, p.ldy, eb) && rows::aligned16(p.dh, p.lddh, es) &&
                  rows::aligned16(p.dn, p.lddn, eb) && rows::aligned16(p.dx, p.lddx, es) && rows::aligned16(p.dy, p.lddy, eb) &&
                  rows::aligned16(p.gate, p.ldg, 4) && rows::aligned16(p.w_post, 0, 4) && rows::aligned16(p.w_pre, 0, 4);
  KTimer kt(c, ARMOR_KC_FORWARD, (double)p.rows * (double)p.d *
            ((p.h ? es : 0) + (p.y ? eb : 0) + (p.dh ? es : 0) + (p.dn ? eb : 0) + (p.dx ? es : 0) + (p.dy ? eb : 0)), s);
  return by_types(g->stream_dtype, g->branch_dtype, [&](auto ts, auto tb) {
    using TS = decltype(ts);
    using TB = decltype(tb);
    return al ? launch_grad<TS, TB, true>(c, p, s) : launch_grad<TS, TB, false>(c, p, s);
  });
}
