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
// The sums over rows: a CTA takes consecutive rows and adds in fp32, an element of the row by one owner, so no order is left to chance: in registers
// where rows go through the ring (the share of w_post, once a gate, in shared memory), in shared memory beyond its widths.  A second kernel
// adds the CTAs' sums in order, in fp64.  A gate's rows may end inside a CTA's: the CTA keeps two sums for the gates at its ends, and writes one
// that lies within its rows at once.
#include "rows_io.cuh"
#include "tc_common.cuh"

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

// ---------------------------------------------------------------------------------------------------------
// Many rows: persistent CTAs take consecutive rows through a ring of rows in shared memory, filled by bulk copies several rows ahead,
// and keep their share of the weights in registers.  (A CTA a row reads the three fp32 weights, 12 bytes an element, for every 8 bytes of a
// bf16 row.)  What bounds these kernels is the issue of instructions, with 16 warps an SM or fewer: hence the arithmetic in pairs, one
// barrier a row, and the copies (100 cycles each) by a warp an array.  Nothing may spill: the ring leaves L1 so little that a spilled
// register costs a trip to L2 (16,384 x 5,120 with an fp32 stream 481 us, without spills 244).  Tried and dropped: sums put down
// and picked up later through an mbarrier instead of the barrier (4,096 x 4,096 63 -> 80 us), rows cut between the CTAs of a cluster (8,192
// columns 147 -> 249), a warp of its own for the copies (17 warps leave 96 registers a thread where 16 leave 128).
constexpr int MAX_STAGES = 6;
struct Ring {
  int stages, stage_bytes;
  uint32_t off[4], bytes[4];           // where an array's row lies in a stage, and its length, 0: not there
  int arrays;                          // of them
};
struct RingBars { uint64_t full[MAX_STAGES]; int abort_flag; };

__device__ __forceinline__ void ring_open(RingBars& b, const Ring& ring) {
  if (threadIdx.x == 0) {
    b.abort_flag = 0;
    for (int k = 0; k < ring.stages; ++k) tc::mbar_init(tc::smem_u32(&b.full[k]), ring.arrays);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
}
// The array that this thread copies.  A row that starts or ends off a 16-byte boundary is copied from the boundary before to the
// one behind: up to 15 bytes more, of the same 16-byte words and never looked at.
struct RingCopy {
  const char* base;                    // the array, null: this thread copies none
  int64_t ld;                          // bytes from row to row
  uint32_t bytes, off;
  __device__ __forceinline__ RingCopy(const Ring& ring, const void* const (&at)[4], const int64_t (&lds)[4]) : base(nullptr), ld(0), bytes(0), off(0) {
    const int per = blockDim.x >= 128 ? 32 : 1;
#pragma unroll
    for (int k = 0; k < 4; ++k)                             // (selected, not indexed: an array in registers has no address)
      if ((int)threadIdx.x == k * per && ring.bytes[k]) { base = static_cast<const char*>(at[k]); ld = lds[k]; bytes = ring.bytes[k]; off = ring.off[k]; }
  }
  __device__ __forceinline__ void operator()(RingBars& b, const Ring& ring, uint8_t* mem, int64_t row, int stage) const {
    if (!base) return;
    const char* const from = base + row * ld;
    const uint32_t skip = (uint32_t)reinterpret_cast<uintptr_t>(from) & 15u, len = (skip + bytes + 15u) & ~15u;
    const uint32_t bar = tc::smem_u32(&b.full[stage]);
    tc::mbar_expect_tx(bar, len);
    tc::bulk_load(tc::smem_u32(mem) + (uint32_t)(stage * ring.stage_bytes) + off, from - skip, len, bar);
  }
};
// A wait that gave up has raised the status word and the others have run on without waits: nothing is in flight towards shared memory
// when the kernel leaves, a bounded wait for the last of every stage.
__device__ __forceinline__ void ring_drain(RingBars& b, const Ring& ring, int64_t rows) {
  if (threadIdx.x != 0 || !*(volatile int*)&b.abort_flag) return;
  for (int k = 0; k < ring.stages && k < rows; ++k) {
    const uint32_t last = (uint32_t)((rows - 1 - k) / ring.stages) & 1u;
    const long long t0 = clock64();
    while (!tc::mbar_try(tc::smem_u32(&b.full[k]), last) && clock64() - t0 < 20000000ll) {}
  }
}
// where row `row` of an array lies in a stage
template <typename T>
__device__ __forceinline__ const T* in_stage(const uint8_t* at, const T* base, int64_t row, int64_t ld, bool al) {
  return reinterpret_cast<const T*>(at + (al ? 0 : (reinterpret_cast<uintptr_t>(base + row * ld) & 15)));
}
// Sums of N (2 or 8) values at once over the CTA: the lanes of a warp halve the values between them before they add (8: 9 shuffles where one
// value at a time takes 40); 32 / N neighbouring lanes end with one each.  Between two uses of a buffer lies the barrier of a use of
// another.
template <int N>
__device__ __forceinline__ void sums_over(float (&v)[N], float (*buf)[32]) {
  constexpr int LANES = 32 / N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
  for (int half = N / 2, o = 16; half > 0; half >>= 1, o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int k = 0; k < half; ++k) {
      const float give = up ? v[k] : v[k + half], keep = up ? v[k + half] : v[k];
      v[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  float t = v[0];
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (lane % LANES == 0) buf[lane / LANES][warp] = t;
  __syncthreads();
  t = 0.f;
  for (int w = lane % LANES; w < warps; w += LANES) t += buf[lane / LANES][w];
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, t, k * LANES);
}

// A thread's share of a row: NU units of U elements.  AL: of consecutive ones; else two elements nt apart, so that rows may start anywhere
// and neighbouring lanes touch neighbouring elements.
template <int U_, int NU_, bool AL>
struct Share {
  static constexpr int U = U_, NU = NU_;
  uint32_t e0, step, nt, n;
  __device__ __forceinline__ Share(int threads, uint32_t n_el) : nt(threads), n(n_el) { e0 = threadIdx.x * (AL ? U : 1); step = threads * U; }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int c = 0; c < NU; ++c) {
      const uint32_t e = e0 + c * step;
      if (e < n) f(c, e);
    }
  }
  template <typename T>
  __device__ __forceinline__ void get(const T* p, uint32_t e, F2 (&v)[U / 2]) const {
    if constexpr (AL) get_u<U>(p + e, v);
    else v[0] = f2(to_f(p[e]), e + nt < n ? to_f(p[e + nt]) : 0.f);
  }
  template <typename T>
  __device__ __forceinline__ void put(T* p, uint32_t e, const F2 (&v)[U / 2]) const {
    if constexpr (AL) put_u<U>(p + e, v);
    else {
      const float2 f = f2_get(v[0]);
      p[e] = from_f<T>(f.x);
      if (e + nt < n) p[e + nt] = from_f<T>(f.y);
    }
  }
  // gate (.) w_post
  __device__ __forceinline__ void gain(const float* w_post, const float* gate, F2 (&G)[NU][U / 2]) const {
    each([&](int c, uint32_t e) {
      F2 g[U / 2];
      if (w_post) get(w_post, e, G[c]);
      if (gate) {
        get(gate, e, g);
#pragma unroll
        for (int i = 0; i < U / 2; ++i) G[c][i] = w_post ? f2_mul(G[c][i], g[i]) : g[i];
      }
    });
  }
};
// (AL: rows on 16-byte boundaries of whole units.  A unit that ends behind its row would take what lies there into the sums and write it.)
template <typename TS, typename TB, int CHUNKS, bool AL>
struct ShareOf {
  static constexpr int U = !AL ? 2 : (sizeof(TS) == 4 || sizeof(TB) == 4 ? 4 : 8);
  typedef Share<U, CHUNKS * 8 / U, AL> type;
};

// HAS_Y: there is a branch
template <typename TS, typename TB, int CHUNKS, int THREADS, bool HAS_Y, bool AL>
__global__ void __launch_bounds__(THREADS, 1)
block_norm_ring_kernel(const NormP p, const Ring ring, int32_t* status) {
  grid_begin();
  typedef typename ShareOf<TS, TB, CHUNKS, AL>::type S;
  constexpr int U = S::U, NU = S::NU;
  extern __shared__ __align__(16) uint8_t stage_mem[];
  __shared__ __align__(8) RingBars bars;
  __shared__ float red[3][2][32];
  const int64_t r_lo = rows_lo(blockIdx.x, p.rows, gridDim.x), r_hi = rows_lo(blockIdx.x + 1, p.rows, gridDim.x);
  ring_open(bars, ring);
  const TS* const x0 = static_cast<const TS*>(p.x);
  const TB* const y0 = static_cast<const TB*>(p.y);
  const RingCopy mine(ring, {x0, y0, nullptr, nullptr}, {p.ldx * (int64_t)sizeof(TS), p.ldy * (int64_t)sizeof(TB), 0, 0});
  auto copy = [&](int64_t row, int stage) { mine(bars, ring, stage_mem, row, stage); };
  for (int64_t r = r_lo; r < r_hi && r < r_lo + ring.stages; ++r) copy(r, (int)(r - r_lo));
  volatile int* const abortp = &bars.abort_flag;
  const S my(blockDim.x, (uint32_t)p.d);
  const uint32_t full0 = tc::smem_u32(bars.full);
  const float inv_d = 1.f / (float)p.d;
  F2 wpre[NU][U / 2], G[NU][U / 2], h[NU][U / 2];
#pragma unroll
  for (int c = 0; c < NU; ++c)
#pragma unroll
    for (int i = 0; i < U / 2; ++i) { wpre[c][i] = f2(1.f); G[c][i] = f2(1.f); }
  if (p.w_pre) my.each([&](int c, uint32_t e) { my.get(p.w_pre, e, wpre[c]); });
  int64_t at = p.gate ? r_lo / p.per_gate : 0, until = p.gate ? (at + 1) * p.per_gate : p.rows;
  if (HAS_Y) my.gain(p.w_post, p.gate ? p.gate + at * p.ldg : nullptr, G);
  // sum y^2 of a row in a stage
  auto square_y = [&](int64_t row, int stage) {
    const TB* const y = in_stage(stage_mem + (size_t)stage * ring.stage_bytes + ring.off[1], y0, row, p.ldy, AL);
    F2 s = 0;
    my.each([&](int, uint32_t e) {
      F2 v[U / 2];
      my.get(y, e, v);
#pragma unroll
      for (int i = 0; i < U / 2; ++i) s = f2_fma(v[i], v[i], s);
    });
    return f2_sum(s);
  };
  // The sum over y of the row to come is formed beside that over h of the row at hand: one barrier a row, and one ahead of the first.
  const bool post = HAS_Y && p.post;
  const F2 a2 = f2(p.a);
  int stage = 0;
  uint32_t phase = 0;
  float r1 = 1.f;
  tc::mbar_wait(full0, 0, abortp, status);
  if (post) {
    float s[2] = {square_y(r_lo, 0), 0.f};
    sums_over(s, red[2]);
    r1 = rsqrtf(s[0] * inv_d + p.eps);
  }
  for (int64_t row = r_lo; row < r_hi; ++row) {
    const int here = stage;
    const uint8_t* const mem = stage_mem + (size_t)here * ring.stage_bytes;
    const TS* const x = in_stage(mem, x0, row, p.ldx, AL);
    const TB* const y = in_stage(mem + ring.off[1], y0, row, p.ldy, AL);
    if (HAS_Y && row == until) { my.gain(p.w_post, p.gate + ++at * p.ldg, G); until += p.per_gate; }
    F2 hh = 0;
    const F2 r12 = f2(r1);
    my.each([&](int c, uint32_t e) {
      F2 v[U / 2], xv[U / 2];
      my.get(x, e, xv);
      if (HAS_Y) my.get(y, e, v);
#pragma unroll
      for (int i = 0; i < U / 2; ++i) {
        h[c][i] = f2_mul(a2, xv[i]);
        if (HAS_Y) h[c][i] = f2_fma(f2_mul(v[i], G[c][i]), r12, h[c][i]);
        hh = f2_fma(h[c][i], h[c][i], hh);
      }
      if (p.h) my.put(static_cast<TS*>(p.h) + row * p.ldh, e, h[c]);
    });
    if (++stage == ring.stages) { stage = 0; phase ^= 1; }
    float s[2] = {f2_sum(hh), 0.f};
    if (row + 1 < r_hi) {
      tc::mbar_wait(full0 + 8 * stage, phase, abortp, status);
      if (post) s[1] = square_y(row + 1, stage);
    }
    sums_over(s, red[row & 1]);
    if (row + ring.stages < r_hi) copy(row + ring.stages, here);       // every thread has read the row
    if (post) r1 = rsqrtf(s[1] * inv_d + p.eps);
    const F2 r2 = f2(p.pre ? rsqrtf(s[0] * inv_d + p.eps) : 1.f);
    my.each([&](int c, uint32_t) {
#pragma unroll
      for (int i = 0; i < U / 2; ++i) h[c][i] = f2_mul(h[c][i], f2_mul(r2, wpre[c][i]));
    });
    if (p.n) my.each([&](int c, uint32_t e) { my.put(static_cast<TB*>(p.n) + row * p.ldn, e, h[c]); });
    if (p.q) {
      unsigned top = 0;
      my.each([&](int c, uint32_t e) {
#pragma unroll
        for (int i = 0; i < U / 2; ++i) {
          const float2 t = f2_get(h[c][i]);
          top = max(top, max(__float_as_uint(t.x) & 0x7fffffffu, AL || e + my.nt < my.n ? __float_as_uint(t.y) & 0x7fffffffu : 0u));
        }
      });
      const RowScale r = row_scale(cta_max(top, red[2]));
      int8_t* const q = p.q + row * p.ldq;
      my.each([&](int c, uint32_t e) {
        float v[U];
#pragma unroll
        for (int i = 0; i < U / 2; ++i) { const float2 t = f2_get(h[c][i]); v[2 * i] = t.x; v[2 * i + 1] = t.y; }
        if constexpr (U == 8) *reinterpret_cast<uint2*>(q + e) = make_uint2(row_round4(v, r), row_round4(v + 4, r));
        else if constexpr (U == 4) *reinterpret_cast<uint32_t*>(q + e) = row_round4(v, r);
        else {
          q[e] = (int8_t)row_round(v[0], r);
          if (e + my.nt < my.n) q[e + my.nt] = (int8_t)row_round(v[1], r);
        }
      });
      if (threadIdx.x == 0) p.q_scale[row] = r.s;
    }
  }
  ring_drain(bars, ring, r_hi - r_lo);
}

struct GradP {
  int64_t rows, d, ldh, ldy, lddh, lddn, lddx, lddy, ldg, per_gate, gates_used;
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
  // dw_pre, dw_post, dgate as wanted: eight floats of a thread and chunk as two times four, [chunk][two][thread], so that a warp's accesses
  // meet no bank twice (eight floats side by side: 2,000 x 14,336 bf16 235 us, so 217)
  extern __shared__ float4 sums[];
  __shared__ float red[2][2][3][32];
  const int64_t d = p.d;
  const int dp = CHUNKS * 2 * blockDim.x;
  const float inv_d = 1.f / (float)d;
  float4* const s_pre = sums + threadIdx.x;
  float4* const s_post = s_pre + (p.dw_pre ? dp : 0);
  float4* const s_gate = s_post + (p.dw_post ? dp : 0);
  const int64_t r_lo = rows_lo(blockIdx.x, p.rows, p.ctas), r_hi = rows_lo(blockIdx.x + 1, p.rows, p.ctas);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
      if (e < d) f(c, e);
    }
  };
  auto zero = [&](float4* at) {
#pragma unroll
    for (int k = 0; k < 2 * CHUNKS; ++k) at[k * blockDim.x] = make_float4(0.f, 0.f, 0.f, 0.f);
  };
  auto add = [&](float4* at, int c, const float (&a)[8], const float (&b)[8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float4& v = at[(2 * c + k) * blockDim.x];
      float4 t = v;
      t.x = fmaf(a[4 * k], b[4 * k], t.x); t.y = fmaf(a[4 * k + 1], b[4 * k + 1], t.y);
      t.z = fmaf(a[4 * k + 2], b[4 * k + 2], t.z); t.w = fmaf(a[4 * k + 3], b[4 * k + 3], t.w);
      v = t;
    }
  };
  // the elements of `at` to a row of d floats
  auto spill = [&](const float4* at, float* out) {
    each([&](int c, int64_t e) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float4 t = at[(2 * c + k) * blockDim.x];
        const float v[4] = {t.x, t.y, t.z, t.w};
        if (ALIGNED && d % 4 == 0) {
          if (e + 4 * k < d) *reinterpret_cast<float4*>(out + e + 4 * k) = t;
          continue;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (e + 4 * k + i < d) out[e + 4 * k + i] = v[i];
      }
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
        for (int i = 0; i < 8; ++i) hv[i] *= r2;
        add(s_pre, c, nv, hv);
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
        float u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = yv[i] * wp[i];
        add(s_gate, c, f[c], u);
      }
      if (gate) {
        raw_get(row_load<ALIGNED>(gate, e, d), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[c][i] *= w[i];
      }
      if (p.dw_post) add(s_post, c, f[c], yv);
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

// The gradient through the same ring.  One barrier a row: sum f y, which needs dh', is taken apart,
//   sum f y = sum (G y) dh + (sum (G y) g - mean(g hbar) / rms(h) sum (G y) h) / rms(h),   G = gate (.) w_post,
// so that all six sums of a row are formed at once.  And one running sum serves both the gate and w_post: t = sum dh' ybar over the rows of a
// gate gives dgate = w_post t, and gate t is what these rows add to dw_post.
//
// HAS_Y: y is read.  Without it there is no norm of it and no gradient of the gate; a gate may still stand between dh' and dy.
// KEEP: a thread's share of the four arrays stays in registers between the sums and the gradients; else it is read (and widened) again.
template <typename TS, typename TB, int CHUNKS, int THREADS, bool HAS_Y, bool AL>
__global__ void __launch_bounds__(THREADS, 1)
block_norm_grad_ring_kernel(const GradP p, const Ring ring, int32_t* status) {
  grid_begin();
  typedef typename ShareOf<TS, TB, CHUNKS, AL>::type S;
  constexpr int U = S::U, NU = S::NU, N_SUMS = HAS_Y ? 8 : 2;
  constexpr bool KEEP = CHUNKS == 1;
  extern __shared__ __align__(16) uint8_t stage_mem[];
  __shared__ __align__(8) RingBars bars;
  __shared__ float red[2][N_SUMS][32];
  const int64_t d = p.d;
  const int64_t r_lo = rows_lo(blockIdx.x, p.rows, p.ctas), r_hi = rows_lo(blockIdx.x + 1, p.rows, p.ctas);
  ring_open(bars, ring);
  const TS* const h0 = static_cast<const TS*>(p.h);
  const TB* const y0 = static_cast<const TB*>(p.y);
  const TS* const dh0 = static_cast<const TS*>(p.dh);
  const TB* const dn0 = static_cast<const TB*>(p.dn);
  const RingCopy mine(ring, {h0, y0, dh0, dn0}, {p.ldh * (int64_t)sizeof(TS), p.ldy * (int64_t)sizeof(TB), p.lddh * (int64_t)sizeof(TS), p.lddn * (int64_t)sizeof(TB)});
  auto copy = [&](int64_t row, int stage) { mine(bars, ring, stage_mem, row, stage); };
  for (int64_t r = r_lo; r < r_hi && r < r_lo + ring.stages; ++r) copy(r, (int)(r - r_lo));
  volatile int* const abortp = &bars.abort_flag;
  const S my(blockDim.x, (uint32_t)d);
  const uint32_t full0 = tc::smem_u32(bars.full);
  float* const s_post = reinterpret_cast<float*>(stage_mem + (size_t)ring.stages * ring.stage_bytes);    // dw_post so far
  const float inv_d = 1.f / (float)d;
  // an array that is not given is read from a row of zeros behind the sums (a thread reads what it has written there)
  const int64_t d8 = (d + 7) / 8 * 8;
  uint8_t* const zeros = reinterpret_cast<uint8_t*>(s_post) + (HAS_Y && p.dw_post ? d8 * 4 : 0);
  uint8_t* const zeros_b = sizeof(TB) == sizeof(TS) ? zeros : zeros + d8 * sizeof(TS);
  if (!p.h || !p.dh || !p.dn) my.each([&](int, uint32_t e) {
    F2 z[U / 2];
#pragma unroll
    for (int i = 0; i < U / 2; ++i) z[i] = 0;
    my.put(reinterpret_cast<TS*>(zeros), e, z);
    my.put(reinterpret_cast<TB*>(zeros_b), e, z);
  });
  F2 wpre[NU][U / 2], G[NU][U / 2], a_pre[NU][U / 2], a_t[NU][U / 2];
#pragma unroll
  for (int c = 0; c < NU; ++c)
#pragma unroll
    for (int i = 0; i < U / 2; ++i) { wpre[c][i] = f2(1.f); G[c][i] = f2(1.f); a_pre[c][i] = 0; a_t[c][i] = 0; }
  if (p.w_pre) my.each([&](int c, uint32_t e) { my.get(p.w_pre, e, wpre[c]); });
  const int64_t g_first = p.gate ? r_lo / p.per_gate : 0;
  int64_t at = g_first, until = p.gate ? (at + 1) * p.per_gate : p.rows;
  // (dy = gate (.) dh' needs no y)
  const bool gated = HAS_Y || (p.gate && p.dy);
  if (gated) my.gain(p.w_post, p.gate ? p.gate + at * p.ldg : nullptr, G);
  if (HAS_Y && p.dw_post) my.each([&](int, uint32_t e) {
    F2 z[U / 2];
#pragma unroll
    for (int i = 0; i < U / 2; ++i) z[i] = 0;
    my.put(s_post, e, z);
  });
  // the rows of a gate are through (or the CTA's share of them): its gradient or a sum for the CTA's first or its last gate, and dw_post
  auto gate_done = [&](int64_t g) {
    const int64_t g0 = g * p.per_gate, g1 = g0 + p.per_gate < p.rows ? g0 + p.per_gate : p.rows;
    float* const out = !p.dgate ? nullptr : (r_lo <= g0 && g1 <= r_hi ? p.dgate + g * d
                                  : p.part + ((int64_t)(part_gate(p) + (g == g_first ? 0 : 1)) * p.ctas + blockIdx.x) * d);
    my.each([&](int c, uint32_t e) {
      F2 w[U / 2], v[U / 2];
      if (out) {
        if (p.w_post) my.get(p.w_post, e, w);
#pragma unroll
        for (int i = 0; i < U / 2; ++i) v[i] = p.w_post ? f2_mul(w[i], a_t[c][i]) : a_t[c][i];
        my.put(out, e, v);
      }
      if (p.dw_post) {
        if (p.gate) my.get(p.gate + g * p.ldg, e, w);
        my.get(static_cast<const float*>(s_post), e, v);
#pragma unroll
        for (int i = 0; i < U / 2; ++i) v[i] = f2_fma(p.gate ? w[i] : f2(1.f), a_t[c][i], v[i]);
        my.put(s_post, e, v);
      }
#pragma unroll
      for (int i = 0; i < U / 2; ++i) a_t[c][i] = 0;
    });
  };
  const F2 a2 = f2(p.a);
  int stage = 0, before = 0;
  uint32_t phase = 0;
  for (int64_t row = r_lo; row < r_hi; ++row) {
    const int here = stage;
    const uint8_t* const mem = stage_mem + (size_t)here * ring.stage_bytes;
    const TS* const h = p.h ? in_stage(mem + ring.off[0], h0, row, p.ldh, AL) : reinterpret_cast<const TS*>(zeros);
    const TB* const y = in_stage(mem + ring.off[1], y0, row, p.ldy, AL);
    const TS* const dh = p.dh ? in_stage(mem + ring.off[2], dh0, row, p.lddh, AL) : reinterpret_cast<const TS*>(zeros);
    const TB* const dn = p.dn ? in_stage(mem + ring.off[3], dn0, row, p.lddn, AL) : reinterpret_cast<const TB*>(zeros_b);
    if (gated && row == until) { my.gain(p.w_post, p.gate + ++at * p.ldg, G); until += p.per_gate; }
    tc::mbar_wait(full0 + 8 * here, phase, abortp, status);
    if (++stage == ring.stages) { stage = 0; phase ^= 1; }
    F2 hv[KEEP ? NU : 1][U / 2], nv[KEEP ? NU : 1][U / 2], yv[KEEP ? NU : 1][U / 2], dv[KEEP ? NU : 1][U / 2];
    F2 q[6] = {0, 0, 0, 0, 0, 0};
    my.each([&](int c, uint32_t e) {
      const int k = KEEP ? c : 0;
      my.get(h, e, hv[k]);
      my.get(dn, e, nv[k]);
      if (HAS_Y) my.get(y, e, yv[k]);
      if (HAS_Y || KEEP) my.get(dh, e, dv[k]);
#pragma unroll
      for (int i = 0; i < U / 2; ++i) {
        const F2 g = f2_mul(nv[k][i], wpre[c][i]);
        q[0] = f2_fma(hv[k][i], hv[k][i], q[0]);
        q[1] = f2_fma(g, hv[k][i], q[1]);
        if (HAS_Y) {
          const F2 u = f2_mul(yv[k][i], G[c][i]);
          q[2] = f2_fma(yv[k][i], yv[k][i], q[2]);
          q[3] = f2_fma(u, dv[k][i], q[3]);
          q[4] = f2_fma(u, g, q[4]);
          q[5] = f2_fma(u, hv[k][i], q[5]);
        }
      }
    });
    float s[N_SUMS];
#pragma unroll
    for (int i = 0; i < N_SUMS; ++i) s[i] = i < 6 ? f2_sum(q[i]) : 0.f;
    sums_over(s, red[row & 1]);
    // KEEP: every thread has read the row, else the row before; its place takes another one
    if (KEEP) {
      if (row + ring.stages < r_hi) copy(row + ring.stages, here);
    } else {
      if (row > r_lo && row - 1 + ring.stages < r_hi) copy(row - 1 + ring.stages, before);
      before = here;
    }
    const float r2 = p.pre ? rsqrtf(s[0] * inv_d + p.eps) : 1.f, m2 = p.pre ? s[1] * inv_d * r2 * r2 : 0.f;
    float r1 = 1.f, m1 = 0.f;
    if (HAS_Y && p.post) {
      r1 = rsqrtf(s[2 % N_SUMS] * inv_d + p.eps);
      m1 = (s[3 % N_SUMS] + r2 * (s[4 % N_SUMS] - m2 * s[5 % N_SUMS])) * inv_d * r1 * r1;
    }
    const F2 r22 = f2(r2), r12 = f2(r1), c2 = f2(-r2 * m2), c1 = f2(-r1 * m1);
    my.each([&](int c, uint32_t e) {
      const int k = KEEP ? c : 0;
      F2 o[U / 2];
      if (!KEEP) {
        my.get(h, e, hv[k]);
        my.get(dn, e, nv[k]);
        my.get(dh, e, dv[k]);
        if (HAS_Y) my.get(y, e, yv[k]);
      }
#pragma unroll
      for (int i = 0; i < U / 2; ++i) {
        dv[k][i] = f2_fma(hv[k][i], c2, f2_fma(f2_mul(nv[k][i], wpre[c][i]), r22, dv[k][i]));           // dh'
        o[i] = f2_mul(a2, dv[k][i]);
        a_pre[c][i] = f2_fma(nv[k][i], f2_mul(hv[k][i], r22), a_pre[c][i]);
        if (HAS_Y) a_t[c][i] = f2_fma(dv[k][i], f2_mul(yv[k][i], r12), a_t[c][i]);
      }
      if (p.dx) my.put(static_cast<TS*>(p.dx) + row * p.lddx, e, o);
      if (HAS_Y) {
#pragma unroll
        for (int i = 0; i < U / 2; ++i) dv[k][i] = f2_fma(yv[k][i], c1, f2_mul(f2_mul(G[c][i], dv[k][i]), r12));
      } else {
#pragma unroll
        for (int i = 0; i < U / 2; ++i) dv[k][i] = f2_mul(G[c][i], dv[k][i]);
      }
      if (p.dy) my.put(static_cast<TB*>(p.dy) + row * p.lddy, e, dv[k]);
    });
    if (HAS_Y && (row + 1 == until || row + 1 == r_hi)) gate_done(at);
  }
  if (p.dw_pre) my.each([&](int c, uint32_t e) { my.put(p.part + ((int64_t)part_pre(p) * p.ctas + blockIdx.x) * d, e, a_pre[c]); });
  if (HAS_Y && p.dw_post) my.each([&](int, uint32_t e) {
    F2 v[U / 2];
    my.get(static_cast<const float*>(s_post), e, v);
    my.put(p.part + ((int64_t)part_post(p) * p.ctas + blockIdx.x) * d, e, v);
  });
  ring_drain(bars, ring, r_hi - r_lo);
}

// The CTAs' sums added up in order: blockIdx.y = 0, 1: the weights' gradients, from 2 on: the gates' that have rows of several CTAs, found
// by the gate or, where gates are more than CTAs, by the border between two CTAs.  32 columns x 32 lanes of CTAs, a thread takes VEC columns.
template <int VEC>
__global__ void __launch_bounds__(1024 / VEC)
block_norm_grad_sums_kernel(const GradP p) {
  grid_begin();
  constexpr int CT = 32 / VEC;                              // threads side by side
  __shared__ double add[32][33];
  const int lane = threadIdx.x / CT, c0 = threadIdx.x % CT * VEC;
  const int64_t col = (int64_t)blockIdx.x * 32 + c0;
  __shared__ int64_t own[4];                                // the gate and the CTAs with its rows (64-bit divisions: by one thread)
  int64_t b0 = 0, b1 = p.ctas, second = p.ctas;
  float* out;
  const float* part;
  const int y = blockIdx.y;
  if (y == 0) { out = p.dw_pre; part = p.part + (int64_t)part_pre(p) * p.ctas * p.d; }
  else if (y == 1) { out = p.dw_post; part = p.part + (int64_t)part_post(p) * p.ctas * p.d; }
  else {
    if (threadIdx.x == 0) {
      int64_t gate = y - 2, first = p.ctas;
      bool none = false;
      if (p.gates_used > p.ctas) {
        const int64_t row = rows_lo(y - 1, p.rows, p.ctas);
        gate = row / p.per_gate;
        none = row == gate * p.per_gate || rows_owner(gate * p.per_gate, p.rows, p.ctas) != y - 2;
      }
      const int64_t g0 = gate * p.per_gate, g1 = g0 + p.per_gate < p.rows ? g0 + p.per_gate : p.rows;
      const int64_t lo = rows_owner(g0, p.rows, p.ctas), hi = rows_owner(g1 - 1, p.rows, p.ctas) + 1;
      // a gate that is not its first CTA's first lies in that CTA's second sum; it is the others' first
      if (rows_lo(lo, p.rows, p.ctas) / p.per_gate != gate) first = lo;
      own[0] = gate; own[1] = lo; own[2] = none ? lo + 1 : hi; own[3] = first;
    }
    __syncthreads();
    b0 = own[1]; b1 = own[2]; second = own[3];
    if (b1 == b0 + 1) return;                               // the CTA has written it
    out = p.dgate + own[0] * p.d;
    part = p.part + (int64_t)part_gate(p) * p.ctas * p.d;
  }
  if (!out) return;
  double t[VEC] = {};
  if (col < p.d) {
    const float* at = part + col;
#pragma unroll 5
    for (int64_t b = b0 + lane; b < b1; b += 32) {
      const float* v = at + (b == second ? p.ctas + b : b) * p.d;
      if (VEC == 4) {
        const float4 f = *reinterpret_cast<const float4*>(v);
        t[0] += f.x; t[1 % VEC] += f.y; t[2 % VEC] += f.z; t[3 % VEC] += f.w;
      } else t[0] += *v;
    }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) add[lane][c0 + i] = t[i];
  __syncthreads();
  // a warp adds a column at a time: the lanes' sums in a fixed tree
  for (int c = threadIdx.x >> 5; c < 32; c += 32 / VEC) {
    double u = add[threadIdx.x & 31][c];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    const int64_t mine = (int64_t)blockIdx.x * 32 + c;
    if ((threadIdx.x & 31) == 0 && mine < p.d) out[mine] = (float)u;
  }
}

// Ring and CTAs an SM for rows of d elements in arrays of these element sizes (0: not read), `kept` bytes of shared memory beside them an
// element, rows in use besides those on their way `held`.  The variants by the threads of a CTA and the registers that leaves each: 512 with
// one chunk of eight elements up to 4,096 (128 registers), 352 with two or three up to 8,448 (168), and where `wide` 512 with up to four.  False:
// too long.
constexpr size_t RING_SMEM = 224 * 1024 + 256;
struct Plan { Ring ring; int ctas, chunks, threads; size_t smem; };
bool plan_ring(int64_t d, bool al, size_t e0, size_t e1, size_t e2, size_t e3, size_t kept, int held, bool wide, Plan& pl) {
  Ring& r = pl.ring;
  const size_t es[4] = {e0, e1, e2, e3};
  if (!wide && d > 8448) return false;
  pl.chunks = wide ? (int)((d + 4095) / 4096) : (d <= 4096 ? 1 : (d <= 5632 ? 2 : 3));
  pl.threads = (int)(((d + 7) / 8 + pl.chunks - 1) / pl.chunks + 31) / 32 * 32;
  size_t stage = 0;
  r.arrays = 0;
  for (int k = 0; k < 4; ++k) {
    r.off[k] = (uint32_t)stage;
    r.bytes[k] = (uint32_t)(es[k] * (size_t)d);
    r.arrays += es[k] != 0;
    stage += es[k] ? (r.bytes[k] + 15) / 16 * 16 + (al ? 0 : 16) : 0;
  }
  r.stage_bytes = (int)stage;
  // as many CTAs as the registers hold, 512 threads or one, with two rows on their way
  const int most = wide ? 16 : 8;                           // (of the gradient's every CTA leaves sums behind)
  for (pl.ctas = pl.threads > 256 ? 1 : (512 / pl.threads < most ? 512 / pl.threads : most); pl.ctas >= 1; --pl.ctas) {
    const size_t room = pl.ctas == 1 ? RING_SMEM : RING_SMEM / (size_t)pl.ctas - 2048, keep = kept * (size_t)((d + 7) / 8 * 8);
    if (room < keep) continue;
    int n = (int)((room - keep) / stage);
    if (n > MAX_STAGES) n = MAX_STAGES;
    if (n >= held + 2 || (n > held && pl.ctas == 1)) {
      r.stages = n;
      pl.smem = (size_t)n * stage + keep;
      return true;
    }
  }
  return false;
}
// a ring kernel of `ctas` CTAs
template <typename K, typename P>
armor_status run_ring(armor_ctx* c, K kernel, PerDeviceOnce& attr, int64_t ctas, const Plan& pl, const P& p, cudaStream_t s) {
  if (ensure_dynamic_smem(attr, c->device, kernel, RING_SMEM) != ARMOR_OK) return ARMOR_ERR_CUDA;
  launch_dependent(kernel, dim3((unsigned)ctas), dim3((unsigned)pl.threads), pl.smem, s, p, pl.ring, c->status);
  return ARMOR_OK;
}
template <typename TS, typename TB, int CHUNKS, int THREADS, bool AL>
armor_status run_norm_ring(armor_ctx* c, int64_t ctas, const Plan& pl, const NormP& p, cudaStream_t s) {
  static PerDeviceOnce with, without;
  return p.y ? run_ring(c, block_norm_ring_kernel<TS, TB, CHUNKS, THREADS, true, AL>, with, ctas, pl, p, s)
             : run_ring(c, block_norm_ring_kernel<TS, TB, CHUNKS, THREADS, false, AL>, without, ctas, pl, p, s);
}
template <typename TS, typename TB, int CHUNKS, int THREADS, bool AL>
armor_status run_grad_ring(armor_ctx* c, int64_t ctas, const Plan& pl, const GradP& p, cudaStream_t s) {
  static PerDeviceOnce with, without;
  return p.y ? run_ring(c, block_norm_grad_ring_kernel<TS, TB, CHUNKS, THREADS, true, AL>, with, ctas, pl, p, s)
             : run_ring(c, block_norm_grad_ring_kernel<TS, TB, CHUNKS, THREADS, false, AL>, without, ctas, pl, p, s);
}

// Rows that the ring's aligned variant takes: no unit of theirs reaches behind their end.  Others on 16-byte boundaries (1,001 columns of
// rows 1,008 apart) go to the variant for rows that start anywhere.
template <typename TS, typename TB>
bool whole_units(int64_t d) { return d % ShareOf<TS, TB, 1, true>::U == 0; }

template <typename TS, typename TB, bool AL>
armor_status launch_norm_ring(armor_ctx* c, int64_t ctas, const Plan& pl, const NormP& p, cudaStream_t s) {
  switch (pl.chunks) {
    case 1: return run_norm_ring<TS, TB, 1, 512, AL>(c, ctas, pl, p, s);
    case 2: return run_norm_ring<TS, TB, 2, 512, AL>(c, ctas, pl, p, s);
    case 3: return run_norm_ring<TS, TB, 3, 512, AL>(c, ctas, pl, p, s);
    default: return run_norm_ring<TS, TB, 4, 512, AL>(c, ctas, pl, p, s);
  }
}
template <typename TS, typename TB, bool AL>
armor_status launch_grad_ring(armor_ctx* c, int64_t ctas, const Plan& pl, const GradP& p, cudaStream_t s) {
  if (pl.chunks == 1) return run_grad_ring<TS, TB, 1, 512, AL>(c, ctas, pl, p, s);
  return pl.chunks == 2 ? run_grad_ring<TS, TB, 2, 352, AL>(c, ctas, pl, p, s) : run_grad_ring<TS, TB, 3, 352, AL>(c, ctas, pl, p, s);
}

template <typename TS, typename TB, bool ALIGNED>
armor_status launch_norm(armor_ctx* c, const NormP& p, int64_t rows, cudaStream_t s) {
  const int64_t units = (p.d + 7) / 8;
  auto threads = [&](int chunks) { return dim3((unsigned)(((units + chunks - 1) / chunks + 31) / 32 * 32)); };
  const bool al = ALIGNED && whole_units<TS, TB>(p.d);
  Plan pl;
  // The ring, or a CTA a row with the row in registers where there are few rows: 400 x 9,216 bf16 10.0 and 8.1 us, 2,000 x 14,336 49 and 60; rows
  // that start anywhere, 2,000 x 9,001 62 and 107, 3,068 x 10,332 with an fp32 stream 110 and 242.
  if (rows > (ALIGNED && p.d > 8192 ? 4 : 2) * c->n_sm && plan_ring(p.d, al, sizeof(TS), p.y ? sizeof(TB) : 0, 0, 0, 0, 1, true, pl)) {
    const int64_t ctas = (int64_t)pl.ctas * c->n_sm < rows ? (int64_t)pl.ctas * c->n_sm : rows;
    if constexpr (ALIGNED) if (al) return launch_norm_ring<TS, TB, true>(c, ctas, pl, p, s);
    return launch_norm_ring<TS, TB, false>(c, ctas, pl, p, s);
  }
  const dim3 grid((unsigned)rows);
  if (units <= 128 || (rows <= 148 && units <= 1024)) launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 1>, grid, threads(1), 0, s, p);
  else if (units <= 512) launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 2>, grid, threads(2), 0, s, p);
  else launch_dependent(block_norm_kernel<TS, TB, ALIGNED, 4>, grid, threads(4), 0, s, p);
  return ARMOR_OK;
}
template <typename TS, typename TB, bool ALIGNED>
armor_status launch_grad(armor_ctx* c, GradP p, cudaStream_t s) {
  const int64_t units = (p.d + 7) / 8;
  const int n_sums = (p.dw_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.dgate ? 1 : 0);
  auto threads = [&](int chunks) { return dim3((unsigned)(((units + chunks - 1) / chunks + 31) / 32 * 32)); };
  const bool al = ALIGNED && whole_units<TS, TB>(p.d);
  Plan pl;
  const size_t kept = (p.dw_post ? 4 : 0) + (p.h && p.dh && p.dn ? 0 : sizeof(TS) + (sizeof(TB) != sizeof(TS) ? sizeof(TB) : 0));
  const bool use_ring = plan_ring(p.d, al, p.h ? sizeof(TS) : 0, p.y ? sizeof(TB) : 0, p.dh ? sizeof(TS) : 0, p.dn ? sizeof(TB) : 0, kept, p.d <= 4096 ? 0 : 1, false, pl);
  // CTAs as many as an SM runs, fewer where the workspace has no room for their sums
  const int64_t parts = (p.dw_pre ? 1 : 0) + (p.dw_post ? 1 : 0) + (p.dgate ? 2 : 0);
  int64_t n = use_ring ? (int64_t)pl.ctas * c->n_sm : 2 * c->n_sm;
  if (n > p.rows) n = p.rows;
  if (parts && n > ws_scratch_bytes(c) / (parts * p.d * 4)) n = ws_scratch_bytes(c) / (parts * p.d * 4);
  if (n < 1) return ARMOR_ERR_WORKSPACE;
  p.ctas = (int)n;
  if (use_ring) {
    armor_status st;
    if constexpr (ALIGNED) st = al ? launch_grad_ring<TS, TB, true>(c, n, pl, p, s) : launch_grad_ring<TS, TB, false>(c, n, pl, p, s);
    else st = launch_grad_ring<TS, TB, false>(c, n, pl, p, s);
    if (st != ARMOR_OK) return st;
  } else if (units <= 1024) {
    static PerDeviceOnce attr;
    if (ensure_dynamic_smem(attr, c->device, block_norm_grad_kernel<TS, TB, ALIGNED, 1>, 98304) != ARMOR_OK) return ARMOR_ERR_CUDA;
    launch_dependent(block_norm_grad_kernel<TS, TB, ALIGNED, 1>, dim3((unsigned)p.ctas), threads(1), (size_t)n_sums * 32 * threads(1).x, s, p);
  } else {
    static PerDeviceOnce attr;
    if (ensure_dynamic_smem(attr, c->device, block_norm_grad_kernel<TS, TB, ALIGNED, 2>, 196608) != ARMOR_OK) return ARMOR_ERR_CUDA;
    launch_dependent(block_norm_grad_kernel<TS, TB, ALIGNED, 2>, dim3((unsigned)p.ctas), threads(2), (size_t)n_sums * 64 * threads(2).x, s, p);
  }
  c->launches++;
  if (n_sums) {
    const int64_t sets = 2 + (p.dgate ? (p.gates_used > p.ctas ? p.ctas - 1 : p.gates_used) : 0);
    const dim3 grid((unsigned)((p.d + 31) / 32), (unsigned)sets);
    if (p.d % 4 == 0) launch_dependent(block_norm_grad_sums_kernel<4>, grid, dim3(256), 0, s, p);
    else launch_dependent(block_norm_grad_sums_kernel<1>, grid, dim3(1024), 0, s, p);
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
  st = by_types(g->stream_dtype, g->branch_dtype, [&](auto ts, auto tb) {
    using TS = decltype(ts);
    using TB = decltype(tb);
    return al ? launch_norm<TS, TB, true>(c, p, p.rows, s) : launch_norm<TS, TB, false>(c, p, p.rows, s);
  });
  c->launches++;
  if (st != ARMOR_OK) return st;
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
  if (!g->y && (g->post || g->dgate)) return ARMOR_ERR_INVALID_ARG;   // (with a gate alone y is read where it is given)
  GradP p{};
  p.rows = g->n_rows; p.d = g->d; p.ldh = g->ldh; p.ldy = g->ldy; p.lddh = g->lddh; p.lddn = g->lddn; p.lddx = g->lddx; p.lddy = g->lddy;
  p.ldg = g->ld_gate; p.per_gate = g->gate ? g->rows_per_gate : 1; p.gates_used = g->gate ? (p.rows - 1) / p.per_gate + 1 : 0;
  p.h = g->pre ? g->h : nullptr; p.y = g->post || g->gate ? g->y : nullptr; p.dh = g->dh; p.dn = g->dn; p.dx = g->dx; p.dy = g->dy;
  p.w_post = g->w_post; p.w_pre = g->w_pre; p.gate = g->gate;
  p.dw_post = g->dw_post; p.dw_pre = g->dw_pre; p.dgate = g->dgate;
  p.part = c->T; p.a = g->residual_scale; p.eps = g->eps; p.post = g->post != 0; p.pre = g->pre != 0;
  const int es = rows_dtype_bytes(g->stream_dtype), eb = rows_dtype_bytes(g->branch_dtype);
  const bool al = rows::aligned16(p.h, p.ldh, es) && rows::aligned16(p.y, p.ldy, eb) && rows::aligned16(p.dh, p.lddh, es) &&
                  rows::aligned16(p.dn, p.lddn, eb) && rows::aligned16(p.dx, p.lddx, es) && rows::aligned16(p.dy, p.lddy, eb) &&
                  rows::aligned16(p.gate, p.ldg, 4) && rows::aligned16(p.w_post, 0, 4) && rows::aligned16(p.w_pre, 0, 4) &&
                  rows::aligned16(p.dgate, 0, 4);
  KTimer kt(c, ARMOR_KC_FORWARD, (double)p.rows * (double)p.d *
            ((p.h ? es : 0) + (p.y ? eb : 0) + (p.dh ? es : 0) + (p.dn ? eb : 0) + (p.dx ? es : 0) + (p.dy ? eb : 0)), s);
  if (p.dgate && p.gates_used < g->n_gates)                 // gates without rows
    ARMOR_CUDA_OK(cudaMemsetAsync(p.dgate + p.gates_used * p.d, 0, (size_t)(g->n_gates - p.gates_used) * (size_t)p.d * 4, s));
  return by_types(g->stream_dtype, g->branch_dtype, [&](auto ts, auto tb) {
    using TS = decltype(ts);
    using TB = decltype(tb);
    return al ? launch_grad<TS, TB, true>(c, p, s) : launch_grad<TS, TB, false>(c, p, s);
  });
}
