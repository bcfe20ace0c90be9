// Attention of few rows a sequence (decoding) over a paged cache of int8 keys and values.
//
// A row is one query head of one new token; the rows of a key head's group share its keys.  With kq, vq the int8 rows and ks, vs their
// scales, for a row of position p:
//   t_j = (q . kq_j) ks_j scale log2 e + log2 vs_j     over j <= p (and j > p - window)
//   w_j = 2^(t_j - m),  O = sum w_j vq_j,  l = sum w_j / vs_j,  o = O / l
// m is a maximum of the t_j seen so far, less RAISED, so that w_j, the weight a value's bytes are taken with, is at most 2^15 and its rounding to
// fp16 is one of 2^-11 of what the value contributes (a weight below 2^-21 of the largest loses bits, 2^-32 of the largest at most).  The bytes themselves are exact in fp16, and so are q's 16-bit numbers after
// a multiplication by a power of two; products and sums are fp32.  l is summed from the unrounded weights.  No row: zeros.
//
// Bound by HBM: 2 (dim + 4) bytes a position and key head.  Each warp takes 16 positions at a time, twice, in the layout that mma.sync m16n8k16 wants of its
// M side, where a product over the dimensions may take them in any order: positions are the M side of the scores, S^T = K Q^T, dimensions the M
// side of O^T = V^T P^T, rows of q the N side of both, eight at a time, so that for up to eight rows nothing is computed twice
// and O takes dim / 4 registers.  (tcgen05 would multiply 128 rows for these eight.)  A byte becomes fp16 by a permutation, 1024 + (byte + 128),
// and a subtraction.  A warp's rows come to shared memory a stage of 32
// positions ahead by tensor copies (TMA) that one lane asks for, 16 rows each, or 32 where pages hold a multiple of 32; pages of other sizes take
// cp.async, each lane the sixteen bytes that it multiplies.  (Always so, the asking took 1,000 to 1,300 of a step's 3,900 cycles, 64 streams 152 us
// for 117.)  No registers wait, and no warp waits for another before the end of a CTA's share.
//
// All positions of all (sequence, key head, tile of rows) units, 192 at a time, and OVERHEAD more steps for each unit, stand in one line that is
// cut into equal shares, one a CTA, whatever the lengths.  A unit that is cut leaves its parts (m, l, O in fp32) in the workspace, and the CTA that comes
// last, by a counter, adds them up in the order of the parts: no CTA waits for another and the bits do not depend on the run.
#include "kv_cache.cuh"
#include "tc_common.cuh"

namespace {

using namespace rows;
using namespace kv;

constexpr int WARPS = 6, THREADS = 32 * WARPS, STEP = 32 * WARPS;      // positions a step of a CTA
constexpr int STAGES = 2;                   // of 32 positions a warp
constexpr int OVERHEAD = 2;                 // what a unit takes beside its steps, in steps: its sequence, q, the first copies, the warps' sums
constexpr int SEQS = 1024;                  // sequences a launch

template <int DIM, int NT>
struct Few {
  static constexpr int R = 8 * NT;          // rows of a tile
  static constexpr int KW = DIM / 16;       // words of a key that a lane holds; steps of the scores' product
  static constexpr int VB = DIM / 8;        // bytes of a value that a lane holds
  static constexpr int PART = R * DIM + 2 * R;     // floats of a part: O, m, l
  static constexpr int CTAS = 2;            // an SM
  static constexpr int K_BYTES = DIM / 64 * 2 * 512, V_BYTES = 4 * 32 * VB;        // of sixteen positions
  static constexpr int STAGE = 2 * (K_BYTES + V_BYTES);                             // of 32: keys, values
  static constexpr int SCALES = WARPS * STAGES * STAGE;                             // behind all stages: 256 bytes of scales for each
  static constexpr bool Q_SHARED = NT > 1;                                          // q in shared memory (registers hold eight rows of it)
  static constexpr int SUMS = WARPS * R * (DIM + 4) * 4;                            // the warps' O, in the place of the stages
  static constexpr int Q_AT = SCALES + WARPS * STAGES * 256, SMEM = Q_AT + (Q_SHARED ? NT * KW * 32 * 8 : 0) + 1024;
  static_assert(SUMS <= SCALES, "");
};
// bytes that a lane copies for itself, complete with wait_copies
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void end_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory"); }
__device__ __forceinline__ float minus_inf() { return -__int_as_float(0x7f800000); }

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// bytes of x (biased by 128) that `sel` picks, as fp16: 1024 + byte, exactly, less 1152
__device__ __forceinline__ uint32_t bytes_half(uint32_t x, uint32_t sel) {
  const uint32_t w = __byte_perm(x, 0x64646464u, sel);
  const uint32_t off = 0x64806480u;         // 1152
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(off));
  return r;
}

struct FewP {
  KvAttend a;
  int64_t limit;                            // rows of a sequence at most: those with more are left out
  float* parts;                             // two of every CTA
  int* counters;                            // one of every CTA, zero between calls
  int wide;                                 // 32 positions that begin at a multiple of 32 share a page: one copy for them
  int32_t* status;
};

struct Unit { int64_t per, steps; int tiles; };       // what all units take, steps of one; tiles of rows
template <int R>
__device__ __forceinline__ Unit units_of(const FewP& p, const Seq& s) {
  Unit u{0, 0, 0};
  const int64_t rows = (int64_t)s.n * p.a.group;
  if (rows < 1 || rows > p.limit) return u;
  u.tiles = (int)((rows + R - 1) / R);
  const int64_t lo = p.a.window ? max((int64_t)0, (int64_t)s.length - s.n + 1 - p.a.window) : 0;
  u.steps = max((int64_t)1, divide((int64_t)s.length + STEP - 1, STEP) - divide(lo, STEP));
  u.per = (u.steps + OVERHEAD) * u.tiles * p.a.c.heads;
  return u;
}

// sixteen rows of a page's head, or 32, swizzled: the bank of a row's sixteen bytes moves with the row
__device__ __forceinline__ void copy_rows(uint32_t dst, const CUtensorMap* map, uint32_t slot, int head, uint32_t page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(0), "r"(slot), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
// where sixteen bytes (chunk) of a row lie then
template <int DIM>
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk) {
  return DIM == 128 ? row * 128 + ((chunk ^ (row & 7)) << 4) : row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
}

// TOGETHER: sixteen positions that begin at a multiple of sixteen share a page: one lane of a warp asks for all of their keys, or values, at once.
// (Every lane asking for its own sixteen bytes took 1,000 to 1,300 cycles of a step's 3,900.)  Else every lane copies what it reads itself.
template <typename T, int DIM, int NT, bool TOGETHER>
__global__ void __launch_bounds__(THREADS, Few<DIM, NT>::CTAS)
kv_attend_few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const FewP p) {
  grid_begin();
  using F = Few<DIM, NT>;
  constexpr int R = F::R;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bars[WARPS * STAGES];
  __shared__ int abort_flag;
  float (*const sO)[R][DIM + 4] = reinterpret_cast<float (*)[R][DIM + 4]>(smem);
  __shared__ float sM[WARPS][R], sL[WARPS][R];
  __shared__ int64_t scan[WARPS];
  __shared__ int64_t at_base;
  __shared__ int at_seq, last_one;
  __shared__ Seq at_s;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane >> 2, part = lane & 3;
  const Cache& c = p.a.c;
  const Batch& b = p.a.b;
  const uint32_t my_bars = tc::smem_u32(&bars[warp * STAGES]);
  if (threadIdx.x == 0) {
    abort_flag = 0;
    if (TOGETHER) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
  }
  if (TOGETHER && lane == 0) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) tc::mbar_init(my_bars + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  uint32_t turn = 0;                                      // steps of this warp so far
  bool ok = true;                                         // all copies came

  // ---- the line of all steps, this CTA's share of it and the sequence that it begins in
  int64_t total, begin, end;
  int n_ctas;
  {
    const int per = (b.n + THREADS - 1) / THREADS, s0 = min(b.n, (int)threadIdx.x * per), s1 = min(b.n, s0 + per);
    int64_t mine = 0;
    for (int i = s0; i < s1; ++i) {
      bool bad;
      const Seq s = sequence(b, i, bad);
      if (bad && blockIdx.x == 0) report(p.status);
      mine += units_of<R>(p, s).per;
    }
    int64_t up_to = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, up_to, o);
      if (lane >= o) up_to += v;
    }
    if (lane == 31) scan[warp] = up_to;
    __syncthreads();
    total = 0;
    int64_t before = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) before += scan[w];
      total += scan[w];
    }
    n_ctas = (int)min((int64_t)gridDim.x, total);
    if ((int)blockIdx.x >= n_ctas) return;
    begin = divide((int64_t)blockIdx.x * total, n_ctas);
    end = divide((int64_t)(blockIdx.x + 1) * total, n_ctas);
    int64_t base = before + up_to - mine;
    if (base <= begin && begin < base + mine)
      for (int i = s0; i < s1; ++i) {
        bool bad;
        const Seq s = sequence(b, i, bad);
        const int64_t w = units_of<R>(p, s).per;
        if (begin < base + w) { at_seq = i; at_base = base; at_s = s; break; }
        base += w;
      }
    __syncthreads();
  }
  int seq = at_seq;
  int64_t base = at_base;
  Seq s = at_s;

  while (begin < end) {
    const Unit un = units_of<R>(p, s);
    if (begin >= base + un.per) {
      bool bad;
      base += un.per;
      s = sequence(b, ++seq, bad);
      continue;
    }
    const int64_t unit = divide(begin - base, un.steps + OVERHEAD), u0 = base + unit * (un.steps + OVERHEAD);
    const int first = (int)(begin - u0), count = (int)(min(end, u0 + un.steps) - begin);
    begin = u0 + un.steps + OVERHEAD;                     // of the unit that comes
    if (count < 1) continue;                              // (the share begins behind its last step)
    const int head = (int)divide(unit, un.tiles), tile = (int)(unit - (int64_t)head * un.tiles);
    const int rows = s.n * p.a.group - tile * R;        // of this tile, if fewer than R
    const int64_t lo_all = p.a.window ? max((int64_t)0, (int64_t)s.length - s.n + 1 - p.a.window) : 0;
    const int step0 = (int)divide(lo_all, STEP) + first;

    // ---- q: rows lane / 4 of each eight, four dimensions for each step of the product, in the order that keys come in
    uint32_t q[F::Q_SHARED ? 1 : NT][F::Q_SHARED ? 1 : F::KW][2];
    uint2* const q_shared = reinterpret_cast<uint2*>(smem + F::Q_AT) + lane;
    float factor;
    {
      const T* const t = nullptr;
      float top = 0.f;
      uint32_t raw[NT][F::KW][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = tile * R + n * 8 + quad;
        const bool there = n * 8 + quad < rows;
        const int i = there ? r / p.a.group : 0, g = there ? r - i * p.a.group : 0;
        const T* const row = static_cast<const T*>(p.a.q) + (int64_t)(s.first + i) * p.a.q_row + (int64_t)(head * p.a.group + g) * p.a.q_head;
#pragma unroll
        for (int h = 0; h < DIM / 64; ++h) {
          const int d = TOGETHER ? part * (DIM / 4) + h * 16 : h * 64 + part * 16;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const Raw8<T> x = !there ? raw_zero<T>() : (p.a.aligned ? raw_load(row + d + 8 * e) : row_load<false>(row, d + 8 * e, DIM));
            raw[n][h * 4 + 2 * e][0] = x.w.x; raw[n][h * 4 + 2 * e][1] = x.w.y;
            raw[n][h * 4 + 2 * e + 1][0] = x.w.z; raw[n][h * 4 + 2 * e + 1][1] = x.w.w;
          }
        }
      }
      int shift = 0;
      if (sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value) {
        // bf16 in fp16: by the power of two that brings the largest finite |q| of the tile to [2^14, 2^15), so that what is lost is below 2^-39 of it
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < F::KW; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 v = unpack2(t, raw[n][k][e]);
              const float x = fabsf(v.x), y = fabsf(v.y);
              if (x < __int_as_float(0x7f800000)) top = fmaxf(top, x);
              if (y < __int_as_float(0x7f800000)) top = fmaxf(top, y);
            }
        top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
        shift = top > 0.f ? min(max(14 - ((int)(__float_as_uint(top) >> 23) - 127), -120), 120) : 0;
      }
      const float up = __int_as_float((127 + shift) << 23);
      factor = p.a.scale * __int_as_float((127 - shift) << 23);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < F::KW; ++k) {
          uint32_t x[2] = {raw[n][k][0], raw[n][k][1]};
          if (!std::is_same<T, __half>::value) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { const float2 v = unpack2(t, x[e]); x[e] = half2_bits(v.x * up, v.y * up); }
          }
          if constexpr (!F::Q_SHARED) { q[n][k][0] = x[0]; q[n][k][1] = x[1]; }
          else if (warp == 0) q_shared[(n * F::KW + k) * 32] = make_uint2(x[0], x[1]);
        }
      if (F::Q_SHARED) __syncthreads();
    }

    // ---- the positions that rows 2 part and 2 part + 1 of each eight see: [low, high)
    int low[NT][2], high[NT][2];
    int inner_lo = 0, inner_hi = 0x7fffffff;            // what all of the tile's rows see
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = n * 8 + 2 * part + e;
        low[n][e] = high[n][e] = 0;
        if (r < rows) {
          const int64_t at = (int64_t)s.length - s.n + (tile * R + r) / p.a.group;
          high[n][e] = (int)max((int64_t)0, at + 1);
          low[n][e] = p.a.window ? (int)max((int64_t)0, at + 1 - p.a.window) : 0;
          inner_lo = max(inner_lo, low[n][e]);
          inner_hi = min(inner_hi, high[n][e]);
        }
      }
    inner_lo = __reduce_max_sync(0xffffffffu, inner_lo);
    inner_hi = __reduce_min_sync(0xffffffffu, inner_hi);

    const int last = max(s.length - 1, 0);
    // ---- 32 positions of a step: a lane looks up the place of one of them, or of the first of its sixteen
    uint8_t* const mine = smem + warp * (STAGES * F::STAGE);
    float* const my_scales = reinterpret_cast<float*>(smem + F::SCALES + warp * (STAGES * 256));
    const uint32_t mine_at = tc::smem_u32(mine), scales_at = tc::smem_u32(my_scales) + lane * 4;
    uint32_t page = 0, slot = 0;
    auto look = [&](int i) {                                // of step i
      int j = (step0 + i) * STEP + warp * 32 + lane;
      j = TOGETHER ? (p.wide ? min(j & ~31, last & ~31) + (lane & 16) : min(j & ~15, last & ~15)) : min(j, last);
      const uint32_t x = quotient((uint32_t)j, c.mul, c.shift);
      slot = (uint32_t)j - x * c.page_size;
      page = x < (uint32_t)b.max_pages ? (uint32_t)b.pages[(int64_t)seq * b.ld + x] : 0xffffffffu;
    };
    unsigned refused = 0;                                   // a bit a position of the step fetched last: it has no page
    auto fetch = [&](uint32_t turn) {                       // what has been looked up, to the stage of that step
      const bool none = page >= c.n_pages;
      if (none) page = slot = 0;
      refused = __ballot_sync(0xffffffffu, none);
      const uint32_t st = turn % STAGES, to = mine_at + st * F::STAGE;
      if constexpr (TOGETHER) {
        const uint32_t page1 = __shfl_sync(0xffffffffu, page, 16), slot1 = __shfl_sync(0xffffffffu, slot, 16), bar = my_bars + 8 * st;
        if (lane == 0) {
          tc::mbar_expect_tx(bar, F::STAGE);
          copy_rows(to, &k_map, slot, head, page, bar);
          copy_rows(to + 2 * F::K_BYTES, &v_map, slot, head, page, bar);
          if (!p.wide) {
            copy_rows(to + F::K_BYTES, &k_map, slot1, head, page1, bar);
            copy_rows(to + 2 * F::K_BYTES + F::V_BYTES, &v_map, slot1, head, page1, bar);
          }
        }
      } else {
        const int64_t row = page * c.page + head * c.head + slot * c.slot;
        const uint32_t k_at = to + lane * 16, v_at = to + 2 * F::K_BYTES + lane * F::VB;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int8_t* const from = c.k + __shfl_sync(0xffffffffu, row, 16 * g + quad + 8 * e) + part * 16;
#pragma unroll
            for (int h = 0; h < DIM / 64; ++h) copy_async<16>(k_at + ((g * 2 + e) * (DIM / 64) + h) * 512, from + h * 64);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            copy_async<F::VB>(v_at + (g * 4 + e) * 32 * F::VB, c.v + __shfl_sync(0xffffffffu, row, 16 * g + 2 * part + (e & 1) + (e >> 1) * 8) + quad * F::VB);
        }
      }
      const int64_t scale = page * c.spage + head * c.shead + (slot + (TOGETHER ? lane & 15 : 0)) * c.sslot;
      copy_async<4>(scales_at + st * 256, c.ks + scale);
      copy_async<4>(scales_at + st * 256 + 128, c.vs + scale);
    };

    float O[NT][DIM / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int d = 0; d < DIM / 16; ++d) O[n][d][0] = O[n][d][1] = O[n][d][2] = O[n][d][3] = 0.f;
      m[n][0] = m[n][1] = minus_inf();
      l[n][0] = l[n][1] = 0.f;
    }

    look(0);
    if (TOGETHER && lane == 0) tc::fence_proxy_async();     // (sums of the unit before lay in the stages)
    if (ok) fetch(turn);
    if (count > 1) look(1);
    end_copies();
    for (int i = 0; i < count; ++i, ++turn) {
      wait_copies<0>();
      if (TOGETHER && ok) {
        const uint32_t bar = my_bars + 8 * (turn % STAGES), parity = (turn / STAGES) & 1;
        if (!tc::mbar_wait_warp(bar, parity, &abort_flag, p.status)) {
          // what comes out is worthless, as the status says; no more copies, and this one once more
          ok = false;
          const long long t0 = clock64();
          while (!tc::mbar_try(bar, parity) && clock64() - t0 < 20000000ll) {}
        }
      }
      __syncwarp();
      const unsigned bad = refused;                         // of this step
      if (i + 1 < count && ok) {
        fetch(turn + 1);
        if (i + 2 < count) look(i + 2);
        end_copies();
      }
      const int j0 = (step0 + i) * STEP + warp * 32;
      if (bad) {
        // (what no row sees may lie on pages that are gone)
        const int64_t at = (int64_t)s.length - s.n, hi = at + (tile * R + min(rows, R) - 1) / p.a.group + 1;
        const int64_t lo = p.a.window ? at + tile * R / p.a.group + 1 - p.a.window : 0;
        if (bad >> lane & 1u && j0 + lane >= lo && j0 + lane < hi) report(p.status);
      }
      const uint8_t* const stage = mine + (turn % STAGES) * F::STAGE;

      // ---- scores of twice sixteen positions
      float t[2][NT][4];
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int n = 0; n < NT; ++n) t[g][n][0] = t[g][n][1] = t[g][n][2] = t[g][n][3] = 0.f;
#pragma unroll
      for (int h = 0; h < DIM / 64; ++h) {
        uint4 x[2][2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) x[g][e] = *reinterpret_cast<const uint4*>(TOGETHER ? stage + g * F::K_BYTES + swizzled<DIM>(quad + 8 * e, part * (DIM / 64) + h)
                                                              : stage + ((g * 2 + e) * (DIM / 64) + h) * 512 + lane * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t b0[NT], b1[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (F::Q_SHARED) {
              const uint2 v = q_shared[(n * F::KW + 4 * h + k) * 32];
              b0[n] = v.x; b1[n] = v.y;
            } else { b0[n] = q[n][4 * h + k][0]; b1[n] = q[n][4 * h + k][1]; }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint32_t x0 = k == 0 ? x[g][0].x : k == 1 ? x[g][0].y : k == 2 ? x[g][0].z : x[g][0].w;
            const uint32_t x1 = k == 0 ? x[g][1].x : k == 1 ? x[g][1].y : k == 2 ? x[g][1].z : x[g][1].w;
            const uint32_t a0 = x0 ^ 0x80808080u, a1 = x1 ^ 0x80808080u;
            const uint32_t a[4] = {bytes_half(a0, 0x4140), bytes_half(a1, 0x4140), bytes_half(a0, 0x4342), bytes_half(a1, 0x4342)};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma(t[g][n], a, b0[n], b1[n]);
          }
        }
      }
      float kr[2][2];
      {
        const float* const scales = my_scales + (turn % STAGES) * 64;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float vs = measure(scales[32 + 16 * g + quad + 8 * e]);
            const float ka = scales[16 * g + quad + 8 * e] * factor, kb = __log2f(vs);
            kr[g][e] = __fdividef(LOWERED, vs);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < 2; ++x) t[g][n][2 * e + x] = fmaf(t[g][n][2 * e + x], ka, kb);
          }
      }
      const bool some_hidden = bad || j0 < inner_lo || j0 + 32 > inner_hi;
      if (some_hidden) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = j0 + 16 * g + quad + 8 * (e >> 1);
              if (bad >> (16 * g + quad + 8 * (e >> 1)) & 1u || j < low[n][e & 1] || j >= high[n][e & 1]) t[g][n][e] = minus_inf();
            }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (!(kr[g][e] == kr[g][e])) kr[g][e] = 1.f;    // (no number: the weight is none either, and 0 where it is not seen)
      }
      // m to their maximum, where that passes it by far
      bool over = false;
      float top[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[n][e] = fmaxf(fmaxf(t[0][n][e], t[0][n][e + 2]), fmaxf(t[1][n][e], t[1][n][e + 2]));
          over |= top[n][e] > m[n][e] + (LAZY + RAISED);
        }
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) top[n][e] = fmaxf(top[n][e], __shfl_xor_sync(0xffffffffu, top[n][e], o));
            const float to = fmaxf(m[n][e], top[n][e] - RAISED);
            f[e] = m[n][e] == to ? 1.f : exp2_fast(m[n][e] - to);       // (nothing yet: 2^-inf)
            m[n][e] = to;
            l[n][e] *= f[e];
          }
#pragma unroll
          for (int d = 0; d < DIM / 16; ++d) { O[n][d][0] *= f[0]; O[n][d][1] *= f[1]; O[n][d][2] *= f[0]; O[n][d][3] *= f[1]; }
        }
      }
      uint32_t P[2][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float m0 = m[n][0] == minus_inf() ? 0.f : m[n][0], m1 = m[n][1] == minus_inf() ? 0.f : m[n][1];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float w0 = exp2_fast(t[g][n][2 * e] - m0), w1 = exp2_fast(t[g][n][2 * e + 1] - m1);
            l[n][0] = fmaf(w0, kr[g][e], l[n][0]);
            l[n][1] = fmaf(w1, kr[g][e], l[n][1]);
            P[g][n][e] = transpose8(half2_bits(w0, w1));
          }
      }

      // ---- O^T += V^T P^T: a lane's dimensions quad DIM / 8 + 2 d, + 1
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t V[4][DIM / 32];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t r = 2 * part + (e & 1) + (e >> 1) * 8;
          const uint8_t* const from = stage + 2 * F::K_BYTES +
                                      (TOGETHER ? g * F::V_BYTES + swizzled<DIM>(r, quad * F::VB / 16) + (quad * F::VB & 15) : (g * 4 + e) * 32 * F::VB + lane * F::VB);
          if constexpr (DIM == 128) {
            const uint4 v = *reinterpret_cast<const uint4*>(from);
            V[e][0] = v.x; V[e][1] = v.y; V[e][2] = v.z; V[e][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(from);
            V[e][0] = v.x; V[e][1] = v.y;
          }
        }
#pragma unroll
        for (int h = 0; h < DIM / 32; ++h) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = V[e][h] ^ 0x80808080u;
          const uint32_t a01 = __byte_perm(v[0], v[1], 0x5140), b01 = __byte_perm(v[0], v[1], 0x7362);
          const uint32_t a23 = __byte_perm(v[2], v[3], 0x5140), b23 = __byte_perm(v[2], v[3], 0x7362);
          const uint32_t lo[4] = {bytes_half(a01, 0x4140), bytes_half(a01, 0x4342), bytes_half(a23, 0x4140), bytes_half(a23, 0x4342)};
          const uint32_t hi[4] = {bytes_half(b01, 0x4140), bytes_half(b01, 0x4342), bytes_half(b23, 0x4140), bytes_half(b23, 0x4342)};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma(O[n][2 * h], lo, P[g][n][0], P[g][n][1]);
            mma(O[n][2 * h + 1], hi, P[g][n][0], P[g][n][1]);
          }
        }
      }
    }

    // ---- the warps' sums to one
    __syncthreads();                                      // (the stages have been read)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], o);
        const int r = n * 8 + 2 * part + e;
        if (quad == 0) { sM[warp][r] = m[n][e]; sL[warp][r] = l[n][e]; }
#pragma unroll
        for (int d = 0; d < DIM / 16; ++d)
          *reinterpret_cast<float2*>(&sO[warp][r][quad * F::VB + 2 * d]) = make_float2(O[n][d][e], O[n][d][e + 2]);
      }
    }
    __syncthreads();
    const bool cut = count < un.steps;
    float* const parts = p.parts;
    const int64_t part_at = 2 * (int64_t)blockIdx.x + (first == 0 ? 1 : 0);
    auto put = [&](int r, int d, float4 o, float l) {     // four dimensions of a row of the output
      const float inv = l == 0.f ? 0.f : LOWERED / l;     // (a row that sees nothing: zeros)
      const int rr = tile * R + r, i = rr / p.a.group, g = rr - i * p.a.group;
      T* const to = static_cast<T*>(p.a.o) + (int64_t)(s.first + i) * p.a.o_row + (int64_t)(head * p.a.group + g) * p.a.o_head + d;
      if (p.a.aligned) {
        const T* const t = nullptr;
        *reinterpret_cast<uint2*>(to) = make_uint2(pack2(t, o.x * inv, o.y * inv), pack2(t, o.z * inv, o.w * inv));
      } else {
        to[0] = from_f<T>(o.x * inv); to[1] = from_f<T>(o.y * inv); to[2] = from_f<T>(o.z * inv); to[3] = from_f<T>(o.w * inv);
      }
    };
    auto weight = [](float m, float top) { return m == -__int_as_float(0x7f800000) ? 0.f : exp2_fast(m - top); };
    for (int u = threadIdx.x; u < R * (DIM / 4); u += THREADS) {
      const int r = u / (DIM / 4), d = u % (DIM / 4) * 4;
      if (r >= rows) break;
      float top = sM[0][r];
#pragma unroll
      for (int w2 = 1; w2 < WARPS; ++w2) top = fmaxf(top, sM[w2][r]);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll
      for (int w2 = 0; w2 < WARPS; ++w2) {
        const float f = weight(sM[w2][r], top);
        const float4 v = *reinterpret_cast<const float4*>(&sO[w2][r][d]);
        sum = fmaf(f, sL[w2][r], sum);
        o.x = fmaf(f, v.x, o.x); o.y = fmaf(f, v.y, o.y); o.z = fmaf(f, v.z, o.z); o.w = fmaf(f, v.w, o.w);
      }
      if (!cut) { put(r, d, o, sum); continue; }
      float* const to = parts + part_at * F::PART;
      *reinterpret_cast<float4*>(to + r * DIM + d) = o;
      if (d == 0) { to[R * DIM + r] = top; to[R * DIM + R + r] = sum; }
    }
    if (cut) {
      // ---- the parts of the unit: those of the CTAs from the one that holds its first step to the one that holds its last
      __threadfence();
      __syncthreads();
      const int64_t c0 = divide((u0 + 1) * n_ctas - 1, total), c1 = divide((u0 + un.steps) * n_ctas - 1, total);
      if (threadIdx.x == 0) {
        const int had = atomicAdd(&p.counters[c0], 1);
        last_one = had == (int)(c1 - c0);
        if (last_one) p.counters[c0] = 0;
      }
      __syncthreads();
      if (last_one) {
        // Each warp adds every WARPS-th part, eight of its rows or more at a time; then the warps' sums as above
        __threadfence();
        const int n_parts = (int)(c1 - c0) + 1;
        auto at = [&](int k) { return parts + (2 * (c0 + k) + (k == 0)) * F::PART; };
        float top[R / 8], sum[R / 8];                     // of rows lane % 8 + 8 k, over the lane's parts
#pragma unroll
        for (int k = 0; k < R / 8; ++k) {
          top[k] = minus_inf();
          for (int x = threadIdx.x >> 3; x < n_parts; x += THREADS / 8) top[k] = fmaxf(top[k], __ldcg(at(x) + R * DIM + 8 * k + (lane & 7)));
          top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 8));
          top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 16));
          if (lane < 8) sM[warp][8 * k + lane] = top[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < R / 8; ++k) {
#pragma unroll
          for (int w2 = 0; w2 < WARPS; ++w2) top[k] = fmaxf(top[k], sM[w2][8 * k + (lane & 7)]);
          sum[k] = 0.f;
        }
        __syncthreads();
        float4 o[R * DIM / 128];                          // four numbers of every 128
#pragma unroll
        for (int u = 0; u < R * DIM / 128; ++u) o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int x = warp; x < n_parts; x += WARPS) {
          const float* const from = at(x);
          float4 v[R * DIM / 128];
#pragma unroll
          for (int u = 0; u < R * DIM / 128; ++u) v[u] = __ldcg(reinterpret_cast<const float4*>(from + u * 128) + lane);
          float f[R / 8];
#pragma unroll
          for (int k = 0; k < R / 8; ++k) {
            f[k] = weight(__ldcg(from + R * DIM + 8 * k + (lane & 7)), top[k]);
            sum[k] = fmaf(f[k], __ldcg(from + R * DIM + R + 8 * k + (lane & 7)), sum[k]);
          }
#pragma unroll
          for (int u = 0; u < R * DIM / 128; ++u) {
            const int r = u * (128 / DIM) + (DIM == 64 ? lane >> 4 : 0);
            const float g = __shfl_sync(0xffffffffu, f[u * (128 / DIM) / 8], r & 7);
            o[u].x = fmaf(g, v[u].x, o[u].x); o[u].y = fmaf(g, v[u].y, o[u].y); o[u].z = fmaf(g, v[u].z, o[u].z); o[u].w = fmaf(g, v[u].w, o[u].w);
          }
        }
#pragma unroll
        for (int u = 0; u < R * DIM / 128; ++u)
          *reinterpret_cast<float4*>(&sO[warp][u * (128 / DIM) + (DIM == 64 ? lane >> 4 : 0)][DIM == 64 ? (lane & 15) * 4 : lane * 4]) = o[u];
#pragma unroll
        for (int k = 0; k < R / 8; ++k)
          if (lane < 8) sL[warp][8 * k + lane] = sum[k];
        __syncthreads();
        for (int u = threadIdx.x; u < R * (DIM / 4); u += THREADS) {
          const int r = u / (DIM / 4), d = u % (DIM / 4) * 4;
          if (r >= rows) break;
          float4 s4 = make_float4(0.f, 0.f, 0.f, 0.f);
          float ls = 0.f;
#pragma unroll
          for (int w2 = 0; w2 < WARPS; ++w2) {
            const float4 v = *reinterpret_cast<const float4*>(&sO[w2][r][d]);
            ls += sL[w2][r];
            s4.x += v.x; s4.y += v.y; s4.z += v.z; s4.w += v.w;
          }
          put(r, d, s4, ls);
        }
      }
    }
    __syncthreads();                                      // (the stages' place is free)
  }
}

}  // namespace

namespace {

// [pages][heads][slots][DIM] of keys or values, so many slots at a time
template <int DIM>
bool make_map(CUtensorMap* map, const Cache& c, int8_t* base, cuuint32_t rows) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = tc::get_encode();
  if (!enc) return false;
  cuuint64_t dims[4] = {DIM, c.page_size, (cuuint64_t)c.heads, c.n_pages}, strides[3] = {(cuuint64_t)c.slot, (cuuint64_t)c.head, (cuuint64_t)c.page};
  cuuint32_t box[4] = {DIM, rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, base, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             DIM == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DIM, int NT, bool TOGETHER>
void launch_typed(armor_ctx* c, FewP p, cudaStream_t s) {
  using F = Few<DIM, NT>;
  static PerDeviceOnce once;
  if (ensure_dynamic_smem(once, c->device, kv_attend_few_kernel<T, DIM, NT, TOGETHER>, F::SMEM) != ARMOR_OK) { c->host_err = ARMOR_ERR_CUDA; return; }
  CUtensorMap k_map{}, v_map{};
  p.wide = p.a.c.page_size % 32 == 0;
  if (TOGETHER && (!make_map<DIM>(&k_map, p.a.c, p.a.c.k, p.wide ? 32 : 16) || !make_map<DIM>(&v_map, p.a.c, p.a.c.v, p.wide ? 32 : 16))) { c->host_err = ARMOR_ERR_CUDA; return; }
  // two parts a CTA have to find room in the workspace (a single CTA leaves none)
  int64_t n = (int64_t)c->n_sm * F::CTAS;
  const int64_t room = ws_scratch_bytes(c) / (2 * F::PART * (int64_t)sizeof(float));
  if (n > room) n = room;
  if (n > ARMOR_KV_COUNTERS) n = ARMOR_KV_COUNTERS;
  if (n < 1) n = 1;
  const Batch all = p.a.b;
  for (int b0 = 0; b0 < all.n; b0 += SEQS) {
    p.a.b.n = all.n - b0 < SEQS ? all.n - b0 : SEQS;
    p.a.b.lengths = all.lengths + b0;
    p.a.b.starts = all.starts + b0;
    p.a.b.pages = all.pages + b0 * all.ld;
    launch_dependent(kv_attend_few_kernel<T, DIM, NT, TOGETHER>, dim3((unsigned)n), dim3(THREADS), F::SMEM, s, k_map, v_map, p);
    c->launches++;
  }
}
template <typename T, int DIM>
void launch_by_rows(armor_ctx* c, const FewP& p, int64_t rows, cudaStream_t s) {
  // (a copy of rows takes strides below 2^40)
  const bool together = p.a.c.page_size % 16 == 0 && (uint64_t)(p.a.c.page | p.a.c.head | p.a.c.slot) < (1ull << 40);
  if (rows <= 8) together ? launch_typed<T, DIM, 1, true>(c, p, s) : launch_typed<T, DIM, 1, false>(c, p, s);
  else together ? launch_typed<T, DIM, 2, true>(c, p, s) : launch_typed<T, DIM, 2, false>(c, p, s);
}

}  // namespace

armor_status launch_kv_attend_few(armor_ctx* c, const KvAttend& a, int64_t limit, cudaStream_t s) {
  FewP p;
  p.a = a;
  p.limit = limit;
  p.status = c->status;
  p.counters = c->kv_counters;
  p.parts = c->T;
  // rows a sequence: as expected, or on average; with a batch of which others have most rows, single tokens
  int64_t rows = (a.max_chunk ? a.max_chunk : (a.b.rows + a.b.n - 1) / a.b.n) * a.group;
  if (rows > limit) rows = a.group;
  KTimer kt(c, ARMOR_KC_FORWARD, 0.0, s);
  if (a.dtype == ARMOR_DTYPE_BF16) {
    if (a.dim == 64) launch_by_rows<__nv_bfloat16, 64>(c, p, rows, s);
    else launch_by_rows<__nv_bfloat16, 128>(c, p, rows, s);
  } else {
    if (a.dim == 64) launch_by_rows<__half, 64>(c, p, rows, s);
    else launch_by_rows<__half, 128>(c, p, rows, s);
  }
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}
