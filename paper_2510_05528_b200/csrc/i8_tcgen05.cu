// Products of int8 rows with a scale each on the tensor cores (tcgen05.mma kind::i8, int32 sums in tensor memory):
//   Y[t][m] = xs[t] ws[m] sum_k Xq[t][k] Wq[m][k] (+ b[m])
// with W dense, or the 2:4 core of a factorised layer given as its kept values (int8, two of every four along k) and their
// positions (tcgen05.mma.sp).  The sums are exact: |q| <= 128, so 131,071 products fit an int32.  On their way out fp32 rounds the sum, the
// product of the scales, and the multiplication of the two with the bias added; a further rounding where Y is bf16 or fp16.
//
// W is the A operand, lanes of an accumulator are its rows and columns are tokens, from one token to many.  One instruction
// multiplies 32 k (dense; 32 bytes of each operand) or 64 (sparse; 32 bytes of kept values, 64 of tokens).  A stage is 128 bytes of W's
// rows: 128 k, or 256.
//
// Positions for one sparse instruction: lane l holds the 64 bits of row l, a nibble for each group of four k in order (the lower
// kept position in bits 0-1, the higher in bits 2-3), in two columns of tensor memory; the selector field is 0.  pack_core_i8_kernel
// writes a stage's positions as two blocks of 128 lanes x 16 bytes, which two tcgen05.cp take to eight columns ahead of the stage's
// four instructions, in order with them.
//
// Every wait is bounded.
#include "rows_io.cuh"
#include "tc_common.cuh"

namespace {

using namespace tc;

constexpr int BM = 128;                             // rows of W a CTA
constexpr int A_BYTES = BM * 128;                   // a stage of W
constexpr int E_BYTES = 128 * 32;                   // positions of a sparse stage

struct I8P {
  void* Y; int64_t ldy; int out;                    // ARMOR_DTYPE_* of Y, or OUT_TWO_BF16
  int64_t second;                                   // elements from the first array of the two to the second
  int pairs;                                        // two neighbouring rows of W may be stored at once
  const float *xs, *ws, *bias;
  int64_t M, N;                                     // rows of W, tokens
  int m_tiles, n_tiles, k_tiles, tile_n;
  int per;                                          // few tokens: k tiles a CTA
  const void* x; int64_t ldx, K;                    // few tokens: the rows of x, where the kernel rounds them itself, and their length
  int x_aligned;
  int ahead;                                        // few tokens: W may be fetched before the wait for the kernel before
  int32_t* status;
};

// K-major rows of 128 bytes, 128-byte swizzle
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) { return smem_desc_sw128(addr, 16, 1024); }
// 128 rows of 16 bytes, groups of eight rows 128 bytes apart, no swizzle
__device__ __forceinline__ uint64_t desc_e(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(128 >> 4) << 16;
  d |= (uint64_t)(128 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  return d;
}
// signed int8 operands, both K-major, int32 sums
__device__ __forceinline__ uint32_t idesc_i8(int m, int n, bool sparse) {
  uint32_t d = sparse ? 1u << 2 : 0u;
  d |= 2u << 4;                   // D format: S32
  d |= 1u << 7;                   // A format: S8
  d |= 1u << 10;                  // B format: S8
  d |= (uint32_t)(n >> 3) << 17;
  d |= (uint32_t)(m >> 4) << 24;
  return d;
}
template <int CTAS, bool SP>
__device__ __forceinline__ void umma_i8(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t tmem_e, uint32_t idesc, uint32_t acc) {
  if (SP && CTAS == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "tcgen05.mma.sp.cta_group::1.kind::i8 [%0], %1, %2, [%3], %4, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(tmem_e), "r"(idesc), "r"(acc) : "memory");
  else if (SP)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
                 "tcgen05.mma.sp.cta_group::2.kind::i8 [%0], %1, %2, [%3], %4, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(tmem_e), "r"(idesc), "r"(acc) : "memory");
  else if (CTAS == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void copy_e(uint32_t taddr, uint64_t sdesc) {
  if (CTAS == 1) asm volatile("tcgen05.cp.cta_group::1.128x128b [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.128x128b [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}

// two neighbouring elements, on a 4-byte boundary, of Y and of the array behind it
__device__ __forceinline__ void put_split(__nv_bfloat16* at, int64_t second, float a, float b) {
  uint32_t hi, lo;
  rows::split2(a, b, hi, lo);
  *reinterpret_cast<uint32_t*>(at) = hi;
  *reinterpret_cast<uint32_t*>(at + second) = lo;
}
__device__ __forceinline__ void store_one(const I8P& p, int64_t tok, int64_t row, float v) {
  const int64_t o = tok * p.ldy + row;
  if (p.out == ARMOR_DTYPE_F32) static_cast<float*>(p.Y)[o] = v;
  else if (p.out == ARMOR_DTYPE_BF16) static_cast<__nv_bfloat16*>(p.Y)[o] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p.Y)[o] = __float2half_rn(v);
}
// rows row, row + 1 (row even) of one token
template <bool SP>
__device__ __forceinline__ void store_two(const I8P& p, int64_t tok, int64_t row, float a, float b) {
  if (p.pairs && row + 1 < p.M) {
    const int64_t o = tok * p.ldy + row;
    if (SP && p.out == OUT_TWO_BF16) put_split(static_cast<__nv_bfloat16*>(p.Y) + o, p.second, a, b);
    else if (p.out == ARMOR_DTYPE_F32) *reinterpret_cast<float2*>(static_cast<float*>(p.Y) + o) = make_float2(a, b);
    else if (p.out == ARMOR_DTYPE_BF16)
      *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.Y) + o) = rows::pack2(static_cast<const __nv_bfloat16*>(nullptr), a, b);
    else *reinterpret_cast<uint32_t*>(static_cast<__half*>(p.Y) + o) = rows::pack2(static_cast<const __half*>(nullptr), a, b);
    return;
  }
  if (row < p.M) store_one(p, tok, row, a);
  if (row + 1 < p.M) store_one(p, tok, row + 1, b);
}

// ---------------------------------------------------------------------------------------------------------
// Few tokens: reading W is the cost.  A CTA takes a row tile, BN tokens and a piece of the contraction; the pieces of a tile are
// a cluster, which adds its int32 sums through distributed shared memory (exact in any order): each CTA has a share of the rows and
// writes their outputs.  W is fetched before the wait for the kernel that rounds the tokens.
//
// X other than int8_t: one token or two, rounded here rather than by a kernel before (which takes longer than the product): every CTA
// finds the largest |x| of the whole row, rounds its piece's part of it and lays it down as the tiles that a TMA load would have brought.
template <int BN, bool SP, typename X>
struct Few {
  static constexpr bool RAW = sizeof(X) > 1;
  static constexpr int B_BYTES = BN * 128 * (SP ? 2 : 1);
  static constexpr int STAGE = A_BYTES + (RAW ? 0 : B_BYTES) + (SP ? E_BYTES : 0);
  static constexpr int TILES = RAW ? 32 * 1024 : 0;                           // all tiles of x of a piece
  static constexpr int SUMS = BN * BM * 4;                                    // a CTA's sums, in the place of the stages
  static constexpr int STAGES = (110 * 1024 - TILES) / STAGE;                 // two CTAs share an SM
  static constexpr int NEED = BN + (SP ? 8 * STAGES : 0);
  static constexpr uint32_t COLS = NEED <= 32 ? 32 : (NEED <= 64 ? 64 : (NEED <= 128 ? 128 : 256));
  static constexpr size_t SMEM = (size_t)(STAGES * STAGE > SUMS ? STAGES * STAGE : SUMS) + TILES + 1024;
  static_assert(STAGES >= 2 && SMEM <= 111 * 1024 && (!RAW || STAGES * STAGE >= SUMS), "");
  static constexpr int MAX_PER = RAW ? TILES / B_BYTES : 1 << 30;
};
constexpr int FEW_THREADS = 192;
// the same place in shared memory of another piece's CTA
__device__ __forceinline__ uint32_t in_piece(uint32_t addr, uint32_t piece) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(piece));
  return r;
}

// The rows of x rounded by threads 64 .. 191: their scales to scale[], the piece's part, k from `from` to `to`, to tiles of BN rows x 128 k
template <int BN, typename X>
__device__ __forceinline__ void round_rows(const I8P& p, uint32_t tiles, float* scale, unsigned (&red)[4], int64_t from, int64_t to) {
  const int id = threadIdx.x - 64, warp = id >> 5, lane = id & 31;
  for (int t = 0; t < (int)p.N; ++t) {
    const X* const x = static_cast<const X*>(p.x) + t * p.ldx;
    auto load = [&](int64_t e) { return p.x_aligned ? rows::row_load<true>(x, e, p.K) : rows::row_load<false>(x, e, p.K); };
    unsigned top = 0;
#pragma unroll 4
    for (int64_t e = id * 8; e < p.K; e += 128 * 8) top = max(top, rows::raw_top(load(e)));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) red[warp] = top;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const rows::RowScale r = rows::row_scale<sizeof(X) == 2>(max(max(red[0], red[1]), max(red[2], red[3])));
    asm volatile("bar.sync 1, 128;" ::: "memory");          // (red is read before the next row writes it)
    if (id == 0) scale[t] = r.s;
    for (int64_t e = from + id * 8; e < to; e += 128 * 8) {
      float v[8];
      rows::raw_get(load(e), v);
      const uint2 q = rows::row_round8<sizeof(X) == 2>(v, r);
      const uint32_t k = (uint32_t)(e - from), b = k & 127u;
      const uint32_t at = tiles + (k >> 7) * (BN * 128) + (uint32_t)t * 128 + ((((b >> 4) ^ ((uint32_t)t & 7u))) << 4) + (b & 8u);
      asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(q.x), "r"(q.y) : "memory");
    }
  }
}

template <int BN, bool SP, typename X>
__global__ void __launch_bounds__(FEW_THREADS, 2)
i8_few_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
              const __grid_constant__ CUtensorMap mapE, const I8P p) {
  using T = Few<BN, SP, X>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bars[2 * T::STAGES + 2];
  __shared__ float own_scale[T::RAW ? BN : 1];
  __shared__ unsigned own_top[4];
  __shared__ uint32_t tmem_base_holder;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[T::STAGES]), tfull = smem_u32(&bars[2 * T::STAGES]);
  const uint32_t rounded = tfull + 8, tiles = smem_u32(smem) + T::STAGES * T::STAGE;
  const int mt = blockIdx.x, piece = blockIdx.y, pieces = gridDim.y;
  const int k0 = piece * p.per, k1 = min(p.k_tiles, k0 + p.per);
  const int64_t tok0 = (int64_t)blockIdx.z * BN;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < T::STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    mbar_init(tfull, 1);
    mbar_init(rounded, 128);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_holder)),
                 "r"(T::COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const bool ahead = p.ahead != 0;
  if (!ahead) grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t tmem_base = tmem_base_holder;
  volatile int* abortp = &abort_flag;

  if (warp == 0) {
    if (lane == 0) {
      auto load_w = [&](int kt, int stage) {
        const uint32_t dst = smem_u32(smem + (size_t)stage * T::STAGE), fb = full0 + 8 * stage;
        mbar_expect_tx(fb, T::STAGE);
        tma_load_2d(dst, &mapA, kt * 128, mt * BM, fb);
        if (SP) tma_load_2d(dst + T::STAGE - E_BYTES, &mapE, 0, (mt * p.k_tiles + kt) * 256, fb);
      };
      auto load_x = [&](int kt, int stage) {
        if (T::RAW) return;
        const uint32_t dst = smem_u32(smem + (size_t)stage * T::STAGE) + A_BYTES, fb = full0 + 8 * stage;
        tma_load_2d(dst, &mapB, kt * (SP ? 256 : 128), (int)tok0, fb);
        if (SP) tma_load_2d(dst + BN * 128, &mapB, kt * 256 + 128, (int)tok0, fb);
      };
      const int pre = min(T::STAGES, k1 - k0);
      for (int i = 0; i < pre; ++i) load_w(k0 + i, i);
      if (ahead) grid_dependency_wait();
      for (int i = 0; i < pre; ++i) load_x(k0 + i, i);
      int stage = pre % T::STAGES; uint32_t phase = pre == T::STAGES ? 1 : 0;
      long long issued = pre;
      bool ok = true;
      for (int kt = k0 + pre; kt < k1; ++kt) {
        if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abortp, p.status)) { ok = false; break; }
        load_w(kt, stage);
        load_x(kt, stage);
        ++issued;
        if (++stage == T::STAGES) { stage = 0; phase ^= 1; }
      }
      if (!ok) {
        for (int back = 1; back <= T::STAGES && back <= issued; ++back) {
          int s = stage - back; uint32_t ph = phase;
          if (s < 0) { s += T::STAGES; ph ^= 1; }
          const long long t0 = clock64();
          while (!mbar_try(full0 + 8 * s, ph) && clock64() - t0 < 20000000ll) {}
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_i8(BM, BN, SP);
      int stage = 0; uint32_t phase = 0;
      bool ok = !T::RAW || mbar_wait(rounded, 0, abortp, p.status);
      for (int kt = k0; kt < k1 && ok; ++kt) {
        if (!mbar_wait(full0 + 8 * stage, phase, abortp, p.status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t sa = smem_u32(smem + (size_t)stage * T::STAGE), sb = T::RAW ? tiles + (uint32_t)((kt - k0) * T::B_BYTES) : sa + A_BYTES;
        const uint32_t meta = tmem_base + BN + (uint32_t)(8 * stage);
        if (SP) {
          copy_e<1>(meta, desc_e(sa + T::STAGE - E_BYTES));
          copy_e<1>(meta + 4, desc_e(sa + T::STAGE - E_BYTES + 2048));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          umma_i8<1, SP>(tmem_base, desc_k(sa + j * 32), desc_k(SP ? sb + (j >> 1) * (BN * 128) + (j & 1) * 64 : sb + j * 32), meta + 2 * j, idesc,
                         (uint32_t)((kt > k0) | (j != 0)));
        umma_commit(empty0 + 8 * stage);
        if (++stage == T::STAGES) { stage = 0; phase ^= 1; }
      }
      if (ok) umma_commit(tfull);
    }
  } else {
    if constexpr (T::RAW) {
      if (ahead) grid_dependency_wait();
      const int64_t width = SP ? 256 : 128, to = k1 * width;
      round_rows<BN, X>(p, tiles, own_scale, own_top, k0 * width, to < p.K ? to : p.K);
      fence_proxy_async();
      mbar_arrive(rounded);
    }
    // the CTA's sums to shared memory, [token][row]: all stages have been read when they are complete
    if (mbar_wait_warp(tfull, 0, abortp, p.status)) {
      tc_fence_after();
      const int q = warp & 3;
      int32_t* const sums = reinterpret_cast<int32_t*>(smem);
#pragma unroll 1
      for (int ch = 0; ch < BN / 16; ++ch) {
        if (tok0 + ch * 16 >= p.N) break;
        uint32_t r[16];
        tmem_ld16(tmem_base + (uint32_t)(ch * 16) + ((uint32_t)(q * 32) << 16), r);
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(ch * 16 + i) * BM + q * 32 + lane] = (int32_t)r[i];
      }
      tc_fence_before();
    }
  }
  __syncwarp();
  if (pieces > 1) cluster_sync_all(); else __syncthreads();
  if (!*abortp) {
    grid_dependency_wait();                                 // (every thread that reads the tokens' scales)
    // Row pairs [u0, u1) of every token.  A lane keeps to a row pair and takes four tokens at a time, so that the loads from the other
    // pieces are under way together.
    const int u0 = 64 * piece / pieces, w = 64 * (piece + 1) / pieces - u0;
    const int nv = (int)(p.N - tok0 < BN ? p.N - tok0 : BN);
    const int wide = w <= 8 ? 8 : (w <= 16 ? 16 : 32), abreast = 32 / wide * (FEW_THREADS / 32);      // tokens side by side
    const uint32_t base = smem_u32(smem);
    for (int u = lane % wide; u < w; u += 32) {
      const int r2 = u0 + u;
      const int64_t row = (int64_t)mt * BM + 2 * r2;
      if (row >= p.M) break;
      const bool two = row + 1 < p.M;
      const float wa = p.ws[row], wb = two ? p.ws[row + 1] : 0.f;
      const float ba = p.bias ? p.bias[row] : 0.f, bb = p.bias && two ? p.bias[row + 1] : 0.f;
      for (int t0 = warp * (32 / wide) + lane / wide; t0 < nv; t0 += 4 * abreast) {
        int32_t a[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
        uint32_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = base + (uint32_t)(min(t0 + i * abreast, nv - 1) * BM + 2 * r2) * 4;
        auto add = [&](int k) {                             // (no branch around a load: its wait would stand inside)
          int32_t x[4], y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t from = pieces > 1 ? in_piece(at[i], (uint32_t)k) : at[i];
            asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(x[i]), "=r"(y[i]) : "r"(from) : "memory");
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) { a[i] += x[i]; b[i] += y[i]; }
        };
        int k = 0;
        for (; k + 2 <= pieces; k += 2) { add(k); add(k + 1); }
        if (k < pieces) add(k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + i * abreast;
          if (t < nv) {
            const float xs = T::RAW ? own_scale[t] : p.xs[tok0 + t];
            store_two<SP>(p, tok0 + t, row, fmaf((float)a[i], xs * wa, ba), fmaf((float)b[i], xs * wb, bb));
          }
        }
      }
    }
  }
  __syncwarp();
  if (pieces > 1) cluster_sync_all(); else __syncthreads(); // nobody leaves while its sums are being read
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(T::COLS) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------------------
// The way out of 32 tokens of a warp's 32 rows: sums from tensor memory (lanes are rows), scaled, and neighbouring lanes swap one value of
// every pair of tokens, so that a lane stores two neighbouring rows of one token.  slot: 32 floats of the warp's own.
template <typename T>
__device__ __forceinline__ void put_two(T* at, float a, float b) { *reinterpret_cast<uint32_t*>(at) = rows::pack2(static_cast<const T*>(nullptr), a, b); }
__device__ __forceinline__ void put_two(float* at, float a, float b) { *reinterpret_cast<float2*>(at) = make_float2(a, b); }
// TWO: OUT_TWO_BF16 (M, ldy and Y's address even: those of a core).
template <typename T, bool TWO = false>
__device__ __forceinline__ void way_out(const I8P& p, uint32_t taddr, int64_t row, int64_t tok0, float ws, float bias, float* slot, int lane) {
  __syncwarp();
  slot[lane] = tok0 + lane < p.N ? p.xs[tok0 + lane] : 0.f;
  __syncwarp();
  uint32_t r[32];
  tmem_ld32(taddr, r);
  const bool odd = lane & 1;
  const int64_t even = row & ~int64_t(1);
  const bool pair = p.pairs && even + 1 < p.M, full = tok0 + 32 <= p.N;
  T* at = static_cast<T*>(p.Y) + (tok0 + odd) * p.ldy + even;
  const int64_t step = 2 * p.ldy;
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const float4 x = *reinterpret_cast<const float4*>(slot + i);
    const float v[4] = {fmaf((float)(int32_t)r[i], x.x * ws, bias), fmaf((float)(int32_t)r[i + 1], x.y * ws, bias),
                        fmaf((float)(int32_t)r[i + 2], x.z * ws, bias), fmaf((float)(int32_t)r[i + 3], x.w * ws, bias)};
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const float got = __shfl_xor_sync(0xffffffffu, odd ? v[k] : v[k + 1], 1);
      const float a = odd ? got : v[k], b = odd ? v[k + 1] : got;
      if (full || tok0 + i + k + odd < p.N) {
        if constexpr (TWO) { if (pair) put_split(at, p.second, a, b); }
        else if (pair) put_two(at, a, b);
        else {
          if (even < p.M) at[0] = rows::from_f<T>(a);
          if (even + 1 < p.M) at[1] = rows::from_f<T>(b);
        }
      }
      at += step;
    }
  }
}

// Many tokens: pairs of CTAs (cta_group::2), a tile of 256 rows of W by up to 256 tokens (sparse: 224), persistent, the next tile's
// products beside the last one's way out (two accumulators).  Each CTA holds 128 rows of W (and their positions, in its tensor
// memory) and half of the tile's tokens.  (Two row tiles to a stage's tokens, with one accumulator each, lose what the second accumulator hides:
// 28672 x 8192, 4,096 tokens dense 600 -> 688 us, sparse 452 -> 499.)
//   full[s]   (even CTA): armed for the bytes of both CTAs, whose loads complete on it
//   empty[s], tfull[2] (both CTAs): tcgen05.commit to the pair
//   tempty[2] (even CTA): an arrival of every epilogue warp of either CTA
template <bool SP>
struct Many {
  static constexpr int MAX_N = SP ? 224 : 256;                                // two accumulators and the positions fit tensor memory
  static constexpr int BH = MAX_N / 2 * 128;                                  // 128 bytes of half the tile's tokens
  static constexpr int E_AT = A_BYTES + BH * (SP ? 2 : 1);
  static constexpr int STAGE = E_AT + (SP ? E_BYTES : 0);
  static constexpr int STAGES = 220 * 1024 / STAGE;
  static constexpr uint32_t META = 2 * MAX_N;
  static constexpr int EPI = 8;                                               // epilogue warps, half of the tokens each four
  static constexpr int THREADS = 64 + 32 * EPI;
  static constexpr size_t SMEM = (size_t)STAGES * STAGE + 1024;
  static_assert(!SP || META + 8 * STAGES <= 512, "tensor memory");
};
constexpr uint32_t MANY_COLS = 512;

constexpr int GROUP_M = 8;                          // row tiles that run side by side: see sparse_tcgen05.cu
__device__ __forceinline__ void tile_to_mn(int tile, int m_tiles, int n_tiles, int& mt, int& nt) {
  const int per_group = GROUP_M * n_tiles;
  const int g = tile / per_group, r = tile - g * per_group;
  const int gm = min(GROUP_M, m_tiles - g * GROUP_M);
  mt = g * GROUP_M + r % gm;
  nt = r / gm;
}

template <bool SP>
__global__ void __launch_bounds__(Many<SP>::THREADS, 1)
i8_many_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
               const __grid_constant__ CUtensorMap mapE, const I8P p) {
  using T = Many<SP>;
  constexpr int STAGES = T::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bars[2 * STAGES + 4];
  __shared__ __align__(16) float slots[T::EPI][32];
  __shared__ uint32_t tmem_base_holder;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]);
  const uint32_t tfull0 = smem_u32(&bars[2 * STAGES]), tempty0 = smem_u32(&bars[2 * STAGES + 2]);
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int n_tiles_total = p.m_tiles * p.n_tiles;          // row tiles of 256
  const int half_n = p.tile_n / 2;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(tfull0 + 8 * s, 1); mbar_init(tempty0 + 8 * s, 2 * T::EPI); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_holder)),
                 "r"(MANY_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                       // both CTAs' barriers exist before anyone signals them
  tc_fence_after();
  grid_begin();                                             // (tensor memory is this CTA's before the next kernel's CTAs start)
  const uint32_t tmem_base = tmem_base_holder;
  volatile int* abortp = &abort_flag;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (both CTAs)
    if (lane == 0) {
      int stage = 0; uint32_t phase = 0; long long issued = 0;
      bool ok = true;
      for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs) {
        int mt, nt;
        tile_to_mn(tile, p.m_tiles, p.n_tiles, mt, nt);
        const int row0 = mt * 256 + (int)rank * 128, tok0 = nt * p.tile_n + (int)rank * half_n;
        for (int kt = 0; kt < p.k_tiles; ++kt) {
          if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abortp, p.status)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(full0 + 8 * stage, 2 * (A_BYTES + (SP ? E_BYTES : 0) + half_n * 128 * (SP ? 2 : 1)));
          const uint32_t fb = map_to_cta(full0 + 8 * stage, 0);
          const uint32_t dst = smem_u32(smem + (size_t)stage * T::STAGE);
          tma_load_2d_pair(dst, &mapA, kt * 128, row0, fb);
          tma_load_2d_pair(dst + A_BYTES, &mapB, kt * (SP ? 256 : 128), tok0, fb);
          if (SP) {
            tma_load_2d_pair(dst + A_BYTES + T::BH, &mapB, kt * 256 + 128, tok0, fb);
            tma_load_2d_pair(dst + T::E_AT, &mapE, 0, ((2 * mt + (int)rank) * p.k_tiles + kt) * 256, fb);
          }
          ++issued;
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
      // tail: the MMAs that read the stages issued last have finished (their commits reach both CTAs), so
      // nothing is in flight towards this CTA's shared memory when it leaves
      for (int back = 1; back <= STAGES && back <= issued; ++back) {
        int s = stage - back; uint32_t ph = phase;
        if (s < 0) { s += STAGES; ph ^= 1; }
        const long long t0 = clock64();
        while (!mbar_try(empty0 + 8 * s, ph) && clock64() - t0 < (ok ? WAIT_CYCLES : 20000000ll)) {}
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (even CTA only)
    if (lane == 0 && rank == 0) {
      const uint64_t da0 = desc_k(smem_u32(smem)), db0 = desc_k(smem_u32(smem) + A_BYTES), de0 = desc_e(smem_u32(smem) + T::E_AT);
      const uint32_t idesc = idesc_i8(256, p.tile_n, SP);
      int stage = 0; uint32_t phase = 0;
      int local = 0;
      bool ok = true;
      for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs, ++local) {
        const int as = local & 1;
        if (!mbar_wait_cluster(tempty0 + 8 * as, ((uint32_t)(local >> 1) & 1u) ^ 1u, abortp, p.status)) { ok = false; break; }
        tc_fence_after();
        const uint32_t tacc = tmem_base + (uint32_t)(as * T::MAX_N);
        for (int kt = 0; kt < p.k_tiles; ++kt) {
          if (!mbar_wait_cluster(full0 + 8 * stage, phase, abortp, p.status)) { ok = false; break; }
          tc_fence_after();
          const uint64_t off = (uint64_t)(uint32_t)(stage * (T::STAGE >> 4));
          const uint32_t meta = tmem_base + T::META + (uint32_t)(8 * stage);
          if (SP) {
            copy_e<2>(meta, de0 + off);
            copy_e<2>(meta + 4, de0 + off + (2048 >> 4));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
            umma_i8<2, SP>(tacc, da0 + off + 2 * j, db0 + off + (SP ? (uint64_t)((j >> 1) * (T::BH >> 4) + 4 * (j & 1)) : (uint64_t)(2 * j)), meta + 2 * j, idesc,
                           (uint32_t)((kt > 0) | (j != 0)));
          umma_commit_pair(empty0 + 8 * stage);
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
        if (ok) umma_commit_pair(tfull0 + 8 * as);
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue warps (both CTAs)
    const int q = warp & 3, half = (warp - 2) >> 2;          // lane quarter; odd or even chunks of 32 tokens
    int local = 0;
    bool ok = true;
    for (int tile = pair; tile < n_tiles_total && ok; tile += n_pairs, ++local) {
      int mt, nt;
      tile_to_mn(tile, p.m_tiles, p.n_tiles, mt, nt);
      const int as = local & 1;
      const int64_t row = (int64_t)mt * 256 + rank * 128 + q * 32 + lane;
      const float ws = row < p.M ? p.ws[row] : 0.f, bias = p.bias && row < p.M ? p.bias[row] : 0.f;
      if (!mbar_wait_warp(tfull0 + 8 * as, (uint32_t)(local >> 1) & 1u, abortp, p.status)) { ok = false; break; }
      tc_fence_after();
#pragma unroll 1
      for (int ch = half; ch < p.tile_n / 32; ch += 2) {
        const int64_t tok0 = (int64_t)nt * p.tile_n + ch * 32;
        if (tok0 >= p.N) break;
        const uint32_t taddr = tmem_base + (uint32_t)(as * T::MAX_N + ch * 32) + ((uint32_t)(q * 32) << 16);
        if (p.out == ARMOR_DTYPE_BF16) way_out<__nv_bfloat16>(p, taddr, row, tok0, ws, bias, slots[warp - 2], lane);
        else if (SP && p.out == OUT_TWO_BF16) way_out<__nv_bfloat16, true>(p, taddr, row, tok0, ws, bias, slots[warp - 2], lane);
        else if (p.out == ARMOR_DTYPE_F32) way_out<float>(p, taddr, row, tok0, ws, bias, slots[warp - 2], lane);
        else way_out<__half>(p, taddr, row, tok0, ws, bias, slots[warp - 2], lane);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(tempty0 + 8 * as, 0));
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                       // neither CTA leaves while its partner may still signal it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(MANY_COLS) : "memory");
  }
}

// int8 rows [rows][cols], box of 128 bytes x box_rows, 128-byte swizzle, zeros outside
bool make_map_i8(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// positions: rows of 16 bytes, a stage's 256 a box
bool make_map_e(CUtensorMap* map, const void* base, int64_t rows) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[2] = {4, (cuuint64_t)rows};
  cuuint64_t strides[1] = {16};
  cuuint32_t box[2] = {4, 256};
  cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One thread for 32 k of a row: their kept values (of eight groups of four) as int8 and the word of their positions.  Places behind
// the core (k of a last stage that is half full, rows of a last tile of 256) keep positions 0 and 1, which meet zeros.
__global__ void __launch_bounds__(256)
pack_core_i8_kernel(const float* __restrict__ S, const uint8_t* __restrict__ Mk, const float* __restrict__ top, int8_t* __restrict__ V,
                    uint32_t* __restrict__ E, float* __restrict__ scale, int64_t d_out, int64_t d_in, int32_t* status) {
  const int64_t k_tiles = (d_in + 255) / 256, words = k_tiles * 8;
  const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = w / words, kw = w - row * words;      // 32 k from 32 kw on
  if (row >= (d_out + 255) / 256 * 256) return;
  uint32_t word = 0x44444444u;
  if (row < d_out && kw * 32 < d_in) {
    const rows::RowScale r = rows::row_scale(__float_as_uint(top[row]));
    if (kw == 0) scale[row] = r.s;
    word = 0;
    uint32_t out[4] = {0u, 0u, 0u, 0u};
    int bad = 0;
    for (int g = 0; g < 8; ++g) {
      const int64_t at = row * (d_in / 4) + kw * 8 + g;
      const unsigned m = Mk[at] & 15u;
      const float4 v = *reinterpret_cast<const float4*>(S + 4 * at);
      const float vals[4] = {v.x, v.y, v.z, v.w};
      int i0 = -1, i1 = -1, cnt = 0;
      for (int i = 0; i < 4; ++i)
        if ((m >> i) & 1u) { if (cnt == 0) i0 = i; else if (cnt == 1) i1 = i; ++cnt; }
      if (cnt > 2) bad = 1;
      if (cnt < 2) {                                        // padded with positions that are not kept, i0 < i1
        if (cnt == 0) { i0 = 0; i1 = 1; }
        else if (i0 < 3) i1 = i0 + 1;
        else { i1 = 3; i0 = 2; }
      }
      float a = 0.f, b = 0.f;
      for (int i = 0; i < 4; ++i) {
        if (i == i0 && ((m >> i) & 1u)) a = vals[i];
        if (i == i1 && ((m >> i) & 1u)) b = vals[i];
      }
      word |= (uint32_t)(i0 | (i1 << 2)) << (4 * g);
      const uint32_t two = (uint32_t)(rows::row_round(a, r) & 255) | ((uint32_t)(rows::row_round(b, r) & 255) << 8);
      out[g >> 1] |= two << (16 * (g & 1));
    }
    *reinterpret_cast<uint4*>(V + row * (d_in / 2) + kw * 16) = make_uint4(out[0], out[1], out[2], out[3]);
    if (bad) atomicAdd(&status[ST_SPARSE_BAD_GROUPS], 1);
  }
  // stage kt of row tile mt: two blocks (128 k each) of 128 lanes x 16 bytes
  const int64_t mt = row / 128, kt = kw / 8;
  E[((mt * k_tiles + kt) * 2 + (kw % 8) / 4) * 512 + (row % 128) * 4 + kw % 4] = word;
}
// the largest kept |S| of a row, as bits in top (row_scale); of a group that keeps more than two, the first two
__global__ void __launch_bounds__(256)
core_top_kernel(const float* __restrict__ S, const uint8_t* __restrict__ Mk, float* __restrict__ top, int64_t d_in) {
  __shared__ float red[1][32];
  const int64_t row = blockIdx.x;
  unsigned m = 0;
  for (int64_t g = threadIdx.x; g < d_in / 4; g += 256) {
    const unsigned k = Mk[row * (d_in / 4) + g] & 15u;
    const float4 v = *reinterpret_cast<const float4*>(S + row * d_in + 4 * g);
    const float vals[4] = {v.x, v.y, v.z, v.w};
    int cnt = 0;
    for (int i = 0; i < 4; ++i)
      if (((k >> i) & 1u) && cnt++ < 2) m = max(m, __float_as_uint(vals[i]) & 0x7fffffffu);
  }
  m = rows::cta_max(m, red);
  if (threadIdx.x == 0) top[row] = __uint_as_float(m);
}

// a dependent launch whose CTAs along y are a cluster
template <typename K>
armor_status launch_few(armor_ctx* c, K kernel, dim3 grid, size_t smem, cudaStream_t s, const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mE,
                        const I8P& p) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid; cfg.blockDim = dim3(FEW_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 1; at[1].val.clusterDim.y = grid.y; at[1].val.clusterDim.z = 1;
  cfg.attrs = at; cfg.numAttrs = grid.y > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, mA, mB, mE, p) != cudaSuccess) return ARMOR_ERR_CUDA;
  c->launches++;
  return ARMOR_OK;
}

// What the few-token kernel takes with tiles of w tokens, in nanoseconds, and the pieces of the contraction with which it takes least: a CTA, two
// an SM, takes its stages at 38 bytes a ns, and 6 ns to add a token of a piece.  Clusters have to find room all at once (28672 x 8192, 320
// tokens, five rounds of three pieces 142 us, pairs of CTAs 94), and the machine holds fewer CTAs in clusters: of 296 what `held` says (the
// occupancy calculator's figures), and some clusters less while the kernel before still rounds many tokens (4096 x 14336, 32 tiles, pieces
// eight and seven: 17 tokens 12.1 and 13.3 us, 24 18.3 and 13.8, 37 19.1 to 21.1 and 14.6).
struct FewPlan { int w, n_tiles, pieces, per; int64_t cost; };
FewPlan few_plan(const armor_ctx* c, const I8P& p, bool sparse, int w) {
  constexpr int held[9] = {0, 296, 296, 279, 284, 280, 270, 259, 264};
  FewPlan best{w, (int)((p.N + w - 1) / w), 0, 0, 0};
  const int64_t stage = A_BYTES + (sparse ? E_BYTES + 256 * w : 128 * w), tiles = (int64_t)p.m_tiles * best.n_tiles;
  const int64_t taken = p.N * p.k_tiles * (sparse ? 256 : 128) > 1 << 18 ? 20 : 0;
  for (int want = 1; want <= 8 && (want == 1 || 2 * want <= p.k_tiles); ++want) {
    const int per = (p.k_tiles + want - 1) / want, pieces = (p.k_tiles + per - 1) / per;
    if (pieces > 1 && tiles * pieces > (int64_t)held[pieces] * c->n_sm / 148 - taken) continue;
    const int64_t waves = (tiles * pieces + 2 * c->n_sm - 1) / (2 * c->n_sm), cost = waves * per * stage / 38 + (pieces - 1) * w * 6;
    if (best.pieces == 0 || cost < best.cost) { best.pieces = pieces; best.per = per; best.cost = cost; }
  }
  return best;
}
template <int BN, bool SP, typename X>
armor_status run_few(armor_ctx* c, const CUtensorMap& mA, const CUtensorMap& mE, const int8_t* xq, int64_t ldx, int64_t K, I8P p, const FewPlan& plan,
                     cudaStream_t s) {
  using T = Few<BN, SP, X>;
  CUtensorMap mB = mA;
  if (!T::RAW && !make_map_i8(&mB, xq, p.N, K, ldx, BN)) return ARMOR_ERR_CUDA;
  static PerDeviceOnce attr;
  if (ensure_dynamic_smem(attr, c->device, i8_few_kernel<BN, SP, X>, T::SMEM) != ARMOR_OK) return ARMOR_ERR_CUDA;
  p.n_tiles = plan.n_tiles;
  p.per = plan.per;
  if (plan.w != BN || (T::RAW && p.per > T::MAX_PER)) return ARMOR_ERR_UNSUPPORTED;              // (rounds_itself has looked)
  return launch_few(c, i8_few_kernel<BN, SP, X>, dim3((unsigned)p.m_tiles, (unsigned)plan.pieces, (unsigned)p.n_tiles), T::SMEM, s, mA, mB, mE, p);
}

template <bool SP>
armor_status product(armor_ctx* c, const CUtensorMap& mA, const CUtensorMap& mE, const int8_t* xq, int64_t ldx, int64_t K, I8P p, cudaStream_t s,
                     int32_t x_dtype = ARMOR_DTYPE_I8) {
  KTimer kt(c, ARMOR_KC_GEMM, 2.0 * (double)p.M * (double)p.N * (double)K, s);      // (dense-equivalent)
  p.status = c->status;
  p.k_tiles = (int)((K + (SP ? 255 : 127)) / (SP ? 256 : 128));
  p.m_tiles = (int)((p.M + 127) / 128);
  FewPlan few = few_plan(c, p, SP, 16);
  if (p.x) {                                                // the kernel rounds x itself (rounds_itself)
    if (x_dtype == ARMOR_DTYPE_F32) return run_few<16, SP, float>(c, mA, mE, nullptr, 0, K, p, few, s);
    if constexpr (!SP) {
      if (x_dtype == ARMOR_DTYPE_BF16) return run_few<16, SP, __nv_bfloat16>(c, mA, mE, nullptr, 0, K, p, few, s);
      if (x_dtype == ARMOR_DTYPE_F16) return run_few<16, SP, __half>(c, mA, mE, nullptr, 0, K, p, few, s);
    }
    return ARMOR_ERR_UNSUPPORTED;
  }
  // Pairs of CTAs, or the few-token kernel with the contraction cut, each with the width of tile that costs least, by what they take
  // beside what both do (nanoseconds): a pair's SM takes its stages at 60 bytes a ns, rounds of them; the other as few_plan has it.  Measured, pairs
  // and pieces: 4096 x 4096, 128 tokens 17.3 and 13.0 us; 8192 x 8192, 192 32.6 and 27.6; 4096 x 14336, 320 47.4 and 31.9; 512 x 8192, 512 30.2 and
  // 19.2; 256 x 14336, 1,024 49 and 26.5; 14336 x 4096, 200 22.9 and 27.6; 8192 x 8192, 300 35 and 43.  Beyond 512 tokens the estimate of the
  // pieces is short (1024 x 1024, 1,024 tokens 11.5 us for 10.5): they have to win by a quarter.  Widths of the pieces: 1024 x 1024, 64
  // tokens, one tile of 64 8.0 us, four of 16 6.4; 14336 x 4096, 96 tokens, a tile of 128 19.1, of 96 16.6.
  using T = Many<SP>;
  constexpr int64_t W_BYTES = A_BYTES + (SP ? E_BYTES : 0);
  const int pairs = c->n_sm / 2, rows256 = (int)((p.M + 255) / 256);
  int64_t least = 0;
  for (int w = T::MAX_N; w >= 64; w -= 32) {
    const int64_t rounds = ((int64_t)rows256 * ((p.N + w - 1) / w) + pairs - 1) / pairs, cost = rounds * (W_BYTES + (SP ? 128 : 64) * w);
    if (w == T::MAX_N || cost < least) { least = cost; p.tile_n = w; }
  }
  for (const int w : {32, 64, 96, 128, 160, 192}) {
    if (w - 32 >= p.N || w > (SP ? 128 : 192)) break;       // (wider ones with positions and twice the tokens leave a CTA no second stage)
    const FewPlan plan = few_plan(c, p, SP, w);
    if (plan.cost < few.cost) few = plan;
  }
  const int64_t many = least * p.k_tiles / 60 + 1000;
  if (p.N <= 32 || (p.N <= 512 && few.cost < many) || (p.N <= 1024 && 4 * few.cost < 3 * many)) {
    if (few.w == 16) return run_few<16, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
    if (few.w == 32) return run_few<32, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
    if (few.w == 64) return run_few<64, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
    if (few.w == 96) return run_few<96, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
    if constexpr (!SP) {
      if (few.w == 160) return run_few<160, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
      if (few.w == 192) return run_few<192, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
    }
    return run_few<128, SP, int8_t>(c, mA, mE, xq, ldx, K, p, few, s);
  }
  p.m_tiles = rows256;
  p.n_tiles = (int)((p.N + p.tile_n - 1) / p.tile_n);
  CUtensorMap mB;
  if (!make_map_i8(&mB, xq, p.N, K, ldx, p.tile_n / 2)) return ARMOR_ERR_CUDA;
  static PerDeviceOnce attr;
  if (ensure_dynamic_smem(attr, c->device, i8_many_kernel<SP>, T::SMEM) != ARMOR_OK) return ARMOR_ERR_CUDA;
  const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
  launch_dependent(i8_many_kernel<SP>, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), dim3(T::THREADS), T::SMEM, LaunchStream(s, false, 2), mA, mB, mE, p);
  c->launches++;
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}

I8P output(void* y, int32_t dtype, int64_t ldy, int64_t n, int64_t n_out, const float* xs, const float* ws, const float* bias, int ahead) {
  I8P p{};
  const int es = dtype == OUT_TWO_BF16 ? 2 : rows_dtype_bytes(dtype);
  p.Y = y; p.ldy = ldy; p.out = dtype; p.second = n * ldy; p.xs = xs; p.ws = ws; p.bias = bias; p.M = n_out; p.N = n; p.ahead = ahead;
  p.pairs = reinterpret_cast<uintptr_t>(y) % (2 * es) == 0 && ldy % 2 == 0;
  return p;
}

I8P with_rows(I8P p, const void* x, int32_t dtype, int64_t ldx, int64_t K) {
  p.x = x; p.ldx = ldx; p.K = K;
  p.x_aligned = rows::aligned16(x, p.N > 1 ? ldx : 8, rows_dtype_bytes(dtype));
  return p;
}

// (rows up to whole tiles of 256: those beyond d_out hold positions too, 0 and 1, for an instruction that covers them)
int64_t core_rows(int64_t d_out) { return (d_out + 255) / 256 * 256; }

}  // namespace

// y [n, n_out] = xq [n, n_in] wq [n_out, n_in]^T; ahead: the kernel before this one wrote xq and xs and nothing else that is read here,
// and waits for the kernel before it ahead of letting this one in
armor_status launch_linear_i8(armor_ctx* c, const int8_t* xq, int64_t ldx, const float* xs, const int8_t* wq, int64_t ldw, const float* ws,
                              const float* bias, void* y, int32_t y_dtype, int64_t ldy, int64_t n, int64_t n_out, int64_t n_in, bool ahead,
                              cudaStream_t s) {
  CUtensorMap mA;
  if (!make_map_i8(&mA, wq, n_out, n_in, ldw, BM)) return ARMOR_ERR_CUDA;
  return product<false>(c, mA, mA, xq, ldx, n_in, output(y, y_dtype, ldy, n, n_out, xs, ws, bias, ahead ? 1 : 0), s);
}

// Whether n rows of x of K elements are rounded by the product's own CTAs: each reads all of x, up to 32 KiB, and the part of a piece fits.
static bool rounds_itself(const armor_ctx* c, bool sparse, int64_t n, int64_t n_out, int64_t K, int32_t dtype) {
  if (n > 2 || n * K * rows_dtype_bytes(dtype) > 32768) return false;
  I8P p{};
  p.k_tiles = (int)((K + (sparse ? 255 : 127)) / (sparse ? 256 : 128));
  p.m_tiles = (int)((n_out + 127) / 128);
  p.N = n;
  const int per = few_plan(c, p, sparse, 16).per;
  return per <= (sparse ? Few<16, true, float>::MAX_PER : Few<16, false, float>::MAX_PER);
}
// The same from rows of x that are not rounded yet; UNSUPPORTED where they have to be rounded first.
armor_status launch_linear_i8_raw(armor_ctx* c, const void* x, int32_t x_dtype, int64_t ldx, const int8_t* wq, int64_t ldw, const float* ws,
                                  const float* bias, void* y, int32_t y_dtype, int64_t ldy, int64_t n, int64_t n_out, int64_t n_in, cudaStream_t s) {
  if (!rounds_itself(c, false, n, n_out, n_in, x_dtype)) return ARMOR_ERR_UNSUPPORTED;
  CUtensorMap mA;
  if (!make_map_i8(&mA, wq, n_out, n_in, ldw, BM)) return ARMOR_ERR_CUDA;
  return product<false>(c, mA, mA, nullptr, 0, n_in, with_rows(output(y, y_dtype, ldy, n, n_out, nullptr, ws, bias, 0), x, x_dtype, ldx, n_in), s, x_dtype);
}
armor_status launch_core_i8_raw(armor_ctx* c, const float* z1, const int8_t* V, const void* E, const float* scale, void* z2, int32_t z2_dtype, int64_t n,
                                bool ahead, cudaStream_t s) {
  if (!rounds_itself(c, true, n, c->d_out, c->d_in, ARMOR_DTYPE_F32)) return ARMOR_ERR_UNSUPPORTED;
  CUtensorMap mA, mE;
  if (!make_map_i8(&mA, V, c->d_out, c->d_in / 2, c->d_in / 2, BM)) return ARMOR_ERR_CUDA;
  if (!make_map_e(&mE, E, core_rows(c->d_out) / 128 * ((c->d_in + 255) / 256) * 256)) return ARMOR_ERR_CUDA;
  return product<true>(c, mA, mE, nullptr, 0, c->d_in, with_rows(output(z2, z2_dtype, c->d_out, n, c->d_out, nullptr, scale, nullptr, ahead ? 1 : 0), z1, ARMOR_DTYPE_F32,
                       c->d_in, c->d_in), s, ARMOR_DTYPE_F32);
}

// The core of a layer in 8 bits: values [d_out, d_in / 2], positions (packed_core_i8_e_bytes), scales [d_out]
size_t packed_core_i8_e_bytes(int64_t d_out, int64_t d_in) { return (size_t)core_rows(d_out) * (size_t)((d_in + 255) / 256) * 32; }
armor_status launch_pack_core_i8(armor_ctx* c, const float* S, const uint8_t* M, int8_t* V, void* E, float* scale, cudaStream_t s) {
  const int64_t words = core_rows(c->d_out) * ((c->d_in + 255) / 256) * 8;
  KTimer kt(c, ARMOR_KC_FORWARD, (double)c->wn * 4.875, s);
  core_top_kernel<<<(unsigned)c->d_out, 256, 0, s>>>(S, M, c->T, c->d_in);
  pack_core_i8_kernel<<<(unsigned)((words + 255) / 256), 256, 0, s>>>(S, M, c->T, V, static_cast<uint32_t*>(E), scale, c->d_out, c->d_in, c->status);
  c->launches += 2;
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}
// z2 [n, d_out] = zq [n, d_in] core^T
armor_status launch_core_i8(armor_ctx* c, const int8_t* zq, const float* zs, const int8_t* V, const void* E, const float* scale, void* z2,
                            int32_t z2_dtype, int64_t n, bool ahead, cudaStream_t s) {
  CUtensorMap mA, mE;
  if (!make_map_i8(&mA, V, c->d_out, c->d_in / 2, c->d_in / 2, BM)) return ARMOR_ERR_CUDA;
  if (!make_map_e(&mE, E, core_rows(c->d_out) / 128 * ((c->d_in + 255) / 256) * 256)) return ARMOR_ERR_CUDA;
  return product<true>(c, mA, mE, zq, c->d_in, c->d_in, output(z2, z2_dtype, c->d_out, n, c->d_out, zs, scale, nullptr, ahead ? 1 : 0), s);
}
