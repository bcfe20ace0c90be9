// Attention of chunks of new tokens over a paged cache of int8 keys and values, on the tensor cores (tcgen05).  The formulas are those of
// kv_attend_few.cu: S = Q Kq^T in fp32, t = S ks factor + log2 vs, weights 2^(t - m) in fp16, O = W Vq, l = sum w / vs, o = O / l.
//
// A unit is a tile of 256 rows (a token and a head of the group each; the heads of a group share keys) of one sequence and key head against the
// blocks of 64 positions that its rows see.  A CTA takes it as two halves of 128 rows, so that the tensor cores have the one half's
// products while the other's weights are formed:
//   warps 0-3, 4-7 : the rows of a half each: S from tensor memory, weights back to places of their own, O rescaled there when the maximum moves by far
//                    (rarely), O out at the end; they also bring q in (fp16, scaled by a power of two where it was bf16).  A lane has 16 of
//                    the block's columns in four rows, not a row (a lane a row reads all positions' numbers: 96 reads of 16 bytes a
//                    warp for 128 positions, each of them 512 bytes into registers, and those took 11,000 cycles; now 64 take 2,900)
//   warps 8-11     : keys from their pages through registers to fp16 in shared memory, four blocks, and the three numbers of a
//                    position (ks factor, log2 vs, 2^-RAISED / vs)
//   warps 12-15    : values likewise
//   warp 16        : the products: Q K^T (both from shared memory), W V (W from tensor memory, V as it lies, contiguous along the dimensions)
//   warp 17        : finds the units of the CTA's share, a few ahead of the others
// Tensor memory: for either half S of a block (64 columns), the weights of two (32 each) and O.  S is read into registers at once, so that the next
// block's scores are formed behind this one's exponentials.
//
// Bound by the products' operands: M 128 N 64 from shared memory takes 80 to 90 cycles here (32 by the rate), and the warp that issues them
// stands meanwhile.  8,192 tokens of 64 heads, causal: 1.45 to 1.48 ms between GPUs, 743 to 760 TFLOP/s; 2,048 after 14,337 of 32 heads, each its own keys: 0.66 to
// 0.70 ms, 738 to 778.
//
// All blocks of all units, and OVERHEAD more for each unit, stand in one line, cut into equal shares for one CTA an SM.  (Without the overhead the CTAs with the
// first tiles of a prompt, of a few blocks each, came last: 8,192 tokens of 64 heads 1.82 ms.)  A unit that is cut leaves its parts in the
// workspace, and kv_join_kernel adds them in their order.  Every wait is bounded; a CTA whose wait ran out goes on without waiting, so
// that no barrier is missed, and the status says that its output is worthless.
#include "kv_cache.cuh"
#include "tc_common.cuh"

namespace {

using namespace rows;
using namespace kv;
using namespace tc;

constexpr int THREADS = 640, HALF = 128, ROWS = 2 * HALF, KEYS = 64;
constexpr int SEQS = 1024;                  // sequences a launch
constexpr int JOIN_ROWS = 16, JOIN_THREADS = 256, JOIN_PARTS = 4;   // rows and threads of a CTA of the join, parts under way (16 x 5 tokens: 128 threads 70 us,
                                            // 256 68, 32 rows of 128 77; 64 tokens after 29,936: 16 CTAs a unit 68 us, 4 127; its maxima first 68, with the sums 64)
constexpr int OVERHEAD = 5;                 // what a unit takes beside its blocks, in blocks: q in, O out, the first maximum (14,000 cycles)

constexpr int NUMBERS = 8;                  // blocks whose positions' numbers are kept

template <int DIM>
struct Tile {
  static constexpr int Q_CHUNK = HALF * 128, CHUNK = KEYS * 128;         // 64 dimensions of a half's rows, of a block's
  static constexpr int Q_BYTES = DIM / 64 * Q_CHUNK, BYTES = DIM / 64 * CHUNK;
  static constexpr int PART = ROWS * (DIM + 2);                 // floats of a part: O, four dimensions of all rows behind one another; m; l
  // q of both halves (their outputs at the end), blocks of keys, of values, the numbers of blocks
  static constexpr int Q0 = 0, K0 = 2 * Q_BYTES, V0 = K0 + STAGES * BYTES, C0 = V0 + STAGES * BYTES;
  static constexpr int CONSTS = 3 * KEYS * 4;                   // for two positions: factors, logarithms (16 bytes); behind those of all: inverses
  static constexpr size_t SMEM = C0 + NUMBERS * CONSTS + 1024;
};

struct Cut { int seq, head, tile, last; };  // a unit whose first part is this CTA's; last: the CTA of its last part (-1: none)

struct TileP {
  KvAttend a;
  int64_t limit;                            // sequences of so many rows or fewer are left out
  float* parts;                             // two of every CTA
  Cut* cuts;                                // one of every CTA
  int whole;                                // no room for parts: units are not cut
  int32_t* status;
};

__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float minus_inf() { return -__int_as_float(0x7f800000); }
__device__ __forceinline__ uint32_t bytes_half(uint32_t x, uint32_t sel) {       // (kv_attend_few.cu)
  const uint32_t w = __byte_perm(x, 0x64646464u, sel);
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0x64806480u));
  return r;
}
// upper half of a descriptor of rows of 128 bytes, swizzled, groups of eight 1024 bytes apart (smem_desc_sw128)
constexpr uint32_t SW128_HI = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ void put16(uint32_t at, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// (the address is made behind the wait for what it holds: see `behind`)
__device__ __forceinline__ void behind(uint32_t& at) { asm volatile("" : "+r"(at)::"memory"); }
__device__ __forceinline__ float4 get16(uint32_t at) {
  float4 v;
  asm("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ float2 get8(uint32_t at) {
  float2 v;
  asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at));
  return v;
}

// fp16 operands, fp32 sums; M = 128
__device__ __forceinline__ uint32_t idesc_f16(int n, int b_mn) {
  return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
__device__ __forceinline__ void umma_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader)
      : "memory");
}
// 32 columns of a warp's lanes, a lane a row; the caller waits
__device__ __forceinline__ void tmem_get32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// 16 rows of 64 columns, dealt out as the accumulators of an mma are: r[4 g ..]: columns 8 g + 2 (lane % 4), + 1 of row lane / 4, then of row lane / 4 + 8
__device__ __forceinline__ void tmem_get_frag(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// the same of 32 columns
__device__ __forceinline__ void tmem_get_frag32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_put_frag32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// the same of pairs of 16-bit numbers: 32 columns of 32 bits, r[2 g ..]: column 4 g + lane % 4 of row lane / 4, then of row lane / 4 + 8
__device__ __forceinline__ void tmem_put_pairs(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

static __device__ __forceinline__ bool wait_warp_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  const long long t0 = clock64();
  bool ok;
#pragma unroll 1
  while (!(ok = mbar_try(bar, parity)) && !*abort_flag) {
    if (clock64() - t0 > WAIT_CYCLES) {
      *abort_flag = 1;
      atomicAdd(&status[ST_WAIT_TIMEOUTS], 1);
      status[ST_LAST_ERR] = ARMOR_ERR_TIMEOUT;
    }
  }
  return ok;
}
// mbar_wait_warp in a few instructions: there are twenty of them here, and the code of all roles has to stay in the instruction cache.  (With that
// one, whose inner loop is unrolled, the kernel had 400 KB.)
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  bool ok = mbar_try(bar, parity);
  if (!ok) ok = wait_warp_slow(bar, parity, abort_flag, status);
  return __all_sync(0xffffffffu, ok);
}

// The same without an answer, for the warp that issues the products: one that goes on after a wait ran out multiplies what is there.
__device__ __forceinline__ void wait_short(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  if (!mbar_try(bar, parity)) wait_warp_slow(bar, parity, abort_flag, status);
  __syncwarp();
}

// ---------------------------------------------------------------- units
// The blocks that a tile's rows see, from `block` on
struct Blocks { int block, count, low; };
__device__ __forceinline__ Blocks blocks_of(const KvAttend& a, const Seq& s, int tile) {
  const int rows = s.n * a.group, r0 = tile * ROWS, r1 = min(rows, r0 + ROWS) - 1;
  const int64_t at = (int64_t)s.length - s.n;
  const int64_t hi = max((int64_t)0, at + r1 / a.group + 1);
  const int64_t lo = a.window ? max((int64_t)0, at + r0 / a.group + 1 - a.window) : 0;
  Blocks b;
  b.low = (int)lo;
  b.block = (int)(lo / KEYS);
  b.count = max(1, (int)((hi + KEYS - 1) / KEYS) - b.block);
  return b;
}
__device__ __forceinline__ int tiles_of(const TileP& p, const Seq& s) {
  const int64_t rows = (int64_t)s.n * p.a.group;
  return rows > p.limit ? (int)((rows + ROWS - 1) / ROWS) : 0;
}

// What a CTA does with a unit, or with a piece of one: count blocks of positions from `block` on (0: there is no more)
struct __align__(16) Segment {
  int count, block;
  int rows;                                 // of the tile, if fewer than ROWS
  int seq, head;
  int first_row;                            // the tile's first row in its group: token r / group, head of the group r % group
  int row0;                                 // the sequence's first row in the packed arrays
  int n, length;                            // its new tokens, its positions
  int part;                                 // the place of the part that is left; -1: the unit is done here
  int low;                                  // the first position that a row of the tile sees
  int pad;
};
constexpr int RING = UNIT_PLACES;

// The CTA's share of the line, walked by one warp
struct Walk {
  const TileP& p;
  const int64_t* prefix;                    // [n + 1] where a sequence begins in the line
  int64_t left;                             // of the share from this segment on
  int seq, head, tile, tiles;
  Seq s;
  int first, count, total, block, low;      // of the segment: its first block in the unit, its blocks, the unit's, the position block of first; the tile's first position
  __device__ __forceinline__ Walk(const TileP& p_, const int64_t* prefix_) : p(p_), prefix(prefix_) {}
  __device__ __forceinline__ void load() {
    bool bad;
    s = sequence(p.a.b, seq, bad);
    tiles = tiles_of(p, s);
  }
  __device__ __forceinline__ void set(int off) {
    const Blocks b = blocks_of(p.a, s, tile);
    total = b.count;
    low = b.low;
    first = off;
    block = b.block + off;
    count = p.whole ? b.count : (int)min(left, (int64_t)(b.count - off));
  }
  __device__ __forceinline__ void start(int64_t begin, int64_t end, int seq_) {
    left = end - begin;
    if (left <= 0) return;
    seq = seq_;
    load();
    const int64_t a_head = divide(prefix[seq + 1] - prefix[seq], p.a.c.heads), off = begin - prefix[seq];
    head = (int)divide(off, a_head);
    int64_t rem = off - head * a_head;
    const int lane = threadIdx.x & 31;
    for (int t0 = 0;; t0 += 32) {
      const int t = t0 + lane;
      const int mine = t < tiles ? blocks_of(p.a, s, t).count + OVERHEAD : 0;
      int64_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const unsigned past = __ballot_sync(0xffffffffu, upto > rem);
      if (past || t0 + 32 >= tiles) {
        const int l = past ? __ffs(past) - 1 : 0;
        tile = t0 + l;
        rem -= __shfl_sync(0xffffffffu, upto, l) - __shfl_sync(0xffffffffu, mine, l);
        break;
      }
      rem -= __shfl_sync(0xffffffffu, upto, 31);
    }
    set((int)rem);
    if (count < 1 || (p.whole && first > 0)) {          // nothing left of this unit; or it is that of the CTA where it begins
      left -= total + OVERHEAD - first;
      advance();
    }
  }
  __device__ __forceinline__ void advance() {
    if (left <= 0) return;
    if (++tile == tiles) {
      tile = 0;
      if (++head == p.a.c.heads) {
        head = 0;
        do { ++seq; } while (seq < p.a.b.n && prefix[seq + 1] == prefix[seq]);
        if (seq >= p.a.b.n) { left = 0; return; }
        load();
      }
    }
    set(0);
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ void next() { left -= total + OVERHEAD - first; advance(); }
};

// eight dimensions from 8 c on of a row of a half in shared memory: rows of 128 bytes, swizzled
template <int DIM>
__device__ __forceinline__ uint32_t row_at(uint32_t base, int row, int c) {
  return base + (c >> 3) * Tile<DIM>::Q_CHUNK + row * 128 + (((c & 7) ^ (row & 7)) << 4);
}

// ALIGNED: rows of q and o start on 16-byte boundaries
template <typename T, int DIM, bool ALIGNED>
__global__ void __launch_bounds__(THREADS, 1)
kv_attend_tile_kernel(const TileP p) {
  using L = Tile<DIM>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  __shared__ __align__(8) uint64_t bars[32 + 2 * RING];
  __shared__ Segment ring[RING];
  __shared__ int64_t prefix[SEQS + 1];
  __shared__ unsigned tops[2][8];
  __shared__ float factors[2];
  __shared__ uint32_t tmem_base_holder;
  __shared__ int abort_flag, at_seq;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_u32(&bars[0]);
  // q of the upper half (Q_PLACES) and of the lower; of either half: S there and read, weights there and multiplied (two places); of the stages: keys,
  // values; the units
  const uint32_t q_full = bar0, q1_full = q_full + 8 * Q_PLACES, s_full = bar0 + 24, s_empty = bar0 + 40, p_full = bar0 + 56, o_done = bar0 + 88,
                 k_full = bar0 + 120, k_empty = bar0 + 152, v_full = bar0 + 184, v_empty = bar0 + 216, t_full = bar0 + 248, r_full = bar0 + 256,
                 r_empty = r_full + 8 * RING;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < Q_PLACES; ++i) mbar_init(q_full + 8 * i, 4);
    mbar_init(q1_full, 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(s_empty + 8 * i, 4);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(p_full + 8 * i, 4);
      mbar_init(o_done + 8 * i, 1);
    }
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(k_full + 8 * i, 2);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_full + 8 * i, 2);
      mbar_init(v_empty + 8 * i, 1);
    }
    mbar_init(t_full, 8);
    for (int i = 0; i < RING; ++i) {
      mbar_init(r_full + 8 * i, 1);
      mbar_init(r_empty + 8 * i, 17);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_holder)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_begin();
  const uint32_t tmem = tmem_base_holder;
  volatile int* const abortp = &abort_flag;
  const Cache& c = p.a.c;
  const Batch& b = p.a.b;

  // ---- the line of all blocks, this CTA's share of it and the sequence that it begins in
  for (int i = warp; i < b.n; i += THREADS / 32) {
    bool bad;
    const Seq s = sequence(b, i, bad);
    if (bad && blockIdx.x == 0 && lane == 0) report(p.status);
    const int tiles = tiles_of(p, s);
    int64_t sum = 0;
    for (int t = lane; t < tiles; t += 32) sum += blocks_of(p.a, s, t).count + OVERHEAD;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) prefix[i + 1] = sum * c.heads;
  }
  if (threadIdx.x == 0) at_seq = 0;
  __syncthreads();
  if (warp == 0) {
    const int per = (b.n + 31) / 32, i0 = min(b.n, lane * per), i1 = min(b.n, i0 + per);
    int64_t sum = 0;
    for (int i = i0; i < i1; ++i) sum += prefix[i + 1];
    int64_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    int64_t run = upto - sum;
    if (lane == 0) prefix[0] = 0;
    for (int i = i0; i < i1; ++i) { run += prefix[i + 1]; prefix[i + 1] = run; }
  }
  __syncthreads();
  const int64_t total = prefix[b.n];
  const int n_ctas = (int)min((int64_t)gridDim.x, total);
  const bool idle = (int)blockIdx.x >= n_ctas;
  const int64_t begin = idle ? 0 : divide((int64_t)blockIdx.x * total, n_ctas), end = idle ? 0 : divide((int64_t)(blockIdx.x + 1) * total, n_ctas);
  for (int i = threadIdx.x; i < b.n; i += THREADS)
    if (prefix[i] <= begin && begin < prefix[i + 1]) at_seq = i;
  if (warp == 17 && lane == 0) p.cuts[blockIdx.x].last = -1;
  __syncthreads();

  auto q_bar = [&](uint32_t n) { return q_full + 8 * ring_place(n, Q_PLACES); };      // of unit n
  // the n-th segment of the share, by a whole warp: false behind the last one.  done: the ring may have its place back
  auto segment = [&](uint32_t n) { return wait_warp(r_full + 8 * ring_place(n, RING), ring_parity(n, RING), abortp, p.status) && ring[n % RING].count > 0; };
  auto arrive = [&](uint32_t bar) {                                     // of a warp
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  auto done = [&](uint32_t n) { arrive(r_empty + 8 * (n % RING)); };
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    const int half = warp >> 2, row = threadIdx.x & 127, quad = lane >> 2, pair = lane & 3;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + half * 128 + lanes, tP = tS + 64, tO = tmem + 256 + half * 128 + lanes;
    uint32_t seg = 0, blocks = 0, turn = 0;                             // segments, blocks of the CTA, blocks of this half
    constexpr int LANES = DIM / 8, MOVES = LANES;                       // a row by so many lanes; 32 rows by so many instructions
    const int c8 = lane % LANES, sub_row = lane / LANES;
    const uint32_t rows_at = smem + L::Q0 + half * L::Q_BYTES;
    for (; segment(seg); ++seg) {
      const Segment& at = ring[seg % RING];                             // (read where it is needed: registers are short)
      const int rows = at.rows - half * HALF;                           // of this half
      auto row_in = [&](int64_t stride, int64_t head_stride) {          // where the lane's row begins in q or o
        const int r = row < rows ? at.first_row + half * HALF + row : 0, tok = r / p.a.group, g = r - tok * p.a.group;
        return (int64_t)(at.row0 + tok) * stride + (int64_t)(at.head * p.a.group + g) * head_stride;
      };
      // ---- q
      {
        uint4 raw[MOVES];
        const int64_t off = row_in(p.a.q_row, p.a.q_head);
#pragma unroll
        for (int i = 0; i < MOVES; ++i) {
          const int rr = i * (32 / LANES) + sub_row;
          const T* const from = static_cast<const T*>(p.a.q) + __shfl_sync(0xffffffffu, off, rr) + 8 * c8;
          raw[i] = (warp & 3) * 32 + rr >= rows ? make_uint4(0u, 0u, 0u, 0u) : row_load<ALIGNED>(from, 0, 8).w;
        }
        int shift = 0;
        if (std::is_same<T, __nv_bfloat16>::value) {
          // by the power of two that brings the largest finite |q| of the tile to [2^14, 2^15): what is lost is below 2^-39 of it
          unsigned top = 0;
#pragma unroll
          for (int i = 0; i < MOVES; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t lo = w[k] & 0x7fffu, hi = (w[k] >> 16) & 0x7fffu;
              if (lo < 0x7f80u) top = max(top, lo);
              if (hi < 0x7f80u) top = max(top, hi);
            }
          }
          top = __reduce_max_sync(0xffffffffu, top);
          if (lane == 0) {
            tops[seg & 1][warp] = top;
            mbar_arrive(t_full);
          }
          wait_warp(t_full, seg & 1, abortp, p.status);
          top = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) top = max(top, *(volatile unsigned*)&tops[seg & 1][i]);
          shift = top ? min(max(14 - ((int)(top >> 7) - 127), -120), 120) : 0;
        }
        if (threadIdx.x == 0) factors[seg & 1] = p.a.scale * __int_as_float((127 - shift) << 23);
        if (rows > 0) {
          const float up = __int_as_float((127 + shift) << 23);
          const T* const t = nullptr;
#pragma unroll
          for (int i = 0; i < MOVES; ++i) {
            uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            if (!std::is_same<T, __half>::value) {
#pragma unroll
              for (int k = 0; k < 4; ++k) { const float2 v = unpack2(t, w[k]); w[k] = pack2(static_cast<const __half*>(nullptr), v.x * up, v.y * up); }
            }
            put16(row_at<DIM>(rows_at, (warp & 3) * 32 + i * (32 / LANES) + sub_row, c8), make_uint4(w[0], w[1], w[2], w[3]));
          }
          fence_proxy_async();
          arrive(half ? q1_full : q_bar(seg));
        }
      }
      if (rows <= 0) { blocks += at.count; done(seg); continue; }
      // ---- the positions that rows lane / 4 + {0, 8, 16, 24} of the warp's see: [low, high); what all of them see
      auto sees = [&](int k, int& low, int& high) {
        const int rr = (warp & 3) * 32 + quad + 8 * k;
        low = 0;
        high = 0x7fffffff;                                              // (a row that does not exist: whatever costs nothing)
        if (rr < rows) {
          const int64_t pos = (int64_t)at.length - at.n + (at.first_row + half * HALF + rr) / p.a.group;
          high = (int)max((int64_t)0, pos + 1);
          low = p.a.window ? (int)max((int64_t)0, pos + 1 - p.a.window) : 0;
        }
      };
      int inner_lo = 0, inner_hi = 0x7fffffff;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        int low, high;
        sees(k, low, high);
        inner_lo = max(inner_lo, low);
        inner_hi = min(inner_hi, high);
      }
      inner_lo = __reduce_max_sync(0xffffffffu, inner_lo);
      inner_hi = __reduce_min_sync(0xffffffffu, inner_hi);
      float m[4] = {minus_inf(), minus_inf(), minus_inf(), minus_inf()};
      F2 l[4] = {f2(0.f), f2(0.f), f2(0.f), f2(0.f)};
      const int count = at.count, block0 = at.block;
      for (int i = 0; i < count; ++i, ++blocks, ++turn) {
        const int j0 = (block0 + i) * KEYS;
        const uint32_t place = turn & 1;
        wait_warp(s_full + 8 * half, turn & 1, abortp, p.status);       // (and the numbers: they are there before the keys)
        tc_fence_after();
        uint32_t consts = smem + L::C0 + (blocks % NUMBERS) * L::CONSTS + 16 * pair;
        behind(consts);
        const uint32_t inverses = consts - 8 * pair + 8 * KEYS;
        F2 t[4][8];
        {
          uint32_t raw[2][32];
#pragma unroll
          for (int e = 0; e < 2; ++e) tmem_get_frag(tS + ((uint32_t)(e * 16) << 16), raw[e]);
          tmem_wait_ld();
          tc_fence_before();
          arrive(s_empty + 8 * half);                                   // (the next block's scores are formed behind this one's weights)
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const float4 ab = get16(consts + 64 * g);
            const F2 fa = f2(ab.x, ab.y), fb = f2(ab.z, ab.w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t* const x = &raw[k >> 1][4 * g + 2 * (k & 1)];
              t[k][g] = f2_fma(f2(__uint_as_float(x[0]), __uint_as_float(x[1])), fa, fb);
            }
          }
        }
        if (j0 < inner_lo || j0 + KEYS > inner_hi) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            int low, high;
            sees(k, low, high);
            low -= j0 + 2 * pair;
            high -= j0 + 2 * pair;
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              float2 v = f2_get(t[k][g]);
              if (8 * g < low || 8 * g >= high) v.x = minus_inf();
              if (8 * g + 1 < low || 8 * g + 1 >= high) v.y = minus_inf();
              t[k][g] = f2(v.x, v.y);
            }
          }
        }
        float top[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 v = f2_get(t[k][0]);
          top[k] = fmaxf(v.x, v.y);
#pragma unroll
          for (int g = 1; g < 8; ++g) { const float2 v = f2_get(t[k][g]); top[k] = max3(top[k], v.x, v.y); }
        }
        // m hardly ever moves behind a row's first blocks
        constexpr float OVER = LAZY + RAISED;
        if (__any_sync(0xffffffffu, top[0] > m[0] + OVER || top[1] > m[1] + OVER || top[2] > m[2] + OVER || top[3] > m[3] + OVER)) {
          float f[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
            top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
            const float to = fmaxf(m[k], top[k] - RAISED);
            f[k] = m[k] == to ? 1.f : exp2_fast(m[k] - to);
            l[k] = f2_mul(l[k], f2(f[k]));
            m[k] = to;
          }
          if (i > 0) {
            wait_warp(o_done + 8 * (2 * half + (place ^ 1)), ((turn - 1) >> 1) & 1, abortp, p.status);   // (the product of the block before)
            tc_fence_after();
#pragma unroll 1
            for (int e = 0; e < DIM / 16; ++e) {
              uint32_t o[16];
              const float f0 = e & 1 ? f[2] : f[0], f1 = e & 1 ? f[3] : f[1];
              const uint32_t where = tO + ((uint32_t)((e & 1) * 16) << 16) + (e >> 1) * 32;
              tmem_get_frag32(where, o);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * (x & 2 ? f1 : f0));
              tmem_put_frag32(where, o);
            }
          }
        }
        F2 minus_m[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) minus_m[k] = f2(m[k] == minus_inf() ? 0.f : -m[k]);
        // (the weights that were here have been multiplied: before these scores, by the same warp)
        uint32_t w[2][16];
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float2 r = get8(inverses + 32 * g);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 x = f2_get(f2_add(t[k][g], minus_m[k]));
            const float e0 = exp2_fast(x.x), e1 = exp2_fast(x.y);
            l[k] = f2_fma(f2(e0, e1), f2(r.x, r.y), l[k]);
            w[k >> 1][2 * g + (k & 1)] = pack2(static_cast<const __half*>(nullptr), e0, e1);
          }
        }
        tmem_put_pairs(tP + 32 * place, w[0]);
        tmem_put_pairs(tP + (16u << 16) + 32 * place, w[1]);
        tmem_wait_st();
        tc_fence_before();
        arrive(p_full + 8 * (2 * half + place));
      }
      // m and l of the lane's row: they lie with the lanes 4 (row % 8) .. + 3, the sums a quarter each
      float row_m = 0.f, sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 v = f2_get(l[k]);
        float x = v.x + v.y;
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        const float s2 = __shfl_sync(0xffffffffu, x, 4 * (lane & 7)), m2 = __shfl_sync(0xffffffffu, m[k], 4 * (lane & 7));
        if (lane >> 3 == k) { sum = s2; row_m = m2; }
      }
      // ---- O out
      wait_warp(o_done + 8 * (2 * half + ((turn - 1) & 1)), ((turn - 1) >> 1) & 1, abortp, p.status);
      tc_fence_after();
      if (at.part >= 0) {
        float* const part = p.parts + (int64_t)at.part * L::PART + 4 * (half * HALF + row);
#pragma unroll 1
        for (int k = 0; k < DIM / 32; ++k) {
          uint32_t o[32];
          tmem_get32(tO + 32 * k, o);
          tmem_wait_ld();
          if (row < rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              *reinterpret_cast<uint4*>(part + (8 * k + e) * 4 * ROWS) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        if (row < rows) {
          float* const ml = p.parts + (int64_t)at.part * L::PART + ROWS * DIM + half * HALF + row;
          ml[0] = row_m;
          ml[ROWS] = sum;
        }
      } else {
        // by way of q's place, so that rows go out whole
        const float inv = sum == 0.f ? 0.f : LOWERED / sum;             // (a row that sees nothing: zeros)
        const T* const t = nullptr;
#pragma unroll 1
        for (int k = 0; k < DIM / 32; ++k) {
          uint32_t o[32];
          tmem_get32(tO + 32 * k, o);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) w[x] = pack2(t, __uint_as_float(o[8 * e + 2 * x]) * inv, __uint_as_float(o[8 * e + 2 * x + 1]) * inv);
            put16(row_at<DIM>(rows_at, row, 4 * k + e), make_uint4(w[0], w[1], w[2], w[3]));
          }
        }
        __syncwarp();
        const int64_t off = row_in(p.a.o_row, p.a.o_head);
#pragma unroll 4
        for (int i = 0; i < MOVES; ++i) {
          const int rr = i * (32 / LANES) + sub_row;
          T* const to = static_cast<T*>(p.a.o) + __shfl_sync(0xffffffffu, off, rr) + 8 * c8;
          uint32_t at16 = row_at<DIM>(rows_at, (warp & 3) * 32 + rr, c8);
          behind(at16);
          const float4 v = get16(at16);
          if ((warp & 3) * 32 + rr >= rows) continue;
          if (ALIGNED) *reinterpret_cast<float4*>(to) = v;
          else {
            const uint32_t w[4] = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
#pragma unroll
            for (int x = 0; x < 8; ++x) reinterpret_cast<unsigned short*>(to)[x] = (unsigned short)(w[x >> 1] >> (16 * (x & 1)));
          }
        }
      }
      done(seg);
    }
  } else if (warp < 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    // Warps 8-11 have the keys and the numbers, 12-15 the values; the first two of each the even blocks, the others the odd ones.  A warp takes 32
    // positions: a lane knows where one of them lies, DIM / 16 lanes load a row.  While a block is stored the rows of the warp's next one
    // are on their way, and the page of the one after that.
    const bool values = warp >= 12;
    const int w = warp & 1;
    constexpr int SUBS = DIM / 16;                                      // lanes of a row
    constexpr int LOADS = SUBS;                                         // rows that a lane takes part in: 32 / (32 / SUBS)
    const int lane_sub = lane % SUBS, lane_row = lane / SUBS;
    const int8_t* const from = (values ? c.v : c.k) + lane_sub * 16;
    uint32_t seg = 0;
    // the block whose page is looked up: the segment's blocks behind it, its sequence, head, first position, length, the lane's position
    int behind = 0, seq = 0, head = 0, low = 0, length = 0, j = 0;
    bool more = true;
    auto step = [&]() {                                                 // on to the next block; more: there is one
      j += KEYS;
      if (behind-- > 0) return;
      more = segment(seg);
      if (more) {
        const Segment& at = ring[seg % RING];
        behind = at.count - 1; seq = at.seq; head = at.head; low = at.low; length = at.length;
        j = at.block * KEYS + w * 32 + lane;
      }
      done(seg++);
    };
    // page: the lane's, or one that there is for a position that has none
    uint32_t page = 0, slot = 0;
    bool seen = false;
    auto look = [&]() {
      page = slot = 0;
      seen = j >= low && j < length;                                    // (what no row sees may lie on pages that are gone)
      if (seen) {
        const uint32_t i = quotient((uint32_t)j, c.mul, c.shift);
        slot = (uint32_t)j - i * c.page_size;
        page = i < (uint32_t)b.max_pages ? (uint32_t)b.pages[(int64_t)seq * b.ld + i] : 0xffffffffu;
      }
    };
    uint4 raw[LOADS];
    float ks = 0.f, vs = 0.f;
    bool there = false;
    int of_head = 0;
    auto load = [&]() {                                                 // of the block whose page has been looked up
      there = seen && page < c.n_pages;
      if (seen && !there) {
        if (!values) report(p.status);
        page = slot = 0;
      }
      const int64_t row = page * c.page + of_head * c.head + slot * c.slot;
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        raw[i] = *reinterpret_cast<const uint4*>(from + __shfl_sync(0xffffffffu, row, i * (32 / SUBS) + lane_row));
      if (!values) {
        const int64_t at = page * c.spage + of_head * c.shead + slot * c.sslot;
        ks = c.ks[at];
        vs = c.vs[at];
      }
    };
    // sixteen bytes of row i as fp16, two pieces of sixteen bytes (the second first in half of the lanes: eight lanes then meet in no bank)
    auto store = [&](uint32_t base) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = w * 32 + i * (32 / SUBS) + lane_row;
        const uint32_t a = raw[i].x ^ 0x80808080u, d = raw[i].y ^ 0x80808080u, e = raw[i].z ^ 0x80808080u, f = raw[i].w ^ 0x80808080u;
        const uint4 lo = make_uint4(bytes_half(a, 0x4140), bytes_half(a, 0x4342), bytes_half(d, 0x4140), bytes_half(d, 0x4342));
        const uint4 hi = make_uint4(bytes_half(e, 0x4140), bytes_half(e, 0x4342), bytes_half(f, 0x4140), bytes_half(f, 0x4342));
        const uint32_t line = base + (lane_sub >> 2) * L::CHUNK + r * 128;
        const uint32_t swap = (lane_sub >> 2) & 1, x = (lane_sub & 3) * 2, k = r & 7;
        put16(line + (((x + swap) ^ k) << 4), swap ? hi : lo);
        put16(line + (((x + 1 - swap) ^ k) << 4), swap ? lo : hi);
      }
    };
    uint32_t of = 0, ahead = 0;                                         // segments: of the loaded block, of the one that is looked up
    uint32_t n = ((uint32_t)(warp >> 1) & 1) - 2;                       // the loaded block (none yet)
    bool one = false;                                                   // there is a loaded block
    auto steps = [&](int times) {
#pragma unroll 1
      for (int e = 0; e < times && more; ++e) step();
      ahead = seg - 1;
      if (more) look();
    };
    const uint32_t full = values ? v_full : k_full, empty = values ? v_empty : k_empty, base = smem + (values ? L::V0 : L::K0);
    steps((int)n + 3);
    for (;; n += 2) {
     if (one) {
      const uint32_t st = n % STAGES;
      if (!values) wait_warp(q_bar(of), ring_parity(of, Q_PLACES), abortp, p.status);        // (the factor)
      wait_warp(empty + 8 * st, ((n / STAGES) & 1) ^ 1, abortp, p.status);
      if (!values) {
        // The numbers of block n - NUMBERS have been read: the keys of block n - STAGES have been multiplied, and those only when the scores of
        // block n - STAGES - 1 had been read, behind the weights of the one before
        const uint32_t at = smem + L::C0 + (n % NUMBERS) * L::CONSTS, k = w * 32 + lane, to = at + (k >> 1) * 16 + (k & 1) * 4;
        const float v = measure(vs);
        const float fa = there ? ks * *(volatile float*)&factors[of & 1] : 0.f, fb = there ? __log2f(v) : minus_inf(), fr = !there ? 0.f : (v == v ? __fdividef(LOWERED, v) : 1.f);    // (no number: the weight is none either, and 0 where it is not seen)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(fa) : "memory");
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + 8), "f"(fb) : "memory");
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 8 * KEYS + 4 * k), "f"(fr) : "memory");
      }
      store(base + st * L::BYTES);
      fence_proxy_async();
      arrive(full + 8 * st);
     }
     if (!more) break;
     one = true;
     // load the block that has been looked up, look up the next one
     of_head = head;
     of = ahead;
     load();
     steps(2);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 16) {
      const uint32_t leader = elect_lane();
      const uint32_t qk = idesc_f16(KEYS, 0), pv = idesc_f16(DIM, 1);
      auto wait = [&](uint32_t bar, uint32_t parity) { wait_short(bar, parity, abortp, p.status); };
      // (Descriptors begin from a value that the compiler knows to be the same in all lanes, so that they are formed in uniform registers.)
      const uint32_t tm = uniform(tmem);
      auto desc = [&](uint32_t at, uint32_t leading) { return (uint64_t)SW128_HI << 32 | (leading >> 4) << 16 | (at >> 4); };
      const uint32_t q0 = smem + L::Q0;
      auto scores = [&](int half, uint32_t st) {
        const uint32_t k0 = uniform(smem + L::K0 + st * L::BYTES), qh = uniform(q0 + half * L::Q_BYTES);
#pragma unroll
        for (int k = 0; k < DIM / 16; ++k)
          umma_ss(leader, tm + half * 128, desc(qh + (k >> 2) * L::Q_CHUNK + (k & 3) * 32, 16), desc(k0 + (k >> 2) * L::CHUNK + (k & 3) * 32, 16), qk, k > 0);
        umma_commit_w(leader, s_full + 8 * half);
      };
      auto values = [&](int half, uint32_t st, uint32_t place, bool acc) {
        const uint32_t v = uniform(smem + L::V0 + st * L::BYTES), w = uniform(tm + half * 128 + 64 + place * 32);
#pragma unroll
        for (int k = 0; k < KEYS / 16; ++k)
          umma_ts(leader, tm + 256 + half * 128, w + k * 8, desc(v + k * 2048, L::CHUNK), pv, acc || k > 0);
        umma_commit_w(leader, o_done + 8 * (2 * half + place));
      };
      uint32_t seg = 0, seg1 = 0, n = 0, turn[2] = {0, 0};
      for (; segment(seg); ++seg) {
        const int count = ring[seg % RING].count, halves = ring[seg % RING].rows > HALF ? 2 : 1;
        done(seg);
        wait(q_bar(seg), ring_parity(seg, Q_PLACES));
        if (halves == 2) wait(q1_full, seg1++ & 1);
        for (int i = -1; i < count; ++i) {
          // the scores of block i + 1, once those of block i have been read; then the values of block i
          const uint32_t next = n + (i < 0 ? 0 : 1), st2 = next % STAGES, st = n % STAGES;
          if (i + 1 < count) wait(k_full + 8 * st2, (next / STAGES) & 1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == halves) break;
            if (i >= 0) wait(s_empty + 8 * h, turn[h] & 1);
            if (i + 1 < count) {
              tc_fence_after();
              scores(h, st2);
              if (h + 1 == halves) umma_commit_w(leader, k_empty + 8 * st2);
            }
          }
          if (i < 0) continue;
          wait(v_full + 8 * st, (n / STAGES) & 1);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == halves) break;
            wait(p_full + 8 * (2 * h + (turn[h] & 1)), (turn[h] >> 1) & 1);
            tc_fence_after();
            values(h, st, turn[h] & 1, i > 0);
            if (h + 1 == halves) umma_commit_w(leader, v_empty + 8 * st);
            ++turn[h];
          }
          ++n;
        }
      }
    } else if (warp == 17) {
      Walk at(p, prefix);
      at.start(begin, end, at_seq);
      for (uint32_t n = 0;; ++n) {
        wait_warp(r_empty + 8 * ring_place(n, RING), ring_parity(n, RING) ^ 1, abortp, p.status);
        const bool cut = at.more() && at.count < at.total;
        if (lane == 0) {
          Segment g{};
          if (at.more()) {
            g.count = at.count; g.block = at.block; g.low = at.low;
            g.rows = at.s.n * p.a.group - at.tile * ROWS; g.first_row = at.tile * ROWS;
            g.seq = at.seq; g.head = at.head; g.row0 = at.s.first; g.n = at.s.n; g.length = at.s.length;
            g.part = cut ? 2 * (int)blockIdx.x + (at.first == 0 ? 1 : 0) : -1;
            if (cut && at.first == 0)                                   // parts up to the CTA that holds the unit's last block
              p.cuts[blockIdx.x] = Cut{at.seq, at.head, at.tile, (int)divide((end - at.left + at.total) * n_ctas - 1, total)};
          }
          ring[n % RING] = g;
          mbar_arrive(r_full + 8 * (n % RING));
        }
        __syncwarp();
        if (!at.more() || *abortp) break;
        at.next();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 16) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

// The parts of units that were cut: CTA x takes the unit whose first part is that of CTA x, JOIN_ROWS rows of it.
template <typename T, int DIM>
__global__ void __launch_bounds__(JOIN_THREADS)
kv_join_kernel(const TileP p) {
  grid_begin();
  using L = Tile<DIM>;
  const Cut cut = p.cuts[blockIdx.x];
  if (cut.last < 0) return;
  bool bad;
  const Seq s = sequence(p.a.b, cut.seq, bad);
  const int rows = s.n * p.a.group - cut.tile * ROWS, c0 = blockIdx.x;
  const int r = blockIdx.y * JOIN_ROWS + threadIdx.x % JOIN_ROWS;
  if (r >= rows) return;
  auto part = [&](int k) { return p.parts + (2 * (int64_t)k + (k == c0)) * L::PART; };
  for (int d = threadIdx.x / JOIN_ROWS * 4; d < DIM; d += JOIN_THREADS / JOIN_ROWS * 4) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float top = minus_inf(), sum = 0.f;
    for (int k0 = c0; k0 <= cut.last; k0 += JOIN_PARTS) {
      float m[JOIN_PARTS], l[JOIN_PARTS], to = top;
      float4 v[JOIN_PARTS];
#pragma unroll
      for (int u = 0; u < JOIN_PARTS; ++u) {
        const float* const from = part(min(k0 + u, cut.last));
        m[u] = k0 + u <= cut.last ? from[ROWS * DIM + r] : minus_inf();
        l[u] = from[ROWS * (DIM + 1) + r];
        v[u] = *reinterpret_cast<const float4*>(from + d * ROWS + 4 * r);
      }
#pragma unroll
      for (int u = 0; u < JOIN_PARTS; ++u) to = fmaxf(to, m[u]);
      const float f0 = top == to ? 1.f : exp2_fast(top - to);             // (nothing yet: 2^-inf)
      top = to;
      sum *= f0;
      o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
      for (int u = 0; u < JOIN_PARTS; ++u) {
        const float f = m[u] == minus_inf() ? 0.f : exp2_fast(m[u] - top);
        sum = fmaf(f, l[u], sum);
        o.x = fmaf(f, v[u].x, o.x); o.y = fmaf(f, v[u].y, o.y); o.z = fmaf(f, v[u].z, o.z); o.w = fmaf(f, v[u].w, o.w);
      }
    }
    const float inv = sum == 0.f ? 0.f : LOWERED / sum;
    const int rr = cut.tile * ROWS + r, tok = rr / p.a.group, g = rr - tok * p.a.group;
    T* const to = static_cast<T*>(p.a.o) + (int64_t)(s.first + tok) * p.a.o_row + (int64_t)(cut.head * p.a.group + g) * p.a.o_head + d;
    const T* const t = nullptr;
    if (p.a.aligned) *reinterpret_cast<uint2*>(to) = make_uint2(pack2(t, o.x * inv, o.y * inv), pack2(t, o.z * inv, o.w * inv));
    else { to[0] = from_f<T>(o.x * inv); to[1] = from_f<T>(o.y * inv); to[2] = from_f<T>(o.z * inv); to[3] = from_f<T>(o.w * inv); }
  }
}

template <typename T, int DIM, bool ALIGNED>
armor_status launch_typed(armor_ctx* c, TileP p, cudaStream_t s) {
  using L = Tile<DIM>;
  static PerDeviceOnce once;
  if (ensure_dynamic_smem(once, c->device, kv_attend_tile_kernel<T, DIM, ALIGNED>, L::SMEM) != ARMOR_OK) return ARMOR_ERR_CUDA;
  const unsigned n = (unsigned)c->n_sm;
  const int64_t part_bytes = (int64_t)L::PART * 4, need = 2 * n * part_bytes;
  p.whole = ws_scratch_bytes(c) < need;
  p.parts = c->T;
  p.cuts = reinterpret_cast<Cut*>(c->kv_cuts);
  const Batch all = p.a.b;
  for (int b0 = 0; b0 < all.n; b0 += SEQS) {
    p.a.b.n = all.n - b0 < SEQS ? all.n - b0 : SEQS;
    p.a.b.lengths = all.lengths + b0;
    p.a.b.starts = all.starts + b0;
    p.a.b.pages = all.pages + b0 * all.ld;
    launch_dependent(kv_attend_tile_kernel<T, DIM, ALIGNED>, dim3(n), dim3(THREADS), L::SMEM, s, p);
    c->launches++;
    if (!p.whole) {
      launch_dependent(kv_join_kernel<T, DIM>, dim3(n, ROWS / JOIN_ROWS), dim3(JOIN_THREADS), 0, s, p);
      c->launches++;
    }
  }
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}

template <typename T, int DIM>
armor_status launch_aligned(armor_ctx* c, const TileP& p, cudaStream_t s) {
  return p.a.aligned ? launch_typed<T, DIM, true>(c, p, s) : launch_typed<T, DIM, false>(c, p, s);
}

}  // namespace

armor_status launch_kv_attend_tile(armor_ctx* c, const KvAttend& a, int64_t limit, cudaStream_t s) {
  TileP p;
  p.a = a;
  p.limit = limit;
  p.status = c->status;
  KTimer kt(c, ARMOR_KC_FORWARD, 0.0, s);
  if (a.dtype == ARMOR_DTYPE_BF16) return a.dim == 64 ? launch_aligned<__nv_bfloat16, 64>(c, p, s) : launch_aligned<__nv_bfloat16, 128>(c, p, s);
  return a.dim == 64 ? launch_aligned<__half, 64>(c, p, s) : launch_aligned<__half, 128>(c, p, s);
}
