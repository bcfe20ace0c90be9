// What the cache's kernels and a program on the host can both ask: where the turns of a pipeline have their barriers, and in which page a position lies.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define KV_BOTH __host__ __device__ __forceinline__
#else
#define KV_BOTH inline
#endif

namespace kv {

// Turn n of a ring of `places` barriers: which of them, and the parity of its phase there.  A wait by parity tells a phase from the one before it
// and from no other, so a role may look for turn n only while the turns of the same place before the last one are known to be through, and
// while turn n + places cannot be.
KV_BOTH uint32_t ring_place(uint32_t n, uint32_t places) { return n % places; }
KV_BOTH uint32_t ring_parity(uint32_t n, uint32_t places) { return (n / places) & 1; }

// The tile kernel's rings: of units, of blocks of keys and of values, of q (upper half of a tile).
// q has two places for the warps that store keys.  They need its factor with a block and look at its barrier then; a pair of them has every second
// block, so of two units that follow each other it may have no block in one (of one block), never in both.  With a block of unit s in hand, the unit
// that it looked at last is s - 1 or s - 2, so that q of s - 2, the turn before at this place, has come (they come in order); and q of s + 2
// has not, since unit s, and with it s + 1, cannot end without the block.  With one place q of s + 1 may be there already when a pair that
// had no block in unit s looks for it, and the parity would be that of a phase to come.
constexpr int UNIT_PLACES = 4, STAGES = 4, Q_PLACES = 2;

// p / d for p < 2^31: p mul >> shift.
// (the rounded-up reciprocal: with 2^(s-1) < d <= 2^s, m = ceil(2^(31+s) / d) is at most 2^32 - 1 for d > 1 and
// exceeds 2^(31+s) / d by less than one, so that p m >> (31 + s) is p / d for all p < 2^31; d = 1: m = 2^31, s = 0)
inline void divisor(uint32_t d, uint32_t& mul, int& shift) {
  int s = 0;
  while ((1ull << s) < d) ++s;
  mul = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
  shift = 31 + s;
}
KV_BOTH uint32_t quotient(uint32_t p, uint32_t mul, int shift) { return (uint32_t)(((uint64_t)p * mul) >> shift); }

}  // namespace kv
