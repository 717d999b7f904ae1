// Dropout whose mask is a function of position: nothing is stored, the backward pass draws the same mask again.  Used by
// the linear-layer kernels and the residual junction.
#pragma once
#include "act_math.cuh"

namespace bimask {

// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): a
// keyed bijection of 128-bit counters.  Eight consecutive elements of a T x C matrix are one block (C % 8 == 0: a block stays in
// its row); the block's number and the call's stream number are the counter, the seed is the key, and element k of the block
// takes 16 of the 128 bits.  Ten rounds are 20 wide multiplications and as many three-way exclusive ors, whose key words come from
// the kernel's arguments: 5 operations per element, and 2.5 to compare and to choose (55 to 65 instructions per block, measured).
struct DropParams {
  uint32_t thr;                      // kept iff the 16 bits are at least thr / 65536 (thr has them at its upper end); 0: no dropout
  float scale;                       // 65536 / (65536 - the threshold)
  uint32_t key[20];                  // the rounds' keys, two words each
  unsigned long long number;         // stream number, to which *counter is added
  const unsigned long long* counter; // device memory, or null
};

DropParams drop_params(const bimask_dropout_args* d);      // null: no dropout (residual_kernels.cu)

// The stream number of this launch.  Reads *counter: only after pdl_wait()
__device__ __forceinline__ unsigned long long drop_number(const DropParams& d) {
  return d.number + (d.thr != 0u && d.counter != nullptr ? *d.counter : 0ull);
}

__device__ __forceinline__ uint4 philox(unsigned long long block, unsigned long long number, const DropParams& d) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)number, c3 = (uint32_t)(number >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ d.key[2 * r];
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ d.key[2 * r + 1];
    c1 = (uint32_t)p1;
    c3 = (uint32_t)p0;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Two elements of a block under their word of random bits: times the scale, or +0 (whatever they were).  The bits below the
// upper 16 do not matter to a comparison with a threshold that has none there.
__device__ __forceinline__ act::Pair drop_pair(act::Pair v, uint32_t bits, uint32_t thr, float scale) {
  float lo, hi;
  act::split(act::mul2(v, act::both(scale)), lo, hi);
  return act::pair((bits << 16) >= thr ? lo : 0.f, bits >= thr ? hi : 0.f);
}
// The multipliers of two elements: `kept` or 0.
__device__ __forceinline__ act::Pair drop_choice(uint32_t bits, uint32_t thr, float kept) {
  return act::pair((bits << 16) >= thr ? kept : 0.f, bits >= thr ? kept : 0.f);
}
__device__ __forceinline__ void drop8(act::Pair (&v)[4], const uint4& r, const DropParams& d) {
  v[0] = drop_pair(v[0], r.x, d.thr, d.scale);
  v[1] = drop_pair(v[1], r.y, d.thr, d.scale);
  v[2] = drop_pair(v[2], r.z, d.thr, d.scale);
  v[3] = drop_pair(v[3], r.w, d.thr, d.scale);
}

__device__ __forceinline__ void drop8(act::Pair (&v)[4], unsigned long long block, unsigned long long number, const DropParams& d) {
  drop8(v, philox(block, number, d), d);
}

}  // namespace bimask
