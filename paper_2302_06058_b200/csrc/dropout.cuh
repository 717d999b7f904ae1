// Dropout whose mask is a function of position: nothing is stored, the backward pass draws the same mask again.  Used by
// the linear-layer kernels and the residual junction.
#pragma once
#include "act_math.cuh"

namespace bimask {

// Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): a
// keyed bijection of 128-bit counters.  Eight consecutive elements of a T x C matrix are one block (C % 8 == 0: a block stays in
// its row); the block's number and the call's stream number are the counter, the seed is the key, and element k of the block
// takes 16 of the 128 bits.  Ten rounds are 20 wide multiplications and 40 additions and exclusive ors: 7 operations per
// element, which fit beside the 22 that an SM can issue while HBM moves one bf16 element in and out.
struct DropParams {
  uint32_t thr;                      // kept iff the 16 bits are at least thr; 0: no dropout
  float scale;                       // 65536 / (65536 - thr)
  uint32_t key0, key1;
  unsigned long long number;         // stream number, to which *counter is added
  const unsigned long long* counter; // device memory, or null
};

DropParams drop_params(const bimask_dropout_args* d);      // null: no dropout (residual_kernels.cu)

struct DropKey { uint32_t k0, k1, n0, n1; };

// reads *counter: only after pdl_wait()
__device__ __forceinline__ DropKey drop_key(const DropParams& d) {
  const unsigned long long n = d.number + (d.thr != 0u && d.counter != nullptr ? *d.counter : 0ull);
  return {d.key0, d.key1, (uint32_t)n, (uint32_t)(n >> 32)};
}

__device__ __forceinline__ uint4 philox(unsigned long long block, const DropKey& key) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = key.n0, c3 = key.n1, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)p1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Two elements of a block under their word of random bits: times the scale, or +0 (whatever they were).
__device__ __forceinline__ act::Pair drop_pair(act::Pair v, uint32_t bits, uint32_t thr, float scale) {
  float lo, hi;
  act::split(act::mul2(v, act::both(scale)), lo, hi);
  return act::pair((bits & 0xFFFFu) >= thr ? lo : 0.f, (bits >> 16) >= thr ? hi : 0.f);
}
__device__ __forceinline__ void drop8(act::Pair (&v)[4], unsigned long long block, const DropKey& key, uint32_t thr, float scale) {
  const uint4 r = philox(block, key);
  v[0] = drop_pair(v[0], r.x, thr, scale);
  v[1] = drop_pair(v[1], r.y, thr, scale);
  v[2] = drop_pair(v[2], r.z, thr, scale);
  v[3] = drop_pair(v[3], r.w, thr, scale);
}

}  // namespace bimask
