// The residual junction between two blocks of a network (norm after a block, dropout, gate, residual scale, norm before the
// next block), its gradient, and dropout alone.  All of them stream: every matrix is read once and written once, a row stays
// in the registers of the warps that share it, and its sums are exchanged by shuffles and one barrier per norm (forward) or row
// (backward).
#include "dropout.cuh"
#include "sm100_ptx.cuh"
#include <algorithm>
#include <type_traits>

namespace bimask {

namespace {

using act::Pair;

// ------------------------------------------------------------------------------------------
// Dropout alone: a flat stream of blocks of eight elements, the next items of a thread on their way.  Bound by HBM: 8192 x 16384 of
// bf16 in 90 us on the device (6.0 TB/s), the generator's wide multiplications two thirds of what their pipe can do meanwhile; 8192 x
// 8192 of fp32 in 99 us (5.4 TB/s).  More items on their way (four) and more CTAs than fit at once were no faster.
// ------------------------------------------------------------------------------------------
constexpr int DROP_THREADS = 256;

template <bool F32>
struct Vec8 {                                             // eight elements as they lie in memory
  uint4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ void unpack8(const Vec8<F32>& v, Pair (&p)[4]) {
  if constexpr (F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      p[2 * h] = act::pair(__uint_as_float(v.w[h].x), __uint_as_float(v.w[h].y));
      p[2 * h + 1] = act::pair(__uint_as_float(v.w[h].z), __uint_as_float(v.w[h].w));
    }
  } else {
    p[0] = bf16_pair(v.w[0].x); p[1] = bf16_pair(v.w[0].y); p[2] = bf16_pair(v.w[0].z); p[3] = bf16_pair(v.w[0].w);
  }
}
template <bool F32>
__device__ __forceinline__ Vec8<F32> pack8(const Pair (&p)[4]) {
  Vec8<F32> v;
  if constexpr (F32) {
    float f[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) act::split(p[k], f[2 * k], f[2 * k + 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v.w[h] = make_uint4(__float_as_uint(f[4 * h]), __float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h + 2]), __float_as_uint(f[4 * h + 3]));
  } else {
    v.w[0] = make_uint4(pack_bf16_p(p[0]), pack_bf16_p(p[1]), pack_bf16_p(p[2]), pack_bf16_p(p[3]));
  }
  return v;
}
template <bool F32>
__device__ __forceinline__ void store8(void* base, long long block, const Pair (&p)[4]) {
  const Vec8<F32> v = pack8<F32>(p);
  uint4* dst = reinterpret_cast<uint4*>(base) + block * (F32 ? 2 : 1);
#pragma unroll
  for (int h = 0; h < (F32 ? 2 : 1); ++h) dst[h] = v.w[h];
}

// A thread's item is 16 bytes: a block of bf16, half a block of fp32 (both halves draw the block's bits: with whole blocks a warp's
// instruction would touch half of each sector).
template <bool F32>
__global__ void __launch_bounds__(DROP_THREADS, 6)
dropout_kernel(const uint4* x, long long items, uint4* y /* may be x */, const __grid_constant__ DropParams d) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned long long number = drop_number(d);
  constexpr int U = 2;
  const long long step = (long long)gridDim.x * DROP_THREADS;
  long long i = (long long)blockIdx.x * DROP_THREADS + threadIdx.x;
  uint4 v[U];
  auto fetch = [&](int u, long long at) {
    if (at < items) v[u] = x[at];
  };
#pragma unroll
  for (int u = 0; u < U; ++u) fetch(u, i + u * step);
  while (i < items) {
#pragma unroll
    for (int u = 0; u < U; ++u, i += step) {
      if (i >= items) break;
      uint4 w = v[u];
      fetch(u, i + U * step);
      if (d.thr != 0u) {
        if constexpr (F32) {
          const uint4 bits = philox((unsigned long long)(i >> 1), number, d);
          float f[4];
          act::split(drop_pair(act::pair(__uint_as_float(w.x), __uint_as_float(w.y)), i & 1 ? bits.z : bits.x, d.thr, d.scale), f[0], f[1]);
          act::split(drop_pair(act::pair(__uint_as_float(w.z), __uint_as_float(w.w)), i & 1 ? bits.w : bits.y, d.thr, d.scale), f[2], f[3]);
          w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        } else {
          Pair p[4];
          unpack8<false>(Vec8<false>{w}, p);
          drop8(p, (unsigned long long)i, number, d);
          w = pack8<false>(p).w[0];
        }
      }
      y[i] = w;
    }
  }
}

// ------------------------------------------------------------------------------------------
// Rows.  A thread owns two blocks of eight columns for good; `warps` warps of a CTA, and two or four CTAs of a cluster where a CTA's are
// not enough, share a row.  A CTA holds as many such groups as its warps give; they work on rows of their own and never meet (named
// barriers).  A group takes two rows per step: what its threads exchange for both travels together, and the two rows' chains
// of dependent instructions run side by side.  The rows of the next step are already on their way: every thread copies its own
// 16-byte pieces into its own places in shared memory (cp.async), so no barrier guards them, no registers wait for them, and
// whoever writes a row in place has its old values safely fetched.
// What bounds these kernels next to HBM is the instructions they issue, so the rows' code has no branches but those of absent
// parts: columns and rows past the end are copied as zeros (from a clamped address, of which cp.async reads nothing) and work like
// the others, but for their stores.
// Why two blocks and two rows per thread: what a step costs beside its blocks is shared by four (two RMS norms and dropout, forward: 304
// instructions per block with one block and two rows per step, 245 with two and two).  8192 x 4096 with two RMS norms and dropout, back
// to back: forward 50 us (floor 41), backward 74 with the sums (floor 61).  A third stage of the ring, three CTAs per SM and parameters
// in shared memory (forward) changed nothing or cost time; so did one row per step with 24 warps in the forward pass, but for rows of
// nine to twelve warps (5120 columns 70 and 66 us).  The backward pass takes it where it pays: bwd_rows.
// ------------------------------------------------------------------------------------------
constexpr int ROWS = 2, VECS = 2, STAGES = 2;
// Threads of a CTA (one per SM).  The backward pass keeps five to eight arrays of a step in registers: 255 of them with two rows per step,
// 168 with one (see bwd_rows).
constexpr int FWD_THREADS = 512;
BIMASK_HD constexpr int bwd_threads(int rows) { return rows == 2 ? 256 : 384; }
constexpr long long CLUSTER_WAIT = 4000000000ll;          // cycles, some two seconds, that a warp waits for its row's other warps
constexpr int MAX_ROW_WARPS = 32;                         // of a cluster of two or four CTAs
static_assert(RESIDUAL_MAX_C == 8 * 32 * VECS * MAX_ROW_WARPS, "eight columns of each of a thread's blocks");

struct ResidualParams {
  uint32_t T, C8;
  int warps, cluster;                // warps per row in a CTA, CTAs per row
  int post, pre;
  float eps_post, eps_pre, alpha, inv_c;
  uint32_t gate_span;                // 0: no gate
  long long gate_pitch8;
  DropParams drop;
  const void* x;
  const uint4* y;
  const uint4* gate;
  const float* scale;
  const float* w_post;
  const float* b_post;
  const float* w_pre;
  const float* b_pre;
  void* xo;
  uint4* n;
  float2* stats_post;
  float2* stats_pre;
  // gradient
  const void* dxo;
  const uint4* dn;
  void* dx;
  uint4* dy;
  uint4* dgate;
  float* sums;                       // [clusters][wanted arrays][C]; null: one cluster takes all rows and leaves the gradients themselves
  float* gate_sums;                  // [units][C]; null: units are whole spans and leave their rows of dgate
  int want;                          // bits: SUM_* arrays that are wanted
  float* dscale;
  float* dw_post;
  float* db_post;
  float* dw_pre;
  float* db_pre;
  int has;                           // bits: HAS_* inputs that there are (others: any valid address, of which nothing is read)
  const float* weight;               // w_post or scale, whichever there is; scale_too: scale if there are both
  const float* scale_too;
  // Rows are given out in units of consecutive ones.  units_per_span: 0, or the units that a gate row's span is cut into.
  uint32_t units, unit_rows, units_per_span;
  // Rows shared by a cluster: where a wait that ran out is reported (or null), its limit, and a warp that gives up by itself (tests).
  int32_t* status;
  long long wait_cycles;
  uint32_t late;                     // 32 * warp + 8 * (number of its meeting modulo 4); above all of them: none
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or as many zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(live ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
__device__ __forceinline__ float2 read_pair(uint32_t at) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float read_word(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ float horizontal(Pair v) {
  float a, b;
  act::split(v, a, b);
  return a + b;
}
__device__ __forceinline__ Pair sum8(const Pair (&v)[4]) { return act::add2(act::add2(v[0], v[1]), act::add2(v[2], v[3])); }
__device__ __forceinline__ Pair dot8(const Pair (&v)[4], const Pair (&w)[4]) {
  return act::add2(act::fma2(v[1], w[1], act::mul2(v[0], w[0])), act::fma2(v[3], w[3], act::mul2(v[2], w[2])));
}

// both numbers times `a`, never fused with an addition that follows
__device__ __forceinline__ Pair scalar_product(Pair v, float a) {
  float lo, hi;
  act::split(v, lo, hi);
  return act::pair(__fmul_rn(lo, a), __fmul_rn(hi, a));
}
__device__ __forceinline__ uint4 read_raw(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// 0 times two bf16, added to `sum`: it stays 0 as long as they are finite, and is NaN from then on
__device__ __forceinline__ void add_nothing(uint32_t v, uint32_t& sum) { asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(v), "r"(0u)); }
// v where m is not 0, else 0
__device__ __forceinline__ Pair where_not_zero(Pair m, Pair v) {
  float m0, m1, v0, v1;
  act::split(m, m0, m1);
  act::split(v, v0, v1);
  return act::pair(m0 != 0.f ? v0 : 0.f, m1 != 0.f ? v1 : 0.f);
}
// eight fp32 parameters of block c
__device__ __forceinline__ void param8(const float* base, uint32_t c, Pair (&p)[4]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(base) + 2 * c), b = __ldg(reinterpret_cast<const float4*>(base) + 2 * c + 1);
  p[0] = act::pair(a.x, a.y); p[1] = act::pair(a.z, a.w); p[2] = act::pair(b.x, b.y); p[3] = act::pair(b.z, b.w);
}
__device__ __forceinline__ void times8(Pair (&v)[4], const Pair (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = act::mul2(v[k], w[k]);
}
__device__ __forceinline__ void plus8(Pair (&v)[4], const Pair (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = act::add2(v[k], w[k]);
}
__device__ __forceinline__ void fill8(Pair (&v)[4], float x) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = act::both(x);
}
// (v - mean) rstd, as one multiplication and addition: off by a rounding of (|v| + |mean|) rstd, like the difference first
template <bool LAYER>
__device__ __forceinline__ void normalise(Pair (&v)[4], float2 st) {
  const Pair rstd = act::both(st.y), shift = act::both(-st.x * st.y);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = LAYER ? act::fma2(v[k], rstd, shift) : act::mul2(v[k], rstd);
}

// columns that a row's warp w holds: blocks 64 w .. 64 w + 63 of the row
__device__ __forceinline__ float columns_of(int w, uint32_t C8) { return 8.f * (float)min(max((int)C8 - 32 * VECS * w, 0), 32 * VECS); }

// Exchange buffers: a group's two, of VALUES values from each of its row's warps (zeros up to a multiple of four warps).  Groups of two
// warps or more, so that four words for two warps are the worst.
template <int VALUES, int THREADS, bool CLUSTER>
struct Exchange {
  static constexpr int WORDS = CLUSTER ? MAX_ROW_WARPS : THREADS / 64 * 4;
  // a cluster's: one barrier per buffer, and a byte for each of the row's warps that is set once the warp has given up
  static constexpr int BARRIERS = 2 * VALUES * WORDS * 4, MARKS = BARRIERS + 16, BYTES = BARRIERS + (CLUSTER ? 16 + MAX_ROW_WARPS : 0);
};
// The CTAs of a cluster meet through values that are counted where they arrive.  A warp whose wait runs out gives up for good: it makes the
// row's results and those of its later rows NaN, and publishes nothing any more.  So no later meeting is ever complete, each of the
// others gives up in the next one at the latest, and no warp is ahead of another by more than one meeting: no value of a later row can
// reach a place, or count for a meeting, that a slower warp still waits for.
//
// Thread 0 of a CTA at the end of a kernel in which some warp of the cluster gave up: values that were sent in the last two meetings may
// still be on their way here.  Of the last one some warps sent none: their bytes are counted as sent, or not expected, so that its
// barrier's phase ends when all that were sent have come.  Of all warps' last meetings there are two at most, one after the other, so that
// their numbers modulo 4 tell which is later; if some warp did not give up, all have been to the very last.  own, last_own: this
// warp of the row's, and its last meeting, modulo 4.
__device__ __noinline__ void settle_meetings(uint32_t marks, uint32_t own, uint32_t last_own, uint32_t all, uint32_t even_bytes, uint32_t odd_bytes) {
  auto last = [&](uint32_t w) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(marks + w) : "memory");
    return v != 0u ? v - 1u : last_own;
  };
  uint32_t late = last(0), behind = 0;                    // the later of the last meetings, the warps that did not publish in it
  for (uint32_t w = 1; w < all; ++w)
    if (((last(w) - late) & 3u) == 1u) late = last(w);
  for (uint32_t w = 0; w < all; ++w) behind += last(w) != late;
  const uint32_t barriers = marks - 16u, at = barriers + ((late & 1u) << 3), before = (late + 3u) & 3u;
  if (behind != 0u) {
    const uint32_t bytes = late & 1u ? odd_bytes : even_bytes;
    // this thread told the barrier to expect all bytes if its warp got as far
    if (last(own) == late) ptx::mbar_complete_tx(at, behind * bytes);
    else ptx::mbar_expect_tx(at, (all - behind) * bytes);
  }
  ptx::mbar_wait_cluster(at, late >> 1, CLUSTER_WAIT);
  ptx::mbar_wait_cluster(barriers + ((before & 1u) << 3), before >> 1, CLUSTER_WAIT);        // over at once if there was none before
}

template <int VALUES, int THREADS, bool CLUSTER>
struct Group {                                            // a thread's place among those that share its rows
  int lane, group, warps;                                 // warps: of the row in this CTA
  int warp;                                               // the thread's warp, counted through the row
  bool alone;                                             // the row is one warp's
  int cluster;                                            // CTAs of the row
  int width;                                              // words of a value
  float inv_columns;                                      // 1 / columns that this warp holds
  float peer_columns[CLUSTER ? MAX_ROW_WARPS / 16 : 1];   // columns of the warps whose values a lane reads
  uint32_t buffer, flip;                                  // address of the buffer in use; buffer ^ flip: the other one
  uint32_t barrier, phase;                                // of a cluster's buffer in use; 16 * its parity
  const ResidualParams& p;

  __device__ __forceinline__ Group(const ResidualParams& params, uint32_t exchange) : p(params) {
    const int w = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    warps = p.warps;
    group = w / warps;
    cluster = p.cluster;
    warp = w - group * warps + (CLUSTER ? (int)ptx::cluster_ctarank() * warps : 0);
    alone = !CLUSTER && warps == 1;
    width = CLUSTER ? MAX_ROW_WARPS : (warps + 3) & ~3;
    inv_columns = 1.f / fmaxf(columns_of(warp, p.C8), 1.f);
    for (int k = 0; k < (CLUSTER ? MAX_ROW_WARPS / 16 : 1); ++k) peer_columns[k] = columns_of((lane & (CLUSTER ? 15 : THREADS / 32 - 1)) + 16 * k, p.C8);
    buffer = exchange + (uint32_t)((alone ? 0 : group) * 2 * VALUES * width * 4);
    flip = buffer ^ (buffer + (uint32_t)(VALUES * width * 4));
    barrier = exchange + Exchange<VALUES, THREADS, CLUSTER>::BARRIERS;
    phase = 0;
  }
  // Value i of this warp, to every CTA that shares the row ...
  __device__ __forceinline__ void publish(int i, float v) const {
    const uint32_t at = buffer + (uint32_t)((i * width + warp) * 4);
    if (!CLUSTER) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
    else
      for (int r = 0; r < cluster; ++r) ptx::st_async_u32(ptx::mapa(at, (uint32_t)r), __float_as_uint(v), ptx::mapa(barrier, (uint32_t)r));
  }
  // values: as many as every warp publishes.  A cluster's CTAs each count the bytes that arrive: the cluster's own barrier also waits for
  // the rows that were just stored (backward, 2^25 values of 8192 columns: bf16 101 us, so 89, fp32 stream 164 and 113; forward 2048 x
  // 16384 83 and 68).  Nobody is a meeting ahead: a warp's next values leave after it has all of this one's.  False, for the whole warp,
  // if they did not come in time: then it does not come here again.
  __device__ __forceinline__ bool meet(int values) {
    if (!CLUSTER) {
      ptx::named_bar_sync(group + 1, 32 * warps);
      return true;
    }
    if (threadIdx.x == 0) ptx::mbar_expect_tx(barrier, (uint32_t)(values * cluster * warps * 4));
    const bool came = (uint32_t)(warp << 5) + phase + (barrier & 8u) != p.late && ptx::mbar_wait_cluster(barrier, phase >> 4, p.wait_cycles);
    return __all_sync(0xFFFFFFFFu, came);
  }
  // After a meeting without the others: the warp's mark with every CTA, 1 more than that meeting's number modulo 4.
  __device__ __forceinline__ void give_up() const {
    if (lane != 0) return;
    for (int r = 0; r < cluster; ++r)
      asm volatile("st.shared::cluster.u8 [%0], %1;" ::"r"(ptx::mapa(marks() + (uint32_t)warp, (uint32_t)r)), "r"(((phase + (barrier & 8u)) >> 3) + 1u) : "memory");
    if (p.status != nullptr) atomicExch(p.status, (int32_t)BIMASK_ETIMEOUT);
  }
  __device__ __forceinline__ uint32_t marks() const { return (barrier & ~8u) + 16u; }
  // ... and all warps' values, after they have met.  Two buffers in turn: who writes one has met the others over the other one, and
  // by then everybody had read this one.
  __device__ __forceinline__ uint32_t published(int i, int w) const { return buffer + (uint32_t)((i * width + w) * 4); }
  __device__ __forceinline__ void turn() {
    buffer ^= flip;
    if (CLUSTER) {
      phase ^= (barrier & 8u) << 1;                       // after the second buffer
      barrier ^= 8u;
    }
  }
  // The end of a kernel whose rows are shared by a cluster: shared memory outlives the peers' writes to it.  even, odd: values that a warp
  // publishes in meetings of such a number.
  __device__ __forceinline__ void finish(bool lost, int even, int odd) const {
    if (!CLUSTER) return;
    if (lost) give_up();
    ptx::cluster_sync();
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < MAX_ROW_WARPS / 16; ++w) {
      uint4 x;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(marks() + 16u * w) : "memory");
      any |= x.x | x.y | x.z | x.w;
    }
    if (any == 0u) return;                                // the same in every CTA of the cluster
    const uint32_t meeting = (phase + (barrier & 8u)) >> 3;                               // the one that was lost, or the next
    if (threadIdx.x == 0) settle_meetings(marks(), (uint32_t)warp, lost ? meeting : (meeting + 3u) & 3u, (uint32_t)(cluster * warps), 4u * even, 4u * odd);
    ptx::cluster_sync();
  }
};

// Sums over a warp of N values at a time: at each step a lane keeps half of its values and hands the others to its partner, until
// it has one left.  The total of value i ends in the lanes i (32 / N) and on.
template <int N>
__device__ __forceinline__ float fold(float (&c)[N], int lane) {
#pragma unroll
  for (int n = N / 2, d = 16; n >= 1; n >>= 1, d >>= 1) {
    const bool hi = (lane & d) != 0;
#pragma unroll
    for (int i = 0; i < n; ++i) c[i] = (hi ? c[i + n] : c[i]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? c[i] : c[i + n], d);
  }
  float v = c[0];
#pragma unroll
  for (int d = 16 / N; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Totals over the row of N values of every thread; false if the row's other CTAs did not come.
template <int N, int THREADS, bool CLUSTER>
__device__ __forceinline__ bool row_totals(Group<N, THREADS, CLUSTER>& g, float (&c)[N]) {
  constexpr int LANES = 32 / N;                           // that share a value
  float v = fold<N>(c, g.lane);
  if (!g.alone) {
    const int i = g.lane / LANES, part = g.lane % LANES;
    if (part == 0) g.publish(i, v);
    if (!g.meet(N)) return false;
    v = 0.f;
#pragma unroll
    for (int k = 0; k < ((CLUSTER ? MAX_ROW_WARPS : THREADS / 32) + 3) / 4; k += LANES) {
      const int w = 4 * (part + k);
      if (w < g.width) {
        float4 x;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(g.published(i, w)) : "memory");
        v += (x.x + x.y) + (x.z + x.w);
      }
    }
#pragma unroll
    for (int d = LANES / 2; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    g.turn();
  }
#pragma unroll
  for (int i = 0; i < N; ++i) c[i] = __shfl_sync(0xFFFFFFFFu, v, i * LANES);
  return true;
}

// 1 / sqrt within 2^-22; of what is below 2^-126 infinity, as of 0
__device__ __forceinline__ float rsqrt_fast(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Mean and 1 / deviation of two rows (LAYER: some norm of this kernel subtracts means; `layer`: this one does).  The squares are taken
// about each warp's own mean, and the warps are put together by M = sum M_w + sum n_w (m_w - m)^2: one exchange, and no difference
// of large squares.  rms: all about zero.  Divided by the columns before they leave a thread, the squares fit fp32 at any width (up to
// 1e18: 16 squares of a difference are 6e37).  False if the rows' other CTAs did not come.
template <bool LAYER, int THREADS, bool CLUSTER>
__device__ __forceinline__ bool row_stats(const Pair (&v)[ROWS][VECS][4], const bool (&ok)[VECS], bool layer, float eps, float inv_c,
                                          Group<4, THREADS, CLUSTER>& g, float2 (&st)[ROWS]) {
  static_assert(ROWS == 2, "two rows are folded together");
  const int half = g.lane >> 4;                           // the row whose totals this lane holds
  float m = 0.f, q[ROWS];
  if (LAYER && layer) {
    float s[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) s[r] = horizontal(act::add2(sum8(v[r][0]), sum8(v[r][1])));
    m = fold<2>(s, g.lane) * g.inv_columns;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const Pair shift = act::both(-__shfl_sync(0xFFFFFFFFu, m, 16 * r));
      q[r] = 0.f;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        Pair d[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) d[k] = act::add2(v[r][j][k], shift);
        q[r] += ok[j] ? horizontal(dot8(d, d)) : 0.f;
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) q[r] = horizontal(act::add2(dot8(v[r][0], v[r][0]), dot8(v[r][1], v[r][1])));
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) q[r] *= inv_c;
  float sq = fold<2>(q, g.lane);
  if (!g.alone) {
    if ((g.lane & 15) == 0) {
      if (LAYER && layer) g.publish(half, m);
      g.publish(2 + half, sq);
    }
    if (!g.meet(LAYER && layer ? 2 * ROWS : ROWS)) return false;
    sq = 0.f;
    constexpr int EACH = CLUSTER ? MAX_ROW_WARPS / 16 : 1, SPREAD = CLUSTER ? 8 : THREADS / 64;
    float own[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int w = (g.lane & (2 * SPREAD - 1)) + 16 * k;
      own[k] = 0.f;
      if (w < g.width) {
        sq += read_word(g.published(2 + half, w));
        if (LAYER && layer) own[k] = read_word(g.published(half, w));
      }
    }
    if (LAYER && layer) {
      m = 0.f;
#pragma unroll
      for (int k = 0; k < EACH; ++k) m = fmaf(g.peer_columns[k], own[k], m);
#pragma unroll
      for (int d = SPREAD; d >= 1; d >>= 1) m += __shfl_xor_sync(0xFFFFFFFFu, m, d);
      m *= inv_c;
#pragma unroll
      for (int k = 0; k < EACH; ++k) sq = fmaf(g.peer_columns[k] * inv_c * (own[k] - m), own[k] - m, sq);
    }
#pragma unroll
    for (int d = SPREAD; d >= 1; d >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, d);
    g.turn();
  }
  const float rstd = rsqrt_fast(sq + eps);
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    st[r] = make_float2(LAYER && layer ? __shfl_sync(0xFFFFFFFFu, m, 16 * r) : 0.f, __shfl_sync(0xFFFFFFFFu, rstd, 16 * r));
  return true;
}

// A group's walk over its units, ROWS rows at a time.  SPAN: units of many rows that end with their gate row's span; else of one
// row (all others of the step are none) or ROWS.
template <int ROWS, bool SPAN>
struct Walk {
  uint32_t unit, t, end;
  __device__ __forceinline__ void enter(const ResidualParams& p) {
    if (!SPAN) {
      t = unit * p.unit_rows;
      end = min(t + p.unit_rows, p.T);
    } else {
      const uint32_t span = unit / p.units_per_span, part = unit - span * p.units_per_span;
      t = span * p.gate_span + part * p.unit_rows;
      end = min(min(t + p.unit_rows, (span + 1) * p.gate_span), p.T);
    }
  }
  __device__ __forceinline__ bool more(const ResidualParams& p) const { return unit < p.units; }
  __device__ __forceinline__ bool last() const { return t + ROWS >= end; }    // of the unit
  __device__ __forceinline__ void next(const ResidualParams& p, uint32_t stride) {
    if (!SPAN) {
      unit += stride;
      enter(p);
    } else {
      t += ROWS;
      if (t >= end) {
        unit += stride;
        if (more(p)) enter(p);
        else t = end = 0;
      }
    }
  }
};

// Shared memory of a CTA: the ring of the threads' pieces, the statistics of every warp's rows, the exchange buffers.
BIMASK_HD constexpr int pitch_of(int threads) { return threads * 16; }      // from a thread's piece to its next
BIMASK_HD constexpr int stats_stage(int rows) { return 2 * rows * 8; }                 // bytes of a warp's statistics: before, after
BIMASK_HD constexpr int stats_bytes(int rows) { return STAGES * (bwd_threads(rows) / 32) * stats_stage(rows); }
// With an fp32 stream the ring has no room for a gate's pieces: it is read from memory (L2) where it is used.
BIMASK_HD constexpr bool gate_in_ring(bool f32, bool gate) { return gate && !f32; }
BIMASK_HD constexpr int fwd_slots(bool f32, bool gate) { return (f32 ? 2 : 1) + 1 + (gate_in_ring(f32, gate) ? 1 : 0); }
BIMASK_HD constexpr int bwd_slots(bool f32, bool gate) { return (f32 ? 4 : 2) + 2 + (gate_in_ring(f32, gate) ? 1 : 0); }
// The backward pass keeps two parameters of the threads' columns beside the ring (from memory they cost it a fifth of the time with
// an fp32 stream, whose ring leaves no first-level cache); only there a cluster's largest exchange buffers leave no room.
BIMASK_HD constexpr bool bwd_keeps_params(bool f32, bool cluster, int values) { return !(f32 && cluster && values == 8); }
BIMASK_HD constexpr int param_bytes(int threads) { return 2 * VECS * 2 * pitch_of(threads); }
BIMASK_HD constexpr int bwd_values(bool post, bool wide) { return !post ? 2 : !wide ? 4 : 8; }
BIMASK_HD constexpr int stage_bytes(int rows, int threads, int slots) { return rows * VECS * slots * pitch_of(threads); }
BIMASK_HD constexpr int ring_bytes(int rows, int threads, int slots) { return STAGES * stage_bytes(rows, threads, slots); }

// A thread's blocks of a row: numbers (clamped ones for loads), and whether they exist.
struct Blocks {
  uint32_t at[VECS], safe[VECS];
  bool ok[VECS];
  __device__ __forceinline__ Blocks(int warp, int lane, uint32_t C8) {
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      at[j] = 32u * (uint32_t)(VECS * warp + j) + (uint32_t)lane;
      ok[j] = at[j] < C8;
      safe[j] = min(at[j], C8 - 1u);
    }
  }
};
// 16 bytes at `at`, and for fp32 the next 16 at `second`
template <bool F32>
__device__ __forceinline__ void read_block(uint32_t at, uint32_t second, Pair (&v)[4]) {
  Vec8<F32> raw;
#pragma unroll
  for (int h = 0; h < (F32 ? 2 : 1); ++h)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.w[h].x), "=r"(raw.w[h].y), "=r"(raw.w[h].z), "=r"(raw.w[h].w)
                 : "r"(h == 0 ? at : second) : "memory");
  unpack8<F32>(raw, v);
}
// Blocks of an fp32 stream are 32 bytes.  If every thread copied its own, an instruction would ask for half of each of 32 sectors and the
// next one for the other halves, and L2 would deliver them twice (8192 x 4096 forward and backward 100 and 150 us, so 80 and 104).  So a
// warp copies its blocks' 1024 bytes as two contiguous halves, lane l the half l % 2 of the blocks l / 2 and 16 + l / 2.  In shared
// memory a block lies in one piece, its halves swapped in every other group of four blocks: eight lanes' reads, or writes, fall into
// different banks.  Stores need no such thing: exchanged to whole sectors they cost the forward pass 10 us.
struct StreamPlace {
  uint32_t first, to, from;                               // first block to copy; offsets within a slot to copy to, to read from
  __device__ __forceinline__ StreamPlace(int warp, int lane) {
    const uint32_t b = (uint32_t)lane >> 1, h = (uint32_t)lane & 1u, base = (threadIdx.x >> 5) * 1024u;
    first = 32u * (uint32_t)(VECS * warp) + b;
    to = base + b * 32u + ((h ^ ((b >> 2) & 1u)) << 4);
    from = base + (uint32_t)lane * 32u + ((((uint32_t)lane >> 2) & 1u) << 4);
  }
};
// block j of the stream matrix of a row into a slot (`slot`: address of the slot's first byte, of thread 0)
template <bool F32>
__device__ __forceinline__ void copy_stream(uint32_t slot, const void* base, unsigned long long row, int j, bool live, const Blocks& b,
                                            const StreamPlace& s, uint32_t C8) {
  if (F32) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t block = s.first + 32u * j + 16u * i;
      copy16(slot + s.to + 512u * i, reinterpret_cast<const uint4*>(base) + (row + min(block, C8 - 1u)) * 2 + (threadIdx.x & 1u), live && block < C8);
    }
  } else {
    copy16(slot + threadIdx.x * 16u, reinterpret_cast<const uint4*>(base) + row + b.safe[j], live && b.ok[j]);
  }
}
template <bool F32>
__device__ __forceinline__ void read_stream(uint32_t slot, const StreamPlace& s, Pair (&v)[4]) {
  const uint32_t at = slot + (F32 ? s.from : threadIdx.x * 16u);
  read_block<F32>(at, at ^ 16u, v);
}
template <int VALUES, int THREADS, bool CLUSTER>
__device__ __forceinline__ void clear_exchange(float* exchange) {
  constexpr int BARRIERS = Exchange<VALUES, THREADS, CLUSTER>::BARRIERS, MARKS = Exchange<VALUES, THREADS, CLUSTER>::MARKS;
  for (int i = threadIdx.x; i < BARRIERS / 4; i += blockDim.x) exchange[i] = 0.f;
  if (CLUSTER) {
    if (threadIdx.x == 0) {
      for (int i = 0; i < MAX_ROW_WARPS / 4; ++i) exchange[MARKS / 4 + i] = 0.f;
      ptx::mbar_init(smem_addr(exchange) + BARRIERS, 1);
      ptx::mbar_init(smem_addr(exchange) + BARRIERS + 8, 1);
      ptx::fence_barrier_init();
    }
    ptx::cluster_sync();                                  // before a peer writes here, and before this CTA writes to a peer
  } else {
    __syncthreads();
  }
}

// every row's blocks times (plus) a vector of parameters, if there is one
template <bool TIMES>
__device__ __forceinline__ void affine(Pair (&v)[ROWS][VECS][4], const float* base, const Blocks& b) {
  if (base == nullptr) return;
#pragma unroll
  for (int j = 0; j < VECS; ++j) {
    Pair w[4];
    param8(base, b.safe[j], w);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (TIMES) times8(v[r][j], w);
      else plus8(v[r][j], w);
    }
  }
}
// a vector of parameters, or ones
__device__ __forceinline__ void param_or_one(const float* base, const Blocks& b, Pair (&w)[VECS][4]) {
  if (base != nullptr) {
#pragma unroll
    for (int j = 0; j < VECS; ++j) param8(base, b.safe[j], w[j]);
  } else {
#pragma unroll
    for (int j = 0; j < VECS; ++j) fill8(w[j], 1.f);
  }
}
// address of a thread's piece: slot of block j of row r
template <int SLOTS, int PITCH>
__device__ __forceinline__ uint32_t piece(uint32_t stage_at, int r, int j, int slot) { return stage_at + ((r * VECS + j) * SLOTS + slot) * PITCH; }

template <bool F32, bool GATE, bool LAYER, bool CLUSTER>
__global__ void __launch_bounds__(FWD_THREADS, 1)
residual_fwd_kernel(const __grid_constant__ ResidualParams p) {
  extern __shared__ __align__(128) float4 smem[];
  constexpr int SLOTS = fwd_slots(F32, GATE), X = 0, Y = F32 ? 2 : 1, G = Y + 1;
  constexpr bool GATE_RING = gate_in_ring(F32, GATE);
  constexpr int PITCH = pitch_of(FWD_THREADS);
  constexpr uint32_t STAGE = stage_bytes(ROWS, FWD_THREADS, SLOTS);
  float* exchange = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(smem) + ring_bytes(ROWS, FWD_THREADS, SLOTS));
  pdl_launch_dependents();
  clear_exchange<4, FWD_THREADS, CLUSTER>(exchange);
  Group<4, FWD_THREADS, CLUSTER> g(p, smem_addr(exchange));
  const Blocks b(g.warp, g.lane, p.C8);
  const StreamPlace place(g.warp, g.lane);
  const uint32_t groups = blockDim.x / (32u * (uint32_t)p.warps);
  const uint32_t stride = CLUSTER ? gridDim.x / (uint32_t)p.cluster : gridDim.x * groups;
  const uint32_t ring = smem_addr(smem) + threadIdx.x * 16u;
  Walk<ROWS, false> work, ahead;
  work.unit = CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x * groups + (uint32_t)g.group;
  work.enter(p);
  ahead = work;
  pdl_wait();
  const unsigned long long number = drop_number(p.drop);
  auto gate_row = [&](uint32_t t) { return p.gate + (long long)(p.gate_span == 1u ? t : t / p.gate_span) * p.gate_pitch8; };
  auto fetch = [&](const Walk<ROWS, false>& w, uint32_t stage) {
    const uint32_t at = ring + stage * STAGE, slot0 = smem_addr(smem) + stage * STAGE;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool live = w.more(p) && w.t + r < w.end;
      const uint32_t t = min(w.t + r, p.T - 1u);
      const unsigned long long row = (unsigned long long)t * p.C8;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        copy_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, X), p.x, row, j, live, b, place, p.C8);
        if (p.y != nullptr) copy16(piece<SLOTS, PITCH>(at, r, j, Y), p.y + row + b.safe[j], live && b.ok[j]);
        if (GATE_RING) copy16(piece<SLOTS, PITCH>(at, r, j, G), gate_row(t) + b.safe[j], live && b.ok[j]);
      }
    }
    copies_commit();
  };
  fetch(ahead, 0);
  uint32_t stage = 0;
  bool lost = false;                                      // this warp has given up
  while (work.more(p)) {
    if (F32) __syncwarp();                                // every lane has read the pieces that are overwritten now
    ahead.next(p, stride);
    fetch(ahead, stage ^ 1u);
    const uint32_t at = ring + stage * STAGE, slot0 = smem_addr(smem) + stage * STAGE;
    bool live[ROWS];
    unsigned long long row[ROWS];
    Pair v[ROWS][VECS][4];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      live[r] = work.t + r < work.end;
      row[r] = (unsigned long long)(work.t + r) * p.C8;
    }
    uint4 bits[ROWS][VECS];
    if (p.drop.thr != 0u) {                               // all blocks of the step together, so that their chains interleave, and before its
#pragma unroll                                            // rows are waited for
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) bits[r][j] = philox(row[r] + b.at[j], number, p.drop);
    }
    copies_wait<1>();
    if (F32) __syncwarp();                                // the stream's pieces are other lanes' copies
    if (p.y != nullptr) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) read_block<false>(piece<SLOTS, PITCH>(at, r, j, Y), 0, v[r][j]);
      if (p.post != BIMASK_NORM_NONE) {
        float2 st[ROWS];
        if (lost = !row_stats<LAYER>(v, b.ok, p.post == BIMASK_NORM_LAYER, p.eps_post, p.inv_c, g, st); lost) break;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          if (p.stats_post != nullptr && b.at[0] == 0 && live[r]) p.stats_post[work.t + r] = st[r];
#pragma unroll
          for (int j = 0; j < VECS; ++j) normalise<LAYER>(v[r][j], st[r]);
        }
        affine<true>(v, p.w_post, b);
        affine<false>(v, p.b_post, b);
      }
      if (p.drop.thr != 0u) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
          for (int j = 0; j < VECS; ++j) drop8(v[r][j], bits[r][j], p.drop);
      }
      if (GATE) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
          for (int j = 0; j < VECS; ++j) {
            Pair w[4];
            if (GATE_RING) read_block<false>(piece<SLOTS, PITCH>(at, r, j, G), 0, w);
            else unpack8<false>(Vec8<false>{__ldg(gate_row(min(work.t + r, p.T - 1u)) + b.safe[j])}, w);
            times8(v[r][j], w);
          }
      }
      affine<true>(v, p.scale, b);
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) fill8(v[r][j], 0.f);
    }
    // alpha x is rounded by itself: that takes off what alpha in fp32 has more or less than its decimal where alpha x has few bits, and ties
    // go to the even side.  (Fused, the excess decided all ties alike: 350 of 98304 sums of bf16 with alpha = 1.7 were rounded the wrong way.)
    // In scalar products, because ptxas fuses packed mul.rn and add.rn where it sees both; for fp32, whose pairs come as such from shared
    // memory, only where alpha is not 1.
    const bool scaled = p.alpha != 1.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        Pair x[4];
        read_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, X), place, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (!F32 || scaled) x[k] = scalar_product(x[k], p.alpha);
          v[r][j][k] = act::add2(x[k], v[r][j][k]);
        }
        if (p.xo != nullptr && live[r] && b.ok[j]) store8<F32>(p.xo, (long long)(row[r] + b.at[j]), v[r][j]);
      }
    if (p.pre != BIMASK_NORM_NONE) {
      float2 st[ROWS];
#pragma unroll
      for (int j = 0; j < VECS; ++j)
        if (!b.ok[j])                                     // whatever came of the zeros there (a bias, an infinite statistic) stays out
#pragma unroll
          for (int r = 0; r < ROWS; ++r) fill8(v[r][j], 0.f);
      if (lost = !row_stats<LAYER>(v, b.ok, p.pre == BIMASK_NORM_LAYER, p.eps_pre, p.inv_c, g, st); lost) break;
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        if (p.stats_pre != nullptr && b.at[0] == 0 && live[r]) p.stats_pre[work.t + r] = st[r];
#pragma unroll
        for (int j = 0; j < VECS; ++j) normalise<LAYER>(v[r][j], st[r]);
      }
      affine<true>(v, p.w_pre, b);
      affine<false>(v, p.b_pre, b);
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j)
          if (live[r] && b.ok[j]) store8<false>(p.n, (long long)(row[r] + b.at[j]), v[r][j]);
    }
    work.next(p, stride);
    stage ^= 1u;
  }
  copies_wait<0>();
  if (CLUSTER && lost) {                                  // the rows that are left
    Pair nan[4];
    fill8(nan, NAN);
    for (; work.more(p); work.next(p, stride))
      for (int r = 0; r < ROWS && work.t + r < work.end; ++r) {
        for (int j = 0; j < VECS; ++j) {
          const long long at = (long long)(work.t + r) * p.C8 + b.at[j];
          if (b.ok[j] && p.xo != nullptr) store8<F32>(p.xo, at, nan);
          if (b.ok[j] && p.pre != BIMASK_NORM_NONE) store8<false>(p.n, at, nan);
        }
        if (p.stats_post != nullptr && b.at[0] == 0) p.stats_post[work.t + r] = make_float2(NAN, NAN);
        if (p.stats_pre != nullptr && b.at[0] == 0) p.stats_pre[work.t + r] = make_float2(NAN, NAN);
      }
  }
  const bool both = p.post != BIMASK_NORM_NONE && p.pre != BIMASK_NORM_NONE;
  auto values = [](int norm) { return LAYER && norm == BIMASK_NORM_LAYER ? 2 * ROWS : ROWS; };
  g.finish(lost, values(both ? p.post : p.post + p.pre), values(both ? p.pre : p.post + p.pre));        // a row's norms in turn
}

// ------------------------------------------------------------------------------------------
// Gradient.  With m the dropout's multiplier, xh and yh the normalised values, r and q their 1 / deviation and w = scale w_post:
//   g = w_pre dn,  E = dx' + r g,  k1 = -r mean(g xh),  k2 = -r mean(g) [layer]
//   D = E + k1 xh + k2;   dx = alpha D;   e = m gate D;   dgate = m D (w yh + scale b_post)
//   dy = q (w e - s2 [layer] - yh s1),  s1 = mean(w e yh),  s2 = mean(w e)
// s1 and s2 seem to need D, and so k1 and k2, first; but D is linear in them: with z = w m gate yh,
//   C s1 = sum z E + k1 sum z xh + k2 sum z   (s2 likewise, without yh),
// so that all sums of a row are taken at once and its threads meet once.  The terms are those of the formula, added in another order.
// Four column sums carry every parameter's gradient: G1 = sum dn xh (w_pre), G2 = sum dn (b_pre), A = sum e yh, B = sum e:
//   dw_post = scale A,  db_post = scale B,  dscale = w_post A + b_post B.
// A thread keeps its columns' sums in registers; each cluster (CTA) leaves one row of partial sums.
// Eight warps per SM with all their registers: what bounds the pass beside HBM is the chain of a step (issue slots 45 % used at
// 8192 x 4096, RMS norms, dropout).  In steps of the build: two exchanges per row 131 us, one 101, absent parts as zeros and the step's
// random bits drawn together 91, parameters beside the ring 79, rows sent for before those 76.
// Columns and rows past the end: dx', dn, y (and m of columns) are zeros, and so is every sum.  What is absent (no norm before, dx' or y)
// is copied as zeros, too, statistics among them: then all that depends on it is zero as it should be.
// GATE: 0 no gate, 1 a gate whose gradient, if wanted, is a row per token, 2 one whose gradient is summed over spans.  WIDE: some norm
// subtracts means, or a sum other than A and G1 is wanted; without, a row has three sums to exchange instead of eight.
// ------------------------------------------------------------------------------------------
enum { SUM_A = 1, SUM_B = 2, SUM_G1 = 4, SUM_G2 = 8 };
enum { HAS_PRE = 1, HAS_DXO = 2, HAS_Y = 4, HAS_POST = 8 };

template <int ROWS, bool F32, int GATE, bool POST, bool WIDE, bool CLUSTER>
__global__ void __launch_bounds__(bwd_threads(ROWS), 1)
residual_bwd_kernel(const __grid_constant__ ResidualParams p) {
  extern __shared__ __align__(128) float4 smem[];
  constexpr int THREADS = bwd_threads(ROWS), STATS_STAGE = stats_stage(ROWS);
  constexpr int SLOTS = bwd_slots(F32, GATE != 0), XB = F32 ? 2 : 1, X = 0, DX = XB, DN = 2 * XB, Y = DN + 1, G = Y + 1;
  constexpr bool GATE_RING = gate_in_ring(F32, GATE != 0);
  constexpr int NV = bwd_values(POST, WIDE);              // a row's sums: g xh, g, z E, z xh, z, w m gate (E, xh, 1)
  constexpr int PITCH = pitch_of(THREADS);
  constexpr uint32_t STAGE = stage_bytes(ROWS, THREADS, SLOTS);
  constexpr bool KEPT = bwd_keeps_params(F32, CLUSTER, NV);
  uint8_t* const after = reinterpret_cast<uint8_t*>(smem) + ring_bytes(ROWS, THREADS, SLOTS) + (KEPT ? param_bytes(THREADS) : 0);
  float* const exchange = reinterpret_cast<float*>(after + stats_bytes(ROWS));
  pdl_launch_dependents();
  clear_exchange<ROWS * NV, THREADS, CLUSTER>(exchange);
  Group<ROWS * NV, THREADS, CLUSTER> g(p, smem_addr(exchange));
  const Blocks b(g.warp, g.lane, p.C8);
  const StreamPlace place(g.warp, g.lane);
  const uint32_t groups = blockDim.x / (32u * (uint32_t)p.warps);
  const uint32_t stride = CLUSTER ? gridDim.x / (uint32_t)p.cluster : gridDim.x * groups;
  const uint32_t ring = smem_addr(smem) + threadIdx.x * 16u;
  const uint32_t stats = smem_addr(after) + (threadIdx.x >> 5) * (STAGES * STATS_STAGE);
  Walk<ROWS, GATE == 2> work, ahead;
  work.unit = CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x * groups + (uint32_t)g.group;
  work.enter(p);
  ahead = work;
  pdl_wait();
  const unsigned long long number = drop_number(p.drop);
  const bool dropped = p.drop.thr != 0u && (p.has & HAS_Y) != 0;
  const bool layer_pre = WIDE && p.pre == BIMASK_NORM_LAYER, layer_post = WIDE && POST && p.post == BIMASK_NORM_LAYER;
  auto gate_row = [&](uint32_t t) { return p.gate + (long long)(p.gate_span == 1u ? t : t / p.gate_span) * p.gate_pitch8; };
  // A gate's block from memory.  Its gradient may take its place: per token while others still read their rows, with spans not before the
  // kernel is over (launch_residual_bwd), so that the loads may pass the stores (8192 x 4096, norm before, 124 us, so 116).
  auto gate_block = [&](uint32_t t, int j) { return GATE == 2 ? __ldg(gate_row(t) + b.safe[j]) : gate_row(t)[b.safe[j]]; };
  auto fetch = [&](const Walk<ROWS, GATE == 2>& w, uint32_t stage) {
    const bool more = w.more(p);
    const uint32_t at = ring + stage * STAGE, slot0 = smem_addr(smem) + stage * STAGE;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool live = more && w.t + r < w.end;
      const uint32_t t = min(w.t + r, p.T - 1u);
      const unsigned long long row = (unsigned long long)t * p.C8;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        const bool there = live && b.ok[j];
        const unsigned long long block = row + b.safe[j];
        copy_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, X), p.xo, row, j, live && (p.has & HAS_PRE), b, place, p.C8);
        copy16(piece<SLOTS, PITCH>(at, r, j, DN), p.dn + block, there && (p.has & HAS_PRE));
        copy_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, DX), p.dxo, row, j, live && (p.has & HAS_DXO), b, place, p.C8);
        copy16(piece<SLOTS, PITCH>(at, r, j, Y), p.y + block, there && (p.has & HAS_Y));
        if (GATE_RING) copy16(piece<SLOTS, PITCH>(at, r, j, G), gate_row(t) + b.safe[j], there);
      }
    }
    if (g.lane < 2 * ROWS) {                              // lanes 0, 1: the rows' statistics before, 2, 3: after
      const uint32_t t = w.t + (uint32_t)(g.lane % ROWS);
      const bool before = g.lane < ROWS;
      copy8(stats + stage * STATS_STAGE + g.lane * 8u, (before ? p.stats_pre : p.stats_post) + min(t, p.T - 1u),
            more && t < w.end && (p.has & (before ? HAS_PRE : HAS_POST)));
    }
    copies_commit();
  };
  Pair sum_a[VECS][4], sum_g1[VECS][4], sum_b[VECS][4], sum_g2[VECS][4], fsum[VECS][4];
#pragma unroll
  for (int j = 0; j < VECS; ++j) {
    fill8(sum_a[j], 0.f);
    fill8(sum_g1[j], 0.f);
    fill8(sum_b[j], 0.f);
    fill8(sum_g2[j], 0.f);
    fill8(fsum[j], 0.f);
  }
  auto leave_unit = [&]() {
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      if (!b.ok[j]) continue;
      if (p.gate_sums != nullptr) store8<true>(p.gate_sums, (long long)work.unit * p.C8 + b.at[j], fsum[j]);
      else store8<false>(p.dgate, (long long)work.unit * p.gate_pitch8 + b.at[j], fsum[j]);
    }
  };
  fetch(ahead, 0);
  // the parameters of this thread's columns, w_pre and scale w_post: from its own pieces after the ring, or from memory
  const uint32_t kept = ring + ring_bytes(ROWS, THREADS, SLOTS);
  auto weights = [&](Pair (&w)[VECS][4]) {
    param_or_one(p.weight, b, w);
    if (POST && p.scale_too != nullptr) {
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        Pair s[4];
        param8(p.scale_too, b.safe[j], s);
        times8(w[j], s);
      }
    }
  };
  auto params = [&](int which, Pair (&w)[VECS][4]) {
    if (KEPT) {
#pragma unroll
      for (int j = 0; j < VECS; ++j) read_block<true>(kept + (uint32_t)(which * VECS + j) * 2 * PITCH, kept + ((uint32_t)(which * VECS + j) * 2 + 1) * PITCH, w[j]);
    } else if (which == 0) {
      param_or_one(p.w_pre, b, w);
    } else {
      weights(w);
    }
  };
  if (KEPT) {
    uint4* mine = reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(smem) + ring_bytes(ROWS, THREADS, SLOTS)) + threadIdx.x;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      Pair w[VECS][4];
      if (which == 0) param_or_one(p.w_pre, b, w);
      else weights(w);
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        const Vec8<true> v = pack8<true>(w[j]);
        mine[(which * VECS + j) * 2 * THREADS] = v.w[0];
        mine[((which * VECS + j) * 2 + 1) * THREADS] = v.w[1];
      }
    }
  }
  uint32_t stage = 0;
  bool lost = false;                                      // this warp has given up
  while (work.more(p)) {
    __syncwarp();                                         // every lane has read the statistics and pieces that are overwritten now
    ahead.next(p, stride);
    fetch(ahead, stage ^ 1u);
    copies_wait<1>();
    __syncwarp();                                         // the statistics, and pieces of an fp32 stream, are other lanes' copies
    const uint32_t at = ring + stage * STAGE, slot0 = smem_addr(smem) + stage * STAGE, st_at = stats + stage * STATS_STAGE;
    bool live[ROWS];
    unsigned long long row[ROWS];
    Pair E[ROWS][VECS][4], xh[ROWS][VECS][4], yh[ROWS][VECS][4], m[ROWS][VECS][4];
    float c[ROWS * NV], r_pre[ROWS], r_post[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      live[r] = work.t + r < work.end;
      row[r] = (unsigned long long)(work.t + r) * p.C8;
    }
    if (p.drop.thr != 0u) {                               // all blocks of the step together: their chains interleave
      uint4 bits[ROWS][VECS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) bits[r][j] = philox(row[r] + b.at[j], number, p.drop);
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
          const float scale = b.ok[j] ? p.drop.scale : 0.f;       // nothing past the end in the sums with z
          m[r][j][0] = drop_choice(bits[r][j].x, p.drop.thr, scale);
          m[r][j][1] = drop_choice(bits[r][j].y, p.drop.thr, scale);
          m[r][j][2] = drop_choice(bits[r][j].z, p.drop.thr, scale);
          m[r][j][3] = drop_choice(bits[r][j].w, p.drop.thr, scale);
        }
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j) fill8(m[r][j], b.ok[j] ? 1.f : 0.f);
    }
    uint32_t odd = 0;                                     // not 0 if a value of y is not finite
    Pair w_pre[VECS][4], w[VECS][4];
    params(0, w_pre);
    params(1, w);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float2 st = read_pair(st_at + 8 * r);
      r_pre[r] = st.y;
      const Pair rs = act::both(st.y);
      Pair s = act::both(0.f), s0 = s;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        Pair gr[4];
        read_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, DX), place, E[r][j]);
        read_stream<F32>(slot0 + piece<SLOTS, PITCH>(0, r, j, X), place, xh[r][j]);
        read_block<false>(piece<SLOTS, PITCH>(at, r, j, DN), 0, gr);
        normalise<WIDE>(xh[r][j], st);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum_g1[j][k] = act::fma2(gr[k], xh[r][j][k], sum_g1[j][k]);
        if (WIDE) plus8(sum_g2[j], gr);
        times8(gr, w_pre[j]);
#pragma unroll
        for (int k = 0; k < 4; ++k) s = act::fma2(gr[k], xh[r][j][k], s);
        if (WIDE) s0 = act::add2(s0, sum8(gr));
#pragma unroll
        for (int k = 0; k < 4; ++k) E[r][j][k] = act::fma2(gr[k], rs, E[r][j][k]);
      }
      c[r * NV] = horizontal(s);
      c[r * NV + 1] = WIDE && layer_pre ? horizontal(s0) : 0.f;
      float2 sq = make_float2(0.f, 1.f);
      if (POST) sq = read_pair(st_at + 8 * (ROWS + r));
      r_post[r] = sq.y;
      Pair ze = act::both(0.f), zx = ze, z0 = ze, te = ze, tx = ze, t0 = ze;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        const uint4 raw = read_raw(piece<SLOTS, PITCH>(at, r, j, Y));
        unpack8<false>(Vec8<false>{raw}, yh[r][j]);
        if (!POST && dropped) {
          add_nothing(raw.x, odd);
          add_nothing(raw.y, odd);
          add_nothing(raw.z, odd);
          add_nothing(raw.w, odd);
        }
        if (POST) {
          normalise<WIDE>(yh[r][j], sq);
          Pair z[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) z[k] = act::mul2(m[r][j][k], w[j][k]);
          if (GATE != 0) {
            Pair gt[4];
            if (GATE_RING) read_block<false>(piece<SLOTS, PITCH>(at, r, j, G), 0, gt);
            else unpack8<false>(Vec8<false>{gate_block(min(work.t + r, p.T - 1u), j)}, gt);
            times8(z, gt);
          }
          if (WIDE) {
#pragma unroll
            for (int k = 0; k < 4; ++k) te = act::fma2(z[k], E[r][j][k], te), tx = act::fma2(z[k], xh[r][j][k], tx);
            t0 = act::add2(t0, sum8(z));
          }
          times8(z, yh[r][j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) ze = act::fma2(z[k], E[r][j][k], ze), zx = act::fma2(z[k], xh[r][j][k], zx);
          if (WIDE) z0 = act::add2(z0, sum8(z));
        }
      }
      if (POST) {
        c[r * NV + 2] = horizontal(ze);
        c[r * NV + 3] = horizontal(zx);
        if (WIDE) {
          c[r * NV + 4] = horizontal(z0);
          c[r * NV + 5] = layer_post ? horizontal(te) : 0.f;
          c[r * NV + 6] = layer_post ? horizontal(tx) : 0.f;
          c[r * NV + 7] = layer_post ? horizontal(t0) : 0.f;
        }
      }
    }
    // What was dropped is 0 in the gradients of gate and scale, too, whatever it was.  0 times it will do as long as it is finite (behind a
    // norm it is); looking whether it is costs 1 to 5 % of the time (a choice for every value 3 to 10; 12608 x 384 and a gate row per 197
    // tokens, bf16: 22.1 us, now 22.7), and up to 27 % where registers were short already: an fp32 stream with a gate that serves spans
    // and a layer norm (43690 x 768: 152 us, now 194).  Looking in the ring, before the step's registers are in use, was no better.
    if (!POST && dropped && odd != 0u) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) yh[r][j][k] = where_not_zero(m[r][j][k], yh[r][j][k]);
    }
    if (lost = !row_totals(g, c); lost) break;
    const Pair alpha = act::both(p.alpha);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float scaled = -r_pre[r] * p.inv_c, f1 = c[r * NV] * scaled, f2 = WIDE ? c[r * NV + 1] * scaled : 0.f;
      float s1 = 0.f, s2 = 0.f;
      if (POST) {
        const float scaled_post = -r_post[r] * p.inv_c;
        s1 = c[r * NV + 2] + f1 * c[r * NV + 3];
        if (WIDE) {
          s1 += f2 * c[r * NV + 4];
          s2 = (c[r * NV + 5] + f1 * c[r * NV + 6] + f2 * c[r * NV + 7]) * scaled_post;
        }
        s1 *= scaled_post;
      }
      const Pair k1 = act::both(f1), k2 = act::both(f2), q1 = act::both(s1), q2 = act::both(s2), rs = act::both(r_post[r]);
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        const bool there = live[r] && b.ok[j];
#pragma unroll
        for (int k = 0; k < 4; ++k) E[r][j][k] = act::fma2(xh[r][j][k], k1, WIDE ? act::add2(E[r][j][k], k2) : E[r][j][k]);      // D
        Pair o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = act::mul2(E[r][j][k], alpha);
        if (p.dx != nullptr && there) store8<F32>(p.dx, (long long)(row[r] + b.at[j]), o);
        times8(E[r][j], m[r][j]);
        if (GATE != 0) {
          Pair gt[4];
          auto read_gate = [&]() {
            if (GATE_RING) read_block<false>(piece<SLOTS, PITCH>(at, r, j, G), 0, gt);
            else unpack8<false>(Vec8<false>{gate_block(min(work.t + r, p.T - 1u), j)}, gt);
          };
          constexpr bool EARLY = !GATE_RING && GATE == 1;  // from memory, where its gradient may take its place
          if (EARLY) read_gate();
          if (GATE == 2 || p.dgate != nullptr) {          // scale u
            Pair u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = act::mul2(yh[r][j][k], w[j][k]);
            if (POST && p.b_post != nullptr) {
              Pair bias[4];
              param8(p.b_post, b.safe[j], bias);
              if (p.scale != nullptr) {
                Pair s[4];
                param8(p.scale, b.safe[j], s);
                times8(bias, s);
              }
              plus8(u, bias);
            }
            if (GATE == 2) {
#pragma unroll
              for (int k = 0; k < 4; ++k) fsum[j][k] = act::fma2(E[r][j][k], u[k], fsum[j][k]);
            } else {
              times8(u, E[r][j]);
              if (there) store8<false>(p.dgate, (long long)(work.t + r) * p.gate_pitch8 + b.at[j], u);
            }
          }
          if (!EARLY) read_gate();
          times8(E[r][j], gt);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) sum_a[j][k] = act::fma2(E[r][j][k], yh[r][j][k], sum_a[j][k]);
        if (POST && WIDE) plus8(sum_b[j], E[r][j]);
        times8(E[r][j], w[j]);
        if (POST) {
#pragma unroll
          for (int k = 0; k < 4; ++k) E[r][j][k] = act::fma2(E[r][j][k], rs, WIDE ? act::fma2(yh[r][j][k], q1, q2) : act::mul2(yh[r][j][k], q1));
        }
        if (there && p.dy != nullptr) store8<false>(p.dy, (long long)(row[r] + b.at[j]), E[r][j]);
      }
    }
    if (GATE == 2 && work.last()) {
      leave_unit();
#pragma unroll
      for (int j = 0; j < VECS; ++j) fill8(fsum[j], 0.f);
    }
    work.next(p, stride);
    stage ^= 1u;
  }
  copies_wait<0>();
  if (CLUSTER && lost) {                                  // the rows that are left
    Pair nan[4];
    fill8(nan, NAN);
    for (int j = 0; j < VECS; ++j) {
      fill8(sum_a[j], NAN);
      fill8(sum_g1[j], NAN);
      fill8(sum_b[j], NAN);
      fill8(sum_g2[j], NAN);
      fill8(fsum[j], NAN);
    }
    for (; work.more(p); work.next(p, stride)) {
      for (int r = 0; r < ROWS && work.t + r < work.end; ++r)
        for (int j = 0; j < VECS; ++j) {
          const long long at = (long long)(work.t + r) * p.C8 + b.at[j];
          if (b.ok[j] && p.dx != nullptr) store8<F32>(p.dx, at, nan);
          if (b.ok[j] && p.dy != nullptr) store8<false>(p.dy, at, nan);
          if (GATE == 1 && b.ok[j] && p.dgate != nullptr) store8<false>(p.dgate, (long long)(work.t + r) * p.gate_pitch8 + b.at[j], nan);
        }
      if (GATE == 2 && work.last()) leave_unit();
    }
  }
  // The groups' sums are added through the ring, in their order.
  int slot = 0;
  auto leave = [&](int which, Pair (&sum)[VECS][4]) {
    if (!(p.want & which)) return;                        // the same for every thread
    if (groups > 1) {
      __syncthreads();
      uint4* mine = reinterpret_cast<uint4*>(smem) + threadIdx.x;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        const Vec8<true> v = pack8<true>(sum[j]);
        mine[2 * j * THREADS] = v.w[0];
        mine[(2 * j + 1) * THREADS] = v.w[1];
      }
      __syncthreads();
    }
    if (g.group == 0) {
      float* const out = p.sums + ((size_t)(CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x) * __popc(p.want) + slot) * p.C8 * 8;
#pragma unroll
      for (int j = 0; j < VECS; ++j) {
        for (uint32_t o = 1; o < groups; ++o) {
          Pair q[4];
          read_block<true>(ring + o * (uint32_t)p.warps * 512u + 2 * j * PITCH, ring + o * (uint32_t)p.warps * 512u + (2 * j + 1) * PITCH, q);
          plus8(sum[j], q);
        }
        if (b.ok[j] && p.sums != nullptr) store8<true>(out, b.at[j], sum[j]);
      }
    }
    ++slot;
  };
  leave(SUM_A, sum_a);
  if (POST && WIDE) leave(SUM_B, sum_b);
  leave(SUM_G1, sum_g1);
  if (WIDE) leave(SUM_G2, sum_g2);
  if (p.sums == nullptr && p.want != 0 && g.group == 0) { // what residual_reduce_kernel makes of the sums
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
      if (!b.ok[j]) continue;
      const uint32_t at = b.at[j];
      if (p.dw_pre != nullptr) store8<true>(p.dw_pre, at, sum_g1[j]);
      if (WIDE && p.db_pre != nullptr) store8<true>(p.db_pre, at, sum_g2[j]);
      Pair s[4], o[4];
      fill8(s, 1.f);
      if (p.scale != nullptr) param8(p.scale, at, s);
      auto scaled = [&](const Pair (&sum)[4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = act::mul2(sum[k], s[k]);
      };
      if (p.dw_post != nullptr) { scaled(sum_a[j]); store8<true>(p.dw_post, at, o); }
      if (WIDE && p.db_post != nullptr) { scaled(sum_b[j]); store8<true>(p.db_post, at, o); }
      if (p.dscale != nullptr) {
        fill8(s, 1.f);
        if (POST && p.w_post != nullptr) param8(p.w_post, at, s);
        scaled(sum_a[j]);
        if (POST && WIDE && p.b_post != nullptr) {
          param8(p.b_post, at, s);
          times8(s, sum_b[j]);
          plus8(o, s);
        }
        store8<true>(p.dscale, at, o);
      }
    }
  }
  g.finish(lost, ROWS * NV, ROWS * NV);
}

// What is left to add up, in one launch.  blockIdx.y below the number of wanted arrays: that array's gradients from the clusters'
// partial sums; a CTA covers eight float4 columns, its 32 row slots take the partial rows in turn and are added through shared memory,
// in a fixed order (A carries dscale with it, and B where dscale has a part from there).  blockIdx.y above: a row of dgate from its
// units, the same way.
struct ResidualReduce {
  const float4* sums;
  int slots, want, C4;
  const float4 *scale, *w_post, *b_post;
  float4 *dscale, *dw_post, *db_post, *dw_pre, *db_pre;
  const float4* gate_sums;
  int units_per_span;
  uint2* dgate;
  long long gate_pitch4, gates;
};
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }

__global__ void __launch_bounds__(256)
residual_reduce_kernel(const __grid_constant__ ResidualReduce p) {
  __shared__ float4 red[2][32][8];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 7, slot = threadIdx.x >> 3;
  const int e = blockIdx.x * 8 + lane, arrays = __popc(p.want);
  pdl_wait();
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  // the sum over `rows` rows of `src`, `step` apart, and over those of its neighbour, in the threads of slot 0
  auto total = [&](const float4* src, int rows, size_t step, bool both, size_t neighbour, float4 (&acc)[2]) {
    acc[0] = acc[1] = zero;
    if (e < p.C4) {
#pragma unroll 5
      for (int s = slot; s < rows; s += 32) {
        acc[0] = add4(acc[0], src[s * step]);
        if (both) acc[1] = add4(acc[1], src[s * step + neighbour]);
      }
    }
    red[0][slot][lane] = acc[0];
    red[1][slot][lane] = acc[1];
    __syncthreads();
#pragma unroll
    for (int half = 16; half >= 1; half >>= 1) {
      if (slot < half) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          acc[i] = add4(acc[i], red[i][slot + half][lane]);
          red[i][slot][lane] = acc[i];
        }
      }
      __syncthreads();
    }
  };
  float4 acc[2];
  if ((int)blockIdx.y >= arrays) {
    const long long stride = gridDim.y - arrays;
    for (long long row = (int)blockIdx.y - arrays; row < p.gates; row += stride) {
      total(p.gate_sums + (size_t)row * p.units_per_span * p.C4 + e, p.units_per_span, p.C4, false, 0, acc);
      if (slot == 0 && e < p.C4) p.dgate[row * p.gate_pitch4 + e] = make_uint2(pack_bf16_f(acc[0].x, acc[0].y), pack_bf16_f(acc[0].z, acc[0].w));
    }
    return;
  }
  int which = p.want;                                     // its bit number blockIdx.y
  for (unsigned k = 0; k < blockIdx.y; ++k) which &= which - 1;
  which &= -which;
  const bool both = which == SUM_A && p.dscale != nullptr && p.b_post != nullptr;        // then B comes next after A
  total(p.sums + (size_t)blockIdx.y * p.C4 + e, p.slots, (size_t)arrays * p.C4, both, p.C4, acc);
  if (slot != 0 || e >= p.C4) return;
  const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
  const float4 s = p.scale != nullptr ? __ldg(p.scale + e) : one;
  if (which == SUM_A) {
    if (p.dw_post != nullptr) p.dw_post[e] = mul4(s, acc[0]);
    if (p.dscale != nullptr) {
      float4 d = mul4(p.w_post != nullptr ? __ldg(p.w_post + e) : one, acc[0]);
      if (both) d = add4(d, mul4(__ldg(p.b_post + e), acc[1]));
      p.dscale[e] = d;
    }
  } else if (which == SUM_B) {
    if (p.db_post != nullptr) p.db_post[e] = mul4(s, acc[0]);
  } else if (which == SUM_G1) {
    p.dw_pre[e] = acc[0];
  } else {
    p.db_pre[e] = acc[0];
  }
}

// ---- plans --------------------------------------------------------------------------------------
struct RowPlan {
  int cluster, warps, groups, threads;                    // CTAs that share a row, its warps in each, rows side by side
  int slots;                                              // clusters (CTAs) of the grid
  long long units, gates;
  int unit_rows, units_per_span;
};

// one_slot: a few rows go to one cluster (two steps cost less than a launch that adds up what several leave).
// ctas: how many the card holds.  span > 1: units end where a gate row's span ends.
RowPlan plan_rows(int rows, int threads, int T, int C, int span, int ctas, bool one_slot = false) {
  RowPlan b = {};
  const int all = (C / 8 + 32 * VECS - 1) / (32 * VECS), most = threads / 32;             // warps of a row, of a CTA
  b.cluster = all > 2 * most ? 4 : all > most ? 2 : 1;
  b.warps = (all + b.cluster - 1) / b.cluster;
  b.groups = threads / 32 / b.warps;
  b.threads = 32 * b.warps * b.groups;
  // Clusters that run at once: of four CTAs 33 on a B200, whose parts hold no multiple of four SMs (with 37 the last four ran by
  // themselves, 2048 x 16384 in 178 us)
  const int clusters = b.cluster == 4 ? ctas * 32 / 148 : ctas / b.cluster;
  const bool few = one_slot && T <= 2 * rows * b.groups;
  const long long room = (long long)(few ? 1 : clusters) * b.groups;
  if (span > 1) {
    const int len = span < T ? span : T;
    b.gates = (T + (long long)span - 1) / span;
    // Fewer rows than groups: one each, but spans of two steps whole (nothing is left to add up then, a launch of 2 us).  Else the units
    // per span whose rounds over the groups take the fewest steps, among the largest number that makes one round or two, and one to
    // four; two steps more for any but one.  (43690 x 768 with spans of 197: three units each, of rows / groups, made 1.1 rounds and 187
    // us; five of 40 rows make two in 118.)
    long long best = 0;
    b.unit_rows = len <= 2 * rows ? len : 1;
    for (int k = 0; k < 6 && T > room; ++k) {
      const long long most_units = (k - 3) * room / b.gates, want = k < 4 ? k + 1 : most_units < len ? most_units : len;
      if (want < 1 || want > len || (want > 1 && want * b.gates > 2 * room + b.gates)) continue;
      const long long unit = ((len + want - 1) / want + rows - 1) / rows * rows, each = (len + unit - 1) / unit;
      const long long steps = (b.gates * each + room - 1) / room * (unit / rows) + (each > 1 ? 2 : 0);
      if (best == 0 || steps < best) {
        best = steps;
        b.unit_rows = each > 1 ? (int)unit : len;
      }
    }
    b.units_per_span = (len + b.unit_rows - 1) / b.unit_rows;
    b.units = b.gates * b.units_per_span;
  } else {
    b.unit_rows = T > room ? rows : 1;                    // fewer rows than groups: one each
    b.units = ((long long)T + b.unit_rows - 1) / b.unit_rows;
  }
  const long long slots = (b.units + b.groups - 1) / b.groups;
  b.slots = (int)(slots < clusters ? slots : clusters);
  if (few) b.slots = 1;
  return b;
}

// Rows per step of the backward pass: two with eight warps per SM, or one with twelve.  One hides less latency per warp and pays for an
// exchange per row, so it is taken where it keeps twice the warps busy or needs no cluster: rows of three, five or six warps (bf16,
// 2^25 values, RMS norms both sides and dropout: 1152 columns 114 -> 93 us, 1536 91 -> 77, 2560 105 -> 91; but 4096 81 -> 95), and of
// nine to twelve (5120 columns 122 -> 94, fp32 stream with a layer norm before 196 -> 148).  A gate per token next to a layer norm leaves
// two rows too few of 255 registers, one row enough of 168 (1024 columns 116 -> 98, 4096 132 -> 104).  Not with a norm after and means:
// eight values per row, of which 168 registers spill (5120 columns 130 -> 145); nor for short rows of an fp32 stream with means and no
// gate (1152 columns 118 -> 133).  Which gradients are wanted plays no part: one alone is added up as it is among the others.  So RMS norms
// with biases, whose gradients need the eight values, too, go by their widths like those without.  With a gate that is the faster side
// (two rows and one, gate per token 2560 columns 221 -> 192, 6144 179 -> 175; per 197 tokens 282 -> 232, 245 -> 207), without one it is up to
// 2560 columns (144 -> 139; fp32 stream 174 -> 179), not above (5120 136 -> 148, 6144 118 -> 139).
int bwd_rows(const bimask_residual_args& a) {
  const int all = (a.C / 8 + 32 * VECS - 1) / (32 * VECS);
  const bool f32 = a.stream_type == BIMASK_TYPE_F32, means = a.post == BIMASK_NORM_LAYER || a.pre == BIMASK_NORM_LAYER;
  if (a.post != BIMASK_NORM_NONE && means) return 2;
  if (all > bwd_threads(2) / 32) return all <= bwd_threads(1) / 32 ? 1 : 2;
  if (a.gate != nullptr && a.gate_span == 1 && means && !f32) return 1;
  return (all == 3 || all == 5 || all == 6) && !(f32 && means && a.gate == nullptr) ? 1 : 2;
}

template <typename K>
int launch_rows(K kernel, const RowPlan& b, int bytes, cudaStream_t s, const ResidualParams& p) {
  const int rc = set_smem_attr<256>(kernel, bytes);        // of one type: 16 kernels forward, up to 72 backward
  if (rc != BIMASK_OK) return rc;
  if (b.cluster == 1) BIMASK_CUDA_OK(launch_pdl(kernel, (unsigned)b.slots, b.threads, (size_t)bytes, s, p));
  else BIMASK_CUDA_OK(launch_pdl_cluster(kernel, (unsigned)(b.slots * b.cluster), b.threads, b.cluster, (size_t)bytes, s, p));
  count_launch();
  return BIMASK_OK;
}

void take_plan(ResidualParams& p, const RowPlan& b) {
  p.warps = b.warps;
  p.cluster = b.cluster;
  p.units = (uint32_t)b.units;
  p.unit_rows = (uint32_t)b.unit_rows;
  p.units_per_span = (uint32_t)b.units_per_span;
}

}  // namespace

static size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Scratch of the backward pass: the clusters' partial sums (four arrays at most), then the units' of a spanned gate, each for T
// tokens and every smaller number.  With spans there are at most 2 T units (a last span that is not full has its empty ones),
// and at most two per group of warps and one more per gate row.
// Either number of rows per step: the query does not know the norms.
static size_t column_sums_bytes(int T, int C, int span) {
  size_t bytes = 0;
  for (int rows = 1; rows <= 2; ++rows) {
    const RowPlan b = plan_rows(rows, bwd_threads(rows), 1, C, 1, PLAN_SMS);
    const long long most = PLAN_SMS / b.cluster, slots = ((span > 1 ? 2ll : 1ll) * T + b.groups - 1) / b.groups;
    bytes = std::max(bytes, up256((size_t)(slots < most ? slots : most) * 4 * C * sizeof(float)));
  }
  return bytes;
}
size_t residual_workspace_bytes(int T, int C, int span) {
  size_t bytes = column_sums_bytes(T, C, span);
  if (span > 1) {
    const long long gates = (T + (long long)span - 1) / span;
    long long units = 0;
    for (int rows = 1; rows <= 2; ++rows) {
      const RowPlan b = plan_rows(rows, bwd_threads(rows), 1, C, 1, PLAN_SMS);
      units = std::max(units, 2ll * (PLAN_SMS / b.cluster) * b.groups + gates);
    }
    bytes += (size_t)(units < 2ll * T ? units : 2ll * T) * C * sizeof(float);
  }
  return bytes;
}

DropParams drop_params(const bimask_dropout_args* d) {
  DropParams p = {};
  p.scale = 1.f;
  if (d == nullptr) return p;
  const uint32_t thr = drop_threshold(d->p);
  p.thr = thr << 16;
  p.scale = (float)(65536.0 / (65536.0 - thr));
  for (int r = 0; r < 10; ++r) {
    p.key[2 * r] = (uint32_t)d->seed + 0x9E3779B9u * r;
    p.key[2 * r + 1] = (uint32_t)(d->seed >> 32) + 0xBB67AE85u * r;
  }
  p.number = d->stream_no;
  p.counter = reinterpret_cast<const unsigned long long*>(d->counter);
  return p;
}

int launch_dropout(const void* x, int type, int T, int C, const bimask_dropout_args& d, void* y, cudaStream_t s) {
  const long long items = (long long)T * (C / (type == BIMASK_TYPE_F32 ? 4 : 8));
  const long long ctas = (items + DROP_THREADS - 1) / DROP_THREADS, most = 6ll * sm_count();
  auto run = [&](auto kern) {
    return launch_pdl(kern, (unsigned)(ctas < most ? ctas : most), DROP_THREADS, 0, s, reinterpret_cast<const uint4*>(x), items,
                      reinterpret_cast<uint4*>(y), drop_params(&d));
  };
  BIMASK_CUDA_OK(type == BIMASK_TYPE_F32 ? run(dropout_kernel<true>) : run(dropout_kernel<false>));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

static ResidualParams residual_params(const bimask_residual_args& a, const ResidualGiveUp* give_up) {
  ResidualParams p = {};
  p.status = a.status_word;
  p.wait_cycles = give_up != nullptr ? give_up->limit_cycles : CLUSTER_WAIT;
  p.late = give_up != nullptr && give_up->late_warp >= 0 ? 32u * give_up->late_warp + 8u * give_up->late_meeting : 0xFFFFFFFFu;
  p.T = (uint32_t)a.T;
  p.C8 = (uint32_t)a.C / 8;
  p.post = a.post;
  p.pre = a.pre;
  p.eps_post = a.eps_post;
  p.eps_pre = a.eps_pre;
  p.alpha = a.alpha;
  p.inv_c = 1.f / (float)a.C;
  p.gate_span = a.gate != nullptr ? (uint32_t)a.gate_span : 0u;
  p.gate_pitch8 = a.gate_pitch / 8;
  p.drop = drop_params(&a.drop);
  p.x = a.x;
  p.y = reinterpret_cast<const uint4*>(a.y);
  p.gate = reinterpret_cast<const uint4*>(a.gate);
  p.scale = a.scale;
  p.w_post = a.w_post;
  p.b_post = a.b_post;
  p.w_pre = a.w_pre;
  p.b_pre = a.b_pre;
  p.xo = a.xo;
  p.n = reinterpret_cast<uint4*>(a.n);
  p.stats_post = reinterpret_cast<float2*>(a.stats_post);
  p.stats_pre = reinterpret_cast<float2*>(a.stats_pre);
  p.dxo = a.dxo;
  p.dn = reinterpret_cast<const uint4*>(a.dn);
  p.dx = a.dx;
  p.dy = reinterpret_cast<uint4*>(a.dy);
  p.dgate = reinterpret_cast<uint4*>(a.dgate);
  return p;
}

int launch_residual_fwd(const bimask_residual_args& a, cudaStream_t s, const ResidualGiveUp* give_up) {
  ResidualParams p = residual_params(a, give_up);
  const RowPlan b = plan_rows(ROWS, FWD_THREADS, a.T, a.C, 1, sm_count());
  take_plan(p, b);
  using Yes = std::true_type;
  using No = std::false_type;
  auto run = [&](auto f32, auto gate, auto layer, auto cluster) -> int {
    constexpr bool F = decltype(f32)::value, G = decltype(gate)::value, L = decltype(layer)::value, K = decltype(cluster)::value;
    return launch_rows(residual_fwd_kernel<F, G, L, K>, b, ring_bytes(ROWS, FWD_THREADS, fwd_slots(F, G)) + Exchange<4, FWD_THREADS, K>::BYTES, s, p);
  };
  const bool means = p.post == BIMASK_NORM_LAYER || p.pre == BIMASK_NORM_LAYER;
  auto pick = [&](auto f32, auto gate) -> int {
    if (b.cluster > 1) return means ? run(f32, gate, Yes(), Yes()) : run(f32, gate, No(), Yes());
    return means ? run(f32, gate, Yes(), No()) : run(f32, gate, No(), No());
  };
  const bool gate = p.gate_span != 0;
  const int rc = a.stream_type == BIMASK_TYPE_F32 ? (gate ? pick(Yes(), Yes()) : pick(Yes(), No())) : (gate ? pick(No(), Yes()) : pick(No(), No()));
  if (rc != BIMASK_OK) return rc;
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_residual_bwd(const bimask_residual_args& a, cudaStream_t s, const ResidualGiveUp* give_up) {
  ResidualParams p = residual_params(a, give_up);
  const bool spanned = a.dgate != nullptr && p.gate_span > 1;
  const bool branch = a.dy || a.dgate || a.dscale || a.dw_post || a.db_post, post = branch && a.post != BIMASK_NORM_NONE;
  p.has = (a.pre != BIMASK_NORM_NONE ? HAS_PRE : 0) | (a.dxo ? HAS_DXO : 0) | (branch && a.y ? HAS_Y : 0) | (post ? HAS_POST : 0);
  const void* some = p.has & HAS_PRE ? a.xo : a.dxo;       // one of the two is there
  if (!(p.has & HAS_PRE)) { p.xo = const_cast<void*>(some); p.dn = reinterpret_cast<const uint4*>(some); p.w_pre = nullptr; }
  if (!(p.has & HAS_DXO)) p.dxo = some;
  if (!(p.has & HAS_Y)) p.y = reinterpret_cast<const uint4*>(some);
  if (!(p.has & HAS_PRE)) p.stats_pre = reinterpret_cast<float2*>(const_cast<void*>(some));
  if (!(p.has & HAS_POST)) p.stats_post = reinterpret_cast<float2*>(const_cast<void*>(some));
  p.weight = post && a.w_post ? a.w_post : branch ? a.scale : nullptr;
  p.scale_too = post && a.w_post ? a.scale : nullptr;
  const bool scale = a.dscale != nullptr;
  p.want = (a.dw_post || scale ? SUM_A : 0) | (a.db_post || (scale && a.b_post) ? SUM_B : 0) | (a.dw_pre ? SUM_G1 : 0) | (a.db_pre ? SUM_G2 : 0);
  p.dscale = a.dscale;
  p.dw_post = a.dw_post;
  p.db_post = a.db_post;
  p.dw_pre = a.dw_pre;
  p.db_pre = a.db_pre;
  const bool wide = (post && p.post == BIMASK_NORM_LAYER) || p.pre == BIMASK_NORM_LAYER || (p.want & (SUM_B | SUM_G2)) != 0;
  const int rows = bwd_rows(a);
  const RowPlan b = plan_rows(rows, bwd_threads(rows), a.T, a.C, spanned ? (int)p.gate_span : 1, PLAN_SMS, true);
  take_plan(p, b);
  if (b.slots > 1) p.sums = reinterpret_cast<float*>(a.ws);
  if (spanned && (b.units_per_span > 1 || (a.dgate == a.gate && a.stream_type == BIMASK_TYPE_F32))) p.gate_sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.ws) + column_sums_bytes(a.T, a.C, (int)p.gate_span));
  using Yes = std::true_type;
  using No = std::false_type;
  auto run_with = [&](auto step, auto f32, auto gate, auto post, auto wide, auto cluster) -> int {
    constexpr bool F = decltype(f32)::value, P = decltype(post)::value, W = decltype(wide)::value, K = decltype(cluster)::value;
    constexpr int G = decltype(gate)::value, R = decltype(step)::value, H = bwd_threads(R);
    constexpr int values = bwd_values(P, W), kept = bwd_keeps_params(F, K, values) ? param_bytes(H) : 0;
    constexpr int bytes = ring_bytes(R, H, bwd_slots(F, G != 0)) + kept + stats_bytes(R) + Exchange<values * R, H, K>::BYTES;
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
    return launch_rows(residual_bwd_kernel<R, F, G, P, W, K>, b, bytes, s, p);
  };
  auto run = [&](auto f32, auto gate, auto post, auto wide, auto cluster) -> int {
    if constexpr (!decltype(cluster)::value)
      if (rows == 1) return run_with(std::integral_constant<int, 1>(), f32, gate, post, wide, cluster);
    return run_with(std::integral_constant<int, 2>(), f32, gate, post, wide, cluster);
  };
  auto pick3 = [&](auto f32, auto gate, auto post) -> int {
    if (b.cluster > 1) return wide ? run(f32, gate, post, Yes(), Yes()) : run(f32, gate, post, No(), Yes());
    return wide ? run(f32, gate, post, Yes(), No()) : run(f32, gate, post, No(), No());
  };
  auto pick2 = [&](auto f32, auto gate) -> int { return post ? pick3(f32, gate, Yes()) : pick3(f32, gate, No()); };
  auto pick = [&](auto f32) -> int {
    if (spanned) return pick2(f32, std::integral_constant<int, 2>());
    if (p.gate_span != 0) return pick2(f32, std::integral_constant<int, 1>());
    return pick2(f32, std::integral_constant<int, 0>());
  };
  const int rc = a.stream_type == BIMASK_TYPE_F32 ? pick(std::true_type()) : pick(std::false_type());
  if (rc != BIMASK_OK) return rc;
  const int arrays = p.sums != nullptr ? __builtin_popcount(p.want) : 0;
  if (arrays != 0 || p.gate_sums != nullptr) {
    ResidualReduce r = {};
    r.sums = reinterpret_cast<const float4*>(p.sums);
    r.slots = b.slots;
    r.want = arrays != 0 ? p.want : 0;
    r.C4 = a.C / 4;
    r.scale = reinterpret_cast<const float4*>(a.scale);
    r.w_post = reinterpret_cast<const float4*>(a.w_post);
    r.b_post = reinterpret_cast<const float4*>(a.b_post);
    r.dscale = reinterpret_cast<float4*>(a.dscale);
    r.dw_post = reinterpret_cast<float4*>(a.dw_post);
    r.db_post = reinterpret_cast<float4*>(a.db_post);
    r.dw_pre = reinterpret_cast<float4*>(a.dw_pre);
    r.db_pre = reinterpret_cast<float4*>(a.db_pre);
    if (p.gate_sums != nullptr) {
      r.gate_sums = reinterpret_cast<const float4*>(p.gate_sums);
      r.units_per_span = b.units_per_span;
      r.dgate = reinterpret_cast<uint2*>(a.dgate);
      r.gate_pitch4 = a.gate_pitch / 4;
      r.gates = b.gates;
    }
    const long long rows = arrays + (r.gates < 4096 ? r.gates : 4096);
    BIMASK_CUDA_OK(launch_pdl(residual_reduce_kernel, dim3((r.C4 + 7) / 8, (unsigned)rows), 256, 0, s, r));
    count_launch();
  }
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

}  // namespace bimask
