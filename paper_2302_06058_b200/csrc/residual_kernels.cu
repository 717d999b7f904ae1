// The residual junction between two blocks of a network (norm after a block, dropout, gate, residual scale, norm before the
// next block), its gradient, and dropout alone.  All of them stream: every matrix is read once and written once, a row stays
// in the registers of the warps that share it, and the statistics are exchanged by shuffles and one barrier per norm.
#include "dropout.cuh"
#include "sm100_ptx.cuh"
#include <type_traits>

namespace bimask {

namespace {

using act::Pair;

// ------------------------------------------------------------------------------------------
// Dropout alone: a flat stream of blocks of eight elements.
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
__device__ __forceinline__ Vec8<F32> load8(const void* base, long long block) {
  Vec8<F32> v;
  const uint4* src = reinterpret_cast<const uint4*>(base) + block * (F32 ? 2 : 1);
#pragma unroll
  for (int h = 0; h < (F32 ? 2 : 1); ++h) v.w[h] = src[h];
  return v;
}
template <bool F32>
__device__ __forceinline__ void store8(void* base, long long block, const Pair (&p)[4]) {
  const Vec8<F32> v = pack8<F32>(p);
  uint4* dst = reinterpret_cast<uint4*>(base) + block * (F32 ? 2 : 1);
#pragma unroll
  for (int h = 0; h < (F32 ? 2 : 1); ++h) dst[h] = v.w[h];
}

template <bool F32>
__global__ void __launch_bounds__(DROP_THREADS)
dropout_kernel(const void* x, long long blocks, void* y /* may be x */, const DropParams d) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned long long number = drop_number(d);
  constexpr int U = 2;
  const long long step = (long long)gridDim.x * DROP_THREADS;
  for (long long i0 = (long long)blockIdx.x * DROP_THREADS + threadIdx.x; i0 < blocks; i0 += U * step) {
    Vec8<F32> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * step < blocks) v[u] = load8<F32>(x, i0 + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * step;
      if (i < blocks) {
        Pair p[4];
        unpack8<F32>(v[u], p);
        if (d.thr != 0u) drop8(p, (unsigned long long)i, number, d);
        store8<F32>(y, i, p);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Rows.  A thread owns one block of eight columns for good; `warps` warps of a CTA, and up to four CTAs of a cluster above 4096
// columns, share a row.  A CTA holds as many such groups as its 16 warps give; they work on rows of their own and never meet (named
// barriers).  A group takes two rows per step: what its threads exchange for both travels together, and the two rows' chains
// of dependent instructions run side by side.  The rows of the next step are already on their way: every thread copies its own
// 16-byte pieces into its own places in shared memory (cp.async), so no barrier guards them, no registers wait for them, and
// whoever writes a row in place has its old values safely fetched.
// What bounds these kernels next to HBM is the instructions they issue, so the rows' code has no branches but those of absent
// parts: columns and rows past the end are copied as zeros (from a clamped address, of which cp.async reads nothing) and work like
// the others, but for their stores.
// ------------------------------------------------------------------------------------------
constexpr int ROWS = 2, STAGES = 2;
constexpr int ROW_THREADS = 512;
constexpr int MAX_ROW_WARPS = 64;                         // of a cluster of four CTAs
static_assert(RESIDUAL_MAX_C == 256 * MAX_ROW_WARPS, "eight columns per thread");

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
  float* sums;                       // [clusters][wanted arrays][C]
  float* gate_sums;                  // [units][C]
  int want;                          // bits: SUM_* arrays that are wanted
  int branch;                        // a gradient of the branch is wanted
  // Rows are given out in units of consecutive ones.  units_per_span: 0, or the units that a gate row's span is cut into.
  uint32_t units, unit_rows, units_per_span;
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
__device__ __forceinline__ void normalise(Pair (&v)[4], float2 st) {
  const Pair rstd = act::both(st.y), shift = act::both(-st.x * st.y);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = act::fma2(v[k], rstd, shift);
}

// columns that a row's warp w holds
__device__ __forceinline__ float columns_of(int w, uint32_t C8) { return 8.f * (float)min(max((int)C8 - 32 * w, 0), 32); }

// Exchange buffers: a group's two, of four values from each of its row's warps, their number made even (zero where there is no
// such warp).  Groups of two warps or more: three words for two warps at worst.
template <bool CLUSTER>
struct Exchange {
  static constexpr int WORDS = CLUSTER ? MAX_ROW_WARPS : ROW_THREADS / 64 * 3;
  static constexpr int BYTES = 2 * 4 * WORDS * 4;
};
template <bool CLUSTER>
struct Group {                                            // a thread's place among those that share its rows
  int lane, group, warps;                                 // warps: of the row in this CTA
  int warp;                                               // the thread's warp, counted through the row
  bool alone;                                             // the row is one warp's
  int cluster;
  float inv_columns;                                      // 1 / columns that this warp holds
  float peer_columns;                                     // columns of warp lane % 16 (only without clusters)
  uint32_t mine, buffer;                                  // address of this warp's first word, and of the buffer in use
  uint32_t flip;
  int width;                                              // words of a value

  __device__ __forceinline__ Group(const ResidualParams& p, uint32_t exchange) {
    const int w = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    warps = p.warps;
    group = w / warps;
    cluster = p.cluster;
    warp = w - group * warps + (CLUSTER ? (int)ptx::cluster_ctarank() * warps : 0);
    alone = !CLUSTER && warps == 1;
    inv_columns = 1.f / fmaxf(columns_of(warp, p.C8), 1.f);
    peer_columns = columns_of(lane & 15, p.C8);
    width = CLUSTER ? MAX_ROW_WARPS : warps + (warps & 1);
    buffer = exchange + (uint32_t)((alone ? 0 : group) * 2 * 4 * width * 4);
    mine = 4u * (uint32_t)warp;
    flip = buffer ^ (buffer + 4u * (uint32_t)width * 4u);
  }
  // Value i of this warp, to every CTA that shares the row ...
  __device__ __forceinline__ void publish(int i, float v) const {
    const uint32_t at = buffer + mine + (uint32_t)(i * width * 4);
    if (!CLUSTER) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
    else
      for (int r = 0; r < cluster; ++r) ptx::st_cluster_u32(ptx::mapa(at, (uint32_t)r), __float_as_uint(v));
  }
  __device__ __forceinline__ void meet() const {
    if (CLUSTER) ptx::cluster_sync();
    else ptx::named_bar_sync(group + 1, 32 * warps);
  }
  // ... and all warps' values, after they have met.  Two buffers in turn: who writes one has met the others over the other one, and
  // by then everybody had read this one.
  __device__ __forceinline__ uint32_t published(int i, int w) const { return buffer + (uint32_t)((i * width + w) * 4); }
  __device__ __forceinline__ void turn() { buffer ^= flip; }
};

// Sums over a warp of two or four values at a time: at each step a lane keeps half of its values and hands the others to its
// partner.  The total of value i ends in the lanes 16 i .. or 8 i ..
__device__ __forceinline__ float fold2(float a, float b, int lane) {
  const bool hi = (lane & 16) != 0;
  float v = (hi ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, hi ? a : b, 16);
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
__device__ __forceinline__ float fold4(const float (&c)[4], int lane) {
  const bool hi = (lane & 16) != 0, mid = (lane & 8) != 0;
  const float k0 = (hi ? c[2] : c[0]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? c[0] : c[2], 16);
  const float k1 = (hi ? c[3] : c[1]) + __shfl_xor_sync(0xFFFFFFFFu, hi ? c[1] : c[3], 16);
  float v = (mid ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, mid ? k0 : k1, 8);
#pragma unroll
  for (int d = 4; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Totals over the row of four values; `folded`: fold4 of the thread's.  Split in two, so that other work can be done in between.
template <bool CLUSTER>
__device__ __forceinline__ void totals_begin(const Group<CLUSTER>& g, float folded) {
  if (!g.alone && (g.lane & 7) == 0) g.publish(g.lane >> 3, folded);
}
template <bool CLUSTER>
__device__ __forceinline__ void totals_end(Group<CLUSTER>& g, float folded, float (&c)[4]) {
  if (!g.alone) {
    g.meet();
    folded = 0.f;
#pragma unroll
    for (int k = 0; k < (CLUSTER ? 4 : 1); ++k) {
      const int w = 2 * (g.lane & 7) + 16 * k;
      if (w < g.width) {
        const float2 v = read_pair(g.published(g.lane >> 3, w));
        folded += v.x + v.y;
      }
    }
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) folded += __shfl_xor_sync(0xFFFFFFFFu, folded, d);
    g.turn();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = __shfl_sync(0xFFFFFFFFu, folded, 8 * i);
}

// Mean and 1 / deviation of two rows.  The squares are taken about each warp's own mean, and the warps are put together by
// M = sum M_w + sum n_w (m_w - m)^2: one exchange, and no difference of large squares.  rms: all about zero.
template <bool CLUSTER>
__device__ __forceinline__ void row_stats(const Pair (&v)[ROWS][4], bool ok, bool layer, float eps, float inv_c, uint32_t C8,
                                          Group<CLUSTER>& g, float2 (&st)[ROWS]) {
  static_assert(ROWS == 2, "two rows are folded together");
  const int half = g.lane >> 4;                           // the row whose totals this lane holds
  float m = 0.f, q[ROWS];
  if (layer) {
    m = fold2(horizontal(sum8(v[0])), horizontal(sum8(v[1])), g.lane) * g.inv_columns;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const Pair shift = act::both(-__shfl_sync(0xFFFFFFFFu, m, 16 * r));
      Pair d[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) d[k] = act::add2(v[r][k], shift);
      q[r] = ok ? horizontal(dot8(d, d)) : 0.f;
    }
  } else {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) q[r] = horizontal(dot8(v[r], v[r]));
  }
  float sq = fold2(q[0], q[1], g.lane);
  if (!g.alone) {
    if ((g.lane & 15) == 0) {
      if (layer) g.publish(half, m);
      g.publish(2 + half, sq);
    }
    g.meet();
    sq = 0.f;
    if (CLUSTER) {
      if (layer) {
        m = 0.f;
        for (int w = g.lane & 15; w < MAX_ROW_WARPS; w += 16) m = fmaf(columns_of(w, C8), read_word(g.published(half, w)), m);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) m += __shfl_xor_sync(0xFFFFFFFFu, m, d);
        m *= inv_c;
      }
      for (int w = g.lane & 15; w < MAX_ROW_WARPS; w += 16) {
        sq += read_word(g.published(2 + half, w));
        if (layer) {
          const float d = read_word(g.published(half, w)) - m;
          sq = fmaf(columns_of(w, C8) * d, d, sq);
        }
      }
    } else {
      const int w = min(g.lane & 15, g.width - 1);
      sq = (g.lane & 15) < g.width ? read_word(g.published(2 + half, w)) : 0.f;
      if (layer) {
        const float own = read_word(g.published(half, w));
        m = g.peer_columns * own;
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) m += __shfl_xor_sync(0xFFFFFFFFu, m, d);
        m *= inv_c;
        sq = fmaf(g.peer_columns * (own - m), own - m, sq);
      }
    }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, d);
    g.turn();
  }
  const float rstd = rsqrtf(fmaf(sq, inv_c, eps));        // two units in the last place
#pragma unroll
  for (int r = 0; r < ROWS; ++r) st[r] = make_float2(layer ? __shfl_sync(0xFFFFFFFFu, m, 16 * r) : 0.f, __shfl_sync(0xFFFFFFFFu, rstd, 16 * r));
}

// A group's walk over its units, ROWS rows at a time.  SPAN: units of many rows that end with their gate row's span; else of one
// row (all others of the step are none) or ROWS.
template <bool SPAN>
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
constexpr int PITCH = ROW_THREADS * 16;                   // from a thread's piece to its next
constexpr int STATS_STAGE = 2 * ROWS * 8;                 // bytes of a warp's statistics: before, after
constexpr int STATS_BYTES = STAGES * (ROW_THREADS / 32) * STATS_STAGE;
BIMASK_HD constexpr int fwd_slots(bool f32, bool gate) { return (f32 ? 2 : 1) + 1 + (gate ? 1 : 0); }
BIMASK_HD constexpr int bwd_slots(bool f32, bool gate) { return (f32 ? 4 : 2) + 2 + (gate ? 1 : 0); }
BIMASK_HD constexpr int ring_bytes(int slots) { return STAGES * ROWS * slots * PITCH; }

template <bool F32>
__device__ __forceinline__ void copy_block(uint32_t dst, const void* base, unsigned long long block, bool live) {
  const uint4* src = reinterpret_cast<const uint4*>(base) + block * (F32 ? 2 : 1);
  copy16(dst, src, live);
  if (F32) copy16(dst + PITCH, src + 1, live);
}
template <bool F32>
__device__ __forceinline__ void read_block(uint32_t at, Pair (&v)[4]) {
  Vec8<F32> raw;
#pragma unroll
  for (int h = 0; h < (F32 ? 2 : 1); ++h)
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.w[h].x), "=r"(raw.w[h].y), "=r"(raw.w[h].z), "=r"(raw.w[h].w)
                 : "r"(at + h * PITCH) : "memory");
  unpack8<F32>(raw, v);
}
template <bool CLUSTER>
__device__ __forceinline__ void clear_exchange(float* exchange) {
  for (int i = threadIdx.x; i < Exchange<CLUSTER>::BYTES / 4; i += blockDim.x) exchange[i] = 0.f;
  if (CLUSTER) ptx::cluster_sync();                       // before a peer writes here, and before this CTA writes to a peer
  else __syncthreads();
}

template <bool F32, bool GATE, bool CLUSTER>
__global__ void __launch_bounds__(ROW_THREADS, 2)
residual_fwd_kernel(const __grid_constant__ ResidualParams p) {
  extern __shared__ float4 smem[];
  constexpr int SLOTS = fwd_slots(F32, GATE), X = 0, Y = F32 ? 2 : 1, G = Y + 1;
  constexpr uint32_t STAGE = ROWS * SLOTS * PITCH;
  float* exchange = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(smem) + ring_bytes(SLOTS));
  pdl_launch_dependents();
  clear_exchange<CLUSTER>(exchange);
  Group<CLUSTER> g(p, smem_addr(exchange));
  const uint32_t col = 32u * (uint32_t)g.warp + (uint32_t)g.lane, colc = min(col, p.C8 - 1u);
  const bool ok = col < p.C8;
  const uint32_t groups = blockDim.x / (32u * (uint32_t)p.warps);
  const uint32_t stride = CLUSTER ? gridDim.x / (uint32_t)p.cluster : gridDim.x * groups;
  const uint32_t ring = smem_addr(smem) + threadIdx.x * 16u;
  Walk<false> work, ahead;
  work.unit = CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x * groups + (uint32_t)g.group;
  work.enter(p);
  ahead = work;
  pdl_wait();
  const unsigned long long number = drop_number(p.drop);
  auto fetch = [&](const Walk<false>& w, uint32_t stage) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool live = ok && w.more(p) && w.t + r < w.end;
      const uint32_t t = min(w.t + r, p.T - 1u), at = ring + stage * STAGE + r * SLOTS * PITCH;
      const unsigned long long block = (unsigned long long)t * p.C8 + colc;
      copy_block<F32>(at + X * PITCH, p.x, block, live);
      if (p.y != nullptr) copy16(at + Y * PITCH, p.y + block, live);
      if (GATE) copy16(at + G * PITCH, p.gate + (long long)(p.gate_span == 1u ? t : t / p.gate_span) * p.gate_pitch8 + colc, live);
    }
    copies_commit();
  };
  fetch(ahead, 0);
  uint32_t stage = 0;
  while (work.more(p)) {
    ahead.next(p, stride);
    fetch(ahead, stage ^ 1u);
    copies_wait<1>();
    bool live[ROWS];
    const uint32_t at = ring + stage * STAGE;
    unsigned long long block[ROWS];
    Pair v[ROWS][4];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      live[r] = ok && work.t + r < work.end;
      block[r] = (unsigned long long)(work.t + r) * p.C8 + col;
    }
    if (p.y != nullptr) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) read_block<false>(at + (r * SLOTS + Y) * PITCH, v[r]);
      if (p.post != BIMASK_NORM_NONE) {
        float2 st[ROWS];
        row_stats(v, ok, p.post == BIMASK_NORM_LAYER, p.eps_post, p.inv_c, p.C8, g, st);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          if (p.stats_post != nullptr && col == 0 && live[r]) p.stats_post[work.t + r] = st[r];
          normalise(v[r], st[r]);
        }
        Pair w[4];
        if (p.w_post != nullptr) {
          param8(p.w_post, colc, w);
#pragma unroll
          for (int r = 0; r < ROWS; ++r) times8(v[r], w);
        }
        if (p.b_post != nullptr) {
          param8(p.b_post, colc, w);
#pragma unroll
          for (int r = 0; r < ROWS; ++r) plus8(v[r], w);
        }
      }
      if (p.drop.thr != 0u) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) drop8(v[r], block[r], number, p.drop);
      }
      if (GATE) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          Pair w[4];
          read_block<false>(at + (r * SLOTS + G) * PITCH, w);
          times8(v[r], w);
        }
      }
      if (p.scale != nullptr) {
        Pair w[4];
        param8(p.scale, colc, w);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) times8(v[r], w);
      }
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) fill8(v[r], 0.f);
    }
    const Pair alpha = act::both(p.alpha);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      Pair x[4];
      read_block<F32>(at + (r * SLOTS + X) * PITCH, x);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[r][k] = act::fma2(x[k], alpha, v[r][k]);
      if (p.xo != nullptr && live[r]) store8<F32>(p.xo, (long long)block[r], v[r]);
    }
    if (p.pre != BIMASK_NORM_NONE) {
      float2 st[ROWS];
      if (!ok) {                                          // whatever came of the zeros there (a bias, an infinite statistic) stays out
#pragma unroll
        for (int r = 0; r < ROWS; ++r) fill8(v[r], 0.f);
      }
      row_stats(v, ok, p.pre == BIMASK_NORM_LAYER, p.eps_pre, p.inv_c, p.C8, g, st);
      Pair w[4];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        if (p.stats_pre != nullptr && col == 0 && live[r]) p.stats_pre[work.t + r] = st[r];
        normalise(v[r], st[r]);
      }
      if (p.w_pre != nullptr) {
        param8(p.w_pre, colc, w);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) times8(v[r], w);
      }
      if (p.b_pre != nullptr) {
        param8(p.b_pre, colc, w);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) plus8(v[r], w);
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
        if (live[r]) store8<false>(p.n, (long long)block[r], v[r]);
    }
    work.next(p, stride);
    stage ^= 1u;
  }
  copies_wait<0>();
  if (CLUSTER) ptx::cluster_sync();                       // shared memory outlives the peers' writes to it
}

// ------------------------------------------------------------------------------------------
// Gradient.  With m the dropout's multiplier, xh and yh the normalised values and u = yh w_post + b_post:
//   D  = dx' + rstd (g - mean(g) [layer] - xh mean(g xh)),  g = w_pre dn;        dx = alpha D
//   e  = m gate D;  dy the same norm formula on scale e w_post;                   dgate = m D scale u
// and four column sums carry every parameter's gradient: G1 = sum dn xh (w_pre), G2 = sum dn (b_pre), A = sum e yh, B = sum e:
//   dw_post = scale A,  db_post = scale B,  dscale = w_post A + b_post B.
// A thread keeps its columns' sums in registers; each cluster (CTA) leaves one row of partial sums.
// Columns and rows past the end: dx', dn and y are zeros, and so are D (its means are left out there) and every sum.
// GATE: 0 no gate, 1 a gate whose gradient, if wanted, is a row per token, 2 one whose gradient is summed over spans.
// ------------------------------------------------------------------------------------------
enum { SUM_A = 1, SUM_B = 2, SUM_G1 = 4, SUM_G2 = 8 };

template <bool F32, int GATE, bool CLUSTER>
__global__ void __launch_bounds__(ROW_THREADS, 1)
residual_bwd_kernel(const __grid_constant__ ResidualParams p) {
  extern __shared__ float4 smem[];
  constexpr int SLOTS = bwd_slots(F32, GATE != 0), XB = F32 ? 2 : 1, X = 0, DX = XB, DN = 2 * XB, Y = DN + 1, G = Y + 1;
  constexpr uint32_t STAGE = ROWS * SLOTS * PITCH;
  uint8_t* const after = reinterpret_cast<uint8_t*>(smem) + ring_bytes(SLOTS);
  float* const exchange = reinterpret_cast<float*>(after + STATS_BYTES);
  pdl_launch_dependents();
  clear_exchange<CLUSTER>(exchange);
  Group<CLUSTER> g(p, smem_addr(exchange));
  const uint32_t col = 32u * (uint32_t)g.warp + (uint32_t)g.lane, colc = min(col, p.C8 - 1u);
  const bool ok = col < p.C8;
  const float inv_c = ok ? p.inv_c : 0.f;
  const uint32_t groups = blockDim.x / (32u * (uint32_t)p.warps);
  const uint32_t stride = CLUSTER ? gridDim.x / (uint32_t)p.cluster : gridDim.x * groups;
  const uint32_t ring = smem_addr(smem) + threadIdx.x * 16u;
  const uint32_t stats = smem_addr(after) + (threadIdx.x >> 5) * (STAGES * STATS_STAGE);
  Walk<GATE == 2> work, ahead;
  work.unit = CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x * groups + (uint32_t)g.group;
  work.enter(p);
  ahead = work;
  pdl_wait();
  const unsigned long long number = drop_number(p.drop);
  const bool pre = p.pre != BIMASK_NORM_NONE, post = p.post != BIMASK_NORM_NONE && p.branch != 0;
  const bool layer_pre = p.pre == BIMASK_NORM_LAYER, layer_post = p.post == BIMASK_NORM_LAYER;
  auto fetch = [&](const Walk<GATE == 2>& w, uint32_t stage) {
    const bool more = w.more(p);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool live = ok && more && w.t + r < w.end;
      const uint32_t t = min(w.t + r, p.T - 1u), at = ring + stage * STAGE + r * SLOTS * PITCH;
      const unsigned long long block = (unsigned long long)t * p.C8 + colc;
      if (pre) {
        copy_block<F32>(at + X * PITCH, p.xo, block, live);
        copy16(at + DN * PITCH, p.dn + block, live);
      }
      if (p.dxo != nullptr) copy_block<F32>(at + DX * PITCH, p.dxo, block, live);
      if (p.y != nullptr) copy16(at + Y * PITCH, p.y + block, live);
      if (GATE != 0) copy16(at + G * PITCH, p.gate + (long long)(p.gate_span == 1u ? t : t / p.gate_span) * p.gate_pitch8 + colc, live);
    }
    if (g.lane < 2 * ROWS) {                              // lanes 0, 1: the rows' statistics before, 2, 3: after
      const uint32_t t = w.t + (g.lane & 1);
      const float2* src = g.lane < 2 ? p.stats_pre : p.stats_post;
      if (src != nullptr) copy8(stats + stage * STATS_STAGE + g.lane * 8u, src + min(t, p.T - 1u), more && t < w.end);
    }
    copies_commit();
  };
  Pair sums[4][4], fsum[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) fill8(sums[a], 0.f);
  fill8(fsum, 0.f);
  fetch(ahead, 0);
  uint32_t stage = 0;
  while (work.more(p)) {
    __syncwarp();                                         // every lane has read the statistics that are overwritten now
    ahead.next(p, stride);
    fetch(ahead, stage ^ 1u);
    copies_wait<1>();
    __syncwarp();                                         // the statistics are other lanes' copies
    bool live[ROWS];
    const uint32_t at = ring + stage * STAGE, st_at = stats + stage * STATS_STAGE;
    unsigned long long block[ROWS];
    Pair D[ROWS][4];
    uint4 bits[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      live[r] = ok && work.t + r < work.end;
      block[r] = (unsigned long long)(work.t + r) * p.C8 + col;
      if (p.dxo != nullptr) read_block<F32>(at + (r * SLOTS + DX) * PITCH, D[r]);
      else fill8(D[r], 0.f);
    }
    auto draw = [&]() {
      if (p.drop.thr != 0u) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) bits[r] = philox(block[r], number, p.drop);
      }
    };
    if (pre) {
      Pair xh[ROWS][4], gr[ROWS][4];
      float c[4], rstd[ROWS];
      Pair w[4];
      if (p.w_pre != nullptr) param8(p.w_pre, colc, w);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float2 st = read_pair(st_at + 8 * r);
        rstd[r] = st.y;
        read_block<F32>(at + (r * SLOTS + X) * PITCH, xh[r]);
        read_block<false>(at + (r * SLOTS + DN) * PITCH, gr[r]);
        normalise(xh[r], st);
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[2][k] = act::fma2(gr[r][k], xh[r][k], sums[2][k]);
        if (p.want & SUM_G2) plus8(sums[3], gr[r]);
        if (p.w_pre != nullptr) times8(gr[r], w);
        c[2 * r] = horizontal(dot8(gr[r], xh[r]));
        c[2 * r + 1] = layer_pre ? horizontal(sum8(gr[r])) : 0.f;
      }
      const float folded = fold4(c, g.lane);
      totals_begin(g, folded);
      draw();                                             // needs nothing of the others: done while they arrive
      totals_end(g, folded, c);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float scaled = -rstd[r] * inv_c;
        const Pair c1 = act::both(c[2 * r] * scaled), rs = act::both(rstd[r]);
        if (layer_pre) {
          const Pair c2 = act::both(c[2 * r + 1] * scaled);
#pragma unroll
          for (int k = 0; k < 4; ++k) D[r][k] = act::add2(D[r][k], c2);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) D[r][k] = act::fma2(gr[r][k], rs, act::fma2(xh[r][k], c1, D[r][k]));
      }
    } else {
      draw();
    }
    if (p.dx != nullptr) {
      const Pair alpha = act::both(p.alpha);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        Pair o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = act::mul2(D[r][k], alpha);
        if (live[r]) store8<F32>(p.dx, (long long)block[r], o);
      }
    }
    if (p.branch) {
      Pair yh[ROWS][4];
      float c[4], rstd[ROWS];
      Pair w[4];                                          // scale w_post
      const bool weighted = p.scale != nullptr || p.w_post != nullptr;
      if (p.w_post != nullptr) param8(p.w_post, colc, w);
      if (p.scale != nullptr) {
        Pair s[4];
        param8(p.scale, colc, s);
        if (p.w_post != nullptr) times8(w, s);
        else
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = s[k];
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        rstd[r] = 1.f;
        if (p.y != nullptr) read_block<false>(at + (r * SLOTS + Y) * PITCH, yh[r]);
        else fill8(yh[r], 0.f);
        if (post) {
          const float2 st = read_pair(st_at + 8 * (ROWS + r));
          rstd[r] = st.y;
          normalise(yh[r], st);
        }
        if (p.drop.thr != 0u) {
          D[r][0] = drop_pair(D[r][0], bits[r].x, p.drop.thr, p.drop.scale);
          D[r][1] = drop_pair(D[r][1], bits[r].y, p.drop.thr, p.drop.scale);
          D[r][2] = drop_pair(D[r][2], bits[r].z, p.drop.thr, p.drop.scale);
          D[r][3] = drop_pair(D[r][3], bits[r].w, p.drop.thr, p.drop.scale);
        }
        if (GATE != 0) {
          if (GATE == 2 || p.dgate != nullptr) {          // scale u
            Pair u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = yh[r][k];
            if (weighted) times8(u, w);
            if (p.b_post != nullptr) {
              Pair b[4];
              param8(p.b_post, colc, b);
              if (p.scale != nullptr) {
                Pair s[4];
                param8(p.scale, colc, s);
                times8(b, s);
              }
              plus8(u, b);
            }
            if (GATE == 2) {
#pragma unroll
              for (int k = 0; k < 4; ++k) fsum[k] = act::fma2(D[r][k], u[k], fsum[k]);
            } else {
              times8(u, D[r]);
              if (live[r]) store8<false>(p.dgate, (long long)(work.t + r) * p.gate_pitch8 + col, u);
            }
          }
          Pair gt[4];
          read_block<false>(at + (r * SLOTS + G) * PITCH, gt);
          times8(D[r], gt);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[0][k] = act::fma2(D[r][k], yh[r][k], sums[0][k]);
        if (p.want & SUM_B) plus8(sums[1], D[r]);
        if (weighted) times8(D[r], w);
      }
      if (post) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          c[2 * r] = horizontal(dot8(D[r], yh[r]));
          c[2 * r + 1] = layer_post ? horizontal(sum8(D[r])) : 0.f;
        }
        const float folded = fold4(c, g.lane);
        totals_begin(g, folded);
        totals_end(g, folded, c);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const float scaled = -rstd[r] * inv_c;
          const Pair c1 = act::both(c[2 * r] * scaled), c2 = act::both(layer_post ? c[2 * r + 1] * scaled : 0.f), rs = act::both(rstd[r]);
#pragma unroll
          for (int k = 0; k < 4; ++k) D[r][k] = act::fma2(D[r][k], rs, act::fma2(yh[r][k], c1, c2));
        }
      }
      if (p.dy != nullptr) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          if (live[r]) store8<false>(p.dy, (long long)block[r], D[r]);
      }
      if (GATE == 2 && work.last()) {
        if (ok) store8<true>(p.gate_sums, (long long)work.unit * p.C8 + col, fsum);
        fill8(fsum, 0.f);
      }
    }
    work.next(p, stride);
    stage ^= 1u;
  }
  copies_wait<0>();
  // the groups' sums are added through the ring, in their order
  int slot = 0;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    if (!(p.want & (1 << a))) continue;                   // the same for every thread
    if (groups > 1) {
      __syncthreads();
      const Vec8<true> v = pack8<true>(sums[a]);
      uint4* mine = reinterpret_cast<uint4*>(smem) + threadIdx.x;
      mine[0] = v.w[0];
      mine[ROW_THREADS] = v.w[1];
      __syncthreads();
    }
    if (g.group == 0 && ok) {
      for (uint32_t o = 1; o < groups; ++o) {
        Pair q[4];
        read_block<true>(ring + o * (uint32_t)p.warps * 512u, q);
        plus8(sums[a], q);
      }
      store8<true>(p.sums, ((long long)(CLUSTER ? blockIdx.x / (uint32_t)p.cluster : blockIdx.x) * __popc(p.want) + slot) * p.C8 + col, sums[a]);
    }
    ++slot;
  }
  if (CLUSTER) ptx::cluster_sync();                       // shared memory outlives the peers' writes to it
}

// The parameters' gradients from the CTAs' partial sums: a CTA covers 8 float4 columns, its 32 row slots take the partial
// rows in turn and are added through shared memory, in a fixed order.
struct ResidualReduce {
  const float4* sums;
  int slots, want, C4;
  const float4 *scale, *w_post, *b_post;
  float4 *dscale, *dw_post, *db_post, *dw_pre, *db_pre;
};
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }

__global__ void __launch_bounds__(256)
residual_reduce_kernel(const ResidualReduce p) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float4 red[32][8];
  const int lane = threadIdx.x & 7, slot = threadIdx.x >> 3;
  const int e = blockIdx.x * 8 + lane;
  const int arrays = __popc(p.want);
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 total[4];
  int at = 0;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    total[a] = zero;
    if (!(p.want & (1 << a))) continue;
    float4 acc = zero;
    if (e < p.C4)
#pragma unroll 8
      for (int s = slot; s < p.slots; s += 32) acc = add4(acc, p.sums[((size_t)s * arrays + at) * p.C4 + e]);
    ++at;
    __syncthreads();
    red[slot][lane] = acc;
    __syncthreads();
#pragma unroll
    for (int half = 16; half >= 1; half >>= 1) {
      if (slot < half) {
        acc = add4(acc, red[slot + half][lane]);
        red[slot][lane] = acc;
      }
      __syncthreads();
    }
    total[a] = acc;
  }
  if (slot != 0 || e >= p.C4) return;
  const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
  const float4 s = p.scale != nullptr ? __ldg(p.scale + e) : one, w = p.w_post != nullptr ? __ldg(p.w_post + e) : one;
  if (p.dw_post != nullptr) p.dw_post[e] = mul4(s, total[0]);
  if (p.db_post != nullptr) p.db_post[e] = mul4(s, total[1]);
  if (p.dscale != nullptr) {
    float4 d = mul4(w, total[0]);
    if (p.b_post != nullptr) d = add4(d, mul4(__ldg(p.b_post + e), total[1]));
    p.dscale[e] = d;
  }
  if (p.dw_pre != nullptr) p.dw_pre[e] = total[2];
  if (p.db_pre != nullptr) p.db_pre[e] = total[3];
}

// dgate of a row that serves a span of tokens: the sum of its units, in order.
__global__ void __launch_bounds__(256)
gate_reduce_kernel(const float4* __restrict__ sums, int units_per_span, long long gates, int C4, uint2* dgate, long long pitch4) {
  pdl_launch_dependents();
  pdl_wait();
  const long long all = gates * C4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += 256ll * gridDim.x) {
    const long long g = i / C4;
    const int c = (int)(i - g * C4);
    const float4* src = sums + g * units_per_span * C4 + c;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int u = 0; u < units_per_span; ++u) acc = add4(acc, src[(long long)u * C4]);
    dgate[g * pitch4 + c] = make_uint2(pack_bf16_f(acc.x, acc.y), pack_bf16_f(acc.z, acc.w));
  }
}

// ---- plans --------------------------------------------------------------------------------------
struct RowPlan {
  int cluster, warps, groups, threads;                    // CTAs that share a row, its warps in each, rows side by side
  int slots;                                              // clusters (CTAs) of the grid
  long long units, gates;
  int unit_rows, units_per_span;
};

// ctas: how many the card holds.  span > 1: units end where a gate row's span ends, and are as many as the groups of warps.
RowPlan plan_rows(int T, int C, int span, int ctas) {
  RowPlan b = {};
  const int all = (C / 8 + 31) / 32;                      // warps of a row
  b.cluster = all > 32 ? 4 : all > 16 ? 2 : 1;
  b.warps = (all + b.cluster - 1) / b.cluster;
  b.groups = ROW_THREADS / 32 / b.warps;
  b.threads = 32 * b.warps * b.groups;
  const long long room = (long long)(ctas / b.cluster) * b.groups;
  if (span > 1) {
    const int len = span < T ? span : T;
    b.gates = (T + (long long)span - 1) / span;
    b.unit_rows = (int)((T + room - 1) / room);
    if (b.unit_rows > 1 && b.unit_rows % ROWS != 0) b.unit_rows += ROWS - b.unit_rows % ROWS;
    if (b.unit_rows > len) b.unit_rows = len;
    b.units_per_span = (len + b.unit_rows - 1) / b.unit_rows;
    b.units = b.gates * b.units_per_span;
  } else {
    b.unit_rows = T > room ? ROWS : 1;                    // fewer rows than groups: one each
    b.units = ((long long)T + b.unit_rows - 1) / b.unit_rows;
  }
  const long long slots = (b.units + b.groups - 1) / b.groups;
  b.slots = (int)(slots < ctas / b.cluster ? slots : ctas / b.cluster);
  return b;
}

template <typename K>
int launch_rows(K kernel, const RowPlan& b, int bytes, cudaStream_t s, const ResidualParams& p) {
  const int rc = set_smem_attr(kernel, bytes);
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
static size_t column_sums_bytes(int T, int C, int span) {
  const RowPlan b = plan_rows(1, C, 1, PLAN_SMS);
  const long long most = PLAN_SMS / b.cluster, slots = ((span > 1 ? 2ll : 1ll) * T + b.groups - 1) / b.groups;
  return up256((size_t)(slots < most ? slots : most) * 4 * C * sizeof(float));
}
size_t residual_workspace_bytes(int T, int C, int span) {
  size_t bytes = column_sums_bytes(T, C, span);
  if (span > 1) {
    const RowPlan b = plan_rows(1, C, 1, PLAN_SMS);
    const long long gates = (T + (long long)span - 1) / span, most = 2ll * (PLAN_SMS / b.cluster) * b.groups + gates;
    bytes += (size_t)(most < 2ll * T ? most : 2ll * T) * C * sizeof(float);
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
  const long long blocks = (long long)T * (C / 8);
  const long long ctas = (blocks + DROP_THREADS - 1) / DROP_THREADS, most = 32ll * sm_count();
  auto run = [&](auto kern) {
    return launch_pdl(kern, (unsigned)(ctas < most ? ctas : most), DROP_THREADS, 0, s, x, blocks, y, drop_params(&d));
  };
  BIMASK_CUDA_OK(type == BIMASK_TYPE_F32 ? run(dropout_kernel<true>) : run(dropout_kernel<false>));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

static ResidualParams residual_params(const bimask_residual_args& a) {
  ResidualParams p = {};
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

int launch_residual_fwd(const bimask_residual_args& a, cudaStream_t s) {
  ResidualParams p = residual_params(a);
  const RowPlan b = plan_rows(a.T, a.C, 1, 2 * sm_count());
  take_plan(p, b);
  auto run = [&](auto f32, auto gate, auto cluster) -> int {
    constexpr bool F = decltype(f32)::value, G = decltype(gate)::value, K = decltype(cluster)::value;
    return launch_rows(residual_fwd_kernel<F, G, K>, b, ring_bytes(fwd_slots(F, G)) + Exchange<K>::BYTES, s, p);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  auto pick = [&](auto f32, auto gate) -> int { return b.cluster > 1 ? run(f32, gate, Yes()) : run(f32, gate, No()); };
  const bool gate = p.gate_span != 0;
  const int rc = a.stream_type == BIMASK_TYPE_F32 ? (gate ? pick(Yes(), Yes()) : pick(Yes(), No())) : (gate ? pick(No(), Yes()) : pick(No(), No()));
  if (rc != BIMASK_OK) return rc;
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_residual_bwd(const bimask_residual_args& a, cudaStream_t s) {
  ResidualParams p = residual_params(a);
  const bool spanned = a.dgate != nullptr && p.gate_span > 1;
  const RowPlan b = plan_rows(a.T, a.C, spanned ? (int)p.gate_span : 1, PLAN_SMS);
  take_plan(p, b);
  p.branch = a.dy || a.dgate || a.dscale || a.dw_post || a.db_post;
  if (!p.branch) { p.y = nullptr; p.stats_post = nullptr; }
  if (p.pre == BIMASK_NORM_NONE) p.stats_pre = nullptr;
  if (p.post == BIMASK_NORM_NONE) p.stats_post = nullptr;
  const bool scale = a.dscale != nullptr;
  p.want = (a.dw_post || scale ? SUM_A : 0) | (a.db_post || (scale && a.b_post) ? SUM_B : 0) | (a.dw_pre ? SUM_G1 : 0) | (a.db_pre ? SUM_G2 : 0);
  p.sums = reinterpret_cast<float*>(a.ws);
  if (spanned) p.gate_sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.ws) + column_sums_bytes(a.T, a.C, (int)p.gate_span));
  auto run = [&](auto f32, auto gate, auto cluster) -> int {
    constexpr bool F = decltype(f32)::value, K = decltype(cluster)::value;
    constexpr int G = decltype(gate)::value, bytes = ring_bytes(bwd_slots(F, G != 0)) + STATS_BYTES + Exchange<K>::BYTES;
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
    return launch_rows(residual_bwd_kernel<F, G, K>, b, bytes, s, p);
  };
  auto pick2 = [&](auto f32, auto gate) -> int { return b.cluster > 1 ? run(f32, gate, std::true_type()) : run(f32, gate, std::false_type()); };
  auto pick = [&](auto f32) -> int {
    if (spanned) return pick2(f32, std::integral_constant<int, 2>());
    if (p.gate_span != 0) return pick2(f32, std::integral_constant<int, 1>());
    return pick2(f32, std::integral_constant<int, 0>());
  };
  const int rc = a.stream_type == BIMASK_TYPE_F32 ? pick(std::true_type()) : pick(std::false_type());
  if (rc != BIMASK_OK) return rc;
  if (p.want != 0) {
    ResidualReduce r = {};
    r.sums = reinterpret_cast<const float4*>(a.ws);
    r.slots = b.slots;
    r.want = p.want;
    r.C4 = a.C / 4;
    r.scale = reinterpret_cast<const float4*>(a.scale);
    r.w_post = reinterpret_cast<const float4*>(a.w_post);
    r.b_post = reinterpret_cast<const float4*>(a.b_post);
    r.dscale = reinterpret_cast<float4*>(a.dscale);
    r.dw_post = reinterpret_cast<float4*>(a.dw_post);
    r.db_post = reinterpret_cast<float4*>(a.db_post);
    r.dw_pre = reinterpret_cast<float4*>(a.dw_pre);
    r.db_pre = reinterpret_cast<float4*>(a.db_pre);
    BIMASK_CUDA_OK(launch_pdl(residual_reduce_kernel, (unsigned)((r.C4 + 7) / 8), 256, 0, s, r));
    count_launch();
  }
  if (p.gate_sums != nullptr) {
    const long long ctas = (b.gates * (a.C / 4) + 255) / 256, most = 8ll * sm_count();
    BIMASK_CUDA_OK(launch_pdl(gate_reduce_kernel, (unsigned)(ctas < most ? ctas : most), 256, 0, s, reinterpret_cast<const float4*>(p.gate_sums),
                              b.units_per_span, b.gates, a.C / 4, reinterpret_cast<uint2*>(a.dgate), a.gate_pitch / 4));
    count_launch();
  }
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

}  // namespace bimask
