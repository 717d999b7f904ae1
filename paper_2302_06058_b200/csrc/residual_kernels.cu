// The residual junction between two blocks of a network (norm after a block, dropout, gate, residual scale, norm before the
// next block), its gradient, and dropout alone.  All of them stream: every matrix is read once and written once, a row stays
// in the registers of the warps that share it, and the statistics are exchanged by shuffles and one barrier per norm.
#include "dropout.cuh"
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
  const DropKey key = drop_key(d);
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
        if (d.thr != 0u) drop8(p, (unsigned long long)i, key, d.thr, d.scale);
        store8<F32>(y, i, p);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Rows.  W warps share a row; thread l of the 32 W takes blocks l, l + 32 W, ... (V of them) of eight columns.  G such
// groups in a CTA work on rows of their own and never meet (named barriers).
// ------------------------------------------------------------------------------------------
struct ResidualParams {
  int T, C8, warps;                  // warps per row
  int post, pre;
  float eps_post, eps_pre, alpha, inv_c;
  int gate_span;                     // 0: no gate
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
  float* sums;                       // [CTAs][wanted arrays][C]
  float* gate_sums;                  // [units][C]
  int want;                          // bits: SUM_* arrays that are wanted
  int branch;                        // a gradient of the branch is wanted
  int unit_rows, units_per_span;     // rows that a group takes at a time, such units in a gate row's span
};

__device__ __forceinline__ void group_sync(int group, int warps) {
  if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(32 * warps) : "memory");
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
__device__ __forceinline__ float sum16(float v) {         // over the lanes' low four bits
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}
__device__ __forceinline__ float horizontal(Pair v) {
  float a, b;
  act::split(v, a, b);
  return a + b;
}

// eight fp32 parameters of block c, or a constant
__device__ __forceinline__ void param8(const float* base, int c, float otherwise, Pair (&p)[4]) {
  if (base != nullptr) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(base) + 2 * c), b = __ldg(reinterpret_cast<const float4*>(base) + 2 * c + 1);
    p[0] = act::pair(a.x, a.y); p[1] = act::pair(a.z, a.w); p[2] = act::pair(b.x, b.y); p[3] = act::pair(b.z, b.w);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = act::both(otherwise);
  }
}

struct Row {                                              // a thread's place in its row
  int lane, warp, group, warps, turn;
  float inv_count;                                        // 1 / columns of the row that this warp holds
  float peer_count;                                       // columns that warp lane % 16 of the group holds
  float2* red;                                            // the group's [2][16]
};

__device__ __forceinline__ float columns_of_warp(int warp, int warps, int V, int C8) {
  int n = 0;
  for (int j = 0; j < V; ++j) n += min(max(C8 - 32 * (warp + j * warps), 0), 32);
  return 8.f * (float)n;
}

__device__ __forceinline__ Row make_row(int warps, int V, int C8, float2* red) {
  Row r;
  const int w = threadIdx.x >> 5;
  r.lane = threadIdx.x & 31;
  r.group = w / warps;
  r.warp = w - r.group * warps;
  r.warps = warps;
  r.turn = 0;
  r.inv_count = 1.f / fmaxf(columns_of_warp(r.warp, warps, V, C8), 1.f);
  r.peer_count = (r.lane & 15) < warps ? columns_of_warp(r.lane & 15, warps, V, C8) : 0.f;
  r.red = red + 32 * r.group;
  return r;
}

// Every warp of the group hands in a pair; lane i of each warp gets warp i % 16's (zero past the last).  Two buffers in
// turn: a warp that writes one has passed the barrier of the other, before which everybody had read this one.
__device__ __forceinline__ float2 exchange(Row& r, float2 mine) {
  float2* buf = r.red + 16 * r.turn;
  r.turn ^= 1;
  if (r.lane == 0) buf[r.warp] = mine;
  group_sync(r.group, r.warps);
  const int i = r.lane & 15;
  return i < r.warps ? buf[i] : make_float2(0.f, 0.f);
}

// Mean and 1 / deviation of a row.  The squares are taken about each warp's own mean, and the warps are put together by
// M = sum M_w + sum n_w (m_w - m)^2: one exchange, and no difference of large squares.  rms: all about zero.
template <int V>
__device__ __forceinline__ float2 row_stats(const Pair (&v)[V][4], const bool (&ok)[V], int kind, float eps, float inv_c, Row& r) {
  const bool layer = kind == BIMASK_NORM_LAYER;
  float mean = 0.f;
  if (layer) {
    Pair a = act::both(0.f);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (ok[j]) a = act::add2(a, act::add2(act::add2(v[j][0], v[j][1]), act::add2(v[j][2], v[j][3])));
    mean = warp_sum(horizontal(a)) * r.inv_count;
  }
  Pair q = act::both(0.f);
  const Pair shift = act::both(-mean);
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (ok[j])
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Pair d = act::add2(v[j][k], shift);
        q = act::fma2(d, d, q);
      }
  float sq = warp_sum(horizontal(q));
  if (r.warps > 1) {
    const float2 e = exchange(r, make_float2(mean, sq));
    float part = e.y;
    if (layer) {
      mean = sum16(r.peer_count * e.x) * inv_c;
      const float d = e.x - mean;
      part = fmaf(r.peer_count * d, d, part);
    }
    sq = sum16(part);
  }
  return make_float2(mean, 1.f / sqrtf(fmaf(sq, inv_c, eps)));
}

// (v - mean) rstd w + b.  The difference first: mean * rstd could be far larger than the result.
__device__ __forceinline__ void normalise(Pair (&v)[4], float2 st) {
  const Pair shift = act::both(-st.x), rstd = act::both(st.y);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = act::mul2(act::add2(v[k], shift), rstd);
}
__device__ __forceinline__ void affine(Pair (&v)[4], const float* w, const float* b, int c) {
  Pair p[4];
  if (w != nullptr) {
    param8(w, c, 1.f, p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = act::mul2(v[k], p[k]);
  }
  if (b != nullptr) {
    param8(b, c, 0.f, p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = act::add2(v[k], p[k]);
  }
}

constexpr int FWD_THREADS = 512;

template <int V, bool F32>
__global__ void __launch_bounds__(FWD_THREADS)
residual_fwd_kernel(const ResidualParams p) {
  __shared__ float2 red[16 * 32];
  pdl_launch_dependents();
  pdl_wait();
  const DropKey key = drop_key(p.drop);
  Row r = make_row(p.warps, V, p.C8, red);
  const int groups = blockDim.x / (32 * p.warps);
  const int l = 32 * r.warp + r.lane;
  int col[V];
  bool ok[V];
#pragma unroll
  for (int j = 0; j < V; ++j) { col[j] = l + 32 * j * p.warps; ok[j] = col[j] < p.C8; }
  for (long long t = (long long)blockIdx.x * groups + r.group; t < p.T; t += (long long)gridDim.x * groups) {
    const long long row = t * p.C8;
    Vec8<F32> xv[V];
    Vec8<false> yv[V], gv[V];
    const long long grow = p.gate_span != 0 ? (t / p.gate_span) * p.gate_pitch8 : 0;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (ok[j]) {
        xv[j] = load8<F32>(p.x, row + col[j]);
        if (p.y != nullptr) yv[j] = load8<false>(p.y, row + col[j]);
        if (p.gate_span != 0) gv[j].w[0] = __ldg(p.gate + grow + col[j]);
      }
    Pair v[V][4];
    if (p.y != nullptr) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (ok[j]) unpack8<false>(yv[j], v[j]);
      }
      if (p.post != BIMASK_NORM_NONE) {
        const float2 st = row_stats<V>(v, ok, p.post, p.eps_post, p.inv_c, r);
        if (p.stats_post != nullptr && l == 0) p.stats_post[t] = st;
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j]) { normalise(v[j], st); affine(v[j], p.w_post, p.b_post, col[j]); }
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (ok[j]) {
          if (p.drop.thr != 0u) drop8(v[j], (unsigned long long)(row + col[j]), key, p.drop.thr, p.drop.scale);
          if (p.gate_span != 0) {
            Pair g[4];
            unpack8<false>(gv[j], g);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[j][k] = act::mul2(v[j][k], g[k]);
          }
          affine(v[j], p.scale, nullptr, col[j]);
        }
    }
    const Pair alpha = act::both(p.alpha);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (ok[j]) {
        Pair x[4];
        unpack8<F32>(xv[j], x);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j][k] = p.y != nullptr ? act::fma2(x[k], alpha, v[j][k]) : act::mul2(x[k], alpha);
        if (p.xo != nullptr) store8<F32>(p.xo, row + col[j], v[j]);
      }
    if (p.pre != BIMASK_NORM_NONE) {
      const float2 st = row_stats<V>(v, ok, p.pre, p.eps_pre, p.inv_c, r);
      if (p.stats_pre != nullptr && l == 0) p.stats_pre[t] = st;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (ok[j]) {
          normalise(v[j], st);
          affine(v[j], p.w_pre, p.b_pre, col[j]);
          store8<false>(p.n, row + col[j], v[j]);
        }
    }
  }
}

// ------------------------------------------------------------------------------------------
// Gradient.  With m the dropout's multiplier, xh and yh the normalised values and u = yh w_post + b_post:
//   D  = dx' + rstd (g - mean(g) [layer] - xh mean(g xh)),  g = w_pre dn;        dx = alpha D
//   e  = m gate D;  dy the same norm formula on scale e w_post;                   dgate = m D scale u
// and four column sums carry every parameter's gradient: G1 = sum dn xh (w_pre), G2 = sum dn (b_pre), A = sum e yh, B = sum e:
//   dw_post = scale A,  db_post = scale B,  dscale = w_post A + b_post B.
// A thread owns its columns for good and keeps the sums in registers; each CTA leaves one row of partial sums.
// ------------------------------------------------------------------------------------------
constexpr int BWD_THREADS = 512;
enum { SUM_A = 1, SUM_B = 2, SUM_G1 = 4, SUM_G2 = 8 };

__device__ __forceinline__ float2 row_sums(float a, float b, bool two, Row& r) {
  a = warp_sum(a);
  if (two) b = warp_sum(b);
  if (r.warps > 1) {
    const float2 e = exchange(r, make_float2(a, b));
    a = sum16(e.x);
    if (two) b = sum16(e.y);
  }
  return make_float2(a, b);
}

// One gate row's span (or any row without one) is worked off in units of consecutive rows.
struct Unit { long long begin, end; };
__device__ __forceinline__ Unit unit_rows(const ResidualParams& p, long long k) {
  if (p.units_per_span == 0) return {k, k + 1};
  const long long span = k / p.units_per_span, part = k - span * p.units_per_span;
  const long long begin = span * p.gate_span + part * p.unit_rows;
  const long long end = min(min(begin + p.unit_rows, (span + 1) * p.gate_span), (long long)p.T);
  return {begin, end};
}

template <int V, bool F32, bool SPAN>
__global__ void __launch_bounds__(BWD_THREADS, 1)
residual_bwd_kernel(const ResidualParams p, long long units) {
  __shared__ float2 red[16 * 32];
  extern __shared__ float4 fold[];                        // [threads][2 V] (one array at a time)
  pdl_launch_dependents();
  pdl_wait();
  const DropKey key = drop_key(p.drop);
  Row r = make_row(p.warps, V, p.C8, red);
  const int groups = blockDim.x / (32 * p.warps);
  const int l = 32 * r.warp + r.lane;
  int col[V];
  bool ok[V];
  Pair sums[4][V][4], fsum[SPAN ? V : 1][4];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    col[j] = l + 32 * j * p.warps;
    ok[j] = col[j] < p.C8;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int k = 0; k < 4; ++k) sums[a][j][k] = act::both(0.f);
  }
  for (long long unit = (long long)blockIdx.x * groups + r.group; unit < units; unit += (long long)gridDim.x * groups) {
    const Unit rows = unit_rows(p, unit);
    if (SPAN)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) fsum[j][k] = act::both(0.f);
    for (long long t = rows.begin; t < rows.end; ++t) {
      const long long row = t * p.C8;
      Vec8<F32> dxv[V], xv[V];
      Vec8<false> dnv[V], yv[V], gv[V];
      const long long grow = p.gate_span != 0 ? (t / p.gate_span) * p.gate_pitch8 : 0;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (ok[j]) {
          if (p.dxo != nullptr) dxv[j] = load8<F32>(p.dxo, row + col[j]);
          if (p.pre != BIMASK_NORM_NONE) {
            dnv[j] = load8<false>(p.dn, row + col[j]);
            xv[j] = load8<F32>(p.xo, row + col[j]);
          }
          if (p.y != nullptr) yv[j] = load8<false>(p.y, row + col[j]);
          if (p.gate_span != 0) gv[j].w[0] = __ldg(p.gate + grow + col[j]);
        }
      Pair D[V][4];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (p.dxo != nullptr && ok[j]) unpack8<F32>(dxv[j], D[j]);
        else
#pragma unroll
          for (int k = 0; k < 4; ++k) D[j][k] = act::both(0.f);
      }
      if (p.pre != BIMASK_NORM_NONE) {
        const float2 st = p.stats_pre[t];
        Pair xh[V][4], g[V][4];
        Pair s1 = act::both(0.f), s2 = act::both(0.f);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j]) {
            unpack8<F32>(xv[j], xh[j]);
            normalise(xh[j], st);
            unpack8<false>(dnv[j], g[j]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              sums[2][j][k] = act::fma2(g[j][k], xh[j][k], sums[2][j][k]);
              sums[3][j][k] = act::add2(sums[3][j][k], g[j][k]);
            }
            affine(g[j], p.w_pre, nullptr, col[j]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              s1 = act::fma2(g[j][k], xh[j][k], s1);
              s2 = act::add2(s2, g[j][k]);
            }
          }
        const bool layer = p.pre == BIMASK_NORM_LAYER;
        const float2 c = row_sums(horizontal(s1), horizontal(s2), layer, r);
        const Pair c1 = act::both(-c.x * p.inv_c), c2 = act::both(layer ? -c.y * p.inv_c : 0.f), rstd = act::both(st.y);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j])
#pragma unroll
            for (int k = 0; k < 4; ++k) D[j][k] = act::fma2(act::fma2(xh[j][k], c1, act::add2(g[j][k], c2)), rstd, D[j][k]);
      }
      if (p.dx != nullptr) {
        const Pair alpha = act::both(p.alpha);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j]) {
            Pair o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = act::mul2(D[j][k], alpha);
            store8<F32>(p.dx, row + col[j], o);
          }
      }
      if (!p.branch) continue;
      Pair yh[V][4];
      float2 st = make_float2(0.f, 1.f);
      if (p.post != BIMASK_NORM_NONE) st = p.stats_post[t];
      Pair s1 = act::both(0.f), s2 = act::both(0.f);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (ok[j]) {
          if (p.y != nullptr) unpack8<false>(yv[j], yh[j]);
          else                                            // not needed: any value
#pragma unroll
            for (int k = 0; k < 4; ++k) yh[j][k] = act::both(0.f);
          if (p.post != BIMASK_NORM_NONE) normalise(yh[j], st);
          if (p.drop.thr != 0u) drop8(D[j], (unsigned long long)(row + col[j]), key, p.drop.thr, p.drop.scale);
          if (p.gate_span != 0) {
            Pair g[4], u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = yh[j][k];
            affine(u, p.w_post, p.b_post, col[j]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (SPAN) fsum[j][k] = act::fma2(D[j][k], u[k], fsum[j][k]);
              else u[k] = act::mul2(D[j][k], u[k]);
            }
            if (!SPAN && p.dgate != nullptr) {
              affine(u, p.scale, nullptr, col[j]);
              store8<false>(p.dgate, grow + col[j], u);
            }
            unpack8<false>(gv[j], g);
#pragma unroll
            for (int k = 0; k < 4; ++k) D[j][k] = act::mul2(D[j][k], g[k]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            sums[0][j][k] = act::fma2(D[j][k], yh[j][k], sums[0][j][k]);
            sums[1][j][k] = act::add2(sums[1][j][k], D[j][k]);
          }
          affine(D[j], p.scale, nullptr, col[j]);
          if (p.post != BIMASK_NORM_NONE) {
            affine(D[j], p.w_post, nullptr, col[j]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              s1 = act::fma2(D[j][k], yh[j][k], s1);
              s2 = act::add2(s2, D[j][k]);
            }
          }
        }
      if (p.post != BIMASK_NORM_NONE) {
        const bool layer = p.post == BIMASK_NORM_LAYER;
        const float2 c = row_sums(horizontal(s1), horizontal(s2), layer, r);
        const Pair c1 = act::both(-c.x * p.inv_c), c2 = act::both(layer ? -c.y * p.inv_c : 0.f), rstd = act::both(st.y);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j])
#pragma unroll
            for (int k = 0; k < 4; ++k) D[j][k] = act::mul2(act::fma2(yh[j][k], c1, act::add2(D[j][k], c2)), rstd);
      }
      if (p.dy != nullptr) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (ok[j]) store8<false>(p.dy, row + col[j], D[j]);
      }
    }
    if (SPAN) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (ok[j]) store8<true>(p.gate_sums, unit * p.C8 + col[j], fsum[j]);
    }
  }
  // the groups' sums are added through shared memory, in their order
  int slot = 0;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    if (!(p.want & (1 << a))) continue;                   // the same for every thread
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (groups > 1) {
        __syncthreads();
        const Vec8<true> v = pack8<true>(sums[a][j]);
        reinterpret_cast<uint4*>(fold)[2 * threadIdx.x] = v.w[0];
        reinterpret_cast<uint4*>(fold)[2 * threadIdx.x + 1] = v.w[1];
        __syncthreads();
      }
      if (r.group == 0 && ok[j]) {
        for (int g = 1; g < groups; ++g) {
          Pair q[4];
          unpack8<true>(load8<true>(fold, l + 32 * p.warps * g), q);
#pragma unroll
          for (int k = 0; k < 4; ++k) sums[a][j][k] = act::add2(sums[a][j][k], q[k]);
        }
        store8<true>(p.sums, ((long long)blockIdx.x * __popc(p.want) + slot) * p.C8 + col[j], sums[a][j]);
      }
    }
    ++slot;
  }
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

// dgate of a row that serves a span of tokens: scale times the sum of its units, in order.
__global__ void __launch_bounds__(256)
gate_reduce_kernel(const float4* __restrict__ sums, int units_per_span, long long gates, int C4, const float4* __restrict__ scale,
                   uint2* dgate, long long pitch4) {
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
    if (scale != nullptr) acc = mul4(acc, __ldg(scale + c));
    dgate[g * pitch4 + c] = make_uint2(pack_bf16_f(acc.x, acc.y), pack_bf16_f(acc.z, acc.w));
  }
}

// ---- plans --------------------------------------------------------------------------------------
struct BwdPlan {
  int vec, warps, groups, threads;                        // blocks of eight per thread, warps per row, rows side by side
  int slots;                                              // CTAs
  int unit_rows, units_per_span;                          // with a gate row per span: rows of a unit
  long long units, gates;
};

BwdPlan plan_bwd(int T, int C, int span) {
  BwdPlan b;
  const int C8 = C / 8;
  b.vec = C8 > 512 ? 2 : 1;
  b.warps = (C8 + 32 * b.vec - 1) / (32 * b.vec);
  b.groups = BWD_THREADS / (32 * b.warps);
  b.threads = 32 * b.warps * b.groups;
  b.unit_rows = 1;
  b.units_per_span = 0;
  b.units = T;
  b.gates = 0;
  if (span > 1) {
    const long long all = (long long)PLAN_SMS * b.groups;
    const int len = span < T ? span : T;
    b.gates = (T + (long long)span - 1) / span;
    b.unit_rows = (int)((T + all - 1) / all);
    if (b.unit_rows > len) b.unit_rows = len;
    b.units_per_span = (len + b.unit_rows - 1) / b.unit_rows;
    b.units = b.gates * b.units_per_span;
  }
  const long long ctas = (b.units + b.groups - 1) / b.groups;
  b.slots = (int)(ctas < PLAN_SMS ? ctas : PLAN_SMS);
  return b;
}

}  // namespace

static size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Scratch of the backward pass: the CTAs' partial sums (four arrays at most), then the units' of a spanned gate, each for T
// tokens and every smaller number.  With spans there are at most 2 T units (a last span that is not full has its empty ones),
// and at most two per group of warps and one more per gate row.
static size_t column_sums_bytes(int T, int C, int span) {
  const BwdPlan b = plan_bwd(1, C, 0);
  const long long ctas = ((span > 1 ? 2ll : 1ll) * T + b.groups - 1) / b.groups;
  return up256((size_t)(ctas < PLAN_SMS ? ctas : PLAN_SMS) * 4 * C * sizeof(float));
}
size_t residual_workspace_bytes(int T, int C, int span) {
  size_t bytes = column_sums_bytes(T, C, span);
  if (span > 1) {
    const long long gates = (T + (long long)span - 1) / span, most = 2ll * PLAN_SMS * plan_bwd(1, C, 0).groups + gates;
    bytes += (size_t)(most < 2ll * T ? most : 2ll * T) * C * sizeof(float);
  }
  return bytes;
}

DropParams drop_params(const bimask_dropout_args* d) {
  DropParams p = {};
  p.scale = 1.f;
  if (d == nullptr) return p;
  p.thr = drop_threshold(d->p);
  p.scale = (float)(65536.0 / (65536.0 - p.thr));
  p.key0 = (uint32_t)d->seed;
  p.key1 = (uint32_t)(d->seed >> 32);
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
  p.T = a.T;
  p.C8 = a.C / 8;
  p.post = a.post;
  p.pre = a.pre;
  p.eps_post = a.eps_post;
  p.eps_pre = a.eps_pre;
  p.alpha = a.alpha;
  p.inv_c = 1.f / (float)a.C;
  p.gate_span = a.gate != nullptr ? a.gate_span : 0;
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
  const int vec = p.C8 > 32 ? 2 : 1;
  p.warps = (p.C8 + 32 * vec - 1) / (32 * vec);
  const int groups = p.warps < 8 ? 8 / p.warps : 1, threads = 32 * p.warps * groups;
  const long long ctas = ((long long)a.T + groups - 1) / groups, most = (long long)sm_count() * (threads > 256 ? 2 : 4);
  auto run = [&](auto kern) { return launch_pdl(kern, (unsigned)(ctas < most ? ctas : most), threads, 0, s, p); };
  const bool f32 = a.stream_type == BIMASK_TYPE_F32;
  BIMASK_CUDA_OK(vec == 1 ? (f32 ? run(residual_fwd_kernel<1, true>) : run(residual_fwd_kernel<1, false>))
                          : (f32 ? run(residual_fwd_kernel<2, true>) : run(residual_fwd_kernel<2, false>)));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_residual_bwd(const bimask_residual_args& a, cudaStream_t s) {
  ResidualParams p = residual_params(a);
  const bool spanned = a.dgate != nullptr && p.gate_span > 1;
  const BwdPlan b = plan_bwd(a.T, a.C, spanned ? p.gate_span : 1);
  p.branch = a.dy || a.dgate || a.dscale || a.dw_post || a.db_post;
  p.warps = b.warps;
  p.unit_rows = b.unit_rows;
  p.units_per_span = b.units_per_span;
  const bool scale = a.dscale != nullptr;
  p.want = (a.dw_post || scale ? SUM_A : 0) | (a.db_post || (scale && a.b_post) ? SUM_B : 0) | (a.dw_pre ? SUM_G1 : 0) | (a.db_pre ? SUM_G2 : 0);
  p.sums = reinterpret_cast<float*>(a.ws);
  if (spanned) p.gate_sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.ws) + column_sums_bytes(a.T, a.C, p.gate_span));
  auto run = [&](auto kern) { return launch_pdl(kern, (unsigned)b.slots, b.threads, (size_t)b.threads * 32, s, p, b.units); };
  auto pick = [&](auto f32, auto span) {
    constexpr bool F = decltype(f32)::value, S = decltype(span)::value;
    return b.vec == 1 ? run(residual_bwd_kernel<1, F, S>) : run(residual_bwd_kernel<2, F, S>);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  const bool f32 = a.stream_type == BIMASK_TYPE_F32;
  BIMASK_CUDA_OK(f32 ? (spanned ? pick(Yes(), Yes()) : pick(Yes(), No())) : (spanned ? pick(No(), Yes()) : pick(No(), No())));
  count_launch();
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
                              b.units_per_span, b.gates, a.C / 4, reinterpret_cast<const float4*>(a.scale), reinterpret_cast<uint2*>(a.dgate),
                              a.gate_pitch / 4));
    count_launch();
  }
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

}  // namespace bimask
