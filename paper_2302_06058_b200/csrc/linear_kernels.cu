// The streaming kernels around a linear layer: 8-bit activation checkpoints written and read, and the gradient through
// the activation and the bias.  All three are bound by HBM.
#include "act_math.cuh"

namespace bimask {

namespace {

// ------------------------------------------------------------------------------------------
// Checkpoint of a bf16 matrix.  A thread takes 16 channels (32 bytes in, 16 out): a block of 32 is a pair of
// neighbouring lanes, so its maximum is one shuffle away and every store is a whole 16 bytes.  Blocks never straddle
// rows (C % 32 == 0): the matrix is a flat stream of C / 32 blocks per token.  Bound by HBM: 8192 x 16384 in 62 us,
// 406 MB at 6.5 TB/s.
// ------------------------------------------------------------------------------------------
constexpr int STREAM_THREADS = 256;

__global__ void __launch_bounds__(STREAM_THREADS)
ckpt_pack_kernel(const uint4* __restrict__ x, long long halves, uint4* __restrict__ q, uint8_t* __restrict__ s) {
  pdl_launch_dependents();
  pdl_wait();
  const long long step = (long long)gridDim.x * STREAM_THREADS;
  // the loop runs for whole warps: `halves` is even, and the lane past the end (if any) is the pair's other half or more
  for (long long i = (long long)blockIdx.x * STREAM_THREADS + threadIdx.x; (i & ~31ll) < halves; i += step) {
    uint4 v[2] = {};
    if (i < halves) { v[0] = __ldg(x + 2 * i); v[1] = __ldg(x + 2 * i + 1); }
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t m2 = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m2 = __vmaxu2(m2, w[k] & 0x7FFF7FFFu);
    m2 = __vmaxu2(m2, __shfl_xor_sync(0xFFFFFFFFu, m2, 1));
    const uint32_t h = max(m2 & 0xFFFFu, m2 >> 16);
    const uint32_t sc = ckpt::scale_of(h);
    const float inv = ckpt::inverse_scale(sc);
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = __byte_perm(ckpt::round_bits(bf16_lo(w[2 * k]), inv), ckpt::round_bits(bf16_hi(w[2 * k]), inv), 0x0040);
      const uint32_t b = __byte_perm(ckpt::round_bits(bf16_lo(w[2 * k + 1]), inv), ckpt::round_bits(bf16_hi(w[2 * k + 1]), inv), 0x0040);
      o[k] = __byte_perm(a, b, 0x5410);
    }
    if (i < halves) {
      q[i] = make_uint4(o[0], o[1], o[2], o[3]);
      if (!(i & 1)) s[i >> 1] = (uint8_t)sc;
    }
  }
}

// The values of a checkpoint, through an activation or as they are.  Eight channels per thread and step, so that the 16-byte
// stores of a warp are contiguous (16 channels as two stores of every other 16 bytes: 84 us for 8192 x 16384 through
// an activation, now 76: 5.3 TB/s); two steps' bytes are loaded at a time.
template <int ACT>
__global__ void __launch_bounds__(STREAM_THREADS)
ckpt_unpack_kernel(const uint2* __restrict__ q, const uint8_t* __restrict__ s, long long eighths, uint4* __restrict__ x) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int U = 2;
  const long long step = (long long)gridDim.x * STREAM_THREADS;
  for (long long i0 = (long long)blockIdx.x * STREAM_THREADS + threadIdx.x; i0 < eighths; i0 += U * step) {
    uint2 v[U];
    uint32_t sb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * step;
      if (i < eighths) { v[u] = __ldg(q + i); sb[u] = __ldg(s + (i >> 2)); }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * step;
      if (i < eighths) {
        const act::Pair sc = act::both(ckpt::scale_value(sb[u]));
        act::Pair z[4];
        ckpt::decode4(v[u].x, sc, z); ckpt::decode4(v[u].y, sc, z + 2);
        x[i] = make_uint4(pack_bf16_p(act::value2<ACT>(z[0])), pack_bf16_p(act::value2<ACT>(z[1])), pack_bf16_p(act::value2<ACT>(z[2])),
                          pack_bf16_p(act::value2<ACT>(z[3])));
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// dZ = dY act'(Z) and db = column sums of dZ in fp32.  A thread owns two groups of eight columns for good, half a tile
// apart (so that a warp's 16-byte loads and stores are contiguous; sixteen values share the polynomial's coefficients)
// and walks over rows, the next three already loading, so the column sums stay in registers; the rows that a CTA takes side
// by side are added through shared memory at its end, in a fixed order, and each CTA leaves one row of partial sums for
// bias_reduce_kernel (no atomics: the result does not depend on timing).  8192 x 16384 in 127 us on the device, 5.3 TB/s
// (the bias gradient alone 47 us); 12608 x 1536 in 22 + 3 us: there the launches and the uneven end of the CTAs are a
// third.  CTA (x, y): column tile x of 2 * half groups of eight, row slot y of gridDim.y.
// ------------------------------------------------------------------------------------------
constexpr int ACTBWD_MAX_THREADS = 512;

template <int ACT>
__global__ void __launch_bounds__(ACTBWD_MAX_THREADS, 1)
act_bwd_kernel(const uint4* dY, const uint2* __restrict__ zq, const uint8_t* __restrict__ zs, int T, int C8, int half, int rows,
               uint4* dZ /* may be dY */, float4* __restrict__ partial) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float red[ACTBWD_MAX_THREADS][17];           // 17: neighbouring threads fall into different banks
  const int g = threadIdx.x / half, lc = threadIdx.x - g * half;
  const int ca = blockIdx.x * 2 * half + lc, cb = ca + half;
  const bool a_ok = g < rows && ca < C8, b_ok = g < rows && cb < C8;
  act::Pair sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = act::both(0.f);
  if (a_ok) {
    const long long stride = (long long)rows * gridDim.y;
    constexpr int U = 3;                                  // rows loaded ahead of the one being worked on
    uint4 d[U][2];
    uint2 z[U][2];
    uint32_t sc[U][2];
    auto fetch = [&](int u, long long t) {
      if (t < T) {
        const long long at = t * C8 + ca;
        d[u][0] = dY[at];
        if (ACT != BIMASK_ACT_NONE) { z[u][0] = __ldg(zq + at); sc[u][0] = __ldg(zs + (at >> 2)); }   // C8 % 4 == 0: (t C8 + c) / 4 is the block
        if (b_ok) {
          d[u][1] = dY[at + half];
          if (ACT != BIMASK_ACT_NONE) { z[u][1] = __ldg(zq + at + half); sc[u][1] = __ldg(zs + ((at + half) >> 2)); }
        }
      }
    };
    long long t = (long long)blockIdx.y * rows + g;
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(u, t + u * stride);
    while (t < T) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (t >= T) break;
        act::Pair v[8], a[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v[4 * h] = bf16_pair(d[u][h].x); v[4 * h + 1] = bf16_pair(d[u][h].y);
          v[4 * h + 2] = bf16_pair(d[u][h].z); v[4 * h + 3] = bf16_pair(d[u][h].w);
          if constexpr (ACT != BIMASK_ACT_NONE) {
            const act::Pair s = act::both(ckpt::scale_value(sc[u][h]));
            ckpt::decode4(z[u][h].x, s, a + 4 * h); ckpt::decode4(z[u][h].y, s, a + 4 * h + 2);
          }
        }
        fetch(u, t + U * stride);
        if constexpr (ACT != BIMASK_ACT_NONE) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = act::mul2(v[k], act::slope2<ACT>(a[k]));
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = act::add2(sum[k], v[k]);
        if (dZ != nullptr) {
          uint4* out = dZ + t * C8 + ca;
          out[0] = make_uint4(pack_bf16_p(v[0]), pack_bf16_p(v[1]), pack_bf16_p(v[2]), pack_bf16_p(v[3]));
          if (b_ok) out[half] = make_uint4(pack_bf16_p(v[4]), pack_bf16_p(v[5]), pack_bf16_p(v[6]), pack_bf16_p(v[7]));
        }
        t += stride;
      }
    }
  }
  if (partial == nullptr) return;
  float s[16];
#pragma unroll
  for (int k = 0; k < 8; ++k) act::split(sum[k], s[2 * k], s[2 * k + 1]);
  if (rows > 1) {
#pragma unroll
    for (int k = 0; k < 16; ++k) red[threadIdx.x][k] = s[k];
    __syncthreads();
    if (g == 0)
      for (int r = 1; r < rows; ++r)
#pragma unroll
        for (int k = 0; k < 16; ++k) s[k] += red[r * half + lc][k];
  }
  if (g == 0 && a_ok) {
    float4* out = partial + (size_t)blockIdx.y * (2 * C8) + 2 * ca;
    out[0] = make_float4(s[0], s[1], s[2], s[3]);
    out[1] = make_float4(s[4], s[5], s[6], s[7]);
    if (b_ok) {
      out[2 * half] = make_float4(s[8], s[9], s[10], s[11]);
      out[2 * half + 1] = make_float4(s[12], s[13], s[14], s[15]);
    }
  }
}

// db[c] = sum over the partial rows, in a fixed order: a CTA covers 8 float4 columns, its 32 row slots take the rows in
// turn and are added through shared memory.
__global__ void __launch_bounds__(256)
bias_reduce_kernel(const float4* __restrict__ partial, int nrows, int n4, float4* __restrict__ out) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float4 red[32][8];
  const int col = threadIdx.x & 7, slot = threadIdx.x >> 3;
  const int e = blockIdx.x * 8 + col;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (e < n4) {
#pragma unroll 8
    for (int r = slot; r < nrows; r += 32) {
      const float4 v = partial[(size_t)r * n4 + e];
      acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
  }
  red[slot][col] = acc;
  __syncthreads();
#pragma unroll
  for (int half = 16; half >= 1; half >>= 1) {
    if (slot < half) {
      const float4 v = red[slot + half][col];
      acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
      red[slot][col] = acc;
    }
    __syncthreads();
  }
  if (slot == 0 && e < n4) out[e] = acc;
}

int stream_grid(long long items) {
  const long long ctas = (items + STREAM_THREADS - 1) / STREAM_THREADS;
  const long long most = 32ll * sm_count();               // four rounds of 2048 threads per SM: SMs far from a memory part take fewer
  return (int)(ctas < most ? ctas : most);
}

struct ActBwdPlan { int half, tiles, rows, threads, slots; };

// Columns: one tile when a row has at most 4096 columns, else tiles of about that size.  One CTA of up to 512 threads per
// SM: as many rows side by side as fit, so that few rows of partial sums are left over.
ActBwdPlan plan_act_bwd(int T, int C) {
  ActBwdPlan p;
  const int C8 = C / 8;
  p.tiles = (C8 + 511) / 512;
  p.half = ((C8 + p.tiles - 1) / p.tiles + 1) / 2;
  p.rows = ACTBWD_MAX_THREADS / p.half;
  if (p.rows > T) p.rows = T;
  p.threads = (p.half * p.rows + 31) / 32 * 32;
  p.slots = PLAN_SMS / p.tiles;
  const int most = (T + p.rows - 1) / p.rows;
  if (p.slots > most) p.slots = most;
  if (p.slots < 1) p.slots = 1;
  return p;
}

}  // namespace

size_t act_bwd_partial_bytes(int T, int C) { return (size_t)plan_act_bwd(T, C).slots * C * sizeof(float); }

int launch_ckpt_pack(const uint16_t* x, int T, int C, int8_t* q, uint8_t* s, cudaStream_t st) {
  const long long halves = (long long)T * (C / 16);
  BIMASK_CUDA_OK(launch_pdl(ckpt_pack_kernel, stream_grid(halves), STREAM_THREADS, 0, st, reinterpret_cast<const uint4*>(x), halves,
                            reinterpret_cast<uint4*>(q), s));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_ckpt_unpack(const int8_t* q, const uint8_t* s, int act, int T, int C, uint16_t* x, cudaStream_t st) {
  const long long eighths = (long long)T * (C / 8);
  auto run = [&](auto kern) {
    return launch_pdl(kern, stream_grid(eighths), STREAM_THREADS, 0, st, reinterpret_cast<const uint2*>(q), s, eighths,
                      reinterpret_cast<uint4*>(x));
  };
  cudaError_t e;
  switch (act) {
    case BIMASK_ACT_RELU: e = run(ckpt_unpack_kernel<BIMASK_ACT_RELU>); break;
    case BIMASK_ACT_GELU: e = run(ckpt_unpack_kernel<BIMASK_ACT_GELU>); break;
    case BIMASK_ACT_GELU_TANH: e = run(ckpt_unpack_kernel<BIMASK_ACT_GELU_TANH>); break;
    case BIMASK_ACT_SILU: e = run(ckpt_unpack_kernel<BIMASK_ACT_SILU>); break;
    default: e = run(ckpt_unpack_kernel<BIMASK_ACT_NONE>); break;
  }
  BIMASK_CUDA_OK(e);
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_act_bwd(const uint16_t* dY, const int8_t* zq, const uint8_t* zs, int act, int T, int C, uint16_t* dZ, float* dbias,
                   float* partial, cudaStream_t st) {
  const ActBwdPlan p = plan_act_bwd(T, C);
  float* part = dbias == nullptr ? nullptr : p.slots == 1 ? dbias : partial;      // one slot: its row is the result
  auto run = [&](auto kern) {
    return launch_pdl(kern, dim3(p.tiles, p.slots), p.threads, 0, st, reinterpret_cast<const uint4*>(dY), reinterpret_cast<const uint2*>(zq),
                      zs, T, C / 8, p.half, p.rows, reinterpret_cast<uint4*>(dZ), reinterpret_cast<float4*>(part));
  };
  cudaError_t e;
  switch (act) {
    case BIMASK_ACT_RELU: e = run(act_bwd_kernel<BIMASK_ACT_RELU>); break;
    case BIMASK_ACT_GELU: e = run(act_bwd_kernel<BIMASK_ACT_GELU>); break;
    case BIMASK_ACT_GELU_TANH: e = run(act_bwd_kernel<BIMASK_ACT_GELU_TANH>); break;
    case BIMASK_ACT_SILU: e = run(act_bwd_kernel<BIMASK_ACT_SILU>); break;
    default: e = run(act_bwd_kernel<BIMASK_ACT_NONE>); break;
  }
  BIMASK_CUDA_OK(e);
  count_launch();
  if (dbias != nullptr && p.slots > 1) {
    BIMASK_CUDA_OK(launch_pdl(bias_reduce_kernel, (C / 4 + 7) / 8, 256, 0, st, reinterpret_cast<const float4*>(partial), p.slots, C / 4,
                              reinterpret_cast<float4*>(dbias)));
    count_launch();
  }
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

}  // namespace bimask
