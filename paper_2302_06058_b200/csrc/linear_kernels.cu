// The streaming kernels around a linear layer: 8-bit activation checkpoints written and read, and the gradient through
// the activation and the bias.  All three are bound by HBM.
#include "act_math.cuh"

namespace bimask {

namespace {

// ------------------------------------------------------------------------------------------
// Checkpoint of a bf16 matrix.  A thread takes 16 channels (32 bytes in, 16 out): a block of 32 is a pair of
// neighbouring lanes, so its maximum is one shuffle away and every store is a whole 16 bytes.  Blocks never straddle
// rows (C % 32 == 0): the matrix is a flat stream of C / 32 blocks per token.
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

// The values of a checkpoint, through an activation or as they are: 16 channels per thread.
template <int ACT>
__global__ void __launch_bounds__(STREAM_THREADS)
ckpt_unpack_kernel(const uint4* __restrict__ q, const uint8_t* __restrict__ s, long long halves, uint4* __restrict__ x) {
  pdl_launch_dependents();
  pdl_wait();
  const long long step = (long long)gridDim.x * STREAM_THREADS;
  for (long long i = (long long)blockIdx.x * STREAM_THREADS + threadIdx.x; i < halves; i += step) {
    const uint4 v = __ldg(q + i);
    const float sc = ckpt::scale_value(__ldg(s + (i >> 1)));
    float z[16];
    ckpt::decode4(v.x, sc, z); ckpt::decode4(v.y, sc, z + 4); ckpt::decode4(v.z, sc, z + 8); ckpt::decode4(v.w, sc, z + 12);
    uint32_t o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = pack_bf16_f(act::value<ACT>(z[2 * k]), act::value<ACT>(z[2 * k + 1]));
    x[2 * i] = make_uint4(o[0], o[1], o[2], o[3]);
    x[2 * i + 1] = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

// ------------------------------------------------------------------------------------------
// dZ = dY act'(Z) and db = column sums of dZ in fp32.  A thread owns eight columns for good and walks over rows, so the
// column sums stay in registers; the rows that a CTA takes side by side are added through shared memory at its end, in
// a fixed order, and each CTA leaves one row of partial sums for bias_reduce_kernel (no atomics: the result does not
// depend on timing).  CTA (x, y): column tile x of `tile8` groups of eight, row slot y of gridDim.y.
// ------------------------------------------------------------------------------------------
constexpr int ACTBWD_MAX_THREADS = 512;

template <int ACT>
__global__ void __launch_bounds__(ACTBWD_MAX_THREADS)
act_bwd_kernel(const uint4* dY, const uint2* __restrict__ zq, const uint8_t* __restrict__ zs, int T, int C8, int tile8, int rows,
               uint4* dZ /* may be dY */, float4* __restrict__ partial) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ float red[ACTBWD_MAX_THREADS][9];            // 9: neighbouring threads fall into different banks
  const int g = threadIdx.x / tile8, lc = threadIdx.x - g * tile8;
  const int c8 = blockIdx.x * tile8 + lc;
  const bool mine = g < rows && c8 < C8;
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = 0.f;
  if (mine) {
    const int stride = rows * (int)gridDim.y;
    constexpr int U = 4;                                  // rows in flight per thread
    for (long long t0 = (long long)blockIdx.y * rows + g; t0 < T; t0 += (long long)U * stride) {
      uint4 d[U];
      uint2 z[U];
      uint32_t sc[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long t = t0 + (long long)u * stride;
        if (t < T) {
          d[u] = dY[t * C8 + c8];
          if (ACT != BIMASK_ACT_NONE) { z[u] = __ldg(zq + t * C8 + c8); sc[u] = __ldg(zs + t * (C8 >> 2) + (c8 >> 2)); }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long t = t0 + (long long)u * stride;
        if (t < T) {
          float v[8] = {bf16_lo(d[u].x), bf16_hi(d[u].x), bf16_lo(d[u].y), bf16_hi(d[u].y),
                        bf16_lo(d[u].z), bf16_hi(d[u].z), bf16_lo(d[u].w), bf16_hi(d[u].w)};
          if (ACT != BIMASK_ACT_NONE) {
            float a[8];
            const float s = ckpt::scale_value(sc[u]);
            ckpt::decode4(z[u].x, s, a); ckpt::decode4(z[u].y, s, a + 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= act::slope<ACT>(a[k]);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) sum[k] += v[k];
          if (dZ != nullptr)
            dZ[t * C8 + c8] = make_uint4(pack_bf16_f(v[0], v[1]), pack_bf16_f(v[2], v[3]), pack_bf16_f(v[4], v[5]), pack_bf16_f(v[6], v[7]));
        }
      }
    }
  }
  if (partial == nullptr) return;
  if (rows > 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k) red[threadIdx.x][k] = sum[k];
    __syncthreads();
    if (g == 0)
      for (int r = 1; r < rows; ++r)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += red[r * tile8 + lc][k];
  }
  if (g == 0 && mine) {
    float4* out = partial + (size_t)blockIdx.y * (2 * C8) + 2 * c8;
    out[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    out[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
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
  const long long most = 148 * 8;                         // 2048 threads per SM
  return (int)(ctas < most ? ctas : most);
}

struct ActBwdPlan { int tile8, tiles, rows, threads, slots; };

// Columns: one tile when a row has at most 2048 columns, else tiles of about that size.  Rows: as many side by side as
// fit 256 threads (at least one); row slots so that every SM holds about 1024 threads, each with four rows in flight.
ActBwdPlan plan_act_bwd(int T, int C) {
  ActBwdPlan p;
  const int C8 = C / 8;
  p.tiles = (C8 + 255) / 256;
  p.tile8 = (C8 + p.tiles - 1) / p.tiles;
  p.rows = 256 / p.tile8 > 0 ? 256 / p.tile8 : 1;
  if (p.rows > T) p.rows = T;
  p.threads = (p.tile8 * p.rows + 31) / 32 * 32;
  int per_sm = 1024 / p.threads;
  if (per_sm < 1) per_sm = 1;
  if (per_sm > 16) per_sm = 16;
  p.slots = 148 * per_sm / p.tiles;
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
  const long long halves = (long long)T * (C / 16);
  auto run = [&](auto kern) {
    return launch_pdl(kern, stream_grid(halves), STREAM_THREADS, 0, st, reinterpret_cast<const uint4*>(q), s, halves,
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
                      zs, T, C / 8, p.tile8, p.rows, reinterpret_cast<uint4*>(dZ), reinterpret_cast<float4*>(part));
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
