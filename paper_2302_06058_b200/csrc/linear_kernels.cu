// The streaming kernels around a linear layer: 8-bit activation checkpoints written and read, and the gradient through
// the activation and the bias.  All three are bound by HBM.
#include "dropout.cuh"

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
// an activation, now 76: 5.3 TB/s); two steps' bytes are loaded at a time.  DROP: dropout of the result; its blocks of eight
// are the threads'.  Then the generator and the GELU keep the multiplying pipe three quarters busy: 134 us; more warps, or fewer
// with more registers, changed nothing.
template <int ACT, bool DROP>
__global__ void __launch_bounds__(STREAM_THREADS, 8)
ckpt_unpack_kernel(const uint2* __restrict__ q, const uint8_t* __restrict__ s, long long eighths, uint4* __restrict__ x, const __grid_constant__ DropParams d) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned long long number = DROP ? drop_number(d) : 0ull;
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
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = act::value2<ACT>(z[k]);
        if constexpr (DROP) drop8(z, (unsigned long long)i, number, d);
        x[i] = make_uint4(pack_bf16_p(z[0]), pack_bf16_p(z[1]), pack_bf16_p(z[2]), pack_bf16_p(z[3]));
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

// ------------------------------------------------------------------------------------------
// The same with dY dropped first.  The generator doubles the instructions per element (254 for a block of eight with a GELU: two
// thirds of the issue slots, of the integer pipe and of the one that multiplies), so this kernel wants warps rather than registers: 32
// of them, a thread with one block of eight columns, and the rows ahead in shared memory, copied by the threads that will use them
// (cp.async: every thread waits for its own pieces only); a row's scale byte, shared by four threads, is loaded a row ahead.
// 8192 x 16384 in 185 us (3.7 TB/s), 12608 x 1536 in 34; in act_bwd_kernel, with 16 warps and rows ahead in registers, 238 and 37.
// ------------------------------------------------------------------------------------------
constexpr int DROPBWD_THREADS = 1024, DROPBWD_STAGES = 4;
constexpr int DROPBWD_SMEM = DROPBWD_STAGES * DROPBWD_THREADS * (16 + 8);

template <int ACT>
__global__ void __launch_bounds__(DROPBWD_THREADS, 1)
act_dropout_bwd_kernel(const uint4* dY, const uint2* __restrict__ zq, const uint8_t* __restrict__ zs, uint32_t T, uint32_t C8, int cols,
                       uint32_t rows, uint4* dZ /* may be dY */, float4* __restrict__ partial, const __grid_constant__ DropParams drop) {
  extern __shared__ uint4 smem[];
  pdl_launch_dependents();
  const uint32_t g = threadIdx.x / (uint32_t)cols, lc = threadIdx.x - g * (uint32_t)cols, c = blockIdx.x * (uint32_t)cols + lc;
  const bool ok = g < rows && c < C8;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
  const uint32_t ring_d = base + threadIdx.x * 16u, ring_q = base + DROPBWD_STAGES * DROPBWD_THREADS * 16u + threadIdx.x * 8u;
  pdl_wait();
  const unsigned long long number = drop_number(drop);
  act::Pair sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = act::both(0.f);
  if (ok) {
    const uint32_t stride = rows * gridDim.y, first = blockIdx.y * rows + g;
    const unsigned long long hop = (unsigned long long)stride * C8;
    unsigned long long at = (unsigned long long)first * C8 + c, lead = at;
    uint32_t ahead = first;
    auto fetch = [&](uint32_t stage) {
      if (ahead < T) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring_d + stage * (DROPBWD_THREADS * 16)), "l"(dY + lead) : "memory");
        if (ACT != BIMASK_ACT_NONE)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ring_q + stage * (DROPBWD_THREADS * 8)), "l"(zq + lead) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      ahead += stride;
      lead += hop;
    };
#pragma unroll
    for (int s = 0; s < DROPBWD_STAGES - 1; ++s) fetch(s);
    uint32_t stage = 0, next_scale = ACT != BIMASK_ACT_NONE && first < T ? __ldg(zs + (at >> 2)) : 0u;
    for (uint32_t t = first; t < T; t += stride, at += hop) {
      const uint32_t scale_byte = next_scale;
      if (ACT != BIMASK_ACT_NONE && t + stride < T) next_scale = __ldg(zs + ((at + hop) >> 2));
      asm volatile("cp.async.wait_group %0;" ::"n"(DROPBWD_STAGES - 2) : "memory");
      uint4 d;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(d.x), "=r"(d.y), "=r"(d.z), "=r"(d.w) : "r"(ring_d + stage * (DROPBWD_THREADS * 16)) : "memory");
      act::Pair v[4] = {bf16_pair(d.x), bf16_pair(d.y), bf16_pair(d.z), bf16_pair(d.w)};
      act::Pair a[4];
      if constexpr (ACT != BIMASK_ACT_NONE) {
        uint2 z;
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(z.x), "=r"(z.y) : "r"(ring_q + stage * (DROPBWD_THREADS * 8)) : "memory");
        const act::Pair scale = act::both(ckpt::scale_value(scale_byte));
        ckpt::decode4(z.x, scale, a);
        ckpt::decode4(z.y, scale, a + 2);
      }
      // into the pieces that the row before this one left
      fetch((stage + DROPBWD_STAGES - 1) % DROPBWD_STAGES);
      stage = (stage + 1) % DROPBWD_STAGES;
      drop8(v, at, number, drop);
      if constexpr (ACT != BIMASK_ACT_NONE) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = act::mul2(v[k], act::slope2<ACT>(a[k]));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] = act::add2(sum[k], v[k]);
      if (dZ != nullptr) dZ[at] = make_uint4(pack_bf16_p(v[0]), pack_bf16_p(v[1]), pack_bf16_p(v[2]), pack_bf16_p(v[3]));
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
  if (partial == nullptr) return;
  // the rows that worked side by side are added in their order; each thread's sums lie in the first of its own pieces and the next
  float s[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) act::split(sum[k], s[2 * k], s[2 * k + 1]);
  float4* fold = reinterpret_cast<float4*>(smem);
  if (rows > 1) {
    fold[threadIdx.x] = make_float4(s[0], s[1], s[2], s[3]);
    fold[DROPBWD_THREADS + threadIdx.x] = make_float4(s[4], s[5], s[6], s[7]);
    __syncthreads();
    if (g == 0)
      for (uint32_t r = 1; r < rows; ++r) {
        const float4 x = fold[r * (uint32_t)cols + lc], y = fold[DROPBWD_THREADS + r * (uint32_t)cols + lc];
        s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
        s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
      }
  }
  if (g == 0 && ok) {
    float4* out = partial + ((size_t)blockIdx.y * C8 + c) * 2;
    out[0] = make_float4(s[0], s[1], s[2], s[3]);
    out[1] = make_float4(s[4], s[5], s[6], s[7]);
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

// The same of the kernel with dropout: `half` is the columns (groups of eight) of a tile, a thread's one.
ActBwdPlan plan_dropout_bwd(int T, int C) {
  ActBwdPlan p;
  const int C8 = C / 8;
  p.tiles = (C8 + DROPBWD_THREADS / 2 - 1) / (DROPBWD_THREADS / 2);
  p.half = (C8 + p.tiles - 1) / p.tiles;
  p.rows = DROPBWD_THREADS / p.half;
  if (p.rows > T) p.rows = T;
  p.threads = (p.half * p.rows + 31) / 32 * 32;
  p.slots = PLAN_SMS / p.tiles;
  const int most = (T + p.rows - 1) / p.rows;
  if (p.slots > most) p.slots = most;
  if (p.slots < 1) p.slots = 1;
  return p;
}

}  // namespace

// enough for either kernel
size_t act_bwd_partial_bytes(int T, int C) {
  const int a = plan_act_bwd(T, C).slots, b = plan_dropout_bwd(T, C).slots;
  return (size_t)(a > b ? a : b) * C * sizeof(float);
}

int launch_ckpt_pack(const uint16_t* x, int T, int C, int8_t* q, uint8_t* s, cudaStream_t st) {
  const long long halves = (long long)T * (C / 16);
  BIMASK_CUDA_OK(launch_pdl(ckpt_pack_kernel, stream_grid(halves), STREAM_THREADS, 0, st, reinterpret_cast<const uint4*>(x), halves,
                            reinterpret_cast<uint4*>(q), s));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_ckpt_unpack(const int8_t* q, const uint8_t* s, int act, int T, int C, uint16_t* x, cudaStream_t st, const bimask_dropout_args* drop) {
  const long long eighths = (long long)T * (C / 8);
  const DropParams d = drop_params(drop);
  auto run = [&](auto kern) {
    return launch_pdl(kern, stream_grid(eighths), STREAM_THREADS, 0, st, reinterpret_cast<const uint2*>(q), s, eighths,
                      reinterpret_cast<uint4*>(x), d);
  };
  cudaError_t e;
#define BIMASK_RUN(ACT) (d.thr != 0u ? run(ckpt_unpack_kernel<ACT, true>) : run(ckpt_unpack_kernel<ACT, false>))
  switch (act) {
    case BIMASK_ACT_RELU: e = BIMASK_RUN(BIMASK_ACT_RELU); break;
    case BIMASK_ACT_GELU: e = BIMASK_RUN(BIMASK_ACT_GELU); break;
    case BIMASK_ACT_GELU_TANH: e = BIMASK_RUN(BIMASK_ACT_GELU_TANH); break;
    case BIMASK_ACT_SILU: e = BIMASK_RUN(BIMASK_ACT_SILU); break;
    default: e = BIMASK_RUN(BIMASK_ACT_NONE); break;
  }
#undef BIMASK_RUN
  BIMASK_CUDA_OK(e);
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

// db from the partial rows
static int launch_bias_reduce(const float* partial, int slots, int C, float* dbias, cudaStream_t st) {
  BIMASK_CUDA_OK(launch_pdl(bias_reduce_kernel, (C / 4 + 7) / 8, 256, 0, st, reinterpret_cast<const float4*>(partial), slots, C / 4,
                            reinterpret_cast<float4*>(dbias)));
  count_launch();
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
    const int rc = launch_bias_reduce(partial, p.slots, C, dbias, st);
    if (rc != BIMASK_OK) return rc;
  }
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

int launch_act_dropout_bwd(const uint16_t* dY, const int8_t* zq, const uint8_t* zs, int act, const bimask_dropout_args& drop, int T, int C,
                           uint16_t* dZ, float* dbias, float* partial, cudaStream_t st) {
  const DropParams d = drop_params(&drop);
  if (d.thr == 0u) return launch_act_bwd(dY, zq, zs, act, T, C, dZ, dbias, partial, st);
  const ActBwdPlan p = plan_dropout_bwd(T, C);
  float* part = dbias == nullptr ? nullptr : p.slots == 1 ? dbias : partial;      // one slot: its row is the result
  auto run = [&](auto kern) -> int {
    const int rc = set_smem_attr(kern, DROPBWD_SMEM);
    if (rc != BIMASK_OK) return rc;
    BIMASK_CUDA_OK(launch_pdl(kern, dim3(p.tiles, p.slots), p.threads, DROPBWD_SMEM, st, reinterpret_cast<const uint4*>(dY),
                              reinterpret_cast<const uint2*>(zq), zs, (uint32_t)T, (uint32_t)C / 8, p.half, (uint32_t)p.rows,
                              reinterpret_cast<uint4*>(dZ), reinterpret_cast<float4*>(part), d));
    count_launch();
    return BIMASK_OK;
  };
  int rc;
  switch (act) {
    case BIMASK_ACT_RELU: rc = run(act_dropout_bwd_kernel<BIMASK_ACT_RELU>); break;
    case BIMASK_ACT_GELU: rc = run(act_dropout_bwd_kernel<BIMASK_ACT_GELU>); break;
    case BIMASK_ACT_GELU_TANH: rc = run(act_dropout_bwd_kernel<BIMASK_ACT_GELU_TANH>); break;
    case BIMASK_ACT_SILU: rc = run(act_dropout_bwd_kernel<BIMASK_ACT_SILU>); break;
    default: rc = run(act_dropout_bwd_kernel<BIMASK_ACT_NONE>); break;
  }
  if (rc == BIMASK_OK && dbias != nullptr && p.slots > 1) rc = launch_bias_reduce(partial, p.slots, C, dbias, st);
  if (rc != BIMASK_OK) return rc;
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

}  // namespace bimask
