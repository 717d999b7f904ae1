// A linear layer for few tokens: the form of generation and of small batches.  Its time is the reading of
// the weights, so the work is cut along the reduction as well: a cluster of `splits` CTAs owns 128 rows x N_TILE tokens,
// each streams its share of the k tiles through a deep ring of stages (the same TMA -> tcgen05.mma pipeline as the large
// products), leaves its fp32 partial sums in its own shared memory, and after a cluster barrier the CTAs add one another's
// parts over distributed shared memory, token by token in rank order -- no workspace, no second kernel, and a result that
// does not depend on timing -- and finish the layer on them: bias, checkpoint, activation, residual, one rounding.
// The tensor core adds into its fp32 accumulator without rounding to nearest, and the error grows with the length of the
// chain; so a chain ends after 32 MMAs (1024 products' worth of 2:4 reduction, 512 dense).  Two accumulators take the
// segments in turn, and the draining warps, idle until the end otherwise, add each finished one to sums in registers,
// rounded to nearest, while the next is under way.  A 2:4 row of 16384 positive products is off by at most
// 5.0e-7 relative (dense operand 3.5e-7); as one chain 3.2e-5 (4.0e-5).  The end of a chain costs the issuing thread 0.06 us.
// One token, 4096 -> 16384 with the weights in HBM: 15.7 us (75.6 MB, 4.8 TB/s over the whole call; without the split and
// the deep ring 34 us); 24 tokens, 16384 -> 4096: 16.9 us (54 us).  Left: start-up, the first loads' latency and the join,
// about 4 us.
#include "gemm_common.cuh"
#include <mutex>

namespace bimask {

namespace {

constexpr int SMALL_THREADS = 256;                       // warp 0 TMA, warp 1 MMA, warps 2-5 drain; all eight finish

template <int N_TILE, int STAGES, bool SPARSE>
struct SmallCfg {
  static constexpr int A_BYTES = SPARSE ? 16384 : 32768;
  static constexpr int B_BYTES = N_TILE * 256;
  static constexpr int E_BYTES = SPARSE ? 2048 : 0;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + E_BYTES;
  static constexpr int SEGMENT = SPARSE ? 8 : 4;         // k tiles per chain: 32 MMAs
  static constexpr int PART_BYTES = N_TILE * 512;        // [token][128 rows] fp32, over the stages once they are done with
  static constexpr int TMEM_COLS = 4 * N_TILE;           // two accumulators, the metadata, rounded up to a power of two
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 + 256;
  static_assert(PART_BYTES <= STAGES * STAGE_BYTES, "the partial sums lie over the stages");
  static_assert(8 * (2 * STAGES + 4) + Unwind::BYTES <= 256, "barriers, tensor-memory address and what leaving needs");
};

struct SmallParams {
  const uint8_t* hw_meta;
  int tiles_k, k_per_split, tiles_m;
  int Mdim, Ndim;
  const float* bias;
  int act;
  const uint16_t* res;
  uint16_t* out;
  int8_t* zq;
  uint8_t* zs;
  int32_t* status_word;
};

template <int N_TILE, int STAGES, bool SPARSE>
__global__ void __launch_bounds__(SMALL_THREADS, 1)
linear_small_kernel(const __grid_constant__ CUtensorMap tmapA, const __grid_constant__ CUtensorMap tmapB, const SmallParams p, int splits) {
  pdl_launch_dependents();
  using C = SmallCfg<N_TILE, STAGES, SPARSE>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  const uint32_t bar_base = base + STAGES * C::STAGE_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  auto tmem_full_bar = [&](uint32_t b) { return bar_base + 8u * (2 * STAGES + b); };
  auto tmem_empty_bar = [&](uint32_t b) { return bar_base + 8u * (2 * STAGES + 2 + b); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + STAGES * C::STAGE_BYTES + 8 * (2 * STAGES + 4));
  const Unwind unwind(tmem_slot);
  volatile int* abort_flag = unwind.abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)ptx::cluster_ctarank();           // = blockIdx.x % splits
  const int tile = (int)blockIdx.x / splits;
  const int tile_m = tile % p.tiles_m, tile_n = tile / p.tiles_m;
  const int m0 = tile_m * 128, n0 = tile_n * N_TILE;
  const int kt_begin = rank * p.k_per_split;
  const int num_kt = min(p.tiles_k, kt_begin + p.k_per_split) - kt_begin;   // >= 1: the host leaves no CTA without work

  if (threadIdx.x == 0) {
    unwind.init();
    for (int s = 0; s < STAGES; ++s) {
      ptx::mbar_init(full_bar(s), 1);
      ptx::mbar_init(empty_bar(s), 1);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      ptx::mbar_init(tmem_full_bar(b), 1);
      ptx::mbar_init(tmem_empty_bar(b), 4);               // the draining warps
    }
    ptx::fence_barrier_init();
    ptx::prefetch_tmap(&tmapA);
    ptx::prefetch_tmap(&tmapB);
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(tmem_slot), C::TMEM_COLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t tmem_meta = tmem_base + 2 * N_TILE;
  pdl_wait();

  if (warp == 0) {
    if (ptx::elect_one()) {
      int it = 0;
      for (; it < num_kt; ++it) {
        const int s = it % STAGES;
        if (!ptx::mbar_wait_bounded(empty_bar(s), ((uint32_t)(it / STAGES) & 1u) ^ 1u, abort_flag, WAIT_BUDGET)) { *abort_flag = 1; break; }
        const int kt = kt_begin + it;
        const uint32_t a_s = base + s * C::STAGE_BYTES, b_s = a_s + C::A_BYTES;
        ptx::mbar_expect_tx(full_bar(s), C::STAGE_BYTES);
        if (SPARSE) {
          ptx::tma_load_2d(a_s, &tmapA, kt * 64, m0, full_bar(s));
          ptx::bulk_load(b_s + C::B_BYTES, p.hw_meta + ((size_t)tile_m * p.tiles_k + kt) * 2048, 2048, full_bar(s));
        } else {
          ptx::tma_load_2d(a_s, &tmapA, kt * 128, m0, full_bar(s));
          ptx::tma_load_2d(a_s + 16384, &tmapA, kt * 128 + 64, m0, full_bar(s));
        }
        ptx::tma_load_2d(b_s, &tmapB, kt * 128, n0, full_bar(s));
        ptx::tma_load_2d(b_s + N_TILE * 128, &tmapB, kt * 128 + 64, n0, full_bar(s));
      }
      *unwind.issued = it;
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t idesc = ptx::idesc_bf16(128, N_TILE, false, false, SPARSE);
      bool ok = true;
      int it = 0;
      for (int seg = 0; it < num_kt && ok; ++seg) {
        const uint32_t buf = (uint32_t)seg & 1u, acc = tmem_base + N_TILE * buf;
        // both accumulators start out free
        if (seg >= 2 && !ptx::mbar_wait_bounded(tmem_empty_bar(buf), ((uint32_t)(seg >> 1) & 1u) ^ 1u, abort_flag, WAIT_BUDGET)) { *abort_flag = 1; break; }
        const int end = min(num_kt, it + C::SEGMENT);
        for (int k = 0; it < end; ++it, ++k) {
          const int s = it % STAGES;
          if (!ptx::mbar_wait_bounded(full_bar(s), (uint32_t)(it / STAGES) & 1u, abort_flag, WAIT_BUDGET)) { *abort_flag = 1; ok = false; break; }
          ptx::tc_fence_after();
          const uint32_t a_s = base + s * C::STAGE_BYTES, b_s = a_s + C::A_BYTES;
          if constexpr (SPARSE) {
            ptx::tmem_cp_128x128b(tmem_meta, ptx::smem_desc(b_s + C::B_BYTES, 0, 128, 0));
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
              ptx::mma_sparse(acc, ptx::smem_desc(a_s + kb * 32, 16, 1024, 2),
                              ptx::smem_desc(b_s + (kb >> 1) * (N_TILE * 128) + (kb & 1) * 64, 16, 1024, 2), tmem_meta + (kb & ~1),
                              idesc | (uint32_t)(kb & 1), (k | kb) != 0);
          } else {
#pragma unroll
            for (int kb = 0; kb < 8; ++kb)
              ptx::mma_dense(acc, ptx::smem_desc(a_s + (kb >> 2) * 16384 + (kb & 3) * 32, 16, 1024, 2),
                             ptx::smem_desc(b_s + (kb >> 2) * (N_TILE * 128) + (kb & 3) * 32, 16, 1024, 2), idesc, (k | kb) != 0);
          }
          ptx::tc_commit(empty_bar(s));
        }
        if (ok) ptx::tc_commit(tmem_full_bar(buf));
      }
    }
  } else if (warp < 6) {
    // segments -> sums in registers (lane = row, a register per token) -> shared memory, [token][row]: a store covers 128
    // contiguous bytes.  The last segment's commit says that every MMA is done with the stages.
    const int q = warp & 3;
    const int ntok = p.Ndim - n0;                         // columns past it hold nothing that anybody reads
    float sum[N_TILE];
#pragma unroll
    for (int t = 0; t < N_TILE; ++t) sum[t] = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int seg = 0; seg * C::SEGMENT < num_kt; ++seg) {
      const uint32_t buf = (uint32_t)seg & 1u;
      ok = ptx::mbar_wait_bounded(tmem_full_bar(buf), (uint32_t)(seg >> 1) & 1u, abort_flag, WAIT_BUDGET);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) { *abort_flag = 1; break; }
      ptx::tc_fence_after();
      const uint32_t acc = tmem_base + N_TILE * buf + ((uint32_t)(32 * q) << 16);
#pragma unroll
      for (int c = 0; c < N_TILE; c += 16) {
        if (c < ntok) {
          uint32_t r[16];
          ptx::tmem_ld_32x16(acc + c, r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int t = 0; t < 16; ++t) sum[c + t] += __uint_as_float(r[t]);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(tmem_empty_bar(buf));
    }
    if (ok) {
      float* part = reinterpret_cast<float*>(base_ptr) + 32 * q + lane;
#pragma unroll
      for (int c = 0; c < N_TILE; c += 16) {
        if (c < ntok) {
#pragma unroll
          for (int t = 0; t < 16; ++t) part[(c + t) * 128] = sum[c + t];
        }
      }
    }
  }

  // every CTA's partial sums are in place (or its abort flag is up: then the results are void, and the status says so)
  ptx::tc_fence_before();
  __syncthreads();
  unwind.leave(full_bar(0), STAGES, warp, p.status_word);
  if (splits > 1) ptx::cluster_sync();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, C::TMEM_COLS);
  }

  // tokens rank, rank + splits, ... are this CTA's to finish, two at a time per warp: lane = four rows
  const int ntok = min(N_TILE, p.Ndim - n0);
  const int row = m0 + 4 * lane;
  const bool rows_ok = row < p.Mdim;                      // Mdim % 32 == 0: true for whole blocks of eight lanes
  float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.bias != nullptr && rows_ok) b = __ldg(reinterpret_cast<const float4*>(p.bias + row));
  constexpr int U = 2, V = 4;                             // tokens per warp at a time, ranks' sums in flight
  for (int t0 = rank + splits * U * warp; t0 < ntok; t0 += splits * U * (SMALL_THREADS / 32)) {
    uint2 res[U];
    float4 sum[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + splits * u;
      res[u] = make_uint2(0u, 0u);
      if (t < ntok && p.res != nullptr && rows_ok)
        res[u] = *reinterpret_cast<const uint2*>(p.res + (size_t)(n0 + t) * p.Mdim + row);   // may be `out`: a plain load
      sum[u] = b;
    }
    for (int s = 0; s < splits; s += V) {                 // in rank order; eight loads in flight
      float4 v[V][U];
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = t0 + splits * u;
          v[k][u] = s + k < splits && t < ntok ? ptx::ld_cluster_v4(ptx::mapa(base + (uint32_t)(t * 512 + 16 * lane), s + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int u = 0; u < U; ++u) { sum[u].x += v[k][u].x; sum[u].y += v[k][u].y; sum[u].z += v[k][u].z; sum[u].w += v[k][u].w; }
    }
    act::Pair z[2 * U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      z[2 * u] = act::pair(sum[u].x, sum[u].y);
      z[2 * u + 1] = act::pair(sum[u].z, sum[u].w);
    }
    if (p.zq != nullptr) {                                // eight lanes = one block of 32 channels
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + splits * u;
        float v[4];
        act::split(z[2 * u], v[0], v[1]);
        act::split(z[2 * u + 1], v[2], v[3]);
        uint32_t h = ckpt::up16(act::max_abs3(act::max_abs3(v[0], v[1], v[2]), v[3], 0.0f));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) h = max(h, __shfl_xor_sync(0xFFFFFFFFu, h, d));
        const uint32_t sc = ckpt::scale_of(h);
        const float inv = ckpt::inverse_scale(sc);
        const uint32_t lo = __byte_perm(ckpt::round_bits(v[0], inv), ckpt::round_bits(v[1], inv), 0x0040);
        const uint32_t hi = __byte_perm(ckpt::round_bits(v[2], inv), ckpt::round_bits(v[3], inv), 0x0040);
        if (t < ntok && rows_ok) {
          const size_t at = (size_t)(n0 + t) * p.Mdim + row;
          *reinterpret_cast<uint32_t*>(p.zq + at) = __byte_perm(lo, hi, 0x5410);
          if ((lane & 7) == 0) p.zs[at >> 5] = (uint8_t)sc;
        }
      }
    }
    act::apply(p.act, z);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + splits * u;
      if (t < ntok && rows_ok)
        *reinterpret_cast<uint2*>(p.out + (size_t)(n0 + t) * p.Mdim + row) =
            make_uint2(pack_bf16_p(act::add2(z[2 * u], bf16_pair(res[u].x))), pack_bf16_p(act::add2(z[2 * u + 1], bf16_pair(res[u].y))));
    }
  }
  __syncthreads();
  if (splits > 1) ptx::cluster_sync();                    // shared memory must outlive the peers' reads of it
}

template <int N_TILE, int STAGES, bool SPARSE>
int run_small(const uint16_t* vals, const void* hw_meta, const uint16_t* X, int Mdim, int Ndim, int Kdim, const LinearEpilogue& le,
              uint16_t* out, int32_t* status_word, cudaStream_t s) {
  using C = SmallCfg<N_TILE, STAGES, SPARSE>;
  CUtensorMap ta, tb;
  int rc;
  if ((rc = make_tmap(&ta, vals, SPARSE ? (uint64_t)Kdim / 2 : (uint64_t)Kdim, (uint64_t)Mdim, 128)) != BIMASK_OK) return rc;
  if ((rc = make_tmap(&tb, X, (uint64_t)Kdim, (uint64_t)Ndim, N_TILE)) != BIMASK_OK) return rc;
  auto kern = linear_small_kernel<N_TILE, STAGES, SPARSE>;
  if ((rc = set_smem_attr(kern, C::SMEM_BYTES)) != BIMASK_OK) return rc;
  SmallParams p;
  p.hw_meta = reinterpret_cast<const uint8_t*>(hw_meta);
  p.tiles_k = (Kdim + 127) / 128;
  p.tiles_m = (Mdim + 127) / 128;
  p.Mdim = Mdim; p.Ndim = Ndim;
  p.bias = le.bias; p.act = le.act; p.res = le.res; p.out = out; p.zq = le.zq; p.zs = le.zs;
  p.status_word = status_word;
  const int tiles = p.tiles_m * ((Ndim + N_TILE - 1) / N_TILE);
  const int splits = linear_small_splits(tiles, p.tiles_k);
  p.k_per_split = (p.tiles_k + splits - 1) / splits;
  BIMASK_CUDA_OK(launch_pdl_cluster(kern, splits * tiles, SMALL_THREADS, splits, C::SMEM_BYTES, s, ta, tb, p, splits));
  count_launch();
  BIMASK_CUDA_OK(cudaGetLastError());
  return BIMASK_OK;
}

template <bool SPARSE>
int run_small_any(const uint16_t* vals, const void* hw_meta, const uint16_t* X, int Mdim, int Ndim, int Kdim, const LinearEpilogue& le,
                  uint16_t* out, int32_t* status_word, cudaStream_t s) {
  // stages: what fits 220 KB (22 / 26 / 34 / 50 KB each, dense 36 / 40 / 48 / 64 KB)
  // Very few tokens: narrower token tiles leave room for more stages of weights.  16- / 32-token tiles, us: 16384 x 4096 at
  // 1, 8, 16 tokens 15.8 / 16.6, 15.8 / 16.0, 15.8 / 15.5; 9600 x 16384 33.8 / 37.1, 33.6 / 34.5, 33.1 / 34.1; 4096 x 4096
  // 7.2 / 7.3, 7.5 / 7.7, 7.6 / 7.7; but 4096 x 16384 16.6 / 16.4, 16.8 / 16.2, 17.0 / 16.5.  Dense operand: 16384 x 4096
  // 24.9 / 25.3, 25.6 / 25.8, 25.4 / 25.4; 4096 x 16384 26.8 / 26.5, 27.2 / 26.7, 26.8 / 26.1.  Smaller layers within 1 %.
  if (Ndim <= 8) return run_small<16, SPARSE ? 10 : 6, SPARSE>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s);
  if (Ndim <= 32) return run_small<32, SPARSE ? 8 : 5, SPARSE>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s);
  if (Ndim <= 64) return run_small<64, SPARSE ? 6 : 4, SPARSE>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s);
  return run_small<128, SPARSE ? 4 : 3, SPARSE>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s);
}

}  // namespace

// Clusters of 1 .. 8 CTAs of this file's kernels that the current device holds at once (one CTA per SM, and a cluster must
// lie within a GPC: 148, 74, 45, 33, 26, 22, 15, 15 on a device whose SMs are spread unevenly).  Asked once per device.
static const int* fit_table() {
  constexpr int DEVICES = 64;
  struct Table { std::atomic<bool> known{false}; int fit[9] = {0, 148, 74, 49, 37, 29, 24, 21, 18}; };
  static Table tables[DEVICES];
  static const Table unknown;                             // no device: nothing is launched by it
  static std::mutex mutex;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEVICES) return unknown.fit;
  Table& t = tables[dev];
  if (t.known.load(std::memory_order_acquire)) return t.fit;
  std::lock_guard<std::mutex> lock(mutex);
  if (t.known.load(std::memory_order_relaxed)) return t.fit;
  using C = SmallCfg<32, 8, true>;
  auto kern = linear_small_kernel<32, 8, true>;
  if (set_smem_attr(kern, C::SMEM_BYTES) != BIMASK_OK) return unknown.fit;        // the launch will say what is wrong
  int fit[9] = {0, sm_count()};
  for (int size = 2; size <= 8; ++size) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)size);
    cfg.blockDim = dim3(SMALL_THREADS);
    cfg.dynamicSmemBytes = C::SMEM_BYTES;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&fit[size], kern, &cfg) != cudaSuccess || fit[size] < 1) {
      cudaGetLastError();
      return unknown.fit;
    }
  }
  for (int size = 1; size <= 8; ++size) t.fit[size] = fit[size];
  t.known.store(true, std::memory_order_release);
  return t.fit;
}

int linear_small_fit(int size) { return fit_table()[size < 1 ? 1 : size > 8 ? 8 : size]; }

// The largest cluster, at most eight (the portable size) and at least four k tiles per CTA, of which all tiles' fit at once: a
// second round costs what the split saves and more.  24 tokens, reduction 4096, in one round / one size larger, in two:
// 20 row tiles 6 / 7 CTAs 7.1 / 12.2 us, 24: 5 / 6 7.4 / 12.6, 28: 4 / 5 7.4 / 12.9, 36: 3 / 4 8.2 / 13.0, 48: 2 / 3
// 9.3 / 14.7; reduction 16384: 20 row tiles 12.7 / 19.2, 36: 18.5 / 26.2.  Four CTAs where six fit would save another
// 4 % at 4096 and lose 2 % at 16384.
int linear_small_splits(int tiles, int k_tiles) {
  int splits = 1;
  if (k_tiles >= 8) {
    const int* fit = fit_table();
    for (int c = 8; c > 1 && splits == 1; --c)
      if (4 * c <= k_tiles && tiles <= fit[c]) splits = c;
  }
  const int per = (k_tiles + splits - 1) / splits;
  return (k_tiles + per - 1) / per;
}

int launch_linear_small(const uint16_t* vals, const void* hw_meta, const uint16_t* X, int Mdim, int Ndim, int Kdim,
                        const LinearEpilogue& le, uint16_t* out, int32_t* status_word, cudaStream_t s) {
  return hw_meta != nullptr ? run_small_any<true>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s)
                            : run_small_any<false>(vals, hw_meta, X, Mdim, Ndim, Kdim, le, out, status_word, s);
}

}  // namespace bimask
