// What the tensor-core kernels share: tile configurations, the convolution geometry, kernel parameters, the tile
// order, the accumulator drain of the 2:4 products, and the host helpers (tensor maps, SM count, shared-memory
// attribute) implemented in gemm_host.cu.
#pragma once
#include "common.cuh"
#include "sm100_ptx.cuh"
#include "act_math.cuh"
#include <cuda.h>
#include <cuda_bf16.h>
#include <atomic>
#include <type_traits>

namespace bimask {


constexpr long long WAIT_BUDGET = 4000000000ll;      // ~2 s of SM clocks
constexpr long long DRAIN_BUDGET = 100000000ll;      // ~50 ms: a load that has been issued lands within microseconds
constexpr int GEMM_THREADS = 192;                    // warp 0 TMA, warp 1 MMA, warps 2-5 epilogue
// The sparse kernels that drain bf16 results use eight epilogue warps (two groups of four, one warp per
// tensor-memory lane quadrant, taking alternate column chunks): products with a short reduction are bound by
// that drain, not by the tensor pipe.
constexpr int EPI_WARPS = 8;
// One more warp per group of four epilogue warps issues the tensor stores of the group's staged chunks (see
// drain_chunks_tma / store_chunks): a tensor store costs its issuing thread a few hundred clocks, which the warps
// that drain tensor memory should not wait for.
constexpr int EPI_GROUPS = EPI_WARPS / 4;
constexpr int PAIR_THREADS = 64 + 32 * EPI_WARPS + 32 * EPI_GROUPS;
// Epilogue staging: per group NT tiles of [32 tokens][128 rows] bf16 (8 KB each), and per group NT "staged" plus NT
// "freed" mbarriers, kept EPI_BAR_OFFSET bytes into the kernels' barrier area.
__host__ __device__ constexpr int epi_staging_bytes(int nt) { return EPI_GROUPS * nt * 8192; }
constexpr uint32_t EPI_BAR_OFFSET = 128;
// Past the 256 bytes of barriers: the checkpoint's scales on their way out, a word per token, 128 bytes per staging tile.
constexpr uint32_t EPI_SCALES_OFFSET = 256;
__host__ __device__ constexpr int epi_scales_bytes(int nt) { return EPI_GROUPS * nt * 128; }


template <int N_TILE, int STAGES, bool SPARSE = true, bool EPI = false>
struct Cfg {
  static constexpr int M_TILE = 128;
  static constexpr int K_TILE = 128;                             // logical reduction elements per stage
  static constexpr int A_BYTES = SPARSE ? 16384 : 32768;         // 128 rows x 64 compressed, or x 128 dense, bf16
  static constexpr int B_BYTES = N_TILE * K_TILE * 2;
  static constexpr int E_BYTES = SPARSE ? 2048 : 0;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + E_BYTES;
  static constexpr int META_COLS = SPARSE ? 4 : 0;
  static constexpr int EPI_NT = SPARSE && !EPI ? 3 : 2;          // staging tiles per epilogue group (the dense stages leave room for two; EPI: even, see below)
  static constexpr int TMEM_COLS = (N_TILE + META_COLS) <= 128 ? 128 : (N_TILE + META_COLS) <= 256 ? 256 : 512;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024 /* alignment slack */ + 256 /* barriers */ +
                                    epi_staging_bytes(EPI_NT) /* epilogue staging */;
};

// ---- leaving a kernel ---------------------------------------------------------------------------
// A role whose wait runs out of budget raises the CTA's abort flag and leaves; the others follow.  Before such a CTA may free
// its tensor memory and end, the MMAs issued so far and the loads in flight into its shared memory must have finished,
// whichever role gave up: the producer may have left long before with everything issued.  In shared memory behind the
// tensor-memory address: the abort flag, the number of loads that the producer issued, a barrier for the MMAs.
struct Unwind {
  volatile int* abort_flag;
  volatile int* issued;
  uint32_t mma_bar;
  __device__ __forceinline__ explicit Unwind(uint32_t* tmem_slot)
      : abort_flag(reinterpret_cast<volatile int*>(tmem_slot + 1)), issued(reinterpret_cast<volatile int*>(tmem_slot + 2)),
        mma_bar(ptx::smem_u32(tmem_slot) + 16u) {}
  static constexpr int BYTES = 24;                                // with the tensor-memory address
  __device__ __forceinline__ void init() const {                  // one thread, before fence_barrier_init
    *abort_flag = 0;
    *issued = 0;
    ptx::mbar_init(mma_bar, 1);
  }
  __device__ __forceinline__ void drain_loads(uint32_t full_bar0, int stages, int issued0, int issued1, uint32_t cta_bytes) const {
    volatile int none = 0;
    for (int k = drain_begin(issued0, issued1, stages); k < drain_end(issued0, issued1); ++k) {
      const uint32_t bar = full_bar0 + 8u * (uint32_t)(k % stages);
      const int settle = drain_settle(k, issued0, issued1);
      if (settle == SETTLE_EXPECT) ptx::mbar_expect_tx(bar, cta_bytes);
      if (settle == SETTLE_COUNT) ptx::mbar_complete_tx(bar, cta_bytes);
      ptx::mbar_wait_bounded(bar, (uint32_t)(k / stages) & 1u, &none, DRAIN_BUDGET);
    }
  }
  // All threads, after the barrier that joins the roles.  Warp 1 issued the MMAs (elect_one picks the same lane each time, and
  // a commit covers what its thread has issued).
  __device__ __forceinline__ void leave(uint32_t full_bar0, int stages, int warp, int32_t* status_word) const {
    if (!*abort_flag) return;
    volatile int none = 0;
    if (warp == 1 && ptx::elect_one()) {
      ptx::tc_commit(mma_bar);
      ptx::mbar_wait_bounded(mma_bar, 0, &none, DRAIN_BUDGET);
    }
    if (threadIdx.x == 0) {
      atomicExch(status_word, (int32_t)BIMASK_ETIMEOUT);
      drain_loads(full_bar0, stages, *issued, *issued, 0u);
    }
    __syncthreads();
  }
  // The same for a CTA pair, cluster barrier included: both leave together.  cta_bytes: one CTA's bytes per stage.
  __device__ __forceinline__ void leave_pair(uint32_t full_bar0, int stages, uint32_t cta_bytes, uint32_t rank, int warp,
                                             int32_t* status_word) const {
    const uint32_t flag = ptx::smem_u32(const_cast<int*>(abort_flag));
    if (threadIdx.x == 0 && *abort_flag) {
      atomicExch(status_word, (int32_t)BIMASK_ETIMEOUT);
      ptx::st_cluster_u32(ptx::mapa(flag, rank ^ 1u), 1u);
    }
    __syncwarp();
    ptx::cluster_sync();
    if (!*abort_flag) return;
    if (rank == 0) {
      volatile int none = 0;
      if (warp == 1 && ptx::elect_one()) {
        ptx::tc_commit_pair(mma_bar, 1);
        ptx::mbar_wait_bounded(mma_bar, 0, &none, DRAIN_BUDGET);
      }
      if (threadIdx.x == 0) {
        const uint32_t peer = ptx::mapa(ptx::smem_u32(const_cast<int*>(issued)), 1);
        drain_loads(full_bar0, stages, *issued, (int)ptx::ld_cluster_u32(peer), cta_bytes);
      }
    }
    __syncthreads();
    ptx::cluster_sync();
  }
};

// A 3x3 convolution as an implicit GEMM: the token operand is an NHWC tensor and a "tile of
// tokens" is a box of wb x hb pixels of nb images, fetched with one 4-D tensor load per 64
// channels, shifted by the filter tap the k index belongs to (pixels outside the image read 0).
//   mode 1 (forward, Eq. 3):        k = (tap, c);  B = x,   shift (+kw-1, +kh-1)
//   mode 2 (input gradient, Eq. 10): k = (tap, i');  B = dy[:, perm], shift (1-kw, 1-kh); the rows of
//           the 2:4 operand for tap (kh, kw) are (kh*3+kw)*C + c.
struct ConvGeom {
  int mode;                 // 0: plain matrix operand
  int H, W, NB;             // grid of the tokens (the convolution's OUTPUT pixels)
  int stride;               // mode 1 / weight gradient: input pixel of output pixel (h, w), tap (kh, kw) is
                            // (stride * h + kh - 1, stride * w + kw - 1); the input tensor map strides by it
  int CB;                   // channels of the token operand (x: C; dy: I)
  int wb, hb, nb;           // pixel box of one load: wb * hb * nb tokens (powers of two)
  int lg_wb, lg_hb;         // their logarithms
  int tiles_w, tiles_h;     // boxes per image
  int kt_per_tap;           // mode 2: 128-wide k tiles per filter tap (I / 128)
  int rows_per_tap;         // mode 2: rows of the 2:4 operand per tap (C)
  // mode 2: the filter taps this launch sums over, in k order: tap id (kh * 3 + kw, selects the operand rows) and the
  // shift of the dy box.  Stride 1: all nine, shift (1 - kw, 1 - kh).  Stride 2: the input pixels of one parity class
  // (h % 2, w % 2) receive gradient through the taps with kh = h + 1 and kw = w + 1 (mod 2) only -- one, two, two and
  // four taps for the four classes -- from dy pixel ((h + 1 - kh) / 2, (w + 1 - kw) / 2); the token grid is then the
  // class's sub-grid and the results go to every second pixel of dx.
  signed char tap_id[9], tap_dw[9], tap_dh[9];
  int out_step, out_h0, out_w0, out_H, out_W;   // token (h, w) is stored at pixel (out_step * h + out_h0, out_step * w + out_w0) of out_H x out_W
};

// Where the results of token pixel (n, h, w) go: element offset of its first channel in the NHWC output.
__device__ __forceinline__ size_t conv_out_pixel(const ConvGeom& g, int n, int h, int w) {
  return ((size_t)n * g.out_H + (g.out_step * h + g.out_h0)) * g.out_W + (g.out_step * w + g.out_w0);
}

__device__ __forceinline__ void conv_box_origin(const ConvGeom& g, int box, int& w0, int& h0, int& n0) {
  w0 = (box % g.tiles_w) * g.wb;
  const int r = box / g.tiles_w;
  h0 = (r % g.tiles_h) * g.hb;
  n0 = (r / g.tiles_h) * g.nb;
}

// Channel offset and pixel shift of the 64-wide half q of k tile kt; valid = false: past the
// reduction length (the loader then reads a box of zeros).
__device__ __forceinline__ void conv_k_coords(const ConvGeom& g, int kt, int q, int Kdim, int& c0, int& dw, int& dh, bool& valid) {
  if (g.mode == 1) {
    const int j = kt * 128 + 64 * q;
    valid = j < Kdim;
    const int tap = j / g.CB;
    c0 = j - tap * g.CB;
    dh = tap / 3 - 1;
    dw = tap % 3 - 1;
  } else {
    const int tap = kt / g.kt_per_tap;
    c0 = (kt - tap * g.kt_per_tap) * 128 + 64 * q;
    valid = true;
    dh = g.tap_dh[tap];
    dw = g.tap_dw[tap];
  }
}

struct GemmParams {
  ConvGeom conv;
  const uint8_t* hw_meta;   // sparse only
  int tiles_k_meta;         // number of 128-wide k tiles in the metadata image
  int Mdim, Ndim, Kdim;     // D is Mdim x Ndim, reduction length Kdim (logical)
  int k_tiles_per_split;    // dense split-K: k tiles handled by one blockIdx.z
  int tiles_m, tiles_n;     // output tiles (CTA pairs along M for the pair kernel)
  int raster_group;         // tiles walked along M before advancing along N
  int n_tile;               // pair kernel: output columns per tile (multiple of 32, <= 256)
  void* out;                // sparse: bf16 [Ndim][Mdim];  dense: fp32 [split][Mdim][Ndim]
  int32_t* status_word;
};


// Tile order.  A linear id walks `group` tiles along M before it advances along N, so that the
// CTAs resident at one time cover a near-square patch of the output and both operands are
// re-used out of L2 instead of being streamed from HBM once per wave.
__device__ __forceinline__ void raster(int id, int tiles_m, int tiles_n, int group, int& tm, int& tn) {
  const int per_group = group * tiles_n;
  const int g = id / per_group;
  const int first = g * group;
  const int gsize = min(group, tiles_m - first);
  const int in = id - g * per_group;
  tm = first + in % gsize;
  tn = in / gsize;
}

// Epilogue of the 2:4 products, form with per-lane global stores (used where a token's address is not affine in
// its index: the pixel boxes of the implicit convolution; drain_chunks_tma below is the form for plain matrices).
// The accumulator holds D[row][token] (row = tensor-memory lane), the result is
// stored token-major, so a chunk of W tokens x the CTA's 128 rows is transposed on its way out by a GROUP of four
// warps, one per tensor-memory lane quadrant:
//   tensor memory -> registers in the accumulator-fragment layout (two 16-lane loads per warp) -> bf16 pairs ->
//   stmatrix.trans into one of the group's two staging tiles [token][128 rows] (256-byte rows; the 16-byte unit
//   index is XOR-ed with the token index mod 8, so the eight rows of a matrix fall into eight different bank
//   groups) -> named barrier -> each warp reads W/4 whole token rows back and writes them with 16-byte stores,
//   256 contiguous bytes per token (whole 128-byte lines).
// The tensor-memory load of the next chunk is issued before the current one is converted and stored.
template <int W>
__device__ __forceinline__ void epi_load(uint32_t taddr, uint32_t (&r)[W], bool zero) {
  if (zero) {
#pragma unroll
    for (int j = 0; j < W; ++j) r[j] = 0u;
  } else if (W == 32) {
    ptx::tmem_ld_16x256b_x4(taddr, &r[0]);                 // lanes 0-15 of the quadrant
    ptx::tmem_ld_16x256b_x4(taddr + (16u << 16), &r[16]);  // lanes 16-31
  } else {
    ptx::tmem_ld_16x256b_x2(taddr, &r[0]);
    ptx::tmem_ld_16x256b_x2(taddr + (16u << 16), &r[W / 2]);
  }
}

__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// `dst`: this lane's row address for token group 0 (see drain_chunks); token group g is GROUP_BYTES further (eight
// token rows of the staging tile).
template <int W, uint32_t GROUP_BYTES = 2048u>
__device__ __forceinline__ void epi_stage(const uint32_t (&r)[W], uint32_t dst) {
#pragma unroll
  for (int g = 0; g < W / 8; ++g)
    ptx::stmatrix_x4_trans(dst + GROUP_BYTES * g, pack_bf16(r[4 * g], r[4 * g + 1]), pack_bf16(r[4 * g + 2], r[4 * g + 3]),
                           pack_bf16(r[W / 2 + 4 * g], r[W / 2 + 4 * g + 1]),
                           pack_bf16(r[W / 2 + 4 * g + 2], r[W / 2 + 4 * g + 3]));
}

// The staging and store half of the drain, shared by the two schedules below: state of one warp of a group.
// `stg`: the group's two staging tiles (2 x W * 256 bytes, 1 KB aligned); `bar_id`: its named barrier.  Every tile
// of the accumulator loop starts with the first staging tile: the callers synchronise the group between two tiles
// (the barrier on which the group agrees that the next accumulator is ready), so the last read-back of one tile is
// over before the next one stages.
// row_of(c, t) returns where token t of chunk c starts in the result (the CTA's first row), or nullptr when that
// token lies outside; rows_valid = how many of the CTA's 128 rows exist (a multiple of 32).
template <int W>
struct DrainWarp {
  uint32_t stg, bar_id, dst, parity;
  int q, lane, unit;
  bool unit_ok;
  __device__ __forceinline__ DrainWarp(uint32_t stg_, uint32_t bar_id_, int q_, int lane_, int rows_valid)
      : stg(stg_), bar_id(bar_id_), parity(0), q(q_), lane(lane_), unit(lane_ & 15), unit_ok(8 * (lane_ & 15) < rows_valid) {
    // stmatrix: lane 8 i + k addresses token k (of a group of eight) of matrix i = rows 32 q + 8 i .. + 7, i.e. unit
    // 4 q + i of the token's 256-byte row
    dst = stg + (uint32_t)(lane & 7) * 256u + ((((uint32_t)(4 * q) + ((uint32_t)lane >> 3)) ^ ((uint32_t)lane & 7u)) << 4);
  }
  // reading back: this warp owns tokens (W/4) q .. (W/4) q + W/4 - 1; per step lanes 0-15 take one token, lanes 16-31
  // the next, 16 bytes (eight rows) per lane
  template <typename RowOf>
  __device__ __forceinline__ void emit(const uint32_t (&r)[W], int c, RowOf& row_of) {
    // Two tiles, one barrier per chunk: a tile is staged again two chunks later, and between the read-back of this
    // chunk and that staging every warp of the group passes the barrier of the chunk in between.
    const uint32_t tile = parity * (uint32_t)(W * 256);
    parity ^= 1u;
    uint16_t* row[W / 8];                                 // where this lane's tokens go: worked out ahead of the barrier
#pragma unroll
    for (int i = 0; i < W / 8; ++i) {
      uint16_t* r0 = row_of(c, (W / 4) * q + 2 * i + (lane >> 4));
      row[i] = (r0 != nullptr && unit_ok) ? r0 + 8 * unit : nullptr;
    }
    epi_stage<W>(r, dst + tile);
    ptx::named_bar_sync(bar_id, 128);
    uint4 v[W / 8];
#pragma unroll
    for (int i = 0; i < W / 8; ++i) {
      const int t = (W / 4) * q + 2 * i + (lane >> 4);
      v[i] = ptx::ld_shared_v4(stg + tile + (uint32_t)t * 256u + (((uint32_t)unit ^ ((uint32_t)t & 7u)) << 4));
    }
#pragma unroll
    for (int i = 0; i < W / 8; ++i)
      if (row[i] != nullptr) *reinterpret_cast<uint4*>(row[i]) = v[i];
  }
};

// After its last tensor-memory read a warp arrives once on `release_bar` (0: nobody waits for the accumulator).
__device__ __forceinline__ void release_accumulator(uint32_t release_bar, int lane) {
  if (release_bar != 0u) {
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive_cluster(release_bar);
  }
}

// The accumulator loop shared by the two write-out forms below: chunks c0, c0 + cstep, ... (< nchunks) of one
// accumulator (column of chunk c: W * c) go through emit(registers, c); one chunk is converted and written while the
// tensor-memory load of the next is in flight.
template <int W, typename Emit>
__device__ __forceinline__ void drain_loop(uint32_t acc, int c0, int cstep, int nchunks, bool zero, uint32_t release_bar,
                                           int lane, Emit&& emit) {
  uint32_t ra[W], rb[W];
  epi_load<W>(acc + W * c0, ra, zero);
#pragma unroll 1
  for (int c = c0; c < nchunks; c += 2 * cstep) {
    if (!zero) ptx::tmem_ld_wait();
    const bool more1 = c + cstep < nchunks;
    if (more1) epi_load<W>(acc + W * (c + cstep), rb, zero); else release_accumulator(release_bar, lane);
    emit(ra, c);
    if (!more1) break;
    if (!zero) ptx::tmem_ld_wait();
    if (c + 2 * cstep < nchunks) epi_load<W>(acc + W * (c + 2 * cstep), ra, zero); else release_accumulator(release_bar, lane);
    emit(rb, c + cstep);
  }
}

// Drains chunks c0, c0 + cstep, ... (< nchunks) of one accumulator; called by the four warps of a group with the
// same arguments except `acc` (the warp's lane quadrant q = warp % 4).  Results leave through per-lane 16-byte
// stores to addresses that row_of supplies (any token-to-address mapping: the implicit convolution's pixel boxes).
template <int W, typename RowOf>
__device__ __forceinline__ void drain_chunks(uint32_t acc, int c0, int cstep, int nchunks, bool zero, uint32_t release_bar,
                                             uint32_t stg, uint32_t bar_id, int q, int lane, int rows_valid, RowOf&& row_of) {
  if (c0 >= nchunks) { release_accumulator(release_bar, lane); return; }
  DrainWarp<W> d(stg, bar_id, q, lane, rows_valid);
  drain_loop<W>(acc, c0, cstep, nchunks, zero, release_bar, lane, [&](const uint32_t (&r)[W], int c) { d.emit(r, c, row_of); });
}

// The same drain for results that are a plain [token][row] matrix: a chunk leaves as two tensor stores (TMA) of
// W tokens x 64 rows, straight from a staging tile, issued by the group's STORE thread (store_chunks below) so
// that the draining warps never wait for a store to be issued.  A staging tile is two halves [W tokens][64 rows] of
// 128-byte token rows in the 128-byte-swizzled layout of the tensor map (16-byte unit index XOR token index mod 8
// -- the same XOR that keeps stmatrix free of bank conflicts).  The group's NT tiles are used in turn over the
// whole kernel (chunk number u of the group -> tile u % NT); two mbarriers per tile hand it back and forth:
//   staged[t]  (4 arrivals: one per draining warp, after stmatrix and a proxy fence)   drain -> store thread
//   freed[t]   (1 arrival: the store thread, once the tile's stores have read it)       store thread -> drain
// `bars`: the group's barriers (NT staged, then NT freed); `u`: the group's chunk counter, carried from call to
// call.  Returns false when a wait ran out of budget (the caller raises the abort flag).
template <int NT>
__device__ __forceinline__ void epi_bars_init(uint32_t bar_area) {
#pragma unroll
  for (int g = 0; g < EPI_GROUPS; ++g)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      ptx::mbar_init(bar_area + EPI_BAR_OFFSET + 8u * (g * 2 * NT + t), 4);
      ptx::mbar_init(bar_area + EPI_BAR_OFFSET + 8u * (g * 2 * NT + NT + t), 1);
    }
}
template <int NT>
__device__ __forceinline__ uint32_t epi_bars_of(uint32_t bar_area, int g) { return bar_area + EPI_BAR_OFFSET + 8u * (g * 2 * NT); }

template <int W, int NT>
__device__ __forceinline__ bool drain_chunks_tma(uint32_t acc, int c0, int cstep, int nchunks, bool zero, uint32_t release_bar,
                                                 uint32_t stg, uint32_t bars, uint32_t& u, int q, int lane,
                                                 volatile int* abort_flag) {
  if (c0 >= nchunks) { release_accumulator(release_bar, lane); return true; }
  // stmatrix: lane 8 i + k addresses token k (of a group of eight) of matrix i = rows 32 q + 8 i .. + 7, i.e. 16-byte
  // unit 4 (q & 1) + i of the token's row in half q >> 1
  const uint32_t dst = stg + (uint32_t)(q >> 1) * (uint32_t)(W * 128) + (uint32_t)(lane & 7) * 128u +
                       ((((uint32_t)(4 * (q & 1)) + ((uint32_t)lane >> 3)) ^ ((uint32_t)lane & 7u)) << 4);
  bool ok = true;
  drain_loop<W>(acc, c0, cstep, nchunks, zero, release_bar, lane, [&](const uint32_t (&r)[W], int) {
    const uint32_t slot = u % NT, use = u / NT;
    ++u;
    if (use > 0 && ok) ok = ptx::mbar_wait_bounded(bars + 8u * (NT + slot), (use - 1u) & 1u, abort_flag, WAIT_BUDGET);
    epi_stage<W, 1024u>(r, dst + slot * 8192u);
    ptx::fence_proxy_async();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bars + 8u * slot);
  });
  return ok;
}

// The store thread's side of drain_chunks_tma, called with the same chunk sequence: waits for a staged tile, issues
// its stores (rows and tokens outside the result are clipped by the tensor map, extent Mdim x Ndim; a store that
// would start outside is not issued), and hands back the tile of the previous chunk once its stores have read it.
// x0: first row of the CTA's 128; y0: first token of chunk 0.  After its last call the thread runs store_finish().
template <int W, int NT>
__device__ __forceinline__ bool store_chunks(const CUtensorMap* tmapD, int c0, int cstep, int nchunks, uint32_t stg,
                                             uint32_t bars, uint32_t& u, int x0, int y0, int Mdim, int Ndim,
                                             volatile int* abort_flag) {
  for (int c = c0; c < nchunks; c += cstep) {
    const uint32_t slot = u % NT, use = u / NT;
    if (!ptx::mbar_wait_bounded(bars + 8u * slot, use & 1u, abort_flag, WAIT_BUDGET)) return false;
    const int y = y0 + W * c;
    if (y < Ndim && x0 < Mdim) {
      ptx::tma_store_2d(tmapD, x0, y, stg + slot * 8192u);
      if (x0 + 64 < Mdim) ptx::tma_store_2d(tmapD, x0 + 64, y, stg + slot * 8192u + (uint32_t)(W * 128));
    }
    ptx::bulk_commit();
    if (u > 0) {
      ptx::bulk_wait_read<1>();
      ptx::mbar_arrive(bars + 8u * (NT + (u - 1u) % NT));
    }
    ++u;
  }
  return true;
}
// Shared memory must outlive the stores that read it.
__device__ __forceinline__ void store_finish() { ptx::bulk_wait_read<0>(); }

// ---- epilogue of a linear layer -----------------------------------------------------------------
// Y = act(D + b) + R, and the checkpoint of D + b, on the way out of the accumulator (EPI instantiations of the product
// kernels).
struct EpiParams {
  const float* bias;        // Mdim, or null
  int mode;                 // 3 BIMASK_ACT_* + 0 (no residual), 1 (residual), 2 (residual and checkpoint)
  int has_res;              // residual R, [Ndim][Mdim] bf16, through its tensor map
  int8_t* zq;               // checkpoint of D + b, [Ndim][Mdim], or null
  uint8_t* zs;              // its scales, [Ndim][Mdim / 32]
};

// The epilogue's arithmetic takes several times the instructions of a plain drain (20 to 30 per result with GELU and a
// checkpoint), and two warps per scheduler do not cover its latencies: the EPI kernels have sixteen draining warps in four
// groups.  Two groups share a RING of staging tiles and its store thread (ring r holds the chunks r, r + 2, ... of every
// tile); the ring's running chunk number n decides which of its two groups takes the chunk (n % 2).  The number of tiles
// per ring is even, so that a tile always serves the same group: an mbarrier's parity tells a waiter only about the phase
// after the last one it saw, and a group that came back to a tile two uses later could pass too early.
constexpr int LIN_EPI_WARPS = 16;
constexpr int LIN_THREADS = 64 + 32 * LIN_EPI_WARPS + 32 * EPI_GROUPS;

// Long reductions.  The tensor core's fp32 sums do not round to nearest, and their error grows with the chain: a sum of
// positive products is off by 1.3e-6 after 64 MMAs, by 3.7e-6 after 128, 3.2e-5 after 512.  So the CTA-pair kernel ends a
// chain after at most 96 (24 k tiles of a 2:4 operand, 12 of a dense one), a tile's chains about equally long; the two
// accumulators take them in turn, and the draining warps add them up (64 columns of one lane quadrant each) in fp32
// registers while the next chain runs.  The total goes back into the last chain's accumulator, from which the tile is drained
// like any other.  96, not 32 as elsewhere: a chain should last longer than the drain of the tile before it, which holds the
// other accumulator meanwhile.  512 rows x 6816 at 2495 tokens: 8.7e-6 -> 1.3e-6, and 30.0 -> 31.4 us; 1536 x 4096 at 8192
// 58.4 -> 60.4; dense 4096 x 4096 at 8192 174 -> 182; at worst 16384 x 4096 at 512 46 -> 51 (one round of tiles, nothing
// to hide the joining under).
__host__ __device__ constexpr int epi_segment(bool sparse) { return sparse ? 24 : 12; }   // k tiles
// Called by all sixteen draining warps; `quadrant`: tensor memory with the warp's lane offset, col0: its first column.  scount:
// running number of the tile's first chain on entry, of its last on return (chain c in accumulator c % nbuf).  The warps go on or
// give up together: a warp whose wait ran out still comes to the barrier.
__device__ __forceinline__ bool join_chains(uint32_t full_bar0, uint32_t empty_bar0, uint32_t quadrant, int col0, int n_tile, int nseg,
                                            uint32_t nbuf, uint32_t& scount, int lane, volatile int* abort_flag) {
  float sum[64];
#pragma unroll
  for (int j = 0; j < 64; ++j) sum[j] = 0.f;
  bool ok = true;
#pragma unroll 1
  for (int seg = 0; seg + 1 < nseg; ++seg, ++scount) {
    const uint32_t buf = scount & (nbuf - 1u), phase = (scount >> (nbuf - 1u)) & 1u;
    if (ok) ok = __all_sync(0xFFFFFFFFu, ptx::mbar_wait_bounded(full_bar0 + 8u * buf, phase, abort_flag, WAIT_BUDGET));
    if (!ok) continue;
    ptx::tc_fence_after();
#pragma unroll
    for (int j = 0; j < 64; j += 16) {
      if (col0 + j < n_tile) {
        uint32_t r[16];
        ptx::tmem_ld_32x16(quadrant + 256u * buf + (uint32_t)(col0 + j), r);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[j + i] += __uint_as_float(r[i]);
      }
    }
    release_accumulator(ptx::mapa(empty_bar0 + 8u * buf, 0), lane);
  }
  const uint32_t buf = scount & (nbuf - 1u), phase = (scount >> (nbuf - 1u)) & 1u;
  if (ok) ok = ptx::mbar_wait_bounded(full_bar0 + 8u * buf, phase, abort_flag, WAIT_BUDGET);
  ok = ptx::named_bar_and(1 + LIN_EPI_WARPS / 4, 32 * LIN_EPI_WARPS, ok);
  if (!ok) return false;
  ptx::tc_fence_after();
#pragma unroll
  for (int j = 0; j < 64; j += 16) {
    if (col0 + j < n_tile) {
      uint32_t r[16];
      ptx::tmem_ld_32x16(quadrant + 256u * buf + (uint32_t)(col0 + j), r);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(sum[j + i] + __uint_as_float(r[i]));
      ptx::tmem_st_32x16(quadrant + 256u * buf + (uint32_t)(col0 + j), r);
    }
  }
  ptx::tmem_st_wait();
  ptx::tc_fence_before();
  ptx::named_bar_sync(1 + LIN_EPI_WARPS / 4, 32 * LIN_EPI_WARPS);     // the chunks are drained by other warps than summed them
  return true;
}

// Checkpoint of one warp's chunk: 32 rows = one block of 32 channels, 32 tokens.  `z` in the accumulator-fragment
// layout (lane = 4 a + b: pair 8 h + 2 g + j holds row 16 h + 8 j + a, tokens 8 g + 2 b + {0, 1}).
//   scales: the maximum of a token's 32 values is four registers and the eight lanes that share b; the halving exchange
//           (two tokens per register, half of the registers sent away at each step) takes 4 shuffles, handing the
//           inverse scales of its eight tokens (powers of two, exact in bf16) back to every lane 3.
//   bytes:  two bytes of a token (rows a and a + 8 of a half) make a 16-bit element, which stmatrix transposes like
//           any other; a lane reads back the 16 bytes of half a block, undoes the pairing and stores them: a token's 32
//           bytes are one whole sector.
// `area`: 32 token rows of 128 bytes of which this warp may use units u0, u0 + 1 (16 bytes each, XOR token mod 8) as
// scratch.  q_out: where token 0's block goes; ntok: tokens of the chunk that exist.  The scales go to shared memory, one
// byte of a word per token (`scales`: this warp's byte of token 0): the store warp writes the four warps' together (bytes
// stored one by one cost 30 of 643 us on the 16384-row layer).
__device__ __forceinline__ void emit_checkpoint(const act::Pair (&z)[16], uint32_t area, uint32_t u0, int lane, int8_t* q_out,
                                                size_t q_pitch, uint32_t scales, int ntok) {
  uint32_t p[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float v[4][2];
#pragma unroll
    for (int m = 0; m < 4; ++m) act::split(z[8 * (m >> 1) + 2 * g + (m & 1)], v[m][0], v[m][1]);
    const float m0 = act::max_abs3(act::max_abs3(v[0][0], v[1][0], v[2][0]), v[3][0], 0.0f);
    const float m1 = act::max_abs3(act::max_abs3(v[0][1], v[1][1], v[2][1]), v[3][1], 0.0f);
    p[g] = __byte_perm(__float_as_uint(m0) + 0xFFFFu, __float_as_uint(m1) + 0xFFFFu, 0x7632);   // both rounded up to 16 bits
  }
  const bool hi = (lane & 16) != 0, mid = (lane & 8) != 0;
  uint32_t k0 = hi ? p[2] : p[0], k1 = hi ? p[3] : p[1];
  k0 = __vmaxu2(k0, __shfl_xor_sync(0xFFFFFFFFu, hi ? p[0] : p[2], 16));
  k1 = __vmaxu2(k1, __shfl_xor_sync(0xFFFFFFFFu, hi ? p[1] : p[3], 16));
  uint32_t k = mid ? k1 : k0;
  k = __vmaxu2(k, __shfl_xor_sync(0xFFFFFFFFu, mid ? k0 : k1, 8));
  k = __vmaxu2(k, __shfl_xor_sync(0xFFFFFFFFu, k, 4));     // tokens 8 g + 2 b + {0, 1}, g = lane / 8
  // ckpt::scale_of on both halves: `raw` is the scale of a block in range, the or'ed part is 255 where a block is not
  const uint32_t raw = __vmaxu2(((k + 0x00010001u) >> 7) & 0x01FF01FFu, 0x00070007u) - 0x00060006u;
  const uint32_t over = (k + 0x00010001u * (0x7FFFu - ckpt::LARGEST)) & 0x80008000u;
  const uint32_t s2 = raw | ((over >> 7) - (over >> 15));
  const int st = 8 * (lane >> 3) + 2 * (lane & 3) + ((lane >> 2) & 1);
  ptx::st_shared_u8(scales + 4u * (uint32_t)st, (lane & 4) ? s2 >> 16 : s2);
  const uint32_t inv2 = (0x00FE00FEu - raw) << 7;         // 2^(127 - s) of both tokens, as bf16
  const uint32_t o8 = __shfl_xor_sync(0xFFFFFFFFu, inv2, 8);
  const uint32_t g0 = mid ? o8 : inv2, g1 = mid ? inv2 : o8;
  const uint32_t h0 = __shfl_xor_sync(0xFFFFFFFFu, g0, 16), h1 = __shfl_xor_sync(0xFFFFFFFFu, g1, 16);
  const uint32_t invs[4] = {hi ? h0 : g0, hi ? h1 : g1, hi ? g0 : h0, hi ? g1 : h1};
  uint32_t w[8];                                          // w[2 g + h]: low half token e = 0, high half e = 1
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const act::Pair inv = act::pair(bf16_lo(invs[g]), bf16_hi(invs[g]));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float a0, a1, b0, b1;
      act::split(act::fma2(z[8 * h + 2 * g], inv, act::both(ckpt::ROUNDER)), a0, a1);
      act::split(act::fma2(z[8 * h + 2 * g + 1], inv, act::both(ckpt::ROUNDER)), b0, b1);
      w[2 * g + h] = __byte_perm(__byte_perm(__float_as_uint(a0), __float_as_uint(b0), 0x0040),
                                 __byte_perm(__float_as_uint(a1), __float_as_uint(b1), 0x0040), 0x5410);
    }
  }
  const uint32_t lt = (uint32_t)lane & 7u, li = (uint32_t)lane >> 3;   // stmatrix: lane 8 i + k addresses token k of matrix i
#pragma unroll
  for (int g = 0; g < 4; g += 2)                          // matrices (g, half 0), (g, half 1), (g + 1, half 0), (g + 1, half 1)
    ptx::stmatrix_x4_trans(area + (8u * (g + (li >> 1)) + lt) * 128u + (((u0 + (li & 1u)) ^ lt) << 4), w[2 * g], w[2 * g + 1],
                           w[2 * g + 2], w[2 * g + 3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = 16 * i + (lane & 15), h = lane >> 4;
    const uint4 v = ptx::ld_shared_v4(area + (uint32_t)t * 128u + (((u0 + (uint32_t)h) ^ lt) << 4));
    if (t < ntok)
      *reinterpret_cast<uint4*>(q_out + (size_t)t * q_pitch + 16 * h) =
          make_uint4(__byte_perm(v.x, v.y, 0x6420), __byte_perm(v.z, v.w, 0x6420), __byte_perm(v.x, v.y, 0x7531), __byte_perm(v.z, v.w, 0x7531));
  }
  __syncwarp();                                           // the scratch area is the warp's again
}

// act(z) + residual, packed to bf16 and staged: straight-line code for each combination.  RES 1: the residual is in the
// staging tile on entry and is read in the fragment layout that stmatrix writes back; 2: it has been read into `res`
// already.  `dst`: this lane's stmatrix row for token group 0.
template <int ACT, int RES>
__device__ __forceinline__ void emit_result(const act::Pair (&z)[16], uint32_t dst, const uint32_t (&res)[16]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    uint32_t y[4];                                        // matrix m: rows 8 m + a, tokens 8 g + 2 b + {0, 1}
    if (RES == 1) ptx::ldmatrix_x4_trans(dst + 1024u * g, y[0], y[1], y[2], y[3]);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      act::Pair v = act::value2<ACT>(z[8 * (m >> 1) + 2 * g + (m & 1)]);
      if (RES != 0) {
        const uint32_t r = RES == 1 ? y[m] : res[4 * g + m];
        v = act::add2(v, act::pair(bf16_lo(r), bf16_hi(r)));
      }
      float lo, hi;
      act::split(v, lo, hi);
      y[m] = pack_bf16_f(lo, hi);
    }
    if (RES == 1) __syncwarp();                           // all lanes have read these eight tokens
    ptx::stmatrix_x4_trans(dst + 1024u * g, y[0], y[1], y[2], y[3]);
  }
}

// The bias of a draining warp's rows in the fragment layout: rows 8 k + lane / 4 of the 32 from row0 on.  Loaded before
// the accumulator is waited for.
__device__ __forceinline__ void epi_bias(const float* bias, int row0, int Mdim, int lane, float (&b)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = (bias != nullptr && row0 < Mdim) ? __ldg(bias + row0 + 8 * k + (lane >> 2)) : 0.f;
}

// One tile's share of a draining warp: the ring's chunks of this tile are c = ring, ring + 2, ... (`first`: the ring's
// index for this tile, 0 or 1; they carry the running numbers n0, n0 + 1, ...), and the group takes those whose number
// is `sub` modulo 2.  n0 is advanced by the ring's count.
// With a residual, `freed[t]` is completed by the arrival of the residual tile of the chunk in staging tile t
// (store_chunks_epi loads it there as soon as the tile's last store has read it), so it is waited for on every use;
// ldmatrix reads the tile in the fragment layout that stmatrix then writes back.
// b: epi_bias of the warp's rows; x0: first row of the CTA's 128; y0: first token of chunk 0.
template <int NT>
__device__ __forceinline__ bool drain_chunks_epi(uint32_t acc, int first, int sub, int nchunks, uint32_t release_bar, uint32_t stg,
                                                 uint32_t bars, uint32_t scales, uint32_t& n0, int q, int lane, const EpiParams& e,
                                                 const float (&b)[4], int x0, int y0, int Mdim, int Ndim, volatile int* abort_flag) {
  static_assert(NT % 2 == 0, "a staging tile serves one group");
  const int count = (nchunks - first + 1) / 2;
  uint32_t n = n0 + (((uint32_t)sub - n0) & 1u);           // the group's first chunk of this tile
  const uint32_t end = n0 + (uint32_t)count;
  if (n >= end) { release_accumulator(release_bar, lane); n0 = end; return true; }
  const uint32_t half = stg + (uint32_t)(q >> 1) * 4096u;
  const uint32_t dst = half + (uint32_t)(lane & 7) * 128u +
                       ((((uint32_t)(4 * (q & 1)) + ((uint32_t)lane >> 3)) ^ ((uint32_t)lane & 7u)) << 4);
  const int row0 = x0 + 32 * q;                           // this warp's 32 rows all exist or none does
  const bool rows_ok = row0 < Mdim;
  bool ok = true;
#pragma unroll 1
  for (; n < end; n += 2) {
    const int c = first + 2 * (int)(n - n0);
    const uint32_t slot = n % NT, use = n / NT;
    act::Pair z[16];
    {
      uint32_t r[32];
      epi_load<32>(acc + 32 * c, r, false);
      ptx::tmem_ld_wait();
      if (n + 2 >= end) release_accumulator(release_bar, lane);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        z[i] = act::add2(act::pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), act::both(b[2 * (i >> 3) + (i & 1)]));
    }
    if (ok) {
      if (e.has_res) ok = ptx::mbar_wait_bounded(bars + 8u * (NT + slot), use & 1u, abort_flag, WAIT_BUDGET);
      else if (use > 0) ok = ptx::mbar_wait_bounded(bars + 8u * (NT + slot), (use - 1u) & 1u, abort_flag, WAIT_BUDGET);
    }
    __syncwarp();
    const uint32_t tile = slot * 8192u;
    uint32_t res[16];
    if (e.zq != nullptr) {
      if (e.has_res) {                                    // the checkpoint's scratch is where the residual lies
#pragma unroll
        for (int g = 0; g < 4; ++g) ptx::ldmatrix_x4_trans(dst + tile + 1024u * g, res[4 * g], res[4 * g + 1], res[4 * g + 2], res[4 * g + 3]);
        __syncwarp();
      }
      const int t0 = y0 + 32 * c;
      emit_checkpoint(z, half + tile, 4u * (q & 1), lane, e.zq + (size_t)t0 * Mdim + row0, (size_t)Mdim, scales + 128u * slot + (uint32_t)q,
                      rows_ok ? Ndim - t0 : 0);
    }
    switch (e.mode) {
#define BIMASK_EMIT(m) case m: emit_result<m / 3, m % 3>(z, dst + tile, res); break;
      BIMASK_EMIT(0) BIMASK_EMIT(1) BIMASK_EMIT(2) BIMASK_EMIT(3) BIMASK_EMIT(4) BIMASK_EMIT(5) BIMASK_EMIT(6) BIMASK_EMIT(7)
      BIMASK_EMIT(8) BIMASK_EMIT(9) BIMASK_EMIT(10) BIMASK_EMIT(11) BIMASK_EMIT(12) BIMASK_EMIT(13) BIMASK_EMIT(14)
#undef BIMASK_EMIT
    }
    ptx::fence_proxy_async();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bars + 8u * slot);
  }
  n0 = end;
  return ok;
}

// The store warp's side.  `walk` yields the ring's chunks one after the other, over all its tiles: next(x0, y) gives
// the first row and token, false past the last.  Lane 0 sends the tiles off; with a checkpoint every lane stores one token's
// scales (`scales`: a word per token and staging tile).  With a residual a second copy of the walk runs NT chunks ahead: the
// residual tile of chunk n + NT is loaded into the staging tile of chunk n once that chunk's store has read it.
template <int NT, typename Walk>
__device__ __forceinline__ bool store_chunks_epi(const CUtensorMap* tmapD, const CUtensorMap* tmapR, const EpiParams& e, uint32_t stg,
                                                 uint32_t bars, uint32_t scales, int lane, int Mdim, int Ndim, volatile int* abort_flag,
                                                 Walk walk) {
  Walk ahead = walk;
  const bool has_res = e.has_res != 0;
  uint32_t loaded = 0;                                    // residual tiles requested so far
  auto load = [&]() {
    int x0, y;
    if (!ahead.next(x0, y)) return;
    const uint32_t slot = loaded % NT, bar = bars + 8u * (NT + slot);
    ptx::mbar_expect_tx(bar, 8192);
    ptx::tma_load_2d(stg + slot * 8192u, tmapR, x0, y, bar);
    ptx::tma_load_2d(stg + slot * 8192u + 4096u, tmapR, x0 + 64, y, bar);
    ++loaded;
  };
  if (has_res && lane == 0)
    for (uint32_t n = 0; n < NT; ++n) load();
  bool ok = true;
  int x0, y;
  for (uint32_t n = 0; walk.next(x0, y); ++n) {
    const uint32_t slot = n % NT, use = n / NT;
    ok = ptx::mbar_wait_bounded(bars + 8u * slot, use & 1u, abort_flag, WAIT_BUDGET);
    ok = __all_sync(0xFFFFFFFFu, ok);
    if (!ok) break;
    if (lane == 0) {
      if (y < Ndim && x0 < Mdim) {
        ptx::tma_store_2d(tmapD, x0, y, stg + slot * 8192u);
        if (x0 + 64 < Mdim) ptx::tma_store_2d(tmapD, x0 + 64, y, stg + slot * 8192u + 4096u);
      }
      ptx::bulk_commit();
    }
    if (e.zq != nullptr && x0 < Mdim) {
      const uint32_t w = ptx::ld_shared_u32(scales + 128u * slot + 4u * (uint32_t)lane);
      if (y + lane < Ndim) {
        uint8_t* out = e.zs + (size_t)(y + lane) * (Mdim >> 5) + (x0 >> 5);
        if (Mdim % 128 == 0) {
          *reinterpret_cast<uint32_t*>(out) = w;
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (x0 + 32 * k < Mdim) out[k] = (uint8_t)(w >> (8 * k));
        }
      }
      __syncwarp();                                       // the words have been read: the tile may be handed back
    }
    // With two tiles, one per group, a tile is handed back as soon as its store has read it: its group cannot go on
    // before (1 % on the 16384-row layers).  With four, the wait goes under the next store.
    if (lane == 0 && (NT <= 2 || n > 0)) {
      ptx::bulk_wait_read<(NT <= 2 ? 0 : 1)>();
      if (has_res) load();
      else ptx::mbar_arrive(bars + 8u * (NT + (NT <= 2 ? slot : (n - 1u) % NT)));
    }
  }
  if (lane == 0) {
    if (has_res) {                                        // no load may be in flight when the kernel ends, whoever gave up
      volatile int none = 0;
      for (uint32_t n = loaded > NT ? loaded - NT : 0; n < loaded; ++n)
        ptx::mbar_wait_bounded(bars + 8u * (NT + n % NT), (n / NT) & 1u, &none, DRAIN_BUDGET);
    }
    store_finish();
  }
  return ok;
}

// The chunks of ring `ring` in the order of the draining warps.  A tile is ROWS accumulators of 128 rows of this CTA,
// `row_step` rows apart, drained one after the other; accumulator m takes the chunks (ring ^ m) & 1, + 2, ...
template <int ROWS>
struct ChunkWalk {
  int tile, step, num_tiles, tiles_m, tiles_n, group;     // the CTA's tiles
  int rows_per_tile, row_off, row_step, n_tile, ring;
  int m, c, x0, y0;                                       // position: accumulator and chunk of the current tile
  __device__ __forceinline__ void enter() {
    if (tile < num_tiles) {
      int tile_m, tile_n;
      raster(tile, tiles_m, tiles_n, group, tile_m, tile_n);
      x0 = tile_m * rows_per_tile + row_off;
      y0 = tile_n * n_tile;
    }
    m = 0;
    c = ring;
  }
  __device__ __forceinline__ bool next(int& x, int& y) {
    while (32 * c >= n_tile) {                            // past the accumulator's last chunk
      if (tile >= num_tiles) return false;
      if (ROWS > 1 && m + 1 < ROWS) {
        ++m;
        c = (ring ^ m) & 1;
      } else {
        tile += step;
        enter();
      }
    }
    if (tile >= num_tiles) return false;
    x = x0 + m * row_step;
    y = y0 + 32 * c;
    c += 2;
    return true;
  }
};
template <int ROWS>
__device__ __forceinline__ ChunkWalk<ROWS> chunk_walk(const GemmParams& p, int tile, int step, int num_tiles, int rows_per_tile, int row_off,
                                                      int row_step, int n_tile, int ring) {
  ChunkWalk<ROWS> w{tile, step, num_tiles, p.tiles_m, p.tiles_n, p.raster_group, rows_per_tile, row_off, row_step, n_tile, ring, 0, 0, 0, 0};
  w.enter();
  return w;
}

// ---- host helpers (gemm_host.cu) -----------------------------------------------------------
// 2-D bf16 tensor map: `inner` contiguous elements per row, `outer` rows, box = 64 x box_rows, 128-byte swizzle,
// out-of-range elements read as zero.
int make_tmap(CUtensorMap* m, const void* ptr, uint64_t inner, uint64_t outer, uint32_t box_rows);
// The metadata image as a 2-D tensor of u32: 256 words per row, two rows per 2048-byte block.
int make_tmap_meta(CUtensorMap* m, const void* ptr, uint64_t blocks);
// fp32 [planes][rows][inner] for stores of 32 x 128 boxes (the dense product's result or its split-K partial sums).
int make_tmap_f32_store(CUtensorMap* m, const void* ptr, uint64_t inner, uint64_t rows, uint64_t planes);
// 4-D bf16 map of an NHWC tensor (channels, W, H, NB) for loads of 64-channel pixel boxes, 128-byte swizzle.
// estride 2: a box takes every second pixel along W and H (wb x hb pixels all the same).
int make_tmap_nhwc_load(CUtensorMap* m, const void* ptr, int CH, int W, int H, int NB, int wb, int hb, int nb, int estride = 1);

// ---- pixel boxes of the implicit convolution ------------------------------------------------
inline int pow2_ceil(int v) { int p = 1; while (p < v) p <<= 1; return p; }
inline int log2_exact(int v) { int l = 0; while ((1 << l) < v) ++l; return l; }

// Pixel boxes of `tokens` tokens: as wide as the image allows (16 or 8), at least 32 tokens per image of the box.
inline void conv_boxes(ConvGeom& g, int tokens) {
  g.wb = g.W > 8 ? 16 : 8;
  int hb = tokens / g.wb;
  const int hp = pow2_ceil(g.H);
  if (hb > hp) hb = hp;
  if (hb < 32 / g.wb) hb = 32 / g.wb;
  g.hb = hb;
  g.nb = tokens / (g.wb * g.hb);
  g.lg_wb = log2_exact(g.wb);
  g.lg_hb = log2_exact(g.hb);
  g.tiles_w = (g.W + g.wb - 1) / g.wb;
  g.tiles_h = (g.H + g.hb - 1) / g.hb;
}

}  // namespace bimask
