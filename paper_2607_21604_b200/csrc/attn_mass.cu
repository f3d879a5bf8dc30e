// Attention weight that every cached key has received: per kv head h and key j
//     mass_out[h][j] = mass_in[h][j] + sum over rows r that see j, heads i of the group of h:
//                      exp(q_ri . k_jh / sqrt(hd) - lse_ri)
// with lse the log-sum-exp of the row, as the attention that produced the row left it.
// The rows of the g = n_q / n_kv query heads of a kv head are stacked (r * g + i); every sum runs
// over them in a fixed order, so equal calls give equal bits.
//
// 16-bit types run on the tensor cores with the keys along M, so that a thread owns one key and its
// sum over the rows needs no shuffle; the score matrix never leaves tensor memory:
//     S^T = K Q^T     tcgen05.mma, two tiles of 128 keys against one tile of up to 256 stacked rows
//     sum             two warp groups, one per key tile: exp2 of a row of S^T, added up in registers
// A CTA keeps 256 keys in shared memory while the rows' Q tiles stream past them (each is used
// twice), then goes on to its next 256 keys.  Two warps work out what each column sees; a tile whose
// columns all see its keys runs without a mask.  The exponentials bound it from below (16 per clock
// and SM: 4096 clocks for 256 keys x 256 rows, 160 us of the 229 us that 512 rows x 40 heads x 32768
// keys take); the rest is the MMA of a group's next tile, which waits for its only buffer.  With few
// rows it is bound by reading K once (16 rows x 32 heads over 12416 keys: 8.9 us, 3.0 TB/s).
// Few keys and many rows: a cluster shares the row tiles of its keys and adds the
// partial sums through distributed shared memory.
#include "tc_common.cuh"
#include <math.h>

namespace {

struct MassParams {
  const void* q;
  const void* k;
  int64_t q_ld, k_ld;
  const float* lse;                  // [R][n_q]
  const int32_t* k_lo;
  const int32_t* k_hi;
  int R, T, n_q, n_kv, g;
  const float* mass_in;              // null: zeros
  float* mass_out;
  float scale;                       // 1 / sqrt(hd)
};

constexpr float LOG2E = 1.4426950408889634f;

// ---- tensor cores
constexpr int BK = 128;              // keys of a tile, two tiles per item
constexpr int M_THREADS = 384;       // warp group 0: TMA and MMA, warp groups 1 and 2: sums
constexpr int M_SLAB = 128 * 128;    // 128 rows of 64 values
// FEW: all stacked rows fit 128 columns.  One Q tile stays as long as the head does, K streams
// through two stages and S^T has two buffers, so that items overlap.  Otherwise row tiles of 256
// columns stream past one K item: an MMA of 256 columns reads its A operand from shared memory half
// as often per column, and the load of the next K hides behind the sums of the last tile (512 rows
// x 40 heads x 32768 keys: 229 us, against 238 us with two buffers of 128 columns).
template <bool FEW> struct MassCfg {
  static constexpr int BQ = FEW ? 128 : 256, NB = FEW ? 2 : 1, KST = FEW ? 2 : 1, QST = FEW ? 1 : 2;
};
template <int HD> constexpr int M_TILE = HD / 64 * M_SLAB;               // 128 rows
// shared memory: K[KST][2 tiles] | Q[QST] | barriers (256 B) | what a column sees, twice | partial sums | flags
template <bool FEW> constexpr int M_COLS = 2 * MassCfg<FEW>::BQ * (4 + 8);
template <int HD, bool FEW> constexpr int M_SMEM = (2 * MassCfg<FEW>::KST + MassCfg<FEW>::QST * MassCfg<FEW>::BQ / 128) * M_TILE<HD> +
                                                   256 + M_COLS<FEW> + 2 * 128 * 4 + 64;
enum { MB_KFULL = 0, MB_KEMPTY = 2, MB_QFULL = 4, MB_QEMPTY = 6,
       MB_SFULL = 8,                          // [2 groups][2 buffers] S^T of a tile is complete
       MB_SEMPTY = 12,                        // [2][2] the group has taken it into registers (4 warps)
       MB_CFULL = 16, MB_CEMPTY = 18,         // [2] what the columns of a tile see has been written / read (2 warps, 8 warps)
       MB_COUNT = 20 };
static_assert(MB_COUNT * 8 + 8 <= 256, "barriers, the tensor-memory slot and the abort flag share 256 bytes");
static_assert(M_SMEM<128, true> <= 232448 && M_SMEM<128, false> <= 232448, "shared memory of one CTA");

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T, int HD, bool FEW>
__global__ void __launch_bounds__(M_THREADS, 1)
mass_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ, const MassParams p,
               int C, int key_items, int n_items, int BR, int q_boxes, uint32_t fmt) {
  using Cfg = MassCfg<FEW>;
  constexpr int TILE = M_TILE<HD>, BQ = Cfg::BQ, NB = Cfg::NB, KST = Cfg::KST, QST = Cfg::QST, Q_BYTES = BQ / 128 * TILE;
  constexpr int OFF_Q = 2 * KST * TILE, OFF_BAR = OFF_Q + QST * Q_BYTES, OFF_COL = OFF_BAR + 256;
  constexpr int OFF_PART = OFF_COL + M_COLS<FEW>, OFF_FLAG = OFF_PART + 2 * 128 * 4, Q_SLAB = BQ * 128;
  extern __shared__ __align__(1024) uint8_t smem[];
  if (tc::smem_u32(smem) & 1023u) return;           // swizzled tiles need 1024-byte alignment (the same in every CTA)
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + MB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* part = reinterpret_cast<float*>(smem + OFF_PART);          // [2][128]
  float* col_z = reinterpret_cast<float*>(smem + OFF_COL);          // [2][BQ] -lse of a column in log2 units
  int2* col_rng = reinterpret_cast<int2*>(col_z + 2 * BQ);          // [2][BQ] its first visible key, and how many follow
  volatile int* flag = reinterpret_cast<volatile int*>(smem + OFF_FLAG);    // [2][2 groups][2 halves] a column needs a mask
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < MB_COUNT; ++i) tc::mbar_init(&bar[i], i >= MB_CEMPTY ? 8 : i >= MB_CFULL ? 2 : i >= MB_SEMPTY ? 4 : 1);
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  // Q tiles hold BR * g rows; what the loads leave out behind them stays zero
  for (int i = threadIdx.x; i < QST * Q_BYTES / 16; i += M_THREADS)
    *reinterpret_cast<uint4*>(smem + OFF_Q + i * 16) = make_uint4(0u, 0u, 0u, 0u);
  tc::fence_proxy_async();
  pdl_wait();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // FEW: consecutive items (of one head, mostly) for each cluster.  Otherwise every n_cl-th, so that
  // masked items (the end of a causal window) spread.
  const int rank = blockIdx.x % C, n_cl = gridDim.x / C, cl = blockIdx.x / C;
  const int item0 = FEW ? (int)((int64_t)n_items * cl / n_cl) : cl, step = FEW ? 1 : n_cl;
  const int item1 = FEW ? (int)((int64_t)n_items * (cl + 1) / n_cl) : n_items;
  const int row_tiles = (p.R + BR - 1) / BR;
  auto head_ends = [&](int item) { return item + 1 == item1 || (item + 1) / key_items != item / key_items; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0) {
      // ------------------------------------------------------------------ TMA producer
      if (lane == 0) {
        tc::prefetch_tmap(&tmK);
        tc::prefetch_tmap(&tmQ);
        // boxes of at most 128 stacked rows, back to back
        const int box_rows = BR / q_boxes, box_bytes = box_rows * p.g * 128;
        bool ok = true;
        int it = 0, n = 0;
        for (int item = item0; item < item1 && ok; item += step, ++it) {
          const int h = item / key_items, j0 = (item % key_items) * (2 * BK), ks = it % KST;
          if (!tc::mbar_wait(&bar[MB_KEMPTY + ks], ((it / KST) & 1) ^ 1, abort_flag)) { ok = false; break; }
          tc::mbar_expect_tx(&bar[MB_KFULL + ks], 2 * TILE);
#pragma unroll
          for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int c = 0; c < HD / 64; ++c)
              tc::tma_load_2d(smem + (2 * ks + w) * TILE + c * M_SLAB, &tmK, h * HD + c * 64, j0 + w * BK, &bar[MB_KFULL + ks]);
          if (FEW && it > 0 && (item - 1) / key_items == h) continue;    // the head's rows are there
          for (int rt = rank; rt < row_tiles; rt += C, ++n) {
            const int qs = n % QST;
            if (!tc::mbar_wait(&bar[MB_QEMPTY + qs], ((n / QST) & 1) ^ 1, abort_flag)) { ok = false; break; }
            tc::mbar_expect_tx(&bar[MB_QFULL + qs], (uint32_t)(q_boxes * box_bytes * (HD / 64)));
            for (int x = 0; x < q_boxes; ++x)
#pragma unroll
              for (int c = 0; c < HD / 64; ++c)
                tc::tma_load_3d(smem + OFF_Q + qs * Q_BYTES + c * Q_SLAB + x * box_bytes, &tmQ, c * 64, h * p.g,
                                rt * BR + x * box_rows, &bar[MB_QFULL + qs]);
          }
        }
        if (!ok) *abort_flag = 1;
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      if (lane == 0) {
        bool ok = true;
        int it = 0, n = 0, nq = 0;                    // items, tiles, Q tiles so far
        for (int item = item0; item < item1 && ok; item += step, ++it) {
          const int ks = it % KST;
          if (!tc::mbar_wait(&bar[MB_KFULL + ks], (it / KST) & 1, abort_flag)) { ok = false; break; }
          for (int rt = rank; rt < row_tiles && ok; rt += C, ++n) {
            const int qs = nq % QST, b = n % NB;
            if (!tc::mbar_wait(&bar[MB_QFULL + qs], (nq / QST) & 1, abort_flag)) { ok = false; break; }
            const int cols = min(BR, p.R - rt * BR) * p.g;
            const uint32_t idesc = tc::idesc_f16(fmt, BK, (cols + 63) / 64 * 64, 0);      // whole chunks: rows of zeros behind the last
            const uint32_t q_addr = tc::smem_u32(smem + OFF_Q + qs * Q_BYTES);
            for (int w = 0; w < 2; ++w) {
              if (!tc::mbar_wait(&bar[MB_SEMPTY + 2 * w + b], ((n / NB) & 1) ^ 1, abort_flag)) { ok = false; break; }
              tc::fence_after_sync();
              const uint32_t k_addr = tc::smem_u32(smem + (2 * ks + w) * TILE);
#pragma unroll
              for (int k = 0; k < HD / 16; ++k)
                tc::mma_f16(tmem_base + w * 256 + b * BQ, tc::smem_desc_k_sw128(k_addr + (k >> 2) * M_SLAB + (k & 3) * 32),
                            tc::smem_desc_k_sw128(q_addr + (k >> 2) * Q_SLAB + (k & 3) * 32), idesc, k != 0);
              tc::mma_commit(&bar[MB_SFULL + 2 * w + b]);
            }
            if (ok && (!FEW || head_ends(item))) { tc::mma_commit(&bar[MB_QEMPTY + qs]); ++nq; }
          }
          if (ok) tc::mma_commit(&bar[MB_KEMPTY + ks]);
        }
        if (!ok) *abort_flag = 1;
      }
    }
    else {
      // ------------------------------------------------------------------ what the columns see
      // In two warps of their own, half of the columns each, all loads in flight together: in the
      // summing warps, or one column after the other, the latency of these loads bounded the kernel.
      constexpr int CPL = BQ / 64;
      const int half = warp - 2;
      int r_in[CPL], head_in[CPL];
#pragma unroll
      for (int x = 0; x < CPL; ++x) {
        const int i = x * 64 + half * 32 + lane;
        r_in[x] = i < BR * p.g ? i / p.g : 0x3fffffff;
        head_in[x] = i % p.g;
      }
      bool ok = true;
      int n = 0;
      for (int item = item0; item < item1 && ok; item += step) {
        const int h = item / key_items, k0 = (item % key_items) * (2 * BK);
        for (int rt = rank; rt < row_tiles; rt += C, ++n) {
          const int cb = n & 1;
          float z[CPL];
          int lo[CPL], hi[CPL];
#pragma unroll
          for (int x = 0; x < CPL; ++x) {
            const int r = min(rt * BR + min(r_in[x], BR), p.R - 1);
            z[x] = __ldg(p.lse + (int64_t)r * p.n_q + h * p.g + head_in[x]);
            lo[x] = __ldg(p.k_lo + r);
            hi[x] = __ldg(p.k_hi + r);
          }
          if (!tc::mbar_wait(&bar[MB_CEMPTY + cb], ((n >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
          bool masked[2] = {false, false};
#pragma unroll
          for (int x = 0; x < CPL; ++x) {
            const int i = x * 64 + half * 32 + lane;
            const bool real = r_in[x] < BR && rt * BR + r_in[x] < p.R;
            lo[x] = max(lo[x], 0);
            hi[x] = min(hi[x], p.T - 1);
            const bool blind = !real || z[x] == -INFINITY || lo[x] > hi[x];     // such a row adds nothing
            // a column of zeros behind the last row needs no mask: exp2(0 - inf) = 0
#pragma unroll
            for (int w = 0; w < 2; ++w)
              masked[w] |= real && (blind || lo[x] > k0 + w * BK || hi[x] < min(k0 + (w + 1) * BK, p.T) - 1);
            col_z[cb * BQ + i] = blind ? -INFINITY : -z[x] * LOG2E;
            // seen <=> (unsigned)(key - first) <= length: never for a blind row (keys are not negative)
            col_rng[cb * BQ + i] = blind ? make_int2(0x7fffffff, 0) : make_int2(lo[x], hi[x] - lo[x]);
          }
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const bool any = __any_sync(0xFFFFFFFFu, masked[w]);
            if (lane == 0) flag[(cb * 2 + w) * 2 + half] = any;
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bar[MB_CFULL + cb]);
        }
      }
      if (!ok && lane == 0) *abort_flag = 1;
    }
  } else {
    // ---------------------------------------------------------------------- a key per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int w = (warp >> 2) - 1, m = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
    const float scale2 = p.scale * LOG2E;
    bool ok = true;
    int n = 0;
    for (int item = item0; item < item1 && ok; item += step) {
      const int h = item / key_items, key = (item % key_items) * (2 * BK) + w * BK + m;
      float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int rt = rank; rt < row_tiles; rt += C, ++n) {
        const int b = n % NB, cb = n & 1;
        const int all_cols = min(BR, p.R - rt * BR) * p.g;
        if (!tc::mbar_wait(&bar[MB_CFULL + cb], (n >> 1) & 1, abort_flag)) { ok = false; break; }
        const bool mask = (flag[(cb * 2 + w) * 2] | flag[(cb * 2 + w) * 2 + 1]) != 0;
        if (!tc::mbar_wait(&bar[MB_SFULL + 2 * w + b], (n / NB) & 1, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
        // 64 columns at a time, the next ones on their way from tensor memory meanwhile
        const uint32_t s_addr = lane_addr + w * 256 + b * BQ;
        const int chunks = (all_cols + 63) / 64;
        float ta[64], tb[64];
        auto fetch = [&](float(&t)[64], int c) {
          tc::tmem_ld32(s_addr + c * 64, *reinterpret_cast<float(*)[32]>(&t[0]));
          tc::tmem_ld32(s_addr + c * 64 + 32, *reinterpret_cast<float(*)[32]>(&t[32]));
        };
        auto arrived = [&](int c) {
          tc::tmem_ld_wait();
          if (c + 1 == chunks) {                          // all of the tile is in registers: its buffer is free
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&bar[MB_SEMPTY + 2 * w + b]);
          }
        };
        auto add = [&](const float(&t)[64], int c) {
          const float* z = col_z + cb * BQ + c * 64;
          const float2 sc = make_float2(scale2, scale2);
          // no branch inside: the loads, exponentials and sums of different columns overlap
          if (!mask) {
#pragma unroll
            for (int i = 0; i < 64; i += 4) {
              const float4 zz = *reinterpret_cast<const float4*>(z + i);
              const float2 x = __ffma2_rn(make_float2(t[i], t[i + 1]), sc, make_float2(zz.x, zz.y));
              const float2 y = __ffma2_rn(make_float2(t[i + 2], t[i + 3]), sc, make_float2(zz.z, zz.w));
              acc[(i >> 1) & 3] = __fadd2_rn(acc[(i >> 1) & 3], make_float2(ex2(x.x), ex2(x.y)));
              acc[((i >> 1) + 1) & 3] = __fadd2_rn(acc[((i >> 1) + 1) & 3], make_float2(ex2(y.x), ex2(y.y)));
            }
          } else {
            const int2* ranges = col_rng + cb * BQ + c * 64;
#pragma unroll
            for (int i = 0; i < 64; i += 2) {
              const float2 zz = *reinterpret_cast<const float2*>(z + i);
              const int4 rng = *reinterpret_cast<const int4*>(ranges + i);
              const float2 x = __ffma2_rn(make_float2(t[i], t[i + 1]), sc, zz);
              const float e0 = ex2(x.x), e1 = ex2(x.y);
              acc[(i >> 1) & 3] = __fadd2_rn(acc[(i >> 1) & 3], make_float2((unsigned)(key - rng.x) <= (unsigned)rng.y ? e0 : 0.f,
                                                                          (unsigned)(key - rng.z) <= (unsigned)rng.w ? e1 : 0.f));
            }
          }
        };
        fetch(ta, 0);
        for (int c = 0; c < chunks; c += 2) {
          arrived(c);
          if (c + 1 < chunks) fetch(tb, c + 1);
          add(ta, c);
          if (c + 1 >= chunks) break;
          arrived(c + 1);
          if (c + 2 < chunks) fetch(ta, c + 2);
          add(tb, c + 1);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bar[MB_CEMPTY + cb]);
      }
      if (!ok) break;
      const float2 s01 = __fadd2_rn(acc[0], acc[1]), s23 = __fadd2_rn(acc[2], acc[3]);
      const float sum = (s01.x + s01.y) + (s23.x + s23.y);
      const int64_t at = (int64_t)h * p.T + key;
      if (C == 1) {
        if (key < p.T) p.mass_out[at] = (p.mass_in ? p.mass_in[at] : 0.f) + sum;
      } else {
        part[w * 128 + m] = sum;
      }
    }
    if (!ok) *abort_flag = 1;
  }
  if (*abort_flag) __nanosleep(200000);
  tc::fence_before_sync();
  __syncthreads();
  if (C > 1) {
    // a cluster has one item: its first CTA adds the parts in rank order
    tc::cluster_sync_all();
    if (rank == 0 && warp >= 4) {
      const int w = (warp >> 2) - 1, m = threadIdx.x & 127, h = item0 / key_items, key = (item0 % key_items) * (2 * BK) + w * BK + m;
      float sum = 0.f;
      for (int c = 0; c < C; ++c) {
        float x;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(tc::map_to_rank(tc::smem_u32(&part[w * 128 + m]), c)) : "memory");
        sum += x;
      }
      const int64_t at = (int64_t)h * p.T + key;
      if (key < p.T) p.mass_out[at] = (p.mass_in ? p.mass_in[at] : 0.f) + sum;
    }
    tc::cluster_sync_all();
  }
  if (warp == 1) {
    __syncwarp();
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem_base, 512);
  }
}

template <typename T, int HD, bool FEW>
int32_t run_tc(const MassParams& p, cudaStream_t st) {
  static bool attr_set = false;
  if (!attr_set) {
    AKVS_CUDA(cudaFuncSetAttribute(mass_tc_kernel<T, HD, FEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, M_SMEM<HD, FEW>));
    attr_set = true;
  }
  // rows of a tile: 1 or 2 boxes whose rows fill whole groups of 8 (a swizzle atom), so that boxes lie back to back
  int box_rows = 128 / p.g, q_boxes = FEW ? 1 : 2;
  if (!FEW) {
    while (box_rows > 1 && box_rows * p.g % 8) --box_rows;
    if (box_rows * p.g % 8) { box_rows = 128 / p.g; q_boxes = 1; }
  }
  const int BR = box_rows * q_boxes;
  const int row_tiles = akvs_cdiv(p.R, BR), key_items = akvs_cdiv(p.T, 2 * BK);
  const int64_t n_items = (int64_t)key_items * p.n_kv;
  if (n_items > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  CUtensorMap tmK, tmQ;
  AKVS_TRY(make_tmap_2d_16bit(&tmK, p.k, p.T, (uint64_t)p.n_kv * HD, (uint64_t)p.k_ld, BK));
  // without rows there is no tile to load either; the map only has to be well formed
  AKVS_TRY(encode_tmap_3d_16bit(&tmQ, p.R > 0 ? p.q : p.k, HD, p.R > 0 ? p.n_q : p.n_kv, p.R > 0 ? p.R : p.T, HD,
                                p.R > 0 ? p.q_ld : p.k_ld, p.g, box_rows));
  int C = 1;
  while (C < 8 && n_items * C * 2 <= 148 && row_tiles >= C * 4) C *= 2;
  const int64_t grid = C > 1 ? n_items * C : (n_items < 148 ? n_items : 148);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(M_THREADS);
  cfg.dynamicSmemBytes = M_SMEM<HD, FEW>;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, mass_tc_kernel<T, HD, FEW>, tmK, tmQ, p, C, key_items, (int)n_items, BR, q_boxes,
                               std::is_same<T, f16>::value ? tc::kF16 : tc::kBF16));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

template <typename T, int HD>
int32_t run_tc(const MassParams& p, cudaStream_t st) {
  // up to 128 stacked rows: one tile of whole rows
  return (int64_t)akvs_cdiv(p.R, 128 / p.g) <= 1 ? run_tc<T, HD, true>(p, st) : run_tc<T, HD, false>(p, st);
}

// ---- CUDA cores: 64 keys per CTA, the stacked rows 64 at a time, 4 x 4 scores per thread.
constexpr int SK = 64, SR = 64, S_THREADS = 256;

template <typename T, int HD>
__device__ __forceinline__ void load_row_chunk(float* dst, const T* src, bool ok) {
  constexpr int V = VecOf<T>::N;
  float x[V];
  if (ok) {
    ld16(src, x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
}

template <typename T, int HD>
__global__ void __launch_bounds__(S_THREADS)
mass_simt_kernel(const __grid_constant__ MassParams p) {
  constexpr int LD = HD + 4, V = VecOf<T>::N, CH = HD / V;
  extern __shared__ __align__(16) float sm[];
  float* kt = sm;                    // [SK][LD]
  float* qt = kt + SK * LD;          // [SR][LD]
  __shared__ float row_lse[SR];
  __shared__ int row_lo[SR], row_hi[SR];
  __shared__ float part[16][SK];
  pdl_trigger();
  pdl_wait();
  const int h = blockIdx.y, j0 = blockIdx.x * SK, tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rows = p.R * p.g;
  for (int i = tid; i < SK * CH; i += S_THREADS) {
    const int j = i / CH, c = i % CH * V;
    load_row_chunk<T, HD>(kt + j * LD + c, (const T*)p.k + (int64_t)min(j0 + j, p.T - 1) * p.k_ld + (int64_t)h * HD + c, j0 + j < p.T);
  }
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int m0 = 0; m0 < rows; m0 += SR) {
    __syncthreads();
    bool any = false;
    if (tid < SR) {
      const int m = m0 + tid, r = min(m, rows - 1) / p.g;
      row_lse[tid] = m < rows ? p.lse[(int64_t)r * p.n_q + h * p.g + m % p.g] : 0.f;
      // a row that sees nothing has lse = -inf and adds nothing
      const bool on = m < rows && row_lse[tid] != -INFINITY;
      row_lo[tid] = on ? p.k_lo[r] : 0x7fffffff;
      row_hi[tid] = on ? p.k_hi[r] : -1;
      any = on && row_lo[tid] < j0 + SK && row_hi[tid] >= j0;
    }
    if (!__syncthreads_or(any)) continue;
    for (int i = tid; i < SR * CH; i += S_THREADS) {
      const int m = m0 + i / CH, c = i % CH * V, mm = min(m, rows - 1);
      load_row_chunk<T, HD>(qt + (i / CH) * LD + c,
                            (const T*)p.q + (int64_t)(mm / p.g) * p.q_ld + (int64_t)(h * p.g + mm % p.g) * HD + c, m < rows);
    }
    __syncthreads();
    float s[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) s[a][b] = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD; c += 4) {
      float4 x[4], y[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) x[a] = *reinterpret_cast<const float4*>(qt + (ty * 4 + a) * LD + c);
#pragma unroll
      for (int b = 0; b < 4; ++b) y[b] = *reinterpret_cast<const float4*>(kt + (tx + 16 * b) * LD + c);
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          s[a][b] = fmaf(x[a].x, y[b].x, fmaf(x[a].y, y[b].y, fmaf(x[a].z, y[b].z, fmaf(x[a].w, y[b].w, s[a][b]))));
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int m = ty * 4 + a, lo = row_lo[m], hi = row_hi[m];
      const float z = row_lse[m];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int j = j0 + tx + 16 * b;
        if (lo <= j && j <= hi) acc[b] += exp2f((s[a][b] * p.scale - z) * LOG2E);
      }
    }
  }
#pragma unroll
  for (int b = 0; b < 4; ++b) part[ty][tx + 16 * b] = acc[b];
  __syncthreads();
  if (tid < SK && j0 + tid < p.T) {
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < 16; ++y) s += part[y][tid];
    const int64_t at = (int64_t)h * p.T + j0 + tid;
    p.mass_out[at] = (p.mass_in ? p.mass_in[at] : 0.f) + s;
  }
}

template <typename T, int HD>
int32_t run_simt(const MassParams& p, cudaStream_t st) {
  constexpr int smem = (SK + SR) * (HD + 4) * 4;
  static bool attr_set = false;
  if (!attr_set) {
    AKVS_CUDA(cudaFuncSetAttribute(mass_simt_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    attr_set = true;
  }
  AKVS_CUDA(launch_pdl(mass_simt_kernel<T, HD>, dim3(akvs_cdiv(p.T, SK), p.n_kv), dim3(S_THREADS), smem, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

}  // namespace

extern "C" int32_t akvs_op_attention_mass(int32_t dtype, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                                          const float* lse, const int32_t* k_lo, const int32_t* k_hi, int32_t R,
                                          int32_t T, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                          const float* mass_in, float* mass_out, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (R < 0 || T < 0) return AKVS_ERR_INVALID_ARG;
  if (n_kv_heads <= 0 || n_q_heads <= 0 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 128 || n_kv_heads > 65535)
    return AKVS_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return AKVS_ERR_UNSUPPORTED;
  if (T == 0) return AKVS_OK;
  if (!mass_out || !k || (R > 0 && (!q || !lse || !k_lo || !k_hi))) return AKVS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)dtype_size(dtype), row = (int64_t)n_kv_heads * head_dim, q_row = (int64_t)n_q_heads * head_dim;
  if (k_ld < row || (R > 0 && q_ld < q_row)) return AKVS_ERR_SHAPE;
  if (!aligned16(k) || k_ld * es % 16 || (R > 0 && (!aligned16(q) || q_ld * es % 16))) return AKVS_ERR_INVALID_ARG;
  if ((int64_t)R * n_q_heads > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  const int64_t out_n = (int64_t)n_kv_heads * T * 4;
  const void* ins[5] = {R > 0 ? q : nullptr, k, lse, k_lo, k_hi};
  const int64_t in_n[5] = {R > 0 ? ((R - 1) * q_ld + q_row) * es : 0, ((T - 1) * k_ld + row) * es, (int64_t)R * n_q_heads * 4,
                           R * 4ll, R * 4ll};
  for (int i = 0; i < 5; ++i)
    if (bytes_overlap(ins[i], in_n[i], mass_out, out_n)) return AKVS_ERR_INVALID_ARG;
  if (mass_in && mass_in != mass_out && bytes_overlap(mass_in, out_n, mass_out, out_n)) return AKVS_ERR_INVALID_ARG;
  MassParams p;
  p.q = q; p.k = k; p.q_ld = q_ld; p.k_ld = k_ld; p.lse = lse; p.k_lo = k_lo; p.k_hi = k_hi;
  p.R = R; p.T = T; p.n_q = n_q_heads; p.n_kv = n_kv_heads; p.g = n_q_heads / n_kv_heads;
  p.mass_in = mass_in; p.mass_out = mass_out;
  p.scale = 1.f / sqrtf((float)head_dim);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using E = decltype(tag);
    if constexpr (std::is_same<E, float>::value)
      return head_dim == 64 ? run_simt<E, 64>(p, st) : run_simt<E, 128>(p, st);
    else
      return head_dim == 64 ? run_tc<E, 64>(p, st) : run_tc<E, 128>(p, st);
  });
}
