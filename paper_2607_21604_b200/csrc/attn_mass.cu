// Attention weight that every cached key has received: per kv head h and key j
//     mass_out[h][j] = mass_in[h][j] + sum over rows r that see j, heads i of the group of h:
//                      exp(q_ri . k_jh / sqrt(hd) - lse_ri)
// with lse the log-sum-exp of the row, as the attention that produced the row left it.
// The rows of the g = n_q / n_kv query heads of a kv head are stacked (r * g + i); every sum runs
// over them in a fixed order, so equal calls give equal bits.
//
// 16-bit types run on the tensor cores with the keys along M, so that a thread owns one key and its
// sum over the rows needs no shuffle; the score matrix never leaves tensor memory:
//     S^T = K Q^T     tcgen05.mma, two tiles of 128 keys against one tile of up to 128 stacked rows
//     sum            two warp groups, one per key tile: exp2 of a row of S^T, added up in registers
// A CTA keeps 256 keys in shared memory while the rows' Q tiles stream past them (each is used
// twice), then goes on to its next 256 keys.  The exponentials bound it: 16 per clock and SM, 2048
// clocks for a tile of 256 keys x 128 rows, against 1050 of the MMAs.  With few rows it is bound by
// reading K once.  Few keys and many rows: a cluster shares the row tiles of its keys and adds the
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
constexpr int BQ = 128;              // stacked rows of a tile at most
constexpr int MK_STAGES = 2, MQ_STAGES = 2, M_THREADS = 384;
constexpr int M_SLAB = 128 * 128;    // 128 rows of 64 values
template <int HD> constexpr int M_TILE = HD / 64 * M_SLAB;
// shared memory: K[2][2 tiles] | Q[2] | barriers (256 B) | per group: what a column sees, [2][128] | partial sums | flags
constexpr int M_COL_BYTES = 2 * 128 * 4 + 2 * 128 * 8;
template <int HD> constexpr int M_SMEM = (2 * MK_STAGES + MQ_STAGES) * M_TILE<HD> + 256 + 2 * M_COL_BYTES + 2 * 128 * 4 + 64;
enum { MB_KFULL = 0, MB_KEMPTY = MB_KFULL + MK_STAGES, MB_QFULL = MB_KEMPTY + MK_STAGES, MB_QEMPTY = MB_QFULL + MQ_STAGES,
       MB_SFULL = MB_QEMPTY + MQ_STAGES,      // [2 groups][2 buffers] S^T of a tile is complete
       MB_SEMPTY = MB_SFULL + 4,              // [2][2] the group has taken it into registers (4 warps)
       MB_COUNT = MB_SEMPTY + 4 };
static_assert(MB_COUNT * 8 + 8 <= 256, "barriers, the tensor-memory slot and the abort flag share 256 bytes");
static_assert(M_SMEM<128> <= 232448, "shared memory of one CTA");

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void group_sync(int grp) { asm volatile("bar.sync %0, 128;" ::"r"(grp + 1) : "memory"); }

template <typename T, int HD>
__global__ void __launch_bounds__(M_THREADS, 1)
mass_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ, const MassParams p,
               int C, int key_items, int n_items, int BR, uint32_t fmt) {
  constexpr int TILE = M_TILE<HD>;
  constexpr int OFF_Q = 2 * MK_STAGES * TILE, OFF_BAR = OFF_Q + MQ_STAGES * TILE, OFF_COL = OFF_BAR + 256;
  constexpr int OFF_PART = OFF_COL + 2 * M_COL_BYTES, OFF_FLAG = OFF_PART + 2 * 128 * 4;
  extern __shared__ __align__(1024) uint8_t smem[];
  if (tc::smem_u32(smem) & 1023u) return;           // swizzled tiles need 1024-byte alignment (the same in every CTA)
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + MB_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* part = reinterpret_cast<float*>(smem + OFF_PART);          // [2][128]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < MB_COUNT; ++i) tc::mbar_init(&bar[i], i >= MB_SEMPTY ? 4 : 1);
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  // Q tiles hold BR * g rows; where g does not divide 128 the last ones are never loaded and stay zero
  for (int i = threadIdx.x; i < MQ_STAGES * TILE / 16; i += M_THREADS)
    *reinterpret_cast<uint4*>(smem + OFF_Q + i * 16) = make_uint4(0u, 0u, 0u, 0u);
  tc::fence_proxy_async();
  pdl_wait();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const int rank = blockIdx.x % C, first = blockIdx.x / C, stride = gridDim.x / C;
  const int row_tiles = (p.R + BR - 1) / BR;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 0) {
      // ------------------------------------------------------------------ TMA producer
      if (lane == 0) {
        tc::prefetch_tmap(&tmK);
        tc::prefetch_tmap(&tmQ);
        const uint32_t q_bytes = (uint32_t)(BR * p.g) * 128u * (HD / 64);
        bool ok = true;
        int it = 0, n = 0;
        for (int item = first; item < n_items && ok; item += stride, ++it) {
          const int h = item / key_items, j0 = (item % key_items) * (2 * BK), ks = it % MK_STAGES;
          if (!tc::mbar_wait(&bar[MB_KEMPTY + ks], ((it / MK_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
          tc::mbar_expect_tx(&bar[MB_KFULL + ks], 2 * TILE);
#pragma unroll
          for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int c = 0; c < HD / 64; ++c)
              tc::tma_load_2d(smem + (2 * ks + w) * TILE + c * M_SLAB, &tmK, h * HD + c * 64, j0 + w * BK, &bar[MB_KFULL + ks]);
          for (int rt = rank; rt < row_tiles; rt += C, ++n) {
            const int qs = n % MQ_STAGES;
            if (!tc::mbar_wait(&bar[MB_QEMPTY + qs], ((n / MQ_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
            tc::mbar_expect_tx(&bar[MB_QFULL + qs], q_bytes);
#pragma unroll
            for (int c = 0; c < HD / 64; ++c)
              tc::tma_load_3d(smem + OFF_Q + qs * TILE + c * M_SLAB, &tmQ, c * 64, h * p.g, rt * BR, &bar[MB_QFULL + qs]);
          }
        }
        if (!ok) *abort_flag = 1;
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      if (lane == 0) {
        bool ok = true;
        int it = 0, n = 0;
        for (int item = first; item < n_items && ok; item += stride, ++it) {
          const int ks = it % MK_STAGES;
          if (!tc::mbar_wait(&bar[MB_KFULL + ks], (it / MK_STAGES) & 1, abort_flag)) { ok = false; break; }
          for (int rt = rank; rt < row_tiles && ok; rt += C, ++n) {
            const int qs = n % MQ_STAGES, b = n & 1;
            if (!tc::mbar_wait(&bar[MB_QFULL + qs], (n / MQ_STAGES) & 1, abort_flag)) { ok = false; break; }
            const int cols = min(BR, p.R - rt * BR) * p.g;
            const uint32_t idesc = tc::idesc_f16(fmt, BK, (cols + 15) / 16 * 16, 0);
            const uint32_t q_addr = tc::smem_u32(smem + OFF_Q + qs * TILE);
            for (int w = 0; w < 2; ++w) {
              if (!tc::mbar_wait(&bar[MB_SEMPTY + 2 * w + b], ((n >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
              tc::fence_after_sync();
              const uint32_t k_addr = tc::smem_u32(smem + (2 * ks + w) * TILE);
#pragma unroll
              for (int k = 0; k < HD / 16; ++k) {
                const uint32_t off = (k >> 2) * M_SLAB + (k & 3) * 32;
                tc::mma_f16(tmem_base + (2 * w + b) * BQ, tc::smem_desc_k_sw128(k_addr + off),
                            tc::smem_desc_k_sw128(q_addr + off), idesc, k != 0);
              }
              tc::mma_commit(&bar[MB_SFULL + 2 * w + b]);
            }
            if (ok) tc::mma_commit(&bar[MB_QEMPTY + qs]);
          }
          if (ok) tc::mma_commit(&bar[MB_KEMPTY + ks]);
        }
        if (!ok) *abort_flag = 1;
      }
    }
  } else {
    // ---------------------------------------------------------------------- a key per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int w = (warp >> 2) - 1, m = threadIdx.x & 127, quad = warp & 3;
    float* col_z = reinterpret_cast<float*>(smem + OFF_COL + w * M_COL_BYTES);        // [2][128] -lse in log2 units
    int2* col_rng = reinterpret_cast<int2*>(col_z + 2 * 128);                         // [2][128] visible keys
    volatile int* flag = reinterpret_cast<volatile int*>(smem + OFF_FLAG) + w * 8;    // [2][4] a column of the quad needs a mask
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
    const float scale2 = p.scale * LOG2E;
    bool ok = true;
    int n = 0;
    for (int item = first; item < n_items && ok; item += stride) {
      const int h = item / key_items, k0 = (item % key_items) * (2 * BK) + w * BK, key = k0 + m;
      const int k_last = min(k0 + BK, p.T) - 1;
      float acc[4] = {0.f, 0.f, 0.f, 0.f};
      for (int rt = rank; rt < row_tiles; rt += C, ++n) {
        const int b = n & 1;
        {
          // this thread describes column m of the tile
          const int r = rt * BR + m / p.g;
          const bool real = m < BR * p.g && r < p.R;
          float z = INFINITY;
          int lo = 0x7fffffff, hi = -1;
          if (real) {
            z = __ldg(p.lse + (int64_t)r * p.n_q + h * p.g + m % p.g);
            lo = __ldg(p.k_lo + r);
            hi = __ldg(p.k_hi + r);
            if (z == -INFINITY) { z = INFINITY; lo = 0x7fffffff; hi = -1; }    // a row that sees nothing adds nothing
          }
          // a column of zeros behind the last row needs no mask: exp2(0 - inf) = 0
          const bool masked = real && !(lo <= k0 && hi >= k_last);
          col_z[b * 128 + m] = -z * LOG2E;
          col_rng[b * 128 + m] = make_int2(lo, hi);
          const bool any = __any_sync(0xFFFFFFFFu, masked);
          if (lane == 0) flag[b * 4 + quad] = any;
        }
        group_sync(w);
        const bool mask = flag[b * 4] || flag[b * 4 + 1] || flag[b * 4 + 2] || flag[b * 4 + 3];
        const int cols = min(BR, p.R - rt * BR) * p.g;
        if (!tc::mbar_wait(&bar[MB_SFULL + 2 * w + b], (n >> 1) & 1, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
        float t[BQ];
        const uint32_t s_addr = lane_addr + (2 * w + b) * BQ;
#pragma unroll
        for (int c = 0; c < BQ / 32; ++c) tc::tmem_ld32(s_addr + c * 32, *reinterpret_cast<float(*)[32]>(&t[c * 32]));
        tc::tmem_ld_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bar[MB_SEMPTY + 2 * w + b]);
#pragma unroll
        for (int c = 0; c < BQ; c += 16) {
          if (c < cols) {                                 // S^T behind the last 16 columns was not written
#pragma unroll
            for (int i = c; i < c + 16; ++i) {
              float e = ex2(fmaf(t[i], scale2, col_z[b * 128 + i]));
              if (mask) {
                const int2 rng = col_rng[b * 128 + i];
                e = rng.x <= key && key <= rng.y ? e : 0.f;
              }
              acc[i & 3] += e;
            }
          }
        }
      }
      if (!ok) break;
      const float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
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
      const int w = (warp >> 2) - 1, m = threadIdx.x & 127, h = first / key_items, key = (first % key_items) * (2 * BK) + w * BK + m;
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

template <typename T, int HD>
int32_t run_tc(const MassParams& p, cudaStream_t st) {
  static bool attr_set = false;
  if (!attr_set) {
    AKVS_CUDA(cudaFuncSetAttribute(mass_tc_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, M_SMEM<HD>));
    attr_set = true;
  }
  const int BR = BQ / p.g;
  const int row_tiles = akvs_cdiv(p.R, BR), key_items = akvs_cdiv(p.T, 2 * BK);
  const int64_t n_items = (int64_t)key_items * p.n_kv;
  if (n_items > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  CUtensorMap tmK, tmQ;
  AKVS_TRY(make_tmap_2d_16bit(&tmK, p.k, p.T, (uint64_t)p.n_kv * HD, (uint64_t)p.k_ld, BK));
  // without rows there is no tile to load either; the map only has to be well formed
  AKVS_TRY(encode_tmap_3d_16bit(&tmQ, p.R > 0 ? p.q : p.k, HD, p.R > 0 ? p.n_q : p.n_kv, p.R > 0 ? p.R : p.T, HD,
                                p.R > 0 ? p.q_ld : p.k_ld, p.g, BR));
  int C = 1;
  while (C < 8 && n_items * C * 2 <= 148 && row_tiles >= C * 4) C *= 2;
  const int64_t grid = C > 1 ? n_items * C : (n_items < 148 ? n_items : 148);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(M_THREADS);
  cfg.dynamicSmemBytes = M_SMEM<HD>;
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
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, mass_tc_kernel<T, HD>, tmK, tmQ, p, C, key_items, (int)n_items, BR,
                               std::is_same<T, f16>::value ? tc::kF16 : tc::kBF16));
  AKVS_LAUNCHED();
  return AKVS_OK;
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
