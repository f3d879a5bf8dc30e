// Linear layers with 4-bit weights for the few rows of a decoding step: y = x W^T,
//     w_nk = c_nk scale_ng + min_ng,  g = k / 64;     y_n = sum_g scale_ng (c_ng . x_g) + min_ng sum(x_g).
// Memory bound by the weights (36 bytes per 64 of them) while the rows are few.  A code becomes an operand of a product by an AND
// and half a shift, as a float16 of few bits that is exact in the tensor cores (code_operands); x is scaled by the power of two
// that brings the largest value of a row and range of columns to [2^14, 2^15), where float16 loses nothing above 2^-39 of it (odd
// columns, which enter with a sixteenth: 2^-35).  A group's products are summed by themselves and scaled in float, so that weights
// are what their codes and records say and nothing is rounded but sums.  Float rows enter as three float16 pieces, which hold all 24
// bits of a value down to 2^-15 of the largest (odd columns: 2^-11); a piece's products are summed by themselves and added in float.
// Root mean square errors of float results are up to 0.2e-6 of y for 16-bit rows and 0.5e-6 for float rows (with codes as an AND
// leaves them, up to 1.4e-6 for float16 and float rows, and 0.5e-6 for bfloat16; 8 rows of 14336 x 4096 12.1 instead of 12.4 us).
//
// Weights are laid out once (akvs_op_linear_q4_pack): blocks of 16 features x 2 groups, 1152 bytes; those of 256 features
// side by side, and so on along the columns, so that every kernel reads long pieces.  A feature's 64 bytes of codes are
// four chunks of 16 bytes, chunk t the columns 16 t .. 16 t + 15 of either group, at place t ^ (feature / 2 % 4): a warp's
// fragment load is 512 contiguous bytes, and 8 threads that read a chunk of a feature each from shared memory meet 8
// different places.
//
// Three kernels, chosen by path_of: `few` (up to 8 rows), `clusters` (to 16 rows, float rows, and x too long for `few`), both
// on mma.sync m16n8k16 with 16 features along M and 8 rows along N; `tc` (more rows) on tcgen05.  All of them add in a fixed
// order: equal calls give equal bits.
//
// The first one below, `clusters`: a CTA has 8 warps of 16 features each, which share x, and a range of columns; the CTAs of a
// cluster share the features and add their sums over distributed shared memory, in the order of the ranges.  16 rows of
// 14336 x 4096 in 17.9 us (1.8 TB/s of weights), bound by the instructions that turn codes into operands and by its start.
#include <cooperative_groups.h>
#include "linear_rule.h"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int LQ_WARPS = 8, LQ_THREADS = LQ_WARPS * 32, LQ_F = LQ_WARPS * 16;        // features of a CTA
constexpr int XG = 8;                                 // groups of x staged at a time
constexpr int LQ_CODES = 1024, LQ_BLOCK = LQ_CODES + 128;      // bytes of 16 features x 128 columns, (scale, minimum) last

// Number of the block of 16 features `tile` and pair of groups `pair`.
__host__ __device__ __forceinline__ int64_t block_of(int tile, int pair, int tiles, int pairs) {
  const int set = tile >> 4, beside = tiles - set * 16 < 16 ? tiles - set * 16 : 16;
  return (int64_t)set * 16 * pairs + (int64_t)pair * beside + (tile & 15);
}

struct LinearQ4Params {
  const void* x;
  int64_t x_ld;
  const uint8_t* w;
  void* y;                                            // T [M][N], or
  const float* h;                                     // float [M][N]: h_out = h + x W^T
  float* h_out;
  int M, N, groups, pairs, groups_per_split;
  int team;                                           // warps that share a tile's columns
};

// A grid of clusters side by side along the features, and of blocks of rows over the two short dimensions.
dim3 row_grid(int64_t ctas, int blocks) { return dim3((unsigned)ctas, blocks < 65535 ? blocks : 65535, akvs_cdiv(blocks, 65535)); }
__device__ __forceinline__ int row_block() { return (int)(blockIdx.z * 65535u + blockIdx.y); }
__device__ __forceinline__ int cluster_number() {
  uint32_t x;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(x));
  return (int)x;
}
__device__ __forceinline__ int cluster_rank() {
  uint32_t x;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(x));
  return (int)x;
}

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bulk_copy(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(tc::smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void add4(float (&d)[4], const float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) d[e] += x[e];
}
// the same with nothing to add to
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Waits, as long as a wait may take, for a copy or products that nobody waited for, since another wait had run out:
// nothing may land in memory that is not this CTA's any more.
__device__ __noinline__ void drain(uint64_t* bar, uint32_t parity) {
  volatile int never = 0;
  tc::mbar_wait(bar, parity, &never);
}

// Shared memory of a CTA: two stages of weights ([pair][8 blocks], 8 groups), two of x.
template <int NT, int PIECES> struct LqSmem {
  static constexpr int PAIR = LQ_WARPS * LQ_BLOCK, W = XG / 2 * PAIR, X = XG * NT * PIECES * 1024;
  static constexpr int XM = NT * 2 * 32 * 4 * (PIECES > 1 ? 2 : 1), XP = NT * 8 * 4;     // sums of x as operands, powers of two of the rows
  static constexpr int XALL = X + XM + XP, BYTES = 2 * W + 2 * XALL;
  static constexpr int RED = (LQ_F + 4) * 4 * 8 * NT;                 // the sums, where the weights were
  static_assert(W % 128 == 0 && XALL % 16 == 0 && RED <= 2 * W, "");
};

// grid (features / 128 x splits, rows / (8 NT)), the splits one cluster
template <typename T, int NT>
__global__ void __launch_bounds__(LQ_THREADS, sizeof(T) == 4 ? 1 : 2)
linear_q4_kernel(const __grid_constant__ LinearQ4Params p) {
  constexpr int PIECES = sizeof(T) == 4 ? 3 : 1, ROWS = 8 * NT;
  using S = LqSmem<NT, PIECES>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[2];
  __shared__ volatile int gave_up;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  const int f_range = cluster_number(), row0 = row_block() * ROWS, f0 = f_range * LQ_F + warp * 16;
  if (row_block() > (p.M - 1) / ROWS) return;         // (a whole cluster)
  const int g0 = cluster_rank() * p.groups_per_split, g1 = min(g0 + p.groups_per_split, p.groups), chunks = (g1 - g0 + XG - 1) / XG;
  const bool mine = f0 < p.N;
  const int tiles = (p.N + 15) / 16, nt = min(LQ_WARPS, tiles - f_range * LQ_WARPS);   // blocks side by side here
  auto pairs = [&](int c) { return min(XG / 2, (g1 - g0 - c * XG + 1) / 2); };       // of a chunk
  auto source = [&](int c, int k) { return p.w + block_of(f_range * LQ_WARPS, g0 / 2 + c * (XG / 2) + k, tiles, p.pairs) * LQ_BLOCK; };
  pdl_trigger();
  // Weights on their way to L2 before this kernel may read anything: a hint, which what is written meanwhile outlives
  if (warp < 2 && lane < XG / 2 && warp < chunks && lane < pairs(warp))
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(source(warp, lane)), "r"(nt * LQ_BLOCK) : "memory");
  if (threadIdx.x == 0) {
    gave_up = 0;
    tc::mbar_init(&full[0], 1);
    tc::mbar_init(&full[1], 1);
    tc::fence_barrier_init();
  }
  __syncthreads();
  pdl_wait();
  auto fetch = [&](int c) {                           // thread 0: weights of chunk c
    tc::mbar_expect_tx(&full[c & 1], pairs(c) * nt * LQ_BLOCK);
    for (int k = 0; k < pairs(c); ++k) bulk_copy(smem + (c & 1) * S::W + k * S::PAIR, source(c, k), nt * LQ_BLOCK, &full[c & 1]);
  };
  if (threadIdx.x == 0)
    for (int c = 0; c < 2 && c < chunks; ++c) fetch(c);

  // x of a chunk: a warp per row, lane = 4 group + t.  Loads and conversion apart, so that products run in between.
  constexpr int V = VecOf<T>::N;
  uint4 raw[NT][16 / V];
  auto load_x = [&](int c) {
#pragma unroll
    for (int rr = 0; rr < NT; ++rr) {
      const int row = row0 + rr * 8 + warp, g = g0 + c * XG + (lane >> 2);
      const T* src = reinterpret_cast<const T*>(p.x) + (int64_t)row * p.x_ld + g * 64 + t * 16;
#pragma unroll
      for (int i = 0; i < 16 / V; ++i)
        raw[rr][i] = row < p.M && g < g1 ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  auto convert_x = [&](int c) {
    uint8_t* xb = smem + 2 * S::W + (c & 1) * S::XALL;
#pragma unroll
    for (int rr = 0; rr < NT; ++rr) {
      float f[16];
#pragma unroll
      for (int i = 0; i < 16 / V; ++i) {
        float y[V];
        if constexpr (sizeof(T) == 4) {
          y[0] = __uint_as_float(raw[rr][i].x); y[1] = __uint_as_float(raw[rr][i].y);
          y[2] = __uint_as_float(raw[rr][i].z); y[3] = __uint_as_float(raw[rr][i].w);
        } else {
          ld16(reinterpret_cast<const T*>(&raw[rr][i]), y);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) f[i * V + e] = y[e];
      }
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(f[e]));
      top = warp_max(top);
      int up = 141 - (int)(__float_as_uint(top) >> 23);               // brings the largest value to [2^14, 2^15)
      up = top == 0.f || !(top < INFINITY) ? 0 : min(up, 126);
      const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        f[e] *= mul;
        s += f[e];
      }
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
      if (lane == 0) *reinterpret_cast<float*>(xb + S::X + S::XM + (rr * 8 + warp) * 4) = __uint_as_float((uint32_t)(127 - up) << 23);
      // the group's sum, below 2^21, as two float16 of a sixty-fourth of it: k = 2 (g % 4), 2 (g % 4) + 1 of half g / 4.  Two hold
      // it to 2^-23 of itself, a float's last bit, or to 2^-33 of the largest value of the columns staged: enough beside 16-bit x; float
      // rows have a third.
      if (t == 0) {
        const float m = s * 0x1p-6f;
        const __half hi = __float2half_rn(m), lo = __float2half_rn(m - __half2float(hi));
        uint8_t* at = xb + S::X + ((rr * 2 + (lane >> 4)) * 32 + warp * 4 + ((lane >> 2) & 3)) * 4;
        *reinterpret_cast<__half2*>(at) = __halves2half2(hi, lo);
        if (PIECES > 1)
          *reinterpret_cast<__half2*>(at + NT * 256) =
              __halves2half2(__float2half_rn(m - __half2float(hi) - __half2float(lo)), __float2half_rn(0.f));
      }
#pragma unroll
      for (int wd = 0; wd < 2; ++wd) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = f[8 * wd + e] * (e & 1 ? CODE_ODD : 1.f);
#pragma unroll
        for (int pc = 0; pc < PIECES; ++pc) {
          uint32_t q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int lo = (i & 1) * 2 + (i >> 1);    // (0 4) (2 6) (1 5)/16 (3 7)/16
            const __half2 hh = __floats2half2_rn(y[lo], y[lo + 4]);
            q[i] = *reinterpret_cast<const uint32_t*>(&hh);
            const float2 back = __half22float2(hh);
            y[lo] -= back.x;
            y[lo + 4] -= back.y;
          }
          *reinterpret_cast<uint4*>(xb + (((((lane >> 2) * NT + rr) * PIECES + pc) * 2 + wd) * 32 + warp * 4 + t) * 16) =
              make_uint4(q[0], q[1], q[2], q[3]);
        }
      }
    }
  };

  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
  load_x(0);
  convert_x(0);
  __syncthreads();
  bool lost = false;
  for (int c = 0; c < chunks; ++c) {
    if (c + 1 < chunks) load_x(c + 1);
    if (!lost && !tc::mbar_wait(&full[c & 1], (c >> 1) & 1, &gave_up)) {
      lost = true;
      gave_up = 1;
      if (threadIdx.x == 0) {                         // what is on its way: this chunk and the next
        drain(&full[c & 1], (c >> 1) & 1);
        if (c + 1 < chunks) drain(&full[(c + 1) & 1], ((c + 1) >> 1) & 1);
      }
    }
    if (mine && !lost) {
      const uint8_t* wb = smem + (c & 1) * S::W + warp * LQ_BLOCK;
      const uint8_t* xb = smem + 2 * S::W + (c & 1) * S::XALL;
      const int gn = min(XG, g1 - g0 - c * XG);
      float sum[NT][4], low[NT][4];                   // of codes; of minima
      uint32_t am[4];                                 // minima of features gr, gr + 8: groups t and t + 4, twice each
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int g = t + 4 * (i >> 1);
        am[i] = 0u;
        if (g < gn)
          am[i] = __byte_perm(*reinterpret_cast<const uint32_t*>(wb + (g >> 1) * S::PAIR + LQ_CODES + (gr + 8 * (i & 1)) * 8 + (g & 1) * 4), 0u, 0x3232u);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[n][e] = low[n][e] = 0.f;
        const uint32_t* xm = reinterpret_cast<const uint32_t*>(xb + S::X) + n * 64 + lane;
        mma16816(low[n], am[0], am[1], am[2], am[3], xm[0], xm[32]);
        if (PIECES > 1) {
          float own[4] = {0.f, 0.f, 0.f, 0.f};
          mma16816(own, am[0], am[1], am[2], am[3], xm[NT * 64], xm[NT * 64 + 32]);
          add4(low[n], own);
        }
      }
#pragma unroll
      for (int g = 0; g < XG; ++g) {
        if (g >= gn) break;
        const uint8_t* blk = wb + (g >> 1) * S::PAIR;
        // (both groups of a block come with one load)
        const uint4 ca = reinterpret_cast<const uint4*>(blk)[gr * 4 + (t ^ ((gr >> 1) & 3))];
        const uint4 cb = reinterpret_cast<const uint4*>(blk)[32 + gr * 4 + (t ^ ((gr >> 1) & 3))];
        const uint32_t wa[2] = {g & 1 ? ca.z : ca.x, g & 1 ? ca.w : ca.y}, wb2[2] = {g & 1 ? cb.z : cb.x, g & 1 ? cb.w : cb.y};
        const float sa = __half2float(*reinterpret_cast<const __half*>(blk + LQ_CODES + gr * 8 + (g & 1) * 4));
        const float sb = __half2float(*reinterpret_cast<const __half*>(blk + LQ_CODES + (gr + 8) * 8 + (g & 1) * 4));
        float d[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
#pragma unroll
        for (int wd = 0; wd < 2; ++wd) {
          uint32_t a0[2], a1[2], b0[2], b1[2];
          code_operands(wa[wd], a0, a1);
          code_operands(wb2[wd], b0, b1);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) {
              const uint4 q = *reinterpret_cast<const uint4*>(xb + ((((g * NT + n) * PIECES + pc) * 2 + wd) * 32 + lane) * 16);
              float own[4] = {0.f, 0.f, 0.f, 0.f};
              float(&to)[4] = PIECES > 1 ? own : d[n];
              mma16816(to, a0[0], b0[0], a0[1], b0[1], q.x, q.y);
              mma16816(to, a1[0], b1[0], a1[1], b1[1], q.z, q.w);
              if (PIECES > 1) add4(d[n], own);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          sum[n][0] = fmaf(sa, d[n][0], sum[n][0]);
          sum[n][1] = fmaf(sa, d[n][1], sum[n][1]);
          sum[n][2] = fmaf(sb, d[n][2], sum[n][2]);
          sum[n][3] = fmaf(sb, d[n][3], sum[n][3]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 pw = *reinterpret_cast<const float2*>(xb + S::X + S::XM + (8 * n + 2 * t) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[n][e] = fmaf(fmaf(sum[n][e], CODE_BACK, low[n][e] * 0x1p6f), e & 1 ? pw.y : pw.x, acc[n][e]);
      }
    }
    if (c + 1 < chunks) convert_x(c + 1);
    __syncthreads();
    if (threadIdx.x == 0 && c + 2 < chunks && !lost) fetch(c + 2);
  }
  float* red = reinterpret_cast<float*>(smem);        // [ROWS][LQ_F + 4], where the weights were
  constexpr int LD = LQ_F + 4;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      red[(8 * n + 2 * t + (e & 1)) * LD + warp * 16 + gr + 8 * (e >> 1)] = lost ? NAN : acc[n][e];
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const int splits = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  // 128 features x ROWS sums, shared out over the cluster's CTAs
  for (int i = rank * LQ_THREADS + threadIdx.x; i < ROWS * LQ_F; i += splits * LQ_THREADS) {
    const int r = i / LQ_F, f = i % LQ_F, row = row0 + r, n = f_range * LQ_F + f;
    if (row >= p.M || n >= p.N) continue;
    float s = 0.f;
#pragma unroll 4
    for (int k = 0; k < splits; ++k) s += *cluster.map_shared_rank(red + r * LD + f, k);
    const int64_t at = (int64_t)row * p.N + n;
    if (p.h_out) p.h_out[at] = p.h[at] + s;
    else reinterpret_cast<T*>(p.y)[at] = from_f_inf<T>(s);
  }
  cluster.sync();                                     // nobody leaves while others read
}

// ---------------------------------------------------------------------------------------------------------------------
// Up to 8 rows, while x fits into shared memory beside the weights under way: one CTA per SM, whose 16 warps form teams of 4,
// 8 or 16.  A team walks FT feature tiles of 16 at a time, its warps share the columns.  x is brought into operand order once
// per CTA; a warp streams its columns through a ring of its own, a pair of groups a stage, so nothing but the sums of the
// tiles is exchanged, once per FT tiles, through shared memory.
// 8 rows of 14336 x 4096: 12.7 us, 2.6 TB/s of weights (a cluster per 128 features, with x converted anew for each: 13.8); of
// 55296 x 5120 40 us, 4.0 TB/s, and one row of it 30 us, 5.3 TB/s of 6.56 (teams of 16 alone: 56 and 37).  One row of 4096 x
// 4096: 4.5 us, 4.9 with weights from memory; clusters 6.2.  Bound by start, x (2.7 us for 8 rows of 4096) and end where weights
// are small, then by issue, some 220 instructions for a pair of groups of two tiles, and by memory for one row.
constexpr int FW_WARPS = 16, FW_THREADS = FW_WARPS * 32, FW_STAGES = 3;
constexpr int FW_MAX_SMEM = 224 * 1024;
__host__ __device__ constexpr int fw_ring(int FT) { return FW_WARPS * FW_STAGES * FT * LQ_BLOCK; }
__host__ __device__ constexpr int fw_ld(int FT) { return FT * 16 + 1; }
__host__ __device__ constexpr int fw_red(int FT) { return 2 * FW_WARPS * 8 * fw_ld(FT) * 4; }      // [2][warp][row][features]

// x in operand order: [group][piece][word][row][t] 16 bytes; sums float [group][8]; powers of two float [pair][8].
__host__ __device__ __forceinline__ int64_t few_x_bytes(int M, int pairs, int pieces) { return (int64_t)pairs * 2 * pieces * 2 * M * 64; }
__host__ __device__ __forceinline__ int64_t few_smem(int FT, int M, int pairs, int pieces) {
  return fw_ring(FT) + fw_red(FT) + few_x_bytes(M, pairs, pieces) + (int64_t)pairs * 3 * 8 * 4;
}

template <typename T, int FT>
__global__ void __launch_bounds__(FW_THREADS, 1)
linear_q4_few_kernel(const __grid_constant__ LinearQ4Params p) {
  constexpr int PIECES = sizeof(T) == 4 ? 3 : 1, V = VecOf<T>::N, STAGE = FT * LQ_BLOCK, LD = fw_ld(FT);
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3, M = p.M;
  float* red = reinterpret_cast<float*>(smem + fw_ring(FT));
  uint8_t* xf = smem + fw_ring(FT) + fw_red(FT);
  float* xsum = reinterpret_cast<float*>(xf + few_x_bytes(M, p.pairs, PIECES));
  float* xpow = xsum + p.pairs * 16;
  // This warp's pairs of groups in every tile of its team; its units are (FT tiles, pair), one after the other.
  const int tiles = (p.N + 15) / 16, sets = (tiles + FT - 1) / FT, per = (p.pairs + p.team - 1) / p.team;
  const int team = warp / p.team, q0 = min(warp % p.team * per, p.pairs), q1 = min(q0 + per, p.pairs);
  const int set0 = team * (int)gridDim.x + (int)blockIdx.x, set_step = FW_WARPS / p.team * (int)gridDim.x;
  const int mine = sets > set0 ? (sets - 1 - set0) / set_step + 1 : 0;
  uint8_t* ring = smem + warp * FW_STAGES * STAGE;
  // The next unit's weights, if there is one, into the next stage.  (FT divides the 16 blocks that lie side by side.)
  int next_set = q0 < q1 ? set0 : sets, next_q = q0, next_n = 0, next_step = 0;
  const uint8_t* next_src = p.w;
  const uint32_t ring0 = tc::smem_u32(ring) + lane * 16;
  uint32_t next_dst = ring0;
  auto seek = [&]() {                                 // the first block of next_set
    if (next_set >= sets) return;
    next_n = min(FT, tiles - next_set * FT) * 72;
    next_step = min(16, tiles - next_set * FT / 16 * 16) * LQ_BLOCK;
    next_src = p.w + block_of(next_set * FT, q0, tiles, p.pairs) * LQ_BLOCK + lane * 16;
  };
  auto fetch = [&]() {
    if (next_set < sets) {
#pragma unroll
      for (int i = 0; i < (FT * 72 + 31) / 32; ++i)
        if (i * 32 + lane < next_n)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(next_dst + i * 512), "l"(next_src + i * 512) : "memory");
      next_src += next_step;
      next_dst = next_dst == ring0 + (FW_STAGES - 1) * STAGE ? ring0 : next_dst + STAGE;
      if (++next_q == q1) {
        next_q = q0;
        next_set += set_step;
        seek();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  seek();
  pdl_trigger();
  // The first tiles on their way to L2 before this kernel may read anything: a hint, which what is written meanwhile outlives
  if (q0 + lane < q1 && lane < 8 && set0 < sets)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;"
                 ::"l"(p.w + block_of(set0 * FT, q0 + lane, tiles, p.pairs) * LQ_BLOCK), "r"(min(FT, tiles - set0 * FT) * LQ_BLOCK)
                 : "memory");
  pdl_wait();
#pragma unroll
  for (int i = 0; i < FW_STAGES; ++i) fetch();

  // x: a thread takes 16 columns of a row at a time, eight threads a pair of groups; loads of several ahead of their use
  constexpr int UN = sizeof(T) == 4 ? 2 : 4;
  const int per_row = p.pairs * 8, all = M * per_row;
  for (int i0 = threadIdx.x; (i0 & ~31) < all; i0 += UN * FW_THREADS) {
    uint4 raw[UN][16 / V];
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int i = i0 + k * FW_THREADS, r = i / per_row, u = i % per_row;
      const T* src = reinterpret_cast<const T*>(p.x) + (int64_t)r * p.x_ld + u * 16;
#pragma unroll
      for (int c = 0; c < 16 / V; ++c)
        raw[k][c] = i < all && u < p.groups * 4 ? __ldg(reinterpret_cast<const uint4*>(src) + c) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int i = i0 + k * FW_THREADS, r = i / per_row, u = i % per_row, g = u >> 2, tt = u & 3;
      if ((i & ~31) >= all) break;                    // (eight threads alike: per_row % 8 == 0)
      float f[16], s = 0.f, top = 0.f;
#pragma unroll
      for (int c = 0; c < 16 / V; ++c) {
        float y[V];
        if constexpr (sizeof(T) == 4) {
          y[0] = __uint_as_float(raw[k][c].x); y[1] = __uint_as_float(raw[k][c].y);
          y[2] = __uint_as_float(raw[k][c].z); y[3] = __uint_as_float(raw[k][c].w);
        } else {
          ld16(reinterpret_cast<const T*>(&raw[k][c]), y);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          f[c * V + e] = y[e];
          s += y[e];
          top = fmaxf(top, fabsf(y[e]));
        }
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (o < 4) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      }
      int up = 141 - (int)(__float_as_uint(top) >> 23);               // brings the largest value to [2^14, 2^15)
      up = top == 0.f || !(top < INFINITY) ? 0 : min(up, 126);
      const float even = __uint_as_float((uint32_t)(up + 127) << 23), odd = even * CODE_ODD;
      if (i >= all) continue;
      if (tt == 0) xsum[g * 8 + r] = s;
      // 2^21 for the codes beside it.  (x beyond 2^120 leaves the floats here, and the row becomes infinities or NaN.)
      if ((u & 7) == 0) xpow[(u >> 3) * 8 + r] = __uint_as_float((uint32_t)(127 - up) << 23) * CODE_BACK;
#pragma unroll
      for (int wd = 0; wd < 2; ++wd) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = f[8 * wd + e] * (e & 1 ? odd : even);
#pragma unroll
        for (int pc = 0; pc < PIECES; ++pc) {
          uint32_t q[4];
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) {
            const int lo = (k4 & 1) * 2 + (k4 >> 1);  // (0 4) (2 6) (1 5)/16 (3 7)/16
            const __half2 hh = __floats2half2_rn(y[lo], y[lo + 4]);
            q[k4] = *reinterpret_cast<const uint32_t*>(&hh);
            if (pc + 1 < PIECES) {
              const float2 back = __half22float2(hh);
              y[lo] -= back.x;
              y[lo + 4] -= back.y;
            }
          }
          *reinterpret_cast<uint4*>(xf + ((((g * PIECES + pc) * 2 + wd) * M + r) * 4 + tt) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
        }
      }
    }
  }
  for (int i = threadIdx.x; i < p.pairs * 24; i += FW_THREADS)        // rows that do not exist
    if ((i & 7) >= M) xsum[i] = 0.f;
  __syncthreads();

  int stage = 0, buf = 0;
  const uint8_t* xl = xf + (gr * 4 + t) * 16;         // this lane's operands of x: M * 64 bytes from one word to the next
  const uint8_t* codes = ring + (gr * 4 + (t ^ ((gr >> 1) & 3))) * 16;
  const uint8_t* records = ring + LQ_CODES + gr * 8;
  const bool row = gr < M;
  const int word = M * 64;
  for (int m = 0; m < mine; ++m, buf ^= 1) {
    const int set = set0 + m * set_step;
    float acc[FT][4];                                 // features gr, gr + 8 of rows 2 t, 2 t + 1
#pragma unroll
    for (int f = 0; f < FT; ++f) acc[f][0] = acc[f][1] = acc[f][2] = acc[f][3] = 0.f;
    const uint8_t* xq = xl + (int64_t)q0 * 4 * PIECES * word;
    const float* sq = xsum + q0 * 16 + 2 * t;
    const float* pq = xpow + q0 * 8 + 2 * t;
    for (int q = q0; q < q1; ++q, xq += 4 * PIECES * word, sq += 16, pq += 8) {
      uint4 x[2][PIECES][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int pc = 0; pc < PIECES; ++pc)
#pragma unroll
          for (int wd = 0; wd < 2; ++wd) {
            x[h][pc][wd] = make_uint4(0u, 0u, 0u, 0u);
            if (row) x[h][pc][wd] = *reinterpret_cast<const uint4*>(xq + ((h * PIECES + pc) * 2 + wd) * word);
          }
      const float2 xs[2] = {*reinterpret_cast<const float2*>(sq), *reinterpret_cast<const float2*>(sq + 8)};
      const float2 pw = *reinterpret_cast<const float2*>(pq);
      asm volatile("cp.async.wait_group %0;" ::"n"(FW_STAGES - 1) : "memory");
      __syncwarp();                                   // every lane's copies are there
      const int at = stage * STAGE;
      if (++stage == FW_STAGES) stage = 0;
      float d[FT][2][4];
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const uint4 ca = *reinterpret_cast<const uint4*>(codes + at + f * LQ_BLOCK), cb = *reinterpret_cast<const uint4*>(codes + at + f * LQ_BLOCK + 512);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int wd = 0; wd < 2; ++wd) {
            uint32_t a0[2], a1[2], b0[2], b1[2];
            code_operands(h ? (wd ? ca.w : ca.z) : (wd ? ca.y : ca.x), a0, a1);
            code_operands(h ? (wd ? cb.w : cb.z) : (wd ? cb.y : cb.x), b0, b1);
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) {
              const uint4 v = x[h][pc][wd];
              const bool first = wd == 0 && pc == 0;
              float own[4];
              float(&to)[4] = PIECES > 1 && !first ? own : d[f][h];
              if (first || PIECES > 1) mma16816_first(to, a0[0], b0[0], a0[1], b0[1], v.x, v.y);
              else mma16816(to, a0[0], b0[0], a0[1], b0[1], v.x, v.y);
              mma16816(to, a1[0], b1[0], a1[1], b1[1], v.z, v.w);
              if (PIECES > 1 && !first) add4(d[f][h], own);
            }
          }
        }
      }
      uint2 ra[FT], rb[FT];
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        ra[f] = *reinterpret_cast<const uint2*>(records + at + f * LQ_BLOCK);
        rb[f] = *reinterpret_cast<const uint2*>(records + at + f * LQ_BLOCK + 64);
      }
      __syncwarp();                                   // the stage is read
      fetch();
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const float2 a0 = __half22float2(*reinterpret_cast<const __half2*>(&ra[f].x)), a1 = __half22float2(*reinterpret_cast<const __half2*>(&ra[f].y));
        const float2 b0 = __half22float2(*reinterpret_cast<const __half2*>(&rb[f].x)), b1 = __half22float2(*reinterpret_cast<const __half2*>(&rb[f].y));
        const float* d0 = d[f][0];
        const float* d1 = d[f][1];
        acc[f][0] = fmaf(fmaf(a1.x, d1[0], a0.x * d0[0]), pw.x, fmaf(a0.y, xs[0].x, fmaf(a1.y, xs[1].x, acc[f][0])));
        acc[f][1] = fmaf(fmaf(a1.x, d1[1], a0.x * d0[1]), pw.y, fmaf(a0.y, xs[0].y, fmaf(a1.y, xs[1].y, acc[f][1])));
        acc[f][2] = fmaf(fmaf(b1.x, d1[2], b0.x * d0[2]), pw.x, fmaf(b0.y, xs[0].x, fmaf(b1.y, xs[1].x, acc[f][2])));
        acc[f][3] = fmaf(fmaf(b1.x, d1[3], b0.x * d0[3]), pw.y, fmaf(b0.y, xs[0].y, fmaf(b1.y, xs[1].y, acc[f][3])));
      }
    }
    float* mr = red + (buf * FW_WARPS + warp) * 8 * LD;
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e) mr[(2 * t + (e & 1)) * LD + f * 16 + gr + 8 * (e >> 1)] = acc[f][e];
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(p.team * 32) : "memory");
    // Four threads a sum, in a fixed order
    for (int i = threadIdx.x % (p.team * 32); i < 4 * M * FT * 16; i += p.team * 32) {
      const int o = i >> 2, part = i & 3, f = o % (FT * 16), r = o / (FT * 16), n = set * FT * 16 + f;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < FW_WARPS / 4; ++w)
        if (w < p.team / 4) s += red[((buf * FW_WARPS + team * p.team + part * (p.team / 4) + w) * 8 + r) * LD + f];
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
      if (part != 0 || n >= p.N) continue;
      const int64_t at = (int64_t)r * p.N + n;
      if (p.h_out) p.h_out[at] = p.h[at] + s;
      else reinterpret_cast<T*>(p.y)[at] = from_f_inf<T>(s);
    }
  }
}

// A warp per block.
__global__ void __launch_bounds__(LQ_THREADS)
linear_q4_pack_kernel(const uint8_t* codes, const uint32_t* recs, int N, int groups, int pairs, uint8_t* out) {
  const int64_t unit = (int64_t)blockIdx.x * LQ_WARPS + (threadIdx.x >> 5);
  const int tiles = (N + 15) / 16;
  if (unit >= (int64_t)tiles * pairs) return;
  const int tile = (int)(unit / pairs);
  const int g0 = (int)(unit % pairs) * 2, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  uint8_t* b = out + block_of(tile, g0 / 2, tiles, pairs) * LQ_BLOCK;
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int64_t n = (int64_t)tile * 16 + gr + 8 * hf;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int g = 0; g < 2; ++g)
      if (n < N && g0 + g < groups) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(codes + (n * groups + g0 + g) * 32 + t * 8);
        w[2 * g] = src[0];
        w[2 * g + 1] = src[1];
      }
    reinterpret_cast<uint4*>(b)[hf * 32 + gr * 4 + (t ^ ((gr >> 1) & 3))] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  const int64_t n = (int64_t)tile * 16 + lane / 2;
  const int g = g0 + (lane & 1);
  reinterpret_cast<uint32_t*>(b + LQ_CODES)[lane] = n < N && g < groups ? recs[n * groups + g] : 0u;
}

template <typename T, int NT>
int32_t launch(const LinearQ4Params& p0, cudaStream_t st) {
  LinearQ4Params p = p0;
  const int tiles = akvs_cdiv(p.N, LQ_F), blocks = akvs_cdiv(p.M, 8 * NT);
  using S = LqSmem<NT, sizeof(T) == 4 ? 3 : 1>;
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)linear_q4_kernel<T, NT>, S::BYTES, smem_set));
  static_assert(XG == 8, "ranges of 512 columns");
  int splits = lq_cluster_ranges((int64_t)tiles * blocks, p.groups, sizeof(T) == 4 ? LQ_FIT_ONE : LQ_FIT_TWO);
  p.groups_per_split = akvs_cdiv(akvs_cdiv(p.groups, splits), XG) * XG;
  splits = akvs_cdiv(p.groups, p.groups_per_split);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = row_grid((int64_t)tiles * splits, blocks);
  cfg.blockDim = dim3(LQ_THREADS);
  cfg.dynamicSmemBytes = S::BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, linear_q4_kernel<T, NT>, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

// ---------------------------------------------------------------------------------------------------------------------
// More rows of a 16-bit type: the same sums on tcgen05.  256 features a CTA (two products of 128) by NB
// rows, a group of 64 columns a step:
//     D[feature][row] = codes[feature][64] x[row][64]        A in tensor memory, B in shared memory, D in tensor memory
//     acc[feature][row] += scale[feature] D                  a thread per feature, NB sums in registers
// Warps of their own turn codes into operands (code_operands, stored to tensor memory, four steps ahead), issue products and
// add them up.  The minima are a product too: 32 groups' minima
// (float16, as they are) against 32 sums of x, each as two float16, make a step of the same form, two steps a stage.
// x is brought into operand order once per call by a kernel of its own (scale of a row, permuted columns, the 128-byte
// swizzle); weights and x arrive by bulk copies, five or six pairs of groups ahead.
// 64 rows of 5120 x 27648 take 37.2 us, 2.2 TB/s of weights, 490 TFLOP/s; of 28672 x 4096 30.5 us; 17 rows take 0.9 of that.  Bound by
// what happens in a step (some 700 clocks, of which the products take 260): codes to tensor memory and sums out of it, 16 warps'
// instructions, waits; by 10 us of start and end, of which x takes 3 and the cluster's sum 3; and by the SMs that clusters of
// one size leave idle (28 of 148 here).
constexpr int TC_F = 256, TC_THREADS = 608;

struct TcParams {
  const uint8_t* w;
  const uint8_t* xt;                                  // [row block][step][NB][64] float16
  const float* pow;                                   // [range][row block][NB]
  void* y;
  const float* h;
  float* h_out;
  int M, N, tiles16, pairs, pairs_per_split, rows_per_block, steps, blocks;
  bool fours;                                         // four results in a row lie together
};

template <int NB> struct TcStage {
  static constexpr int X = NB * 128, BYTES = 2 * X + 16 * LQ_BLOCK, COUNT = NB == 64 ? 5 : 6;
  static constexpr int SMEM = COUNT * BYTES + 1024;
  static_assert(BYTES % 1024 == 0 && NB * (TC_F + 4) * 4 <= COUNT * BYTES, "");
};

// Steps of minima: 32 groups each, two at a time.
__host__ __device__ __forceinline__ int lq_min_steps(int groups) { return (groups + 63) / 64 * 2; }

// grid (rows of all blocks, ranges of columns): a range has its own power of two, since its CTA sums by itself.
constexpr int ROWS_THREADS = 256;
template <typename T, int NB>
__global__ void __launch_bounds__(ROWS_THREADS)
linear_q4_rows_kernel(const T* x, int64_t x_ld, int M, int rows_per_block, int groups, int pairs, int pairs_per_split, uint8_t* xt,
                      float* pow) {
  constexpr int KEEP = 4;
  __shared__ float tops[ROWS_THREADS / 32];
  pdl_wait();
  pdl_trigger();                                      // after the wait: the products' kernel reads weights without its own
  const int block = blockIdx.x / NB, n = blockIdx.x % NB, row = block * rows_per_block + n, lane = threadIdx.x & 31;
  const bool ok = n < rows_per_block && row < M;
  const int steps = 2 * pairs + lq_min_steps(groups), p0 = blockIdx.y * pairs_per_split, p1 = min(p0 + pairs_per_split, pairs);
  const int v0 = 16 * p0, v1 = 16 * p1;               // vectors of eight columns, a padded group included
  const T* src = x + (int64_t)(ok ? row : 0) * x_ld;
  uint4 kept[KEEP];
  float top = 0.f;
  auto fetch = [&](int v) {
    return ok && v < v1 && v < groups * 8 ? __ldg(reinterpret_cast<const uint4*>(src) + v) : make_uint4(0u, 0u, 0u, 0u);
  };
  auto peak = [&](const uint4& w) {
    float f[8];
    ld16(reinterpret_cast<const T*>(&w), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i) kept[i] = fetch(v0 + threadIdx.x + i * ROWS_THREADS);
#pragma unroll
  for (int i = 0; i < KEEP; ++i) peak(kept[i]);
  for (int v = v0 + threadIdx.x + KEEP * ROWS_THREADS; v < v1; v += ROWS_THREADS) peak(fetch(v));
  top = warp_max(top);
  if (lane == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  top = warp_max(tops[lane & (ROWS_THREADS / 32 - 1)]);
  int up = 141 - (int)(__float_as_uint(top) >> 23);   // brings the largest value to [2^14, 2^15)
  up = top == 0.f || !(top < INFINITY) ? 0 : min(up, 126);
  const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
  if (threadIdx.x == 0) pow[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = __uint_as_float((uint32_t)(127 - up) << 23);
  uint8_t* out = xt + (int64_t)block * steps * (NB * 128) + n * 128;
  auto put = [&](int v, const uint4& w) {             // (a warp's 32 vectors, of which the first 16 or all exist)
    float f[8], s = 0.f;
    ld16(reinterpret_cast<const T*>(&w), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] *= mul;
      s += f[e];
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    const int g = v >> 3, c = v & 7;
    if (v >= v1) return;
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int lo = (i & 1) * 2 + (i >> 1);          // (0 4) (2 6) (1 5)/16 (3 7)/16
      const float k = i < 2 ? 1.f : CODE_ODD;
      const __half2 hh = __floats2half2_rn(f[lo] * k, f[lo + 4] * k);
      q[i] = *reinterpret_cast<const uint32_t*>(&hh);
    }
    *reinterpret_cast<uint4*>(out + (int64_t)g * (NB * 128) + ((c ^ (n & 7)) << 4)) = make_uint4(q[0], q[1], q[2], q[3]);
    if (c == 0 && g < groups) {
      const float m = s * 0x1p-6f;                    // below 2^15
      const __half hi = __float2half_rn(m), lo = __float2half_rn(m - __half2float(hi));
      const int i = g & 31;
      *reinterpret_cast<__half2*>(out + (int64_t)(2 * pairs + (g >> 5)) * (NB * 128) + (((i >> 2) ^ (n & 7)) << 4) + (i & 3) * 4) =
          __halves2half2(hi, lo);
    }
  };
#pragma unroll
  for (int i = 0; i < KEEP; ++i)
    if (v0 + (int)(threadIdx.x & ~31) + i * ROWS_THREADS < v1) put(v0 + threadIdx.x + i * ROWS_THREADS, kept[i]);
  for (int v = v0 + threadIdx.x + KEEP * ROWS_THREADS; v0 + ((v - v0) & ~31) < v1; v += ROWS_THREADS) put(v, fetch(v));
  if (p1 == pairs)
    for (int g = groups + threadIdx.x; g < lq_min_steps(groups) * 32; g += ROWS_THREADS) {       // no groups: zeros
      const int i = g & 31;
      *reinterpret_cast<uint32_t*>(out + (int64_t)(2 * pairs + (g >> 5)) * (NB * 128) + (((i >> 2) ^ (n & 7)) << 4) + (i & 3) * 4) = 0u;
    }
}

// Waits of the warps below, on shared-memory addresses: one try, and only then the long way, suspended, where polling would
// take issue slots from the warps that work.  Bounded like mbar_wait; a wait that ran out sets the flag, which ends all
// others, and the results become NaN.
__device__ __noinline__ void wait_on(uint32_t bar, uint32_t parity, volatile int* gave_up) {
  const long long t0 = clock64();
  for (;;) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
    if (ok || *gave_up) return;
    if (clock64() - t0 > tc::kWaitCycles) *gave_up = 1;
  }
}
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}\n"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  if (!ok) wait_on(bar, parity, gave_up);
}
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// 16 columns of this thread's lane in tensor memory
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
                 "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
               : "r"(taddr) : "memory");
}

// grid (features / 256 x splits, row blocks), the splits one cluster.  Warps 0 - 7: codes to operands, a thread per
// feature; 8 - 15: sums, a thread per feature; 16, 17: products of either tile; 18: copies.
// A thread that issues products waits at one barrier a step (84 cycles even when it is open) and signals one: operands are
// there and the place for the products is free; the warps that read the sums give back operands and x as well.  With codes and
// sums in the same warps, one after the other, a step took 1180 cycles, with a barrier for each of these things 1100.
template <typename T, int NB>
__global__ void __launch_bounds__(TC_THREADS, 1)
linear_q4_tc_kernel(const __grid_constant__ TcParams p) {
  using S = TcStage<NB>;
  constexpr int ST = S::COUNT, NA = 4, ND = 128 / NB;   // operands and products in flight
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[ST], empty[ST], ready[2][NA], summed[2][NA], d_full[2][ND], done[2];
  __shared__ float scales[2][NA][128];
  __shared__ uint32_t minima[32][256];
  __shared__ uint32_t tmem_base;
  __shared__ volatile int gave_up;
  uint8_t* ring = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // The order of stages, for all roles: two steps of codes for every pair of groups, and after the last pair of 64 groups, or
  // of this range, two steps of their minima.  Stage i uses slots 2 (i % 2) and the next one of operands.
  const int f_range = cluster_number(), block = row_block();
  if (block >= p.blocks) return;                      // (a whole cluster)
  const int p0 = cluster_rank() * p.pairs_per_split, p1 = min(p0 + p.pairs_per_split, p.pairs);
  auto ends = [&](int pr) { return (pr & 31) == 31 || pr + 1 == p1; };
  const int n_stages = p1 - p0 + (p1 + 31) / 32 - p0 / 32;
  if (threadIdx.x == 0) {
    gave_up = 0;
    for (int i = 0; i < ST; ++i) {
      tc::mbar_init(&full[i], 1);
      tc::mbar_init(&empty[i], 16);                   // 8 warps have the codes, 8 the sums of both steps
    }
    for (int j = 0; j < 2; ++j) {
      for (int i = 0; i < NA; ++i) {
        tc::mbar_init(&ready[j][i], 8);               // 4 warps wrote operands, 4 read the products ND steps before
        tc::mbar_init(&summed[j][i], 4);
      }
      for (int i = 0; i < ND; ++i) tc::mbar_init(&d_full[j][i], 1);
      tc::mbar_init(&done[j], 1);
    }
    tc::fence_barrier_init();
  }
  if (warp == 16) {
    tc::tmem_alloc(&tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tmem_base;
  auto d_col = [&](int tile, int b) { return tmem + (uint32_t)((tile * ND + b) * NB); };
  auto a_col = [&](int tile, int b) { return tmem + 256u + (uint32_t)((tile * NA + b) * 32); };
  const uint8_t* xt = p.xt + (int64_t)block * p.steps * S::X;
  const uint32_t full0 = tc::smem_u32(full), empty0 = tc::smem_u32(empty);
  float2 acc[NB / 2];

  if (warp == 18) {
    // ---- copies: a stage of codes is the blocks of 256 features, one piece, and two steps of x
    if (tc::elect_one()) {
      const uint8_t* w0 = p.w + block_of(f_range * 16, 0, p.tiles16, p.pairs) * LQ_BLOCK;
      const int bytes = min(16, p.tiles16 - f_range * 16) * LQ_BLOCK;
      auto weights = [&](int st, int pr, bool minima) {
        tc::mbar_expect_tx(&full[st], 2 * S::X + (minima ? 0 : bytes));
        if (!minima) bulk_copy(ring + st * S::BYTES + 2 * S::X, w0 + (int64_t)pr * bytes, bytes, &full[st]);
      };
      auto columns = [&](int st, int pr, bool minima) {
        bulk_copy(ring + st * S::BYTES, xt + (int64_t)(minima ? 2 * p.pairs + pr / 32 * 2 : 2 * pr) * S::X, 2 * S::X, &full[st]);
      };
      struct Place { int pr; bool minima; };
      auto next = [&](Place& c) {
        if (!c.minima && ends(c.pr)) { c.minima = true; return; }
        c.minima = false;
        ++c.pr;
      };
      // weights of the first stages before x is in operand order
      Place c = {p0, false}, x = c;
      const int first = min(ST, n_stages);
      for (int i = 0; i < first; ++i, next(c)) weights(i, c.pr, c.minima);
      pdl_wait();
      for (int i = 0; i < first; ++i, next(x)) columns(i, x.pr, x.minima);
      int st = 0;
      uint32_t sp = 0;
      int issued = first;
      for (; issued < n_stages; ++issued, next(c)) {
        wait(empty0 + st * 8, sp, &gave_up);
        if (gave_up) break;
        weights(st, c.pr, c.minima);
        columns(st, c.pr, c.minima);
        if (++st == ST) { st = 0; sp ^= 1; }
      }
      // nothing is left in flight, whoever gave up: the last copies have arrived
      for (int i = issued - first; i < issued; ++i) drain(&full[i % ST], (i / ST) & 1);
    }
    __syncwarp();
  } else if (warp >= 16) {
    // ---- products of tile j.  x has arrived where the codes have.
    const int j = warp - 16;
    if (tc::elect_one()) {
      constexpr uint32_t idesc = tc::idesc_f16(tc::kF16, 128, NB, 0);
      const uint64_t desc0 = tc::smem_desc_k_sw128(tc::smem_u32(ring));
      const uint32_t ready0 = tc::smem_u32(ready[j]);
      uint64_t desc = desc0;
      int st = 0;
      for (int i = 0; i < n_stages; ++i) {
        const uint32_t par = i & 1, ph = (i >> 1) & 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          wait(ready0 + par * 16 + h * 8, ph, &gave_up);
          tc::fence_after_sync();
          const uint32_t dc = d_col(j, h) + (ND == 4 ? par * 2 * NB : 0), ac = a_col(j, h) + par * 64;
          const uint64_t bd = desc + h * (S::X >> 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) tc::mma_f16_ts(dc, ac + 8 * e, bd + 2 * e, idesc, e > 0);
          tc::mma_commit(&d_full[j][(ND == 4 ? par * 2 : 0) + h]);
        }
        desc += S::BYTES >> 4;
        if (++st == ST) { st = 0; desc = desc0; }
      }
      tc::mma_commit(&done[j]);
      drain(&done[j], 0);                             // tensor memory is given back below
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ---- sums, a thread per feature
    const int j = (warp >> 2) & 1, f = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ready0 = tc::smem_u32(ready[j]), summed0 = tc::smem_u32(summed[j]);
    const uint32_t d_full0 = tc::smem_u32(d_full[j]);
#pragma unroll
    for (int n = 0; n < NB / 2; ++n) acc[n] = make_float2(0.f, 0.f);
    if (lane < ND) arrive(ready0 + lane * 8);         // the places for the first products are free
    int st = 0;
    for (int i = 0; i < n_stages; ++i) {
      const uint32_t par = i & 1, ph = (i >> 1) & 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t d = (ND == 4 ? par * 2 : 0) + h, slot = par * 2 + h;
        wait(d_full0 + d * 8, ND == 4 ? ph : par, &gave_up);
        tc::fence_after_sync();
        const float scale = scales[j][slot][f];
        const float2 s2 = make_float2(scale, scale);
        const uint32_t at = d_col(j, 0) + lanes + d * NB;
#pragma unroll
        for (int c = 0; c < NB / 16; ++c) {
          float v[16];
          tmem_ld16(at + 16 * c, v);
          tc::tmem_ld_wait();
#pragma unroll
          for (int n = 0; n < 8; ++n) acc[c * 8 + n] = __ffma2_rn(make_float2(v[2 * n], v[2 * n + 1]), s2, acc[c * 8 + n]);
        }
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (ND == 4 ? i + 2 < n_stages : i + 1 < n_stages) arrive(ready0 + (ND == 4 ? slot : slot ^ 2u) * 8);
          arrive(summed0 + slot * 8);
          if (h == 1) arrive(empty0 + st * 8);
        }
      }
      if (++st == ST) st = 0;
    }
  } else {
    // ---- codes to operands, a thread per feature; the next stage's codes are read while this one's are turned
    const int j = warp >> 2, f = (warp & 3) * 32 + lane, fr = f & 15;  // feature f of tile j, its row in its block
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ready0 = tc::smem_u32(ready[j]), summed0 = tc::smem_u32(summed[j]);
    const uint8_t* blk = ring + 2 * S::X + (j * 8 + (f >> 4)) * LQ_BLOCK;
    const uint8_t* chunk[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) chunk[t] = blk + (fr * 4 + (t ^ ((fr >> 1) & 3))) * 16;
    const uint8_t* record = blk + LQ_CODES + fr * 8;
    int st = 0, i = 0;
    uint32_t sp = 0;
    struct Codes { uint4 c[4]; uint2 r; };
    auto read = [&](Codes& k) {
      wait(full0 + st * 8, sp, &gave_up);
      const uint32_t at = st * S::BYTES;
#pragma unroll
      for (int t = 0; t < 4; ++t) k.c[t] = *reinterpret_cast<const uint4*>(chunk[t] + at);
      k.r = *reinterpret_cast<const uint2*>(record + at);
    };
    auto release = [&]() {
      __syncwarp();
      if (lane == 0) arrive(empty0 + st * 8);
      if (++st == ST) { st = 0; sp ^= 1; }
    };
    auto put = [&](const uint32_t (&a)[32], float scale, int h) {
      const uint32_t slot = (i & 1) * 2 + h;
      // what this slot held two stages ago is done with
      if (i > 1) wait(summed0 + slot * 8, ((i >> 1) + 1) & 1, &gave_up);
      tc::fence_after_sync();
      scales[j][slot][f] = scale;
      tc::tmem_st32(a_col(j, 0) + slot * 32 + lanes, a);
      tc::tmem_st_wait();
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) arrive(ready0 + slot * 8);
    };
    auto turn = [&](const Codes& k, int h) {
      uint32_t a[32];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t first[2], second[2], *at = a + (2 * t + w) * 4;
          code_operands(h == 0 ? (w ? k.c[t].y : k.c[t].x) : (w ? k.c[t].w : k.c[t].z), first, second);
          at[0] = first[0]; at[1] = first[1]; at[2] = second[0]; at[3] = second[1];
        }
      put(a, __half2float(__ushort_as_half((unsigned short)((h == 0 ? k.r.x : k.r.y) & 0xFFFFu))) * CODE_BACK, h);
    };
    // A pair's stage; `next` is read on the way.  The window of 64 groups' minima is this thread's own.
    auto pair = [&](const Codes& k, Codes& next, int pr) {
      minima[pr & 31][threadIdx.x] = __byte_perm(k.r.x, k.r.y, 0x7632u);       // (the record is read last: the codes are here)
      release();
      turn(k, 0);
      const bool end = ends(pr);
      if (!end) read(next);
      turn(k, 1);
      ++i;
      if (!end) return;
      // minima of 64 groups, twice each (their x sums are two float16); groups of another range or of none: zeros
      wait(full0 + st * 8, sp, &gave_up);
      release();
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        uint32_t a[32];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = (pr & ~31) + h * 16 + e;
          const uint32_t m = at >= p0 && at <= pr ? minima[h * 16 + e][threadIdx.x] : 0u;
          a[2 * e] = __byte_perm(m, 0u, 0x1010u);
          a[2 * e + 1] = __byte_perm(m, 0u, 0x3232u);
        }
        put(a, 0x1p6f, h);
      }
      ++i;
      if (pr + 1 < p1) read(next);
    };
    Codes k0, k1;
    read(k0);
    for (int pr = p0; pr < p1; pr += 2) {
      pair(k0, k1, pr);
      if (pr + 1 < p1) pair(k1, k0, pr + 1);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  // Sums of the cluster's ranges, in their order: [NB][256] floats in each CTA's shared memory, where the ring was.  The
  // rows' powers of two are fetched meanwhile, and each thread has several sums under way: one after the other, with a
  // load of the power in each, this took 5 us for 64 rows, and takes 1 us in one CTA, 3 us in a cluster of 8: the 56 KB that a
  // CTA reads from the others.  (Sums stored to the shared memory of a row's owner instead: 1 us more.)
  cg::cluster_group cluster = cg::this_cluster();
  const int splits = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  float* red = reinterpret_cast<float*>(ring);
  float* pws = reinterpret_cast<float*>(&minima[0][0]);
  static_assert(sizeof(minima) >= 8 * NB * 4, "powers of up to 8 ranges");
  constexpr int LD = TC_F + 4, UN = 8;
  const bool lost = gave_up;
  pdl_wait();                                         // every thread that writes results: h and pow of kernels before
  if (warp >= 8 && warp < 16) {
    const int f = threadIdx.x - 256;
#pragma unroll
    for (int n = 0; n < NB / 2; ++n) {
      red[(2 * n) * LD + f] = lost ? NAN : acc[n].x;
      red[(2 * n + 1) * LD + f] = lost ? NAN : acc[n].y;
    }
  } else if (warp < 8) {
    for (int i = threadIdx.x; i < splits * NB; i += 256)
      pws[i] = __ldcg(p.pow + ((int64_t)(i / NB) * p.blocks + block) * NB + i % NB);
  }
  cluster.sync();
  pdl_trigger();
  // number i of four features of a row: its place in shared memory, and the results
  auto place = [&](int i) { return i / (TC_F / 4) * LD + i % (TC_F / 4) * 4; };
  auto put = [&](int i, const float (&s)[4]) {
    const int row = block * p.rows_per_block + i / (TC_F / 4), n = f_range * TC_F + i % (TC_F / 4) * 4;
    if (row >= p.M || n >= p.N) return;
    const int64_t at = (int64_t)row * p.N + n;
    if (p.fours && p.h_out) {
      const float4 h = *reinterpret_cast<const float4*>(p.h + at);
      *reinterpret_cast<float4*>(p.h_out + at) = make_float4(h.x + s[0], h.y + s[1], h.z + s[2], h.w + s[3]);
    } else if (p.fours) {
      alignas(8) T y[4] = {from_f_inf<T>(s[0]), from_f_inf<T>(s[1]), from_f_inf<T>(s[2]), from_f_inf<T>(s[3])};
      *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.y) + at) = *reinterpret_cast<const uint2*>(y);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (n + e >= p.N) break;
        if (p.h_out) p.h_out[at + e] = p.h[at + e] + s[e];
        else reinterpret_cast<T*>(p.y)[at + e] = from_f_inf<T>(s[e]);
      }
    }
  };
  const int all = p.rows_per_block * (TC_F / 4);
  if (splits == 1) {
    for (int i0 = threadIdx.x; i0 < all; i0 += UN * TC_THREADS) {
      float4 v[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u)
        if (i0 + u * TC_THREADS < all) v[u] = *reinterpret_cast<const float4*>(red + place(i0 + u * TC_THREADS));
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int i = i0 + u * TC_THREADS;
        if (i >= all) break;
        const float w = pws[i / (TC_F / 4)], s[4] = {v[u].x * w, v[u].y * w, v[u].z * w, v[u].w * w};
        put(i, s);
      }
    }
  } else {
    for (int i = rank * TC_THREADS + threadIdx.x; i < all; i += splits * TC_THREADS) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      for (int k0 = 0; k0 < splits; k0 += UN) {
        float4 v[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u)
          if (k0 + u < splits) v[u] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(red + place(i), k0 + u));
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          if (k0 + u >= splits) break;
          const float w = pws[(k0 + u) * NB + i / (TC_F / 4)];
          s[0] = fmaf(v[u].x, w, s[0]);
          s[1] = fmaf(v[u].y, w, s[1]);
          s[2] = fmaf(v[u].z, w, s[2]);
          s[3] = fmaf(v[u].w, w, s[3]);
        }
      }
      put(i, s);
    }
  }
  cluster.sync();                                     // nobody leaves while others read
  if (warp == 16) tc::tmem_dealloc(tmem, 512);
}

template <typename T, int FT>
int32_t launch_few(const LinearQ4Params& p, cudaStream_t st) {
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)linear_q4_few_kernel<T, FT>, FW_MAX_SMEM, smem_set));
  const int sets = akvs_cdiv(p.N, 16 * FT);
  AKVS_CUDA(launch_pdl(linear_q4_few_kernel<T, FT>, dim3(sets < 148 ? sets : 148), dim3(FW_THREADS),
                       (size_t)few_smem(FT, p.M, p.pairs, sizeof(T) == 4 ? 3 : 1), st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

// Row blocks of a call: up to 64 rows each, as even as they go.
int tc_blocks(int M) { return akvs_cdiv(M, 64); }
int tc_rows(int M) { return M <= 32 ? 32 : 64; }
int64_t tc_scratch(int M, int K) {
  const int groups = K / 64, pairs = (groups + 1) / 2, nb = tc_rows(M);
  return (int64_t)tc_blocks(M) * nb * (128ll * (2 * pairs + lq_min_steps(groups)) + 8 * 4) + 256;
}

// How many clusters of k CTAs of the kernel run at once (0: a cluster of that size does not), asked once per device and size.
template <typename T, int NB>
int32_t clusters_at_a_time(int k, int& fit) {
  static std::atomic<int> known[64][LQ_MAX_RANGES + 1];              // one more than fit
  int dev = 0;
  AKVS_CUDA(cudaGetDevice(&dev));
  fit = known[dev & 63][k].load(std::memory_order_relaxed) - 1;
  if (fit >= 0) return AKVS_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(k, 148);
  cfg.blockDim = dim3(TC_THREADS);
  cfg.dynamicSmemBytes = TcStage<NB>::SMEM;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = k;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&fit, linear_q4_tc_kernel<T, NB>, &cfg) != cudaSuccess) {
    cudaGetLastError();                               // not an error of this call: other sizes may do; asked again the next time
    fit = 0;
    return AKVS_OK;
  }
  fit = fit < 0 ? 0 : fit;
  known[dev & 63][k].store(fit + 1, std::memory_order_relaxed);
  return AKVS_OK;
}

template <typename T, int NB>
int32_t launch_tc(const LinearQ4Params& l, void* scratch, cudaStream_t st) {
  using S = TcStage<NB>;
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)linear_q4_tc_kernel<T, NB>, S::SMEM, smem_set));
  TcParams p;
  const int blocks = tc_blocks(l.M), tiles = akvs_cdiv(l.N, TC_F);
  p.w = l.w; p.y = l.y; p.h = l.h; p.h_out = l.h_out; p.M = l.M; p.N = l.N; p.pairs = l.pairs;
  p.tiles16 = akvs_cdiv(l.N, 16);
  p.fours = l.N % 4 == 0 && (l.h_out ? (reinterpret_cast<uintptr_t>(l.h) | reinterpret_cast<uintptr_t>(l.h_out)) % 16 == 0
                                     : reinterpret_cast<uintptr_t>(l.y) % 8 == 0);
  p.rows_per_block = akvs_cdiv(l.M, blocks);
  p.steps = 2 * l.pairs + lq_min_steps(l.groups);
  p.xt = reinterpret_cast<uint8_t*>(scratch);
  const int64_t x_bytes = (int64_t)blocks * p.steps * S::X;
  p.pow = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(scratch) + x_bytes);
  // One CTA an SM; how many clusters fit at a time depends on how many SMs a part of the GPU has.
  int fit[LQ_MAX_RANGES + 1] = {};
  for (int k = 1; k <= LQ_MAX_RANGES && (k == 1 || l.pairs / k >= 4); ++k) AKVS_TRY((clusters_at_a_time<T, NB>(k, fit[k])));
  int splits = lq_ranges((int64_t)tiles * blocks, l.pairs, fit);
  if (splits == 0) return AKVS_ERR_CUDA;
  p.pairs_per_split = akvs_cdiv(l.pairs, splits);
  splits = akvs_cdiv(l.pairs, p.pairs_per_split);
  p.blocks = blocks;
  AKVS_CUDA(launch_pdl(linear_q4_rows_kernel<T, NB>, dim3(blocks * NB, splits), dim3(ROWS_THREADS), 0, st, reinterpret_cast<const T*>(l.x),
                       l.x_ld, l.M, p.rows_per_block, l.groups, l.pairs, p.pairs_per_split, reinterpret_cast<uint8_t*>(scratch),
                       const_cast<float*>(p.pow)));
  AKVS_LAUNCHED();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = row_grid((int64_t)tiles * splits, blocks);
  cfg.blockDim = dim3(TC_THREADS);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, linear_q4_tc_kernel<T, NB>, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

// Which kernel.  Few rows: one CTA per SM while x fits into its shared memory.  tcgen05: from 17 rows on; its start (x in
// order, tensor memory, the cluster's sum) costs some 10 us, but a step less than the clusters' where these have more columns than
// their SMs can share, so it also takes fewer rows there.
enum class Path { few, clusters, tc };
Path path_of(int dtype, int M, int N, int K) {
  const int pairs = (K / 64 + 1) / 2;
  if (M <= 8 && few_smem(1, M, pairs, dtype == AKVS_F32 ? 3 : 1) <= FW_MAX_SMEM) return Path::few;
  if (dtype != AKVS_F32 && (M > 16 || lq_prefers_tensor(M, N, K / 64))) return Path::tc;
  return Path::clusters;
}

// What a grid holds, with up to 8 ranges of columns; beyond that lie only calls whose x or y no GPU holds.
bool fits_a_grid(int dtype, int M, int N, int K) {
  switch (path_of(dtype, M, N, K)) {
    case Path::few: return true;
    case Path::clusters: return (int64_t)akvs_cdiv(M, 8) * akvs_cdiv(N, LQ_F) <= 0x7fffffff / 8;
    default:
      return (int64_t)tc_blocks(M) * akvs_cdiv(N, TC_F) <= 0x7fffffff / 8 && tc_blocks(M) < 1 << 25 && (double)tc_blocks(M) * (K + 4096.0) < 1e14;
  }
}

int32_t linear(int32_t dtype, const void* x, int64_t x_ld, const void* w, int64_t w_bytes, void* y, const float* h, float* h_out,
               int32_t M, int32_t N, int32_t K, void* scratch, int64_t scratch_size, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (M < 0 || N <= 0 || K <= 0) return AKVS_ERR_INVALID_ARG;
  const int64_t need = akvs_linear_q4_bytes(N, K), es = (int64_t)dtype_size(dtype);
  if (need < 0) return AKVS_ERR_SHAPE;
  if (M == 0) return AKVS_OK;
  void* out = h_out ? (void*)h_out : y;
  if (!x || !w || !out || (h_out && !h)) return AKVS_ERR_INVALID_ARG;
  if (x_ld < K || w_bytes < need) return AKVS_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(w) || x_ld * es % 16 || reinterpret_cast<uintptr_t>(out) % (h_out ? 4 : es) ||
      reinterpret_cast<uintptr_t>(h) % 4)
    return AKVS_ERR_INVALID_ARG;
  const int64_t room = akvs_op_linear_q4_scratch_bytes(dtype, M, N, K);
  if (room < 0) return AKVS_ERR_TOO_LARGE;
  const int64_t x_n = ((M - 1) * x_ld + K) * es, out_n = (int64_t)M * N * (h_out ? 4 : es);
  if (bytes_overlap(x, x_n, out, out_n) || bytes_overlap(w, need, out, out_n) || (h_out && h != h_out && bytes_overlap(h, out_n, out, out_n)))
    return AKVS_ERR_INVALID_ARG;
  if (room > 0) {
    if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || scratch_size < room) return AKVS_ERR_WORKSPACE;
    if (bytes_overlap(x, x_n, scratch, room) || bytes_overlap(w, need, scratch, room) || bytes_overlap(out, out_n, scratch, room) ||
        (h_out && bytes_overlap(h, out_n, scratch, room)))
      return AKVS_ERR_INVALID_ARG;
  }
  LinearQ4Params p = {x, x_ld, reinterpret_cast<const uint8_t*>(w), y, h, h_out, M, N, K / 64, (K / 64 + 1) / 2, 0, 0};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    const Path path = path_of(dtype, M, N, K);
    if (path == Path::few) {
      // As few rounds of teams as there can be: 16 warps share the columns where an SM has one tile, 8 up to two, 4 beyond
      // (8 rows of 55296 x 5120: 40 us, with one team of 16 56).  Two tiles at a time read x half as often, where teams of
      // four have more than one round and x leaves the room (one row of 11008 x 2048: 5.6 us, with one tile 6.2).
      const int tiles = akvs_cdiv(N, 16);
      p.team = tiles <= 148 ? 16 : tiles <= 2 * 148 ? 8 : 4;
      return tiles > 4 * 148 && few_smem(2, M, p.pairs, sizeof(T) == 4 ? 3 : 1) <= FW_MAX_SMEM ? launch_few<T, 2>(p, st) : launch_few<T, 1>(p, st);
    }
    if constexpr (sizeof(T) == 4) {
      return launch<T, 1>(p, st);
    } else {
      if (path == Path::tc) return tc_rows(M) == 32 ? launch_tc<T, 32>(p, scratch, st) : launch_tc<T, 64>(p, scratch, st);
      return M <= 8 ? launch<T, 1>(p, st) : launch<T, 2>(p, st);
    }
  });
}

}  // namespace

extern "C" int64_t akvs_linear_q4_bytes(int32_t N, int32_t K) {
  if (N <= 0 || N > 0x7fffff00 || K <= 0 || K % 64) return -1;
  return ((int64_t)N + 15) / 16 * ((K / 64 + 1) / 2) * LQ_BLOCK;
}

extern "C" int64_t akvs_op_linear_q4_scratch_bytes(int32_t dtype, int32_t M, int32_t N, int32_t K) {
  if ((dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) || M < 0 || akvs_linear_q4_bytes(N, K) < 0 || !fits_a_grid(dtype, M, N, K))
    return -1;
  return path_of(dtype, M, N, K) == Path::tc ? tc_scratch(M, K) : 0;
}

extern "C" int32_t akvs_op_linear_q4_pack(const void* codes, const void* meta, int32_t N, int32_t K, void* packed, void* stream) {
  if (N <= 0 || K <= 0) return AKVS_ERR_INVALID_ARG;
  const int64_t bytes = akvs_linear_q4_bytes(N, K);
  if (bytes < 0) return AKVS_ERR_SHAPE;
  if (!codes || !meta || !packed) return AKVS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(codes) & 3) || (reinterpret_cast<uintptr_t>(meta) & 3) || !aligned16(packed)) return AKVS_ERR_INVALID_ARG;
  if (bytes_overlap(codes, (int64_t)N * K / 2, packed, bytes) || bytes_overlap(meta, (int64_t)N * K / 16, packed, bytes)) return AKVS_ERR_INVALID_ARG;
  const int64_t blocks = (bytes / LQ_BLOCK + LQ_WARPS - 1) / LQ_WARPS;
  if (blocks > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  linear_q4_pack_kernel<<<(unsigned)blocks, LQ_THREADS, 0, reinterpret_cast<cudaStream_t>(stream)>>>(
      reinterpret_cast<const uint8_t*>(codes), reinterpret_cast<const uint32_t*>(meta), N, K / 64, (K / 64 + 1) / 2,
      reinterpret_cast<uint8_t*>(packed));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

extern "C" int32_t akvs_op_linear_q4(int32_t dtype, const void* x, int64_t x_ld, const void* packed, int64_t packed_bytes, void* y,
                                     int32_t M, int32_t N, int32_t K, void* scratch, int64_t scratch_bytes, void* stream) {
  return linear(dtype, x, x_ld, packed, packed_bytes, y, nullptr, nullptr, M, N, K, scratch, scratch_bytes, stream);
}

extern "C" int32_t akvs_op_linear_q4_residual(int32_t dtype, const void* x, int64_t x_ld, const void* packed, int64_t packed_bytes,
                                              const float* h, float* h_out, int32_t M, int32_t N, int32_t K, void* scratch,
                                              int64_t scratch_bytes, void* stream) {
  if (M > 0 && !h_out) return AKVS_ERR_INVALID_ARG;
  return linear(dtype, x, x_ld, packed, packed_bytes, nullptr, h, h_out, M, N, K, scratch, scratch_bytes, stream);
}
