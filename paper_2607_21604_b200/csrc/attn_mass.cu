// Attention weight that every cached key has received: per kv head h and key j
//     mass_out[h][j] = mass_in[h][j] + sum over rows r that see j, heads i of the group of h:
//                      exp(q_ri . k_jh / sqrt(hd) - lse_ri)
// with lse the log-sum-exp of the row, as the attention that produced the row left it.
// The rows of the g = n_q / n_kv query heads of a kv head are stacked (r * g + i); every sum runs
// over them in a fixed order, so equal calls give equal bits.
//
// 16-bit types run on the tensor cores with the keys along M, so that a thread owns one key and its
// sum over the rows needs no shuffle; the score matrix never leaves tensor memory:
//     S^T = K Q^T     tcgen05.mma, two tiles of 128 keys against one tile of stacked rows
//     sum             two warp groups, one per key tile: exp2 of a row of S^T, added up in registers
// A CTA keeps 256 keys while the rows' Q tiles stream past them (each is used twice), then goes on to
// its next 256 keys.  Two warps work out what each column sees; a tile whose columns all see its
// keys runs without a mask.  With many rows the exponentials bound it (16 per clock and SM), with few
// rows reading K once (16 rows x 32 heads over 12416 keys: 9.4 us, 2.8 TB/s; 7.4 us with K in L2).  Few
// keys and many rows: a cluster shares the row tiles of its keys and adds the partial sums through
// distributed shared memory.
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
constexpr int M_THREADS = 384;       // warp group 0: TMA, MMA and columns; warp groups 1 and 2: sums
constexpr int M_SLAB = 128 * 128;    // 128 rows of 64 values

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row of a tile is a column of S^T: BR rows x g heads, rows from rt * BR.
struct Cols { int BR, gb; };

// What the columns of a tile see, worked out by NWARP warps (`half` of them) for the summing warps, with
// all loads of a lane in flight together.  col_z: -lse in log2 units; col_rng: first visible key and how
// many follow; flag[w][half]: some column of the half needs a mask for key tile w.
template <int BQ, int NWARP>
struct ColumnLane {                  // a lane's columns, the same in every tile: row and head inside it
  static constexpr int N = BQ / (32 * NWARP);
  static_assert(BQ % (32 * NWARP) == 0, "every lane has as many columns");
  int r_in[N], head_in[N];           // r_in = BR: a column that is never loaded
  __device__ __forceinline__ ColumnLane(const Cols& cl, int half, int lane) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = (x * NWARP + half) * 32 + lane;
      r_in[x] = min(i / cl.gb, cl.BR);
      head_in[x] = i % cl.gb;
    }
  }
};
template <int BQ, int NWARP, int NW>
struct ColumnLoad {                  // NW: key tiles of an item
  static constexpr int N = BQ / (32 * NWARP);
  float z[N];
  int lo[N], hi[N];
  __device__ __forceinline__ void fetch(const MassParams& p, const Cols& cl, const ColumnLane<BQ, NWARP>& ln, int rt, int h) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int r = min(rt * cl.BR + ln.r_in[x], p.R - 1);
      z[x] = __ldg(p.lse + (int64_t)r * p.n_q + h * p.g + ln.head_in[x]);
      lo[x] = __ldg(p.k_lo + r);
      hi[x] = __ldg(p.k_hi + r);
    }
  }
  __device__ __forceinline__ void store(const MassParams& p, const Cols& cl, const ColumnLane<BQ, NWARP>& ln, int rt, int k0, int half,
                                        int lane, float* col_z, int2* col_rng, volatile int* flag) const {
    bool masked[NW] = {};
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = (x * NWARP + half) * 32 + lane;
      const bool real = ln.r_in[x] < cl.BR && rt * cl.BR + ln.r_in[x] < p.R;
      const int a = max(lo[x], 0), b = min(hi[x], p.T - 1);
      const bool blind = !real || z[x] == -INFINITY || a > b;              // such a column adds nothing
      // columns of zeros behind the last row ask for no mask (add_columns)
#pragma unroll
      for (int w = 0; w < NW; ++w)
        masked[w] |= real && (blind || a > k0 + w * BK || b < min(k0 + (w + 1) * BK, p.T) - 1);
      col_z[i] = blind ? -INFINITY : -z[x] * LOG2E;
      // seen <=> (unsigned)(key - first) <= length: never for a blind column (keys are not negative)
      col_rng[i] = blind ? make_int2(0x7fffffff, 0) : make_int2(a, b - a);
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const bool any = __any_sync(0xFFFFFFFFu, masked[w]);
      if (lane == 0) flag[w * NWARP + half] = any;
    }
    __syncwarp();
  }
};

// N columns of a key's row of S^T: no branch inside, so that the loads, exponentials and sums of
// different columns overlap.  Columns behind the last row hold a row of zeros and a z of -inf: exp2(0 - inf)
// = 0 without a mask, unless the key holds an infinity or a NaN, with which 0 gives NaN.  Such columns end
// a tile, so the last column shows it, and its NaN turns the mask on (for a real column, too: it changes
// no result).  One compare and vote per 64 columns: 512 rows x 40 heads over 32768 keys 238.8 -> 239.6 us.
template <int N>
__device__ __forceinline__ void add_columns(const float (&t)[N], const float* z, const int2* ranges, bool mask, int key,
                                            float scale2, float2 (&acc)[4]) {
  const float2 sc = make_float2(scale2, scale2);
  mask |= __any_sync(0xFFFFFFFFu, t[N - 1] != t[N - 1]) != 0;
  if (!mask) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 zz = *reinterpret_cast<const float4*>(z + i);
      const float2 x = __ffma2_rn(make_float2(t[i], t[i + 1]), sc, make_float2(zz.x, zz.y));
      const float2 y = __ffma2_rn(make_float2(t[i + 2], t[i + 3]), sc, make_float2(zz.z, zz.w));
      acc[(i >> 1) & 3] = __fadd2_rn(acc[(i >> 1) & 3], make_float2(ex2(x.x), ex2(x.y)));
      acc[((i >> 1) + 1) & 3] = __fadd2_rn(acc[((i >> 1) + 1) & 3], make_float2(ex2(y.x), ex2(y.y)));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 zz = *reinterpret_cast<const float2*>(z + i);
      const int4 rng = *reinterpret_cast<const int4*>(ranges + i);
      const float2 x = __ffma2_rn(make_float2(t[i], t[i + 1]), sc, zz);
      const float e0 = ex2(x.x), e1 = ex2(x.y);
      acc[(i >> 1) & 3] = __fadd2_rn(acc[(i >> 1) & 3], make_float2((unsigned)(key - rng.x) <= (unsigned)rng.y ? e0 : 0.f,
                                                                  (unsigned)(key - rng.z) <= (unsigned)rng.w ? e1 : 0.f));
    }
  }
}
__device__ __forceinline__ float total(const float2 (&acc)[4]) {
  const float2 a = __fadd2_rn(acc[0], acc[1]), b = __fadd2_rn(acc[2], acc[3]);
  return (a.x + a.y) + (b.x + b.y);
}

// A 128-byte-swizzled operand `bytes` further on in shared memory.  The address sits in the descriptor's
// low bits in units of 16 bytes, so a constant is added instead of building it anew.
__device__ __forceinline__ uint64_t desc_at(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }

// Bounded waits all over: whoever runs out raises the flag, and the others follow.
struct Waiter {
  uint64_t* bar;
  volatile int* abort_flag;
  __device__ __forceinline__ bool operator()(int b, uint32_t parity) const { return tc::mbar_wait(&bar[b], parity & 1, abort_flag); }
};

// -- few rows: all columns fit one tile of 128.  The Q tile stays as long as the head does, K streams
// through two stages by TMA and S^T has two buffers, so that items overlap; bound by reading K.
namespace few {
constexpr int BQ = 128, KST = 2;
template <int HD> constexpr int TILE = HD / 64 * M_SLAB;
// shared memory: K[2][2 tiles] | Q | barriers (256 B) | what a column sees, twice | flags
template <int HD> constexpr int SMEM = (2 * KST + 1) * TILE<HD> + 256 + 2 * BQ * 12 + 64;
enum { KFULL = 0, KEMPTY = 2, QFULL = 4, QEMPTY = 5, SFULL = 6 /*[2 groups][2]*/, SEMPTY = 10, CFULL = 14, CEMPTY = 16, COUNT = 18 };
static_assert(COUNT * 8 + 8 <= 256 && SMEM<128> <= 232448, "shared memory of one CTA");

template <typename T, int HD>
__global__ void __launch_bounds__(M_THREADS, 1)
mass_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ, const MassParams p,
                const Cols cols, int key_items, int n_items, uint32_t fmt) {
  constexpr int OFF_Q = 2 * KST * TILE<HD>, OFF_BAR = OFF_Q + TILE<HD>, OFF_COL = OFF_BAR + 256, OFF_FLAG = OFF_COL + 2 * BQ * 12;
  extern __shared__ __align__(1024) uint8_t smem[];
  if (tc::smem_u32(smem) & 1023u) return;           // swizzled tiles need 1024-byte alignment
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* col_z = reinterpret_cast<float*>(smem + OFF_COL);
  int2* col_rng = reinterpret_cast<int2*>(col_z + 2 * BQ);
  volatile int* flag = reinterpret_cast<volatile int*>(smem + OFF_FLAG);    // [2][2 groups][2 halves]
  const Waiter wait{bar, abort_flag};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < COUNT; ++i) tc::mbar_init(&bar[i], i >= CEMPTY ? 8 : i >= CFULL ? 2 : i >= SEMPTY ? 4 : 1);
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  for (int i = threadIdx.x; i < TILE<HD> / 16; i += M_THREADS)      // what the load leaves out behind the rows stays zero
    *reinterpret_cast<uint4*>(smem + OFF_Q + i * 16) = make_uint4(0u, 0u, 0u, 0u);
  tc::fence_proxy_async();
  pdl_wait();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // consecutive items, of one head mostly
  const int item0 = (int)((int64_t)n_items * blockIdx.x / gridDim.x), item1 = (int)((int64_t)n_items * (blockIdx.x + 1) / gridDim.x);
  const bool rows = p.R > 0;
  const int n_cols = p.R * p.g;
  auto head_ends = [&](int item) { return item + 1 == item1 || (item + 1) / key_items != item / key_items; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    bool ok = true;
    if (warp == 0 && lane == 0) {
      // ------------------------------------------------------------------ TMA producer
      tc::prefetch_tmap(&tmK);
      tc::prefetch_tmap(&tmQ);
      int nq = 0;
      for (int item = item0, it = 0; item < item1; ++item, ++it) {
        const int h = item / key_items, j0 = (item % key_items) * (2 * BK), ks = it % KST;
        if (!(ok = wait(KEMPTY + ks, (it / KST) ^ 1))) break;
        tc::mbar_expect_tx(&bar[KFULL + ks], 2 * TILE<HD>);
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int c = 0; c < HD / 64; ++c)
            tc::tma_load_2d(smem + (2 * ks + w) * TILE<HD> + c * M_SLAB, &tmK, h * HD + c * 64, j0 + w * BK, &bar[KFULL + ks]);
        if (!rows || (it > 0 && (item - 1) / key_items == h)) continue;      // the head's rows are there
        if (!(ok = wait(QEMPTY, nq ^ 1))) break;
        tc::mbar_expect_tx(&bar[QFULL], (uint32_t)(cols.BR * cols.gb) * 128u * (HD / 64));
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) tc::tma_load_3d(smem + OFF_Q + c * M_SLAB, &tmQ, c * 64, h * p.g, 0, &bar[QFULL]);
        ++nq;
      }
    } else if (warp == 1 && lane == 0) {
      // ------------------------------------------------------------------ MMA issuer
      const uint32_t idesc = tc::idesc_f16(fmt, BK, (n_cols + 63) / 64 * 64, 0);      // whole chunks of 64 columns
      const uint64_t q_desc = tc::smem_desc_k_sw128(tc::smem_u32(smem + OFF_Q)), k_desc = tc::smem_desc_k_sw128(tc::smem_u32(smem));
      int nq = 0;
      for (int item = item0, it = 0; item < item1 && ok; ++item, ++it) {
        const int ks = it % KST, b = it & 1;
        if (!(ok = wait(KFULL + ks, it / KST))) break;
        if (rows) {
          if (!(ok = wait(QFULL, nq))) break;
          for (int w = 0; w < 2; ++w) {
            if (!(ok = wait(SEMPTY + 2 * w + b, (it >> 1) ^ 1))) break;
            tc::fence_after_sync();
            const uint64_t kd = desc_at(k_desc, (2 * ks + w) * TILE<HD>);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint32_t off = (k >> 2) * M_SLAB + (k & 3) * 32;
              tc::mma_f16(tmem_base + w * 256 + b * BQ, desc_at(kd, off), desc_at(q_desc, off), idesc, k != 0);
            }
            tc::mma_commit(&bar[SFULL + 2 * w + b]);
          }
          if (!ok) break;
          if (head_ends(item)) { tc::mma_commit(&bar[QEMPTY]); ++nq; }
        }
        tc::mma_commit(&bar[KEMPTY + ks]);
      }
    } else if (warp >= 2 && rows) {
      // ------------------------------------------------------------------ what the columns see
      const ColumnLane<BQ, 2> ln(cols, warp - 2, lane);
      ColumnLoad<BQ, 2, 2> cl;
      for (int item = item0, it = 0; item < item1; ++item, ++it) {
        const int h = item / key_items, cb = it & 1;
        if (it == 0 || (item - 1) / key_items != h) cl.fetch(p, cols, ln, 0, h);
        if (!(ok = wait(CEMPTY + cb, (it >> 1) ^ 1))) break;
        cl.store(p, cols, ln, 0, (item % key_items) * (2 * BK), warp - 2, lane, col_z + cb * BQ, col_rng + cb * BQ, flag + cb * 4);
        if (lane == 0) tc::mbar_arrive(&bar[CFULL + cb]);
      }
    }
    if (!ok) *abort_flag = 1;
  } else {
    // ---------------------------------------------------------------------- a key per thread
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int w = (warp >> 2) - 1, m = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
    bool ok = true;
    for (int item = item0, it = 0; item < item1; ++item, ++it) {
      const int h = item / key_items, key = (item % key_items) * (2 * BK) + w * BK + m, b = it & 1;
      const int64_t at = (int64_t)h * p.T + key;
      const float old = p.mass_in && key < p.T ? p.mass_in[at] : 0.f;
      float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      if (rows) {
        if (!(ok = wait(CFULL + b, it >> 1))) break;
        const bool mask = (flag[(b * 2 + w) * 2] | flag[(b * 2 + w) * 2 + 1]) != 0;
        if (!(ok = wait(SFULL + 2 * w + b, it >> 1))) break;
        tc::fence_after_sync();
        // 64 columns at a time, the next ones on their way from tensor memory meanwhile
        const uint32_t s_addr = lane_addr + w * 256 + b * BQ;
        const int chunks = (n_cols + 63) / 64;
        float ta[64], tb[64];
        auto fetch = [&](float(&t)[64], int c) {
          tc::tmem_ld32(s_addr + c * 64, *reinterpret_cast<float(*)[32]>(&t[0]));
          tc::tmem_ld32(s_addr + c * 64 + 32, *reinterpret_cast<float(*)[32]>(&t[32]));
        };
        auto taken = [&]() {                              // all of the tile is in registers: its buffer is free
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bar[SEMPTY + 2 * w + b]);
        };
        const float* z = col_z + b * BQ;
        const int2* rng = col_rng + b * BQ;
        fetch(ta, 0);
        tc::tmem_ld_wait();
        if (chunks > 1) fetch(tb, 1);
        else taken();
        add_columns<64>(ta, z, rng, mask, key, p.scale * LOG2E, acc);
        if (chunks > 1) {
          tc::tmem_ld_wait();
          taken();
          add_columns<64>(tb, z + 64, rng + 64, mask, key, p.scale * LOG2E, acc);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bar[CEMPTY + b]);
      }
      if (key < p.T) p.mass_out[at] = old + total(acc);
    }
    if (!ok) {                                            // a wait ran out: NaN rather than masses that lack terms
      *abort_flag = 1;
      for (int item = item0; item < item1; ++item) {
        const int key = (item % key_items) * (2 * BK) + w * BK + m;
        if (key < p.T) p.mass_out[(int64_t)(item / key_items) * p.T + key] = NAN;
      }
    }
  }
  if (*abort_flag) __nanosleep(200000);
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem_base, 512);
  }
}
}  // namespace few

// -- many rows: tiles of up to 256 columns stream past the K of 256 keys.  The width halves what an MMA
// reads of its A operand per column and spreads a tile's barriers over more work; one buffer of S^T per
// group is all that fits then, and a group's next product waits until its last columns are taken.
// 512 rows x 40 heads x 32768 keys: 220 to 240 us, of which the exponentials are 160 us (16 per clock and
// SM).  Built and measured instead of it: 128 columns with two buffers 238 us (against 229); an issuing
// thread per group (and a warp less for the columns) 237 us; K in tensor memory as the A operand with
// tiles of 96 columns, two groups of two buffers 276 us, three groups of one buffer 253 us; exp2 of an
// eighth / a quarter / half of the columns by a polynomial on the FMA units 235 / 239 / 261 us (against
// 236): two warps per scheduler do not hide its chain.
namespace many {
constexpr int BQ = 256, QST = 2;
template <int HD> constexpr int KTILE = HD / 64 * M_SLAB;                // 128 keys
template <int HD> constexpr int QTILE = HD / 64 * BQ * 128;
// shared memory: K[2 tiles] | Q[2] | barriers (256 B) | what a column sees, twice | partial sums | flags
template <int HD> constexpr int SMEM = 2 * KTILE<HD> + QST * QTILE<HD> + 256 + 2 * BQ * 12 + 2 * 128 * 4 + 64;
enum { QFULL = 0, QEMPTY = QFULL + QST, KFULL = QEMPTY + QST, KEMPTY, SFULL /*[2 groups]*/, SEMPTY = SFULL + 2, CFULL = SEMPTY + 2,
       CEMPTY = CFULL + 2, COUNT = CEMPTY + 2 };
static_assert(COUNT * 8 + 8 <= 256 && SMEM<128> <= 232448, "shared memory of one CTA");

template <typename T, int HD>
__global__ void __launch_bounds__(M_THREADS, 1)
mass_many_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ, const MassParams p,
                 int C, int key_items, int n_items, int BR, int q_boxes, uint32_t fmt) {
  constexpr int OFF_Q = 2 * KTILE<HD>, OFF_BAR = OFF_Q + QST * QTILE<HD>, OFF_COL = OFF_BAR + 256, OFF_PART = OFF_COL + 2 * BQ * 12;
  constexpr int OFF_FLAG = OFF_PART + 2 * 128 * 4, Q_SLAB = BQ * 128;
  extern __shared__ __align__(1024) uint8_t smem[];
  if (tc::smem_u32(smem) & 1023u) return;           // swizzled tiles need 1024-byte alignment (the same in every CTA)
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* part = reinterpret_cast<float*>(smem + OFF_PART);          // [2][128]
  float* col_z = reinterpret_cast<float*>(smem + OFF_COL);          // [2][BQ] -lse of a column in log2 units
  int2* col_rng = reinterpret_cast<int2*>(col_z + 2 * BQ);          // [2][BQ] its first visible key, and how many follow
  volatile int* flag = reinterpret_cast<volatile int*>(smem + OFF_FLAG);    // [2][2 groups][2 halves] a column needs a mask
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < COUNT; ++i) tc::mbar_init(&bar[i], i >= CEMPTY ? 8 : i >= CFULL ? 2 : i >= SEMPTY ? 4 : 1);
    *abort_flag = 0;
    tc::fence_barrier_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_slot, 512);
    tc::tmem_relinquish();
  }
  // Q tiles hold BR * g rows; what the loads leave out behind them stays zero
  for (int i = threadIdx.x; i < QST * QTILE<HD> / 16; i += M_THREADS)
    *reinterpret_cast<uint4*>(smem + OFF_Q + i * 16) = make_uint4(0u, 0u, 0u, 0u);
  tc::fence_proxy_async();
  pdl_wait();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // every n_cl-th item for a cluster, so that masked items (the end of a causal window) spread
  const int rank = blockIdx.x % C, item0 = blockIdx.x / C, step = gridDim.x / C;
  const int row_tiles = (p.R + BR - 1) / BR;

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
        for (int item = item0; item < n_items && ok; item += step, ++it) {
          const int h = item / key_items, j0 = (item % key_items) * (2 * BK);
          if (!tc::mbar_wait(&bar[KEMPTY], (it & 1) ^ 1, abort_flag)) { ok = false; break; }
          tc::mbar_expect_tx(&bar[KFULL], 2 * KTILE<HD>);
#pragma unroll
          for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int c = 0; c < HD / 64; ++c)
              tc::tma_load_2d(smem + w * KTILE<HD> + c * M_SLAB, &tmK, h * HD + c * 64, j0 + w * BK, &bar[KFULL]);
          for (int rt = rank; rt < row_tiles; rt += C, ++n) {
            const int qs = n % QST;
            if (!tc::mbar_wait(&bar[QEMPTY + qs], ((n / QST) & 1) ^ 1, abort_flag)) { ok = false; break; }
            tc::mbar_expect_tx(&bar[QFULL + qs], (uint32_t)(q_boxes * box_bytes * (HD / 64)));
            for (int x = 0; x < q_boxes; ++x)
#pragma unroll
              for (int c = 0; c < HD / 64; ++c)
                tc::tma_load_3d(smem + OFF_Q + qs * QTILE<HD> + c * Q_SLAB + x * box_bytes, &tmQ, c * 64, h * p.g,
                                rt * BR + x * box_rows, &bar[QFULL + qs]);
          }
        }
        if (!ok) *abort_flag = 1;
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      if (lane == 0) {
        bool ok = true;
        int it = 0, n = 0;
        for (int item = item0; item < n_items && ok; item += step, ++it) {
          if (!tc::mbar_wait(&bar[KFULL], it & 1, abort_flag)) { ok = false; break; }
          for (int rt = rank; rt < row_tiles && ok; rt += C, ++n) {
            const int qs = n % QST;
            if (!tc::mbar_wait(&bar[QFULL + qs], (n / QST) & 1, abort_flag)) { ok = false; break; }
            const int cols = min(BR, p.R - rt * BR) * p.g;
            const uint32_t idesc = tc::idesc_f16(fmt, BK, (cols + 63) / 64 * 64, 0);      // whole chunks: rows of zeros behind the last
            const uint32_t q_addr = tc::smem_u32(smem + OFF_Q + qs * QTILE<HD>);
            for (int w = 0; w < 2; ++w) {
              if (!tc::mbar_wait(&bar[SEMPTY + w], (n & 1) ^ 1, abort_flag)) { ok = false; break; }
              tc::fence_after_sync();
              const uint32_t k_addr = tc::smem_u32(smem + w * KTILE<HD>);
#pragma unroll
              for (int k = 0; k < HD / 16; ++k)
                tc::mma_f16(tmem_base + w * BQ, tc::smem_desc_k_sw128(k_addr + (k >> 2) * M_SLAB + (k & 3) * 32),
                            tc::smem_desc_k_sw128(q_addr + (k >> 2) * Q_SLAB + (k & 3) * 32), idesc, k != 0);
              tc::mma_commit(&bar[SFULL + w]);
            }
            if (ok) tc::mma_commit(&bar[QEMPTY + qs]);
          }
          if (ok) tc::mma_commit(&bar[KEMPTY]);
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
      for (int item = item0; item < n_items && ok; item += step) {
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
          if (!tc::mbar_wait(&bar[CEMPTY + cb], ((n >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
          bool masked[2] = {false, false};
#pragma unroll
          for (int x = 0; x < CPL; ++x) {
            const int i = x * 64 + half * 32 + lane;
            const bool real = r_in[x] < BR && rt * BR + r_in[x] < p.R;
            lo[x] = max(lo[x], 0);
            hi[x] = min(hi[x], p.T - 1);
            const bool blind = !real || z[x] == -INFINITY || lo[x] > hi[x];     // such a row adds nothing
            // a column of zeros behind the last row asks for no mask (add_columns)
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
          if (lane == 0) tc::mbar_arrive(&bar[CFULL + cb]);
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
    for (int item = item0; item < n_items && ok; item += step) {
      const int h = item / key_items, key = (item % key_items) * (2 * BK) + w * BK + m;
      float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int rt = rank; rt < row_tiles; rt += C, ++n) {
        const int cb = n & 1;
        const int all_cols = min(BR, p.R - rt * BR) * p.g;
        if (!tc::mbar_wait(&bar[CFULL + cb], (n >> 1) & 1, abort_flag)) { ok = false; break; }
        const bool mask = (flag[(cb * 2 + w) * 2] | flag[(cb * 2 + w) * 2 + 1]) != 0;
        if (!tc::mbar_wait(&bar[SFULL + w], n & 1, abort_flag)) { ok = false; break; }
        tc::fence_after_sync();
        // 64 columns at a time, the next ones on their way from tensor memory meanwhile
        const uint32_t s_addr = lane_addr + w * BQ;
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
            if (lane == 0) tc::mbar_arrive(&bar[SEMPTY + w]);
          }
        };
        auto add = [&](const float(&t)[64], int c) {
          add_columns<64>(t, col_z + cb * BQ + c * 64, col_rng + cb * BQ + c * 64, mask, key, scale2, acc);
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
        if (lane == 0) tc::mbar_arrive(&bar[CEMPTY + cb]);
      }
      if (!ok) break;
      const float sum = total(acc);
      const int64_t at = (int64_t)h * p.T + key;
      if (C == 1) {
        if (key < p.T) p.mass_out[at] = (p.mass_in ? p.mass_in[at] : 0.f) + sum;
      } else {
        part[w * 128 + m] = sum;
      }
    }
    if (!ok) {                                            // a wait ran out: NaN rather than masses that lack terms
      *abort_flag = 1;
      part[w * 128 + m] = NAN;
      for (int item = item0; item < n_items && C == 1; item += step) {
        const int key = (item % key_items) * (2 * BK) + w * BK + m;
        if (key < p.T) p.mass_out[(int64_t)(item / key_items) * p.T + key] = NAN;
      }
    }
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
}  // namespace many

template <typename T, int HD>
int32_t run_tc(const MassParams& p, cudaStream_t st) {
  static std::atomic<uint64_t> few_set{0}, many_set{0};
  AKVS_CUDA(smem_opt_in((const void*)few::mass_few_kernel<T, HD>, few::SMEM<HD>, few_set));
  AKVS_CUDA(smem_opt_in((const void*)many::mass_many_kernel<T, HD>, many::SMEM<HD>, many_set));
  const uint32_t fmt = std::is_same<T, f16>::value ? tc::kF16 : tc::kBF16;
  const bool rows = p.R > 0, is_few = (int64_t)p.R * p.g <= few::BQ;
  const int key_items = akvs_cdiv(p.T, 2 * BK);
  const int64_t n_items = (int64_t)key_items * p.n_kv;
  if (n_items > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  // rows of a tile: one or two boxes, whose rows fill whole groups of 8 (a swizzle atom) where there are two
  int box_rows = 128 / p.g, boxes = 1;
  if (!is_few) {
    int b = box_rows;
    while (b > 1 && b * p.g % 8) --b;
    if (b * p.g % 8 == 0) { box_rows = b; boxes = 2; }
  }
  const Cols cols = {box_rows * boxes, p.g};
  CUtensorMap tmK, tmQ;
  AKVS_TRY(make_tmap_2d_16bit(&tmK, p.k, p.T, (uint64_t)p.n_kv * HD, (uint64_t)p.k_ld, BK));
  // without rows there is no tile to load either; the map only has to be well formed
  AKVS_TRY(encode_tmap_3d_16bit(&tmQ, rows ? p.q : p.k, HD, rows ? p.n_q : p.n_kv, rows ? p.R : p.T, HD, rows ? p.q_ld : p.k_ld,
                                p.g, box_rows));
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(M_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  if (is_few) {
    cfg.gridDim = dim3((unsigned)(n_items < 148 ? n_items : 148));
    cfg.dynamicSmemBytes = few::SMEM<HD>;
    cfg.numAttrs = 1;
    AKVS_CUDA(cudaLaunchKernelEx(&cfg, few::mass_few_kernel<T, HD>, tmK, tmQ, p, cols, key_items, (int)n_items, fmt));
  } else {
    const int row_tiles = akvs_cdiv(p.R, cols.BR);
    int C = 1;
    while (C < 8 && n_items * C * 2 <= 148 && row_tiles >= C * 4) C *= 2;
    cfg.gridDim = dim3((unsigned)(C > 1 ? n_items * C : n_items < 148 ? n_items : 148));
    cfg.dynamicSmemBytes = many::SMEM<HD>;
    attr[1].val.clusterDim.x = C;
    cfg.numAttrs = 2;
    AKVS_CUDA(cudaLaunchKernelEx(&cfg, many::mass_many_kernel<T, HD>, tmK, tmQ, p, C, key_items, (int)n_items, cols.BR, boxes, fmt));
  }
  AKVS_LAUNCHED();
  return AKVS_OK;
}

// ---- CUDA cores (float): 64 keys per CTA, the stacked rows SR at a time, SR/16 x 4 scores per thread.
// 64 rows a tile are bound by the products (64 rows x 16 heads over 20000 keys: 189 us, 28 TFLOP/s); up to
// 16 rows take small tiles, which leave room for more CTAs on an SM to read K.  Few keys and many rows: a
// cluster shares the row tiles and adds its sums through distributed shared memory.
constexpr int SK = 64, S_THREADS = 256;

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

template <typename T, int HD, int SR>
__global__ void __launch_bounds__(S_THREADS)
mass_simt_kernel(const __grid_constant__ MassParams p, int C) {
  constexpr int LD = HD + 4, V = VecOf<T>::N, CH = HD / V, RPT = SR / 16;
  extern __shared__ __align__(16) float sm[];
  float* kt = sm;                    // [SK][LD]
  float* qt = kt + SK * LD;          // [SR][LD]
  __shared__ float row_lse[SR];
  __shared__ int row_lo[SR], row_hi[SR];
  __shared__ float part[16][SK];
  pdl_trigger();
  pdl_wait();
  const int rank = blockIdx.x % C, h = blockIdx.y, j0 = blockIdx.x / C * SK, tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rows = p.R * p.g;
  for (int i = tid; i < SK * CH; i += S_THREADS) {
    const int j = i / CH, c = i % CH * V;
    load_row_chunk<T, HD>(kt + j * LD + c, (const T*)p.k + (int64_t)min(j0 + j, p.T - 1) * p.k_ld + (int64_t)h * HD + c, j0 + j < p.T);
  }
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int m0 = rank * SR; m0 < rows; m0 += C * SR) {
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
    float s[RPT][4];
#pragma unroll
    for (int a = 0; a < RPT; ++a)
#pragma unroll
      for (int b = 0; b < 4; ++b) s[a][b] = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD; c += 4) {
      float4 x[RPT], y[4];
#pragma unroll
      for (int a = 0; a < RPT; ++a) x[a] = *reinterpret_cast<const float4*>(qt + (ty * RPT + a) * LD + c);
#pragma unroll
      for (int b = 0; b < 4; ++b) y[b] = *reinterpret_cast<const float4*>(kt + (tx + 16 * b) * LD + c);
#pragma unroll
      for (int a = 0; a < RPT; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          s[a][b] = fmaf(x[a].x, y[b].x, fmaf(x[a].y, y[b].y, fmaf(x[a].z, y[b].z, fmaf(x[a].w, y[b].w, s[a][b]))));
    }
#pragma unroll
    for (int a = 0; a < RPT; ++a) {
      const int m = ty * RPT + a, lo = row_lo[m], hi = row_hi[m];
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
  __shared__ float tot[SK];
  if (tid < SK) {
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < 16; ++y) s += part[y][tid];
    tot[tid] = s;
  }
  if (C > 1) tc::cluster_sync_all();
  if (rank == 0 && tid < SK && j0 + tid < p.T) {
    float s = tot[tid];
    for (int c = 1; c < C; ++c) {
      float x;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(tc::map_to_rank(tc::smem_u32(&tot[tid]), c)) : "memory");
      s += x;
    }
    const int64_t at = (int64_t)h * p.T + j0 + tid;
    p.mass_out[at] = (p.mass_in ? p.mass_in[at] : 0.f) + s;
  }
  if (C > 1) tc::cluster_sync_all();
}

template <typename T, int HD, int SR>
int32_t run_simt(const MassParams& p, cudaStream_t st) {
  constexpr int smem = (SK + SR) * (HD + 4) * 4;
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)mass_simt_kernel<T, HD, SR>, smem, smem_set));
  const int64_t ctas = (int64_t)akvs_cdiv(p.T, SK) * p.n_kv;
  const int row_tiles = akvs_cdiv((int64_t)p.R * p.g, SR);
  int C = 1;
  while (C < 8 && ctas * C * 2 <= 296 && row_tiles >= C * 2) C *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(akvs_cdiv(p.T, SK) * C), p.n_kv);
  cfg.blockDim = dim3(S_THREADS);
  cfg.dynamicSmemBytes = smem;
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
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, mass_simt_kernel<T, HD, SR>, p, C));
  AKVS_LAUNCHED();
  return AKVS_OK;
}
template <typename T, int HD>
int32_t run_simt(const MassParams& p, cudaStream_t st) {
  return (int64_t)p.R * p.g <= 16 ? run_simt<T, HD, 16>(p, st) : run_simt<T, HD, 64>(p, st);
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
