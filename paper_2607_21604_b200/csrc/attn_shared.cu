// Attention of many sequences over one shared context and their own tokens.
//
// S sequences share the context K/V (P tokens, kept once); each holds its own K/V besides
// (len[s] tokens in a slot of `cap`).  Row i of the n rows of a sequence sees the whole context
// and the first len[s] - (n - 1 - i) of its own tokens:
//     x_j = q . k_j / sqrt(hd),   lse = log sum_j exp(x_j),   out = sum_j exp(x_j - lse) v_j.
// The sum splits over key ranges: a range gives (m, l, O) = (max x, sum exp(x - m),
// sum exp(x - m) v), and ranges join by rescaling to the common maximum.
//
//  1. The context is read once for all rows: the g = n_q / n_kv query heads of all R rows that
//     share a kv head are stacked (row-major: r * g + i), and the key range is split over CTAs;
//     each leaves (m, l, O) of its rows in scratch, in float.
//  2. One cluster per (sequence, kv head) runs the sequence's own tokens, joins them with the
//     context's parts and writes the rows.  The launch overlaps the first (it waits for it only
//     before it reads the parts).
//
// Context, 16-bit types and more than one tile of 16 stacked rows: the tcgen05 attention kernel
// (attn_tc.cu) on 128 stacked rows per CTA, so that K and V are read once for up to 128 of them.
// The rest, and all own tokens, are memory bound with few rows: K and V go from global memory straight into the operand
// registers of mma.sync m16n8k16, whose contraction index may be permuted at will (for Q K^T a
// lane's 16-byte chunk of K and of Q supplies four of its k positions; for P V a lane's chunk
// of V supplies one column of eight tiles), so no shared-memory staging stands between a load
// and its use.  Probabilities enter P V as a 16-bit value and the 16-bit rounding of what it
// lost: with one 16-bit value alone the rounding of P would cost the output as much accuracy
// as its own final rounding.  Scores, maxima, sums and O are float.
#include "tc_common.cuh"
#include <math.h>

namespace {

constexpr int DIR_WARPS = 4, DIR_THREADS = DIR_WARPS * 32;
constexpr int MT = 16;                        // stacked rows of a tile (the M of one mma)
constexpr int MAX_C = 8;                      // portable cluster size
constexpr float NO_MAX = -1.0e30f;            // running maximum before any key: exp2(x - NO_MAX) is never formed for x = -inf rows
constexpr float LN2 = 0.69314718f, LOG2E = 1.4426950408889634f;

struct SharedParams {
  const void* q;
  int64_t q_ld;                               // elements between rows of q
  int R, n_q, n_kv, g;
  const void* pk;
  const void* pv;
  int P;
  int64_t p_ld;
  const void* sk;
  const void* sv;
  int S, cap;
  int64_t s_ld, s_seq;
  const int32_t* s_len;
  const int32_t* q_off;                       // null: row s belongs to sequence s
  void* out;
  float* lse;
  float* part_o;                              // [splits][R * n_q][hd]
  float2* part_ml;                            // [splits][R * n_q] (m in log2 units, l)
  int splits, split_len;
  float scale_log2;                           // log2(e) / sqrt(hd)
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  if constexpr (std::is_same<T, bf16>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<bf16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<f16>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Which stacked rows a tile holds and how many keys each of them sees.
struct Tile {
  int r0, j0, count;                          // first row, first stacked index, stacked rows in all
  int h;                                      // kv head
  int len, n;                                 // own tokens and rows of the sequence (own tokens only)
  __device__ __forceinline__ bool valid(int m) const { return j0 + m < count; }
  __device__ __forceinline__ int row(int m, int g) const { return r0 + (j0 + m) / g; }
  __device__ __forceinline__ int head(int m, int g) const { return h * g + (j0 + m) % g; }
};

// floats between rows of a joined O: 16-byte rows that start in different banks
template <int HD> constexpr int o_ld = HD + 4;

// ---- 16-bit core: keys [start, end) of k/v (rows `ld` apart); row m sees keys below lim(m).
// Leaves O (unnormalised) in raw[16][HD + 4] and (m, l) in cm / cl.
template <typename T, int HD, typename Lim>
__device__ __forceinline__ void core(const SharedParams& p, const Tile& tl, const T* k, const T* v, int64_t ld, int start,
                                     int end, int all_see, const Lim& lim, float* raw, float* cm, float* cl) {
  constexpr int KC = HD / 32, VC = HD / 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  uint32_t qa[2][KC][4];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int m = gr + 8 * s;
    const bool ok = tl.valid(m);
    const T* q = reinterpret_cast<const T*>(p.q) + (ok ? (int64_t)tl.row(m, p.g) * p.q_ld + (int64_t)tl.head(m, p.g) * HD : 0);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const uint4 x = ok ? __ldcg(reinterpret_cast<const uint4*>(q + 32 * c + 8 * t)) : make_uint4(0u, 0u, 0u, 0u);
      qa[s][c][0] = x.x; qa[s][c][1] = x.y; qa[s][c][2] = x.z; qa[s][c][3] = x.w;
    }
  }
  const int limit[2] = {min(lim(gr), end), min(lim(gr + 8), end)};
  float o[VC][8][4];
#pragma unroll
  for (int a = 0; a < VC; ++a)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[a][i][e] = 0.f;
  float mx[2] = {NO_MAX, NO_MAX}, sum[2] = {0.f, 0.f};

  for (int key0 = start + warp * 16; key0 < end; key0 += DIR_WARPS * 16) {
    uint4 kr[2][KC], vr[4][VC];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const T* kp = k + (int64_t)min(key0 + hf * 8 + gr, end - 1) * ld + 8 * t;
#pragma unroll
      for (int c = 0; c < KC; ++c) kr[hf][c] = __ldcg(reinterpret_cast<const uint4*>(kp + 32 * c));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + 2 * t + (i & 1) + (i >> 1) * 8;
      const T* vp = v + (int64_t)min(key, end - 1) * ld + 8 * gr;
      // rows behind the end may hold anything, NaN included, and 0 * NaN is not 0
#pragma unroll
      for (int c = 0; c < VC; ++c)
        vr[i][c] = key < end ? __ldcg(reinterpret_cast<const uint4*>(vp + 64 * c)) : make_uint4(0u, 0u, 0u, 0u);
    }
    float sc[2][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      sc[hf][0] = sc[hf][1] = sc[hf][2] = sc[hf][3] = 0.f;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        mma16816<T>(sc[hf], qa[0][c][0], qa[1][c][0], qa[0][c][1], qa[1][c][1], kr[hf][c].x, kr[hf][c].y);
        mma16816<T>(sc[hf], qa[0][c][2], qa[1][c][2], qa[0][c][3], qa[1][c][3], kr[hf][c].z, kr[hf][c].w);
      }
    }
    const bool every = key0 + 16 <= all_see;        // all rows see all 16 keys
    float pr[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {                   // rows gr and gr + 8
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = key0 + (e >> 1) * 8 + 2 * t + (e & 1);
        const float y = sc[e >> 1][2 * s + (e & 1)] * p.scale_log2;
        x[e] = every || key < limit[s] ? y : -INFINITY;
      }
      float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const float m_new = fmaxf(mx[s], top);
      if (__any_sync(0xFFFFFFFFu, m_new != mx[s])) {
        const float f = ex2(mx[s] - m_new);
        sum[s] *= f;
#pragma unroll
        for (int a = 0; a < VC; ++a)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[a][i][2 * s] *= f;
            o[a][i][2 * s + 1] *= f;
          }
      }
      mx[s] = m_new;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pr[s][e] = ex2(x[e] - m_new);
        sum[s] += pr[s][e];
      }
    }
    if (every || all_see >= end) {
      uint32_t hi[4], lo[4];                        // A operand: (row, keys 2t..), (row + 8, ..), keys + 8
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = i & 1, e = (i >> 1) * 2;
        hi[i] = pack2<T>(pr[s][e], pr[s][e + 1]);
        const float2 h2 = unpack2<T>(hi[i]);
        lo[i] = pack2<T>(pr[s][e] - h2.x, pr[s][e + 1] - h2.y);
      }
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        const uint32_t w[4][4] = {{vr[0][c].x, vr[0][c].y, vr[0][c].z, vr[0][c].w},
                                  {vr[1][c].x, vr[1][c].y, vr[1][c].z, vr[1][c].w},
                                  {vr[2][c].x, vr[2][c].y, vr[2][c].z, vr[2][c].w},
                                  {vr[3][c].x, vr[3][c].y, vr[3][c].z, vr[3][c].w}};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t sel = (i & 1) ? 0x7632u : 0x5410u;
          const uint32_t b0 = __byte_perm(w[0][i >> 1], w[1][i >> 1], sel);
          const uint32_t b1 = __byte_perm(w[2][i >> 1], w[3][i >> 1], sel);
          mma16816<T>(o[c][i], hi[0], hi[1], hi[2], hi[3], b0, b1);
          mma16816<T>(o[c][i], lo[0], lo[1], lo[2], lo[3], b0, b1);
        }
      }
    } else {
      // Keys that some rows see and others do not (a sequence's last rows): a hidden key must not
      // reach a row even if its V is infinite or NaN, so each row adds what it sees by itself.
      for (int kk = 0; kk < 16; ++kk) {
        const int key = key0 + kk;
        if (key >= end) break;
        const int src = (lane & ~3) | ((kk & 7) >> 1);
        const int e = (kk >> 3) * 2 + (kk & 1);
        float pa = e == 0 ? pr[0][0] : e == 1 ? pr[0][1] : e == 2 ? pr[0][2] : pr[0][3];
        float pb = e == 0 ? pr[1][0] : e == 1 ? pr[1][1] : e == 2 ? pr[1][2] : pr[1][3];
        pa = __shfl_sync(0xFFFFFFFFu, pa, src);
        pb = __shfl_sync(0xFFFFFFFFu, pb, src);
        const T* vp = v + (int64_t)key * ld + 16 * t;
#pragma unroll
        for (int c = 0; c < VC; ++c) {
          float x[2][8];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(vp + 64 * c + 8 * b));
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 y = unpack2<T>(ws[i]);
              x[b][2 * i] = y.x;
              x[b][2 * i + 1] = y.y;
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
              if (key < limit[0]) o[c][i][e2] = fmaf(pa, x[e2][i], o[c][i][e2]);
              if (key < limit[1]) o[c][i][2 + e2] = fmaf(pb, x[e2][i], o[c][i][2 + e2]);
            }
        }
      }
    }
  }
  // join the warps
  __shared__ float wm[DIR_WARPS][MT], wl[DIR_WARPS][MT];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    sum[s] += __shfl_xor_sync(0xFFFFFFFFu, sum[s], 1);
    sum[s] += __shfl_xor_sync(0xFFFFFFFFu, sum[s], 2);
    if (t == 0) { wm[warp][gr + 8 * s] = mx[s]; wl[warp][gr + 8 * s] = sum[s]; }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int m = gr + 8 * s;
    float top = wm[0][m];
#pragma unroll
    for (int w = 1; w < DIR_WARPS; ++w) top = fmaxf(top, wm[w][m]);
    const float f = ex2(mx[s] - top);
    float* dst = raw + (warp * MT + m) * o_ld<HD> + 16 * t;
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int i = 0; i < 8; i += 4)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float4*>(dst + 64 * c + 8 * e + i) =
              make_float4(o[c][i][2 * s + e] * f, o[c][i + 1][2 * s + e] * f, o[c][i + 2][2 * s + e] * f, o[c][i + 3][2 * s + e] * f);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < MT * HD / 4; i += DIR_THREADS) {
    float4* at = reinterpret_cast<float4*>(raw + (i / (HD / 4)) * o_ld<HD> + i % (HD / 4) * 4);
    float4 a = *at;
#pragma unroll
    for (int w = 1; w < DIR_WARPS; ++w) {
      const float4 b = *reinterpret_cast<float4*>(reinterpret_cast<float*>(at) + w * MT * o_ld<HD>);
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
    *at = a;
  }
  if (threadIdx.x < MT) {
    const int m = threadIdx.x;
    float top = wm[0][m], l = 0.f;
    for (int w = 1; w < DIR_WARPS; ++w) top = fmaxf(top, wm[w][m]);
    for (int w = 0; w < DIR_WARPS; ++w) l += wl[w][m] * ex2(wm[w][m] - top);
    cm[m] = top;
    cl[m] = l;
  }
  __syncthreads();
}

// ---- float core: the same on the CUDA cores, 32 keys at a time through shared memory.
constexpr int FK = 32;
template <int HD, typename Lim>
__device__ __forceinline__ void core_f32(const SharedParams& p, const Tile& tl, const float* k, const float* v, int64_t ld,
                                         int start, int end, const Lim& lim, float* raw, float* cm, float* cl) {
  constexpr int LD = HD + 4, OC = HD / 32;
  float* kt = raw;                            // [FK][LD]
  float* vt = kt + FK * LD;                   // [FK][LD]
  float* qt = vt + FK * LD;                   // [MT][LD]
  float* pt = qt + MT * LD;                   // [MT][FK + 1]
  const int m = threadIdx.x >> 3, e = threadIdx.x & 7;
  for (int i = threadIdx.x; i < MT * HD / 4; i += DIR_THREADS) {
    const int mm = i / (HD / 4), c = i % (HD / 4) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tl.valid(mm))
      x = __ldcg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + (int64_t)tl.row(mm, p.g) * p.q_ld +
                                                 (int64_t)tl.head(mm, p.g) * HD + c));
    *reinterpret_cast<float4*>(qt + mm * LD + c) = x;
  }
  const int limit = min(lim(m), end);
  float4 o[OC];
#pragma unroll
  for (int c = 0; c < OC; ++c) o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
  float mx = NO_MAX, sum = 0.f;
  for (int key0 = start; key0 < end; key0 += FK) {
    __syncthreads();
    for (int i = threadIdx.x; i < FK * HD / 4; i += DIR_THREADS) {
      const int kk = i / (HD / 4), c = i % (HD / 4) * 4;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
      if (key0 + kk < end) {
        a = __ldcg(reinterpret_cast<const float4*>(k + (int64_t)(key0 + kk) * ld + c));
        b = __ldcg(reinterpret_cast<const float4*>(v + (int64_t)(key0 + kk) * ld + c));
      }
      *reinterpret_cast<float4*>(kt + kk * LD + c) = a;
      *reinterpret_cast<float4*>(vt + kk * LD + c) = b;
    }
    __syncthreads();
    float x[FK / 8];
#pragma unroll
    for (int j = 0; j < FK / 8; ++j) x[j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD; c += 4) {
      const float4 a = *reinterpret_cast<const float4*>(qt + m * LD + c);
#pragma unroll
      for (int j = 0; j < FK / 8; ++j) {
        const float4 b = *reinterpret_cast<const float4*>(kt + (e + 8 * j) * LD + c);
        x[j] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, x[j]))));
      }
    }
    float top = mx;
#pragma unroll
    for (int j = 0; j < FK / 8; ++j) {
      x[j] = key0 + e + 8 * j < limit ? x[j] * p.scale_log2 : -INFINITY;
      top = fmaxf(top, x[j]);
    }
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
    const float f = exp2f(mx - top);
    mx = top;
    sum *= f;
#pragma unroll
    for (int c = 0; c < OC; ++c) { o[c].x *= f; o[c].y *= f; o[c].z *= f; o[c].w *= f; }
#pragma unroll
    for (int j = 0; j < FK / 8; ++j) {
      const float y = exp2f(x[j] - top);
      sum += y;
      pt[m * (FK + 1) + e + 8 * j] = y;
    }
    __syncwarp();                             // a row's eight threads are in one warp
    const int n = min(FK, limit - key0);      // hidden keys are not touched: their V may be NaN
    for (int kk = 0; kk < n; ++kk) {
      const float y = pt[m * (FK + 1) + kk];
#pragma unroll
      for (int c = 0; c < OC; ++c) {
        const float4 b = *reinterpret_cast<const float4*>(vt + kk * LD + 32 * c + 4 * e);
        o[c].x = fmaf(y, b.x, o[c].x); o[c].y = fmaf(y, b.y, o[c].y);
        o[c].z = fmaf(y, b.z, o[c].z); o[c].w = fmaf(y, b.w, o[c].w);
      }
    }
    __syncwarp();
  }
#pragma unroll
  for (int s = 4; s > 0; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
  __syncthreads();                            // the key tile becomes the output tile
#pragma unroll
  for (int c = 0; c < OC; ++c) *reinterpret_cast<float4*>(raw + m * LD + 32 * c + 4 * e) = o[c];
  if (e == 0) { cm[m] = mx; cl[m] = sum; }
  __syncthreads();
}

template <typename T, int HD> constexpr int direct_smem() {
  return std::is_same<T, float>::value ? (2 * FK * (HD + 4) + MT * (HD + 4) + MT * (FK + 1)) * 4
                                       : DIR_WARPS * MT * (HD + 4) * 4;
}

template <typename T, int HD, typename Lim>
__device__ __forceinline__ void run_core(const SharedParams& p, const Tile& tl, const void* k, const void* v, int64_t ld,
                                         int start, int end, int all_see, const Lim& lim, float* raw, float* cm, float* cl) {
  if constexpr (std::is_same<T, float>::value)
    core_f32<HD>(p, tl, (const float*)k, (const float*)v, ld, start, end, lim, raw, cm, cl);
  else
    core<T, HD>(p, tl, (const T*)k, (const T*)v, ld, start, end, all_see, lim, raw, cm, cl);
}

// ---- 1. context: grid (split, kv head, tile of 16 stacked rows)
template <typename T, int HD>
__global__ void __launch_bounds__(DIR_THREADS)
context_direct_kernel(const __grid_constant__ SharedParams p) {
  extern __shared__ __align__(16) float raw[];
  __shared__ float cm[MT], cl[MT];
  pdl_wait();
  pdl_trigger();                              // after the wait: see own_join_kernel
  const int split = blockIdx.x, h = blockIdx.y;
  const Tile tl{0, (int)blockIdx.z * MT, p.R * p.g, h, 0, 0};
  const int start = split * p.split_len, end = min(start + p.split_len, p.P);
  run_core<T, HD>(p, tl, (const T*)p.pk + (int64_t)h * HD, (const T*)p.pv + (int64_t)h * HD, p.p_ld, start, end, end,
                  [&](int) { return end; }, raw, cm, cl);
  const int64_t rows = (int64_t)p.R * p.n_q;
  for (int i = threadIdx.x; i < MT * HD / 4; i += DIR_THREADS) {
    const int m = i / (HD / 4), c = i % (HD / 4) * 4;
    if (tl.valid(m))
      *reinterpret_cast<float4*>(p.part_o + ((int64_t)split * rows + (int64_t)tl.row(m, p.g) * p.n_q + tl.head(m, p.g)) * HD + c) =
          *reinterpret_cast<const float4*>(raw + m * o_ld<HD> + c);
  }
  if (threadIdx.x < MT && tl.valid(threadIdx.x))
    p.part_ml[(int64_t)split * rows + (int64_t)tl.row(threadIdx.x, p.g) * p.n_q + tl.head(threadIdx.x, p.g)] =
        make_float2(cm[threadIdx.x], cl[threadIdx.x]);
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float ld_cluster1(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void add_scaled(float4& a, const float4& b, float f) {
  a.x = fmaf(b.x, f, a.x); a.y = fmaf(b.y, f, a.y); a.z = fmaf(b.z, f, a.z); a.w = fmaf(b.w, f, a.w);
}

// ---- 2. own tokens and the join: cluster of C CTAs per (sequence, kv head), the own tokens split
// over the cluster; CTA c joins the rows m = c mod C of each tile.  grid (S * C, n_kv, tiles in flight)
template <typename T, int HD>
__global__ void __launch_bounds__(DIR_THREADS)
own_join_kernel(const __grid_constant__ SharedParams p, int C) {
  extern __shared__ __align__(16) float raw[];
  __shared__ __align__(16) float cm[MT], cl[MT];
  pdl_trigger();
  const int s = blockIdx.x / C, rank = blockIdx.x % C, h = blockIdx.y;
  // A CTA of this kernel starts once every CTA of the context's kernel has passed its own wait, so
  // q, the own tokens, lengths and offsets (older than that kernel) are complete in L2 and are read
  // there; only the parts, which that kernel writes, need a wait of this one.  Without a context
  // the kernel before is a stranger: wait for it first.
  if (p.splits == 0) pdl_wait();
  int r0 = s, r1 = s + 1;
  if (p.q_off) {
    r0 = min(max(__ldcg(p.q_off + s), 0), p.R);
    r1 = min(max(__ldcg(p.q_off + s + 1), r0), p.R);
  }
  const int n = r1 - r0;
  const int len = p.cap > 0 ? min(max(__ldcg(p.s_len + s), 0), p.cap) : 0;
  const int64_t rows = (int64_t)p.R * p.n_q;
  const T* k = (const T*)p.sk + (int64_t)s * p.s_seq + (int64_t)h * HD;
  const T* v = (const T*)p.sv + (int64_t)s * p.s_seq + (int64_t)h * HD;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int LPR = HD / 4, RPW = 32 / LPR;       // lanes of a row, rows a warp joins at a time
  for (int j0 = blockIdx.z * MT; j0 < n * p.g; j0 += gridDim.z * MT) {
    const Tile tl{r0, j0, n * p.g, h, len, n};
    // row i of the sequence sees len - (n - 1 - i) own tokens: the tile's first row the fewest
    auto lim = [&](int m) { return tl.valid(m) ? len - (n - 1 - (j0 + m) / p.g) : len; };
    const int most = max(0, lim(min(MT, n * p.g - j0) - 1)), fewest = max(0, lim(0));
    const int chunk = (((most + C - 1) / C + 63) / 64) * 64;
    const int start = min(rank * chunk, most), end = min(start + chunk, most);
    run_core<T, HD>(p, tl, k, v, p.s_ld, start, end, min(fewest, end), lim, raw, cm, cl);
    pdl_wait();
    if (C > 1) tc::cluster_sync_all();
    for (int m0 = rank + warp * RPW * C; m0 < MT; m0 += DIR_WARPS * RPW * C) {
      const int m = m0 + (lane / LPR) * C;
      const bool ok = m < MT && tl.valid(m);
      const int c4 = (lane % LPR) * 4;
      const int64_t at = ok ? (int64_t)tl.row(m, p.g) * p.n_q + tl.head(m, p.g) : 0;
      const int mm = ok ? m : 0;
      float top = NO_MAX;
      for (int c = 0; c < C; ++c) top = fmaxf(top, C > 1 ? ld_cluster1(tc::map_to_rank(tc::smem_u32(&cm[mm]), c)) : cm[mm]);
      if (ok)
        for (int i = 0; i < p.splits; ++i) top = fmaxf(top, __ldcg(p.part_ml + i * rows + at).x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
      for (int c = 0; c < C; ++c) {
        if (C > 1) {
          const float f = ex2(ld_cluster1(tc::map_to_rank(tc::smem_u32(&cm[mm]), c)) - top);
          l += f * ld_cluster1(tc::map_to_rank(tc::smem_u32(&cl[mm]), c));
          add_scaled(o, ld_cluster4(tc::map_to_rank(tc::smem_u32(raw + mm * o_ld<HD> + c4), c)), f);
        } else {
          const float f = ex2(cm[mm] - top);
          l += f * cl[mm];
          add_scaled(o, *reinterpret_cast<const float4*>(raw + mm * o_ld<HD> + c4), f);
        }
      }
      if (ok) {
#pragma unroll 4
        for (int i = 0; i < p.splits; ++i) {
          const float2 ml = __ldcg(p.part_ml + i * rows + at);
          const float f = ex2(ml.x - top);
          l = fmaf(f, ml.y, l);
          add_scaled(o, __ldcg(reinterpret_cast<const float4*>(p.part_o + (i * rows + at) * HD + c4)), f);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;          // nothing visible: zeros, lse = -inf
        T* dst = reinterpret_cast<T*>(p.out) + at * HD + c4;
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        } else {
          uint2 w;
          w.x = pack2<T>(o.x * inv, o.y * inv);
          w.y = pack2<T>(o.z * inv, o.w * inv);
          *reinterpret_cast<uint2*>(dst) = w;
        }
        if (c4 == 0) p.lse[at] = l == 0.f ? -INFINITY : (top + log2f(l)) * LN2;
      }
    }
    if (C > 1) tc::cluster_sync_all();              // the tile's parts stay until the cluster has read them
    else __syncthreads();
  }
  pdl_wait();                                       // a CTA without rows, too: the next kernel relies on it
}

struct Plan { bool tc; int splits, split_len; };

// How the context is cut.
Plan plan_context(bool is16, int R, int P, int g, int n_kv, int hd) {
  if (P == 0 || R == 0) return {false, 0, 0};
  if (is16 && (int64_t)R * g > MT) {
    // One CTA per SM.  In units of a key tile: rounds of CTAs times (a CTA's tiles + 6 for its start
    // and end), plus writing and reading the parts at memory speed (a tile takes about 0.7 us).
    const int64_t base = (int64_t)akvs_cdiv(R, 128 / g) * n_kv;
    const int tiles = akvs_cdiv(P, 128);
    const double part = 2.0 * R * g * n_kv * (hd + 2) * 4 / 6.4e6 / 0.7;
    int best = 1;
    double best_cost = 1e300;
    for (int s = 1; s <= tiles && s <= 148; ++s) {
      const double cost = (double)((base * s + 147) / 148) * (akvs_cdiv(tiles, s) + 6) + part * s;
      if (cost < best_cost) { best_cost = cost; best = s; }
    }
    const int len = akvs_cdiv(tiles, best) * 128;
    return {true, akvs_cdiv(P, len), len};
  }
  // A CTA runs 64 keys at a time; two CTAs fit an SM.
  const int64_t base = (int64_t)n_kv * akvs_cdiv((int64_t)R * g, MT);
  int splits = (int)(base >= 296 ? 1 : akvs_cdiv(296, base));
  const int most = akvs_cdiv(P, 128);
  if (splits > most) splits = most;
  const int len = akvs_cdiv(akvs_cdiv(P, splits), 64) * 64;
  return {false, akvs_cdiv(P, len), len};
}

int64_t parts_bytes(int splits, int R, int n_q, int hd) {
  const int64_t rows = (int64_t)splits * R * n_q;
  return akvs_align_up(rows * hd * 4, 256) + akvs_align_up(rows * 8, 256) + 256;
}

template <typename T, int HD>
int32_t run(SharedParams& p, int dtype, bool tc, cudaStream_t st) {
  constexpr int smem = direct_smem<T, HD>();
  static_assert(smem <= 48 * 1024, "the direct kernels stay below the size that needs an attribute");
  if (p.splits > 0 && tc) {
    AKVS_TRY(launch_attention_parts_tc(dtype, HD, p.q, p.q_ld, p.pk, p.pv, p.p_ld, p.R, p.P, p.n_q, p.n_kv, p.split_len,
                                       p.part_o, p.part_ml, st));
  } else if (p.splits > 0) {
    const int64_t tiles = akvs_cdiv((int64_t)p.R * p.g, MT);
    if (tiles > 65535) return AKVS_ERR_TOO_LARGE;
    AKVS_CUDA(launch_pdl(context_direct_kernel<T, HD>, dim3(p.splits, p.n_kv, (unsigned)tiles), dim3(DIR_THREADS), smem, st, p));
    AKVS_LAUNCHED();
  }
  if (p.S == 0) return AKVS_OK;
  // Tiles in flight per sequence: one is all there is for a row per sequence and up to 16 heads per
  // kv head; ragged batches get room for twice the mean, and a CTA walks what is left.
  const int z = p.q_off ? (int)min((int64_t)64, ((int64_t)akvs_cdiv(p.R, p.S) * p.g * 2 + MT - 1) / MT) : akvs_cdiv(p.g, MT);
  // Few sequences with long slots: a cluster shares the own tokens of one (256 keys or more each).
  int C = 1;
  while (C < MAX_C && (int64_t)p.S * p.n_kv * z * C * 2 <= 296 && p.cap / (C * 2) >= 256) C *= 2;
  if (C == 1 && (int64_t)p.S * p.n_kv * z * 4 <= 148 && p.splits > 8) C = 4;   // the join alone is worth four SMs
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.S * C), p.n_kv, z < 1 ? 1 : z);
  cfg.blockDim = dim3(DIR_THREADS);
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
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, own_join_kernel<T, HD>, p, C));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

bool heads_ok(int32_t n_q, int32_t n_kv) { return n_kv > 0 && n_q > 0 && n_q % n_kv == 0 && n_q / n_kv <= 128 && n_kv <= 65535; }

}  // namespace

extern "C" int64_t akvs_op_attention_shared_scratch_bytes(int32_t R, int32_t P, int32_t n_q_heads, int32_t n_kv_heads,
                                                          int32_t head_dim) {
  if (R < 0 || P < 0 || !heads_ok(n_q_heads, n_kv_heads) || (head_dim != 64 && head_dim != 128)) return -1;
  const int g = n_q_heads / n_kv_heads;       // the larger of the two ways the types take
  const int a = plan_context(true, R, P, g, n_kv_heads, head_dim).splits, b = plan_context(false, R, P, g, n_kv_heads, head_dim).splits;
  return parts_bytes(a > b ? a : b, R, n_q_heads, head_dim);
}

extern "C" int32_t akvs_op_attention_shared(int32_t dtype, const void* q, int64_t q_ld, int32_t R, const void* ctx_k,
                                            const void* ctx_v, int64_t ctx_ld, int32_t P, const void* own_k,
                                            const void* own_v, int64_t own_ld, int64_t own_seq_ld, int32_t S, int32_t cap,
                                            const int32_t* own_len, const int32_t* q_off, int32_t n_q_heads,
                                            int32_t n_kv_heads, int32_t head_dim, void* out, float* lse, void* scratch,
                                            int64_t scratch_size, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (R < 0 || P < 0 || S < 0 || cap < 0) return AKVS_ERR_INVALID_ARG;
  if (!heads_ok(n_q_heads, n_kv_heads)) return AKVS_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return AKVS_ERR_UNSUPPORTED;
  if (!q_off && R < S) return AKVS_ERR_SHAPE;
  if (R == 0 || S == 0) return AKVS_OK;
  const int64_t es = (int64_t)dtype_size(dtype), row = (int64_t)n_kv_heads * head_dim, q_row = (int64_t)n_q_heads * head_dim;
  if (!q || !out || !lse || (P > 0 && (!ctx_k || !ctx_v)) || (cap > 0 && (!own_k || !own_v || !own_len)))
    return AKVS_ERR_INVALID_ARG;
  if (q_ld < q_row || (P > 0 && ctx_ld < row) || (cap > 0 && (own_ld < row || own_seq_ld < 0))) return AKVS_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(out) || q_ld * es % 16 || (P > 0 && (!aligned16(ctx_k) || !aligned16(ctx_v) || ctx_ld * es % 16)) ||
      (cap > 0 && (!aligned16(own_k) || !aligned16(own_v) || own_ld * es % 16 || own_seq_ld * es % 16)))
    return AKVS_ERR_INVALID_ARG;
  if ((int64_t)R * n_q_heads > 0x7fffffff || (int64_t)S * MAX_C > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  const Plan pl = plan_context(dtype != AKVS_F32, R, P, n_q_heads / n_kv_heads, n_kv_heads, head_dim);
  const int64_t need = parts_bytes(pl.splits, R, n_q_heads, head_dim);
  if (pl.splits > 0 && (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || scratch_size < need)) return AKVS_ERR_WORKSPACE;
  const int64_t ctx_n = P > 0 ? ((P - 1) * ctx_ld + row) * es : 0;
  const int64_t own_n = cap > 0 ? ((S - 1) * own_seq_ld + (cap - 1) * own_ld + row) * es : 0;
  const void* ins[7] = {q, ctx_k, ctx_v, own_k, own_v, own_len, q_off};
  const int64_t in_n[7] = {((R - 1) * q_ld + q_row) * es, ctx_n, ctx_n, own_n, own_n, cap > 0 ? S * 4ll : 0, q_off ? (S + 1) * 4ll : 0};
  const void* outs[3] = {out, lse, scratch};
  const int64_t out_n[3] = {R * q_row * es, (int64_t)R * n_q_heads * 4, pl.splits > 0 ? need : 0};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 7; ++i)
      if (bytes_overlap(ins[i], in_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
    for (int i = 0; i < o; ++i)
      if (bytes_overlap(outs[i], out_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
  }
  SharedParams p;
  p.q = q; p.q_ld = q_ld; p.R = R; p.n_q = n_q_heads; p.n_kv = n_kv_heads; p.g = n_q_heads / n_kv_heads;
  p.pk = ctx_k; p.pv = ctx_v; p.P = P; p.p_ld = ctx_ld;
  p.sk = own_k; p.sv = own_v; p.S = S; p.cap = cap; p.s_ld = own_ld; p.s_seq = own_seq_ld; p.s_len = own_len; p.q_off = q_off;
  p.out = out; p.lse = lse;
  p.splits = pl.splits; p.split_len = pl.split_len;
  const int64_t rows = (int64_t)pl.splits * R * n_q_heads;
  p.part_o = reinterpret_cast<float*>(scratch);
  p.part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(scratch) + akvs_align_up(rows * head_dim * 4, 256));
  p.scale_log2 = LOG2E / sqrtf((float)head_dim);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    return head_dim == 64 ? run<T, 64>(p, dtype, pl.tc, st) : run<T, 128>(p, dtype, pl.tc, st);
  });
}
