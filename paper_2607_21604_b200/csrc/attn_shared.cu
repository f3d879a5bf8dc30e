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
//  2. A sequence's own tokens give further parts of the same form.  This launch needs nothing of
//     the first and runs beside it, on SMs that it leaves idle.
//  3. The parts of a row are joined and the row is written.
//
// Context, 16-bit types and more than 16 stacked rows: the tcgen05 attention kernel (attn_tc.cu) on
// 128 stacked rows per CTA, so that K and V are read once for up to 128 of them.  The rest, and all
// own tokens, are memory bound with few rows, on mma.sync m16n8k16 with the ROWS along N, so that 4
// or 5 heads fill most of a tile (with the rows along M twice as many products were issued, and
// their rate, not the memory's, bounded the kernel):
//     S^T = K Q^T      16 keys x 8 rows, 8 products for head_dim 128
//     O^T += V^T P^T   16 columns x 8 rows x 16 keys, P^T turned by movmatrix
// A warp keeps a tile of 8 or 16 stacked rows and streams keys through a cp.async ring of its own (16
// keys a stage, two stages in flight).  The contraction index of S^T and the columns of O^T may be
// permuted at will, so fragments are plain 16-byte loads: a lane's chunk of K and of Q supplies four
// of its k positions, and its chunks of four V rows, paired by byte permutes, eight columns.
// In these tiles probabilities enter P V as a 16-bit value and the 16-bit rounding of what it lost: with
// one 16-bit value alone, as in the tcgen05 kernel (which explains it), the rounding of P costs the output
// as much accuracy as its own final rounding.  Scores, maxima, sums and O are float.
#include "tc_common.cuh"
#include <float.h>
#include <math.h>

namespace {

constexpr int DIR_WARPS = 4, DIR_THREADS = DIR_WARPS * 32;
constexpr int MT = 16;                        // stacked rows of the largest tile
constexpr int ST = 3;                         // stages of a warp's ring, 16 keys each
constexpr int MAX_OWN_SPLITS = 64;
constexpr float NO_MAX = -FLT_MAX;            // running maximum before any key: below every finite score (in log2
                                              // units they are products with less than 0.2), and exp2(-inf - NO_MAX) = 0
// How far below the largest score the reference of the exponentials is, in log2 units: float16 ends at
// 2^-24, and with 2^7 for the largest weight all weights are held to 2^-32 of it (without, 30000 keys of
// 2^-26 beside one of 1 lost a quarter of what they add to the output).
template <typename T> constexpr float BELOW = std::is_same<T, f16>::value ? 7.f : 0.f;
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
  float* part_o;                              // [splits + own_splits][R * n_q][hd]
  float2* part_ml;                            // [splits + own_splits][R * n_q] (m in log2 units, l)
  int splits, split_len;                      // of the context
  int own_splits;                             // of every sequence's own tokens
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
// Two values of a row of the output.  float16 saturates where rounded weights carry a mean of the largest V
// past the type's end, but an infinity stays one (pack2 alone would make it the largest finite value).
template <typename T> __device__ __forceinline__ uint32_t round2(float a, float b) { return pack2<T>(a, b); }
template <> __device__ __forceinline__ uint32_t round2<f16>(float a, float b) {
  auto end = [](float x) { return fabsf(x) > 65504.f && fabsf(x) < INFINITY ? copysignf(65504.f, x) : x; };
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(end(b)), "f"(end(a)));
  return r;
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<bf16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<f16>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Which stacked rows a tile holds.
struct Tile {
  int r0, j0, count, h;                       // first row, first stacked index, stacked rows in all, kv head
  __device__ __forceinline__ bool valid(int m) const { return j0 + m < count; }
  __device__ __forceinline__ int row(int m, int g) const { return r0 + (j0 + m) / g; }
  __device__ __forceinline__ int head(int m, int g) const { return h * g + (j0 + m) % g; }
};

// ---- 16-bit types: what a warp keeps of its tile while keys pass by.
template <int HD> constexpr int STAGE = 16 * HD * 4;       // bytes: 16 rows of K, 16 rows of V
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
// Copies chunk c of row `row` (of 16) of K and V into a stage.  Places are exchanged so that the eight
// lanes of a shared-memory phase hit different banks: a K read takes 4 chunks of two neighbouring
// rows, a V read 2 chunks of four even rows.  Rows behind the end may hold anything, NaN included,
// and 0 * NaN is not 0: they arrive as zeros.
template <typename T, int HD>
__device__ __forceinline__ void copy_chunk(uint32_t stage, const T* k, const T* v, int64_t ld, int key, int end, int row, int c) {
  constexpr int CH = HD / 8;
  const bool ok = key < end;
  const int64_t at = (int64_t)(ok ? key : end - 1) * ld + c * 8;
  cp16(stage + (row * CH + (c ^ ((row & 1) << 2))) * 16, k + at, ok);
  cp16(stage + STAGE<HD> / 2 + (row * CH + (c ^ (row & 6))) * 16, v + at, ok);
}

// P^T of 8 keys x 8 rows from the layout of S^T (a key per lane group) to that of an operand (a row per
// lane group).
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// NT: 8 NT stacked rows.  Lane = 4 gr + t.
template <typename T, int HD, int NT>
struct WarpTile {
  static constexpr int KC = HD / 32, VC = HD / 64, CH = HD / 8;
  uint32_t qb[NT][KC][4];                     // row 8 x + gr, chunk 4 c + t
  int limit[NT][2];                           // rows 8 x + 2 t + e see the keys below these
  float o[NT][VC][4][4];                      // row 8 x + 2 t + e, column 64 c + 8 gr + 2 i + s at [x][c][i][2 s + e]
  float mx[NT][2], sum[NT][2];                // reference of the exponentials (the largest score less BELOW), their sum

  template <typename Lim>
  __device__ __forceinline__ void begin(const SharedParams& p, const Tile& tl, int end, const Lim& lim) {
    const int lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int m = 8 * x + gr;
      const bool ok = tl.valid(m);
      const T* q = reinterpret_cast<const T*>(p.q) + (ok ? (int64_t)tl.row(m, p.g) * p.q_ld + (int64_t)tl.head(m, p.g) * HD : 0);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const uint4 w = ok ? __ldcg(reinterpret_cast<const uint4*>(q + 32 * c + 8 * t)) : make_uint4(0u, 0u, 0u, 0u);
        qb[x][c][0] = w.x; qb[x][c][1] = w.y; qb[x][c][2] = w.z; qb[x][c][3] = w.w;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        limit[x][e] = min(lim(8 * x + 2 * t + e), end);
        mx[x][e] = NO_MAX;
        sum[x][e] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x][c][i][e] = 0.f;
    }
  }

  // 16 keys from key0, staged at `ks`; no key from `end` on exists, all rows see those below all_see.
  __device__ __forceinline__ void step(uint32_t ks, int key0, int end, int all_see, float scale_log2) {
    const int lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
    const uint32_t vs = ks + STAGE<HD> / 2;
    float pr[NT][4];                                // [2 half + e]: key 8 half + gr, row 2 t + e
#pragma unroll
    for (int x = 0; x < NT; ++x) pr[x][0] = pr[x][1] = pr[x][2] = pr[x][3] = 0.f;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int at = ((4 * c + t) ^ ((gr & 1) << 2)) * 16;      // rows gr and gr + 8 exchange alike
      const uint4 a = lds16(ks + gr * CH * 16 + at), b = lds16(ks + (gr + 8) * CH * 16 + at);
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        mma16816<T>(pr[x], a.x, b.x, a.y, b.y, qb[x][c][0], qb[x][c][1]);
        mma16816<T>(pr[x], a.z, b.z, a.w, b.w, qb[x][c][2], qb[x][c][3]);
      }
    }
    const bool every = key0 + 16 <= all_see;        // all rows see all 16 keys
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      float m_new[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float y = __fmul_rn(pr[x][2 * hf + e], scale_log2);      // not fused with the subtraction below: both round alike
          pr[x][2 * hf + e] = every || key0 + 8 * hf + gr < limit[x][e] ? y : -INFINITY;
        }
        float top = fmaxf(pr[x][e], pr[x][2 + e]);
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
        m_new[e] = fmaxf(mx[x][e], top - BELOW<T>);
      }
      if (__any_sync(0xFFFFFFFFu, m_new[0] != mx[x][0] || m_new[1] != mx[x][1])) {
        const float f[2] = {ex2(mx[x][0] - m_new[0]), ex2(mx[x][1] - m_new[1])};
        sum[x][0] *= f[0];
        sum[x][1] *= f[1];
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][c][i][e] *= f[e & 1];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[x][e] = m_new[e];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          pr[x][2 * hf + e] = ex2(pr[x][2 * hf + e] - m_new[e]);
          sum[x][e] += pr[x][2 * hf + e];
        }
      }
    }
    if (every || all_see >= end) {
      uint32_t hi[NT][2], lo[NT][2];                // B operand: keys 2 t, 2 t + 1 (and + 8) of row gr
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const uint32_t h = pack2<T>(pr[x][2 * hf], pr[x][2 * hf + 1]);
          const float2 h2 = unpack2<T>(h);
          hi[x][hf] = turn8x8(h);
          lo[x][hf] = turn8x8(pack2<T>(pr[x][2 * hf] - h2.x, pr[x][2 * hf + 1] - h2.y));
        }
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        uint32_t w[4][4];                           // rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9; columns 64 c + 8 gr ..
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 2 * t + (i & 1) + (i >> 1) * 8;
          const uint4 v = lds16(vs + (row * CH + ((8 * c + gr) ^ (row & 6))) * 16);
          w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a0 = __byte_perm(w[0][i], w[1][i], 0x5410u), a1 = __byte_perm(w[0][i], w[1][i], 0x7632u);
          const uint32_t a2 = __byte_perm(w[2][i], w[3][i], 0x5410u), a3 = __byte_perm(w[2][i], w[3][i], 0x7632u);
#pragma unroll
          for (int x = 0; x < NT; ++x) {
            mma16816<T>(o[x][c][i], a0, a1, a2, a3, hi[x][0], hi[x][1]);
            mma16816<T>(o[x][c][i], a0, a1, a2, a3, lo[x][0], lo[x][1]);
          }
        }
      }
    } else {
      // Keys that some rows see and others do not (a sequence's last rows): a hidden key must not
      // reach a row even if its V is infinite or NaN, so each row adds what it sees by itself.
      for (int kk = 0; kk < 16; ++kk) {
        const int key = key0 + kk;
        if (key >= end) break;
        float v[VC][8];
#pragma unroll
        for (int c = 0; c < VC; ++c) {
          const uint4 w = lds16(vs + (kk * CH + ((8 * c + gr) ^ (kk & 6))) * 16);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 y = unpack2<T>(ws[i]);
            v[c][2 * i] = y.x;
            v[c][2 * i + 1] = y.y;
          }
        }
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float y = __shfl_sync(0xFFFFFFFFu, kk < 8 ? pr[x][e] : pr[x][2 + e], (kk & 7) * 4 + t);
            if (key < limit[x][e])
#pragma unroll
              for (int c = 0; c < VC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) o[x][c][i >> 1][2 * (i & 1) + e] = fmaf(y, v[c][i], o[x][c][i >> 1][2 * (i & 1) + e]);
          }
      }
    }
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sum[x][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[x][e], 4);
        sum[x][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[x][e], 8);
        sum[x][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[x][e], 16);
      }
  }

  // columns 64 c + 8 gr + 4 half .. of row 8 x + 2 t + e
  __device__ __forceinline__ float4 quad(int x, int e, int c, int half, float f) const {
    return make_float4(o[x][c][2 * half][e] * f, o[x][c][2 * half][2 + e] * f, o[x][c][2 * half + 1][e] * f,
                       o[x][c][2 * half + 1][2 + e] * f);
  }
};

// A warp alone: keys start, start + step, ... (16 at a time) below `end`, through its own ring.
template <typename T, int HD, int NT, typename Lim>
__device__ __forceinline__ void warp_core(const SharedParams& p, const Tile& tl, const T* k, const T* v, int64_t ld, int start,
                                          int end, int step, int all_see, const Lim& lim, uint32_t ring, WarpTile<T, HD, NT>& wt) {
  constexpr int CH = HD / 8;
  const int lane = threadIdx.x & 31;
  auto issue = [&](int n) {
    const int key0 = start + n * step;
    if (key0 < end) {
#pragma unroll
      for (int i = 0; i < 16 * CH / 32; ++i) {
        const int row = (i * 32 + lane) / CH, c = (i * 32 + lane) % CH;
        copy_chunk<T, HD>(ring + (n % ST) * STAGE<HD>, k, v, ld, key0 + row, end, row, c);
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int n = 0; n < ST - 1; ++n) issue(n);
  wt.begin(p, tl, end, lim);
  int n = 0;
  for (int key0 = start; key0 < end; key0 += step, ++n) {
    cp_wait<ST - 2>();
    __syncwarp();                             // every lane's copies are there, and the stage before is read
    issue(n + ST - 1);
    wt.step(ring + (n % ST) * STAGE<HD>, key0, end, all_see, p.scale_log2);
  }
  cp_wait<0>();
  wt.finish();
}

// Row m's part into scratch, from a row of O in shared memory.
template <int HD>
__device__ __forceinline__ void store_part(const SharedParams& p, const Tile& tl, int part, int m, int c4, float4 o) {
  const int64_t row = (int64_t)part * p.R * p.n_q + (int64_t)tl.row(m, p.g) * p.n_q + tl.head(m, p.g);
  *reinterpret_cast<float4*>(p.part_o + row * HD + c4) = o;
}
__device__ __forceinline__ void store_ml(const SharedParams& p, const Tile& tl, int part, int m, float mx, float l) {
  p.part_ml[(int64_t)part * p.R * p.n_q + (int64_t)tl.row(m, p.g) * p.n_q + tl.head(m, p.g)] = make_float2(mx, l);
}

// A warp's whole tile into scratch, from its registers.
template <typename T, int HD, int NT>
__device__ __forceinline__ void store_tile(const SharedParams& p, const Tile& tl, int part, const WarpTile<T, HD, NT>& wt) {
  const int lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int m = 8 * x + 2 * t + e;
      if (!tl.valid(m)) continue;
#pragma unroll
      for (int c = 0; c < HD / 64; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half) store_part<HD>(p, tl, part, m, 64 * c + 8 * gr + 4 * half, wt.quad(x, e, c, half, 1.f));
      if (gr == 0) store_ml(p, tl, part, m, wt.mx[x][e], wt.sum[x][e]);
    }
}

// One tile, the CTA's warps taking turns over its keys; joins them and leaves the part in scratch.
template <typename T, int HD, int NT, typename Lim>
__device__ __forceinline__ void cta_part(const SharedParams& p, const Tile& tl, const T* k, const T* v, int64_t ld, int start,
                                         int end, int all_see, const Lim& lim, uint8_t* smem, int part) {
  constexpr int TR = 8 * NT, LD = HD + 4;     // 16-byte rows that start in different banks
  __shared__ float wm[DIR_WARPS][TR], wl[DIR_WARPS][TR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  float* raw = reinterpret_cast<float*>(smem);
  WarpTile<T, HD, NT> acc;
  warp_core<T, HD, NT>(p, tl, k, v, ld, start + warp * 16, end, DIR_WARPS * 16, all_see, lim,
                       tc::smem_u32(smem) + warp * ST * STAGE<HD>, acc);
  if (gr == 0)
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e) { wm[warp][8 * x + 2 * t + e] = acc.mx[x][e]; wl[warp][8 * x + 2 * t + e] = acc.sum[x][e]; }
  __syncthreads();                            // the rings become the warps' rows of O
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int m = 8 * x + 2 * t + e;
      float top = wm[0][m];
#pragma unroll
      for (int w = 1; w < DIR_WARPS; ++w) top = fmaxf(top, wm[w][m]);
      const float f = ex2(acc.mx[x][e] - top);
      float* dst = raw + (warp * TR + m) * LD + 8 * gr;
#pragma unroll
      for (int c = 0; c < HD / 64; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half) *reinterpret_cast<float4*>(dst + 64 * c + 4 * half) = acc.quad(x, e, c, half, f);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < TR * HD / 4; i += DIR_THREADS) {
    const int m = i / (HD / 4), c4 = i % (HD / 4) * 4;
    if (!tl.valid(m)) continue;
    float4 a = *reinterpret_cast<const float4*>(raw + m * LD + c4);
#pragma unroll
    for (int w = 1; w < DIR_WARPS; ++w) {
      const float4 b = *reinterpret_cast<const float4*>(raw + (w * TR + m) * LD + c4);
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
    store_part<HD>(p, tl, part, m, c4, a);
  }
  if (threadIdx.x < TR && tl.valid(threadIdx.x)) {
    const int m = threadIdx.x;
    float top = wm[0][m], l = 0.f;
    for (int w = 1; w < DIR_WARPS; ++w) top = fmaxf(top, wm[w][m]);
    for (int w = 0; w < DIR_WARPS; ++w) l += wl[w][m] * ex2(wm[w][m] - top);
    store_ml(p, tl, part, m, top, l);
  }
  __syncthreads();                            // before another tile reuses the shared memory
}

// ---- float core: 16 stacked rows on the CUDA cores, 64 keys at a time through shared memory.  A thread
// forms 2 x 4 scores, then 4 rows x 4 columns of O: 6 and 2 shared-memory reads of 16 bytes for 32 and 16
// products of 4 (a thread per row with 4 keys, 5 reads for 16 products, took 363 us where this takes
// 145 us: 50 rows x 16 heads over 5000 keys).
constexpr int FK = 64, FP_LD = MT + 4;
template <int HD, typename Lim>
__device__ __forceinline__ void cta_part_f32(const SharedParams& p, const Tile& tl, const float* k, const float* v, int64_t ld,
                                             int start, int end, int all_see, const Lim& lim, uint8_t* smem, int part) {
  constexpr int LD = HD + 4, CH = HD / 4;
  float* kt = reinterpret_cast<float*>(smem); // [FK][LD]
  float* vt = kt + FK * LD;                   // [FK][LD]
  float* qt = vt + FK * LD;                   // [MT][LD]
  float* pt = qt + MT * LD;                   // [FK][FP_LD]: probabilities, a key per row
  float* ft = pt + FK * FP_LD;                // [MT]: what O is rescaled by
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rp = tid >> 4, kq = tid & 15;     // scores of rows 2 rp, 2 rp + 1 and keys kq + 16 j
  const int col = lane % CH * 4, sub = lane / CH;      // O: rows 4 warp .., columns col ..; head_dim 64: the half-warps share the keys
  for (int i = tid; i < MT * CH; i += DIR_THREADS) {
    const int m = i / CH, c = i % CH * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tl.valid(m))
      x = __ldcg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + (int64_t)tl.row(m, p.g) * p.q_ld +
                                                 (int64_t)tl.head(m, p.g) * HD + c));
    *reinterpret_cast<float4*>(qt + m * LD + c) = x;
  }
  int limit[2], o_limit[4];
#pragma unroll
  for (int a = 0; a < 2; ++a) limit[a] = min(lim(2 * rp + a), end);
#pragma unroll
  for (int r = 0; r < 4; ++r) o_limit[r] = min(lim(4 * warp + r), end);
  float4 o[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
  float mx[2] = {NO_MAX, NO_MAX}, sum[2] = {0.f, 0.f};
  for (int key0 = start; key0 < end; key0 += FK) {
    __syncthreads();                          // the tile before is read
    for (int i = tid; i < FK * CH; i += DIR_THREADS) {
      const int kk = i / CH, c = i % CH * 4;
      const bool ok = key0 + kk < end;        // keys behind the end arrive as zeros
      const int64_t at = (int64_t)(ok ? key0 + kk : end - 1) * ld + c;
      cp16(tc::smem_u32(kt + kk * LD + c), k + at, ok);
      cp16(tc::smem_u32(vt + kk * LD + c), v + at, ok);
    }
    cp_commit();
    cp_wait<0>();
    __syncthreads();
    float x[2][4];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[a][j] = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD; c += 4) {
      float4 q[2], y[4];
#pragma unroll
      for (int a = 0; a < 2; ++a) q[a] = *reinterpret_cast<const float4*>(qt + (2 * rp + a) * LD + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(kt + (kq + 16 * j) * LD + c);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[a][j] = fmaf(q[a].x, y[j].x, fmaf(q[a].y, y[j].y, fmaf(q[a].z, y[j].z, fmaf(q[a].w, y[j].w, x[a][j]))));
    }
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      float top = mx[a];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[a][j] = key0 + kq + 16 * j < limit[a] ? __fmul_rn(x[a][j], p.scale_log2) : -INFINITY;
        top = fmaxf(top, x[a][j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, w));
      const float f = exp2f(mx[a] - top);
      mx[a] = top;
      sum[a] *= f;
      if (kq == 0) ft[2 * rp + a] = f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[a][j] = exp2f(x[a][j] - top);
        sum[a] += x[a][j];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(pt + (kq + 16 * j) * FP_LD + 2 * rp) = make_float2(x[0][j], x[1][j]);
    __syncthreads();
    const float4 f4 = *reinterpret_cast<const float4*>(ft + 4 * warp);
    const float fr[4] = {f4.x, f4.y, f4.z, f4.w};
#pragma unroll
    for (int r = 0; r < 4; ++r) { o[r].x *= fr[r]; o[r].y *= fr[r]; o[r].z *= fr[r]; o[r].w *= fr[r]; }
    const bool every = key0 + FK <= all_see || all_see >= end;
    auto add = [&](int kk, bool check) {
      const float4 y4 = *reinterpret_cast<const float4*>(pt + kk * FP_LD + 4 * warp);
      const float4 b = *reinterpret_cast<const float4*>(vt + kk * LD + col);
      const float y[4] = {y4.x, y4.y, y4.z, y4.w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!check || key0 + kk < o_limit[r]) {       // a hidden key's V may be NaN: it is not touched
          o[r].x = fmaf(y[r], b.x, o[r].x); o[r].y = fmaf(y[r], b.y, o[r].y);
          o[r].z = fmaf(y[r], b.z, o[r].z); o[r].w = fmaf(y[r], b.w, o[r].w);
        }
    };
    if (every) {
#pragma unroll 8
      for (int kk = sub; kk < FK; kk += 32 / CH) add(kk, false);
    } else {
      for (int kk = sub; kk < FK; kk += 32 / CH) add(kk, true);
    }
  }
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) sum[a] += __shfl_xor_sync(0xFFFFFFFFu, sum[a], w);
  if constexpr (CH < 32) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      o[r].x += __shfl_xor_sync(0xFFFFFFFFu, o[r].x, CH); o[r].y += __shfl_xor_sync(0xFFFFFFFFu, o[r].y, CH);
      o[r].z += __shfl_xor_sync(0xFFFFFFFFu, o[r].z, CH); o[r].w += __shfl_xor_sync(0xFFFFFFFFu, o[r].w, CH);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (sub == 0 && tl.valid(4 * warp + r)) store_part<HD>(p, tl, part, 4 * warp + r, col, o[r]);
#pragma unroll
  for (int a = 0; a < 2; ++a)
    if (kq == 0 && tl.valid(2 * rp + a)) store_ml(p, tl, part, 2 * rp + a, mx[a], sum[a]);
  __syncthreads();                            // before another tile reuses the shared memory
}

template <typename T, int HD> constexpr int direct_smem() {
  return std::is_same<T, float>::value ? (2 * FK * (HD + 4) + MT * (HD + 4) + FK * FP_LD + MT) * 4 : DIR_WARPS * ST * STAGE<HD>;
}

template <typename T, int HD, int NT, typename Lim>
__device__ __forceinline__ void tile_part(const SharedParams& p, const Tile& tl, const T* k, const T* v, int64_t ld, int start,
                                          int end, int all_see, const Lim& lim, uint8_t* smem, int part) {
  if constexpr (std::is_same<T, float>::value)
    cta_part_f32<HD>(p, tl, k, v, ld, start, end, all_see, lim, smem, part);
  else
    cta_part<T, HD, NT>(p, tl, k, v, ld, start, end, all_see, lim, smem, part);
}

// ---- 1. context, one split of it, for one tile of stacked rows
template <typename T, int HD, int NT>
__device__ __forceinline__ void context_tile(const SharedParams& p, int split, int h, int tile, uint8_t* smem) {
  const Tile tl{0, tile * 8 * NT, p.R * p.g, h};
  const int start = split * p.split_len, end = min(start + p.split_len, p.P);
  tile_part<T, HD, NT>(p, tl, (const T*)p.pk + (int64_t)h * HD, (const T*)p.pv + (int64_t)h * HD, p.p_ld, start, end, end,
                   [&](int) { return end; }, smem, split);
}

// The rows of sequence s and how many of its tokens are filled.
struct Seq { int r0, n, len; };
__device__ __forceinline__ Seq sequence(const SharedParams& p, int s) {
  Seq q;
  int r1 = s + 1;
  q.r0 = s;
  if (p.q_off) {
    q.r0 = min(max(__ldcg(p.q_off + s), 0), p.R);
    r1 = min(max(__ldcg(p.q_off + s + 1), q.r0), p.R);
  }
  q.n = r1 - q.r0;
  q.len = p.cap > 0 ? min(max(__ldcg(p.s_len + s), 0), p.cap) : 0;
  return q;
}

// ---- 2. own tokens of a sequence, one split of them, tile z of nz in flight.
// WIDE (sequences of many rows, one split): every warp has a tile of its own and runs all its keys.
template <typename T, int HD, int NT, bool WIDE>
__device__ __forceinline__ void own_tiles(const SharedParams& p, int s, int split, int h, int z, int nz, uint8_t* smem) {
  const Seq sq = sequence(p, s);
  const T* k = (const T*)p.sk + (int64_t)s * p.s_seq + (int64_t)h * HD;
  const T* v = (const T*)p.sv + (int64_t)s * p.s_seq + (int64_t)h * HD;
  const int count = sq.n * p.g;
  constexpr int TILES = WIDE ? DIR_WARPS : 1, TR = 8 * NT;
  const int warp = threadIdx.x >> 5;
  for (int j0 = (z * TILES + (WIDE ? warp : 0)) * TR; j0 < count; j0 += nz * TILES * TR) {
    const Tile tl{sq.r0, j0, count, h};
    // row i of the sequence sees len - (n - 1 - i) own tokens: the tile's first row the fewest
    auto lim = [&](int m) { return tl.valid(m) ? sq.len - (sq.n - 1 - (j0 + m) / p.g) : sq.len; };
    const int most = max(0, lim(min(TR, count - j0) - 1)), fewest = max(0, lim(0));
    if constexpr (WIDE) {
      WarpTile<T, HD, NT> wt;
      warp_core<T, HD, NT>(p, tl, k, v, p.s_ld, 0, most, 16, min(fewest, most), lim, tc::smem_u32(smem) + warp * ST * STAGE<HD>, wt);
      store_tile<T, HD, NT>(p, tl, p.splits, wt);
      __syncwarp();                           // the ring is read
    } else {
      const int chunk = ((most + p.own_splits - 1) / p.own_splits + 63) / 64 * 64;
      const int start = min(split * chunk, most), end = min(start + chunk, most);
      tile_part<T, HD, NT>(p, tl, k, v, p.s_ld, start, end, min(fewest, end), lim, smem, p.splits + split);
    }
  }
}

// beside the tcgen05 kernel: grid (sequence * own split, kv head, tiles in flight)
template <typename T, int HD, int NT, bool WIDE>
__global__ void __launch_bounds__(DIR_THREADS)
own_kernel(const __grid_constant__ SharedParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  // A CTA of this kernel starts once every CTA of the context's kernel has passed its own wait, so
  // q, the own tokens, lengths and offsets (older than that kernel) are complete in L2 and are read
  // there.
  pdl_trigger();
  own_tiles<T, HD, NT, WIDE>(p, blockIdx.x / p.own_splits, blockIdx.x % p.own_splits, blockIdx.y, blockIdx.z, gridDim.z, smem);
  // The join waits for this grid alone: its last CTA ends after the context's kernel.
  if (blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1 && blockIdx.z == gridDim.z - 1) pdl_wait();
}

// context and own tokens in one launch: the first n_ctx CTAs of a kv head take the context
template <typename T, int HD, int NT, bool WIDE>
__global__ void __launch_bounds__(DIR_THREADS)
direct_kernel(const __grid_constant__ SharedParams p, int n_ctx, int own_z) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_wait();
  pdl_trigger();                              // after the wait: the join reads lengths and offsets without its own
  int x = blockIdx.x;
  if (x < n_ctx) {
    context_tile<T, HD, NT>(p, x % p.splits, blockIdx.y, x / p.splits, smem);
  } else {
    x -= n_ctx;
    const int z = x % own_z, sx = x / own_z;
    own_tiles<T, HD, NT, WIDE>(p, sx / p.own_splits, sx % p.own_splits, blockIdx.y, z, own_z, smem);
  }
}

// ---- 3. join: WPR warps per row, which share its parts.  grid (sequence, kv head, rows in flight)
template <typename T, int HD, int WPR>
__global__ void __launch_bounds__(DIR_THREADS)
join_kernel(const __grid_constant__ SharedParams p) {
  constexpr int V = HD / 32, RPC = DIR_WARPS / WPR, UN = 8;    // values of a lane, rows of a CTA, parts in flight
  __shared__ float jo[DIR_WARPS][HD], jm[DIR_WARPS], jl[DIR_WARPS];
  pdl_trigger();
  const int s = blockIdx.x, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % WPR;
  const int parts = p.splits + p.own_splits;
  if (parts == 0) pdl_wait();                 // no kernel of this call before this one: a stranger's results
  const Seq sq = sequence(p, s);              // older than the kernels before, which have started: no wait
  pdl_wait();
  const int mine = parts > sub ? (parts - sub + WPR - 1) / WPR : 0;
  const int64_t rows = (int64_t)p.R * p.n_q;
  const int count = sq.n * p.g;
  for (int j0 = blockIdx.z * RPC; j0 < count; j0 += gridDim.z * RPC) {
    const int j = j0 + warp / WPR;
    const bool ok = j < count;
    const int64_t at = (int64_t)(sq.r0 + (ok ? j : 0) / p.g) * p.n_q + h * p.g + (ok ? j : 0) % p.g;
    float mx = NO_MAX, l = 0.f, o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int b = 0; b < mine; b += 32) {
      const bool have = b + lane < mine;
      const float2 ml = have ? __ldcg(p.part_ml + (int64_t)(sub + (b + lane) * WPR) * rows + at) : make_float2(NO_MAX, 0.f);
      const float top = fmaxf(mx, warp_max(ml.x));
      const float w = have ? ex2(ml.x - top) : 0.f, f = ex2(mx - top);
      l = l * f + warp_sum(w * ml.y);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] *= f;
      mx = top;
      const int n = min(32, mine - b);
      for (int c = 0; c < n; c += UN) {
        float x[UN][V];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          if (c + u >= n) break;               // (the same for the whole warp)
          const float* src = p.part_o + ((int64_t)(sub + (b + c + u) * WPR) * rows + at) * HD + lane * V;
          if constexpr (V == 4) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(src));
            x[u][0] = y.x; x[u][1] = y.y; x[u][2] = y.z; x[u][3] = y.w;
          } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(src));
            x[u][0] = y.x; x[u][1] = y.y;
          }
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          if (c + u >= n) break;
          const float wu = __shfl_sync(0xFFFFFFFFu, w, c + u);
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = fmaf(wu, x[u][i], o[i]);
        }
      }
    }
    if constexpr (WPR > 1) {
#pragma unroll
      for (int i = 0; i < V; ++i) jo[warp][lane * V + i] = o[i];
      if (lane == 0) { jm[warp] = mx; jl[warp] = l; }
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int w = 1; w < WPR; ++w) {
          const float top = fmaxf(mx, jm[warp + w]), f = ex2(mx - top), e = ex2(jm[warp + w] - top);
          l = l * f + jl[warp + w] * e;
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = o[i] * f + jo[warp + w][lane * V + i] * e;
          mx = top;
        }
      }
      __syncthreads();
    }
    if (ok && sub == 0) {
      const float inv = l == 0.f ? 0.f : 1.f / l;              // nothing visible: zeros, lse = -inf
      T* dst = reinterpret_cast<T*>(p.out) + at * HD + lane * V;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) dst[i] = o[i] * inv;
      } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = round2<T>(o[i] * inv, o[i + 1] * inv);
      }
      if (lane == 0) p.lse[at] = l == 0.f ? -INFINITY : (mx + log2f(l)) * LN2;
    }
  }
}

struct Plan { bool tc; int splits, split_len, own_splits; bool wide; int nt, z; };      // nt: tiles of 8 nt rows

// How the context and the own tokens are cut.
Plan make_plan(bool is16, int R, int P, int S, int cap, int g, int n_kv, int hd, bool ragged) {
  Plan pl = {false, 0, 0, 0, false, 2, 1};
  if (R == 0 || S == 0) return pl;
  // Up to one tile of stacked rows on mma.sync, more on tcgen05: over 12416 tokens of 8 kv heads one
  // tile takes 17.2 us on mma.sync, two tiles 22.0 us against 18.3 us on tcgen05, four 42.8 against 20.8.
  if (P > 0 && is16 && (int64_t)R * g > MT) {
    // One CTA per SM, longer key ranges first: every split but the last has `len` tiles, the last what is
    // left.  In units of a key tile (0.85 us), with 9 for a CTA's start and end, the CTAs of the last split
    // fill what the last round of the others leaves idle.  The mean of that end and of the work per SM
    // counts, since CTAs do not run in step and own tokens use idle SMs, plus writing and reading the
    // parts at memory speed (58 row blocks x 2 heads over 128 tiles: 108 + 20 tiles 137 us, 64 + 64 146 us;
    // one row block x 8 heads over 97 tiles: 11 splits 19.5 us, 17 splits 22.6 us; figures
    // with K and V in L2, before the branch for far scores added 1 to 2 %).
    const int64_t base = (int64_t)akvs_cdiv(R, 128 / g) * n_kv;
    const int tiles = akvs_cdiv(P, 128);
    const double part = 2.0 * R * g * n_kv * (hd + 2) * 4 / 6.4e6 / 0.85;
    int best = tiles, last = 0;
    double best_cost = 1e300;
    auto consider = [&](int len, double uneven) {
      const int s = (tiles + len - 1) / len, longs = s > 1 ? (s - 1) * (int)base : 0, q = longs / 148, r = longs % 148;
      const double a = len + 9, b = tiles - (s - 1) * len + 9;
      double end;
      const int64_t fit = r > 0 ? (int)(a / b) * (148 - r) : 0;        // last ones that end with the others
      if (r > 0 && fit >= base) end = (q + 1) * a;
      else end = (q + (r > 0)) * a + (double)((base - fit + 147) / 148) * b;
      const double work = (longs * a + base * b) * (1.0 / 148);
      const double cost = uneven * (0.5 * (end + work) + part * s);
      if (cost < best_cost) { best_cost = cost; best = len; }
    };
    for (int s = 1; s <= tiles && (s == 1 || base * s <= 3 * 148); ++s) {
      const int even = (tiles + s - 1) / s;
      if (even == last) continue;
      last = even;
      consider(even, 1.0);
      // a last split so short that k of its CTAs take as long as one of the others; it has to gain 2 %
      // over equal ones, which leave idle SMs to the own tokens from the start (32 row blocks and heads
      // over 256 tiles with 268 MB of own tokens: 4 equal splits 126 us, 4 x 58 + 24 tiles 128 us)
      const int r = s > 1 ? (s - 1) * (int)base % 148 : 0, k = r > 0 ? ((int)base + 147 - r) / (148 - r) : 1;
      if (k > 1) {
        const int len = (int)((k * (tiles + 9.0) - 9) / (1 + (double)k * (s - 1))) + 1;
        if (len < tiles) consider(len, 1.02);
      }
    }
    pl.tc = true;
    pl.split_len = best * 128;
  } else if (P > 0) {
    // Two CTAs fit an SM; one runs 64 keys at a time.
    if (is16 && (int64_t)R * g <= 8) pl.nt = 1;
    const int64_t base = (int64_t)n_kv * akvs_cdiv((int64_t)R * g, 8 * pl.nt);
    const int units = akvs_cdiv(P, 64);
    const int splits = (int)(base >= 296 ? 1 : akvs_cdiv(296, base));
    pl.split_len = akvs_cdiv(units, splits < units ? splits : units) * 64;
  }
  if (P > 0) pl.splits = akvs_cdiv(P, pl.split_len);
  // Stacked rows of a sequence: g, or the mean of a ragged batch.  Ragged batches get room for twice
  // the mean at once, and a CTA walks what is left.
  const int64_t stacked = ragged ? (int64_t)akvs_cdiv(R, S) * g * 2 : g;
  pl.wide = is16 && ragged && (int64_t)akvs_cdiv(R, S) * g > MT;
  if (is16 && (P == 0 || pl.tc) && !ragged && g <= 8) pl.nt = 1;
  const int64_t tiles = (stacked + 8 * pl.nt - 1) / (8 * pl.nt), z = pl.wide ? (tiles + DIR_WARPS - 1) / DIR_WARPS : tiles;
  pl.z = (int)(z < 64 ? z : 64);
  if (cap > 0) {
    pl.own_splits = 1;
    // Few sequences: their tokens are split while CTAs are missing and a split keeps 128 keys.
    while (!pl.wide && pl.own_splits < MAX_OWN_SPLITS && (int64_t)S * n_kv * pl.z * pl.own_splits * 2 <= 296 &&
           cap / (pl.own_splits * 2) >= 128)
      pl.own_splits *= 2;
  }
  return pl;
}

int64_t parts_bytes(int64_t rows, int hd) { return akvs_align_up(rows * hd * 4, 256) + akvs_align_up(rows * 8, 256) + 256; }
int64_t part_rows(const Plan& pl, int R, int n_q) { return (int64_t)(pl.splits + pl.own_splits) * R * n_q; }

// Rows of parts of any plan for up to R rows, P context tokens, cap own ones and any number of sequences:
// it grows with each of them, which a single plan's need does not (fewer rows are split further).
int64_t part_rows_bound(bool is16, int R, int P, int cap, int g, int n_kv) {
  const int64_t n_q = (int64_t)n_kv * g;
  auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
  auto most = [](int64_t a, int64_t b) { return a > b ? a : b; };
  int64_t ctx = 0;
  // mma.sync and float: up to ceil(296 / base) splits of 64 keys or more, base >= r * n_q / MT
  const int64_t r = is16 ? least(R, MT / g) : R;
  if (r > 0) ctx = least(least(akvs_cdiv(P, 64), akvs_cdiv(296, n_kv)) * r * n_q, 296 * MT + r * n_q);
  // tcgen05: at most 3 * 148 CTAs or one split, base >= r * n_q / 128
  if (is16 && (int64_t)R * g > MT)
    ctx = most(ctx, least(least(akvs_cdiv(P, 128), most(1, 3 * 148 / n_kv)) * R * n_q, most((int64_t)R * n_q, 3 * 148 * 128)));
  // Own tokens: `own` splits of S sequences of r rows have S * n_kv * z * own <= 296, or are one split.  One row
  // each: r = S, g <= MT * z.  Ragged 16 bits: r * g <= MT * S, or one split (wide).  Ragged float: z >= r * g / (8 S),
  // or z = 64, where 4 splits of one kv head or 2 of two are the most.
  int own = cap > 0;
  while (own > 0 && own < MAX_OWN_SPLITS && (int64_t)n_kv * own * 2 <= 296 && cap / (own * 2) >= 128) own *= 2;
  const int64_t all = (int64_t)R * n_q, deep = is16 || n_kv > 2 ? 1 : 4 / n_kv;
  return ctx + least(own * all, most(deep * all, 296 * MT));
}

template <typename T, int HD, int NT, bool WIDE>
int32_t launch_direct(const SharedParams& p, const Plan& pl, cudaStream_t st) {
  constexpr int smem = direct_smem<T, HD>();
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)direct_kernel<T, HD, NT, WIDE>, smem, smem_set));
  const int64_t n_ctx = (int64_t)p.splits * akvs_cdiv((int64_t)p.R * p.g, 8 * NT);
  const int64_t grid = n_ctx + (int64_t)p.S * p.own_splits * pl.z;
  if (grid > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  AKVS_CUDA(launch_pdl(direct_kernel<T, HD, NT, WIDE>, dim3((unsigned)grid, p.n_kv), dim3(DIR_THREADS), smem, st, p, (int)n_ctx,
                       pl.z));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

template <typename T, int HD, int NT, bool WIDE>
int32_t launch_own(const SharedParams& p, const Plan& pl, cudaStream_t st) {
  constexpr int smem = direct_smem<T, HD>();
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)own_kernel<T, HD, NT, WIDE>, smem, smem_set));
  AKVS_CUDA(launch_pdl(own_kernel<T, HD, NT, WIDE>, dim3((unsigned)(p.S * p.own_splits), p.n_kv, pl.z), dim3(DIR_THREADS), smem, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

template <typename T, int HD>
int32_t run(SharedParams& p, int dtype, const Plan& pl, cudaStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (pl.tc) {
      AKVS_TRY(launch_attention_parts_tc(dtype, HD, p.q, p.q_ld, p.pk, p.pv, p.p_ld, p.R, p.P, p.n_q, p.n_kv, p.split_len,
                                         p.part_o, p.part_ml, st));
      if (p.own_splits > 0) {
        if (pl.wide) AKVS_TRY((launch_own<T, HD, 2, true>(p, pl, st)));
        else if (pl.nt == 2) AKVS_TRY((launch_own<T, HD, 2, false>(p, pl, st)));
        else AKVS_TRY((launch_own<T, HD, 1, false>(p, pl, st)));
      }
    } else if (p.splits + p.own_splits > 0) {
      if (pl.wide) AKVS_TRY((launch_direct<T, HD, 2, true>(p, pl, st)));
      else if (pl.nt == 2) AKVS_TRY((launch_direct<T, HD, 2, false>(p, pl, st)));
      else AKVS_TRY((launch_direct<T, HD, 1, false>(p, pl, st)));
    }
  } else if (p.splits + p.own_splits > 0) {
    AKVS_TRY((launch_direct<T, HD, 2, false>(p, pl, st)));
  }
  // Few rows with many parts: four warps share a row's parts.  CTAs in flight: what the SMs hold at a
  // time; more of them would start late and find little.
  const bool few = (int64_t)p.R * p.n_q <= 2048 && p.splits + p.own_splits > 8;
  const int64_t rows = p.q_off ? (int64_t)akvs_cdiv(p.R, p.S) * p.g * 2 : p.g, per = few ? 1 : DIR_WARPS;
  const int64_t fit = akvs_cdiv(148 * 15, (int64_t)p.S * p.n_kv), need = (rows + per - 1) / per;
  const dim3 grid(p.S, p.n_kv, (unsigned)(need < fit ? need : fit < 1 ? 1 : fit));
  if (few) AKVS_CUDA(launch_pdl(join_kernel<T, HD, 4>, grid, dim3(DIR_THREADS), 0, st, p));
  else AKVS_CUDA(launch_pdl(join_kernel<T, HD, 1>, grid, dim3(DIR_THREADS), 0, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

bool heads_ok(int32_t n_q, int32_t n_kv) { return n_kv > 0 && n_q > 0 && n_q % n_kv == 0 && n_q / n_kv <= 128 && n_kv <= 65535; }

}  // namespace

extern "C" int64_t akvs_op_attention_shared_scratch_bytes(int32_t dtype, int32_t R, int32_t P, int32_t S, int32_t cap,
                                                          int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return -1;
  if (R < 0 || P < 0 || S < 0 || cap < 0 || !heads_ok(n_q_heads, n_kv_heads) || (head_dim != 64 && head_dim != 128)) return -1;
  if ((int64_t)R * n_q_heads > 0x7fffffff) return -1;
  return parts_bytes(part_rows_bound(dtype != AKVS_F32, R, P, cap, n_q_heads / n_kv_heads, n_kv_heads), head_dim);
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
  if ((int64_t)R * n_q_heads > 0x7fffffff || (int64_t)S * MAX_OWN_SPLITS > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  const int32_t used = q_off ? R : S;             // rows behind the last sequence's get no parts
  const Plan pl = make_plan(dtype != AKVS_F32, used, P, S, cap, n_q_heads / n_kv_heads, n_kv_heads, head_dim, q_off != nullptr);
  const int64_t rows = part_rows(pl, used, n_q_heads), need = parts_bytes(rows, head_dim);
  if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || scratch_size < need) return AKVS_ERR_WORKSPACE;
  const int64_t ctx_n = P > 0 ? ((P - 1) * ctx_ld + row) * es : 0;
  const int64_t own_n = cap > 0 ? ((S - 1) * own_seq_ld + (cap - 1) * own_ld + row) * es : 0;
  const void* ins[7] = {q, ctx_k, ctx_v, own_k, own_v, own_len, q_off};
  const int64_t in_n[7] = {((R - 1) * q_ld + q_row) * es, ctx_n, ctx_n, own_n, own_n, cap > 0 ? S * 4ll : 0, q_off ? (S + 1) * 4ll : 0};
  const void* outs[3] = {out, lse, scratch};
  const int64_t out_n[3] = {R * q_row * es, (int64_t)R * n_q_heads * 4, need};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 7; ++i)
      if (bytes_overlap(ins[i], in_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
    for (int i = 0; i < o; ++i)
      if (bytes_overlap(outs[i], out_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
  }
  SharedParams p;
  p.q = q; p.q_ld = q_ld; p.R = used; p.n_q = n_q_heads; p.n_kv = n_kv_heads; p.g = n_q_heads / n_kv_heads;
  p.pk = ctx_k; p.pv = ctx_v; p.P = P; p.p_ld = ctx_ld;
  p.sk = own_k; p.sv = own_v; p.S = S; p.cap = cap; p.s_ld = own_ld; p.s_seq = own_seq_ld; p.s_len = own_len; p.q_off = q_off;
  p.out = out; p.lse = lse;
  p.splits = pl.splits; p.split_len = pl.split_len; p.own_splits = pl.own_splits;
  p.part_o = reinterpret_cast<float*>(scratch);
  p.part_ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(scratch) + akvs_align_up(rows * head_dim * 4, 256));
  p.scale_log2 = LOG2E / sqrtf((float)head_dim);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    return head_dim == 64 ? run<T, 64>(p, dtype, pl, st) : run<T, 128>(p, dtype, pl, st);
  });
}
