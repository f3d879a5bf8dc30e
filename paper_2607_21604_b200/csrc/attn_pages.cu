// Attention of new rows over the 4-bit pages of their sequences.
//
// Row i of the n new rows of sequence s sees the first len[s] - (n - 1 - i) of its tokens:
//     x_j = q . k_j / sqrt(hd),   lse = log sum_j exp(x_j),   out = sum_j exp(x_j - lse) v_j,
// with k_j and v_j given by codes c in 0..15 and a (scale, minimum) per group of 64 values:
//     q . k_j  = sum_g scale_jg (q_g . c_jg) + min_jg sum(q_g)
//     out_g    = sum_j (p_j scale_jg) c_jg + sum_j p_j min_jg
// so the codes enter the tensor cores as the whole numbers they are, exactly, and the records go to the scores
// and to the weights.  Nothing is dequantised.
//
// Memory bound: 144 bytes a token and kv head (head_dim 128) for the g query heads that share it, so a warp has
// few rows and many codes.  Products are mma.sync m16n8k16 with the ROWS along N (S^T = K Q^T: 16 keys x 8 rows,
// O^T += V^T P^T: 16 columns x 8 rows x 16 keys; P^T turned by movmatrix).  A code becomes an operand by an AND and half a
// shift, as a float16 c 2^-21 or 16 c 2^-21 (K), or by an AND alone as a bfloat16 c 2^-133 or 16 c 2^-133 (V); all are exact in the
// tensor cores.  The powers of two go to the other side: a row of q is scaled by a power of two so that its largest value lies in
// [2^14, 2^15), where float16 loses nothing above 2^-39 of it (odd values, which enter with a sixteenth: 2^-35); weights carry
// 2^100.
// The tensor cores cut sums off below their last bit, so a long sum of codes, all of them positive, comes out low, and
// the minima's term, which is as large, does not forgive that.  Odd tokens therefore enter with 15 - c (the complement,
// in the AND's own instruction) and minus their weight, and 15 times the weight joins the minima's term: the sums stay
// near zero (floats, 4000 tokens of about equal weight: 1.1e-5 off before).  They also line products up by their exponents, and the
// leading zeros of a subnormal are lost with it; so K's codes are not taken as an AND leaves them (scores of few float16 rows
// were 1e-6 off), nor V's for float rows (16 c 2^-133 throughout).  For float rows a piece's products are summed by themselves and
// added in float, rounded instead of cut off: root mean square errors of up to 0.6e-6 of the output for up to 11680 tokens
// (1.4e-6 with the AND alone).  8 float rows of 32 / 8 heads over 6000 tokens each: 30 us.
// A weight enters as a bfloat16 and the bfloat16 of what its rounding lost (2^-17 of itself; float rows: three of
// them).  That is little beside the output's own rounding (float16: 7e-6 beside 2.1e-4).  Up to 4 stacked rows (rows x query
// heads of a kv head) leave half of N free: there the columns 4 .. 7 repeat the rows, and take the lost parts in the same
// product.
//
// Work: a CTA of 4 warps takes 16 of a page's 64 tokens per warp, straight from global memory into registers (the
// page's layout is that of the fragments), one page ahead, the pages after it on their way to L2.  All
// (sequence, tile of rows, page) triples of a kv head form one list, in order, that is cut into equal parts, one per
// CTA, whatever the lengths; a CTA leaves (max, sum, O) of every stretch it holds in scratch, and a second kernel
// joins the stretches of a row in a fixed order.
// 64 rows of 40 / 8 heads over 500 to 12416 tokens each (490 MB): 137 us, 3.6 TB/s of 6.56.  Not memory but the issue slots
// (half of them taken) and the chains between products bound it: AND, shift and scale around every product of a few
// rows.  One page at a time with 16 warps an SM, 1, 3, 4 and 6 pages between a load and its request, 2 and 4 CTAs an SM: 137 to 172.
// Tiles of 16 rows and float rows leave room for 2 CTAs an SM, and the list is cut for as many (16 sequences of 8 rows over 6000
// tokens each, 32 / 8 heads: 120 us cut for three, 95 so).  A tile reads all of its pages, so a question of 128 rows over 12000 tokens
// takes 163 us; its 16-bit values read out and given to the shared attention take 56.
// One row of 32 / 8 heads over 8576 tokens: 12.2 us, of which 9 are a chain of loads (length, page numbers, pages), a step or two
// and the four warps' join, and 3 the second kernel.
#include "pages.cuh"
#include <float.h>
#include <math.h>

namespace {

constexpr int PA_WARPS = 4, PA_THREADS = PA_WARPS * 32;
constexpr int PA_CTAS = 148;                          // of all kv heads, times the CTAs that an SM holds
constexpr int ctas_of_an_sm(int TR, int type_size) { return TR == 16 || type_size == 4 ? 2 : 3; }
constexpr int AHEAD = 2;                              // pages between a load and the request that brings its page to L2
constexpr float NO_MAX = -FLT_MAX;                    // reference before any key: exp2(-inf - NO_MAX) = 0
constexpr float LN2 = 0.69314718f, LOG2E = 1.4426950408889634f;

struct PagesParams {
  const void* q;
  int64_t q_ld;
  int R, n_q, n_kv, g;
  const uint8_t* pool;
  int64_t page_ld;
  int n_pages;
  const int32_t* table;
  int64_t table_ld;
  int width, S;
  const int32_t* len;
  const int32_t* off;                                 // null: row s belongs to sequence s
  void* out;
  float* lse;
  float* part_o;                                      // [slot][n_kv][TR][hd]
  float2* part_ml;                                    // [slot][n_kv][TR] (reference in log2 units, sum)
  longlong2* plan;                                    // [S]: first unit and first tile of a sequence
  int workers;                                        // CTAs of a kv head
  int64_t slots;                                      // room in scratch: offsets that overlap find none
  float scale_log2;                                   // log2(e) / sqrt(hd)
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
__device__ __forceinline__ void add4(float (&d)[4], const float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) d[e] += x[e];
}
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float2 twice(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float part2(float2 a, int e) { return e ? a.y : a.x; }
__device__ __forceinline__ float2 half2f(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float2 bf2f(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }

template <int TR> __host__ __device__ __forceinline__ int tiles_of(int n, int g) { return (n * g + TR - 1) / TR; }

// A warp's 16 tokens of a page.  words: [half][..] of K (tokens gr, gr + 8) and V (tokens 2 t, 2 t + 1 and 8 more).
template <int HD> struct Stage {
  static constexpr int W = HD / 32, G = HD / 64;
  using B = PageBlock<HD>;
  uint32_t k[2][W], v[2][W], km[2][G], vm[2][G];
  static __device__ __forceinline__ void words(uint32_t (&w)[2][W], uint32_t (&m)[2][G], const uint8_t* at, const uint8_t* rec) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      if constexpr (HD == 128) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(at + hf * 4 * HD));
        const uint2 c = __ldcg(reinterpret_cast<const uint2*>(rec + hf * 8 * G * 4));
        w[hf][0] = a.x; w[hf][1] = a.y; w[hf][2] = a.z; w[hf][3] = a.w;
        m[hf][0] = c.x; m[hf][1] = c.y;
      } else {
        const uint2 a = __ldcg(reinterpret_cast<const uint2*>(at + hf * 4 * HD));
        w[hf][0] = a.x; w[hf][1] = a.y;
        m[hf][0] = __ldcg(reinterpret_cast<const uint32_t*>(rec + hf * 8 * G * 4));
      }
    }
  }
  __device__ __forceinline__ void load_k(const uint8_t* block, int warp, int lane) {
    words(k, km, block + warp * 8 * HD + lane * (HD / 8), block + 2 * B::KC + (warp * 16 + (lane >> 2)) * G * 4);
  }
  __device__ __forceinline__ void load_v(const uint8_t* block, int warp, int lane) {
    words(v, vm, block + B::KC + warp * 8 * HD + lane * (HD / 8), block + 2 * B::KC + B::META + (warp * 16 + (lane >> 2)) * G * 4);
  }
};

// What a warp keeps of a tile of TR stacked rows while tokens pass by.  Lane = 4 gr + t.
template <typename T, int HD, int TR> struct RowTile {
  static constexpr bool PAIR = TR == 4;               // columns 4 .. 7 repeat the rows and take the lost parts
  static constexpr int NT = TR == 16 ? 2 : 1, G = HD / 64, PIECES = sizeof(T) == 4 ? 3 : 1, WP = sizeof(T) == 4 ? 3 : 2;
  uint32_t qb[NT][PIECES][G][2][4];                   // row 8 x + gr: per word pairs (0 4) (2 6) (1 5)/16 (3 7)/16
  float2 rf[NT], qs[NT][G];                           // rows 8 x + 2 t, 2 t + 1: power of two and scale, sums of q
  int lim[NT][2];                                     // it sees the tokens below
  float o[NT][G][4][4];                               // [j][2 c + e]: value 64 g + 8 gr + 2 j + c (times 16 for c = 1)
  float2 om[NT][G];                                   // sums of weights times minima, this lane's tokens
  float2 mx[NT], sum[NT];                             // reference of the exponentials, their sum

  __device__ __forceinline__ void begin(const PagesParams& p, const PageSeq& sq, int j0, int h) {
    const int lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3, count = sq.n * p.g;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int j = j0 + (PAIR ? (gr & 3) : 8 * x + gr);
      const bool ok = j < count;
      const T* q = reinterpret_cast<const T*>(p.q) + (ok ? (int64_t)(sq.r0 + j / p.g) * p.q_ld + (int64_t)(h * p.g + j % p.g) * HD : 0);
      float f[G][16], top = 0.f, s[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        constexpr int V = VecOf<T>::N;
        s[g] = 0.f;
#pragma unroll
        for (int c = 0; c < 16; c += V) {
          float y[V];
          if (ok) {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(q + 64 * g + 16 * t + c));
            if constexpr (sizeof(T) == 4) {
              y[0] = __uint_as_float(w.x); y[1] = __uint_as_float(w.y); y[2] = __uint_as_float(w.z); y[3] = __uint_as_float(w.w);
            } else {
              ld16(reinterpret_cast<const T*>(&w), y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            f[g][c + e] = y[e];
            s[g] += y[e];
            top = fmaxf(top, fabsf(y[e]));
          }
        }
        s[g] += __shfl_xor_sync(0xFFFFFFFFu, s[g], 1);
        s[g] += __shfl_xor_sync(0xFFFFFFFFu, s[g], 2);
      }
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      // 2^up brings the largest value to [2^14, 2^15).  Rows with an infinity or a NaN end as NaN.
      int up = 141 - (int)(__float_as_uint(top) >> 23);
      up = top == 0.f || !(top < INFINITY) ? 0 : min(up, 100);
      // Beyond 2^115 the power below leaves the floats: such a row is NaN, as one with an infinity is.
      const float mul = up < -100 ? NAN : __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = f[g][8 * w + e] * mul * (e & 1 ? CODE_ODD : 1.f);
#pragma unroll
          for (int pc = 0; pc < PIECES; ++pc)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int lo = (i & 1) * 2 + (i >> 1);  // (0 4) (2 6) (1 5) (3 7)
              const __half2 hh = __floats2half2_rn(y[lo], y[lo + 4]);
              qb[x][pc][g][w][i] = *reinterpret_cast<const uint32_t*>(&hh);
              const float2 back = __half22float2(hh);
              y[lo] -= back.x;
              y[lo + 4] -= back.y;
            }
        }
      float rfe[2], qse[2][G];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = PAIR ? (2 * t + e) & 3 : 2 * t + e, from = 4 * m;
        const int ju = j0 + 8 * x + m;
        lim[x][e] = ju < count ? min(sq.len, max(0, sq.len - (sq.n - 1 - ju / p.g))) : sq.len;
        rfe[e] = __shfl_sync(0xFFFFFFFFu, __uint_as_float((uint32_t)(127 - up) << 23), from) * p.scale_log2 * CODE_BACK;
#pragma unroll
        for (int g = 0; g < G; ++g) qse[e][g] = __shfl_sync(0xFFFFFFFFu, s[g], from) * p.scale_log2;
      }
      rf[x] = make_float2(rfe[0], rfe[1]);
      mx[x] = make_float2(NO_MAX, NO_MAX);
      sum[x] = make_float2(0.f, 0.f);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        qs[x][g] = make_float2(qse[0][g], qse[1][g]);
        om[x][g] = make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x][g][j4][e] = 0.f;
    }
  }

  // The warp's 16 tokens of NP pages, from key0 on in the first of them.  ALL: every row sees every one of them.
  // `read_k` and `read_v` fetch what comes next, as soon as the registers are free.
  template <bool ALL, int NP, typename FK, typename FV>
  __device__ __forceinline__ void step(Stage<HD> (&st)[NP], int key0, const FK& read_k, const FV& read_v) {
    const int lane = threadIdx.x & 31, gr = lane >> 2;
    float2 s[NP][NT][2];                              // scores of token gr + 8 hf: rows 2 t, 2 t + 1
    bool sees[NP][NT][2][2];
    {
      float d[NP][NT][G][4];
#pragma unroll
      for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int g = 0; g < G; ++g) d[n][x][g][0] = d[n][x][g][1] = d[n][x][g][2] = d[n][x][g][3] = 0.f;
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int n = 0; n < NP; ++n) {
            uint32_t a0[2], a1[2], b0[2], b1[2];
            code_operands(st[n].k[0][2 * g + w], a0, a1);
            code_operands(st[n].k[1][2 * g + w], b0, b1);
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
              for (int pc = 0; pc < PIECES; ++pc) {
                const uint32_t(&q)[4] = qb[x][pc][g][w];
                float own[4] = {0.f, 0.f, 0.f, 0.f};
                float(&to)[4] = PIECES > 1 ? own : d[n][x][g];
                mma16816<f16>(to, a0[0], b0[0], a0[1], b0[1], q[0], q[1]);
                mma16816<f16>(to, a1[0], b1[0], a1[1], b1[1], q[2], q[3]);
                if constexpr (PIECES > 1) add4(d[n][x][g], own);
              }
          }
      float2 ks[NP][2][G];                            // (scale, minimum) of tokens gr and gr + 8
#pragma unroll
      for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int g = 0; g < G; ++g) ks[n][hf][g] = half2f(st[n].km[hf][g]);
      read_k();
#pragma unroll
      for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            float2 z = mul2(twice(ks[n][hf][0].y), qs[x][0]);
            float2 y = mul2(twice(ks[n][hf][0].x), make_float2(d[n][x][0][2 * hf], d[n][x][0][2 * hf + 1]));
            if constexpr (G == 2) {
              z = __ffma2_rn(twice(ks[n][hf][1].y), qs[x][1], z);
              y = __ffma2_rn(twice(ks[n][hf][1].x), make_float2(d[n][x][1][2 * hf], d[n][x][1][2 * hf + 1]), y);
            }
            s[n][x][hf] = __ffma2_rn(y, rf[x], z);
            if constexpr (!ALL) {
              const int key = key0 + n * 64 + 8 * hf + gr;
              sees[n][x][hf][0] = key < lim[x][0];
              sees[n][x][hf][1] = key < lim[x][1];
              s[n][x][hf] = make_float2(sees[n][x][hf][0] ? s[n][x][hf].x : -INFINITY, sees[n][x][hf][1] ? s[n][x][hf].y : -INFINITY);
            }
          }
    }
    // The reference of the exponentials is raised only when a score exceeds it by more than 2^8; weights above 1 are
    // as good as those below.
    float2 top[NT];
    bool raise = false;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      top[x] = make_float2(fmaxf(s[0][x][0].x, s[0][x][1].x), fmaxf(s[0][x][0].y, s[0][x][1].y));
#pragma unroll
      for (int n = 1; n < NP; ++n)
        top[x] = make_float2(fmaxf(fmaxf(top[x].x, s[n][x][0].x), s[n][x][1].x), fmaxf(fmaxf(top[x].y, s[n][x][0].y), s[n][x][1].y));
      raise = raise || top[x].x > mx[x].x + 8.f || top[x].y > mx[x].y + 8.f;
    }
    if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const float tops[2] = {top[x].x, top[x].y}, old[2] = {mx[x].x, mx[x].y};
        float now[2], f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = tops[e];
          m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
          m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
          now[e] = m > old[e] + 8.f ? m : old[e];     // a row's bits do not depend on its neighbours
          f[e] = ex2(old[e] - now[e]);
        }
        mx[x] = make_float2(now[0], now[1]);
        const float2 f2 = make_float2(f[0], f[1]);
        sum[x] = mul2(sum[x], f2);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          om[x][g] = mul2(om[x][g], f2);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][g][j][e] *= f[e & 1];
        }
      }
    }
    const float vpow = gr & 1 ? -0x1p100f : 0x1p100f, odd15 = gr & 1 ? 15.f : 0.f;
    uint32_t pb[NP][NT][G][WP][2];                    // B operands: tokens 2 t, 2 t + 1 (and 8 more) of row gr
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        float2 vs[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float2 r = half2f(st[n].vm[hf][g]);
          vs[g] = make_float2(r.x * vpow, fmaf(r.x, odd15, r.y));
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          const float2 dm = __fadd2_rn(s[n][x][hf], make_float2(-mx[x].x, -mx[x].y));
          const float2 y = make_float2(ex2(dm.x), ex2(dm.y));
          sum[x] = __fadd2_rn(sum[x], y);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float2 w = mul2(y, twice(vs[g].x));
            float2 m = __ffma2_rn(y, twice(vs[g].y), om[x][g]);
            if constexpr (!ALL) {                     // records that a row does not see may hold anything
              w = make_float2(sees[n][x][hf][0] ? w.x : 0.f, sees[n][x][hf][1] ? w.y : 0.f);
              m = make_float2(sees[n][x][hf][0] ? m.x : om[x][g].x, sees[n][x][hf][1] ? m.y : om[x][g].y);
            }
            om[x][g] = m;
            uint32_t part[WP];
#pragma unroll
            for (int i = 0; i < WP; ++i) {
              part[i] = pack_bf16x2(w.x, w.y);
              if (i + 1 < WP) {
                const float2 back = bf2f(part[i]);
                w = __fadd2_rn(w, make_float2(-back.x, -back.y));
              }
            }
            if constexpr (PAIR) {
              pb[n][x][g][0][hf] = turn8x8((lane & 2) ? part[1] : part[0]);
            } else {
#pragma unroll
              for (int i = 0; i < WP; ++i) pb[n][x][g][i][hf] = turn8x8(part[i]);
            }
          }
        }
      }
    // the upper halves hold odd tokens; float rows have all codes 4 bits up
    auto lo = [](uint32_t w) { return PIECES > 1 ? (w << 4 & 0x00F000F0u) ^ 0x00F00000u : (w & 0x000F000Fu) ^ 0x000F0000u; };
    auto hi4 = [](uint32_t w) { return (w & 0x00F000F0u) ^ 0x00F00000u; };
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int c = 0; c < 2; ++c) {                 // values 0 .. 3, 4 .. 7 of the lane's eight
          const uint32_t a = st[n].v[0][2 * g + c], b = st[n].v[1][2 * g + c], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i = 0; i < (PAIR ? 1 : WP); ++i) {
              const uint32_t b0 = pb[n][x][g][i][0], b1 = pb[n][x][g][i][1];
              float own[2][4] = {};
              float(&to0)[4] = PIECES > 1 ? own[0] : o[x][g][2 * c];
              float(&to1)[4] = PIECES > 1 ? own[1] : o[x][g][2 * c + 1];
              mma16816<bf16>(to0, lo(a), hi4(a), lo(b), hi4(b), b0, b1);
              mma16816<bf16>(to1, lo(a8), hi4(a8), lo(b8), hi4(b8), b0, b1);
              if constexpr (PIECES > 1) {
                add4(o[x][g][2 * c], own[0]);
                add4(o[x][g][2 * c + 1], own[1]);
              }
            }
        }
    read_v();
  }

  // Sums over the lanes that share a row; O in its own units.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < NT; ++x) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        sum[x].x += __shfl_xor_sync(0xFFFFFFFFu, sum[x].x, w);
        sum[x].y += __shfl_xor_sync(0xFFFFFFFFu, sum[x].y, w);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          om[x][g].x += __shfl_xor_sync(0xFFFFFFFFu, om[x][g].x, w);
          om[x][g].y += __shfl_xor_sync(0xFFFFFFFFu, om[x][g].y, w);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float y = o[x][g][j][e];
            if constexpr (PAIR) y += __shfl_xor_sync(0xFFFFFFFFu, y, 2);
            o[x][g][j][e] = fmaf(y, PIECES > 1 || (e & 2) ? 0x1p29f : 0x1p33f, e & 1 ? om[x][g].y : om[x][g].x);
          }
    }
  }
};

template <int HD, int TR> constexpr int attn_smem() { return PA_WARPS * TR * (HD + 4) * 4; }

// Pages pg0 .. pg0 + np - 1 of sequence s for the tile of rows from j0 on; leaves the part in `slot`.
template <typename T, int HD, int TR>
__device__ __forceinline__ void stretch(const PagesParams& p, const PageSeq& sq, int s, int j0, int pg0, int np, int64_t slot, int h,
                                        float* raw) {
  using B = PageBlock<HD>;
  using Tile = RowTile<T, HD, TR>;
  constexpr int NT = Tile::NT, G = Tile::G, LD = HD + 4;
  __shared__ float wm[PA_WARPS][TR], wl[PA_WARPS][TR];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane >> 2, t = lane & 3;
  const int32_t* row = p.table + (int64_t)s * p.table_ld + pg0;
  constexpr int NP = NT == 1 && sizeof(T) == 2 ? 2 : 1;         // pages at a time: two where the registers hold them
  int window = 0, ids = lane < np ? __ldcg(row + lane) : -1;
  auto block = [&](int i) -> const uint8_t* {         // page i of the stretch, or null
    if ((i & ~31) != window) {
      window = i & ~31;
      ids = window + lane < np ? __ldcg(row + window + lane) : -1;
    }
    const int id = __shfl_sync(0xFFFFFFFFu, ids, i & 31);
    return id < 0 || id >= p.n_pages ? nullptr : p.pool + (int64_t)id * p.page_ld + (int64_t)h * B::BYTES;
  };
  const int all_see = max(0, sq.len - (sq.n - 1 - j0 / p.g)), key0 = pg0 * 64 + warp * 16;
  const int whole = max(0, min(np, all_see / 64 - pg0));        // pages that all rows see to the end
  const uint8_t* at[NP];
  auto find = [&](int i) -> bool {                    // pages i .. i + NP - 1, all there and whole
    if (i + NP > whole) return false;
    bool ok = true;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      at[n] = block(i + n);
      ok = ok && at[n] != nullptr;
    }
    // the page AHEAD, to L2: a warp in turn asks for it
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if ((i & 31) + n + AHEAD < 32 && ((i + n) & (PA_WARPS - 1)) == warp) {
        const uint8_t* far = block(i + n + AHEAD);
        if (far && lane == 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(far), "r"(B::BYTES) : "memory");
      }
    return ok;
  };
  Stage<HD> st[NP];
  auto read_k = [&]() {
#pragma unroll
    for (int n = 0; n < NP; ++n) st[n].load_k(at[n], warp, lane);
  };
  auto read_v = [&]() {
#pragma unroll
    for (int n = 0; n < NP; ++n) st[n].load_v(at[n], warp, lane);
  };
  bool more = find(0);
  if (more) {
    read_k();
    read_v();
  }
  Tile tile;
  tile.begin(p, sq, j0, h);
  int i = 0;
  while (more) {
    const int now = i;
    i += NP;
    more = find(i);
    tile.template step<true, NP>(st, key0 + now * 64, [&]() { if (more) read_k(); }, [&]() { if (more) read_v(); });
  }
  for (; i < np; ++i) {                               // pages that end within, single ones, gaps
    const uint8_t* page = block(i);
    if (!page) continue;
    Stage<HD> one[1];
    one[0].load_k(page, warp, lane);
    one[0].load_v(page, warp, lane);
    tile.template step<false, 1>(one, key0 + i * 64, []() {}, []() {});
  }
  tile.finish();
  // Join the four warps.
  if (gr == 0 && (!Tile::PAIR || t < 2))
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e) { wm[warp][8 * x + 2 * t + e] = part2(tile.mx[x], e); wl[warp][8 * x + 2 * t + e] = part2(tile.sum[x], e); }
  __syncthreads();
  if (!Tile::PAIR || t < 2)
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = 8 * x + 2 * t + e;
        float top = wm[0][m];
#pragma unroll
        for (int w = 1; w < PA_WARPS; ++w) top = fmaxf(top, wm[w][m]);
        const float f = ex2(part2(tile.mx[x], e) - top);
        float* dst = raw + (warp * TR + m) * LD + 8 * gr;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            *reinterpret_cast<float4*>(dst + 64 * g + 4 * j) =
                make_float4(tile.o[x][g][2 * j][e] * f, tile.o[x][g][2 * j][2 + e] * f, tile.o[x][g][2 * j + 1][e] * f,
                            tile.o[x][g][2 * j + 1][2 + e] * f);
      }
  __syncthreads();
  const int64_t base = (slot * p.n_kv + h) * TR;
  for (int i = threadIdx.x; i < TR * HD / 4; i += PA_THREADS) {
    const int m = i / (HD / 4), c4 = i % (HD / 4) * 4;
    float4 a = *reinterpret_cast<const float4*>(raw + m * LD + c4);
#pragma unroll
    for (int w = 1; w < PA_WARPS; ++w) {
      const float4 b = *reinterpret_cast<const float4*>(raw + (w * TR + m) * LD + c4);
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
    *reinterpret_cast<float4*>(p.part_o + (base + m) * HD + c4) = a;
  }
  if (threadIdx.x < TR) {
    const int m = threadIdx.x;
    float top = wm[0][m], l = 0.f;
    for (int w = 1; w < PA_WARPS; ++w) top = fmaxf(top, wm[w][m]);
    for (int w = 0; w < PA_WARPS; ++w) l += wl[w][m] * ex2(wm[w][m] - top);
    p.part_ml[base + m] = make_float2(top, l);
  }
  __syncthreads();                                    // before another stretch uses the shared memory
}

__device__ __forceinline__ int64_t units_per_worker(int64_t total, int workers) { return total == 0 ? 1 : (total + workers - 1) / workers; }

// grid (workers, kv heads)
template <typename T, int HD, int TR>
__global__ void __launch_bounds__(PA_THREADS, ctas_of_an_sm(TR, sizeof(T)))
attention_pages_kernel(const __grid_constant__ PagesParams p) {
  extern __shared__ __align__(16) float raw[];
  __shared__ int64_t sums[PA_WARPS], rest[PA_WARPS], start_unit, start_tile;
  __shared__ int tsums[PA_WARPS], start_seq;
  __shared__ PageSeq start_of;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, w = blockIdx.x, h = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  const int64_t room = (int64_t)p.width * 64;
  auto units = [&](const PageSeq& q, int& tiles) -> int64_t {
    tiles = tiles_of<TR>(q.n, p.g);
    return (int64_t)tiles * ((q.len + 63) / 64);
  };
  // The list: units of all sequences, and where this CTA's share begins.  128 sequences at a time; lengths of up to 128
  // are read once.
  const bool planner = w == 0 && h == 0;              // leaves the list's outline for the join
  int64_t total = 0, u0 = 0, u1 = 0, per = 1, run = 0, trun = 0;
  if (p.S == 1) {                                     // nothing to search
    const PageSeq q = page_sequence(p.off, p.len, 0, p.R, room);
    int ti;
    total = units(q, ti);
    per = units_per_worker(total, p.workers);
    u0 = w * per;
    u1 = min(u0 + per, total);
    if (tid == 0) { start_seq = 0; start_unit = start_tile = 0; start_of = q; }
    __syncthreads();
  }
  for (int b = 0; p.S > 1 && b < p.S && (b == 0 || planner || run <= u0); b += PA_THREADS) {
    const int s = b + tid;
    PageSeq q = {0, 0, 0};
    if (s < p.S) q = page_sequence(p.off, p.len, s, p.R, room);
    int ti = 0;
    const int64_t c = units(q, ti);
    int64_t ci = c, later = 0;
    int tin = ti, dummy;
    if (b == 0)
      for (int k = tid + PA_THREADS; k < p.S; k += PA_THREADS) later += units(page_sequence(p.off, p.len, k, p.R, room), dummy);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, ci, o);
      const int y = __shfl_up_sync(0xFFFFFFFFu, tin, o);
      if (lane >= o) { ci += x; tin += y; }
      later += __shfl_xor_sync(0xFFFFFFFFu, later, o);
    }
    if (lane == 31) { sums[warp] = ci; tsums[warp] = tin; rest[warp] = later; }
    __syncthreads();
    int64_t before = run, tbefore = trun;
#pragma unroll
    for (int i = 0; i < PA_WARPS; ++i) {
      if (i < warp) { before += sums[i]; tbefore += tsums[i]; }
      run += sums[i];
      trun += tsums[i];
      if (b == 0) total += sums[i] + rest[i];
    }
    if (b == 0) {
      per = units_per_worker(total, p.workers);
      u0 = w * per;
      u1 = min(u0 + per, total);
    }
    before += ci - c;
    tbefore += tin - ti;
    if (planner && s < p.S) p.plan[s] = make_longlong2(before, tbefore);
    if (c > 0 && before <= u0 && u0 < before + c && u0 < u1) { start_seq = s; start_unit = before; start_tile = tbefore; start_of = q; }
    __syncthreads();
  }
  if (u0 >= u1) return;
  int s = start_seq;
  int64_t first = start_unit, tile0 = start_tile;
  PageSeq sq = start_of;
  for (int64_t u = u0; u < u1;) {
    const int tiles = tiles_of<TR>(sq.n, p.g), pages = (sq.len + 63) / 64;
    const int64_t c = (int64_t)tiles * pages;
    if (u - first >= c) {                             // the next sequence
      first += c;
      tile0 += tiles;
      sq = page_sequence(p.off, p.len, ++s, p.R, room);
      continue;
    }
    const int z = (int)((u - first) / pages), pg = (int)((u - first) % pages);
    const int np = (int)min((int64_t)(pages - pg), u1 - u);
    if ((uint64_t)(w + tile0 + z) < (uint64_t)p.slots) stretch<T, HD, TR>(p, sq, s, z * TR, pg, np, w + tile0 + z, h, raw);
    u += np;
  }
}

// grid (sequence, kv head, rows in flight): WPR warps join the stretches of one stacked row
template <typename T, int HD, int TR, int WPR>
__global__ void __launch_bounds__(PA_THREADS)
pages_join_kernel(const __grid_constant__ PagesParams p) {
  constexpr int V = HD / 32, UN = WPR > 1 ? 16 : 8, RPC = PA_WARPS / WPR;    // values of a lane, parts in flight, rows of a CTA
  __shared__ float jo[PA_WARPS][HD], jm[PA_WARPS], jl[PA_WARPS];
  pdl_trigger();
  const int s = blockIdx.x, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % WPR;
  const int64_t room = (int64_t)p.width * 64;
  // lengths and offsets are older than the kernel before, whose CTAs have all passed their wait: no wait for them
  const PageSeq sq = page_sequence(p.off, p.len, s, p.R, room), lq = page_sequence(p.off, p.len, p.S - 1, p.R, room);
  const int pages = (sq.len + 63) / 64, count = sq.n * p.g;
  pdl_wait();
  const longlong2 zero = make_longlong2(0, 0), at0 = p.S == 1 ? zero : __ldcg(p.plan + s);
  const int64_t total = (p.S == 1 ? 0 : __ldcg(p.plan + p.S - 1).x) + (int64_t)tiles_of<TR>(lq.n, p.g) * ((lq.len + 63) / 64);
  const int64_t per = units_per_worker(total, p.workers);
  for (int j0 = blockIdx.z * RPC; j0 < count; j0 += gridDim.z * RPC) {
    const bool ok = j0 + warp / WPR < count;
    const int j = ok ? j0 + warp / WPR : j0, z = j / TR, m = j % TR;
    const int64_t u = at0.x + (int64_t)z * pages;
    const int64_t w0 = u / per, w1 = pages ? (u + pages - 1) / per : w0 - 1;
    const int64_t slot0 = w0 + at0.y + z;
    const int all = slot0 >= 0 && slot0 + (w1 - w0) < p.slots ? (int)(w1 - w0 + 1) : 0, n = all > sub ? (all - sub + WPR - 1) / WPR : 0;
    float mx = NO_MAX, l = 0.f, o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.f;
    for (int b = 0; b < n; b += 32) {
      const bool have = b + lane < n;
      const float2 ml = have ? __ldcg(p.part_ml + ((slot0 + sub + (b + lane) * WPR) * p.n_kv + h) * TR + m) : make_float2(NO_MAX, 0.f);
      const int cnt = min(32, n - b);
      float x[UN][V];
      auto fetch = [&](int c) {
#pragma unroll
        for (int k = 0; k < UN; ++k) {
          if (c + k >= cnt) break;                    // (the same for the whole warp)
          const float* src = p.part_o + (((slot0 + sub + (b + c + k) * WPR) * p.n_kv + h) * TR + m) * HD + lane * V;
          if constexpr (V == 4) {
            const float4 y = __ldcg(reinterpret_cast<const float4*>(src));
            x[k][0] = y.x; x[k][1] = y.y; x[k][2] = y.z; x[k][3] = y.w;
          } else {
            const float2 y = __ldcg(reinterpret_cast<const float2*>(src));
            x[k][0] = y.x; x[k][1] = y.y;
          }
        }
      };
      fetch(0);
      const float top = fmaxf(mx, warp_max(ml.x));
      const float wt = have ? ex2(ml.x - top) : 0.f, f = ex2(mx - top);
      l = l * f + warp_sum(wt * ml.y);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] *= f;
      mx = top;
      for (int c = 0; c < cnt; c += UN) {
        if (c > 0) fetch(c);
#pragma unroll
        for (int k = 0; k < UN; ++k) {
          if (c + k >= cnt) break;
          const float wk = __shfl_sync(0xFFFFFFFFu, wt, c + k);
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = fmaf(wk, x[k][i], o[i]);
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
    if (!ok || sub != 0) continue;
    const int64_t row = (int64_t)(sq.r0 + j / p.g) * p.n_q + h * p.g + j % p.g;
    const float inv = l == 0.f ? 0.f : 1.f / l;       // nothing visible: zeros, lse = -inf
    T* dst = reinterpret_cast<T*>(p.out) + row * HD + lane * V;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < V; ++i) dst[i] = o[i] * inv;
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack2_inf<T>(o[i] * inv, o[i + 1] * inv);
    }
    if (lane == 0) p.lse[row] = l == 0.f ? -INFINITY : (mx + log2f(l)) * LN2;
  }
}

// Rows of a tile: 4 or 8 where a sequence has no more of them (the mean, of a ragged batch), else 16.  Float rows
// have three times the operands: 8.
int tile_rows(int dtype, int R, int S, int g, bool ragged) {
  if (dtype == AKVS_F32) return 8;
  const int64_t stacked = ragged ? (int64_t)akvs_cdiv(R, S) * g : g;
  return stacked <= 4 ? 4 : stacked <= 8 ? 8 : 16;
}
int workers_of(int n_kv, int per_sm) { return n_kv >= PA_CTAS * per_sm ? 1 : PA_CTAS * per_sm / n_kv; }
// Slots x rows of a slot: a stretch per CTA and one more per tile that it ends in; at most this for any tile
// size, so that the size grows with R and S.
int64_t slot_rows(int R, int S, int n_kv, int g) { return (int64_t)(workers_of(n_kv, 3) + S) * 16 + (int64_t)R * g; }
int64_t scratch_need(int R, int S, int n_kv, int g, int hd) {
  const int64_t rows = slot_rows(R, S, n_kv, g) * n_kv;
  return akvs_align_up(rows * hd * 4, 256) + akvs_align_up(rows * 8, 256) + akvs_align_up(S * 16ll, 256) + 256;
}

template <typename T, int HD, int TR>
int32_t run(const PagesParams& p, cudaStream_t st) {
  constexpr int smem = attn_smem<HD, TR>();
  static_assert(smem <= 48 * 1024, "no opt-in needed");
  AKVS_CUDA(launch_pdl(attention_pages_kernel<T, HD, TR>, dim3(p.workers, p.n_kv), dim3(PA_THREADS), smem, st, p));
  AKVS_LAUNCHED();
  // Few rows may have many stretches: four warps share a row's.
  const bool few = (int64_t)p.R * p.n_q <= 2048;
  const int64_t rows = p.off ? (int64_t)akvs_cdiv(p.R, p.S) * p.g * 2 : p.g, per = few ? 1 : PA_WARPS;
  const int64_t fit = akvs_cdiv(148 * 15, (int64_t)p.S * p.n_kv), want = (rows + per - 1) / per;
  const dim3 grid(p.S, p.n_kv, (unsigned)(want < fit ? want : fit < 1 ? 1 : fit));
  if (few) AKVS_CUDA(launch_pdl(pages_join_kernel<T, HD, TR, 4>, grid, dim3(PA_THREADS), 0, st, p));
  else AKVS_CUDA(launch_pdl(pages_join_kernel<T, HD, TR, 1>, grid, dim3(PA_THREADS), 0, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

bool heads_ok(int32_t n_q, int32_t n_kv) { return n_kv > 0 && n_q > 0 && n_q % n_kv == 0 && n_q / n_kv <= 128 && n_kv <= 65535; }

}  // namespace

extern "C" int64_t akvs_op_attention_pages_scratch_bytes(int32_t R, int32_t S, int32_t n_q_heads, int32_t n_kv_heads,
                                                         int32_t head_dim) {
  if (R < 0 || S < 0 || !heads_ok(n_q_heads, n_kv_heads) || (head_dim != 64 && head_dim != 128)) return -1;
  if ((int64_t)R * n_q_heads > 0x7fffffff) return -1;
  return scratch_need(R, S, n_kv_heads, n_q_heads / n_kv_heads, head_dim);
}

extern "C" int32_t akvs_op_attention_pages(int32_t dtype, const void* q, int64_t q_ld, int32_t R, const void* pool, int64_t page_ld,
                                           int32_t n_pages, const int32_t* table, int64_t table_ld, int32_t width,
                                           const int32_t* seq_len, const int32_t* q_off, int32_t S, int32_t n_q_heads,
                                           int32_t n_kv_heads, int32_t head_dim, void* out, float* lse, void* scratch,
                                           int64_t scratch_size, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (R < 0 || S < 0 || width < 0 || n_pages < 0) return AKVS_ERR_INVALID_ARG;
  if (!heads_ok(n_q_heads, n_kv_heads)) return AKVS_ERR_SHAPE;
  if (head_dim != 64 && head_dim != 128) return AKVS_ERR_UNSUPPORTED;
  if (!q_off && R < S) return AKVS_ERR_SHAPE;
  if (R == 0 || S == 0) return AKVS_OK;
  const int64_t es = (int64_t)dtype_size(dtype), q_row = (int64_t)n_q_heads * head_dim, block = akvs_page_bytes(n_kv_heads, head_dim);
  if (!q || !out || !lse || !seq_len || (width > 0 && !table) || (n_pages > 0 && !pool)) return AKVS_ERR_INVALID_ARG;
  if (q_ld < q_row || table_ld < width || (n_pages > 0 && page_ld < block)) return AKVS_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(out) || !aligned16(pool) || q_ld * es % 16 || page_ld % 16) return AKVS_ERR_INVALID_ARG;
  if ((int64_t)R * n_q_heads > 0x7fffffff || width > 0x7fffffff / 64) return AKVS_ERR_TOO_LARGE;
  const int32_t used = q_off ? R : S, g = n_q_heads / n_kv_heads;     // rows behind the last sequence's get no parts
  const int64_t need = scratch_need(used, S, n_kv_heads, g, head_dim);
  if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || scratch_size < need) return AKVS_ERR_WORKSPACE;
  const void* ins[5] = {q, pool, table, seq_len, q_off};
  const int64_t in_n[5] = {((R - 1) * q_ld + q_row) * es, n_pages > 0 ? (n_pages - 1) * page_ld + block : 0,
                           width > 0 ? ((S - 1) * table_ld + width) * 4 : 0, S * 4ll, q_off ? (S + 1) * 4ll : 0};
  const void* outs[3] = {out, lse, scratch};
  const int64_t out_n[3] = {R * q_row * es, (int64_t)R * n_q_heads * 4, need};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 5; ++i)
      if (bytes_overlap(ins[i], in_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
    for (int i = 0; i < o; ++i)
      if (bytes_overlap(outs[i], out_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
  }
  PagesParams p;
  p.q = q; p.q_ld = q_ld; p.R = used; p.n_q = n_q_heads; p.n_kv = n_kv_heads; p.g = g;
  p.pool = reinterpret_cast<const uint8_t*>(pool); p.page_ld = page_ld; p.n_pages = n_pages;
  p.table = table; p.table_ld = table_ld; p.width = width; p.S = S; p.len = seq_len; p.off = q_off;
  p.out = out; p.lse = lse;
  const int64_t rows = slot_rows(used, S, n_kv_heads, g) * n_kv_heads;
  char* at = reinterpret_cast<char*>(scratch);
  p.part_o = reinterpret_cast<float*>(at);
  p.part_ml = reinterpret_cast<float2*>(at + akvs_align_up(rows * head_dim * 4, 256));
  p.plan = reinterpret_cast<longlong2*>(at + akvs_align_up(rows * head_dim * 4, 256) + akvs_align_up(rows * 8, 256));
  const int tr = tile_rows(dtype, used, S, g, q_off != nullptr);
  p.workers = workers_of(n_kv_heads, ctas_of_an_sm(tr, (int)es));
  p.slots = slot_rows(used, S, n_kv_heads, g) / tr;
  p.scale_log2 = LOG2E / sqrtf((float)head_dim);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    if constexpr (sizeof(T) == 4) {
      return head_dim == 64 ? run<T, 64, 8>(p, st) : run<T, 128, 8>(p, st);
    } else {
      if (tr == 4) return head_dim == 64 ? run<T, 64, 4>(p, st) : run<T, 128, 4>(p, st);
      if (tr == 8) return head_dim == 64 ? run<T, 64, 8>(p, st) : run<T, 128, 8>(p, st);
      return head_dim == 64 ? run<T, 64, 16>(p, st) : run<T, 128, 16>(p, st);
    }
  });
}
