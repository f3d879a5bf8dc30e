// Norm of queries and keys per head with the position rotation in the same pass:
//     y = x * rsqrt(mean(x^2) + eps) * gain              over the head_dim values of one head
//     out[i]        = y[i] cos(a_i) - y[i + hd/2] sin(a_i)
//     out[i + hd/2] = y[i + hd/2] cos(a_i) + y[i] sin(a_i),    a_i = pos * base^(-2i/hd)
// Memory bound: every value is read once and written once (7 flops each), q and k in one launch
// (11648 rows x 48 heads of 128, 16 bits: 52 us, 5.5 TB/s; one row 2.1 us).
// A head is shared by LPH lanes; a lane holds one 16-byte chunk of the lower half and the partner
// chunk of the upper half, so the rotation needs no exchange and the sum of squares log2(LPH)
// shuffles.  A warp keeps its row's cosines and sines in registers and walks the heads of the
// row; few rows are cut into more warps by heads, which then repeat the row's angles.
// All arithmetic is float with one rounding at the store.  Angles: the turn count
// pos * base^(-2i/hd) / 2pi is formed and reduced to [-1/2, 1/2] in double (a float angle of a
// far position has no correct digits left after the reduction), then split into a float and its
// remainder, which enters as a first-order correction.
#include "common.cuh"
#include <math.h>

namespace {

constexpr int QKN_THREADS = 256, QKN_BLOCKS = 4;      // per SM: 64 registers a thread
constexpr int QKN_MAX_HALF = 128;           // head_dim <= 256

struct QkNormParams {
  const void* x[2];                         // q, k
  void* y[2];
  const float* gain[2];
  int64_t ld_x[2], ld_y[2];                 // elements between rows
  const int32_t* pos;
  int n, heads[2];
  int units_per_row, heads_per_unit;        // a warp walks heads_per_unit heads of one row
  float eps;
  double turns[QKN_MAX_HALF];               // base^(-2i/hd) / 2pi
};

__device__ __forceinline__ void unpack(const uint4& w, float (&o)[4], float) {
  o[0] = __uint_as_float(w.x); o[1] = __uint_as_float(w.y); o[2] = __uint_as_float(w.z); o[3] = __uint_as_float(w.w);
}
template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float (&o)[8], T) {
  ld16(reinterpret_cast<const T*>(&w), o);
}

template <typename T, int HD>
__global__ void __launch_bounds__(QKN_THREADS, QKN_BLOCKS)
qk_norm_rope_kernel(const __grid_constant__ QkNormParams p) {
  constexpr int V = VecOf<T>::N, HALF = HD / 2, LPH = HALF / V, HPW = 32 / LPH;
  __shared__ double turns[HALF];
  __shared__ __align__(16) float gains[2][HD];
  pdl_trigger();
  for (int i = threadIdx.x; i < HALF; i += QKN_THREADS) turns[i] = p.turns[i];
  pdl_wait();
  for (int i = threadIdx.x; i < 2 * HD; i += QKN_THREADS)
    if (p.heads[i / HD] > 0) gains[i / HD][i % HD] = p.gain[i / HD][i % HD];
  __syncthreads();
  const int64_t unit = (int64_t)blockIdx.x * (QKN_THREADS / 32) + (threadIdx.x >> 5);
  if (unit >= (int64_t)p.n * p.units_per_row) return;
  const int r = (int)(unit / p.units_per_row);
  const int h0 = (int)(unit % p.units_per_row) * p.heads_per_unit;
  const int n_heads = p.heads[0] + p.heads[1];
  const int h1 = min(h0 + p.heads_per_unit, n_heads);
  const int lane = threadIdx.x & 31, sub = lane / LPH, c = (lane % LPH) * V;

  // The next group's chunks are on their way while a group is worked on, in the 8 registers of their
  // packed form: the kernel lives on the number of warps that fit.
  uint4 nlo, nhi;
  auto fetch = [&](int hh) {
    if (hh < h1) {
      const int w = hh >= p.heads[0];
      const uint4* x = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.x[w]) + (int64_t)r * p.ld_x[w] +
                                                      (int64_t)(hh - (w ? p.heads[0] : 0)) * HD + c);
      nlo = __ldcs(x);
      nhi = __ldcs(x + LPH);
    } else {
      nlo = nhi = make_uint4(0u, 0u, 0u, 0u);
    }
  };
  fetch(h0 + sub);

  float cs[V], sn[V];
  const double at = (double)p.pos[r];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const double t = at * turns[c + i];
    const double f = t - rint(t);
    const float hi = (float)f;
    const float lo = (float)(f - (double)hi) * 6.2831853f;
    float s_, c_;
    sincospif(2.f * hi, &s_, &c_);
    sn[i] = fmaf(c_, lo, s_);
    cs[i] = fmaf(-s_, lo, c_);
  }

  for (int h = h0 + sub; h - sub < h1; h += HPW) {
    float lo[V], hi[V];
    unpack(nlo, lo, T{});
    unpack(nhi, hi, T{});
    fetch(h + HPW);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
    const float scale = rsqrtf(ss * (1.f / HD) + p.eps);
    if (h >= h1) continue;
    const int w = h >= p.heads[0];
    float olo[V], ohi[V];
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 gl = *reinterpret_cast<const float4*>(&gains[w][c + i]), gh = *reinterpret_cast<const float4*>(&gains[w][HALF + c + i]);
      const float ga[4] = {gl.x, gl.y, gl.z, gl.w}, gb[4] = {gh.x, gh.y, gh.z, gh.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = lo[i + e] * scale * ga[e], b = hi[i + e] * scale * gb[e];
        olo[i + e] = a * cs[i + e] - b * sn[i + e];
        ohi[i + e] = b * cs[i + e] + a * sn[i + e];
      }
    }
    T* y = reinterpret_cast<T*>(p.y[w]) + (int64_t)r * p.ld_y[w] + (int64_t)(h - (w ? p.heads[0] : 0)) * HD + c;
    st16(y, olo);
    st16(y + HALF, ohi);
  }
}

template <typename T, int HD>
int32_t run(QkNormParams& p, cudaStream_t st) {
  constexpr int HPW = 32 / (HD / 2 / VecOf<T>::N);
  const int n_heads = p.heads[0] + p.heads[1];
  // Few rows: one group of heads per warp, so that all SMs get work.  Many rows: up to 16 groups,
  // which share the angles of their row.
  int groups = akvs_cdiv(n_heads, HPW), per = 1;
  while (per < 16 && per < groups && (int64_t)p.n * akvs_cdiv(groups, per * 2) >= 148 * 64) per *= 2;
  p.units_per_row = akvs_cdiv(groups, per);
  p.heads_per_unit = akvs_cdiv(groups, p.units_per_row) * HPW;       // even shares
  const int64_t blocks = ((int64_t)p.n * p.units_per_row + QKN_THREADS / 32 - 1) / (QKN_THREADS / 32);
  if (blocks > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  AKVS_CUDA(launch_pdl(qk_norm_rope_kernel<T, HD>, dim3((unsigned)blocks), dim3(QKN_THREADS), 0, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

}  // namespace

extern "C" int32_t akvs_op_qk_norm_rope(int32_t dtype, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                                        const float* q_gain, const float* k_gain, const int32_t* pos, int32_t n,
                                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float eps,
                                        float rope_base, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                                        void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (n < 0 || n_q_heads < 0 || n_kv_heads < 0 || (int64_t)n_q_heads + n_kv_heads > (1 << 20)) return AKVS_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !(rope_base > 0.f) || isinf(eps) || isinf(rope_base)) return AKVS_ERR_INVALID_ARG;
  if (head_dim != 32 && head_dim != 64 && head_dim != 128 && head_dim != 256) return AKVS_ERR_UNSUPPORTED;
  if (n == 0 || n_q_heads + n_kv_heads == 0) return AKVS_OK;
  if (!pos || (n_q_heads > 0 && (!q || !q_gain || !q_out)) || (n_kv_heads > 0 && (!k || !k_gain || !k_out)))
    return AKVS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)dtype_size(dtype);
  QkNormParams p;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const float* gain[2] = {q_gain, k_gain};
  const int64_t ld[2] = {q_ld, k_ld}, ld_out[2] = {q_out_ld, k_out_ld};
  const int heads[2] = {n_q_heads, n_kv_heads};
  for (int i = 0; i < 2; ++i) {
    p.x[i] = in[i]; p.y[i] = out[i]; p.gain[i] = gain[i]; p.ld_x[i] = ld[i]; p.ld_y[i] = ld_out[i]; p.heads[i] = heads[i];
    if (heads[i] == 0) continue;
    const int64_t row = (int64_t)heads[i] * head_dim;
    if (ld[i] < row || ld_out[i] < row) return AKVS_ERR_SHAPE;
    if (!aligned16(in[i]) || !aligned16(out[i]) || ld[i] * es % 16 || ld_out[i] * es % 16) return AKVS_ERR_INVALID_ARG;
  }
  for (int o = 0; o < 2; ++o) {
    if (heads[o] == 0) continue;
    const int64_t bytes = ((n - 1) * ld_out[o] + (int64_t)heads[o] * head_dim) * es;
    if (bytes_overlap(pos, n * 4ll, out[o], bytes)) return AKVS_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
      if (heads[i] > 0 && bytes_overlap(gain[i], head_dim * 4ll, out[o], bytes)) return AKVS_ERR_INVALID_ARG;
  }
  // In place is one tensor with one stride; any other overlap would be read after it was written.
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 2; ++i) {
      if (heads[o] == 0 || heads[i] == 0) continue;
      if (o == i && in[i] == out[o] && ld[i] == ld_out[o]) continue;
      if (rows_overlap(in[i], ld[i] * es, heads[i] * (int64_t)head_dim * es, out[o], ld_out[o] * es,
                       heads[o] * (int64_t)head_dim * es, n))
        return AKVS_ERR_INVALID_ARG;
    }
  if (heads[0] > 0 && heads[1] > 0 &&
      rows_overlap(out[0], ld_out[0] * es, heads[0] * (int64_t)head_dim * es, out[1], ld_out[1] * es,
                   heads[1] * (int64_t)head_dim * es, n))
    return AKVS_ERR_INVALID_ARG;
  p.pos = pos; p.n = n; p.eps = eps;
  // base^(-2i/hd) / 2pi by repeated products in extended precision: one power, no table kept
  const long double ratio = powl((long double)rope_base, -2.0L / head_dim);
  long double f = 0.159154943091895335768883763372514362L;
  for (int i = 0; i < head_dim / 2; ++i, f *= ratio) p.turns[i] = (double)f;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    switch (head_dim) {
      case 32: return run<T, 32>(p, st);
      case 64: return run<T, 64>(p, st);
      case 128: return run<T, 128>(p, st);
      default: return run<T, 256>(p, st);
    }
  });
}
