// Rotation of queries and keys by their positions: pairs (i, i + rot/2) or (2i, 2i + 1) of the first `rot`
// values of a head, the rest as it is, with frequencies scaled for contexts longer than the trained one:
//     (a, b) -> m (a cos - b sin, b cos + a sin),   angle = pos f_i,   i < rot/2
// The f_i are formed on the host, per call, in extended precision (akvs.h has the formulas) and travel as
// kernel parameters: turns f_i / 2pi in double.
// Memory bound: every value is read once and written once, q and k in one launch.  A lane holds one
// 16-byte chunk (interleaved pairs lie inside it) or a chunk and its partner rot/2 further (half layout),
// or a chunk that is only copied; it keeps its cosines and sines in registers and walks the heads of the
// row.  Angles are reduced to [-1/2, 1/2] turns in double and enter the cosine as a float and its
// remainder: a float angle of a far position has no correct digits left.  All arithmetic on values is
// float with one rounding at the store.
// 11648 rows of 40 + 8 heads of 128, half of each turned, in 58 us: 4.9 TB/s, of 6.56 that a copy reaches (1 us more with CTAs
// of 256 threads, 3 with three heads' loads ahead of their use, 6 with fewer heads a warp, which then form their
// angles more often; 2 of them look for infinities of float16); one row in 1.8 us, the time of a launch.
// Rotated parts whose halves do not start on 16 bytes (rot = 20, say) take a kernel that moves single
// values, a lane per pair: 172 us for those rows with 20 of 128 values turned.
#include "common.cuh"
#include <math.h>

namespace {

constexpr int RS_THREADS = 128, RS_MAX_HD = 256, RS_MAX_PAIRS = RS_MAX_HD / 2;

struct RopeParams {
  const void* x[2];                         // q, k
  void* y[2];
  int64_t ld_x[2], ld_y[2];                 // elements between rows
  const int32_t* pos;
  int n, heads[2], hd, rot;
  int rot_slots, slots;                     // chunks (or pairs of them) of a head that turn, and all of them
  int lanes, slot_blocks;                   // lanes of a head, warps that share a head with more than 32 slots
  int units_per_row, heads_per_unit;        // a warp walks heads_per_unit heads of one row
  float mag;
  double turns[RS_MAX_PAIRS];
};

// m cos and m sin of pos * turns
__device__ __forceinline__ float2 turn(double pos, double turns, float mag) {
  const double t = pos * turns, f = t - rint(t);
  const float hi = (float)f, lo = (float)(f - (double)hi) * 6.2831853f;
  float s, c;
  sincospif(2.f * hi, &s, &c);
  return make_float2(mag * fmaf(-s, lo, c), mag * fmaf(c, lo, s));
}

template <typename T>
__device__ __forceinline__ void unpack16(const uint4& w, float (&o)[VecOf<T>::N]) {
  if constexpr (sizeof(T) == 4) {
    o[0] = __uint_as_float(w.x); o[1] = __uint_as_float(w.y); o[2] = __uint_as_float(w.z); o[3] = __uint_as_float(w.w);
  } else {
    ld16(reinterpret_cast<const T*>(&w), o);
  }
}

template <typename T, bool INTER>
__global__ void __launch_bounds__(RS_THREADS)
rope_scaled_kernel(const __grid_constant__ RopeParams p) {
  constexpr int V = VecOf<T>::N, PAIRS = INTER ? V / 2 : V;
  __shared__ double turns[RS_MAX_PAIRS];
  pdl_trigger();
  for (int i = threadIdx.x; i < p.rot / 2; i += RS_THREADS) turns[i] = p.turns[i];
  pdl_wait();
  __syncthreads();
  const int64_t unit = (int64_t)blockIdx.x * (RS_THREADS / 32) + (threadIdx.x >> 5);
  const int per_row = p.units_per_row * p.slot_blocks;
  if (unit >= (int64_t)p.n * per_row) return;
  const int r = (int)(unit / per_row), rest = (int)(unit % per_row);
  const int h0 = rest / p.slot_blocks * p.heads_per_unit, n_heads = p.heads[0] + p.heads[1], h1 = min(h0 + p.heads_per_unit, n_heads);
  const int lane = threadIdx.x & 31, sub = lane / p.lanes, hpw = 32 / p.lanes;
  const int slot = rest % p.slot_blocks * 32 + lane % p.lanes;
  if (sub >= hpw || slot >= p.slots) return;                        // no lane waits for another below
  const bool turns_it = slot < p.rot_slots;
  const int at = turns_it ? slot * V : p.rot + (slot - p.rot_slots) * V, half = p.rot / 2;
  const bool two = !INTER && turns_it;

  uint4 nlo, nhi = make_uint4(0u, 0u, 0u, 0u);
  auto fetch = [&](int h) {
    if (h < h1) {
      const int w = h >= p.heads[0];
      const T* x = reinterpret_cast<const T*>(p.x[w]) + (int64_t)r * p.ld_x[w] + (int64_t)(h - (w ? p.heads[0] : 0)) * p.hd + at;
      nlo = __ldcs(reinterpret_cast<const uint4*>(x));
      if (two) nhi = __ldcs(reinterpret_cast<const uint4*>(x + half));
    }
  };
  fetch(h0 + sub);

  float cs[PAIRS], sn[PAIRS];
  if (turns_it) {
    const double pos = (double)p.pos[r];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      const float2 t = turn(pos, turns[slot * PAIRS + i], p.mag);
      cs[i] = t.x;
      sn[i] = t.y;
    }
  }

  for (int h = h0 + sub; h < h1; h += hpw) {
    const uint4 a4 = nlo, b4 = nhi;
    fetch(h + hpw);
    const int w = h >= p.heads[0];
    T* y = reinterpret_cast<T*>(p.y[w]) + (int64_t)r * p.ld_y[w] + (int64_t)(h - (w ? p.heads[0] : 0)) * p.hd + at;
    if (!turns_it) {
      *reinterpret_cast<uint4*>(y) = a4;
    } else if constexpr (INTER) {
      float a[V], o[V];
      unpack16<T>(a4, a);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        o[2 * i] = a[2 * i] * cs[i] - a[2 * i + 1] * sn[i];
        o[2 * i + 1] = a[2 * i + 1] * cs[i] + a[2 * i] * sn[i];
      }
      st16_inf(y, o);
    } else {
      float a[V], b[V], oa[V], ob[V];
      unpack16<T>(a4, a);
      unpack16<T>(b4, b);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        oa[i] = a[i] * cs[i] - b[i] * sn[i];
        ob[i] = b[i] * cs[i] + a[i] * sn[i];
      }
      st16_inf(y, oa);
      st16_inf(y + half, ob);
    }
  }
}

// Any even rot: lane i has the pairs i, i + 32, ...; a warp walks the heads of its unit.
template <typename T, bool INTER>
__global__ void __launch_bounds__(RS_THREADS)
rope_scaled_values_kernel(const __grid_constant__ RopeParams p) {
  constexpr int MAX = RS_MAX_PAIRS / 32;
  pdl_trigger();
  pdl_wait();
  const int64_t unit = (int64_t)blockIdx.x * (RS_THREADS / 32) + (threadIdx.x >> 5);
  if (unit >= (int64_t)p.n * p.units_per_row) return;
  const int r = (int)(unit / p.units_per_row), lane = threadIdx.x & 31, half = p.rot / 2;
  const int h0 = (int)(unit % p.units_per_row) * p.heads_per_unit, h1 = min(h0 + p.heads_per_unit, p.heads[0] + p.heads[1]);
  float cs[MAX], sn[MAX];
  const double pos = (double)p.pos[r];
#pragma unroll
  for (int k = 0; k < MAX; ++k)
    if (lane + 32 * k < half) {
      const float2 t = turn(pos, p.turns[lane + 32 * k], p.mag);
      cs[k] = t.x;
      sn[k] = t.y;
    }
  for (int h = h0; h < h1; ++h) {
    const int w = h >= p.heads[0];
    const int64_t head = (int64_t)(h - (w ? p.heads[0] : 0)) * p.hd;
    const T* x = reinterpret_cast<const T*>(p.x[w]) + (int64_t)r * p.ld_x[w] + head;
    T* y = reinterpret_cast<T*>(p.y[w]) + (int64_t)r * p.ld_y[w] + head;
#pragma unroll
    for (int k = 0; k < MAX; ++k) {
      const int i = lane + 32 * k;
      if (i >= half) break;
      const int ia = INTER ? 2 * i : i, ib = INTER ? 2 * i + 1 : i + half;
      const float a = to_f(x[ia]), b = to_f(x[ib]);
      y[ia] = from_f_inf<T>(a * cs[k] - b * sn[k]);
      y[ib] = from_f_inf<T>(b * cs[k] + a * sn[k]);
    }
    for (int i = p.rot + lane; i < p.hd; i += 32) y[i] = x[i];
  }
}

template <typename T, bool INTER>
int32_t run(RopeParams& p, bool in_place, cudaStream_t st) {
  constexpr int V = VecOf<T>::N;
  const int n_heads = p.heads[0] + p.heads[1];
  const bool chunks = p.rot % (INTER ? V : 2 * V) == 0;
  p.rot_slots = p.rot / (INTER ? V : 2 * V);
  p.slots = p.rot_slots + (in_place ? 0 : (p.hd - p.rot) / V);        // in place the rest stays where it is
  p.lanes = p.slots < 32 ? p.slots : 32;
  p.slot_blocks = akvs_cdiv(p.slots, 32);
  const int hpw = chunks ? 32 / p.lanes : 1;
  // Few rows: one group of heads per warp, so that all SMs get work.  Many rows: up to 16 groups,
  // which share the angles of their row.
  int groups = akvs_cdiv(n_heads, hpw), per = 1;
  while (per < 16 && per < groups && (int64_t)p.n * akvs_cdiv(groups, per * 2) >= 148 * 64) per *= 2;
  p.units_per_row = akvs_cdiv(groups, per);
  p.heads_per_unit = akvs_cdiv(groups, p.units_per_row) * hpw;        // even shares
  const int64_t units = (int64_t)p.n * p.units_per_row * (chunks ? p.slot_blocks : 1);
  const int64_t blocks = (units + RS_THREADS / 32 - 1) / (RS_THREADS / 32);
  if (blocks > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  const dim3 grid((unsigned)blocks), cta(RS_THREADS);
  if (chunks) AKVS_CUDA(launch_pdl(rope_scaled_kernel<T, INTER>, grid, cta, 0, st, p));
  else AKVS_CUDA(launch_pdl(rope_scaled_values_kernel<T, INTER>, grid, cta, 0, st, p));
  AKVS_LAUNCHED();
  return AKVS_OK;
}

// Turns per position of every pair, and the magnitude.
int32_t frequencies(const akvs_rope_desc& d, RopeParams& p) {
  const long double two_pi = 6.283185307179586476925286766559005768L, s = d.factor;
  const int half = d.rot_dim / 2;
  long double base = d.base;
  if (d.scaling == AKVS_ROPE_NTK) base *= powl(s, (long double)d.rot_dim / (d.rot_dim - 2));
  const long double ratio = powl(base, -2.0L / d.rot_dim);
  double first = 0, last = 1;
  if (d.scaling == AKVS_ROPE_YARN) {
    auto at = [&](double turns) { return d.rot_dim * log(d.orig_ctx / ((double)two_pi * turns)) / (2 * log((double)d.base)); };
    first = fmax(floor(at(d.high)), 0.0);
    last = fmin(ceil(at(d.low)), d.rot_dim - 1.0);
  }
  long double f = 1.0L;
  for (int i = 0; i < half; ++i, f *= ratio) {
    long double g = f;
    if (d.scaling == AKVS_ROPE_LINEAR) g = f / s;
    if (d.scaling == AKVS_ROPE_BANDS || d.scaling == AKVS_ROPE_YARN) {
      const double x = d.scaling == AKVS_ROPE_BANDS ? ((double)(d.orig_ctx * f / two_pi) - d.low) / ((double)d.high - d.low)
                                                    : 1.0 - (i - first) / fmax(last - first, 0.001);
      const double keep = fmin(fmax(x, 0.0), 1.0);
      g = f * (keep + (1 - keep) / s);
    }
    p.turns[i] = (double)(g / two_pi);
  }
  p.mag = d.magnitude != 0.f ? d.magnitude : d.scaling == AKVS_ROPE_YARN && d.factor > 1.f ? (float)(0.1 * log((double)d.factor) + 1) : 1.f;
  return AKVS_OK;
}

bool finite_positive(float x) { return x > 0.f && !isinf(x); }

}  // namespace

extern "C" int32_t akvs_op_rope_scaled(int32_t dtype, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                                       const int32_t* pos, int32_t n, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t head_dim, const akvs_rope_desc* rope, void* q_out, int64_t q_out_ld,
                                       void* k_out, int64_t k_out_ld, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (!rope || n < 0 || n_q_heads < 0 || n_kv_heads < 0 || (int64_t)n_q_heads + n_kv_heads > (1 << 20)) return AKVS_ERR_INVALID_ARG;
  if (head_dim <= 0 || head_dim % 8 || head_dim > RS_MAX_HD) return AKVS_ERR_UNSUPPORTED;
  const akvs_rope_desc& d = *rope;
  if (d.layout != AKVS_ROPE_HALF && d.layout != AKVS_ROPE_INTERLEAVED) return AKVS_ERR_UNSUPPORTED;
  if (d.scaling < AKVS_ROPE_PLAIN || d.scaling > AKVS_ROPE_YARN) return AKVS_ERR_UNSUPPORTED;
  if (d.rot_dim < 2 || d.rot_dim % 2 || d.rot_dim > head_dim || (d.scaling == AKVS_ROPE_NTK && d.rot_dim == 2)) return AKVS_ERR_SHAPE;
  if (!finite_positive(d.base) || !(d.magnitude >= 0.f) || isinf(d.magnitude)) return AKVS_ERR_INVALID_ARG;
  if (d.scaling != AKVS_ROPE_PLAIN && !finite_positive(d.factor)) return AKVS_ERR_INVALID_ARG;
  if (d.scaling == AKVS_ROPE_BANDS || d.scaling == AKVS_ROPE_YARN) {
    if (!finite_positive(d.orig_ctx) || !finite_positive(d.high) || !(d.low >= 0.f) || !(d.low < d.high)) return AKVS_ERR_INVALID_ARG;
    if (d.scaling == AKVS_ROPE_YARN && (d.low == 0.f || !(d.base > 1.f))) return AKVS_ERR_INVALID_ARG;
  }
  if (n == 0 || n_q_heads + n_kv_heads == 0) return AKVS_OK;
  if (!pos || (n_q_heads > 0 && (!q || !q_out)) || (n_kv_heads > 0 && (!k || !k_out))) return AKVS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)dtype_size(dtype);
  RopeParams p;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int64_t ld[2] = {q_ld, k_ld}, ld_out[2] = {q_out_ld, k_out_ld};
  const int heads[2] = {n_q_heads, n_kv_heads};
  bool in_place = true;
  for (int i = 0; i < 2; ++i) {
    p.x[i] = in[i]; p.y[i] = out[i]; p.ld_x[i] = ld[i]; p.ld_y[i] = ld_out[i]; p.heads[i] = heads[i];
    if (heads[i] == 0) continue;
    const int64_t row = (int64_t)heads[i] * head_dim;
    if (ld[i] < row || ld_out[i] < row) return AKVS_ERR_SHAPE;
    if (!aligned16(in[i]) || !aligned16(out[i]) || ld[i] * es % 16 || ld_out[i] * es % 16) return AKVS_ERR_INVALID_ARG;
    if (bytes_overlap(pos, n * 4ll, out[i], ((n - 1) * ld_out[i] + row) * es)) return AKVS_ERR_INVALID_ARG;
    in_place = in_place && in[i] == out[i] && ld[i] == ld_out[i];
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
  p.pos = pos; p.n = n; p.hd = head_dim; p.rot = d.rot_dim;
  AKVS_TRY(frequencies(d, p));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    return d.layout == AKVS_ROPE_HALF ? run<T, false>(p, in_place, st) : run<T, true>(p, in_place, st);
  });
}
