// Attention weight that every cached key has received: per kv head h and key j
//     mass_out[h][j] = mass_in[h][j] + sum over rows r that see j, heads i of the group of h:
//                      exp(q_ri . k_jh / sqrt(hd) - lse_ri)
// with lse the log-sum-exp of the row, as the attention that produced the row left it.
// The rows of the g = n_q / n_kv query heads of a kv head are stacked (r * g + i); every sum runs
// over them in a fixed order, so equal calls give equal bits.
#include "common.cuh"
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
    return head_dim == 64 ? run_simt<E, 64>(p, st) : run_simt<E, 128>(p, st);
  });
}
