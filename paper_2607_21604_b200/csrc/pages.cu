// A cache in pages of 64 tokens, 4 bits a value: new K/V rows into it, values out of it, copies of pages.
//
// Quantiser, per token, kv head and group of 64 values (32-bit round-to-nearest operations, no contraction, the
// same bits as the quantiser of the unit cache in elem.cu):
//     scale = half((max - min) / 15), min16 = half(min), code = clamp(rint((x - min16) / scale), 0, 15).
// 8 lanes share a group and hold 8 values each (one 16-byte load of a 16-bit type), minimum and maximum are three
// shuffles, and a lane's codes are one word of the page.  A division per value made the kernel compute bound
// (12416 rows x 8 heads of 128: 376 instructions for 256 values, 52 us): a product with the scale's reciprocal is off
// by less than 2^-17 for quotients up to 15, so the code is decided by it unless the quotient lies within 2^-16 of the
// middle of two codes, and only then divided for (30 us; with the arithmetic in pairs of values 25.6).  Bound by issue: 180
// instructions for 256 values, at 2.5 TB/s of 6.56.  Reading the same rows back takes 21.4 us: 14 MB in, 51 MB out, 3 TB/s, bound
// by the chain offsets, page number, codes and by the sectors that half words of V of one token meet (four times its bytes, from
// L2).  A new token of 16 sequences takes 4.7 us, a launch and the same chain.  CTAs of 128 threads: 44 us for both kernels
// against 46 with 256 and 49 with 512.
#include "pages.cuh"

namespace {

constexpr int PG_THREADS = 128;

struct RowsParams {
  const void* k;
  const void* v;
  int64_t k_ld, v_ld;                       // elements between rows
  void* k_out;                              // pages_read: [R][n_kv][hd]
  void* v_out;
  int R, S, n_kv;
  const int32_t* off;                       // null: row s belongs to sequence s
  const int32_t* len;
  const int32_t* table;
  int64_t table_ld;
  int width, n_pages;
  uint8_t* pool;
  int64_t page_ld;                          // bytes between pages
  int warps_per_row;
};

// Where row r goes: its page's bytes and token within it, or null.  One warp, all lanes alike.  Offsets and length come in one
// go, a lane per sequence, so that only the page's number is read after them.
__device__ __forceinline__ uint8_t* place(const RowsParams& p, int r, int& tok) {
  const int64_t room = (int64_t)p.width * 64;
  int s = r;
  PageSeq q = {0, 0, 0};
  if (p.off) {
    const int lane = threadIdx.x & 31;
    for (int b = 0;; b += 32) {             // how many sequences end at or before r
      if (b >= p.S) return nullptr;
      const bool have = b + lane < p.S;
      if (have) q = page_sequence(p.off, p.len, b + lane, p.R, room);
      const int n = __popc(__ballot_sync(0xFFFFFFFFu, have && q.r0 + q.n <= r));
      s = b + n;
      if (n == 32) continue;
      q.r0 = __shfl_sync(0xFFFFFFFFu, q.r0, n);
      q.n = __shfl_sync(0xFFFFFFFFu, q.n, n);
      q.len = __shfl_sync(0xFFFFFFFFu, q.len, n);
      break;
    }
    if (s >= p.S) return nullptr;
  } else {
    q = page_sequence(p.off, p.len, s, p.R, room);
  }
  const int at = q.len - q.n + (r - q.r0);
  if (r < q.r0 || r >= q.r0 + q.n || at < 0) return nullptr;
  const int page = __ldcg(p.table + (int64_t)s * p.table_ld + at / 64);
  if (page < 0 || page >= p.n_pages) return nullptr;
  tok = at % 64;
  return p.pool + (int64_t)page * p.page_ld;
}

// A lane's eight values and their codes.
template <typename T> struct Eight {
  uint4 w[sizeof(T) == 4 ? 2 : 1];
  __device__ __forceinline__ void load(const T* src) {
    w[0] = __ldcs(reinterpret_cast<const uint4*>(src));
    if constexpr (sizeof(T) == 4) w[1] = __ldcs(reinterpret_cast<const uint4*>(src) + 1);
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
    if constexpr (sizeof(T) == 4) {
      x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y); x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
      x[4] = __uint_as_float(w[1].x); x[5] = __uint_as_float(w[1].y); x[6] = __uint_as_float(w[1].z); x[7] = __uint_as_float(w[1].w);
    } else {
      ld16(reinterpret_cast<const T*>(&w[0]), x);
    }
  }
};

__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float s, float m) {
  if (s == 0.f) return 0u;
  const float2 magic = make_float2(12582912.f, 12582912.f);           // 1.5 2^23: adding it rounds to whole numbers, ties to even
  const float2 minus = make_float2(-12582912.f, -12582912.f), of15 = make_float2(15.f, 15.f), m2 = make_float2(-m, -m);
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));               // (s is 2^-24 or more)
  r *= 1.f / 15.f;
  float edge = 0.f;                                   // how near a quotient comes to the middle of two codes
  float2 c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 d = __fadd2_rn(make_float2(x[2 * e], x[2 * e + 1]), m2);
    const float2 t = make_float2(__saturatef(d.x * r), __saturatef(d.y * r));       // a fifteenth of the quotient; NaN becomes 0
    c[e] = __fadd2_rn(__ffma2_rn(t, of15, magic), minus);
    const float2 off = __ffma2_rn(t, of15, make_float2(-c[e].x, -c[e].y));
    edge = fmaxf(edge, fmaxf(fabsf(off.x), fabsf(off.y)));
  }
  // whole numbers below 2^16, four codes each
  const float2 k = make_float2(256.f, 256.f), a = __ffma2_rn(c[1], k, c[0]), b = __ffma2_rn(c[3], k, c[2]);
  uint32_t word = (__float_as_uint(fmaf(a.y, 16.f, a.x) + magic.x) & 0xFFFFu) | __float_as_uint(fmaf(b.y, 16.f, b.x) + magic.x) << 16;
  if (edge > 0.5f - 0x1p-16f) {
    word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      word |= (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[e], m), s)), 0.f), 15.f) << (4 * e);
  }
  return word;
}

// An item is K or V of one kv head of a row: HD / 8 lanes.
template <typename T, int HD>
__global__ void __launch_bounds__(PG_THREADS)
pages_append_kernel(const __grid_constant__ RowsParams p) {
  using B = PageBlock<HD>;
  constexpr int LPI = HD / 8, IPW = 32 / LPI, UN = sizeof(T) == 4 ? 2 : 4;      // items of a warp at a time, steps in flight
  pdl_trigger();
  pdl_wait();
  const int64_t unit = (int64_t)blockIdx.x * (PG_THREADS / 32) + (threadIdx.x >> 5);
  if (unit >= (int64_t)p.R * p.warps_per_row) return;
  const int r = (int)(unit / p.warps_per_row), lane = threadIdx.x & 31, l = lane % LPI, g = l >> 3, i = l & 7;
  const int items = 2 * p.n_kv, stride = p.warps_per_row * IPW;
  const T* kr = reinterpret_cast<const T*>(p.k) + (int64_t)r * p.k_ld + l * 8;
  const T* vr = reinterpret_cast<const T*>(p.v) + (int64_t)r * p.v_ld + l * 8;
  uint8_t* page = nullptr;
  int tok = 0;
  bool placed = false;
  for (int first = (int)(unit % p.warps_per_row) * IPW; first < items; first += UN * stride) {
    Eight<T> in[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int it = first + u * stride + lane / LPI;
      if (it < items) in[u].load(it >= p.n_kv ? vr + (int64_t)(it - p.n_kv) * HD : kr + (int64_t)it * HD);
      else in[u] = {};
    }
    if (!placed) {                                    // while the first values are on their way
      page = place(p, r, tok);
      if (!page) return;
      placed = true;
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      if (first + u * stride >= items) break;
      const int it = first + u * stride + lane / LPI, is_v = it >= p.n_kv, h = it - is_v * p.n_kv;
      float x[8];
      in[u].values(x);
      float mn = x[0], mx = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) { mn = fminf(mn, x[e]); mx = fmaxf(mx, x[e]); }
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) {
        mn = fminf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
      }
      const __half s16 = __float2half_rn(__fdiv_rn(__fsub_rn(mx, mn), 15.f)), m16 = __float2half_rn(mn);
      const uint32_t word = codes_of(x, __half2float(s16), __half2float(m16));
      if (it >= items) continue;
      uint8_t* block = page + (int64_t)h * B::BYTES;
      if (is_v) {
        *reinterpret_cast<uint16_t*>(block + B::v_half(tok, g, i, 0)) = (uint16_t)word;
        *reinterpret_cast<uint16_t*>(block + B::v_half(tok, g, i, 1)) = (uint16_t)(word >> 16);
      } else {
        *reinterpret_cast<uint32_t*>(block + B::k_word(tok, g, i)) = word;
      }
      if (i == 0) *reinterpret_cast<__half2*>(block + B::record(is_v, tok, g)) = __halves2half2(s16, m16);
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(PG_THREADS)
pages_read_kernel(const __grid_constant__ RowsParams p) {
  using B = PageBlock<HD>;
  constexpr int LPI = HD / 8, IPW = 32 / LPI;
  pdl_trigger();
  pdl_wait();
  const int64_t unit = (int64_t)blockIdx.x * (PG_THREADS / 32) + (threadIdx.x >> 5);
  if (unit >= (int64_t)p.R * p.warps_per_row) return;
  const int r = (int)(unit / p.warps_per_row), lane = threadIdx.x & 31, l = lane % LPI, g = l >> 3, i = l & 7;
  int tok = 0;
  const uint8_t* page = place(p, r, tok);
  if (!page) return;
  constexpr int UN = 4, V = VecOf<T>::N;              // items of a lane in flight
  const int items = 2 * p.n_kv, stride = p.warps_per_row * IPW;
  for (int first = (int)(unit % p.warps_per_row) * IPW + lane / LPI; first < items; first += UN * stride) {
    uint32_t word[UN], rec[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int it = first + u * stride, is_v = it >= p.n_kv, h = it - is_v * p.n_kv;
      if (it >= items) break;
      const uint8_t* block = page + (int64_t)h * B::BYTES;
      word[u] = is_v ? __ldcg(reinterpret_cast<const uint16_t*>(block + B::v_half(tok, g, i, 0))) |
                           (uint32_t)__ldcg(reinterpret_cast<const uint16_t*>(block + B::v_half(tok, g, i, 1))) << 16
                     : __ldcg(reinterpret_cast<const uint32_t*>(block + B::k_word(tok, g, i)));
      rec[u] = __ldcg(reinterpret_cast<const uint32_t*>(block + B::record(is_v, tok, g)));
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int it = first + u * stride, is_v = it >= p.n_kv, h = it - is_v * p.n_kv;
      if (it >= items) break;
      const float2 sm = __half22float2(*reinterpret_cast<const __half2*>(&rec[u]));
      T* dst = reinterpret_cast<T*>(is_v ? p.v_out : p.k_out) + ((int64_t)r * p.n_kv + h) * HD + l * 8;
#pragma unroll
      for (int c = 0; c < 8; c += V) {
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = fmaf((float)((word[u] >> (4 * (c + e))) & 15u), sm.x, sm.y);
        st16_inf(dst + c, y);                         // (a record's minimum may be infinite)
      }
    }
  }
}

constexpr int CP_THREADS = 256, CP_UNROLL = 4;

// grid (pieces of a page, pairs, layers)
__global__ void __launch_bounds__(CP_THREADS)
pages_copy_kernel(uint8_t* pool, int64_t layer_ld, int64_t page_ld, int64_t page_bytes, int n_pages, const int32_t* src,
                  const int32_t* dst, int n_layers) {
  pdl_trigger();
  pdl_wait();
  const int a = __ldcg(src + blockIdx.y), b = __ldcg(dst + blockIdx.y);
  if (a < 0 || b < 0 || a >= n_pages || b >= n_pages || a == b) return;
  const int64_t at = ((int64_t)blockIdx.x * CP_UNROLL * CP_THREADS + threadIdx.x) * 16;
  for (int l = blockIdx.z; l < n_layers; l += gridDim.z) {
    const uint8_t* x = pool + l * layer_ld + a * page_ld + at;
    uint8_t* y = pool + l * layer_ld + b * page_ld + at;
    uint4 w[CP_UNROLL];
#pragma unroll
    for (int i = 0; i < CP_UNROLL; ++i)
      if (at + i * CP_THREADS * 16 < page_bytes) w[i] = __ldcs(reinterpret_cast<const uint4*>(x + i * CP_THREADS * 16));
#pragma unroll
    for (int i = 0; i < CP_UNROLL; ++i)
      if (at + i * CP_THREADS * 16 < page_bytes) __stcs(reinterpret_cast<uint4*>(y + i * CP_THREADS * 16), w[i]);
  }
}

int32_t block_bytes(int hd) { return hd == 64 ? PageBlock<64>::BYTES : PageBlock<128>::BYTES; }

// What append and read have in common: `p` but for the tensors, and its checks.
int32_t rows_params(RowsParams& p, int32_t R, int32_t S, const int32_t* off, const int32_t* len, const int32_t* table,
                    int64_t table_ld, int32_t width, int32_t n_pages, int32_t n_kv, int32_t hd, const void* pool, int64_t page_ld) {
  if (R < 0 || S < 0 || width < 0 || n_pages < 0) return AKVS_ERR_INVALID_ARG;
  if (n_kv <= 0 || n_kv > 65535) return AKVS_ERR_SHAPE;
  if (hd != 64 && hd != 128) return AKVS_ERR_UNSUPPORTED;
  if (!off && R < S) return AKVS_ERR_SHAPE;
  if (R == 0 || S == 0) return AKVS_OK;
  if (!len || (width > 0 && !table) || (n_pages > 0 && !pool)) return AKVS_ERR_INVALID_ARG;
  if (table_ld < width || (n_pages > 0 && page_ld < (int64_t)n_kv * block_bytes(hd))) return AKVS_ERR_SHAPE;
  if (!aligned16(pool) || page_ld % 16) return AKVS_ERR_INVALID_ARG;
  p.R = off ? R : S; p.S = S; p.n_kv = n_kv; p.off = off; p.len = len; p.table = table; p.table_ld = table_ld; p.width = width;
  p.n_pages = n_pages; p.page_ld = page_ld;
  return AKVS_OK;
}

// Warps of a row: few rows are spread over the SMs, many take two items a warp's lane group.
int warps_per_row(int R, int n_kv, int hd) {
  const int steps = akvs_cdiv(2 * n_kv, 32 / (hd / 8));
  int w = steps;
  while (w > 1 && (int64_t)R * w >= 148 * 64) w = (w + 1) / 2;
  return w;
}

}  // namespace

extern "C" int64_t akvs_page_bytes(int32_t n_kv_heads, int32_t head_dim) {
  if (n_kv_heads <= 0 || n_kv_heads > 65535 || (head_dim != 64 && head_dim != 128)) return -1;
  return (int64_t)n_kv_heads * block_bytes(head_dim);
}

extern "C" int32_t akvs_op_pages_append(int32_t dtype, const void* k, int64_t k_ld, const void* v, int64_t v_ld, int32_t R,
                                        const int32_t* row_off, const int32_t* seq_len, int32_t S, const int32_t* table,
                                        int64_t table_ld, int32_t width, int32_t n_kv_heads, int32_t head_dim, void* pool,
                                        int64_t page_ld, int32_t n_pages, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  RowsParams p = {};
  AKVS_TRY(rows_params(p, R, S, row_off, seq_len, table, table_ld, width, n_pages, n_kv_heads, head_dim, pool, page_ld));
  if (R == 0 || S == 0 || width == 0 || n_pages == 0) return AKVS_OK;
  if (!k || !v) return AKVS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)dtype_size(dtype), row = (int64_t)n_kv_heads * head_dim;
  if (k_ld < row || v_ld < row) return AKVS_ERR_SHAPE;
  if (!aligned16(k) || !aligned16(v) || k_ld * es % 16 || v_ld * es % 16) return AKVS_ERR_INVALID_ARG;
  const int64_t bytes = (n_pages - 1) * page_ld + n_kv_heads * block_bytes(head_dim);
  const void* ins[5] = {k, v, row_off, seq_len, table};
  const int64_t in_n[5] = {((p.R - 1) * k_ld + row) * es, ((p.R - 1) * v_ld + row) * es, row_off ? (S + 1) * 4ll : 0, S * 4ll,
                           ((S - 1) * table_ld + width) * 4};
  for (int i = 0; i < 5; ++i)
    if (bytes_overlap(ins[i], in_n[i], pool, bytes)) return AKVS_ERR_INVALID_ARG;
  p.k = k; p.v = v; p.k_ld = k_ld; p.v_ld = v_ld; p.pool = reinterpret_cast<uint8_t*>(pool);
  p.warps_per_row = warps_per_row(p.R, n_kv_heads, head_dim);
  const int64_t blocks = ((int64_t)p.R * p.warps_per_row + PG_THREADS / 32 - 1) / (PG_THREADS / 32);
  if (blocks > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    const dim3 grid((unsigned)blocks), cta(PG_THREADS);
    if (head_dim == 64) AKVS_CUDA(launch_pdl(pages_append_kernel<T, 64>, grid, cta, 0, st, p));
    else AKVS_CUDA(launch_pdl(pages_append_kernel<T, 128>, grid, cta, 0, st, p));
    AKVS_LAUNCHED();
    return AKVS_OK;
  });
}

extern "C" int32_t akvs_op_pages_read(int32_t dtype, const void* pool, int64_t page_ld, int32_t n_pages, const int32_t* table,
                                      int64_t table_ld, int32_t width, const int32_t* row_off, const int32_t* seq_len, int32_t S,
                                      int32_t R, int32_t n_kv_heads, int32_t head_dim, void* k_out, void* v_out, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  RowsParams p = {};
  AKVS_TRY(rows_params(p, R, S, row_off, seq_len, table, table_ld, width, n_pages, n_kv_heads, head_dim, pool, page_ld));
  if (R == 0 || S == 0 || width == 0 || n_pages == 0) return AKVS_OK;
  if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return AKVS_ERR_INVALID_ARG;
  const int64_t out_n = (int64_t)R * n_kv_heads * head_dim * (int64_t)dtype_size(dtype);
  const void* ins[4] = {pool, row_off, seq_len, table};
  const int64_t in_n[4] = {(n_pages - 1) * page_ld + n_kv_heads * block_bytes(head_dim), row_off ? (S + 1) * 4ll : 0, S * 4ll,
                           ((S - 1) * table_ld + width) * 4};
  for (int i = 0; i < 4; ++i)
    if (bytes_overlap(ins[i], in_n[i], k_out, out_n) || bytes_overlap(ins[i], in_n[i], v_out, out_n)) return AKVS_ERR_INVALID_ARG;
  if (bytes_overlap(k_out, out_n, v_out, out_n)) return AKVS_ERR_INVALID_ARG;
  p.k_out = k_out; p.v_out = v_out; p.pool = reinterpret_cast<uint8_t*>(const_cast<void*>(pool));
  p.warps_per_row = warps_per_row(p.R, n_kv_heads, head_dim);
  const int64_t blocks = ((int64_t)p.R * p.warps_per_row + PG_THREADS / 32 - 1) / (PG_THREADS / 32);
  if (blocks > 0x7fffffff) return AKVS_ERR_TOO_LARGE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dispatch_dtype(dtype, [&](auto tag) -> int32_t {
    using T = decltype(tag);
    const dim3 grid((unsigned)blocks), cta(PG_THREADS);
    if (head_dim == 64) AKVS_CUDA(launch_pdl(pages_read_kernel<T, 64>, grid, cta, 0, st, p));
    else AKVS_CUDA(launch_pdl(pages_read_kernel<T, 128>, grid, cta, 0, st, p));
    AKVS_LAUNCHED();
    return AKVS_OK;
  });
}

extern "C" int32_t akvs_op_pages_copy(void* pool, int64_t layer_ld, int64_t page_ld, int64_t page_bytes, int32_t n_layers,
                                      int32_t n_pages, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  if (n_layers < 0 || n_pages < 0 || n < 0 || page_bytes < 0) return AKVS_ERR_INVALID_ARG;
  if (n == 0 || n_layers == 0 || n_pages == 0 || page_bytes == 0) return AKVS_OK;
  if (!pool || !src || !dst) return AKVS_ERR_INVALID_ARG;
  if (page_ld < page_bytes || (n_layers > 1 && layer_ld < (n_pages - 1) * page_ld + page_bytes)) return AKVS_ERR_SHAPE;
  if (!aligned16(pool) || page_ld % 16 || page_bytes % 16 || (n_layers > 1 && layer_ld % 16)) return AKVS_ERR_INVALID_ARG;
  const int64_t bytes = (n_layers > 1 ? (n_layers - 1) * layer_ld : 0) + (n_pages - 1) * page_ld + page_bytes;
  if (bytes_overlap(src, n * 4ll, pool, bytes) || bytes_overlap(dst, n * 4ll, pool, bytes)) return AKVS_ERR_INVALID_ARG;
  const int64_t pieces = (page_bytes + CP_UNROLL * CP_THREADS * 16 - 1) / (CP_UNROLL * CP_THREADS * 16);
  if (pieces > 0x7fffffff || n > 65535) return AKVS_ERR_TOO_LARGE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)pieces, (unsigned)n, (unsigned)(n_layers < 65535 ? n_layers : 65535));
  AKVS_CUDA(launch_pdl(pages_copy_kernel, grid, dim3(CP_THREADS), 0, st, reinterpret_cast<uint8_t*>(pool), layer_ld, page_ld, page_bytes,
                       n_pages, src, dst, n_layers));
  AKVS_LAUNCHED();
  return AKVS_OK;
}
