// Eviction from a cache by accumulated attention weight.  Per layer and kv head the first
// `n_sink` and the last `n_recent` tokens stay, and of the others the heaviest until `budget`
// tokens are kept (ties to the smaller index); the kept tokens' K, V and mass are packed in
// ascending token order.
//
// One launch: a cluster of C CTAs owns one (layer, head) row of masses, keeps it in shared memory as
// order-preserving 32-bit keys, and fixes the key of the last kept token in four passes of 8 bits;
// the 256-bin histograms of the CTAs are added up through distributed shared memory.  Counts of
// greater and equal keys per warp then give every kept token its place without a sort, and the
// cluster moves its head's K/V of the kept tokens, 16 bytes per lane, an equal share per CTA.
// Selection is latency bound (a row is read once from memory), so a call with few rows spreads
// each over up to 8 SMs; the copies are memory bound and nearly all of the operator's bytes.
// 8 heads of 128, 16 bits: 32 layers, 12416 to 4096 tokens, 214 us (5.1 TB/s over all, 5.7 in the copies);
// one layer, 8320 to 2048 tokens, 16.7 us (15.2 us from L2), of which the selection is 9 us.
#include "tc_common.cuh"

namespace {

constexpr int SEL_THREADS = 512, SEL_WARPS = SEL_THREADS / 32;
static_assert(SEL_THREADS >= 256, "a thread per bin");
constexpr int COPY_UN = 4;                         // tokens of a lane in flight
constexpr int SEL_MAX_C = 8;                       // portable cluster size (16 measured slower: 17.3 against 15.2 us on a layer)
constexpr int SEL_MAX_SEG = 50 * 1024;             // keys of a CTA's shared memory (200 KB, beside 18 KB of counts)

// Order of the masses as unsigned integers: greater mass, greater key; -0 equals +0, NaN is the
// smallest of all, so that a broken mass is the first to go.
__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return 0u;
  const uint32_t u = __float_as_uint(m + 0.f);     // -0 + 0 = +0
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_mass(uint32_t k) {
  return k == 0u ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float((k >> 31) ? (k & 0x7FFFFFFFu) : ~k);
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

template <bool CACHED>
__global__ void __launch_bounds__(SEL_THREADS)
evict_kernel(const float* __restrict__ mass, int T, int n_sink, int n_recent, int budget, int seg, int32_t* idx,
             float* __restrict__ mass_out, const uint4* __restrict__ k, const uint4* __restrict__ v, int n_kv, int log_cph,
             int64_t layer_ld, int64_t tok_ld, uint4* __restrict__ k_out, uint4* __restrict__ v_out) {
  extern __shared__ uint32_t keys[];               // [seg] when CACHED
  __shared__ uint32_t hist[2][256];                // this CTA's counts, read by the cluster
  __shared__ uint32_t sub[SEL_WARPS][256];         // a warp's own: masses share exponents, and bins would be fought over
  __shared__ uint32_t warp_part[SEL_WARPS];
  __shared__ uint32_t found[3];                    // bin, keys still wanted from it, keys in it
  __shared__ uint32_t cnt[2];                      // this CTA's kept-for-sure and tied tokens
  __shared__ uint32_t w_sure[SEL_WARPS], w_tied[SEL_WARPS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int C = gridDim.x;
  const uint32_t rank = tc::cluster_ctarank();
  const int row = blockIdx.y;
  const int t0 = min((int64_t)rank * seg, (int64_t)T), t1 = min((int64_t)t0 + seg, (int64_t)T);
  const int n = t1 - t0;
  pdl_trigger();
  pdl_wait();
  const float* m = mass + (int64_t)row * T + t0;
  if (CACHED) {
#pragma unroll 8
    for (int i = tid; i < n; i += SEL_THREADS) keys[i] = mass_key(__ldg(m + i));
  }
  auto key = [&](int i) { return CACHED ? keys[i] : mass_key(__ldg(m + i)); };
  auto sync_cluster = [&]() {
    if (C > 1) tc::cluster_sync_all();
    else __syncthreads();
  };
  const int from = max(n_sink - t0, 0), to = min(T - n_recent - t0, n);    // candidates of this CTA

  uint32_t want = (uint32_t)(budget - n_sink - n_recent);
  uint32_t prefix = 0, mask = 0;
  for (int i = tid; i < SEL_WARPS * 256; i += SEL_THREADS) (&sub[0][0])[i] = 0;
  __syncthreads();
  if (want > 0) {                                  // the same in all CTAs of the cluster
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      uint32_t* hb = hist[pass & 1];
      // the loads of a batch before its counting: a key at a time, each would wait for the one before
      constexpr int UN = 8;
      for (int j0 = from + tid; j0 < to; j0 += UN * SEL_THREADS) {
        uint32_t kx[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) kx[u] = key(min(j0 + u * SEL_THREADS, to - 1));
#pragma unroll
        for (int u = 0; u < UN; ++u)
          if (j0 + u * SEL_THREADS < to && (kx[u] & mask) == prefix) atomicAdd(&sub[warp][(kx[u] >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < SEL_WARPS; ++w) { sum += sub[w][tid]; sub[w][tid] = 0; }
        hb[tid] = sum;
      }
      sync_cluster();
      // total of each bin, greatest bin first: thread i holds bin 255 - i
      uint32_t total = 0;
      if (tid < 256) {
        const uint32_t a = tc::smem_u32(&hb[255 - tid]);
        uint32_t part[SEL_MAX_C];
#pragma unroll
        for (int c = 0; c < SEL_MAX_C; ++c) part[c] = c < C ? ld_cluster(tc::map_to_rank(a, c)) : 0u;
#pragma unroll
        for (int c = 0; c < SEL_MAX_C; ++c) total += part[c];
      }
      uint32_t incl = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += up;
      }
      if (lane == 31) warp_part[warp] = incl;
      __syncthreads();
      if (tid < 256) {
#pragma unroll
        for (int w = 0; w < 7; ++w) incl += w < warp ? warp_part[w] : 0u;
        if (incl >= want && incl - total < want) {
          found[0] = 255 - tid;
          found[1] = want - (incl - total);
          found[2] = total;
        }
      }
      __syncthreads();
      prefix |= found[0] << shift;
      mask |= 255u << shift;
      want = found[1];
      if (want == found[2]) break;                 // the whole bin stays: its other bits do not matter
    }
  }
  // kept: keys whose masked bits are above `cut`, and the first `ties` of those that equal it
  if (budget == n_sink + n_recent) mask = 0xFFFFFFFFu;
  const uint32_t cut = budget > n_sink + n_recent ? prefix : 0xFFFFFFFFu;   // no key is all ones
  const uint32_t ties = budget > n_sink + n_recent ? want : 0u;

  // every warp owns a run of consecutive tokens: count, exchange, then place
  const int per = (seg + SEL_THREADS - 1) / SEL_THREADS * 32;
  const int a = min(warp * per, n), b = min(a + per, n);
  // bit 0: kept for sure; bit 1: tied with the last kept one
  auto look = [&](int i, uint32_t& kx) {
    const int j = i + lane, t = t0 + j;
    kx = key(min(j, n - 1));
    const bool in = j < b, f = (t < n_sink) | (t >= T - n_recent);
    return (in & (f | ((kx & mask) > cut)) ? 1 : 0) | (in & !f & ((kx & mask) == cut) ? 2 : 0);
  };
  uint32_t sure = 0, tied = 0;
#pragma unroll 8
  for (int i = a; i < b; i += 32) {
    uint32_t kx;
    const int is = look(i, kx);
    sure += __popc(__ballot_sync(0xFFFFFFFFu, is & 1));
    tied += __popc(__ballot_sync(0xFFFFFFFFu, is & 2));
  }
  if (lane == 0) { w_sure[warp] = sure; w_tied[warp] = tied; }
  __syncthreads();
  if (warp == 0) {
    const uint32_t s = __reduce_add_sync(0xFFFFFFFFu, lane < SEL_WARPS ? w_sure[lane] : 0u);
    const uint32_t t = __reduce_add_sync(0xFFFFFFFFu, lane < SEL_WARPS ? w_tied[lane] : 0u);
    if (lane == 0) { cnt[0] = s; cnt[1] = t; }
  }
  sync_cluster();
  uint32_t before_s = 0, before_t = 0;
  // lane c holds the counts of CTA c, then of warp c
  if (lane < (int)rank) {
    before_s = ld_cluster(tc::map_to_rank(tc::smem_u32(&cnt[0]), lane));
    before_t = ld_cluster(tc::map_to_rank(tc::smem_u32(&cnt[1]), lane));
  }
  if (lane < warp) { before_s += w_sure[lane]; before_t += w_tied[lane]; }
  before_s = __reduce_add_sync(0xFFFFFFFFu, before_s);
  before_t = __reduce_add_sync(0xFFFFFFFFu, before_t);
  int32_t* out = idx + (int64_t)row * budget;
  float* mo = mass_out + (int64_t)row * budget;
#pragma unroll 8
  for (int i = a; i < b; i += 32) {
    uint32_t kx;
    const int is = look(i, kx);
    const uint32_t bs = __ballot_sync(0xFFFFFFFFu, is & 1), bt = __ballot_sync(0xFFFFFFFFu, is & 2);
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t my_s = before_s + __popc(bs & below), my_t = before_t + __popc(bt & below);
    if ((is & 1) | ((is & 2) != 0 & my_t < ties)) {
      const uint32_t at = my_s + min(my_t, ties);
      out[at] = t0 + i + lane;
      mo[at] = key_mass(kx);
    }
    before_s += __popc(bs);
    before_t += __popc(bt);
  }
  sync_cluster();                                  // every CTA's indices are written, and its counts read

  // this CTA's share of the kept tokens: lanes of a head's 16-byte chunks, COPY_UN tokens each
  const int l = row / n_kv, h = row % n_kv, cph = 1 << log_cph, tpw = 32 >> log_cph;
  const int b0 = (int)((int64_t)budget * rank / C), b1 = (int)((int64_t)budget * (rank + 1) / C);
  const int64_t src0 = l * layer_ld + (int64_t)h * cph + (lane & (cph - 1));
  const int64_t dst0 = ((int64_t)l * budget * n_kv + h) * cph + (lane & (cph - 1));
  for (int t = b0 + warp * tpw + (lane >> log_cph); t < b1; t += SEL_WARPS * tpw * COPY_UN) {
    uint4 x[COPY_UN], y[COPY_UN];
#pragma unroll
    for (int u = 0; u < COPY_UN; ++u) {
      const int tu = t + u * SEL_WARPS * tpw;
      if (tu < b1) {
        const int64_t at = src0 + (int64_t)__ldcg(out + tu) * tok_ld;
        x[u] = __ldcs(k + at);
        y[u] = __ldcs(v + at);
      }
    }
#pragma unroll
    for (int u = 0; u < COPY_UN; ++u) {
      const int tu = t + u * SEL_WARPS * tpw;
      if (tu < b1) {
        const int64_t at = dst0 + (int64_t)tu * n_kv * cph;
        __stcs(k_out + at, x[u]);
        __stcs(v_out + at, y[u]);
      }
    }
  }
}

}  // namespace

extern "C" int32_t akvs_op_evict(int32_t dtype, const float* mass, const void* k, const void* v, int64_t layer_ld,
                                 int64_t tok_ld, int32_t n_layers, int32_t T, int32_t n_kv_heads, int32_t head_dim,
                                 int32_t budget, int32_t n_sink, int32_t n_recent, int32_t* idx, void* k_out,
                                 void* v_out, float* mass_out, void* stream) {
  if (dtype != AKVS_F32 && dtype != AKVS_BF16 && dtype != AKVS_F16) return AKVS_ERR_UNSUPPORTED;
  if (n_layers < 0 || T < 0 || n_kv_heads <= 0 || budget < 0 || n_sink < 0 || n_recent < 0) return AKVS_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return AKVS_ERR_UNSUPPORTED;
  if (budget > T || (int64_t)n_sink + n_recent > budget) return AKVS_ERR_SHAPE;
  if (n_layers == 0 || budget == 0) return AKVS_OK;
  if (!mass || !k || !v || !idx || !k_out || !v_out || !mass_out) return AKVS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)dtype_size(dtype), row = (int64_t)n_kv_heads * head_dim;
  if (tok_ld < row || layer_ld < 0 || (n_layers > 1 && layer_ld < (T - 1) * tok_ld + row)) return AKVS_ERR_SHAPE;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_out) || !aligned16(v_out) || tok_ld * es % 16 || layer_ld * es % 16)
    return AKVS_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)n_layers * n_kv_heads;
  if (rows > 65535 || n_layers > 65535) return AKVS_ERR_TOO_LARGE;
  const int64_t in_bytes = ((n_layers - 1) * layer_ld + (int64_t)(T - 1) * tok_ld + row) * es;
  const void* ins[3] = {mass, k, v};
  const int64_t in_n[3] = {rows * T * 4, in_bytes, in_bytes};
  const void* outs[4] = {idx, k_out, v_out, mass_out};
  const int64_t out_n[4] = {rows * budget * 4, n_layers * budget * row * es, n_layers * budget * row * es, rows * budget * 4};
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < 3; ++i)
      if (bytes_overlap(ins[i], in_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
    for (int i = 0; i < o; ++i)
      if (bytes_overlap(outs[i], out_n[i], outs[o], out_n[o])) return AKVS_ERR_INVALID_ARG;
  }
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  static std::atomic<uint64_t> smem_set{0};
  AKVS_CUDA(smem_opt_in((const void*)evict_kernel<true>, SEL_MAX_SEG * 4, smem_set));
  // Rows are spread over clusters while SMs would idle and a CTA's share is still worth it (512
  // keys), and as far as the keys need the room; beyond that they are re-read from memory.
  int C = 1;
  while (C < SEL_MAX_C && ((rows * C * 2 <= 148 && T / C > 1024) || akvs_cdiv(T, C) > SEL_MAX_SEG)) C *= 2;
  const int seg = akvs_cdiv(T, C);
  const bool cached = seg <= SEL_MAX_SEG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C, (unsigned)rows);
  cfg.blockDim = dim3(SEL_THREADS);
  cfg.dynamicSmemBytes = cached ? (size_t)seg * 4 : 0;
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
  const int64_t cph = head_dim * es / 16;              // 8, 16 or 32 chunks of a head
  const int log_cph = cph == 8 ? 3 : cph == 16 ? 4 : 5;
  AKVS_CUDA(cudaLaunchKernelEx(&cfg, cached ? evict_kernel<true> : evict_kernel<false>, mass, (int)T, (int)n_sink,
                               (int)n_recent, (int)budget, seg, idx, mass_out, (const uint4*)k, (const uint4*)v,
                               (int)n_kv_heads, log_cph, layer_ld * es / 16, tok_ld * es / 16, (uint4*)k_out, (uint4*)v_out));
  AKVS_LAUNCHED();
  return AKVS_OK;
}
