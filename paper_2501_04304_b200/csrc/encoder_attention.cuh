// Attention with full-precision scores over an encoder's states and over a paged 8-bit cache:
//
//     O_i = sum_j w_ij V_j / sum_j w_ij,   w_ij = 2^(t_ij - m_i),   t_ij = log2(e) scale Q_i . K_j,   m_i >= max_j t_ij
//
// over the keys that row i sees; a row that sees none gives zeros.
#pragma once

#include "kv_cache.cuh"
#include "self_attention.cuh"

namespace dgq {

struct EncAttnArgs {
  dgq_rows Q, K, V, O;          // strides of dimensions of size 1 are 0
  int B, Hq, Hkv, nq, nk, d;    // nq: most queries of a request; nk: most keys
  float scale_log2;             // log2(e) * scale
  const int32_t* kv_lens;       // dev [B] or null (all nk)
  // the cache (K and V above unused)
  const int8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  int n_pages, page, max_pages;
  const int32_t* table;         // dev [B, max_pages]
  const int32_t* q_start;       // dev [B + 1] or null (nq queries each)
  int64_t n_rows;
  int causal;
};

// What a block needs to know of its request.
struct EncRequest {
  int nq, len;       // queries, keys
  int64_t q_row;     // first row of Q and O, where they are packed
};
__device__ __forceinline__ EncRequest enc_request(const EncAttnArgs& a, int b) {
  EncRequest r;
  r.nq = a.nq;
  r.q_row = 0;
  r.len = a.kv_lens ? min(max(a.kv_lens[b], 0), a.nk) : a.nk;
  if (a.q_start) {
    const int64_t s = a.q_start[b], e = a.q_start[b + 1];
    const int64_t first = min(max(s, (int64_t)0), a.n_rows);
    const int64_t n = min(max(e - first, (int64_t)0), a.n_rows - first);
    r.q_row = first;
    r.nq = (int)min(n, (int64_t)a.nq);
    if (s < 0 || e < s || r.nq != e - s) record_error(DGQ_ERR_INVALID_ARG);
  }
  return r;
}
// Keys that query i of the request sees.
__device__ __forceinline__ int enc_sees(const EncAttnArgs& a, const EncRequest& r, int i) {
  return a.causal ? max(r.len - r.nq + i + 1, 0) : r.len;
}

// One warp for one query row and head: a lane has a key of 32 for the scores, every 32nd feature for the product.
template <bool BF, bool CACHED>
__global__ void __launch_bounds__(128) enc_attn_rows_kernel(const __grid_constant__ EncAttnArgs a) {
  __shared__ float sq[4][KV_MAX_D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t at = (int64_t)blockIdx.x * 4 + warp;
  pdl_launch_dependents();
  pdl_wait();
  if (at >= (int64_t)a.B * a.nq * a.Hq) return;
  const int h = (int)(at % a.Hq), i = (int)(at / a.Hq % a.nq), b = (int)(at / a.Hq / a.nq);
  const int g = h / (a.Hq / a.Hkv);
  const EncRequest rq = enc_request(a, b);
  if (i >= rq.nq) return;
  const uint16_t* q = (const uint16_t*)a.Q.ptr + b * a.Q.batch + (rq.q_row + i) * a.Q.token + h * a.Q.head;
  for (int u = lane; u < a.d / 2; u += 32) {
    const float2 f = unpack16<BF>(reinterpret_cast<const uint32_t*>(q)[u]);
    sq[warp][2 * u] = f.x;
    sq[warp][2 * u + 1] = f.y;
  }
  __syncwarp();
  const int sees = enc_sees(a, rq, i), row_bytes = kv_row_bytes(a.d);
  float o[(KV_MAX_D + 31) / 32] = {};
  float m = -INFINITY, z = 0.f;
  for (int j0 = 0; j0 < sees; j0 += 32) {
    const int j = j0 + lane;
    bool real = j < sees;
    float t = -INFINITY, vs = 1.f;
    const int8_t* vc = nullptr;
    if (CACHED) {
      const int p = real ? a.table[(int64_t)b * a.max_pages + j / a.page] : 0;
      if (p < 0 || p >= a.n_pages) {
        real = false;
        record_error(DGQ_ERR_INVALID_ARG);
      }
      if (real) {
        const int64_t ph = (int64_t)p * a.Hkv + g;
        const int8_t* kc = a.k_codes + (ph * a.page + j % a.page) * row_bytes;
        vc = a.v_codes + (ph * a.page + j % a.page) * row_bytes;
        float dot = 0.f;
        for (int c = 0; c < a.d; ++c) dot = fmaf(sq[warp][c], (float)kc[c], dot);
        t = dot * (a.k_scale[ph] * a.scale_log2);
        vs = a.v_scale[ph];
      }
    } else if (real) {
      const uint32_t* k = (const uint32_t*)((const uint16_t*)a.K.ptr + b * a.K.batch + (int64_t)j * a.K.token + g * a.K.head);
      float dot = 0.f;
      for (int c = 0; c < a.d / 2; ++c) {
        const float2 f = unpack16<BF>(k[c]);
        dot = fmaf(sq[warp][2 * c], f.x, dot);
        dot = fmaf(sq[warp][2 * c + 1], f.y, dot);
      }
      t = dot * a.scale_log2;
    }
    float top = t;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    const float m1 = fmaxf(m, top);
    const float base = m1 == -INFINITY ? 0.f : m1;
    const float p = real ? exp2f(t - base) : 0.f;
    const float fall = m == -INFINITY ? 0.f : exp2f(m - base);
    m = m1;
    z = z * fall + p;
#pragma unroll
    for (int e = 0; e < (KV_MAX_D + 31) / 32; ++e) o[e] *= fall;
    const unsigned some = __ballot_sync(0xFFFFFFFFu, real);
    for (int jj = 0; jj < 32; ++jj) {
      if (!(some >> jj & 1)) continue;
      const float w = __shfl_sync(0xFFFFFFFFu, p * vs, jj);
      const int8_t* c8 = (const int8_t*)__shfl_sync(0xFFFFFFFFu, (unsigned long long)vc, jj);
      const uint16_t* v = CACHED ? nullptr : (const uint16_t*)a.V.ptr + b * a.V.batch + (int64_t)(j0 + jj) * a.V.token + g * a.V.head;
#pragma unroll
      for (int e = 0; e < (KV_MAX_D + 31) / 32; ++e)
        if (lane + 32 * e < a.d) o[e] = fmaf(w, CACHED ? (float)c8[lane + 32 * e] : unpack16<BF>((uint32_t)v[lane + 32 * e]).x, o[e]);
    }
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, x);
  uint16_t* out = (uint16_t*)a.O.ptr + b * a.O.batch + (rq.q_row + i) * a.O.token + h * a.O.head;
#pragma unroll
  for (int e = 0; e < (KV_MAX_D + 31) / 32; ++e)
    if (lane + 32 * e < a.d) out[lane + 32 * e] = (uint16_t)pack16<BF>(z == 0.f ? 0.f : o[e] / z, 0.f);
}

template <bool BF, bool CACHED>
static dgq_status enc_attn_launch(const EncAttnArgs& a, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.nq * a.Hq;
  if (rows / 4 >= INT_MAX) return DGQ_ERR_UNSUPPORTED;
  DGQ_CUDA_OK(launch_pdl(enc_attn_rows_kernel<BF, CACHED>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, stream, a));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

}  // namespace dgq

extern "C" dgq_status dgq_encoder_attn(const dgq_rows* Q, const dgq_rows* K, const dgq_rows* V, const dgq_rows* O,
                                       int dtype, int B, int Hq, int Hkv, int nq, int nk, int d, float scale,
                                       const int32_t* kv_lens, void* stream) {
  using namespace dgq;
  if (!rows_pointer_ok(Q) || !rows_pointer_ok(K) || !rows_pointer_ok(V) || !rows_pointer_ok(O) || B <= 0 || Hq <= 0 || Hkv <= 0 ||
      nq <= 0 || nk <= 0 || d <= 0 || Hq % Hkv || (dtype != DGQ_F16 && dtype != DGQ_BF16) || !std::isfinite(scale))
    return DGQ_ERR_INVALID_ARG;
  if (d % 8 || d > KV_MAX_D) return DGQ_ERR_UNSUPPORTED;
  dgq_status st;
  if ((st = rows_check(*Q, B, nq, Hq, false)) != DGQ_OK || (st = rows_check(*K, B, nk, Hkv, false)) != DGQ_OK ||
      (st = rows_check(*V, B, nk, Hkv, false)) != DGQ_OK || (st = rows_check(*O, B, nq, Hq, true)) != DGQ_OK)
    return st;
  EncAttnArgs a = {};
  a.Q = rows_normal(*Q, B, nq, Hq);
  a.K = rows_normal(*K, B, nk, Hkv);
  a.V = rows_normal(*V, B, nk, Hkv);
  a.O = rows_normal(*O, B, nq, Hq);
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.nq = nq;
  a.nk = nk;
  a.d = d;
  a.scale_log2 = (float)(1.4426950408889634 * (double)scale);
  a.kv_lens = kv_lens;
  return dtype == DGQ_BF16 ? enc_attn_launch<true, false>(a, (cudaStream_t)stream) : enc_attn_launch<false, false>(a, (cudaStream_t)stream);
}

extern "C" dgq_status dgq_cached_attn(const dgq_kv_cache* cache, const dgq_rows* Q, const dgq_rows* O, int dtype, int B,
                                      int Hq, int64_t n_rows, const int32_t* q_start, int max_nq, const int32_t* block_table,
                                      int max_pages, const int32_t* kv_lens, int causal, float scale, void* stream) {
  using namespace dgq;
  dgq_status st = kv_cache_check(cache);
  if (st != DGQ_OK) return st;
  if (!rows_pointer_ok(Q) || !rows_pointer_ok(O) || B <= 0 || Hq <= 0 || max_nq <= 0 || !block_table || max_pages <= 0 || !kv_lens ||
      (q_start && n_rows <= 0) || Hq % cache->n_heads || (dtype != DGQ_F16 && dtype != DGQ_BF16) || !std::isfinite(scale))
    return DGQ_ERR_INVALID_ARG;
  if ((int64_t)max_pages * cache->page > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  const int64_t qb = q_start ? 1 : B, qn = q_start ? n_rows : max_nq;
  if ((st = rows_check(*Q, qb, qn, Hq, false)) != DGQ_OK || (st = rows_check(*O, qb, qn, Hq, true)) != DGQ_OK) return st;
  EncAttnArgs a = {};
  a.Q = rows_normal(*Q, qb, qn, Hq);
  a.O = rows_normal(*O, qb, qn, Hq);
  a.B = B;
  a.Hq = Hq;
  a.Hkv = cache->n_heads;
  a.nq = max_nq;
  a.nk = max_pages * cache->page;
  a.d = cache->d;
  a.scale_log2 = (float)(1.4426950408889634 * (double)scale);
  a.kv_lens = kv_lens;
  a.k_codes = (const int8_t*)cache->k;
  a.v_codes = (const int8_t*)cache->v;
  a.k_scale = cache->k_scale;
  a.v_scale = cache->v_scale;
  a.n_pages = cache->n_pages;
  a.page = cache->page;
  a.max_pages = max_pages;
  a.table = block_table;
  a.q_start = q_start;
  a.n_rows = n_rows;
  a.causal = causal != 0;
  return dtype == DGQ_BF16 ? enc_attn_launch<true, true>(a, (cudaStream_t)stream) : enc_attn_launch<false, true>(a, (cudaStream_t)stream);
}
