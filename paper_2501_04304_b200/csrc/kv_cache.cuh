// A paged key/value cache in 8 bits: block tables and slot maps from lengths, rows in, values out.
//
//     s = max |x| / 127 over the rows of one page and head,   code = clamp(rint(x / s), -127, 127),   value = code * s
//
// All three kernels move bytes; none has arithmetic that counts.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace dgq {

constexpr int KV_MAX_D = 160;
constexpr int KV_MAX_PAGE = 128;

__host__ __device__ inline int kv_row_bytes(int d) { return (d + 15) & ~15; }

// ------------------------------------------------------------------ 16-bit tensors with strides
static inline bool rows_pointer_ok(const dgq_rows* r) { return r && r->ptr; }
// Strides of one tensor [B, n, H, d]; `out` marks one that is written, which may not broadcast.
static dgq_status rows_check(const dgq_rows& r, int64_t B, int64_t n, int64_t H, bool out) {
  const int64_t size[3] = {B, n, H}, stride[3] = {r.batch, r.token, r.head};
  for (int i = 0; i < 3; ++i) {
    if (size[i] <= 1) continue;
    if (stride[i] < 0 || (stride[i] == 0 && (out || i == 1))) return DGQ_ERR_INVALID_ARG;
  }
  if (!aligned16(r.ptr)) return DGQ_ERR_ALIGNMENT;
  for (int i = 0; i < 3; ++i) {
    if (size[i] <= 1) continue;
    if (stride[i] % 8) return DGQ_ERR_ALIGNMENT;
    if (stride[i] >= (1ll << 38)) return DGQ_ERR_UNSUPPORTED;  // a tensor map holds strides below 2^40 bytes
  }
  return DGQ_OK;
}
// The strides as the kernels use them: 0 where the dimension has one element.
static dgq_rows rows_normal(const dgq_rows& r, int64_t B, int64_t n, int64_t H) {
  dgq_rows x = r;
  if (B <= 1) x.batch = 0;
  if (n <= 1) x.token = 0;
  if (H <= 1) x.head = 0;
  return x;
}
static dgq_status kv_cache_check(const dgq_kv_cache* c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || c->n_pages <= 0 || c->n_heads <= 0 || c->page <= 0 || c->d <= 0)
    return DGQ_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v)) return DGQ_ERR_ALIGNMENT;
  if ((c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) || c->d % 8 || c->d > KV_MAX_D ||
      (int64_t)c->n_pages * c->page > INT_MAX || c->n_heads > 65535)
    return DGQ_ERR_UNSUPPORTED;
  return DGQ_OK;
}

#ifdef __CUDACC__
// ------------------------------------------------------------------ 16-bit elements, two at a time
template <bool BF>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
  if (BF) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (BF) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ------------------------------------------------------------------ block tables and slot maps
struct KvPlanArgs {
  const int32_t *lens, *n_new, *free_pages;
  int32_t *table, *token_start, *kv_lens, *slots, *used;
  int B, n_free, max_pages, page, n_slots;
};

constexpr int PLAN_WARPS = 8;

__device__ __forceinline__ void plan_lengths(const KvPlanArgs& a, int b, int& len, int& add, bool& bad) {
  const int64_t cap = min((int64_t)a.max_pages * a.page, (int64_t)INT_MAX);
  const int l = a.lens[b], n = a.n_new[b];
  len = (int)min((int64_t)max(l, 0), cap);
  add = (int)min((int64_t)max(n, 0), cap - len);
  bad |= l < 0 || n < 0 || (int64_t)l + n > cap;
}

// A warp has one request, a block eight in a row.  Every block adds up the tokens and pages of all requests before its own by
// itself (at most a few reads a thread, from L2), so that one launch does it all; the totals it gets on the way say where the
// unused end of the slot map begins.  The largest case writes 1.8 MB; what bounds it is the launch and two dependent
// rounds of loads.
__global__ void __launch_bounds__(PLAN_WARPS * 32) kv_plan_kernel(const KvPlanArgs a) {
  __shared__ long long part[PLAN_WARPS][4];
  __shared__ long long own[PLAN_WARPS][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b0 = blockIdx.x * PLAN_WARPS, b = b0 + warp;
  pdl_launch_dependents();
  pdl_wait();
  bool bad = false;
  // tokens and pages before this block's requests, and of all requests
  long long sum[4] = {0, 0, 0, 0};
  for (int i = threadIdx.x; i < a.B; i += PLAN_WARPS * 32) {
    int len, add;
    plan_lengths(a, i, len, add, bad);
    const int pages = (int)(((long long)len + add + a.page - 1) / a.page - ((long long)len + a.page - 1) / a.page);
    sum[2] += add;
    sum[3] += pages;
    if (i < b0) {
      sum[0] += add;
      sum[1] += pages;
    }
  }
  int len = 0, add = 0;
  if (b < a.B) plan_lengths(a, b, len, add, bad);
  const int have = (int)(((long long)len + a.page - 1) / a.page), need = (int)(((long long)len + add + a.page - 1) / a.page);
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], o);
  if (lane == 0) {
    for (int k = 0; k < 4; ++k) part[warp][k] = sum[k];
    own[warp][0] = add;
    own[warp][1] = need - have;
  }
  __syncthreads();
  long long start = 0, taken = 0, total = 0, all_pages = 0;
  for (int w = 0; w < PLAN_WARPS; ++w) {
    start += part[w][0];
    taken += part[w][1];
    total += part[w][2];
    all_pages += part[w][3];
  }
  for (int w = 0; w < warp; ++w) {
    start += own[w][0];
    taken += own[w][1];
  }
  if (total > INT_MAX || total > a.n_slots || all_pages > a.n_free) bad = true;
  if (b < a.B) {
    int32_t* row = a.table + (int64_t)b * a.max_pages;
    if (lane == 0) {
      a.token_start[b] = (int32_t)min(start, (long long)INT_MAX);
      a.kv_lens[b] = len + add;
    }
    // the page of the tokens that the request has already begun
    int first = -1;
    if (have > 0 && len % a.page) {
      first = row[have - 1];
      if (first < 0) bad = true;
    }
    const auto new_page = [&](int i) {
      const long long at = taken + i;
      return at < a.n_free ? a.free_pages[at] : -1;
    };
    for (int i = lane; i < need - have; i += 32) row[have + i] = new_page(i);
    for (int i = lane; i < add; i += 32) {
      const long long t = start + i;
      if (t >= a.n_slots) break;
      const int pos = len + i, pi = pos / a.page;
      const int page = pi < have ? first : new_page(pi - have);
      a.slots[t] = page < 0 ? -1 : page * a.page + pos % a.page;
    }
  }
  for (long long t = min(total, (long long)a.n_slots) + blockIdx.x * (PLAN_WARPS * 32) + threadIdx.x; t < a.n_slots;
       t += (long long)gridDim.x * (PLAN_WARPS * 32))
    a.slots[t] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.token_start[a.B] = (int32_t)min(total, (long long)INT_MAX);
    *a.used = (int32_t)min(all_pages, (long long)a.n_free);
  }
  if (bad) record_error(DGQ_ERR_INVALID_ARG);
}

// ------------------------------------------------------------------ rows in
struct KvWriteArgs {
  const uint16_t* x[2];     // K and V rows
  int64_t token[2], head[2];
  int8_t* codes[2];
  float* scale[2];
  const int32_t* slots;
  int64_t T;
  int n_pages, n_heads, page, d, chunk;
};

constexpr int WRITE_THREADS = 128;

// A block takes the runs of rows of one page that begin among its `chunk` tokens, for one head of K or V: largest value, scale,
// codes.  The rows are read twice, the second time from L1.
template <bool BF>
__global__ void __launch_bounds__(WRITE_THREADS) kv_write_kernel(const KvWriteArgs a) {
  __shared__ float red[WRITE_THREADS / 32];
  __shared__ int s_len[WRITE_THREADS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, which = blockIdx.z;
  const uint16_t* x = a.x[which] + (int64_t)h * a.head[which];
  const int64_t ldx = a.token[which];
  const int row_bytes = kv_row_bytes(a.d), units = a.d / 8;
  const int n_slots = a.n_pages * a.page;
  pdl_launch_dependents();
  pdl_wait();
  const int64_t t_end = min(a.T, (int64_t)(blockIdx.x + 1) * a.chunk);
  for (int64_t t = (int64_t)blockIdx.x * a.chunk; t < t_end;) {
    const int slot = a.slots[t];
    const int r0 = slot % a.page;
    if (slot < 0 || slot >= n_slots) {
      if (slot >= n_slots && tid == 0) record_error(DGQ_ERR_INVALID_ARG);
      ++t;
      continue;
    }
    if (r0 > 0 && t > 0 && a.slots[t - 1] == slot - 1) {  // the run began before: another block's, or done
      ++t;
      continue;
    }
    // length of the run: thread i looks at row i
    const bool in = t + tid < a.T && r0 + tid < a.page && a.slots[t + tid] == slot + tid;
    const unsigned ball = __ballot_sync(0xFFFFFFFFu, in);
    if (lane == 0) s_len[warp] = ball == 0xFFFFFFFFu ? 32 : __ffs(~ball) - 1;
    __syncthreads();
    int n = 0;
    for (int w = 0; w < WRITE_THREADS / 32; ++w) {
      n += s_len[w];
      if (s_len[w] < 32) break;
    }
    const uint16_t* rows = x + t * ldx;
    float top = 0.f;
    for (int u = tid; u < n * units; u += WRITE_THREADS) {
      const int r = u / units, c = u - r * units;
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(rows + r * ldx) + c);
      const uint32_t w4[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack16<BF>(w4[i]);
        top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) red[warp] = top;
    const int64_t ph = (int64_t)(slot / a.page) * a.n_heads + h;
    float* scale = a.scale[which] + ph;
    const float held = r0 > 0 ? *scale : 0.f;
    __syncthreads();  // also: everyone has read the old scale and the run's length
    for (int w = 0; w < WRITE_THREADS / 32; ++w) top = fmaxf(top, red[w]);
    float s = __fmul_rn(top, 1.0f / 127.0f);
    if (r0 > 0) s = fmaxf(s, held);
    int8_t* page = a.codes[which] + ph * a.page * row_bytes;
    if (r0 > 0 && s > held) {
      for (int u = tid; u < r0 * (row_bytes / 16); u += WRITE_THREADS) {
        uint4* p = reinterpret_cast<uint4*>(page) + u;
        uint4 q = *p;
        uint32_t w4[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t o = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float c = (float)(int8_t)(w4[i] >> (8 * k));
            const int v = __float2int_rn(fminf(fmaxf(rintf(__fdiv_rn(__fmul_rn(c, held), s)), -127.f), 127.f));
            o |= (uint32_t)(v & 0xFF) << (8 * k);
          }
          w4[i] = o;
        }
        *p = make_uint4(w4[0], w4[1], w4[2], w4[3]);
      }
    }
    for (int u = tid; u < n * units; u += WRITE_THREADS) {
      const int r = u / units, c = u - r * units;
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(rows + r * ldx) + c);
      const uint32_t w4[4] = {q.x, q.y, q.z, q.w};
      uint32_t o[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack16<BF>(w4[i]);
        const float y0 = s > 0.f ? __fdiv_rn(f.x, s) : 0.f, y1 = s > 0.f ? __fdiv_rn(f.y, s) : 0.f;
        const int v0 = __float2int_rn(fminf(fmaxf(rintf(y0), -127.f), 127.f));
        const int v1 = __float2int_rn(fminf(fmaxf(rintf(y1), -127.f), 127.f));
        o[i >> 1] |= ((uint32_t)(v0 & 0xFF) | (uint32_t)(v1 & 0xFF) << 8) << (16 * (i & 1));
      }
      int8_t* dst = page + (int64_t)(r0 + r) * row_bytes + c * 8;
      *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
      if (c == units - 1 && (a.d & 8)) *reinterpret_cast<uint2*>(dst + 8) = make_uint2(0, 0);
    }
    if (tid == 0) *scale = s;
    t += n;
    __syncthreads();  // red and s_len are free again
  }
}

// ------------------------------------------------------------------ values out
struct KvReadArgs {
  uint16_t* y[2];
  int64_t token[2], head[2];
  const int8_t* codes[2];
  const float* scale[2];
  const int32_t* slots;
  int64_t n_units;  // T * heads * d / 8
  int n_pages, n_heads, page, d;
};

// One thread: eight values of K and the same eight of V.
template <bool BF>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvReadArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int units = a.d / 8, row_bytes = kv_row_bytes(a.d);
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < a.n_units; i += gridDim.x * 256ll) {
    const int c = (int)(i % units);
    const int64_t th = i / units;
    const int h = (int)(th % a.n_heads);
    const int64_t t = th / a.n_heads;
    const int slot = a.slots[t];
    const bool real = slot >= 0 && slot < a.n_pages * a.page;
    if (slot >= a.n_pages * a.page) record_error(DGQ_ERR_INVALID_ARG);
    const int64_t ph = real ? (int64_t)(slot / a.page) * a.n_heads + h : 0;
    const int64_t at = real ? (ph * a.page + slot % a.page) * row_bytes + c * 8 : 0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint2 q = make_uint2(0, 0);
      float s = 0.f;
      if (real) {
        q = *reinterpret_cast<const uint2*>(a.codes[w] + at);
        s = a.scale[w][ph];
      }
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t two = (k < 2 ? q.x : q.y) >> (16 * (k & 1));
        o[k] = pack16<BF>(__fmul_rn((float)(int8_t)two, s), __fmul_rn((float)(int8_t)(two >> 8), s));
      }
      *reinterpret_cast<uint4*>(a.y[w] + t * a.token[w] + h * a.head[w] + c * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}
#endif

}  // namespace dgq

extern "C" dgq_status dgq_kv_plan(const int32_t* lens, const int32_t* n_new, int B, const int32_t* free_pages, int n_free,
                                  int32_t* block_table, int max_pages, int page, int32_t* token_start, int32_t* kv_lens,
                                  int32_t* slots, int n_slots, int32_t* used, void* stream) {
  using namespace dgq;
  if (!lens || !n_new || !block_table || !token_start || !kv_lens || !used || B <= 0 || max_pages <= 0 || n_free < 0 || n_slots < 0 ||
      (!free_pages && n_free) || (!slots && n_slots))
    return DGQ_ERR_INVALID_ARG;
  // blocks read all lengths while others write theirs
  const auto apart = [&](const int32_t* in, const int32_t* out, int64_t n) { return in + B <= out || out + n <= in; };
  if (!apart(lens, kv_lens, B) || !apart(n_new, kv_lens, B) || !apart(lens, token_start, B + 1ll) || !apart(n_new, token_start, B + 1ll))
    return DGQ_ERR_INVALID_ARG;
  if (page != 16 && page != 32 && page != 64 && page != 128) return DGQ_ERR_UNSUPPORTED;
  KvPlanArgs a{lens, n_new, free_pages, block_table, token_start, kv_lens, slots, used, B, n_free, max_pages, page, n_slots};
  DGQ_CUDA_OK(launch_pdl(kv_plan_kernel, dim3((unsigned)((B + PLAN_WARPS - 1) / PLAN_WARPS)), dim3(PLAN_WARPS * 32), 0,
                         (cudaStream_t)stream, a));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

extern "C" dgq_status dgq_kv_write(const dgq_kv_cache* cache, const dgq_rows* K, const dgq_rows* V, int dtype, int64_t T,
                                   const int32_t* slots, void* stream) {
  using namespace dgq;
  dgq_status st = kv_cache_check(cache);
  if (st != DGQ_OK) return st;
  if (!rows_pointer_ok(K) || !rows_pointer_ok(V) || !slots || T <= 0 || (dtype != DGQ_F16 && dtype != DGQ_BF16))
    return DGQ_ERR_INVALID_ARG;
  if ((st = rows_check(*K, 1, T, cache->n_heads, false)) != DGQ_OK || (st = rows_check(*V, 1, T, cache->n_heads, false)) != DGQ_OK)
    return st;
  KvWriteArgs a;
  const dgq_rows in[2] = {rows_normal(*K, 1, T, cache->n_heads), rows_normal(*V, 1, T, cache->n_heads)};
  for (int i = 0; i < 2; ++i) {
    a.x[i] = (const uint16_t*)in[i].ptr;
    a.token[i] = in[i].token;
    a.head[i] = in[i].head;
    a.codes[i] = (int8_t*)(i ? cache->v : cache->k);
    a.scale[i] = i ? cache->v_scale : cache->k_scale;
  }
  a.slots = slots;
  a.T = T;
  a.n_pages = cache->n_pages;
  a.n_heads = cache->n_heads;
  a.page = cache->page;
  a.d = cache->d;
  // single tokens (each its own run) want a block each while they fit on the GPU at once; many tokens come as runs
  a.chunk = T * cache->n_heads * 2 > 148 * 16 * 4 ? 16 : 1;
  const int64_t blocks = (T + a.chunk - 1) / a.chunk;
  if (blocks > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  DGQ_CUDA_OK(launch_pdl(dtype == DGQ_BF16 ? kv_write_kernel<true> : kv_write_kernel<false>,
                         dim3((unsigned)blocks, (unsigned)cache->n_heads, 2), dim3(WRITE_THREADS), 0, (cudaStream_t)stream, a));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

extern "C" dgq_status dgq_kv_read(const dgq_kv_cache* cache, const int32_t* slots, int64_t T, const dgq_rows* K,
                                  const dgq_rows* V, int dtype, void* stream) {
  using namespace dgq;
  dgq_status st = kv_cache_check(cache);
  if (st != DGQ_OK) return st;
  if (!rows_pointer_ok(K) || !rows_pointer_ok(V) || !slots || T <= 0 || (dtype != DGQ_F16 && dtype != DGQ_BF16))
    return DGQ_ERR_INVALID_ARG;
  if ((st = rows_check(*K, 1, T, cache->n_heads, true)) != DGQ_OK || (st = rows_check(*V, 1, T, cache->n_heads, true)) != DGQ_OK)
    return st;
  KvReadArgs a;
  const dgq_rows out[2] = {rows_normal(*K, 1, T, cache->n_heads), rows_normal(*V, 1, T, cache->n_heads)};
  for (int i = 0; i < 2; ++i) {
    a.y[i] = (uint16_t*)out[i].ptr;
    a.token[i] = out[i].token;
    a.head[i] = out[i].head;
    a.codes[i] = (const int8_t*)(i ? cache->v : cache->k);
    a.scale[i] = i ? cache->v_scale : cache->k_scale;
  }
  a.slots = slots;
  a.n_units = T * cache->n_heads * (cache->d / 8);
  a.n_pages = cache->n_pages;
  a.n_heads = cache->n_heads;
  a.page = cache->page;
  a.d = cache->d;
  int sms = 0;
  DGQ_CUDA_OK(sm_count(&sms));
  const int64_t blocks = std::min<int64_t>((a.n_units + 255) / 256, (int64_t)sms * 32);
  DGQ_CUDA_OK(launch_pdl(dtype == DGQ_BF16 ? kv_read_kernel<true> : kv_read_kernel<false>, dim3((unsigned)blocks), dim3(256), 0,
                         (cudaStream_t)stream, a));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}
