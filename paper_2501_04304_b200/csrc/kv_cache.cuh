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
static inline int kv_log2(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

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
  int B, n_free, max_pages, page, page_log2, n_slots;
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
// unused end of the slot map begins.  That reads B * B / 8 lengths in all: 2048 requests, which write 1.25 MB, are bound by the launch
// and two dependent rounds of loads.
__global__ void __launch_bounds__(PLAN_WARPS * 32) kv_plan_kernel(const KvPlanArgs a) {
  __shared__ long long part[PLAN_WARPS][4];
  __shared__ long long own[PLAN_WARPS][2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b0 = blockIdx.x * PLAN_WARPS, b = b0 + warp;
  pdl_wait();
  bool bad = false;
  const auto pages_of = [&](long long tokens) { return (int)((tokens + a.page - 1) >> a.page_log2); };
  // tokens and pages before this block's requests, and of all requests
  long long sum[4] = {0, 0, 0, 0};
#pragma unroll 4
  for (int i = threadIdx.x; i < a.B; i += PLAN_WARPS * 32) {
    int len, add;
    plan_lengths(a, i, len, add, bad);
    const int pages = pages_of((long long)len + add) - pages_of(len);
    sum[2] += add;
    sum[3] += pages;
    if (i < b0) {
      sum[0] += add;
      sum[1] += pages;
    }
  }
  int len = 0, add = 0;
  if (b < a.B) plan_lengths(a, b, len, add, bad);
  const int have = pages_of(len), need = pages_of((long long)len + add);
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
  pdl_launch_dependents();  // at the top, the next call's blocks came in before this one's had read: 10.1 us a call back to back, 6.4 here
  if (total > INT_MAX || total > a.n_slots || all_pages > a.n_free) bad = true;
  if (b < a.B) {
    int32_t* row = a.table + (int64_t)b * a.max_pages;
    if (lane == 0) {
      a.token_start[b] = (int32_t)min(start, (long long)INT_MAX);
      a.kv_lens[b] = len + add;
    }
    // a page whose slots 31 bits hold: a larger number's would be those of another page
    const auto page_ok = [&](int p) { return p >= 0 && p <= INT_MAX >> a.page_log2; };
    // the page of the tokens that the request has already begun
    int first = -1;
    if (have > 0 && (len & (a.page - 1))) {
      first = row[have - 1];
      bad |= !page_ok(first);
    }
    const auto new_page = [&](int i) {
      const long long at = taken + i;
      return at < a.n_free ? a.free_pages[at] : -1;
    };
    for (int i = lane; i < need - have; i += 32) {
      const int p = new_page(i);
      bad |= !page_ok(p);
      row[have + i] = p;
    }
    for (int i = lane; i < add; i += 32) {
      const long long t = start + i;
      if (t >= a.n_slots) break;
      const int pos = len + i, pi = pos >> a.page_log2;
      const int page = pi < have ? first : new_page(pi - have);
      a.slots[t] = !page_ok(page) ? -1 : (page << a.page_log2) + (pos & (a.page - 1));
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
  int n_pages, n_heads, page, page_log2, d, chunk;
};

constexpr int WRITE_THREADS = 128;
constexpr int WRITE_HELD = 4;  // sixteen-byte pieces of a thread that stay in registers between the two passes

// Largest magnitude of two 16-bit numbers against `top`, in the type itself (exact); NaN stays NaN.
template <bool BF>
__device__ __forceinline__ uint32_t absmax16(uint32_t top, uint32_t x) {
  x &= 0x7FFF7FFFu;
  if (BF) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&top), *reinterpret_cast<const __nv_bfloat162*>(&x));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2*>(&top), *reinterpret_cast<const __half2*>(&x));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Two 16-bit numbers with 0 for those that are not finite: all bits of their exponent are set.
template <bool BF>
__device__ __forceinline__ uint32_t finite16(uint32_t x) {
  constexpr uint32_t E = BF ? 0x7F80u : 0x7C00u;
  if ((x & E) == E) x &= 0xFFFF0000u;
  if ((x >> 16 & E) == E) x &= 0x0000FFFFu;
  return x;
}
// Codes of four 16-bit numbers: rint(x / s), the quotient rounded to fp32.  x * inv is within 127 * 2^-23 of it, so the two round to the
// same whole number unless a border of two codes is that near; `near` then tells that these (a few in 10^5, half the largest value
// among them) have to be divided.  Adding 1.5 * 2^23 rounds to a whole number, whose low byte is the code; no clamp is needed:
// |x| <= 127 s up to the last bit of s.
__device__ __forceinline__ uint32_t low_bytes(const float (&t)[4]) {
  return __byte_perm(__byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040),
                     __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t codes_by_division(float4 x, float s) {
  const float t[4] = {__fadd_rn(__fdiv_rn(x.x, s), 12582912.f), __fadd_rn(__fdiv_rn(x.y, s), 12582912.f),
                      __fadd_rn(__fdiv_rn(x.z, s), 12582912.f), __fadd_rn(__fdiv_rn(x.w, s), 12582912.f)};
  return low_bytes(t);
}
template <bool BF>
__device__ __forceinline__ uint32_t codes_of4(uint32_t a, uint32_t b, float inv, float& near) {
  const unsigned long long magic = pack_f32x2(12582912.f, 12582912.f), minus = pack_f32x2(-12582912.f, -12582912.f);
  const unsigned long long inv2 = pack_f32x2(inv, inv), one = pack_f32x2(-1.f, -1.f), zero = 0ull;
  const float2 lo = unpack16<BF>(a), hi = unpack16<BF>(b);
  float t[4], d[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned long long y = fma_f32x2(i ? pack_f32x2(hi.x, hi.y) : pack_f32x2(lo.x, lo.y), inv2, zero);
    const unsigned long long u = add_f32x2(y, magic);
    unpack_f32x2(u, t[2 * i], t[2 * i + 1]);
    unpack_f32x2(fma_f32x2(add_f32x2(u, minus), one, y), d[2 * i], d[2 * i + 1]);
  }
  near = fmaxf(near, fmaxf(fmaxf(fabsf(d[0]), fabsf(d[1])), fmaxf(fabsf(d[2]), fabsf(d[3]))));
  return low_bytes(t);
}
__device__ __forceinline__ float code_as_float(uint32_t biased_word, int i) {
  return __uint_as_float(__byte_perm(biased_word, 0x4B000000u, 0x7540 + i)) - 8388736.f;  // 2^23 + 128
}

// Largest magnitude of sixteen bytes of a row against `top`.
template <bool BF>
__device__ __forceinline__ uint32_t absmax_piece(uint32_t top, const uint4& y) {
  return absmax16<BF>(absmax16<BF>(absmax16<BF>(absmax16<BF>(top, y.x), y.y), y.z), y.w);
}
// The same over THREADS threads, keys and values; all have then read what they needed of the page's old scales.
template <bool BF, int THREADS>
__device__ __forceinline__ void absmax_all(uint32_t (&top2)[2], uint32_t (*red)[WRITE_THREADS / 32]) {
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top2[w] = absmax16<BF>(top2[w], __shfl_xor_sync(0xFFFFFFFFu, top2[w], o));
  if (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) {
      red[0][threadIdx.x >> 5] = top2[0];
      red[1][threadIdx.x >> 5] = top2[1];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
      top2[0] = absmax16<BF>(top2[0], red[0][i]);
      top2[1] = absmax16<BF>(top2[1], red[1][i]);
    }
  } else {
    __syncwarp();
  }
}
// A page's scale from its largest new magnitude and the one it has (0: none).
template <bool BF>
__device__ __forceinline__ float page_scale(uint32_t top2, float held) {
  const float2 top = unpack16<BF>(top2);
  // a scale below the smallest normal number would have no inverse
  float s = fmaxf(top.x, top.y);
  s = s > 0.f ? fmaxf(__fmul_rn(s, 1.0f / 127.0f), 1.17549435e-38f) : 0.f;
  return fmaxf(s, held);
}
// The codes of a page's first rows from one scale to a larger one.
template <int THREADS>
__device__ __forceinline__ void round_old_codes(int8_t* page, int rows, int row_bytes, float held, float s) {
#pragma unroll 1
  for (int u = threadIdx.x % THREADS; u < rows * (row_bytes / 16); u += THREADS) {
    uint4* p = reinterpret_cast<uint4*>(page) + u;
    uint4 y = *p;
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {  // the words move up: four divisions of code instead of sixteen
      const uint32_t x = y.x ^ 0x80808080u;
      y = make_uint4(y.y, y.z, y.w, codes_by_division(make_float4(__fmul_rn(code_as_float(x, 0), held), __fmul_rn(code_as_float(x, 1), held),
                                                                  __fmul_rn(code_as_float(x, 2), held), __fmul_rn(code_as_float(x, 3), held)), s));
    }
    *p = y;
  }
}
// Eight codes; the last ones of a row with the zeros that fill it up.
__device__ __forceinline__ void put_codes(int8_t* to, uint32_t lo, uint32_t hi, bool fill) {
  *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
  if (fill) *reinterpret_cast<uint2*>(to + 8) = make_uint2(0, 0);
}
template <bool BF>
__device__ __forceinline__ void put_divided(int8_t* to, const uint4& y, float s, bool fill) {
  const float2 f0 = unpack16<BF>(y.x), f1 = unpack16<BF>(y.y), f2 = unpack16<BF>(y.z), f3 = unpack16<BF>(y.w);
  put_codes(to, codes_by_division(make_float4(f0.x, f0.y, f1.x, f1.y), s), codes_by_division(make_float4(f2.x, f2.y, f3.x, f3.y), s), fill);
}

// The tokens of a call seen from a run, which goes on to the next usable slot of another page.
struct KvRun {
  const KvWriteArgs& a;
  int64_t t;  // its first token
  int slot;
  __device__ __forceinline__ bool usable(int s) const { return s >= 0 && s < a.n_pages << a.page_log2; }
  // Slot s of token i + lane and which of the 32 are the run's; true: it ends among them.
  __device__ __forceinline__ bool look(int64_t i, int& s, unsigned& in) const {
    i += threadIdx.x & 31;
    s = i < a.T ? a.slots[i] : -1;
    const bool here = usable(s) && (s >> a.page_log2) == (slot >> a.page_log2);
    const unsigned end = __ballot_sync(0xFFFFFFFFu, i >= a.T || (usable(s) && !here));
    in = __ballot_sync(0xFFFFFFFFu, here) & (end ? (1u << (__ffs(end) - 1)) - 1u : 0xFFFFFFFFu);
    return end != 0;
  }
  // The first token from i on whose slot is usable, T if none is left.  Stretches of skipped tokens may be long (the end of a slot map with
  // room for more): 1024 at a time where that many are left, all loads in front of the first use.
  __device__ __forceinline__ int64_t next_usable(int64_t i) const {
    const int lane = threadIdx.x & 31;
    for (bool first = true; i < a.T; first = false) {
      const bool wide = !first && i + 1024 <= a.T;
      unsigned at = 1024;
      if (wide) {
        // from a sixteen-byte boundary, at most three tokens back, which are skipped ones
        i -= (int64_t)(((reinterpret_cast<uintptr_t>(a.slots) >> 2) + (uint64_t)i) & 3);
        int4 s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = reinterpret_cast<const int4*>(a.slots + i)[k * 32 + lane];
#pragma unroll
        for (int k = 7; k >= 0; --k) {
          const unsigned j = k * 128 + lane * 4;
          at = usable(s[k].x) ? j : usable(s[k].y) ? j + 1 : usable(s[k].z) ? j + 2 : usable(s[k].w) ? j + 3 : at;
        }
      } else {
        int s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = i + k * 32 + lane < a.T ? a.slots[i + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 7; k >= 0; --k) at = usable(s[k]) ? k * 32 + lane : at;
      }
      at = __reduce_min_sync(0xFFFFFFFFu, at);
      if (at < 1024) return i + at;
      i += wide ? 1024 : 256;
    }
    return a.T;
  }
  // The last usable slot of the tokens in front of i, -1 if there is none.
  __device__ __forceinline__ int last_before(int64_t i) const {
    const int lane = threadIdx.x & 31;
    for (; i > 0; i -= 256) {
      int s[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] = i > k * 32 + lane ? a.slots[i - 1 - k * 32 - lane] : -1;
      unsigned back = 256;
#pragma unroll
      for (int k = 7; k >= 0; --k) back = usable(s[k]) ? k * 32 + lane : back;
      back = __reduce_min_sync(0xFFFFFFFFu, back);
      if (back < 256) return a.slots[i - 1 - back];
    }
    return -1;
  }
};

// A run with rows left out or skipped tokens between its rows, or with values that are not finite, which count as 0: first the token of
// every row of the page, then two passes over them.
template <bool BF, int THREADS>
__device__ __forceinline__ void kv_write_gaps(const KvWriteArgs& a, const KvRun& run, int h, long long* token_of, uint32_t (*red)[WRITE_THREADS / 32]) {
  const int lane = threadIdx.x & 31, tid = threadIdx.x % THREADS;
  const int row_bytes = kv_row_bytes(a.d), units = a.d / 8, r0 = run.slot & (a.page - 1);
  const int step = THREADS / units, r_first = tid / units, c = tid - r_first * units;
  const int64_t ph = (int64_t)(run.slot >> a.page_log2) * a.n_heads + h;
  float held[2] = {0.f, 0.f};
  if (r0 > 0) {
    held[0] = a.scale[0][ph];
    held[1] = a.scale[1][ph];
  }
  if (THREADS == 32 || threadIdx.x < 32) {
    __syncwarp();
    for (int r = lane; r < a.page; r += 32) token_of[r] = -1;
    __syncwarp();
    int top = -1;
    for (int64_t i = run.t; top < a.page - 1;) {
      int s;
      unsigned in;
      const bool end = run.look(i, s, in);
      const int row = in >> lane & 1u ? s & (a.page - 1) : -1;
      int most = row;  // of the lanes up to this one
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, most, o);
        if (lane >= o) most = max(most, y);
      }
      const int before = __shfl_up_sync(0xFFFFFFFFu, most, 1);
      if (row > (lane ? max(before, top) : top)) token_of[row] = i + lane;  // one that is not above all before it is skipped
      top = max(top, __shfl_sync(0xFFFFFFFFu, most, 31));
      if (end) break;
      i += 32;
      if (!in) i = run.next_usable(i);
    }
    __syncwarp();
  }
  if (THREADS > 32) __syncthreads();
  bool odd = false;
  const auto piece = [&](int w, long long token) {
    const uint4 y = __ldg(reinterpret_cast<const uint4*>(a.x[w] + (int64_t)h * a.head[w] + c * 8 + token * a.token[w]));
    const uint4 f = make_uint4(finite16<BF>(y.x), finite16<BF>(y.y), finite16<BF>(y.z), finite16<BF>(y.w));
    odd |= f.x != y.x || f.y != y.y || f.z != y.z || f.w != y.w;
    return f;
  };
  uint32_t top2[2] = {0, 0};
  if (r_first < step)
#pragma unroll 1
    for (int r = r0 + r_first; r < a.page; r += step) {
      const long long token = token_of[r];
      if (token < 0) continue;
#pragma unroll
      for (int w = 0; w < 2; ++w) top2[w] = absmax_piece<BF>(top2[w], piece(w, token));
    }
  if (odd) record_error(DGQ_ERR_INVALID_ARG);
  absmax_all<BF, THREADS>(top2, red);
#pragma unroll 1
  for (int w = 0; w < 2; ++w) {
    const float s = page_scale<BF>(top2[w], held[w]);
    int8_t* page = a.codes[w] + (ph << a.page_log2) * row_bytes;
    if (r0 > 0 && s > held[w]) round_old_codes<THREADS>(page, r0, row_bytes, held[w], s);
    if (r_first < step)
#pragma unroll 1
      for (int r = r0 + r_first; r < a.page; r += step) {
        const long long token = token_of[r];
        if (token >= 0) put_divided<BF>(page + r * row_bytes + c * 8, piece(w, token), s > 0.f ? s : 1.f, c == units - 1 && (a.d & 8));
      }
    if (tid == 0) a.scale[w][ph] = s;
  }
}

// THREADS (one warp, or the block for large pages) take the runs that begin among `chunk` tokens, for one head's keys and values at
// once: largest values, scales, codes.  A run is all that a call brings for one page, whatever tokens are skipped and rows left out in
// it: one scale has to come out of it, and the old codes are rounded to it once.  Most runs' rows follow one another, fit the registers
// and are read once.  What bounds it is the chain slots, rows, maximum, codes of a run, so keys and values go through it together and
// few tokens share a warp only where the GPU is full without.  64 prompts of 20 to 77 rows of 20 x 64 into pages of 16 and out again:
// 43 us with a block per run, a division per value and a second read; 18.2 with a warp for keys and one for values; 16.6 with one
// warp for both.  Looking for a run's end behind gaps and for values that are not finite costs 1.5 us of that case with changing inputs
// (19.6 -> 21.1; 256 single tokens 19.5 -> 20.7); 64 tokens in a slot map with room for 64, 960 and 8128 more 0.2, 0.8 and 8 us.
// Without the bound on registers the compiler takes 120 for runs with gaps and fewer blocks share an SM (22.2 us for the tokens); a
// bound for six blocks spills (23.0 us for the prompts).
template <bool BF, int THREADS>
__global__ void __launch_bounds__(WRITE_THREADS, 5) kv_write_kernel(const __grid_constant__ KvWriteArgs a) {
  __shared__ uint32_t red[2][WRITE_THREADS / 32];
  __shared__ long long row_token[WRITE_THREADS];  // of a run with gaps: 32 rows for each warp (pages up to 32) or 128 for the block
  constexpr int GROUPS = WRITE_THREADS / THREADS;
  const int tid = threadIdx.x % THREADS, lane = threadIdx.x & 31;
  const int h = blockIdx.y;
  const int row_bytes = kv_row_bytes(a.d), units = a.d / 8;
  KvRun run{a, 0, 0};
  pdl_launch_dependents();
  pdl_wait();
  const int64_t t0 = ((int64_t)blockIdx.x * GROUPS + threadIdx.x / THREADS) * a.chunk;
  // Which of the tokens begin a run: those whose page is not that of the nearest usable slot before them, however far back that is.
  unsigned begins;
  int mine = -1;
  {
    const int64_t t = t0 + lane;
    const int64_t back = t0 - 32 + lane;
    int before = back >= 0 && back < a.T ? a.slots[back] : -1;
    if (lane < a.chunk && t < a.T) {
      mine = a.slots[t];
      if (mine >= 0 && !run.usable(mine) && h == 0) record_error(DGQ_ERR_INVALID_ARG);
    }
    const unsigned real = __ballot_sync(0xFFFFFFFFu, run.usable(mine)), seen = __ballot_sync(0xFFFFFFFFu, run.usable(before));
    if (!real) return;
    if (seen) before = __shfl_sync(0xFFFFFFFFu, before, 31 - __clz(seen));
    else before = run.last_before(t0 - 32);
    const unsigned lower = real & ((1u << lane) - 1u);
    const int inside = __shfl_sync(0xFFFFFFFFu, mine, lower ? 31 - __clz(lower) : 0);
    const int prev = lower ? inside : before;
    const bool same = run.usable(mine) && prev >= 0 && (prev >> a.page_log2) == (mine >> a.page_log2);
    if (same && prev >= mine && h == 0) record_error(DGQ_ERR_INVALID_ARG);
    begins = __ballot_sync(0xFFFFFFFFu, run.usable(mine) && !same);
  }
  // a thread has the same piece of rows tid / units, + step, ...
  const int step = THREADS / units, r_first = tid / units, c = tid - r_first * units;
  const bool works = r_first < step, fill = c == units - 1 && (a.d & 8);
  unsigned gapped = 0;  // runs with gaps or values that are not finite, which come last
  for (; begins; begins &= begins - 1) {
    const int at = __ffs(begins) - 1;
    const int64_t t = t0 + at;
    const int slot = __shfl_sync(0xFFFFFFFFu, mine, at), r0 = slot & (a.page - 1);
    const int64_t ph = (int64_t)(slot >> a.page_log2) * a.n_heads + h;
    float held[2] = {0.f, 0.f};
    if (r0 > 0) {
      held[0] = a.scale[0][ph];
      held[1] = a.scale[1][ph];
    }
    // n rows follow one another, row r0 + i being token t + i; `gaps`: there are more
    run.t = t;
    run.slot = slot;
    int n = 0;
    bool gaps = false;
    for (int64_t i = t;;) {
      int s;
      unsigned in;
      const bool end = run.look(i, s, in);
      unsigned rest = in;
      if (i - t == n) {
        const unsigned direct = __ballot_sync(0xFFFFFFFFu, (unsigned)s - (unsigned)slot == (unsigned)(n + lane)) & in;
        const int more = direct == 0xFFFFFFFFu ? 32 : __ffs(~direct) - 1;
        n += more;
        rest = more == 32 ? 0u : in >> more;
      }
      gaps = rest != 0;
      if (gaps || end || r0 + n == a.page) break;
      i += 32;
      if (i - t != n) i = run.next_usable(i);  // the rows that follow one another have ended
      if (i >= a.T) break;
    }
    if (gaps) {
      gapped |= 1u << at;
      continue;
    }
    const uint16_t* rows[2];
    uint4 q[2][WRITE_HELD];
    uint32_t top2[2] = {0, 0};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      rows[w] = a.x[w] + (int64_t)h * a.head[w] + c * 8 + t * a.token[w];
#pragma unroll
      for (int k = 0; k < WRITE_HELD; ++k) {
        if (k * step >= n) break;
        const int r = r_first + k * step;
        q[w][k] = make_uint4(0, 0, 0, 0);
        if (works && r < n) q[w][k] = __ldg(reinterpret_cast<const uint4*>(rows[w] + r * a.token[w]));
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int k = 0; k < WRITE_HELD; ++k) {
        if (k * step >= n) break;
        top2[w] = absmax_piece<BF>(top2[w], q[w][k]);
      }
    if (works)
#pragma unroll 2
      for (int r = r_first + WRITE_HELD * step; r < n; r += step)
#pragma unroll
        for (int w = 0; w < 2; ++w) top2[w] = absmax_piece<BF>(top2[w], __ldg(reinterpret_cast<const uint4*>(rows[w] + r * a.token[w])));
    absmax_all<BF, THREADS>(top2, red);
    if (finite16<BF>(top2[0]) != top2[0] || finite16<BF>(top2[1]) != top2[1]) {
      gapped |= 1u << at;
      if (THREADS > 32) __syncthreads();  // red is free again
      continue;
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float s = page_scale<BF>(top2[w], held[w]);
      const float inv = s > 0.f ? __fdiv_rn(1.0f, s) : 0.f;
      int8_t* page = a.codes[w] + (ph << a.page_log2) * row_bytes;
      if (r0 > 0 && s > held[w]) round_old_codes<THREADS>(page, r0, row_bytes, held[w], s);
      int8_t* dst = page + r0 * row_bytes + c * 8;
      float near = 0.f;
      if (works) {
#pragma unroll
        for (int k = 0; k < WRITE_HELD; ++k) {
          if (k * step >= n) break;
          if (r_first + k * step < n)
            put_codes(dst + (r_first + k * step) * row_bytes, codes_of4<BF>(q[w][k].x, q[w][k].y, inv, near), codes_of4<BF>(q[w][k].z, q[w][k].w, inv, near), fill);
        }
#pragma unroll 1
        for (int r = r_first + WRITE_HELD * step; r < n; r += step) {
          const uint4 y = __ldg(reinterpret_cast<const uint4*>(rows[w] + r * a.token[w]));
          put_codes(dst + r * row_bytes, codes_of4<BF>(y.x, y.y, inv, near), codes_of4<BF>(y.z, y.w, inv, near), fill);
        }
        if (near > 0.49998f) {
#pragma unroll 1
          for (int r = r_first; r < n; r += step) put_divided<BF>(dst + r * row_bytes, __ldg(reinterpret_cast<const uint4*>(rows[w] + r * a.token[w])), s, fill);
        }
      }
      if (tid == 0) a.scale[w][ph] = s;
    }
    if (THREADS > 32) __syncthreads();  // red is free again
  }
  for (; gapped; gapped &= gapped - 1) {
    const int at = __ffs(gapped) - 1;
    run.t = t0 + at;
    run.slot = __shfl_sync(0xFFFFFFFFu, mine, at);
    kv_write_gaps<BF, THREADS>(a, run, h, row_token + threadIdx.x / THREADS * (WRITE_THREADS / GROUPS), red);
    if (THREADS > 32) __syncthreads();
  }
}

// ------------------------------------------------------------------ values out
struct KvReadArgs {
  uint16_t* y[2];
  int64_t token[2], head[2];
  const int8_t* codes[2];
  const float* scale[2];
  const int32_t* slots;
  int64_t T;
  uint32_t per_row, per_units;   // 2^32 / n rounded up: the high half of a product with it is the quotient
  int n_pages, n_heads, page, page_log2, d, tokens;
};

constexpr int READ_UNITS = 512;  // most pieces of a block's tokens (a token may have more)

// Two codes (bytes i, i + 1 of a biased word) as values.
template <bool BF>
__device__ __forceinline__ uint32_t values_of2(uint32_t w, int i, float s) {
  return pack16<BF>(__fmul_rn(code_as_float(w, i), s), __fmul_rn(code_as_float(w, i + 1), s));
}

// A block has `tokens` tokens, a thread a piece of eight codes of K and the same of V at a time: sixteen bytes out, next to its
// neighbours' (two pieces a thread wrote halves of sectors and took 14.7 us instead of 12.0 for 256 requests' last pages of 8 x
// 128).  The index arithmetic stays in 32 bits: quotients of a block's piece numbers come from one multiplication.
template <bool BF>
__global__ void __launch_bounds__(256) kv_read_kernel(const __grid_constant__ KvReadArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int row_bytes = kv_row_bytes(a.d), units = a.d / 8, per_token = a.n_heads * units, n_slots = a.n_pages << a.page_log2;
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
  const int pieces = (int)min((int64_t)a.tokens, a.T - t0) * per_token;
  for (int u = threadIdx.x; u < pieces; u += 256) {
    const int tl = per_token == 1 ? u : a.tokens == 1 ? 0 : (int)__umulhi((uint32_t)u, a.per_row), in = u - tl * per_token;
    const int h = units == 1 ? in : (int)__umulhi((uint32_t)in, a.per_units), c = in - h * units;
    const int slot = a.slots[t0 + tl];
    const bool real = slot >= 0 && slot < n_slots;
    if (slot >= n_slots) record_error(DGQ_ERR_INVALID_ARG);
    uint2 q[2] = {make_uint2(0, 0), make_uint2(0, 0)};
    float s[2] = {0.f, 0.f};
    if (real) {
      const int64_t ph = (int64_t)(slot >> a.page_log2) * a.n_heads + h;
      const int64_t at = ((ph << a.page_log2) + (slot & (a.page - 1))) * row_bytes + c * 8;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        q[w] = __ldg(reinterpret_cast<const uint2*>(a.codes[w] + at));
        s[w] = __ldg(a.scale[w] + ph);
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t x = q[w].x ^ 0x80808080u, y = q[w].y ^ 0x80808080u;
      *reinterpret_cast<uint4*>(a.y[w] + (t0 + tl) * a.token[w] + h * a.head[w] + c * 8) =
          make_uint4(values_of2<BF>(x, 0, s[w]), values_of2<BF>(x, 2, s[w]), values_of2<BF>(y, 0, s[w]), values_of2<BF>(y, 2, s[w]));
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
  KvPlanArgs a{lens, n_new, free_pages, block_table, token_start, kv_lens, slots, used, B, n_free, max_pages, page, kv_log2(page), n_slots};
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
  a.page_log2 = kv_log2(cache->page);
  // sixteen tokens to a warp where that still fills the GPU: they are one or two runs of a prompt; single tokens (each its own
  // run) want a warp each
  int sms = 0;
  DGQ_CUDA_OK(sm_count(&sms));
  const int group = cache->page > 32 ? WRITE_THREADS : 32;
  a.chunk = 16;
  while (a.chunk > 1 && T * cache->n_heads / a.chunk * group < (int64_t)sms * 768) a.chunk /= 4;
  const int64_t per_block = (int64_t)a.chunk * (WRITE_THREADS / group), blocks = (T + per_block - 1) / per_block;
  if (blocks > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  const auto kernel = dtype == DGQ_BF16 ? (group == 32 ? kv_write_kernel<true, 32> : kv_write_kernel<true, WRITE_THREADS>)
                                        : (group == 32 ? kv_write_kernel<false, 32> : kv_write_kernel<false, WRITE_THREADS>);
  DGQ_CUDA_OK(launch_pdl(kernel, dim3((unsigned)blocks, (unsigned)cache->n_heads), dim3(WRITE_THREADS), 0, (cudaStream_t)stream, a));
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
  const int units = cache->d / 8, per_token = units * cache->n_heads;
  a.T = T;
  a.tokens = (int)std::min<int64_t>(std::max(1, READ_UNITS / per_token), T);
  a.per_row = (uint32_t)((1ull << 32) / per_token + 1);
  a.per_units = (uint32_t)((1ull << 32) / units + 1);
  a.n_pages = cache->n_pages;
  a.n_heads = cache->n_heads;
  a.page = cache->page;
  a.page_log2 = kv_log2(cache->page);
  a.d = cache->d;
  const int64_t blocks = (T + a.tokens - 1) / a.tokens;
  if (blocks > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  DGQ_CUDA_OK(launch_pdl(dtype == DGQ_BF16 ? kv_read_kernel<true> : kv_read_kernel<false>, dim3((unsigned)blocks), dim3(256), 0,
                         (cudaStream_t)stream, a));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}
