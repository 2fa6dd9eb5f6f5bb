// Group normalisation of channels-last maps, with an addend per image and channel and an activation, as 16-bit values or as
// the codes of the next layer.
//
//     u = x + add[b, c],   y = (u - mean_bg) / sqrt(var_bg + eps) * gamma_c + beta_c,   v = y  or  y / (1 + e^-y)
//
// mean and var over the P pixels and C / n_groups channels of a group g of image b.
//
// Two kernels.  The first one adds up x and x^2 of every channel over a slab of rows, in 64 bits, puts the addend in (sum u =
// sum x + n add, sum u^2 = sum x^2 + 2 add sum x + n add^2) and leaves one pair of sums for each group and slab.  In 64 bits the
// difference of the two sums is good to 2^-52 mean^2 / var, so that there is no second pass over the values; a conversion and
// two additions an element are what the 64-bit units do at the rate at which memory delivers 16-bit values.  The second kernel adds the
// slabs up in a fixed order (every block for itself), turns them into one factor and one addend per channel and passes over
// the map once more.  No atomics: a result does not depend on the order in which blocks run.
#pragma once

#include "kv_cache.cuh"
#include "groups.cuh"

namespace dgq {

constexpr int GN_MAX_C = 4096;
constexpr int GN_THREADS = 256;
constexpr int GN_SLABS = 296;  // slabs of rows over all images, two blocks for each multiprocessor

struct GnArgs {
  const uint16_t* X;
  int64_t xb, xp;  // strides of images and pixels, in elements
  const uint16_t* add;
  int64_t ld_add;
  const float *gamma, *beta;  // may be null: 1 and 0
  uint16_t* Y;
  int64_t yb, yp;
  int P, C, n_groups;
  int slabs, slab_rows;  // of the first kernel
  int rows;              // of a block of the second kernel
  double eps;
  double2* part;  // [B][slabs][n_groups]
  // codes
  uint8_t* Xq;
  const int16_t* perm;       // [K_pad], -1 = padding
  const uint8_t* chunk_group;  // [K_pad / 16]
  const int32_t* row_group;  // [row_period], null if there is one row group
  const float* inv_scale;    // [R][G]
  const int32_t* zp;
  int K_pad, G, R, row_period, bits, quads;
};

// Rows of a slab, and how many slabs an image has.
static inline void gn_slabs(int B, int P, int* slabs, int* rows) {
  const int want = std::max(1, std::min((GN_SLABS + B - 1) / B, P));
  *rows = (P + want - 1) / want;
  *slabs = (P + *rows - 1) / *rows;
}
static inline size_t gn_workspace(int B, int P, int n_groups) {
  int slabs, rows;
  gn_slabs(B, P, &slabs, &rows);
  return (size_t)B * slabs * n_groups * sizeof(double2);
}

#ifdef __CUDACC__

__device__ __forceinline__ float gn_up(uint16_t h, bool bf) {
  return bf ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}

// ------------------------------------------------------------------ sums
// A thread has eight neighbouring channels of every n-th row of the slab.
template <bool BF>
__global__ void __launch_bounds__(GN_THREADS) gn_sums_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  double2* acc = reinterpret_cast<double2*>(gn_smem);  // [lines][C]
  const int tid = threadIdx.x, nvec = a.C >> 3, b = blockIdx.y;
  const int lines = max(1, GN_THREADS / nvec);
  const int p0 = blockIdx.x * a.slab_rows, p1 = min(a.P, p0 + a.slab_rows);
  pdl_launch_dependents();
  pdl_wait();
  const int line = nvec <= GN_THREADS ? tid / nvec : 0;
  if (line < lines)
    for (int v = nvec <= GN_THREADS ? tid - line * nvec : tid; v < nvec; v += GN_THREADS) {
      double s[8], q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = q[i] = 0.0;
      const uint16_t* src = a.X + (int64_t)b * a.xb + v * 8;
#pragma unroll 4
      for (int p = p0 + line; p < p1; p += lines) {
        const uint4 x = *reinterpret_cast<const uint4*>(src + p * a.xp);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = unpack16<BF>(w[i]);
          const double d0 = (double)f.x, d1 = (double)f.y;
          s[2 * i] += d0;
          q[2 * i] = fma(d0, d0, q[2 * i]);
          s[2 * i + 1] += d1;
          q[2 * i + 1] = fma(d1, d1, q[2 * i + 1]);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[line * a.C + v * 8 + i] = make_double2(s[i], q[i]);
    }
  __syncthreads();
  // one warp per group
  const int cpg = a.C / a.n_groups, lane = tid & 31;
  for (int g = tid >> 5; g < a.n_groups; g += GN_THREADS / 32) {
    double s = 0.0, q = 0.0;
    for (int i = lane; i < cpg * lines; i += 32) {
      const int l = i / cpg, c = g * cpg + i - l * cpg;
      const double2 t = acc[l * a.C + c];
      const double e = a.add ? (double)gn_up(a.add[(int64_t)b * a.ld_add + c], BF) : 0.0;
      const double n = (double)max(0, (p1 - p0 - l + lines - 1) / lines);
      s += fma(n, e, t.x);
      q += fma(e, fma(n, e, 2.0 * t.x), t.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      q += __shfl_xor_sync(0xffffffffu, q, o);
    }
    if (lane == 0) a.part[((int64_t)b * a.slabs + blockIdx.x) * a.n_groups + g] = make_double2(s, q);
  }
}

// ------------------------------------------------------------------ factors
// Mean and 1 / sqrt(var + eps) of every group of image b, into `stat` [n_groups].  A negative difference of the sums (all values
// equal) counts as 0, NaN stays NaN.
__device__ __forceinline__ void gn_stats(const GnArgs& a, int b, double2* stat) {
  const double n = (double)a.P * (double)(a.C / a.n_groups);
  for (int g = threadIdx.x; g < a.n_groups; g += GN_THREADS) {
    double s = 0.0, q = 0.0;
    const double2* p = a.part + (int64_t)b * a.slabs * a.n_groups + g;
#pragma unroll 8
    for (int k = 0; k < a.slabs; ++k) {
      const double2 t = p[(int64_t)k * a.n_groups];
      s += t.x;
      q += t.y;
    }
    const double mean = s / n;
    double var = fma(-mean, mean, q / n);
    if (var < 0.0) var = 0.0;
    stat[g] = make_double2(mean, 1.0 / sqrt(var + a.eps));
  }
  __syncthreads();
}
// y = (x + shift) * factor + beta of channel c: shift, factor, beta.  The shift stands apart so that a constant map, whose deviation is
// nothing next to its mean, gives beta.
__device__ __forceinline__ float3 gn_channel(const GnArgs& a, const double2* stat, int b, int c, bool bf) {
  const double2 t = stat[c / (a.C / a.n_groups)];
  const double f = a.gamma ? t.y * (double)a.gamma[c] : t.y;
  const double e = a.add ? (double)gn_up(a.add[(int64_t)b * a.ld_add + c], bf) : 0.0;
  return make_float3((float)(e - t.x), (float)f, a.beta ? a.beta[c] : 0.f);
}

// y / (1 + e^-y); for y down to -inf the quotient's limit 0 comes out as -0 (the exponential is infinite, its reciprocal 0), for -inf as NaN.
__device__ __forceinline__ float gn_silu(float y) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return y * r;
}

// ------------------------------------------------------------------ values
template <bool BF, bool SILU>
__global__ void __launch_bounds__(GN_THREADS) gn_values_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  double2* stat = reinterpret_cast<double2*>(gn_smem);  // [n_groups]
  const int tid = threadIdx.x, nvec = a.C >> 3, b = blockIdx.y;
  const int lines = max(1, GN_THREADS / nvec);
  const int p0 = blockIdx.x * a.rows, p1 = min(a.P, p0 + a.rows);
  pdl_launch_dependents();
  pdl_wait();
  gn_stats(a, b, stat);
  const int line = nvec <= GN_THREADS ? tid / nvec : 0;
  if (line >= lines) return;
  for (int v = nvec <= GN_THREADS ? tid - line * nvec : tid; v < nvec; v += GN_THREADS) {
    float3 k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = gn_channel(a, stat, b, v * 8 + i, BF);
    const uint16_t* src = a.X + (int64_t)b * a.xb + v * 8;
    uint16_t* dst = a.Y + (int64_t)b * a.yb + v * 8;
    for (int p = p0 + line; p < p1; p += 4 * lines) {
      uint4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (p + j * lines < p1) x[j] = *reinterpret_cast<const uint4*>(src + (p + j * lines) * a.xp);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (p + j * lines < p1) {
          uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = unpack16<BF>(w[i]);
            float y0 = fmaf(f.x + k[2 * i].x, k[2 * i].y, k[2 * i].z), y1 = fmaf(f.y + k[2 * i + 1].x, k[2 * i + 1].y, k[2 * i + 1].z);
            if (SILU) y0 = gn_silu(y0), y1 = gn_silu(y1);
            w[i] = pack16<BF>(y0, y1);
          }
          *reinterpret_cast<uint4*>(dst + (p + j * lines) * a.yp) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
  }
}

// ------------------------------------------------------------------ codes
// A code next to a border of two codes, or of a zero-point that the short form has no room for, in 64 bits.
__device__ __noinline__ uint32_t gn_code_exact(const GnArgs& a, const double2* stat, bool silu, bool bf, float x, int b, int c, float inv,
                                               int z, bool centred) {
  const double2 t = stat[c / (a.C / a.n_groups)];
  const double u = (double)x + (a.add ? (double)gn_up(a.add[(int64_t)b * a.ld_add + c], bf) : 0.0);
  double v = fma((u - t.x) * t.y, a.gamma ? (double)a.gamma[c] : 1.0, a.beta ? (double)a.beta[c] : 0.0);
  if (silu) v = v / (1.0 + exp(-v));
  const double q = fmin(fmax(rint(v * (double)inv) + (double)z, 0.0), (double)((1 << a.bits) - 1));
  return (uint32_t)((int)q - (centred ? z : 0)) & 0xFFu;
}

// A thread has eight neighbouring channels of four rows at a time: it puts the four codes of a channel into one word at the channel's
// place in the padded row, in shared memory, and the words of 16 places are turned into 16 bytes of four rows on the way out.
template <bool BF, bool SILU, bool CENTRED, bool ROWS>
__global__ void __launch_bounds__(GN_THREADS) gn_codes_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  const int tid = threadIdx.x, nvec = a.C >> 3, b = blockIdx.y;
  uint32_t* words = reinterpret_cast<uint32_t*>(gn_smem);                        // [quads][K_pad], K_pad a multiple of 32
  double2* stat = reinterpret_cast<double2*>(words + (size_t)a.quads * a.K_pad);  // [n_groups]
  float4* chan = reinterpret_cast<float4*>(stat + a.n_groups);                    // [8][nvec] shift, factor, beta, place and group
  float2* cell = reinterpret_cast<float2*>(chan + a.C);                           // [R][G] 1 / s, -Z (infinite: by the long form)
  const int L = (1 << a.bits) - 1;
  const int p0 = blockIdx.x * a.rows, p1 = min(a.P, p0 + a.rows);
  pdl_launch_dependents();
  for (int i = tid; i < a.R * a.G; i += GN_THREADS) {
    const int z = __ldg(a.zp + i);
    cell[i] = make_float2(__ldg(a.inv_scale + i), abs(z) <= 65535 ? (float)-z : INFINITY);
  }
  for (int i = tid; i < a.K_pad; i += GN_THREADS) {
    const int c = __ldg(a.perm + i);
    if (c >= 0) chan[(c & 7) * nvec + (c >> 3)].w = __int_as_float(i | (int)__ldg(a.chunk_group + (i >> 4)) << 16);
  }
  pdl_wait();
  gn_stats(a, b, stat);
  for (int c = tid; c < a.C; c += GN_THREADS) {
    const float3 k = gn_channel(a, stat, b, c, BF);
    float4& to = chan[(c & 7) * nvec + (c >> 3)];
    to.x = k.x, to.y = k.y, to.z = k.z;
  }
  __syncthreads();
  const uint16_t* src = a.X + (int64_t)b * a.xb;
  const int64_t row0 = (int64_t)b * a.P;
  auto row_group = [&](int p) { return ROWS ? __ldg(a.row_group + (row0 + p) % a.row_period) * a.G : 0; };
  for (int p = p0; p < p1; p += 4 * a.quads) {
    for (int task = tid; task < a.quads * nvec; task += GN_THREADS) {
      const int quad = task / nvec, v = task - quad * nvec, r = p + 4 * quad;
      if (r >= p1) break;
      uint32_t x[4][4];
      int rg[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = min(r + j, p1 - 1);
        const uint4 t = *reinterpret_cast<const uint4*>(src + row * a.xp + v * 8);
        x[j][0] = t.x, x[j][1] = t.y, x[j][2] = t.z, x[j][3] = t.w;
        rg[j] = row_group(row);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 k = chan[i * nvec + v];
        const int place = __float_as_int(k.w), g = place >> 16;
        float2 t = cell[rg[0] + g];
        uint32_t code[4];
        float f[4];
        bool near_border = false;
        const float fixed = 0x1p-22f * (0.6f * fabsf(k.z) + 0.3f * fabsf(k.x * k.y));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (ROWS && j) t = cell[rg[j] + g];
          const float2 pair = unpack16<BF>(x[j][i >> 1]);
          f[j] = i & 1 ? pair.y : pair.x;
          const float y = fmaf(f[j] + k.x, k.y, k.z), w = (SILU ? gn_silu(y) : y) * t.x;
          // The code is off by less than `off` of a step: the rounded shift and sum, their product with the rounded factor and the sum
          // with beta by 2^-24 (3 |y| + 2 |beta| + |shift factor|), a SiLU's slope of at most 1.1 times that; the exponential's argument and
          // result, the sum, the reciprocal and the two products by 1.9 * 2^-22 |y|.
          const float off = t.x * fmaf(fabsf(y), 2.9f * 0x1p-22f, fixed);
          const float magic = CENTRED ? 12582912.f : 12582912.f - t.y;
          const float c = fminf(fmaxf(w, t.y), t.y + (float)L), m = c + magic;
          near_border |= !(fabsf(c - (m - magic)) + off < 0.5f);
          code[j] = __float_as_uint(m);
        }
        if (near_border)
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            const int at = (ROWS ? row_group(min(r + j, p1 - 1)) : 0) + g;
            const float xj = j == 0 ? f[0] : j == 1 ? f[1] : j == 2 ? f[2] : f[3];
            const uint32_t e = gn_code_exact(a, stat, SILU, BF, xj, b, v * 8 + i, cell[at].x, __ldg(a.zp + at), CENTRED);
            if (j == 0) code[0] = e;
            else if (j == 1) code[1] = e;
            else if (j == 2) code[2] = e;
            else code[3] = e;
          }
        words[quad * a.K_pad + (place & 0xFFFF)] = __byte_perm(__byte_perm(code[0], code[1], 0x0040), __byte_perm(code[2], code[3], 0x0040), 0x5410);
      }
    }
    // padding: the clamped zero-point, 0 in the zero-centred layout
    if (ROWS || p == p0)
      for (int i = tid; i < a.quads * a.K_pad; i += GN_THREADS) {
        const int quad = i / a.K_pad, at = i - quad * a.K_pad;
        if (__ldg(a.perm + at) >= 0) continue;
        uint32_t w = 0;
        if (!CENTRED) {
          const int g = __ldg(a.chunk_group + (at >> 4));
#pragma unroll
          for (int j = 0; j < 4; ++j) w |= (uint32_t)min(max(__ldg(a.zp + row_group(min(p + 4 * quad + j, p1 - 1)) + g), 0), L) << (8 * j);
        }
        words[i] = w;
      }
    __syncthreads();
    const int chunks = a.K_pad >> 4;
    for (int task = tid; task < a.quads * chunks; task += GN_THREADS) {
      const int quad = task / chunks, ch = task - quad * chunks, r = p + 4 * quad;
      if (r >= p1) break;
      const uint4* s = reinterpret_cast<const uint4*>(words + quad * a.K_pad + ch * 16);
      uint32_t out[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 w = s[i];
        const uint32_t lo01 = __byte_perm(w.x, w.y, 0x5140), hi01 = __byte_perm(w.x, w.y, 0x7362);
        const uint32_t lo23 = __byte_perm(w.z, w.w, 0x5140), hi23 = __byte_perm(w.z, w.w, 0x7362);
        out[0][i] = __byte_perm(lo01, lo23, 0x5410);
        out[1][i] = __byte_perm(lo01, lo23, 0x7632);
        out[2][i] = __byte_perm(hi01, hi23, 0x5410);
        out[3][i] = __byte_perm(hi01, hi23, 0x7632);
      }
      uint8_t* dst = a.Xq + (row0 + r) * a.K_pad + ch * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r + j < p1) *reinterpret_cast<uint4*>(dst + (int64_t)j * a.K_pad) = make_uint4(out[j][0], out[j][1], out[j][2], out[j][3]);
    }
    __syncthreads();
  }
}
#endif

// ------------------------------------------------------------------ host
static dgq_status gn_check(const dgq_rows* X, const void* add, int64_t ld_add, int dtype, int B, int P, int C, int n_groups, float eps, int act) {
  if (!rows_pointer_ok(X) || B <= 0 || P <= 0 || C <= 0 || n_groups <= 0 || C % n_groups || (dtype != DGQ_F16 && dtype != DGQ_BF16) ||
      (act != DGQ_ACT_NONE && act != DGQ_ACT_SILU) || !(eps > 0.f) || !std::isfinite(eps) || (add && B > 1 && ld_add < 0))
    return DGQ_ERR_INVALID_ARG;
  if (C % 8 || C > GN_MAX_C || P > (1 << 30) || B > 65535) return DGQ_ERR_UNSUPPORTED;
  return rows_check(*X, B, P, 1, false);
}
static void gn_fill(GnArgs& a, const dgq_rows* X, const void* add, int64_t ld_add, const float* gamma, const float* beta, int B, int P, int C,
                    int n_groups, float eps, void* workspace) {
  const dgq_rows x = rows_normal(*X, B, P, 1);
  a.X = (const uint16_t*)x.ptr;
  a.xb = x.batch;
  a.xp = x.token;
  a.add = (const uint16_t*)add;
  a.ld_add = B > 1 ? ld_add : 0;
  a.gamma = gamma;
  a.beta = beta;
  a.P = P;
  a.C = C;
  a.n_groups = n_groups;
  a.eps = (double)eps;
  a.part = (double2*)workspace;
  gn_slabs(B, P, &a.slabs, &a.slab_rows);
}
static dgq_status gn_workspace_check(int B, int P, int n_groups, const void* workspace, size_t bytes) {
  if (!workspace || bytes < gn_workspace(B, P, n_groups)) return DGQ_ERR_WORKSPACE;
  return (reinterpret_cast<uintptr_t>(workspace) & 255u) ? DGQ_ERR_ALIGNMENT : DGQ_OK;
}
constexpr size_t GN_SMEM_MAX = 200 * 1024;
// Opts a kernel in to more shared memory than 48 KB, once per device.
template <typename K>
static cudaError_t gn_opt_in(K kernel, std::atomic<bool>* done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && done[dev].load())) return e;
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)GN_SMEM_MAX)) != cudaSuccess) return e;
  if (dev < 64) done[dev].store(true);
  return cudaSuccess;
}
template <bool BF>
static dgq_status gn_sums(const GnArgs& a, int B, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  DGQ_CUDA_OK(gn_opt_in(gn_sums_kernel<BF>, done));
  const size_t smem = (size_t)std::max(1, GN_THREADS / (a.C / 8)) * a.C * sizeof(double2);
  DGQ_CUDA_OK(launch_pdl(gn_sums_kernel<BF>, dim3(a.slabs, B), dim3(GN_THREADS), smem, stream, a));
  g_launches += 1;
  return DGQ_OK;
}
template <bool BF, bool SILU>
static dgq_status gn_values(GnArgs& a, int B, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  DGQ_CUDA_OK(gn_opt_in(gn_values_kernel<BF, SILU>, done));
  dgq_status st = gn_sums<BF>(a, B, stream);
  if (st != DGQ_OK) return st;
  a.rows = a.slab_rows;
  DGQ_CUDA_OK(launch_pdl(gn_values_kernel<BF, SILU>, dim3((a.P + a.rows - 1) / a.rows, B), dim3(GN_THREADS), a.n_groups * sizeof(double2), stream, a));
  g_launches += 1;
  return DGQ_OK;
}
template <bool BF, bool SILU, bool CENTRED, bool ROWS>
static dgq_status gn_codes(GnArgs& a, int B, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  DGQ_CUDA_OK(gn_opt_in(gn_codes_kernel<BF, SILU, CENTRED, ROWS>, done));
  dgq_status st = gn_sums<BF>(a, B, stream);
  if (st != DGQ_OK) return st;
  a.rows = (a.slab_rows + 3) / 4 * 4;
  // as many quads of rows as the threads have work for, within 48 KB
  a.quads = std::max(1, std::min({GN_THREADS / (a.C / 8), 48 * 1024 / (a.K_pad * 4), a.rows / 4}));
  const size_t smem = (size_t)a.quads * a.K_pad * 4 + a.n_groups * sizeof(double2) + a.C * sizeof(float4) + (size_t)a.R * a.G * sizeof(float2);
  static_assert((GN_MAX_C + 40 * DGQ_MAX_GROUPS) * 4 + GN_MAX_C * 32 + DGQ_MAX_GROUPS * DGQ_MAX_GROUPS * 8 <= GN_SMEM_MAX, "one quad of the widest layer");
  DGQ_CUDA_OK(launch_pdl(gn_codes_kernel<BF, SILU, CENTRED, ROWS>, dim3((a.P + a.rows - 1) / a.rows, B), dim3(GN_THREADS), smem, stream, a));
  g_launches += 1;
  return DGQ_OK;
}
template <bool BF, bool SILU>
static dgq_status gn_codes_pick(GnArgs& a, int B, bool centred, cudaStream_t stream) {
  if (a.row_group) return centred ? gn_codes<BF, SILU, true, true>(a, B, stream) : gn_codes<BF, SILU, false, true>(a, B, stream);
  return centred ? gn_codes<BF, SILU, true, false>(a, B, stream) : gn_codes<BF, SILU, false, false>(a, B, stream);
}

}  // namespace dgq

extern "C" dgq_status dgq_group_norm_workspace_bytes(int B, int P, int C, int n_groups, size_t* bytes) {
  if (!bytes || B <= 0 || P <= 0 || C <= 0 || n_groups <= 0 || C % n_groups) return DGQ_ERR_INVALID_ARG;
  *bytes = dgq::gn_workspace(B, P, n_groups);
  return DGQ_OK;
}

extern "C" dgq_status dgq_group_norm(const dgq_rows* X, const void* add, int64_t ld_add, const float* gamma, const float* beta,
                                     const dgq_rows* Y, int dtype, int B, int P, int C, int n_groups, float eps, int act,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  using namespace dgq;
  if (!rows_pointer_ok(Y)) return DGQ_ERR_INVALID_ARG;
  dgq_status st = gn_check(X, add, ld_add, dtype, B, P, C, n_groups, eps, act);
  if (st != DGQ_OK || (st = rows_check(*Y, B, P, 1, true)) != DGQ_OK) return st;
  if (P > 1 && Y->token < C) return DGQ_ERR_INVALID_ARG;
  if ((st = gn_workspace_check(B, P, n_groups, workspace, workspace_bytes)) != DGQ_OK) return st;
  GnArgs a = {};
  gn_fill(a, X, add, ld_add, gamma, beta, B, P, C, n_groups, eps, workspace);
  const dgq_rows y = rows_normal(*Y, B, P, 1);
  a.Y = (uint16_t*)y.ptr;
  a.yb = y.batch;
  a.yp = y.token;
  const cudaStream_t s = (cudaStream_t)stream;
  if (dtype == DGQ_BF16) return act == DGQ_ACT_SILU ? gn_values<true, true>(a, B, s) : gn_values<true, false>(a, B, s);
  return act == DGQ_ACT_SILU ? gn_values<false, true>(a, B, s) : gn_values<false, false>(a, B, s);
}

extern "C" dgq_status dgq_group_norm_quantize(const dgq_groups* g, int timestep, int layout, const dgq_rows* X, const void* add,
                                              int64_t ld_add, const float* gamma, const float* beta, int dtype, int B, int P,
                                              int n_groups, float eps, int act, void* Xq, void* workspace, size_t workspace_bytes,
                                              void* stream) {
  using namespace dgq;
  if (!g || !Xq || (layout != DGQ_CODES_U8 && layout != DGQ_CODES_S8_CENTRED) || timestep < 0 || timestep >= g->T) return DGQ_ERR_INVALID_ARG;
  dgq_status st = gn_check(X, add, ld_add, dtype, B, P, g->C, n_groups, eps, act);
  if (st != DGQ_OK) return st;
  if (!aligned16(Xq)) return DGQ_ERR_ALIGNMENT;
  if (!g->filled[timestep]) return DGQ_ERR_NOT_CALIBRATED;
  const size_t trow = (size_t)timestep * g->R * g->G;
  const int L = (1 << g->bits) - 1;
  if (layout == DGQ_CODES_S8_CENTRED)
    for (int i = 0; i < g->R * g->G; ++i)
      if (g->zp[trow + i] > 128 || g->zp[trow + i] < L - 127) return DGQ_ERR_UNSUPPORTED;
  if ((st = gn_workspace_check(B, P, n_groups, workspace, workspace_bytes)) != DGQ_OK) return st;
  int dev = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  if (dev != g->device) return DGQ_ERR_INVALID_ARG;
  GnArgs a = {};
  gn_fill(a, X, add, ld_add, gamma, beta, B, P, g->C, n_groups, eps, workspace);
  a.Xq = (uint8_t*)Xq;
  a.perm = g->d_perm;
  a.chunk_group = g->d_chunk_group;
  a.row_group = g->R > 1 ? g->d_row_group : nullptr;
  a.inv_scale = g->d_inv_scale + trow;
  a.zp = g->d_zp + trow;
  a.K_pad = g->K_pad;
  a.G = g->G;
  a.R = g->R;
  a.row_period = g->P;
  a.bits = g->bits;
  const bool centred = layout == DGQ_CODES_S8_CENTRED;
  const cudaStream_t s = (cudaStream_t)stream;
  if (dtype == DGQ_BF16) return act == DGQ_ACT_SILU ? gn_codes_pick<true, true>(a, B, centred, s) : gn_codes_pick<true, false>(a, B, centred, s);
  return act == DGQ_ACT_SILU ? gn_codes_pick<false, true>(a, B, centred, s) : gn_codes_pick<false, false>(a, B, centred, s);
}
