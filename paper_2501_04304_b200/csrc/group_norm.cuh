// Group normalisation of channels-last maps, with an addend per image and channel and an activation, as 16-bit values or as
// the codes of the next layer.
//
//     u = x + add[b, c],   y = (u - mean_bg) / sqrt(var_bg + eps) * gamma_c + beta_c,   v = y  or  y / (1 + e^-y)
//
// mean and var over the P pixels and C / n_groups channels of a group g of image b.
#pragma once

#include <cooperative_groups.h>

#include "kv_cache.cuh"
#include "groups.cuh"

namespace dgq {

constexpr int GN_MAX_C = 4096;
constexpr int GN_MAX_PIXELS = 1 << 30;
constexpr int GN_MAX_CODE_GROUPS = 2048;  // into codes: what shared memory holds beside the widest row
constexpr int GN_MAX_THREADS = 512;  // one thread for every eight channels of the widest row
constexpr size_t GN_SMEM_MAX = 232448 - 8 * 1024;  // beside what a kernel declares
// 1 / deviation below which (bf16 only) 32 bits may not hold the differences from the mean, nor with full precision what they are multiplied with
constexpr float GN_FAR = 0x1p-60f;

struct GnArgs {
  const uint16_t* X;
  int64_t xb, xp;  // strides of images and pixels, in elements
  const uint16_t* add;
  int64_t ld_add;
  const float *gamma, *beta;  // may be null: 1 and 0
  uint16_t* Y;
  int64_t yb, yp;
  int P, C, n_groups, cpg;  // cpg: channels of a group
  int nvec;                 // eights of channels of a block's rows
  float per_nvec, per_cpg;  // 1 / nvec, 1 / cpg
  int lines;                // rows that a block has under way at a time
  float per_lines;          // 1 / lines
  int log_cluster;          // blocks of a cluster (one kernel, sums)
  int slab_rows, clusters;  // sums: rows of a block, clusters of an image
  int early;                // sums: the second kernel's blocks may come in at once
  int past;                 // values: outputs of 48 MiB and more go past L2
  int rows;                 // values and codes: rows of a block
  float eps;
  double count, per_count;  // P cpg, 1 / (P cpg)
  double2* part;  // [B][clusters][n_groups]
  // codes
  uint8_t* Xq;
  const int16_t* perm;         // [K_pad], -1 = padding
  const uint8_t* chunk_group;  // [K_pad / 16]
  const int32_t* row_group;    // [row_period], null if there is one row group
  const float* inv_scale;      // [R][G]
  const int32_t* zp;
  int K_pad, G, R, row_period, bits, centred, quads, buffers;
  float per_chunks;  // 16 / K_pad
};

#ifdef __CUDACC__

// x / n for 0 <= x < 2^20 and the rounded reciprocal of n: half a step more than the numerator keeps the rounding on the right side.
__device__ __forceinline__ int gn_div(int x, float reciprocal) { return (int)(((float)x + 0.5f) * reciprocal); }
// Keeps the compiler from working a number out again in every round of a loop.
__device__ __forceinline__ void gn_keep(int& x) { asm volatile("" : "+r"(x)); }
__device__ __forceinline__ float gn_up(uint16_t h, bool bf) {
  return bf ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}
__device__ __forceinline__ unsigned long long mul_f32x2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
template <bool BF>
__device__ __forceinline__ unsigned long long gn_pair(uint32_t w) {
  const float2 f = unpack16<BF>(w);
  return pack_f32x2(f.x, f.y);
}

// y / (1 + e^-y) of two values with three special-function operations: the reciprocal is that of the product of both denominators e0 and e1.  The
// exponents stop at 2^60, so that the product stays in range; what that leaves of a value below -41 is less than 2^-60 |y| (a bound on y itself would
// leave nothing, and cost 2 % of a large map's time).  ANY: e1 / (e0 e1) first, since y e1 leaves the range where y is beyond 2^68; else y is not
// (gn_far_silu) and y e1 is there before the reciprocal (large fp16 maps: 45.7 against 47.7 us for 1 x 262144 x 128; bf16 takes the same for both, and on
// the chip the question costs more than the product).
__device__ __forceinline__ void gn_silu_parts(float y0, float y1, float k0, float k1, float& e0, float& e1, float& per) {
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(fminf(y0 * k0, 60.f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(fminf(y1 * k1, 60.f)));
  e0 += 1.f, e1 += 1.f;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(per) : "f"(e0 * e1));
}
template <bool ANY>
__device__ __forceinline__ void gn_silu2(float y0, float y1, float& v0, float& v1) {
  float e0, e1, per;
  gn_silu_parts(y0, y1, -1.4426950408889634f, -1.4426950408889634f, e0, e1, per);
  v0 = ANY ? y0 * (e1 * per) : y0 * e1 * per;
  v1 = ANY ? y1 * (e0 * per) : y1 * e0 * per;
}
// Whether y may be beyond 2^68: a value is at most 2^21 deviations from its group's mean.
__device__ __forceinline__ bool gn_far_silu(float gamma, float beta) { return fmaxf(fabsf(gamma), fabsf(beta)) > 0x1p46f; }
// y / (1 + e^-y) of one value
__device__ __forceinline__ float gn_silu(float y) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return y * r;
}

// f(channel, value) of eight 16-bit values one after the other, for the few of which 32 bits hold no part of the formula.
template <bool BF, typename F>
__device__ __forceinline__ uint4 gn_each(uint4 x, F f) {
  unsigned long long lo = x.x | (unsigned long long)x.y << 32, hi = x.z | (unsigned long long)x.w << 32;
#pragma unroll 1
  for (int c = 0; c < 8; ++c) {  // values leave at the bottom, results enter at the top
    const unsigned long long y = pack16<BF>(f(c, gn_up((uint16_t)lo, BF)), 0.f) & 0xFFFFu;
    lo = lo >> 16 | hi << 48;
    hi = hi >> 16 | y << 48;
  }
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// ------------------------------------------------------------------ eight channels and their groups
// Eight neighbouring channels lie in at most two groups where a group has four channels or at least seven (SEG 2: a part of each, the
// second one may be empty), else every channel counts as a part of its own (SEG 8).  What threads have summed up for the parts stands
// in shared memory as [part][line][eight].
struct GnParts {
  int first, split;  // group of channel 0, channels of it
  __device__ __forceinline__ GnParts(int v, int cpg, float per_cpg) {
    first = gn_div(v * 8, per_cpg);
    split = min(8, (first + 1) * cpg - v * 8);
  }
};
// The entries of a group: calls f(index of the entry in [part][line][eight], its line, channels) for those of lane `sub` of `width`.
template <int SEG, typename F>
__device__ __forceinline__ void gn_entries(int g, int cpg, int lines, int all_lines, int nvec, int sub, int width, F f) {
  const int from = g * cpg, to = from + cpg, first = SEG == 8 ? from : from >> 3, n = (SEG == 8 ? to : (to + 7) >> 3) - first;
  const float per_n = __fdividef(1.f, (float)n);
  int line = gn_div(sub, per_n), i = sub - line * n;
  const int dl = gn_div(width, per_n), di = width - dl * n;
  while (line < lines) {
    if (SEG == 8) {
      const int c = first + i;
      f(((c & 7) * all_lines + line) * nvec + (c >> 3), line, 1);
    } else {
      const int v = first + i, c0 = v * 8;  // the group's channels of it come first or, behind those of the group before, second
      f(((c0 >= from ? 0 : all_lines) + line) * nvec + v, line, min(c0 + 8, to) - max(c0, from));
    }
    line += dl, i += di;
    if (i >= n) i -= n, ++line;
  }
}
// Lanes that share a group when a block of n_threads has n groups: 2 to this power, up to 32.
__device__ __forceinline__ int gn_width(int n_threads, int n) {
  int w = 5;
  while (w > 0 && n << w > n_threads) --w;
  return w;
}

// What eight channels have of their own, asked for before the statistics are waited for.
struct GnEight {
  float gamma[8], beta[8];
  uint32_t add[4];
  __device__ __forceinline__ void request_scale(const GnArgs& a, int c0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      gamma[i] = a.gamma ? a.gamma[c0 + i] : 1.f;
      beta[i] = a.beta ? a.beta[c0 + i] : 0.f;
    }
  }
  __device__ __forceinline__ void request_add(const GnArgs& a, int b, int c0) {
    const uint16_t* e = a.add + (int64_t)b * a.ld_add + c0;
#pragma unroll
    for (int i = 0; i < 4; ++i) add[i] = a.add ? e[2 * i] | (uint32_t)e[2 * i + 1] << 16 : 0u;
  }
  __device__ __forceinline__ float addend(int i, bool bf) const { return gn_up((uint16_t)(i & 1 ? add[i >> 1] >> 16 : add[i >> 1]), bf); }
};

// ------------------------------------------------------------------ one kernel: the map stays on the chip
// A cluster has some channels (whole groups) of one image, a block of it some of the rows, a thread eight channels of some of
// them, which it brings into shared memory once and then goes over twice.  Statistics: a thread's sums of x and x^2 of a channel count
// from the channel's first value, which loses no more than the number of its rows times 2^-24 (a value that is far from the others is a part
// of their deviation too); they become means and squared deviations, which the threads of a block and the blocks of the cluster join
// relative to the first one's mean (by the same reason no worse than the number of threads times 2^-24, and that only where all the
// deviation is that first thread's; in 64 bits their chains took 0.4 us).  Blocks write theirs into each other's shared memory, so that one barrier
// of the cluster is all.  (bf16 has values whose squares, or sums with the addend, 32 bits do not hold: groups whose deviations are not
// finite are gone over once more with everything 2^-100 times as large, statistics and values.)
// What bounds it where the map is small: the chain of reading, joining, waiting for the cluster and writing, about a microsecond each.
struct GnChipStat {
  // dev: sum of squared deviations, then 1 / sqrt(var + eps); NaN where a sum is not finite; negative, of 2^-100 times the values, as mean is too, where
  // that takes the scaled form
  float mean, dev;
};
template <bool BF, bool SILU, int SEG>
__global__ void __maxnreg__(80) gn_chip_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  const int tid = threadIdx.x, n_threads = blockDim.x, nv = a.nvec, lines = a.lines, W = nv * 8, groups = gn_div(W, a.per_cpg);
  const int rank = blockIdx.x, S = gridDim.x, b = blockIdx.z;
  uint4* rows = reinterpret_cast<uint4*>(gn_smem) + tid;                                         // piece k of this thread: rows[k * n_threads]
  float2* parts = reinterpret_cast<float2*>(gn_smem + (size_t)a.rows * n_threads * 16);          // [SEG][lines][nv]
  GnChipStat* stat = reinterpret_cast<GnChipStat*>(parts + SEG * lines * nv);                    // [groups] of the image
  GnChipStat* all = stat + groups;                                                               // [1 or, bf16, 2][S][groups] of the blocks
  // rows of a rank: P / S of them and one of the remaining ones
  const int share = a.P >> a.log_cluster, spare = a.P & (S - 1);
  const int p0 = rank * share + min(rank, spare), R = share + (rank < spare);
  int line = gn_div(tid, a.per_nvec), v = tid - line * nv;
  gn_keep(line), gn_keep(v);
  const int full = gn_div(R, a.per_lines), more = R - full * lines;  // rows of a line: full, one more for the first ones
  const int n = line < lines ? full + (line < more) : 0;             // rows of this thread
  const GnParts part(v, a.cpg, a.per_cpg);
  const int c0 = blockIdx.y * W + v * 8;
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  if (S > 1) cluster.barrier_arrive();  // (waited for before the first access to another block's shared memory: it has started by then)
  pdl_wait();
  {
    const uint16_t* src = a.X + (int64_t)b * a.xb + (p0 + line) * a.xp + c0;
    uint32_t to = smem_u32(rows);
#pragma unroll 4
    for (int k = 0; k < n; ++k, src += lines * a.xp, to += n_threads * 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
  }
  GnEight of;
  if (n > 0) of.request_add(a, b, c0), of.request_scale(a, c0);
  auto addend = [&](int i) { return of.addend(i, BF); };
  asm volatile("cp.async.wait_all;" ::: "memory");
  // Statistics of the block's groups into `stat`; false if one of them is not finite.  SCALED does those over that are not.
  auto attempt = [&](auto scaled) {
    constexpr bool SCALED = decltype(scaled)::value;
    constexpr float unit = SCALED ? 0x1p-100f : 1.f;
    auto value = [&](uint32_t w) { return SCALED ? mul_f32x2(gn_pair<BF>(w), pack_f32x2(unit, unit)) : gn_pair<BF>(w); };
    bool finite = true;
    const float per_all = (float)a.per_count;
    auto settle = [&](int g, float mean, float dev) {
      const float var = dev * per_all;
      if (!SCALED) {
        stat[g] = GnChipStat{mean, dev < INFINITY ? __frsqrt_rn(var + a.eps) : __int_as_float(0x7FC00000)};
        finite &= dev < INFINITY;
      } else if (isnan(stat[g].dev)) {
        stat[g] = GnChipStat{mean, dev < INFINITY ? -__frsqrt_rn(var + fmaxf(a.eps * unit * unit, 0x1p-126f)) : __int_as_float(0x7FC00000)};
      }
    };
    if (n > 0) {
      unsigned long long s2[4] = {0, 0, 0, 0}, q2[4] = {0, 0, 0, 0}, minus[4];
      float m[8], q[8];
      {
        const uint4 x = rows[0];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          unpack_f32x2(value(w[i]), m[2 * i], m[2 * i + 1]);
          minus[i] = pack_f32x2(-m[2 * i], -m[2 * i + 1]);
        }
      }
#pragma unroll 4
      for (int j = 1; j < n; ++j) {
        const uint4 x = rows[j * n_threads];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned long long d = add_f32x2(value(w[i]), minus[i]);
          s2[i] = add_f32x2(s2[i], d);
          q2[i] = fma_f32x2(d, d, q2[i]);
        }
      }
      const float fn = (float)n, per_n = __frcp_rn(fn);
      float mean[SEG] = {}, dev[SEG] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float t[2], u[2];
        unpack_f32x2(s2[i], t[0], t[1]);
        unpack_f32x2(q2[i], u[0], u[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = 2 * i + h;
          const float off = t[h] * per_n;
          m[c] += fmaf(addend(c), unit, off);
          q[c] = fmaf(-off, t[h], u[h]);
          if (SEG == 8) mean[c] = m[c], dev[c] = q[c];
          else mean[0] += c < part.split ? m[c] : 0.f, mean[1] += c < part.split ? 0.f : m[c];
        }
      }
      if (SEG == 2) {
        mean[0] = __fdividef(mean[0], (float)part.split), mean[1] = __fdividef(mean[1], (float)max(1, 8 - part.split));
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float d = m[c] - (c < part.split ? mean[0] : mean[1]), t = fmaf(fn * d, d, q[c]);
          dev[0] += c < part.split ? t : 0.f, dev[1] += c < part.split ? 0.f : t;
        }
      }
#pragma unroll
      for (int i = 0; i < SEG; ++i) parts[(i * lines + line) * nv + v] = make_float2(mean[i], dev[i]);
    }
    __syncthreads();
    const int log_width = gn_width(n_threads, groups), width = 1 << log_width, used = min(lines, R);
    const int per_round = n_threads >> log_width;
    const float per_own = __frcp_rn((float)(R * a.cpg));
    // sums over the lanes that share a group of n (m - m0) and n (m - m0)^2
    auto join = [&](float& t, float& u, int lanes) {
      for (int o = lanes >> 1; o > 0; o >>= 1) {
        t += __shfl_xor_sync(0xffffffffu, t, o);
        u += __shfl_xor_sync(0xffffffffu, u, o);
      }
    };
    GnChipStat* mine = all + (SCALED ? groups * S : 0);  // [S][groups], everybody's
    if (S > 1 && !SCALED) cluster.barrier_wait();
    for (int g0 = 0; g0 < groups; g0 += per_round) {
      const int g = min(g0 + (tid >> log_width), groups - 1), sub = tid & (width - 1);  // (spare lanes do the last group again)
      const int from = g * a.cpg;
      const float m0 = parts[(SEG == 8 ? (from & 7) * lines * nv : from & 7 ? lines * nv : 0) + (from >> 3)].x;
      float t = 0.f, u = 0.f;
      gn_entries<SEG>(g, a.cpg, used, lines, nv, sub, width, [&](int at, int l, int channels) {
        const float2 p = parts[at];
        const float d = p.x - m0, c = (float)((full + (l < more)) * channels);
        t = fmaf(c, d, t);
        u += fmaf(c * d, d, p.y);
      });
      join(t, u, width);
      const float off = t * per_own;
      const GnChipStat r = {m0 + off, fmaf(-off, t, u)};
      const bool real = g0 + (tid >> log_width) < groups;
      if (S == 1) {
        if (sub == 0 && real) settle(g, r.mean, r.dev);
      } else if (real) {
        for (int to = sub; to < S; to += width) *cluster.map_shared_rank(mine + rank * groups + g, to) = r;
      }
    }
    if (S > 1) {
      cluster.sync();
      // sixteen lanes per group, one for each block
      for (int g0 = 0; g0 < groups; g0 += n_threads / 16) {
        const int g = min(g0 + tid / 16, groups - 1), r = tid & 15;
        const GnChipStat z = r < S ? mine[r * groups + g] : GnChipStat{0.f, 0.f};
        const float m0 = __shfl_sync(0xffffffffu, z.mean, tid & 16);
        const float d = r < S ? z.mean - m0 : 0.f, c = (float)(share + (r < spare)) * (float)a.cpg;
        float t = c * d, u = fmaf(t, d, z.dev);
        join(t, u, 16);
        const float off = t * per_all;
        if (r == 0 && g0 + tid / 16 < groups) settle(g, m0 + off, fmaf(-off, t, u));
      }
    }
    return finite;
  };
  // (the same answer in every block of the cluster: they have joined the same numbers)
  const bool finite = attempt(std::false_type{});
  auto group = [&](int c) { return SEG == 8 ? gn_div(v * 8 + c, a.per_cpg) : part.first + (c < part.split ? 0 : 1); };
  if (BF) {
    if (__syncthreads_or(!finite)) {
      attempt(std::true_type{});
      __syncthreads();
      bool far = false;
      for (int c = 0; c < 8; ++c) far |= stat[group(c)].dev < 0.f;
      if (far) {
        uint16_t* dst = a.Y + (int64_t)b * a.yb + (p0 + line) * a.yp + c0;
#pragma unroll 1
        for (int k = 0; k < n; ++k, dst += lines * a.yp)
          *reinterpret_cast<uint4*>(dst) = gn_each<BF>(rows[k * n_threads], [&](int c, float x) {
            const GnChipStat st = stat[group(c)];
            const float unit = st.dev < 0.f ? 0x1p-100f : 1.f;
            const float e = a.add ? gn_up(a.add[(int64_t)b * a.ld_add + c0 + c], BF) : 0.f;
            // (the sum first, as in the statistics: equal sums are equal to their mean)
            const float y = fmaf((fmaf(x, unit, e * unit) - st.mean) * fabsf(st.dev), a.gamma ? a.gamma[c0 + c] : 1.f, a.beta ? a.beta[c0 + c] : 0.f);
            return SILU ? gn_silu(y) : y;
          });
        return;
      }
    }
  } else {
    __syncthreads();
  }
  pdl_launch_dependents();  // (earlier, the next kernel's blocks would crowd this one's)
  if (n > 0) {
    unsigned long long shift[4], factor[4], beta[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float t[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = 2 * i + h;
        const GnChipStat st = stat[group(c)];
        t[h][0] = addend(c) - st.mean;
        t[h][1] = st.dev * of.gamma[c];
      }
      shift[i] = pack_f32x2(t[0][0], t[1][0]);
      factor[i] = pack_f32x2(t[0][1], t[1][1]);
      beta[i] = pack_f32x2(of.beta[2 * i], of.beta[2 * i + 1]);
    }
    uint16_t* dst = a.Y + (int64_t)b * a.yb + (p0 + line) * a.yp + c0;
#pragma unroll 2
    for (int k = 0; k < n; ++k, dst += lines * a.yp) {
      const uint4 x = rows[k * n_threads];
      uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned long long y = fma_f32x2(add_f32x2(gn_pair<BF>(w[i]), shift[i]), factor[i], beta[i]);
        float y0, y1;
        unpack_f32x2(y, y0, y1);
        if (SILU) gn_silu2<true>(y0, y1, y0, y1);
        w[i] = pack16<BF>(y0, y1);
      }
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// ------------------------------------------------------------------ two kernels: sums ...
// For maps that do not fit, and for codes, which a row's whole width is permuted into.  The first kernel adds up x and x^2 of every channel
// over a slab of rows, in 64 bits, puts the addend in (sum u = sum x + n add, sum u^2 = sum x^2 + 2 add sum x + n add^2) and leaves one
// pair of sums for each group and cluster of slabs.  In 64 bits the difference of the two sums is good to 2^-52 mean^2 / var, or add^2 / var where an addend
// takes off what the values have, so that there is
// no second pass over the values; a conversion and two additions an element are what the 64-bit units do at the rate at which memory delivers 16-bit
// values.  The second kernel adds the clusters up in a fixed order (every block for itself), turns them into a shift and a factor per
// channel and passes over the map once more.  No atomics: a result does not depend on the order in which blocks run.
// Rows come in through a ring of pieces in shared memory that each thread fills and empties for itself, GN_RING of them under way: with
// the loads in registers, four at a time, 63 MB took 25 us.
constexpr int GN_RING = 8;
struct GnRing {
  uint32_t at;  // of this thread's first piece
  uint32_t step;
  __device__ __forceinline__ GnRing(const void* smem, int tid, int n_threads) : at(smem_u32(smem) + tid * 16), step(n_threads * 16) {}
  // piece k from `src`, if it is there; one group each
  __device__ __forceinline__ void request(int k, const uint16_t* src, bool there) const {
    if (there) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + (k % GN_RING) * step), "l"(src) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // piece k, when pieces up to k + GN_RING - 2 have been requested
  __device__ __forceinline__ uint4 take(int k) const {
    asm volatile("cp.async.wait_group %0;" ::"n"(GN_RING - 2) : "memory");
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at + (k % GN_RING) * step) : "memory");
    return x;
  }
};

template <bool BF, int SEG>
__global__ void __launch_bounds__(GN_MAX_THREADS) gn_sums_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  const int tid = threadIdx.x, n_threads = blockDim.x, nv = a.nvec, lines = a.lines, b = blockIdx.y;
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int S = 1 << a.log_cluster, rank = blockIdx.x & (S - 1), per_block = (a.n_groups + S - 1) >> a.log_cluster;
  double2* all = reinterpret_cast<double2*>(gn_smem);  // [S][per_block] of the cluster's blocks, of the groups that this one joins
  double2* parts = all + S * per_block;                // [SEG][lines][nv], in the ring's place
  cluster.barrier_arrive();  // (waited for before the first access to another block's shared memory: it has started by then)
  const int p0 = min((int64_t)a.P, (int64_t)blockIdx.x * a.slab_rows), p1 = min((int64_t)a.P, (int64_t)p0 + a.slab_rows), used = min(lines, p1 - p0);
  const int line = gn_div(tid, a.per_nvec), v = tid - line * nv;
  const GnRing ring(parts, tid, n_threads);
  if (a.early) pdl_launch_dependents();
  pdl_wait();
  double2 t[SEG];
#pragma unroll
  for (int i = 0; i < SEG; ++i) t[i] = make_double2(0.0, 0.0);
  if (line < used) {
    double s[8], q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = q[i] = 0.0;
    const int rows = (p1 - p0 - line + lines - 1) / lines;
    const int64_t step = lines * a.xp;
    const uint16_t* src = a.X + (int64_t)b * a.xb + (p0 + line) * a.xp + v * 8;
#pragma unroll
    for (int k = 0; k < GN_RING - 1; ++k, src += step) ring.request(k, src, k < rows);
#pragma unroll 2
    for (int k = 0; k < rows; ++k, src += step) {
      const uint4 x = ring.take(k);
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
      ring.request(k + GN_RING - 1, src, k + GN_RING - 1 < rows);  // into the piece before this one
    }
    const GnParts part(v, a.cpg, a.per_cpg);
    const double n = (double)rows;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (a.add) {
        const double e = (double)gn_up(a.add[(int64_t)b * a.ld_add + v * 8 + i], BF);
        q[i] = fma(e, fma(n, e, 2.0 * s[i]), q[i]);
        s[i] = fma(n, e, s[i]);
      }
      if (SEG == 8) t[i] = make_double2(s[i], q[i]);
      else if (i < part.split) t[0].x += s[i], t[0].y += q[i];
      else t[1].x += s[i], t[1].y += q[i];
    }
  }
  if (!a.early) pdl_launch_dependents();
  __syncthreads();  // the ring is empty
  if (line < used)
#pragma unroll
    for (int i = 0; i < SEG; ++i) parts[(i * lines + line) * nv + v] = t[i];
  __syncthreads();
  cluster.barrier_wait();
  const int log_width = gn_width(n_threads, a.n_groups), width = 1 << log_width, per_round = n_threads >> log_width;
  for (int g0 = 0; g0 < a.n_groups; g0 += per_round) {
    const int g = min(g0 + (tid >> log_width), a.n_groups - 1), sub = tid & (width - 1);
    double s = 0.0, q = 0.0;
    gn_entries<SEG>(g, a.cpg, used, lines, nv, sub, width, [&](int at, int, int) {
      s += parts[at].x;
      q += parts[at].y;
    });
    for (int o = width >> 1; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      q += __shfl_xor_sync(0xffffffffu, q, o);
    }
    // to the block that joins this group's: the groups are dealt out to the blocks of the cluster in turn
    if (g0 + (tid >> log_width) < a.n_groups && sub == 0) *cluster.map_shared_rank(all + rank * per_block + (g >> a.log_cluster), g & (S - 1)) = make_double2(s, q);
  }
  cluster.sync();
  for (int i = tid, g = rank + (tid << a.log_cluster); g < a.n_groups; i += n_threads, g += n_threads << a.log_cluster) {
    double2 t = all[i];
    for (int r = 1; r < S; ++r) t.x += all[r * per_block + i].x, t.y += all[r * per_block + i].y;
    a.part[((int64_t)b * a.clusters + (blockIdx.x >> a.log_cluster)) * a.n_groups + g] = t;
  }
}

// Mean and 1 / sqrt(var + eps) of every group of image b, into `stat` [n_groups].  A negative difference of the sums (all values
// equal) counts as 0, NaN stays NaN.
// `meanwhile` is called between the requests and their arrival: loads of its own come behind the few that everybody waits for.
template <typename F>
__device__ __forceinline__ void gn_stats(const GnArgs& a, int b, double2* stat, F meanwhile) {
  const int tid = threadIdx.x, n_threads = blockDim.x;
  const int log_width = gn_width(n_threads, a.n_groups), width = 1 << log_width, per_round = n_threads >> log_width;
  for (int g0 = 0; g0 < a.n_groups; g0 += per_round) {
    const int g = min(g0 + (tid >> log_width), a.n_groups - 1), sub = tid & (width - 1);
    double s = 0.0, q = 0.0;
    const double2* p = a.part + (int64_t)b * a.clusters * a.n_groups + g;
    double2 t[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) t[i] = sub + i * width < a.clusters ? p[(int64_t)(sub + i * width) * a.n_groups] : make_double2(0.0, 0.0);
    if (g0 == 0) meanwhile();
#pragma unroll
    for (int i = 0; i < 5; ++i) s += t[i].x, q += t[i].y;
    for (int k = sub + 5 * width; k < a.clusters; k += width) {
      const double2 u = p[(int64_t)k * a.n_groups];
      s += u.x;
      q += u.y;
    }
    for (int o = width >> 1; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      q += __shfl_xor_sync(0xffffffffu, q, o);
    }
    // s / count, rounded: a map of equal values has them for its mean, and nothing is left of u - mean, whatever it is multiplied with
    double mean = s * a.per_count;
    mean = fma(fma(-a.count, mean, s), a.per_count, mean);
    double var = fma(-mean, mean, q * a.per_count);
    if (var < 0.0) var = 0.0;
    if (sub == 0) stat[g] = make_double2(mean, rsqrt(var + (double)a.eps));
  }
  __syncthreads();
}
// y = (x + shift) * factor + beta.  The shift stands apart so that a constant map, whose deviation is nothing next to its mean, gives
// beta.  Where 16 bits have no addend their zeros add nothing.
__device__ __forceinline__ float2 gn_channel(const GnEight& k, const double2& stat, int i, bool bf) {
  return make_float2((float)((double)k.addend(i, bf) - stat.x), (float)stat.y * k.gamma[i]);
}

// Whether that leaves the range of 32 bits (see GN_FAR; a constant map may have no deviation and a mean beyond it).
__device__ __forceinline__ bool gn_far(const double2& stat, float shift) { return stat.y < (double)GN_FAR || fabsf(shift) > 0x1p126f; }

// ------------------------------------------------------------------ ... and values ...
template <bool BF, bool SILU>
__global__ void __launch_bounds__(GN_MAX_THREADS) gn_values_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  double2* stat = reinterpret_cast<double2*>(gn_smem);  // [n_groups]
  const int tid = threadIdx.x, nv = a.nvec, lines = a.lines, b = blockIdx.y;
  // last rows first: the sums have read them last
  const int p0 = (int)(gridDim.x - 1 - blockIdx.x) * a.rows, p1 = min(a.P, p0 + a.rows);
  const int line = gn_div(tid, a.per_nvec), v = tid - line * nv;
  const GnRing ring(stat + a.n_groups, tid, blockDim.x);
  pdl_wait();
  const int rows = line < lines && p0 + line < p1 ? (p1 - p0 - line + lines - 1) / lines : 0;
  const int64_t step = lines * a.xp;
  const uint16_t* src = a.X + (int64_t)b * a.xb + (p0 + line) * a.xp + v * 8;
  GnEight own;
  if (rows > 0) own.request_scale(a, v * 8), own.request_add(a, b, v * 8);
  gn_stats(a, b, stat, [&]() {
#pragma unroll
    for (int k = 0; k < GN_RING - 1; ++k, src += step) ring.request(k, src, k < rows);
  });
  if (rows == 0) return;
  unsigned long long shift[4], factor[4], beta[4];
  bool far = false;  // whether this takes 64 bits
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t0 = gn_channel(own, stat[gn_div(v * 8 + 2 * i, a.per_cpg)], 2 * i, BF), t1 = gn_channel(own, stat[gn_div(v * 8 + 2 * i + 1, a.per_cpg)], 2 * i + 1, BF);
    shift[i] = pack_f32x2(t0.x, t1.x);
    factor[i] = pack_f32x2(t0.y, t1.y);
    beta[i] = pack_f32x2(own.beta[2 * i], own.beta[2 * i + 1]);
    if (BF) far |= gn_far(stat[gn_div(v * 8 + 2 * i, a.per_cpg)], t0.x) || gn_far(stat[gn_div(v * 8 + 2 * i + 1, a.per_cpg)], t1.x);
    else if (SILU) far |= gn_far_silu(own.gamma[2 * i], own.beta[2 * i]) || gn_far_silu(own.gamma[2 * i + 1], own.beta[2 * i + 1]);
  }
  uint16_t* dst = a.Y + (int64_t)b * a.yb + (p0 + line) * a.yp + v * 8;
  if ((BF || SILU) && far) {
#pragma unroll 1
    for (int k = 0; k < rows; ++k, src += step, dst += lines * a.yp) {
      *reinterpret_cast<uint4*>(dst) = gn_each<BF>(ring.take(k), [&](int i, float x) {
        const int c = v * 8 + i;
        const double2 st = stat[gn_div(c, a.per_cpg)];
        const double u = (double)x + (a.add ? (double)gn_up(a.add[(int64_t)b * a.ld_add + c], BF) : 0.0);
        const float y = (float)fma((u - st.x) * st.y, a.gamma ? (double)a.gamma[c] : 1.0, a.beta ? (double)a.beta[c] : 0.0);
        return SILU ? gn_silu(y) : y;
      });
      ring.request(k + GN_RING - 1, src, k + GN_RING - 1 < rows);
    }
    return;
  }
#pragma unroll 2
  for (int k = 0; k < rows; ++k, src += step, dst += lines * a.yp) {
    const uint4 x = ring.take(k);
    if (k + GN_RING >= rows) pdl_launch_dependents();
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned long long y = fma_f32x2(add_f32x2(gn_pair<BF>(w[i]), shift[i]), factor[i], beta[i]);
      float y0, y1;
      unpack_f32x2(y, y0, y1);
      if (SILU) gn_silu2<BF>(y0, y1, y0, y1);
      w[i] = pack16<BF>(y0, y1);
    }
    ring.request(k + GN_RING - 1, src, k + GN_RING - 1 < rows);  // into the piece before this one
    // what would push out of L2 the map that is still to be read goes past it
    if (a.past) __stcs(reinterpret_cast<uint4*>(dst), make_uint4(w[0], w[1], w[2], w[3]));
    else *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ------------------------------------------------------------------ ... or codes
// A code next to a border of two codes, or of a zero-point that the short form has no room for, in 64 bits.
__device__ __noinline__ uint32_t gn_code_exact(const GnArgs& a, const double2* stat, bool silu, bool bf, float x, int b, int c, float inv,
                                               int z, bool centred) {
  const double2 t = stat[c / a.cpg];
  const double u = (double)x + (a.add ? (double)gn_up(a.add[(int64_t)b * a.ld_add + c], bf) : 0.0);
  double v = fma((u - t.x) * t.y, a.gamma ? (double)a.gamma[c] : 1.0, a.beta ? (double)a.beta[c] : 0.0);
  if (silu) v = v / (1.0 + exp(-v));
  const double q = fmin(fmax(rint(v * (double)inv) + (double)z, 0.0), (double)((1 << a.bits) - 1));
  return (uint32_t)((int)q - (centred ? z : 0)) & 0xFFu;
}

// The short form of a code: u = (act(y) / s - lo) / L with lo = -Z, cut off at 0 and 1, then L u + M + 1/2 + w 2^-f with M = 2^(23 - f),
// whose bits are the code and f bits of fraction below it.  It is settled if the fraction is more than 2 w, w being how far 32 bits may
// have t = act(y) / s off, in units of 2^-f.  In steps: shift, sum, factor, their product and the sum with beta by 2^-24 (4 |y| +
// 3 |beta| + |shift factor|), a SiLU's slope of at most 1.1 times that; its exponential's argument and result, the sums, the reciprocal and the
// products by 2.2 * 2^-22 of |v| for y > 0, where |y| <= |v| + 0.28, and by 2^-22 where y < 0 and y^2 e^y < 0.55; the rounded 1 / (s L) and
// lo / L and the two sums behind them by 2^-24 (|t| + 2 |lo| + 3 L).  In all 2^-22 (5 max(|lo|, |lo + L|) + L + 4 + inv (2.1 + 0.9 |beta| +
// 0.3 |shift factor| + 2^-17 |gamma|)), t beyond the ends of the range being cut off there, and one unit for the last sum's own rounding; the term of gamma
// is what a SiLU leaves of an argument far below nought, 2^-60 |y| with |y - beta| <= 2^21 |gamma|.  That holds as long as no
// number leaves the range of 32 bits: a value is at most 2^21 deviations from its group's mean, so that deviations up to 2^60 (all that fp16 has) keep it
// below 2^81, where a factor below 2^-126 costs less than 2^-69; groups of larger ones take the long form.
constexpr uint32_t GN_ALWAYS = 0x7FFF;  // the limit of channels whose codes all take the long form
__device__ __forceinline__ float gn_fixed(float shift, float factor, float gamma, float beta) {
  return 2.1f + 0.9f * fabsf(beta) + 0.3f * fabsf(shift * factor) + 0x1p-17f * fabsf(gamma);
}
// w; GN_ALWAYS where it is too large, or a scale so far out that the short form's factors may leave the range of 32 bits
template <bool EIGHT>
__device__ __forceinline__ uint32_t gn_limit(float inv, float lo, float Lf, float fixed) {
  const float off = 0x1p-22f * fmaf(5.f, fmaxf(fabsf(lo), fabsf(lo + Lf)), fmaf(inv, fixed, Lf + 4.f)) * (EIGHT ? 32768.f : 65536.f);
  return off < 8000.f && inv > 1e-30f && inv < 1e30f ? (uint32_t)off + 2u : GN_ALWAYS;
}
// M + 1/2 + w 2^-f: w counts units in the last place
template <bool EIGHT>
__device__ __forceinline__ float gn_bias(uint32_t w) { return __uint_as_float((EIGHT ? 0x43804000u : 0x43008000u) + (w == GN_ALWAYS ? 0u : w)); }
// What a fraction has to be below to be too near to a border (the fraction's f bits at the top of 16)
template <bool EIGHT>
__device__ __forceinline__ uint32_t gn_below(uint32_t w) { return w == GN_ALWAYS ? 0x10000u : (2u * w + 1u) << (EIGHT ? 1 : 0); }
__device__ __forceinline__ float gn_fma_sat(float a, float b, float c) {
  float d;
  asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// A thread has eight neighbouring channels of four rows at a time: it puts the four codes of a channel into one word at the channel's
// place in the padded row, in shared memory, and the words of 16 places are turned into 16 bytes of four rows on the way out.  Codes next to a border
// (one in some ten thousand) are noted in a list, two channels and four rows at a time, worked out in 64 bits by all threads together
// behind the last row and stored over what was written (each on the spot by its own warp: 8 x 4096 x 960 into 6 bits took 129 us, of which
// the other warps of the block waited 60); where the list is full they are worked out on the spot.  EIGHT: codes of 8 bits, f = 15, else 16.
// ROWS: pixel groups, so that scale and zero-point change from row to row.
// Of each 16 places' words the four quarters lie in an order that changes with every second 16, so that neighbouring threads read them from
// different banks on the way out.
__device__ __forceinline__ int gn_shuffle(int place) { return place ^ ((place >> 5 & 3) << 2); }  // (its own inverse)
constexpr int GN_LIST = 512;
template <bool BF, bool SILU, bool EIGHT, bool ROWS>
__global__ void __maxnreg__(64) gn_codes_kernel(const __grid_constant__ GnArgs a) {
  extern __shared__ __align__(16) unsigned char gn_smem[];
  __shared__ uint2 list[GN_LIST];  // first row, first channel
  __shared__ int listed;
  __shared__ unsigned int widest;  // (ROWS) the largest fixed part, as bits
  __shared__ int n_pads;           // (ROWS)
  const int tid = threadIdx.x, n_threads = blockDim.x, nv = a.nvec, b = blockIdx.y;
  const int set_words = a.quads * a.K_pad;
  uint32_t* words = reinterpret_cast<uint32_t*>(gn_smem);                                   // [buffers][quads][K_pad], K_pad a multiple of 32
  double2* stat = reinterpret_cast<double2*>(words + (size_t)a.buffers * set_words);         // [n_groups]
  // [4][4][nv], of channels 2 i and 2 i + 1: shift, factor | beta, places in bytes (16 bits each), groups (later, unless ROWS: limits) |
  // -log2 e over the scale of the factor, -lo / L | what takes the zero-points out of four codes, bias, -
  // Factor and beta have 1 / (s L) in them unless ROWS, and beta has -lo / L where there is no SiLU.
  float4* chan = reinterpret_cast<float4*>(stat + a.n_groups);
  float4* cell = chan + 4 * 4 * nv;  // [R][G] 1 / (s L), -lo / L, 1 / s (ROWS, later: w), Z
  // ROWS: [2][4 quads] first cell of each row of a round; places of padding in bytes, groups << 16
  int* row_cells = reinterpret_cast<int*>(cell + a.R * a.G);
  uint32_t* pads = reinterpret_cast<uint32_t*>(row_cells + 8 * a.quads);
  const int L = (1 << a.bits) - 1;
  const float Lf = (float)L, per_L = __fdividef(1.f, Lf);
  const bool centred = a.centred;
  const int p0 = (int)(gridDim.x - 1 - blockIdx.x) * a.rows, p1 = min(a.P, p0 + a.rows);
  const int64_t row0 = (int64_t)b * a.P;
  if (tid == 0) listed = 0, widest = 0, n_pads = 0;
  if (ROWS) __syncthreads();
#pragma unroll 4
  for (int i = tid; i < a.R * a.G; i += n_threads) {
    const int z = __ldg(a.zp + i);
    const float inv = __ldg(a.inv_scale + i);
    cell[i] = make_float4(inv * per_L, (float)z * per_L, inv, __int_as_float(z));
  }
  auto place_of = [&](int c) -> uint16_t& {
    return reinterpret_cast<uint16_t*>(&reinterpret_cast<uint32_t*>(&chan[(((c & 7) >> 1) * 4 + 1) * nv + (c >> 3)])[2])[c & 1];
  };
#pragma unroll 4
  for (int i = tid; i < a.K_pad; i += n_threads) {
    const int c = __ldg(a.perm + i), g = __ldg(a.chunk_group + (i >> 4));
    if (c >= 0) {
      place_of(c) = (uint16_t)(4 * gn_shuffle(i));
      (&place_of(c))[2] = (uint16_t)g;
    } else if (ROWS) {
      pads[atomicAdd(&n_pads, 1)] = 4 * gn_shuffle(i) | g << 16;  // (in any order)
    } else {  // padding: the clamped zero-point, 0 in the zero-centred layout
      const uint32_t w = centred ? 0u : 0x01010101u * (uint32_t)min(max(__ldg(a.zp + g), 0), L);
      for (int k = gn_shuffle(i); k < a.buffers * set_words; k += a.K_pad) words[k] = w;
    }
  }
  // a thread's channels and quad are the same in every round
  int quad = gn_div(tid, a.per_nvec), v = tid - quad * nv;
  gn_keep(quad), gn_keep(v);
  const bool active = quad < a.quads;
  const uint16_t* src = a.X + (int64_t)b * a.xb + (p0 + 4 * quad) * a.xp + v * 8;
  const int64_t src_step = 4 * a.quads * a.xp;
  int position = 0, advance = 0, next = 0;  // of the quad's first row among the pixel positions of the grouping
  if (ROWS) {
    position = (int)((row0 + p0 + 4 * quad) % a.row_period);
    advance = 4 * a.quads % a.row_period;
  }
  uint32_t w[4][4];
  auto request = [&](int r) {  // four rows from r
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (active && r + j < p1) x = *reinterpret_cast<const uint4*>(src + j * a.xp);
      w[j][0] = x.x, w[j][1] = x.y, w[j][2] = x.z, w[j][3] = x.w;
    }
    src += src_step;
    if (ROWS && v == 0 && active) {
      int at = position;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        row_cells[(next * a.quads + quad) * 4 + j] = __ldg(a.row_group + at) * a.G;
        if (++at == a.row_period) at = 0;
      }
      position += advance;
      if (position >= a.row_period) position -= a.row_period;
      next ^= 1;
    }
  };
  pdl_wait();
  {
    // two neighbouring channels for a thread; what belongs to the first two pairs is asked for before the statistics are waited for
    const int pairs = a.C >> 1;
    float2 gamma[2], beta[2];
    uint32_t add[2];
    auto own = [&](int z, int pair) {
      if (pair >= pairs) return;
      const int c = 2 * pair;
      gamma[z] = a.gamma ? make_float2(a.gamma[c], a.gamma[c + 1]) : make_float2(1.f, 1.f);
      beta[z] = a.beta ? make_float2(a.beta[c], a.beta[c + 1]) : make_float2(0.f, 0.f);
      const uint16_t* e = a.add + (int64_t)b * a.ld_add + c;
      add[z] = a.add ? e[0] | (uint32_t)e[1] << 16 : 0u;
    };
    own(0, tid);
    own(1, tid + n_threads);
    gn_stats(a, b, stat, [&]() { request(p0 + 4 * quad); });  // (ends in a barrier: places and cells are set)
    for (int pair = tid, z = 0; pair < pairs; pair += n_threads, ++z) {
      if (z >= 2) own(0, pair);
      const bool second = z == 1;
      const int at = (pair & 3) * 4 * nv + (pair >> 2);
      float4& one = chan[at + nv];
      const uint32_t places = __float_as_uint(one.z), groups = __float_as_uint(one.w);
      float t[2][6];  // shift, factor, beta, exponent's factor, -lo / L, zero-points
      uint32_t w = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const double2 st = stat[gn_div(2 * pair + h, a.per_cpg)];
        const float2 g2 = second ? gamma[1] : gamma[0], b2 = second ? beta[1] : beta[0];
        const uint32_t e2 = second ? add[1] : add[0];
        const float be = h ? b2.y : b2.x;
        t[h][0] = (float)((double)gn_up((uint16_t)(h ? e2 >> 16 : e2), BF) - st.x);
        t[h][1] = (float)st.y * (h ? g2.y : g2.x);
        t[h][2] = be;
        t[h][3] = t[h][4] = t[h][5] = 0.f;
        const float fixed = BF && st.y < (double)GN_FAR ? INFINITY : gn_fixed(t[h][0], t[h][1], h ? g2.y : g2.x, be);
        if (ROWS) {
          atomicMax(&widest, fixed < INFINITY ? __float_as_uint(fixed) : 0x7F800000u);  // (any order gives the same)
        } else {
          const float4 z4 = cell[groups >> (16 * h) & 0xFFFFu];
          w = max(w, gn_limit<EIGHT>(z4.z, -(float)__float_as_int(z4.w), Lf, fixed));  // one limit for both channels
          t[h][1] *= z4.x;
          t[h][2] = SILU ? be * z4.x : fmaf(be, z4.x, z4.y);
          t[h][3] = __fdividef(-1.4426950408889634f, z4.x);
          t[h][4] = z4.y;
          t[h][5] = __uint_as_float(0x80808080u - 0x01010101u * __float_as_uint(z4.w));
        }
      }
      const uint32_t below = min(gn_below<EIGHT>(w), 0xFFFFu);
      chan[at] = make_float4(t[0][0], t[1][0], t[0][1], t[1][1]);
      one = make_float4(t[0][2], t[1][2], __uint_as_float(places), __uint_as_float(ROWS ? groups : below | below << 16));
      if (!ROWS) {
        chan[at + 2 * nv] = make_float4(t[0][3], t[1][3], t[0][4], t[1][4]);
        chan[at + 3 * nv] = make_float4(t[0][5], t[1][5], gn_bias<EIGHT>(w), 0.f);
      }
    }
  }
  __syncthreads();
  if (ROWS) {
    for (int i = tid; i < a.R * a.G; i += n_threads) {
      const float4 t = cell[i];
      cell[i].z = __uint_as_float(gn_limit<EIGHT>(t.z, -(float)__float_as_int(t.w), Lf, __uint_as_float(widest)));
    }
    __syncthreads();
  }
  // the code of one value, in 64 bits
  auto exact = [&](int p, int c) {
    const uint16_t value = a.X[(int64_t)b * a.xb + p * a.xp + c];
    const int at = (ROWS ? __ldg(a.row_group + (row0 + p) % a.row_period) * a.G : 0) + __ldg(a.chunk_group + (place_of(c) >> 6));
    return gn_code_exact(a, stat, SILU, BF, gn_up(value, BF), b, c, ROWS ? __ldg(a.inv_scale + at) : cell[at].z, __float_as_int(cell[at].w), centred);
  };
  // this thread's first 16 places on the way out, the same in every round
  int chunks = a.K_pad >> 4, out_quad = gn_div(tid, a.per_chunks), out_chunk = tid - out_quad * chunks;
  gn_keep(out_quad), gn_keep(out_chunk), gn_keep(chunks);
  uint32_t my_words = smem_u32(words + quad * a.K_pad);  // flips between the two sets
  for (int p = p0, round = 0; p < p1; p += 4 * a.quads, ++round) {
    const int r = p + 4 * quad;
    if (active && r < p1) {
      int4 rg = make_int4(0, 0, 0, 0);
      if (ROWS) rg = *reinterpret_cast<const int4*>(row_cells + ((round & 1) * a.quads + quad) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 k0 = chan[i * 4 * nv + v], k1 = chan[(i * 4 + 1) * nv + v];
        float4 k2 = k0, k3 = k0;
        if (!ROWS) {
          if (SILU) k2 = chan[(i * 4 + 2) * nv + v];
          k3 = chan[(i * 4 + 3) * nv + v];
        }
        const uint32_t places = __float_as_uint(k1.z);
        uint32_t m[2][4];
        bool near_border = false;
        uint32_t zero[2] = {0, 0};  // (ROWS, zero-centred) the rows' zero-points
        float4 c0 = make_float4(0.f, 0.f, 0.f, 0.f), c1 = c0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = unpack16<BF>(w[j][i]);
          float y0 = f.x + k0.x, y1 = f.y + k0.y, bias0 = k3.z, bias1 = k3.z;  // (NaN is cut off to the lower end)
          if (ROWS) {
            const int mine = j == 0 ? rg.x : j == 1 ? rg.y : j == 2 ? rg.z : rg.w, before = j == 1 ? rg.x : j == 2 ? rg.y : rg.z;
            if (j == 0 || mine != before) {  // (rows next to each other are mostly of one group)
              c0 = cell[mine + (int)(__float_as_uint(k1.w) & 0xFFFFu)], c1 = cell[mine + (int)(__float_as_uint(k1.w) >> 16)];
            }
            y0 = fmaf(y0, k0.z, k1.x), y1 = fmaf(y1, k0.w, k1.y);
            if (SILU) gn_silu2<true>(y0, y1, y0, y1);
            y0 = gn_fma_sat(y0, c0.x, c0.y), y1 = gn_fma_sat(y1, c1.x, c1.y);
            bias0 = gn_bias<EIGHT>(__float_as_uint(c0.z)), bias1 = gn_bias<EIGHT>(__float_as_uint(c1.z));
            m[0][j] = __float_as_uint(fmaf(y0, Lf, bias0)) << (EIGHT ? 1 : 0);
            m[1][j] = __float_as_uint(fmaf(y1, Lf, bias1)) << (EIGHT ? 1 : 0);
            near_border |= (m[0][j] & 0xFFFFu) < gn_below<EIGHT>(__float_as_uint(c0.z)) || (m[1][j] & 0xFFFFu) < gn_below<EIGHT>(__float_as_uint(c1.z));
            zero[0] |= (__float_as_uint(c0.w) & 0xFFu) << (8 * j);
            zero[1] |= (__float_as_uint(c1.w) & 0xFFu) << (8 * j);
          } else if (SILU) {
            y0 = fmaf(y0, k0.z, k1.x), y1 = fmaf(y1, k0.w, k1.y);
            float e0, e1, per;
            gn_silu_parts(y0, y1, k2.x, k2.y, e0, e1, per);
            y0 = gn_fma_sat(y0, e1 * per, k2.z), y1 = gn_fma_sat(y1, e0 * per, k2.w);
          } else {
            y0 = gn_fma_sat(y0, k0.z, k1.x), y1 = gn_fma_sat(y1, k0.w, k1.y);
          }
          if (!ROWS) {
            m[0][j] = __float_as_uint(fmaf(y0, Lf, bias0)) << (EIGHT ? 1 : 0);
            m[1][j] = __float_as_uint(fmaf(y1, Lf, bias1)) << (EIGHT ? 1 : 0);
          }
        }
        if (!ROWS) {
          // the least fractions: low halves of two rows side by side
          const uint32_t f0 = __vminu2(__byte_perm(m[0][0], m[0][1], 0x5410), __byte_perm(m[0][2], m[0][3], 0x5410));
          const uint32_t f1 = __vminu2(__byte_perm(m[1][0], m[1][1], 0x5410), __byte_perm(m[1][2], m[1][3], 0x5410));
          const uint32_t below = __float_as_uint(k1.w);
          near_border = below == 0xFFFFFFFFu || __vminu2(__vminu2(f0, f1), below) != below;
        }
        uint32_t word[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          word[h] = __byte_perm(__byte_perm(m[h][0], m[h][1], 0x0062), __byte_perm(m[h][2], m[h][3], 0x0062), 0x5410);
          if (centred) {
            // codes of 8 bits have the zero-point 128; fewer bits leave the upper one free, so that no byte borrows from the next
            if (EIGHT) word[h] ^= 0x80808080u;
            else if (ROWS) word[h] = __vsub4(word[h], zero[h]);
            else word[h] = (word[h] + __float_as_uint(h ? k3.y : k3.x)) ^ 0x80808080u;
          }
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(my_words + (h ? places >> 16 : places & 0xFFFFu)), "r"(word[h]) : "memory");
        }
        if (near_border) {
          const int at = atomicAdd(&listed, 1);
          if (at < GN_LIST) {
            list[at] = make_uint2(r, v * 8 + 2 * i);
          } else {
#pragma unroll 1
            for (int j = 0; j < 8; ++j)
              if (r + (j & 3) < p1)
                asm volatile("st.shared.u8 [%0], %1;" ::"r"(my_words + (j >> 2 ? places >> 16 : places & 0xFFFFu) + (j & 3)),
                             "r"(exact(r + (j & 3), v * 8 + 2 * i + (j >> 2)))
                             : "memory");
          }
        }
      }
    }
    request(r + 4 * a.quads);  // arrives while this round's rows leave
    uint32_t* out_words = words + (a.buffers == 2 && (round & 1) ? set_words : 0);
    if (ROWS) {  // padding
      const int count = n_pads;
      const float per_count = __fdividef(1.f, (float)count);
      for (int i = tid; i < count * a.quads; i += n_threads) {
        const int q = gn_div(i, per_count);
        const uint32_t pad = pads[i - q * count];
        uint32_t word = 0;
        if (!centred) {
          const int* rows = row_cells + ((round & 1) * a.quads + q) * 4;
#pragma unroll
          for (int j = 0; j < 4; ++j) word |= (uint32_t)min(max(__float_as_int(cell[rows[j] + (int)(pad >> 16)].w), 0), L) << (8 * j);
        }
        out_words[q * a.K_pad + (int)(pad & 0xFFFFu) / 4] = word;
      }
    }
    __syncthreads();
    if (p + 4 * a.quads >= p1) pdl_launch_dependents();  // (earlier, the next kernel's blocks would crowd this one's)
    for (int q = out_quad, ch = out_chunk; q < a.quads;) {
      const int row = p + 4 * q;
      if (row >= p1) break;
      const uint4* s = reinterpret_cast<const uint4*>(out_words + q * a.K_pad + ch * 16);
      uint32_t out[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 t = s[i ^ (ch >> 1 & 3)];
        const uint32_t lo01 = __byte_perm(t.x, t.y, 0x5140), hi01 = __byte_perm(t.x, t.y, 0x7362);
        const uint32_t lo23 = __byte_perm(t.z, t.w, 0x5140), hi23 = __byte_perm(t.z, t.w, 0x7362);
        out[0][i] = __byte_perm(lo01, lo23, 0x5410);
        out[1][i] = __byte_perm(lo01, lo23, 0x7632);
        out[2][i] = __byte_perm(hi01, hi23, 0x5410);
        out[3][i] = __byte_perm(hi01, hi23, 0x7632);
      }
      uint8_t* dst = a.Xq + (row0 + row) * a.K_pad + ch * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (row + j < p1) *reinterpret_cast<uint4*>(dst + j * a.K_pad) = make_uint4(out[j][0], out[j][1], out[j][2], out[j][3]);
      ch += n_threads;
      while (ch >= chunks) ch -= chunks, ++q;
    }
    // (with two sets of words the next round's barrier says that this round's have been read)
    if (a.buffers == 1) __syncthreads();
    else my_words += round & 1 ? -4 * set_words : 4 * set_words;
  }
  __syncthreads();  // the rows are written, the list is complete
  for (int k = tid; k < min(listed, GN_LIST) * 8; k += n_threads) {
    const int p = (int)list[k >> 3].x + (k & 3), c = (int)list[k >> 3].y + (k >> 2 & 1);
    if (p < p1) a.Xq[(row0 + p) * a.K_pad + gn_shuffle(place_of(c) >> 2)] = (uint8_t)exact(p, c);
  }
}
#endif

// ------------------------------------------------------------------ host
// Whether eight neighbouring channels lie in at most two groups.
static inline bool gn_two_parts(int cpg) { return cpg == 4 || cpg >= 7; }
static inline int gn_gcd(int a, int b) { return b ? gn_gcd(b, a % b) : a; }

// The sums' kernel: lines of rows of a block, rows of a block, blocks of a cluster, clusters of an image.  Two blocks for each
// multiprocessor over all images (the numbers do not depend on the device, so that the workspace does not either), at least two
// rows for each line.
struct GnSumsPlan {
  int nvec, lines, threads, rows, cluster, clusters;
};
static inline GnSumsPlan gn_sums_plan(int B, int P, int C) {
  GnSumsPlan s;
  s.nvec = std::max(1, C / 8);
  s.lines = std::max(1, 256 / s.nvec);
  s.threads = (s.lines * s.nvec + 31) / 32 * 32;
  const int most = (P - 1) / (2 * s.lines) + 1;
  int slabs = std::max(1, std::min((296 + B - 1) / B, most));
  s.cluster = slabs >= 128 ? 16 : slabs >= 8 ? 8 : slabs >= 4 ? 4 : slabs >= 2 ? 2 : 1;
  s.clusters = (slabs + s.cluster - 1) / s.cluster;
  slabs = s.clusters * s.cluster;
  s.rows = (P - 1) / slabs + 1;
  return s;
}
static inline size_t gn_sums_bytes(int B, int P, int C, int n_groups) {
  return (size_t)B * gn_sums_plan(B, P, C).clusters * n_groups * sizeof(double2);
}

// The one kernel for values: eights of channels of a block (whole groups), blocks of a cluster, lines of rows of a block, rows
// of a thread, bytes of shared memory.  ok: whether the map fits that way.
struct GnChipPlan {
  bool ok;
  int nvec, cluster, lines, rows, threads;
  size_t smem;
};
static inline GnChipPlan gn_chip_plan(int B, int P, int C, int cpg) {
  GnChipPlan s = {};
  const int unit = cpg / gn_gcd(cpg, 8), units = C / 8 / unit;  // eights of channels that are whole groups
  // at least 64 bytes of a row, so that few sectors are fetched by two blocks
  int k = 1;
  while (k < units && (k * unit < 4 || units % k)) ++k;
  s.nvec = k * unit;
  if (s.nvec > GN_MAX_THREADS) return s;
  const int64_t blocks = (int64_t)B * (units / k);
  for (int cluster = 1; cluster <= 16 && cluster <= P; cluster *= 2) {
    const int rows = (P - 1) / cluster + 1;
    // about 256 threads, so that several blocks fit a multiprocessor (and clusters of eight the GPU: of blocks that each fill one, a
    // sixteenth cluster waits for the others), two rows a thread at least
    const int lines = std::min(std::max(1, 256 / s.nvec), std::max(1, (rows + 1) / 2)), threads = (lines * s.nvec + 31) / 32 * 32;
    const int per_thread = (rows - 1) / lines + 1;
    if (per_thread > 64) continue;
    const size_t smem = (size_t)per_thread * threads * 16 + (size_t)(gn_two_parts(cpg) ? 2 : 8) * lines * s.nvec * sizeof(float2) +
                        (size_t)(1 + 2 * cluster) * (s.nvec * 8 / cpg) * 8;
    if (smem > GN_SMEM_MAX) continue;
    if (s.ok && cluster > 8) break;
    s.ok = true;
    s.cluster = cluster, s.lines = lines, s.threads = threads, s.rows = per_thread, s.smem = smem;
    // further split while blocks are few or large
    const int64_t bytes = (int64_t)rows * s.nvec * 16;
    if ((blocks * cluster >= 96 && bytes <= 48 * 1024) || bytes <= 16 * 1024) break;
  }
  // Blocks that fill a multiprocessor each, in several rounds, read, join and write one after the other: two kernels are faster then (with a SiLU, one
  // kernel against two: 1 x 16384 x 1280 46.8 and 37.9 us, 2 x 9216 x 960 39.7 and 29.2, 4 x 4096 x 960 36 and 27, 8 x 4096 x 960 62 and 43, 8 x 16384 x
  // 320 79 and 54).  In one round one is (64 blocks, 1 x 4096 x 960: 12.5 and 15.6), though not where sixteen clusters of eight, one of which has to
  // wait, count as one round here (128 blocks, 2 x 4096 x 960: 23.8 and 18.7).  Of smaller blocks neither is for all (8 x 4096 x 640 33.0 and 32.5,
  // 2 x 9216 x 640 19.2 and 22.8, 2 x 9216 x 1280 35.1 and 40.4; without an activation 30.5 and 27.6, 18.2 and 19.7, 33.0 and 30.3).
  if (s.smem > 110 * 1024 && blocks * s.cluster > 148) s.ok = false;
  return s;
}

static dgq_status gn_check(const dgq_rows* X, const void* add, int64_t ld_add, int dtype, int B, int P, int C, int n_groups, float eps, int act) {
  if (!rows_pointer_ok(X) || B <= 0 || P <= 0 || C <= 0 || n_groups <= 0 || C % n_groups || (dtype != DGQ_F16 && dtype != DGQ_BF16) ||
      (act != DGQ_ACT_NONE && act != DGQ_ACT_SILU) || !(eps >= 0x1p-126f) || !std::isfinite(eps) || (add && B > 1 && ld_add < 0))
    return DGQ_ERR_INVALID_ARG;
  if (C % 8 || C > GN_MAX_C || P > GN_MAX_PIXELS || B > 65535) return DGQ_ERR_UNSUPPORTED;
  return rows_check(*X, B, P, 1, false);
}
// Whether two rows of C elements of an output with pixels at least C apart meet: rows p of image 0 and q of image d do if d * batch lies within C of (p - q) * token.
static bool gn_overlap(const dgq_rows& y, int B, int P, int C) {
  if (B == 1) return false;
  if (P == 1 || y.batch < C) return y.batch < C;
  if (y.token >= (B - 1) * y.batch + C) return false;  // pixels outermost
  for (int64_t d = 1; d < B; ++d) {
    const int64_t p = d * y.batch / y.token, past = d * y.batch % y.token;
    if (p >= P) return false;  // images outermost from here on
    if (past < C || (p + 1 < P && y.token - past < C)) return true;
  }
  return false;
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
  a.cpg = C / n_groups;
  a.eps = eps;
  a.part = (double2*)workspace;
  a.per_cpg = 1.f / (float)a.cpg;
  a.count = (double)P * (double)a.cpg;
  a.per_count = 1.0 / a.count;
}
static void gn_shape(GnArgs& a, int nvec, int lines) {
  a.nvec = nvec;
  a.lines = lines;
  a.per_nvec = 1.f / (float)nvec;
  a.per_lines = 1.f / (float)lines;
}
static dgq_status gn_workspace_check(size_t need, const void* workspace, size_t bytes) {
  if (!need) return DGQ_OK;
  if (!workspace || bytes < need) return DGQ_ERR_WORKSPACE;
  return (reinterpret_cast<uintptr_t>(workspace) & 255u) ? DGQ_ERR_ALIGNMENT : DGQ_OK;
}

// A launch in clusters that follows the kernel before it as launch_pdl does.  `done`: whether the kernel has been opted in to its shared
// memory, and to clusters of sixteen, on a device.
static cudaError_t gn_launch(void (*kernel)(GnArgs), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t stream, const GnArgs& a,
                             std::atomic<bool>* done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !done[dev].load()) {
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)GN_SMEM_MAX)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess)
      return e;
    if (dev < 64) done[dev].store(true);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  if ((e = cudaLaunchKernelEx(&cfg, kernel, a)) == cudaSuccess) g_launches += 1;
  return e;
}

template <bool BF, int SEG>
static dgq_status gn_sums(GnArgs a, int B, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const GnSumsPlan s = gn_sums_plan(B, a.P, a.C);
  gn_shape(a, s.nvec, s.lines);
  a.slab_rows = s.rows;
  // Where a map is small the second kernel's first steps hide behind this one's; where it is large its blocks would take the places of this one's.
  a.early = (int64_t)B * a.P * a.C <= 8 << 20;
  a.clusters = s.clusters;
  a.log_cluster = s.cluster == 16 ? 4 : s.cluster == 8 ? 3 : s.cluster / 2;
  const size_t smem = (size_t)(a.n_groups + s.cluster) * sizeof(double2) + std::max((size_t)SEG * s.lines * s.nvec * sizeof(double2), (size_t)s.threads * GN_RING * 16);
  DGQ_CUDA_OK(gn_launch(gn_sums_kernel<BF, SEG>, dim3(s.clusters * s.cluster, B), s.threads, smem, s.cluster, stream, a, done));
  return DGQ_OK;
}
template <bool BF>
static dgq_status gn_sums_pick(GnArgs& a, int B, cudaStream_t stream) {
  a.clusters = gn_sums_plan(B, a.P, a.C).clusters;
  return gn_two_parts(a.cpg) ? gn_sums<BF, 2>(a, B, stream) : gn_sums<BF, 8>(a, B, stream);
}

template <bool BF, bool SILU, int SEG>
static dgq_status gn_chip(GnArgs& a, int B, const GnChipPlan& p, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  gn_shape(a, p.nvec, p.lines);
  a.rows = p.rows;
  a.log_cluster = p.cluster == 16 ? 4 : p.cluster == 8 ? 3 : p.cluster / 2;
  DGQ_CUDA_OK(gn_launch(gn_chip_kernel<BF, SILU, SEG>, dim3(p.cluster, a.C / 8 / a.nvec, B), p.threads, p.smem, p.cluster, stream, a, done));
  return DGQ_OK;
}

template <bool BF, bool SILU>
static dgq_status gn_values(GnArgs& a, int B, cudaStream_t stream) {
  const GnChipPlan p = gn_chip_plan(B, a.P, a.C, a.cpg);
  if (p.ok) {
    return gn_two_parts(a.cpg) ? gn_chip<BF, SILU, 2>(a, B, p, stream) : gn_chip<BF, SILU, 8>(a, B, p, stream);
  }
  static std::atomic<bool> done[64];
  const dgq_status st = gn_sums_pick<BF>(a, B, stream);
  if (st != DGQ_OK) return st;
  gn_shape(a, a.C / 8, std::max(1, 256 / (a.C / 8)));
  const int threads = (a.lines * a.nvec + 31) / 32 * 32;
  const int step = 4 * a.lines, rounds = (int)(((int64_t)B * a.P + 444ll * step - 1) / (444ll * step));  // three blocks for each multiprocessor
  a.rows = (int)std::min<int64_t>((int64_t)rounds * step, 1 << 30);
  // (without an activation 8 x 4096 x 960 38.4 -> 37.0 us, 4 x 65536 x 128 39.7 -> 38.8, 1 x 262144 x 128 41.2 -> 40.7; with a SiLU, below and from twice
  // that size on the same to 0.5 % either way)
  a.past = (int64_t)B * a.P * a.C >= 24 << 20;
  DGQ_CUDA_OK(gn_launch(gn_values_kernel<BF, SILU>, dim3((a.P - 1) / a.rows + 1, B), threads,
                        a.n_groups * sizeof(double2) + (size_t)threads * GN_RING * 16, 1, stream, a, done));
  return DGQ_OK;
}
template <bool BF, bool SILU, bool EIGHT, bool ROWS>
static dgq_status gn_codes(GnArgs& a, int B, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const dgq_status st = gn_sums_pick<BF>(a, B, stream);
  if (st != DGQ_OK) return st;
  gn_shape(a, a.C / 8, 1);
  a.per_chunks = 16.f / (float)a.K_pad;
  // as many quads of rows as 256 threads have, within 48 KB
  a.quads = std::max(1, std::min({256 / a.nvec, 48 * 1024 / (a.K_pad * 4), (a.P + 3) / 4}));
  const int threads = (a.quads * a.nvec + 31) / 32 * 32, step = 4 * a.quads;
  const size_t fixed = a.n_groups * sizeof(double2) + (size_t)a.C / 2 * 4 * sizeof(float4) + (size_t)a.R * a.G * sizeof(float4) +
                       (ROWS ? (size_t)a.quads * 32 + (size_t)(a.K_pad - a.C) * 4 : 0);
  const size_t set = (size_t)a.quads * a.K_pad * 4;
  static_assert((GN_MAX_C + 39 * DGQ_MAX_GROUPS) * 4 + GN_MAX_CODE_GROUPS * 16 + GN_MAX_C / 2 * 64 + DGQ_MAX_GROUPS * DGQ_MAX_GROUPS * 16 + 32 +
                        39 * DGQ_MAX_GROUPS * 4 <=
                    GN_SMEM_MAX,
                "one quad of the widest row");
  // one wave of blocks, as many as registers (64 a thread) and shared memory (with 5 KB of the kernel's own and the system's) allow
  auto fit = [&](int buffers) { return std::max<int>(1, std::min<size_t>(1024 / threads, 233472 / (fixed + buffers * set + 5 * 1024 + 512))); };
  // (one set fits beside any table, two do not beside the widest row with the most groups and cells)
  a.buffers = fit(2) == fit(1) && fixed + 2 * set <= GN_SMEM_MAX ? 2 : 1;
  const int64_t wave = 148ll * fit(a.buffers) * step, rounds = ((int64_t)B * a.P + wave - 1) / wave;
  if (rounds == 1) a.buffers = 1;
  a.rows = (int)std::min<int64_t>(rounds * step, 1 << 30);
  DGQ_CUDA_OK(gn_launch(gn_codes_kernel<BF, SILU, EIGHT, ROWS>, dim3((a.P - 1) / a.rows + 1, B), threads, fixed + a.buffers * set, 1,
                        stream, a, done));
  return DGQ_OK;
}
template <bool BF, bool SILU>
static dgq_status gn_codes_pick(GnArgs& a, int B, cudaStream_t stream) {
  if (a.row_group) return a.bits == 8 ? gn_codes<BF, SILU, true, true>(a, B, stream) : gn_codes<BF, SILU, false, true>(a, B, stream);
  return a.bits == 8 ? gn_codes<BF, SILU, true, false>(a, B, stream) : gn_codes<BF, SILU, false, false>(a, B, stream);
}

}  // namespace dgq

extern "C" dgq_status dgq_group_norm_workspace_bytes(int B, int P, int C, int n_groups, int quantize, size_t* bytes) {
  using namespace dgq;
  if (!bytes || B <= 0 || P <= 0 || C <= 0 || n_groups <= 0 || C % n_groups) return DGQ_ERR_INVALID_ARG;
  if (C % 8 || C > GN_MAX_C || P > GN_MAX_PIXELS || B > 65535) return DGQ_ERR_UNSUPPORTED;
  *bytes = !quantize && gn_chip_plan(B, P, C, C / n_groups).ok ? 0 : gn_sums_bytes(B, P, C, n_groups);
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
  const size_t need = gn_chip_plan(B, P, C, C / n_groups).ok ? 0 : gn_sums_bytes(B, P, C, n_groups);
  if ((st = gn_workspace_check(need, workspace, workspace_bytes)) != DGQ_OK) return st;
  if (gn_overlap(*Y, B, P, C)) return DGQ_ERR_INVALID_ARG;
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
  if (n_groups > GN_MAX_CODE_GROUPS) return DGQ_ERR_UNSUPPORTED;
  if (!g->filled[timestep]) return DGQ_ERR_NOT_CALIBRATED;
  const size_t trow = (size_t)timestep * g->R * g->G;
  const int L = (1 << g->bits) - 1;
  if (layout == DGQ_CODES_S8_CENTRED)
    for (int i = 0; i < g->R * g->G; ++i)
      if (g->zp[trow + i] > 128 || g->zp[trow + i] < L - 127) return DGQ_ERR_UNSUPPORTED;
  if ((st = gn_workspace_check(gn_sums_bytes(B, P, g->C, n_groups), workspace, workspace_bytes)) != DGQ_OK) return st;
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
  a.centred = layout == DGQ_CODES_S8_CENTRED;
  const cudaStream_t s = (cudaStream_t)stream;
  if (dtype == DGQ_BF16) return act == DGQ_ACT_SILU ? gn_codes_pick<true, true>(a, B, s) : gn_codes_pick<true, false>(a, B, s);
  return act == DGQ_ACT_SILU ? gn_codes_pick<false, true>(a, B, s) : gn_codes_pick<false, false>(a, B, s);
}
