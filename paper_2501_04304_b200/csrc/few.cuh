// Products of few 16-bit rows with 4-bit weights.
//
//     Y[m, n] = bias[n] + sum_g s[n, g] sum_{k in g} q[n, k] act(X[m, k]),   q in -8 .. 7, one fp16 scale for `group` input channels
//
// The weights are read once and bound the call.  They lie in tiles of 16 outputs x 64 input channels, 512 bytes, in the
// order in which the lanes of a warp need them as the first operand of mma.sync (16 outputs x 16 channels): one 16-byte load per lane is
// four steps.  Eight rows of X are the second operand.  Which channel stands at which place of a step is free as long as
// both operands agree, so that a lane's part of a row is two times 16 contiguous bytes.  A code becomes a 16-bit float by two bit
// operations (its bits under those of a power of two) and one exact subtraction; products with whole numbers of 4 bits are exact in the
// accumulator's 32 bits, where also the scales are applied, group by group.
#pragma once

#include <new>

#include "group_norm.cuh"

struct dgq_few_weight {
  int N = 0, K = 0, group = 0;
  int tiles = 0, blocks = 0, n_groups = 0;  // ceil(N / 16), ceil(K / 64), ceil(K / group)
  unsigned char* d_slab = nullptr;
  uint4* d_codes = nullptr;     // [tiles][blocks][32]
  uint32_t* d_scale = nullptr;  // [tiles][scale columns][8]: fp16 scales of outputs r and r + 8
  int device = 0;
};

namespace dgq {

constexpr int FEW_MOST = (1 << 20) - 16;      // outputs and input channels: at most 65535 tiles of 16
constexpr int FEW_MOST_ROWS = (1 << 21) - 32;  // 65535 times 32

// Scale columns of a tile: the groups of whole blocks (a group of 128 has two blocks).
__host__ __device__ inline int few_columns(int blocks, int group) { return group == 32 ? 2 * blocks : group == 64 ? blocks : (blocks + 1) / 2; }

#ifdef __CUDACC__

// ------------------------------------------------------------------ weights
// Place of code (r of 16, k of 64) of a tile: word of the tile and shift.  Lane 4 (r % 8) + c has channels 8 c .. 8 c + 7 of either half of
// the block, of outputs r % 8 and r % 8 + 8; its words 0 and 1 are those of the first half, four channels each (so that two steps
// are 32 neighbouring channels, the smallest group).  In a word, nibble i and nibble 4 + i are the two halves of operand register i:
// channels 0, 1 of the lower output, of the upper one, channels 2, 3 of the lower, of the upper.
__host__ __device__ inline void few_place(int r, int k, int* word, int* shift) {
  const int lane = 4 * (r & 7) + ((k >> 3) & 3), j = 2 * (k >> 5) + ((k >> 2) & 1), reg = (r >> 3) + 2 * ((k >> 1) & 1), half = k & 1;
  *word = lane * 4 + j;
  *shift = 4 * (reg + 4 * half);
}

struct FewPackArgs {
  const __half* W;         // [N][K], or null
  const int8_t* wq;        // [N][K]
  const __half* scales;    // [N][n_groups]
  int N, K, group, n_groups, blocks, columns;
  uint32_t* codes;
  __half* scale_out;
  int* bad;
};

// One block per tile of 16 outputs and 128 input channels; a thread has eight channels of one output.
__global__ void __launch_bounds__(256) few_pack_kernel(const FewPackArgs a) {
  __shared__ uint32_t words[2][128];
  const int tid = threadIdx.x, r = tid >> 4, k0 = blockIdx.x * 128 + (tid & 15) * 8, n = blockIdx.y * 16 + r;
  words[tid >> 7][tid & 127] = 0;
  __syncthreads();
  const int per = a.group / 8;  // threads of a group
  const bool in = n < a.N && k0 < a.K;
  int q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  bool bad = false;
  __half s = __ushort_as_half(0);
  if (a.W) {
    // s = max |w| / 7 rounded up, so that no code is beyond 7; code = rint(w / s)
    float w[8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = in ? __half2float(a.W[(size_t)n * a.K + k0 + i]) : 0.f;
      bad |= !(fabsf(w[i]) < INFINITY);
      top = fmaxf(top, fabsf(w[i]));
    }
    for (int o = 1; o < per; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    s = __float2half_ru(__fdiv_ru(top, 7.f));
    const float f = __half2float(s);
    if (top > 0.f)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = (int)rintf(__fdiv_rn(w[i], f));
  } else if (in) {
    s = a.scales[(size_t)n * a.n_groups + k0 / a.group];
    bad |= !(fabsf(__half2float(s)) < INFINITY);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      q[i] = a.wq[(size_t)n * a.K + k0 + i];
      bad |= q[i] < -8 || q[i] > 7;
    }
  }
  if (bad) *a.bad = 1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int word, shift;
    few_place(r, (k0 + i) & 63, &word, &shift);
    atomicOr(&words[(tid & 15) >> 3][word], (uint32_t)((q[i] + 8) & 15) << shift);
  }
  __syncthreads();
  const int block = blockIdx.x * 2 + (tid >> 7);
  if (block < a.blocks) a.codes[((size_t)blockIdx.y * a.blocks + block) * 128 + (tid & 127)] = words[tid >> 7][tid & 127];
  const int column = k0 / a.group;
  if ((tid & 15) % per == 0 && column < a.columns)
    a.scale_out[((size_t)blockIdx.y * a.columns + column) * 16 + (r & 7) * 2 + (r >> 3)] = in ? s : __ushort_as_half(0);
}

// ------------------------------------------------------------------ products
struct FewArgs {
  const uint4* codes;
  const uint32_t* scale;
  const uint16_t* X;
  int64_t ldx;
  const uint16_t* bias;
  uint16_t* Y;
  int64_t ldy;
  int M, N, K, blocks, columns, tiles;
};

constexpr int FEW_WARPS = 8;

// Codes -> two 16-bit floats each.  fp16: 1024 + q has q in its low bits, 1024 + 16 q in bits 4 to 7.  bf16: 128 + q.
template <bool BF>
__device__ __forceinline__ void few_widen(uint32_t w, uint32_t (&r)[4]) {
  if (BF) {
    const __nv_bfloat162 off = __floats2bfloat162_rn(-136.f, -136.f), one = __floats2bfloat162_rn(1.f, 1.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
      const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&t), one, off);
      r[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
  } else {
    const __half2 off = __floats2half2_rn(-1032.f, -1032.f), off16 = __floats2half2_rn(-72.f, -72.f), by16 = __floats2half2_rn(0.0625f, 0.0625f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t x = i ? w >> 8 : w, t0 = (x & 0x000F000Fu) | 0x64006400u, t1 = (x & 0x00F000F0u) | 0x64006400u;
      const __half2 v0 = __hadd2(*reinterpret_cast<const __half2*>(&t0), off);
      const __half2 v1 = __hfma2(*reinterpret_cast<const __half2*>(&t1), by16, off16);
      r[2 * i] = *reinterpret_cast<const uint32_t*>(&v0);
      r[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&v1);
    }
  }
}
template <bool BF>
__device__ __forceinline__ void few_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// NT tiles of outputs and MT times eight rows for a block, whose warps take every eighth block of 64 channels.
template <bool BF, bool SILU, int GROUP, int NT, int MT>
__global__ void __launch_bounds__(FEW_WARPS * 32) few_kernel(const __grid_constant__ FewArgs a) {
  __shared__ float part[FEW_WARPS][MT * 8][NT * 16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
  const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * MT * 8;
  pdl_launch_dependents();
  pdl_wait();
  float acc[NT][MT][4] = {};
#pragma unroll 2
  for (int kb = warp; kb < a.blocks; kb += FEW_WARPS) {
    uint4 w[NT];
    uint32_t s[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int tile = min(tile0 + t, a.tiles - 1);
      w[t] = __ldg(a.codes + ((size_t)tile * a.blocks + kb) * 32 + lane);
      const uint32_t* sc = a.scale + (size_t)tile * a.columns * 8 + r;
      if (GROUP == 32) {
        s[t][0] = __ldg(sc + kb * 16);
        s[t][1] = __ldg(sc + kb * 16 + 8);
      } else {
        s[t][0] = __ldg(sc + (GROUP == 64 ? kb : kb >> 1) * 8);
      }
    }
    uint32_t x[MT][8];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int row = m0 + 8 * m + r, k = kb * 64 + 8 * c;
      const uint4* src = reinterpret_cast<const uint4*>(a.X + row * a.ldx + k);
      const uint4 z = make_uint4(0, 0, 0, 0);
      const uint4 x0 = row < a.M && k < a.K ? __ldg(src) : z, x1 = row < a.M && k + 32 < a.K ? __ldg(src + 4) : z;
      x[m][0] = x0.x, x[m][1] = x0.y, x[m][2] = x0.z, x[m][3] = x0.w;
      x[m][4] = x1.x, x[m][5] = x1.y, x[m][6] = x1.z, x[m][7] = x1.w;
      if (SILU)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = unpack16<BF>(x[m][i]);
          x[m][i] = pack16<BF>(gn_silu(f.x), gn_silu(f.y));
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t words[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
      float d[MT][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t op[4];
        few_widen<BF>(words[j], op);
        if (j == 0 || (GROUP == 32 && j == 2))
#pragma unroll
          for (int m = 0; m < MT; ++m) d[m][0] = d[m][1] = d[m][2] = d[m][3] = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m) few_mma<BF>(d[m], op, x[m][2 * j], x[m][2 * j + 1]);
        if (j == 3 || (GROUP == 32 && j == 1)) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&s[t][GROUP == 32 ? j >> 1 : 0]));
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            acc[t][m][0] = fmaf(d[m][0], f.x, acc[t][m][0]);
            acc[t][m][1] = fmaf(d[m][1], f.x, acc[t][m][1]);
            acc[t][m][2] = fmaf(d[m][2], f.y, acc[t][m][2]);
            acc[t][m][3] = fmaf(d[m][3], f.y, acc[t][m][3]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[warp][8 * m + 2 * c + (i & 1)][16 * t + r + (i & 2) * 4] = acc[t][m][i];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 8 * NT * 16; i += FEW_WARPS * 32) {
    const int m = i / (NT * 16), o = i - m * (NT * 16), row = m0 + m, n = tile0 * 16 + o;
    if (row >= a.M || n >= a.N) continue;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < FEW_WARPS; ++k) y += part[k][m][o];
    if (a.bias) y += gn_up(a.bias[n], BF);
    a.Y[row * a.ldy + n] = (uint16_t)pack16<BF>(y, 0.f);
  }
}
#endif

// ------------------------------------------------------------------ host
static dgq_status few_build(const __half* W, const int8_t* wq, const __half* scales, int N, int K, int group, dgq_few_weight** out,
                            cudaStream_t stream) {
  if (!out || N <= 0 || K <= 0 || (group != 32 && group != 64 && group != 128)) return DGQ_ERR_INVALID_ARG;
  if (K % 8 || N > FEW_MOST || K > FEW_MOST) return DGQ_ERR_UNSUPPORTED;
  dgq_few_weight* w = new (std::nothrow) dgq_few_weight();
  if (!w) return DGQ_ERR_CUDA;
  w->N = N;
  w->K = K;
  w->group = group;
  w->tiles = (N + 15) / 16;
  w->blocks = (K + 63) / 64;
  w->n_groups = (K + group - 1) / group;
  const int columns = few_columns(w->blocks, group);
  const size_t code_bytes = (size_t)w->tiles * w->blocks * 512, scale_bytes = ((size_t)w->tiles * columns * 32 + 255) / 256 * 256;
  dgq_status st = DGQ_OK;
  auto ok = [&](cudaError_t e) {
    if (st == DGQ_OK && e != cudaSuccess) st = DGQ_ERR_CUDA;
    return st == DGQ_OK;
  };
  int bad = 0;
  if (ok(cudaGetDevice(&w->device)) && ok(pool_alloc((void**)&w->d_slab, code_bytes + scale_bytes + 256, stream))) {
    w->d_codes = reinterpret_cast<uint4*>(w->d_slab);
    w->d_scale = reinterpret_cast<uint32_t*>(w->d_slab + code_bytes);
    int* d_bad = reinterpret_cast<int*>(w->d_slab + code_bytes + scale_bytes);
    FewPackArgs a = {W, wq, scales, N, K, group, w->n_groups, w->blocks, columns, reinterpret_cast<uint32_t*>(w->d_codes),
                     reinterpret_cast<__half*>(w->d_scale), d_bad};
    if (ok(cudaMemsetAsync(d_bad, 0, sizeof(int), stream))) {
      few_pack_kernel<<<dim3((w->blocks + 1) / 2, w->tiles), 256, 0, stream>>>(a);
      g_launches += 1;
      ok(cudaGetLastError());
      ok(cudaMemcpyAsync(&bad, d_bad, sizeof(int), cudaMemcpyDeviceToHost, stream));
      ok(cudaStreamSynchronize(stream));
    }
  }
  if (st == DGQ_OK && bad) st = DGQ_ERR_INVALID_ARG;
  if (st != DGQ_OK) {
    pool_free(w->d_slab);
    delete w;
    return st;
  }
  *out = w;
  return DGQ_OK;
}

template <bool BF, bool SILU, int GROUP, int NT>
static dgq_status few_launch(const FewArgs& a, cudaStream_t stream) {
  const int mt = std::min((a.M + 7) / 8, 4);
  const dim3 grid((a.tiles + NT - 1) / NT, (a.M + mt * 8 - 1) / (mt * 8));
  auto kernel = mt == 1 ? few_kernel<BF, SILU, GROUP, NT, 1> : mt == 2 ? few_kernel<BF, SILU, GROUP, NT, 2>
              : mt == 3 ? few_kernel<BF, SILU, GROUP, NT, 3> : few_kernel<BF, SILU, GROUP, NT, 4>;
  DGQ_CUDA_OK(launch_pdl(kernel, grid, dim3(FEW_WARPS * 32), 0, stream, a));
  g_launches += 1;
  return DGQ_OK;
}
template <bool BF, bool SILU>
static dgq_status few_pick(const FewArgs& a, int group, cudaStream_t stream) {
  return group == 32 ? few_launch<BF, SILU, 32, 1>(a, stream) : group == 64 ? few_launch<BF, SILU, 64, 1>(a, stream) : few_launch<BF, SILU, 128, 1>(a, stream);
}

}  // namespace dgq

extern "C" dgq_status dgq_few_weight_prepare(const void* W, int N, int K, int group, dgq_few_weight** out, void* stream) {
  if (!W) return DGQ_ERR_INVALID_ARG;
  return dgq::few_build((const __half*)W, nullptr, nullptr, N, K, group, out, (cudaStream_t)stream);
}

extern "C" dgq_status dgq_few_weight_from_codes(const int8_t* wq, const void* scales, int N, int K, int group, dgq_few_weight** out,
                                                void* stream) {
  if (!wq || !scales) return DGQ_ERR_INVALID_ARG;
  return dgq::few_build(nullptr, wq, (const __half*)scales, N, K, group, out, (cudaStream_t)stream);
}

extern "C" dgq_status dgq_few_weight_destroy(dgq_few_weight* w) {
  if (!w) return DGQ_OK;
  dgq::pool_free(w->d_slab);
  delete w;
  return DGQ_OK;
}

extern "C" dgq_status dgq_few_weight_export(const dgq_few_weight* w, int8_t* wq, uint16_t* scales) {
  using namespace dgq;
  if (!w) return DGQ_ERR_INVALID_ARG;
  DeviceScope on(w->device);
  DGQ_CUDA_OK(on.err);
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  DGQ_CUDA_OK(cudaThreadExchangeStreamCaptureMode(&mode));
  const int columns = few_columns(w->blocks, w->group);
  std::vector<uint32_t> codes(wq ? (size_t)w->tiles * w->blocks * 128 : 0);
  std::vector<uint16_t> sc(scales ? (size_t)w->tiles * columns * 16 : 0);
  cudaStream_t stream = nullptr;
  cudaError_t e = own_stream(&stream);
  if (e == cudaSuccess && wq) e = cudaMemcpyAsync(codes.data(), w->d_codes, codes.size() * 4, cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess && scales) e = cudaMemcpyAsync(sc.data(), w->d_scale, sc.size() * 2, cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  cudaThreadExchangeStreamCaptureMode(&mode);
  if (e != cudaSuccess) return DGQ_ERR_CUDA;
  for (int n = 0; n < w->N; ++n) {
    if (wq)
      for (int k = 0; k < w->K; ++k) {
        int word, shift;
        few_place(n & 15, k & 63, &word, &shift);
        wq[(size_t)n * w->K + k] = (int8_t)((int)((codes[((size_t)(n >> 4) * w->blocks + (k >> 6)) * 128 + word] >> shift) & 15) - 8);
      }
    if (scales)
      for (int g = 0; g < w->n_groups; ++g)
        scales[(size_t)n * w->n_groups + g] = sc[((size_t)(n >> 4) * columns + g) * 16 + (n & 7) * 2 + ((n >> 3) & 1)];
  }
  return DGQ_OK;
}

extern "C" dgq_status dgq_linear_few(const dgq_few_weight* w, const void* X, int64_t ldx, int dtype, int M, int act, const void* bias,
                                     void* Y, int64_t ldy, void* stream) {
  using namespace dgq;
  if (!w || !X || !Y || M <= 0 || (dtype != DGQ_F16 && dtype != DGQ_BF16) || (act != DGQ_ACT_NONE && act != DGQ_ACT_SILU) ||
      (M > 1 && (ldx < 0 || ldy < w->N)))
    return DGQ_ERR_INVALID_ARG;
  if (!aligned16(X) || (M > 1 && ldx % 8)) return DGQ_ERR_ALIGNMENT;
  if (M > FEW_MOST_ROWS) return DGQ_ERR_UNSUPPORTED;
  int dev = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  if (dev != w->device) return DGQ_ERR_INVALID_ARG;
  FewArgs a = {w->d_codes, w->d_scale, (const uint16_t*)X, M > 1 ? ldx : 0, (const uint16_t*)bias, (uint16_t*)Y, M > 1 ? ldy : 0,
               M, w->N, w->K, w->blocks, few_columns(w->blocks, w->group), w->tiles};
  const cudaStream_t s = (cudaStream_t)stream;
  if (dtype == DGQ_BF16) return act == DGQ_ACT_SILU ? few_pick<true, true>(a, w->group, s) : few_pick<true, false>(a, w->group, s);
  return act == DGQ_ACT_SILU ? few_pick<false, true>(a, w->group, s) : few_pick<false, false>(a, w->group, s);
}
