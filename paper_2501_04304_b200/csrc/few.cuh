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
  uint32_t* d_scale = nullptr;  // [tiles][scale columns][8]: fp16 scales of outputs r and r + 8 (groups of 32: [tiles][blocks][8][2])
  int device = 0;
};

namespace dgq {

constexpr int FEW_MOST = (1 << 20) - 16;      // outputs and input channels: at most 65535 tiles of 16
constexpr int FEW_MOST_ROWS = (1 << 21) - 32;  // 65535 times 32

// Scale columns of a tile: the groups of whole blocks (a group of 128 has two blocks).
__host__ __device__ inline int few_columns(int blocks, int group) { return group == 32 ? 2 * blocks : group == 64 ? blocks : (blocks + 1) / 2; }

// Place of a scale in a tile's columns, in pairs of fp16.
__host__ __device__ inline int few_scale_place(int column, int r, int group) {
  return group == 32 ? ((column >> 1) * 8 + r) * 2 + (column & 1) : column * 8 + r;
}
// A warp may read this many blocks behind the end of a tile (the rows are zeros there): the next tile's, or what lies behind the last one,
// of which the scales are zeros.
constexpr int FEW_BEYOND = 64;
// Warps of a block with the rows in shared memory: 72 registers a thread, 128 with 32 rows (at 72 300 bytes spill: 79 -> 123 us for 32 x 8192 x 28672).
__host__ __device__ constexpr int few_most_warps(int mt) { return mt == 4 ? 16 : 26; }

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
  int aligned;  // eight values lie at a multiple of their size
};
// Eight neighbouring values as the registers of one load, where they are aligned.
template <typename T, typename V>
__device__ __forceinline__ void few_load8(const T* p, bool aligned, V& v) {
  static_assert(sizeof(V) == 8 * sizeof(T), "eight values");
  if (aligned) {
    v = __ldg(reinterpret_cast<const V*>(p));
  } else {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = p[i];
    memcpy(&v, t, sizeof(V));
  }
}

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
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (in) few_load8(a.W + (size_t)n * a.K + k0, a.aligned, raw);
    const uint32_t h[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = gn_up((uint16_t)(i & 1 ? h[i >> 1] >> 16 : h[i >> 1]), false);
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
    uint2 raw;
    few_load8(a.wq + (size_t)n * a.K + k0, a.aligned, raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      q[i] = (int8_t)((i < 4 ? raw.x : raw.y) >> (8 * (i & 3)));
      bad |= q[i] < -8 || q[i] > 7;
    }
  }
  if (bad) *a.bad = 1;
  // four neighbouring channels of an output lie in one word, with those of the output eight further
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    uint32_t v = 0;
    int word = 0, shift;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      few_place(r, ((k0 + i) & 63) + j, &word, &shift);
      v |= (uint32_t)((q[i + j] + 8) & 15) << shift;
    }
    atomicOr(&words[(tid & 15) >> 3][word], v);
  }
  __syncthreads();
  const int block = blockIdx.x * 2 + (tid >> 7);
  if (block < a.blocks) a.codes[((size_t)blockIdx.y * a.blocks + block) * 128 + (tid & 127)] = words[tid >> 7][tid & 127];
  const int column = k0 / a.group;
  if ((tid & 15) % per == 0 && column < a.columns)
    a.scale_out[((size_t)blockIdx.y * a.columns * 8 + few_scale_place(column, r & 7, a.group)) * 2 + (r >> 3)] = in ? s : __ushort_as_half(0);
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
  int log_columns;  // 1 where two blocks share a scale column (groups of 128)
  int log_wk, wn;   // warps of a block: 2^log_wk along the input channels, wn along the outputs
};

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

// the same from zero
template <bool BF>
__device__ __forceinline__ void few_mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// The warps' parts of a block's outputs, joined in a fixed order in shared memory, [2^log_wk][rows][outputs], and stored.
template <bool BF, int MT>
__device__ __forceinline__ void few_join(const FewArgs& a, unsigned char* smem, const float* acc, int wk, int wn, int rows, int m0) {
  const int tid = threadIdx.x, n_threads = blockDim.x, r = (tid & 31) >> 2, c = tid & 3, width = a.wn * 16;
  float* part = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * m + 2 * c + (i & 1);
      if (row < rows) part[(wk * rows + row) * width + wn * 16 + r + (i & 2) * 4] = acc[m * 4 + i];
    }
  __syncthreads();
  const float per_width = 1.f / (float)width;
  for (int i = tid; i < rows * width; i += n_threads) {
    const int m = gn_div(i, per_width), o = i - m * width, n = blockIdx.x * width + o;
    if (n >= a.N) continue;
    float y = 0.f;
    for (int k = 0; k < 1 << a.log_wk; ++k) y += part[(k * rows + m) * width + o];
    if (a.bias) y += gn_up(a.bias[n], BF);
    a.Y[(m0 + m) * a.ldy + n] = (uint16_t)pack16<BF>(y, 0.f);
  }
}

// Up to eight rows as they are: a block has one tile, its warps split the input channels (four neighbouring blocks of 64 of a chunk for each),
// and every lane reads its part of its row straight from memory, which the multiprocessor's blocks do at about the same time, a block of 64 ahead;
// weights are asked for four blocks ahead.  No barriers, and shared memory for the join alone (7 x 5000 x 10007: 10.6 to 12.6 us; with the rows in
// shared memory, three chunks of 4 x 4 blocks, 17).  Registers would hold 32 warps a multiprocessor, few_plan asks for sixteen.
template <bool BF, bool G32>
__global__ void __launch_bounds__(512, 2) few_rows_kernel(const __grid_constant__ FewArgs a) {
  extern __shared__ __align__(16) unsigned char few_smem[];
  const int tid = threadIdx.x, wk = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3, tile = blockIdx.x;
  const int per_chunk = 4 << a.log_wk, chunks = (a.blocks + per_chunk - 1) >> (2 + a.log_wk);
  uint4 w[4];
  uint2 s[4];
  const uint4* codes = a.codes + ((size_t)tile * a.blocks + wk * 4) * 32 + lane;
  const uint32_t* scales = a.scale + (size_t)tile * a.columns * 8 + (G32 ? (wk * 4 * 8 + r) * 2 : (wk * 4 >> a.log_columns) * 8 + r);
  const int scale_step = G32 ? per_chunk * 16 : (per_chunk >> a.log_columns) * 8;
  auto weights = [&](int i) {
    w[i] = __ldg(codes + i * 32);
    if (G32) s[i] = __ldg(reinterpret_cast<const uint2*>(scales + i * 16));
    else s[i].x = __ldg(scales + (a.log_columns ? i >> 1 : i) * 8);
  };
  // (columns behind the last row are worked out and dropped)
  const uint16_t* row = a.X + min(r, a.M - 1) * a.ldx + wk * 256 + c * 8;
  int left = a.K - wk * 256 - c * 8;  // channels from this lane's first one to the end of the row
  uint4 x[2][2];
  auto rows = [&](int i) {
    const uint4 none = make_uint4(0, 0, 0, 0);
    x[i & 1][0] = i * 64 < left ? __ldg(reinterpret_cast<const uint4*>(row + i * 64)) : none;
    x[i & 1][1] = i * 64 + 32 < left ? __ldg(reinterpret_cast<const uint4*>(row + i * 64 + 32)) : none;
  };
  float acc[4] = {};
  // the weight is the caller's own object, complete since it was made: asked for before the kernel in front has ended
#pragma unroll
  for (int i = 0; i < 4; ++i) weights(i);
  pdl_wait();
  rows(0);
  for (int ch = 0; ch < chunks; ++ch) {
    codes += per_chunk * 32, scales += scale_step;  // those of the next chunk
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < 3) {
        rows(i + 1);
      } else if (ch + 1 < chunks) {
        row += per_chunk * 64, left -= per_chunk * 64;
        rows(0);
      } else {
        pdl_launch_dependents();
      }
      const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      const uint4 x0 = x[i & 1][0], x1 = x[i & 1][1];
      const uint32_t b[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
      float d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t op[4];
        few_widen<BF>(words[j], op);
        if (j == 0 || (G32 && j == 2)) few_mma_first<BF>(d, op, b[2 * j], b[2 * j + 1]);
        else few_mma<BF>(d, op, b[2 * j], b[2 * j + 1]);
        if (j == 3 || (G32 && j == 1)) {
          const uint32_t pair = G32 && j == 3 ? s[i].y : s[i].x;
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&pair));
          acc[0] = fmaf(d[0], f.x, acc[0]);
          acc[1] = fmaf(d[1], f.x, acc[1]);
          acc[2] = fmaf(d[2], f.y, acc[2]);
          acc[3] = fmaf(d[3], f.y, acc[3]);
        }
      }
      if (ch + 1 < chunks) weights(i);
    }
  }
  few_join<BF, 1>(a, few_smem, acc, wk, 0, a.M, 0);
}

// A block has wn tiles of outputs and MT times eight rows.  Its warps split the input channels (2^log_wk ways, every warp four neighbouring blocks
// of 64 of a chunk) and the tiles; the rows of a chunk stand in shared memory for all of them, three chunks in turn, so that one barrier a chunk is
// enough.  A warp's weights are asked for a chunk ahead, in registers.  A SiLU's results enter as a 16-bit number and what it leaves of
// the 32-bit one, rounded too: rounded once only, they would put half as much error again on the result's own.  (Half a step of half a step, 2^-16 or
// 2^-22 of the result; in fp16 at least 2^-25, the second number being subnormal where the result is below 1/8; and the 32-bit SiLU's own error.)
template <bool BF, bool G32, int MT, bool SILU>
__global__ void __launch_bounds__(few_most_warps(MT) * 32) few_kernel(const __grid_constant__ FewArgs a) {
  extern __shared__ __align__(16) unsigned char few_smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;
  const int wk = warp & ((1 << a.log_wk) - 1), wn = warp >> a.log_wk;
  const int tile = min((int)blockIdx.x * a.wn + wn, a.tiles - 1), m0 = blockIdx.y * MT * 8, rows = min(MT * 8, a.M - m0);
  const int per_chunk = 4 << a.log_wk, chunks = (a.blocks + per_chunk - 1) >> (2 + a.log_wk);
  const int pitch = per_chunk * 128 + 64, part = rows * pitch, set = SILU ? 2 * part : part;  // bytes; rows start in different halves of the banks
  uint4 w[4];
  uint2 s[4];
  const uint4* codes = a.codes + ((size_t)tile * a.blocks + wk * 4) * 32 + lane;
  const uint32_t* scales = a.scale + (size_t)tile * a.columns * 8 + (G32 ? (wk * 4 * 8 + r) * 2 : (wk * 4 >> a.log_columns) * 8 + r);
  const int scale_step = G32 ? per_chunk * 16 : (per_chunk >> a.log_columns) * 8;
  auto weights = [&](int i) {
    w[i] = __ldg(codes + i * 32);
    if (G32) s[i] = __ldg(reinterpret_cast<const uint2*>(scales + i * 16));
    else s[i].x = __ldg(scales + (a.log_columns ? i >> 1 : i) * 8);
  };
  // Rows of chunk `ch` into shared memory, eight channels (which are in or out as a whole) of every wn-th row for a thread.
  const int piece = tid & ((32 << a.log_wk) - 1);
  auto stage = [&](int ch, int buffer) {
    const int k = (ch * per_chunk * 8 + piece) * 8;
    const bool in = k < a.K;
    const uint16_t* src = a.X + (m0 + wn) * a.ldx + (in ? k : 0);
    uint32_t to = smem_u32(few_smem) + buffer * set + wn * pitch + piece * 16;
    for (int row = wn; row < rows; row += a.wn, src += a.wn * a.ldx, to += a.wn * pitch) {
      if (!SILU) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(in ? 16 : 0) : "memory");
      } else {
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (in) {
          x = __ldg(reinterpret_cast<const uint4*>(src));
          uint32_t* h = reinterpret_cast<uint32_t*>(&x);
          uint32_t* l = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const float2 f = unpack16<BF>(h[z]);
            const float v0 = gn_silu(f.x), v1 = gn_silu(f.y);
            h[z] = pack16<BF>(v0, v1);
            const float2 g = unpack16<BF>(h[z]);
            // (an infinity leaves nothing: inf - inf would be NaN)
            l[z] = pack16<BF>(g.x < INFINITY ? v0 - g.x : 0.f, g.y < INFINITY ? v1 - g.y : 0.f);
          }
        }
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + part), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
      }
    }
  };
  // where this lane's part of the rows lies (columns behind the last row are worked out and dropped)
  int mine[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) mine[m] = min(8 * m + r, rows - 1) * pitch + c * 16 + wk * 512;
  float acc[MT][4] = {};
  // the weight is the caller's own object, complete since it was made: asked for before the kernel in front has ended
#pragma unroll
  for (int i = 0; i < 4; ++i) weights(i);
  pdl_wait();
  stage(0, 0);
  asm volatile("cp.async.commit_group;" ::: "memory");
  if (chunks > 1) stage(1, 1);
  asm volatile("cp.async.commit_group;" ::: "memory");
  int buffer = 0;
  for (int ch = 0; ch < chunks; ++ch) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();  // chunk ch is there, and everybody is done with the one before, whose place the one after the next takes
    const int free = buffer == 0 ? 2 : buffer - 1;
    if (ch + 2 < chunks) stage(ch + 2, free);
    else pdl_launch_dependents();
    asm volatile("cp.async.commit_group;" ::: "memory");
    const unsigned char* from = few_smem + buffer * set;
    buffer = buffer == 2 ? 0 : buffer + 1;
    codes += per_chunk * 32, scales += scale_step;  // those of the next chunk
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // 32 rows: a lane's part of all of them at once, of which the compiler makes the better order; fewer: one half after the other, for the registers
      constexpr int HALVES = MT == 4 && !SILU ? 1 : 2;
      const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      float d[MT][4];
#pragma unroll
      for (int half = 0; half < HALVES; ++half) {
        uint32_t x[MT][8 / HALVES];
        uint4 y[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint4* p = reinterpret_cast<const uint4*>(from + mine[m] + i * 128 + half * 64);
          const uint4 x0 = p[0];
          x[m][0] = x0.x, x[m][1] = x0.y, x[m][2] = x0.z, x[m][3] = x0.w;
          if constexpr (SILU) y[m] = *reinterpret_cast<const uint4*>(from + mine[m] + i * 128 + half * 64 + part);
          if constexpr (HALVES == 1) {
            const uint4 x1 = p[4];
            x[m][4] = x1.x, x[m][5] = x1.y, x[m][6] = x1.z, x[m][7] = x1.w;
          }
        }
#pragma unroll
        for (int k = 0; k < 4 / HALVES; ++k) {
          const int j = half * 2 + k;
          uint32_t op[4];
          few_widen<BF>(words[j], op);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (j == 0 || (G32 && j == 2)) few_mma_first<BF>(d[m], op, x[m][2 * k], x[m][2 * k + 1]);
            else few_mma<BF>(d[m], op, x[m][2 * k], x[m][2 * k + 1]);
            if constexpr (SILU) few_mma<BF>(d[m], op, k ? y[m].z : y[m].x, k ? y[m].w : y[m].y);
          }
          if (j == 3 || (G32 && j == 1)) {
            const uint32_t pair = G32 && j == 3 ? s[i].y : s[i].x;
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&pair));
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              acc[m][0] = fmaf(d[m][0], f.x, acc[m][0]);
              acc[m][1] = fmaf(d[m][1], f.x, acc[m][1]);
              acc[m][2] = fmaf(d[m][2], f.y, acc[m][2]);
              acc[m][3] = fmaf(d[m][3], f.y, acc[m][3]);
            }
          }
        }
      }
      if (ch + 1 < chunks) weights(i);
    }
  }
  __syncthreads();  // the rows' places are free
  few_join<BF, MT>(a, few_smem, &acc[0][0], wk, wn, rows, m0);
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
  const size_t beyond = FEW_BEYOND * 512;  // of codes; of scales at most an eighth of it
  dgq_status st = DGQ_OK;
  auto ok = [&](cudaError_t e) {
    if (st == DGQ_OK && e != cudaSuccess) st = DGQ_ERR_CUDA;
    return st == DGQ_OK;
  };
  int bad = 0;
  if (ok(cudaGetDevice(&w->device)) && ok(pool_alloc((void**)&w->d_slab, code_bytes + scale_bytes + beyond + 256, stream))) {
    w->d_codes = reinterpret_cast<uint4*>(w->d_slab);
    w->d_scale = reinterpret_cast<uint32_t*>(w->d_slab + code_bytes);
    int* d_bad = reinterpret_cast<int*>(w->d_slab + code_bytes + scale_bytes + beyond);
    FewPackArgs a = {W, wq, scales, N, K, group, w->n_groups, w->blocks, columns, reinterpret_cast<uint32_t*>(w->d_codes),
                     reinterpret_cast<__half*>(w->d_scale), d_bad,
                     W ? aligned16(W) : (reinterpret_cast<uintptr_t>(wq) & 7u) == 0};
    const size_t scale_end = code_bytes + (size_t)w->tiles * columns * 32;
    if (ok(cudaMemsetAsync(w->d_slab + scale_end, 0, code_bytes + scale_bytes + beyond + sizeof(int) - scale_end, stream))) {
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

constexpr size_t FEW_SMEM_MAX = 208 * 1024;
// How a product is dealt out: warps along the input channels (a power of two) and along the outputs, eights of rows.
struct FewPlan {
  int log_wk, wn, mt;
  size_t smem;
};
static FewPlan few_plan(int M, int tiles, int blocks, bool silu) {
  FewPlan p;
  p.mt = M <= 8 ? 1 : M <= 16 ? 2 : 4;
  const int rows = std::min(M, p.mt * 8);
  const int64_t units = (int64_t)tiles * ((M + p.mt * 8 - 1) / (p.mt * 8));
  // sixteen warps for each multiprocessor (eight with 32 rows), four
  // blocks of 64 channels for a warp at least
  p.log_wk = 0;
  const int most = p.mt == 4 ? 2 : p.mt == 2 ? 3 : 4, warps = p.mt == 4 ? 8 : 16;
  while (p.log_wk < most && units << p.log_wk < warps * 148 && (4 << p.log_wk) < blocks) ++p.log_wk;
  // (a SiLU's results take twice the place: the channels are split less where they do not fit)
  auto staged = [&]() {
    const int per_chunk = 4 << p.log_wk, sets = std::min((blocks + per_chunk - 1) / per_chunk, 3);
    return (size_t)sets * rows * (per_chunk * 128 + 64) * (silu ? 2 : 1);
  };
  while (p.log_wk > 0 && staged() > FEW_SMEM_MAX) --p.log_wk;
  // Along the outputs, with more than eight rows, which would be read over and over: the most that fill the multiprocessors as evenly as any other
  // number does.
  p.wn = 1;
  double best = 0.;
  for (int wn = 1; p.mt > 1 && wn << p.log_wk <= few_most_warps(p.mt); ++wn) {
    const int64_t n = (units + wn - 1) / wn, rounds = (n + 147) / 148;
    const double full = (double)units / (double)(rounds * 148 * wn);
    if (full > 0.97 * best) best = std::max(best, full), p.wn = wn;
  }
  p.smem = std::max(staged(), (size_t)(1 << p.log_wk) * rows * p.wn * 16 * sizeof(float));
  return p;
}

template <bool BF, bool G32, int MT, bool SILU>
static dgq_status few_launch(const FewArgs& a, const FewPlan& p, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  int dev = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  if (dev >= 64 || !done[dev].load()) {
    DGQ_CUDA_OK(cudaFuncSetAttribute(few_kernel<BF, G32, MT, SILU>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FEW_SMEM_MAX));
    if (dev < 64) done[dev].store(true);
  }
  const dim3 grid((a.tiles + p.wn - 1) / p.wn, (a.M + MT * 8 - 1) / (MT * 8));
  DGQ_CUDA_OK(launch_pdl(few_kernel<BF, G32, MT, SILU>, grid, dim3((p.wn << p.log_wk) * 32), p.smem, stream, a));
  g_launches += 1;
  return DGQ_OK;
}
template <bool BF, bool G32, bool SILU>
static dgq_status few_rows(const FewArgs& a, const FewPlan& p, cudaStream_t stream) {
  return p.mt == 1 ? few_launch<BF, G32, 1, SILU>(a, p, stream) : p.mt == 2 ? few_launch<BF, G32, 2, SILU>(a, p, stream) : few_launch<BF, G32, 4, SILU>(a, p, stream);
}
template <bool BF, bool G32>
static dgq_status few_pick(const FewArgs& a, const FewPlan& p, bool silu, cudaStream_t stream) {
  if (silu) return few_rows<BF, G32, true>(a, p, stream);
  if (p.mt > 1) return p.mt == 2 ? few_launch<BF, G32, 2, false>(a, p, stream) : few_launch<BF, G32, 4, false>(a, p, stream);
  DGQ_CUDA_OK(launch_pdl(few_rows_kernel<BF, G32>, dim3(a.tiles), dim3(32 << p.log_wk), (size_t)(1 << p.log_wk) * a.M * 16 * sizeof(float), stream, a));
  g_launches += 1;
  return DGQ_OK;
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
        scales[(size_t)n * w->n_groups + g] = sc[((size_t)(n >> 4) * columns * 8 + few_scale_place(g, n & 7, w->group)) * 2 + ((n >> 3) & 1)];
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
  const bool silu = act == DGQ_ACT_SILU;
  const FewPlan p = few_plan(M, w->tiles, w->blocks, silu);
  const FewArgs a = {w->d_codes, w->d_scale, (const uint16_t*)X, M > 1 ? ldx : 0, (const uint16_t*)bias, (uint16_t*)Y, M > 1 ? ldy : 0, M, w->N, w->K,
                     w->blocks, few_columns(w->blocks, w->group), w->tiles, w->group == 128, p.log_wk, p.wn};
  const cudaStream_t s = (cudaStream_t)stream;
  if (dtype == DGQ_BF16) return w->group == 32 ? few_pick<true, true>(a, p, silu, s) : few_pick<true, false>(a, p, silu, s);
  return w->group == 32 ? few_pick<false, true>(a, p, silu, s) : few_pick<false, false>(a, p, silu, s);
}
