// Attention with full-precision scores over an encoder's states and over a paged 8-bit cache:
//
//     O_i = sum_j w_ij V_j / sum_j w_ij,   w_ij = 2^(t_ij - m_i),   t_ij = log2(e) scale Q_i . K_j
//
// over the keys that row i sees; a row that sees none gives zeros.  Any m_i gives the same quotient; the kernels keep one that the
// largest t_ij so far exceeds by 8 at most.
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
  int n_pages, page, page_log2, max_pages;
  const int32_t* table;         // dev [B, max_pages]
  const int32_t* q_start;       // dev [B + 1] or null (nq queries each)
  int64_t n_rows;
  int causal;
  int bf;                       // Q and O are bf16
  int by_length;                // blocks take the requests longest first (at most EA_SORTED of them)
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

// The request of a given rank by length, for all threads of a block: where blocks run in several rounds, the last ones to start
// should be short.  A thread counts one request's rank, so this goes up to as many requests as the smallest block has threads; more
// are taken in their order.
constexpr int EA_SORTED = 128;
__device__ __forceinline__ int enc_request_of_rank(const EncAttnArgs& a, int rank) {
  __shared__ int lens[EA_SORTED], found;
  const int j = threadIdx.x;
  if (j < a.B) lens[j] = a.kv_lens[j];
  __syncthreads();
  if (j < a.B) {
    int r = 0;
    for (int k = 0; k < a.B; ++k) r += lens[k] > lens[j] || (lens[k] == lens[j] && k < j);
    if (r == rank) found = j;
  }
  __syncthreads();
  return found;
}

// ------------------------------------------------------------------ many query rows: tcgen05
constexpr int EA_Q = 128;                 // query rows of a tile
constexpr int EA_K = 128;                 // keys of a block
constexpr int EA_PANEL = 128 * 128;       // bytes of 64 features of 128 rows
constexpr int EA_MOST = 1 << 30;          // queries or keys of a request (sums of an index and a block stay below 2^31)
constexpr float EA_LAZY = 8.0f;           // a row's reference follows its maximum once that is 2^8 above it

// NT: query tiles of a block.  Over 16-bit keys one, and two blocks to an SM, whose starts, products and softmaxes then drift apart
// and run under each other (2 x 10 x 4096 x 64 over 4173 keys: 153 us, with two tiles in one block 191; 128 features 214 and 277).
// Over a cache two, which share the work of widening every code (2 x 16 of 4 x 2048 x 128 over 6000 codes: 283 us, with one 489); their
// 608 threads have 96 registers each and spill 76 bytes for heads to 128 and 8 to 64, the 448 for heads to 160 (128 registers) 52.
template <int NP, bool CACHED>
struct EaCfg {
  static constexpr int NT = CACHED && NP <= 2 ? 2 : 1;
  static constexpr int BLOCKS = CACHED || NP == 3 ? 1 : 2;   // per SM
  static constexpr bool OWN_P = NP != 2;              // weights have tensor memory of their own (else they lie over the scores)
  static constexpr int KST = BLOCKS == 2 && NP == 2 ? 1 : 2, VST = NP == 3 ? 1 : KST;
  static constexpr int SOFTMAX_WARPS = 4 * NT;
  static constexpr int WARP_TMA = SOFTMAX_WARPS, WARP_MMA = SOFTMAX_WARPS + 1;  // one issuing warp per tile
  static constexpr int CONV_WARP0 = SOFTMAX_WARPS + 1 + NT;  // CACHED: the first CONV warps bring in keys, the others values
  static constexpr int CONV = 4;
  static constexpr int WARPS = CONV_WARP0 + (CACHED ? 2 * CONV : 0);
  static constexpr int THREADS = WARPS * 32;
  static constexpr int TMEM = BLOCKS == 2 ? 256 : 512;
  static constexpr int TMEM_P = OWN_P ? NT * 128 : 0, P_STRIDE = OWN_P ? 64 : 128;
  static constexpr int TMEM_O = OWN_P ? NT * 192 : NT * 128, O_STRIDE = NP * 64;
  static constexpr int TILE = NP * EA_PANEL;
  static constexpr int OFF_K = NT * TILE, OFF_V = OFF_K + KST * TILE, OFF_SH = OFF_V + VST * TILE;
  static constexpr int SMEM = 1024 + OFF_SH + 1024;
  static_assert(SMEM * BLOCKS <= 232448 - 1024 * (BLOCKS - 1), "shared memory budget");
  static_assert(TMEM_O + NT * O_STRIDE <= TMEM, "tensor memory budget");
};

// Of sixteen keys of a cache: t = S * k, weight 2^(t + lv) with lv = log2 of the page's value scale, its inverse.
struct EaPage {
  float k, lv, iv, pad;
};

struct EaShared {
  uint64_t q_full;
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], v_clean;
  uint64_t s_full[2], p_full[2], o_done[2];
  uint32_t tmem_base;
  int abort_flag;
  EaPage page[4][8];  // four key blocks of eight groups
};
static_assert(sizeof(EaShared) <= 1024, "shared block");

struct EaMaps {
  CUtensorMap q, k, v, o;
  int q_b, k_b, k_h, v_b, v_h;  // 0 where the tensor broadcasts along the dimension (its extent is then 1)
  int q_h, o_b, o_h;
};

// kind::f16 instruction descriptor with both operands' type and the sign of A.
__device__ __forceinline__ uint32_t ea_idesc(int n, bool b_mn_major, bool bf, bool negate_a) {
  return (1u << 4) | ((bf ? 1u : 0u) << 7) | ((bf ? 1u : 0u) << 10) | ((negate_a ? 1u : 0u) << 13) |
         ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(EA_Q >> 4) << 24);
}
// Nothing that uses r moves in front of this (of a wait for its load before it).
__device__ __forceinline__ void pin32(uint32_t (&r)[32]) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                    "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                    "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                    "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

// Boxes of 64 features x 32 rows x 1 head out of shared memory (rows of 128 bytes, swizzled); rows and features beyond the tensor's
// are left out.
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* m, const void* src, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
               : "memory");
}
// Features c .. c + 7 of an output row into its place in such a box.
__device__ __forceinline__ void stage_out(unsigned char* slab, int panel_bytes, int row, int c, uint4 y) {
  *reinterpret_cast<uint4*>(slab + (c >> 6) * panel_bytes + row * 128 + ((((c >> 3) & 7) ^ (row & 7)) << 4)) = y;
}

// Four codes as four 16-bit numbers, exactly.  fp16: 0x64 in front of a byte is 1024 + byte.  bf16: 0x43 in front of the low seven
// bits is 128 + those, in front of the sign bit alone 128 or 256.
template <bool BF>
__device__ __forceinline__ void codes_to_16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (BF) {
    const uint32_t y0 = __byte_perm(w, 0x43434343u, 0x4140), y1 = __byte_perm(w, 0x43434343u, 0x4342);
    const uint32_t a0 = y0 & 0xFF7FFF7Fu, b0 = y0 & 0xFF80FF80u, a1 = y1 & 0xFF7FFF7Fu, b1 = y1 & 0xFF80FF80u;
    const __nv_bfloat162 r0 = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a0), *reinterpret_cast<const __nv_bfloat162*>(&b0));
    const __nv_bfloat162 r1 = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a1), *reinterpret_cast<const __nv_bfloat162*>(&b1));
    lo = *reinterpret_cast<const uint32_t*>(&r0);
    hi = *reinterpret_cast<const uint32_t*>(&r1);
  } else {
    const uint32_t x = w ^ 0x80808080u, bias = 0x64806480u;
    const uint32_t y0 = __byte_perm(x, 0x64646464u, 0x4140), y1 = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 r0 = __hsub2(*reinterpret_cast<const __half2*>(&y0), *reinterpret_cast<const __half2*>(&bias));
    const __half2 r1 = __hsub2(*reinterpret_cast<const __half2*>(&y1), *reinterpret_cast<const __half2*>(&bias));
    lo = *reinterpret_cast<const uint32_t*>(&r0);
    hi = *reinterpret_cast<const uint32_t*>(&r1);
  }
}

// Both good to 2^-22 for normal numbers.
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The page of a request's token, or -1 (recorded) where the table says nothing usable.
__device__ __forceinline__ int ea_page_of(const EncAttnArgs& a, int b, int token) {
  const int p = __ldg(a.table + (int64_t)b * a.max_pages + (token >> a.page_log2));
  if (p >= 0 && p < a.n_pages) return p;
  record_error(DGQ_ERR_INVALID_ARG);
  return -1;
}

// The constants of sixteen keys that begin at `token`.  A page of zeros has no scale of its own: 2^-40 keeps its weights
// (which count in the row sum) within range whatever the other pages' scales are; others are held above 2^-100.
__device__ __forceinline__ EaPage ea_page_scales(const EncAttnArgs& a, int b, int g, int token, float scale_log2) {
  EaPage c{1.17549435e-38f, -INFINITY, 0.f, 0.f};
  const int p = ea_page_of(a, b, token);
  if (p < 0) return c;
  const int64_t ph = (int64_t)p * a.Hkv + g;
  const float vs = __ldg(a.v_scale + ph);
  const float v = vs == 0.f ? 9.094947e-13f : fmaxf(vs, 7.8886091e-31f);
  c.k = fmaxf(__ldg(a.k_scale + ph) * scale_log2, 1.17549435e-38f);
  c.lv = lg2_approx(v);
  c.iv = rcp_approx(v);
  return c;
}

template <int NP, bool BF, bool CACHED>
__global__ void __launch_bounds__(EaCfg<NP, CACHED>::THREADS, EaCfg<NP, CACHED>::BLOCKS)
enc_attn_tiles_kernel(const __grid_constant__ EaMaps maps, const __grid_constant__ EncAttnArgs a) {
  using Cfg = EaCfg<NP, CACHED>;
  constexpr int NT = Cfg::NT, KST = Cfg::KST, VST = Cfg::VST;
  constexpr bool P_BF = BF && !CACHED;  // codes are whole numbers of 8 bits: fp16 holds them and three more bits of the weight
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  unsigned char* sQ = smem;
  unsigned char* sK = smem + Cfg::OFF_K;
  unsigned char* sV = smem + Cfg::OFF_V;
  EaShared* sh = reinterpret_cast<EaShared*>(smem + Cfg::OFF_SH);
  volatile int* abort_flag = &sh->abort_flag;

  const int n_tiles = (a.nq + EA_Q * NT - 1) / (EA_Q * NT);
  // the tiles that see most come first where that differs
  const int tile = a.causal ? n_tiles - 1 - (int)(blockIdx.x % n_tiles) : (int)(blockIdx.x % n_tiles);
  const int h = (int)(blockIdx.x / n_tiles) % a.Hq;
  int b = (int)(blockIdx.x / n_tiles) / a.Hq;
  const int g = h / (a.Hq / a.Hkv);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(&sh->q_full, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh->k_full[i], CACHED ? Cfg::CONV : 1);
      mbar_init(&sh->v_full[i], CACHED ? Cfg::CONV : 1);
      mbar_init(&sh->k_empty[i], NT);
      mbar_init(&sh->v_empty[i], NT);
      mbar_init(&sh->s_full[i], 1);
      mbar_init(&sh->p_full[i], 4);
      mbar_init(&sh->o_done[i], 1);
    }
    mbar_init(&sh->v_clean, 1);
    sh->abort_flag = 0;
    fence_barrier_init();
  }
  // Tensor memory is taken once the kernel before has ended: a block that held it while it waits could keep a block of that one from
  // its own.
  pdl_wait();
  if (warp == Cfg::WARP_MMA) {
    tmem_alloc(&sh->tmem_base, Cfg::TMEM);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();  // not before this block has its tensor memory: a block of the next kernel could take it and wait for this one
  const uint32_t tmem_base = sh->tmem_base;

  if (a.by_length) b = enc_request_of_rank(a, b);
  const EncRequest rq = enc_request(a, b);
  const int row0 = tile * (EA_Q * NT);
  // keys and key blocks that each tile walks: as many as its last row sees
  int most[2] = {0, 0}, nbt[2] = {0, 0};
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int first = row0 + t * EA_Q;
    if (first < rq.nq) most[t] = enc_sees(a, rq, min(first + EA_Q, rq.nq) - 1);
    nbt[t] = (most[t] + EA_K - 1) / EA_K;
  }
  const int nb = max(nbt[0], nbt[1]);
  // columns of block j that a tile computes, in sixteens
  const auto columns = [](int keys, int j) { return (min(EA_K, keys - j * EA_K) + 15) & ~15; };
  // value rows behind the length meet weights of 0, which an infinity or NaN there would not survive
  const bool clean = !CACHED && rq.len < a.nk && rq.len % EA_K != 0;
  const float scale_log2 = fabsf(a.scale_log2);  // the sign is the MMA's
  const int ksteps = (a.d + 15) / 16, dp = ksteps * 16;

  if (warp == Cfg::WARP_TMA) {
    // ------------------------------------------------------------ loads
    const int panels = (a.d + 63) / 64;  // panels of NP that hold features
    if (lane == 0) {
      tma_prefetch_desc(&maps.q);
      if (!CACHED) {
        tma_prefetch_desc(&maps.k);
        tma_prefetch_desc(&maps.v);
      }
    }
    if (lane == 0 && nb > 0) {
      mbar_arrive_expect_tx(&sh->q_full, (uint32_t)(NT * panels * EA_PANEL));
      for (int t = 0; t < NT; ++t)
        for (int p = 0; p < panels; ++p)
          tma_load_4d(sQ + t * Cfg::TILE + p * EA_PANEL, &maps.q, &sh->q_full, p * 64, h * maps.q_h, (int)rq.q_row + row0 + t * EA_Q, b * maps.q_b);
      for (int j = 0; !CACHED && j < nb; ++j) {
        const uint32_t ks = (uint32_t)j % KST, vs = (uint32_t)j % VST;
        mbar_wait_handover(smem_u32(&sh->k_empty[ks]), (((uint32_t)j / KST) & 1u) ^ 1u, abort_flag);
        mbar_arrive_expect_tx(&sh->k_full[ks], (uint32_t)(panels * EA_PANEL));
        for (int p = 0; p < panels; ++p)
          tma_load_4d(sK + ks * Cfg::TILE + p * EA_PANEL, &maps.k, &sh->k_full[ks], p * 64, g * maps.k_h, j * EA_K, b * maps.k_b);
        mbar_wait_handover(smem_u32(&sh->v_empty[vs]), (((uint32_t)j / VST) & 1u) ^ 1u, abort_flag);
        mbar_arrive_expect_tx(&sh->v_full[vs], (uint32_t)(panels * EA_PANEL));
        for (int p = 0; p < panels; ++p)
          tma_load_4d(sV + vs * Cfg::TILE + p * EA_PANEL, &maps.v, &sh->v_full[vs], p * 64, g * maps.v_h, j * EA_K, b * maps.v_b);
        if (*abort_flag) break;
      }
    }
    __syncwarp();
    if (clean && nb > 0) {
      const uint32_t vs = (uint32_t)(nb - 1) % VST;
      const int real = rq.len - (nb - 1) * EA_K;
      mbar_wait_handover(smem_u32(&sh->v_full[vs]), ((uint32_t)(nb - 1) / VST) & 1u, abort_flag);
      for (int k = lane; k < (EA_K - real) * NP * 8; k += 32) {
        const int r = real + k / (NP * 8), c = k % (NP * 8);
        *reinterpret_cast<uint4*>(sV + vs * Cfg::TILE + (c >> 3) * EA_PANEL + r * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->v_clean);
    }
    __syncwarp();
  } else if (warp == Cfg::WARP_MMA || (NT == 2 && warp == Cfg::WARP_MMA + 1)) {
    // ------------------------------------------------------------ products
    // One warp per tile issues its scores of block j + 1 and its O += P V of block j, so that neither tile's hand-overs wait
    // behind the other's; a tile's softmax runs under the other tile's products.  The weights' hand-over also says that the
    // scores have been read.
    const int t = NT == 2 ? warp - Cfg::WARP_MMA : 0;
    const uint32_t idesc_pv = ea_idesc(dp, true, P_BF, false);
    constexpr uint32_t HI = smem_desc_hi(1024, 2);
    const uint32_t q_lo = smem_desc_lo(smem_u32(sQ)) + (uint32_t)(t * Cfg::TILE >> 4), k_lo = smem_desc_lo(smem_u32(sK));
    const uint32_t v_lo = ((smem_u32(sV) & 0x3FFFFu) >> 4) | ((uint32_t)(EA_PANEL >> 4) << 16);
    const uint32_t s_full = smem_u32(&sh->s_full[t]), p_full = smem_u32(&sh->p_full[t]), o_done = smem_u32(&sh->o_done[t]);
    const int keys = t == 0 ? most[0] : most[1], blocks = t == 0 ? nbt[0] : nbt[1];
    auto scores = [&](int j) {
      const uint32_t ks = (uint32_t)j % KST, b_lo = k_lo + ks * (uint32_t)(Cfg::TILE >> 4);
      const uint32_t idesc_qk = ea_idesc(columns(keys, j), false, BF, a.scale_log2 < 0.f);
      mbar_wait_handover(smem_u32(&sh->k_full[ks]), ((uint32_t)j / KST) & 1u, abort_flag);
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < NP * 4; ++k) {
          if (k >= ksteps) break;
          const uint32_t off = (uint32_t)(((k >> 2) * EA_PANEL + (k & 3) * 32) >> 4);
          mma_f16_lohi(tmem_base + t * 128, q_lo + off, HI, b_lo + off, HI, idesc_qk, k > 0 ? 1u : 0u);
        }
        mma_commit_addr(s_full);
        mma_commit_addr(smem_u32(&sh->k_empty[ks]));
      }
      __syncwarp();
    };
    if (blocks > 0) {
      mbar_wait_handover(smem_u32(&sh->q_full), 0, abort_flag);
      scores(0);
    }
    for (int j = 0; j < blocks; ++j) {
      const uint32_t vs = (uint32_t)j % VST;
      mbar_wait_handover(p_full, (uint32_t)j & 1u, abort_flag);
      tc_fence_after();
      if (Cfg::OWN_P && j + 1 < blocks) scores(j + 1);
      mbar_wait_handover(smem_u32(&sh->v_full[vs]), ((uint32_t)j / VST) & 1u, abort_flag);
      if (clean && j == nb - 1) mbar_wait_handover(smem_u32(&sh->v_clean), 0, abort_flag);
      tc_fence_after();
      const uint32_t a_tmem = tmem_base + Cfg::TMEM_P + t * Cfg::P_STRIDE, d_tmem = tmem_base + Cfg::TMEM_O + t * Cfg::O_STRIDE;
      const uint32_t b_lo = v_lo + vs * (uint32_t)(Cfg::TILE >> 4);
      const int n = columns(keys, j) / 16;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < EA_K / 16; ++k) {
          if (k >= n) break;
          mma_f16_ts(d_tmem, a_tmem + k * 8, b_lo + (uint32_t)(k * 2048 >> 4), HI, idesc_pv, (j > 0 || k > 0) ? 1u : 0u);
        }
        mma_commit_addr(o_done);
        mma_commit_addr(smem_u32(&sh->v_empty[vs]));
      }
      __syncwarp();
      if (!Cfg::OWN_P && j + 1 < blocks) scores(j + 1);
      if ((j & 7) == 7 && *abort_flag) break;
    }
    // blocks that only the other tile walks
    for (int j = blocks; NT == 2 && j < nb && !*abort_flag; ++j) {
      const uint32_t ks = (uint32_t)j % KST, vs = (uint32_t)j % VST;
      mbar_wait_handover(smem_u32(&sh->k_full[ks]), ((uint32_t)j / KST) & 1u, abort_flag);
      if (lane == 0) mbar_arrive(&sh->k_empty[ks]);
      mbar_wait_handover(smem_u32(&sh->v_full[vs]), ((uint32_t)j / VST) & 1u, abort_flag);
      if (lane == 0) mbar_arrive(&sh->v_empty[vs]);
    }
    __syncwarp();
  } else if (CACHED && warp >= Cfg::CONV_WARP0) {
    // ------------------------------------------------------------ codes to 16 bits
    // Half of these warps bring in keys, half values: sixteen codes a load, the next block's first loads in registers while
    // this one's stage is still in use.
    const bool values = warp >= Cfg::CONV_WARP0 + Cfg::CONV;
    constexpr int N = Cfg::CONV * 32;
    const int tid = (warp - Cfg::CONV_WARP0) % Cfg::CONV * 32 + lane;
    const int row_bytes = kv_row_bytes(a.d), units = row_bytes / 16;
    constexpr int BATCH = NP * 512 / N < 8 ? NP * 512 / N : 8, BATCHES = (NP * 512 / N + BATCH - 1) / BATCH;
    const int8_t* codes = values ? a.v_codes : a.k_codes;
    const int st_n = values ? VST : KST;
    uint4 x[BATCH];
    auto load = [&](int j, int batch) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int u = tid + (batch * BATCH + i) * N;
        const int r = u / units, c = u - r * units, token = j * EA_K + r;
        x[i] = make_uint4(0, 0, 0, 0);
        if (r >= EA_K || token >= rq.len) continue;
        const int p = ea_page_of(a, b, token);
        if (p >= 0)
          x[i] = __ldg(reinterpret_cast<const uint4*>(codes + ((((int64_t)p * a.Hkv + g) << a.page_log2) + (token & (a.page - 1))) * row_bytes) + c);
      }
    };
    if (nb > 0) load(0, 0);
    for (int j = 0; j < nb; ++j) {
      const int st = j % st_n;
      unsigned char* stage = (values ? sV : sK) + st * Cfg::TILE;
      uint64_t* empty = values ? &sh->v_empty[st] : &sh->k_empty[st];
      uint64_t* full = values ? &sh->v_full[st] : &sh->k_full[st];
      EaPage pg;
      if (!values && tid < 8) {
        const int token = j * EA_K + tid * 16;
        pg = EaPage{1.17549435e-38f, -INFINITY, 0.f, 0.f};
        if (token < rq.len) pg = ea_page_scales(a, b, g, token, scale_log2);
      }
      mbar_wait_handover(smem_u32(empty), (((uint32_t)j / st_n) & 1u) ^ 1u, abort_flag);
      if (!values && tid < 8) sh->page[j & 3][tid] = pg;
#pragma unroll
      for (int batch = 0; batch < BATCHES; ++batch) {
        if (batch > 0) load(j, batch);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int u = tid + (batch * BATCH + i) * N;
          const int r = u / units, c = u - r * units;
          if (r >= EA_K) continue;
          uint32_t y[8];
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (BF && !values) codes_to_16<true>(w[k], y[2 * k], y[2 * k + 1]);
            else codes_to_16<false>(w[k], y[2 * k], y[2 * k + 1]);
          }
          unsigned char* row = stage + (c >> 2) * EA_PANEL + r * 128;
          const int c0 = (c & 3) * 2, sw = r & 7;
          *reinterpret_cast<uint4*>(row + ((c0 ^ sw) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(row + (((c0 + 1) ^ sw) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(full);
      if (j + 1 < nb) load(j + 1, 0);
      if (*abort_flag) break;
    }
    __syncwarp();
  } else if (warp < Cfg::SOFTMAX_WARPS) {
    // ------------------------------------------------------------ softmax
    // One thread has one row of a tile.  Its weights are powers of two relative to a reference that need not be the row's maximum:
    // a later block starts with the reference it finds and looks for a larger maximum on the way; only when that is more than
    // 2^8 above is the block done again.  Where the weights lie over the scores the maximum has to come first.
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t t_lane = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_s = t_lane + t * 128, t_p = t_lane + Cfg::TMEM_P + t * Cfg::P_STRIDE, t_o = t_lane + Cfg::TMEM_O + t * Cfg::O_STRIDE;
    const uint32_t o_done = smem_u32(&sh->o_done[t]);
    const int i = row0 + t * EA_Q + row;
    const int keys = t == 0 ? most[0] : most[1], blocks = t == 0 ? nbt[0] : nbt[1];
    const int sees = i < rq.nq ? enc_sees(a, rq, i) : keys;  // rows that are not there are not written
    float m = -INFINITY;   // the reference
    float z = 0.f;
    for (int j = 0; j < blocks; ++j) {
      mbar_wait_handover(smem_u32(&sh->s_full[t]), (uint32_t)j & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      const int n = columns(keys, j), valid = sees - j * EA_K;  // columns below `valid` are keys that the row sees
      const EaPage* pages = sh->page[j & 3];
      auto hide = [&](int c, uint32_t (&r)[32]) {
        pin32(r);
        if (valid < c + 32) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (c + k >= valid) r[k] = 0xFF800000u;
        }
      };
      // the largest exponent of 32 columns that begin at c
      auto most_of = [&](int c, const uint32_t (&r)[32], float top) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int k = half * 16; k < half * 16 + 16; k += 4) {
            m0 = max3(m0, __uint_as_float(r[k]), __uint_as_float(r[k + 1]));
            m1 = max3(m1, __uint_as_float(r[k + 2]), __uint_as_float(r[k + 3]));
          }
          const float f = CACHED ? pages[c / 16 + half].k : scale_log2, off = CACHED ? pages[c / 16 + half].lv : 0.f;
          top = fmaxf(top, fmaf(fmaxf(m0, m1), f, off));
        }
        return top;
      };
      // their weights in pairs, added to z2
      auto weigh = [&](int c, const uint32_t (&r)[32], float base, unsigned long long& z2, uint32_t (&pk)[16]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float f = scale_log2, off = -base, iv = 1.f;
          if (CACHED) {
            const EaPage pg = pages[c / 16 + half];
            f = pg.k;
            off = pg.lv - base;
            iv = pg.iv;
          }
          const unsigned long long f2 = pack_f32x2(f, f), off2 = pack_f32x2(off, off);
          unsigned long long zc = 0ull;
#pragma unroll
          for (int k = 0; k < 16; k += 2) {
            const unsigned long long x2 = fma_f32x2(pack_f32x2(__uint_as_float(r[half * 16 + k]), __uint_as_float(r[half * 16 + k + 1])), f2, off2);
            float x0, x1;
            unpack_f32x2(x2, x0, x1);
            const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
            zc = add_f32x2(zc, pack_f32x2(e0, e1));
            pk[half * 8 + k / 2] = pack16<P_BF>(e0, e1);
          }
          z2 = CACHED ? fma_f32x2(zc, pack_f32x2(iv, iv), z2) : add_f32x2(zc, z2);
        }
      };
      auto after_product = [&]() {  // of the block before: its weights have been read, the accumulator is complete
        mbar_wait_handover(o_done, (uint32_t)(j - 1) & 1u, abort_flag);
        __syncwarp();
        tc_fence_after();
      };
      auto follow = [&](float top) {
        const float m1 = fmaxf(m, top);
        const float fall = m1 == -INFINITY ? 1.f : ex2_approx(m - m1);  // m = -inf: 0
        m = m1;
        z *= fall;
        tmem_st_wait();
        after_product();
#pragma unroll 1
        for (int c = 0; c < dp; c += 16) {
          uint32_t o[16];
          tmem_ld16(t_o + c, o);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fall);
          tmem_st16(t_o + c, o);
        }
      };
      unsigned long long z2 = 0ull;
      // Whole blocks run without a branch; the loops below serve the others.
      const bool whole = __all_sync(0xFFFFFFFFu, valid >= EA_K);
      bool done = false;
      if (whole && (j > 0 || !Cfg::OWN_P)) {
        uint32_t x[2][32];
        if (!Cfg::OWN_P) {
          float top = -INFINITY;
          tmem_ld32(t_s, x[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_ld_wait();
            pin32(x[c & 1]);
            if (c < 3) tmem_ld32(t_s + (c + 1) * 32, x[(c + 1) & 1]);
            top = most_of(c * 32, x[c & 1], top);
          }
          if (j == 0) m = top;
          else if (__any_sync(0xFFFFFFFFu, top > m + EA_LAZY)) follow(top);
        }
        const float base = m == -INFINITY ? 0.f : m;
        float top = -INFINITY;
        tmem_ld32(t_s, x[0]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tmem_ld_wait();
          pin32(x[c & 1]);
          if (c < 3) tmem_ld32(t_s + (c + 1) * 32, x[(c + 1) & 1]);
          if (Cfg::OWN_P) top = most_of(c * 32, x[c & 1], top);
          uint32_t pk[16];
          weigh(c * 32, x[c & 1], base, z2, pk);
          if (Cfg::OWN_P && c == 0 && j > 0) after_product();
          tmem_st16(t_p + c * 16, pk);
        }
        done = !Cfg::OWN_P || !__any_sync(0xFFFFFFFFu, top > m + EA_LAZY);
      }
      if (!done) {
        float top = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < n; c += 32) {
          uint32_t r[32];
          tmem_ld32(t_s + c, r);
          tmem_ld_wait();
          hide(c, r);
          top = most_of(c, r, top);
        }
        if (j == 0) m = top;
        else if (__any_sync(0xFFFFFFFFu, top > m + EA_LAZY)) follow(top);
        const float base = m == -INFINITY ? 0.f : m;
        if (Cfg::OWN_P && j > 0) after_product();
        z2 = 0ull;
#pragma unroll 1
        for (int c = 0; c < n; c += 32) {
          uint32_t r[32], pk[16];
          tmem_ld32(t_s + c, r);
          tmem_ld_wait();
          hide(c, r);
          weigh(c, r, base, z2, pk);
          tmem_st16(t_p + c / 2, pk);
        }
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->p_full[t]);
      z += __uint_as_float((uint32_t)z2) + __uint_as_float((uint32_t)(z2 >> 32));
    }
    if (blocks > 0) {
      mbar_wait_handover(o_done, (uint32_t)(blocks - 1) & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
    }
    // Outputs leave through the tile's queries, which every product has read: written row by row they would be sixteen bytes of a
    // sector at a time (the kernel for few keys, 8 x 16 of 4 heads of 4096 x 64 over 77: 56.2 us, 48.1 this way).
    const float inv = sees > 0 && (z > 0.f || z != z) ? 1.f / z : 0.f;
    unsigned char* slab = sQ + t * Cfg::TILE + (warp & 3) * 32 * 128;
    uint16_t* out = (uint16_t*)a.O.ptr + b * a.O.batch + (rq.q_row + i) * a.O.token + h * a.O.head;
    const int first = row0 + t * EA_Q + (warp & 3) * 32;           // the warp's rows
    // rows behind a packed request's are another one's; where a tile has no block its queries may still be on their way
    const bool boxed = blocks > 0 && (!a.q_start || first + 32 <= rq.nq);
#pragma unroll 1
    for (int c = 0; c < a.d; c += 32) {
      uint32_t o[32];
      if (blocks > 0) {
        tmem_ld32(t_o + c, o);
        tmem_ld_wait();
        pin32(o);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (c + e * 8 >= a.d) break;
        uint32_t y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          y[k] = blocks > 0 && sees > 0 ? pack16<BF>(__uint_as_float(o[e * 8 + 2 * k]) * inv, __uint_as_float(o[e * 8 + 2 * k + 1]) * inv) : 0u;
        const uint4 y4 = make_uint4(y[0], y[1], y[2], y[3]);
        if (boxed) stage_out(slab, EA_PANEL, lane, c + e * 8, y4);
        else if (i < rq.nq) *reinterpret_cast<uint4*>(out + c + e * 8) = y4;
      }
    }
    if (boxed && first < rq.nq) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        for (int p = 0; p * 64 < a.d; ++p)
          tma_store_4d(&maps.o, slab + p * EA_PANEL, p * 64, h * maps.o_h, (int)rq.q_row + first, b * maps.o_b);
        bulk_commit();
        bulk_wait_read0();
      }
      __syncwarp();
    }
  }

  // ------------------------------------------------------------ common exit
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // give copies that may still be in flight time to land before the block's shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 200000) {
    }
    __syncthreads();
  }
  if (warp == Cfg::WARP_MMA) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::TMEM);
  }
}

// [B, n, H, d] with strides as a 4-D tensor (d, H, n, B), boxes of 64 features x `rows` rows of one head.  A dimension along which
// the tensor broadcasts has extent 1, and the kernel's coordinate there is 0.
static bool ea_encode(CUtensorMap* m, const dgq_rows& r, int64_t B, int64_t n, int64_t H, int d, bool bf, uint32_t rows, int* use_b, int* use_h) {
  *use_b = r.batch != 0;
  *use_h = r.head != 0;
  const uint64_t dims[4] = {(uint64_t)d, *use_h ? (uint64_t)H : 1u, (uint64_t)n, *use_b ? (uint64_t)B : 1u};
  const auto bytes = [&](int64_t s) { return (uint64_t)(s ? s * 2 : (int64_t)kv_row_bytes(d) * 2); };
  const uint64_t strides[3] = {bytes(r.head), bytes(r.token), bytes(r.batch)};
  const uint32_t box[4] = {64, 1, rows, 1};
  return encode_map(m, r.ptr, 4, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                    bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16);
}

template <int NP, bool BF, bool CACHED>
static dgq_status ea_launch_tiles(const EncAttnArgs& a, cudaStream_t stream) {
  using Cfg = EaCfg<NP, CACHED>;
  static std::atomic<bool> attr_set[64];
  int dev = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  if (dev >= 64 || !attr_set[dev].load()) {
    DGQ_CUDA_OK(cudaFuncSetAttribute(enc_attn_tiles_kernel<NP, BF, CACHED>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::SMEM));
    if (dev < 64) attr_set[dev].store(true);
  }
  const int64_t grid = (int64_t)a.B * a.Hq * ((a.nq + EA_Q * Cfg::NT - 1) / (EA_Q * Cfg::NT));
  if (grid > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  EaMaps maps;
  std::memset(&maps, 0, sizeof(maps));
  if (!ea_encode(&maps.q, a.Q, a.q_start ? 1 : a.B, a.q_start ? a.n_rows : a.nq, a.Hq, a.d, BF, 128, &maps.q_b, &maps.q_h)) return DGQ_ERR_CUDA;
  if (!CACHED && (!ea_encode(&maps.k, a.K, a.B, a.nk, a.Hkv, a.d, BF, 128, &maps.k_b, &maps.k_h) ||
                  !ea_encode(&maps.v, a.V, a.B, a.nk, a.Hkv, a.d, BF, 128, &maps.v_b, &maps.v_h)))
    return DGQ_ERR_CUDA;
  if (!ea_encode(&maps.o, a.O, a.q_start ? 1 : a.B, a.q_start ? a.n_rows : a.nq, a.Hq, a.d, BF, 32, &maps.o_b, &maps.o_h)) return DGQ_ERR_CUDA;
  int sms = 0;
  DGQ_CUDA_OK(sm_count(&sms));
  EncAttnArgs aa = a;
  aa.by_length = a.kv_lens && a.B > 1 && a.B <= EA_SORTED && grid > Cfg::BLOCKS * sms;
  DGQ_CUDA_OK(launch_pdl(enc_attn_tiles_kernel<NP, BF, CACHED>, dim3((unsigned)grid), dim3(Cfg::THREADS), (size_t)Cfg::SMEM, stream, maps, aa));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

// ------------------------------------------------------------------ few query rows: keys split over warps and blocks
// The n x G rows of a request's queries that share a key head are columns of S^T = K Q^T (mma.m16n8k16: sixteen keys, eight
// columns), so that a key or value is read once for up to 32 of them (16 for heads beyond 128), straight from memory into the operand's
// registers; more columns are blocks of their own, which read the keys again, for a request with fewer queries than others too.  Which
// features a lane's sixteen bytes hold is the lane's choice as long as Q's fragment follows it.  Weights turn into the second
// product's operand O^T = V^T P by transposing 8 x 8 tiles between lanes.  Codes become fp16 in registers (1.25 instructions a
// code for keys, 1.5 for values).  Each warp has its own running maximum and sums; the warps of a block meet in shared memory,
// the blocks of a request in the shared memory of their cluster, in a fixed order.  Beyond 16 columns heads of 72 to 128 take all 255
// registers and spill 436 bytes (over codes 268), heads beyond 128 with 16 columns 44 (over codes none).
enum { EF_I8 = 0, EF_F16 = 1, EF_BF16 = 2 };
constexpr int EF_SPLITS = 16;   // most blocks of a cluster

template <int SRC, int DC, int NTL>
struct EfCfg {
  static constexpr bool I8 = SRC == EF_I8;
  static constexpr int DMAX = DC == 1 ? 64 : DC == 2 ? 128 : 160;
  static constexpr int KU = I8 ? 16 : 8;                    // features in sixteen bytes of a key
  static constexpr int KR = (DMAX / KU + 3) / 4;            // such loads of a lane per key
  static constexpr int KW = I8 ? 4 : 2;                     // MMA steps per load
  static constexpr int KSTEPS = KR * KW;
  static constexpr int VB = I8 && DC == 1 ? 8 : 16;         // bytes of a value row per lane and load
  static constexpr int VU = I8 ? VB : 8;                    // features in them
  static constexpr int VR = (DMAX / VU + 7) / 8;
  static constexpr int MT = VR * VU / 2;                    // tiles of sixteen features
  static constexpr int GR = I8 && DC < 3 ? 2 : 1;           // groups of sixteen keys per step
  static constexpr int CH = GR * 16;
  static constexpr int WARPS = 4, N = NTL * 8;
  static constexpr int O_LD = DMAX + 4;
  static constexpr int SMEM_Q = NTL * KSTEPS * 32 * 8;
  static constexpr int SMEM_O = WARPS * N * O_LD * 4;
  static constexpr int SMEM = SMEM_Q + SMEM_O + (3 * WARPS + 3) * N * 4;
};

template <bool BF>
__device__ __forceinline__ void ef_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint2 b) {
  if (BF)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
  else
    mma_f16(c, a0, a1, a2, a3, b.x, b.y);
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Bytes 0, 1 (lo) or 2, 3 (hi) of biased codes as two fp16 numbers.
__device__ __forceinline__ uint32_t biased_lo(uint32_t x) {
  const uint32_t y = __byte_perm(x, 0x64646464u, 0x4140), bias = 0x64806480u;
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&y), *reinterpret_cast<const __half2*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t biased_hi(uint32_t x) {
  const uint32_t y = __byte_perm(x, 0x64646464u, 0x4342), bias = 0x64806480u;
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&y), *reinterpret_cast<const __half2*>(&bias));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 ld_stream16(const void* p) {
  uint4 x;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
  return x;
}
__device__ __forceinline__ uint2 ld_stream8(const void* p) {
  uint2 x;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(x.x), "=r"(x.y) : "l"(p));
  return x;
}

template <int SRC, int DC, int NTL>
__global__ void __launch_bounds__(128) enc_attn_few_kernel(const __grid_constant__ EncAttnArgs a, int splits) {
  using Cfg = EfCfg<SRC, DC, NTL>;
  constexpr bool I8 = Cfg::I8;
  constexpr bool M_BF = SRC == EF_BF16;       // type of both products' operands; codes: fp16
  const bool bf = I8 ? a.bf != 0 : M_BF;      // type of Q and O
  constexpr int GR = Cfg::GR, KR = Cfg::KR, KW = Cfg::KW, VR = Cfg::VR, MT = Cfg::MT, N = Cfg::N, KSTEPS = Cfg::KSTEPS;
  extern __shared__ unsigned char smem_dyn[];
  uint2* sQ = reinterpret_cast<uint2*>(smem_dyn);
  float* sO = reinterpret_cast<float*>(smem_dyn + Cfg::SMEM_Q);  // [warp][column][feature]
  float* sM = sO + Cfg::SMEM_O / 4;                              // [warp][column]
  float* sZ = sM + Cfg::WARPS * N;
  float* sF = sZ + Cfg::WARPS * N;
  float* cM = sF + Cfg::WARPS * N;                               // the block's maximum, sum and the columns' factors
  float* cZ = cM + N;
  float* sC = cZ + N;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, lg = lane >> 2, lt = lane & 3;
  const int group = a.Hq / a.Hkv;
  const int split = (int)blockIdx.x % splits;  // heads lie in x too, so that a request's blocks are dealt out together
  const int g = (int)(blockIdx.x / splits) % a.Hkv, col0 = (int)blockIdx.y * N;
  int b = (int)(blockIdx.x / splits) / a.Hkv;
  pdl_wait();
  if (a.by_length) b = enc_request_of_rank(a, b);
  const EncRequest rq = enc_request(a, b);

  // this block's keys: whole steps, the same number for every block of the cluster but the last ones
  const int steps = (rq.len + Cfg::CH - 1) / Cfg::CH, share = (steps + splits - 1) / splits;
  const int step1 = min((split + 1) * share, steps);
  int step = split * share + warp;

  // ------------------------------------------------------------ loads of a step
  // Nothing here is conditional on a lane: a piece beyond a row is another one's instead (Q is zero there, or the feature is not
  // written; a 16-bit key's, which may hold an infinity, becomes zero), a group of absent keys is page 0's (their weights are 0), and
  // a 16-bit row beyond the keys is the last one's.
  const int row_bytes = I8 ? kv_row_bytes(a.d) : a.d * 2;
  uint4 kx[GR][2][KR];
  uint4 vx[GR][4][VR];
  float ks[GR], vs[GR];
  int page_next[GR];
  const int32_t* table = I8 ? a.table + (int64_t)b * a.max_pages : nullptr;
  int kc[KR], vc[VR];  // offset of a lane's pieces in a row
#pragma unroll
  for (int r = 0; r < KR; ++r) kc[r] = (lt + 4 * r) * 16 < row_bytes ? (lt + 4 * r) * 16 : 0;
#pragma unroll
  for (int r = 0; r < VR; ++r) vc[r] = (lg + 8 * r) * Cfg::VB < row_bytes ? (lg + 8 * r) * Cfg::VB : 0;
  const bool short_rows = !I8 && row_bytes < KR * 64;
  const uint8_t* k_rows = I8 ? nullptr : (const uint8_t*)a.K.ptr + 2 * (b * a.K.batch + g * a.K.head);
  const uint8_t* v_rows = I8 ? nullptr : (const uint8_t*)a.V.ptr + 2 * (b * a.V.batch + g * a.V.head);
  auto find_pages = [&](int st) {
    if (!I8 || st >= step1) return;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const int key = st * Cfg::CH + i * 16;
      page_next[i] = key < rq.len ? __ldg(table + (key >> a.page_log2)) : -1;
    }
  };
  auto load_k = [&](int st) {
    if (st >= step1) return;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const int key = st * Cfg::CH + i * 16;
      if (I8) {
        const int p = page_next[i];
        const bool real = p >= 0 && p < a.n_pages;
        if (!real && key < rq.len) record_error(DGQ_ERR_INVALID_ARG);
        const int64_t ph = real ? (int64_t)p * a.Hkv + g : 0;
        ks[i] = __ldg(a.k_scale + ph);
        vs[i] = real ? __ldg(a.v_scale + ph) : -1.f;  // negative: absent
        const uint8_t* base = (const uint8_t*)a.k_codes + ((ph << a.page_log2) + (key & (a.page - 1))) * row_bytes + lg * row_bytes;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int r = 0; r < KR; ++r) kx[i][hh][r] = ld_stream16(base + hh * 8 * row_bytes + kc[r]);
      } else {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint8_t* base = k_rows + 2 * a.K.token * min(key + lg + 8 * hh, rq.len - 1);
#pragma unroll
          for (int r = 0; r < KR; ++r) {
            kx[i][hh][r] = ld_stream16(base + kc[r]);
            if (short_rows && (lt + 4 * r) * 16 >= row_bytes) kx[i][hh][r] = make_uint4(0, 0, 0, 0);
          }
        }
      }
    }
  };
  auto load_v = [&](int st) {
    if (st >= step1) return;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const int key = st * Cfg::CH + i * 16;
      const uint8_t* base = nullptr;
      if (I8) {
        const int p = page_next[i];
        const int64_t ph = p >= 0 && p < a.n_pages ? (int64_t)p * a.Hkv + g : 0;
        base = (const uint8_t*)a.v_codes + ((ph << a.page_log2) + (key & (a.page - 1))) * row_bytes + 2 * lt * row_bytes;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int row = (k & 1) + 8 * (k >> 1);
        const uint8_t* at = I8 ? base + row * row_bytes : v_rows + 2 * a.V.token * min(key + 2 * lt + row, rq.len - 1);
#pragma unroll
        for (int r = 0; r < VR; ++r) {
          if (Cfg::VB == 16) {
            vx[i][k][r] = ld_stream16(at + vc[r]);
          } else {
            const uint2 x = ld_stream8(at + vc[r]);
            vx[i][k][r].x = x.x;
            vx[i][k][r].y = x.y;
          }
        }
      }
    }
  };
  find_pages(step);
  load_k(step);
  load_v(step);
  find_pages(step + Cfg::WARPS);

  // ------------------------------------------------------------ Q as the second operand
  auto q_row = [&](int col) -> const uint16_t* {
    const int i = col / group, h = g * group + col % group;
    if (i >= rq.nq) return nullptr;
    return (const uint16_t*)a.Q.ptr + b * a.Q.batch + (rq.q_row + i) * a.Q.token + h * a.Q.head;
  };
  for (int c = warp; c < N; c += Cfg::WARPS) {
    // bf16 queries over codes: a power of two brings the row's largest value to 1 .. 2, so that fp16 holds what bf16 does
    // (but for what is 2^24 times smaller than the largest)
    float norm = 1.f;
    if (I8 && bf) {
      const uint16_t* q = q_row(col0 + c);
      float top = 0.f;
      if (q)
        for (int k = lane; k < a.d; k += 32) top = fmaxf(top, fabsf(__uint_as_float((uint32_t)q[k] << 16)));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
      const int e = (int)(__float_as_uint(top) >> 23) - 127;
      if (top > 0.f && e < 128) norm = __uint_as_float((uint32_t)(127 - min(max(e, -126), 126)) << 23);
    }
    if (lane == 0) sC[c] = norm;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < NTL * KSTEPS * 32; i += 128) {
    const int l = i & 31, k = (i >> 5) % KSTEPS, nt = (i >> 5) / KSTEPS;
    const int c = nt * 8 + (l >> 2), f = ((l & 3) + 4 * (k / KW)) * Cfg::KU + (k % KW) * 4;
    const uint16_t* q = q_row(col0 + c);
    uint2 x = make_uint2(0, 0);
    if (q && f < a.d) x = *reinterpret_cast<const uint2*>(q + f);
    if (I8 && bf) {
      const float2 lo = unpack16<true>(x.x), hi = unpack16<true>(x.y);
      const float n = sC[c];
      x = make_uint2(pack16<false>(lo.x * n, lo.y * n), pack16<false>(hi.x * n, hi.y * n));
    }
    sQ[i] = x;
  }
  __syncthreads();
  float f[NTL][2];
  int sees[NTL][2];
#pragma unroll
  for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int c = nt * 8 + 2 * lt + k, i = (col0 + c) / group;
      f[nt][k] = a.scale_log2 / sC[c];
      sees[nt][k] = i < rq.nq ? enc_sees(a, rq, i) : 0;
    }

  // ------------------------------------------------------------ the keys
  float m[NTL][2], z[NTL][2], o[MT][NTL][4];
#pragma unroll
  for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      m[nt][k] = -INFINITY;
      z[nt][k] = 0.f;
    }
#pragma unroll
  for (int j = 0; j < MT; ++j)
#pragma unroll
    for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[j][nt][k] = 0.f;
  uint2 qf[NTL == 1 ? KSTEPS : 1];
  if (NTL == 1) {
#pragma unroll
    for (int k = 0; k < KSTEPS; ++k) qf[k] = sQ[k * 32 + lane];
  }

  for (; step < step1; step += Cfg::WARPS) {
    float s[GR][NTL][4];
#pragma unroll
    for (int i = 0; i < GR; ++i)
#pragma unroll
      for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[i][nt][k] = 0.f;
#pragma unroll
    for (int r = 0; r < KR; ++r)
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        uint32_t x[GR][4];
#pragma unroll
        for (int i = 0; i < GR; ++i) {
          if (I8) {
            const uint4 &p = kx[i][0][r], &q = kx[i][1][r];
            const uint32_t u = (w == 0 ? p.x : w == 1 ? p.y : w == 2 ? p.z : p.w) ^ 0x80808080u;
            const uint32_t v = (w == 0 ? q.x : w == 1 ? q.y : w == 2 ? q.z : q.w) ^ 0x80808080u;
            x[i][0] = biased_lo(u);
            x[i][1] = biased_lo(v);
            x[i][2] = biased_hi(u);
            x[i][3] = biased_hi(v);
          } else {
            x[i][0] = w ? kx[i][0][r].z : kx[i][0][r].x;
            x[i][1] = w ? kx[i][1][r].z : kx[i][1][r].x;
            x[i][2] = w ? kx[i][0][r].w : kx[i][0][r].y;
            x[i][3] = w ? kx[i][1][r].w : kx[i][1][r].y;
          }
        }
#pragma unroll
        for (int nt = 0; nt < NTL; ++nt) {
          const uint2 q = NTL == 1 ? qf[r * KW + w] : sQ[(nt * KSTEPS + r * KW + w) * 32 + lane];
#pragma unroll
          for (int i = 0; i < GR; ++i) ef_mma<M_BF>(s[i][nt], x[i][0], x[i][1], x[i][2], x[i][3], q);
        }
      }
    // exponents, in units that include the value's scale
    float fk[GR], lv[GR], iv[GR];
    int key[GR];
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      key[i] = step * Cfg::CH + i * 16 + lg;
      fk[i] = 1.f;
      lv[i] = 0.f;
      iv[i] = 1.f;
      if (I8) {
        const float v = vs[i] == 0.f ? 9.094947e-13f : fmaxf(vs[i], 7.8886091e-31f);
        fk[i] = ks[i];
        lv[i] = vs[i] < 0.f ? -INFINITY : lg2_approx(v);
        iv[i] = rcp_approx(v);
        if (vs[i] < 0.f) key[i] = INT_MAX - 8;
      }
    }
    load_k(step + Cfg::WARPS);
    bool move = false;
    float top[NTL][2];
#pragma unroll
    for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[nt][k] = -INFINITY;
#pragma unroll
        for (int i = 0; i < GR; ++i) {
          const float fc = f[nt][k] * fk[i];
          s[i][nt][k] = key[i] < sees[nt][k] ? fmaf(s[i][nt][k], fc, lv[i]) : -INFINITY;
          s[i][nt][k + 2] = key[i] + 8 < sees[nt][k] ? fmaf(s[i][nt][k + 2], fc, lv[i]) : -INFINITY;
          top[nt][k] = max3(top[nt][k], s[i][nt][k], s[i][nt][k + 2]);
        }
        move |= top[nt][k] > m[nt][k] + EA_LAZY;
      }
    if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
      for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float t = fmaxf(top[nt][k], m[nt][k]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, x));
          const float fall = t == -INFINITY ? 1.f : ex2_approx(m[nt][k] - t);
          m[nt][k] = t;
          z[nt][k] *= fall;
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            o[j][nt][k] *= fall;
            o[j][nt][k + 2] *= fall;
          }
        }
    }
    const bool ragged = (step + 1) * Cfg::CH > rq.len;  // the last step: a row read in the place of one that is not there has weight 0, which NaN would survive
    uint2 pf[GR][NTL];
#pragma unroll
    for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
      for (int i = 0; i < GR; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float base = m[nt][k] == -INFINITY ? 0.f : m[nt][k];
          s[i][nt][k] = ex2_approx(s[i][nt][k] - base);
          s[i][nt][k + 2] = ex2_approx(s[i][nt][k + 2] - base);
          z[nt][k] = fmaf(s[i][nt][k] + s[i][nt][k + 2], iv[i], z[nt][k]);
        }
        pf[i][nt].x = transpose8x8(pack16<M_BF>(s[i][nt][0], s[i][nt][1]));
        pf[i][nt].y = transpose8x8(pack16<M_BF>(s[i][nt][2], s[i][nt][3]));
      }
#pragma unroll
    for (int i = 0; i < GR; ++i)
#pragma unroll
      for (int r = 0; r < VR; ++r)
#pragma unroll
        for (int w = 0; w < Cfg::VB / 4; ++w) {
          uint32_t x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4& p = vx[i][k][r];
            x[k] = w == 0 ? p.x : w == 1 ? p.y : w == 2 ? p.z : p.w;
            if (!I8 && ragged && step * Cfg::CH + 2 * lt + (k & 1) + 8 * (k >> 1) >= rq.len) x[k] = 0;
          }
          if (I8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] ^= 0x80808080u;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t y0 = __byte_perm(x[0], x[1], half ? 0x7362 : 0x5140), y1 = __byte_perm(x[2], x[3], half ? 0x7362 : 0x5140);
              const uint32_t a0 = biased_lo(y0), a1 = biased_hi(y0), a2 = biased_lo(y1), a3 = biased_hi(y1);
#pragma unroll
              for (int nt = 0; nt < NTL; ++nt) ef_mma<M_BF>(o[r * (Cfg::VU / 2) + w * 2 + half][nt], a0, a1, a2, a3, pf[i][nt]);
            }
          } else {
            const uint32_t a0 = __byte_perm(x[0], x[1], 0x5410), a1 = __byte_perm(x[0], x[1], 0x7632);
            const uint32_t a2 = __byte_perm(x[2], x[3], 0x5410), a3 = __byte_perm(x[2], x[3], 0x7632);
#pragma unroll
            for (int nt = 0; nt < NTL; ++nt) ef_mma<M_BF>(o[r * 4 + w][nt], a0, a1, a2, a3, pf[i][nt]);
          }
        }
    load_v(step + Cfg::WARPS);
    find_pages(step + 2 * Cfg::WARPS);
  }

  pdl_launch_dependents();  // blocks of the next kernel that wait from the start take 0.6 us of 16 x 16 x 1 x 64 over 1000 keys (12.4 us)
  // ------------------------------------------------------------ the warps of the block
#pragma unroll
  for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float t = z[nt][k];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, x);
      if (lg == 0) {
        sM[warp * N + nt * 8 + 2 * lt + k] = m[nt][k];
        sZ[warp * N + nt * 8 + 2 * lt + k] = t;
      }
    }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int feature = (lg + 8 * (j / (Cfg::VU / 2))) * Cfg::VU + (j % (Cfg::VU / 2)) * 2;
    if (feature < Cfg::DMAX) {
#pragma unroll
      for (int nt = 0; nt < NTL; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          *reinterpret_cast<float2*>(sO + (warp * N + nt * 8 + 2 * lt + k) * Cfg::O_LD + feature) = make_float2(o[j][nt][k], o[j][nt][k + 2]);
    }
  }
  __syncthreads();
  if (threadIdx.x < N) {
    const int c = threadIdx.x;
    float top = sM[c];
#pragma unroll
    for (int w = 1; w < Cfg::WARPS; ++w) top = fmaxf(top, sM[w * N + c]);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < Cfg::WARPS; ++w) {
      const float fall = top == -INFINITY ? 0.f : ex2_approx(sM[w * N + c] - top);
      sF[w * N + c] = fall;
      sum = fmaf(sZ[w * N + c], fall, sum);
    }
    cM[c] = top;
    cZ[c] = sum;
  }
  __syncthreads();
  const int quads = a.d / 4;
  const int cols = min(N, rq.nq * group - col0);  // columns that exist (none: negative)
  auto of_block = [&](int c, int q) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < Cfg::WARPS; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(sO + (w * N + c) * Cfg::O_LD + q * 4);
      const float fall = sF[w * N + c];
      x = make_float4(fmaf(y.x, fall, x.x), fmaf(y.y, fall, x.y), fmaf(y.z, fall, x.z), fmaf(y.w, fall, x.w));
    }
    return x;
  };
  auto put = [&](int c, int q, float4 x, float sum) {
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const int i = (col0 + c) / group, h = g * group + (col0 + c) % group;
    uint16_t* out = (uint16_t*)a.O.ptr + b * a.O.batch + (rq.q_row + i) * a.O.token + h * a.O.head;
    *reinterpret_cast<uint2*>(out + q * 4) = bf ? make_uint2(pack16<true>(x.x * inv, x.y * inv), pack16<true>(x.z * inv, x.w * inv))
                                                : make_uint2(pack16<false>(x.x * inv, x.y * inv), pack16<false>(x.z * inv, x.w * inv));
  };
  if (splits == 1) {
    for (int u = threadIdx.x; u < cols * quads; u += 128) put(u / quads, u % quads, of_block(u / quads, u % quads), cZ[u / quads]);
    return;
  }
  // ------------------------------------------------------------ the blocks of the cluster
  // Every block leaves its sum in its first slab (a thread reads and writes the same place), then adds up its share of the
  // columns' features over all blocks.
  for (int u = threadIdx.x; u < cols * quads; u += 128) {
    const int c = u / quads, q = u % quads;
    const float4 x = of_block(c, q);
    *reinterpret_cast<float4*>(sO + c * Cfg::O_LD + q * 4) = x;
  }
  const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  cluster.sync();
  for (int u = threadIdx.x * splits + split; u < cols * quads; u += 128 * splits) {
    const int c = u / quads, q = u % quads;
    float top = -INFINITY;
    for (int r = 0; r < splits; r += 4) {
      float t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = *cluster.map_shared_rank(cM + c, min(r + k, splits - 1));
      top = fmaxf(top, fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
    }
    float sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = 0; r < splits; r += 4) {
      // four blocks' loads before the first use: one round trip between the SMs for all
      float t[4], z4[4];
      float4 y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int from = min(r + k, splits - 1);
        t[k] = *cluster.map_shared_rank(cM + c, from);
        z4[k] = *cluster.map_shared_rank(cZ + c, from);
        y[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(sO + c * Cfg::O_LD + q * 4, from));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float fall = r + k >= splits || top == -INFINITY ? 0.f : ex2_approx(t[k] - top);
        sum = fmaf(z4[k], fall, sum);
        x = make_float4(fmaf(y[k].x, fall, x.x), fmaf(y[k].y, fall, x.y), fmaf(y[k].z, fall, x.z), fmaf(y[k].w, fall, x.w));
      }
    }
    put(c, q, x, sum);
  }
  cluster.sync();  // nobody leaves while its shared memory is being read
}

template <int SRC, int DC, int NTL>
static dgq_status ef_launch(const EncAttnArgs& a, cudaStream_t stream) {
  using Cfg = EfCfg<SRC, DC, NTL>;
  const auto kernel = enc_attn_few_kernel<SRC, DC, NTL>;
  static std::atomic<bool> attr_set[64];
  int dev = 0, sms = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  DGQ_CUDA_OK(sm_count(&sms));
  if (dev >= 64 || !attr_set[dev].load()) {
    DGQ_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::SMEM));
    DGQ_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));  // clusters of 16
    if (dev < 64) attr_set[dev].store(true);
  }
  const int64_t columns = (int64_t)a.nq * (a.Hq / a.Hkv), blocks_z = (columns + Cfg::N - 1) / Cfg::N;
  // Blocks that share a head's keys: two to four rounds of the GPU while every warp keeps four steps, and at least one block an
  // SM while every warp has a step (64 requests of 300 to 8000 keys, 8 heads of 128: 147 us with one block a head,
  // 131 with two, 136 with four, 169 with eight; longest first 108 with two; a block costs about 7 us beside its keys).  Clusters of sixteen take long to start and have
  // to be worth it (1 x 8 heads of 64 rows over 600 keys of 128: 31.7 us with sixteen, 17.5 with eight).
  const int64_t steps = ((int64_t)a.nk + Cfg::CH - 1) / Cfg::CH, base = a.B * (int64_t)a.Hkv * blocks_z;
  int splits = 1;
  while (splits < EF_SPLITS && ((base * splits < 6 * sms && steps >= splits * 2 * Cfg::WARPS * 4) || (base * splits < sms && steps > splits * Cfg::WARPS && splits < 8)))
    splits *= 2;
  const int64_t blocks = base / blocks_z * splits;
  if (blocks > INT_MAX || blocks_z > 65535) return DGQ_ERR_UNSUPPORTED;
  EncAttnArgs aa = a;
  aa.by_length = a.kv_lens && a.B > 1 && a.B <= EA_SORTED && blocks > 4 * sms;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)blocks_z);
  cfg.blockDim = dim3(128);
  cfg.dynamicSmemBytes = Cfg::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  DGQ_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, aa, splits));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

template <int SRC, int DC>
static dgq_status ef_launch_columns(const EncAttnArgs& a, cudaStream_t stream) {
  const int64_t columns = (int64_t)a.nq * (a.Hq / a.Hkv);
  if (columns <= 8) return ef_launch<SRC, DC, 1>(a, stream);
  if (columns <= 16 || DC == 3) return ef_launch<SRC, DC, 2>(a, stream);
  return ef_launch<SRC, DC, DC == 3 ? 2 : 4>(a, stream);
}
template <bool BF, bool CACHED>
static dgq_status ef_launch_size(const EncAttnArgs& a, cudaStream_t stream) {
  constexpr int SRC = CACHED ? EF_I8 : BF ? EF_BF16 : EF_F16;
  if (a.d <= 64) return ef_launch_columns<SRC, 1>(a, stream);
  if (a.d <= 128) return ef_launch_columns<SRC, 2>(a, stream);
  return ef_launch_columns<SRC, 3>(a, stream);
}

// ------------------------------------------------------------------ many query rows, few keys
// All keys of a head are one block of scores: a thread block brings keys and values in once (widened, if they are codes) and walks
// tiles of 128 query rows, of all query heads that share them.  No running maximum: a row's is known before its weights.  Two
// threads have a row, one half of its columns each; weights lie over the scores, each half's over its own.  Two thread blocks
// share an SM: the chain of a tile (scores, maximum, weights, product, output) is several times the work in it.
template <int NP, bool CACHED>
struct EsCfg {
  static constexpr int KEYS = NP == 1 ? 192 : 128;         // most keys: scores and outputs in 256 columns of tensor memory
  static constexpr int PANEL = KEYS * 128;                 // bytes of 64 features of the keys
  static constexpr int QST = NP == 1 ? 2 : 1;              // query tiles in shared memory
  static constexpr int SOFTMAX_WARPS = 8, WARP_TMA = 8, WARP_MMA = 9, THREADS = 320;
  static constexpr int TMEM_O = KEYS;
  static constexpr int QTILE = NP * EA_PANEL;
  // outputs have a tile's room of their own beside two query tiles, else they take the queries'
  static constexpr int OFF_O = QST == 2 ? 2 * QTILE : 0;
  static constexpr int OFF_K = QST == 2 ? 3 * QTILE : QTILE, OFF_V = OFF_K + NP * PANEL, OFF_SH = OFF_V + NP * PANEL;
  static constexpr int SMEM = 1024 + OFF_SH + 1024 + 4 * 128 * 4;
  static_assert(2 * SMEM <= 232448 - 2048, "two blocks share an SM");
  static_assert(KEYS + NP * 64 <= 256, "tensor memory budget");
};

struct EsShared {
  uint64_t q_full[2], q_empty[2], kv_full, v_clean, s_full, p_full, o_done;
  uint32_t tmem_base;
  int abort_flag;
  EaPage page[14];  // a thread's last thirty-two columns may begin with its last sixteen
};
static_assert(sizeof(EsShared) <= 1024, "shared block");

__device__ __forceinline__ void pin16(uint32_t (&r)[16]) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
               "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
template <int NP, bool BF, bool CACHED>
__global__ void __launch_bounds__(EsCfg<NP, CACHED>::THREADS, 2)
enc_attn_short_kernel(const __grid_constant__ EaMaps maps, const __grid_constant__ EncAttnArgs a, int chunk_tiles) {
  using Cfg = EsCfg<NP, CACHED>;
  constexpr bool P_BF = BF && !CACHED;
  constexpr int QST = Cfg::QST, PANEL = Cfg::PANEL;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  unsigned char* sQ = smem;
  unsigned char* sK = smem + Cfg::OFF_K;
  unsigned char* sV = smem + Cfg::OFF_V;
  EsShared* sh = reinterpret_cast<EsShared*>(smem + Cfg::OFF_SH);
  float* tops = reinterpret_cast<float*>(smem + Cfg::OFF_SH + 1024);  // [half][row]: what a row's two threads tell each other
  float* sums = tops + 256;
  volatile int* abort_flag = &sh->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // tiles of a key head: those of its first query head, of its second, ...
  const int group = a.Hq / a.Hkv, per_head = (a.nq + EA_Q - 1) / EA_Q, all = per_head * group;
  const int n_chunks = (all + chunk_tiles - 1) / chunk_tiles;
  const int chunk = (int)(blockIdx.x % n_chunks), g = (int)(blockIdx.x / n_chunks) % a.Hkv, b = (int)(blockIdx.x / n_chunks) / a.Hkv;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh->q_full[i], 1);
      mbar_init(&sh->q_empty[i], QST == 2 ? 1 : 4);
    }
    mbar_init(&sh->kv_full, CACHED ? Cfg::SOFTMAX_WARPS : 1);
    mbar_init(&sh->v_clean, 1);
    mbar_init(&sh->s_full, 1);
    mbar_init(&sh->p_full, Cfg::SOFTMAX_WARPS);
    mbar_init(&sh->o_done, 1);
    sh->abort_flag = 0;
    fence_barrier_init();
  }
  // Tensor memory is taken once the kernel before has ended: a block that held it while it waits could keep a block of that one from
  // its own.
  pdl_wait();
  if (warp == Cfg::WARP_MMA) {
    tmem_alloc(&sh->tmem_base, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();  // not before this block has its tensor memory: a block of the next kernel could take it and wait for this one
  const uint32_t tmem_base = sh->tmem_base;

  const EncRequest rq = enc_request(a, b);
  const int n = (rq.len + 15) & ~15, n0 = (n + 16) / 32 * 16;  // columns, and those of a row's first thread
  const int ksteps = (a.d + 15) / 16, dp = ksteps * 16, panels = (a.d + 63) / 64;
  const int tile0 = chunk * chunk_tiles, tile1 = min(tile0 + chunk_tiles, all);
  const bool clean = !CACHED && rq.len < a.nk && rq.len % 16 != 0;  // value rows behind the length, as in the kernel above
  // A tile that a request with fewer queries than others does not have is passed over by all roles.
  const auto real = [&](int tile) { return tile % per_head * EA_Q < rq.nq && rq.len > 0; };

  if (warp == Cfg::WARP_TMA) {
    // ------------------------------------------------------------ loads
    int r = 0;
    for (int tile = tile0; tile < tile1 && !*abort_flag; ++tile) {
      if (!real(tile)) continue;
      if (lane == 0) {
        const int qb = r % QST;
        mbar_wait_handover(smem_u32(&sh->q_empty[qb]), ((uint32_t)(r / QST) & 1u) ^ 1u, abort_flag);
        mbar_arrive_expect_tx(&sh->q_full[qb], (uint32_t)(panels * EA_PANEL));
        for (int p = 0; p < panels; ++p)
          tma_load_4d(sQ + qb * Cfg::QTILE + p * EA_PANEL, &maps.q, &sh->q_full[qb], p * 64, (g * group + tile / per_head) * maps.q_h,
                      (int)rq.q_row + tile % per_head * EA_Q, b * maps.q_b);
        if (!CACHED && r == 0) {
          const int boxes = (rq.len + 63) / 64;
          mbar_arrive_expect_tx(&sh->kv_full, (uint32_t)(2 * boxes * panels * 64 * 128));
          for (int p = 0; p < panels; ++p)
            for (int i = 0; i < boxes; ++i) {
              tma_load_4d(sK + p * PANEL + i * 64 * 128, &maps.k, &sh->kv_full, p * 64, g * maps.k_h, i * 64, b * maps.k_b);
              tma_load_4d(sV + p * PANEL + i * 64 * 128, &maps.v, &sh->kv_full, p * 64, g * maps.v_h, i * 64, b * maps.v_b);
            }
        }
      }
      __syncwarp();
      if (clean && r == 0) {
        mbar_wait_handover(smem_u32(&sh->kv_full), 0, abort_flag);
        for (int k = lane; k < (n - rq.len) * NP * 8; k += 32) {
          const int row = rq.len + k / (NP * 8), c = k % (NP * 8);
          *reinterpret_cast<uint4*>(sV + (c >> 3) * PANEL + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->v_clean);
        __syncwarp();
      }
      ++r;
    }
    __syncwarp();
  } else if (warp == Cfg::WARP_MMA) {
    // ------------------------------------------------------------ products
    const uint32_t idesc_qk = ea_idesc(n, false, BF, a.scale_log2 < 0.f), idesc_pv = ea_idesc(dp, true, P_BF, false);
    constexpr uint32_t HI = smem_desc_hi(1024, 2);
    const uint32_t q_lo = smem_desc_lo(smem_u32(sQ)), k_lo = smem_desc_lo(smem_u32(sK));
    const uint32_t v_lo = ((smem_u32(sV) & 0x3FFFFu) >> 4) | ((uint32_t)(PANEL >> 4) << 16);
    int r = 0;
    for (int tile = tile0; tile < tile1 && !*abort_flag; ++tile) {
      if (!real(tile)) continue;
      const int qb = r % QST;
      if (r == 0) {
        mbar_wait_handover(smem_u32(&sh->kv_full), 0, abort_flag);
        if (clean) mbar_wait_handover(smem_u32(&sh->v_clean), 0, abort_flag);
      }
      mbar_wait_handover(smem_u32(&sh->q_full[qb]), (uint32_t)(r / QST) & 1u, abort_flag);
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < NP * 4; ++k) {
          if (k >= ksteps) break;
          const uint32_t in = (uint32_t)((k & 3) * 32 >> 4);
          mma_f16_lohi(tmem_base, q_lo + (uint32_t)((qb * Cfg::QTILE + (k >> 2) * EA_PANEL) >> 4) + in, HI,
                       k_lo + (uint32_t)((k >> 2) * PANEL >> 4) + in, HI, idesc_qk, k > 0 ? 1u : 0u);
        }
        mma_commit_addr(smem_u32(&sh->s_full));
        if (QST == 2) mma_commit_addr(smem_u32(&sh->q_empty[qb]));
      }
      __syncwarp();
      mbar_wait_handover(smem_u32(&sh->p_full), (uint32_t)r & 1u, abort_flag);
      tc_fence_after();
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < Cfg::KEYS / 16; ++k) {
          if (k * 16 >= n) break;
          const uint32_t at = k * 16 < n0 ? k * 8 : n0 + (k * 16 - n0) / 2;
          mma_f16_ts(tmem_base + Cfg::TMEM_O, tmem_base + at, v_lo + (uint32_t)(k * 2048 >> 4), HI, idesc_pv, k > 0 ? 1u : 0u);
        }
        mma_commit_addr(smem_u32(&sh->o_done));
      }
      __syncwarp();
      ++r;
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const float scale_log2 = fabsf(a.scale_log2);
    if (CACHED) {
      const int row_bytes = kv_row_bytes(a.d), units = row_bytes / 16;
#pragma unroll 2
      for (int u = threadIdx.x; u < n * units; u += Cfg::SOFTMAX_WARPS * 32) {
        const int row = u / units, c = u - row * units;
        uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        const int p = row < rq.len ? ea_page_of(a, b, row) : -1;
        if (p >= 0) {
          const int64_t at = ((((int64_t)p * a.Hkv + g) << a.page_log2) + (row & (a.page - 1))) * row_bytes + c * 16;
          x[0] = __ldg(reinterpret_cast<const uint4*>(a.k_codes + at));
          x[1] = __ldg(reinterpret_cast<const uint4*>(a.v_codes + at));
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t y[8];
          const uint32_t x4[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (BF && w == 0) codes_to_16<true>(x4[k], y[2 * k], y[2 * k + 1]);
            else codes_to_16<false>(x4[k], y[2 * k], y[2 * k + 1]);
          }
          unsigned char* to = (w ? sV : sK) + (c >> 2) * PANEL + row * 128;
          const int c0 = (c & 3) * 2, sw = row & 7;
          *reinterpret_cast<uint4*>(to + ((c0 ^ sw) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(to + (((c0 + 1) ^ sw) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
      }
      if (threadIdx.x < 14) sh->page[threadIdx.x] = threadIdx.x < n / 16 ? ea_page_scales(a, b, g, threadIdx.x * 16, scale_log2) : EaPage{1.f, 0.f, 1.f, 0.f};
      fence_proxy_async_smem();
      named_bar_sync(1, Cfg::SOFTMAX_WARPS * 32);
      if (lane == 0) mbar_arrive(&sh->kv_full);
    }
    const int half = warp >> 2, row = (warp & 3) * 32 + lane, bar = 2 + (warp & 3);
    const uint32_t t_lane = tmem_base + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_lane + Cfg::TMEM_O;
    const int c0 = half ? n0 : 0, nc = half ? n - n0 : n0;  // this thread's columns
    const int valid = rq.len - c0;                          // those below are keys
    const uint32_t t_s = t_lane + c0;
    const EaPage* pages = sh->page + c0 / 16;
    const int f_half = (a.d / 8 + 1) / 2 * 8, f0 = half ? f_half : 0, f1 = half ? a.d : f_half;  // its features of the outputs
    unsigned char* slab = smem + Cfg::OFF_O + (warp & 3) * 32 * 128;
    // Thirty-two columns at a time, those beyond this thread's hidden like those behind the keys.
    const int shown = min(valid, nc);
    auto fetch = [&](int c, uint32_t (&x)[32]) {
      tmem_ld32(t_s + c, x);
      tmem_ld_wait();
      pin32(x);
      if (shown < c + 32) {
#pragma unroll
        for (int k = 0; k < 32; ++k)
          if (c + k >= shown) x[k] = 0xFF800000u;
      }
    };
    int r = 0;
    for (int tile = tile0; tile < tile1; ++tile) {
      const int i = tile % per_head * EA_Q + row, h = g * group + tile / per_head;
      uint16_t* out = (uint16_t*)a.O.ptr + b * a.O.batch + (rq.q_row + i) * a.O.token + h * a.O.head;
      if (!real(tile)) {
        if (i < rq.nq)
          for (int c = half * 8; c < a.d; c += 16) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
        continue;
      }
      mbar_wait_handover(smem_u32(&sh->s_full), (uint32_t)r & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      float top = -INFINITY;
#pragma unroll 1
      for (int c = 0; c < nc; c += 32) {
        uint32_t x[32];
        fetch(c, x);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
          for (int k = e * 16; k < e * 16 + 16; k += 4) {
            m0 = max3(m0, __uint_as_float(x[k]), __uint_as_float(x[k + 1]));
            m1 = max3(m1, __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
          }
          const float f = CACHED ? pages[c / 16 + e].k : scale_log2, off = CACHED ? pages[c / 16 + e].lv : 0.f;
          top = fmaxf(top, fmaf(fmaxf(m0, m1), f, off));
        }
      }
      tops[half * 128 + row] = top;
      if (QST == 2 && half == 0 && lane == 0) bulk_wait_read0();  // the tile before has left the outputs' room
      named_bar_sync(bar, 64);
      top = fmaxf(top, tops[(half ^ 1) * 128 + row]);
      const float base = top == -INFINITY ? 0.f : top;
      unsigned long long z2 = 0ull;
#pragma unroll 1
      for (int c = 0; c < nc; c += 32) {  // weights take the front half of this thread's columns, behind what has been read
        uint32_t x[32], pk[16];
        fetch(c, x);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float f = CACHED ? pages[c / 16 + e].k : scale_log2, off = (CACHED ? pages[c / 16 + e].lv : 0.f) - base;
          const unsigned long long f2 = pack_f32x2(f, f), off2 = pack_f32x2(off, off);
          unsigned long long zc = 0ull;
#pragma unroll
          for (int k = e * 16; k < e * 16 + 16; k += 2) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), f2, off2), x0, x1);
            const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
            zc = add_f32x2(zc, pack_f32x2(e0, e1));
            pk[k >> 1] = pack16<P_BF>(e0, e1);
          }
          if (CACHED) z2 = fma_f32x2(zc, pack_f32x2(pages[c / 16 + e].iv, pages[c / 16 + e].iv), z2);
          else z2 = add_f32x2(zc, z2);
        }
        tmem_st16(t_s + c / 2, pk);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->p_full);
      float z = __uint_as_float((uint32_t)z2) + __uint_as_float((uint32_t)(z2 >> 32));
      sums[half * 128 + row] = z;
      named_bar_sync(bar, 64);
      z += sums[(half ^ 1) * 128 + row];
      const float inv = z > 0.f || z != z ? 1.f / z : 0.f;
      mbar_wait_handover(smem_u32(&sh->o_done), (uint32_t)r & 1u, abort_flag);
      __syncwarp();
      tc_fence_after();
      const int first = tile % per_head * EA_Q + (warp & 3) * 32;  // the warp's rows
      const bool boxed = !a.q_start || first + 32 <= rq.nq;
#pragma unroll 1
      for (int c = f0; c < f1; c += 16) {
        uint32_t o[16];  // features beyond f1 are read for nothing, within the accumulator's columns
        tmem_ld16(t_o + c, o);
        tmem_ld_wait();
        pin16(o);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = pack16<BF>(__uint_as_float(o[e * 8 + 2 * k]) * inv, __uint_as_float(o[e * 8 + 2 * k + 1]) * inv);
          const uint4 y4 = make_uint4(y[0], y[1], y[2], y[3]);
          if (c + e * 8 >= f1) continue;
          if (boxed) stage_out(slab, EA_PANEL, lane, c + e * 8, y4);
          else if (i < rq.nq) *reinterpret_cast<uint4*>(out + c + e * 8) = y4;
        }
      }
      fence_proxy_async_smem();
      named_bar_sync(bar, 64);
      if (half == 0 && lane == 0) {
        if (boxed && first < rq.nq) {
          for (int p = 0; p * 64 < a.d; ++p)
            tma_store_4d(&maps.o, slab + p * EA_PANEL, p * 64, h * maps.o_h, (int)rq.q_row + first, b * maps.o_b);
          bulk_commit();
        }
        if (QST == 1) {
          bulk_wait_read0();
          mbar_arrive(&sh->q_empty[0]);
        }
      }
      ++r;
    }
    if (half == 0 && lane == 0) bulk_wait_read0();
  }

  // ------------------------------------------------------------ common exit
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // give copies that may still be in flight time to land before the block's shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 200000) {
    }
    __syncthreads();
  }
  if (warp == Cfg::WARP_MMA) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, 256);
  }
}

template <int NP, bool BF, bool CACHED>
static dgq_status es_launch(const EncAttnArgs& a, cudaStream_t stream) {
  using Cfg = EsCfg<NP, CACHED>;
  const auto kernel = enc_attn_short_kernel<NP, BF, CACHED>;
  static std::atomic<bool> attr_set[64];
  int dev = 0, sms = 0;
  DGQ_CUDA_OK(cudaGetDevice(&dev));
  DGQ_CUDA_OK(sm_count(&sms));
  if (dev >= 64 || !attr_set[dev].load()) {
    DGQ_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::SMEM));
    if (dev < 64) attr_set[dev].store(true);
  }
  // Tiles of a block: it costs about 3 us beside them, a tile 1 us (2 x 8 heads of 4096 x 40 over 77 keys: 14.5 us with one tile a
  // block, 11.9 with two, 14.0 with three, 19.7 with eight).  Where requests have different numbers of queries, two rounds of
  // blocks at least, so that they even out (8 x 8 heads of 1024 to 4096 x 40 over 20 to 154: 29.3 us with three, 33.1 with eight).
  const int64_t all = (int64_t)((a.nq + EA_Q - 1) / EA_Q) * (a.Hq / a.Hkv), heads = a.B * (int64_t)a.Hkv;
  if (all * heads > INT_MAX) return DGQ_ERR_UNSUPPORTED;
  int tiles = 1;
  float best = 3.4e38f;
  for (int c = 1; c <= 64 && c <= all; ++c) {
    const int64_t blocks = heads * ((all + c - 1) / c), rounds = (blocks + 2 * sms - 1) / (2 * sms);
    if (a.q_start && c > 1 && rounds < 2) break;
    const float time = rounds * (3.f + c);
    if (time < best) {
      best = time;
      tiles = c;
    }
  }
  EaMaps maps;
  std::memset(&maps, 0, sizeof(maps));
  if (!ea_encode(&maps.q, a.Q, a.q_start ? 1 : a.B, a.q_start ? a.n_rows : a.nq, a.Hq, a.d, BF, 128, &maps.q_b, &maps.q_h)) return DGQ_ERR_CUDA;
  if (!CACHED && (!ea_encode(&maps.k, a.K, a.B, a.nk, a.Hkv, a.d, BF, 64, &maps.k_b, &maps.k_h) ||
                  !ea_encode(&maps.v, a.V, a.B, a.nk, a.Hkv, a.d, BF, 64, &maps.v_b, &maps.v_h)))
    return DGQ_ERR_CUDA;
  if (!ea_encode(&maps.o, a.O, a.q_start ? 1 : a.B, a.q_start ? a.n_rows : a.nq, a.Hq, a.d, BF, 32, &maps.o_b, &maps.o_h)) return DGQ_ERR_CUDA;
  const int64_t grid = heads * ((all + tiles - 1) / tiles);
  DGQ_CUDA_OK(launch_pdl(kernel, dim3((unsigned)grid), dim3(Cfg::THREADS), (size_t)Cfg::SMEM, stream, maps, a, tiles));
  g_launches += 1;
  DGQ_CUDA_OK(cudaGetLastError());
  return DGQ_OK;
}

// ------------------------------------------------------------------ launch
// Whether a few tiles of query rows, which leave most SMs without work, take longer than the kernel that splits keys.  Fitted to 72
// shapes of 8 to 128 key heads, 17 to 128 rows, 600 and 4000 keys (time in us): a block of 128 keys for a tile, sixteen keys for
// thirty-two rows of one head over the whole GPU.  1 x 8 heads of 64 rows over 4000 keys of 64: 44 by tiles, 16 split; codes of
// 128: 90 and 27; 8 x 16 heads: 46 and 115, 100 and 160.
static bool ef_is_faster(const EncAttnArgs& a, bool cached, int sms) {
  if (a.nq > 256) return false;
  const int rows = cached && a.d <= 128 ? 2 * EA_Q : EA_Q, columns = a.d <= 128 ? 32 : 16;
  const double blocks = (double)a.B * a.Hq * ((a.nq + rows - 1) / rows), places = sms * (cached || a.d > 128 ? 1.0 : 2.0);
  const double block_us = cached ? 2.6 : a.d <= 64 ? 1.25 : a.d <= 128 ? 1.8 : 2.3;
  const double tiles_us = std::ceil(blocks / places) * (6.0 + std::ceil((double)a.nk / EA_K) * block_us);
  const double unit_us = 1e-3 * (cached ? (a.d <= 64 ? 1.1 : 2.1) : a.d <= 64 ? 1.5 : 3.6);
  const double units = (double)a.B * a.Hkv * std::ceil((double)a.nq * (a.Hq / a.Hkv) / columns) * (a.nk / 16.0);
  return 11.0 + 1.1 * units * unit_us < 0.9 * tiles_us;
}

template <bool BF, bool CACHED>
static dgq_status enc_attn_launch(const EncAttnArgs& a, cudaStream_t stream) {
  if (a.nq <= 16) return ef_launch_size<BF, CACHED>(a, stream);
  EncAttnArgs t = a;
  if (t.scale_log2 == 0.f) t.scale_log2 = 1.17549435e-38f;  // hidden keys are -inf, which 0 would make NaN
  // Few keys: 8 x 16 of 4 heads of 4096 x 64 over 77 keys 48 us as one block of scores, 82 by blocks of 128; over 192 58 and 99.
  if (!a.causal && a.d <= 64 && a.nk <= EsCfg<1, CACHED>::KEYS) return es_launch<1, BF, CACHED>(t, stream);
  if (!a.causal && a.d > 64 && a.d <= 128 && a.nk <= EsCfg<2, CACHED>::KEYS) return es_launch<2, BF, CACHED>(t, stream);
  int sms = 0;
  DGQ_CUDA_OK(sm_count(&sms));
  if (ef_is_faster(a, CACHED, sms)) return ef_launch_size<BF, CACHED>(a, stream);
  if (a.d <= 64) return ea_launch_tiles<1, BF, CACHED>(t, stream);
  if (a.d <= 128) return ea_launch_tiles<2, BF, CACHED>(t, stream);
  return ea_launch_tiles<3, BF, CACHED>(t, stream);
}

}  // namespace dgq

extern "C" dgq_status dgq_encoder_attn(const dgq_rows* Q, const dgq_rows* K, const dgq_rows* V, const dgq_rows* O,
                                       int dtype, int B, int Hq, int Hkv, int nq, int nk, int d, float scale,
                                       const int32_t* kv_lens, void* stream) {
  using namespace dgq;
  if (!rows_pointer_ok(Q) || !rows_pointer_ok(K) || !rows_pointer_ok(V) || !rows_pointer_ok(O) || B <= 0 || Hq <= 0 || Hkv <= 0 ||
      nq <= 0 || nk <= 0 || d <= 0 || Hq % Hkv || (dtype != DGQ_F16 && dtype != DGQ_BF16) || !std::isfinite(scale))
    return DGQ_ERR_INVALID_ARG;
  if (d % 8 || d > KV_MAX_D || nq > EA_MOST || nk > EA_MOST) return DGQ_ERR_UNSUPPORTED;
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
  a.bf = dtype == DGQ_BF16;
  return a.bf ? enc_attn_launch<true, false>(a, (cudaStream_t)stream) : enc_attn_launch<false, false>(a, (cudaStream_t)stream);
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
  if ((int64_t)max_pages * cache->page > EA_MOST || max_nq > EA_MOST || (q_start && n_rows > EA_MOST)) return DGQ_ERR_UNSUPPORTED;
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
  a.page_log2 = kv_log2(cache->page);
  a.max_pages = max_pages;
  a.table = block_table;
  a.q_start = q_start;
  a.n_rows = n_rows;
  a.causal = causal != 0;
  a.bf = dtype == DGQ_BF16;
  return a.bf ? enc_attn_launch<true, true>(a, (cudaStream_t)stream) : enc_attn_launch<false, true>(a, (cudaStream_t)stream);
}
