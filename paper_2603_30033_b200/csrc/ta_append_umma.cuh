// Append to a paged latent cache on tcgen05: [K | V] = X [U3 | Ut3], latent RoPE on K, rows scattered to their pages;
// one launch, nothing between X and the pages touches memory.
//
// One CTA multiplies MT tiles of 128 token rows (A, K-major) with the factors as they lie in memory (B, MN-major), all
// columns of both or of one of them, over a share of d.  The S CTAs of a cluster share the rows and split d: a batch of
// a few tokens is bound by reading the factors, which S (times two) SMs then do at once, and a long prompt whose row
// tiles do not fill the GPU gets more CTAs without reading X or the factors twice.  The sum over the cluster goes
// through the caller's workspace, i.e. the L2 cache:
//   unit       32 columns x 128 rows of fp32 sums; the units of a cluster are dealt evenly to its CTAs
//   every CTA  writes the others' units, meets them at the cluster's barrier, reads its own units back and adds them in
//              the order of the shares (its own share straight from TMEM): no atomics, the result does not depend on
//              timing
// (Through distributed shared memory, written or read, the same exchange moved about 13 bytes per cycle and SM: 128 KB
// per CTA took 10 thousand cycles of the 16384-token call, and 7 of the 16 thousand cycles of the 64-token call.)
//   epilogue   thread = token row: rotation at the row's position (angles formed while the products run), one rounding
//              to bf16, 64 adjacent bytes of eight rows per store instruction
// Bounds: X read once and the pages written once when T is large; per-CTA bytes of X and the factors over L2 otherwise,
// which is what the choice of MT, S and the column split minimises (append_plan).
//   warp 0  TMA producer      warp 1  TMEM, MMA issue      warps 2..9  epilogue, two per TMEM lane quadrant
#pragma once

#include "ta_paged.cuh"
#include "ta_sm100.cuh"

namespace ta {
namespace append {

using namespace sm100;

constexpr int BM = 128, BK = 64, UC = 32;        // UC: columns of a unit
constexpr int THREADS = 320;
constexpr int MAX_STAGES = 8;
constexpr int RING_BYTES = 192 * 1024;
constexpr size_t SMEM_BYTES = 1024 + (size_t)RING_BYTES;
constexpr int A_BYTES = BM * BK * 2, BOX_BYTES = 64 * BK * 2, UNIT_BYTES = UC * BM * 4;
// A finished unit's rounded rows wait for their stores in the idle ring, a place per unit: places used again would have
// to wait for the stores (64 single tokens 11.5 -> 12.7 us on the GPU).  A CTA finishes 16 units at most, 512 columns of
// TMEM.
constexpr int MAX_UNITS = 512 / UC, STAGED_BYTES = UC * BM * 2;
static_assert(MAX_UNITS * STAGED_BYTES <= RING_BYTES, "all units of a CTA fit into the ring");
constexpr int MAX_S = 8;
constexpr int CSU = 2;                           // units per thread whose angles are formed ahead

// A factor [d, width] and where its products go.
struct Part {
  bf16* pool;
  int width;          // r3 or t3, a multiple of 32, at most 256
  int rope;           // 1: rotated before rounding
};
struct Params {
  int T, d, S, MT;               // token rows, embedding width, CTAs per cluster, row tiles per CTA
  int n_parts;                   // parts a CTA computes: n_parts of part[], from part[blockIdx.y] on
  Part part[2];
  const int32_t *tok_start, *cache_len;
  int B, pos0;
  PagedView pv;
  float* part_sums;              // S > 1: [part, when split][cluster][share][unit][128 x UC]
  int y_units;                   // units of a cluster of the first part (split)
  unsigned int* err;
};

// TMEM columns of one accumulator
__host__ __device__ constexpr uint32_t acc_cols(int width) { return width <= 32 ? 32u : (width <= 64 ? 64u : (width <= 128 ? 128u : 256u)); }
__host__ __device__ inline int boxes(int width) { return (width + 63) / 64; }

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(THREADS, 1)
k_append(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmB0, const __grid_constant__ CUtensorMap tmB1,
         const Params p, const dec::RopeTurns turns) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full_bar[MAX_STAGES], empty_bar[MAX_STAGES], acc_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring = smem_raw + (base - smem_u32(smem_raw));
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int S = p.S, MT = p.MT, s = (int)(blockIdx.x % (unsigned)S);
  const int m0 = (int)(blockIdx.x / (unsigned)S) * MT * BM;
  Abort ab{&abort_flag, p.err};
  // this CTA's parts, their place among a row tile's TMEM columns, and the K blocks of its share of d
  const Part p0 = p.part[blockIdx.y];
  const Part p1 = p.n_parts > 1 ? p.part[1] : Part{nullptr, 0, 0};
  const int width = p0.width + p1.width;
  const uint32_t c1 = acc_cols(p0.width);                                  // first column of the second part
  const uint32_t tile_cols = c1 + (p1.width ? acc_cols(p1.width) : 0u);
  uint32_t ncols = 32;
  while (ncols < tile_cols * (uint32_t)MT) ncols *= 2;
  const int nb = boxes(p0.width) + (p1.width ? boxes(p1.width) : 0);
  const uint32_t stage_bytes = (uint32_t)(MT * A_BYTES + nb * BOX_BYTES);
  const int stages = min(MAX_STAGES, (int)(RING_BYTES / stage_bytes));
  const int nkb = p.d / BK, kb0 = (int)((long)nkb * s / S), kb1 = (int)((long)nkb * (s + 1) / S);
  // units of the cluster: (row tile, column chunk); this CTA finishes [u0, u1)
  const int upt = width / UC, units = MT * upt;
  const int u0 = units * s / S, u1 = units * (s + 1) / S;

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < MAX_STAGES; ++i) { mbar_init(&full_bar[i], 1); mbar_init(&empty_bar[i], 1); }
    mbar_init(&acc_bar, 1);
    fence_barrier_init();
  }
  pdl_enter();
  if (warp == 1) {
    tmem_alloc(&tmem_slot, ncols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  bool ok = true;
  AppendDst dst[2];
  float2 cs[CSU][UC / 2];
  const int q = warp % 4, hf = (warp - 2) >> 2, rloc = q * 32 + lane;
  if (warp == 0) {
    if (elect_one()) {
      tma_prefetch_desc(&tmX); tma_prefetch_desc(&tmB0); tma_prefetch_desc(&tmB1);
      const CUtensorMap* tb0 = blockIdx.y == 0 ? &tmB0 : &tmB1;
      int issued = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++issued) {
        const int i = kb - kb0, st = i % stages;
        if (!mbar_wait(&empty_bar[st], ((i / stages) & 1) ^ 1, ab)) break;
        mbar_expect_tx(&full_bar[st], stage_bytes);
        uint8_t* a = ring + (size_t)st * stage_bytes;
        uint8_t* b = a + MT * A_BYTES;
        for (int t = 0; t < MT; ++t) tma_load_2d(a + t * A_BYTES, &tmX, &full_bar[st], kb * BK, m0 + t * BM);
        for (int j = 0; j < boxes(p0.width); ++j) tma_load_2d(b + j * BOX_BYTES, tb0, &full_bar[st], j * 64, kb * BK);
        b += boxes(p0.width) * BOX_BYTES;
        if (p1.width)
          for (int j = 0; j < boxes(p1.width); ++j) tma_load_2d(b + j * BOX_BYTES, &tmB1, &full_bar[st], j * 64, kb * BK);
      }
      if (ab.raised()) mbar_drain_ring(full_bar, issued, stages);     // the copies in flight end before the CTA does
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint32_t id0 = umma_idesc_bf16(BM, (uint32_t)p0.width) | (1u << 16), id1 = umma_idesc_bf16(BM, (uint32_t)p1.width) | (1u << 16);
      for (int kb = kb0; kb < kb1; ++kb) {
        const int i = kb - kb0, st = i % stages;
        if (!(ok = mbar_wait(&full_bar[st], (i / stages) & 1, ab))) break;
        tc_fence_after();
        const uint32_t a = smem_u32(ring + (size_t)st * stage_bytes), b = a + MT * A_BYTES;
        for (int t = 0; t < MT; ++t) {
          const uint64_t da = umma_desc_kmajor_sw128(a + t * A_BYTES);
          const uint64_t db0 = umma_desc_mnmajor_sw128(b, BOX_BYTES);
          const uint64_t db1 = umma_desc_mnmajor_sw128(b + boxes(p0.width) * BOX_BYTES, BOX_BYTES);
          const uint32_t d = tmem + (uint32_t)t * tile_cols;
#pragma unroll
          for (int k = 0; k < BK / 16; ++k)
            umma_ss(d, da + (uint64_t)(k * 2), db0 + (uint64_t)(k * 128), id0, (i | k) != 0 ? 1u : 0u);
          if (p1.width) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k)
              umma_ss(d + c1, da + (uint64_t)(k * 2), db1 + (uint64_t)(k * 128), id1, (i | k) != 0 ? 1u : 0u);
          }
        }
        umma_commit(&empty_bar[st]);
      }
      umma_commit(&acc_bar);
    }
  } else {
    // ------------------------------- epilogue warps -------------------------------
    // while the products run: where this thread's rows go
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      dst[t].row = -1; dst[t].pos = 0;
      const int row = m0 + t * BM + rloc;
      if (t < MT && row < p.T) dst[t] = append_dst(row, p.tok_start, p.cache_len, p.B, p.pos0, p.pv, p.err);
    }
    // ... and the angles of its first two units, where they are rotated (all of its rotated units, unless r3 > 128 or
    // the CTA finishes two row tiles by itself)
#pragma unroll
    for (int k = 0; k < CSU; ++k) {
      const int u = u0 + hf + 2 * k, t = u / upt, c = (u % upt) * UC;
      if (u < u1 && c < p0.width && p0.rope)
#pragma unroll
        for (int e = 0; e < UC / 2; ++e) cs[k][e] = dec::rope_at((t == 0 ? dst[0] : dst[1]).pos, turns, c / 2 + e);
    }
    ok = mbar_wait(&acc_bar, 0, ab);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
  }
  auto unit_tmem = [&](int u) -> uint32_t {
    const int t = u / upt, c = (u % upt) * UC;
    return tmem + (uint32_t)t * tile_cols + (c < p0.width ? (uint32_t)c : c1 + (uint32_t)(c - p0.width)) + ((uint32_t)(q * 32) << 16);
  };
  // rows of this warp that exist: none of the others' sums are needed
  auto warp_rows = [&](int u) -> bool { return m0 + (u / upt) * BM + q * 32 < p.T; };
  // 16-byte chunk `ch` of row `row` of a staged unit: a warp's rows of one chunk are adjacent, and the four chunks of one
  // row lie on different banks
  auto chunk_at = [&](int slot, int row, int ch) -> uint32_t {
    return (uint32_t)(slot * STAGED_BYTES + ch * (BM * 16) + ((row ^ ch) << 4));
  };
  // this cluster's partial sums, [share][unit][chunk][row] of 16 bytes
  float4* const part = reinterpret_cast<float4*>(p.part_sums) + ((long)blockIdx.y * (gridDim.x / S) * p.y_units + (long)(blockIdx.x / S) * units) * S * (UNIT_BYTES / 16);
  [[maybe_unused]] const long part_n = (long)S * units * (UNIT_BYTES / 16);
  if (S > 1) {
    if (warp >= 2 && ok) {
      for (int u = hf; u < units; u += 2) {
        if ((u >= u0 && u < u1) || !warp_rows(u)) continue;
        uint32_t r[32];
        tmem_ld32(unit_tmem(u), r);
        tmem_ld_wait();
        const long at = ((long)s * units + u) * (UNIT_BYTES / 16) + rloc;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (TA_IDX_OK(p.err, at + e * BM, 1, part_n))
            __stcg(part + at + e * BM, make_float4(__uint_as_float(r[4 * e]), __uint_as_float(r[4 * e + 1]), __uint_as_float(r[4 * e + 2]),
                                                   __uint_as_float(r[4 * e + 3])));
      }
    }
    __syncwarp();
    cluster_sync();                     // orders the writes above before the reads below, across the cluster
  }
  if (warp >= 2 && ok) {
    auto finish = [&](int u, bool have, const float2 (&a)[UC / 2]) {
      const int t = u / upt, c = (u % upt) * UC;
      const AppendDst& to = t == 0 ? dst[0] : dst[1];
      float v[32];
      {
        uint32_t r[32];
        tmem_ld32(unit_tmem(u), r);
        tmem_ld_wait();
        if (S == 1) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.f;
          for (int o = 0; o < S; ++o) {           // in the order of the shares of d
            if (o == s) {
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] += __uint_as_float(r[e]);
            } else {
              const long at = ((long)o * units + u) * (UNIT_BYTES / 16) + rloc;
              float4 w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) w[e] = TA_IDX_OK(p.err, at + e * BM, 1, part_n) ? __ldcg(part + at + e * BM) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int e = 0; e < 8; ++e) { v[4 * e] += w[e].x; v[4 * e + 1] += w[e].y; v[4 * e + 2] += w[e].z; v[4 * e + 3] += w[e].w; }
            }
          }
        }
      }
      const bool first = c < p0.width;
      if (first && p0.rope) {
#pragma unroll
        for (int e = 0; e < UC / 2; ++e) {
          const float2 cse = have ? a[e] : dec::rope_at(to.pos, turns, c / 2 + e);
          const float xe = v[2 * e], xo = v[2 * e + 1];
          v[2 * e] = xe * cse.x - xo * cse.y;
          v[2 * e + 1] = xe * cse.y + xo * cse.x;
        }
      }
      // the rounded row into this thread's own place in the idle ring ...
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<uint4*>(ring + chunk_at(u - u0, rloc, e)) =
            make_uint4(pack_bf16(v[8 * e], v[8 * e + 1]), pack_bf16(v[8 * e + 2], v[8 * e + 3]), pack_bf16(v[8 * e + 4], v[8 * e + 5]),
                       pack_bf16(v[8 * e + 6], v[8 * e + 7]));
      __syncwarp();
      // ... and from there to the pages, the 64 bytes of eight rows per store instruction
      bf16* pool = first ? p0.pool : p1.pool;
      const int wd = first ? p0.width : p1.width, cc = (first ? c : c - p0.width) + (lane & 3) * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rr = i * 8 + lane / 4;
        const long row = __shfl_sync(0xffffffffu, to.row, rr);
        const uint4 w = *reinterpret_cast<const uint4*>(ring + chunk_at(u - u0, q * 32 + rr, lane & 3));
        if (row >= 0 && TA_IDX_OK(p.err, row * wd + cc, 8, (long)p.pv.n_pages * p.pv.page_size * wd))
          *reinterpret_cast<uint4*>(pool + row * wd + cc) = w;
      }
    };
#pragma unroll
    for (int k = 0; k < CSU; ++k) {
      const int u = u0 + hf + 2 * k;
      if (u < u1 && warp_rows(u)) finish(u, true, cs[k]);
    }
    for (int u = u0 + hf + 2 * CSU; u < u1; u += 2)
      if (warp_rows(u)) finish(u, false, cs[0]);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, ncols);
}

// How a call is divided: MT row tiles per CTA, S shares of d per cluster, and whether the two factors go to different
// CTAs. The CTA's time is taken as proportional to the bytes it moves into shared memory, times the waves of one CTA
// per SM; a share of d costs the partial sums once to the L2 cache and back.
struct Plan {
  int MT, S, split_parts;
};
inline Plan append_plan(int T, int d, int w0, int w1, int sms) {
  Plan best{1, 1, 0};
  double best_cost = -1;
  const int tiles = (T + BM - 1) / BM, nkb = d / BK;
  for (int mt = 1; mt <= 2; ++mt)
    for (int split = 0; split <= (w1 > 0 ? 1 : 0); ++split)
      for (int S = 1; S <= MAX_S && S <= nkb; S *= 2) {
        const int width = split ? (w0 > w1 ? w0 : w1) : w0 + w1;
        const uint32_t cols = split ? acc_cols(width) : acc_cols(w0) + (w1 ? acc_cols(w1) : 0u);
        if (mt > tiles || cols * mt > 512) continue;
        const long ctas = (long)((tiles + mt - 1) / mt) * S * (split ? 2 : 1);
        const long waves = (ctas + sms - 1) / sms;
        const int rows = T < mt * BM ? T : mt * BM;
        const double bytes = 2.0 * ((double)rows + width) * d / S + (S > 1 ? 2.0 * 4.0 * rows * width / S : 0.0) + 16384.0;
        const double cost = waves * bytes;
        if (best_cost < 0 || cost < best_cost) { best_cost = cost; best = Plan{mt, S, split}; }
      }
  return best;
}
// Bytes of partial sums the plan needs.
inline size_t append_part_bytes(const Plan& q, int T, int w0, int w1) {
  if (q.S == 1) return 0;
  const size_t clusters = ((size_t)T + q.MT * BM - 1) / (q.MT * BM);
  return clusters * q.S * q.MT * BM * sizeof(float) * (q.split_parts ? 2 * (size_t)(w0 > w1 ? w0 : w1) : (size_t)w0 + w1);
}

}  // namespace append
}  // namespace ta
