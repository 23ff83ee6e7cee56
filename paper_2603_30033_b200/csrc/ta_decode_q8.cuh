// Decode attention over a paged latent cache held in 8 bits (Eq. 9) on tcgen05 tensor cores.
//
// The bytes of the cache bound the step, and there are half as many as in bf16: a tile of 128 keys, 32 KB of codes, is due
// every 1450 cycles per SM at the copy rate, where the bf16 kernel's tile has 2900.  So the codes are never converted: the
// tiles go to the tensor cores as TMA wrote them (kind::f8f6f4), and everything else is arranged around that.
//
//   S^T [128 keys x 32 heads] = K_codes * q^T      The query is carried as three e4m3 numbers per coordinate (the rounded
//       value, the rounded rest, the rest's rounded rest: 2^-12 of it together), which are three products into one
//       accumulator.  Its own scale is a power of two per sequence.  Two numbers (2^-8) would move scores of a standard
//       deviation of 2 by what the rounding of y to bf16 moves the output.
//   p 2^k' [128 keys x 32 heads]                   A thread owns a key, so the row's scales are two numbers of its own: 2^k
//       multiplies the scores, 2^k' the weight of the value row, as a term of the exponent.  The sums are of p alone.
//   O^T [t3 x 32 heads] += V_codes^T * (p 2^k')    The weight is carried as three e5m2 numbers: the upper byte of an f16, the
//       upper byte of what is left, and of what is left then, rounded (2^-10 together; a byte's worth of an f16 is an e5m2,
//       so this is masking and exact subtraction).  e5m2 for its range: with the reference maximum at 2^11 .. 2^15, weights
//       down to 2^-27 of the largest count in full precision or to 2^-28 absolute.  The three are 96 columns of one product
//       and of the accumulator, and are added up once per segment.
//
// Two softmax warpgroups take tiles in turn, each with its own scores, weights, running maxima, sums and accumulator (two of
// each fit TMEM here), so that a tile's chain of waits has the time of two tiles; the bf16 kernel's warpgroups share every
// tile.  What agreement on a tile still takes is one vote over a warpgroup: whether any score lies more than 2^15 above its
// head's reference.  Then, at the first tile of a segment and seldom after, the maxima are taken and the accumulator rescaled.
// At the end of a (CTA, sequence) segment one warpgroup hands its part to the other through its weights' buffer.
//
//   warp 0       TMA producer: pages of codes, and their scale bytes by plain bulk copies
//   warp 1       TMEM allocation, MMA issue: scores two tiles ahead of the values
//   warps 2, 3   split the next segment's queries; put the new token's row into the tile that holds it
//   warps 4 + 4 g .. 7 + 4 g   softmax warpgroup g: tiles g, g + 2, ...
// TMEM columns: S_0 [0, 32), S_1 [32, 64), O_0 [64, 160), O_1 [160, 256).
// Every wait is bounded (Abort).
#pragma once

#include "ta_common.cuh"
#include "ta_decode.cuh"
#include "ta_decode_umma.cuh"
#include "ta_q8.cuh"
#include "ta_sm100.cuh"

#include <cuda_fp16.h>

namespace ta {
namespace decq {

using namespace sm100;
using decu::ex2;
using decu::warp_max;

constexpr int TK = 128;                          // keys per tile
constexpr int NWG = 2, THREADS = 128 + 128 * NWG;
constexpr int NH = 32;                           // head columns
constexpr int TILE_BYTES = TK * 128;             // rows of 128 bytes, the last of them zeros where a rank is smaller
constexpr int RING_BYTES = 10 * TILE_BYTES;      // five K + V stages, or ten of one shared pool
constexpr int MAX_STAGES = 10;
constexpr int PIECES = 3;
constexpr int QPIECE_BYTES = NH * 128, QBUF_BYTES = PIECES * QPIECE_BYTES;
constexpr int PBUF_BYTES = TK * 128;             // a key's 96 weights in a row of 128 bytes
constexpr int SCALE_BYTES = 2 * TK;              // of a stage
// ring | queries of two segments | weights of two tiles | scales
constexpr size_t SMEM_BYTES = 1024 + (size_t)RING_BYTES + 2 * QBUF_BYTES + 2 * PBUF_BYTES + MAX_STAGES * SCALE_BYTES;
static_assert(SMEM_BYTES <= 225 * 1024, "one CTA's shared memory, with the static part");
constexpr float kTop = 15.f, kStart = 11.f;      // weights reach 2^kTop at most, the largest is 2^kStart when a reference is set

struct Params {
  int B, nH, Lmax, r3, t3;
  int shared_kv;           // 1: one pool, the K tile is the V tile
  const int32_t* cache_len;
  const uint8_t *Ks, *Vs;  // scale bytes of the pools
  const bf16* qhat;        // [2][B, nH, r3] per-head queries in units of log2: rounded values, rounded rests
  const uint32_t* qmax;    // [B][4] bits of the largest |q| of each 32 coordinates
  const uint8_t *knew, *vnew;      // [B, r3], [B, t3] codes of the new rows
  const uint8_t* new_scale;        // [B][2] their scale bytes
  float* part_o;           // [grid + B][t3 / 4][32][4]
  float* part_ml;          // [grid + B][32][2]  (reference in log2 units, sum)
  unsigned int* err;
  PagedView pv;
  int* seq_cta;            // [B][2] first and last CTA that holds a part of the sequence, for the join
};

// Instruction descriptor: D fp32, A e4m3, B of `b_format` (0 e4m3, 1 e5m2), shape M x N (x 32).
__host__ __device__ constexpr uint32_t idesc_f8(uint32_t b_format, uint32_t M, uint32_t N) {
  return (1u << 4) | (b_format << 10) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
      "}\n"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 16-byte chunk of a row of 128 bytes, 128-byte swizzle
__device__ __forceinline__ uint32_t swz(int row, int chunk) { return (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

// Sums of v[h] over the 32 lanes of the warp; lane h returns that of v[h].  At each level a lane hands half of its values on.
__device__ __forceinline__ float lane_sums(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int half = 16; half >= 1; half >>= 1) {
    const bool up = lane & half;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float mine = up ? v[i + half] : v[i], give = up ? v[i] : v[i + half];
      v[i] = mine + __shfl_xor_sync(0xffffffffu, give, half);
    }
  }
  return v[0];
}

__global__ void __launch_bounds__(THREADS, 1)
k_dec_attn_q8(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full_bar[MAX_STAGES], empty_bar[MAX_STAGES], patched[MAX_STAGES], q_full[2], q_empty[2];
  __shared__ uint64_t s_full[NWG], s_free[NWG], p_full[NWG], p_free[NWG], o_read[NWG], handed[NWG], taken[NWG], wg_bar[NWG], wanted;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float q_scale[8];                   // of segment i at i & 7: the queries are split at most three segments ahead
  __shared__ uint32_t votes[NWG][2];             // a byte per warp, by parity of the warpgroup's tiles
  __shared__ float max_s[NWG][4][NH], sum_s[NWG][4][NH], hand_m[NWG][NH], hand_l[NWG][NH];
  __shared__ long long wtot_s[THREADS / 32];
  __shared__ int loc_b;
  __shared__ long long loc_first;

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* ring = smem_raw + (base - smem_u32(smem_raw));
  uint8_t* qbuf = ring + RING_BYTES;
  uint8_t* pbuf = qbuf + 2 * QBUF_BYTES;
  uint8_t* scales = pbuf + 2 * PBUF_BYTES;
  const int STAGES = p.shared_kv ? 10 : 5;
  const int stage_bytes = p.shared_kv ? TILE_BYTES : 2 * TILE_BYTES;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Abort ab{&abort_flag, p.err};

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
      mbar_init(&patched[s], 2);          // the new token's row is in its place: one arrival per helping warp
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 2);
      mbar_init(&q_empty[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], 4);           // the scores are in registers
      mbar_init(&p_full[i], 4);           // the weights are in shared memory
      mbar_init(&p_free[i], 1);           // the product that read them is complete
      mbar_init(&o_read[i], 4);           // the accumulator of a finished segment has been read
      mbar_init(&handed[i], 4);           // warpgroup i has laid its part of a segment down ...
      mbar_init(&taken[i], 4);            // ... and the other one has picked it up
      mbar_init(&wg_bar[i], 4);
    }
    mbar_init(&wanted, 1);                // the next tile with a new token's row has arrived
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_slot, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // ---- this CTA's range of the flat tile list (see k_dec_attn_umma) ----
  int lo, hi;
  long excl;
  const long total = dec::block_tile_scan(p.cache_len, p.B, p.Lmax, lo, hi, excl, wtot_s);
  const long parts = min((long)gridDim.x, total);
  const long t_begin = min(dec::cta_first_tile(blockIdx.x, total, parts), total);
  const long t_end = min(dec::cta_first_tile(blockIdx.x + 1, total, parts), total);
  {
    long f = excl;
    for (int b = lo; b < hi; ++b) {
      const long nt = dec::tiles_of(dec::clamp_len(p.cache_len[b], p.Lmax));
      if (t_begin >= f && t_begin < f + nt) { loc_b = b; loc_first = f; }
      f += nt;
    }
  }
  __syncthreads();
  const bool have_work = t_begin < t_end;
  const int n_tiles = (int)(t_end - t_begin);
  decu::Walk w;
  if (have_work) w.init(p, t_begin, t_end, loc_b, (long)loc_first);
  auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {
    const bool good = mbar_wait(bar, parity, ab);
    return __all_sync(0xffffffffu, good);
  };

  // 88 x 128 + 208 x 256 = 64512 = 168 x 384 registers, what the CTA was launched with
  if (warp < 4) {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
   if (have_work && warp == 0) {
    // ------------------------------- TMA producer -------------------------------
    if (elect_one()) { tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV); }
    __syncwarp();
    const int ps = p.pv.page_size;
    const int box_rows = ps < TK ? ps : TK, n_box = TK / box_rows, kinds = p.shared_kv ? 1 : 2;
    // page of box `lane` of the tile that ww is positioned on; -1 where the box holds no cached row
    auto lookup = [&](const decu::Walk& ww, long t) -> int {
      const int r = ww.k0(t) + lane * box_rows;
      return (lane < n_box && r < ww.L) ? p.pv.table[(long)ww.b * p.pv.max_pages + r / ps] : -1;
    };
    struct Box { int pg, in_page; uint32_t bytes; bool mine, good; };
    auto box_of = [&](const decu::Walk& ww, long t, int pg) -> Box {
      const int row = ww.k0(t) + lane * box_rows;
      Box x;
      x.mine = lane < n_box && row < ww.L;
      x.good = x.mine && pg >= 0 && pg < p.pv.n_pages;
      if (x.mine && !x.good) {
        atomicOr(p.err, (unsigned)TA_DEVERR_BAD_PAGE);
        pg = p.pv.n_pages;                         // outside the tensor: the box is filled with zeros
      }
      x.pg = pg;
      x.in_page = row % ps;
      x.bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, x.mine)) * kinds * box_rows * 128 +
                           __popc(__ballot_sync(0xffffffffu, x.good)) * kinds * box_rows);
      return x;
    };
    auto load_tile = [&](const Box& x, int s) {
      uint8_t* sc = scales + s * SCALE_BYTES + lane * box_rows;
      if (x.mine && !x.good)                       // rows of zeros: any scale but NaN
        for (int i = 0; i < box_rows; i += 16)
          for (int k = 0; k < kinds; ++k) *reinterpret_cast<uint4*>(sc + k * TK + i) = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
      __syncwarp();
      if (lane == 0) mbar_expect_tx(&full_bar[s], x.bytes);
      __syncwarp();
      if (x.mine) {
        uint8_t* kt = ring + (size_t)s * stage_bytes + lane * box_rows * 128;
        tma_load_3d(kt, &tmK, &full_bar[s], 0, x.in_page, x.pg);
        if (kinds == 2) tma_load_3d(kt + TILE_BYTES, &tmV, &full_bar[s], 0, x.in_page, x.pg);
        if (x.good) {
          const long at = (long)x.pg * ps + x.in_page;
          bulk_load(sc, p.Ks + at, box_rows, &full_bar[s]);
          if (kinds == 2) bulk_load(sc + TK, p.Vs + at, box_rows, &full_bar[s]);
        }
      }
    };
    // A CTA whose tiles all fit into the ring requests them before the wait for the query kernel (see k_dec_attn_umma).
    decu::Walk wn = w, wp = w;                     // the next tile to be looked up, to be requested
    const int ahead = n_tiles <= STAGES ? n_tiles : 0;
    int pg_next = lookup(wn, t_begin);
    auto request = [&](int i, bool wait) -> bool { // tile i; the page of tile i + 1 is on its way
      const int pg = pg_next;
      if (i + 1 < n_tiles) {
        wn.seek(t_begin + i + 1);
        pg_next = lookup(wn, t_begin + i + 1);
      }
      wp.seek(t_begin + i);
      const Box x = box_of(wp, t_begin + i, pg);
      const int s = i % STAGES;
      if (wait && !wait_all(&empty_bar[s], ((i / STAGES) & 1) ^ 1)) return false;
      load_tile(x, s);
      return true;
    };
    int it = 0;
    for (; it < ahead; ++it) (void)request(it, false);
    pdl_enter();
    for (; it < n_tiles; ++it)
      if (!request(it, true)) break;
    if (ab.raised()) mbar_drain_ring(full_bar, it, STAGES);      // the copies in flight end before the CTA does
   } else if (have_work && warp == 1) {
    // ------------------------------- MMA issuer ---------------------------------
    pdl_enter();
    if (elect_one()) {
      const uint32_t idesc_qk = idesc_f8(0, TK, NH);
      const uint32_t idesc_pv = idesc_f8(1, TK, PIECES * NH) | (1u << 15) | (1u << 16);      // both with their M / N index contiguous
      const int ksteps = p.r3 / 32;
      const uint64_t dq0 = umma_desc_kmajor_sw128(smem_u32(qbuf));
      const uint64_t dk0 = umma_desc_kmajor_sw128(smem_u32(ring));
      const uint64_t dv0 = umma_desc_mnmajor_sw128(smem_u32(ring) + (p.shared_kv ? 0u : (uint32_t)TILE_BYTES), TILE_BYTES);
      const uint64_t dp0 = umma_desc_mnmajor_sw128(smem_u32(pbuf), PBUF_BYTES);
      const uint64_t stage_step = (uint64_t)(stage_bytes >> 4);
      uint32_t begun = 0;                          // per warpgroup, 16 bits each: segments in which it has had a tile
      // the two tiles between score issue and value issue: stage << 1 | first of its warpgroup's in the segment
      uint32_t h1 = 0, h2 = 0;
      auto issue_pv = [&](int it, uint32_t code) -> bool {
        const int g = it & 1, st = (int)(code >> 1);
        if (!mbar_wait(&p_full[g], (uint32_t)((it >> 1) & 1), ab)) return false;
        if (code & 1u) {
          const uint32_t n = (begun >> (16 * g)) & 0xffffu;
          // the accumulator of the segment before must have been read
          if (n > 0 && !mbar_wait(&o_read[g], (n - 1) & 1, ab)) return false;
          begun = (begun & ~(0xffffu << (16 * g))) | (((n == 2 ? 1 : n + 1)) << (16 * g));      // 0, then 1 and 2 in turn
        }
        tc_fence_after();
        const uint64_t dv = dv0 + stage_step * (uint64_t)st, dp = dp0 + (uint64_t)(g * (PBUF_BYTES >> 4));
        const uint32_t d = tmem + 64u + (uint32_t)g * 96u;
#pragma unroll
        for (int ks = 0; ks < TK / 32; ++ks)
          umma_f8(d, dv + (uint64_t)(ks * 256), dp + (uint64_t)(ks * 256), idesc_pv, (ks != 0 || !(code & 1u)) ? 1u : 0u);
        umma_commit(&p_free[g]);
        umma_commit(&empty_bar[st]);
        return true;
      };
      int seg = -1, st = 0, seg_it = 0;
      uint32_t st_par = 0, pp = 0;                 // parity of the ring; of each stage's patches
      bool ok = true;
      for (int it = 0; it < n_tiles + 2 && ok; ++it) {
        uint32_t code = 0;
        if (it < n_tiles) {
          const long t = t_begin + it;
          const int g = it & 1;
          w.seek(t);
          if (w.seg_start(t)) {
            ++seg;
            seg_it = it;
            if (!(ok = mbar_wait(&q_full[seg & 1], (uint32_t)((seg >> 1) & 1), ab))) break;
          }
          if (!(ok = mbar_wait(&full_bar[st], st_par, ab))) break;
          if (w.last_tile(t)) {
            mbar_arrive(&wanted);
            if (!(ok = mbar_wait(&patched[st], (pp >> st) & 1u, ab))) break;
            pp ^= 1u << st;
          }
          // the scores of tile it - 2 are in registers
          if (it >= 2 && !(ok = mbar_wait(&s_free[g], (uint32_t)(((it >> 1) - 1) & 1), ab))) break;
          tc_fence_after();
          const uint64_t dk = dk0 + stage_step * (uint64_t)st, dq = dq0 + (uint64_t)((seg & 1) * (QBUF_BYTES >> 4));
          const uint32_t d = tmem + (uint32_t)g * 32u;
#pragma unroll
          for (int pc = 0; pc < PIECES; ++pc)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              if (ks < ksteps)
                umma_f8(d, dk + (uint64_t)(ks * 2), dq + (uint64_t)(pc * (QPIECE_BYTES >> 4) + ks * 2), idesc_qk, (pc | ks) != 0 ? 1u : 0u);
          umma_commit(&s_full[g]);
          if (w.seg_end(t)) umma_commit(&q_empty[seg & 1]);
          code = ((uint32_t)st << 1) | (it - seg_it < 2 ? 1u : 0u);
          if (++st == STAGES) { st = 0; st_par ^= 1u; }
        }
        if (it >= 2) ok = issue_pv(it - 2, h2);
        h2 = h1;
        h1 = code;
      }
    }
   } else if (have_work) {
    // ------------------------------- helpers ------------------------------------
    pdl_enter();
    const int hid = threadIdx.x - 64;
    const int nch = p.r3 / 16;                     // 16-byte chunks of a query's codes
    decu::Walk wq = w;                             // the segment whose queries are split
    int tq = 0, n_q = 0, n_wanted = 0;
    bool ok = true;
    auto split_queries = [&]() -> bool {           // of the segment that starts at tile tq
      const int qb = n_q & 1;
      wq.seek(t_begin + tq);
      const long row0 = (long)wq.b * p.nH;
      const uint4 mx = *reinterpret_cast<const uint4*>(p.qmax + 4 * (long)wq.b);
      const int byte = q8::scale_byte(max(max(mx.x, mx.y), max(mx.z, mx.w)));
      const float inv = q8::inverse(byte);
      if (!wait_all(&q_empty[qb], (uint32_t)(((n_q >> 1) & 1) ^ 1))) return false;
      uint8_t* dst = qbuf + qb * QBUF_BYTES;
      for (int i = hid; i < NH * nch; i += 64) {
        const int h = i / nch, ch = i - h * nch;
        uint4 out[PIECES] = {};
        if (h < p.nH && TA_IDX_OK(p.err, (row0 + h) * p.r3 + ch * 16, 16, (long)p.B * p.nH * p.r3)) {
          const bf16* src = p.qhat + (row0 + h) * p.r3 + ch * 16;
          const bf16* rest = src + (long)p.B * p.nH * p.r3;
          uint4 a[2], b[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            a[e] = reinterpret_cast<const uint4*>(src)[e];
            b[e] = reinterpret_cast<const uint4*>(rest)[e];
          }
          const uint32_t aw[8] = {a[0].x, a[0].y, a[0].z, a[0].w, a[1].x, a[1].y, a[1].z, a[1].w};
          const uint32_t bw[8] = {b[0].x, b[0].y, b[0].z, b[0].w, b[1].x, b[1].y, b[1].z, b[1].w};
          uint32_t* o = reinterpret_cast<uint32_t*>(out);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x0 = (__uint_as_float(aw[e] << 16) + __uint_as_float(bw[e] << 16)) * inv;
            float x1 = (__uint_as_float(aw[e] & 0xffff0000u) + __uint_as_float(bw[e] & 0xffff0000u)) * inv;
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) {
              const uint32_t c = q8::codes2(x0, x1);
              const float2 v = q8::values2(c);
              x0 -= v.x; x1 -= v.y;
              o[pc * 4 + (e >> 1)] |= c << (16 * (e & 1));
            }
          }
        }
#pragma unroll
        for (int pc = 0; pc < PIECES; ++pc) *reinterpret_cast<uint4*>(dst + pc * QPIECE_BYTES + swz(h, ch)) = out[pc];
      }
      if (hid == 0) q_scale[n_q & 7] = q8::scale(byte);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[qb]);
      ++n_q;
      tq = min(n_tiles, (int)(wq.first + wq.nt - t_begin));
      return true;
    };
    ok = split_queries();
    for (int it0 = 0; it0 < n_tiles && ok;) {
      w.seek(t_begin + it0);
      const int it1 = min(n_tiles, (int)(w.first + w.nt - t_begin));      // end of the segment
      if (tq < n_tiles && !(ok = split_queries())) break;
      const long tl = t_begin + it1 - 1;
      if (w.last_tile(tl)) {
        // the tile with the new token: its row, and zeros behind it as values (their weights are zero, but the slots may
        // hold anything)
        const int s = (it1 - 1) % STAGES, row = w.L - w.k0(tl);
        const int kch = p.r3 / 16, vch = p.t3 / 16;
        uint4 nk = make_uint4(0u, 0u, 0u, 0u);     // lanes 0 .. 7 of the warps: chunks of the key, of the value
        if (hid < kch) nk = reinterpret_cast<const uint4*>(p.knew + (long)w.b * p.r3)[hid];
        else if (hid >= 32 && hid - 32 < vch) nk = reinterpret_cast<const uint4*>(p.vnew + (long)w.b * p.t3)[hid - 32];
        const uint8_t ns = lane == 0 ? p.new_scale[2 * (long)w.b + (warp - 2)] : 0;
        // (the issuer's word, not full_bar: these warps do not follow the ring, whose rounds they could not tell apart)
        if (!(ok = wait_all(&wanted, (uint32_t)(n_wanted & 1)))) break;
        ++n_wanted;
        uint8_t* kt = ring + (size_t)s * stage_bytes;
        uint8_t* vt = p.shared_kv ? kt : kt + TILE_BYTES;
        if (hid < kch && !p.shared_kv) *reinterpret_cast<uint4*>(kt + swz(row, hid)) = nk;
        if (hid >= 32 && hid - 32 < vch) *reinterpret_cast<uint4*>(vt + swz(row, hid - 32)) = nk;
        if (lane == 0) scales[s * SCALE_BYTES + (warp - 2) * TK + row] = ns;
        for (int i = (row + 1) * 8 + hid; i < TK * 8; i += 64) *reinterpret_cast<uint4*>(vt + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&patched[s]);
      }
      it0 = it1;
    }
   }
  } else {
   asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
   if (have_work) {
    pdl_enter();
    // ------------------------------- softmax warpgroups --------------------------
    const int g = (warp - 4) / 4;               // tiles g, g + 2, ...
    const int q = warp % 4;                     // TMEM lane quadrant
    const int tid = q * 32 + lane;              // key of a score tile / value coordinate of O^T
    const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
    const uint32_t tm_s = tmem + (uint32_t)g * 32u + lane_addr, tm_o = tmem + 64u + (uint32_t)g * 96u + lane_addr;
    uint8_t* const my_p = pbuf + g * PBUF_BYTES;
    uint32_t wg_phase = 0, pp = 0;              // parity of each stage's patches
    int n_handed[NWG] = {};                     // parts handed over so far by either warpgroup
    bool ok = true, owe = false;                // owe: my part lies in the weights' buffer until it is taken
    auto wg_sync = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(&wg_bar[g]);
      const bool good = mbar_wait(&wg_bar[g], wg_phase & 1, ab);
      ++wg_phase;
      return __all_sync(0xffffffffu, good);
    };
    int seg = 0;
    for (int it0 = 0; it0 < n_tiles && ok; ++seg) {
      w.seek(t_begin + it0);
      const int it1 = min(n_tiles, (int)(w.first + w.nt - t_begin));
      const bool last_seg = w.last_tile(t_begin + it1 - 1);
      const int mine0 = it0 + ((it0 ^ g) & 1);
      float m[NH], l[NH], m_lane = -INFINITY;   // reference of head h; sum of this thread's keys; m[lane]
#pragma unroll
      for (int h = 0; h < NH; ++h) { m[h] = -INFINITY; l[h] = 0.f; }
      int it = mine0;
      for (; it < it1 && ok; it += 2) {
        const int st = it % STAGES, j = it >> 1;
        const bool last = last_seg && it == it1 - 1;
        if (!(ok = wait_all(&s_full[g], (uint32_t)(j & 1)))) break;
        // long complete: for the scale bytes, which other proxies and threads wrote
        if (!(ok = wait_all(&full_bar[st], (uint32_t)((it / STAGES) & 1)))) break;
        if (last && !(ok = wait_all(&patched[st], (pp >> st) & 1u))) break;
        tc_fence_after();
        uint32_t sr[NH];
        tmem_ld32(tm_s, sr);
        const uint8_t* sc = scales + st * SCALE_BYTES + tid;
        const int kb = sc[0], vb = p.shared_kv ? kb : sc[TK];
        float kq = q8::scale(kb) * q_scale[seg & 7], ev = vb == q8::kNan ? NAN : (float)(vb - 127);
        float inv = vb == q8::kNan ? NAN : q8::scale(254 - vb);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[g]);        // the scores of tile it + 2 may overwrite the buffer
        const bool none = last && w.k0(t_begin + it) + tid > w.L;      // keys past the new token do not exist
        if (none) { ev = 0.f; inv = 0.f; }
        float a[NH], over = -INFINITY;                 // log2 of p 2^k'
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          a[h] = none ? -INFINITY : fmaf(__uint_as_float(sr[h]), kq, ev);
          over = fmaxf(over, a[h] - m[h]);
        }
        const bool vote = __any_sync(0xffffffffu, over > kTop);
        if (lane == 0) reinterpret_cast<uint8_t*>(&votes[g][j & 1])[q] = vote ? 1 : 0;
        if (!(ok = wg_sync())) break;
        bool free_seen = false;
        if (*reinterpret_cast<volatile uint32_t*>(&votes[g][j & 1]) != 0u) {
          // ---- new references: the tile's maxima where they are needed ----
          float mine = -INFINITY;
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            const float mx = warp_max(a[h]);
            if (lane == h) mine = mx;
          }
          max_s[g][q][lane] = mine;
          if (!(ok = wg_sync())) break;
          const float mt = fmaxf(fmaxf(max_s[g][0][lane], max_s[g][1][lane]), fmaxf(max_s[g][2][lane], max_s[g][3][lane]));
          const bool need = mt - m_lane > kTop;
          const float m_new = need ? mt - kStart : m_lane;
          const float f_lane = need ? ex2(m_lane - m_new) : 1.f;       // exp2(-inf) = 0 on the first tile
          float f[NH];
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            f[h] = __shfl_sync(0xffffffffu, f_lane, h);
            m[h] = __shfl_sync(0xffffffffu, m_new, h);
            l[h] *= f[h];
          }
          m_lane = m_new;
          if (it > mine0) {
            // the product of the tile before must be complete before its accumulator is rescaled
            if (!(ok = wait_all(&p_free[g], (uint32_t)((j - 1) & 1)))) break;
            free_seen = true;
            tc_fence_after();
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) {
              uint32_t o[NH];
              tmem_ld32(tm_o + pc * NH, o);
              tmem_ld_wait();
#pragma unroll
              for (int h = 0; h < NH; ++h) o[h] = __float_as_uint(__uint_as_float(o[h]) * f[h]);
              tmem_st32(tm_o + pc * NH, o);
            }
            tmem_st_wait();
          }
        }
        // the product of tile it - 2 must have finished reading the weights' buffer, and a part laid down there be taken
        if (it >= 2 && !free_seen && !(ok = wait_all(&p_free[g], (uint32_t)((j - 1) & 1)))) break;
        if (owe) {
          if (!(ok = wait_all(&taken[g], (uint32_t)((n_handed[g] - 1) & 1)))) break;
          owe = false;
        }
        // ---- weights in three bytes; sums ----
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t out[PIECES][4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t hv[2], piece[PIECES][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = half * 16 + u * 4 + e * 2;
              const float w0 = ex2(a[h] - m[h]), w1 = ex2(a[h + 1] - m[h + 1]);
              l[h] = fmaf(w0, inv, l[h]);
              l[h + 1] = fmaf(w1, inv, l[h + 1]);
              const __half2 x = __floats2half2_rn(w0, w1);
              hv[e] = *reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
              for (int pc = 0; pc < PIECES; ++pc) {
                if (pc == PIECES - 1) {
                  piece[pc][e] = hv[e] + 0x00800080u;            // round the last one; all are positive
                } else {
                  piece[pc][e] = hv[e];
                  const uint32_t top = hv[e] & 0xff00ff00u;
                  const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&hv[e]), *reinterpret_cast<const __half2*>(&top));
                  hv[e] = *reinterpret_cast<const uint32_t*>(&rest);
                }
              }
            }
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) out[pc][u] = __byte_perm(piece[pc][0], piece[pc][1], 0x7531);
          }
#pragma unroll
          for (int pc = 0; pc < PIECES; ++pc)
            *reinterpret_cast<uint4*>(my_p + swz(tid, pc * 2 + half)) = make_uint4(out[pc][0], out[pc][1], out[pc][2], out[pc][3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[g]);
      }
      if (!ok) break;
      const int fin = (it1 - 1) & 1;                   // the warpgroup of the last tile finishes the segment
      const bool two = it1 - it0 >= 2;                 // the other one has a part too
      if (mine0 < it1) {
        const int jl = (it - 2) >> 1;
        if (!(ok = wait_all(&p_free[g], (uint32_t)(jl & 1)))) break;     // the product of my last tile is complete
        tc_fence_after();
        float o[NH];
        {
          uint32_t c0[NH], c1[NH];
          tmem_ld32(tm_o, c0);
          tmem_ld32(tm_o + NH, c1);
          tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < NH; ++h) o[h] = __uint_as_float(c0[h]) + __uint_as_float(c1[h]);
          tmem_ld32(tm_o + 2 * NH, c0);
          tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < NH; ++h) o[h] += __uint_as_float(c0[h]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&o_read[g]);        // the next segment may overwrite the accumulator
        sum_s[g][q][lane] = lane_sums(l);
        if (!(ok = wg_sync())) break;
        float l_lane = sum_s[g][0][lane] + sum_s[g][1][lane] + sum_s[g][2][lane] + sum_s[g][3][lane];
        if (g != fin) {
          float* part = reinterpret_cast<float*>(my_p);                // [32][128]
#pragma unroll
          for (int h = 0; h < NH; ++h) part[h * 128 + tid] = o[h];
          if (q == 0) { hand_m[g][lane] = m_lane; hand_l[g][lane] = l_lane; }
          __syncwarp();
          if (lane == 0) mbar_arrive(&handed[g]);
          owe = true;
        } else {
          if (two) {
            const int x = g ^ 1;
            if (!(ok = wait_all(&handed[x], (uint32_t)(n_handed[x] & 1)))) break;
            const float mo = hand_m[x][lane], mn = fmaxf(m_lane, mo);
            const float fm = ex2(m_lane - mn), fo = ex2(mo - mn);
            l_lane = l_lane * fm + hand_l[x][lane] * fo;
            m_lane = mn;
            const float* part = reinterpret_cast<const float*>(pbuf + x * PBUF_BYTES);
#pragma unroll
            for (int h = 0; h < NH; ++h)
              o[h] = o[h] * __shfl_sync(0xffffffffu, fm, h) + part[h * 128 + tid] * __shfl_sync(0xffffffffu, fo, h);
            __syncwarp();
            if (lane == 0) mbar_arrive(&taken[x]);
          }
          if (tid == 0) {
            if (t_begin <= w.first && TA_IDX_OK(p.err, 2 * w.b, 2, 2L * p.B)) p.seq_cta[2 * w.b] = (int)blockIdx.x;
            if (last_seg && TA_IDX_OK(p.err, 2 * w.b, 2, 2L * p.B)) p.seq_cta[2 * w.b + 1] = (int)blockIdx.x;
          }
          const long slot = (long)blockIdx.x + w.b;    // one per (CTA, sequence) pair that can occur
          if (TA_IDX_OK(p.err, slot, 1, (long)gridDim.x + p.B)) {
            if (q == 0) reinterpret_cast<float2*>(p.part_ml)[slot * NH + lane] = make_float2(m_lane, l_lane);
            if (tid < p.t3) {
              float* dst = p.part_o + slot * NH * p.t3 + (long)(tid / 4) * NH * 4 + tid % 4;
#pragma unroll
              for (int h = 0; h < NH; ++h) dst[h * 4] = o[h];
            }
          }
        }
      }
      if (two) ++n_handed[fin ^ 1];
      if (last_seg) pp ^= 1u << ((it1 - 1) % STAGES);
      it0 = it1;
    }
   }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, 256);
}

// The prefix that all sequences share, as the attention kernel of all rows reads it: values of the codes, bf16 (exact), row
// after row; one pool with RoPE: the keys rotated, in two halves (see k_prefix_rotate), and the rows.  A thread per eight
// columns of a row.
__global__ void __launch_bounds__(256) k_prefix_unpack_q8(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale_bytes,
                                                          const int32_t* __restrict__ table, int n_pages, int page_size, bf16* __restrict__ out,
                                                          bf16* __restrict__ rot, long lo, int P, int r, const dec::RopeTurns turns,
                                                          unsigned int* err) {
  pdl_enter();
  const int per = r / 8;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long)P * per) return;
  const int n = (int)(i / per), c = (int)(i % per) * 8;
  const int pg = table[n / page_size];
  float f[8] = {};
  if (pg >= 0 && pg < n_pages) {
    const long row = (long)pg * page_size + n % page_size;
    const float s = q8::scale(scale_bytes[row]);
    q8::values8(*reinterpret_cast<const uint2*>(codes + row * r + c), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= s;
  } else {
    atomicOr(err, (unsigned)TA_DEVERR_BAD_PAGE);
  }
  const long at = (long)n * r + c;
  if (!TA_IDX_OK(err, at, 8, lo)) return;
  uint32_t w[4], wl[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(f[2 * e], f[2 * e + 1]);
  *reinterpret_cast<uint4*>(out + at) = make_uint4(w[0], w[1], w[2], w[3]);
  if (!rot) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 cs = dec::rope_at(n, turns, c / 2 + e);
    const float re = f[2 * e] * cs.x - f[2 * e + 1] * cs.y, ro = f[2 * e] * cs.y + f[2 * e + 1] * cs.x;
    w[e] = pack_bf16(re, ro);
    const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
    wl[e] = pack_bf16(re - v.x, ro - v.y);
  }
  *reinterpret_cast<uint4*>(rot + at) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(rot + lo + at) = make_uint4(wl[0], wl[1], wl[2], wl[3]);
}

}  // namespace decq
}  // namespace ta
