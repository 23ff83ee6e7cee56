// Attention of ALL query rows of a batch (B sequences x n_H heads) to one shared prefix of the latent cache, on
// tcgen05.
//
// Every row attends to the same keys, so the prefix is a plain product pair S = Q K^T, O = P V with M = B n_H rows: the
// cache is read once per 256 rows instead of once per sequence, and the step turns from HBM bound into tensor bound.
//   row block   256 query rows = two tiles of 128, one per softmax warpgroup (thread = row = TMEM lane)
//   unit        (row block, tile of 128 keys); the flat list of units, row block by row block, is divided evenly over
//               one CTA per SM, so any mix of few rows with a long prefix and many rows with a short one fills the GPU.
//               A CTA leaves one partial (max, sum, unnormalised O) per row block it touched, in slot (CTA + row
//               block).
//   warp 0      TMA producer (all lanes: one page box of the tile per lane), ring of K and V tiles in order of need
//   warp 1      TMEM, MMA issue:  S_w = Qhi_w K^T + Qlo_w K^T ;  O_w += P_w V
//   warps 4..7, 8..11   softmax warpgroup w
// TMEM columns: S_0 [0,128) S_1 [128,256) O_0 [256,384) O_1 [384,512).  P_w (bf16) overwrites the first 64 columns of
// S_w: the next scores of the same tile are issued behind the P V product that reads it, in the same thread's order.
// While one warpgroup is in its softmax the tensor core works for the other; P is handed over in two halves, so that P
// V starts while the second half is exponentiated.
// (Both warpgroups on every tile, half a row per thread, was measured: the exchange of the row maxima and the phases in
// which neither of them uses the exponential unit cost more than the shorter hand-over gains, 5050 cycles per unit
// against 4800 here, of which 48 MMAs take 64 each.)
//
// The kernel follows the streaming kernel of the sequences' own keys in the stream but does not depend on it: what it
// reads was complete before that kernel let it be launched.  So its CTAs start as the streaming kernel's leave their
// SMs, and it only waits for that kernel at its end (so that the join, which waits for this kernel, finds both
// complete).
//
// The query is carried as two bf16 halves, as in the paged streaming kernel.  The second half costs a third of the
// tensor time (its eight MMAs per tile next to eight for the first half and eight for P V).
// KLO: so are the keys, which one un-rotated pool with RoPE makes necessary (k_prefix_rotate): rotated keys rounded
// once moved every score by 2^-9 of its size, and scores of a standard deviation of 8 the output by up to 2e-2 of its
// norm.  A unit then has three tiles, K, its rests and V: S_w = Qhi_w K^T + Qlo_w K^T + Qhi_w Klo^T.  At ranks above 64
// the ring just holds one unit, which is enough to go on: the scores of the next one need its two key tiles while V is
// still in use.
// The value tile is used where it lies (MN-major B operand).
// Slots past the prefix in its last page may hold anything: their scores are replaced by -inf, their value rows by
// zeros.
#pragma once

#include "ta_common.cuh"
#include "ta_decode.cuh"
#include "ta_sm100.cuh"

namespace ta {
namespace prefix {

using namespace sm100;

constexpr int TQ = 128, TK = 128;         // rows of a tile, keys of a tile
constexpr int RB = 2 * TQ;                // rows of a block
constexpr int THREADS = 384;
constexpr int SUB_BYTES = 128 * 64 * 2;   // [128 rows x 64 columns] bf16
constexpr int MAX_BUF = 6;
constexpr int TILE_BYTES = 224 * 1024;    // queries and ring
// All shared memory is dynamic, so that its start, and with it the tiles', is 1024-byte aligned (checked) and nothing
// is lost to alignment.
struct Ctl {
  uint64_t q_full, q_empty, kv_full[MAX_BUF], kv_empty[MAX_BUF], s_full[2], p_half[2], p_full[2], o_full[2], o_read[2], patched;
  uint32_t tmem_slot;
  int abort_flag;
};
constexpr size_t SMEM_BYTES = (size_t)TILE_BYTES + sizeof(Ctl);
static_assert(SMEM_BYTES <= 227 * 1024, "one CTA's shared memory");
constexpr float kRescaleThreshold = 8.f;

// Where a tile's rows lie: pages of `page_size` rows listed in `table`, or (table == nullptr) one after another.
struct Rows {
  const int32_t* table;
  int n_pages, page_size;
};

struct Params {
  int R, P, r3, t3;        // query rows, keys of the prefix, ranks
  int n_kt, n_rb;          // key tiles, row blocks
  Rows k, v;
  float* part_o;           // [grid + n_rb][t3 / 4][RB][4]: a warp's rows are adjacent, for its stores and for the reader's heads
  float* part_ml;          // [grid + n_rb][RB][2]   (max in log2 units, sum)
  unsigned int* err;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// The CTA that works on unit t when `total` units are divided over `grid` CTAs (see dec::cta_first_tile).
__device__ __forceinline__ long owner_of(long t, long total, long grid) { return ((t + 1) * grid - 1) / total; }

// KS = r3 / 16: with the number of K steps known the issue of an MMA takes about as long as the MMA; with a test in
// front of each one the issuing thread set the pace (5900 against 5050 cycles per unit of two score tiles).
template <int KS, bool KLO>
__global__ void __launch_bounds__(THREADS, 1)
k_prefix_attn(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
              const __grid_constant__ CUtensorMap tmV, const Params p) {
  constexpr int NT = KLO ? 3 : 2;                          // tiles of a unit in the ring: keys, (their rests,) values
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023u) {                            // never: the tiles' swizzle needs it
    if (threadIdx.x == 0) atomicOr(p.err, (unsigned)TA_DEVERR_BAD_INDEX);
    return;
  }
  Ctl& ctl = *reinterpret_cast<Ctl*>(smem + TILE_BYTES);
  uint64_t &q_full = ctl.q_full, &q_empty = ctl.q_empty, &patched = ctl.patched;
  uint64_t *kv_full = ctl.kv_full, *kv_empty = ctl.kv_empty, *s_full = ctl.s_full, *p_half = ctl.p_half, *p_full = ctl.p_full,
           *o_full = ctl.o_full, *o_read = ctl.o_read;
  const int ksub = (p.r3 + 63) / 64, vsub = (p.t3 + 63) / 64;
  const int q_tile = 2 * ksub * SUB_BYTES;                 // one tile's rows: first halves, second halves
  uint8_t* ring = smem + 2 * q_tile;
  const int buf_bytes = max(ksub, vsub) * SUB_BYTES;
  const int n_buf = min(MAX_BUF, (TILE_BYTES - 2 * q_tile) / buf_bytes);     // 3 at ranks above 64
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Abort ab{&ctl.abort_flag, p.err};

  if (threadIdx.x == 0) {
    ctl.abort_flag = 0;
    mbar_init(&q_full, 1);
    mbar_init(&q_empty, 1);
    for (int i = 0; i < MAX_BUF; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_half[i], 4);         // the first 64 keys' P is in TMEM: one arrival per warp of the group
      mbar_init(&p_full[i], 4);         // all of it
      mbar_init(&o_full[i], 1);         // the P V product is complete
      mbar_init(&o_read[i], 4);         // the accumulator of a finished segment has been read
    }
    mbar_init(&patched, 4);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&ctl.tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem_slot;

  const long total = (long)p.n_rb * p.n_kt;
  const long u_begin = dec::cta_first_tile(blockIdx.x, total, gridDim.x);
  const long u_end = dec::cta_first_tile(blockIdx.x + 1, total, gridDim.x);
  const bool ragged = p.P % TK != 0;                       // the last key tile is not full

  if (warp < 4) {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
   if (warp == 0) {
    // ------------------------------- TMA producer -------------------------------
    if (elect_one()) { tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV); }
    __syncwarp();
    // page of box `lane` of key tile kt; -1 where this lane has none
    auto lookup = [&](const Rows& r, int kt) -> int {
      const int rows = min(r.page_size, TK), row = kt * TK + lane * rows;
      if (lane * rows >= TK || row >= p.P) return -1;
      return r.table ? r.table[row / r.page_size] : row / r.page_size;
    };
    int kt = (int)(u_begin % p.n_kt);
    int pk_next = lookup(p.k, kt), pv_next = lookup(p.v, kt);      // the tables are inputs of the call
    int n = 0, seg = 0;                                            // ring buffers filled so far, segments
    bool ok = true;
    auto load = [&](const Rows& r, const CUtensorMap* tm, int kt_, int pg, int nsub) -> bool {
      const int rows = min(r.page_size, TK), row = kt_ * TK + lane * rows;
      const bool mine = lane * rows < TK && row < p.P;
      if (mine && (pg < 0 || pg >= r.n_pages)) {
        atomicOr(p.err, (unsigned)TA_DEVERR_BAD_PAGE);
        pg = r.n_pages;                                            // outside the tensor: filled with zeros
      }
      const int s = n % n_buf;
      if (!__all_sync(0xffffffffu, mbar_wait(&kv_empty[s], ((n / n_buf) & 1) ^ 1, ab))) return false;
      const uint32_t n_mine = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine));
      if (lane == 0) mbar_expect_tx(&kv_full[s], n_mine * (uint32_t)(nsub * rows * 128));
      __syncwarp();
      if (mine)
        for (int kk = 0; kk < nsub; ++kk)
          tma_load_3d(ring + (size_t)s * buf_bytes + kk * SUB_BYTES + lane * rows * 128, tm, &kv_full[s], kk * 64, row % r.page_size, pg);
      ++n;
      return true;
    };
    for (long u = u_begin; u < u_end && ok; ++u) {
      const int rb = (int)(u / p.n_kt);
      kt = (int)(u - (long)rb * p.n_kt);
      if (u == u_begin || kt == 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(&q_empty, (seg & 1) ^ 1, ab));
        if (!ok) break;
        const int nw = (p.R - rb * RB) > TQ ? 2 : 1;
        if (lane == 0) {
          mbar_expect_tx(&q_full, (uint32_t)(nw * q_tile));
          for (int w = 0; w < nw; ++w)
            for (int kk = 0; kk < 2 * ksub; ++kk)                  // the second halves lie R rows behind the first
              tma_load_2d(smem + w * q_tile + kk * SUB_BYTES, &tmQ, &q_full, (kk % ksub) * 64, rb * RB + w * TQ + (kk < ksub ? 0 : p.R));
        }
        ++seg;
      }
      const int pk = pk_next, pv = pv_next;
      if (u + 1 < u_end) {
        const int nx = kt + 1 < p.n_kt ? kt + 1 : 0;
        pk_next = lookup(p.k, nx);
        pv_next = lookup(p.v, nx);
      }
      ok = load(p.k, &tmK, kt, pk, ksub);
      if (KLO) ok = ok && load(p.k, &tmK, kt, pk + p.n_kt, ksub);  // the rests lie n_kt tiles behind
      ok = ok && load(p.v, &tmV, kt, pv, vsub);
    }
    if (!ok) {                                                     // aborted: the copies in flight end before the CTA does
      mbar_drain_ring(kv_full, n, n_buf);
      mbar_drain_ring(&q_full, seg, 1);
    }
   } else if (warp == 1) {
    // ------------------------------- MMA issuer ---------------------------------
    if (elect_one()) {
      const uint32_t idesc_qk = umma_idesc_bf16(TQ, TK);
      const uint32_t idesc_pv = umma_idesc_bf16(TQ, (uint32_t)p.t3) | (1u << 16);     // B = V tile, MN-major
      const uint64_t dq0 = umma_desc_kmajor_sw128(smem_u32(smem));
      const uint64_t dk0 = umma_desc_kmajor_sw128(smem_u32(ring));
      const uint64_t dv0 = umma_desc_mnmajor_sw128(smem_u32(ring), SUB_BYTES);
      auto issue_qk = [&](int w, int s, int sl) {            // ring buffers of the keys and of their rests
        const uint64_t dk = dk0 + (uint64_t)(s * (buf_bytes >> 4));
        const uint64_t dq = dq0 + (uint64_t)((w * q_tile) >> 4), dl = dq + (uint64_t)((ksub * SUB_BYTES) >> 4);
        const uint32_t d = tmem + (uint32_t)w * 128u;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint64_t o = (uint64_t)((ks >> 2) * (SUB_BYTES >> 4) + (ks & 3) * 2);
          umma_ss(d, dq + o, dk + o, idesc_qk, ks != 0 ? 1u : 0u);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint64_t o = (uint64_t)((ks >> 2) * (SUB_BYTES >> 4) + (ks & 3) * 2);
          umma_ss(d, dl + o, dk + o, idesc_qk, 1u);
        }
        if constexpr (KLO) {
          const uint64_t dkl = dk0 + (uint64_t)(sl * (buf_bytes >> 4));
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const uint64_t o = (uint64_t)((ks >> 2) * (SUB_BYTES >> 4) + (ks & 3) * 2);
            umma_ss(d, dq + o, dkl + o, idesc_qk, 1u);
          }
        }
        umma_commit(&s_full[w]);
      };
      int n = 0;                          // ring buffers consumed so far
      uint32_t pf = 0, od = 0, begun = 0; // per warpgroup, a bit each: parity of p_full, of o_read, any segment before
      int seg = 0, n_patch = 0;
      bool ok = true;
      for (long u = u_begin; u < u_end && ok;) {
        const int rb = (int)(u / p.n_kt), kt0 = (int)(u - (long)rb * p.n_kt);
        const int nt = (int)min((long)(p.n_kt - kt0), u_end - u);
        const int nw = (p.R - rb * RB) > TQ ? 2 : 1;
        if (!(ok = mbar_wait(&q_full, (uint32_t)(seg & 1), ab))) break;
        // the keys in buffer n and, KLO, their rests in buffer n + 1 have arrived / are used no more
        auto keys_full = [&]() -> bool {
          return mbar_wait(&kv_full[n % n_buf], (uint32_t)((n / n_buf) & 1), ab) &&
                 (!KLO || mbar_wait(&kv_full[(n + 1) % n_buf], (uint32_t)(((n + 1) / n_buf) & 1), ab));
        };
        auto keys_done = [&]() {
          umma_commit(&kv_empty[n % n_buf]);
          if (KLO) umma_commit(&kv_empty[(n + 1) % n_buf]);
          n += NT - 1;
        };
        if (!(ok = keys_full())) break;
        tc_fence_after();
        for (int w = 0; w < nw; ++w) issue_qk(w, n % n_buf, (n + 1) % n_buf);
        keys_done();
        if (nt == 1) umma_commit(&q_empty);
        for (int i = 0; i < nt && ok; ++i) {
          const int sv = n % n_buf;
          if (!(ok = mbar_wait(&kv_full[sv], (uint32_t)((n / n_buf) & 1), ab))) break;
          ++n;
          if (ragged && kt0 + i == p.n_kt - 1) {
            if (!(ok = mbar_wait(&patched, (uint32_t)(n_patch & 1), ab))) break;
            ++n_patch;
          }
          for (int w = 0; w < nw && ok; ++w) {
            if (!(ok = mbar_wait_poll(&p_half[w], (pf >> w) & 1u, ab))) break;
            if (i == 0) {                 // the accumulator of the group's previous segment must have been read
              if ((begun >> w) & 1u) {
                if (!(ok = mbar_wait(&o_read[w], (od >> w) & 1u, ab))) break;
                od ^= 1u << w;
              }
              begun |= 1u << w;
            }
            tc_fence_after();
            const uint64_t dv = dv0 + (uint64_t)(sv * (buf_bytes >> 4));
            const uint32_t a = tmem + (uint32_t)w * 128u, d = tmem + 256u + (uint32_t)w * 128u;
            // the product starts with the keys whose P is there while the group still works on the others
#pragma unroll
            for (int ks = 0; ks < TK / 32; ++ks)
              umma_ts(d, a + (uint32_t)ks * 8u, dv + (uint64_t)(ks * 128), idesc_pv, (i | ks) != 0 ? 1u : 0u);
            if (!(ok = mbar_wait_poll(&p_full[w], (pf >> w) & 1u, ab))) break;
            pf ^= 1u << w;
            tc_fence_after();
#pragma unroll
            for (int ks = TK / 32; ks < TK / 16; ++ks)
              umma_ts(d, a + (uint32_t)ks * 8u, dv + (uint64_t)(ks * 128), idesc_pv, 1u);
            umma_commit(&o_full[w]);
            if (i + 1 < nt) {
              if (w == 0 && !(ok = keys_full())) break;
              issue_qk(w, n % n_buf, (n + 1) % n_buf);
            }
          }
          if (!ok) break;
          umma_commit(&kv_empty[sv]);
          if (i + 1 < nt) {
            keys_done();
            if (i + 2 == nt) umma_commit(&q_empty);        // the segment's last scores are issued
          }
        }
        ++seg;
        u += nt;
      }
    }
   }
  } else {
   // launched with 168 registers x 384 threads = 64512 = 128 x 72 + 256 x 216
   asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
   // ------------------------------- softmax warpgroups --------------------------
   const int w = (warp - 4) / 4, q = warp % 4, rloc = q * 32 + lane;
   const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
   const uint32_t tm_s = tmem + (uint32_t)w * 128u + lane_addr, tm_o = tmem + 256u + (uint32_t)w * 128u + lane_addr;
   auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {
     const bool good = mbar_wait(bar, parity, ab);
     return __all_sync(0xffffffffu, good);
   };
   int jt = 0;                            // tiles of this group so far
   int n = 0;                             // ring buffers of the segments before this one
   bool ok = true;
   for (long u = u_begin; u < u_end && ok;) {
     const int rb = (int)(u / p.n_kt), kt0 = (int)(u - (long)rb * p.n_kt);
     const int nt = (int)min((long)(p.n_kt - kt0), u_end - u);
     const int row = rb * RB + w * TQ + rloc;
     const bool present = (p.R - rb * RB) > w * TQ;        // uniform in the group
     float m_used = -INFINITY, l = 0.f;
     for (int i = 0; present && i < nt && ok; ++i, ++jt) {
       const int k0 = (kt0 + i) * TK;
       const bool last = ragged && k0 + TK > p.P;
       if (last && w == 0) {
         // value rows past the prefix must not be trusted: zeros (a zero row is zero in any swizzle)
         // (KLO: the tile before it in its buffer may be the previous unit's values, which nothing here has waited for
         // yet; until they have come, their buffer's barrier shows the parity that is waited for next)
         if (KLO && i > 0 && !(ok = wait_all(&o_full[w], (uint32_t)((jt - 1) & 1)))) break;
         const int nv = n + NT * i + NT - 1, s = nv % n_buf;
         if (!(ok = wait_all(&kv_full[s], (uint32_t)((nv / n_buf) & 1)))) break;
         if (k0 + rloc >= p.P)
           for (int kk = 0; kk < vsub; ++kk)
#pragma unroll
             for (int c = 0; c < 8; ++c)
               *reinterpret_cast<uint4*>(ring + (size_t)s * buf_bytes + kk * SUB_BYTES + rloc * 128 + c * 16) = make_uint4(0u, 0u, 0u, 0u);
         fence_proxy_async_smem();
         __syncwarp();
         if (lane == 0) mbar_arrive(&patched);
       }
       if (!(ok = wait_all(&s_full[w], (uint32_t)(jt & 1)))) break;
       tc_fence_after();
       uint32_t sr[128];
       {
         uint32_t (*c)[32] = reinterpret_cast<uint32_t (*)[32]>(sr);
         tmem_ld32(tm_s + 0, c[0]);
         tmem_ld32(tm_s + 32, c[1]);
         tmem_ld32(tm_s + 64, c[2]);
         tmem_ld32(tm_s + 96, c[3]);
         tmem_ld_wait();
       }
       if (last) {
#pragma unroll
         for (int c = 0; c < 128; ++c)
           if (k0 + c >= p.P) sr[c] = 0xff800000u;          // -inf
       }
       float mt;
       {
         float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
         for (int c = 0; c < 128; c += 8) {
           m0 = max3(m0, __uint_as_float(sr[c]), __uint_as_float(sr[c + 1]));
           m1 = max3(m1, __uint_as_float(sr[c + 2]), __uint_as_float(sr[c + 3]));
           m2 = max3(m2, __uint_as_float(sr[c + 4]), __uint_as_float(sr[c + 5]));
           m3 = max3(m3, __uint_as_float(sr[c + 6]), __uint_as_float(sr[c + 7]));
         }
         mt = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
       }
       // the reference maximum only moves when it would grow by more than a factor of 256: the accumulator is rescaled
       // rarely
       const bool need = mt > m_used + kRescaleThreshold;   // every tile holds a key: mt > -inf, and the first tile needs
       if (__any_sync(0xffffffffu, need)) {
         const float m_new = need ? mt : m_used;
         const float f = need ? dec::ex2(m_used - m_new) : 1.f;
         if (i > 0) {
           if (!(ok = wait_all(&o_full[w], (uint32_t)((jt - 1) & 1)))) break;
           tc_fence_after();
           for (int ch = 0; ch < p.t3 / 32; ++ch) {
             uint32_t o[32];
             tmem_ld32(tm_o + ch * 32, o);
             tmem_ld_wait();
#pragma unroll
             for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
             tmem_st32(tm_o + ch * 32, o);
           }
         }
         l *= f;
         m_used = m_new;
       }
       const float2 negm = make_float2(-m_used, -m_used);
       float2 rs[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
       for (int half = 0; half < 2; ++half) {
#pragma unroll
         for (int c = half * 32; c < half * 32 + 32; ++c) {
           const float2 x = __fadd2_rn(make_float2(__uint_as_float(sr[2 * c]), __uint_as_float(sr[2 * c + 1])), negm);
           const float2 e = make_float2(dec::ex2(x.x), dec::ex2(x.y));
           rs[c & 3] = __fadd2_rn(rs[c & 3], e);
           sr[c] = pack_bf16(e.x, e.y);
         }
         tmem_st32(tm_s + half * 32, reinterpret_cast<uint32_t (*)[32]>(sr)[half]);
         tmem_st_wait();
         tc_fence_before();
         __syncwarp();
         if (lane == 0) mbar_arrive(half ? &p_full[w] : &p_half[w]);
       }
       // (the sum of the exponentials before their rounding to bf16; of the rounded ones, as the streaming kernel takes
       // it, rows under growing scores were off by 1.7e-3 instead of 1.8e-3 in the median, 2.3e-3 instead of 3.1e-3 at
       // most, and the 64-sequence document step took 92.0 instead of 91.0 us: not kept)
       const float2 r01 = __fadd2_rn(rs[0], rs[1]), r23 = __fadd2_rn(rs[2], rs[3]);
       l += (r01.x + r01.y) + (r23.x + r23.y);
     }
     if (!ok) break;
     if (present) {
       if (!(ok = wait_all(&o_full[w], (uint32_t)((jt - 1) & 1)))) break;
       tc_fence_after();
       const long slot = (long)blockIdx.x + rb;
       const bool slot_ok = row < p.R && TA_IDX_OK(p.err, slot, 1, (long)gridDim.x + p.n_rb);
       float4* dst = reinterpret_cast<float4*>(p.part_o) + slot * RB * (p.t3 / 4) + w * TQ + rloc;
       for (int ch = 0; ch < p.t3 / 32; ++ch) {
         uint32_t o[32];
         tmem_ld32(tm_o + ch * 32, o);
         tmem_ld_wait();
         if (slot_ok)
#pragma unroll
           for (int c = 0; c < 8; ++c)
             dst[(long)(ch * 8 + c) * RB] = make_float4(__uint_as_float(o[4 * c]), __uint_as_float(o[4 * c + 1]), __uint_as_float(o[4 * c + 2]),
                                                        __uint_as_float(o[4 * c + 3]));
       }
       tc_fence_before();
       __syncwarp();
       if (lane == 0) mbar_arrive(&o_read[w]);               // the next segment may overwrite the accumulator
       if (slot_ok) *reinterpret_cast<float2*>(p.part_ml + (slot * RB + w * TQ + rloc) * 2) = make_float2(m_used, l);
     }
     n += NT * nt;
     u += nt;
   }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, 512);
  pdl_enter();
}

// One pool with latent RoPE holds un-rotated rows: the prefix's keys, rotated at positions 0 .. P - 1 and laid one
// after another, for the call's attention kernel: bf16 [P, r3], and `lo` elements behind it the rounded rests.  A
// thread per 8 columns of a row.
__global__ void __launch_bounds__(256) k_prefix_rotate(const bf16* __restrict__ pool, const Rows rows, bf16* __restrict__ out, long lo,
                                                       int P, int r3, const dec::RopeTurns turns, unsigned int* err) {
  pdl_enter();
  const int per = r3 / 8;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long)P * per) return;
  const int n = (int)(i / per), c = (int)(i % per) * 8;
  const int pg = rows.table[n / rows.page_size];
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (pg >= 0 && pg < rows.n_pages) v = *reinterpret_cast<const uint4*>(pool + ((long)pg * rows.page_size + n % rows.page_size) * r3 + c);
  else atomicOr(err, (unsigned)TA_DEVERR_BAD_PAGE);
  uint32_t wv[4] = {v.x, v.y, v.z, v.w}, wl[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[e]));
    const float2 cs = dec::rope_at(n, turns, c / 2 + e);
    const float re = x.x * cs.x - x.y * cs.y, ro = x.x * cs.y + x.y * cs.x;
    wv[e] = pack_bf16(re, ro);
    const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[e]));
    wl[e] = pack_bf16(re - f.x, ro - f.y);
  }
  const long at = (long)n * r3 + c;
  if (TA_IDX_OK(err, at, 8, lo)) {
    *reinterpret_cast<uint4*>(out + at) = make_uint4(wv[0], wv[1], wv[2], wv[3]);
    *reinterpret_cast<uint4*>(out + lo + at) = make_uint4(wl[0], wl[1], wl[2], wl[3]);
  }
}

}  // namespace prefix
}  // namespace ta
