// Decode attention over a paged latent cache held in 8 bits (Eq. 9) on tcgen05 tensor cores.
//
// The bytes of the cache bound the step, and there are half as many as in bf16: a tile of 128 keys, 32 KB of codes, is due
// every 1450 cycles per SM at the copy rate, where the bf16 kernel's tile has 2900.  So the codes are never converted: the
// tiles go to the tensor cores as TMA wrote them (kind::f8f6f4), and everything else is arranged around that.
//
//   S^T [128 keys x 32 heads] = K_codes * q^T      The query is carried as three e4m3 numbers per coordinate (the rounded
//       value, the rounded rest, the rest's rounded rest: 2^-12 of it together), 96 columns of one product that are added up
//       when they are read (as three products into one accumulator the key tile was read three times: at N = 32 an
//       instruction takes the 40 cycles of its 4 KB of A from shared memory, and the tensor core was the limit).  Its own scale
//       is a power of two per sequence.  Two numbers (2^-8) would move scores of a standard deviation of 2 by what the
//       rounding of y to bf16 moves the output.  (It is how much the scores differ that counts: what the rounding adds to a part
//       that all keys share is the same for all.  1000 nats of it: y 1.6e-3 off, as without.)
//   p 2^k' [128 keys x 32 heads]                   A thread owns a key, so the row's scales are two numbers of its own: 2^k
//       multiplies the scores, 2^k' the weight of the value row, as a term of the exponent.  The sums are of p alone.
//   O^T [t3 x 32 heads] += V_codes^T * (p 2^k')    The weight is carried as three e5m2 numbers: the upper byte of an f16, the
//       upper byte of 8 times what is left, and of 8 times what is left then, rounded (2^-10 together; a byte's worth of an f16
//       is an e5m2, so this is masking and exact subtraction).  The three are 96 columns of one product and of the accumulator,
//       and are added up once per segment.  With a head's largest weight at 2^4 .. 2^15, all are held to 2^-27 of the largest.
//       (Without the factors, for which their columns have room, to 2^-21: 12000 equal weights behind one of e^14 times theirs
//       came out 6% off; the factors cost 1 us of 109.)
//
// Everything goes by steps of 256 keys.  The two softmax warpgroups take a half each, with scores, weights, running maxima, sums
// and an accumulator of its own (TMEM has room for two of each here; the bf16 kernel's warpgroups share every tile's heads and
// its accumulator).  What the threads of one have to agree on is one vote per step: whether any score lies more than 2^kTop
// above its head's reference.  Half of the weights are formed while it is counted.  At the first step of a segment and seldom
// after (64 ragged sequences of random rows: 2 to 9 of a CTA's 35 steps, 2000 cycles each; with
// kStart = 8 the step takes 119 us instead of 109), the maxima are taken and the accumulator rescaled where a reference moved.
// At the end of a (CTA, sequence) segment warpgroup 1 hands its part to warpgroup 0 through its weights' buffer.
// 64 ragged sequences to 32768 tokens (1.3 million keys, 347 MB: 54 us at the copy rate): 90 us.  A CTA's 35 steps take 2600
// to 3000 cycles each, what the bytes and the softmax warps' chains (2100) need, and about 25 thousand cycles go to the
// division of the work, the first pass over cold code and the last segment's end.  What was tried: references and sums in
// registers with everything of a step formed at once (300 bytes of spills, 126 us); four softmax warpgroups of 16 heads
// (113); a pass over the loop before the queries are there, for the code (109); all scores loaded at once, or the accumulator
// rescaled behind the weights instead of in front of them (both 110, with spills).
//
//   warp 0       TMA producer of keys and values
//   warp 1       TMEM allocation, MMA issue of the scores, a step ahead of the values
//   warp 2       MMA issue of the values; scale bytes
//   warp 3       splits the next segment's queries (the first's: warps 4 ..); puts the new token's row into the tile that holds it
//   warps 4 + 4 g .. 7 + 4 g   softmax warpgroup g: keys 128 g .. 128 g + 127 of a step
// A warp that works alone gets through about a hundred instructions in a thousand cycles, waits and issues among them, and a
// step of 128 keys was too short for that: with the warpgroups on alternate tiles of 128 keys one warp or another of the
// first four set the pace (110 to 94 us for 1.3 million keys, whatever was moved from one to another; six of them instead of
// four took the softmax warps' issue slots and registers, 108 us).
// TMEM columns: S_0 [0, 96), S_1 [96, 192), O_0 [192, 288), O_1 [288, 384).
// Every wait is bounded (Abort).
#pragma once

#include "ta_common.cuh"
#include "ta_decode.cuh"
#include "ta_decode_umma.cuh"
#include "ta_prefix_attn.cuh"
#include "ta_q8.cuh"
#include "ta_sm100.cuh"

#include <cuda_fp16.h>
#include <limits.h>

namespace ta {
namespace decq {

using namespace sm100;
using decu::ex2;
using prefix::max3;

constexpr int TK = 128, SK = 2 * TK;             // keys of a warpgroup, of a step
constexpr int NWG = 2, THREADS = 128 + 128 * NWG;
constexpr int NH = 32;                           // head columns
constexpr int STEP_BYTES = SK * 128;             // rows of 128 bytes, the last of them zeros where a rank is smaller
// Keys and values in rings of their own: keys are done with when their scores are, values a softmax later.
constexpr int K_STAGES = 2, V_STAGES = 3;
constexpr int MAX_STAGES = K_STAGES + V_STAGES;  // of one shared pool, whose rows are both
constexpr int RING_BYTES = MAX_STAGES * STEP_BYTES;
constexpr int PIECES = 3, PC = PIECES * NH;      // columns of a product
constexpr uint32_t TMEM_COLS = 512, TMEM_O = NWG * PC;
constexpr int QPIECE_BYTES = NH * 128, QBUF_BYTES = PIECES * QPIECE_BYTES;
constexpr int PBUF_BYTES = TK * 128;             // a key's 96 weights in a row of 128 bytes
constexpr int S_SLOTS = 4, S_AHEAD = 3;          // steps whose scale bytes have a place (a power of two), how far they run ahead
// rings | queries of two segments | weights of two warpgroups | scales
constexpr size_t SMEM_BYTES = 1024 + (size_t)RING_BYTES + 2 * QBUF_BYTES + 2 * PBUF_BYTES + S_SLOTS * 2 * SK;
static_assert(SMEM_BYTES <= 224 * 1024, "one CTA's shared memory, with the static part");
// Weights reach 2^kTop at most; the largest is 2^(kStart - 1) to 2^(kStart + 1) when a reference is set, from a maximum of kFine at most.
constexpr float kTop = 15.f, kStart = 5.f, kFine = 256.f;
// What references are set by is this much less for a row of zeros: below any other row's (scales are 2^-96 and more), and no more
// than leaves its weights, 2^(kTop + kZeroRow) at most, in fp32.  The sums are in units of 2^kSumUnit, so that a million such weights
// fit.  Upwards there is room for scales of 2^87: then 2^-24 of the largest weight is 2^-126 of the sum's unit.
constexpr float kZeroRow = 108.f;
constexpr int kSumUnit = 20;
constexpr float kRestUp = 8.f;                  // what a piece leaves of a weight is below 2^(kTop - 3)

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
// 16-byte chunk of a row of 128 bytes, 128-byte swizzle
__device__ __forceinline__ uint32_t swz(int row, int chunk) { return (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); }

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// pairs of fp32 numbers
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ uint64_t pairu(uint32_t lo, uint32_t hi) { return pack2(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// Scale bytes of rows that no page holds: they are rows of zeros, with any scale but NaN.
__device__ __align__(16) const uint8_t g_ones[16] = {127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127};

// This CTA's steps [0, n), sequence by sequence: a segment is its part of one.
struct Segments {
  const int32_t* cache_len;
  int Lmax, n;
  int b, L, it0, it1, k0;      // sequence, its cached rows; steps [it0, it1); first key
  bool head, tail;             // the sequence begins / ends (with the new token, key L) in it
  __device__ void init(const Params& p, long t_begin, int n_, int b0, long first) {
    cache_len = p.cache_len; Lmax = p.Lmax; n = n_;
    b = b0;
    L = dec::clamp_len(cache_len[b], Lmax);
    const int done = (int)(t_begin - first), left = dec::tiles_of<SK>(L) - done;
    it0 = 0; it1 = min(n, left);
    k0 = done * SK;
    head = done == 0; tail = left <= n;
  }
  __device__ bool more() const { return it0 < n; }
  __device__ void next() {
    it0 = it1;
    if (it0 >= n) return;
    ++b;
    L = dec::clamp_len(cache_len[b], Lmax);
    const int nt = dec::tiles_of<SK>(L);
    it1 = min(n, it0 + nt);
    k0 = 0;
    head = true; tail = it0 + nt <= n;
  }
  // whether warpgroup 1 has any of the keys of step it
  __device__ bool both(int it) const { return k0 + (it - it0) * SK + TK <= L; }
};

// Page entries of a CTA's steps in turn: lane i has box i (a page, or 128 rows of one) of a step.  Without divisions in the loop,
// which is one warp's chain of instructions.
struct Place { int pg, in_page, rows; };         // entry, first row in the page, whether the box has cached rows
struct Lookup {
  Segments g;
  const int32_t* entry;                          // this lane's of the next step
  int it, rows_left, in_page, my_row, page0, in0, L_next;
  __device__ void init(const Params& p, const Segments& s, int lane) {
    g = s;
    it = 0;
    const int ps = p.pv.page_size, box_rows = min(ps, TK), n_box = SK / box_rows, off = lane * box_rows;
    my_row = lane < n_box ? off : INT_MAX;
    page0 = off / ps; in0 = off % ps;
    rows_left = g.L - g.k0;
    in_page = (g.k0 + off) % ps;
    entry = p.pv.table + (long)g.b * p.pv.max_pages + (g.k0 + off) / ps;
  }
  __device__ Place next(const Params& p) {
    Place x{-1, in_page, 0};
    if (it < g.n) {
      if (my_row < rows_left) {
        x.rows = 1;
        x.pg = *entry;
      }
      if (++it == g.it1) {
        g.next();
        rows_left = g.L;
        in_page = in0;
        entry = p.pv.table + (long)g.b * p.pv.max_pages + page0;
      } else {
        const int ps = p.pv.page_size;
        rows_left -= SK;
        in_page += SK;
        if (ps <= TK) { in_page -= SK; entry += SK >> (31 - __clz(ps)); }
        else if (in_page >= ps) { in_page -= ps; ++entry; }      // a larger page size is a multiple of 128, at least 256
      }
    }
    return x;
  }
};

// Scale byte of a sequence's queries
__device__ __forceinline__ int query_byte(const Params& p, int b) {
  const uint4 mx = *reinterpret_cast<const uint4*>(p.qmax + 4 * (long)b);
  return q8::scale_byte(max(max(mx.x, mx.y), max(mx.z, mx.w)));
}
// Sixteen coordinates (chunk item % 8 of the row) of head item / 8 in three pieces, zeros where there is no head or coordinate
__device__ __forceinline__ void split_query(const Params& p, int b, int item, float inv, uint8_t* dst) {
  const int h = item >> 3, ch = item & 7;
  const long at = ((long)b * p.nH + h) * p.r3 + ch * 16, half = (long)p.B * p.nH * p.r3;
  uint4 out[PIECES] = {};
  if (h < p.nH && ch * 16 < p.r3 && TA_IDX_OK(p.err, at, 16, half)) {
    uint4 a[2], b4[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      a[e] = reinterpret_cast<const uint4*>(p.qhat + at)[e];
      b4[e] = reinterpret_cast<const uint4*>(p.qhat + half + at)[e];
    }
    const uint32_t aw[8] = {a[0].x, a[0].y, a[0].z, a[0].w, a[1].x, a[1].y, a[1].z, a[1].w};
    const uint32_t bw[8] = {b4[0].x, b4[0].y, b4[0].z, b4[0].w, b4[1].x, b4[1].y, b4[1].z, b4[1].w};
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

__global__ void __launch_bounds__(THREADS, 1)
k_dec_attn_q8(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t kfull[K_STAGES], kempty[K_STAGES], vfull[MAX_STAGES], vempty[MAX_STAGES], sfull[S_SLOTS], q_full[2], q_empty[2];
  __shared__ uint64_t s_full[NWG], s_free[NWG], p_full[NWG], p_free[NWG], o_read[NWG], wg_bar[NWG], handed, taken, wanted, patched, q_first;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float q_scale[8];                   // of segment i at i & 7: the queries are split at most three segments ahead
  __shared__ uint32_t votes[NWG][2];             // a byte per warp, by parity of the step
  __shared__ float max_s[NWG][4][NH], sum_s[NWG][4][NH], hand_m[NH], hand_l[NH], hand_f[NH];
  __shared__ __align__(16) float up_s[NWG][4][NH], neg_s[NWG][4][NH];      // a warp's own: minus the references, minus their rise
  __shared__ long long wtot_s[THREADS / 32];
  __shared__ int loc_b;
  __shared__ long long loc_first;

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const ring = smem_raw + (base - smem_u32(smem_raw));
  uint8_t* const qbuf = ring + RING_BYTES;
  uint8_t* const pbuf = qbuf + 2 * QBUF_BYTES;
  uint8_t* const scales = pbuf + 2 * PBUF_BYTES;
  const bool shared = p.shared_kv;
  const int VS = shared ? MAX_STAGES : V_STAGES;
  uint8_t* const vring = ring + (shared ? 0 : K_STAGES * STEP_BYTES);      // one shared pool: no ring of keys
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Abort ab{&abort_flag, p.err};

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(&vfull[s], 1);
      mbar_init(&vempty[s], 1);
    }
    for (int s = 0; s < K_STAGES; ++s) {
      mbar_init(&kfull[s], 1);
      mbar_init(&kempty[s], 1);
    }
    for (int s = 0; s < S_SLOTS; ++s) mbar_init(&sfull[s], 32);      // one arrival per copying lane, when its bytes are there
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1);
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], 4);           // the scores are in registers
      mbar_init(&p_full[i], 4);           // the weights are in shared memory
      mbar_init(&p_free[i], 1);           // the product that read them is complete
      mbar_init(&o_read[i], 4);           // the accumulator of a finished segment has been read
      mbar_init(&wg_bar[i], 4);
    }
    mbar_init(&handed, 4);                // warpgroup 1 has laid its part of a segment down ...
    mbar_init(&taken, 4);                 // ... and warpgroup 0 has picked it up
    mbar_init(&wanted, 1);                // the next step with a new token's row has arrived ...
    mbar_init(&patched, 1);               // ... and the row is in its place
    mbar_init(&q_first, 4 * NWG);         // the first segment's queries
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(&tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // ---- this CTA's range of the flat list of steps (see k_dec_attn_umma) ----
  int lo, hi;
  long excl;
  const long total = dec::block_tile_scan<SK>(p.cache_len, p.B, p.Lmax, lo, hi, excl, wtot_s);
  const long parts = min((long)gridDim.x, total);
  const long t_begin = min(dec::cta_first_tile(blockIdx.x, total, parts), total);
  const long t_end = min(dec::cta_first_tile(blockIdx.x + 1, total, parts), total);
  {
    long f = excl;
    for (int b = lo; b < hi; ++b) {
      const long nt = dec::tiles_of<SK>(dec::clamp_len(p.cache_len[b], p.Lmax));
      if (t_begin >= f && t_begin < f + nt) { loc_b = b; loc_first = f; }
      f += nt;
    }
  }
  __syncthreads();
  const bool have_work = t_begin < t_end;
  const int n_steps = (int)(t_end - t_begin);
  Segments sg;
  if (have_work) sg.init(p, t_begin, n_steps, loc_b, (long)loc_first);
  auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {
    const bool good = mbar_wait(bar, parity, ab);
    return __all_sync(0xffffffffu, good);
  };
  // Two barriers at once: one after the other, each costs a warp a hundred cycles of its chain even when it is complete.
  auto wait_both = [&](uint64_t* bar0, uint32_t parity0, uint64_t* bar1, uint32_t parity1) -> bool {
    const bool r0 = mbar_try_wait(bar0, parity0), r1 = mbar_try_wait(bar1, parity1);
    if (__all_sync(0xffffffffu, r0 && r1)) return true;
    return wait_all(bar0, parity0) && wait_all(bar1, parity1);
  };

  // 88 x 128 + 208 x 256 = 64512 = 168 x 384 registers, what the CTA was launched with
  if (warp < 4) {
   asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
   if (have_work && warp == 0) {
    // ------------------------------- TMA producer -------------------------------
    if (elect_one()) { tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV); }
    __syncwarp();
    const int box_rows = min(p.pv.page_size, TK);
    Lookup look;
    look.init(p, sg, lane);
    Place cur = look.next(p);
    int n = 0, sk = 0, sv = 0;                     // steps requested so far; stages, and the parities that their release has
    uint32_t k_par = 1, v_par = 1;
    auto request = [&](bool wait) -> bool {        // the next step
      const Place nxt = look.next(p);              // on its way while this step's stages are waited for
      int pg = cur.pg;
      if (cur.rows && (pg < 0 || pg >= p.pv.n_pages)) {
        atomicOr(p.err, (unsigned)TA_DEVERR_BAD_PAGE);
        pg = p.pv.n_pages;                         // outside the tensor: the box is filled with zeros
      }
      const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, cur.rows)) * box_rows * 128);
      if (wait && !(shared ? wait_all(&vempty[sv], v_par) : wait_both(&kempty[sk], k_par, &vempty[sv], v_par))) return false;
      if (lane == 0) {
        if (!shared) mbar_expect_tx(&kfull[sk], bytes);
        mbar_expect_tx(&vfull[sv], bytes);
      }
      __syncwarp();
      if (cur.rows) {
        if (!shared) tma_load_3d(ring + sk * STEP_BYTES + look.my_row * 128, &tmK, &kfull[sk], 0, cur.in_page, pg);
        tma_load_3d(vring + sv * STEP_BYTES + look.my_row * 128, &tmV, &vfull[sv], 0, cur.in_page, pg);
      }
      ++n;
      if (++sk == K_STAGES) { sk = 0; k_par ^= 1u; }
      if (++sv == VS) { sv = 0; v_par ^= 1u; }
      cur = nxt;
      return true;
    };
    // A CTA whose steps all fit into the rings requests them before the wait for the query kernel (see k_dec_attn_umma).
    const int ahead = n_steps <= K_STAGES ? n_steps : 0;
    int it = 0;
    for (; it < ahead; ++it) (void)request(false);
    pdl_enter();
    for (; it < n_steps; ++it)
      if (!request(true)) break;
    if (ab.raised()) {                             // the copies in flight end before the CTA does
      if (!shared) mbar_drain_ring(kfull, n, K_STAGES);
      mbar_drain_ring(vfull, n, VS);
    }
   } else if (have_work && warp == 1) {
    // ------------------------------- issuer of the scores -----------------------
    pdl_enter();
    if (elect_one()) {
      const uint32_t idesc_qk = idesc_f8(0, TK, PC);
      const int ksteps = p.r3 / 32;
      const uint64_t dq0 = umma_desc_kmajor_sw128(smem_u32(qbuf));
      const uint64_t dk0 = umma_desc_kmajor_sw128(smem_u32(ring));
      int sv = 0, sk = 0, seg = 0, n_patch = 0;    // stages
      uint32_t v_par = 0, k_par = 0;               // parity of the rings
      uint32_t used = 0, par = 0;                  // per warpgroup, a bit each: any scores before; parity of their being taken
      bool ok = true;
      for (; sg.more() && ok; sg.next(), ++seg) {
        const uint64_t dq = dq0 + (uint64_t)((seg & 1) * (QBUF_BYTES >> 4));
        if (!(ok = seg == 0 ? mbar_wait(&q_first, 0, ab) : mbar_wait(&q_full[seg & 1], (uint32_t)(((seg - 1) >> 1) & 1), ab))) break;
        for (int it = sg.it0; it < sg.it1; ++it) {
          const bool last = sg.tail && it == sg.it1 - 1;
          if (!shared && !(ok = mbar_wait(&kfull[sk], k_par, ab))) break;
          if ((shared || last) && !(ok = mbar_wait(&vfull[sv], v_par, ab))) break;
          if (last) {
            mbar_arrive(&wanted);
            if (!(ok = mbar_wait(&patched, (uint32_t)(n_patch & 1), ab))) break;
            ++n_patch;
          }
          const uint64_t dk = dk0 + (uint64_t)((shared ? sv : sk) * (STEP_BYTES >> 4));
          const int nw = sg.both(it) ? 2 : 1;
          for (int g = 0; g < nw && ok; ++g) {
            // the step before's scores are in registers
            if ((used >> g) & 1u) {
              if (!(ok = mbar_wait(&s_free[g], (par >> g) & 1u, ab))) break;
              par ^= 1u << g;
            }
            used |= 1u << g;
            tc_fence_after();
            const uint32_t d = tmem + (uint32_t)(g * PC);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              if (ks < ksteps) umma_f8(d, dk + (uint64_t)(g * (TK * 128 >> 4) + ks * 2), dq + (uint64_t)(ks * 2), idesc_qk, ks != 0 ? 1u : 0u);
            umma_commit(&s_full[g]);
          }
          if (!ok) break;
          if (!shared) umma_commit(&kempty[sk]);
          if (++sv == VS) { sv = 0; v_par ^= 1u; }
          if (++sk == K_STAGES) { sk = 0; k_par ^= 1u; }
        }
        if (ok) umma_commit(&q_empty[seg & 1]);
      }
    }
   } else if (have_work && warp == 2) {
    // ------------------------------- issuer of the values; scales ---------------
    // Scale bytes by cp.async, 16 rows of a kind per lane, S_AHEAD steps ahead of the values.  (As bulk copies they took the
    // producer 700 cycles per 128 keys to issue; as loads into registers, by these lanes or by the softmax threads for
    // themselves, they were waited for, 1200 cycles.)
    const int ps = p.pv.page_size, box_rows = min(ps, TK);
    const int kind = lane >> 4, row = (lane & 15) * 16, box = row / box_rows, in_box = row - box * box_rows;
    const uint8_t* const pool = (kind == 0 ? p.Ks : p.Vs) + in_box;
    Lookup look;
    look.init(p, sg, lane);
    Place cur = look.next(p);
    int n_req = 0;
    auto request = [&]() {                         // of the next step, if there is one
      if (n_req >= n_steps) return;
      const Place nxt = look.next(p);
      const int pg = __shfl_sync(0xffffffffu, cur.pg, box), rows = __shfl_sync(0xffffffffu, cur.rows, box);
      const int in_page = __shfl_sync(0xffffffffu, cur.in_page, box);
      const uint8_t* const src = rows && pg >= 0 && pg < p.pv.n_pages ? pool + (long)pg * ps + in_page : g_ones;
      const int slot = n_req & (S_SLOTS - 1);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(scales + slot * 2 * SK + kind * SK + row)), "l"(src) : "memory");
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sfull[slot])) : "memory");
      cur = nxt;
      ++n_req;
    };
    if (n_steps > K_STAGES) pdl_enter();           // see the producer
    for (int i = 0; i < S_AHEAD; ++i) request();
    if (n_steps <= K_STAGES) pdl_enter();
    const uint32_t idesc_pv = idesc_f8(1, TK, PC) | (1u << 15) | (1u << 16);      // both with their M / N index contiguous
    const uint64_t dv0 = umma_desc_mnmajor_sw128(smem_u32(vring), TK * 128);
    const uint64_t dp0 = umma_desc_mnmajor_sw128(smem_u32(pbuf), PBUF_BYTES);
    uint32_t v_par = 0;
    uint32_t par = 0, used = 0, o_par = 0;         // per warpgroup, a bit each: parity of the weights; any segment before; its accumulator's
    int sv = 0;
    bool ok = true;
    for (; sg.more() && ok; sg.next()) {
      uint32_t begun = 0;                          // ... in this segment
      for (int it = sg.it0; it < sg.it1 && ok; ++it) {
        const int nw = sg.both(it) ? 2 : 1;
        for (int g = 0; g < nw; ++g) {
          if (g == 0) ok = wait_both(&vfull[sv], v_par, &p_full[0], par & 1u);      // (the patches came before the scores)
          else ok = wait_all(&p_full[1], par >> 1);
          if (!ok) break;
          par ^= 1u << g;
          const bool first = !((begun >> g) & 1u);
          if (first && ((used >> g) & 1u)) {
            // the accumulator of the segment before must have been read
            if (!(ok = wait_all(&o_read[g], (o_par >> g) & 1u))) break;
            o_par ^= 1u << g;
          }
          begun |= 1u << g;
          used |= 1u << g;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t dv = dv0 + (uint64_t)(sv * (STEP_BYTES >> 4) + g * (TK * 128 >> 4)), dp = dp0 + (uint64_t)(g * (PBUF_BYTES >> 4));
            const uint32_t d = tmem + TMEM_O + (uint32_t)(g * PC);
#pragma unroll
            for (int ks = 0; ks < TK / 32; ++ks)
              umma_f8(d, dv + (uint64_t)(ks * 256), dp + (uint64_t)(ks * 256), idesc_pv, (ks != 0 || !first) ? 1u : 0u);
            umma_commit(&p_free[g]);
            if (g == nw - 1) umma_commit(&vempty[sv]);
          }
          __syncwarp();
        }
        if (++sv == VS) { sv = 0; v_par ^= 1u; }
        request();                                 // S_AHEAD steps on: into a slot whose step has had its weights taken
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
   } else if (have_work) {
    // ------------------------------- queries, new rows --------------------------
    pdl_enter();
    Segments sq = sg;                              // the segment whose queries are split next
    sq.next();                                     // (the softmax warps do the first one's)
    int n_q = 1, n_wanted = 0;
    bool ok = true;
    auto split_next = [&]() -> bool {
      const int qb = n_q & 1;
      const int byte = query_byte(p, sq.b);
      if (!wait_all(&q_empty[qb], (uint32_t)(((n_q >> 1) & 1) ^ 1))) return false;
#pragma unroll 2
      for (int i = lane; i < NH * 8; i += 32) split_query(p, sq.b, i, q8::inverse(byte), qbuf + qb * QBUF_BYTES);
      if (lane == 0) q_scale[n_q & 7] = q8::scale(byte);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[qb]);
      ++n_q;
      sq.next();
      return true;
    };
    for (; sg.more() && ok; sg.next()) {
      // the next segment's queries in time, unless this one's last step is almost there (a split takes 3000 cycles)
      if (sg.it1 - sg.it0 > 2 && sq.more() && !(ok = split_next())) break;
      if (!sg.tail) continue;
      // the step with the new token: its row, and zeros behind it as values (their weights are zero, but the slots may hold
      // anything)
      const int it = sg.it1 - 1, row = sg.L - (sg.k0 + (it - sg.it0) * SK), end = row < TK ? TK : SK;
      const int kch = p.r3 / 16, vch = p.t3 / 16;
      uint4 nr = make_uint4(0u, 0u, 0u, 0u);       // lanes 0 .. 7: chunks of the key; 8 .. 15: of the value
      if (lane < kch) nr = reinterpret_cast<const uint4*>(p.knew + (long)sg.b * p.r3)[lane];
      else if (lane >= 8 && lane - 8 < vch) nr = reinterpret_cast<const uint4*>(p.vnew + (long)sg.b * p.t3)[lane - 8];
      const uint8_t ns = lane < 2 ? p.new_scale[2 * (long)sg.b + lane] : 0;
      // (the issuer's word, not vfull: this warp does not follow the ring, whose rounds it could not tell apart)
      if (!(ok = wait_all(&wanted, (uint32_t)(n_wanted & 1)))) break;
      ++n_wanted;
      const int slot = it & (S_SLOTS - 1);
      if (!(ok = wait_all(&sfull[slot], (uint32_t)((it / S_SLOTS) & 1)))) break;
      if (lane < 2) scales[slot * 2 * SK + lane * SK + row] = ns;
      uint8_t* vt = vring + (size_t)(it % VS) * STEP_BYTES;
      uint8_t* kt = shared ? vt : ring + (size_t)(it % K_STAGES) * STEP_BYTES;
      if (lane < kch && !shared) *reinterpret_cast<uint4*>(kt + swz(row, lane)) = nr;
      // (a value's whole line, of which a narrower row leaves zeros: where no box was requested nobody else fills it, and the
      // softmax warps look for rows of zeros by the line)
      if (lane >= 8 && lane < 16) *reinterpret_cast<uint4*>(vt + swz(row, lane - 8)) = nr;
#pragma unroll 4
      for (int i = (row + 1) * 8 + lane; i < end * 8; i += 32) *reinterpret_cast<uint4*>(vt + i * 16) = make_uint4(0u, 0u, 0u, 0u);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&patched);
      if (sg.it1 - sg.it0 <= 2 && sq.more()) ok = split_next();
    }
   }
  } else {
   asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
   if (have_work) {
    // ------------------------------- softmax warpgroups --------------------------
    const int g = (warp - 4) / 4;               // half of every step
    const int q = warp % 4;                     // TMEM lane quadrant
    const int tid = q * 32 + lane;              // key of the half / value coordinate of O^T
    const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
    const uint32_t tm_s = tmem + (uint32_t)(g * PC) + lane_addr, tm_o = tm_s + TMEM_O;
    uint8_t* const my_p = pbuf + g * PBUF_BYTES;
    uint32_t wg_phase = 0, n_mine = 0, n_handed = 0;      // steps in which this warpgroup had keys; parts handed over so far
    pdl_enter();
    {
      // the first segment's queries, on which everything waits: a thread per sixteen numbers (by the warp that does the others'
      // 5000 cycles, here 1000)
      const int byte = query_byte(p, sg.b);
      split_query(p, sg.b, (int)threadIdx.x - 128, q8::inverse(byte), qbuf);
      if (threadIdx.x == 128) q_scale[0] = q8::scale(byte);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_first);
    }
    bool ok = true, owe = false;                // owe: my part lies in the weights' buffer until it is taken
    auto wg_sync = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(&wg_bar[g]);
      const bool good = mbar_wait(&wg_bar[g], wg_phase & 1, ab);
      ++wg_phase;
      return __all_sync(0xffffffffu, good);
    };
    int seg = 0;
    for (; sg.more() && ok; sg.next(), ++seg) {
      uint64_t l2[NH / 2];                      // pairs of heads: sums of this thread's keys
      float m_lane = 0.f;                       // reference of head `lane`
      neg_s[g][q][lane] = 0.f;
      __syncwarp();
#pragma unroll
      for (int h = 0; h < NH / 2; ++h) l2[h] = 0;
      int first = 1;
#pragma unroll 1
      for (int it = sg.it0; it < sg.it1 && ok; ++it) {
        asm volatile("" : "+r"(first));         // no copy of the loop for the first step
        if (g == 1 && !sg.both(it)) break;      // (the last step only)
        const uint32_t par = n_mine & 1u;
        const int slot = it & (S_SLOTS - 1);
        if (!(ok = wait_both(&sfull[slot], (uint32_t)((it / S_SLOTS) & 1), &s_full[g], par))) break;
        tc_fence_after();
        const uint8_t* sc = scales + slot * 2 * SK + g * TK + tid;
        const int kb = sc[0], vb = sc[SK];
        const float kq = q8::scale(kb) * q_scale[seg & 7];
        const float ev = vb == q8::kNan ? NAN : (float)(vb - 127);
        float inv = vb == q8::kNan ? NAN : q8::scale(max(254 - kSumUnit - vb, 0)), low = 0.f;
        if (__any_sync(0xffffffffu, vb == 127)) {
          // A row of zeros has the scale 1, among value rows of 2^-30 too, whose weights it would push below what their bytes hold;
          // as would one with a key that most queries like, among any.  It adds nothing to the output, whatever its weight: that
          // goes into the sum as it is, into the product as zero, and into references as if 2^-kZeroRow.  (Other rows come here only
          // with a largest number of 224 to 448; the tile has not been waited for otherwise.)
          if (!(ok = wait_all(&vfull[it % VS], (uint32_t)((it / VS) & 1)))) break;
          if (vb == 127) {
            const uint8_t* const row = vring + (size_t)(it % VS) * STEP_BYTES + (g * TK + tid) * 128;
            uint32_t any = 0;
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              const uint4 v = *reinterpret_cast<const uint4*>(row + ((c ^ (tid & 7)) << 4));
              any |= v.x | v.y | v.z | v.w;
            }
            if ((any & 0x7f7f7f7fu) == 0) low = kZeroRow;
          }
        }
        // log2 of p 2^k', relative to the references (by halves, for the registers)
        const uint64_t kq2 = pack2(kq, kq), ev2 = pack2(ev, ev);
        float a[NH];
#pragma unroll
        for (int h0 = 0; h0 < NH; h0 += 16) {
          uint32_t s0[16], s1[16], s2[16];
          tmem_ld16(tm_s + h0, s0);
          tmem_ld16(tm_s + NH + h0, s1);
          tmem_ld16(tm_s + 2 * NH + h0, s2);
          tmem_ld_wait();
#pragma unroll
          for (int h = 0; h < 16; h += 4) {
            const float4 neg = *reinterpret_cast<const float4*>(&neg_s[g][q][h0 + h]);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const int i = h + e;
              const uint64_t s = add2(add2(pairu(s0[i], s0[i + 1]), pairu(s1[i], s1[i + 1])), pairu(s2[i], s2[i + 1]));
              unpack2(fma2(s, kq2, add2(ev2, e == 0 ? pack2(neg.x, neg.y) : pack2(neg.z, neg.w))), a[h0 + i], a[h0 + i + 1]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[g]);       // the next step's scores may overwrite the buffer
        if (sg.tail && it == sg.it1 - 1 && sg.k0 + (it - sg.it0) * SK + g * TK + tid > sg.L) {
          // keys past the new token do not exist: weights of zero whatever the scores are
          inv = 0.f;
#pragma unroll
          for (int h = 0; h < NH; ++h) a[h] = -INFINITY;
        }
        const uint64_t inv2 = pack2(inv, inv);
        bool free_seen = n_mine == 0;                  // the step before's product has read the weights
        uint32_t out[2][PIECES][4];
        uint64_t sum[NH / 4];
        // ---- weights in three bytes, of heads 16 half ..; sums ----
        auto weights = [&](int half, uint64_t* into) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t hv[2], piece[PIECES][2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = half * 16 + u * 4 + e * 2;
              const float w0 = ex2(a[h]), w1 = ex2(a[h + 1]);
              into[u * 2 + e] = fma2(pack2(w0, w1), inv2, l2[h / 2]);
              const __half2 x = __floats2half2_rn(w0, w1);
              hv[e] = *reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
              for (int pc = 0; pc < PIECES; ++pc) {
                if (pc == PIECES - 1) {
                  piece[pc][e] = hv[e] + 0x00800080u;            // round the last one; all are positive
                } else {
                  piece[pc][e] = hv[e];
                  const uint32_t top = hv[e] & 0xff00ff00u;
                  const __half2 rest = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&hv[e]), *reinterpret_cast<const __half2*>(&top)),
                                               __float2half2_rn(kRestUp));
                  hv[e] = *reinterpret_cast<const uint32_t*>(&rest);
                }
              }
            }
#pragma unroll
            for (int pc = 0; pc < PIECES; ++pc) out[half][pc][u] = __byte_perm(piece[pc][0], piece[pc][1], 0x7531);
          }
        };
        int renew = first;
        int coarse = 0;                                // a bit per head: its reference was set from a maximum too large for bf16
#pragma unroll 1
        for (;;) {
          if (renew) {
            // ---- new references: the maxima of these keys where they are needed ----
            // Of pairs of heads in bf16 (a reference only has to be near), by a butterfly whose levels keep half of the pairs
            // each: lane 2 i + {0, 1} is left with pair i.  The rounding is half a step, 2^-8 of the maximum: up to kFine it
            // leaves the largest weight within a factor of two of 2^kStart.  Beyond, the reference can lie above every score by more
            // than the weights have bits (from 2^13 on it left them all zero, and the output with them), and nothing but a
            // second round here, on what is left of the scores, would bring it down again.
            uint32_t mx[NH / 2];
            const uint64_t low2 = pack2(-low, -low);
#pragma unroll
            for (int h = 0; h < NH / 2; ++h) {
              float x, y;
              unpack2(add2(pack2(a[2 * h], a[2 * h + 1]), low2), x, y);
              mx[h] = pack_bf16(x, y);
            }
#pragma unroll
            for (int lev = 8; lev >= 1; lev >>= 1) {
              const bool upper = lane & (2 * lev);
#pragma unroll
              for (int h = 0; h < lev; ++h) {
                const uint32_t keep = upper ? mx[h + lev] : mx[h], give = upper ? mx[h] : mx[h + lev];
                mx[h] = max_bf16x2(keep, __shfl_xor_sync(0xffffffffu, give, 2 * lev));
              }
            }
            mx[0] = max_bf16x2(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], 1));
            max_s[g][q][lane] = __uint_as_float(lane & 1 ? mx[0] & 0xffff0000u : mx[0] << 16);
            if (!(ok = wg_sync())) break;
            // by how much the reference of head `lane` rises (it is 0 until the first step sets it)
            const float mt = fmaxf(fmaxf(max_s[g][0][lane], max_s[g][1][lane]), fmaxf(max_s[g][2][lane], max_s[g][3][lane]));
            const bool move = mt >= kTop || first || (coarse >> lane & 1);
            const float up = move ? mt - kStart : 0.f;
            coarse = (int)__ballot_sync(0xffffffffu, move && fabsf(mt) > kFine && fabsf(mt) < INFINITY);
            m_lane += up;
            up_s[g][q][lane] = -up;
            neg_s[g][q][lane] = -m_lane;
            __syncwarp();
#pragma unroll
            for (int h = 0; h < NH; h += 4) {
              const float4 u = *reinterpret_cast<const float4*>(&up_s[g][q][h]);
              a[h] += u.x; a[h + 1] += u.y; a[h + 2] += u.z; a[h + 3] += u.w;
            }
            if (!first) {
              // (A reference comes down in a second round only, after a rise by more than kFine - kStart, which has left zeros of
              // the sums and of the accumulator.)
              // the product of the step before must be complete before its accumulator is rescaled
              if (!free_seen && !(ok = wait_all(&p_free[g], par ^ 1u))) break;
              free_seen = true;
              tc_fence_after();
#pragma unroll
              for (int h = 0; h < NH; h += 2) {
                const float2 u = *reinterpret_cast<const float2*>(&up_s[g][q][h]);
                l2[h / 2] = mul2(l2[h / 2], pack2(ex2(fminf(u.x, 0.f)), ex2(fminf(u.y, 0.f))));
              }
#pragma unroll 1
              for (int h0 = 0; h0 < NH; h0 += 8) {
                if (!__any_sync(0xffffffffu, up != 0.f && lane >> 3 == h0 >> 3)) continue;      // none of these heads' (all warps alike)
                uint32_t o[PIECES][8];
#pragma unroll
                for (int pc = 0; pc < PIECES; ++pc) tmem_ld8(tm_o + pc * NH + h0, o[pc]);
                tmem_ld_wait();
#pragma unroll
                for (int h = 0; h < 8; h += 2) {
                  const float2 u = *reinterpret_cast<const float2*>(&up_s[g][q][h0 + h]);
                  const uint64_t f = pack2(ex2(fminf(u.x, 0.f)), ex2(fminf(u.y, 0.f)));
#pragma unroll
                  for (int pc = 0; pc < PIECES; ++pc) {
                    float x, y;
                    unpack2(mul2(pairu(o[pc][h], o[pc][h + 1]), f), x, y);
                    o[pc][h] = __float_as_uint(x); o[pc][h + 1] = __float_as_uint(y);
                  }
                }
#pragma unroll
                for (int pc = 0; pc < PIECES; ++pc) tmem_st8(tm_o + pc * NH + h0, o[pc]);
              }
              tmem_st_wait();
            }
            first = first && coarse;
          }
          // The vote is counted while half of the weights are formed, on the strength of there being none as a rule.
          float over = -INFINITY;
#pragma unroll
          for (int h = 0; h < NH; h += 2) over = max3(over, a[h], a[h + 1]);
          const uint32_t ph = wg_phase & 1u;
          const bool vote = __any_sync(0xffffffffu, over - low > kTop);
          if (lane == 0) {
            reinterpret_cast<uint8_t*>(&votes[g][ph])[q] = vote ? 1 : 0;
            mbar_arrive(&wg_bar[g]);
          }
          weights(0, sum);
          if (!(ok = wait_all(&wg_bar[g], ph))) break;
          ++wg_phase;
          renew = ((int)*reinterpret_cast<volatile uint32_t*>(&votes[g][ph]) | coarse) != 0;
          if (!renew) break;
        }
        if (!ok) break;
#pragma unroll
        for (int h = 0; h < NH / 4; ++h) l2[h] = sum[h];
        weights(1, l2 + NH / 4);
        if (low != 0.f) {
#pragma unroll
          for (int i = 0; i < 2 * PIECES * 4; ++i) (&out[0][0][0])[i] = 0;
        }
        if (!free_seen && !(ok = wait_all(&p_free[g], par ^ 1u))) break;
        if (owe) {                                     // a part laid down in the weights' buffer must have been taken
          if (!(ok = wait_all(&taken, (n_handed - 1) & 1u))) break;
          owe = false;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int pc = 0; pc < PIECES; ++pc)
            *reinterpret_cast<uint4*>(my_p + swz(tid, pc * 2 + half)) = make_uint4(out[half][pc][0], out[half][pc][1], out[half][pc][2], out[half][pc][3]);
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[g]);
        ++n_mine;
      }
      if (!ok) break;
      const bool two = sg.both(sg.it0);                // warpgroup 1 has a part too
      if (g == 0 || two) {
        if (!(ok = wait_all(&p_free[g], (n_mine - 1) & 1u))) break;      // the product of my last step is complete
        tc_fence_after();
        // the sums, over the keys of the warpgroup's threads, through its weights' buffer: thread by thread, then a head a lane
        {
          uint64_t* const mine = reinterpret_cast<uint64_t*>(my_p + tid * 128);
#pragma unroll
          for (int h = 0; h < NH / 2; h += 2) *reinterpret_cast<ulonglong2*>(mine + ((h + 2 * tid) & (NH / 2 - 1))) = make_ulonglong2(l2[h], l2[h + 1]);
          __syncwarp();
          float t = 0.f;
#pragma unroll 4
          for (int i = q * 32; i < q * 32 + 32; ++i) t += reinterpret_cast<const float*>(my_p + i * 128)[(lane + 4 * i) & (NH - 1)];
          sum_s[g][q][lane] = t;
        }
        if (!(ok = wg_sync())) break;
        float l_lane = sum_s[g][0][lane] + sum_s[g][1][lane] + sum_s[g][2][lane] + sum_s[g][3][lane];
        // the accumulator, its three parts added up, [32 heads][32 groups of four coordinates], groups swizzled
#pragma unroll 1
        for (int h0 = 0; h0 < NH; h0 += 8) {
          uint32_t c0[8], c1[8], c2[8];
          tmem_ld8(tm_o + h0, c0);
          tmem_ld8(tm_o + NH + h0, c1);
          tmem_ld8(tm_o + 2 * NH + h0, c2);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            reinterpret_cast<float*>(my_p)[(h0 + e) * 128 + (((tid >> 2) ^ (h0 + e)) << 2) + (tid & 3)] =
                __uint_as_float(c0[e]) + (__uint_as_float(c1[e]) + __uint_as_float(c2[e]) * (1.f / kRestUp)) * (1.f / kRestUp);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&o_read[g]);        // the next segment may overwrite the accumulator
        // From here on references are of the weights alone, without the scales (exponents in which parts would differ by more than
        // fp32 holds, one of rows of zeros and one of large values): the sum becomes a number of [1, 2).
        const int e2 = min(max((int)(__float_as_uint(l_lane) >> 23) - 127, -126), 126);
        const float f2 = q8::scale(127 - e2);
        l_lane *= f2;
        m_lane += (float)(e2 + kSumUnit);
        float fm = f2 * (1.f / (1 << kSumUnit)), fo = 0.f;      // of head `lane`: what my part and the other one are multiplied by
        if (g == 1) {
          if (q == 0) { hand_m[lane] = m_lane; hand_l[lane] = l_lane; hand_f[lane] = fm; }
        } else if (two) {
          if (!(ok = wait_all(&handed, n_handed & 1u))) break;
          const float mo = hand_m[lane], mn = fmaxf(m_lane, mo), um = ex2(m_lane - mn), uo = ex2(mo - mn);
          fm *= um; fo = hand_f[lane] * uo;
          l_lane = l_lane * um + hand_l[lane] * uo;
          m_lane = mn;
        }
        if (g == 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&handed);
          owe = true;
        } else {
          // joined and stored by head: lane = head, four coordinates at a time (a thread's own coordinate of one head after
          // another, 16 adjacent bytes per four lanes, took 5000 cycles)
          const long slot = (long)blockIdx.x + sg.b;   // one per (CTA, sequence) pair that can occur
          const bool slot_ok = TA_IDX_OK(p.err, slot, 1, (long)gridDim.x + p.B);
          if (!(ok = wg_sync())) break;
          float4* const dst = reinterpret_cast<float4*>(p.part_o + slot * NH * p.t3) + lane;
          const float4 *const a4 = reinterpret_cast<const float4*>(my_p) + lane * 32, *const b4 = reinterpret_cast<const float4*>(pbuf + PBUF_BYTES) + lane * 32;
#pragma unroll 2
          for (int c = q; c < p.t3 / 4; c += 4) {
            float4 v = a4[c ^ lane];
            v.x *= fm; v.y *= fm; v.z *= fm; v.w *= fm;
            if (two) {
              const float4 u = b4[c ^ lane];
              v.x = fmaf(u.x, fo, v.x); v.y = fmaf(u.y, fo, v.y); v.z = fmaf(u.z, fo, v.z); v.w = fmaf(u.w, fo, v.w);
            }
            if (slot_ok) dst[c * NH] = v;
          }
          __syncwarp();
          if (two && lane == 0) mbar_arrive(&taken);
          if (tid == 0) {
            if (sg.head && TA_IDX_OK(p.err, 2 * sg.b, 2, 2L * p.B)) p.seq_cta[2 * sg.b] = (int)blockIdx.x;
            if (sg.tail && TA_IDX_OK(p.err, 2 * sg.b, 2, 2L * p.B)) p.seq_cta[2 * sg.b + 1] = (int)blockIdx.x;
          }
          if (slot_ok && q == 0) reinterpret_cast<float2*>(p.part_ml)[slot * NH + lane] = make_float2(m_lane, l_lane);
        }
      }
      if (two) ++n_handed;
    }
   }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

// The prefix that all sequences share, as the attention kernel of all rows reads it: values of the codes, bf16 (exact), row
// after row; one pool with RoPE: the keys rotated, in two halves (see k_prefix_rotate), and the rows.  A thread per eight
// columns of UNPACK_ROWS rows, blockIdx.y the pool.
// Runs beside the query kernel: when that one lets this one start, the kernels in front of it are complete, calls before among
// them, and it writes neither the prefix's pages nor what this one writes.  (Step behind 32768 tokens, 100 us: 1.3 more behind it
// with a launch per pool; 0.8 more with a row per thread, found by long divisions.)
struct UnpackPart {
  const uint8_t *codes, *scales;
  bf16 *out, *rot;         // rot: null unless the keys are rotated
  int r;
};
constexpr int UNPACK_THREADS = 256, UNPACK_ROWS = 4;
__host__ __device__ inline int unpack_block_rows(int r) { return UNPACK_THREADS / (r / 8) * UNPACK_ROWS; }
__global__ void __launch_bounds__(UNPACK_THREADS) k_prefix_unpack_q8(const UnpackPart first, const UnpackPart second, const int32_t* __restrict__ table,
                                                          int n_pages, int page_size, long rows, int P, const dec::RopeTurns turns,
                                                          unsigned int* err) {
  const UnpackPart& u = blockIdx.y == 0 ? first : second;
  const int r = u.r, per = r / 8, at_once = UNPACK_THREADS / per;
  const int mine = (int)threadIdx.x / per, c = ((int)threadIdx.x - mine * per) * 8;
  const long lo = rows * r, n0 = (long)blockIdx.x * (at_once * UNPACK_ROWS) + mine;
  const uint8_t* src[UNPACK_ROWS];
  float sc[UNPACK_ROWS];
  uint2 codes[UNPACK_ROWS];
#pragma unroll
  for (int k = 0; k < UNPACK_ROWS; ++k) {
    const long n = n0 + k * at_once;
    src[k] = nullptr;
    sc[k] = 0.f;
    if (mine < at_once && n < P) {
      const int slot = (int)n, j = slot / page_size, pg = table[j];
      if (pg >= 0 && pg < n_pages) {
        const long row = (long)pg * page_size + (slot - j * page_size);
        src[k] = u.codes + row * r + c;
        sc[k] = q8::scale(u.scales[row]);
      } else {
        atomicOr(err, (unsigned)TA_DEVERR_BAD_PAGE);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < UNPACK_ROWS; ++k) codes[k] = src[k] ? *reinterpret_cast<const uint2*>(src[k]) : make_uint2(0u, 0u);
#pragma unroll
  for (int k = 0; k < UNPACK_ROWS; ++k) {
    const long n = n0 + k * at_once, at = n * r + c;
    if (mine >= at_once || n >= P || !TA_IDX_OK(err, at, 8, lo)) continue;
    float f[8];
    q8::values8(codes[k], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= sc[k];
    uint32_t w[4], wl[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(f[2 * e], f[2 * e + 1]);
    *reinterpret_cast<uint4*>(u.out + at) = make_uint4(w[0], w[1], w[2], w[3]);
    if (u.rot) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 cs = dec::rope_at((int)n, turns, c / 2 + e);
        const float re = f[2 * e] * cs.x - f[2 * e + 1] * cs.y, ro = f[2 * e] * cs.y + f[2 * e + 1] * cs.x;
        w[e] = pack_bf16(re, ro);
        const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
        wl[e] = pack_bf16(re - v.x, ro - v.y);
      }
      *reinterpret_cast<uint4*>(u.rot + at) = make_uint4(w[0], w[1], w[2], w[3]);
      *reinterpret_cast<uint4*>(u.rot + lo + at) = make_uint4(wl[0], wl[1], wl[2], wl[3]);
    }
  }
  pdl_enter();
}

}  // namespace decq
}  // namespace ta
