// Paged decode step for small work: one launch, a cluster of eight CTAs per sequence, everything between the token and
// y on chip.
//
// A step over a short cache is a chain of dependent small products: projections of the token, queries, attention,
// output core, output.  As launches each link costs a kernel boundary (about 2 us, and as much host time), ten times
// the work in it.
// Here the links go through distributed shared memory: what a CTA computes is sent to the CTAs that need it by
// st.async, which counts the bytes on the receiver's mbarrier, so that a link costs one way through the cluster and no
// fence.
//   1  projections x [U2 | U3 | Ut3]: CTA r takes the r-th eighth of d; everybody receives the partial sums.
//   2  v[a, :] = sum_j (x U2)_j C[a, j, :]: CTA r takes an eighth of the (a, eight columns) pairs, everybody receives
//      them; every CTA then forms all queries q_h = scale sum_a U1[h, a] v[a, :], rotated.
//   3  the keys of the sequence, prefix first, are split evenly over the eight CTAs: keys and values are shared by all
//      heads, so a split over heads would read them eight times.  Rows come by cp.async; the first two tiles are
//      requested before anything is computed, pages are looked up two tiles ahead.  Running maximum and sum per head;
//      CTA 0 starts from the new token.
//   4  the partial outputs' column groups of eight go to the CTAs that own them (group g: CTA g mod 8), which join the
//      eight partials by their maxima and sums and form u[a, c] = sum_h Ut1[h, a] o_h[c] and their columns' share of
//      z[j] = sum_a sum_c Ct[a, j, c] u[a, c], received by everybody.
//   5  y = z Ut2^T: CTA r takes an eighth of the rows.
// All arithmetic is fp32 from the stored values on (the tensor-core path carries q and z as two bf16 numbers each);
// only what is stored is rounded.  Sums are taken in a fixed order.  The weights are read once per sequence and the
// scores take FMAs, so that this form is for small batches of short contexts only: see cluster_step_pays.
//
// Bounded by latency: d 768, 12 heads, ranks 64, one sequence of 37 tokens 11.2 us (19.3 as four launches), of which
// 1.4 wait for the first loads and 0.6 to 1.5 go to each later phase; a tile of 64 keys per CTA 1.3 us (scores and
// values are issue and shared-memory bound).  Exchanges by cluster barrier and remote reads, with less of the rest
// overlapped, were 16.3 us.
#include "ta_paged.cuh"
#include "ta_cluster.cuh"

#include <algorithm>

namespace ta {
namespace pgc {

using namespace cluster;

constexpr int CL = 8, THREADS = 512, WARPS = THREADS / 32;
constexpr int TK = 64;                                 // keys per tile
constexpr int TPR = THREADS / TK;                      // threads that copy a row
constexpr float kLog2e = 1.4426950408889634f;

// Division by a number that the launch fixes, for dividends below 2^20: (x + 1/2) / d is at least 1 / (2 d) from a
// whole number and computed to x / d * 2^-22.  An integer division is some 150 cycles of latency, and a step has a
// dozen between its links.
struct Div {
  int d;
  float inv;
  __host__ explicit Div(int v) : d(v), inv(1.f / (float)v) {}
  __device__ __forceinline__ int operator()(int x) const { return __float2int_rz(((float)x + 0.5f) * inv); }
};

template <typename T>
struct Params {
  const T *x, *C, *U1, *U2, *U3, *Ct, *Ut1, *Ut2, *Ut3;
  T *y, *K, *V;
  PagedView pv;
  const int32_t *cache_len, *prefix_table;
  int B, d, nH, r1, r2, r3, t1, t2, t3, Lmax, P, append, one_pool, rope;
  float scale;
  dec::RopeTurns turns;
  unsigned int* err;
  // columns of the projections, of a key and of a value in groups of eight; (four heads, eight columns) pairs; ...
  Div nc3, ch3, ch, combos, half, t1d, t2d, nc, nh8;
  int G, KS, SA, rpw, cs_log;
  explicit Params(const tucker_attn_desc& e, bool shared)
      : nc3((e.r2 + e.r3 + (shared ? 0 : e.t3)) / 8), ch3(e.r3 / 8), ch(e.t3 / 8), combos((e.n_H + 3) / 4 * (e.t3 / 8)),
        half(e.r3 / 2), t1d(e.t1), t2d(e.t2), nc(e.t2 / 8), nh8(e.n_H * 8) {
    G = THREADS / nc3.d;
    KS = std::min(TK / 4, THREADS / combos.d);
    SA = THREADS / e.t2;
    rpw = 32 / nc.d;
    const int quads = (e.n_H + 3) / 4;
    cs_log = quads * 4 <= WARPS ? 2 : 1;               // 2^cs_log shares of a score's columns: about one task per warp
  }
};

// Shared memory (offsets in bytes, multiples of 16).
template <typename T>
struct Layout {
  int kp, vp, stage;                                   // bytes of a key row, a value row, a stage of the ring
  int ring, xs, part, q, gat, sum, xq, v, u1, s, orc, mlg, w, oc, u, ut1, zg, total;
  __host__ __device__ Layout(int d, int nH, int r1, int r2, int r3, int t1, int t2, int t3, bool one_pool) {
    const int N = r2 + r3 + t3, nco = (t3 / 8 + CL - 1) / CL;
    kp = r3 * (int)sizeof(T) + 16;                     // one 16-byte column on per row: 32 rows read at one column hit all banks
    vp = one_pool ? 0 : t3 * (int)sizeof(T) + 16;
    stage = TK * (kp + vp);
    int off = 0;
    auto take = [&](int floats) { const int o_ = off; off += (floats * 4 + 15) / 16 * 16; return o_; };
    ring = off; off += 2 * stage > THREADS * 128 ? 2 * stage : THREADS * 128;   // afterwards: 32 partial outputs per thread
    xs = take((d + CL - 1) / CL);
    part = q = take(nH * r3 > THREADS * 8 ? nH * r3 : THREADS * 8);      // partial projections, then queries, then partials of z
    gat = take(CL * N);
    sum = take(N > t2 ? N : t2);
    xq = take(N > t2 ? N : t2);                        // x U2, new key (rotated), new value; at the end z
    v = take(r1 * r3);
    u1 = take(nH * r1);
    s = take(WARPS * 4 * TK);                          // [shares of the columns][heads][keys]
    orc = take(nco * CL * nH * 8);
    mlg = take(CL * nH * 2);
    w = take(CL * nH);
    oc = take(nco * nH * 8);
    u = take(nco * t1 * 8);
    ut1 = take(nH * t1);
    zg = take(CL * t2);
    total = off;
  }
};

__device__ __forceinline__ void cp16(void* dst, const void* src, bool there) {      // zeros where there is no row
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Eight consecutive elements as stored, and as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(w[e] << 16);
      f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// Dot products over columns [c_beg, c_end) of two keys (rows `step` bytes apart) with four heads.
template <typename T>
__device__ __forceinline__ void scores(const char* row, int step, const float* const (&q)[4], int c_beg, int c_end, float (&acc)[2][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[0][i] = acc[1][i] = 0.f;
#pragma unroll 2
  for (int c = c_beg; c < c_end; c += 8) {
    Raw8<T> k0, k1;
    float f0[8], f1[8];
    k0.load(reinterpret_cast<const T*>(row) + c);
    k1.load(reinterpret_cast<const T*>(row + step) + c);
    k0.get(f0);
    k1.get(f1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 a = *reinterpret_cast<const float4*>(q[i] + c), b = *reinterpret_cast<const float4*>(q[i] + c + 4);
      const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[0][i] = fmaf(w[e], f0[e], acc[0][i]);
        acc[1][i] = fmaf(w[e], f1[e], acc[1][i]);
      }
    }
  }
}

template <typename T>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(THREADS, 1) k_pg_step(const __grid_constant__ Params<T> p) {
  extern __shared__ __align__(16) char sm[];
  const Layout<T> lay(p.d, p.nH, p.r1, p.r2, p.r3, p.t1, p.t2, p.t3, p.one_pool);
  auto at = [&](int off) { return reinterpret_cast<float*>(sm + off); };
  float *const xs = at(lay.xs), *const part = at(lay.part), *const gat = at(lay.gat), *const sum_s = at(lay.sum), *const xq = at(lay.xq);
  float *const v_s = at(lay.v), *const u1_s = at(lay.u1), *const q_s = at(lay.q), *const s_s = at(lay.s), *const orc = at(lay.orc);
  float *const mlg = at(lay.mlg), *const w_s = at(lay.w), *const oc_s = at(lay.oc), *const u_s = at(lay.u), *const ut1_s = at(lay.ut1);
  float* const zg = at(lay.zg);
  __shared__ uint64_t bar_x, bar_v, bar_o, bar_z;      // one per exchange
  __shared__ float2 cs_s[64];                          // (cos, sin) of the new token's position
  __shared__ float m_s[32], l_s[32], al_s[32];
  __shared__ long dst_s;                               // row of the new token, -1: not written (by this CTA)
  __shared__ long rows_s[2][TK];                       // pool rows of the keys of a tile, -1: none

  const int b = blockIdx.x / CL, rank = blockIdx.x % CL, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int d = p.d, nH = p.nH, r1 = p.r1, r2 = p.r2, r3 = p.r3, t1 = p.t1, t2 = p.t2, t3 = p.t3;
  const int tp = p.one_pool ? 0 : t3, N = r2 + r3 + tp; // projected columns (one pool: the value row is the key row)
  const int ch = p.ch.d, nco = (ch - rank + CL - 1) / CL;      // column groups of the output; those of this CTA
  if (tid == 0) {
    sm100::mbar_init(&bar_x, 1); sm100::mbar_init(&bar_v, 1); sm100::mbar_init(&bar_o, 1); sm100::mbar_init(&bar_z, 1);
    sm100::fence_barrier_init();
    sm100::mbar_expect_tx(&bar_x, CL * N * 4);
    sm100::mbar_expect_tx(&bar_v, r1 * r3 * 4);
    sm100::mbar_expect_tx(&bar_o, CL * nH * (nco * 32 + 8));
    sm100::mbar_expect_tx(&bar_z, CL * t2 * 4);
  }
  cluster_arrive();                                    // "started, ready to receive": waited for before anything is sent
  pdl_enter();
  // ---- everything that needs nothing is requested first ----
  int L = p.cache_len[b];
  const int k_beg = (int)((long)d * rank / CL), k_end = (int)((long)d * (rank + 1) / CL);
  const T xv0 = k_beg + tid < k_end ? p.x[(long)b * d + k_beg + tid] : T(0.f);
  const int G = p.G, pg = p.nc3(tid), pn = (tid - pg * p.nc3.d) * 8;      // projections: thread = (eight columns, share of the rows)
  const T* F;
  int ldf;
  if (pn < r2) { F = p.U2 + pn; ldf = r2; }
  else if (pn < r2 + r3) { F = p.U3 + (pn - r2); ldf = r3; }
  else { F = p.Ut3 + (pn - r2 - r3); ldf = t3; }
  constexpr int PF = 16 / (int)sizeof(T);              // rows in flight per thread
  Raw8<T> f[PF];
  auto rows_of = [&](int k0) {
#pragma unroll
    for (int e = 0; e < PF; ++e) {
      if (pg < G && k0 + e * G < k_end) f[e].load(F + (long)(k0 + e * G) * ldf);
      else f[e].zero();
    }
  };
  rows_of(k_beg + pg);
  const T u10 = tid < nH * r1 ? p.U1[tid] : T(0.f), ut10 = tid < nH * t1 ? p.Ut1[tid] : T(0.f);

  if (k_beg + tid < k_end) xs[tid] = to_f(xv0);
  for (int k = k_beg + tid + THREADS; k < k_end; k += THREADS) xs[k - k_beg] = to_f(p.x[(long)b * d + k]);
  __syncthreads();

  bool write = p.append;
  if (L < 0 || L >= p.Lmax) {
    if (tid == 0 && rank == 0) atomicOr(p.err, (unsigned)TA_DEVERR_BAD_CACHE_LEN);
    L = L < 0 ? 0 : p.Lmax - 1;
    write = false;                                     // a page is not written on the strength of a clamped length
  }
  // this CTA's keys: [key_beg, key_beg + n_keys) of the prefix and the cached slots together
  const long keys = (long)p.P + L, key_beg = keys * rank / CL;
  const int n_keys = (int)(keys * (rank + 1) / CL - key_beg), tiles = (n_keys + TK - 1) / TK;
  const int32_t* const table = p.pv.table + (long)b * p.pv.max_pages;
  // Page entry of a key (prefix and slots together) and its place in the page; the entry is checked when it is used.
  auto entry = [&](long key, int& in_page) -> int {
    const bool own = key >= p.P;
    const int slot = (int)(own ? key - p.P : key), e = slot / p.pv.page_size;
    in_page = slot - e * p.pv.page_size;
    return own ? table[e] : p.prefix_table[e];
  };
  auto row_of = [&](int pg, int in_page) -> long {     // -1: no such page (flagged)
    if (pg >= 0 && pg < p.pv.n_pages) return (long)pg * p.pv.page_size + in_page;
    atomicOr(p.err, (unsigned)TA_DEVERR_BAD_PAGE);
    return -1;
  };
  const int kc = r3 * (int)sizeof(T) / 16, vc = tp * (int)sizeof(T) / 16;
  auto request = [&](int tile) {                       // one commit group per call, also without rows
    if (tile < tiles) {
      char* const st = sm + lay.ring + (tile & 1) * lay.stage;
      const int j = tid / TPR;
      const long row = rows_s[tile & 1][j];
      [[maybe_unused]] const long rows = (long)p.pv.n_pages * p.pv.page_size;
      const bool there = row >= 0 && TA_IDX_OK(p.err, row, 1, rows);
      const char* const k = reinterpret_cast<const char*>(p.K + (there ? row : 0) * r3);
      const char* const v = reinterpret_cast<const char*>(p.V + (there ? row : 0) * t3);
#pragma unroll 4
      for (int c = tid % TPR; c < kc; c += TPR) cp16(st + j * lay.kp + c * 16, k + c * 16, there);
#pragma unroll 4
      for (int c = tid % TPR; c < vc; c += TPR) cp16(st + TK * lay.kp + j * lay.vp + c * 16, v + c * 16, there);
    }
    cp_commit();
  };
  // page entries of the first two tiles, and of the new token's row
  int pg0 = 0, in0 = 0;
  const bool has0 = tid < 2 * TK ? tid < n_keys : (tid == 2 * TK && write && rank == 0);
  if (has0) pg0 = entry(tid < 2 * TK ? key_beg + tid : keys, in0);

  // ---- 1: projections ----
  {
    float acc[8] = {};
    for (int k0 = k_beg + pg; k0 < k_end; k0 += PF * G) {
      if (k0 != k_beg + pg) rows_of(k0);
#pragma unroll
      for (int e = 0; e < PF; ++e) {
        const float xv = k0 + e * G < k_end ? xs[k0 + e * G - k_beg] : 0.f;
        float ff[8];
        f[e].get(ff);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(xv, ff[i], acc[i]);
      }
    }
    if (pg < G) {
      *reinterpret_cast<float4*>(part + pg * N + pn) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(part + pg * N + pn + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
    }
  }
  if (tid < nH * r1) u1_s[tid] = to_f(u10);
  if (tid < nH * t1) ut1_s[tid] = to_f(ut10);
  for (int i = tid + THREADS; i < nH * r1; i += THREADS) u1_s[i] = to_f(p.U1[i]);
  for (int i = tid + THREADS; i < nH * t1; i += THREADS) ut1_s[i] = to_f(p.Ut1[i]);
  if (tid <= 2 * TK) {
    const long row0 = has0 ? row_of(pg0, in0) : -1;
    if (tid < 2 * TK) rows_s[tid / TK][tid % TK] = row0;
    else dst_s = row0;
  }
  // v's first rows of the core (a warp per slice a and eight columns) and, towards L2, what the last phases read
  const int units = r1 * p.ch3.d, un_beg = units * rank / CL, un_end = units * (rank + 1) / CL;
  constexpr int PC = 4;
  Raw8<T> cpre[PC];
  auto core_rows = [&](int un, int j0) {
    const int a = p.ch3(un), c = (un - a * p.ch3.d) * 8;
#pragma unroll
    for (int e = 0; e < PC; ++e) {
      const int j = j0 + lane + 32 * e;
      if (un < un_end && j < r2) cpre[e].load(p.C + ((long)a * r2 + j) * r3 + c);
      else cpre[e].zero();
    }
  };
  core_rows(un_beg + warp, 0);
  {
    const unsigned cl = (unsigned)(t1 * t2 * t3) * sizeof(T) / (CL * 128), ul = (unsigned)(d * t2) * sizeof(T) / (CL * 128);
    const char *c0 = reinterpret_cast<const char*>(p.Ct) + (size_t)rank * cl * 128, *u0 = reinterpret_cast<const char*>(p.Ut2) + (size_t)rank * ul * 128;
    for (unsigned i = tid; i < cl; i += THREADS) asm volatile("prefetch.global.L2 [%0];" ::"l"(c0 + i * 128u));
    for (unsigned i = tid; i < ul; i += THREADS) asm volatile("prefetch.global.L2 [%0];" ::"l"(u0 + i * 128u));
  }
  __syncthreads();
  for (int c = tid; c < N; c += THREADS) {
    float t = 0.f;
#pragma unroll 8
    for (int k = 0; k < G; ++k) t += part[k * N + c];
    sum_s[c] = t;
  }
  if (p.rope && tid >= THREADS - r3 / 2) {             // the last two warps, which have the least to add up
    const int i = THREADS - 1 - tid;
    cs_s[i] = dec::rope_at(p.P + L, p.turns, i);
  }
  __syncthreads();
  cluster_wait();
  for (int i = tid; i < N * (CL / 4); i += THREADS) {
    const int c = i / CL * 4;
    send4(gat + rank * N + c, i % CL, &bar_x, *reinterpret_cast<const float4*>(sum_s + c));
  }
  request(0);
  request(1);
  bool came = received(&bar_x, p.err);
  for (int c = tid; c < N; c += THREADS) {
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < CL; ++r) t += gat[r * N + c];
    xq[c] = t;
  }
  __syncthreads();
  // ---- 2: v, and the new token's row ----
  for (int un = un_beg + warp; un < un_end; un += WARPS) {
    float acc[8] = {};
    for (int j0 = 0; j0 < r2; j0 += 32 * PC) {
      if (un != un_beg + warp || j0 != 0) core_rows(un, j0);
#pragma unroll
      for (int e = 0; e < PC; ++e) {
        const int j = j0 + lane + 32 * e;
        const float xv = j < r2 ? xq[j] : 0.f;
        float ff[8];
        cpre[e].get(ff);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(xv, ff[i], acc[i]);
      }
    }
    // sums over the lanes, halving the columns a lane holds as long as it holds more than one: column = bits 4, 3, 2 of
    // the lane
#pragma unroll
    for (int st = 0; st < 3; ++st) {
      const int keep = 4 >> st, bit = 16 >> st;
      const bool up = lane & bit;
#pragma unroll
      for (int i = 0; i < keep; ++i) {
        const float give = up ? acc[i] : acc[i + keep], mine = up ? acc[i + keep] : acc[i];
        acc[i] = mine + __shfl_xor_sync(0xffffffffu, give, bit);
      }
    }
    acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], 2);
    acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], 1);
    float* const dst = v_s + un * 8 + (lane >> 4 & 1) * 4 + (lane >> 3 & 1) * 2 + (lane >> 2 & 1);      // un * 8 = a r3 + column
    send(dst, lane & 3, &bar_v, acc[0]);
    send(dst, (lane & 3) + 4, &bar_v, acc[0]);
  }
  const int vofs = p.one_pool ? r2 : r2 + r3;          // the new value row in xq; the new key, rotated in place, at r2
  if (p.rope && tid < r3 / 2) {
    const float xe = xq[r2 + 2 * tid], xo = xq[r2 + 2 * tid + 1];
    const float2 cs = cs_s[tid];
    xq[r2 + 2 * tid] = xe * cs.x - xo * cs.y;
    xq[r2 + 2 * tid + 1] = xe * cs.y + xo * cs.x;
  }
  came &= received(&bar_v, p.err);
  // queries, in units of log2
  for (int i = tid; i < nH * (r3 / 2); i += THREADS) {
    const int h = p.half(i), c = i - h * p.half.d;
    float xe = 0.f, xo = 0.f;
#pragma unroll 8
    for (int a = 0; a < r1; ++a) {
      const float uu = u1_s[h * r1 + a];
      const float2 vv = reinterpret_cast<const float2*>(v_s + a * r3)[c];
      xe = fmaf(uu, vv.x, xe);
      xo = fmaf(uu, vv.y, xo);
    }
    xe *= p.scale * kLog2e; xo *= p.scale * kLog2e;
    const float2 cs = p.rope ? cs_s[c] : make_float2(1.f, 0.f);
    reinterpret_cast<float2*>(q_s + h * r3)[c] = make_float2(xe * cs.x - xo * cs.y, xe * cs.y + xo * cs.x);
  }
  __syncthreads();
  // ---- 3: attention.  Values: thread = (four heads, eight columns, key subset); CTA 0 starts from the new token ----
  const int KS = p.KS, ks = p.combos(tid), cmb = tid - ks * p.combos.d, hq = p.ch(cmb) * 4, vcol = (cmb - p.ch(cmb) * ch) * 8;
  float acc[4][8] = {};
  for (int h = warp; h < nH; h += WARPS) {
    float t = 0.f;
    if (rank == 0) {
      for (int c = lane; c < r3; c += 32) t = fmaf(q_s[h * r3 + c], xq[r2 + c], t);
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    }
    if (lane == 0) {
      m_s[h] = rank == 0 ? t : -INFINITY;
      l_s[h] = rank == 0 ? 1.f : 0.f;
    }
  }
  if (rank == 0 && ks == 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[0][i] = acc[1][i] = acc[2][i] = acc[3][i] = xq[vofs + vcol + i];
  const int cs_log = p.cs_log, CS = 1 << cs_log, quads = (nH + 3) / 4;
  for (int t = 0; t < tiles; ++t) {
    const char* const st = sm + lay.ring + (t & 1) * lay.stage;
    const char* const vt = p.one_pool ? st : st + TK * lay.kp;
    const int vpitch = p.one_pool ? lay.kp : lay.vp;
    const int here = min(TK, n_keys - t * TK);
    if (t == 0) cp_wait<1>();
    else cp_wait<0>();
    __syncthreads();                                   // the tile is there for all; the one before it is done with
    if (t >= 1) request(t + 1);
    const int i2 = (t + 2) * TK + tid;                 // the tile after the next
    const bool has2 = tid < TK && i2 < n_keys;
    int pg2 = 0, in2 = 0;
    if (has2) pg2 = entry(key_beg + i2, in2);
    for (int task = warp; task < CS * quads; task += WARPS) {      // task = (share of the columns, four heads), lane = two keys
      const int share = task & (CS - 1), hb = (task >> cs_log) * 4;
      const float* qh[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) qh[i] = q_s + min(hb + i, nH - 1) * r3;
      float a[2][4];
      scores<T>(st + lane * lay.kp, 32 * lay.kp, qh, (p.ch3.d * share >> cs_log) * 8, (p.ch3.d * (share + 1) >> cs_log) * 8, a);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (hb + i < nH) {
          float* const dst = s_s + (share * nH + hb + i) * TK + lane;
          dst[0] = a[0][i];
          dst[32] = a[1][i];
        }
    }
    if (tid < TK) rows_s[t & 1][tid] = has2 ? row_of(pg2, in2) : -1;
    __syncthreads();
    for (int h = warp; h < nH; h += WARPS) {
      float sc[TK / 32], mt = -INFINITY;
#pragma unroll
      for (int e = 0; e < TK / 32; ++e) {
        const int j = lane + 32 * e;
        sc[e] = s_s[h * TK + j];
        sc[e] += s_s[(nH + h) * TK + j];
        if (CS > 2) sc[e] += s_s[(2 * nH + h) * TK + j] + s_s[(3 * nH + h) * TK + j];
        if (j >= here) sc[e] = -INFINITY;
        mt = fmaxf(mt, sc[e]);
      }
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, off));
      const float mo = m_s[h], mn = fmaxf(mo, mt), mr = mn == -INFINITY ? 0.f : mn;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < TK / 32; ++e) {
        const float pe = dec::ex2(sc[e] - mr);
        s_s[h * TK + lane + 32 * e] = pe;
        sum += pe;
      }
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      __syncwarp();
      if (lane == 0) {
        const float al = dec::ex2(mo - mr);
        al_s[h] = al;
        l_s[h] = fmaf(l_s[h], al, sum);
        m_s[h] = mn;
      }
    }
    __syncthreads();
    if (ks < KS) {
      int ho[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ho[i] = min(hq + i, nH - 1);
        const float al = al_s[ho[i]];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i][e] *= al;
      }
      for (int kb = ks; kb * 4 < here; kb += KS) {     // rows behind `here` are zeros, their weights too
        float wt[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 w4 = *reinterpret_cast<const float4*>(s_s + ho[i] * TK + kb * 4);
          wt[i][0] = w4.x; wt[i][1] = w4.y; wt[i][2] = w4.z; wt[i][3] = w4.w;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          Raw8<T> vv;
          float ff[8];
          vv.load(reinterpret_cast<const T*>(vt + (kb * 4 + k) * vpitch) + vcol);
          vv.get(ff);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[i][e] = fmaf(wt[i][k], ff[e], acc[i][e]);
        }
      }
    }
  }
  cp_wait<0>();
  __syncthreads();
  // Key subsets joined through the ring's memory; the sums go to the owners of their columns, maxima and sums to
  // everybody.
  {
    float* const red = at(lay.ring);
    if (ks < KS) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (hq + e < nH)
#pragma unroll
          for (int i = 0; i < 8; i += 4)
            reinterpret_cast<float4*>(red)[((ks * nH + hq + e) * 2 + i / 4) * ch + vcol / 8] =      // neighbours next to each other
                make_float4(acc[e][i], acc[e][i + 1], acc[e][i + 2], acc[e][i + 3]);
    }
    if (tid < nH * CL) send2(mlg + (rank * nH + tid / CL) * 2, tid % CL, &bar_o, make_float2(m_s[tid / CL], l_s[tid / CL]));
    __syncthreads();
    for (int i = tid; i < nH * t3 / 4; i += THREADS) {
      float4 s = reinterpret_cast<const float4*>(red)[i];
#pragma unroll 4
      for (int k = 1; k < KS; ++k) {
        const float4 o = reinterpret_cast<const float4*>(red + k * nH * t3)[i];
        s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
      }
      const int hh = p.ch(i), g = i - hh * ch, h = hh >> 1;    // i = (head, half of the eight columns, group)
      send4(orc + (((g / CL) * CL + rank) * nH + h) * 8 + (hh & 1) * 4, g % CL, &bar_o, s);
    }
  }
  // ---- 4: join and output core.  z: thread = (row j, share of this CTA's (column group, slice a) pairs) ----
  const int SA = p.SA, za = p.t2d(tid), zj = tid - za * t2, pairs = nco * t1;
  constexpr int PZ = 4;
  Raw8<T> zr4[PZ];
  auto z_rows = [&](int i0) {
#pragma unroll
    for (int e = 0; e < PZ; ++e) {
      const int i = i0 + e * SA, gi = p.t1d(i), a = i - gi * t1;
      if (za < SA && i < pairs) zr4[e].load(p.Ct + ((long)a * t2 + zj) * t3 + (rank + gi * CL) * 8);
      else zr4[e].zero();
    }
  };
  z_rows(za);
  // the new token's row, where its stores are in nobody's way
  {
    [[maybe_unused]] const long rows = (long)p.pv.n_pages * p.pv.page_size;
    if (dst_s >= 0 && TA_IDX_OK(p.err, dst_s, 1, rows)) {
      if (tid < t3) put(p.V + dst_s * t3 + tid, xq[vofs + tid]);
      if (!p.one_pool && tid >= THREADS - r3) put(p.K + dst_s * r3 + tid - (THREADS - r3), xq[r2 + tid - (THREADS - r3)]);
    }
  }
  came &= received(&bar_o, p.err);
  if (tid < nH) {
    float m = -INFINITY, l = 0.f, wr[CL];
#pragma unroll
    for (int r = 0; r < CL; ++r) m = fmaxf(m, mlg[(r * nH + tid) * 2]);
#pragma unroll
    for (int r = 0; r < CL; ++r) {
      wr[r] = dec::ex2(mlg[(r * nH + tid) * 2] - m);   // no keys: 0
      l = fmaf(mlg[(r * nH + tid) * 2 + 1], wr[r], l);
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int r = 0; r < CL; ++r) w_s[r * nH + tid] = wr[r] * inv;
  }
  __syncthreads();
  for (int i = tid; i < nco * nH * 8; i += THREADS) {
    const int g = p.nh8(i), hc = i - g * nH * 8, h = hc / 8;
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < CL; ++r) t = fmaf(w_s[r * nH + h], orc[(g * CL + r) * nH * 8 + hc], t);
    oc_s[i] = t;
  }
  __syncthreads();
  for (int i = tid; i < pairs * 8; i += THREADS) {
    const int g = p.t1d(i / 8), a = i / 8 - g * t1, c = i % 8;
    float t = 0.f;
#pragma unroll 4
    for (int h = 0; h < nH; ++h) t = fmaf(ut1_s[h * t1 + a], oc_s[(g * nH + h) * 8 + c], t);
    u_s[i] = t;
  }
  __syncthreads();
  {
    float zacc = 0.f;
    if (za < SA)
      for (int i0 = za; i0 < pairs; i0 += PZ * SA) {
        if (i0 != za) z_rows(i0);
#pragma unroll
        for (int e = 0; e < PZ; ++e) {
          if (i0 + e * SA >= pairs) break;
          float ff[8];
          zr4[e].get(ff);
          const float4 ua = *reinterpret_cast<const float4*>(u_s + (i0 + e * SA) * 8), ub = *reinterpret_cast<const float4*>(u_s + (i0 + e * SA) * 8 + 4);
          zacc = fmaf(ff[0], ua.x, zacc); zacc = fmaf(ff[1], ua.y, zacc); zacc = fmaf(ff[2], ua.z, zacc); zacc = fmaf(ff[3], ua.w, zacc);
          zacc = fmaf(ff[4], ub.x, zacc); zacc = fmaf(ff[5], ub.y, zacc); zacc = fmaf(ff[6], ub.z, zacc); zacc = fmaf(ff[7], ub.w, zacc);
        }
      }
    if (za < SA) part[za * t2 + zj] = zacc;
  }
  // ---- 5: y.  Lane = (row of rpw, eight columns of the factor's row); the first rows are requested before z is there
  const int nc = p.nc.d, rpw = p.rpw, sub = p.nc(lane), cz = lane - sub * nc;
  constexpr int YU = 4;
  const int y_step = WARPS * rpw, y0 = k_beg + warp * rpw + sub;      // rows [k_beg, k_end), y_step of them at a time
  Raw8<T> yv[YU];
  auto y_rows = [&](int j0) {
#pragma unroll
    for (int k = 0; k < YU; ++k) {
      const int j = j0 + k * y_step;
      if (sub < rpw && j < k_end) yv[k].load(p.Ut2 + (long)j * t2 + cz * 8);
      else yv[k].zero();
    }
  };
  y_rows(y0);
  __syncthreads();
  if (tid < t2) {
    float t = 0.f;
    for (int k = 0; k < SA; ++k) t += part[k * t2 + tid];
    sum_s[tid] = t;
  }
  __syncthreads();
  for (int i = tid; i < t2 * (CL / 4); i += THREADS) {
    const int j = i / CL * 4;
    send4(zg + rank * t2 + j, i % CL, &bar_z, *reinterpret_cast<const float4*>(sum_s + j));
  }
  came &= received(&bar_z, p.err);
  if (tid < t2) {
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < CL; ++r) t += zg[r * t2 + tid];
    xq[tid] = t;
  }
  __syncthreads();
  const float4 za4 = *reinterpret_cast<const float4*>(xq + cz * 8), zb4 = *reinterpret_cast<const float4*>(xq + cz * 8 + 4);
  const float zr[8] = {za4.x, za4.y, za4.z, za4.w, zb4.x, zb4.y, zb4.z, zb4.w};
  for (int j0 = y0; j0 - sub < k_end; j0 += YU * y_step) {
    if (j0 != y0) y_rows(j0);
    float t[YU];
#pragma unroll
    for (int k = 0; k < YU; ++k) {
      float ff[8];
      yv[k].get(ff);
      t[k] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) t[k] = fmaf(zr[e], ff[e], t[k]);
    }
    for (int off = 1; off < nc; off <<= 1)             // sums over the nc lanes of a row
#pragma unroll
      for (int k = 0; k < YU; ++k) {
        const float o = __shfl_down_sync(0xffffffffu, t[k], off);
        if (cz + off < nc) t[k] += o;
      }
#pragma unroll
    for (int k = 0; k < YU; ++k) {
      const int j = j0 + k * y_step;
      if (sub < rpw && cz == 0 && j < k_end && TA_IDX_OK(p.err, (long)b * d + j, 1, (long)p.B * d)) put(p.y + (long)b * d + j, t[k]);
    }
  }
  if (!came) {                                         // a wait ran out: y is void, and what comes late must find this CTA here
    stay_for(&bar_x); stay_for(&bar_v); stay_for(&bar_o); stay_for(&bar_z);
  }
}

template <typename T>
int smem_bytes(const tucker_attn_desc& d, bool one_pool) {
  return Layout<T>(d.d_model, d.n_H, d.r1, d.r2, d.r3, d.t1, d.t2, d.t3, one_pool).total;
}
constexpr int kMaxSmem = 225 * 1024;

// Clusters of this kernel that the current device runs at once (one CTA per SM: 15 on B200, whose GPCs are not all
// multiples of eight SMs), asked once per device; 0: the runtime cannot tell.
template <typename T>
int clusters_at_once() {
  static std::mutex mu;
  static int known[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (known[dev] == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CL);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = kMaxSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CL; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static PerDeviceFlag attr_smem;
    int n = 0;
    if (ensure_dynamic_smem(attr_smem, (const void*)k_pg_step<T>, kMaxSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k_pg_step<T>, &cfg) != cudaSuccess)
      (void)cudaGetLastError();
    known[dev] = n > 0 ? n : -1;
  }
  return std::max(known[dev], 0);
}

template <typename T>
int launch(Problem& p) {
  const tucker_attn_desc& d = p.d;
  Params<T> g(d, p.shared_kv);
  g.x = (const T*)p.X; g.C = (const T*)p.C; g.U1 = (const T*)p.U1; g.U2 = (const T*)p.U2; g.U3 = (const T*)p.U3;
  g.Ct = (const T*)p.Ct; g.Ut1 = (const T*)p.Ut1; g.Ut2 = (const T*)p.Ut2; g.Ut3 = (const T*)p.Ut3;
  g.y = (T*)p.Y; g.K = (T*)p.Kc; g.V = (T*)p.Vc;
  g.pv = p.pv; g.cache_len = p.cache_len; g.prefix_table = p.prefix_table;
  g.B = d.B; g.d = d.d_model; g.nH = d.n_H; g.r1 = d.r1; g.r2 = d.r2; g.r3 = d.r3; g.t1 = d.t1; g.t2 = d.t2; g.t3 = d.t3;
  g.Lmax = p.Lmax; g.P = p.prefix_len; g.append = p.append; g.one_pool = p.shared_kv; g.rope = d.rope;
  g.scale = p.scale; g.turns = rope_turns(d); g.err = p.dev_err;
  static PerDeviceFlag attr;
  TA_CUDA_TRY(ensure_dynamic_smem(attr, (const void*)k_pg_step<T>, kMaxSmem));
  prof_begin(p);
  (void)launch_pdl(k_pg_step<T>, dim3((unsigned)d.B * CL), dim3(THREADS), (size_t)smem_bytes<T>(d, p.shared_kv), p.stream, g);
  TA_LAUNCH_CHECK(p);
  prof_end(p);
  return TA_OK;
}

}  // namespace pgc

bool cluster_step_supported(const tucker_attn_desc& d, bool one_pool) {
  auto ok8 = [](int r, int most) { return r % 8 == 0 && r <= most; };
  if (!ok8(d.r2, 256) || !ok8(d.t2, 256) || !ok8(d.r3, 128) || !ok8(d.t3, 128) || d.d_model % 8) return false;
  if (d.n_H > 32 || d.r1 > 32 || d.t1 > 32 || (d.flags & TA_FLAG_FORCE_GENERIC)) return false;
  if (one_pool && d.rope) return false;                // the cached rows would have to be rotated
  return (d.dtype == TA_DTYPE_F32 ? pgc::smem_bytes<float>(d, one_pool) : pgc::smem_bytes<bf16>(d, one_pool)) <= pgc::kMaxSmem;
}

// Whether this form is the faster one, by the longest sequence the table can hold.  All in us, fitted to the device
// time of whole steps over d 768 to 4096, 8 to 32 heads, ranks 64 to 128 and 1 to 36 sequences (w = heads * (r3 + t3)):
//   here          10 + 3.2 (bf16) or 2.3 (fp32) per MB of weights + (2.9 + w / 940) per 1024 keys, for every wave of
//                 clusters
//   tensor cores  20.5 + 1.6 per MB of weights, hardly more with keys and sequences as far as the rule reaches
//   generic       30 + 1.6 per MB of weights + 0.8 per 1000 keys of all sequences and 1536 of w
// E.g. d 768, 12 heads, ranks 64, here / there: bf16, 1 sequence of 64 keys 11.6 / 19.9, 1024 14.1 / 19.5, 3000 22.7 /
// 19.6; 15 of 2048 19.0 / 27.6; 16 (a second wave) of 1024 27.6 / 23.6; fp32, 1 of 64 12.2 / 31.4, 4 of 2048 19.8 /
// 41.2, 36 of 8192 146 / 505.
// d 4096, 32 heads, ranks 128, 4 of 64 keys 25.2 / 27.2, of 1024 33.0 / 27.7.
bool cluster_step_pays(const tucker_attn_desc& d, int64_t slots, int32_t prefix_len, bool tensor_cores) {
  const bool f32 = d.dtype == TA_DTYPE_F32;
  const int at_once = f32 ? pgc::clusters_at_once<float>() : pgc::clusters_at_once<bf16>();
  if (at_once == 0) return false;
  const double mb = ((double)d.d_model * (d.r2 + d.r3 + d.t2 + d.t3) + (double)d.r1 * d.r2 * d.r3 + (double)d.t1 * d.t2 * d.t3) * (f32 ? 4e-6 : 2e-6);
  const double keys = (double)slots + prefix_len, w = (double)d.n_H * (d.r3 + d.t3);
  const double waves = (d.B + at_once - 1) / at_once;
  const double here = waves * (10. + (f32 ? 2.3 : 3.2) * mb + keys / 1024. * (2.9 + w / 940.));
  const double there = tensor_cores ? 20.5 + 1.6 * mb : 30. + 1.6 * mb + 0.8e-3 * d.B * keys * w / 1536.;
  return here < there;
}

int cluster_paged_decode(Problem& p) { return p.d.dtype == TA_DTYPE_F32 ? pgc::launch<float>(p) : pgc::launch<bf16>(p); }

}  // namespace ta
