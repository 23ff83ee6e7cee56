// Output side of the paged decode step: joins the partials of a sequence -- those of its own keys (streaming kernel)
// and of the shared prefix (prefix kernel) -- by their maxima and sums and applies the output-side core:
//   o_h = merged, normalised output of head h;  u[a, :] = sum_h Ut1[h, a] o_h;  z[j] = sum_a sum_c Ct[a, j, c] u[a, c]
// A cluster of CL CTAs per sequence (8, 4 or 2: the most that still lets all of them run at once, two CTAs per SM).
// CTA y merges t3 / CL value columns of all heads (every partial is read once per sequence, where CTAs that split the
// rows of z would each have to merge everything), forms its columns of u, hands them to the other CTAs through
// distributed shared memory, and computes t2 / CL rows of z.  For small batches (paged_out_fuses_y) it goes on to y = z
// Ut2^T: z is handed round the cluster and every CTA computes d / CL outputs, each sequence reading the factor again,
// which a launch and its boundary outweigh as long as there are few.  One user with a long cache has a partial from
// every SM: the maxima, weights and sums of the partials are spread over all warps instead of walked by one.
// The kernels before it fill their SMs, so that next to nothing of this one overlaps them: it takes the CTAs that hold
// a sequence from the streaming kernel instead of scanning the lengths.
#pragma once

#include "ta_cluster.cuh"
#include "ta_common.cuh"
#include "ta_decode.cuh"
#include "ta_paged.cuh"
#include "ta_prefix_attn.cuh"

namespace ta {
namespace pgout {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_PART = 2 * dec::MAX_GRID;      // partials of one head: one per CTA of either attention kernel at most

struct Params {
  int B, nH, t1, t2, t3, z_half;
  const int* seq_cta;                            // [B][2]
  const float *part_o, *part_ml;                 // own keys: [grid + B][t3 / 4][32][4], [grid + B][32][2]
  int grid;
  const float *pre_o, *pre_ml;                   // prefix: [grid_p + n_rb][t3 / 4][RB][4], [..][RB][2]
  int grid_p, n_kt, n_rb;                        // n_rb = 0: no prefix
  const bf16 *Ct, *Ut1;
  bf16* z;                                       // [B, 2 z_half]: rounded values, rounded rests
  const bf16* Ut2;                               // not null: y = z Ut2^T here, z stays on chip
  bf16* y;                                       // [B, d]
  int d;
  unsigned int* err;
};

__host__ __device__ inline size_t smem_bytes(int cl, int t1, int t3, int nH, bool with_prefix) {
  const int parts = with_prefix ? MAX_PART : dec::MAX_GRID;
  return sizeof(float) * ((size_t)parts * 64 + (size_t)t1 * t3 + ((size_t)nH * t1 + 1) / 2 * 2 + (size_t)THREADS * 4 + 32 * (128 / cl));
}

template <int CL>
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(THREADS, 2) k_pg_out(const Params p) {
  constexpr int MAX_COLS = 128 / CL;
  extern __shared__ __align__(16) float sm[];
  const int t3 = p.t3, cw = t3 / CL, q4 = cw / 4;          // columns of this CTA (t3 = 64, 96 or 128), as float4
  float4* red_s = reinterpret_cast<float4*>(sm);           // [THREADS]
  float* o_s = sm + THREADS * 4;                           // [32][MAX_COLS]
  float* u_s = o_s + 32 * MAX_COLS;                        // [t1][t3]
  float* ut1_s = u_s + p.t1 * t3;                          // [nH][t1]
  float2* w_s = reinterpret_cast<float2*>(ut1_s + (p.nH * p.t1 + 1) / 2 * 2);      // [partials][32]: (max, sum), then (weight, -)
  __shared__ float hm_s[WARPS][32], hl_s[WARPS][32];
  __shared__ float z_s[256];
  const int b = blockIdx.x / CL, y = blockIdx.x % CL, c0 = y * cw;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int jn = p.t2 / CL, jbeg = y * jn;
  __shared__ uint64_t bar_u, bar_z;                        // everybody's columns of u; (fused y) everybody's rows of z
  if (tid == 0) {
    sm100::mbar_init(&bar_u, 1);
    sm100::mbar_init(&bar_z, 1);
    sm100::fence_barrier_init();
    sm100::mbar_expect_tx(&bar_u, p.t1 * t3 * 4);
    if (p.Ut2) sm100::mbar_expect_tx(&bar_z, p.t2 * 4);
  }
  cluster::cluster_arrive();                               // "started, ready to receive": waited for before anything is sent
  // z: lane = (slice a of rpl, 16-byte chunk) of a row of the core
  const int nch = t3 / 8, rpl = 32 / nch;                  // 8, 12 or 16 chunks; 4, 2 or 2 slices at a time
  const int ga = lane / nch, ch = lane % nch;
  const uint4* Cq = reinterpret_cast<const uint4*>(p.Ct);
  auto core = [&](int jl, int a) -> uint4 {
    return (jl < jn && ga < rpl && a < p.t1) ? Cq[((long)a * p.t2 + jbeg + jl) * nch + ch] : make_uint4(0u, 0u, 0u, 0u);
  };
  {
    // this CTA's rows of the core towards L2 (a long cache streamed through it has pushed them out) while the partials
    // are merged
    const char* rows = reinterpret_cast<const char*>(p.Ct) + (long)jbeg * t3 * 2;
    const int lines = (jn * t3 * 2 + 127) / 128;
    for (int a = warp; a < p.t1; a += WARPS)
      for (int i = lane; i < lines; i += 32)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(rows + (long)a * p.t2 * t3 * 2 + i * 128));
  }
  for (int i = tid; i < p.nH * p.t1; i += THREADS) ut1_s[i] = __bfloat162float(p.Ut1[i]);
  // The prefix's partials of head h (rows of a sequence may lie in two row blocks): first slot, number, row in the
  // block.
  __shared__ int ps0_s[32], pc_s[32];
  if (warp == 0) {
    int slot0 = 0, cnt = 0;
    if (p.n_rb > 0 && lane < p.nH) {
      const int rb = (b * p.nH + lane) / prefix::RB;
      const long tot = (long)p.n_rb * p.n_kt, f = (long)rb * p.n_kt;
      const int first = (int)prefix::owner_of(f, tot, p.grid_p), last = (int)prefix::owner_of(f + p.n_kt - 1, tot, p.grid_p);
      slot0 = first + rb;
      cnt = last - first + 1;
      if (!TA_IDX_OK(p.err, slot0, cnt, (long)p.grid_p + p.n_rb)) cnt = 0;
    }
    ps0_s[lane] = slot0;
    pc_s[lane] = cnt;
  }
  __syncthreads();
  // Up to here only inputs of the call were read; the partials come from the kernels before this one.
  pdl_enter();
  const int noted = p.seq_cta[2 * b], np = noted_parts(noted, p.seq_cta[2 * b + 1], p.grid), i0 = np > 0 ? noted : 0;
  if (np == 0 && tid == 0) atomicOr(p.err, (unsigned)TA_DEVERR_WAIT_TIMEOUT);      // the streaming kernel gave up: y is void
  // ---- weights: warp w takes the partials w, w + WARPS, ... of all heads (lane = head) ----
  {
    const int h = lane, pc = pc_s[h], prl = (b * p.nH + h) % prefix::RB;
    const long ps0 = ps0_s[h];
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + (long)(i0 + b) * 32 + h;
    const float2* pml = reinterpret_cast<const float2*>(p.pre_ml) + ps0 * prefix::RB + prl;
    float m = -INFINITY;
#pragma unroll 2
    for (int k = warp; k < np; k += WARPS) {
      const float2 v = ml[(long)k * 32];
      w_s[k * 32 + h] = v;
      m = fmaxf(m, v.x);
    }
#pragma unroll 2
    for (int k = warp; k < pc; k += WARPS) {
      const float2 v = pml[(long)k * prefix::RB];
      w_s[(np + k) * 32 + h] = v;
      m = fmaxf(m, v.x);
    }
    hm_s[warp][h] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) m = fmaxf(m, hm_s[w][h]);      // finite: a sequence's own part holds the new token
    float l = 0.f;
    for (int k = warp; k < np; k += WARPS) {
      float2& v = w_s[k * 32 + h];
      v.x = dec::ex2(v.x - m);
      l = fmaf(v.y, v.x, l);
    }
    for (int k = warp; k < pc; k += WARPS) {
      float2& v = w_s[(np + k) * 32 + h];
      v.x = dec::ex2(v.x - m);
      l = fmaf(v.y, v.x, l);
    }
    hl_s[warp][h] = l;
  }
  __syncthreads();
  // ---- merge: item = (four columns, head), heads adjacent (512 bytes per load of 32 heads) ----
  // (partials dealt over groups of threads)
  const int items = p.nH * q4, groups = min(16, THREADS / items);
  {
    const int g = tid / items, it = tid % items, h = it % p.nH, c = c0 + it / p.nH * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (g < groups) {
      const int pc = pc_s[h], prl = (b * p.nH + h) % prefix::RB;
      const long ps0 = ps0_s[h];
      const float* po = p.part_o + (long)(i0 + b) * 32 * t3 + ((long)(c / 4) * 32 + h) * 4;
      const float* pp = p.pre_o + ps0 * prefix::RB * t3 + ((long)(c / 4) * prefix::RB + prl) * 4;
      auto add = [&](const float* src, long stride, int n, int w0) {
        constexpr int PF = 6;           // partials in flight per thread
        for (int k0 = g; k0 < n; k0 += PF * groups) {
          float4 v[PF];
#pragma unroll
          for (int e = 0; e < PF; ++e) {
            const int k = k0 + e * groups;
            v[e] = k < n ? *reinterpret_cast<const float4*>(src + (long)k * stride) : make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll
          for (int e = 0; e < PF; ++e) {
            const int k = k0 + e * groups;
            const float wt = k < n ? w_s[(w0 + k) * 32 + h].x : 0.f;
            acc.x = fmaf(wt, v[e].x, acc.x); acc.y = fmaf(wt, v[e].y, acc.y);
            acc.z = fmaf(wt, v[e].z, acc.z); acc.w = fmaf(wt, v[e].w, acc.w);
          }
        }
      };
      add(po, 32L * t3, np, 0);
      add(pp, (long)prefix::RB * t3, pc, np);
    }
    red_s[tid] = acc;
  }
  // the first slices of this warp's first two rows of the core: requested here, used behind two barriers
  uint4 pre[2][4];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int e = 0; e < 4; ++e) pre[r][e] = core(warp + r * WARPS, e * rpl + ga);
  __syncthreads();
  if (tid < items) {
    const int h = tid % p.nH;
    float4 s = red_s[tid];
    for (int g = 1; g < groups; ++g) {
      const float4 v = red_s[g * items + tid];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) l += hl_s[w][h];
    const float inv = 1.f / l;
    *reinterpret_cast<float4*>(o_s + h * MAX_COLS + tid / p.nH * 4) = make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv);
  }
  __syncthreads();
  cluster::cluster_wait();
  // ---- this CTA's columns of u, to every CTA of the cluster ----
  for (int i = tid; i < p.t1 * cw; i += THREADS) {
    const int a = i / cw, c = i % cw;
    float acc = 0.f;
    for (int h = 0; h < p.nH; ++h) acc = fmaf(ut1_s[h * p.t1 + a], o_s[h * MAX_COLS + c], acc);
#pragma unroll
    for (int r = 0; r < CL; ++r) cluster::send(&u_s[a * t3 + c0 + c], r, &bar_u, acc);
  }
  bool came = cluster::received(&bar_u, p.err);
  // ---- z: a warp per row ----
  auto dot = [&](const uint4 (&v)[2][4], int a0, float (&acc)[2]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int a = a0 + e * rpl + ga;
      if (ga < rpl && a < p.t1) {
        const float4 u0 = reinterpret_cast<const float4*>(u_s + a * t3 + ch * 8)[0];
        const float4 u1 = reinterpret_cast<const float4*>(u_s + a * t3 + ch * 8)[1];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t wv[4] = {v[r][e].x, v[r][e].y, v[r][e].z, v[r][e].w};
          const float2 k0 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[0]));
          const float2 k1 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[1]));
          const float2 k2 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[2]));
          const float2 k3 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[3]));
          float t = acc[r];
          t = fmaf(u0.x, k0.x, t); t = fmaf(u0.y, k0.y, t); t = fmaf(u0.z, k1.x, t); t = fmaf(u0.w, k1.y, t);
          t = fmaf(u1.x, k2.x, t); t = fmaf(u1.y, k2.y, t); t = fmaf(u1.z, k3.x, t); t = fmaf(u1.w, k3.y, t);
          acc[r] = t;
        }
      }
    }
  };
  for (int jl = warp; jl < jn; jl += 2 * WARPS) {            // two rows at a time
    float acc[2] = {0.f, 0.f};
    for (int a0 = 0; a0 < p.t1; a0 += 4 * rpl) {
      if (jl != warp || a0 != 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) pre[r][e] = core(jl + r * WARPS, a0 + e * rpl + ga);
      }
      dot(pre, a0, acc);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int j = jbeg + jl + r * WARPS;
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], off);
      if (p.Ut2) {
        if (lane < CL && jl + r * WARPS < jn) cluster::send(&z_s[j], (uint32_t)lane, &bar_z, acc[r]);
      } else if (lane == 0 && jl + r * WARPS < jn && TA_IDX_OK(p.err, (long)b * 2 * p.z_half + p.z_half + j, 1, (long)p.B * 2 * p.z_half)) {
        const bf16 zh = __float2bfloat16_rn(acc[r]);
        p.z[(long)b * 2 * p.z_half + j] = zh;
        p.z[(long)b * 2 * p.z_half + p.z_half + j] = __float2bfloat16_rn(acc[r] - __bfloat162float(zh));
      }
    }
  }
  if (p.Ut2) {
    // ---- y: lane = (row of rpw, 16-byte chunk of the factor's row); a lane's eight values of z stay in registers ----
    came &= cluster::received(&bar_z, p.err);
    const int nc = p.t2 / 8, rpw = 32 / nc, sub = lane / nc, cz = lane % nc;
    const bool on = sub < rpw;
    float zr[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) zr[e] = z_s[cz * 8 + e];
    const uint4* F = reinterpret_cast<const uint4*>(p.Ut2);
    const int rows = p.d / CL, end = (y + 1) * rows;
    constexpr int YU = 4;                  // row groups in flight per warp
    for (int j0 = y * rows + warp * rpw * YU; j0 < end; j0 += WARPS * rpw * YU) {
      uint4 v[YU];
#pragma unroll
      for (int k = 0; k < YU; ++k) {
        const int j = j0 + k * rpw + sub;
        v[k] = (on && j < end) ? F[(long)j * nc + cz] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < YU; ++k) {
        const int j = j0 + k * rpw + sub;
        const uint32_t wv[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&wv[e]));
          t = fmaf(zr[2 * e], f.x, t);
          t = fmaf(zr[2 * e + 1], f.y, t);
        }
        for (int off = 1; off < nc; off <<= 1) {           // sum over the nc lanes of the row
          const float o = __shfl_down_sync(0xffffffffu, t, off);
          if (cz + off < nc) t += o;
        }
        if (on && cz == 0 && j < end && TA_IDX_OK(p.err, (long)b * p.d + j, 1, (long)p.B * p.d)) p.y[(long)b * p.d + j] = __float2bfloat16_rn(t);
      }
    }
  } else if (y == 0) {
    for (int j = p.t2 + tid; j < p.z_half; j += THREADS)
      if (TA_IDX_OK(p.err, (long)b * 2 * p.z_half + p.z_half + j, 1, (long)p.B * 2 * p.z_half)) {
        p.z[(long)b * 2 * p.z_half + j] = __float2bfloat16_rn(0.f);
        p.z[(long)b * 2 * p.z_half + p.z_half + j] = __float2bfloat16_rn(0.f);
      }
  }
  if (!came) {                                             // a wait ran out: what comes late must find this CTA here
    cluster::stay_for(&bar_u);
    if (p.Ut2) cluster::stay_for(&bar_z);
  }
}

}  // namespace pgout
}  // namespace ta
