// Shape-generic FMA kernels of the paged cache: append, decode, decode behind a shared prefix; fp32 storage, and bf16
// shapes the tensor-core kernels do not cover.  Everything between the inputs and the outputs is fp32.
//
// Unlike the contiguous decode step's generic kernel, which walks a whole sequence in one block, the keys are split
// over blocks and joined by their (max, sum, output) partials: a step with few sequences still fills the GPU.
#include "ta_gemm_fma.cuh"
#include "ta_paged.cuh"
#include "ta_q8.cuh"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace ta {
namespace {

using fma::ld;
using fma::st;
__device__ __forceinline__ float ld(const e4m3* p) { return q8::value(p->v); }      // without its row's scale

// ---------------------------------------------------------------------------------------
// 32 x 32 tile of A [M, K] B [K, N], fp32 accumulation.  512 threads: eight groups of 64 threads take an eighth of
// every 128-deep K block each (4 x 4 outputs per thread) and are summed through shared memory at the end, so that the
// short and narrow products of a decode step (few rows, K = d) have eight times the threads a plain tile would and a
// round trip to memory covers 128 of K.  The next K block is in registers while the current one is multiplied.
// ---------------------------------------------------------------------------------------
constexpr int GM = 32, GN = 32, GK = 128, GG = 8, GT = 64 * GG;

struct TileSmem {
  union {
    struct { float a[GK][GM + 1], b[GK][GN + 1]; } in;
    float part[GG][GM][GN + 1];
  };
};

struct MatB {              // element (k, n) at k * sk + n * sn
  long sk, sn;
};

// K blocks [k_beg, K).  On return s.part[0] holds the tile (rows and columns past the edge are zero); all threads are
// synchronised.
template <typename TA, typename TB>
__device__ __forceinline__ void gemm_tile(const TA* __restrict__ A, long lda, const TB* __restrict__ Bm, MatB sb, int M, int N, int k_beg,
                                          int K, int m0, int n0, TileSmem& s) {
  const int tid = threadIdx.x, grp = tid / 64, tx = tid % 8, ty = (tid % 64) / 8;
  float acc[4][4] = {};
  float ra[8], rb[8];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int idx = tid + i * GT;
      const int m = idx / GK, k = k0 + idx % GK;
      ra[i] = (m0 + m < M && k < K) ? ld(A + (long)(m0 + m) * lda + k) : 0.f;
      const int n = sb.sn == 1 ? idx % GN : idx / GK, kb = k0 + (sb.sn == 1 ? idx / GN : idx % GK);
      rb[i] = (n0 + n < N && kb < K) ? ld(Bm + (long)kb * sb.sk + (long)(n0 + n) * sb.sn) : 0.f;
    }
  };
  fetch(k_beg);
  for (int k0 = k_beg; k0 < K; k0 += GK) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int idx = tid + i * GT;
      s.in.a[idx % GK][idx / GK] = ra[i];
      if (sb.sn == 1) s.in.b[idx / GN][idx % GN] = rb[i];
      else s.in.b[idx % GK][idx / GK] = rb[i];
    }
    __syncthreads();
    if (k0 + GK < K) fetch(k0 + GK);
#pragma unroll
    for (int kk = 0; kk < GK / GG; ++kk) {
      const int k = grp * (GK / GG) + kk;
      float a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = s.in.a[k][ty * 4 + i]; b[i] = s.in.b[k][tx * 4 + i]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s.part[grp][ty * 4 + i][tx * 4 + j] = acc[i][j];
  __syncthreads();
  for (int i = tid; i < GM * GN; i += GT) {
    float c = 0.f;
#pragma unroll
    for (int g = 0; g < GG; ++g) c += s.part[g][i / GN][i % GN];
    s.part[0][i / GN][i % GN] = c;       // read above by this thread only
  }
  __syncthreads();
}

// C [M, N] (ld ldc) = A B for up to three (B, C) pairs that share A and K: blockIdx.z = share of K * pairs + pair.  The
// shares' products lie `split` elements apart and are added up by whoever reads them.
template <typename TB, typename TC>
struct GemmPart {
  const TB* B;
  MatB sb;
  TC* C;
  long ldc;
  int N;
  long split;
};
template <typename TA, typename TB, typename TC>
struct GemmArgs {
  const TA* A;
  long lda;
  int M, K, parts, kb_per_split;   // kb_per_split: GK-deep blocks of K per share
  GemmPart<TB, TC> part[3];
};
template <typename TA, typename TB, typename TC>
__global__ void __launch_bounds__(GT) k_pg_gemm(const GemmArgs<TA, TB, TC> g) {
  pdl_enter();
  __shared__ TileSmem s;
  const GemmPart<TB, TC> pt = g.part[blockIdx.z % g.parts];
  const int share = blockIdx.z / g.parts, k_beg = share * g.kb_per_split * GK;
  const int m0 = blockIdx.x * GM, n0 = blockIdx.y * GN;
  if (n0 >= pt.N) return;
  gemm_tile(g.A, g.lda, pt.B, pt.sb, g.M, pt.N, k_beg, min(g.K, k_beg + g.kb_per_split * GK), m0, n0, s);
  for (int i = threadIdx.x; i < GM * GN; i += GT) {
    const int m = m0 + i / GN, n = n0 + i % GN;
    if (m < g.M && n < pt.N) st(pt.C + share * pt.split + (long)m * pt.ldc + n, s.part[0][i / GN][i % GN]);
  }
}

// Rotation frequency of coordinate pair i of r; (cos, sin) at a position: dec::rope_cos_sin_theta.
__device__ __forceinline__ double pair_theta(int i, int r, double base) { return pow(base, -2.0 * (double)i / (double)r); }
constexpr int kMaxPairs = 544;      // r3 / 2; shape_ok() bounds r3 well below this

// ---------------------------------------------------------------------------------------
// Append: 32 tokens x 32 latent coordinates per block; blockIdx.z = 0 keys, 1 values.
// ---------------------------------------------------------------------------------------
template <typename T>
struct AppendArgs {
  const T *X, *U3, *Ut3;
  T *K, *V;
  PagedView pv;
  const int32_t *tok_start, *cache_len;
  int B, T_, d, r3, t3, rope, pos0;
  int keys_shared;      // 1: only the value rows are written (one pool; un-rotated rows when rope)
  double base;
  dec::RopeTurns turns; // of the first 128 pairs; those behind are formed from `base`
  unsigned int* err;
};
template <typename T>
__global__ void __launch_bounds__(GT) k_pg_append(const AppendArgs<T> g) {
  pdl_enter();
  __shared__ TileSmem s;
  __shared__ long row_s[GM];
  __shared__ int pos_s[GM];
  __shared__ unsigned long long turn_s[GN / 2];
  const bool is_k = blockIdx.z == 0 && !g.keys_shared;
  const int r = is_k ? g.r3 : g.t3;
  const int m0 = blockIdx.x * GM, n0 = blockIdx.y * GN;
  if (n0 >= r) return;
  if (is_k && g.rope && threadIdx.x >= 64 && threadIdx.x < 64 + GN / 2) {
    const int i = n0 / 2 + threadIdx.x - 64;
    if (i < 128) {
      turn_s[threadIdx.x - 64] = g.turns.turn[i];
    } else {
      const double turns = pair_theta(i, r, g.base) * 0.15915494309189535;
      turn_s[threadIdx.x - 64] = (unsigned long long)((turns - floor(turns)) * 18446744073709551616.0);
    }
  }
  if (threadIdx.x < GM) {
    AppendDst dst;
    dst.row = -1; dst.pos = 0;
    if (m0 + (int)threadIdx.x < g.T_)
      dst = append_dst(m0 + threadIdx.x, g.tok_start, g.cache_len, g.B, g.pos0, g.pv, g.err);
    row_s[threadIdx.x] = dst.row;
    pos_s[threadIdx.x] = dst.pos;
  }
  MatB sb = {r, 1};
  gemm_tile(g.X, (long)g.d, is_k ? g.U3 : g.Ut3, sb, g.T_, r, 0, g.d, m0, n0, s);
  T* pool = is_k ? g.K : g.V;
  for (int i = threadIdx.x; i < GM * GN; i += GT) {
    const int m = i / GN, c = i % GN, n = n0 + c;
    if (row_s[m] < 0 || n >= r) continue;
    float v = s.part[0][m][c];
    if (is_k && g.rope) {            // r3 is even and tiles start at even columns: both halves of a pair are here
      const float other = s.part[0][m][c ^ 1];
      const float2 cs = dec::rope_cos_sin_turn(pos_s[m], turn_s[c >> 1]);
      v = (c & 1) ? other * cs.y + v * cs.x : v * cs.x - other * cs.y;
    }
    if (TA_IDX_OK(g.err, row_s[m] * r + n, 1, (long)g.pv.n_pages * g.pv.page_size * r)) st(pool + row_s[m] * r + n, v);
  }
}

// w[a, b, c] = sum_q qt[b, q] C[a, q, c].  A block forms 32 columns of one slice for four sequences: thread (c, g) of
// 32 x 8 walks the rows q = g, g + 8, ..., the eight sums per column are joined through shared memory.
constexpr int WB = 4;
template <typename T>
__global__ void __launch_bounds__(256) k_pg_w(const float* __restrict__ qt_parts, int shares, const T* __restrict__ C,
                                              float* __restrict__ w, int B, int r1, int r2, int r3) {
  pdl_enter();
  extern __shared__ float qt[];                 // [WB][r2]
  __shared__ float red[8][WB][32];
  for (int i = threadIdx.x; i < WB * r2; i += 256) {
    const int b = blockIdx.x * WB + i / r2;
    float t = 0.f;
    if (b < B)
#pragma unroll 4
      for (int k = 0; k < shares; ++k) t += qt_parts[((long)k * B + b) * r2 + i % r2];
    qt[i] = t;
  }
  __syncthreads();
  const int b0 = blockIdx.x * WB, a = blockIdx.y, c = blockIdx.z * 32 + threadIdx.x % 32, g = threadIdx.x / 32;
  float acc[WB] = {};
  if (c < r3)
#pragma unroll 4
    for (int q = g; q < r2; q += 8) {
      const float v = ld(C + ((long)a * r2 + q) * r3 + c);
#pragma unroll
      for (int i = 0; i < WB; ++i)
        acc[i] = fmaf(qt[i * r2 + q], v, acc[i]);
    }
#pragma unroll
  for (int i = 0; i < WB; ++i) red[g][i][threadIdx.x % 32] = acc[i];
  __syncthreads();
  if (g < WB && b0 + g < B && c < r3) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t += red[k][g][threadIdx.x % 32];
    w[((long)a * B + b0 + g) * r3 + c] = t;
  }
}

// ---------------------------------------------------------------------------------------
// Per-head queries and the new token: w [r1][B][r3] = qt C[a];  qhat[b, h] = scale * sum_a U1[h, a] w[a, b], rotated at
// the new token's position prefix_len + cache_len[b]; the new key rotated in place; both appended.  C: the pools' type.
// An 8-bit cache's new rows go on as the cache stores them (one pool with RoPE: the key is the stored row, rotated).
// ---------------------------------------------------------------------------------------
template <typename T, typename C>
__global__ void __launch_bounds__(256) k_pg_queries(const float* __restrict__ w, const T* __restrict__ U1, float* __restrict__ qhat,
                                                    const float* __restrict__ k_parts, const float* __restrict__ v_parts, int shares,
                                                    float* __restrict__ knew, float* __restrict__ vnew, C* __restrict__ K,
                                                    C* __restrict__ V, uint8_t* __restrict__ Ks, uint8_t* __restrict__ Vs, const PagedView pv, const int32_t* __restrict__ cache_len,
                                                    int B, int nH, int r1, int r3, int t3, int Lmax, int prefix_len, float scale, int rope,
                                                    double base, const dec::RopeFreqs freqs, int append, int shared_kv, int shared_rope, unsigned int* err) {
  constexpr bool kQ8 = std::is_same<C, e4m3>::value;
  pdl_enter();
  const int b = blockIdx.x;
  __shared__ long dst_s;
  __shared__ float2 cs_s[kMaxPairs];          // (cos, sin) of the new token's position
  int L = cache_len[b];
  if (L < 0 || L >= Lmax) {
    if (threadIdx.x == 0 && blockIdx.y == 0) atomicOr(err, (unsigned)TA_DEVERR_BAD_CACHE_LEN);
    L = L < 0 ? 0 : Lmax - 1;
    append = 0;                               // a page is not written on the strength of a clamped length
  }
  const int half = (r3 + 1) / 2;
  if (rope)
    for (int i = threadIdx.x; i < r3 / 2; i += blockDim.x)
      cs_s[i] = dec::rope_cos_sin_theta(prefix_len + L, i < 128 ? freqs.theta[i] : pair_theta(i, r3, base));
  __syncthreads();
  for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < nH * half; i += gridDim.y * blockDim.x) {
    const int h = i / half, c = 2 * (i % half);
    float xe = 0.f, xo = 0.f;
#pragma unroll 4
    for (int a = 0; a < r1; ++a) {
      const float u = ld(U1 + (long)h * r1 + a);
      const float* wr = w + ((long)a * B + b) * r3 + c;
      xe = fmaf(u, wr[0], xe);
      if (c + 1 < r3) xo = fmaf(u, wr[1], xo);
    }
    xe *= scale; xo *= scale;
    float* q = qhat + ((long)b * nH + h) * r3 + c;
    if (rope) {
      const float2 cs = cs_s[c >> 1];
      q[0] = xe * cs.x - xo * cs.y;
      q[1] = xe * cs.y + xo * cs.x;
    } else {
      q[0] = xe;
      if (c + 1 < r3) q[1] = xo;
    }
  }
  if (blockIdx.y != 0) return;
  if (threadIdx.x == 0) dst_s = append ? paged_row(pv.table + (long)b * pv.max_pages, L, pv, err) : -1;
  for (int i = threadIdx.x; i < half; i += blockDim.x) {
    float xe = 0.f, xo = 0.f;
    for (int k = 0; k < shares; ++k) {
      const float* px = k_parts + ((long)k * B + b) * r3 + 2 * i;
      xe += px[0];
      if (2 * i + 1 < r3) xo += px[1];
    }
    const float2 cs = rope && !(kQ8 && shared_rope) ? cs_s[i] : make_float2(1.f, 0.f);
    knew[(long)b * r3 + 2 * i] = xe * cs.x - xo * cs.y;
    if (2 * i + 1 < r3) knew[(long)b * r3 + 2 * i + 1] = xe * cs.y + xo * cs.x;
  }
  for (int c = threadIdx.x; c < t3; c += blockDim.x) {
    float t = 0.f;
    for (int k = 0; k < shares; ++k) t += v_parts[((long)k * B + b) * t3 + c];
    vnew[(long)b * t3 + c] = t;
  }
  __syncthreads();
  [[maybe_unused]] const long rows = (long)pv.n_pages * pv.page_size;
  if constexpr (kQ8) {
    __shared__ uint32_t amax_s[2];
    if (threadIdx.x < 2) amax_s[threadIdx.x] = 0;
    __syncthreads();
    const bool write = dst_s >= 0 && TA_IDX_OK(err, dst_s, 1, rows);
    for (int part = 0; part < 2; ++part) {         // one pool: the value row is the pool's
      const int r = part == 0 ? r3 : t3;
      float* row = (part == 0 ? knew : vnew) + (long)b * r;
      uint32_t a = 0;
      for (int c = threadIdx.x; c < r; c += blockDim.x) a = max(a, q8::abs_bits(row[c]));
      atomicMax(&amax_s[part], a);
      __syncthreads();
      const int byte = q8::scale_byte(amax_s[part]);
      const float inv = q8::inverse(byte), sc = q8::scale(byte);
      const bool put = write && (part == 1 || !shared_kv);
      for (int c = threadIdx.x; c < r; c += blockDim.x) {
        const uint32_t code = q8::codes2(row[c] * inv, 0.f);
        row[c] = q8::values2(code).x * sc;
        if (put) (part == 0 ? K : V)[dst_s * r + c].v = (uint8_t)code;
      }
      if (put && threadIdx.x == 0) (part == 0 ? Ks : Vs)[dst_s] = (uint8_t)byte;
    }
    if (shared_rope) {
      __syncthreads();
      for (int i = threadIdx.x; i < half; i += blockDim.x) {
        const float xe = vnew[(long)b * r3 + 2 * i], xo = vnew[(long)b * r3 + 2 * i + 1];
        knew[(long)b * r3 + 2 * i] = xe * cs_s[i].x - xo * cs_s[i].y;
        knew[(long)b * r3 + 2 * i + 1] = xe * cs_s[i].y + xo * cs_s[i].x;
      }
    }
    return;
  } else {
  if (dst_s < 0) return;
  if (!shared_kv && TA_IDX_OK(err, dst_s, 1, rows))
    for (int c = threadIdx.x; c < r3; c += blockDim.x) st(K + dst_s * r3 + c, knew[(long)b * r3 + c]);
  if (TA_IDX_OK(err, dst_s, 1, rows))      // one pool: the value row, which is the un-rotated latent row
    for (int c = threadIdx.x; c < t3; c += blockDim.x) st(V + dst_s * t3 + c, vnew[(long)b * t3 + c]);
  }
}

// ---------------------------------------------------------------------------------------
// Attention partials of 16 query rows against one share of a list of keys.
//   own part    grid (ceil(nH / 16), splits, B): rows = heads of sequence z, keys = its cached slots and the new token
//   prefix      grid (ceil(B nH / 16), splits, 1): rows = all heads of all sequences, keys = the prefix
// Thread (row, l) of 16 x 16: scores of keys l and l + 16 of a 32-key tile, then output columns 4 l + 64 i .. + 3.
// Partial of (row, split): max, sum, unnormalised output; a share without keys leaves max = -inf, sum = 0, and its
// output is not written (and not read).
// ---------------------------------------------------------------------------------------
constexpr int AR = 16, AK = 32, kMaxO4 = 8;       // t3 <= 64 * kMaxO4
__host__ __device__ inline int pitch4(int r) { return (r + 3) / 4 * 4 + 4; }
__host__ __device__ inline size_t pg_attn_smem(int r3, int t3) {
  return sizeof(float) * ((size_t)(AR + AK) * pitch4(r3) + (size_t)AK * pitch4(t3) + AR * (AK + 1)) + sizeof(long) * AK;
}
template <typename T>
struct AttnArgs {
  const float* q;          // [rows, r3]
  const T *K, *V;          // pools
  const uint8_t *Ks, *Vs;  // scale bytes of an 8-bit cache's rows
  PagedView pv;            // table: row z of it is used (the prefix: its only row)
  const int32_t* cache_len;// nullptr: the prefix, n_keys keys
  const float *knew, *vnew;// [B, r3] rotated, [B, t3]
  int rows_per_z, n_keys, Lmax, r3, t3, splits;
  int rotate_keys, pos_base;   // one pool with latent RoPE: keys are formed by rotation; position of slot 0
  double base;
  float *part_o, *part_ml; // [z * rows_per_z + row][splits][t3] / [..][splits][2]
  unsigned int* err;
};
__device__ __forceinline__ float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 ld4(const bf16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
  return make_float4(a.x, a.y, b.x, b.y);
}

__device__ __forceinline__ float4 ld4(const e4m3* p) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  const float2 a = q8::values2(w), b = q8::values2(w >> 16);
  return make_float4(a.x, a.y, b.x, b.y);
}

// Rows of a tile to shared memory, zero-padded to the pitch.  VEC: r is a multiple of 4, so that rows can be read four
// elements at a time (a tile's loads are then in flight together instead of one after another).
template <bool VEC, typename T>
__device__ __forceinline__ void load_rows(float* __restrict__ out, const T* __restrict__ pool, const uint8_t* __restrict__ scales,
                                          const float* __restrict__ fresh, const long* __restrict__ rows_s, int r, int pitch) {
  constexpr bool kQ8 = std::is_same<T, e4m3>::value;
  if (VEC) {
    const int n4 = pitch / 4;
#pragma unroll 4
    for (int i = threadIdx.x; i < AK * n4; i += 256) {
      const int j = i / n4, c = (i - j * n4) * 4;
      const long rw = rows_s[j];
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c < r) {
        if (rw == -2) v = ld4(fresh + c);
        else if (rw >= 0) {
          v = ld4(pool + rw * r + c);
          if constexpr (kQ8) {
            const float sc = q8::scale(scales[rw]);
            v.x *= sc; v.y *= sc; v.z *= sc; v.w *= sc;
          }
        }
      }
      *reinterpret_cast<float4*>(out + j * pitch + c) = v;
    }
  } else {
    for (int i = threadIdx.x; i < AK * pitch; i += 256) {
      const int j = i / pitch, c = i - j * pitch;
      const long rw = rows_s[j];
      float v = c >= r ? 0.f : (rw == -2 ? fresh[c] : (rw >= 0 ? ld(pool + rw * r + c) : 0.f));
      if constexpr (kQ8)
        if (c < r && rw >= 0) v *= q8::scale(scales[rw]);
      out[i] = v;
    }
  }
}

template <bool VEC, typename T>
__global__ void __launch_bounds__(256) k_pg_attn(const AttnArgs<T> g) {
  pdl_enter();
  extern __shared__ __align__(16) float sm[];
  __shared__ double theta_s[kMaxPairs];
  const int rp = pitch4(g.r3), tp = pitch4(g.t3);
  float* qs = sm;                       // [AR][rp]
  float* Kt = qs + AR * rp;             // [AK][rp]
  float* Vt = Kt + AK * rp;             // [AK][tp]
  float* ps = Vt + AK * tp;             // [AR][AK + 1]
  long* rows_s = reinterpret_cast<long*>(ps + AR * (AK + 1));   // AR * (AK + 1) is even: 8-byte aligned
  const int tid = threadIdx.x, r = tid / 16, l = tid % 16;
  const int split = blockIdx.y, row0 = blockIdx.x * AR, z = blockIdx.z;
  const int row = row0 + r;
  const bool valid = row < g.rows_per_z;
  int L = 0, limit = g.n_keys;
  if (g.cache_len) {
    L = g.cache_len[z];
    L = L < 0 ? 0 : (L >= g.Lmax ? g.Lmax - 1 : L);
    limit = L + 1;
  }
  const int tiles = (limit + AK - 1) / AK;
  const int t_beg = (int)((long)tiles * split / g.splits), t_end = (int)((long)tiles * (split + 1) / g.splits);
  const int32_t* table = g.pv.table + (long)z * g.pv.max_pages;
  if (g.rotate_keys)
    for (int i = tid; i < g.r3 / 2; i += 256) theta_s[i] = pair_theta(i, g.r3, g.base);
  for (int i = tid; i < AR * rp; i += 256) {
    const int rr = i / rp, c = i % rp;
    qs[i] = (row0 + rr < g.rows_per_z && c < g.r3) ? g.q[((long)z * g.rows_per_z + row0 + rr) * g.r3 + c] : 0.f;
  }
  float m = -INFINITY, lsum = 0.f;
  float4 o[kMaxO4];
#pragma unroll
  for (int i = 0; i < kMaxO4; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int n4 = (g.r3 + 3) / 4;
  for (int t = t_beg; t < t_end; ++t) {
    const int k0 = t * AK;
    __syncthreads();
    if (tid < AK) {                     // -1: no such row (zeros), -2: the new token
      const int s = k0 + tid;
      rows_s[tid] = s >= limit ? -1 : (g.cache_len && s == L ? -2 : paged_row(table, s, g.pv, g.err));
    }
    __syncthreads();
    load_rows<VEC>(Kt, g.K, g.Ks, g.knew + (long)z * g.r3, rows_s, g.r3, rp);
    load_rows<VEC>(Vt, g.V, g.Vs, g.vnew + (long)z * g.t3, rows_s, g.t3, tp);
    __syncthreads();
    if (g.rotate_keys) {                // one pool with latent RoPE: the key is the cached row, rotated (the new token's is already)
      const int half = g.r3 / 2;
      for (int i = tid; i < AK * half; i += 256) {
        const int j = i / half, c = i - j * half;
        if (rows_s[j] < 0) continue;
        const float2 cs = dec::rope_cos_sin_theta(g.pos_base + k0 + j, theta_s[c]);
        float* px = Kt + j * rp + 2 * c;
        const float xe = px[0], xo = px[1];
        px[0] = xe * cs.x - xo * cs.y;
        px[1] = xe * cs.y + xo * cs.x;
      }
      __syncthreads();
    }
    float s0 = 0.f, s1 = 0.f;
    const float4* q4 = reinterpret_cast<const float4*>(qs + r * rp);
    const float4* ka = reinterpret_cast<const float4*>(Kt + l * rp);
    const float4* kb = reinterpret_cast<const float4*>(Kt + (l + 16) * rp);
    for (int c = 0; c < n4; ++c) {
      const float4 q = q4[c], a = ka[c], b = kb[c];
      s0 = fmaf(q.x, a.x, s0); s0 = fmaf(q.y, a.y, s0); s0 = fmaf(q.z, a.z, s0); s0 = fmaf(q.w, a.w, s0);
      s1 = fmaf(q.x, b.x, s1); s1 = fmaf(q.y, b.y, s1); s1 = fmaf(q.z, b.z, s1); s1 = fmaf(q.w, b.w, s1);
    }
    if (k0 + l >= limit) s0 = -INFINITY;
    if (k0 + l + 16 >= limit) s1 = -INFINITY;
    float mt = fmaxf(s0, s1);
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, d));
    const float mn = fmaxf(m, mt);      // a tile holds at least one key below `limit`
    const float p0 = expf(s0 - mn), p1 = expf(s1 - mn), f = expf(m - mn);
    float pt = p0 + p1;
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) pt += __shfl_xor_sync(0xffffffffu, pt, d);
    lsum = lsum * f + pt;
    m = mn;
    ps[r * (AK + 1) + l] = p0;
    ps[r * (AK + 1) + l + 16] = p1;
    __syncwarp();                       // a row's 16 threads are half a warp
#pragma unroll
    for (int i = 0; i < kMaxO4; ++i)
      if (4 * l + 64 * i < g.t3) { o[i].x *= f; o[i].y *= f; o[i].z *= f; o[i].w *= f; }
    for (int j = 0; j < AK; ++j) {
      const float p = ps[r * (AK + 1) + j];
      const float4* v4 = reinterpret_cast<const float4*>(Vt + j * tp);
#pragma unroll
      for (int i = 0; i < kMaxO4; ++i)
        if (4 * l + 64 * i < g.t3) {
          const float4 v = v4[l + 16 * i];
          o[i].x = fmaf(p, v.x, o[i].x); o[i].y = fmaf(p, v.y, o[i].y);
          o[i].z = fmaf(p, v.z, o[i].z); o[i].w = fmaf(p, v.w, o[i].w);
        }
    }
  }
  if (!valid) return;
  const long slot = ((long)z * g.rows_per_z + row) * g.splits + split;
  if (l == 0) { g.part_ml[2 * slot] = m; g.part_ml[2 * slot + 1] = lsum; }
  if (t_beg >= t_end) return;
  float* po = g.part_o + slot * g.t3;
#pragma unroll
  for (int i = 0; i < kMaxO4; ++i) {
    const int c = 4 * l + 64 * i;
    const float v[4] = {o[i].x, o[i].y, o[i].z, o[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < g.t3) po[c + e] = v[e];
  }
}

// ---------------------------------------------------------------------------------------
// o[b, h] from the partials of its own keys (splits_o) and of the prefix (splits_p, may be 0).  A block per (b, h); the
// partials are dealt over its eight warps, whose sums are joined in order.
// ---------------------------------------------------------------------------------------
constexpr int kMaxSplits = 128;       // of either kind, see pick_splits
__global__ void __launch_bounds__(256) k_pg_merge(const float* __restrict__ po, const float* __restrict__ ml, int splits_o,
                                                  const float* __restrict__ po_p, const float* __restrict__ ml_p, int splits_p,
                                                  float* __restrict__ o, int t3) {
  pdl_enter();
  __shared__ float w_s[2 * kMaxSplits], red_s[8], acc_s[8][64];
  const long row = blockIdx.x;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const float2* a = reinterpret_cast<const float2*>(ml) + row * splits_o;
  const float2* p = reinterpret_cast<const float2*>(ml_p) + row * splits_p;
  const int n = splits_o + splits_p;    // at most 256: one partial per thread
  const float2 v = tid < n ? (tid < splits_o ? a[tid] : p[tid - splits_o]) : make_float2(-INFINITY, 0.f);
  float m = v.x;
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (lane == 0) red_s[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, red_s[i]);      // the new token's share holds a key: finite
  const float wt = v.y > 0.f ? expf(v.x - m) : 0.f;        // a share without keys wrote no output
  if (tid < n) w_s[tid] = wt;
  float l = v.y * wt;
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
  __syncthreads();                      // red_s is read above
  if (lane == 0) red_s[warp] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) l += red_s[i];
  const float inv = 1.f / l;
  for (int c0 = 0; c0 < t3; c0 += 64) { // 64 columns at a time, two per lane
    float s0 = 0.f, s1 = 0.f;
    const int c = c0 + lane;
#pragma unroll 4
    for (int i = warp; i < n; i += 8) {
      const float wi = w_s[i];
      if (wi == 0.f) continue;
      const float* src = i < splits_o ? po + (row * splits_o + i) * t3 : po_p + (row * splits_p + (i - splits_o)) * t3;
      if (c < t3) s0 = fmaf(wi, src[c], s0);
      if (c + 32 < t3) s1 = fmaf(wi, src[c + 32], s1);
    }
    acc_s[warp][lane] = s0;
    acc_s[warp][lane + 32] = s1;
    __syncthreads();
    if (tid < 64 && c0 + tid < t3) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t += acc_s[i][tid];
      o[row * t3 + c0 + tid] = t * inv;
    }
    __syncthreads();
  }
}

// Output-side core: u[b, a, c] = sum_h Ut1[h, a] o[b, h, c];  z[b, j] = sum_a sum_c Ct[a, j, c] u[b, a, c] (a warp per
// j).
template <typename T>
__global__ void __launch_bounds__(256) k_pg_u(const float* __restrict__ o, const T* __restrict__ Ut1, float* __restrict__ u, int B,
                                              int nH, int t1, int t3) {
  pdl_enter();
  const long total = (long)B * t1 * t3;
  for (long i = blockIdx.x * 256L + threadIdx.x; i < total; i += gridDim.x * 256L) {
    const int c = (int)(i % t3), a = (int)((i / t3) % t1), b = (int)(i / ((long)t3 * t1));
    float acc = 0.f;
#pragma unroll 4
    for (int h = 0; h < nH; ++h) acc = fmaf(ld(Ut1 + (long)h * t1 + a), o[((long)b * nH + h) * t3 + c], acc);
    u[i] = acc;
  }
}
template <typename T>
__global__ void __launch_bounds__(256) k_pg_z(const float* __restrict__ u, const T* __restrict__ Ct, float* __restrict__ z, int t1,
                                              int t2, int t3) {
  pdl_enter();
  const int b = blockIdx.y, j = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
  if (j >= t2) return;
  float acc = 0.f;
  const float* ub = u + (long)b * t1 * t3;
#pragma unroll 8
  for (int i = lane; i < t1 * t3; i += 32) {
    const int a = i / t3, c = i - a * t3;
    acc = fmaf(ld(Ct + ((long)a * t2 + j) * t3 + c), ub[i], acc);
  }
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
  if (lane == 0) z[(long)b * t2 + j] = acc;
}

// ---- host side ----------------------------------------------------------------------------------------------------

constexpr int kMaxAttnSmem = 200 * 1024, kMaxQuerySmem = 160 * 1024;
bool shape_ok(const tucker_attn_desc& d) {
  return d.t3 <= 64 * kMaxO4 && d.r3 <= 2 * kMaxPairs && pg_attn_smem(d.r3, d.t3) <= kMaxAttnSmem &&
         WB * (size_t)d.r2 * sizeof(float) <= kMaxQuerySmem;
}

// SMs that the shares are laid out for: B200's, whatever device is current, so that a workspace query does not depend on
// it.
constexpr int kSms = 148;
// Shares per list of keys: about two blocks per SM, no more than there are tiles.
int pick_splits(long blocks, long keys) {
  const long tiles = (keys + AK - 1) / AK;
  return (int)std::max<long>(1, std::min<long>(std::min<long>(tiles, kMaxSplits), (2 * kSms + blocks - 1) / blocks));
}
int own_splits(const tucker_attn_desc& d, int64_t Lmax) { return pick_splits((long)d.B * ((d.n_H + AR - 1) / AR), Lmax); }
int prefix_splits(const tucker_attn_desc& d, int32_t P) { return P > 0 ? pick_splits(((long)d.B * d.n_H + AR - 1) / AR, P) : 0; }

// Shares of K = d of the new tokens' projections: one 128-deep block each while few tiles would otherwise be all there
// is.
int proj_shares(const tucker_attn_desc& d) {
  const int kb = (d.d_model + GK - 1) / GK;
  return d.B <= 4 * GM ? std::min(kb, 8) : 1;
}

struct Ws {
  float *qt_parts, *k_parts, *v_parts, *knew, *vnew, *w, *qhat, *po, *ml, *po_p, *ml_p, *o, *u, *z;
};
size_t carve(const tucker_attn_desc& d, int64_t Lmax, int32_t P, char* base, Ws* out) {
  Carver c(base);
  Ws t;
  const size_t B = d.B, rows = B * d.n_H, so = own_splits(d, Lmax), sp = prefix_splits(d, P);
  const size_t sh = proj_shares(d);
  t.qt_parts = c.take<float>(sh * B * d.r2);
  t.k_parts = c.take<float>(sh * B * d.r3);
  t.v_parts = c.take<float>(sh * B * d.t3);
  t.knew = c.take<float>(B * d.r3);
  t.vnew = c.take<float>(B * d.t3);
  t.w = c.take<float>(B * d.r1 * d.r3);
  t.qhat = c.take<float>(rows * d.r3);
  t.po = c.take<float>(rows * so * d.t3);
  t.ml = c.take<float>(rows * so * 2);
  t.po_p = c.take<float>(rows * sp * d.t3);
  t.ml_p = c.take<float>(rows * sp * 2);
  t.o = c.take<float>(rows * d.t3);
  t.u = c.take<float>(B * d.t1 * d.t3);
  t.z = c.take<float>(B * d.t2);
  if (out) *out = t;
  return c.off;
}

template <typename TA, typename TB, typename TC>
int launch_gemm(Problem& p, const GemmArgs<TA, TB, TC>& g, int max_n) {
  const int kb = (g.K + GK - 1) / GK, shares = (kb + g.kb_per_split - 1) / g.kb_per_split;
  (void)launch_pdl(k_pg_gemm<TA, TB, TC>, dim3((g.M + GM - 1) / GM, (max_n + GN - 1) / GN, g.parts * shares), dim3(GT), 0, p.stream, g);
  TA_LAUNCH_CHECK(p);
  return TA_OK;
}

template <typename T>
int attn(Problem& p, const AttnArgs<T>& g, int zs) {
  const size_t smem = pg_attn_smem(g.r3, g.t3);
  const bool vec = g.r3 % 4 == 0 && g.t3 % 4 == 0;
  const auto kernel = vec ? k_pg_attn<true, T> : k_pg_attn<false, T>;
  static PerDeviceFlag attr_vec, attr_any;
  TA_CUDA_TRY(ensure_dynamic_smem(vec ? attr_vec : attr_any, (const void*)kernel, kMaxAttnSmem));
  (void)launch_pdl(kernel, dim3((g.rows_per_z + AR - 1) / AR, g.splits, zs), dim3(256), smem, p.stream, g);
  TA_LAUNCH_CHECK(p);
  return TA_OK;
}

template <typename T, typename C>      // C: the pools' type
int decode_typed(Problem& p) {
  const tucker_attn_desc& d = p.d;
  const int P = p.prefix_len;
  Ws w;
  carve(d, p.Lmax, P, p.ws, &w);
  int rc;
  const int kb = (d.d_model + GK - 1) / GK, per = (kb + proj_shares(d) - 1) / proj_shares(d), shares = (kb + per - 1) / per;
  {
    GemmArgs<T, T, float> g = {};
    g.A = (const T*)p.X; g.lda = d.d_model; g.M = d.B; g.K = d.d_model; g.parts = 3; g.kb_per_split = per;
    g.part[0] = {(const T*)p.U2, {d.r2, 1}, w.qt_parts, d.r2, d.r2, (long)d.B * d.r2};
    g.part[1] = {(const T*)p.U3, {d.r3, 1}, w.k_parts, d.r3, d.r3, (long)d.B * d.r3};
    g.part[2] = {(const T*)p.Ut3, {d.t3, 1}, w.v_parts, d.t3, d.t3, (long)d.B * d.t3};
    if ((rc = launch_gemm(p, g, std::max(d.r2, std::max(d.r3, d.t3))))) return rc;
  }
  static PerDeviceFlag attr_w;
  TA_CUDA_TRY(ensure_dynamic_smem(attr_w, (const void*)k_pg_w<T>, kMaxQuerySmem));
  (void)launch_pdl(k_pg_w<T>, dim3((d.B + WB - 1) / WB, d.r1, (d.r3 + 31) / 32), dim3(256), WB * d.r2 * sizeof(float), p.stream, w.qt_parts,
                   shares, (const T*)p.C, w.w, d.B, d.r1, d.r2, d.r3);
  TA_LAUNCH_CHECK(p);
  (void)launch_pdl(k_pg_queries<T, C>, dim3(d.B, std::max(1, std::min(8, 2 * kSms / d.B))), dim3(256), 0, p.stream, w.w, (const T*)p.U1, w.qhat,
                   w.k_parts, w.v_parts, shares, w.knew, w.vnew, (C*)p.Kc, (C*)p.Vc, p.Ks, p.Vs, p.pv, p.cache_len, d.B, d.n_H, d.r1, d.r3, d.t3, p.Lmax,
                   P, p.scale, d.rope, (double)d.rope_base, rope_freqs(d), p.append, p.shared_kv, p.shared_rope, p.dev_err);
  TA_LAUNCH_CHECK(p);
  AttnArgs<C> a = {};
  a.q = w.qhat; a.K = (const C*)p.Kc; a.V = (const C*)p.Vc; a.Ks = p.Ks; a.Vs = p.Vs; a.pv = p.pv; a.cache_len = p.cache_len;
  a.knew = w.knew; a.vnew = w.vnew; a.rows_per_z = d.n_H; a.Lmax = p.Lmax; a.r3 = d.r3; a.t3 = d.t3;
  a.splits = own_splits(d, p.Lmax); a.rotate_keys = p.shared_rope; a.pos_base = P; a.base = (double)d.rope_base;
  a.part_o = w.po; a.part_ml = w.ml; a.err = p.dev_err;
  prof_begin(p);
  if ((rc = attn(p, a, d.B))) return rc;
  const int sp = prefix_splits(d, P);
  if (P > 0) {
    a.pv.table = p.prefix_table; a.pv.max_pages = (P + p.pv.page_size - 1) / p.pv.page_size;
    a.cache_len = nullptr; a.n_keys = P; a.pos_base = 0; a.rows_per_z = d.B * d.n_H; a.splits = sp;
    a.part_o = w.po_p; a.part_ml = w.ml_p;
    if ((rc = attn(p, a, 1))) return rc;
  }
  prof_end(p);
  const int rows = d.B * d.n_H;
  (void)launch_pdl(k_pg_merge, dim3(rows), dim3(256), 0, p.stream, w.po, w.ml, own_splits(d, p.Lmax), w.po_p, w.ml_p, sp, w.o, d.t3);
  TA_LAUNCH_CHECK(p);
  (void)launch_pdl(k_pg_u<T>, dim3((unsigned)std::min<long>(kSms * 8, ((long)d.B * d.t1 * d.t3 + 255) / 256)), dim3(256), 0, p.stream, w.o,
                   (const T*)p.Ut1, w.u, d.B, d.n_H, d.t1, d.t3);
  TA_LAUNCH_CHECK(p);
  (void)launch_pdl(k_pg_z<T>, dim3((d.t2 + 7) / 8, d.B), dim3(256), 0, p.stream, w.u, (const T*)p.Ct, w.z, d.t1, d.t2, d.t3);
  TA_LAUNCH_CHECK(p);
  GemmArgs<float, T, T> g = {};
  g.A = w.z; g.lda = d.t2; g.M = d.B; g.K = d.t2; g.parts = 1; g.kb_per_split = (d.t2 + GK - 1) / GK;
  g.part[0] = {(const T*)p.Ut2, {1, d.t2}, (T*)p.Y, d.d_model, d.d_model, 0};
  return launch_gemm(p, g, d.d_model);
}

template <typename T>
int append_q8_typed(Problem& p, const int32_t* tok_start, int32_t T_) {
  const tucker_attn_desc& d = p.d;
  Carver c(p.ws);
  float* k = p.shared_kv ? nullptr : c.take<float>((size_t)T_ * d.r3);
  float* v = c.take<float>((size_t)T_ * d.t3);
  GemmArgs<T, T, float> g = {};
  g.A = (const T*)p.X; g.lda = d.d_model; g.M = T_; g.K = d.d_model; g.kb_per_split = (d.d_model + GK - 1) / GK;
  g.part[g.parts++] = {(const T*)p.Ut3, {d.t3, 1}, v, d.t3, d.t3, 0};
  if (k) g.part[g.parts++] = {(const T*)p.U3, {d.r3, 1}, k, d.r3, d.r3, 0};
  const int rc = launch_gemm(p, g, k ? std::max(d.r3, d.t3) : d.t3);
  if (rc) return rc;
  return q8_store_rows(p, k ? k : v, v, TA_DTYPE_F32, k && d.rope, tok_start, T_);
}

template <typename T>
int append_typed(Problem& p, const int32_t* tok_start, int32_t T_) {
  const tucker_attn_desc& d = p.d;
  AppendArgs<T> g = {};
  g.X = (const T*)p.X; g.U3 = (const T*)p.U3; g.Ut3 = (const T*)p.Ut3;
  g.K = (T*)p.Kc; g.V = (T*)p.Vc; g.pv = p.pv; g.tok_start = tok_start; g.cache_len = p.cache_len;
  g.B = d.B; g.T_ = T_; g.d = d.d_model; g.r3 = d.r3; g.t3 = d.t3; g.rope = d.rope; g.pos0 = d.pos0;
  g.keys_shared = p.shared_kv; g.base = (double)d.rope_base; g.turns = rope_turns(d); g.err = p.dev_err;
  const int wide = p.shared_kv ? d.t3 : std::max(d.r3, d.t3);
  (void)launch_pdl(k_pg_append<T>, dim3((T_ + GM - 1) / GM, (wide + GN - 1) / GN, p.shared_kv ? 1 : 2), dim3(GT), 0, p.stream, g);
  TA_LAUNCH_CHECK(p);
  return TA_OK;
}

}  // namespace

size_t generic_paged_decode_workspace(const tucker_attn_desc& d, int64_t Lmax, int32_t prefix_len) {
  return shape_ok(d) ? carve(d, Lmax, prefix_len, nullptr, nullptr) : 0;
}

int generic_paged_decode(Problem& p) {
  if (!shape_ok(p.d)) return TA_ERR_UNSUPPORTED_SHAPE;
  if (p.q8) return p.d.dtype == TA_DTYPE_F32 ? decode_typed<float, e4m3>(p) : decode_typed<bf16, e4m3>(p);
  return p.d.dtype == TA_DTYPE_F32 ? decode_typed<float, float>(p) : decode_typed<bf16, bf16>(p);
}

size_t generic_q8_append_workspace(const tucker_attn_desc& d, int32_t T, bool one_pool) {
  Carver c(nullptr);
  if (!one_pool) c.take<float>((size_t)T * d.r3);
  c.take<float>((size_t)T * d.t3);
  return c.off;
}

int generic_paged_append(Problem& p, const int32_t* tok_start, int32_t T) {
  if (p.q8) return p.d.dtype == TA_DTYPE_F32 ? append_q8_typed<float>(p, tok_start, T) : append_q8_typed<bf16>(p, tok_start, T);
  return p.d.dtype == TA_DTYPE_F32 ? append_typed<float>(p, tok_start, T) : append_typed<bf16>(p, tok_start, T);
}

}  // namespace ta
