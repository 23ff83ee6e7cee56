// Rows of the 8-bit paged cache: latent rows quantised into their pages, and read back.
//
// Both move each byte once and compute next to nothing: 1.5 to 2.5 times as many bytes per element on the row side as on the
// page side.  LPR lanes hold one row, eight numbers each (16 bytes of bf16, 8 of codes), so that a row's largest number is a
// shuffle away and a warp's loads and stores are whole rows next to each other.  A row's place (its sequence, the table, two
// divisions) is 80 instructions and a chain of loads.  One lane finds it, not all of the row's, and where there are more rows than
// the GPU has threads for, a warp finds those of kRows times as many rows at once.  112 thousand rows of 128 and 128 read (87 MB, 13.4 us
// at the copy rate): 27.3 us with a search per thread, 25.6 with four rows each, 14.8 with a search per row as well; 23 thousand
// rows stored 8.3 -> 6.8.
#include "ta_paged.cuh"
#include "ta_q8.cuh"

#include <algorithm>

namespace ta {
namespace {

constexpr int kThreads = 256, kMaxSteps = 5, kRows = 4;         // rows of up to 32 * 8 * kMaxSteps numbers

struct RowsArgs {
  const void* rows_in[2];    // store: [T, r] of type T, keys and values
  void* rows_out[2];         // read
  uint8_t* codes[2];         // pools
  uint8_t* scales[2];
  int r[2];
  PagedView pv;
  const int32_t *tok_start, *slots;      // slots: [B] tokens cached before (store) or first slot (read)
  int B, T, pos0;
  int rope;                  // store: keys are rotated on their way
  double base;
  dec::RopeTurns turns;      // of the first 128 pairs; those behind are formed from `base`
  unsigned int* err;
};

__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16* p, float (&f)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
    w[e] = *reinterpret_cast<const uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// Places of a warp's rows t0, t0 + 1 ..: lane i looks row i up.  Row -1: no cache row for it; `room`: whether the row is a token
// of a sequence that its table has room for.
struct Places {
  long row;
  int pos;
  bool room;
  __device__ __forceinline__ Places(const RowsArgs& g, long t0, int n, int lane, int pos0) : row(-1), pos(0), room(false) {
    if (lane >= n || t0 + lane >= g.T) return;
    const AppendDst d = append_dst((int)(t0 + lane), g.tok_start, g.slots, g.B, pos0, g.pv, g.err, &room);
    pos = d.pos;
    if (d.row >= 0 && TA_IDX_OK(g.err, d.row, 1, (long)g.pv.n_pages * g.pv.page_size)) row = d.row;
  }
};

// VEC: both widths are multiples of eight, so that a row's pieces of eight are whole and aligned.
template <typename T, int LPR, int STEPS, bool VEC, int ROWS>
__global__ void __launch_bounds__(kThreads) k_q8_store(const __grid_constant__ RowsArgs g) {
  pdl_enter();
  constexpr int W = 32 / LPR;                    // rows of a warp at a time
  const int part = blockIdx.y, r = g.r[part], lane = threadIdx.x % 32, sub = lane % LPR;
  const long t0 = ((long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * (W * ROWS);
  const T* const rows = static_cast<const T*>(g.rows_in[part]);
  float v[ROWS][STEPS][8];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const long t = t0 + i * W + lane / LPR;
    const bool there = t < g.T;
    const T* row = rows + (there ? t : 0) * r;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = (s * LPR + sub) * 8;
      if (VEC) {
        if (there && c < r) load8(row + c, v[i][s]);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][s][e] = 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][s][e] = there && c + e < r ? to_f(row[c + e]) : 0.f;
      }
    }
  }
  const Places mine(g, t0, W * ROWS, lane, g.pos0);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int from = i * W + lane / LPR;
    const long dst = __shfl_sync(0xffffffffu, mine.row, from);
    if (g.rope && part == 0) {
      const int pos = __shfl_sync(0xffffffffu, mine.pos, from);
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = (s * LPR + sub) * 4 + e;
          if (2 * k < r) {
            const float2 cs = k < 128 ? dec::rope_cos_sin_turn(pos, g.turns.turn[k])
                                      : dec::rope_cos_sin_theta(pos, pow(g.base, -2.0 * (double)k / (double)r));
            const float xe = v[i][s][2 * e], xo = v[i][s][2 * e + 1];
            v[i][s][2 * e] = xe * cs.x - xo * cs.y;
            v[i][s][2 * e + 1] = xe * cs.y + xo * cs.x;
          }
        }
    }
    uint32_t a = 0;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) a = max(a, q8::abs_bits(v[i][s][e]));
#pragma unroll
    for (int off = LPR / 2; off >= 1; off >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, off));
    if (dst < 0) continue;
    const int byte = q8::scale_byte(a);
    const float inv = q8::inverse(byte);
    uint8_t* out = g.codes[part] + dst * r;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = (s * LPR + sub) * 8;
      const uint2 w = q8::codes8(v[i][s], inv);
      if (VEC) {
        if (c < r) *reinterpret_cast<uint2*>(out + c) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < r) out[c + e] = (uint8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
      }
    }
    if (sub == 0) g.scales[part][dst] = (uint8_t)byte;
  }
}

template <typename T, int LPR, int STEPS, bool VEC, int ROWS>
__global__ void __launch_bounds__(kThreads) k_q8_read(const __grid_constant__ RowsArgs g) {
  pdl_enter();
  constexpr int W = 32 / LPR;
  const int part = blockIdx.y, r = g.r[part], lane = threadIdx.x % 32, sub = lane % LPR;
  const long t0 = ((long)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * (W * ROWS);
  const Places mine(g, t0, W * ROWS, lane, 0);
  const float my_scale = mine.row >= 0 ? q8::scale(g.scales[part][mine.row]) : 0.f;
  const uint8_t* in[ROWS];
  float sc[ROWS];
  bool room[ROWS], have[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int from = i * W + lane / LPR;
    const long src = __shfl_sync(0xffffffffu, mine.row, from);
    room[i] = __shfl_sync(0xffffffffu, (int)mine.room, from) != 0;
    sc[i] = __shfl_sync(0xffffffffu, my_scale, from);
    have[i] = src >= 0;
    in[i] = g.codes[part] + (have[i] ? src : 0) * r;
  }
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int c = (s * LPR + sub) * 8;
    uint2 w[ROWS];
    if (VEC) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) w[i] = have[i] && c < r ? *reinterpret_cast<const uint2*>(in[i] + c) : make_uint2(0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (!room[i]) continue;
      T* row = static_cast<T*>(g.rows_out[part]) + (t0 + i * W + lane / LPR) * r;
      if (VEC) {
        if (c < r) {
          float f[8];
          q8::values8(w[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] *= sc[i];
          store8(row + c, f);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < r) put(row + c + e, have[i] ? q8::value(in[i][c + e]) * sc[i] : 0.f);
      }
    }
  }
}

template <typename T, int LPR, int STEPS, bool VEC, int ROWS>
int launch_rows(Problem& p, const RowsArgs& g, bool store, int parts) {
  const long per = (long)kThreads / LPR * ROWS;
  prof_begin(p);
  (void)launch_pdl(store ? k_q8_store<T, LPR, STEPS, VEC, ROWS> : k_q8_read<T, LPR, STEPS, VEC, ROWS>, dim3((unsigned)((g.T + per - 1) / per), parts),
                   dim3(kThreads), 0, p.stream, g);
  prof_end(p);
  TA_LAUNCH_CHECK(p);
  return TA_OK;
}
template <typename T, int LPR, int STEPS, bool VEC>
int launch(Problem& p, const RowsArgs& g, bool store, int parts) {
  if constexpr (VEC && STEPS == 1)
    if ((long)g.T * parts * LPR > 2048L * sm_count()) return launch_rows<T, LPR, STEPS, VEC, kRows>(p, g, store, parts);      // more lanes than the GPU holds threads
  return launch_rows<T, LPR, STEPS, VEC, 1>(p, g, store, parts);
}

template <typename T>
int dispatch(Problem& p, const RowsArgs& g, bool store, int parts) {
  const int wide = parts > 1 ? std::max(g.r[0], g.r[1]) : g.r[0];
  const bool vec = g.r[0] % 8 == 0 && g.r[1] % 8 == 0;
  if (!vec) return wide <= 256 ? launch<T, 32, 1, false>(p, g, store, parts) : launch<T, 32, kMaxSteps, false>(p, g, store, parts);
  if (wide <= 64) return launch<T, 8, 1, true>(p, g, store, parts);
  if (wide <= 128) return launch<T, 16, 1, true>(p, g, store, parts);
  if (wide <= 256) return launch<T, 32, 1, true>(p, g, store, parts);
  return launch<T, 32, kMaxSteps, true>(p, g, store, parts);
}

RowsArgs args_of(const Problem& p, const int32_t* tok_start, int32_t T) {
  const tucker_attn_desc& d = p.d;
  RowsArgs g = {};
  g.codes[0] = (uint8_t*)p.Kc; g.codes[1] = (uint8_t*)p.Vc; g.scales[0] = p.Ks; g.scales[1] = p.Vs;
  g.r[0] = d.r3; g.r[1] = d.t3; g.pv = p.pv; g.tok_start = tok_start; g.slots = p.cache_len; g.B = d.B; g.T = T;
  g.pos0 = d.pos0; g.err = p.dev_err;
  return g;
}

}  // namespace

bool q8_rows_supported(const tucker_attn_desc& d) { return std::max(d.r3, d.t3) <= 256 * kMaxSteps; }

int q8_store_rows(Problem& p, const void* Krows, const void* Vrows, int dtype, bool rope, const int32_t* tok_start, int32_t T) {
  RowsArgs g = args_of(p, tok_start, T);
  g.rows_in[0] = Krows; g.rows_in[1] = Vrows;
  if (rope) { g.rope = 1; g.base = (double)p.d.rope_base; g.turns = rope_turns(p.d); }
  return dtype == TA_DTYPE_F32 ? dispatch<float>(p, g, true, p.shared_kv ? 1 : 2) : dispatch<bf16>(p, g, true, p.shared_kv ? 1 : 2);
}

int q8_read_rows(Problem& p, void* Krows, void* Vrows, const int32_t* tok_start, int32_t T) {
  RowsArgs g = args_of(p, tok_start, T);
  g.rows_out[0] = Krows; g.rows_out[1] = Vrows;
  return p.d.dtype == TA_DTYPE_F32 ? dispatch<float>(p, g, false, p.shared_kv ? 1 : 2) : dispatch<bf16>(p, g, false, p.shared_kv ? 1 : 2);
}

}  // namespace ta
