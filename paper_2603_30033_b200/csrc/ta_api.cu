// C ABI entry points: argument validation, path selection, workspace sizing, error word.
#include "ta_common.cuh"

#include <math.h>

namespace ta {

__device__ unsigned int g_device_error_word = 0;

static thread_local int tl_last_path = 0;
static thread_local int tl_last_launches = 0;
static thread_local cudaEvent_t tl_prof_start = nullptr;
static thread_local cudaEvent_t tl_prof_stop = nullptr;

static unsigned int* device_error_ptr() {
  // one address per device; looked up lazily, cached per device ordinal
  static unsigned int* cache[kMaxDevices] = {nullptr};
  static std::mutex m;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  std::lock_guard<std::mutex> lock(m);
  if (!cache[dev]) {
    void* ptr = nullptr;
    if (cudaGetSymbolAddress(&ptr, g_device_error_word) != cudaSuccess) return nullptr;
    cache[dev] = static_cast<unsigned int*>(ptr);
  }
  return cache[dev];
}

unsigned int* device_error_word() { return device_error_ptr(); }

static bool desc_ok(const tucker_attn_desc* d, bool decode) {
  if (!d) return false;
  if (d->B <= 0 || d->d_model <= 0 || d->n_H <= 0) return false;
  if (!decode && d->N <= 0) return false;
  if (d->d_model % d->n_H) return false;
  if (d->r1 <= 0 || d->r2 <= 0 || d->r3 <= 0 || d->t1 <= 0 || d->t2 <= 0 || d->t3 <= 0) return false;
  if (d->rope && (d->r3 % 2)) return false;
  if (d->rope && !(d->rope_base > 0.f)) return false;
  if (d->dtype != TA_DTYPE_F32 && d->dtype != TA_DTYPE_BF16) return false;
  return true;
}

static float resolve_scale(const tucker_attn_desc& d) {
  return d.scale > 0.f ? d.scale : (float)(1.0 / sqrt((double)d.d_model / (double)d.n_H));
}

static bool use_fast_fwd(const tucker_attn_desc& d) {
  return d.dtype == TA_DTYPE_BF16 && !(d.flags & TA_FLAG_FORCE_GENERIC) && fast_fwd_supported(d);
}
static bool use_fast_decode(const tucker_attn_desc& d, int32_t Lmax) {
  return d.dtype == TA_DTYPE_BF16 && !(d.flags & TA_FLAG_FORCE_GENERIC) && fast_decode_supported(d, Lmax);
}

// Shared key / value projection (Sec. 3.1, L^KV = X U3): the caller passes the SAME factor for U3 and Ut3.
// Without RoPE the latent keys are then the latent values, so one projection and one cache serve both.
// With latent RoPE the one cache holds the un-rotated latent rows (the values); keys are rotated when used.
static bool shared_kv_weights(const tucker_attn_desc& d, const void* U3, const void* Ut3) {
  return U3 == Ut3 && d.r3 == d.t3;
}

// A paged cache's host-side description.  Slots are counted in 32 bits: max_pages * page_size + `before` (the tokens in
// front of slot 0) must stay below 2^31 - 4096, so that a tile that starts at an existing slot ends in 32 bits.
static bool paged_ok(const tucker_paged_cache* c, int64_t before) {
  if (!c || !c->K || !c->V || !c->block_table) return false;
  if (c->n_pages <= 0 || c->page_size <= 0 || c->max_pages <= 0 || before < 0) return false;
  return (int64_t)c->max_pages * c->page_size + before < ((int64_t)1 << 31) - 4096;
}
static int64_t paged_slots(const tucker_paged_cache& c) { return (int64_t)c.max_pages * c.page_size; }

// Either kind of paged cache; the 8-bit one has scales.
struct CacheArgs {
  tucker_paged_cache c;
  uint8_t *Ks, *Vs;
  int q8;
  bool one_pool() const { return c.K == c.V; }
};
static CacheArgs cache_args(const tucker_paged_cache* c) { return CacheArgs{c ? *c : tucker_paged_cache{}, nullptr, nullptr, 0}; }
static CacheArgs cache_args(const tucker_paged_cache_q8* c) {
  if (!c) return CacheArgs{};
  return CacheArgs{{c->K, c->V, c->block_table, c->n_pages, c->page_size, c->max_pages}, (uint8_t*)c->Ks, (uint8_t*)c->Vs, 1};
}

// Grid limits of the paged kernels.
static bool paged_batch_ok(const tucker_attn_desc& d) { return d.B <= 65535 && (int64_t)d.B * d.n_H <= (1 << 24); }

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static bool cache_ok(const CacheArgs& a, int64_t before) {
  if (!paged_ok(&a.c, before)) return false;
  if (!aligned16(a.c.K) || !aligned16(a.c.V)) return false;
  return !a.q8 || (a.Ks && a.Vs && aligned16(a.Ks) && aligned16(a.Vs) && (a.Ks == a.Vs) == a.one_pool());
}
static void put_cache(Problem& p, const CacheArgs& a) {
  p.Kc = a.c.K; p.Vc = a.c.V; p.Ks = a.Ks; p.Vs = a.Vs; p.q8 = a.q8;
  p.paged = 1;
  p.pv = PagedView{a.c.block_table, a.c.n_pages, a.c.page_size, a.c.max_pages};
  p.shared_kv = a.one_pool() ? 1 : 0;
  p.shared_rope = (p.shared_kv && p.d.rope) ? 1 : 0;
}

}  // namespace ta

using namespace ta;

extern "C" {

size_t tucker_attn_fwd_workspace_bytes(const tucker_attn_desc* desc) {
  if (!desc_ok(desc, false)) return 0;
  return use_fast_fwd(*desc) ? fast_fwd_workspace(*desc) : generic_fwd_workspace(*desc);
}

size_t tucker_attn_decode_workspace_bytes(const tucker_attn_desc* desc, int32_t Lmax) {
  if (!desc_ok(desc, true) || Lmax <= 0) return 0;
  return use_fast_decode(*desc, Lmax) ? fast_decode_workspace(*desc, Lmax) : generic_decode_workspace(*desc, Lmax);
}

int tucker_attn_fwd(const tucker_attn_desc* desc, const void* X, const void* C, const void* U1, const void* U2,
                    const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3, void* Y,
                    void* Kcache_out, void* Vcache_out, int32_t Lmax, void* workspace, size_t workspace_bytes,
                    void* cuda_stream) {
  if (!desc_ok(desc, false)) return TA_ERR_INVALID_ARG;
  if (!X || !C || !U1 || !U2 || !U3 || !Ct || !Ut1 || !Ut2 || !Ut3 || !Y || !workspace) return TA_ERR_INVALID_ARG;
  if ((Kcache_out == nullptr) != (Vcache_out == nullptr)) return TA_ERR_INVALID_ARG;
  if (Kcache_out && Lmax < desc->N) return TA_ERR_INVALID_ARG;
  if (Kcache_out && Kcache_out == Vcache_out && !shared_kv_weights(*desc, U3, Ut3)) return TA_ERR_INVALID_ARG;
  const void* ptrs[] = {X, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Y};
  for (const void* q : ptrs)
    if (!aligned16(q)) return TA_ERR_INVALID_ARG;
  if (Kcache_out && (!aligned16(Kcache_out) || !aligned16(Vcache_out))) return TA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return TA_ERR_INVALID_ARG;
  const bool fast = use_fast_fwd(*desc);
  const size_t need = fast ? fast_fwd_workspace(*desc) : generic_fwd_workspace(*desc);
  if (need == 0) return TA_ERR_UNSUPPORTED_SHAPE;
  if (workspace_bytes < need) return TA_ERR_WORKSPACE_TOO_SMALL;
  Problem p = {};
  p.d = *desc;
  p.scale = resolve_scale(*desc);
  p.X = X; p.C = C; p.U1 = U1; p.U2 = U2; p.U3 = U3; p.Ct = Ct; p.Ut1 = Ut1; p.Ut2 = Ut2; p.Ut3 = Ut3;
  p.Y = Y; p.Kc = Kcache_out; p.Vc = Vcache_out; p.Lmax = Lmax;
  p.cache_len = nullptr; p.append = 0;
  const bool one_cache = shared_kv_weights(*desc, U3, Ut3) && Kcache_out == Vcache_out;
  p.shared_kv = (one_cache && !desc->rope) ? 1 : 0;                   // one projection serves keys and values
  p.shared_rope = (one_cache && desc->rope && Kcache_out) ? 1 : 0;    // rotated keys computed, un-rotated rows cached
  p.ws = static_cast<char*>(workspace); p.ws_bytes = workspace_bytes;
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.launches = 0;
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  const int rc = fast ? fast_fwd(p) : generic_fwd(p);
  tl_last_path = fast ? 2 : 1;
  tl_last_launches = p.launches;
  return rc;
}

int tucker_attn_decode(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                       const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                       void* Kcache, void* Vcache, int32_t Lmax, const int32_t* cache_len, int32_t append, void* y,
                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!desc_ok(desc, true)) return TA_ERR_INVALID_ARG;
  if (!x || !C || !U1 || !U2 || !U3 || !Ct || !Ut1 || !Ut2 || !Ut3 || !y || !workspace) return TA_ERR_INVALID_ARG;
  if (!Kcache || !Vcache || !cache_len || Lmax <= 0) return TA_ERR_INVALID_ARG;
  if (Kcache == Vcache && !shared_kv_weights(*desc, U3, Ut3)) return TA_ERR_INVALID_ARG;
  const void* ptrs[] = {x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, y, Kcache, Vcache};
  for (const void* q : ptrs)
    if (!aligned16(q)) return TA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return TA_ERR_INVALID_ARG;
  const bool fast = use_fast_decode(*desc, Lmax);
  const size_t need = fast ? fast_decode_workspace(*desc, Lmax) : generic_decode_workspace(*desc, Lmax);
  if (need == 0) return TA_ERR_UNSUPPORTED_SHAPE;
  if (workspace_bytes < need) return TA_ERR_WORKSPACE_TOO_SMALL;
  Problem p = {};
  p.d = *desc;
  p.scale = resolve_scale(*desc);
  p.X = x; p.C = C; p.U1 = U1; p.U2 = U2; p.U3 = U3; p.Ct = Ct; p.Ut1 = Ut1; p.Ut2 = Ut2; p.Ut3 = Ut3;
  p.Y = y; p.Kc = Kcache; p.Vc = Vcache; p.Lmax = Lmax;
  p.cache_len = cache_len; p.append = append ? 1 : 0;
  p.shared_kv = (Kcache == Vcache) ? 1 : 0;
  p.shared_rope = (p.shared_kv && desc->rope) ? 1 : 0;
  p.ws = static_cast<char*>(workspace); p.ws_bytes = workspace_bytes;
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.launches = 0;
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  const int rc = fast ? fast_decode(p) : generic_decode(p);
  tl_last_path = fast ? 2 : 1;
  tl_last_launches = p.launches;
  return rc;
}

// Whether a step runs in its one-launch form, which needs no workspace.
static bool paged_decode_fast(const tucker_attn_desc& d, const CacheArgs& a) { return fast_paged_supported(d, a.c.page_size); }
static bool paged_decode_small(const tucker_attn_desc& d, const CacheArgs& a, int32_t prefix_len) {
  return paged_batch_ok(d) && cluster_step_supported(d, a.one_pool(), a.q8) &&
         cluster_step_pays(d, paged_slots(a.c), prefix_len, paged_decode_fast(d, a), a.q8);
}
static size_t paged_decode_need(const tucker_attn_desc& d, const CacheArgs& a, int32_t prefix_len) {
  if (!paged_batch_ok(d)) return 0;
  if (paged_decode_small(d, a, prefix_len)) return TA_WORKSPACE_NONE;
  if (paged_decode_fast(d, a)) return fast_paged_workspace(d, prefix_len, a.one_pool(), a.q8);
  return generic_paged_decode_workspace(d, paged_slots(a.c), prefix_len);
}
static size_t paged_decode_query(const tucker_attn_desc* desc, const CacheArgs& a, int32_t prefix_len) {
  return desc_ok(desc, true) && paged_ok(&a.c, prefix_len) ? paged_decode_need(*desc, a, prefix_len) : 0;
}

size_t tucker_attn_decode_paged_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache* cache) {
  return paged_decode_query(desc, cache_args(cache), 0);
}
size_t tucker_attn_decode_paged_q8_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache_q8* cache) {
  return paged_decode_query(desc, cache_args(cache), 0);
}
size_t tucker_attn_decode_prefix_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache* cache,
                                                 int32_t prefix_len) {
  return paged_decode_query(desc, cache_args(cache), prefix_len);
}
size_t tucker_attn_decode_prefix_q8_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache_q8* cache,
                                                    int32_t prefix_len) {
  return paged_decode_query(desc, cache_args(cache), prefix_len);
}

static int paged_decode(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                        const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                        const CacheArgs& a, const int32_t* cache_len, const int32_t* prefix_table,
                        int32_t prefix_len, int32_t append, void* y, void* workspace, size_t workspace_bytes,
                        void* cuda_stream) {
  if (!desc_ok(desc, true) || !cache_ok(a, prefix_len)) return TA_ERR_INVALID_ARG;
  if (!x || !C || !U1 || !U2 || !U3 || !Ct || !Ut1 || !Ut2 || !Ut3 || !y) return TA_ERR_INVALID_ARG;
  if (!cache_len || (prefix_len > 0 && !prefix_table)) return TA_ERR_INVALID_ARG;
  if (a.one_pool() && !shared_kv_weights(*desc, U3, Ut3)) return TA_ERR_INVALID_ARG;
  const void* ptrs[] = {x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, y};
  for (const void* q : ptrs)
    if (!aligned16(q)) return TA_ERR_INVALID_ARG;
  const size_t need = paged_decode_need(*desc, a, prefix_len);
  const bool small = need == TA_WORKSPACE_NONE;
  if (!small && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))) return TA_ERR_INVALID_ARG;
  if (need == 0) return TA_ERR_UNSUPPORTED_SHAPE;
  if (!small && workspace_bytes < need) return TA_ERR_WORKSPACE_TOO_SMALL;
  Problem p = {};
  p.d = *desc;
  p.scale = resolve_scale(*desc);
  p.X = x; p.C = C; p.U1 = U1; p.U2 = U2; p.U3 = U3; p.Ct = Ct; p.Ut1 = Ut1; p.Ut2 = Ut2; p.Ut3 = Ut3;
  p.Y = y; p.Lmax = (int32_t)paged_slots(a.c);
  p.cache_len = cache_len; p.append = append ? 1 : 0;
  put_cache(p, a);
  p.prefix_table = prefix_table; p.prefix_len = prefix_len;
  p.ws = static_cast<char*>(workspace); p.ws_bytes = workspace_bytes;
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  const bool fast = paged_decode_fast(*desc, a);
  const int rc = small ? cluster_paged_decode(p) : (fast ? fast_decode(p) : generic_paged_decode(p));
  tl_last_path = small ? 3 : (fast ? 2 : 1);
  tl_last_launches = p.launches;
  return rc;
}

int tucker_attn_decode_prefix(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                              const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                              const tucker_paged_cache* cache, const int32_t* cache_len, const int32_t* prefix_table,
                              int32_t prefix_len, int32_t append, void* y, void* workspace, size_t workspace_bytes,
                              void* cuda_stream) {
  return paged_decode(desc, x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, cache_args(cache), cache_len, prefix_table, prefix_len, append, y,
                      workspace, workspace_bytes, cuda_stream);
}
int tucker_attn_decode_prefix_q8(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                                 const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                                 const tucker_paged_cache_q8* cache, const int32_t* cache_len, const int32_t* prefix_table,
                                 int32_t prefix_len, int32_t append, void* y, void* workspace, size_t workspace_bytes,
                                 void* cuda_stream) {
  return paged_decode(desc, x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, cache_args(cache), cache_len, prefix_table, prefix_len, append, y,
                      workspace, workspace_bytes, cuda_stream);
}
int tucker_attn_decode_paged(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                             const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                             const tucker_paged_cache* cache, const int32_t* cache_len, int32_t append, void* y,
                             void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return paged_decode(desc, x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, cache_args(cache), cache_len, nullptr, 0, append, y, workspace,
                      workspace_bytes, cuda_stream);
}
int tucker_attn_decode_paged_q8(const tucker_attn_desc* desc, const void* x, const void* C, const void* U1, const void* U2,
                                const void* U3, const void* Ct, const void* Ut1, const void* Ut2, const void* Ut3,
                                const tucker_paged_cache_q8* cache, const int32_t* cache_len, int32_t append, void* y,
                                void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return paged_decode(desc, x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, cache_args(cache), cache_len, nullptr, 0, append, y, workspace,
                      workspace_bytes, cuda_stream);
}

static size_t append_query(const tucker_attn_desc* desc, const CacheArgs& a, int32_t T) {
  if (!desc_ok(desc, true) || !paged_ok(&a.c, desc->pos0) || T < 0) return 0;
  size_t need = 0;
  if (T > 0 && fast_append_supported(*desc)) need = fast_append_workspace(*desc, T, a.one_pool());
  else if (T > 0 && a.q8) need = generic_q8_append_workspace(*desc, T, a.one_pool());
  return need < 256 ? 256 : need;
}

size_t tucker_cache_append_paged_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache* cache, int32_t T) {
  return append_query(desc, cache_args(cache), T);
}
size_t tucker_cache_append_paged_q8_workspace_bytes(const tucker_attn_desc* desc, const tucker_paged_cache_q8* cache, int32_t T) {
  return append_query(desc, cache_args(cache), T);
}

static int append_tokens(const tucker_attn_desc* desc, const void* X, const void* U3, const void* Ut3, const CacheArgs& a,
                         const int32_t* cache_len, const int32_t* tok_start, int32_t T, void* workspace, size_t workspace_bytes,
                         void* cuda_stream) {
  if (!desc_ok(desc, true) || !cache_ok(a, desc->pos0) || T < 0) return TA_ERR_INVALID_ARG;
  if (!U3 || !Ut3 || !cache_len || !tok_start || !workspace || (T > 0 && !X)) return TA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return TA_ERR_INVALID_ARG;
  if (a.one_pool() && !shared_kv_weights(*desc, U3, Ut3)) return TA_ERR_INVALID_ARG;
  const void* ptrs[] = {X, U3, Ut3};
  for (const void* q : ptrs)
    if (!aligned16(q)) return TA_ERR_INVALID_ARG;
  if (a.q8 && !q8_rows_supported(*desc)) return TA_ERR_UNSUPPORTED_SHAPE;
  if (workspace_bytes < append_query(desc, a, T)) return TA_ERR_WORKSPACE_TOO_SMALL;
  Problem p = {};
  p.d = *desc;
  p.X = X; p.U3 = U3; p.Ut3 = Ut3; p.cache_len = cache_len;
  p.ws = static_cast<char*>(workspace); p.ws_bytes = workspace_bytes;
  put_cache(p, a);
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  const bool fast = fast_append_supported(*desc);
  const int rc = T == 0 ? TA_OK : (fast ? fast_append(p, tok_start, T) : generic_paged_append(p, tok_start, T));
  tl_last_path = fast ? 2 : 1;
  tl_last_launches = p.launches;
  return rc;
}

int tucker_cache_append_paged(const tucker_attn_desc* desc, const void* X, const void* U3, const void* Ut3,
                              const tucker_paged_cache* cache, const int32_t* cache_len, const int32_t* tok_start, int32_t T,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return append_tokens(desc, X, U3, Ut3, cache_args(cache), cache_len, tok_start, T, workspace, workspace_bytes, cuda_stream);
}
int tucker_cache_append_paged_q8(const tucker_attn_desc* desc, const void* X, const void* U3, const void* Ut3,
                                 const tucker_paged_cache_q8* cache, const int32_t* cache_len, const int32_t* tok_start, int32_t T,
                                 void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return append_tokens(desc, X, U3, Ut3, cache_args(cache), cache_len, tok_start, T, workspace, workspace_bytes, cuda_stream);
}

// Rows into (store) or out of an 8-bit cache.
static int move_rows(const tucker_attn_desc* desc, const void* Krows, const void* Vrows, const CacheArgs& a, const int32_t* slots,
                     const int32_t* tok_start, int32_t T, bool store, void* cuda_stream) {
  if (!desc_ok(desc, true) || !cache_ok(a, 0) || T < 0) return TA_ERR_INVALID_ARG;
  if (!slots || !tok_start || (T > 0 && (!Krows || !Vrows))) return TA_ERR_INVALID_ARG;
  if (!aligned16(Krows) || !aligned16(Vrows)) return TA_ERR_INVALID_ARG;
  if (a.one_pool() ? (desc->r3 != desc->t3 || Krows != Vrows) : (!store && T > 0 && Krows == Vrows)) return TA_ERR_INVALID_ARG;
  if (!q8_rows_supported(*desc)) return TA_ERR_UNSUPPORTED_SHAPE;
  Problem p = {};
  p.d = *desc;
  p.cache_len = slots;
  put_cache(p, a);
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  int rc = TA_OK;
  if (T > 0)
    rc = store ? q8_store_rows(p, Krows, Vrows, desc->dtype, false, tok_start, T)
               : q8_read_rows(p, const_cast<void*>(Krows), const_cast<void*>(Vrows), tok_start, T);
  tl_last_path = 1;
  tl_last_launches = p.launches;
  return rc;
}

int tucker_cache_store_paged_q8(const tucker_attn_desc* desc, const void* Krows, const void* Vrows,
                                const tucker_paged_cache_q8* cache, const int32_t* cache_len, const int32_t* tok_start, int32_t T,
                                void* cuda_stream) {
  return move_rows(desc, Krows, Vrows, cache_args(cache), cache_len, tok_start, T, true, cuda_stream);
}
int tucker_cache_read_paged_q8(const tucker_attn_desc* desc, const tucker_paged_cache_q8* cache, const int32_t* slot_start,
                               const int32_t* tok_start, int32_t T, void* Krows, void* Vrows, void* cuda_stream) {
  return move_rows(desc, Krows, Vrows, cache_args(cache), slot_start, tok_start, T, false, cuda_stream);
}

const char* tucker_attn_status_string(int status) {
  switch (status) {
    case TA_OK: return "ok";
    case TA_ERR_INVALID_ARG: return "invalid argument";
    case TA_ERR_UNSUPPORTED_SHAPE: return "unsupported shape";
    case TA_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
    case TA_ERR_CUDA: return "CUDA error";
    case TA_ERR_DEVICE_TIMEOUT: return "device-side wait timed out";
    default: return "unknown status";
  }
}

int tucker_attn_last_device_error(void* cuda_stream) {
  unsigned int* ptr = device_error_ptr();
  if (!ptr) return TA_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  unsigned int host = 0;
  if (cudaMemcpyAsync(&host, ptr, sizeof(host), cudaMemcpyDeviceToHost, s) != cudaSuccess) return TA_ERR_CUDA;
  if (cudaMemsetAsync(ptr, 0, sizeof(host), s) != cudaSuccess) return TA_ERR_CUDA;
  if (cudaStreamSynchronize(s) != cudaSuccess) return TA_ERR_CUDA;
  return (int)host;
}

static bool hosvd_args_ok(int32_t d, int32_t nH, int32_t r1, int32_t r2, int32_t r3) {
  return d > 0 && d <= 8192 && nH > 0 && nH <= 64 && r1 >= 1 && r1 <= nH && r2 >= 1 && r2 <= d && r3 >= 1 && r3 <= d;
}

size_t tucker_hosvd_workspace_bytes(int32_t d_model, int32_t n_H, int32_t r2, int32_t r3) {
  if (!hosvd_args_ok(d_model, n_H, 1, r2, r3)) return 0;
  return hosvd_workspace(n_H, d_model, d_model, r2, r3);
}

int tucker_hosvd_init(int32_t d_model, int32_t n_H, int32_t r1, int32_t r2, int32_t r3, const float* W, float* C,
                      float* U1, float* U2, float* U3, float* spectra, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
  if (!hosvd_args_ok(d_model, n_H, r1, r2, r3)) return TA_ERR_INVALID_ARG;
  if (!W || !C || !U1 || !U2 || !U3 || !workspace) return TA_ERR_INVALID_ARG;
  if (!aligned16(W) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return TA_ERR_INVALID_ARG;
  if (workspace_bytes < hosvd_workspace(n_H, d_model, d_model, r2, r3)) return TA_ERR_WORKSPACE_TOO_SMALL;
  Problem p = {};
  p.ws = static_cast<char*>(workspace); p.ws_bytes = workspace_bytes;
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  p.prof_start = tl_prof_start; p.prof_stop = tl_prof_stop;
  if (!p.dev_err) return TA_ERR_CUDA;
  const int rc = hosvd_run(p, n_H, d_model, d_model, r1, r2, r3, W, C, U1, U2, U3, spectra);
  tl_last_path = 2;
  tl_last_launches = p.launches;
  return rc;
}

int tucker_mha_weight_tensors(int32_t d_model, int32_t n_H, const float* WQ, const float* WK, const float* WV,
                              const float* WO, float* W, float* Wt, void* cuda_stream) {
  if (d_model <= 0 || n_H <= 0 || d_model % n_H || !WQ || !WK || !WV || !WO || !W || !Wt) return TA_ERR_INVALID_ARG;
  Problem p = {};
  p.stream = static_cast<cudaStream_t>(cuda_stream);
  p.dev_err = device_error_ptr();
  if (!p.dev_err) return TA_ERR_CUDA;
  const int rc = mha_weight_tensors_run(p, d_model, n_H, WQ, WK, WV, WO, W, Wt);
  tl_last_launches = p.launches;
  return rc;
}

int tucker_attn_sync_status(void* cuda_stream) {
  const int word = tucker_attn_last_device_error(cuda_stream);
  if (word < 0) return word;
  if (word & TA_DEVERR_WAIT_TIMEOUT) return TA_ERR_DEVICE_TIMEOUT;
  if (word & (TA_DEVERR_BAD_CACHE_LEN | TA_DEVERR_BAD_PAGE)) return TA_ERR_INVALID_ARG;
  if (word & TA_DEVERR_BAD_INDEX) return TA_ERR_CUDA;
  return TA_OK;
}

int tucker_attn_bounds_checked(void) {
#ifdef TA_BOUNDS_CHECK
  return 1;
#else
  return 0;
#endif
}

int tucker_attn_selftest_wait_timeout(int32_t budget_us, int32_t* out, void* cuda_stream) {
  if (budget_us <= 0 || budget_us > 100000 || !out) return TA_ERR_INVALID_ARG;
  unsigned int* ptr = device_error_ptr();
  if (!ptr) return TA_ERR_CUDA;
  return wait_selftest(ptr, budget_us, out, static_cast<cudaStream_t>(cuda_stream));
}

int tucker_attn_selftest_cluster_wait(int32_t budget_us, int32_t* out, void* cuda_stream) {
  if (budget_us <= 0 || budget_us > 100000 || !out) return TA_ERR_INVALID_ARG;
  unsigned int* ptr = device_error_ptr();
  if (!ptr) return TA_ERR_CUDA;
  return cluster_wait_selftest(ptr, budget_us, out, static_cast<cudaStream_t>(cuda_stream));
}

int tucker_attn_set_profile_events(void* ev_start, void* ev_stop) {
  if ((ev_start == nullptr) != (ev_stop == nullptr)) return TA_ERR_INVALID_ARG;
  tl_prof_start = static_cast<cudaEvent_t>(ev_start);
  tl_prof_stop = static_cast<cudaEvent_t>(ev_stop);
  return TA_OK;
}

int tucker_attn_last_path(void) { return tl_last_path; }
int tucker_attn_last_launch_count(void) { return tl_last_launches; }

}  // extern "C"
