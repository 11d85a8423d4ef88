// C ABI entry points: argument validation and launches on the caller's stream.
#include "mdss.h"

#include <hip/hip_runtime.h>

#include "cache.h"
#include "common.h"

namespace {

constexpr int32_t kAbiVersion = 1;

// B = 0 is an empty batch: after the shape and parameter checks an entry point
// returns MDSS_OK without reading, writing or launching anything.
mdss_status check_shape(int64_t B, int64_t V) {
  if (B < 0 || B > MDSS_MAX_B || V < 2 || V > MDSS_MAX_V) return MDSS_ESHAPE;
  return MDSS_OK;
}

bool workspace_ok(const void* ws, size_t bytes, size_t need) {
  return ws && bytes >= need && (reinterpret_cast<uintptr_t>(ws) % 256) == 0;
}

mdss_status check_k(int32_t K, int32_t s_max) {
  if (K != 2 && K != 3) return MDSS_EUNSUPPORTED;
  if (K == 3 && (s_max < 1 || s_max > MDSS_K3_MAX_SUPPORT)) return MDSS_EUNSUPPORTED;
  return MDSS_OK;
}

mdss_status from_hip(hipError_t e) { return e == hipSuccess ? MDSS_OK : MDSS_EDEVICE; }

// ---- cache and beams
constexpr int64_t kMaxTokens = 1LL << 24, kMaxPages = 1LL << 24;

mdss_status check_cache(const mdss_cache* c) {
  if (!c) return MDSS_EINVAL;
  if (c->layers < 1 || c->layers > 65535 || c->heads < 1 || c->heads > 1024 || c->pages < 1 || c->pages > kMaxPages)
    return MDSS_ESHAPE;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256) return MDSS_EUNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return MDSS_EUNSUPPORTED;
  return MDSS_OK;
}

// The pool's own pointers, once there is work to do.
bool cache_pointers(const mdss_cache* c) {
  return c->k && c->v && c->k_exp && c->v_exp &&
         ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15) == 0;
}

mdss::CacheView cache_view(const mdss_cache* c) {
  mdss::CacheView v;
  v.k = c->k;
  v.v = c->v;
  v.k_exp = c->k_exp;
  v.v_exp = c->v_exp;
  v.layers = c->layers;
  v.heads = c->heads;
  v.d = c->head_dim;
  v.page_shift = __builtin_ctz((unsigned)c->page_size);
  v.pages = c->pages;
  return v;
}

mdss_status check_rows(int64_t S, int64_t width) {
  if (S < 0 || S > MDSS_MAX_B || width < 1 || width > INT32_MAX || S * width > INT32_MAX) return MDSS_ESHAPE;
  return MDSS_OK;
}

mdss_status check_tokens(int64_t T, int64_t S, bool uniform) {
  if (T < 0 || T > kMaxTokens || (uniform && S > 0 && T % S != 0)) return MDSS_ESHAPE;
  return MDSS_OK;
}

mdss_status check_rope(const mdss_rope* r, int64_t head_dim) {
  if (!r) return MDSS_EINVAL;
  if (head_dim < 1 || r->pairs < 1 || 2 * (int64_t)r->pairs > head_dim) return MDSS_ESHAPE;
  if (!(r->magnitude > 0.0f) || r->magnitude > 65536.0f || (reinterpret_cast<uintptr_t>(r->frequencies) & 7)) return MDSS_EINVAL;
  return MDSS_OK;
}

mdss::Rope rope_view(const mdss_rope* r, int32_t inverse) {
  mdss::Rope v;
  v.freq = r->frequencies;
  v.pairs = r->pairs;
  v.interleaved = r->interleaved != 0;
  v.magnitude = r->magnitude;
  v.sign = inverse ? -1.0f : 1.0f;
  v.bound = (float)(1.4142135623730951 * (double)r->magnitude);
  return v;
}

mdss_status check_beams(int64_t B, int64_t W, int64_t n) {
  if (W < 1 || W > MDSS_MAX_BEAMS || n < 1 || n > MDSS_MAX_BEAMS || B < 0 || B * W > 65535 || B * n > 65535 ||
      B > 65535)
    return MDSS_ESHAPE;
  return MDSS_OK;
}

}  // namespace

extern "C" {

int32_t mdss_abi_version(void) { return kAbiVersion; }

const char* mdss_status_string(mdss_status s) {
  switch (s) {
    case MDSS_OK: return "ok";
    case MDSS_EINVAL: return "invalid argument (null pointer or bad value)";
    case MDSS_ESHAPE: return "invalid shape (B outside [0, MDSS_MAX_B], V outside [2, MDSS_MAX_V], or a size of the cache or beams out of range)";
    case MDSS_EUNSUPPORTED: return "unsupported configuration (K out of range, K = 3 with s_max out of range, s outside [1, MDSS_TLP_MAX_S], or a cache's head or page size)";
    case MDSS_EDEVICE: return "HIP error while launching";
    case MDSS_EWORKSPACE: return "workspace missing or too small (allocation-free call: sizes beyond MDSS_NOALLOC_SCRATCH_BYTES)";
  }
  return "unknown status";
}

size_t mdss_workspace_bytes(int64_t B, int64_t V, int32_t K, int32_t s_max) {
  if (check_shape(B, V) != MDSS_OK || check_k(K, s_max) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes(B, V, K, s_max);
}

mdss_status mdss_induced_dist(const float* p, const float* q, int64_t B, int64_t V, int32_t K, int32_t s_max,
                              float* r, int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if ((s = check_k(K, s_max)) != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  const size_t need = mdss::workspace_bytes(B, V, K, s_max);
  if (!workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  return from_hip(
      mdss::launch_induced(p, q, B, V, K, s_max, r, row_status, workspace, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_pair(int64_t B, int64_t V) {
  if (check_shape(B, V) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes_pair(B, V);
}

mdss_status mdss_induced_dist_pair(const float* p, const float* q1, const float* q2, int64_t B, int64_t V, float* r,
                                   int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !q2 || !r) return MDSS_EINVAL;
  const size_t need = mdss::workspace_bytes_pair(B, V);
  if (!workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_pair(p, q1, q2, B, V, r, row_status, workspace,
                                            static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_intermediate_pair(const float* p, const float* q1, const float* q2, const int32_t* drafts,
                                          const float* u, uint64_t seed, uint64_t offset, int64_t B, int64_t V,
                                          int32_t* sel_index, int32_t* sel_token, int32_t* row_status,
                                          void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !q2 || !drafts || !sel_index || !sel_token) return MDSS_EINVAL;
  return from_hip(mdss::launch_select_pair(p, q1, q2, drafts, u, seed, offset, B, V, sel_index, sel_token,
                                           row_status, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_successive(int64_t B, int64_t V) {
  if (check_shape(B, V) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes_pair(B, V);
}

mdss_status mdss_induced_dist_successive(const float* p, const float* q, int64_t B, int64_t V, int32_t K,
                                         float* r_stages, int32_t* row_status, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (K < 2 || K > MDSS_SUCCESSIVE_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r_stages) return MDSS_EINVAL;
  const size_t need = mdss::workspace_bytes_pair(B, V);
  if (!workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_successive(p, q, B, V, K, r_stages, row_status, workspace,
                                                  static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_successive(const float* p, const float* q, const float* r_stages, const int32_t* drafts,
                                   const float* u_sel, uint64_t seed, uint64_t offset, int64_t B, int64_t V,
                                   int32_t K, int32_t* sel_index, int32_t* sel_token, int32_t* row_status,
                                   void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (K < 2 || K > MDSS_SUCCESSIVE_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !drafts || !sel_index || !sel_token) return MDSS_EINVAL;
  if (K > 2 && !r_stages) return MDSS_EINVAL;
  return from_hip(mdss::launch_select_successive(p, q, r_stages, drafts, u_sel, seed, offset, B, V, K, sel_index,
                                                 sel_token, row_status, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_truncate_alphabet(const float* p, int64_t B, int64_t V, int32_t m, float* p_trunc, double* mass0,
                                   int32_t* row_status, void* stream) {
  if (m < 1) return MDSS_EINVAL;
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (B == 0) return MDSS_OK;
  if (!p || !p_trunc || !mass0) return MDSS_EINVAL;
  return from_hip(mdss::launch_alphabet_truncate(p, B, V, m, p_trunc, mass0, row_status,
                                                 static_cast<hipStream_t>(stream)));
}

mdss_status mdss_alphabet_post(const float* p, const float* p_trunc, const double* mass0, const int32_t* token,
                               const float* u2, uint64_t seed, uint64_t offset, int64_t B, int64_t V,
                               int32_t* out_token, uint8_t* kept, void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (B == 0) return MDSS_OK;
  if (!p || !p_trunc || !mass0 || !token || !out_token || !kept) return MDSS_EINVAL;
  return from_hip(mdss::launch_alphabet_post(p, p_trunc, mass0, token, u2, seed, offset, B, V, out_token, kept,
                                             static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_optimum(int64_t B, int64_t V) {
  if (check_shape(B, V) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes_optimum(B, V);
}

mdss_status mdss_optimal_acceptance(const float* p, const float* q, int64_t B, int64_t V, int32_t K, double* pstar,
                                    int32_t* kstar, int32_t* row_status, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (K < 2 || K > MDSS_OPTIMUM_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !pstar) return MDSS_EINVAL;
  const size_t need = mdss::workspace_bytes_optimum(B, V);
  if (!workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_optimum(p, q, B, V, K, pstar, kstar, row_status, workspace,
                                       static_cast<hipStream_t>(stream)));
}

mdss_status mdss_acceptance(const float* p, const float* r, int64_t B, int64_t V, double* accept,
                            int32_t* row_status, void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (B == 0) return MDSS_OK;
  if (!p || !r || !accept) return MDSS_EINVAL;
  return from_hip(mdss::launch_acceptance(p, r, B, V, accept, row_status, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_tlp(int64_t B, int64_t V, int32_t tail) {
  if (check_shape(B, V) != MDSS_OK || (tail != MDSS_TLP_SORTED && tail != MDSS_TLP_HALF) || B == 0) return 0;
  return mdss::workspace_bytes_tlp(B, V, tail);
}

mdss_status mdss_truncated_lp(const float* p, const float* q1, const float* q2, int64_t B, int64_t V, int32_t s,
                              int32_t tail, float* r, int32_t* omega1, double* w, double* accept,
                              int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  if (tail != MDSS_TLP_SORTED && tail != MDSS_TLP_HALF) return MDSS_EINVAL;
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (s < 1 || s > MDSS_TLP_MAX_S) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !r || !omega1 || !w) return MDSS_EINVAL;
  const size_t need = mdss::workspace_bytes_tlp(B, V, tail);
  if (!workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_tlp(p, q1, q2, B, V, s, tail, r, omega1, w, accept, row_status, workspace,
                                   static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_truncated_lp(const float* p, const float* q1, const float* q2, const int32_t* drafts,
                                     const float* u, uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t s,
                                     int32_t tail, const int32_t* omega1, const double* w, int32_t* sel_index,
                                     int32_t* sel_token, int32_t* row_status, void* stream) {
  if (tail != MDSS_TLP_SORTED && tail != MDSS_TLP_HALF) return MDSS_EINVAL;
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (s < 1 || s > MDSS_TLP_MAX_S) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !drafts || !omega1 || !w || !sel_index || !sel_token) return MDSS_EINVAL;
  return from_hip(mdss::launch_select_tlp(p, q1, q2, drafts, u, seed, offset, B, V, s, tail, omega1, w, sel_index,
                                          sel_token, row_status, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_expsum(int64_t B, int64_t V, int32_t K) {
  if (check_shape(B, V) != MDSS_OK || K < 2 || K > MDSS_MAX_K || B == 0) return 0;
  return mdss::workspace_bytes_expsum(B, V, 1);
}

mdss_status mdss_induced_dist_expsum(const float* p, const float* q, int64_t B, int64_t V, int32_t K, float* r,
                                     int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_expsum(B, V, 1))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_expsum(p, q, nullptr, B, V, K, r, row_status, workspace,
                                              static_cast<hipStream_t>(stream)));
}

mdss_status mdss_induced_dist_topk_expsum(const float* p, const float* q, int64_t B, int64_t V, int32_t K,
                                          int32_t s_max, float* r, int32_t* row_status, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K || s_max < 1 || s_max > MDSS_K3_MAX_SUPPORT) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  return from_hip(
      mdss::launch_induced_topk_expsum(p, q, B, V, K, s_max, r, row_status, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_induced_dist_topk_expsum_sums(const float* p, const float* q, int64_t B, int64_t V, int32_t K,
                                               int32_t s_max, float* r, int32_t* row_status, void* accept_workspace,
                                               size_t accept_workspace_bytes, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K || s_max < 1 || s_max > MDSS_K3_MAX_SUPPORT) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  if (!workspace_ok(accept_workspace, accept_workspace_bytes, mdss::workspace_bytes_accept(B, V)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_topk_expsum(p, q, B, V, K, s_max, r, row_status,
                                                   static_cast<hipStream_t>(stream),
                                                   static_cast<double*>(accept_workspace)));
}

mdss_status mdss_step_topk_expsum(const float* p, const float* q, const int32_t* drafts, const float* u,
                                  uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t K, int32_t s_max,
                                  float* r, int32_t* sel_index, int32_t* sel_token, int32_t* out_token,
                                  uint8_t* accepted, double* residual_mass, int32_t* row_status,
                                  void* accept_workspace, size_t accept_workspace_bytes, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K || s_max < 1 || s_max > MDSS_K3_MAX_SUPPORT) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r || !drafts || !out_token || !accepted) return MDSS_EINVAL;
  if (!workspace_ok(accept_workspace, accept_workspace_bytes, mdss::workspace_bytes_accept(B, V)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_step_topk_expsum(p, q, drafts, u, seed, offset, B, V, K, s_max, r, sel_index,
                                                sel_token, out_token, accepted, residual_mass, row_status,
                                                static_cast<double*>(accept_workspace),
                                                static_cast<hipStream_t>(stream)));
}

mdss_status mdss_induced_dist_expsum_noalloc(const float* p, const float* q, int64_t B, int64_t V, int32_t K,
                                             float* r, int32_t* row_status, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  if (mdss::workspace_bytes_expsum(B, V, 1) > (size_t)MDSS_NOALLOC_SCRATCH_BYTES) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_expsum_noalloc(p, q, B, V, K, r, row_status, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_pair_expsum(int64_t B, int64_t V) {
  if (check_shape(B, V) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes_expsum(B, V, 2);
}

mdss_status mdss_induced_dist_pair_expsum(const float* p, const float* q1, const float* q2, int64_t B, int64_t V,
                                          float* r, int32_t* row_status, void* workspace, size_t workspace_bytes,
                                          void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !q2 || !r) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_expsum(B, V, 2))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_expsum(p, q1, q2, B, V, 2, r, row_status, workspace,
                                              static_cast<hipStream_t>(stream)));
}

mdss_status mdss_induced_dist_successive_expsum(const float* p, const float* q, int64_t B, int64_t V, int32_t K,
                                                float* r_stages, int32_t* row_status, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  const mdss_status st = check_shape(B, V);
  if (st != MDSS_OK) return st;
  if (K < 2 || K > MDSS_SUCCESSIVE_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r_stages) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_expsum(B, V, 2))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_successive_expsum(p, q, B, V, K, r_stages, row_status, workspace,
                                                         static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_intermediate(const float* p, const float* q, const int32_t* drafts, const float* u,
                                     uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t K,
                                     int32_t* sel_index, int32_t* sel_token, int32_t* row_status, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !drafts || !sel_index || !sel_token) return MDSS_EINVAL;
  return from_hip(mdss::launch_select(p, q, drafts, u, seed, offset, B, V, K, sel_index, sel_token, row_status,
                                      static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_accept(int64_t B, int64_t V) {
  if (check_shape(B, V) != MDSS_OK || B == 0) return 0;
  return mdss::workspace_bytes_accept(B, V);
}

mdss_status mdss_accept_or_resample(const float* p, const float* r, const int32_t* sel_token, const float* u,
                                    uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t* out_token,
                                    uint8_t* accepted, float* residual, double* residual_mass, int32_t* row_status,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !r || !sel_token || !out_token || !accepted) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_accept(B, V))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_accept(p, r, sel_token, u, seed, offset, B, V, out_token, accepted, residual,
                                      residual_mass, row_status, workspace, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_accept(const float* p, const float* q, const float* r, const int32_t* drafts,
                               const float* u, uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t K,
                               int32_t* sel_index, int32_t* sel_token, int32_t* out_token, uint8_t* accepted,
                               float* residual, double* residual_mass, int32_t* row_status, void* workspace,
                               size_t workspace_bytes, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r || !drafts || !out_token || !accepted) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_accept(B, V))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_select_accept(p, q, nullptr, r, drafts, u, seed, offset, B, V, K, sel_index,
                                             sel_token, out_token, accepted, residual, residual_mass, row_status,
                                             workspace, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_induced_dist_expsum_sums(const float* p, const float* q, int64_t B, int64_t V, int32_t K, float* r,
                                          int32_t* row_status, void* workspace, size_t workspace_bytes,
                                          void* accept_workspace, size_t accept_workspace_bytes, void* stream) {
  const mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_expsum(B, V, 1))) return MDSS_EWORKSPACE;
  if (!workspace_ok(accept_workspace, accept_workspace_bytes, mdss::workspace_bytes_accept(B, V)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_induced_expsum(p, q, nullptr, B, V, K, r, row_status, workspace,
                                              static_cast<hipStream_t>(stream),
                                              static_cast<double*>(accept_workspace)));
}

mdss_status mdss_select_accept_sums(const float* p, const float* q, const float* r, const int32_t* drafts,
                                    const float* u, uint64_t seed, uint64_t offset, int64_t B, int64_t V, int32_t K,
                                    int32_t* sel_index, int32_t* sel_token, int32_t* out_token, uint8_t* accepted,
                                    double* residual_mass, int32_t* row_status, void* accept_workspace,
                                    size_t accept_workspace_bytes, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (K < 2 || K > MDSS_MAX_K) return MDSS_EUNSUPPORTED;
  if (B == 0) return MDSS_OK;
  if (!p || !q || !r || !drafts || !out_token || !accepted) return MDSS_EINVAL;
  if (!workspace_ok(accept_workspace, accept_workspace_bytes, mdss::workspace_bytes_accept(B, V)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_select_accept_sums(p, q, nullptr, r, drafts, u, seed, offset, B, V, K, sel_index,
                                                  sel_token, out_token, accepted, residual_mass, row_status,
                                                  accept_workspace, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_select_accept_pair(const float* p, const float* q1, const float* q2, const float* r,
                                    const int32_t* drafts, const float* u, uint64_t seed, uint64_t offset,
                                    int64_t B, int64_t V, int32_t* sel_index, int32_t* sel_token,
                                    int32_t* out_token, uint8_t* accepted, float* residual, double* residual_mass,
                                    int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_shape(B, V);
  if (s != MDSS_OK) return s;
  if (B == 0) return MDSS_OK;
  if (!p || !q1 || !q2 || !r || !drafts || !out_token || !accepted) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_accept(B, V))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_select_accept(p, q1, q2, r, drafts, u, seed, offset, B, V, 2, sel_index, sel_token,
                                             out_token, accepted, residual, residual_mass, row_status, workspace,
                                             static_cast<hipStream_t>(stream)));
}

mdss_status mdss_cache_append(const mdss_cache* cache, int32_t layer, const void* key, int64_t key_token_stride,
                              int64_t key_head_stride, const void* value, int64_t value_token_stride,
                              int64_t value_head_stride, mdss_dtype dtype, int64_t T, const int32_t* starts,
                              const int32_t* table, int64_t width, const int32_t* lengths, int64_t S,
                              int32_t* row_status, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_tokens(T, S, !starts)) != MDSS_OK) return s;
  if (layer < 0 || layer >= cache->layers || key_token_stride < 0 || key_head_stride < 0 || value_token_stride < 0 ||
      value_head_stride < 0)
    return MDSS_EINVAL;
  if (dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (S == 0 || T == 0) return MDSS_OK;
  if (!cache_pointers(cache) || !key || !value || !table || !lengths) return MDSS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(key) | reinterpret_cast<uintptr_t>(value)) & 1) return MDSS_EINVAL;
  const mdss::CacheRows rows = {starts, table, lengths, T, width, (int)S};
  return from_hip(mdss::launch_cache_append(cache_view(cache), layer, key, value, dtype, key_token_stride,
                                            key_head_stride, value_token_stride, value_head_stride, rows, row_status,
                                            static_cast<hipStream_t>(stream)));
}

mdss_status mdss_rotary(const void* x, int64_t x_token_stride, int64_t x_head_stride, mdss_dtype dtype, int64_t T, int64_t heads,
                        int64_t head_dim, const int32_t* positions, const mdss_rope* rope, int32_t inverse, void* out,
                        int64_t out_token_stride, int64_t out_head_stride, void* stream) {
  const mdss_status s = check_rope(rope, head_dim);
  if (s != MDSS_OK) return s;
  if (T < 0 || T > kMaxTokens || heads < 1 || head_dim > 65536 || heads > INT32_MAX / head_dim) return MDSS_ESHAPE;
  if (dtype != MDSS_F32 && dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (x_token_stride < 0 || x_head_stride < 0 || (T > 1 && out_token_stride < head_dim) || (heads > 1 && out_head_stride < head_dim))
    return MDSS_EINVAL;
  // (no two rows of out in one place: tokens lie past each other's heads, or heads past each other's tokens)
  if (T > 1 && heads > 1 && (out_token_stride - head_dim) / (heads - 1) < out_head_stride &&
      (out_head_stride - head_dim) / (T - 1) < out_token_stride)
    return MDSS_EINVAL;
  if (T == 0) return MDSS_OK;
  if (!x || !out || !positions || !rope->frequencies) return MDSS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & (dtype == MDSS_F32 ? 3 : 1)) return MDSS_EINVAL;
  if (x == out && ((T > 1 && x_token_stride != out_token_stride) || (heads > 1 && x_head_stride != out_head_stride))) return MDSS_EINVAL;
  return from_hip(mdss::launch_rotary(x, x_token_stride, x_head_stride, dtype, T, heads, head_dim, positions, rope_view(rope, inverse), out,
                                      out_token_stride, out_head_stride, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_cache_append_rotary(const mdss_cache* cache, int32_t layer, const void* key, int64_t key_token_stride,
                                     int64_t key_head_stride, const void* value, int64_t value_token_stride,
                                     int64_t value_head_stride, mdss_dtype dtype, int64_t T, const int32_t* starts,
                                     const int32_t* table, int64_t width, const int32_t* lengths, int64_t S,
                                     const mdss_rope* rope, const int32_t* positions, const void* q, int64_t q_token_stride,
                                     int64_t q_head_stride, int64_t heads_q, void* q_out, int32_t* row_status, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rope(rope, cache->head_dim)) != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_tokens(T, S, !starts)) != MDSS_OK) return s;
  if (heads_q < 0 || heads_q % cache->heads || heads_q / cache->heads > 1024 || T * heads_q > INT32_MAX) return MDSS_ESHAPE;
  if (layer < 0 || layer >= cache->layers || key_token_stride < 0 || key_head_stride < 0 || value_token_stride < 0 ||
      value_head_stride < 0 || q_token_stride < 0 || q_head_stride < 0)
    return MDSS_EINVAL;
  if (dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (S == 0 || T == 0) return MDSS_OK;
  if (!cache_pointers(cache) || !key || !value || !table || !lengths || !rope->frequencies) return MDSS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(key) | reinterpret_cast<uintptr_t>(value)) & 1) return MDSS_EINVAL;
  if (heads_q > 0 && (!q || !q_out || q == q_out || (reinterpret_cast<uintptr_t>(q) & 1) || (reinterpret_cast<uintptr_t>(q_out) & 15)))
    return MDSS_EINVAL;
  const mdss::CacheRows rows = {starts, table, lengths, T, width, (int)S};
  const mdss::AppendTurn turn = {rope_view(rope, 0), positions, q, q_out, q_token_stride, q_head_stride, heads_q * cache->head_dim,
                                 cache->head_dim, (int)(heads_q / cache->heads)};
  return from_hip(mdss::launch_cache_append(cache_view(cache), layer, key, value, dtype, key_token_stride, key_head_stride,
                                            value_token_stride, value_head_stride, rows, row_status,
                                            static_cast<hipStream_t>(stream), &turn));
}

mdss_status mdss_cache_shared(const mdss_cache* cache, int64_t T, const int32_t* starts, const int32_t* table, int64_t width,
                              const int32_t* lengths, int64_t S, const int32_t* groups, int64_t G, int32_t least,
                              int32_t* tokens, int32_t* group_rows, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_tokens(T, S, !starts)) != MDSS_OK) return s;
  if (G < 0 || G > MDSS_MAX_B) return MDSS_ESHAPE;
  if (least < 0) return MDSS_EINVAL;
  if (S == 0 && G == 0) return MDSS_OK;
  if (G > 0 && (!groups || !group_rows)) return MDSS_EINVAL;
  if (S > 0 && (!table || !lengths || !tokens)) return MDSS_EINVAL;
  const mdss::CacheRows rows = {starts, table, lengths, T, width, (int)S};
  return from_hip(mdss::launch_cache_shared(cache_view(cache), rows, groups, G, least, tokens, group_rows,
                                            static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_attention_shared(const mdss_cache* cache, int64_t T, int64_t S, int64_t G, int64_t width, int64_t heads_q,
                                             int32_t uniform, int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own) {
  if (check_cache(cache) != MDSS_OK || check_rows(S, width) != MDSS_OK || check_tokens(T, S, uniform) != MDSS_OK || G < 0 ||
      G > MDSS_MAX_B || heads_q < 1 || heads_q % cache->heads || heads_q / cache->heads > 1024 || T * heads_q > INT32_MAX || S == 0 ||
      T == 0)
    return 0;
  return mdss::workspace_bytes_attention_shared(cache_view(cache), T, S, G, width, heads_q, uniform != 0, max_new, max_group,
                                                max_shared, max_own);
}

mdss_status mdss_cache_attention_shared(const mdss_cache* cache, int32_t layer, const void* q, int64_t q_token_stride,
                                        int64_t q_head_stride, mdss_dtype dtype, int64_t T, int64_t heads_q,
                                        const int32_t* starts, const int32_t* table, int64_t width, const int32_t* lengths,
                                        int64_t S, const int32_t* tokens, const int32_t* group_rows, int64_t G, float scale,
                                        int64_t max_new, int64_t max_group, int64_t max_shared, int64_t max_own, void* out,
                                        float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_tokens(T, S, !starts)) != MDSS_OK) return s;
  if (G < 0 || G > MDSS_MAX_B || heads_q < 1 || heads_q % cache->heads || heads_q / cache->heads > 1024 || T * heads_q > INT32_MAX)
    return MDSS_ESHAPE;
  if (layer < 0 || layer >= cache->layers || q_token_stride < 0 || q_head_stride < 0 || max_new < 0 || max_group < 0 ||
      max_shared < 0 || max_own < 0)
    return MDSS_EINVAL;
  if (dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (S == 0 || T == 0) return MDSS_OK;
  if (!cache_pointers(cache) || !q || !table || !lengths || !tokens || (G > 0 && !group_rows) || !out) return MDSS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q) & 1) || (reinterpret_cast<uintptr_t>(out) & 15)) return MDSS_EINVAL;
  const mdss::CacheView c = cache_view(cache);
  const size_t need = mdss::workspace_bytes_attention_shared(c, T, S, G, width, heads_q, !starts, max_new, max_group, max_shared,
                                                             max_own);
  if (need > 0 && !workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  const mdss::CacheRows rows = {starts, table, lengths, T, width, (int)S};
  return from_hip(mdss::launch_cache_attention_shared(c, layer, q, dtype, heads_q, q_token_stride, q_head_stride, rows, tokens,
                                                      group_rows, G, scale, max_new, max_group, max_shared, max_own, out, lse,
                                                      workspace, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_attention(const mdss_cache* cache, int64_t T, int64_t S, int64_t width, int64_t heads_q,
                                      int32_t uniform, int64_t max_new, int64_t max_length) {
  if (check_cache(cache) != MDSS_OK || check_rows(S, width) != MDSS_OK || check_tokens(T, S, uniform) != MDSS_OK ||
      heads_q < 1 || heads_q % cache->heads || heads_q / cache->heads > 1024 ||
      T * heads_q > INT32_MAX || S == 0 || T == 0)
    return 0;
  return mdss::workspace_bytes_attention(cache_view(cache), T, S, width, heads_q, max_new, max_length, uniform != 0);
}

mdss_status mdss_cache_attention(const mdss_cache* cache, int32_t layer, const void* q, int64_t q_token_stride,
                                 int64_t q_head_stride, mdss_dtype dtype, int64_t T, int64_t heads_q,
                                 const int32_t* starts, const int32_t* table, int64_t width, const int32_t* lengths,
                                 int64_t S, float scale, int64_t max_new, int64_t max_length, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_tokens(T, S, !starts)) != MDSS_OK) return s;
  if (heads_q < 1 || heads_q % cache->heads || heads_q / cache->heads > 1024 || T * heads_q > INT32_MAX)
    return MDSS_ESHAPE;
  if (layer < 0 || layer >= cache->layers || q_token_stride < 0 || q_head_stride < 0 || max_new < 0 || max_length < 0)
    return MDSS_EINVAL;
  if (dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (S == 0 || T == 0) return MDSS_OK;
  if (!cache_pointers(cache) || !q || !table || !lengths || !out) return MDSS_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q) & 1) || (reinterpret_cast<uintptr_t>(out) & 15)) return MDSS_EINVAL;
  const mdss::CacheView c = cache_view(cache);
  const size_t need = mdss::workspace_bytes_attention(c, T, S, width, heads_q, max_new, max_length, !starts);
  if (need > 0 && !workspace_ok(workspace, workspace_bytes, need)) return MDSS_EWORKSPACE;
  const mdss::CacheRows rows = {starts, table, lengths, T, width, (int)S};
  return from_hip(mdss::launch_cache_attention(c, layer, q, dtype, heads_q, q_token_stride, q_head_stride, rows, scale,
                                               max_new, max_length, out, lse, workspace,
                                               static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_cache_fork(const mdss_cache* cache, int64_t S_out) {
  if (check_cache(cache) != MDSS_OK || check_rows(S_out, 1) != MDSS_OK) return 0;
  return mdss::workspace_bytes_cache_fork(cache->pages, S_out);
}

mdss_status mdss_cache_fork(const mdss_cache* cache, const int32_t* table, const int32_t* lengths, int64_t S,
                            int64_t width, const int32_t* refs, const int32_t* parent, const int32_t* keep,
                            const int32_t* grow, int64_t S_out, int32_t* table_out, int32_t* lengths_out,
                            int32_t* refs_out, int32_t* row_status, void* workspace, size_t workspace_bytes,
                            void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if ((s = check_rows(S_out, width)) != MDSS_OK) return s;
  if (!parent && S_out > S) return MDSS_EINVAL;
  if (!cache_pointers(cache) || !refs || !refs_out) return MDSS_EINVAL;
  if (S > 0 && (!table || !lengths)) return MDSS_EINVAL;
  if (S_out > 0 && (!table_out || !lengths_out)) return MDSS_EINVAL;
  if ((table && table_out == table) || (lengths && lengths_out == lengths)) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_cache_fork(cache->pages, S_out)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_cache_fork(cache_view(cache), table, lengths, S, width, refs, parent, keep, grow, S_out,
                                          table_out, lengths_out, refs_out, row_status, workspace,
                                          static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_cache_compact(const mdss_cache* cache) {
  return check_cache(cache) == MDSS_OK ? mdss::workspace_bytes_cache_compact(cache->pages) : 0;
}

mdss_status mdss_cache_compact(const mdss_cache* cache, const int32_t* table, const int32_t* lengths, int64_t S,
                               int64_t width, const int32_t* refs, int32_t* table_out, int32_t* refs_out,
                               int32_t* used, void* workspace, size_t workspace_bytes, void* stream) {
  mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if ((s = check_rows(S, width)) != MDSS_OK) return s;
  if (!cache_pointers(cache) || !refs || !refs_out || refs_out == refs || !used) return MDSS_EINVAL;
  if (S > 0 && (!table || !lengths || !table_out)) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_cache_compact(cache->pages)))
    return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_cache_compact(cache_view(cache), table, lengths, S, width, refs, table_out, refs_out,
                                             used, workspace, static_cast<hipStream_t>(stream)));
}

mdss_status mdss_cache_copy(const mdss_cache* cache, const int32_t* src, const int32_t* dst, int64_t n, void* stream) {
  const mdss_status s = check_cache(cache);
  if (s != MDSS_OK) return s;
  if (n < 0 || n > kMaxPages) return MDSS_ESHAPE;
  if (n == 0) return MDSS_OK;
  if (!cache_pointers(cache) || !src || !dst) return MDSS_EINVAL;
  return from_hip(mdss::launch_cache_copy(cache_view(cache), src, dst, n, static_cast<hipStream_t>(stream)));
}

size_t mdss_workspace_bytes_beam(int64_t B, int64_t W, int64_t V, int64_t n) {
  if (check_beams(B, W, n) != MDSS_OK || V < 1 || V > MDSS_MAX_V || B == 0) return 0;
  return mdss::workspace_bytes_beam(B, W, V, n);
}

mdss_status mdss_beam_select(const void* logits, mdss_dtype dtype, int64_t row_stride, const float* scores,
                             const uint8_t* done, int64_t B, int64_t W, int64_t V, int64_t n, int32_t eos,
                             int32_t* parent, int32_t* token, float* score_out, uint8_t* done_out,
                             int32_t* row_status, void* workspace, size_t workspace_bytes, void* stream) {
  const mdss_status s = check_beams(B, W, n);
  if (s != MDSS_OK) return s;
  if (V < 1 || V > MDSS_MAX_V || row_stride < V) return MDSS_ESHAPE;
  if (dtype != MDSS_F32 && dtype != MDSS_BF16 && dtype != MDSS_F16) return MDSS_EUNSUPPORTED;
  if (eos < -1 || eos >= V) return MDSS_EINVAL;
  if (B == 0) return MDSS_OK;
  if (!logits || !scores || !parent || !token || !score_out || !done_out) return MDSS_EINVAL;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == MDSS_F32 ? 4 : 2)) return MDSS_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, mdss::workspace_bytes_beam(B, W, V, n))) return MDSS_EWORKSPACE;
  return from_hip(mdss::launch_beam_select(logits, dtype, row_stride, scores, done, B, W, V, n, eos, parent, token,
                                           score_out, done_out, row_status, workspace,
                                           static_cast<hipStream_t>(stream)));
}

mdss_status mdss_beam_reorder(const void* state, const int32_t* parent, int64_t B, int64_t W, int64_t n,
                              int64_t row_bytes, void* out, void* stream) {
  const mdss_status s = check_beams(B, W, n);
  if (s != MDSS_OK) return s;
  if (row_bytes < 0) return MDSS_ESHAPE;
  if (B == 0 || row_bytes == 0) return MDSS_OK;
  if (!state || !parent || !out || out == state) return MDSS_EINVAL;
  return from_hip(mdss::launch_beam_reorder(state, parent, B, W, n, row_bytes, out, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
