// C ABI of the cache's other forms: packed rings and the decode step over them, trees of drafted tokens.  Argument validation,
// workspaces, launches; errors as in api.hip.
#include "host_api.hpp"

using namespace rattn;

namespace {

constexpr int TREE_NODES = 64;   // one 64-bit mask of ancestors

template <typename... P> bool all_aligned(const P*... p) { return (aligned16(p) && ...); }
template <typename... P> bool any_null(const P*... p) { return (!p || ...); }

rattn_status tree_dims(const rattn_tree_params* p, TreeDims* td) {
  if (!p) return fail(RATTN_ERR_INVALID_ARG, "params is NULL");
  const rattn_decode_params d = {p->N, p->Hq, p->Hkv, p->D, p->window, p->dtype, p->softmax_scale, p->rms_eps, p->feature_map};
  DecodeDims dd;
  const rattn_status s = decode_dims(&d, &dd);
  if (s != RATTN_OK) return s;
  if (p->nodes < 1) return fail(RATTN_ERR_INVALID_ARG, "nodes must be >= 1 (got %d)", p->nodes);
  if (p->nodes > TREE_NODES) return fail(RATTN_ERR_UNSUPPORTED, "nodes must be <= %d (got %d)", TREE_NODES, p->nodes);
  if (p->Hq > 65535) return fail(RATTN_ERR_UNSUPPORTED, "Hq must be <= 65535 (got %d)", p->Hq);
  // a node's rows are addressed with 32-bit byte offsets, a launch has 2^31 work-groups at most
  if ((long long)p->nodes * p->Hkv * p->D * 4 >= (1ll << 31) || (long long)p->N * p->Hq * p->nodes >= (1ll << 31))
    return fail(RATTN_ERR_UNSUPPORTED, "N, heads and nodes too large");
  *td = TreeDims();
  td->N = dd.N; td->M = p->nodes; td->Hq = dd.Hq; td->Hkv = dd.Hkv; td->D = dd.D; td->W = dd.W; td->G = dd.G;
  td->scale = dd.scale; td->eps = dd.eps; td->phi = dd.phi;
  return RATTN_OK;
}

// the ring pointers of a tree call: both scales or neither
rattn_status check_rings(const void* k_ring, const void* k_scale, const void* v_ring, const void* v_scale) {
  if (any_null(k_ring, v_ring)) return fail(RATTN_ERR_INVALID_ARG, "k_ring and v_ring must be non-NULL");
  if (!k_scale != !v_scale) return fail(RATTN_ERR_INVALID_ARG, "packed rings need k_scale and v_scale, others neither");
  if (!all_aligned((const char*)k_ring, (const char*)k_scale, (const char*)v_ring, (const char*)v_scale))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  return RATTN_OK;
}

}  // namespace

extern "C" {

rattn_status rattn_ring_pack(const rattn_decode_params* p, const void* k_ring, const void* v_ring, void* k_codes, void* k_scale,
                             void* v_codes, void* v_scale, void* stream) {
  DecodeDims dd;
  const rattn_status s = decode_dims(p, &dd);
  if (s != RATTN_OK) return s;
  if (any_null(k_ring, v_ring, k_codes, k_scale, v_codes, v_scale))
    return fail(RATTN_ERR_INVALID_ARG, "k_ring, v_ring, k_codes, k_scale, v_codes, v_scale must be non-NULL");
  if (!all_aligned((const char*)k_ring, (const char*)v_ring, (char*)k_codes, (char*)k_scale, (char*)v_codes, (char*)v_scale))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  ring_pack(p->dtype, (long long)dd.N * dd.Hkv * dd.W * dd.D, k_ring, v_ring, k_codes, k_scale, v_codes, v_scale, (hipStream_t)stream);
  return check_launch("rattn_ring_pack");
}

rattn_status rattn_ring_unpack(const rattn_decode_params* p, const void* k_codes, const void* k_scale, const void* v_codes,
                               const void* v_scale, void* k_ring, void* v_ring, void* stream) {
  DecodeDims dd;
  const rattn_status s = decode_dims(p, &dd);
  if (s != RATTN_OK) return s;
  if (any_null(k_ring, v_ring, k_codes, k_scale, v_codes, v_scale))
    return fail(RATTN_ERR_INVALID_ARG, "k_codes, k_scale, v_codes, v_scale, k_ring, v_ring must be non-NULL");
  if (!all_aligned((const char*)k_codes, (const char*)k_scale, (const char*)v_codes, (const char*)v_scale, (char*)k_ring, (char*)v_ring))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  ring_unpack(p->dtype, (long long)dd.N * dd.Hkv * dd.W * dd.D, k_codes, k_scale, v_codes, v_scale, k_ring, v_ring, (hipStream_t)stream);
  return check_launch("rattn_ring_unpack");
}

rattn_status rattn_decode_packed_workspace_bytes(const rattn_decode_params* p, size_t* bytes) {
  DecodeDims dd;
  const rattn_status s = decode_dims(p, &dd);
  if (s != RATTN_OK) return s;
  if (bytes) *bytes = decode_split(dd, 1).bytes;
  return RATTN_OK;
}

rattn_status rattn_decode_step_packed(const rattn_decode_params* p, const void* q, const void* k_new, const void* v_new,
                                      const int32_t* pos, void* k_codes, void* k_scale, void* v_codes, void* v_scale,
                                      float* state, const float* gamma_swa, const float* gamma_rla, void* o, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  DecodeDims dd;
  const rattn_status s = decode_dims(p, &dd);
  if (s != RATTN_OK) return s;
  if (any_null(q, k_new, v_new, k_codes, k_scale, v_codes, v_scale, (void*)state, o, (const void*)pos))
    return fail(RATTN_ERR_INVALID_ARG, "q, k_new, v_new, pos, k_codes, k_scale, v_codes, v_scale, state, o must be non-NULL");
  if (!all_aligned((const char*)q, (const char*)k_new, (const char*)v_new, (char*)k_codes, (char*)k_scale, (char*)v_codes,
                   (char*)v_scale, (char*)state, (char*)o, (char*)workspace))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const size_t need = decode_split(dd, 1).bytes;
  if (workspace && workspace_bytes < need)
    return fail(RATTN_ERR_WORKSPACE, "decode step needs %zu workspace bytes (or none), got %zu", need, workspace_bytes);
  if (workspace && need > 0) { dd.workspace = workspace; dd.nonce = decode_nonce(); }
  decode_step_packed(dd, p->dtype, q, k_new, v_new, pos, k_codes, k_scale, v_codes, v_scale, state, gamma_swa, gamma_rla, o,
                     (hipStream_t)stream);
  return check_launch("rattn_decode_step_packed");
}

rattn_status rattn_tree_workspace_bytes(const rattn_tree_params* p, int32_t packed, size_t* bytes) {
  TreeDims td;
  const rattn_status s = tree_dims(p, &td);
  if (s != RATTN_OK) return s;
  if (bytes) *bytes = tree_plan(td, p->dtype, packed != 0).bytes;
  return RATTN_OK;
}

rattn_status rattn_tree_step(const rattn_tree_params* p, const void* q, const void* k, const void* v, const int32_t* parent,
                             const int32_t* count, const int32_t* pos, const void* k_ring, const void* k_scale,
                             const void* v_ring, const void* v_scale, const float* state, const float* gamma_swa,
                             const float* gamma_rla, void* o, void* workspace, size_t workspace_bytes, void* stream) {
  TreeDims td;
  rattn_status s = tree_dims(p, &td);
  if (s != RATTN_OK) return s;
  if (any_null(q, k, v, (const void*)parent, (const void*)pos, (const void*)state, (const void*)o))
    return fail(RATTN_ERR_INVALID_ARG, "q, k, v, parent, pos, state, o must be non-NULL");
  s = check_rings(k_ring, k_scale, v_ring, v_scale);
  if (s != RATTN_OK) return s;
  if (!all_aligned((const char*)q, (const char*)k, (const char*)v, (const char*)state, (char*)o, (char*)workspace))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const size_t need = tree_plan(td, p->dtype, k_scale != nullptr).bytes;
  if (workspace && workspace_bytes < need)
    return fail(RATTN_ERR_WORKSPACE, "tree step needs %zu workspace bytes (or none), got %zu", need, workspace_bytes);
  if (workspace && need > 0) { td.workspace = workspace; td.nonce = decode_nonce(); }
  const TreeTensors t = {q, k, v, parent, count, pos, const_cast<void*>(k_ring), const_cast<void*>(k_scale), const_cast<void*>(v_ring),
                         const_cast<void*>(v_scale), const_cast<float*>(state), gamma_swa, gamma_rla, o};
  tree_step(td, p->dtype, t, (hipStream_t)stream);
  return check_launch("rattn_tree_step");
}

rattn_status rattn_tree_commit(const rattn_tree_params* p, const void* k, const void* v, const int32_t* parent,
                               const int32_t* accepted, const int32_t* pos, void* k_ring, void* k_scale, void* v_ring,
                               void* v_scale, float* state, void* stream) {
  TreeDims td;
  rattn_status s = tree_dims(p, &td);
  if (s != RATTN_OK) return s;
  if (any_null(k, v, (const void*)parent, (const void*)accepted, (const void*)pos, (const void*)state))
    return fail(RATTN_ERR_INVALID_ARG, "k, v, parent, accepted, pos, state must be non-NULL");
  s = check_rings(k_ring, k_scale, v_ring, v_scale);
  if (s != RATTN_OK) return s;
  if (!all_aligned((const char*)k, (const char*)v, (const char*)state))
    return fail(RATTN_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  const TreeTensors t = {nullptr, k, v, parent, nullptr, pos, k_ring, k_scale, v_ring, v_scale, state, nullptr, nullptr, nullptr};
  tree_commit(td, p->dtype, t, accepted, (hipStream_t)stream);
  return check_launch("rattn_tree_commit");
}

}  // extern "C"
