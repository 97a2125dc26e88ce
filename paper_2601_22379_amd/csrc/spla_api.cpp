// Device entry points of the C ABI: argument checks, then the kernel
// launches of each call on the caller's stream.
#include <hip/hip_runtime.h>

#include <mutex>

#include "spla_kernels.h"

using spla::Dims;

namespace spla {

int compute_units() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
  if (cached[dev] == 0) {
    int v = 0;
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v < 1)
      v = 256;
    cached[dev] = v;
  }
  return cached[dev];
}

}  // namespace spla

namespace {

int32_t check_cache(const spla_config* cfg, const spla_cache* c) {
  if (!c) return SPLA_ERR_INVALID_ARG;
  if (!c->k_cache || !c->v_cache || !c->blk_stats || !c->lin_state || !c->lin_norm || !c->seq_lens)
    return SPLA_ERR_INVALID_ARG;
  if ((cfg->kv_pages > 0) != (c->block_table != nullptr)) return SPLA_ERR_INVALID_ARG;
  return SPLA_OK;
}

int32_t check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return SPLA_OK;
  if (!ws || have < need) return SPLA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) % SPLA_WORKSPACE_ALIGN != 0) return SPLA_ERR_WORKSPACE;
  return SPLA_OK;
}

struct PhaseMark {
  const spla_events* ev;
  hipStream_t st;
  int p;
  PhaseMark(const spla_events* e, hipStream_t s, int phase) : ev(e), st(s), p(phase) {
    if (ev && ev->start[p]) hipEventRecord((hipEvent_t)ev->start[p], st);
  }
  ~PhaseMark() {
    if (ev && ev->stop[p]) hipEventRecord((hipEvent_t)ev->stop[p], st);
  }
};

#define SPLA_TRY(expr)                               \
  do {                                               \
    hipError_t e_ = (expr);                          \
    if (e_ != hipSuccess) return SPLA_ERR_HIP;       \
  } while (0)

// k_step, v_step (or NULL): a step's token whose rank-one update of S_bar the
// decode's sparse pass applies (step_fusable shapes); the single launch also
// appends its rows and statistics, before the separate launches they are
// appended already and ws.appended holds the tokens each sequence received.
int32_t run_decode(const spla_config* cfg, const spla_cache* cache, const void* q,
                   const float* w, void* out, int32_t* sel_idx, void* ws, size_t ws_bytes,
                   const spla_events* ev, hipStream_t st, const void* k_step = nullptr,
                   const void* v_step = nullptr) {
  const Dims m = spla::make_dims(*cfg);
  const spla::DecodeWs L = spla::decode_ws_layout(m);
  char* base = static_cast<char*>(ws);
  if (spla::use_fused_decode(m) && !(cfg->flags & SPLA_FLAG_SEPARATE_KERNELS)) {
    PhaseMark pm(ev, st, SPLA_PHASE_DECODE);
    if (k_step)
      SPLA_TRY(spla::launch_decode_fused_step(m, *cfg, *cache, k_step, v_step, q, w, out, sel_idx,
                                              L, base, st));
    else
      SPLA_TRY(spla::launch_decode_fused(m, *cfg, *cache, q, w, out, sel_idx, L, base, st));
    return SPLA_OK;
  }
  // the selection runs in its own launch, or in the scoring launch's last
  // workgroup of each head, or in the sparse launch (the select phase empty)
  const bool in_sparse = spla::sparse_selects(m, k_step != nullptr);
  const bool in_score = !in_sparse && spla::score_selects(m);
  {
    PhaseMark pm(ev, st, SPLA_PHASE_SCORE);
    if (in_score)
      SPLA_TRY(spla::launch_score_select(m, *cfg, *cache, q, L, base, sel_idx, st));
    else
      SPLA_TRY(spla::launch_score(m, *cfg, *cache, q, L, base, st));
  }
  {
    PhaseMark pm(ev, st, SPLA_PHASE_SELECT);  // empty when folded into another launch
    if (!in_sparse && !in_score) SPLA_TRY(spla::launch_select(m, *cache, L, base, sel_idx, st));
  }
  {
    PhaseMark pm(ev, st, SPLA_PHASE_SPARSE);
    SPLA_TRY(spla::launch_sparse(m, *cfg, *cache, q, w, out, sel_idx, L, base, st, k_step,
                                 v_step));
  }
  {
    PhaseMark pm(ev, st, SPLA_PHASE_MERGE);
    SPLA_TRY(spla::launch_merge(m, *cfg, w, out, L, base, st));
  }
  return SPLA_OK;
}

int32_t check_decode_args(const spla_config* cfg, const spla_cache* cache, const void* q,
                          const float* w, void* out, void* ws, size_t ws_bytes) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if (!q || !w || !out) return SPLA_ERR_INVALID_ARG;
  if (out == q) return SPLA_ERR_INVALID_ARG;
  size_t need = 0;
  spla_workspace_bytes(cfg, &need);
  return check_ws(ws, ws_bytes, need);
}

}  // namespace

extern "C" int32_t spla_reset(const spla_config* cfg, const spla_cache* cache, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  size_t b[SPLA_CACHE_NUM_BUFFERS];
  spla_cache_bytes(cfg, b);
  hipStream_t st = static_cast<hipStream_t>(stream);
  SPLA_TRY(spla::launch_reset(*cache, b, st));
  return SPLA_OK;
}

extern "C" int32_t spla_workspace_init(const spla_config* cfg, void* ws, size_t ws_bytes,
                                       void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  size_t need = 0;
  spla_workspace_bytes(cfg, &need);
  if ((s = check_ws(ws, ws_bytes, need)) != SPLA_OK) return s;
  SPLA_TRY(spla::launch_fill_zero(ws, need, static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_append(const spla_config* cfg, const spla_cache* cache, const void* k_new,
                               const void* v_new, int32_t max_new, const int32_t* n_new,
                               void* workspace, size_t workspace_bytes, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if (max_new < 0) return SPLA_ERR_INVALID_ARG;
  if (max_new > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  if (max_new == 0) return SPLA_OK;
  if (!k_new || !v_new) return SPLA_ERR_INVALID_ARG;
  size_t need = 0;
  spla_append_workspace_bytes(cfg, max_new, &need);
  if ((s = check_ws(workspace, workspace_bytes, need)) != SPLA_OK) return s;
  const Dims m = spla::make_dims(*cfg);
  const spla::AppendWs L = spla::append_ws_layout(m, max_new);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (spla::append_fusable(m)) {  // the lengths advance in its last launch
    SPLA_TRY(spla::launch_append_fused(m, *cache, k_new, v_new, max_new, n_new, L,
                                       static_cast<char*>(workspace), st));
  } else {
    SPLA_TRY(spla::launch_append_blocks(m, *cache, k_new, v_new, max_new, n_new, st));
    SPLA_TRY(spla::launch_append_state(m, *cache, k_new, v_new, max_new, n_new, L,
                                       static_cast<char*>(workspace), st));
    SPLA_TRY(spla::launch_append_finish(m, *cache, max_new, n_new, st));
  }
  return SPLA_OK;
}

extern "C" int32_t spla_decode_ex(const spla_config* cfg, const spla_cache* cache, const void* q,
                                  const float* w, void* out, int32_t* sel_idx, void* ws,
                                  size_t ws_bytes, const spla_events* ev, void* stream) {
  int32_t s = check_decode_args(cfg, cache, q, w, out, ws, ws_bytes);
  if (s != SPLA_OK) return s;
  return run_decode(cfg, cache, q, w, out, sel_idx, ws, ws_bytes, ev,
                    static_cast<hipStream_t>(stream));
}

extern "C" int32_t spla_decode(const spla_config* cfg, const spla_cache* cache, const void* q,
                               const float* w, void* out, int32_t* sel_idx, void* ws,
                               size_t ws_bytes, void* stream) {
  return spla_decode_ex(cfg, cache, q, w, out, sel_idx, ws, ws_bytes, nullptr, stream);
}

extern "C" int32_t spla_step_ex(const spla_config* cfg, const spla_cache* cache, const void* k_new,
                                const void* v_new, const void* q, const float* w, void* out,
                                int32_t* sel_idx, void* ws, size_t ws_bytes,
                                const spla_events* ev, void* stream) {
  int32_t s = check_decode_args(cfg, cache, q, w, out, ws, ws_bytes);
  if (s != SPLA_OK) return s;
  if (!k_new || !v_new) return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // the append's last workgroup of each sequence advances its length (the
  // counters: the workspace's item lines, zero between calls)
  const spla::DecodeWs L = spla::decode_ws_layout(m);
  char* base = static_cast<char*>(ws);
  int32_t* fin = reinterpret_cast<int32_t*>(base + L.sync) + spla::sync_layout(m).items_done;
  if (spla::step_fusable(m)) {
    // the token's rows and statistics first (in one launch with the decode
    // where that is one); its rank-one update of S_bar is applied by the
    // decode's sparse pass to the rows it reads anyway
    {
      PhaseMark pm(ev, st, SPLA_PHASE_APPEND);
      if (!spla::use_fused_decode(m) || (cfg->flags & SPLA_FLAG_SEPARATE_KERNELS))
        SPLA_TRY(spla::launch_append_one(m, *cache, k_new, v_new, st, false, fin,
                                         reinterpret_cast<int32_t*>(base + L.appended)));
    }
    return run_decode(cfg, cache, q, w, out, sel_idx, ws, ws_bytes, ev, st, k_new, v_new);
  }
  {
    PhaseMark pm(ev, st, SPLA_PHASE_APPEND);
    SPLA_TRY(spla::launch_append_one(m, *cache, k_new, v_new, st, true, fin));
  }
  return run_decode(cfg, cache, q, w, out, sel_idx, ws, ws_bytes, ev, st);
}

extern "C" int32_t spla_step(const spla_config* cfg, const spla_cache* cache, const void* k_new,
                             const void* v_new, const void* q, const float* w, void* out,
                             int32_t* sel_idx, void* ws, size_t ws_bytes, void* stream) {
  return spla_step_ex(cfg, cache, k_new, v_new, q, w, out, sel_idx, ws, ws_bytes, nullptr, stream);
}

extern "C" int32_t spla_prefill_ex(const spla_config* cfg, const spla_cache* cache,
                                   int32_t n_tokens, const void* k_new, const void* v_new,
                                   const void* q, const float* w, void* out, int32_t* sel_idx,
                                   void* ws, size_t ws_bytes, const spla_events* ev,
                                   void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if (!q || !w || !out || out == q) return SPLA_ERR_INVALID_ARG;
  if (n_tokens < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  if (n_tokens == 0) return SPLA_OK;
  if (!k_new || !v_new) return SPLA_ERR_INVALID_ARG;
  size_t need = 0;
  spla_prefill_workspace_bytes(cfg, n_tokens, &need);
  if ((s = check_ws(ws, ws_bytes, need)) != SPLA_OK) return s;
  const Dims m = spla::make_dims(*cfg);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // per position: the rows of token t, the queries at t, their outputs
  const size_t kv_step = (size_t)m.bh * m.d * m.elem;
  const size_t q_step = (size_t)m.batch * m.hq * m.d * m.elem;
  const size_t sel_step = (size_t)m.bh * m.k;
  const char* kb = static_cast<const char*>(k_new);
  const char* vb = static_cast<const char*>(v_new);
  const char* qb = static_cast<const char*>(q);
  char* ob = static_cast<char*>(out);
  if (spla::use_chunked_prefill(m)) {
    const spla::PrefillWs L = spla::prefill_ws_layout(m, n_tokens);
    // chunks of about equal size
    const int n_chunks = (n_tokens - 1) / L.T + 1, step = (n_tokens - 1) / n_chunks + 1;
    for (int32_t c0 = 0; c0 < n_tokens; c0 += step) {
      const int T = n_tokens - c0 < step ? n_tokens - c0 : step;
      SPLA_TRY(spla::launch_prefill_chunk(m, *cfg, *cache, T, kb + c0 * kv_step,
                                          vb + c0 * kv_step, qb + c0 * q_step, w,
                                          ob + c0 * q_step,
                                          sel_idx ? sel_idx + c0 * sel_step : nullptr, L,
                                          static_cast<char*>(ws), ev, st));
    }
    return SPLA_OK;
  }
  // the decode workspace: its item lines count the append's workgroups; it
  // comes unprepared, so its synchronisation area is cleared first
  char* sync = static_cast<char*>(ws) + spla::decode_ws_layout(m).sync;
  SPLA_TRY(spla::launch_fill_zero(sync, (size_t)spla::sync_layout(m).words * 4, st));
  int32_t* fin = reinterpret_cast<int32_t*>(sync) + spla::sync_layout(m).items_done;
  for (int32_t t = 0; t < n_tokens; ++t) {
    SPLA_TRY(spla::launch_append_one(m, *cache, kb + t * kv_step, vb + t * kv_step, st, true,
                                     fin));
    if ((s = run_decode(cfg, cache, qb + t * q_step, w, ob + t * q_step,
                        sel_idx ? sel_idx + t * sel_step : nullptr, ws, ws_bytes, nullptr, st)) !=
        SPLA_OK)
      return s;
  }
  return SPLA_OK;
}

extern "C" int32_t spla_prefill(const spla_config* cfg, const spla_cache* cache, int32_t n_tokens,
                                const void* k_new, const void* v_new, const void* q,
                                const float* w, void* out, int32_t* sel_idx, void* ws,
                                size_t ws_bytes, void* stream) {
  return spla_prefill_ex(cfg, cache, n_tokens, k_new, v_new, q, w, out, sel_idx, ws, ws_bytes,
                         nullptr, stream);
}

// ---- rotary positions and exact attention ------------------------------------
namespace {

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// rows of `heads` heads at a stride of `stride` elements
bool good_rows(const Dims& m, const void* p, int64_t stride, int heads) {
  return p && aligned16(p) && stride >= (int64_t)heads * m.d && stride * m.elem % 16 == 0;
}

}  // namespace

extern "C" int32_t spla_rotate(const spla_config* cfg, const spla_rope* rope, int32_t n_tokens,
                               const int32_t* positions, const int32_t* seq_lens, const void* q,
                               int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k,
                               int64_t k_stride, void* k_out, int64_t k_out_stride,
                               int32_t transpose, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = spla::check_rope(*cfg, rope)) != SPLA_OK) return s;
  if (n_tokens < 0 || (transpose != 0 && transpose != 1)) return SPLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPLA_OK;
  if ((!q && !k) || (q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr))
    return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  if (q && (!good_rows(m, q, q_stride, m.hq) || !good_rows(m, q_out, q_out_stride, m.hq)))
    return SPLA_ERR_INVALID_ARG;
  if (k && (!good_rows(m, k, k_stride, m.hkv) || !good_rows(m, k_out, k_out_stride, m.hkv)))
    return SPLA_ERR_INVALID_ARG;
  if ((q == q_out && q_stride != q_out_stride) || (k == k_out && k_stride != k_out_stride))
    return SPLA_ERR_INVALID_ARG;
  const int64_t nb = m.batch;
  const spla::RotateSet a{q, q_out, nb * q_stride, q_stride, m.d, nb * q_out_stride, q_out_stride,
                          m.d, q ? m.hq : 0};
  const spla::RotateSet b{k, k_out, nb * k_stride, k_stride, m.d, nb * k_out_stride, k_out_stride,
                          m.d, k ? m.hkv : 0};
  const spla::RotateRows rows{n_tokens, m.batch, positions, positions ? nullptr : seq_lens, nullptr,
                              nullptr};
  SPLA_TRY(spla::launch_rotate(m, *rope, rows, a, b, transpose != 0,
                               static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_append_rope(const spla_config* cfg, const spla_cache* cache,
                                    const spla_rope* rope, const void* k_new, const void* v_new,
                                    int32_t max_new, const int32_t* n_new,
                                    const int32_t* pos_shift, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if ((s = spla::check_rope(*cfg, rope)) != SPLA_OK) return s;
  if (max_new < 0) return SPLA_ERR_INVALID_ARG;
  if (max_new > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  if (max_new == 0) return SPLA_OK;
  if (!k_new || !v_new || !aligned16(k_new) || !aligned16(v_new)) return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  const spla::AppendRopeWs L = spla::append_rope_ws_layout(m, max_new, rope->rot_dim);
  if ((s = check_ws(workspace, workspace_bytes, (size_t)L.total)) != SPLA_OK) return s;
  char* ws = static_cast<char*>(workspace);
  if (max_new == 1) {
    SPLA_TRY(spla::launch_append_rope_one(m, *cache, *rope, k_new, v_new, n_new, pos_shift,
                                          reinterpret_cast<int32_t*>(ws + L.count),
                                          static_cast<hipStream_t>(stream)));
    return SPLA_OK;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  const spla::AppendWs A = spla::append_ws_layout(m, max_new);
  const bool one_pass = spla::append_fusable(m);
  if (spla::append_rotates(m, rope->rot_dim)) {
    SPLA_TRY(spla::launch_append_fused(m, *cache, k_new, v_new, max_new, n_new, A, ws + L.append,
                                       st, rope, pos_shift));
    return SPLA_OK;
  }
  const int64_t s_h = (int64_t)max_new * m.d, s_b = s_h * m.hkv;
  const spla::RotateSet set{k_new, ws + L.k_rot, m.d, s_b, s_h, m.d, s_b, s_h, m.hkv};
  const spla::RotateRows rows{max_new, m.batch, nullptr, cache->seq_lens, pos_shift, n_new};
  SPLA_TRY(spla::launch_rotate(m, *rope, rows, set, spla::RotateSet{}, false, st));
  const void* kr = ws + L.k_rot;
  if (one_pass) {
    const spla_rope none{};
    SPLA_TRY(spla::launch_append_fused(m, *cache, kr, v_new, max_new, n_new, A, ws + L.append, st,
                                       &none));
    return SPLA_OK;
  }
  SPLA_TRY(spla::launch_append_blocks(m, *cache, kr, v_new, max_new, n_new, st));
  SPLA_TRY(spla::launch_append_state(m, *cache, kr, v_new, max_new, n_new, A, ws + L.append, st,
                                     true, true));
  return SPLA_OK;
}

extern "C" int32_t spla_attend(const spla_config* cfg, const spla_cache* cache, int32_t n_tokens,
                               const void* q, const spla_attend_opts* opts, void* out, float* lse,
                               void* workspace, size_t workspace_bytes, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if (n_tokens < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  const spla_attend_opts o = opts ? *opts : spla_attend_opts{};
  if (o.softcap != 0.f && !(o.softcap >= SPLA_SOFTCAP_MIN && o.softcap <= SPLA_SOFTCAP_MAX))
    return SPLA_ERR_INVALID_ARG;  // (NaN too)
  if (n_tokens == 0) return SPLA_OK;
  if (!q || !out || out == q || !aligned16(q) || !aligned16(out)) return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  const spla::AttendWs L = spla::attend_ws_layout(m, n_tokens);
  if ((s = check_ws(workspace, workspace_bytes, (size_t)L.total)) != SPLA_OK) return s;
  SPLA_TRY(spla::launch_attend(m, *cfg, *cache, n_tokens, q, o, out, lse, L,
                               static_cast<char*>(workspace), static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

// ---- per-head norms with the rotation, the 8-bit cache -------------------------
namespace {

// What spla_norm_rotate and its gradients check alike.
int32_t check_norm(const spla_config* cfg, const spla_rope* rope, int32_t n_tokens,
                   const float* q_weight, const float* k_weight, int32_t per_head, double eps) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = spla::check_rope(*cfg, rope)) != SPLA_OK) return s;
  if (n_tokens < 0 || (per_head != 0 && per_head != 1)) return SPLA_ERR_INVALID_ARG;
  if (!(eps >= 0.0) || !(eps <= 1.7976931348623157e308)) return SPLA_ERR_INVALID_ARG;  // (NaN too)
  if (!aligned16(q_weight) || !aligned16(k_weight)) return SPLA_ERR_INVALID_ARG;
  return SPLA_OK;
}

spla::NormSet norm_set(const Dims& m, const void* x, int64_t xs, void* y, int64_t ys, int heads,
                       const float* w, bool per_head, const void* g, int64_t gs) {
  const int64_t nb = m.batch;
  return spla::NormSet{{x, y, nb * xs, xs, m.d, nb * ys, ys, m.d, x ? heads : 0},
                       w, per_head ? m.d : 0, g, nb * gs, gs};
}

int32_t check_cache8(const spla_config* cfg, const spla_cache8* c) {
  if (!c) return SPLA_ERR_INVALID_ARG;
  if (!c->k_codes || !c->v_codes || !c->scales || !c->seq_lens || !c->counters)
    return SPLA_ERR_INVALID_ARG;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return SPLA_ERR_INVALID_ARG;
  if ((cfg->kv_pages > 0) != (c->block_table != nullptr)) return SPLA_ERR_INVALID_ARG;
  return SPLA_OK;
}

}  // namespace

extern "C" int32_t spla_norm_rotate(const spla_config* cfg, const spla_rope* rope,
                                    int32_t n_tokens, const int32_t* positions,
                                    const int32_t* seq_lens, const float* q_weight,
                                    const float* k_weight, int32_t weight_per_head, double eps,
                                    const void* q, int64_t q_stride, void* q_out,
                                    int64_t q_out_stride, const void* k, int64_t k_stride,
                                    void* k_out, int64_t k_out_stride, void* stream) {
  int32_t s = check_norm(cfg, rope, n_tokens, q_weight, k_weight, weight_per_head, eps);
  if (s != SPLA_OK) return s;
  if (n_tokens == 0) return SPLA_OK;
  if ((!q && !k) || (q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr))
    return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  if (q && (!good_rows(m, q, q_stride, m.hq) || !good_rows(m, q_out, q_out_stride, m.hq)))
    return SPLA_ERR_INVALID_ARG;
  if (k && (!good_rows(m, k, k_stride, m.hkv) || !good_rows(m, k_out, k_out_stride, m.hkv)))
    return SPLA_ERR_INVALID_ARG;
  if ((q == q_out && q_stride != q_out_stride) || (k == k_out && k_stride != k_out_stride))
    return SPLA_ERR_INVALID_ARG;
  const spla::NormSet a = norm_set(m, q, q_stride, q_out, q_out_stride, m.hq, q_weight,
                                   weight_per_head, nullptr, 0);
  const spla::NormSet b = norm_set(m, k, k_stride, k_out, k_out_stride, m.hkv, k_weight,
                                   weight_per_head, nullptr, 0);
  const spla::RotateRows rows{n_tokens, m.batch, positions, positions ? nullptr : seq_lens, nullptr,
                              nullptr};
  SPLA_TRY(spla::launch_norm_rotate(m, *rope, eps, rows, a, b, static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_norm_rotate_grad(
    const spla_config* cfg, const spla_rope* rope, int32_t n_tokens, const int32_t* positions,
    const int32_t* seq_lens, const float* q_weight, const float* k_weight, int32_t weight_per_head,
    double eps, const void* q, int64_t q_stride, const void* q_grad, int64_t q_grad_stride,
    void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, const void* k_grad,
    int64_t k_grad_stride, void* k_out, int64_t k_out_stride, float* q_weight_grad,
    float* k_weight_grad, void* workspace, size_t workspace_bytes, void* stream) {
  int32_t s = check_norm(cfg, rope, n_tokens, q_weight, k_weight, weight_per_head, eps);
  if (s != SPLA_OK) return s;
  const Dims m = spla::make_dims(*cfg);
  if (n_tokens > 0) {
    if ((!q && !k) || (q != nullptr) != (q_out != nullptr) ||
        (k != nullptr) != (k_out != nullptr) || (q != nullptr) != (q_grad != nullptr) ||
        (k != nullptr) != (k_grad != nullptr))
      return SPLA_ERR_INVALID_ARG;
    if (q && (!good_rows(m, q, q_stride, m.hq) || !good_rows(m, q_out, q_out_stride, m.hq) ||
              !good_rows(m, q_grad, q_grad_stride, m.hq)))
      return SPLA_ERR_INVALID_ARG;
    if (k && (!good_rows(m, k, k_stride, m.hkv) || !good_rows(m, k_out, k_out_stride, m.hkv) ||
              !good_rows(m, k_grad, k_grad_stride, m.hkv)))
      return SPLA_ERR_INVALID_ARG;
    if ((q && q == q_out && q_stride != q_out_stride) ||
        (k && k == k_out && k_stride != k_out_stride) ||
        (q && q_grad == q_out && q_grad_stride != q_out_stride) ||
        (k && k_grad == k_out && k_grad_stride != k_out_stride))
      return SPLA_ERR_INVALID_ARG;
    // a weight's gradient goes with its rows
    if ((q_weight_grad && !q) || (k_weight_grad && !k)) return SPLA_ERR_INVALID_ARG;
  }
  const spla::NormGradWs L = spla::norm_grad_ws_layout(m, n_tokens);
  const bool sums = q_weight_grad || k_weight_grad;
  if (sums && (s = check_ws(workspace, workspace_bytes, (size_t)L.total)) != SPLA_OK) return s;
  if (n_tokens == 0 && !sums) return SPLA_OK;
  const spla::NormSet a = norm_set(m, q, q_stride, q_out, q_out_stride, m.hq, q_weight,
                                   weight_per_head, q_grad, q_grad_stride);
  const spla::NormSet b = norm_set(m, k, k_stride, k_out, k_out_stride, m.hkv, k_weight,
                                   weight_per_head, k_grad, k_grad_stride);
  const spla::RotateRows rows{n_tokens, m.batch, positions, positions ? nullptr : seq_lens, nullptr,
                              nullptr};
  SPLA_TRY(spla::launch_norm_rotate_grad(m, *rope, eps, rows, a, b, q_weight_grad, k_weight_grad, L,
                                         static_cast<char*>(workspace),
                                         static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_reset8(const spla_config* cfg, const spla_cache8* cache, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache8(cfg, cache)) != SPLA_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(stream);
  SPLA_TRY(spla::launch_fill_zero(cache->seq_lens, (size_t)cfg->batch * 4, st));
  SPLA_TRY(spla::launch_fill_zero(cache->counters, (size_t)cfg->batch * spla::kSyncLine * 4, st));
  return SPLA_OK;
}

extern "C" int32_t spla_append8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                                const void* k_new, int64_t k_stride, const void* v_new,
                                int64_t v_stride, const int32_t* n_new, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache8(cfg, cache)) != SPLA_OK) return s;
  if (n_tokens < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  if (n_tokens == 0) return SPLA_OK;
  const Dims m = spla::make_dims(*cfg);
  if (!good_rows(m, k_new, k_stride, m.hkv) || !good_rows(m, v_new, v_stride, m.hkv))
    return SPLA_ERR_INVALID_ARG;
  SPLA_TRY(spla::launch_append8(m, *cache, n_tokens, k_new, k_stride, v_new, v_stride, n_new,
                                static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_read8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                              const int32_t* first, void* k_out, void* v_out, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache8(cfg, cache)) != SPLA_OK) return s;
  if (n_tokens < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPLA_OK;
  if ((!k_out && !v_out) || !aligned16(k_out) || !aligned16(v_out) || k_out == v_out)
    return SPLA_ERR_INVALID_ARG;
  SPLA_TRY(spla::launch_read8(spla::make_dims(*cfg), *cache, n_tokens, first, k_out, v_out,
                              static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

extern "C" int32_t spla_attend8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                                const void* q, const spla_attend8_opts* opts, void* out,
                                float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache8(cfg, cache)) != SPLA_OK) return s;
  if (n_tokens < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens > cfg->max_seq_len) return SPLA_ERR_CAPACITY;
  const spla_attend8_opts o = opts ? *opts : spla_attend8_opts{};
  const float c = o.attend.softcap;
  if (c != 0.f && !(c >= SPLA_SOFTCAP_MIN && c <= SPLA_SOFTCAP_MAX))
    return SPLA_ERR_INVALID_ARG;  // (NaN too)
  if (o.window < 0 || o.sinks < 0) return SPLA_ERR_INVALID_ARG;
  if (n_tokens == 0) return SPLA_OK;
  if (!q || !out || out == q || !aligned16(q) || !aligned16(out)) return SPLA_ERR_INVALID_ARG;
  const Dims m = spla::make_dims(*cfg);
  const size_t need = (size_t)spla::attend8_ws_bytes(m, n_tokens);
  if ((s = check_ws(workspace, workspace_bytes, need)) != SPLA_OK) return s;
  const spla::AttendWs L =
      spla::attend8_ws_layout(m, n_tokens, spla::attend8_keys(m, n_tokens, o));
  SPLA_TRY(spla::launch_attend8(m, *cfg, *cache, n_tokens, q, o, out, lse, L,
                                static_cast<char*>(workspace), static_cast<hipStream_t>(stream)));
  return SPLA_OK;
}

// ---- decode without a caller workspace (callers that cannot allocate) ------
// The decode workspace of spla_decode_noalloc: one copy of this array per
// device, held by every GPU the library runs on until the process ends. In
// host code `scratch` only names the array; its device address is taken once
// per device with hipGetSymbolAddress and only that address is handed to
// kernels.
static __device__ __align__(256) unsigned char scratch[SPLA_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch[kMaxDevices] = {};

// Device address of the current device's scratch; the first call on a device
// takes it (with that device current) and zero-fills the array on `st`.
int32_t device_scratch(hipStream_t st, void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SPLA_ERR_HIP;
  if (dev < 0 || dev >= kMaxDevices) return SPLA_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch[dev]) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return SPLA_ERR_HIP;
    if (spla::launch_fill_zero(p, SPLA_NOALLOC_SCRATCH_BYTES, st) != hipSuccess)
      return SPLA_ERR_HIP;
    g_scratch[dev] = p;
  }
  *out = g_scratch[dev];
  return SPLA_OK;
}

}  // namespace

extern "C" int32_t spla_decode_noalloc(const spla_config* cfg, const spla_cache* cache,
                                       const void* q, const float* w, void* out,
                                       int32_t* sel_idx, void* stream) {
  int32_t s = spla_validate(cfg);
  if (s != SPLA_OK) return s;
  if ((s = check_cache(cfg, cache)) != SPLA_OK) return s;
  if (!q || !w || !out || out == q) return SPLA_ERR_INVALID_ARG;
  size_t need = 0;
  spla_workspace_bytes(cfg, &need);
  if (need > (size_t)SPLA_NOALLOC_SCRATCH_BYTES) return SPLA_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  void* base = nullptr;
  if ((s = device_scratch(st, &base)) != SPLA_OK) return s;
  const Dims m = spla::make_dims(*cfg);
  const spla::DecodeWs L = spla::decode_ws_layout(m);
  // the counters (single launch, selection folded into the scoring launch,
  // two-stage selection) must start at zero; the previous call may have
  // left other data there (another layout), so the synchronisation area is
  // cleared with a fill kernel on every call
  SPLA_TRY(spla::launch_fill_zero(static_cast<char*>(base) + L.sync, (size_t)(L.total - L.sync),
                                  st));
  return run_decode(cfg, cache, q, w, out, sel_idx, base, need, nullptr, st);
}
