// C-ABI entry points: argument checks, then stage launchers. No entry point allocates or synchronises, except
// madakv_poll_status, which synchronises the stream to read the device status word.
#include <initializer_list>

#include "common.cuh"

using namespace madakv;

extern "C" {

int madakv_abi_version(void) { return 4; }

const char* madakv_status_string(int s) {
  switch (s) {
    case MADAKV_OK: return "ok";
    case MADAKV_EINVAL: return "invalid argument";
    case MADAKV_ESHAPE: return "bad shape";
    case MADAKV_EALIGN: return "misaligned pointer or stride";
    case MADAKV_EWORKSPACE: return "workspace too small";
    case MADAKV_ECAPACITY: return "ragged cache capacity exceeded";
    case MADAKV_EUNSUPPORTED: return "unsupported dtype, head_dim or window";
    case MADAKV_ECUDA: return "CUDA runtime error";
    case MADAKV_ETIMEOUT: return "bounded device wait expired";
    case MADAKV_ESTATIC: return "problem exceeds the built-in scratch of madakv_decode_attn_static";
    default: return "unknown status";
  }
}

int madakv_workspace_bytes(const madakv_config* cfg, size_t* bytes_out) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!bytes_out) return MADAKV_EINVAL;
  *bytes_out = ws_layout(*cfg).total;
  return MADAKV_OK;
}

int madakv_workspace_bytes_attn(const madakv_config* cfg, size_t* bytes_out) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!bytes_out) return MADAKV_EINVAL;
  *bytes_out = ws_bytes_attn(*cfg);
  return MADAKV_OK;
}

int madakv_score(const madakv_config* cfg, const void* q_win, madakv_strides sq, const void* k, madakv_strides sk,
                 const int32_t* seq_len, float* lse, float* psi, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!q_win || !k || !seq_len || !psi) return MADAKV_EINVAL;
  if (!aligned16(q_win) || !aligned16(k) || !aligned16(psi) || ((uintptr_t)seq_len & 3) || ((uintptr_t)lse & 3))
    return MADAKV_EALIGN;
  if (!strides_ok(*cfg, sq) || !strides_ok(*cfg, sk)) return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_score(*cfg, q_win, sq, k, sk, seq_len, lse, psi, ws, (cudaStream_t)stream);
}

static int check_score_lse(const madakv_config* cfg, const void* q_win, madakv_strides sq, const void* k, madakv_strides sk,
                           const int32_t* seq_len, const float* lse, const float* psi, const void* ws, size_t ws_bytes) {
  if (const int rc = check_config(cfg)) return rc;
  if (!q_win || !k || !seq_len || !lse || !psi) return MADAKV_EINVAL;
  if (!aligned16(q_win) || !aligned16(k) || !aligned16(psi) || ((uintptr_t)seq_len & 3) || ((uintptr_t)lse & 3))
    return MADAKV_EALIGN;
  if (!strides_ok(*cfg, sq) || !strides_ok(*cfg, sk)) return MADAKV_EALIGN;
  return check_ws(*cfg, ws, ws_bytes);
}

int madakv_score_lse(const madakv_config* cfg, const void* q_win, madakv_strides sq, const void* k, madakv_strides sk,
                     const int32_t* seq_len, const float* lse, float* psi, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_score_lse(cfg, q_win, sq, k, sk, seq_len, lse, psi, ws, ws_bytes)) return rc;
  return launch_score_lse(*cfg, q_win, sq, k, sk, seq_len, lse, psi, ws, (cudaStream_t)stream);
}

int madakv_score_kept(const madakv_config* cfg, const void* q_win, madakv_strides sq, const void* k, madakv_strides sk,
                      const int32_t* seq_len, const float* lse, int32_t* win_len, float* psi, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_score_lse(cfg, q_win, sq, k, sk, seq_len, lse, psi, ws, ws_bytes);
  if (rc) return rc;
  if (!win_len) return MADAKV_EINVAL;
  if ((uintptr_t)win_len & 3) return MADAKV_EALIGN;
  if ((rc = launch_window_check(*cfg, seq_len, win_len, ws, (cudaStream_t)stream))) return rc;
  return launch_score_lse(*cfg, q_win, sq, k, sk, seq_len, lse, psi, ws, (cudaStream_t)stream);
}

int madakv_allocate(const madakv_config* cfg, const float* psi, const uint8_t* mask, const int32_t* seq_len,
                    const int32_t* budget, double* mass, double* pref, int32_t* demand, double* phi, int32_t* budgets,
                    void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!psi || !mask || !seq_len || !budget || !mass || !pref || !demand || !phi || !budgets) return MADAKV_EINVAL;
  if (!aligned16(psi) || ((uintptr_t)mass & 7) || ((uintptr_t)pref & 7) || ((uintptr_t)phi & 7) ||
      ((uintptr_t)demand & 7) || ((uintptr_t)budgets & 7) || ((uintptr_t)seq_len & 3) || ((uintptr_t)budget & 3))
    return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_allocate(*cfg, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws, (cudaStream_t)stream);
}

int madakv_allocate_layer(const madakv_config* cfg, int32_t layer, const float* psi, const uint8_t* mask,
                          const int32_t* seq_len, const int32_t* budget, double* mass, double* pref, int32_t* demand,
                          double* phi, int32_t* budgets, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (layer < 0 || layer >= cfg->n_layers) return MADAKV_ESHAPE;
  // psi may be null: mass, pref and demand of the layer then come from madakv_demand_layer
  if (!mask || !seq_len || !budget || !mass || !pref || !demand || !phi || !budgets) return MADAKV_EINVAL;
  if (!aligned16(psi) || ((uintptr_t)mass & 7) || ((uintptr_t)pref & 7) || ((uintptr_t)phi & 7) ||
      ((uintptr_t)demand & 7) || ((uintptr_t)budgets & 7) || ((uintptr_t)seq_len & 3) || ((uintptr_t)budget & 3))
    return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_allocate_layer(*cfg, layer, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws,
                               (cudaStream_t)stream);
}

int madakv_demand_layer(const madakv_config* cfg, const float* psi, const uint8_t* mask, const int32_t* seq_len,
                        double* mass, double* pref, int32_t* demand, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!psi || !mask || !seq_len || !mass || !pref || !demand) return MADAKV_EINVAL;
  if (!aligned16(psi) || ((uintptr_t)mass & 7) || ((uintptr_t)pref & 7) || ((uintptr_t)demand & 7) ||
      ((uintptr_t)seq_len & 3))
    return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_demand_layer(*cfg, psi, mask, seq_len, mass, pref, demand, ws, (cudaStream_t)stream);
}

int madakv_select(const madakv_config* cfg, const float* psi, const uint8_t* mask, const int32_t* seq_len,
                  const int32_t* budgets, int32_t* kept_len, int64_t* seg_off, int32_t* kept_idx, int64_t capacity,
                  void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!psi || !mask || !seq_len || !budgets || !kept_len || !seg_off || !kept_idx) return MADAKV_EINVAL;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(psi) || ((uintptr_t)budgets & 7) || ((uintptr_t)kept_len & 3) || ((uintptr_t)seg_off & 7) ||
      ((uintptr_t)kept_idx & 3) || ((uintptr_t)seq_len & 3))
    return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_select(*cfg, psi, mask, seq_len, budgets, kept_len, seg_off, kept_idx, capacity, ws,
                       (cudaStream_t)stream);
}

int madakv_compact(const madakv_config* cfg, const void* k, const void* v, madakv_strides skv, const int32_t* kept_idx,
                   const int64_t* seg_off, const int32_t* kept_len, void* k_c, void* v_c, int64_t capacity, void* ws,
                   size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!k || !v || !kept_idx || !seg_off || !kept_len || !k_c || !v_c) return MADAKV_EINVAL;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_c) || !aligned16(v_c) || ((uintptr_t)kept_idx & 3) ||
      ((uintptr_t)seg_off & 7) || ((uintptr_t)kept_len & 3))
    return MADAKV_EALIGN;
  if (!strides_ok(*cfg, skv)) return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_compact(*cfg, k, v, skv, kept_idx, seg_off, kept_len, k_c, v_c, capacity, ws, (cudaStream_t)stream);
}

int madakv_decode_attn(const madakv_config* cfg, int32_t layer, const void* q, const void* k_new, const void* v_new,
                       void* k_c, void* v_c, const int64_t* seg_off, int32_t* kept_len, int64_t capacity, void* out,
                       float* lse_out, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!q || !k_c || !v_c || !seg_off || !kept_len || !out) return MADAKV_EINVAL;
  if ((k_new == nullptr) != (v_new == nullptr)) return MADAKV_EINVAL;
  if (layer < -1 || layer >= cfg->n_layers) return MADAKV_ESHAPE;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_c) || !aligned16(v_c) ||
      !aligned16(out) || ((uintptr_t)seg_off & 7) || ((uintptr_t)kept_len & 3) || ((uintptr_t)lse_out & 3))
    return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_decode(*cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, capacity, out, lse_out, nullptr, ws,
                       (cudaStream_t)stream);
}

// What a tracking call may be given. `track.acc` null: no tracking.
static int check_tracking(const Tracking& track) {
  if ((track.acc == nullptr) != (track.scores == nullptr)) return MADAKV_EINVAL;
  if ((track.kept_idx == nullptr) != (track.position == nullptr)) return MADAKV_EINVAL;
  if (!track.acc && track.kept_idx) return MADAKV_EINVAL;
  if (track.acc && !(track.decay >= 0.0f && track.decay <= 1.0f)) return MADAKV_EINVAL;
  if (((uintptr_t)track.acc & 3) || ((uintptr_t)track.scores & 15) || ((uintptr_t)track.kept_idx & 3) ||
      ((uintptr_t)track.position & 3))
    return MADAKV_EALIGN;
  return MADAKV_OK;
}

int madakv_decode_attn_track(const madakv_config* cfg, int32_t layer, const void* q, const void* k_new, const void* v_new,
                             void* k_c, void* v_c, const int64_t* seg_off, int32_t* kept_len, int64_t capacity, void* out,
                             float* lse_out, float* acc, float* scratch, int32_t* kept_idx, const int32_t* position,
                             float decay, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  const Tracking track{acc, scratch, kept_idx, position, decay};
  if (!q || !k_c || !v_c || !seg_off || !kept_len || !out || !acc) return MADAKV_EINVAL;
  if ((k_new == nullptr) != (v_new == nullptr)) return MADAKV_EINVAL;
  if (layer < -1 || layer >= cfg->n_layers) return MADAKV_ESHAPE;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_c) || !aligned16(v_c) ||
      !aligned16(out) || ((uintptr_t)seg_off & 7) || ((uintptr_t)kept_len & 3) || ((uintptr_t)lse_out & 3))
    return MADAKV_EALIGN;
  if ((rc = check_tracking(track))) return rc;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_decode(*cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, capacity, out, lse_out, &track, ws,
                       (cudaStream_t)stream);
}

int madakv_compact_quant(const madakv_config* cfg, const void* k, const void* v, madakv_strides skv, const int32_t* kept_idx,
                         const int64_t* seg_off, const int32_t* kept_len, uint8_t* k_code, void* k_par, uint8_t* v_code,
                         void* v_par, int64_t capacity, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!k || !v || !kept_idx || !seg_off || !kept_len || !k_code || !k_par || !v_code || !v_par) return MADAKV_EINVAL;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_code) || !aligned16(k_par) || !aligned16(v_code) || !aligned16(v_par) ||
      ((uintptr_t)kept_idx & 3) || ((uintptr_t)seg_off & 7) || ((uintptr_t)kept_len & 3))
    return MADAKV_EALIGN;
  if (!strides_ok(*cfg, skv)) return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_compact_quant(*cfg, k, v, skv, kept_idx, seg_off, kept_len, k_code, k_par, v_code, v_par, capacity,
                              (cudaStream_t)stream);
}

int madakv_expand_quant(const madakv_config* cfg, const int64_t* rows, int64_t n_rows, const uint8_t* k_code,
                        const void* k_par, const uint8_t* v_code, const void* v_par, int64_t capacity, void* k_out,
                        void* v_out, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!k_code || !k_par || !v_code || !v_par || !k_out || !v_out) return MADAKV_EINVAL;
  if (n_rows < 0) return MADAKV_ESHAPE;
  if (capacity <= 0 || (!rows && n_rows > capacity)) return MADAKV_ECAPACITY;
  if (((uintptr_t)rows & 7) || !aligned16(k_code) || !aligned16(k_par) || !aligned16(v_code) || !aligned16(v_par) ||
      !aligned16(k_out) || !aligned16(v_out))
    return MADAKV_EALIGN;
  if (n_rows == 0) return MADAKV_OK;
  return launch_expand_quant(*cfg, rows, n_rows, k_code, k_par, v_code, v_par, capacity, k_out, v_out, (cudaStream_t)stream);
}

int madakv_decode_attn_quant(const madakv_config* cfg, int32_t layer, const void* q, const void* k_new, const void* v_new,
                             uint8_t* k_code, void* k_par, uint8_t* v_code, void* v_par, const int64_t* seg_off,
                             int32_t* kept_len, int64_t capacity, void* out, float* lse_out, float* acc, float* scratch,
                             int32_t* kept_idx, const int32_t* position, float decay, void* ws, size_t ws_bytes,
                             void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  const Tracking track{acc, scratch, kept_idx, position, decay};
  if (!q || !k_code || !k_par || !v_code || !v_par || !seg_off || !kept_len || !out) return MADAKV_EINVAL;
  if ((k_new == nullptr) != (v_new == nullptr)) return MADAKV_EINVAL;
  if (layer < -1 || layer >= cfg->n_layers) return MADAKV_ESHAPE;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(k_code) || !aligned16(k_par) ||
      !aligned16(v_code) || !aligned16(v_par) || !aligned16(out) || ((uintptr_t)seg_off & 7) || ((uintptr_t)kept_len & 3) ||
      ((uintptr_t)lse_out & 3))
    return MADAKV_EALIGN;
  if ((rc = check_tracking(track))) return rc;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_decode_quant(*cfg, layer, q, k_new, v_new, k_code, k_par, v_code, v_par, seg_off, kept_len, capacity, out,
                             lse_out, acc ? &track : nullptr, ws, (cudaStream_t)stream);
}

// The two forms of eviction differ in the arrays whose rows move.
static int evict(const madakv_config* cfg, int32_t layer, const int32_t* limit, int32_t recent, float* acc, int32_t* kept_idx,
                 const int64_t* seg_off, int32_t* kept_len, int64_t capacity, const RowArray (&rows)[4], void* ws,
                 size_t ws_bytes, void* stream) {
  if (!limit || !acc || !kept_idx || !seg_off || !kept_len) return MADAKV_EINVAL;
  if (recent < 0) return MADAKV_EINVAL;
  if (layer < -1 || layer >= cfg->n_layers) return MADAKV_ESHAPE;
  if (capacity <= 0) return MADAKV_ECAPACITY;
  for (const RowArray& r : rows)
    if (!aligned16(r.base)) return MADAKV_EALIGN;
  if (((uintptr_t)limit & 3) || ((uintptr_t)acc & 3) || ((uintptr_t)kept_idx & 3) || ((uintptr_t)seg_off & 7) ||
      ((uintptr_t)kept_len & 3))
    return MADAKV_EALIGN;
  int rc;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_evict(*cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, capacity, rows, (cudaStream_t)stream);
}

int madakv_evict(const madakv_config* cfg, int32_t layer, const int32_t* limit, int32_t recent, float* acc, int32_t* kept_idx,
                 const int64_t* seg_off, int32_t* kept_len, int64_t capacity, void* k_c, void* v_c, void* ws,
                 size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!k_c || !v_c) return MADAKV_EINVAL;
  const int row = cfg->head_dim * elem_bytes(*cfg);
  return evict(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, capacity, {{k_c, row}, {v_c, row}, {nullptr, 0}, {nullptr, 0}},
               ws, ws_bytes, stream);
}

int madakv_evict_quant(const madakv_config* cfg, int32_t layer, const int32_t* limit, int32_t recent, float* acc,
                       int32_t* kept_idx, const int64_t* seg_off, int32_t* kept_len, int64_t capacity, uint8_t* k_code,
                       void* k_par, uint8_t* v_code, void* v_par, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!k_code || !k_par || !v_code || !v_par) return MADAKV_EINVAL;
  const int code = cfg->head_dim / 2, par = cfg->head_dim / 8;
  return evict(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, capacity,
               {{k_code, code}, {k_par, par}, {v_code, code}, {v_par, par}}, ws, ws_bytes, stream);
}

static bool all_strides_ok(const madakv_config& c, std::initializer_list<madakv_strides> all) {
  for (const madakv_strides& s : all)
    if (!strides_ok(c, s)) return false;
  return true;
}
// No dimension of more than one element of what a call writes has stride 0.
static bool rows_apart(int64_t batch, int64_t layers, int64_t heads, const madakv_strides& s) {
  return (batch <= 1 || s.batch) && (layers <= 1 || s.layer) && (heads <= 1 || s.head);
}

static int prefill(const madakv_config* cfg, int32_t layer, PromptCall a, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!a.q || !a.k || !a.v || !a.out) return MADAKV_EINVAL;
  if ((a.k_off != nullptr) == (a.seq_len != nullptr) || (a.q_off && a.q_len)) return MADAKV_EINVAL;
  if (layer < 0 || layer >= cfg->n_layers || a.q_rows <= 0 || a.k_rows <= 0) return MADAKV_ESHAPE;
  if (a.q_rows > 0x7fffffffll || a.k_rows > 0x7fffffffll) return MADAKV_EUNSUPPORTED;
  if (a.q_off) a.sq.batch = a.so.batch = 0;  // (packed: not used, whatever stands there)
  if (a.k_off) a.sk.batch = a.sv.batch = 0;
  if (!aligned16(a.q) || !aligned16(a.k) || !aligned16(a.v) || !aligned16(a.out) || !aligned16(a.q_win) || ((uintptr_t)a.q_off & 7) ||
      ((uintptr_t)a.k_off & 7) || ((uintptr_t)a.q_len & 3) || ((uintptr_t)a.seq_len & 3) || ((uintptr_t)a.lse_out & 3) ||
      ((uintptr_t)a.lse_win & 3) || ((uintptr_t)a.win_len & 3))
    return MADAKV_EALIGN;
  if (!all_strides_ok(*cfg, {a.sq, a.sk, a.sv, a.so})) return MADAKV_EALIGN;
  if (!rows_apart(a.q_off ? 1 : cfg->batch, 1, cfg->n_q_heads, a.so)) return MADAKV_EINVAL;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  a.part_rows = attn_part_rows(*cfg, ws_bytes);
  return launch_prefill_attn(*cfg, layer, a, ws, (cudaStream_t)stream);
}

int madakv_prefill_attn(const madakv_config* cfg, int32_t layer, const void* q, madakv_strides sq, int64_t q_rows,
                        const int64_t* q_off, const int32_t* q_len, const void* k, madakv_strides sk, const void* v,
                        madakv_strides sv, int64_t k_rows, const int64_t* k_off, const int32_t* seq_len, void* out,
                        madakv_strides so, float* lse_out, void* q_win, float* lse_win, void* ws, size_t ws_bytes, void* stream) {
  return prefill(cfg, layer, {q, sq, q_rows, q_off, q_len, k, sk, v, sv, k_rows, k_off, seq_len, out, so, lse_out, q_win, lse_win, nullptr, 0},
                 ws, ws_bytes, stream);
}

int madakv_prefill_attn_keep(const madakv_config* cfg, int32_t layer, const void* q, madakv_strides sq, int64_t q_rows,
                             const int64_t* q_off, const int32_t* q_len, const void* k, madakv_strides sk, const void* v,
                             madakv_strides sv, int64_t k_rows, const int64_t* k_off, const int32_t* seq_len, void* out,
                             madakv_strides so, float* lse_out, void* q_win, float* lse_win, int32_t* win_len, void* ws,
                             size_t ws_bytes, void* stream) {
  if (!q_win || !lse_win || !win_len) return MADAKV_EINVAL;
  return prefill(cfg, layer, {q, sq, q_rows, q_off, q_len, k, sk, v, sv, k_rows, k_off, seq_len, out, so, lse_out, q_win, lse_win, win_len, 0},
                 ws, ws_bytes, stream);
}

// What the two calls on drafted trees share.
static int check_tree(const madakv_config* cfg, int32_t layer, const TreeCall& a, const void* k_c, const void* v_c,
                      const int32_t* kept_len) {
  if (!a.k_tree || !a.v_tree || !a.mask || !k_c || !v_c || !a.seg_off || !kept_len) return MADAKV_EINVAL;
  if (layer < -1 || layer >= cfg->n_layers || a.nodes <= 0) return MADAKV_ESHAPE;
  if (a.nodes > 64) return MADAKV_EUNSUPPORTED;
  if (a.capacity <= 0) return MADAKV_ECAPACITY;
  if (!aligned16(a.k_tree) || !aligned16(a.v_tree) || !aligned16(k_c) || !aligned16(v_c) || ((uintptr_t)a.mask & 7) ||
      ((uintptr_t)a.n_nodes & 3) || ((uintptr_t)a.seg_off & 7) || ((uintptr_t)kept_len & 3))
    return MADAKV_EALIGN;
  return all_strides_ok(*cfg, {a.sk, a.sv}) ? MADAKV_OK : MADAKV_EALIGN;
}

int madakv_tree_attn(const madakv_config* cfg, int32_t layer, int32_t nodes, const void* q, madakv_strides sq, const void* k_tree,
                     madakv_strides sk, const void* v_tree, madakv_strides sv, const uint64_t* mask, const int32_t* n_nodes,
                     const void* k_c, const void* v_c, const int64_t* seg_off, const int32_t* kept_len, int64_t capacity,
                     void* out, madakv_strides so, float* lse_out, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  TreeCall a{nodes, q, sq, k_tree, sk, v_tree, sv, mask, n_nodes, seg_off, capacity, 0};
  if (!q || !out) return MADAKV_EINVAL;
  if ((rc = check_tree(cfg, layer, a, k_c, v_c, kept_len))) return rc;
  if (!aligned16(q) || !aligned16(out) || ((uintptr_t)lse_out & 3) || !all_strides_ok(*cfg, {sq, so})) return MADAKV_EALIGN;
  if (!rows_apart(cfg->batch, layer < 0 ? cfg->n_layers : 1, cfg->n_q_heads, so)) return MADAKV_EINVAL;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  a.part_rows = attn_part_rows(*cfg, ws_bytes);
  return launch_tree_attn(*cfg, layer, a, k_c, v_c, kept_len, out, so, lse_out, ws, (cudaStream_t)stream);
}

int madakv_tree_commit(const madakv_config* cfg, int32_t layer, int32_t nodes, const uint64_t* mask, const int32_t* n_nodes,
                       const int32_t* node, const void* k_tree, madakv_strides sk, const void* v_tree, madakv_strides sv, void* k_c,
                       void* v_c, const int64_t* seg_off, int32_t* kept_len, int64_t capacity, float* acc, int32_t* kept_idx,
                       const int32_t* position, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  const TreeCall a{nodes, nullptr, sk, k_tree, sk, v_tree, sv, mask, n_nodes, seg_off, capacity, 0};
  if (!node || (kept_idx == nullptr) != (position == nullptr)) return MADAKV_EINVAL;
  if ((rc = check_tree(cfg, layer, a, k_c, v_c, kept_len))) return rc;
  if (((uintptr_t)node & 3) || ((uintptr_t)acc & 3) || ((uintptr_t)kept_idx & 3) || ((uintptr_t)position & 3)) return MADAKV_EALIGN;
  if ((rc = check_ws(*cfg, ws, ws_bytes))) return rc;
  return launch_tree_commit(*cfg, layer, a, node, k_c, v_c, kept_len, acc, kept_idx, position, ws, (cudaStream_t)stream);
}

int madakv_poll_status(void* ws, void* stream, int32_t* status_out) {
  if (!ws || !status_out) return MADAKV_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  if (cudaStreamSynchronize(st) != cudaSuccess) return MADAKV_ECUDA;
  int32_t s = 0;
  if (cudaMemcpyAsync(&s, ws, sizeof(s), cudaMemcpyDeviceToHost, st) != cudaSuccess) return MADAKV_ECUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return MADAKV_ECUDA;
  if (s != 0 && cudaMemsetAsync(ws, 0, sizeof(s), st) != cudaSuccess) return MADAKV_ECUDA;
  *status_out = s;
  return MADAKV_OK;
}

}  // extern "C"
