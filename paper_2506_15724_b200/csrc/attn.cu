// Host side of prompt attention and attention of drafted trees: the parameters of a call and the kernel that takes it.
#include "attn_common.cuh"

namespace madakv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

AttnParams base_params(const madakv_config& c, int layer, void* ws, int part_rows) {
  AttnParams p = {};
  p.B = c.batch;
  p.L = c.n_layers;
  p.Hq = c.n_q_heads;
  p.Hkv = c.n_kv_heads;
  p.g = c.n_q_heads / c.n_kv_heads;
  p.g_inverse = (65536 + p.g - 1) / p.g;
  p.layer = layer;
  p.causal = c.causal;
  p.w = c.window;
  p.n_max = c.max_seq_len;
  p.scale2 = scale_of(c) * kLog2e;
  p.ws = ws;
  p.part_rows = part_rows;
  return p;
}
int launch(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st) {
  if (c.dtype == MADAKV_F32) return launch_attn_split(p, c, tree, st);
  const int rc = launch_attn_tc(p, c, tree, st);
  return rc >= 0 ? rc : launch_attn_plain(p, c, tree, st);
}

}  // namespace

int launch_prefill_attn(const madakv_config& c, int layer, const PromptCall& a, void* ws, cudaStream_t st) {
  AttnParams p = base_params(c, layer, ws, a.part_rows);
  if (p.g > kMaxGroup) return MADAKV_EUNSUPPORTED;
  const int64_t e = elem_bytes(c);
  auto at = [&](const void* x, const madakv_strides& s) { return (void*)((char*)x + layer * s.layer * e); };
  p.q = at(a.q, a.sq);
  p.sq = a.sq;
  p.q_rows = a.q_rows;
  p.q_off = a.q_off;
  p.q_len = a.q_len;
  p.k = at(a.k, a.sk);
  p.sk = a.sk;
  p.v = at(a.v, a.sv);
  p.sv = a.sv;
  p.k_rows = a.k_rows;
  p.k_off = a.k_off;
  p.seq_len = a.seq_len;
  p.out = at(a.out, a.so);
  p.so = a.so;
  p.lse_out = a.lse_out;
  p.q_win = a.q_win;
  p.lse_win = a.lse_win;
  p.win_len = a.win_len;
  // (calls that hold every key's query leave no earlier row in a window)
  const bool whole = p.q_off ? p.q_off == p.k_off && p.q_rows >= p.k_rows : !p.q_len && (p.q_rows >= p.k_rows || p.q_rows >= p.n_max);
  if (p.win_len && !whole)
    if (const int rc = launch_window_move(p, c, st)) return rc;
  return launch(p, c, false, st);
}

int launch_tree_attn(const madakv_config& c, int layer, const TreeCall& a, const void* k_c, const void* v_c, const int32_t* kept_len,
                     void* out, madakv_strides so, float* lse_out, void* ws, cudaStream_t st) {
  AttnParams p = base_params(c, layer, ws, a.part_rows);
  if (p.g > kMaxGroup) return MADAKV_EUNSUPPORTED;
  p.q = a.q;
  p.sq = a.sq;
  p.q_rows = a.nodes;
  p.k = a.k_tree;
  p.sk = a.sk;
  p.v = a.v_tree;
  p.sv = a.sv;
  p.k_c = k_c;
  p.v_c = v_c;
  p.seg_off = a.seg_off;
  p.kept_len = kept_len;
  p.capacity = a.capacity;
  p.mask = a.mask;
  p.n_nodes = a.n_nodes;
  p.n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  p.out = out;
  p.so = so;
  p.lse_out = lse_out;
  return launch(p, c, true, st);
}

}  // namespace madakv
