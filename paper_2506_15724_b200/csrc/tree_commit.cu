// The accepted path of a drafted tree appended to every head's segment: the rows of the nodes that the accepted node's mask names, in
// ascending order, go behind the segment's last row. A block has one segment. Nothing is computed; a call on one layer is bound by the
// chain of its loads (accepted node, its mask, the rows).
#include "common.cuh"

namespace madakv {
namespace {

constexpr int NT = 256, kNodes = 64;

struct CommitParams {
  const char *k_tree, *v_tree;
  madakv_strides sk, sv;  // in bytes
  const uint64_t* mask;
  const int32_t *n_nodes, *node, *position;
  char *k_c, *v_c;
  const int64_t* seg_off;
  int32_t *kept_len, *kept_idx;
  float* acc;
  void* ws;
  int64_t capacity;
  int L, Hkv, layer, T, row_bytes;
};

__global__ void __launch_bounds__(NT) tree_commit_kernel(const __grid_constant__ CommitParams p) {
  __shared__ int path[kNodes];
  pdl_wait();
  pdl_go();
  const int y = blockIdx.x, u = p.layer < 0 ? y : (y / p.Hkv * p.L + p.layer) * p.Hkv + y % p.Hkv;
  const int b = u / p.Hkv / p.L, l = u / p.Hkv % p.L, h = u % p.Hkv;
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  const int len = p.kept_len[u], node = p.node[b];
  const int nodes = p.n_nodes ? max(0, min(p.n_nodes[b], p.T)) : p.T;
  const int first = p.position ? p.position[b] : 0;
  if (node < 0) return;  // nothing accepted
  if (node >= nodes) {
    if (threadIdx.x == 0) set_status(p.ws, MADAKV_ESHAPE);
    return;
  }
  const uint64_t bits = p.mask[(int64_t)b * p.T + node] & (nodes >= 64 ? ~0ull : (1ull << nodes) - 1);
  const int rows = __popcll(bits);
  // a segment that selection refused, or without room for all of the path, is left as it is
  if (off < 0 || end < off || end > p.capacity || len < 0 || off + (int64_t)len + rows > end) {
    if (threadIdx.x == 0) set_status(p.ws, MADAKV_ECAPACITY);
    return;
  }
  const int t = threadIdx.x;
  if (t < kNodes && bits >> t & 1) path[__popcll(bits & ((1ull << t) - 1))] = t;
  __syncthreads();  // (also: all have read the length)
  const int64_t row = off + len;
  if (t == 0) p.kept_len[u] = len + rows;
  if (t < rows) {
    if (p.acc) p.acc[row + t] = 0.f;
    if (p.kept_idx) p.kept_idx[row + t] = first + t;
  }
  const char* k = p.k_tree + b * p.sk.batch + l * p.sk.layer + h * p.sk.head;
  const char* v = p.v_tree + b * p.sv.batch + l * p.sv.layer + h * p.sv.head;
  const int pieces = p.row_bytes / 16;
  for (int x = t; x < rows * pieces; x += NT) {
    const int i = x / pieces, c = x % pieces * 16, n = path[i];
    const uint4 kk = *reinterpret_cast<const uint4*>(k + n * p.sk.token + c);
    const uint4 vv = *reinterpret_cast<const uint4*>(v + n * p.sv.token + c);
    *reinterpret_cast<uint4*>(p.k_c + (row + i) * p.row_bytes + c) = kk;
    *reinterpret_cast<uint4*>(p.v_c + (row + i) * p.row_bytes + c) = vv;
  }
}

}  // namespace

int launch_tree_commit(const madakv_config& c, int layer, const TreeCall& a, const int32_t* node, void* k_c, void* v_c,
                       int32_t* kept_len, float* acc, int32_t* kept_idx, const int32_t* position, void* ws, cudaStream_t st) {
  const int64_t e = elem_bytes(c);
  auto in_bytes = [&](madakv_strides s) { return madakv_strides{s.batch * e, s.layer * e, s.head * e, s.token * e}; };
  CommitParams p{(const char*)a.k_tree, (const char*)a.v_tree, in_bytes(a.sk), in_bytes(a.sv), a.mask, a.n_nodes, node, position,
                 (char*)k_c, (char*)v_c, a.seg_off, kept_len, kept_idx, acc, ws, a.capacity, c.n_layers, c.n_kv_heads, layer, a.nodes,
                 (int)(c.head_dim * e)};
  const int n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  launch_pdl(tree_commit_kernel, dim3((unsigned)n_sel), dim3(NT), 0, st, p);
  return launch_status();
}

}  // namespace madakv
