// Accumulated attention weight (Eq. 7's sum, over the decode steps instead of the proxy tokens):
//   acc[row] = decay * acc[row] + sum over the group's heads of exp2(logit - lse)
// with the logits and log2-sum-exps that the decode kernel before it has left. Bound by the logits it reads, 4 g bytes a row.
#include "common.cuh"

namespace madakv {
namespace {

constexpr int NT = 256;
constexpr int kRows = 1024;  // rows of a block at a time

struct AccumulateParams {
  const int64_t* seg_off;
  const int32_t* kept_len;
  const float* scores;
  const float* lse2;
  float* acc;
  int64_t capacity;
  float decay;
  int L, Hq, Hkv, g, layer, blocks;  // blocks per segment
};

__global__ void __launch_bounds__(NT) accumulate_kernel(const __grid_constant__ AccumulateParams p) {
  pdl_wait();
  pdl_go();
  const int y = blockIdx.x / p.blocks, x = blockIdx.x % p.blocks;
  const int u = p.layer < 0 ? y : (y / p.Hkv * p.L + p.layer) * p.Hkv + y % p.Hkv;
  const int len = p.kept_len[u];
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  if (off < 0 || len < 0 || off + len > end || end > p.capacity) return;  // (as attention sees it: an empty segment)
  const float* lse2 = p.lse2 + (int64_t)(u / p.Hkv) * p.Hq + u % p.Hkv * p.g;
  for (int r = x * NT + threadIdx.x; r < len; r += p.blocks * NT) {
    const float* s = p.scores + (off + r) * p.g;
    float w = 0.f;
    bool lost = false;
    for (int i = 0; i < p.g; ++i) {
      const float z = lse2[i];
      lost |= z != z;
      if (z < INFINITY) w += exp2f(s[i] - z);
    }
    if (!lost) p.acc[off + r] = fmaf(p.decay, p.acc[off + r], w);
  }
}

}  // namespace

int launch_accumulate(const madakv_config& c, int layer, const int64_t* seg_off, const int32_t* kept_len, int64_t capacity,
                      const Tracking& track, void* ws, cudaStream_t st) {
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  const int n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  const int64_t rows = capacity / units < longest ? capacity / units : longest;
  const int64_t want = rows / kRows + 1, most = n_sel < 4096 ? 4096 / n_sel : 1;
  const AccumulateParams p{seg_off, kept_len, track.scores, tracking_lse2(c, ws), track.acc, capacity, track.decay, c.n_layers,
                           c.n_q_heads, c.n_kv_heads, c.n_q_heads / c.n_kv_heads, layer, (int)(want < most ? want : most)};
  launch_pdl(accumulate_kernel, dim3((unsigned)n_sel * p.blocks), dim3(NT), 0, st, p);
  return launch_status();
}

}  // namespace madakv
