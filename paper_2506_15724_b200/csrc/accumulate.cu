// Accumulated attention weight (Eq. 7's sum, over the decode steps instead of the proxy tokens):
//   acc[row] = decay * acc[row] + sum over the group's heads of exp2(logit - lse)
// with the logits and log2-sum-exps that the decode kernel before it has left. Bound by the logits, 4 g bytes a row that are written and
// read (896 segments of 2512 rows, 7 heads: 29 us beside 122 of attention on 4 bits), and on one layer by being a second, dependent
// launch (8 segments of 2952 rows: 2.7 us).
#include "common.cuh"

namespace madakv {
namespace {

constexpr int NT = 256;

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

// G: at least the heads of a group; a thread has ROWS rows' logits on their way at once.
template <int G, int ROWS>
__global__ void __launch_bounds__(NT) accumulate_kernel(const __grid_constant__ AccumulateParams p) {
  pdl_wait();
  pdl_go();
  const int y = blockIdx.x / p.blocks, x = blockIdx.x % p.blocks;
  const int u = p.layer < 0 ? y : (y / p.Hkv * p.L + p.layer) * p.Hkv + y % p.Hkv;
  const int len = p.kept_len[u];
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  const float* lse2 = p.lse2 + (int64_t)(u / p.Hkv) * p.Hq + u % p.Hkv * p.g;
  float z[G];
  bool lost = false;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    z[i] = i < p.g ? lse2[i] : INFINITY;  // +inf: the head adds nothing
    lost |= z[i] != z[i];
  }
  // (as attention sees it: an empty segment; or one whose rows did not arrive)
  if (off < 0 || len < 0 || off + len > end || end > p.capacity || lost) return;
  for (int r0 = x * NT * ROWS + threadIdx.x; r0 < len; r0 += p.blocks * NT * ROWS) {
    float s[ROWS][G], old[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      const int r = r0 + j * NT;
      old[j] = r < len && p.decay > 0.f ? p.acc[off + r] : 0.f;  // (decay 0 forgets whatever was there)
#pragma unroll
      for (int i = 0; i < G; ++i) s[j][i] = r < len && i < p.g ? p.scores[(off + r) * p.g + i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i)
        if (z[i] < INFINITY) w += exp2f(s[j][i] - z[i]);
      if (r0 + j * NT < len) p.acc[off + r0 + j * NT] = fmaf(p.decay, old[j], w);
    }
  }
}

}  // namespace

int launch_accumulate(const madakv_config& c, int layer, const int64_t* seg_off, const int32_t* kept_len, int64_t capacity,
                      const Tracking& track, void* ws, cudaStream_t st) {
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  const int n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  const int64_t rows = capacity / units < longest ? capacity / units : longest;
  const int g = c.n_q_heads / c.n_kv_heads;
  AccumulateParams p{seg_off, kept_len, track.scores, tracking_lse2(c, ws), track.acc, capacity, track.decay, c.n_layers,
                     c.n_q_heads, c.n_kv_heads, g, layer, 1};
  auto go = [&](auto kernel, int rows_each) {
    const int64_t want = rows / (NT * rows_each) + 1, most = n_sel < 8192 ? 8192 / n_sel : 1;
    p.blocks = (int)(want < most ? want : most);
    launch_pdl(kernel, dim3((unsigned)n_sel * p.blocks), dim3(NT), 0, st, p);
    return launch_status();
  };
  if (g == 1) return go(accumulate_kernel<1, 4>, 4);
  if (g == 2) return go(accumulate_kernel<2, 4>, 4);
  if (g <= 4) return go(accumulate_kernel<4, 2>, 2);
  if (g <= 8) return go(accumulate_kernel<8, 2>, 2);
  return go(accumulate_kernel<16, 1>, 1);
}

}  // namespace madakv
