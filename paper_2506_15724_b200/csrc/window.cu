// The proxy tokens' queries and log-sum-exps from one chunk of a prompt to the next. A chunk of m queries brings the window's last m rows; where m is
// less than the window the rows before them are those that the chunks before have left, m places further up. A launch ahead of the attention moves
// them, a block to a head, in place: pieces go up in ascending order, those of a turn of the block are all read before any of them is
// written, and what later turns read lies behind what earlier ones wrote. Bound by the chain length, row, row's new place: 2.8 us for 28 heads of
// 128 and 22 rows to move, 6.7 for 8 sequences and 12 rows. And the check that windows are those of the prompt that is scored.
#include "attn_common.cuh"

namespace madakv {
namespace {

constexpr int NT = 256;

template <int ROW_BYTES>
__global__ void __launch_bounds__(NT) window_move_kernel(const __grid_constant__ AttnParams p) {
  constexpr int P = ROW_BYTES / 16;  // 16-byte pieces of a row
  pdl_wait();
  pdl_go();
  const int b = blockIdx.x / p.Hq, keys = prompt_keys(p, b), m = prompt_queries(p, b, keys);
  if (m == 0 || m >= min(p.w, keys)) return;  // (nothing new; or all rows are the call's own)
  const bool kept = p.causal && p.win_len[b * p.L + p.layer] == keys - m;
  const int rows = p.w - m;
  const int64_t first = (((int64_t)b * p.L + p.layer) * p.Hq + blockIdx.x % p.Hq) * p.w;
  float* lse = p.lse_win + first;
  uint4* q = reinterpret_cast<uint4*>((char*)p.q_win + first * ROW_BYTES);
  for (int x0 = 0; x0 < rows * P; x0 += NT) {
    const int x = x0 + threadIdx.x;
    const bool in = x < rows * P;
    const uint4 piece = in && kept ? q[x + m * P] : make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (in) q[x] = piece;
  }
  for (int r0 = 0; r0 < rows; r0 += NT) {
    const int r = r0 + threadIdx.x;
    const float y = r < rows && kept ? lse[r + m] : -INFINITY;
    __syncthreads();
    if (r < rows) lse[r] = y;
  }
}

// Windows that an eviction goes on from: of a sequence of n keys all layers' have to be complete for n keys and either all new or all those that an
// eviction has gone on from before (its repetition): a layer that a new prompt has not reached still has the last one's. A warp to a sequence.
__global__ void __launch_bounds__(NT) window_check_kernel(const int32_t* seq_len, int32_t* win_len, int B, int L, int n_max, void* ws) {
  pdl_wait();
  pdl_go();
  const int b = blockIdx.x * (NT / 32) + threadIdx.x / 32, lane = threadIdx.x % 32;
  if (b >= B) return;
  const int n = clamped_len(seq_len, b, n_max);
  bool fresh = false, used = false, other = false;
  for (int l = lane; l < L; l += 32) {
    const int held = win_len[b * L + l];
    fresh |= held == n;
    used |= held == ~n;
    other |= held != n && held != ~n;
  }
  fresh = __any_sync(0xffffffffu, fresh);
  used = __any_sync(0xffffffffu, used);
  if (n > 0 && (__any_sync(0xffffffffu, other) || (fresh && used))) {
    if (lane == 0) set_status(ws, MADAKV_ESHAPE);
    return;
  }
  for (int l = lane; l < L; l += 32) win_len[b * L + l] = ~n;
}

}  // namespace

int launch_window_check(const madakv_config& c, const int32_t* seq_len, int32_t* win_len, void* ws, cudaStream_t st) {
  launch_pdl(window_check_kernel, dim3((unsigned)((c.batch + NT / 32 - 1) / (NT / 32))), dim3(NT), 0, st, seq_len, win_len, c.batch, c.n_layers, c.max_seq_len, ws);
  return launch_status();
}

int launch_window_move(const AttnParams& p, const madakv_config& c, cudaStream_t st) {
  const int64_t blocks = (int64_t)p.B * p.Hq;
  if (blocks > 0x7fffffffll) return MADAKV_EUNSUPPORTED;
  auto kernel = c.head_dim * elem_bytes(c) == 128 ? window_move_kernel<128> : c.head_dim * elem_bytes(c) == 256 ? window_move_kernel<256> : window_move_kernel<512>;
  launch_pdl(kernel, dim3((unsigned)blocks), dim3(NT), 0, st, p);
  return launch_status();
}

}  // namespace madakv
