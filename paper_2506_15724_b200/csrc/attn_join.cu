// Shares of the keys joined: a row's result is the sum of its shares' results, each brought to the largest of their maxima, over the sum of
// their weights, in the order of the shares. A launch of its own, a warp to a row, so that all of the GPU takes part. (The block of an item
// that was done last, on its own: 17300 clocks for 112 rows of 4 shares, 30 us and more for 256 rows of 8.)
#include <type_traits>

#include "attn_common.cuh"

namespace madakv {
namespace {

constexpr int NT = 256, kRowsOfBlock = NT / 32;

template <typename T, int D, bool kTree>
__global__ void __launch_bounds__(NT) attn_join_kernel(const __grid_constant__ AttnParams p) {
  constexpr int V = D / 32, N = 8;  // columns of a lane; shares on their way at once
  using Piece = std::conditional_t<V == 4, float4, float2>;
  __shared__ AttnItem s_item;
  __shared__ int s_there;
  pdl_wait();
  pdl_go();
  const int per = (p.tile_rows + kRowsOfBlock - 1) / kRowsOfBlock, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const unsigned y = blockIdx.x / per;
  const int r = (int)(blockIdx.x % per) * kRowsOfBlock + warp;
  // (results are on their way before it is known how many of the places hold some: what the others hold is not used)
  const int64_t first = (int64_t)y * p.slots * p.tile_rows + r;
  const Piece* part = reinterpret_cast<const Piece*>(p.part + first * D) + lane;
  const bool row_there = r < p.tile_rows;
  float2 ml = row_there && lane < p.slots ? __ldcg(p.part_ml + first + lane * p.tile_rows) : make_float2(-INFINITY, 0.f);
  Piece v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = row_there && i < p.slots ? __ldcg(part + (int64_t)i * p.tile_rows * 32) : Piece();
  if (warp == 0) {
    AttnItem it;
    const bool there = kTree ? tree_item(p, y, it) : prompt_item(p, y, it);
    if (lane == 0) s_item = it, s_there = there;
  }
  __syncthreads();
  if (!s_there) return;
  const AttnItem& it = s_item;
  const int nb = shares_of(p, item_tiles<kTree>(p, it));
  if (nb == 1 || r >= min(p.tile_q, it.n_q - it.q0) * p.g) return;  // (one share: its block has written the result)
  if (lane >= nb) ml = make_float2(-INFINITY, 0.f);
  float acc[V] = {}, top = ml.x;
#pragma unroll
  for (int i = 16; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
  const float fac = exp2f(ml.x - (top == -INFINITY ? 0.f : top));
  float sum = ml.y * fac;
#pragma unroll
  for (int i = 16; i >= 1; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
  for (int i0 = 0; i0 < nb; i0 += N) {
    if (i0 > 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = i0 + i < nb ? __ldcg(part + (int64_t)(i0 + i) * p.tile_rows * 32) : Piece();
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i0 + i >= nb) break;
      const float f = __shfl_sync(0xffffffffu, fac, i0 + i);  // (0 beyond the last share)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += reinterpret_cast<const float*>(&v[i])[e] * f;
    }
  }
  const int t = it.q0 + group_of(p, r), j = r - group_of(p, r) * p.g;
  const float z = row_factor(sum);
  T* to = reinterpret_cast<T*>(p.out) + it.out_at + t * p.so.token + j * p.so.head + lane * V;
#pragma unroll
  for (int e = 0; e < V; e += 2) {
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<__nv_bfloat162*>(to + e) = __floats2bfloat162_rn(acc[e] * z, acc[e + 1] * z);
    else
      *reinterpret_cast<float2*>(to + e) = make_float2(acc[e] * z, acc[e + 1] * z);
  }
  int64_t win = 0;
  const bool proxy = lane == 0 && store_row_lse(p, it, t, j, row_lse(top, sum), win);
  if (!__any_sync(0xffffffffu, proxy)) return;
  win = __shfl_sync(0xffffffffu, win, 0);
  const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.q) + it.q_at + t * p.sq.token + j * p.sq.head);
  uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.q_win) + win * D);
  if (lane < D * (int)sizeof(T) / 16) dst[lane] = src[lane];
}

}  // namespace

int launch_attn_join(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st) {
  const int64_t blocks = p.n_items * ((p.tile_rows + kRowsOfBlock - 1) / kRowsOfBlock);
  auto go = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    if (tree)
      launch_pdl(attn_join_kernel<T, D, true>, dim3((unsigned)blocks), dim3(NT), 0, st, p);
    else
      launch_pdl(attn_join_kernel<T, D, false>, dim3((unsigned)blocks), dim3(NT), 0, st, p);
    return launch_status();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (c.dtype == MADAKV_F32) return c.head_dim == 64 ? go(float(), D64()) : go(float(), D128());
  return c.head_dim == 64 ? go(__nv_bfloat16(), D64()) : go(__nv_bfloat16(), D128());
}

}  // namespace madakv
