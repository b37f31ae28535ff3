// Attention of a prompt and of drafted trees with scalar fp32 arithmetic on bf16 rows, for strides that tensor copies cannot take (a
// dimension of stride 0, layers and sequences that do not lie evenly):
//   out = sum_i p_i v_i / sum_i p_i,  p_i = exp2(scale * log2(e) * q . k_i - m),  lse = (m + log2(sum_i p_i)) ln 2
// with m the running maximum of the row's logits; sums and maxima are kept in fp32 and corrected when m grows, so one pass over
// the keys is enough. A block has 64 rows and goes through its keys 64 at a time.
#include <type_traits>

#include "attn_common.cuh"

namespace madakv {
namespace {

constexpr int M = 64, N = 64, NT = 256;

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 halves(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}

// Four elements of a row as fp32, or zeros.
using T = __nv_bfloat16;
__device__ __forceinline__ float4 load4(const T* src, bool there) {
  if (!there) return make_float4(0.f, 0.f, 0.f, 0.f);
  const uint2 x = *reinterpret_cast<const uint2*>(src);
  return make_float4(bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y));
}
__device__ __forceinline__ void store4(T* dst, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <int D>
struct Smem {
  static constexpr int PITCH = D + 4, PPITCH = N + 4;  // (rows 16 bytes further: the 16-byte loads of 8 lanes meet all banks)
  float q[M * PITCH];
  union {
    float k[N * PITCH];
    float p[M * PPITCH];
  };
  float v[N * PITCH];
  AttnItem item;
  int there;
};

template <int D, bool kTree>
__global__ void __launch_bounds__(NT, 2) attn_plain_kernel(const __grid_constant__ AttnParams p) {
  extern __shared__ __align__(16) unsigned char raw[];
  using S = Smem<D>;
  S& sm = *reinterpret_cast<S*>(raw);
  constexpr int C4 = D / 4, CO = D / 64;  // float4 pieces of a row; float4 columns of a thread's results
  pdl_wait();
  pdl_go();
  const unsigned y = blockIdx.x / p.slots;
  const int slot = blockIdx.x % p.slots;
  if constexpr (!kTree) fill_window<D * (int)sizeof(T)>(p, threadIdx.x, NT);
  if (threadIdx.x < 32) {
    AttnItem it;
    const bool there = kTree ? tree_item(p, y, it) : prompt_item(p, y, it);
    if (threadIdx.x == 0) {
      sm.item = it;
      sm.there = there;
    }
  }
  __syncthreads();
  if (!sm.there) return;
  const AttnItem& it = sm.item;
  const int rows = min(p.tile_q, it.n_q - it.q0) * p.g;  // rows of the tile that are queries
  if (rows <= 0) return;
  // keys that any row sees, in tiles; a tree's own nodes are a tile behind the segment's
  const int tiles = item_tiles<kTree>(p, it), main_tiles = tiles - (kTree ? 1 : 0), nb = shares_of(p, tiles);
  if (slot >= nb) return;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;

  float m[4], l[4];
  float4 o[4][CO];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < CO; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  {
    const T* q = reinterpret_cast<const T*>(p.q) + it.q_at;
    for (int x = tid; x < M * C4; x += NT) {
      const int r = x / C4, c = x % C4 * 4;
      const bool there = r < rows;
      *reinterpret_cast<float4*>(sm.q + r * S::PITCH + c) =
          load4(q + (there ? (int64_t)(it.q0 + group_of(p, r)) * p.sq.token + (r - group_of(p, r) * p.g) * p.sq.head + c : 0), there);
    }
    int visible[4];  // keys that the thread's rows see
    uint64_t nodes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = ty * 4 + i, t = it.q0 + group_of(p, r);
      visible[i] = r >= rows ? 0 : (kTree || !p.causal ? it.n_keys : max(0, min(it.n_keys, t + it.shift + 1)));
      nodes[i] = kTree && r < rows ? node_mask(p, it, t) : 0;
    }
    int begin, end;
    share_tiles(nb, tiles, slot, begin, end);
    for (int tile = begin; tile < end; ++tile) {
      const bool own = kTree && tile == main_tiles;  // the tree's nodes
      const int first = own ? 0 : tile * N, there = own ? it.nodes : it.n_keys - first;
      const T *k, *v;
      int64_t sk, sv;
      if (kTree && !own) {
        k = reinterpret_cast<const T*>(p.k_c) + (it.key_row + first) * D;
        v = reinterpret_cast<const T*>(p.v_c) + (it.key_row + first) * D;
        sk = sv = D;
      } else {
        sk = p.sk.token;
        sv = p.sv.token;
        k = reinterpret_cast<const T*>(p.k) + it.k_at + first * sk;
        v = reinterpret_cast<const T*>(p.v) + it.v_at + first * sv;
      }
      __syncthreads();  // (the tile before is done with)
      for (int x = tid; x < N * C4; x += NT) {
        const int r = x / C4, c = x % C4 * 4;
        const bool in = r < there;
        *reinterpret_cast<float4*>(sm.k + r * S::PITCH + c) = load4(k + (in ? r * sk + c : 0), in);
        *reinterpret_cast<float4*>(sm.v + r * S::PITCH + c) = load4(v + (in ? r * sv + c : 0), in);
      }
      __syncthreads();
      // logits of rows 4 ty + i, keys tx + 16 j: sums over even and odd elements apart
      uint64_t acc[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0;
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(sm.q + (ty * 4 + i) * S::PITCH + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(sm.k + (tx + 16 * j) * S::PITCH + c);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[i][j] = fma2(pair(a[i].x, a[i].y), pair(b[j].x, b[j].y), acc[i][j]);
            acc[i][j] = fma2(pair(a[i].z, a[i].w), pair(b[j].z, b[j].w), acc[i][j]);
          }
      }
      float s[4][4], f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float top = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = tx + 16 * j;
          const bool see = own ? nodes[i] >> key & 1 : first + key < visible[i];
          const float2 h = halves(acc[i][j]);
          s[i][j] = see ? (h.x + h.y) * p.scale2 : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int x = 8; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float base = top == -INFINITY ? 0.f : top;
        f[i] = exp2f(m[i] - base);
        m[i] = top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += s[i][j] = exp2f(s[i][j] - base);
        l[i] = l[i] * f[i] + sum;  // (of this thread's keys)
#pragma unroll
        for (int c = 0; c < CO; ++c) o[i][c].x *= f[i], o[i][c].y *= f[i], o[i][c].z *= f[i], o[i][c].w *= f[i];
      }
      __syncthreads();  // (all are done with the keys, in whose place the weights go)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sm.p[(ty * 4 + i) * S::PPITCH + tx + 16 * j] = s[i][j];
      __syncwarp();  // (a warp reads the weights of its own rows only)
#pragma unroll 2
      for (int x = 0; x < N; x += 4) {
        float4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(sm.p + (ty * 4 + i) * S::PPITCH + x);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < CO; ++c) {
            const float4 b = *reinterpret_cast<const float4*>(sm.v + (x + e) * S::PITCH + tx * 4 + 64 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float z = e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w;
              o[i][c].x = fmaf(z, b.x, o[i][c].x), o[i][c].y = fmaf(z, b.y, o[i][c].y);
              o[i][c].z = fmaf(z, b.z, o[i][c].z), o[i][c].w = fmaf(z, b.w, o[i][c].w);
            }
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 8; x >= 1; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
  }
  auto finish_row = [&](int r, float mm, float ll) {  // log-sum-exp and proxy query of a row, by 16 threads
    const int t = it.q0 + group_of(p, r), j = r - group_of(p, r) * p.g;
    int64_t win = 0;
    bool copy = false;
    if (tx == 0) copy = store_row_lse(p, it, t, j, row_lse(mm, ll), win);
    const unsigned half = 0xffffu << (tid & 16);
    copy = __shfl_sync(half, copy, tid & 16);
    win = __shfl_sync(half, win, tid & 16);
    if (!copy) return;
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.q) + it.q_at + t * p.sq.token + j * p.sq.head);
    uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.q_win) + win * D);
    for (int x = tx; x < D * (int)sizeof(T) / 16; x += 16) dst[x] = src[x];
  };
  T* out = reinterpret_cast<T*>(p.out) + it.out_at;
  if (nb == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = ty * 4 + i;
      if (r >= rows) continue;
      const float z = row_factor(l[i]);
      T* dst = out + (int64_t)(it.q0 + group_of(p, r)) * p.so.token + (r - group_of(p, r) * p.g) * p.so.head;
#pragma unroll
      for (int c = 0; c < CO; ++c)
        store4(dst + tx * 4 + 64 * c, make_float4(o[i][c].x * z, o[i][c].y * z, o[i][c].z * z, o[i][c].w * z));
      finish_row(r, m[i], l[i]);
    }
    return;
  }
  auto part_row = [&](int x, int r) { return ((int64_t)y * p.slots + x) * p.tile_rows + r; };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i;
    if (r >= rows) continue;
    const int64_t at = part_row(slot, r);
#pragma unroll
    for (int c = 0; c < CO; ++c) *reinterpret_cast<float4*>(p.part + at * D + tx * 4 + 64 * c) = o[i][c];
    if (tx == 0) p.part_ml[at] = make_float2(m[i], l[i]);
  }
}

template <int D, bool kTree>
int run(AttnParams p, const madakv_config& c, cudaStream_t st) {
  p.tile_q = M / p.g;
  attn_items(p, kTree);
  if (p.n_items == 0) p.n_items = 1;  // (the window's missing rows are still filled)
  attn_slots(p, c, kTree, N, {15.f, 15.f, 10.f, 2});
  auto kernel = attn_plain_kernel<D, kTree>;
  if (p.n_items * p.slots > 0x7fffffffll) return MADAKV_EUNSUPPORTED;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>)) != cudaSuccess) return MADAKV_ECUDA;
  launch_pdl(kernel, dim3((unsigned)(p.n_items * p.slots)), dim3(NT), sizeof(Smem<D>), st, p);
  const int rc = launch_status();
  return rc || p.slots == 1 ? rc : launch_attn_join(p, c, kTree, st);
}

}  // namespace

int launch_attn_plain(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st) {
  if (c.head_dim == 64) return tree ? run<64, true>(p, c, st) : run<64, false>(p, c, st);
  return tree ? run<128, true>(p, c, st) : run<128, false>(p, c, st);
}

}  // namespace madakv
