// Stage 4b with a cache in 4 bits: gather the kept K/V rows and quantise them on the way; and the way back for single rows.
//
// A row is shared by D / 4 lanes of a warp, four elements each, in the order of the row's 16-bit words: a warp reads whole rows of
// the source and writes whole rows of codes.
#include <type_traits>

#include "quant.cuh"

namespace madakv {
namespace {

constexpr int NT = 256;

struct CompactQuantParams {
  const char* k;
  const char* v;
  uint8_t* k_code;
  uint8_t* v_code;
  uint32_t* k_par;
  uint32_t* v_par;
  const int32_t* kept_idx;
  const int64_t* seg_off;
  const int32_t* kept_len;
  int64_t capacity;
  int64_t stride_b, stride_l, stride_h, stride_t;  // bytes
  int L, Hkv, n_max, headroom, blocks;             // blocks per unit
};

template <typename T, int D>
__global__ void __launch_bounds__(NT) compact_quant_kernel(const __grid_constant__ CompactQuantParams p) {
  using R = QuantRow<D>;
  constexpr int RPB = NT / R::LANES;  // rows of the block at a time
  pdl_wait();
  pdl_go();
  const int u = blockIdx.x / p.blocks, x = blockIdx.x % p.blocks;
  const int len = p.kept_len[u];
  const int64_t off = p.seg_off[u];
  // a segment that selection refused (MADAKV_ECAPACITY: it would end beyond the cache) has no index list: skip it
  if (off < 0 || off + len + p.headroom > p.capacity) return;
  const int h = u % p.Hkv, l = (u / p.Hkv) % p.L, b = u / (p.Hkv * p.L);
  const int lane = threadIdx.x % R::LANES, sub = threadIdx.x / R::LANES;
  const int G = lane % R::NG, i = lane / R::NG;
  const int64_t src_base = b * p.stride_b + l * p.stride_l + h * p.stride_h + (32 * G + 4 * i) * (int)sizeof(T);
  for (int row0 = x * RPB; row0 < len; row0 += p.blocks * RPB) {  // (all lanes of a warp stay: they exchange extremes)
    const int r = row0 + sub;
    int idx = r < len ? p.kept_idx[off + r] : -1;
    if (idx >= p.n_max) idx = -1;
    float kx[4] = {0.f, 0.f, 0.f, 0.f}, vx[4] = {0.f, 0.f, 0.f, 0.f};
    if (idx >= 0) {
      load4(reinterpret_cast<const T*>(p.k + src_base + (int64_t)idx * p.stride_t), kx);
      load4(reinterpret_cast<const T*>(p.v + src_base + (int64_t)idx * p.stride_t), vx);
    }
    uint32_t kc, kp, vc, vp;
    quantise4<D>(kx, kc, kp);
    quantise4<D>(vx, vc, vp);
    if (idx >= 0) {
      const int64_t dst = off + r;
      reinterpret_cast<uint16_t*>(p.k_code)[dst * (D / 4) + lane] = (uint16_t)kc;
      reinterpret_cast<uint16_t*>(p.v_code)[dst * (D / 4) + lane] = (uint16_t)vc;
      if (i == 0) {
        p.k_par[dst * R::NG + G] = kp;
        p.v_par[dst * R::NG + G] = vp;
      }
    }
  }
}

struct ExpandParams {
  const int64_t* rows;
  const uint8_t* k_code;
  const uint8_t* v_code;
  const uint32_t* k_par;
  const uint32_t* v_par;
  void* k_out;
  void* v_out;
  int64_t n_rows, capacity;
};

__device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&x)[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <typename T, int D>
__global__ void __launch_bounds__(NT) expand_quant_kernel(const __grid_constant__ ExpandParams p) {
  using R = QuantRow<D>;
  constexpr int RPB = NT / R::LANES;
  pdl_wait();
  pdl_go();
  const int lane = threadIdx.x % R::LANES, G = lane % R::NG, i = lane / R::NG;
  for (int64_t r = (int64_t)blockIdx.x * RPB + threadIdx.x / R::LANES; r < p.n_rows; r += (int64_t)gridDim.x * RPB) {
    const int64_t row = p.rows ? p.rows[r] : r;
    float kx[4] = {0.f, 0.f, 0.f, 0.f}, vx[4] = {0.f, 0.f, 0.f, 0.f};
    if (row >= 0 && row < p.capacity) {
      values4(reinterpret_cast<const uint16_t*>(p.k_code)[row * (D / 4) + lane], p.k_par[row * R::NG + G], kx);
      values4(reinterpret_cast<const uint16_t*>(p.v_code)[row * (D / 4) + lane], p.v_par[row * R::NG + G], vx);
    }
    store4(reinterpret_cast<T*>(p.k_out) + r * D + 32 * G + 4 * i, kx);
    store4(reinterpret_cast<T*>(p.v_out) + r * D + 32 * G + 4 * i, vx);
  }
}

// f(T(), D) for the config's type and head_dim.
template <typename F>
int for_type(const madakv_config& c, F f) {
  if (c.dtype == MADAKV_F32)
    c.head_dim == 64 ? f(float(), std::integral_constant<int, 64>()) : f(float(), std::integral_constant<int, 128>());
  else
    c.head_dim == 64 ? f(__nv_bfloat16(), std::integral_constant<int, 64>()) : f(__nv_bfloat16(), std::integral_constant<int, 128>());
  return launch_status();
}

}  // namespace

int launch_compact_quant(const madakv_config& c, const void* k, const void* v, madakv_strides s, const int32_t* kept_idx,
                         const int64_t* seg_off, const int32_t* kept_len, uint8_t* k_code, void* k_par, uint8_t* v_code,
                         void* v_par, int64_t capacity, cudaStream_t st) {
  const int e = elem_bytes(c);
  CompactQuantParams p;
  p.k = (const char*)k;
  p.v = (const char*)v;
  p.k_code = k_code;
  p.v_code = v_code;
  p.k_par = (uint32_t*)k_par;
  p.v_par = (uint32_t*)v_par;
  p.kept_idx = kept_idx;
  p.seg_off = seg_off;
  p.kept_len = kept_len;
  p.capacity = capacity;
  p.stride_b = s.batch * e;
  p.stride_l = s.layer * e;
  p.stride_h = s.head * e;
  p.stride_t = s.token * e;
  p.L = c.n_layers;
  p.Hkv = c.n_kv_heads;
  p.n_max = c.max_seq_len;
  p.headroom = c.max_new_tokens;
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, rows = capacity / units + 1;
  const int64_t per_block = 32, want = (rows + per_block - 1) / per_block, most = ((1 << 20) + units - 1) / units;
  p.blocks = (int)(want < most ? want : most);
  if (units * p.blocks > 0x7fffffff) return MADAKV_EUNSUPPORTED;
  return for_type(c, [&](auto t, auto d) {
    launch_pdl(compact_quant_kernel<decltype(t), decltype(d)::value>, dim3((unsigned)(units * p.blocks)), dim3(NT), 0, st, p);
  });
}

int launch_expand_quant(const madakv_config& c, const int64_t* rows, int64_t n_rows, const uint8_t* k_code, const void* k_par,
                        const uint8_t* v_code, const void* v_par, int64_t capacity, void* k_out, void* v_out, cudaStream_t st) {
  const ExpandParams p{rows, k_code, v_code, (const uint32_t*)k_par, (const uint32_t*)v_par, k_out, v_out, n_rows, capacity};
  const int64_t rpb = NT / (c.head_dim / 4), want = (n_rows + rpb - 1) / rpb;
  const unsigned grid = (unsigned)(want < (1 << 20) ? want : (1 << 20));
  return for_type(c, [&](auto t, auto d) {
    launch_pdl(expand_quant_kernel<decltype(t), decltype(d)::value>, dim3(grid), dim3(NT), 0, st, p);
  });
}

}  // namespace madakv
