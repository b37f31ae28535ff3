// Stage 5 on a cache in 4 bits: cache append (Eq. 4, the row quantised on the way) and decode attention (Eq. 5).
//
// The rows of a segment are shared out over blocks as in decode.cu. A row is shared by D / 4 lanes, four elements each, which turn
// its codes into values; the g query heads of the KV group share every row read; online softmax in the log2 domain, fp32 accumulation.
#include <type_traits>

#include "decode_common.cuh"
#include "quant.cuh"

namespace madakv {
namespace {

constexpr int NT = 128;

template <typename T, int D, int G, bool kTrack>
__global__ void __launch_bounds__(NT) decode_quant_kernel(const __grid_constant__ DecodeParams p) {
  using R = QuantRow<D>;
  constexpr int LANES = R::LANES, GROUPS = NT / LANES, U = 4;
  __shared__ __align__(16) float s_o[GROUPS * G * D];
  __shared__ float s_m[GROUPS * G], s_l[GROUPS * G];
  __shared__ __align__(16) float b_o[G * D];
  __shared__ float b_m[G], b_l[G], fac[G * kDecodeSlots];
  pdl_wait();
  pdl_go();
  const int y = blockIdx.x / p.slots, slot = blockIdx.x % p.slots;
  const int u = unit_of(p, y);
  const SegView view = segment_view(p, u, slot == 0 && threadIdx.x == 0);
  const int len = view.len, nb = segment_blocks(p, len);
  int row_begin, row_end;
  block_rows(nb, len, slot, row_begin, row_end);  // (empty beyond the nb-th block)
  const int h = u % p.Hkv, bl = u / p.Hkv;
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES, gi = lane % R::NG;
  const int first = 32 * gi + 4 * (lane / R::NG);  // the lane's elements
  if (slot < nb) {
    const int64_t off = p.seg_off[u];
    uint16_t *kc = reinterpret_cast<uint16_t*>(p.k_c) + off * (D / 4) + lane, *vc = reinterpret_cast<uint16_t*>(p.v_c) + off * (D / 4) + lane;
    uint32_t *kp = reinterpret_cast<uint32_t*>(p.k_par) + off * R::NG + gi, *vp = reinterpret_cast<uint32_t*>(p.v_par) + off * R::NG + gi;
    if (view.new_row >= row_begin && view.new_row < row_end) {
      if (threadIdx.x < 32) {
        float x[4];
        uint32_t codes, par;
        load4(reinterpret_cast<const T*>(p.k_new) + (int64_t)u * D + first, x);
        quantise4<D>(x, codes, par);
        if (grp == 0) {
          kc[(int64_t)view.new_row * (D / 4)] = (uint16_t)codes;
          if (lane < R::NG) kp[(int64_t)view.new_row * R::NG] = par;
        }
        load4(reinterpret_cast<const T*>(p.v_new) + (int64_t)u * D + first, x);
        quantise4<D>(x, codes, par);
        if (grp == 0) {
          vc[(int64_t)view.new_row * (D / 4)] = (uint16_t)codes;
          if (lane < R::NG) vp[(int64_t)view.new_row * R::NG] = par;
        }
      }
      __syncthreads();
    }
    float qr[G][4], m[G], l[G], o[G][4];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) qr[i][c] = o[i][c] = 0.f;
      if (i < p.g) load4(reinterpret_cast<const T*>(p.q) + ((int64_t)bl * p.Hq + h * p.g + i) * D + first, qr[i]);
#pragma unroll
      for (int c = 0; c < 4; ++c) qr[i][c] *= p.scale2;
    }
    for (int r0 = row_begin; r0 < row_end; r0 += GROUPS * U) {
      float sc[G][U], vf[U][4];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int64_t r = min(r0 + GROUPS * j + grp, row_end - 1);
        float kf[4];
        values4(kc[r * (D / 4)], kp[r * R::NG], kf);
        values4(vc[r * (D / 4)], vp[r * R::NG], vf[j]);
#pragma unroll
        for (int i = 0; i < G; ++i) sc[i][j] = qr[i][0] * kf[0] + qr[i][1] * kf[1] + qr[i][2] * kf[2] + qr[i][3] * kf[3];
      }
#pragma unroll
      for (int sh = LANES / 2; sh >= 1; sh >>= 1)
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int j = 0; j < U; ++j) sc[i][j] += __shfl_xor_sync(0xffffffffu, sc[i][j], sh);
#pragma unroll
      for (int i = 0; i < G; ++i) {
        float mn = m[i];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int r = r0 + GROUPS * j + grp;
          if (kTrack && lane == i && i < p.g && r < row_end) p.scores[(off + r) * p.g + i] = sc[i][j];
          if (r >= row_end) sc[i][j] = -INFINITY;
          mn = fmaxf(mn, sc[i][j]);
        }
        const float base = mn == -INFINITY ? 0.f : mn;
        const float f = fast_ex2(m[i] - base);
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][c] *= f;
        m[i] = mn;
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const float w = fast_ex2(sc[i][j] - base);
          l[i] += w;
          if (r0 + GROUPS * j + grp < row_end) {  // (the row read in its place may hold anything)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[i][c] = fmaf(w, vf[j][c], o[i][c]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < G; ++i) {
      if (lane == 0) {
        s_m[grp * G + i] = m[i];
        s_l[grp * G + i] = l[i];
      }
      *reinterpret_cast<float4*>(s_o + (grp * G + i) * D + first) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
    }
    __syncthreads();
    for (int x = threadIdx.x; x < p.g * D; x += NT) {
      const int i = x / D, c = x % D;
      float M = -INFINITY, Lsum = 0.f, O = 0.f;
#pragma unroll
      for (int gq = 0; gq < GROUPS; ++gq) M = fmaxf(M, s_m[gq * G + i]);
#pragma unroll
      for (int gq = 0; gq < GROUPS; ++gq) {
        const float f = part_weight(s_m[gq * G + i], M);
        Lsum += s_l[gq * G + i] * f;
        O += s_o[(gq * G + i) * D + c] * f;
      }
      b_o[i * D + c] = O;
      if (c == 0) {
        b_m[i] = M;
        b_l[i] = Lsum;
      }
    }
    __syncthreads();
  }
  finish_segment<T, D, NT, true>(p, b_o, b_m, b_l, fac, u, y, slot, nb, view);
}

template <typename T, int D>
int run(DecodeParams p, const madakv_config& c, int splits, cudaStream_t st) {
  if (p.g > (sizeof(T) == 2 ? 16 : 8)) return MADAKV_EUNSUPPORTED;
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  const int64_t rows = p.capacity / units < longest ? p.capacity / units : longest;
  const int64_t want = 3 * rows / 512 + 1, most = 888 / p.n_sel < 1 ? 1 : 888 / p.n_sel < kDecodeSlots ? 888 / p.n_sel : kDecodeSlots;
  p.slots = (int)(want < most ? want : most);
  if (p.slots > splits) p.slots = splits;
  if (p.n_sel > kCounters) p.slots = 1;
  p.min_rows = 256;
  p.part_ml = reinterpret_cast<float2*>(p.part + (int64_t)c.batch * c.n_layers * c.n_q_heads * p.slots * D);
  auto go = [&](auto heads) {
    constexpr int G = decltype(heads)::value;
    const dim3 grid((unsigned)p.n_sel * p.slots);
    if (p.scores)
      launch_pdl(decode_quant_kernel<T, D, G, true>, grid, dim3(NT), 0, st, p);
    else
      launch_pdl(decode_quant_kernel<T, D, G, false>, grid, dim3(NT), 0, st, p);
    return launch_status();
  };
  if (p.g <= 2) return go(std::integral_constant<int, 2>());
  if (p.g <= 4) return go(std::integral_constant<int, 4>());
  if (p.g <= 8) return go(std::integral_constant<int, 8>());
  if constexpr (sizeof(T) == 2) return go(std::integral_constant<int, 16>());
  return MADAKV_EUNSUPPORTED;
}

}  // namespace

int launch_decode_quant(const madakv_config& c, int layer, const void* q, const void* k_new, const void* v_new, uint8_t* k_code,
                        void* k_par, uint8_t* v_code, void* v_par, const int64_t* seg_off, int32_t* kept_len, int64_t capacity,
                        void* out, float* lse_out, const Tracking* track, void* ws, cudaStream_t st) {
  DecodeParams p = decode_params(c, layer, q, k_new, v_new, k_code, v_code, seg_off, kept_len, capacity, out, lse_out, track, ws);
  p.k_par = k_par;
  p.v_par = v_par;
  const int splits = ws_layout(c).decode_splits;
  int rc;
  if (c.dtype == MADAKV_F32)
    rc = c.head_dim == 64 ? run<float, 64>(p, c, splits, st) : run<float, 128>(p, c, splits, st);
  else
    rc = c.head_dim == 64 ? run<__nv_bfloat16, 64>(p, c, splits, st) : run<__nv_bfloat16, 128>(p, c, splits, st);
  return rc || !track ? rc : launch_accumulate(c, layer, seg_off, kept_len, capacity, *track, ws, st);
}

}  // namespace madakv
