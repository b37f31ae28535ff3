// Stage 4b with a cache in 4 bits: gather the kept K/V rows and quantise them on the way; and the way back for single rows.
//
// A row is shared by lanes of 16 bytes: with 8 (bf16) or 4 (fp32) elements each, 4 or 8 lanes hold a group. HBM takes 29 clocks of an
// SM for a row of K and V (d = 128, bf16: 672 bytes), so that a partition has 116 issue slots for 8 elements of every lane. What keeps
// to that:
//   - a thread has two rows of K and of V at a time. Their groups' extremes meet in log2(lanes) exchanges; then each lane of a group
//     works out (step, mid) for one of the four, and they are handed round: the division is made once per group, not per lane
//   - a code is one fused multiply-add: (x - mid) / step + 8 in units of 2^-16, rounded to a whole number by the constant it is added
//     to. It is off by less than 0.6 units, so the bits above the 16th are the code unless the lower 16 are all zero: then x is on
//     a border, and the bits are right, or just below one. bf16 numbers that are no smaller than step / 256 cannot be that near to a
//     border without being on it (x, mid and step are multiples of 2^-15 of step's power of two), which spares most of them a closer
//     look (every other warp has an element on a border); the others, and fp32, are decided by the exact products of step.
//   - groups with elements outside the sixteen cells (a mid that is large beside step and was rounded), with extreme steps or without
//     one go the exact way altogether
// 1024 units of 1638 rows (d = 128, bf16) take 273 us, 0.64 of the copy bandwidth, bound by the instructions issued (980 with a division
// in fp64 for every code; 238 without looking for elements near borders; 294 with their magnitudes compared as pairs of 16 bits); one
// layer of 4 units of 2048 rows 4.9 us.
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

template <typename T>
struct Lane16;
template <>
struct Lane16<float> {
  static constexpr int N = 4;
  __device__ static void values(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  using Extremes = float2;
  __device__ static Extremes extremes(const uint4& v) {
    float x[4];
    values(v, x);
    float lo = min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3])), hi = max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3]));
#pragma unroll
    for (int off = 1; off < 8; off *= 2) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, off));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, off));
    }
    return make_float2(lo, hi);
  }
  __device__ static float low(Extremes e) { return e.x; }
  __device__ static float high(Extremes e) { return e.y; }
  __device__ static uint32_t par(float lo, float hi) { return group_par(lo, hi); }
  __device__ static bool may_touch(const float (&)[4], float, float) { return true; }
};
template <>
struct Lane16<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static void values(const uint4& v, float (&x)[8]) {
    x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
  }
  __device__ static __nv_bfloat162 two(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
  using Extremes = uint32_t;  // (least, -largest): both get smaller
  __device__ static uint32_t least(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmin2_nan(two(a), two(b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  __device__ static Extremes extremes(const uint4& v) {
    const uint32_t sign = 0x80008000u, a = least(least(v.x, v.y), least(v.z, v.w));
    const uint32_t b = least(least(v.x ^ sign, v.y ^ sign), least(v.z ^ sign, v.w ^ sign));
    uint32_t w = least(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
    for (int off = 1; off < 4; off *= 2) w = least(w, __shfl_xor_sync(0xffffffffu, w, off));
    return w;
  }
  __device__ static float low(Extremes e) { return bf16_lo(e); }
  __device__ static float high(Extremes e) { return -bf16_hi(e); }
  // group_par() in fp32. The sum and the difference of two bf16 numbers are exact or so far from a tie of the roundings that follow that
  // they might be; halves where they would overflow.
  __device__ static uint32_t par(float lo, float hi) {
    const bool huge = hi > 1e38f || lo < -1e38f;
    const float h = huge ? 0.5f : 1.f, sum = __fadd_rn(h * lo, h * hi), diff = __fsub_rn(h * hi, h * lo);
    const float mid = huge ? sum : 0.5f * sum, step = __fdiv_rn(diff, huge ? 7.5f : 15.f);
    const __nv_bfloat162 r = __floats2bfloat162_rn(step, mid);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&r);
    return isfinite(bf16_lo(w)) && isfinite(bf16_hi(w)) ? w : 0x7fc07fc0u;
  }
  // Whether an element (or mid, unless it is 0) is smaller than step / 256.
  __device__ static bool may_touch(const float (&x)[8], float step, float mid) {
    float m = mid == 0.f ? step : fabsf(mid);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fminf(m, fabsf(x[e]));
    return m < step * (1.f / 256.f);
  }
};

constexpr float kUnit = 65536.f;             // 2^16 units to a code
constexpr float kWhole = 12582912.f;         // 1.5 2^23: a float added to it is rounded to a whole number in its lower bits

// 65536 / step where the fast way holds for the group, else NaN.
__device__ __forceinline__ float units_per(uint32_t par, float lo, float hi) {
  const float step = bf16_lo(par), mid = bf16_hi(par);
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
  const float a = fmaf(lo - mid, inv, 8.f), b = fmaf(hi - mid, inv, 8.f);
  return step > 1e-30f && step < 1e30f && a > 0.001f && b < 15.999f ? kUnit * inv : NAN;
}

// The codes of a lane's elements, four in each half of the word; and whether they have to be worked out the exact way.
template <typename T>
__device__ __forceinline__ uint32_t codes_of(const uint4& raw, uint32_t par, float units, bool& unsure) {
  constexpr int N = Lane16<T>::N;
  const float step = bf16_lo(par), mid = bf16_hi(par);
  float x[N];
  Lane16<T>::values(raw, x);
  uint32_t t[N];
#pragma unroll
  for (int e = 0; e < N; ++e) t[e] = __float_as_uint(fmaf(x[e] - mid, units, 8.f * kUnit + kWhole));
  unsure = !(units == units);
  if (Lane16<T>::may_touch(x, step, mid)) {
    uint32_t least = t[0] & 0xffffu;
#pragma unroll
    for (int e = 1; e < N; ++e) least = min(least, t[e] & 0xffffu);
    unsure |= least == 0;
  }
  uint32_t half[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    // codes 0 and 2 in the bytes of the low half, 1 and 3 in those of the high half; then all of them in the low half
    const uint32_t c = (__byte_perm(t[e], t[e + 1], 0x7632) & 0x000f000fu) + (__byte_perm(t[e + 2], t[e + 3], 0x7632) & 0x000f000fu) * 256u;
    half[e / 4] = c | c >> 12;
  }
  return __byte_perm(half[0], half[1], 0x5410);
}
template <typename T>
__device__ __forceinline__ uint32_t exact_codes(const uint4& raw, uint32_t par, float units) {
  const float step = bf16_lo(par), mid = bf16_hi(par);
  float x[Lane16<T>::N];
  Lane16<T>::values(raw, x);
  uint32_t codes = 0;
  if (units == units) {
#pragma unroll
    for (int e = 0; e < Lane16<T>::N; ++e) {
      // d + rest = x - mid exactly; the border that the element is near to, should the lower bits be zero, is an exact product
      const float d = x[e] - mid, y = d - x[e], rest = (x[e] - (d - y)) + (-mid - y), at = fmaf(d, units, 8.f * kUnit + kWhole);
      const float border = (at - (8.f * kUnit + kWhole)) * (1.f / kUnit) * step;
      const uint32_t t = __float_as_uint(at) - ((__float_as_uint(at) & 0xffffu) == 0 && (d < border || (d == border && rest < 0.f)));
      codes |= (t >> 16 & 15u) << (16 * (e / 4) + 4 * (e % 4));
    }
  } else {
#pragma unroll
    for (int e = 0; e < Lane16<T>::N; ++e) codes |= code_of(x[e], step, mid) << (16 * (e / 4) + 4 * (e % 4));
  }
  return codes;
}

// Stores a lane's part of a row of codes at `dst`: two half-words of neighbouring groups make a word, so the lanes GL apart exchange what
// the other one stores.
template <typename T, int D>
__device__ __forceinline__ void store_codes(uint32_t* dst, uint32_t codes, int G, int in_group, bool valid) {
  constexpr int NG = QuantRow<D>::NG, N = Lane16<T>::N;
  const bool odd = G % 2;
  const uint32_t got = __shfl_xor_sync(0xffffffffu, N == 4 ? codes : odd ? codes : codes >> 16, 32 / N);
  if (!valid) return;
  if constexpr (N == 8) {  // elements 8 in_group .. + 3 are half-word 2 in_group, + 4 .. + 7 the next
    dst[(2 * in_group + odd) * (NG / 2) + G / 2] = odd ? __byte_perm(got, codes, 0x7610) : __byte_perm(codes, got, 0x5410);
  } else if (!odd) {
    dst[in_group * (NG / 2) + G / 2] = __byte_perm(codes, got, 0x5410);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(NT, 4) compact_quant_kernel(const __grid_constant__ CompactQuantParams p) {
  using R = QuantRow<D>;
  using V = Lane16<T>;
  constexpr int LPR = D / V::N;   // lanes per row
  constexpr int GL = 32 / V::N;   // lanes per group: 4 or 8
  constexpr int SPAN = NT / LPR;  // rows of the block's threads side by side
  pdl_wait();
  pdl_go();
  const int u = blockIdx.x / p.blocks, x = blockIdx.x % p.blocks;
  const int len = p.kept_len[u];
  const int64_t off = p.seg_off[u];
  // a segment that selection refused (MADAKV_ECAPACITY: it would end beyond the cache) has no index list: skip it
  if (off < 0 || off + len + p.headroom > p.capacity) return;
  const int h = u % p.Hkv, l = (u / p.Hkv) % p.L, b = u / (p.Hkv * p.L);
  const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const int G = lane / GL, in_group = lane % GL;
  const int64_t src_base = b * p.stride_b + l * p.stride_l + h * p.stride_h + lane * 16;
  for (int row0 = x * 2 * SPAN; row0 < len; row0 += p.blocks * 2 * SPAN) {  // (all lanes of a warp stay: they exchange extremes)
    int idx[2];
    uint4 raw[4];  // K and V of the first row, of the second
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = row0 + j * SPAN + sub;
      idx[j] = r < len ? __ldg(p.kept_idx + off + r) : -1;
      if (idx[j] >= p.n_max) idx[j] = -1;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      raw[2 * j] = raw[2 * j + 1] = make_uint4(0u, 0u, 0u, 0u);
      if (idx[j] >= 0) {
        const int64_t src = src_base + (int64_t)idx[j] * p.stride_t;
        raw[2 * j] = __ldg(reinterpret_cast<const uint4*>(p.k + src));
        raw[2 * j + 1] = __ldg(reinterpret_cast<const uint4*>(p.v + src));
      }
    }
    typename V::Extremes ends = V::extremes(raw[0]);  // of the lane's own one of the four
#pragma unroll
    for (int j = 1; j < 4; ++j) {
      const typename V::Extremes other = V::extremes(raw[j]);
      if (in_group % 4 == j) ends = other;
    }
    const float lo = V::low(ends), hi = V::high(ends);
    const uint32_t own = V::par(lo, hi);
    const float own_units = units_per(own, lo, hi);
    if (in_group < 4) {
      const int j = in_group / 2;
      if (idx[j] >= 0) (in_group % 2 ? p.v_par : p.k_par)[(off + row0 + j * SPAN + sub) * R::NG + G] = own;
    }
    uint32_t unsure = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bool again;
      const uint32_t codes = codes_of<T>(raw[j], __shfl_sync(0xffffffffu, own, j, 4), __shfl_sync(0xffffffffu, own_units, j, 4), again);
      uint32_t* dst = reinterpret_cast<uint32_t*>(j % 2 ? p.v_code : p.k_code) + (off + row0 + j / 2 * SPAN + sub) * (D / 8);
      store_codes<T, D>(dst, codes, G, in_group, idx[j / 2] >= 0);
      unsure |= (uint32_t)(again && idx[j / 2] >= 0) << j;
    }
    // (kept apart, with the rows read once more, so that it costs the others nothing)
    unsure = __reduce_or_sync(0xffffffffu, unsure);
#pragma unroll 1
    for (; unsure; unsure &= unsure - 1) {
      const int j = __ffs(unsure) - 1, i = j / 2 ? idx[1] : idx[0];
      uint4 row = make_uint4(0u, 0u, 0u, 0u);
      if (i >= 0) row = __ldg(reinterpret_cast<const uint4*>((j % 2 ? p.v : p.k) + src_base + (int64_t)i * p.stride_t));
      uint32_t* dst = reinterpret_cast<uint32_t*>(j % 2 ? p.v_code : p.k_code) + (off + row0 + j / 2 * SPAN + sub) * (D / 8);
      const uint32_t codes = exact_codes<T>(row, __shfl_sync(0xffffffffu, own, j, 4), __shfl_sync(0xffffffffu, own_units, j, 4));
      store_codes<T, D>(dst, codes, G, in_group, i >= 0);
    }
  }
}

// Rows of K and of V that a thread has on their way. Reading back writes most of its bytes: 1.7 M rows, d = 128, bf16, in 210 us, 0.83 of
// the copy bandwidth (253 with one row and a block for every 16 rows).
constexpr int kExpandRows = 2;

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

__device__ __forceinline__ void store16(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&a);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// fp32 values of four codes in a half-word: a code's bits under an exponent that makes them the integer part, then one subtraction and
// one fused multiply-add, the only rounding.
__device__ __forceinline__ void values4(uint32_t codes, float step, float mid, float* x) {
  const uint32_t y = codes << 4;
  x[0] = fmaf(__uint_as_float((y & 0xf0u) | 0x49000000u) - 524295.5f, step, mid);      // 2^19 + code, in units of 2^-4
  x[1] = fmaf(__uint_as_float((y & 0xf00u) | 0x47000000u) - 32775.5f, step, mid);      // 2^15
  x[2] = fmaf(__uint_as_float((y & 0xf000u) | 0x45000000u) - 2055.5f, step, mid);      // 2^11
  x[3] = fmaf(__uint_as_float((y & 0xf0000u) | 0x43000000u) - 135.5f, step, mid);      // 2^7
}

template <typename T, int D>
__global__ void __launch_bounds__(NT) expand_quant_kernel(const __grid_constant__ ExpandParams p) {
  using R = QuantRow<D>;
  constexpr int N = Lane16<T>::N, LPR = D / N, GL = 32 / N, SPAN = NT / LPR;
  pdl_wait();
  pdl_go();
  const int lane = threadIdx.x % LPR, G = lane / GL, in_group = lane % GL;
  for (int64_t r0 = (int64_t)blockIdx.x * SPAN * kExpandRows + threadIdx.x / LPR; r0 < p.n_rows; r0 += (int64_t)gridDim.x * SPAN * kExpandRows) {
    int64_t row[kExpandRows];
    uint32_t code[kExpandRows][2], par[kExpandRows][2];
#pragma unroll
    for (int i = 0; i < kExpandRows; ++i) {
      const int64_t r = r0 + i * SPAN;
      row[i] = r < p.n_rows ? (p.rows ? __ldg(p.rows + r) : r) : -1;
      if (row[i] >= p.capacity) row[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < kExpandRows; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        code[i][j] = par[i][j] = 0u;  // (zeros)
        if (row[i] < 0) continue;
        const uint16_t* half = reinterpret_cast<const uint16_t*>(j ? p.v_code : p.k_code) + row[i] * (D / 4) + N / 4 * in_group * R::NG + G;
        code[i][j] = __ldg(half) | (N == 8 ? (uint32_t)__ldg(half + R::NG) << 16 : 0u);
        par[i][j] = __ldg((j ? p.v_par : p.k_par) + row[i] * R::NG + G);
      }
#pragma unroll
    for (int i = 0; i < kExpandRows; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t r = r0 + i * SPAN;
        if (r >= p.n_rows) continue;
        float x[N];
#pragma unroll
        for (int e = 0; e < N; e += 4) values4(code[i][j] >> (4 * e) & 0xffffu, bf16_lo(par[i][j]), bf16_hi(par[i][j]), x + e);
        store16(reinterpret_cast<T*>(j ? p.v_out : p.k_out) + r * D + lane * N, x);
      }
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
  // rows of a block: as many as leave 16 blocks for every SM, 32 to 256 (1024 units of 1638 rows, 32 / 64 / 256 / 512 rows a block, in an earlier state: 370 / 330 / 300 / 302 us; 4 of
  // 2048 rows: 5.9 / 7.0 / 14.4 with 32 / 64 / 256)
  const int64_t share = capacity / (148 * 16) / 32 * 32, per_block = share < 32 ? 32 : share > 256 ? 256 : share;
  const int64_t want = (rows + per_block - 1) / per_block, most = ((1 << 20) + units - 1) / units;
  p.blocks = (int)(want < most ? want : most);
  if (units * p.blocks > 0x7fffffff) return MADAKV_EUNSUPPORTED;
  return for_type(c, [&](auto t, auto d) {
    launch_pdl(compact_quant_kernel<decltype(t), decltype(d)::value>, dim3((unsigned)(units * p.blocks)), dim3(NT), 0, st, p);
  });
}

int launch_expand_quant(const madakv_config& c, const int64_t* rows, int64_t n_rows, const uint8_t* k_code, const void* k_par,
                        const uint8_t* v_code, const void* v_par, int64_t capacity, void* k_out, void* v_out, cudaStream_t st) {
  const ExpandParams p{rows, k_code, v_code, (const uint32_t*)k_par, (const uint32_t*)v_par, k_out, v_out, n_rows, capacity};
  const int64_t rpb = NT / (c.head_dim * elem_bytes(c) / 16) * kExpandRows, want = (n_rows + rpb - 1) / rpb;
  const unsigned grid = (unsigned)(want < 148 * 64 ? want : 148 * 64);
  return for_type(c, [&](auto t, auto d) {
    launch_pdl(expand_quant_kernel<decltype(t), decltype(d)::value>, dim3(grid), dim3(NT), 0, st, p);
  });
}

}  // namespace madakv
