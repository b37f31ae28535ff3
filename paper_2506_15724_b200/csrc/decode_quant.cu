// Stage 5 on a cache in 4 bits: cache append (Eq. 4, the row quantised on the way) and decode attention (Eq. 5).
//
// Bound by HBM at 160 bytes a row (d = 128) only if little is done per code: an SM gets a row of K and V, 256 codes, in seven clocks.
// So the codes go into the tensor cores as they are and the groups' (step, mid) are applied to sums.
//   logits   q . k = sum over groups of step sum q code + (mid - 7.5 step) sum q, the sums over codes by m16n8k16 products of 16 rows
//            with 8 heads; a row's step meets four numbers per thread and group. The second part is one more product, of the rows'
//            (step, mid) words as they lie in the cache with multiples of the queries' sums in three bf16 terms.
//   values   sum of w v = sum of (w step) (code - 7.5) + w mid: the weights take the step of every group before they are rounded to
//            bf16 for the product with the codes; mid is summed up in fp32
// K's codes become fp16 operands (k_operands) and the queries, scaled by a power of two per head, fp16 numbers, in which they are exact;
// V's become bf16 (v_operands), whose range the weights times step need: 16 + code, and 23.5 times the sum of the weights is taken
// off at the end, from one more product, with ones, per group. The order of codes in a row is that of the
// operands: a lane's words are one piece of 16 bytes (K) or 8 (V) a row, pairs along d for K, and of two rows for V.
// fp32: queries as three fp16 terms and weights as three bf16 terms, whose products are exact and whose sum is fp32 again; V's
// operands are code - 7.5 then, so that no sum loses bits to the 23.5.
// A warp has tiles of 32 rows of its own, read ahead into a ring in shared memory by asynchronous copies.
// 1024 segments of 1638 rows, g = 1: 83 us, 0.50 of the copy bandwidth; 8 of 131071, g = 4: 50 us, 0.52. No unit is full (shifts, permutations
// and conversions, two clocks each, 59 % of their pipe; issue 57 %, tensor cores 23 %, DRAM 38 %): three warps a partition go through
// a serial chain per tile.
#include <cuda_fp16.h>

#include <type_traits>

#include "decode_common.cuh"
#include "quant.cuh"

namespace madakv {
namespace {

constexpr int kTile = 32;    // rows of a warp at a time
constexpr int kAhead = 3;    // stages of a warp's ring

template <int D, int kWarps>
struct QuantTile {
  using R = QuantRow<D>;
  static constexpr int K_CODE = 0, K_PAR = kTile * R::CODE_BYTES, V_CODE = K_PAR + kTile * R::PAR_BYTES,
                       V_PAR = V_CODE + kTile * R::CODE_BYTES, STAGE = V_PAR + kTile * R::PAR_BYTES;
  static constexpr int WARP = kAhead * STAGE;
  static constexpr int FRESH = kWarps * WARP;  // the appended row: codes and parameters of K, then of V
  static constexpr int QUERIES = FRESH + 2 * (R::CODE_BYTES + R::PAR_BYTES);
  static_assert(QUERIES % 16 == 0, "read in 16-byte pieces");
  // the queries of 8 NH heads: operands of every term, then [8 NH] scales and [8 NH][NG] sums
  static constexpr int query_bytes(int NH, int terms) { return NH * (R::NG * terms * 512 + 32 + 32 * R::NG); }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // an 8 x 8 matrix of 16-bit elements, two of a row per lane
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// Rows kTile apart from a tile's base for the 8 row slots of a product: slots 2 t and 2 t + 1 are neighbours, slots 0, 2, 4, 6 are rows
// 0, 3, 4, 7, so that neither the loads of K (all slots) nor of V (every other slot) meet more than twice in a bank.
__device__ __forceinline__ int slot_row(int s) { return s ^ ((s >> 1) & 1); }

// The four fp16 operand registers of eight codes, the e-th of either half-word: the codes themselves. Codes 0 and 1 stand in the lower
// bits of a mantissa under the exponent of 1024 without a shift, codes 2 and 3 after one; an addition or a fused multiply-add, on a
// pipe that has little else to do, takes the 1024 off.
__device__ __forceinline__ void k_operands(uint32_t x, uint32_t (&r)[4]) {
  const uint32_t y = x >> 8;
  const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f), less = __floats2half2_rn(-64.f, -64.f), base = __floats2half2_rn(1024.f, 1024.f);
  r[0] = (x & 0x000f000fu) | 0x64006400u;
  r[1] = (x & 0x00f000f0u) | 0x64006400u;
  r[2] = (y & 0x000f000fu) | 0x64006400u;
  r[3] = (y & 0x00f000f0u) | 0x64006400u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 v = *reinterpret_cast<__half2*>(&r[e]), c = e % 2 ? __hfma2(v, sixteenth, less) : __hsub2(v, base);
    r[e] = *reinterpret_cast<const uint32_t*>(&c);
  }
}
// The four bf16 operand registers of eight codes: 16 + code, or code - 7.5. (128 + code, which the lowest four bits give without a shift,
// costs the sums of 130000 flat weights as much as the rounding of the result.)
template <bool kExact>
__device__ __forceinline__ void v_operands(uint32_t x, uint32_t (&r)[4]) {
  r[0] = ((x << 3) & 0x00780078u) | 0x41804180u;
  r[1] = ((x >> 1) & 0x00780078u) | 0x41804180u;
  r[2] = ((x >> 5) & 0x00780078u) | 0x41804180u;
  r[3] = ((x >> 9) & 0x00780078u) | 0x41804180u;
  if constexpr (kExact) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 v = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&r[e]), __floats2bfloat162_rn(23.5f, 23.5f));
      r[e] = *reinterpret_cast<const uint32_t*>(&v);
    }
  }
}
// c (+)= a b in fp16.
__device__ __forceinline__ void mma_codes(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_codes_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// The nearest fp16 numbers of x and y; what is left of the two stays in them.
__device__ __forceinline__ uint32_t next_halves(float& x, float& y) {
  const __half2 h = __floats2half2_rn(x, y);
  x -= __low2float(h);
  y -= __high2float(h);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
// (a0, a1) += k (b0, b1), and (a0, a1) = k (b0, b1), as one instruction each.
__device__ __forceinline__ void fma_pair(float& a0, float& a1, float k, float b0, float b1) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_of(k, k)), "l"(pair_of(b0, b1)), "l"(pair_of(a0, a1)));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(r));
}
__device__ __forceinline__ void mul_pair(float& a0, float& a1, float k, float b0, float b1) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_of(k, k)), "l"(pair_of(b0, b1)));
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(a1) : "l"(r));
}
// A product whose sums start from zero.
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// The n-th bf16 term of x and y (0: the nearest; what is left goes on to the next).
__device__ __forceinline__ uint32_t next_term(float& x, float& y) {
  const uint32_t w = pack_bf16x2(x, y);
  x -= bf16_lo(w);
  y -= bf16_hi(w);
  return w;
}

// NH: groups of eight query heads.
template <typename T, int D, int NH, int kWarps, bool kTrack>
__global__ void __launch_bounds__(32 * kWarps, kWarps > 4 ? 1 : NH == 1 ? 3 : 2) decode_quant_kernel(const __grid_constant__ DecodeParams p) {
  using R = QuantRow<D>;
  using QT = QuantTile<D, kWarps>;
  constexpr int NT = 32 * kWarps;
  constexpr int NG = R::NG;
  constexpr bool kExact = sizeof(T) == 4;
  constexpr int TERMS = kExact ? 3 : 1;
  constexpr int KW = D / 32, VW = D / 64;  // words of a row that a lane takes of K and of V
  constexpr int OPITCH = D + 4;            // floats from one head's merged row to the next
  static_assert(8 * NH * (OPITCH + 2) * 4 <= QT::WARP && 16 * kDecodeSlots * 4 <= QT::WARP, "the merge reuses the rings");
  extern __shared__ __align__(128) unsigned char dsmem[];
  pdl_wait();
  pdl_go();
  const int y = blockIdx.x / p.slots, slot = blockIdx.x % p.slots;
  const int u = unit_of(p, y);
  const SegView view = segment_view(p, u, slot == 0 && threadIdx.x == 0);
  const int len = view.len, nb = segment_blocks(p, len);
  int row_begin, row_end;
  block_rows(nb, len, slot, row_begin, row_end);  // (empty beyond the nb-th block)
  const int h = u % p.Hkv, bl = u / p.Hkv;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int gid = lane / 4, t = lane % 4;  // fragment coordinates: row slots gid and gid + 8, columns (heads) 2 t and 2 t + 1
  float* so = reinterpret_cast<float*>(dsmem + warp * QT::WARP);  // the warp's result, once its ring is done with
  float* bo = reinterpret_cast<float*>(dsmem + QT::WARP);         // the block's: [8 NH][D], [8 NH], [8 NH]
  if (slot < nb) {
    const int64_t off = p.seg_off[u];
    const char* src[4] = {(const char*)p.k_c + off * R::CODE_BYTES, (const char*)p.k_par + off * R::PAR_BYTES,
                          (const char*)p.v_c + off * R::CODE_BYTES, (const char*)p.v_par + off * R::PAR_BYTES};
    unsigned char* ring = dsmem + warp * QT::WARP;
    const uint32_t ring_a = smem_addr(ring);
    const bool owner = view.new_row >= row_begin && view.new_row < row_end;
    auto load_tile = [&](int r, int stage) {
      const uint32_t dst = ring_a + stage * QT::STAGE;
      if (r + kTile <= row_end && !(owner && r + kTile > view.new_row)) {  // whole: each array is one stretch of bytes
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int bytes = a % 2 ? R::PAR_BYTES : R::CODE_BYTES, piece = bytes < 16 ? 8 : 16;
          const uint32_t to = dst + (a == 0 ? QT::K_CODE : a == 1 ? QT::K_PAR : a == 2 ? QT::V_CODE : QT::V_PAR) + lane * piece;
          const char* from = src[a] + (int64_t)r * bytes + lane * piece;
#pragma unroll
          for (int x = 0; x < kTile * bytes / (32 * piece); ++x) {
            if (piece == 16)
              cp_async16(to + x * 32 * piece, from + x * 32 * piece, true);
            else
              cp_async8(to + x * 32 * piece, from + x * 32 * piece, true);
          }
        }
        return;
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int bytes = a % 2 ? R::PAR_BYTES : R::CODE_BYTES;
        const int piece = bytes < 16 ? 8 : 16, per_row = bytes / piece;
        const uint32_t to = dst + (a == 0 ? QT::K_CODE : a == 1 ? QT::K_PAR : a == 2 ? QT::V_CODE : QT::V_PAR);
#pragma unroll
        for (int x = lane; x < kTile * per_row; x += 32) {
          const int rr = x / per_row;
          // (rows behind the share and the appended one, which another thread is writing, are zeros)
          const bool valid = r + rr < row_end && r + rr != view.new_row;
          const char* from = src[a] + (int64_t)(r + (valid ? rr : 0)) * bytes + x % per_row * piece;
          if (piece == 16)
            cp_async16(to + x * 16, from, valid);
          else
            cp_async8(to + x * 8, from, valid);
        }
      }
    };
    const int r_first = row_begin + kTile * warp;
#pragma unroll
    for (int s = 0; s < kAhead - 1; ++s) {
      if (r_first + kTile * kWarps * s < row_end) load_tile(r_first + kTile * kWarps * s, s);
      cp_async_commit();
    }
    // the appended row: quantised into the cache and, for the tile that holds it, into shared memory
    if (owner) {
      if (warp < 2) {
        const int l = lane % R::LANES, G = l % NG;
        float x[4];
        uint32_t codes, par;
        load4(reinterpret_cast<const T*>(warp ? p.v_new : p.k_new) + (int64_t)u * D + 32 * G + 4 * (l / NG), x);
        quantise4<D>(x, codes, par);
        unsigned char* fresh = dsmem + QT::FRESH + warp * (R::CODE_BYTES + R::PAR_BYTES);
        const int64_t row = off + view.new_row;
        if (lane < R::LANES) {
          reinterpret_cast<uint16_t*>(fresh)[l] = (uint16_t)codes;
          reinterpret_cast<uint16_t*>(warp ? p.v_c : p.k_c)[row * (D / 4) + l] = (uint16_t)codes;
        }
        if (lane < NG) {
          reinterpret_cast<uint32_t*>(fresh + R::CODE_BYTES)[l] = par;
          reinterpret_cast<uint32_t*>(warp ? p.v_par : p.k_par)[row * NG + l] = par;
        }
      }
    }

    // queries as operands: products j = 0, 1 of group G pair element 8 t + 2 j + {0, 1} with 8 t + 4 + 2 j + {0, 1}. The same for all
    // warps: they lie in shared memory, 16 bytes of every lane together, and the first warps make a group each
    uint4* queries = reinterpret_cast<uint4*>(dsmem + QT::QUERIES) + lane;
    float* scales = reinterpret_cast<float*>(dsmem + QT::QUERIES + NH * NG * TERMS * 512);
    float* sums = scales + 8 * NH;
    if (warp < NG) {
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        const int head = 8 * n + gid;
        float x[8], top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (head < p.g) {
          const T* q = reinterpret_cast<const T*>(p.q) + ((int64_t)bl * p.Hq + h * p.g + head) * D + 8 * t;
#pragma unroll
          for (int G = 0; G < NG; ++G) {
            float v[8];
            load4(q + 32 * G, *reinterpret_cast<float(*)[4]>(v));
            load4(q + 32 * G + 4, *reinterpret_cast<float(*)[4]>(v + 4));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              top = fmaxf(top, fabsf(v[e]));
              if (G == warp) x[e] = v[e];
            }
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // the head's largest element comes to [2^14, 2^15), where fp16 holds what is 2^-29 of it or more, unless that would take the scale that
        // undoes it below fp32's normal numbers (queries below 2^-108 at the usual scale; a scale of 0 would make NaN of the rows behind
        // a share); an infinity makes the head NaN
        const int room = min(126, max(1, (int)(__float_as_uint(p.scale2) >> 23)) - 1);
        const int k = min(room, 14 - ((int)(__float_as_uint(top) >> 23) - 127));
        const float up = __uint_as_float((uint32_t)(k + 127) << 23);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e] *= up;
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (t == 0) {
          sums[head * NG + warp] = sum;
          if (warp == 0) scales[head] = top < INFINITY ? p.scale2 * __uint_as_float((uint32_t)(127 - k) << 23) : NAN;
        }
#pragma unroll
        for (int term = 0; term < TERMS; ++term) {
          uint4 w;
          w.x = next_halves(x[0], x[4]);
          w.y = next_halves(x[1], x[5]);
          w.z = next_halves(x[2], x[6]);
          w.w = next_halves(x[3], x[7]);
          queries[((n * TERMS + term) * NG + warp) * 32] = w;
        }
      }
    }
    __syncthreads();
    uint32_t qm[NH][3];  // the sums as operands against (step, mid) words: lane t has group t's
    float scale[NH][2];  // of heads 2 t and 2 t + 1: what the scaling took, and the softmax's scale
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float sum = t < NG ? sums[(8 * n + gid) * NG + t] : 0.f, off_sum = -7.5f * sum;
#pragma unroll
      for (int term = 0; term < 3; ++term) qm[n][term] = next_term(off_sum, sum);
      scale[n][0] = scales[8 * n + 2 * t];
      scale[n][1] = scales[8 * n + 2 * t + 1];
    }
    float m[NH][2], l[NH][2];
    float o[NH][NG][2][4], ones[NH][NG][4], mids[NH][NG][2];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int G = 0; G < NG; ++G) {
        mids[n][G][0] = mids[n][G][1] = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) ones[n][G][c] = o[n][G][0][c] = o[n][G][1][c] = 0.f;
      }
    }
    for (int it = 0;; ++it) {
      const int r = r_first + kTile * kWarps * it;
      if (r >= row_end) break;
      const int ahead = r + kTile * kWarps * (kAhead - 1);
      if (ahead < row_end) load_tile(ahead, (it + kAhead - 1) % kAhead);
      cp_async_commit();
      cp_async_wait<kAhead - 1>();
      __syncwarp();
      unsigned char* st = ring + it % kAhead * QT::STAGE;
      if (owner && view.new_row >= r && view.new_row < r + kTile) {  // (a tile of the block before may reach behind its share, as far as this row)
        const int row = view.new_row - r;
        const uint32_t* fresh = reinterpret_cast<const uint32_t*>(dsmem + QT::FRESH);
        constexpr int CW = R::CODE_BYTES / 4;
        if (lane < CW) {
          reinterpret_cast<uint32_t*>(st + QT::K_CODE)[row * CW + lane] = fresh[lane];
          reinterpret_cast<uint32_t*>(st + QT::V_CODE)[row * CW + lane] = fresh[CW + NG + lane];
        }
        if (lane < NG) {
          reinterpret_cast<uint32_t*>(st + QT::K_PAR)[row * NG + lane] = fresh[CW + lane];
          reinterpret_cast<uint32_t*>(st + QT::V_PAR)[row * NG + lane] = fresh[2 * CW + NG + lane];
        }
        __syncwarp();
      }

      // logits of row slots gid (c = 0, 1) and gid + 8 (c = 2, 3) of both halves, heads 2 t (c even) and 2 t + 1
      float s[NH][2][4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t kw[2][KW], kp[2][NG], own_par[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 16 * half + 8 * e + slot_row(gid);
#pragma unroll
          for (int x = 0; x < KW; ++x) kw[e][x] = reinterpret_cast<const uint32_t*>(st + QT::K_CODE)[row * (D / 8) + t * KW + x];
#pragma unroll
          for (int G = 0; G < NG; ++G) kp[e][G] = reinterpret_cast<const uint32_t*>(st + QT::K_PAR)[row * NG + G];
          own_par[e] = reinterpret_cast<const uint32_t*>(st + QT::K_PAR)[row * NG + t % NG];
        }
        const uint32_t ap[4] = {own_par[0], own_par[1], own_par[0], own_par[1]};
#pragma unroll
        for (int n = 0; n < NH; ++n) {  // sum over groups of (mid - 7.5 step) sum q
          mma_first(s[n][half], ap, qm[n][2], 0u);
          mma_bf16_16816(s[n][half], ap, qm[n][0], qm[n][1]);
        }
#pragma unroll
        for (int G = 0; G < NG; ++G) {
          uint32_t a[2][4];
#pragma unroll
          for (int e = 0; e < 2; ++e)  // elements 8 t .. + 3 of the group in the low half, + 4 .. + 7 in the high
            k_operands(__byte_perm(kw[e][G / 2], kw[e][KW / 2 + G / 2], G % 2 ? 0x7632 : 0x5410), a[e]);
          const uint32_t a0[4] = {a[0][0], a[1][0], a[0][1], a[1][1]}, a1[4] = {a[0][2], a[1][2], a[0][3], a[1][3]};
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            float c[4];
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term) {
              const uint4 q = queries[((n * TERMS + term) * NG + G) * 32];
              if (term == TERMS - 1)
                mma_codes_first(c, a0, q.x, q.y);
              else
                mma_codes(c, a0, q.x, q.y);
              mma_codes(c, a1, q.z, q.w);
            }
            fma_pair(s[n][half][0], s[n][half][1], bf16_lo(kp[0][G]), c[0], c[1]);
            fma_pair(s[n][half][2], s[n][half][3], bf16_lo(kp[1][G]), c[2], c[3]);
          }
        }
      }
      if constexpr (kTrack) {
        float* dst = p.scores + (off + r + slot_row(gid)) * p.g + 2 * t;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 2; ++e, dst += 8 * p.g)
            if (r + 16 * half + 8 * e + slot_row(gid) < row_end) {
#pragma unroll
              for (int n = 0; n < NH; ++n) {
                if (8 * n + 2 * t < p.g) dst[8 * n] = s[n][half][2 * e] * scale[n][0];
                if (8 * n + 2 * t + 1 < p.g) dst[8 * n + 1] = s[n][half][2 * e + 1] * scale[n][1];
              }
            }
      }
      if (r + kTile > row_end) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (r + 16 * half + 8 * e + slot_row(gid) >= row_end) {
#pragma unroll
              for (int n = 0; n < NH; ++n) s[n][half][2 * e] = s[n][half][2 * e + 1] = -INFINITY;
            }
      }
      // one softmax step; the weights become w, the sums of the steps before get their factor
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(fmaxf(s[n][0][e], s[n][0][e + 2]), fmaxf(s[n][1][e], s[n][1][e + 2]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          // m is the largest logit as the weights' exponents see it, scaled and rounded: while it stays, the factor of the sums is exactly 1
          // (against the product before its rounding it would be off by up to half a step of m in every tile, always the same way)
          const float mn = fmaxf(m[n][e], mx * scale[n][e]), base = mn == -INFINITY ? 0.f : mn;
          f[e] = fast_ex2(m[n][e] - base);
          m[n][e] = mn;
          float sum = 0.f;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < 2; ++j) sum += s[n][half][2 * j + e] = fast_ex2(fmaf(s[n][half][2 * j + e], scale[n][e], -base));
          l[n][e] = l[n][e] * f[e] + sum;
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
          for (int G = 0; G < NG; ++G) {
            mids[n][G][0] *= f[0];
            mids[n][G][1] *= f[1];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              ones[n][G][c] *= f[c & 1];
              o[n][G][0][c] *= f[c & 1];
              o[n][G][1][c] *= f[c & 1];
            }
          }
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t vw[4][VW], vp[2][NG];
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // rows of slots 2 t, 2 t + 1, 2 t + 8, 2 t + 9
          const int row = 16 * half + 8 * (e >> 1) + slot_row(2 * t + (e & 1));
#pragma unroll
          for (int x = 0; x < VW; ++x) vw[e][x] = reinterpret_cast<const uint32_t*>(st + QT::V_CODE)[row * (D / 8) + gid * VW + x];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int G = 0; G < NG; ++G)
            vp[e][G] = reinterpret_cast<const uint32_t*>(st + QT::V_PAR)[(16 * half + 8 * e + slot_row(gid)) * NG + G];
#pragma unroll
        for (int G = 0; G < NG; ++G) {
          uint32_t a[2][4];
#pragma unroll
          for (int e = 0; e < 2; ++e)
            v_operands<kExact>(__byte_perm(vw[2 * e][G / 2], vw[2 * e + 1][G / 2], G % 2 ? 0x7632 : 0x5410), a[e]);
          const uint32_t a0[4] = {a[0][0], a[0][1], a[1][0], a[1][1]}, a1[4] = {a[0][2], a[0][3], a[1][2], a[1][3]};
          const uint32_t one[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
          const float step[2] = {bf16_lo(vp[0][G]), bf16_lo(vp[1][G])}, mid[2] = {bf16_hi(vp[0][G]), bf16_hi(vp[1][G])};
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            float w[4];
            mul_pair(w[0], w[1], step[0], s[n][half][0], s[n][half][1]);
            mul_pair(w[2], w[3], step[1], s[n][half][2], s[n][half][3]);
            fma_pair(mids[n][G][0], mids[n][G][1], mid[0], s[n][half][0], s[n][half][1]);
            fma_pair(mids[n][G][0], mids[n][G][1], mid[1], s[n][half][2], s[n][half][3]);
            float part[2][4];
#pragma unroll
            for (int term = 0; term < TERMS; ++term) {
              const uint32_t b0 = transposed(next_term(w[0], w[1])), b1 = transposed(next_term(w[2], w[3]));
              if constexpr (kExact) {
                // (sums of 16 rows of their own: the products' adder cuts bits off that a running sum of many rows would miss)
                if (term == 0) {
                  mma_first(part[0], a0, b0, b1);
                  mma_first(part[1], a1, b0, b1);
                } else {
                  mma_bf16_16816(part[0], a0, b0, b1);
                  mma_bf16_16816(part[1], a1, b0, b1);
                }
              } else {
                mma_bf16_16816(o[n][G][0], a0, b0, b1);
                mma_bf16_16816(o[n][G][1], a1, b0, b1);
                mma_bf16_16816(ones[n][G], one, b0, b1);
              }
            }
            if constexpr (kExact) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                o[n][G][0][j] += part[0][j];
                o[n][G][1][j] += part[1][j];
              }
            }
          }
        }
      }
      __syncwarp();  // the stage is refilled from here on
    }
    cp_async_wait<0>();
    __syncwarp();
    // the warp's state into its own area: o [8 NH][OPITCH], m [8 NH], l [8 NH]
    float* sm = so + 8 * NH * OPITCH;
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int head = 8 * n + 2 * t + e;
#pragma unroll
        for (int sh = 4; sh <= 16; sh *= 2) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], sh);
        if (gid == 0) {
          sm[head] = m[n][e];
          sm[8 * NH + head] = l[n][e];
        }
#pragma unroll
        for (int G = 0; G < NG; ++G) {
          float add = mids[n][G][e];
#pragma unroll
          for (int sh = 4; sh <= 16; sh *= 2) add += __shfl_xor_sync(0xffffffffu, add, sh);
          if (!kExact) add = fmaf(-23.5f, ones[n][G][e], add);
          *reinterpret_cast<float4*>(so + head * OPITCH + 32 * G + 4 * gid) = make_float4(
              o[n][G][0][e] + add, o[n][G][0][e + 2] + add, o[n][G][1][e] + add, o[n][G][1][e + 2] + add);
        }
      }
    __syncthreads();
    // (every thread sums what it reads before anything is written: the block's result lies in the second warp's area)
    constexpr int PER = (8 * NH * D + NT - 1) / NT;
    float O[PER], M[PER], L[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int x = threadIdx.x + j * NT, i = x / D, c = x % D;
      if (i >= p.g) break;
      float mw[kWarps];
      M[j] = -INFINITY;
      O[j] = L[j] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        mw[w] = reinterpret_cast<const float*>(dsmem + w * QT::WARP)[8 * NH * OPITCH + i];
        M[j] = fmaxf(M[j], mw[w]);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float* wo = reinterpret_cast<const float*>(dsmem + w * QT::WARP);
        const float fw = part_weight(mw[w], M[j]);
        L[j] += wo[8 * NH * OPITCH + 8 * NH + i] * fw;
        O[j] += wo[i * OPITCH + c] * fw;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int x = threadIdx.x + j * NT, i = x / D, c = x % D;
      if (i >= p.g) break;
      bo[x] = O[j];
      if (c == 0) {
        bo[8 * NH * D + i] = M[j];
        bo[8 * NH * D + 8 * NH + i] = L[j];
      }
    }
    __syncthreads();
  }
  finish_segment<T, D, NT, true>(p, bo, bo + 8 * NH * D, bo + 8 * NH * D + 8 * NH, reinterpret_cast<float*>(dsmem), u, y, slot, nb, view);
}

template <typename T, int D>
int run(DecodeParams p, const madakv_config& c, int splits, cudaStream_t st) {
  if (p.g > (sizeof(T) == 2 ? 16 : 8)) return MADAKV_EUNSUPPORTED;
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  const int64_t rows = p.capacity / units < longest ? p.capacity / units : longest;
  const int resident = 148 * (p.g <= 8 ? 3 : 2);
  // few long segments: one block of as many warps as fit an SM, so that all SMs get the same share (8 segments of 131071 rows: 51 us,
  // 32 blocks of four warps for each of them 75)
  const bool big = p.n_sel <= 20 && p.n_sel * rows >= 148 * 768;
  const int blocks = big ? 148 : resident;
  // otherwise as many blocks of four warps as are resident at once. Calls of more segments than that give each one block: finishing a
  // segment that blocks share takes longer than the more even end saves (1024 segments of 1638 rows, g = 1: 84.8 us with one block,
  // 91-94 where the longer ones have two, 101 at shares of 1024; 896 of 2512, g = 7 and tracking: 159, 154-158, 164)
  const int64_t want = 3 * rows / 256 + 1, most = blocks / p.n_sel < 1 ? 1 : blocks / p.n_sel < kDecodeSlots ? blocks / p.n_sel : kDecodeSlots;
  p.slots = (int)(want < most ? want : most);
  if (p.slots > splits) p.slots = splits;
  if (p.n_sel > kCounters) p.slots = 1;
  p.min_rows = 128;
  p.part_ml = reinterpret_cast<float2*>(p.part + (int64_t)c.batch * c.n_layers * c.n_q_heads * p.slots * D);
  auto go = [&](auto groups, auto warps, auto track) {
    constexpr int W = decltype(warps)::value;
    auto kernel = decode_quant_kernel<T, D, decltype(groups)::value, W, decltype(track)::value>;
    constexpr int bytes = QuantTile<D, W>::QUERIES + QuantTile<D, W>::query_bytes(decltype(groups)::value, sizeof(T) == 4 ? 3 : 1);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return (int)MADAKV_ECUDA;
    launch_pdl(kernel, dim3((unsigned)p.n_sel * p.slots), dim3(32 * W), bytes, st, p);
    return launch_status();
  };
  auto sized = [&](auto groups, auto warps) { return p.scores ? go(groups, warps, std::true_type()) : go(groups, warps, std::false_type()); };
  constexpr std::integral_constant<int, 1> one;
  constexpr std::integral_constant<int, 2> two;
  constexpr std::integral_constant<int, 4> four;
  constexpr std::integral_constant<int, 8> eight;
  constexpr std::integral_constant<int, 12> twelve;
  if (p.g <= 8) return big ? sized(one, twelve) : sized(one, four);
  if constexpr (sizeof(T) == 2) return big ? sized(two, eight) : sized(two, four);
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
