// Device code that the decode kernels share: the parameters of a call, what a block works on, the merge of a segment's blocks,
// bulk copies with bounded waits, the warp-level matrix product.
#pragma once

#include "common.cuh"

namespace madakv {
namespace {

constexpr int kDecodeSlots = 32;    // blocks per segment at most

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct DecodeParams {
  const void* q;
  const void* k_new;
  const void* v_new;
  void* k_c;
  void* v_c;
  const int64_t* seg_off;
  int32_t* kept_len;
  int64_t capacity;
  void* out;
  float* lse_out;
  float* part;        // slots > 1: [B*L*Hq, slots, D] partial outputs, then [B*L*Hq, slots, 2] their (max, sum)
  float2* part_ml;
  unsigned* counter;  // slots > 1: one per segment of the call, zero when it begins and when it ends
  void* ws;
  int L, Hq, Hkv, g, layer, slots, n_sel, min_rows;
  float scale2;
  int hold_copies;        // test of waits that run out: no row is copied
  long long wait_clocks;  // bound of a wait for a copy
  // tracking (all null in a call without it): logits in the log2 domain [capacity, g], the heads' log2-sum-exps [B*L*Hq], and
  // where an appended row gets its position and its weight's start
  float* scores;
  float* lse2;
  float* acc;
  int32_t* kept_idx;
  const int32_t* position;
  // the cache in 4 bits: (step, mid) of every row's groups; its codes stand in the place of k_c and v_c
  void* k_par;
  void* v_par;
};

__device__ __forceinline__ float fast_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ int unit_of(const DecodeParams& p, int y) {
  // y enumerates the (sequence, KV head) pairs of the selected layer, or all units when layer < 0
  if (p.layer < 0) return y;
  const int b = y / p.Hkv, h = y % p.Hkv;
  return (b * p.L + p.layer) * p.Hkv + h;
}

// Rows of unit u's segment that attention may read. A segment that selection refused (it, with its headroom, ends
// beyond the cache: MADAKV_ECAPACITY was reported and neither indices nor rows were written) counts as empty, and so
// does one whose length does not fit its own slot: nothing beyond `capacity` rows is ever touched.
__device__ __forceinline__ bool segment_refused(const DecodeParams& p, int u) {
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  return off < 0 || end < off || end > p.capacity;
}
__device__ __forceinline__ int segment_rows(const DecodeParams& p, int u) {
  const int len = p.kept_len[u];
  if (segment_refused(p, u) || len < 0 || p.seg_off[u] + (int64_t)len > p.seg_off[u + 1]) return 0;
  return len;
}
// The blocks of a segment of `len` rows: how many take part, and the rows of block x (a multiple of 16 each, so
// that the 16-row chunks of the warps never straddle two blocks). Block 0 always takes part: an empty segment still
// gets a well-defined partial.
__device__ __forceinline__ int segment_blocks(const DecodeParams& p, int len) {
  return max(1, min(p.slots, (len + p.min_rows - 1) / p.min_rows));
}
__device__ __forceinline__ void block_rows(int nb, int len, int x, int& row_begin, int& row_end) {
  const int share = ((len + nb - 1) / nb + 15) / 16 * 16;
  row_begin = min(len, x * share);
  row_end = min(len, row_begin + share);
}

// What a block of unit u works on. When the call appends (Eq. 4), the new row is part of the attention: the one block
// whose share holds it copies it from k_new / v_new into the cache and reads it from there, all others see the old
// rows only. kept_len itself is bumped by the block that merges, after every block of the segment has read the old value.
// A segment without room for the row (or one that selection refused) is left as it is and MADAKV_ECAPACITY is recorded.
struct SegView {
  int len;      // rows attention covers, the appended one included
  int new_row;  // its index in the segment, or -1
};
__device__ __forceinline__ SegView segment_view(const DecodeParams& p, int u, bool reporter) {
  SegView v;
  v.len = segment_rows(p, u);
  v.new_row = -1;
  if (p.k_new) {
    const int len = p.kept_len[u];
    if (segment_refused(p, u) || len < 0 || p.seg_off[u] + (int64_t)len + 1 > p.seg_off[u + 1]) {
      if (reporter) set_status(p.ws, MADAKV_ECAPACITY);
    } else {
      v.new_row = len;
      v.len = len + 1;
    }
  }
  return v;
}
// The owner of the appended row (the block whose rows include it) stores it into the cache.
template <int ROW_BYTES>
__device__ __forceinline__ void store_new_row(const DecodeParams& p, int u, int64_t off, const SegView& v, int row_begin,
                                              int row_end) {
  constexpr int LPR = ROW_BYTES / 16;
  if (v.new_row < row_begin || v.new_row >= row_end || (int)threadIdx.x >= LPR) return;
  const int64_t row = off + v.new_row;
  const uint4 kv = *reinterpret_cast<const uint4*>((const char*)p.k_new + (int64_t)u * ROW_BYTES + threadIdx.x * 16);
  const uint4 vv = *reinterpret_cast<const uint4*>((const char*)p.v_new + (int64_t)u * ROW_BYTES + threadIdx.x * 16);
  *reinterpret_cast<uint4*>((char*)p.k_c + row * ROW_BYTES + threadIdx.x * 16) = kv;
  *reinterpret_cast<uint4*>((char*)p.v_c + row * ROW_BYTES + threadIdx.x * 16) = vv;
}

template <typename T>
struct Vec16;
template <>
struct Vec16<float> {
  static constexpr int N = 4;
  __device__ static void load(const void* p, float* f) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  }
  __device__ static void cvt(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
};
template <>
struct Vec16<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static void load(const void* p, float* f) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
  }
  __device__ static void cvt(const uint4& v, float* f) {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
  }
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// The weight of a partial with maximum m against the overall maximum M.
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.f : exp2f(m - M); }

constexpr float kLost = -1.f;  // in the place of a sum of weights: a wait for the rows ran out
// Four results of one query head: `o` unnormalised, l their sum of weights.
// A sum of weights that is not a number gives 0, or NaN with kNan (the cache in 4 bits).
template <typename T, int D, bool kNan = false>
__device__ __forceinline__ void store4(const DecodeParams& p, int64_t row, int c, float4 o, float l) {
  const float none = l < 0.f || (kNan && l != l) ? NAN : 0.f;
  const float r0 = l > 0.f ? o.x / l : none, r1 = l > 0.f ? o.y / l : none, r2 = l > 0.f ? o.z / l : none, r3 = l > 0.f ? o.w / l : none;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.out) + row * D + c) = make_float4(r0, r1, r2, r3);
  } else {
    const __nv_bfloat162 a = __floats2bfloat162_rn(r0, r1), b = __floats2bfloat162_rn(r2, r3);
    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * D + c) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
}
template <bool kNan = false>
__device__ __forceinline__ void store_lse(const DecodeParams& p, int64_t row, float M, float l) {
  if (p.lse_out) p.lse_out[row] = l > 0.f ? (M + log2f(l)) * kLn2 : (l < 0.f || (kNan && l != l) ? NAN : -INFINITY);
  // for accumulate_kernel: +inf, no weight of this head counts; NaN, the segment's rows did not arrive
  if (p.lse2) p.lse2[row] = l > 0.f ? M + log2f(l) : (l < 0.f ? NAN : INFINITY);
}
// The segment is one row longer from now on: done by one thread, after every block of the segment has read the old length. An
// appended row starts without weight.
__device__ __forceinline__ void finish_append(const DecodeParams& p, int u, const SegView& view) {
  if (view.new_row < 0) return;
  p.kept_len[u] = view.len;
  const int64_t row = p.seg_off[u] + view.new_row;
  if (p.acc) p.acc[row] = 0.f;
  if (p.kept_idx) p.kept_idx[row] = p.position[u / (p.L * p.Hkv)];
}

// The end of a block: its results lie in shared memory (bo [g][D] unnormalised, bm and bl [g], complete behind a barrier of
// the block); they are combined with those of the segment's other blocks, in block order. fac: kDecodeSlots * g floats of
// shared memory. `nb` blocks of the segment have results; the others arrive at the counter all the same, so that the last
// one knows that all have read the segment's length.
template <typename T, int D, int NTHR, bool kNan = false>
__device__ __forceinline__ void finish_segment(const DecodeParams& p, const float* bo, const float* bm, const float* bl, float* fac,
                                               int u, int y, int slot, int nb, SegView view) {
  constexpr int C4 = D / 4;
  const int h = u % p.Hkv, blr = u / p.Hkv;
  const int64_t row0 = (int64_t)blr * p.Hq + h * p.g;
  if (p.slots == 1) {
    for (int x = threadIdx.x; x < p.g * C4; x += NTHR) {
      const int i = x / C4, c = x % C4 * 4;
      store4<T, D, kNan>(p, row0 + i, c, *reinterpret_cast<const float4*>(bo + i * D + c), bl[i]);
      if (c == 0) store_lse<kNan>(p, row0 + i, bm[i], bl[i]);
    }
    if (threadIdx.x == 0) finish_append(p, u, view);
    return;
  }
  if (slot < nb) {
    for (int x = threadIdx.x; x < p.g * C4; x += NTHR) {
      const int i = x / C4, c = x % C4 * 4;
      __stcg(reinterpret_cast<float4*>(p.part + ((row0 + i) * p.slots + slot) * D + c),
             *reinterpret_cast<const float4*>(bo + i * D + c));
    }
    if ((int)threadIdx.x < p.g) __stcg(p.part_ml + (row0 + threadIdx.x) * p.slots + slot, make_float2(bm[threadIdx.x], bl[threadIdx.x]));
  }
  __shared__ unsigned s_last;
  __syncthreads();
  if (threadIdx.x == 0) s_last = arrive_inc(p.counter + y, (unsigned)p.slots - 1u);  // (wraps to 0: ready for the next call)
  __syncthreads();
  if (s_last != (unsigned)p.slots - 1u) return;
  if (threadIdx.x == 0) finish_append(p, u, view);
  // weights of the partials, and every head's maximum and sum; the first partials are on their way meanwhile
  __shared__ float s_l[16];
  constexpr int kFirst = 8, kHeads = (16 * 32 + NTHR - 1) / NTHR;  // heads per warp at most
  float2 ml[kHeads];
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int i = (int)threadIdx.x / 32 + j * (NTHR / 32), s = threadIdx.x % 32;
    ml[j] = i < p.g && s < nb ? __ldcg(p.part_ml + (row0 + i) * p.slots + s) : make_float2(-INFINITY, 0.f);
  }
  float4 v[kFirst];
  auto load_parts = [&](int x, int s0) {
    const float4* src = reinterpret_cast<const float4*>(p.part + (row0 + x / C4) * p.slots * D + x % C4 * 4);
#pragma unroll
    for (int s = 0; s < kFirst; ++s) v[s] = s0 + s < nb ? __ldcg(src + (s0 + s) * C4) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  if ((int)threadIdx.x < p.g * C4) load_parts(threadIdx.x, 0);
#pragma unroll
  for (int j = 0; j < kHeads; ++j) {
    const int i = (int)threadIdx.x / 32 + j * (NTHR / 32), s = threadIdx.x % 32;
    if (i >= p.g) break;
    const float m = ml[j].x;
    float M = m;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    const float f = part_weight(m, M);
    float l = ml[j].y * f;
    if (s < nb) fac[i * kDecodeSlots + s] = f;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if (__any_sync(0xffffffffu, ml[j].y < 0.f)) l = kLost;
    if (s == 0) {
      s_l[i] = l;
      store_lse<kNan>(p, row0 + i, M, l);
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < p.g * C4; x += NTHR) {
    const int i = x / C4, c = x % C4 * 4;
    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < nb; s0 += kFirst) {
      if (s0 || x != (int)threadIdx.x) load_parts(x, s0);
#pragma unroll
      for (int s = 0; s < kFirst; ++s) {
        const float f = s0 + s < nb ? fac[i * kDecodeSlots + s0 + s] : 0.f;
        O.x += v[s].x * f;
        O.y += v[s].y * f;
        O.z += v[s].z * f;
        O.w += v[s].w * f;
      }
    }
    store4<T, D, kNan>(p, row0 + i, c, O, s_l[i]);
  }
}

// ---- bulk copies ---------------------------------------------------------------------------------------------------------
constexpr long long kCopyWait = 4000000000ll;  // ~2 s: bound of a wait for a copy
constexpr long long kLandWait = 2000000ll;     // ~1 ms: what copies in flight get to land once a wait has run out

__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait. False if it runs out, here or in another thread of the block; that is reported where there is a workspace.
__device__ __forceinline__ bool bar_wait(const DecodeParams& p, uint64_t* bar, uint32_t parity, volatile int* gave_up) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity)) {
    if (*gave_up) return false;
    if (clock64() - t0 > p.wait_clocks) {
      *gave_up = 1;
      if (p.ws) set_status(p.ws, MADAKV_ETIMEOUT);
    }
  }
  return true;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(smem_addr(bar))
               : "memory");
}

// ---- warp-level matrix product -------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// ---- host ----------------------------------------------------------------------------------------------------------------
// What every kernel of a call with a workspace gets. (slots, min_rows and part_ml follow from the kernel that is chosen.)
inline DecodeParams decode_params(const madakv_config& c, int layer, const void* q, const void* k_new, const void* v_new, void* k_c,
                                  void* v_c, const int64_t* seg_off, int32_t* kept_len, int64_t capacity, void* out, float* lse_out,
                                  const Tracking* track, void* ws) {
  const WsLayout wl = ws_layout(c);
  DecodeParams p = {};
  p.q = q;
  p.k_new = k_new;
  p.v_new = v_new;
  p.k_c = k_c;
  p.v_c = v_c;
  p.seg_off = seg_off;
  p.kept_len = kept_len;
  p.capacity = capacity;
  p.out = out;
  p.lse_out = lse_out;
  p.part = reinterpret_cast<float*>((char*)ws + wl.decode_off);
  p.counter = reinterpret_cast<unsigned*>((char*)ws + kHeaderBytes);
  p.ws = ws;
  p.L = c.n_layers;
  p.Hq = c.n_q_heads;
  p.Hkv = c.n_kv_heads;
  p.g = c.n_q_heads / c.n_kv_heads;
  p.layer = layer;
  p.n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  p.scale2 = scale_of(c) * kLog2e;
  p.hold_copies = 0;
  p.wait_clocks = kCopyWait;
  if (track) {
    p.scores = track->scores;
    p.lse2 = tracking_lse2(c, ws);
    p.acc = track->acc;
    p.kept_idx = track->kept_idx;
    p.position = track->position;
  }
  return p;
}

}  // namespace
}  // namespace madakv
