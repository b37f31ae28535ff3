// Attention of a prompt and of drafted trees on the tensor cores (bf16):
//   S = Q K^T,  P = exp2(scale * log2(e) * S - m),  O = sum over the tiles of keys of P V,  out = O / sum P
// A block is resident on every SM and goes through work items; an item is two tiles of 128 rows (query, head of the group) of one KV
// head and the 128-key tiles that they see. Everything stays on the SM: S and O of both tiles of rows in tensor memory (4 x 128 columns), P
// over the S that it was made of, as the product's left operand, K and V in a ring of stages that both tiles of rows read.
//   warps 0-3, 4-7   a row per thread: weights of the first and the second tile, results
//   warps 8, 9       matrix products; copies of keys and values, a thread each
//   warp 10          the items one after the other, ahead of the others
//   warp 11          copies of queries; rows of V behind the last key become zeros before the products see them (weights of 0 do not
//                    keep a NaN out, and other sequences' rows or none at all stand there; in K they only make logits that are masked)
// The products of one tile of rows run under the exponentials of the other: S0 S1 | O0 S0' O1 S1' | ... (heads of 64: P is apart from
// S, and S of the next tile of keys runs under a row's own exponentials too: S0' O1 S1' O0' | ...)
// An item whose rows fill one tile only takes the keys in turn: even tiles of keys go to the first accumulator, odd ones to the
// second, and the two are joined at the end.
// The reference m that weights are taken against is the maximum of the row's first tile of keys. It stays, without a look at later
// maxima, until a tile's weights add up to more than 2^16; only then the tile is done again with its maximum, and O and the sum are scaled down. bf16
// weights and fp32 sums have the range for it, relative errors are the same, and numerator and denominator share the factor.
#include "attn_tmem.cuh"

namespace madakv {
namespace {

constexpr int kRows = 128, kKeys = 128, kThreads = 384, kRing = 4;
constexpr float kMostSum = 65536.f;   // of a tile's weights, against the reference

template <int D, bool kTree>
struct Geo {
  static constexpr int kTile = 128 * D * 2;  // bytes of 128 rows: D / 64 blocks of 128 rows of 128 bytes, swizzled
  // Bytes of 64 columns of a tile's results, on their way out: prompts only. (Trees, which stream from memory, need the stage of keys more:
  // 896 segments 290 us with five, 297 with four.)
  static constexpr int kOut = kTree ? 0 : 128 * 128;
  static constexpr int kStages = D == 64 ? 10 : kTree ? 5 : 4;
  // Tensor memory columns: S and O of either tile of rows, and where narrow heads leave room P, which else lies over the S that it was
  // made of. Apart, S of the next tile of keys is computed as soon as S is in registers, and no product stands in a row's chain
  // (32 / 8 heads of 64, 16384 tokens: 1519 -> 1426 us, 772 TFLOP/s).
  static constexpr bool kApart = D == 64;
  static constexpr int kO = 256, kP = kApart ? kO + 2 * D : 0, kPStep = kApart ? 64 : 128;
};

struct Work {
  AttnItem it;
  unsigned y;
  int slot, nb;          // share of the keys, shares that take part
  int begin, end, end0;  // tiles of keys; where the first tile of rows stops
  int main_tiles;        // tiles of keys before the tree's own
  int dual, tok0, tok1;  // one tile of rows only; queries of the tiles
  int q_row, q_outer;    // where the copies of queries begin
  int valid;
};

struct Barriers {
  uint64_t full[10], empty[10], s_full[2], s_empty[2], p_full[2], o_tile[2], o_done[2], q_full, q_empty, item_full[kRing], item_empty[kRing], pair, landed[2], mended[2], out_free[2], out_there[2], drain;
  Work ring[kRing];
  float2 stats[2][kRows];
  uint32_t tmem;
  int abort;
  int mend_stage[2];  // where the copies that landed[] counts go
};
template <int D, bool kTree>
constexpr int smem_bytes() {
  return 2 * Geo<D, kTree>::kTile + Geo<D, kTree>::kStages * Geo<D, kTree>::kTile + 2 * Geo<D, kTree>::kOut + (int)sizeof(Barriers);
}
static_assert(smem_bytes<128, false>() <= 227 * 1024 && smem_bytes<128, true>() <= 227 * 1024 && smem_bytes<64, false>() <= 227 * 1024, "shared memory of a block");

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d_plain(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
__device__ __forceinline__ void tma_store_5d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3, int c4) {
  asm volatile("cp.async.bulk.tensor.5d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5, %6}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1),
               "r"(c2), "r"(c3), "r"(c4)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// Descriptor of V as the operand whose rows are the contraction: 64 columns (128 bytes) by 8 keys are 1024 bytes, swizzled; the next
// 8 keys follow 1024 bytes on (the stride offset, as for the other operands), the next 64 columns a block of 128 keys on.
__device__ __forceinline__ uint32_t v_desc_lo(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | ((uint32_t)(kKeys * 128 >> 4) << 16); }
__host__ __device__ constexpr uint32_t instr_desc_pv(int n) { return instr_desc_bf16(n) | (1u << 16); }

// 2^x of two numbers without the exponential unit, the longest part of narrow heads' chain: x = j + f, |f| <= 1/2; 2^f as the polynomial of
// degree 5 with the least largest relative error (7.5e-8, by exchange; 2.1e-7 with its roundings, as good as the unit's), j added to its
// exponent. From -127 down 2^-149, which bf16 rounds to 0 (a key that is not seen has no weight, whatever its value), off by at most 2^-127 from
// there to -126; above 2^16 from there up and for NaN: the tile is then done again, by the unit.
// (Of 8 pairs one: 32 / 8 heads of 64, 16384 tokens 1426 -> 1359 us, 809 TFLOP/s; of 16 pairs one or three and of 4 pairs one gain less,
// of 8 pairs three nothing. Heads of 128, which the products bound, lose by any.)
__device__ __forceinline__ void exp2_pair(float& lo, float& hi) {
  constexpr float kC0 = 1.00000012f, kC1 = 0.693146944f, kC2 = 0.240221202f, kC3 = 0.0555071309f, kC4 = 0.00967554096f, kC5 = 0.00132764725f;
  constexpr float kRound = 12582912.f;  // 1.5 * 2^23: a sum's last bit is 1
  auto clamp = [](float x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(-127.f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(127.f));
    return x;
  };
  auto both = [](float x) { return pack2(x, x); };
  const uint64_t x = pack2(clamp(lo), clamp(hi)), t = add2(x, both(kRound)), f = fma2(add2(t, both(-kRound)), both(-1.f), x);
  const uint64_t top = fma2(fma2(f, both(kC5), both(kC4)), f, both(kC3));
  const uint64_t y = fma2(fma2(fma2(top, f, both(kC2)), f, both(kC1)), f, both(kC0));
  float t0, t1;
  unpack2(t, t0, t1);
  unpack2(y, lo, hi);
  lo = __uint_as_float((__float_as_uint(t0) << 23) + __float_as_uint(lo));
  hi = __uint_as_float((__float_as_uint(t1) << 23) + __float_as_uint(hi));
}

// The tile that copy number i of an item brings, and whether it is V: as the products ask for them. K0 V0 K1 V1 ... where both tiles of
// rows read every tile of keys; K0 K1 V0 K2 V1 ... where they take them in turn.
__device__ __forceinline__ void copy_of(bool dual, int tiles, int i, int& tile, bool& is_v) {
  if (!dual || tiles == 1) {
    tile = i / 2;
    is_v = i & 1;
  } else if (i == 0) {
    tile = 0;
    is_v = false;
  } else if (i == 2 * tiles - 1) {
    tile = tiles - 1;
    is_v = true;
  } else {  // 1: K1, 2: V0, 3: K2, 4: V1, ...
    tile = i & 1 ? (i + 1) / 2 : i / 2 - 1;
    is_v = !(i & 1);
  }
}
// Keys of the sequence, or nodes, in a tile of 128.
__device__ __forceinline__ int keys_there(const Work& w, int tile, bool own) { return own ? w.it.nodes : w.it.n_keys - tile * kKeys; }

template <int D, bool kTree>
__global__ void __launch_bounds__(kThreads, 1)
    attn_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_tk,
                   const __grid_constant__ CUtensorMap map_tv, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_out,
                   const __grid_constant__ AttnParams p) {
  extern __shared__ __align__(1024) unsigned char base[];
  constexpr int TILE = Geo<D, kTree>::kTile, NST = Geo<D, kTree>::kStages, BLOCK = kRows * 128;
  constexpr bool kApart = Geo<D, kTree>::kApart;
  constexpr int kO = Geo<D, kTree>::kO, kP = Geo<D, kTree>::kP, kPStep = Geo<D, kTree>::kPStep;
  const uint32_t q_smem = smem_u32(base), ring_smem = q_smem + 2 * TILE, out_smem = ring_smem + NST * TILE;
  Barriers& sb = *reinterpret_cast<Barriers*>(base + 2 * TILE + NST * TILE + 2 * Geo<D, kTree>::kOut);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (q_smem & 1023) {  // (the swizzle pattern is one of addresses; the driver places dynamic shared memory so)
    if (threadIdx.x == 0) set_status(p.ws, MADAKV_ECUDA);
    return;
  }

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) mbar_init(&sb.full[i], 1), mbar_init(&sb.empty[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sb.s_full[i], 1);
      mbar_init(&sb.s_empty[i], 4);
      mbar_init(&sb.o_tile[i], 1);
      mbar_init(&sb.p_full[i], 4);
      mbar_init(&sb.o_done[i], 1);
    }
    mbar_init(&sb.q_full, 1);
    mbar_init(&sb.q_empty, 1);
    for (int i = 0; i < kRing; ++i) mbar_init(&sb.item_full[i], 1), mbar_init(&sb.item_empty[i], 1 + 1 + 1 + 8);
    mbar_init(&sb.pair, 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sb.landed[i], 1);
      mbar_init(&sb.mended[i], 1);
      mbar_init(&sb.out_free[i], 1);
      mbar_init(&sb.out_there[i], 4);
    }
    mbar_init(&sb.drain, 1);
    sb.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sb.tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sb.tmem;
  pdl_wait();
  pdl_go();
  Waiter wait{&sb.abort, reinterpret_cast<int32_t*>(p.ws), p.wait_clocks};
  const int tok_m = p.tile_q / 2;  // queries of a tile of rows

  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---- weights and results -------------------------------------------------------------------------------------------
    const int s = warp / 4, r = (warp % 4) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)((warp % 4) * 32) << 16), s_tm = lanes + s * 128, o_tm = lanes + kO + s * D, p_tm = lanes + kP + s * kPStep;
    const int r_q = group_of(p, r), r_head = r - r_q * p.g;
    const uint64_t scale2x = pack2(p.scale2, p.scale2);
    uint32_t n_s = 0, n_o = 0, n_pair = 0, n_out = 0;  // tiles of keys done, meetings of the eight warps, copies of results
    auto meet = [&] {  // (each half has waited for its own accumulator's products and goes on to read the other half's)
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sb.pair);
      wait.all(&sb.pair, n_pair++ & 1, kSiteTile);
      tc_fence_after();
    };
    for (uint32_t round = 0;; ++round) {
      const Work& w = sb.ring[round % kRing];
      if (!wait.all(&sb.item_full[round % kRing], round / kRing & 1, kSiteQFull) || !w.valid) break;
      const AttnItem& it = w.it;
      const bool dual = w.dual;
      const int mt = dual ? 0 : s;
      const int t = it.q0 + mt * tok_m + r_q;
      const bool valid = r_q < (mt ? w.tok1 : w.tok0);
      const bool active = __any_sync(0xffffffffu, valid);
      const int visible = !valid ? 0x7fffffff : kTree || !p.causal ? it.n_keys : min(it.n_keys, t + it.shift + 1);
      const int visible_all = __reduce_min_sync(0xffffffffu, visible);
      uint64_t nodes = 0;
      if constexpr (kTree) nodes = valid ? node_mask(p, it, t) : 0;
      float m = -INFINITY, l = 0.f;
      const int stride = dual ? 2 : 1, tile_end = dual || s ? w.end : w.end0;
      int tile = w.begin + (dual ? s : 0);
      const bool some = tile < tile_end;
      bool look = true;  // rows without a reference, or with one of huge logits
      for (bool first = true; tile < tile_end; tile += stride, first = false) {
        if (!wait.all(&sb.s_full[s], n_s & 1, kSiteFull)) break;
        tc_fence_after();
        if (active) {
          uint32_t z[kKeys];
#pragma unroll
          for (int c = 0; c < kKeys; c += 32) tmem_ld32(s_tm + c, z + c);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < kKeys; c += 32) tie32(z + c);
          if (kApart) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sb.s_empty[s]);
          }
          if (kTree && tile == w.main_tiles) {
#pragma unroll
            for (int c = 0; c < kKeys; ++c)
              if (c >= 64 || !(nodes >> c & 1)) z[c] = 0xff800000u;
          } else if ((tile + 1) * kKeys > visible_all) {
            const int left = visible - tile * kKeys;
#pragma unroll
            for (int c = 0; c < kKeys; ++c)
              if (c >= left) z[c] = 0xff800000u;
          }
          // weights of the tile to where the product reads them; their sum is good where they were taken against a fit reference
          float ref = m;
          auto weights = [&](auto exact) {
            const float off = ref == -INFINITY ? 0.f : -ref * p.scale2;
            const uint64_t off2 = pack2(off, off);
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              uint32_t w2[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float lo, hi;
                unpack2(fma2(pack2u(z[32 * h + 2 * i], z[32 * h + 2 * i + 1]), scale2x, off2), lo, hi);
                if (kApart && !exact.value && i % 8 == 1) {
                  exp2_pair(lo, hi);
                } else {
                  lo = ex2(lo);
                  hi = ex2(hi);
                }
                sum[i & 1] = add2(sum[i & 1], pack2(lo, hi));
                w2[i] = pack_bf16x2(lo, hi);
              }
              if (kApart && h == 0) {  // (the product of the tile before may still read its weights)
                if (!first) wait.all(&sb.o_tile[s], (n_s - 1) & 1, kSiteDrain);
                tc_fence_after();
              }
              tmem_st16(p_tm + 16 * h, w2);
            }
            float lo, hi;
            unpack2(add2(sum[0], sum[1]), lo, hi);
            return lo + hi;
          };
          float part = 0.f;
          if (!look) part = weights(std::false_type());
          if (look || !__all_sync(0xffffffffu, part <= kMostSum || !valid)) {
            float top[2] = {m, -INFINITY};
#pragma unroll
            for (int c = 0; c < kKeys; c += 4) {
              top[0] = max3f(top[0], __uint_as_float(z[c]), __uint_as_float(z[c + 1]));
              top[1] = max3f(top[1], __uint_as_float(z[c + 2]), __uint_as_float(z[c + 3]));
            }
            const float now = fmaxf(top[0], top[1]), f = m == -INFINITY ? 0.f : ex2((m - now) * p.scale2);
            l *= f;
            m = ref = now;
            const bool huge = valid && beyond_rounding(m, p.scale2);
            look = __any_sync(0xffffffffu, huge || (valid && m == -INFINITY));
            if (huge) {
              ref = 0.f;
#pragma unroll
              for (int c = 0; c < kKeys; ++c) z[c] = __float_as_uint(__uint_as_float(z[c]) - m);
            }
            // (P over S: S of this tile has arrived, so the product before it, which was issued before, is done)
            if (!first) {
              if (kApart && !wait.all(&sb.o_tile[s], (n_s - 1) & 1, kSiteDrain)) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                tmem_ld16(o_tm + c, o);
                tmem_wait_ld();
                tie16(o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                tmem_st16(o_tm + c, o);
              }
            }
            part = weights(std::true_type());
          }
          l += part;
          tmem_wait_st();
        } else if (kApart) {
          if (lane == 0) mbar_arrive(&sb.s_empty[s]);
          if (!first && !wait.all(&sb.o_tile[s], (n_s - 1) & 1, kSiteDrain)) break;  // (p_full's phases are passed one by one)
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sb.p_full[s]);
        ++n_s;
      }
      // ---- results ----
      if (some) wait.all(&sb.o_done[s], n_o++ & 1, kSiteDrain);
      tc_fence_after();
      float f0 = 1.f, f1 = 0.f;  // factors of this thread's row in the accumulators that it reads
      if (dual) {
        // the second accumulator's rows join the first's: each half of the warps takes half of the columns of both
        sb.stats[s][r] = make_float2(m, l);
        meet();
        const float2 a = sb.stats[0][r], b = sb.stats[1][r];
        m = fmaxf(a.x, b.x);
        const float at = m == -INFINITY ? 0.f : m;
        f0 = a.x == -INFINITY ? 0.f : ex2((a.x - at) * p.scale2);
        f1 = b.x == -INFINITY ? 0.f : ex2((b.x - at) * p.scale2);
        l = a.y * f0 + b.y * f1;
        if (a.y != a.y || b.y != b.y) l = NAN;
      }
      const bool has0 = dual ? w.end > w.begin : some, has1 = dual && w.end > w.begin + 1;
      const uint32_t o0 = dual ? lanes + kO : o_tm, o1 = lanes + kO + D;
      const int c_begin = dual ? s * (D / 2) : 0, c_end = dual ? c_begin + D / 2 : D;
      const bool split = w.nb > 1;
      const float norm = split ? 1.f : row_factor(l);
      const int64_t row = ((int64_t)w.y * p.slots + w.slot) * p.tile_rows + mt * tok_m * p.g + r;
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + it.out_at + (int64_t)t * p.so.token + r_head * p.so.head;
      if (!kTree && p.copy_out && !dual && !split && (mt ? w.tok1 : w.tok0) == tok_m) {
        // a whole tile of rows: 64 columns at a time through shared memory, swizzled, and out by a copy. (Rows as they stand in the threads
        // are 32 lines a store, 2000 clocks a tile: 16 sequences of 1024 tokens 171 -> 165 us, 8 of 4096 995 -> 976.)
        const bool none = !(l > 0.f || l != l);
        for (int c = 0; c < D; c += 64) {
          if (warp % 4 == 0 && lane == 0) {
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            mbar_arrive(&sb.out_free[s]);
          }
          __syncwarp();
          if (!wait.all(&sb.out_free[s], n_out & 1, kSiteDrain)) break;
#pragma unroll
          for (int h = 0; h < 64; h += 32) {
            uint32_t a[32];
            tmem_ld32(o_tm + c + h, a);
            tmem_wait_ld();
            tie32(a);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              a[i] = none || !some ? 0u : pack_bf16x2(__uint_as_float(a[2 * i]) * norm, __uint_as_float(a[2 * i + 1]) * norm);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(out_smem + s * Geo<D, kTree>::kOut + r * 128 + (((h / 8 + i) ^ (r & 7)) << 4)),
                           "r"(a[4 * i]), "r"(a[4 * i + 1]), "r"(a[4 * i + 2]), "r"(a[4 * i + 3])
                           : "memory");
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sb.out_there[s]);
          if (warp % 4 == 0) {
            if (!wait.all(&sb.out_there[s], n_out & 1, kSiteDrain)) break;
            if (lane == 0) tma_store_5d(&map_out, out_smem + s * Geo<D, kTree>::kOut, c, 0, w.q_row + mt * tok_m, it.h, w.q_outer);
          }
          ++n_out;
        }
      } else if (active && !wait.dead) {
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += 32) {
          uint32_t a[32], b[32];
          __syncwarp();
          tmem_ld32(o0 + c, a);
          if (dual) tmem_ld32(o1 + c, b);
          tmem_wait_ld();
          tie32(a);
          if (dual) tie32(b);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float v = has0 ? __uint_as_float(a[i]) * f0 : 0.f;
            if (has1) v += __uint_as_float(b[i]) * f1;
            a[i] = __float_as_uint(v * norm);
          }
          if (!valid) continue;
          if (split) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) store32(p.part + row * D + c + i, a + i, true);
          } else {
            const bool none = !(l > 0.f || l != l);
#pragma unroll
            for (int i = 0; i < 16; ++i) a[i] = none ? 0u : pack_bf16x2(__uint_as_float(a[2 * i]), __uint_as_float(a[2 * i + 1]));
            store32(dst + c, a, p.wide_out);
            store32(dst + c + 16, a + 8, p.wide_out);
          }
        }
        if (valid && (!dual || s == 0)) {
          if (split) p.part_ml[row] = make_float2(m * p.scale2, l);
        }
      }
      auto finish = [&](int tt, int j, float lse) {
        int64_t win;
        if (!store_row_lse(p, it, tt, j, lse, win)) return;
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.q) + it.q_at + tt * p.sq.token + j * p.sq.head;
        __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(p.q_win) + win * D;
#pragma unroll 1
        for (int c = 0; c < D; c += 64) {
          uint32_t x[32];
#pragma unroll
          for (int i = 0; i < 4; ++i) load32(src + c + 16 * i, x + 8 * i, p.wide_q);
#pragma unroll
          for (int i = 0; i < 4; ++i) store32(to + c + 16 * i, x + 8 * i, p.wide_q);
        }
      };
      if (!split && valid && (!dual || s == 0) && !wait.dead) finish(t, r_head, row_lse(m * p.scale2, l));
      tc_fence_before();
      if (dual) meet();  // (both accumulators have been read before either is written again)
      __syncwarp();
      if (lane == 0) mbar_arrive(&sb.item_empty[round % kRing]);
      if (wait.dead) break;
    }
    if (!kTree && warp % 4 == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 8) {
      // ---- matrix products: one thread ----------------------------------------------------------------------------------
      if (elect_one()) {
        // This thread's chain (weights there -> their product -> the next S) is a row's too: stages are waited for ahead of the weights, and
        // where they are is counted, not worked out.
        constexpr uint32_t kQk = instr_desc_bf16(kKeys), kPv = instr_desc_pv(D);
        uint32_t cur = 0, cur_phase = 0, n_p0 = 0, n_p1 = 0, n_q = 0;
        const uint32_t q_desc = smem_desc_lo(q_smem), ring_desc = smem_desc_lo(ring_smem), v_desc = v_desc_lo(ring_smem);
        struct Stage {
          uint32_t st, phase;
        };
        auto next_stage = [&] {
          const Stage at{cur, cur_phase};
          if (++cur == NST) cur = 0, cur_phase ^= 1;
          return at;
        };
        auto landed = [&](Stage g) { return wait(&sb.full[g.st], g.phase, kSiteFull); };
        uint32_t n_l[2] = {0, 0};
        auto logits = [&](auto slot, uint32_t q, Stage g) {
          if (kApart) {
            if (!wait(&sb.s_empty[slot.value], (n_l[slot.value]++ & 1) ^ 1, kSiteTEmpty)) return;
            tc_fence_after();
          }
          const uint32_t k = ring_desc + g.st * (TILE >> 4);
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const uint32_t at = (i / 4) * (BLOCK >> 4) + (i % 4) * 2;
            umma_bf16(tmem + slot.value * 128, q + at, k + at, kQk, i > 0);
          }
          umma_commit(&sb.s_full[slot.value]);
        };
        auto results = [&](auto slot, uint32_t& n_p, Stage g, bool begun) {
          const uint32_t v = v_desc + g.st * (TILE >> 4);
          if (!wait(&sb.p_full[slot.value], n_p & 1, kSiteTEmpty)) return false;
          ++n_p;
          tc_fence_after();
#pragma unroll
          for (int i = 0; i < kKeys / 16; ++i)
            umma_bf16_ts(tmem + kO + slot.value * D, tmem + kP + slot.value * kPStep + i * 8, v + i * (16 * 128 >> 4), kPv, begun || i > 0);
          if (kApart) umma_commit(&sb.o_tile[slot.value]);
          return true;
        };
        using Slot0 = std::integral_constant<int, 0>;
        using Slot1 = std::integral_constant<int, 1>;
        for (uint32_t round = 0;; ++round) {
          const Work& w = sb.ring[round % kRing];
          if (!wait(&sb.item_full[round % kRing], round / kRing & 1, kSiteQFull) || !w.valid) break;
          const bool dual = w.dual;
          const int tiles = w.end - w.begin, n0 = w.end0 - w.begin;
          mbar_arrive(&sb.item_empty[round % kRing]);
          if (tiles == 0) continue;
          if (!wait(&sb.q_full, n_q++ & 1, kSiteQFull)) break;
          if (dual) {
            auto begin = [&](auto slot) {
              const Stage k = next_stage();
              if (!landed(k)) return;
              tc_fence_after();
              logits(slot, q_desc, k);
              umma_commit(&sb.empty[k.st]);
            };
            begin(Slot0());
            if (tiles > 1) begin(Slot1());
            if (tiles <= 2) umma_commit(&sb.q_empty);
            auto step = [&](auto slot, uint32_t& n_p, int t) {
              const bool more = t + 2 < tiles;
              const Stage v = next_stage(), k = more ? next_stage() : v;
              if (!landed(v) || (more && !landed(k))) return false;
              tc_fence_after();
              if (kApart && more) logits(slot, q_desc, k);
              if (!results(slot, n_p, v, t >= 2)) return false;
              if (!kApart && more) logits(slot, q_desc, k);
              if (!more) umma_commit(&sb.o_done[slot.value]);
              umma_commit(&sb.empty[v.st]);
              if (more) umma_commit(&sb.empty[k.st]);
              if (t + 3 == tiles) umma_commit(&sb.q_empty);
              return true;
            };
            for (int t = 0; t < tiles; t += 2) {
              if (!step(Slot0(), n_p0, t)) break;
              if (t + 1 < tiles && !step(Slot1(), n_p1, t + 1)) break;
            }
          } else {
            const uint32_t q1 = q_desc + (TILE >> 4);
            Stage k = next_stage();
            if (!landed(k)) break;
            tc_fence_after();
            if (n0 > 0) logits(Slot0(), q_desc, k);
            logits(Slot1(), q1, k);
            umma_commit(&sb.empty[k.st]);
            if (tiles == 1) umma_commit(&sb.q_empty);
            if constexpr (kApart) {
              // S of the next tile, then O of the other tile of rows, whose weights are there first: they are half a turn apart
              Stage v = k, v_before = k;
              for (int t = 0; t <= tiles; ++t) {
                const bool more = t + 1 < tiles;
                if (t < tiles) v = next_stage();
                if (more) {
                  k = next_stage();
                  if (!landed(k)) break;
                  tc_fence_after();
                }
                if (t + 1 < n0) logits(Slot0(), q_desc, k);
                if (t > 0) {
                  if (!results(Slot1(), n_p1, v_before, t > 1)) break;
                  if (t == tiles) umma_commit(&sb.o_done[1]);
                  umma_commit(&sb.empty[v_before.st]);
                }
                if (more) {
                  logits(Slot1(), q1, k);
                  umma_commit(&sb.empty[k.st]);
                  if (t + 2 == tiles) umma_commit(&sb.q_empty);
                }
                if (t < tiles) {
                  if (!landed(v)) break;
                  if (t < n0 && !results(Slot0(), n_p0, v, t > 0)) break;
                  if (t + 1 == n0) umma_commit(&sb.o_done[0]);
                }
                v_before = v;
              }
            } else {
              for (int t = 0; t < tiles; ++t) {
                const bool more = t + 1 < tiles;
                const Stage v = next_stage();
                if (more) k = next_stage();
                if (!landed(v) || (more && !landed(k))) break;
                if (t < n0 && !results(Slot0(), n_p0, v, t > 0)) break;
                if (t + 1 < n0) logits(Slot0(), q_desc, k);
                if (t + 1 == n0) umma_commit(&sb.o_done[0]);
                if (!results(Slot1(), n_p1, v, t > 0)) break;
                if (more) logits(Slot1(), q1, k);
                if (!more) umma_commit(&sb.o_done[1]);
                umma_commit(&sb.empty[v.st]);
                if (more) umma_commit(&sb.empty[k.st]);
                if (t + 2 == tiles) umma_commit(&sb.q_empty);
              }
            }
          }
          if (wait.dead) break;
        }
        if (wait.dead) {  // products in flight end before the block does
          umma_commit(&sb.drain);
          const long long t0 = clock64();
          while (!mbar_try(&sb.drain, 0) && clock64() - t0 < kWaitCycles) {}
        }
      }
    } else if (warp == 9) {
      // ---- copies: one thread, which alone waits for stages to become free (a barrier's phases have two names only) -----------
      if (elect_one()) {
        uint32_t seq = 0, n_mend = 0;
        for (uint32_t round = 0;; ++round) {
          const Work& w = sb.ring[round % kRing];
          if (!wait(&sb.item_full[round % kRing], round / kRing & 1, kSiteQFull) || !w.valid) break;
          const int tiles = w.end - w.begin, h = kTree ? 0 : w.it.h, b = kTree || p.k_off ? 0 : w.it.b;
          for (int i = 0; i < 2 * tiles; ++i) {
            int tile;
            bool is_v;
            copy_of(w.dual, tiles, i, tile, is_v);
            tile += w.begin;
            const bool own = kTree && tile == w.main_tiles;
            const uint32_t n = seq + i, st = n % NST;
            if (!wait(&sb.empty[st], (n / NST & 1) ^ 1, kSiteStage)) break;
            uint64_t* bar = &sb.full[st];
            if (is_v && keys_there(w, tile, own) < kKeys) {
              const uint32_t e = n_mend & 1;
              if (!wait(&sb.mended[e], (n_mend / 2 & 1) ^ 1, kSiteTile)) break;
              sb.mend_stage[e] = (int)st;
              bar = &sb.landed[e];
              ++n_mend;
            }
            if (p.hold_copies) continue;
            mbar_expect_tx(bar, TILE);
            const uint32_t dst = ring_smem + st * TILE;
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
              if (own)
                tma_load_5d_plain(dst + x * BLOCK, is_v ? &map_tv : &map_tk, bar, x * 64, 0, w.it.h, w.it.unit / p.Hkv % p.L, w.it.b);
              else
                tma_load_4d(dst + x * BLOCK, is_v ? &map_v : &map_k, bar, x * 64, (int)(w.it.key_row + tile * kKeys), h, b);
            }
          }
          if (wait.dead) break;
          mbar_arrive(&sb.item_empty[round % kRing]);
          seq += 2 * tiles;
        }
        if (wait.dead) {  // copies in flight land before the block ends
          const long long t0 = clock64();
          while (clock64() - t0 < 2000000ll) {}
        }
      }
    } else if (warp == 10) {
      // ---- the items: in rounds over the blocks, to and fro, so that every block gets its share of long ones ----------------
      uint32_t round = 0;
      for (unsigned pass = 0;; ++pass) {
        const unsigned at = pass * gridDim.x + (pass & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        Work w;
        // (all items of a share before the next share: tiles of rows that read the same keys do so at the same time)
        w.slot = p.slots == 1 ? 0 : (int)(at / (unsigned)p.n_items);
        w.y = p.slots == 1 ? at : at % (unsigned)p.n_items;
        bool there = true;
        if (kTree && p.order) {
          there = at < (unsigned)p.order[0];
          w.y = there ? (unsigned)p.order[1 + at] : 0u;
        }
        there = there && (kTree ? tree_item(p, w.y, w.it) : prompt_item(p, w.y, w.it));
        w.valid = p.slots == 1 ? there : w.slot < p.slots;
        if (w.valid) {
          if (!there) continue;
          const AttnItem& it = w.it;
          const int toks = min(p.tile_q, it.n_q - it.q0);
          if (toks <= 0) continue;
          w.tok0 = min(tok_m, toks);
          w.tok1 = toks - w.tok0;
          w.dual = w.tok1 == 0;
          const int tiles = item_tiles<kTree>(p, it);
          w.main_tiles = tiles - (kTree ? 1 : 0);
          const int seen0 = kTree || !p.causal ? it.n_keys : max(0, min(it.n_keys, it.q0 + w.tok0 + it.shift));  // by the first tile of rows
          const int tiles0 = (seen0 + kKeys - 1) / kKeys + (kTree ? 1 : 0);
          w.nb = shares_of(p, tiles);
          if (w.slot >= w.nb) continue;
          share_tiles(w.nb, tiles, w.slot, w.begin, w.end);
          w.end0 = max(w.begin, min(w.end, tiles0));
          w.q_row = (int)((!kTree && p.q_off ? p.q_off[it.b] : 0) + it.q0);
          w.q_outer = kTree && p.layer < 0 ? it.unit / p.Hkv : !kTree && p.q_off ? 0 : it.b;
        }
        if (!wait.all(&sb.item_empty[round % kRing], (round / kRing & 1) ^ 1, kSiteFlag)) break;
        if (lane == 0) {
          sb.ring[round % kRing] = w;
          mbar_arrive(&sb.item_full[round % kRing]);
        }
        __syncwarp();
        ++round;
        if (!w.valid) break;
      }
    } else {
      if constexpr (!kTree) fill_window<D * 2>(p, lane, 32);
      // ---- queries, rows of V behind the last key -----------------------------------------------------------------------------
      uint32_t n_mend = 0, n_q = 0;
      for (uint32_t round = 0;; ++round) {
        const Work& w = sb.ring[round % kRing];
        if (!wait.all(&sb.item_full[round % kRing], round / kRing & 1, kSiteQFull) || !w.valid) break;
        if (w.end > w.begin) {
          if (!wait.all(&sb.q_empty, (n_q++ & 1) ^ 1, kSiteQEmpty)) break;
          if (elect_one()) {
            const int tiles_of_rows = w.dual ? 1 : 2;
            mbar_expect_tx(&sb.q_full, (uint32_t)(tiles_of_rows * tok_m * p.g * D * 2));
            for (int mt = 0; mt < tiles_of_rows; ++mt)
#pragma unroll
              for (int x = 0; x < D / 64; ++x)
                tma_load_5d_plain(q_smem + mt * TILE + x * BLOCK, &map_q, &sb.q_full, x * 64, 0, w.q_row + mt * tok_m, w.it.h, w.q_outer);
          }
          __syncwarp();
        }
        for (int tile = max(w.begin, w.main_tiles - 1); tile < w.end; ++tile) {
          const int there = keys_there(w, tile, kTree && tile == w.main_tiles);
          if (there >= kKeys) continue;
          const uint32_t e = n_mend & 1;
          if (!wait.all(&sb.landed[e], n_mend / 2 & 1, kSiteTile)) break;
          ++n_mend;
          const int st = sb.mend_stage[e];
          unsigned char* v = base + 2 * TILE + st * TILE;
          for (int x = there * 8 + lane; x < kKeys * 8; x += 32)
#pragma unroll
            for (int half = 0; half < D / 64; ++half) *reinterpret_cast<uint4*>(v + half * BLOCK + x * 16) = make_uint4(0, 0, 0, 0);
          fence_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sb.full[st]);
            mbar_arrive(&sb.mended[e]);
          }
        }
        if (wait.dead) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sb.item_empty[round % kRing]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// The items of a tree call by what they cost, the most first, in classes: blocks take them in rounds, to and fro, and end together. (896
// segments of 1000 to 4000 rows, trees of 6 to 41 nodes, in the order of memory: blocks end up to 30 % apart.) One block.
constexpr int kClasses = 1024;
__global__ void __launch_bounds__(kClasses) order_kernel(const __grid_constant__ AttnParams p, float classes_per_cost) {
  __shared__ int start[kClasses], warps[kClasses / 32];
  const int tid = threadIdx.x;
  start[tid] = 0;
  pdl_wait();
  pdl_go();
  __syncthreads();
  auto class_of = [&](unsigned i) {
    AttnItem it;
    tree_item(p, i, it);
    const int queries = min(p.tile_q, it.n_q - it.q0);
    if (queries <= 0) return -1;
    // (a tile of keys takes 1.7 us for two tiles of rows, 0.95 for one; an item 4 us beside)
    const float cost = item_tiles<true>(p, it) * (queries > p.tile_q / 2 ? 1.7f : 0.95f) + 4.f;
    return max(0, kClasses - 1 - (int)(cost * classes_per_cost));
  };
  for (unsigned i = tid; i < (unsigned)p.n_items; i += kClasses) {
    const int c = class_of(i);
    if (c >= 0) atomicAdd(&start[c], 1);
  }
  __syncthreads();
  const int own = start[tid];
  int sum = own;
#pragma unroll
  for (int i = 1; i < 32; i *= 2) {
    const int x = __shfl_up_sync(0xffffffffu, sum, i);
    if (tid % 32 >= i) sum += x;
  }
  if (tid % 32 == 31) warps[tid / 32] = sum;
  __syncthreads();
  if (tid < 32) {
    int x = warps[tid], all = x;
#pragma unroll
    for (int i = 1; i < 32; i *= 2) {
      const int z = __shfl_up_sync(0xffffffffu, all, i);
      if (tid >= i) all += z;
    }
    warps[tid] = all - x;
    if (tid == 31) p.order[0] = all;
  }
  __syncthreads();
  start[tid] = warps[tid / 32] + sum - own;
  __syncthreads();
  for (unsigned i = tid; i < (unsigned)p.n_items; i += kClasses) {
    const int c = class_of(i);
    if (c >= 0) p.order[1 + atomicAdd(&start[c], 1)] = (int)i;  // (within a class in any order: results do not depend on it)
  }
}

// [batch, layers, heads, rows, d] with element strides, boxes of 128 rows by 64 elements; without layers in four dimensions.
bool make_rows_map(CUtensorMap* map, const void* base, int d, int64_t rows, int heads, int layers, int batch, madakv_strides s) {
  if ((heads > 1 && s.head <= 0) || (layers > 1 && s.layer <= 0) || (batch > 1 && s.batch <= 0)) return false;
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const int rank = layers ? 5 : 4;
  const cuuint64_t batches = (cuuint64_t)batch;
  const cuuint64_t dims[5] = {(cuuint64_t)d, (cuuint64_t)rows, (cuuint64_t)heads, layers ? (cuuint64_t)layers : batches, batches};
  auto bytes = [&](int64_t v) { return (cuuint64_t)((v > 0 ? v : d) * 2); };  // (a dimension of extent 1 never advances)
  const cuuint64_t strides[4] = {bytes(s.token), bytes(s.head), bytes(layers ? s.layer : s.batch), bytes(s.batch)};
  for (const cuuint64_t x : strides)
    if (x % 16 || x >= ((cuuint64_t)1 << 40)) return false;
  const cuuint32_t box[5] = {64, kKeys, 1, 1, 1}, one[5] = {1, 1, 1, 1, 1};
  auto encode = [&] {
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  // (a driver call: in a host thread whose first CUDA call this is it needs the context that the runtime makes)
  int dev;
  return encode() || (cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && encode());
}

// Queries as (d, head of the group, query, KV head, outer), boxes of `queries` queries of a whole group: rows of the tile in their order.
bool make_query_map(CUtensorMap* map, const void* base, int d, int g, int64_t rows, int heads, int64_t outer, int64_t outer_stride, madakv_strides s,
                    int queries) {
  EncodeTiledFn fn = encode_fn();
  if (!fn || (g * heads > 1 && s.head <= 0) || (outer > 1 && outer_stride <= 0)) return false;
  const cuuint64_t dims[5] = {(cuuint64_t)d, (cuuint64_t)g, (cuuint64_t)rows, (cuuint64_t)heads, (cuuint64_t)outer};
  auto bytes = [&](int64_t v) { return (cuuint64_t)((v > 0 ? v : d) * 2); };
  const cuuint64_t strides[4] = {bytes(s.head), bytes(s.token), bytes(s.head * g), bytes(outer_stride)};
  for (const cuuint64_t x : strides)
    if (x % 16 || x >= ((cuuint64_t)1 << 40)) return false;
  const cuuint32_t box[5] = {64, (cuuint32_t)g, (cuuint32_t)queries, 1, 1}, one[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kTree>
int run(AttnParams p, const madakv_config& c, cudaStream_t st) {
  CUtensorMap mk, mv, tk, tv, mq, mo;
  p.tile_q = kRows / p.g * 2;
  if constexpr (kTree) {
    const madakv_strides rows{0, 0, 0, D};
    if (p.capacity >= 0x7fffffffll || !make_rows_map(&mk, p.k_c, D, p.capacity, 1, 0, 1, rows) || !make_rows_map(&mv, p.v_c, D, p.capacity, 1, 0, 1, rows) ||
        !make_rows_map(&tk, p.k, D, p.q_rows, p.Hkv, p.L, p.B, p.sk) || !make_rows_map(&tv, p.v, D, p.q_rows, p.Hkv, p.L, p.B, p.sv))
      return -1;
  } else {
    const int batch = p.k_off ? 1 : p.B;
    if (!make_rows_map(&mk, p.k, D, p.k_rows, p.Hkv, 0, batch, p.sk) || !make_rows_map(&mv, p.v, D, p.k_rows, p.Hkv, 0, batch, p.sv)) return -1;
    tk = mk;
    tv = mv;
  }
  // (behind the others: they have seen to it that this thread has a context)
  const bool all = kTree && p.layer < 0;
  if (all && p.B > 1 && p.L > 1 && p.sq.batch != p.L * p.sq.layer) return -1;
  const int64_t outer = all ? (int64_t)p.B * p.L : !kTree && p.q_off ? 1 : p.B;
  const void* q = kTree && !all ? (const char*)p.q + p.layer * p.sq.layer * 2 : p.q;
  if (!make_query_map(&mq, q, D, p.g, p.q_rows, p.Hkv, outer, all && p.L > 1 ? p.sq.layer : p.sq.batch, p.sq, p.tile_q / 2)) return -1;
  p.copy_out = !kTree && make_query_map(&mo, p.out, D, p.g, p.q_rows, p.Hkv, outer, p.so.batch, p.so, p.tile_q / 2);
  if (!p.copy_out) mo = mq;
  attn_items(p, kTree);
  // (28 / 4 heads, one token, 512 keys: 11 us whole, 14 in two shares; 1024 keys: 14.1 and in four 14.6; 2048: 20.7 and in eight 15.4)
  attn_slots(p, c, kTree, kKeys, {0.85f, 1.7f, 4.f, 8});
  attn_waits(p);
  if (p.n_items * p.slots > 0x7ffffff0ll) return MADAKV_EUNSUPPORTED;
  auto wide = [](const void* x, const madakv_strides& t) {
    return ((uintptr_t)x % 32 | t.batch * 2 % 32 | t.layer * 2 % 32 | t.head * 2 % 32 | t.token * 2 % 32) == 0;
  };
  p.wide_out = wide(p.out, p.so);
  p.wide_q = wide(p.q, p.sq) && (uintptr_t)p.q_win % 32 == 0;
  if (kTree && p.slots == 1 && p.n_items > 148 && p.n_items < (int64_t)p.part_rows * D) {
    p.order = reinterpret_cast<int*>(p.part);  // (no shares: the place of their results is free)
    const float most = 1.7f * (float)(((int64_t)c.max_seq_len + c.max_new_tokens) / kKeys + 2) + 4.f;
    launch_pdl(order_kernel, dim3(1), dim3(kClasses), 0, st, p, (kClasses - 1) / most);
    if (const int rc = launch_status()) return rc;
  }
  auto kernel = attn_tc_kernel<D, kTree>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D, kTree>()) != cudaSuccess) return MADAKV_ECUDA;
  // (few works: as many blocks as all get the same number of them)
  const int64_t works = p.n_items * p.slots, each = p.slots > 1 ? (works + 147) / 148 : 1;
  const int64_t blocks = (works + each - 1) / each;
  launch_pdl(kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks < 148 ? blocks : 148)), dim3(kThreads), smem_bytes<D, kTree>(), st, mk, mv, tk, tv, mq, mo, p);
  const int rc = launch_status();
  return rc || p.slots == 1 ? rc : launch_attn_join(p, c, kTree, st);
}

}  // namespace

int launch_attn_tc(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st) {
  if (c.head_dim == 64) return tree ? run<64, true>(p, c, st) : run<64, false>(p, c, st);
  return tree ? run<128, true>(p, c, st) : run<128, false>(p, c, st);
}

}  // namespace madakv
