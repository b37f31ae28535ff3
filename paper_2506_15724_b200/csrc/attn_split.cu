// Attention of a prompt and of drafted trees in fp32 on the tensor cores: every operand as three bf16 terms that add up to it exactly
// (8 leading bits each), a product as the six partial products not below 2^-24 of it, the small ones first, with fp32 sums:
//   S = Q K^T,  P = exp2(scale * log2(e) * S - m),  O = (O + P' V') * exp2(m' - m)
// with m the maximum up to the tile before which it was last looked at: it stays until a tile's weights add up to more than 2^16 (fp32 has
// the range, relative errors are the same), and only then the tile is done again with its maximum.
// The tensor core truncates where it adds, so the results of a tile of keys are summed up on their own and added to O, which a row's thread
// has in registers, with rounding to the nearest. A block has one item: 128 rows, and its share of their keys, N at a time.
//   warps 0-3    a row per thread: weights, results
//   warps 4-11   operands: loads of fp32 rows, their terms to shared memory as the products read them (zeros behind the last key)
//   warp 12      the matrix products, one thread
// The rows of the next tile are on their way from memory while those of one are split, and K of the next tile goes before V of this one,
// which its products need later (half the chain of a tile).
// Bound by the chain of a tile, warps 0-3 (three terms of every weight, O added up) and the six products (6 x 512 clocks for
// 128 x 128 x 64 twice; the tensor pipe takes twice that for tiles as narrow): three prompts of 2503 tokens, 8 heads of 64, take 173 us; 4096
// tokens, 28 / 4 heads of 128, 708 us, 170 TFLOP/s; by fp32 multiply-adds 660 us, and the pipe for those could not take it below 300.
#include "attn_tmem.cuh"

namespace madakv {
namespace {

constexpr int kRows = 128, kThreads = 512, kTerms = 3;
constexpr float kMostSum = 65536.f;  // of a tile's weights, against the reference

template <int D>
struct Geo {
  static constexpr int N = D == 64 ? 128 : 64;      // keys of a tile
  static constexpr int kBlocks = D / 64;            // blocks of 64 columns: rows of 128 bytes, swizzled
  static constexpr int kQBlock = kRows * 128, kQTerm = kBlocks * kQBlock, kQ = kTerms * kQTerm;
  static constexpr int kBlock = N * 128, kTerm = kBlocks * kBlock, kTile = kTerms * kTerm;
  static constexpr int kKeyBuffers = D == 64 ? 2 : 1;
  static constexpr int kS = 0, kP = 2 * N, kO = kP + kTerms * N / 2;  // tensor memory columns: two S, the terms of P, O of a tile
  static_assert(kO + D <= kTmemCols, "tensor memory");
};
struct Barriers {
  uint64_t q_full, k_full[2], k_empty[2], v_full, v_empty, s_full[2], p_full, o_full, drain;
  AttnItem item;
  int there, abort;
  uint32_t tmem;
};
template <int D>
constexpr int smem_bytes() {
  return Geo<D>::kQ + (Geo<D>::kKeyBuffers + 1) * Geo<D>::kTile + (int)sizeof(Barriers);
}
static_assert(smem_bytes<64>() <= 227 * 1024 && smem_bytes<128>() <= 227 * 1024, "shared memory of a block");

// The three terms of two values, packed: the leading 16 bits of what is left, three times.
__device__ __forceinline__ void split2(float a, float b, uint32_t (&t)[kTerms]) {
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
    t[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
    b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
  }
}
// An infinity as the largest finite bf16 number: its products with terms that are 0 would not be numbers.
__device__ __forceinline__ float finite(float x) { return fabsf(x) == INFINITY ? copysignf(3.38953139e38f, x) : x; }

// The terms of 8 elements to shared memory, a term's place `term` bytes behind the one before.
__device__ __forceinline__ void put8(float4 a, float4 b, uint32_t dst, int term) {
  const float big = fmaxf(max3f(max3f(fabsf(a.x), fabsf(a.y), fabsf(a.z)), fabsf(a.w), fabsf(b.x)), max3f(fabsf(b.y), fabsf(b.z), fabsf(b.w)));
  if (big == INFINITY) {
    a = make_float4(finite(a.x), finite(a.y), finite(a.z), finite(a.w));
    b = make_float4(finite(b.x), finite(b.y), finite(b.z), finite(b.w));
  }
  uint32_t t[4][kTerms];
  split2(a.x, a.y, t[0]);
  split2(a.z, a.w, t[1]);
  split2(b.x, b.y, t[2]);
  split2(b.z, b.w, t[3]);
#pragma unroll
  for (int k = 0; k < kTerms; ++k)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + k * term), "r"(t[0][k]), "r"(t[1][k]), "r"(t[2][k]), "r"(t[3][k]) : "memory");
}

template <int D, bool kTree>
__global__ void __launch_bounds__(kThreads, 1) attn_split_kernel(const __grid_constant__ AttnParams p) {
  extern __shared__ __align__(1024) unsigned char base[];
  using G = Geo<D>;
  constexpr int N = G::N;
  const uint32_t q_smem = smem_u32(base), k_smem = q_smem + G::kQ, v_smem = k_smem + G::kKeyBuffers * G::kTile;
  Barriers& sb = *reinterpret_cast<Barriers*>(base + G::kQ + (G::kKeyBuffers + 1) * G::kTile);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (q_smem & 1023) {  // (the swizzle pattern is one of addresses; the driver places dynamic shared memory so)
    if (threadIdx.x == 0) set_status(p.ws, MADAKV_ECUDA);
    return;
  }
  if (threadIdx.x == 0) {
    mbar_init(&sb.q_full, 128);
    for (int i = 0; i < 2; ++i) mbar_init(&sb.k_full[i], 256), mbar_init(&sb.k_empty[i], 1), mbar_init(&sb.s_full[i], 1);
    mbar_init(&sb.v_full, 256);
    mbar_init(&sb.v_empty, 1);
    mbar_init(&sb.p_full, 4);
    mbar_init(&sb.o_full, 1);
    mbar_init(&sb.drain, 1);
    sb.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sb.tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  pdl_go();
  const unsigned y = blockIdx.x / p.slots;
  const int slot = blockIdx.x % p.slots;
  if (warp == 0) {
    AttnItem it;
    const bool there = kTree ? tree_item(p, y, it) : prompt_item(p, y, it);
    if (lane == 0) sb.item = it, sb.there = there;
  }
  if constexpr (!kTree) {
    if (warp == 13) fill_window<D * 4>(p, lane, 32);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sb.tmem;
  const AttnItem& it = sb.item;
  const int queries = sb.there ? min(p.tile_q, it.n_q - it.q0) : 0;
  const int tiles_all = sb.there ? item_tiles<kTree>(p, it) : 0, main_tiles = tiles_all - (kTree ? 1 : 0), nb = shares_of(p, tiles_all);
  int begin = 0, end = 0;
  if (queries > 0 && slot < nb) share_tiles(nb, tiles_all, slot, begin, end);
  const int tiles = end - begin;
  const bool works = queries > 0 && slot < nb;
  Waiter wait{&sb.abort, reinterpret_cast<int32_t*>(p.ws), p.wait_clocks};

  if (warp < 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 240;");
    if (works) {
      // ---- weights and results ---------------------------------------------------------------------------------------------
      const int r = warp * 32 + lane, r_q = group_of(p, r), r_head = r - r_q * p.g, t = it.q0 + r_q;
      const bool valid = r_q < queries, active = __any_sync(0xffffffffu, valid);
      const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
      const int visible = !valid ? 0x7fffffff : kTree || !p.causal ? it.n_keys : min(it.n_keys, t + it.shift + 1);
      const int visible_all = __reduce_min_sync(0xffffffffu, visible);
      uint64_t nodes = 0;
      if constexpr (kTree) nodes = valid ? node_mask(p, it, t) : 0;
      if (tiles > 0) {  // the row's query, while the other warps bring keys
        const float4* src = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + it.q_at + (int64_t)t * p.sq.token + r_head * p.sq.head);
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
          const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
          put8(valid ? src[2 * c] : none, valid ? src[2 * c + 1] : none, q_smem + (c / 8) * G::kQBlock + r * 128 + ((c % 8) ^ (r & 7)) * 16, G::kQTerm);
        }
        fence_async();
        mbar_arrive(&sb.q_full);
      }
      float m = -INFINITY, l = 0.f, o[D];
#pragma unroll
      for (int c = 0; c < D; ++c) o[c] = 0.f;
      auto add_tile = [&] {  // O of the tile before
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint32_t x[32];
          tmem_ld32(lanes + G::kO + c, x);
          tmem_wait_ld();
          tie32(x);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[c + i] += __uint_as_float(x[i]);
        }
      };
      const uint64_t scale2x = pack2(p.scale2, p.scale2);
      bool look = true;  // rows without a reference, or with one of huge logits
      for (int x = 0; x < tiles; ++x) {
        if (!wait.all(&sb.s_full[x & 1], x >> 1 & 1, kSiteFull)) break;
        tc_fence_after();
        float f = 1.f, part = 0.f;
        uint32_t z[N];
        float ref = m;
        bool fresh = look;  // the reference is the maximum so far with this tile's (else it has been for a while)
        while (active) {
#pragma unroll
          for (int c = 0; c < N; c += 32) tmem_ld32(lanes + G::kS + (x & 1) * N + c, z + c);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < N; c += 32) tie32(z + c);
          const int tile = begin + x;
          if (kTree && tile == main_tiles) {
#pragma unroll
            for (int c = 0; c < N; ++c)
              if (c >= 64 || !(nodes >> c & 1)) z[c] = 0xff800000u;
          } else if ((tile + 1) * N > visible_all) {
            const int left = visible - tile * N;
#pragma unroll
            for (int c = 0; c < N; ++c)
              if (c >= left) z[c] = 0xff800000u;
          }
          if (fresh) {
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < N; c += 4) {
              top[0] = max3f(top[0], __uint_as_float(z[c]), __uint_as_float(z[c + 1]));
              top[1] = max3f(top[1], __uint_as_float(z[c + 2]), __uint_as_float(z[c + 3]));
            }
            const float now = fmaxf(m, fmaxf(top[0], top[1]));
            f = m == -INFINITY ? 0.f : ex2((m - now) * p.scale2);
            m = ref = now;
            const bool huge = valid && beyond_rounding(m, p.scale2);
            look = __any_sync(0xffffffffu, huge || (valid && m == -INFINITY));
            if (huge) {
              ref = 0.f;
#pragma unroll
              for (int c = 0; c < N; ++c) z[c] = __float_as_uint(__uint_as_float(z[c]) - m);
            }
          }
          const float off = ref == -INFINITY ? 0.f : -ref * p.scale2;
          const uint64_t off2 = pack2(off, off);
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int c = 0; c < N; c += 2) {
            float lo, hi;
            unpack2(fma2(pack2u(z[c], z[c + 1]), scale2x, off2), lo, hi);
            lo = ex2(lo);
            hi = ex2(hi);
            sum[c >> 1 & 1] = add2(sum[c >> 1 & 1], pack2(lo, hi));
            z[c] = __float_as_uint(lo);
            z[c + 1] = __float_as_uint(hi);
          }
          float lo, hi;
          unpack2(add2(sum[0], sum[1]), lo, hi);
          part = lo + hi;
          if (fresh || __all_sync(0xffffffffu, part <= kMostSum || !valid)) break;
          fresh = true;
        }
        l = l * f + part;
        if (x > 0) {  // (the product of the tile before is done: its results are added, its weights may be written over)
          if (!wait.all(&sb.o_full, (x - 1) & 1, kSiteDrain)) break;
          tc_fence_after();
          if (active) {
            add_tile();
            if (fresh) {
#pragma unroll
              for (int c = 0; c < D; ++c) o[c] *= f;
            }
          }
        }
        if (active) {
#pragma unroll
          for (int c = 0; c < N; c += 32) {
            uint32_t w[kTerms][16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              uint32_t term[kTerms];
              split2(__uint_as_float(z[c + 2 * i]), __uint_as_float(z[c + 2 * i + 1]), term);
#pragma unroll
              for (int k = 0; k < kTerms; ++k) w[k][i] = term[k];
            }
#pragma unroll
            for (int k = 0; k < kTerms; ++k) tmem_st16(lanes + G::kP + k * (N / 2) + c / 2, w[k]);
          }
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sb.p_full);
      }
      if (tiles > 0 && wait.all(&sb.o_full, (tiles - 1) & 1, kSiteDrain)) {
        tc_fence_after();
        if (active) add_tile();
      }
      tc_fence_before();
      // ---- results ----
      const bool split = nb > 1;
      const float norm = split ? 1.f : row_factor(l);
      const int64_t row = ((int64_t)y * p.slots + slot) * p.tile_rows + r;
      float* dst = split ? p.part + row * D : reinterpret_cast<float*>(p.out) + it.out_at + (int64_t)t * p.so.token + r_head * p.so.head;
      auto finish = [&](int tt, int j, float lse) {
        int64_t win;
        if (!store_row_lse(p, it, tt, j, lse, win)) return;
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(p.q) + it.q_at + tt * p.sq.token + j * p.sq.head);
        uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<float*>(p.q_win) + win * D);
#pragma unroll 4
        for (int i = 0; i < D / 4; ++i) to[i] = src[i];
      };
      if (valid && !wait.dead) {
        const bool none = !split && !(l > 0.f || l != l);
#pragma unroll
        for (int c = 0; c < D; c += 8) {
          uint32_t x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = none ? 0u : __float_as_uint(o[c + i] * norm);
          store32(dst + c, x, split || p.wide_out);
        }
        if (split) p.part_ml[row] = make_float2(m * p.scale2, l);
        else finish(t, r_head, row_lse(m * p.scale2, l));
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (!works || tiles == 0) {
    } else if (warp < 12) {
      // ---- operands ----------------------------------------------------------------------------------------------------------
      const int tid = threadIdx.x - 128;
      constexpr int CPR = D / 8;  // pieces of 8 elements of a row
      // Four pieces of 8 elements of a thread, of the rows that at(row) says (null: zeros), from piece x0 on ...
      struct Pieces {
        float4 a[4], b[4];
      };
      auto fetch = [&](Pieces& w, int x0, auto at) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int x = x0 + i * 256;
          const float* src = at(x / CPR);
          w.a[i] = src ? *reinterpret_cast<const float4*>(src + x % CPR * 8) : make_float4(0.f, 0.f, 0.f, 0.f);
          w.b[i] = src ? *reinterpret_cast<const float4*>(src + x % CPR * 8 + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      // ... and their terms to shared memory
      auto put = [&](Pieces& w, int x0, uint32_t to, int block, int term) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int x = x0 + i * 256, r = x / CPR, c = x % CPR;
          put8(w.a[i], w.b[i], to + (c / 8) * block + r * 128 + ((c % 8) ^ (r & 7)) * 16, term);
        }
      };
      auto rows_of = [&](int x, bool is_v) {
        const int tile = begin + x;
        const bool own = kTree && tile == main_tiles;
        const int there = x >= tiles ? 0 : own ? it.nodes : it.n_keys - tile * N;
        const float* from;
        int64_t step;
        if (kTree && !own) {
          from = reinterpret_cast<const float*>(is_v ? p.v_c : p.k_c) + (it.key_row + tile * N) * D;
          step = D;
        } else {
          step = is_v ? p.sv.token : p.sk.token;
          from = reinterpret_cast<const float*>(is_v ? p.v : p.k) + (is_v ? it.v_at : it.k_at) + (own ? 0 : (int64_t)tile * N * step);
        }
        return [=](int r) -> const float* { return r < there ? from + r * step : nullptr; };
      };
      static_assert(N * CPR == 4 * 256, "a tile of keys is four pieces a thread");
      Pieces k, v;  // (a tile's rows are on their way while the rows before are split)
      fetch(k, tid, rows_of(0, false));
      // K of the next tile goes before V of this one: V's place is free when the product of the tile before is done, S should not wait for it.
      auto put_k = [&](int x) {
        const int buf = G::kKeyBuffers == 2 ? x & 1 : 0, use = G::kKeyBuffers == 2 ? x >> 1 : x;
        if (!wait.all(&sb.k_empty[buf], (use & 1) ^ 1, kSiteStage)) return;
        put(k, tid, k_smem + buf * G::kTile, G::kBlock, G::kTerm);
        fence_async();
        mbar_arrive(&sb.k_full[buf]);
      };
      if (!p.hold_copies) {
        fetch(v, tid, rows_of(0, true));
        put_k(0);
        fetch(k, tid, rows_of(1, false));
        for (int x = 0; x < tiles && !wait.dead; ++x) {
          if (x + 1 < tiles) {
            put_k(x + 1);
            fetch(k, tid, rows_of(x + 2, false));
          }
          if (!wait.all(&sb.v_empty, (x & 1) ^ 1, kSiteStage)) break;
          put(v, tid, v_smem, G::kBlock, G::kTerm);
          fence_async();
          mbar_arrive(&sb.v_full);
          fetch(v, tid, rows_of(x + 1, true));
        }
      }
    } else if (warp == 12) {
      // ---- matrix products: one thread ----------------------------------------------------------------------------------------
      if (elect_one()) {
        constexpr uint32_t kQk = instr_desc_bf16(N), kPv = instr_desc_bf16(D) | (1u << 16);  // (V's rows are the contraction)
        constexpr int kA[6] = {2, 0, 1, 1, 0, 0}, kB[6] = {0, 2, 1, 0, 1, 0};  // the small products first
        const uint32_t q_desc = smem_desc_lo(q_smem), k_desc = smem_desc_lo(k_smem);
        const uint32_t v_desc = ((v_smem & 0x3FFFFu) >> 4) | ((uint32_t)(G::kBlock >> 4) << 16);
        auto logits = [&](int x) {
          const int buf = G::kKeyBuffers == 2 ? x & 1 : 0, use = G::kKeyBuffers == 2 ? x >> 1 : x;
          if (!wait(&sb.k_full[buf], use & 1, kSiteFull)) return false;
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < 6; ++i) {
            const uint32_t a = q_desc + ((kA[i] * G::kQTerm) >> 4), b = k_desc + ((buf * G::kTile + kB[i] * G::kTerm) >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_bf16(tmem + G::kS + (x & 1) * N, a + (k / 4) * (G::kQBlock >> 4) + (k % 4) * 2, b + (k / 4) * (G::kBlock >> 4) + (k % 4) * 2, kQk,
                        i + k > 0);
          }
          umma_commit(&sb.s_full[x & 1]);
          umma_commit(&sb.k_empty[buf]);
          return true;
        };
        bool ok = wait(&sb.q_full, 0, kSiteQFull) && logits(0);
        for (int x = 0; ok && x < tiles; ++x) {
          if (x + 1 < tiles && !logits(x + 1)) break;
          if (!wait(&sb.v_full, x & 1, kSiteFull) || !wait(&sb.p_full, x & 1, kSiteTEmpty)) break;
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < 6; ++i) {
            const uint32_t a = tmem + G::kP + kA[i] * (N / 2), b = v_desc + ((kB[i] * G::kTerm) >> 4);
#pragma unroll
            for (int k = 0; k < N / 16; ++k) umma_bf16_ts(tmem + G::kO, a + k * 8, b + k * (16 * 128 >> 4), kPv, i + k > 0);
          }
          umma_commit(&sb.o_full);
          umma_commit(&sb.v_empty);
        }
        if (wait.dead) {  // products in flight end before the block does
          umma_commit(&sb.drain);
          const long long t0 = clock64();
          while (!mbar_try(&sb.drain, 0) && clock64() - t0 < kWaitCycles) {}
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

template <int D, bool kTree>
int run(AttnParams p, const madakv_config& c, cudaStream_t st) {
  p.tile_q = kRows / p.g;
  attn_items(p, kTree);
  if (p.n_items == 0) p.n_items = 1;  // (the window's missing rows are still filled)
  attn_slots(p, c, kTree, Geo<D>::N, {4.7f, 4.7f, 10.f, 2});
  if (p.n_items * p.slots > 0x7ffffff0ll) return MADAKV_EUNSUPPORTED;
  attn_waits(p);
  p.wide_out = ((uintptr_t)p.out % 32 | p.so.batch * 4 % 32 | p.so.layer * 4 % 32 | p.so.head * 4 % 32 | p.so.token * 4 % 32) == 0;
  auto kernel = attn_split_kernel<D, kTree>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>()) != cudaSuccess) return MADAKV_ECUDA;
  launch_pdl(kernel, dim3((unsigned)(p.n_items * p.slots)), dim3(kThreads), smem_bytes<D>(), st, p);
  const int rc = launch_status();
  return rc || p.slots == 1 ? rc : launch_attn_join(p, c, kTree, st);
}

}  // namespace

int launch_attn_split(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st) {
  if (c.head_dim == 64) return tree ? run<64, true>(p, c, st) : run<64, false>(p, c, st);
  return tree ? run<128, true>(p, c, st) : run<128, false>(p, c, st);
}

}  // namespace madakv
