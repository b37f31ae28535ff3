// Eviction while decoding: a segment with more rows than its limit keeps those of the largest accumulated weight, in place.
//
//   which   the c-th largest of the order (protected, weight, lower row first): a histogram of the rows' leading 11 bits, from the top,
//           finds the bin it lies in (a quarter of an octave of weights); up to 512 rows in that bin are compared with one another, more
//           are counted by further digits
//   where   rows [0, c) that go are holes, rows from c on that stay fill them, the j-th hole with the j-th such row: no row that is
//           read is written, so all moves run at once, and only those rows move (a stable compaction would move half the segment to
//           evict one row)
// One block per segment. A call of few is bound by its chain of barriers, one of many by instructions (1024 segments of 1702 rows: 28 us, 59 % of
// the issue slots, 22 % of DRAM), neither by the 8 bytes a row that it reads. Threads keep their rows' keys in registers; segments
// that are too long for that read them from memory every time (8 of 40000 rows: 51 us, 8 of 12000, in registers: 16).
#include <limits.h>

#include <type_traits>

#include "common.cuh"

namespace madakv {
namespace {

// Threads of a block and rows of a thread whose keys stay in registers: what a block takes is mostly what its warps do between barriers,
// so calls of many segments take few warps each (1024 segments of 1702 rows, 64 of them too many, us with 128 x 24 / 256 x 12 / 512 x 6:
// 28.5 / 31 / 33), calls that leave the SMs a block or two take more (4 of 2049: 6.4 / 4.8 / 4.4).
constexpr int kBits = 11, kBins = 1 << kBits;
constexpr int kCandidates = 512;         // rows of a bin that are compared with one another
constexpr int kList = 1024;              // rows moved between two barriers
constexpr int kMaxRows = 3 << 19;        // longest segment: a bit per row lies in shared memory
constexpr uint32_t kSafe = 0xffffffffu;  // in the place of a protected row's weight

struct EvictParams {
  const int32_t* limit;
  float* acc;
  int32_t* kept_idx;
  const int64_t* seg_off;
  int32_t* kept_len;
  int64_t capacity;
  RowArray rows[4];
  int recent, L, Hkv, layer, max_rows;
};

struct EvictShared {
  int hist[kBins];
  uint64_t candidates[kCandidates];
  int to[kList], from[kList];
  int warp_sums[32];
  int bin, above, in, n_candidates;
  uint64_t last;
};

// Sum over the block of one int per thread; and the sum of those before the thread.
template <int NT>
__device__ __forceinline__ int block_sum(int v, int* warp_sums, int* before = nullptr) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int x = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  const int sums = lane < NT / 32 ? warp_sums[lane] : 0;
  if (before) *before = (int)__reduce_add_sync(0xffffffffu, lane < warp ? sums : 0) + x - v;
  return __reduce_add_sync(0xffffffffu, sums);
}

// One 64-bit number per row, larger for a row that goes earlier into the kept set; all different.
__device__ __forceinline__ uint64_t place(uint32_t key, int row) { return ((uint64_t)key << 32) | (uint32_t)~row; }

template <int NT, int kKeys, int PIECE, bool kInRegisters>
__device__ __forceinline__ void evict_segment(const EvictParams& p, EvictShared& sh, uint32_t* stays, int u, int64_t off, int len, int limit) {
  const float* acc = p.acc + off;
  const int32_t* pos = p.kept_idx + off;
  uint32_t key[kKeys];
  int at[kKeys];
  float weight[kKeys];
  int newest = INT_MIN;
  for (int b = threadIdx.x; b < kBins; b += NT) sh.hist[b] = 0;
  if (threadIdx.x == 0) sh.n_candidates = 0;
  if constexpr (kInRegisters) {
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
      const int r = k * NT + threadIdx.x;
      at[k] = r < len ? pos[r] : INT_MIN;
      weight[k] = r < len ? acc[r] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kKeys; ++k) newest = max(newest, at[k]);
  } else {
    for (int r = threadIdx.x; r < len; r += NT) newest = max(newest, pos[r]);
  }
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (threadIdx.x % 32 == 0) sh.warp_sums[threadIdx.x / 32] = newest;
  __syncthreads();
  newest = __reduce_max_sync(0xffffffffu, threadIdx.x % 32 < NT / 32 ? sh.warp_sums[threadIdx.x % 32] : INT_MIN);
  const int64_t young = (int64_t)newest - p.recent;
  if constexpr (kInRegisters) {
#pragma unroll
    for (int k = 0; k < kKeys; ++k) key[k] = at[k] > young ? kSafe : psi_key(weight[k]);
  }
  // f(row, key) for every row of the thread, in strides of the block
  auto each = [&](auto f) {
    if constexpr (kInRegisters) {
#pragma unroll
      for (int k = 0; k < kKeys; ++k)
        if (k * NT + (int)threadIdx.x < len) f(k * NT + (int)threadIdx.x, key[k]);
    } else {
      for (int r = threadIdx.x; r < len; r += NT) f(r, pos[r] > young ? kSafe : psi_key(acc[r]));
    }
  };
  // the bin, from the top, in which the count of rows reaches `need`
  auto walk = [&](int need) {
    constexpr int PER = kBins / NT;
    int mine[PER], sum = 0, before;
#pragma unroll
    for (int j = 0; j < PER; ++j) sum += mine[j] = sh.hist[kBins - 1 - (threadIdx.x * PER + j)];
    block_sum<NT>(sum, sh.warp_sums, &before);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (before < need && before + mine[j] >= need) {
        sh.bin = kBins - 1 - (threadIdx.x * PER + j);
        sh.above = before;
        sh.in = mine[j];
      }
      before += mine[j];
    }
    __syncthreads();
  };
  each([&](int, uint32_t k) { atomicAdd(&sh.hist[k >> (32 - kBits)], 1); });
  __syncthreads();
  const int c = max(limit, sh.hist[kBins - 1]);  // (only protected rows have that bin: the largest weight is infinity)
  if (c >= len) return;
  uint64_t last = ~0ull;  // the place of the last row that stays (c = 0: none does)
  if (c > 0) {
    walk(c);
    int need = c - sh.above, shift = 64 - kBits;
    uint64_t prefix = (uint64_t)sh.bin << shift;
    const int in = sh.in;
    if (need < in && in <= kCandidates) {
      const uint32_t bin = sh.bin;
      each([&](int r, uint32_t k) {
        if (k >> (32 - kBits) == bin) sh.candidates[atomicAdd(&sh.n_candidates, 1)] = place(k, r);
      });
      __syncthreads();
      for (int i = threadIdx.x; i < in; i += NT) {
        const uint64_t own = sh.candidates[i];
        int larger = 0;
        for (int j = 0; j < in; ++j) larger += sh.candidates[j] > own;
        if (larger == need - 1) sh.last = own;
      }
      __syncthreads();
      prefix = sh.last;
    } else {
      while (need < sh.in) {  // (else all rows of the bin stay)
        const uint64_t known = ~0ull << shift;  // the bits that the digits so far have settled
        shift = shift > kBits ? shift - kBits : 0;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += NT) sh.hist[b] = 0;
        __syncthreads();
        each([&](int r, uint32_t k) {
          const uint64_t x = place(k, r);
          if (((x ^ prefix) & known) == 0) atomicAdd(&sh.hist[(x >> shift) & (kBins - 1)], 1);
        });
        __syncthreads();
        walk(need);
        prefix |= (uint64_t)sh.bin << shift;  // (the last digit overlaps the one before it; what the two share agrees)
        need -= sh.above;
      }
    }
    last = prefix;
  }
  // a bit per row: it stays
  const int words = (len + 31) / 32;
  if constexpr (kInRegisters) {
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
      const int r = k * NT + threadIdx.x;
      const uint32_t bits = __ballot_sync(0xffffffffu, c > 0 && r < len && place(key[k], r) >= last);
      if (threadIdx.x % 32 == 0 && r < len) stays[r / 32] = bits;
    }
  } else {
    for (int w = threadIdx.x / 32; w < words; w += NT / 32) {
      const int r = w * 32 + threadIdx.x % 32;
      const uint32_t k = r < len ? (pos[r] > young ? kSafe : psi_key(acc[r])) : 0u;
      const uint32_t bits = __ballot_sync(0xffffffffu, c > 0 && r < len && place(k, r) >= last);
      if (threadIdx.x % 32 == 0) stays[w] = bits;
    }
  }
  __syncthreads();
  // every thread's words, one stretch each: holes below c, rows to move from c on (as many of the ones as of the others)
  const int per = (words + NT - 1) / NT, w0 = min(words, (int)threadIdx.x * per), w1 = min(words, w0 + per);
  auto below = [&](int w) { return w * 32 + 32 <= c ? ~0u : w * 32 >= c ? 0u : (1u << (c - w * 32)) - 1u; };
  int holes = 0, movers = 0, hole0, mover0;
  for (int w = w0; w < w1; ++w) {
    holes += __popc(~stays[w] & below(w));
    movers += __popc(stays[w] & ~below(w));
  }
  int n;
  if constexpr (kInRegisters) {  // (both counts fit half a word)
    n = block_sum<NT>(holes | movers << 16, sh.warp_sums, &hole0) & 0xffff;
    mover0 = hole0 >> 16;
    hole0 &= 0xffff;
  } else {
    block_sum<NT>(holes, sh.warp_sums, &hole0);
    n = block_sum<NT>(movers, sh.warp_sums, &mover0);
  }
  int first[5] = {0, 0, 0, 0, 0};  // pieces of a row before each array
#pragma unroll
  for (int t = 0; t < 4; ++t) first[t + 1] = first[t] + p.rows[t].bytes / PIECE;
  for (int j0 = 0; j0 < n; j0 += kList) {
    int a = hole0, b = mover0;
    for (int w = w0; w < w1; ++w) {
      for (uint32_t bits = ~stays[w] & below(w); bits; bits &= bits - 1, ++a)
        if (a >= j0 && a < j0 + kList) sh.to[a - j0] = w * 32 + __ffs(bits) - 1;
      for (uint32_t bits = stays[w] & ~below(w); bits; bits &= bits - 1, ++b)
        if (b >= j0 && b < j0 + kList) sh.from[b - j0] = w * 32 + __ffs(bits) - 1;
    }
    __syncthreads();
    const int m = min(kList, n - j0), pieces = m * first[4];
    for (int j = threadIdx.x; j < m; j += NT) {
      const float w = acc[sh.from[j]];
      const int32_t q = pos[sh.from[j]];
      p.acc[off + sh.to[j]] = w;
      p.kept_idx[off + sh.to[j]] = q;
    }
    constexpr int U = 4;
    using Piece = typename std::conditional<PIECE == 16, uint4, uint2>::type;
    for (int x0 = threadIdx.x; x0 < pieces; x0 += U * NT) {
      Piece v[U];
      Piece* dst[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int x = x0 + i * NT;
        dst[i] = nullptr;
        if (x >= pieces) continue;
        const int j = x / first[4], q = x % first[4], t = (q >= first[1]) + (q >= first[2]) + (q >= first[3]);
        const int bytes = t == 0 ? p.rows[0].bytes : t == 1 ? p.rows[1].bytes : t == 2 ? p.rows[2].bytes : p.rows[3].bytes;
        const int begin = t == 0 ? 0 : t == 1 ? first[1] : t == 2 ? first[2] : first[3];
        char* base = (char*)(t == 0 ? p.rows[0].base : t == 1 ? p.rows[1].base : t == 2 ? p.rows[2].base : p.rows[3].base);
        v[i] = *reinterpret_cast<const Piece*>(base + (off + sh.from[j]) * bytes + (q - begin) * PIECE);
        dst[i] = reinterpret_cast<Piece*>(base + (off + sh.to[j]) * bytes + (q - begin) * PIECE);
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (dst[i]) *dst[i] = v[i];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) p.kept_len[u] = c;
}

template <int NT, int kKeys, int PIECE>
__global__ void __launch_bounds__(NT) evict_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t stays[];  // a bit per row
  __shared__ EvictShared sh;
  pdl_wait();
  pdl_go();
  const int u = p.layer < 0 ? blockIdx.x : (blockIdx.x / p.Hkv * p.L + p.layer) * p.Hkv + blockIdx.x % p.Hkv;
  const int len = p.kept_len[u], limit = max(0, p.limit[u]);
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  if (off < 0 || end > p.capacity || off + len > end || len > p.max_rows || len <= limit) return;
  if (len <= kKeys * NT)
    evict_segment<NT, kKeys, PIECE, true>(p, sh, stays, u, off, len, limit);
  else
    evict_segment<NT, kKeys, PIECE, false>(p, sh, stays, u, off, len, limit);
}

}  // namespace

int launch_evict(const madakv_config& c, int layer, const int32_t* limit, int recent, float* acc, int32_t* kept_idx,
                 const int64_t* seg_off, int32_t* kept_len, int64_t capacity, const RowArray (&rows)[4], cudaStream_t st) {
  EvictParams p = {limit, acc, kept_idx, seg_off, kept_len, capacity, {rows[0], rows[1], rows[2], rows[3]}, recent, c.n_layers, c.n_kv_heads, layer, 0};
  const int n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  int64_t longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  if (longest > kMaxRows) return MADAKV_EUNSUPPORTED;
  const int64_t mean = capacity / ((int64_t)c.batch * c.n_layers * c.n_kv_heads);
  if (capacity < longest) longest = capacity;
  p.max_rows = (int)longest;
  const size_t smem = (size_t)(longest + 31) / 32 * 4;
  bool wide = true;
  for (const RowArray& r : rows) wide = wide && r.bytes % 16 == 0;
  auto go = [&](auto kernel, int threads) {
    // (the kernel's bound belongs to the process, and calls of other configs may come from other threads: the same for all)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRows / 8) != cudaSuccess) return (int)MADAKV_ECUDA;
    launch_pdl(kernel, dim3((unsigned)n_sel), dim3(threads), smem, st, p);
    return launch_status();
  };
  // keys of segments up to half as long again as the mean in registers
  const int64_t most = mean + mean / 2;
  if (most <= 128 * 24 && n_sel > 2 * 148) return wide ? go(evict_kernel<128, 24, 16>, 128) : go(evict_kernel<128, 24, 8>, 128);
  if (most <= 4096) return wide ? go(evict_kernel<512, 8, 16>, 512) : go(evict_kernel<512, 8, 8>, 512);
  return wide ? go(evict_kernel<1024, 12, 16>, 1024) : go(evict_kernel<1024, 12, 8>, 1024);
}

}  // namespace madakv
