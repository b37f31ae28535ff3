// Eviction while decoding: a segment with more rows than its limit keeps those of the largest accumulated weight, in place.
//
//   which   the c-th largest of the order (protected, weight, lower row first) is found digit by digit from the top, with a histogram of
//           the rows that agree on the digits so far; a row stays if its place in that order is above or at it
//   where   rows [0, c) that go are holes, rows from c on that stay fill them, the j-th hole with the j-th such row: no row that is
//           read is written, so all moves run at once, and only those rows move (a stable compaction would move half the segment to
//           evict one row)
// One block per segment.
#include <limits.h>

#include "common.cuh"

namespace madakv {
namespace {

constexpr int NT = 512;
constexpr int kBits = 11, kBins = 1 << kBits;
constexpr int kList = 2048;             // rows moved between two barriers
constexpr int kMaxRows = 3 << 19;       // longest segment: a bit per row lies in shared memory
constexpr uint32_t kSafe = 0xffffffffu; // in the place of a protected row's weight

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

// Sum over the block of one int per thread; and the sum of those before the thread.
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
  int total = 0, base = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    if (w == warp) base = total;
    total += warp_sums[w];
  }
  if (before) *before = base + x - v;
  return total;
}

// One 64-bit number per row, larger for a row that goes earlier into the kept set; all different.
__device__ __forceinline__ uint64_t place(uint32_t key, int row) { return ((uint64_t)key << 32) | (uint32_t)~row; }

template <int PIECE>
__global__ void __launch_bounds__(NT) evict_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t stays[];  // a bit per row
  __shared__ int hist[kBins];
  __shared__ int warp_sums[NT / 32];
  __shared__ int s_bin, s_above, s_in;
  __shared__ int to[kList], from[kList];
  pdl_wait();
  pdl_go();
  const int u = p.layer < 0 ? blockIdx.x : (blockIdx.x / p.Hkv * p.L + p.layer) * p.Hkv + blockIdx.x % p.Hkv;
  const int len = p.kept_len[u], limit = max(0, p.limit[u]);
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  if (off < 0 || end > p.capacity || off + len > end || len > p.max_rows || len <= limit) return;
  const float* acc = p.acc + off;
  const int32_t* pos = p.kept_idx + off;
  // protected rows: those of the `recent` newest positions
  int newest = INT_MIN;
  for (int r = threadIdx.x; r < len; r += NT) newest = max(newest, pos[r]);
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) newest = max(newest, __shfl_xor_sync(0xffffffffu, newest, o));
  if (threadIdx.x % 32 == 0) warp_sums[threadIdx.x / 32] = newest;
  __syncthreads();
  for (int w = 0; w < NT / 32; ++w) newest = max(newest, warp_sums[w]);
  const int64_t young = (int64_t)newest - p.recent;
  auto key_of = [&](int r) { return pos[r] > young ? kSafe : psi_key(acc[r]); };
  int safe = 0;
  for (int r = threadIdx.x; r < len; r += NT) safe += pos[r] > young;
  safe = block_sum(safe, warp_sums);
  const int c = max(limit, safe);
  if (c >= len) return;
  // the place of the last row that stays (c = 0: none does)
  uint64_t last = ~0ull;
  if (c > 0) {
    uint64_t prefix = 0;
    int need = c;
    uint64_t known = 0;  // the bits that the digits so far have settled
    for (int shift = 64 - kBits;; known = ~0ull << shift, shift = shift > kBits ? shift - kBits : 0) {
      for (int b = threadIdx.x; b < kBins; b += NT) hist[b] = 0;
      __syncthreads();
      for (int r = threadIdx.x; r < len; r += NT) {
        const uint64_t x = place(key_of(r), r);
        if (((x ^ prefix) & known) == 0) atomicAdd(&hist[(x >> shift) & (kBins - 1)], 1);
      }
      __syncthreads();
      // bins from the top: the one in which the count reaches `need`
      constexpr int PER = kBins / NT;
      int mine[PER], sum = 0, before;
#pragma unroll
      for (int j = 0; j < PER; ++j) sum += mine[j] = hist[kBins - 1 - (threadIdx.x * PER + j)];
      block_sum(sum, warp_sums, &before);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (before < need && before + mine[j] >= need) {
          s_bin = kBins - 1 - (threadIdx.x * PER + j);
          s_above = before;
          s_in = mine[j];
        }
        before += mine[j];
      }
      __syncthreads();
      prefix |= (uint64_t)s_bin << shift;  // (the last digit overlaps the one before it; what the two share agrees)
      need -= s_above;
      if (need == s_in || shift == 0) break;  // all rows of the bin stay
    }
    last = prefix;
  }
  // a bit per row: it stays
  const int words = (len + 31) / 32;
  for (int w = threadIdx.x / 32; w < words; w += NT / 32) {
    const int r = w * 32 + threadIdx.x % 32;
    const uint32_t bits = __ballot_sync(0xffffffffu, c > 0 && r < len && place(key_of(r), r) >= last);
    if (threadIdx.x % 32 == 0) stays[w] = bits;
  }
  __syncthreads();
  // every thread's words, one stretch each: holes below c, rows to move from c on
  const int per = (words + NT - 1) / NT, w0 = min(words, (int)threadIdx.x * per), w1 = min(words, w0 + per);
  auto below = [&](int w) { return w * 32 + 32 <= c ? ~0u : w * 32 >= c ? 0u : (1u << (c - w * 32)) - 1u; };
  int holes = 0, movers = 0, hole0, mover0;
  for (int w = w0; w < w1; ++w) {
    holes += __popc(~stays[w] & below(w));
    movers += __popc(stays[w] & ~below(w));
  }
  block_sum(holes, warp_sums, &hole0);
  const int n = block_sum(movers, warp_sums, &mover0);
  for (int j0 = 0; j0 < n; j0 += kList) {
    int a = hole0, b = mover0;
    for (int w = w0; w < w1; ++w) {
      for (uint32_t bits = ~stays[w] & below(w); bits; bits &= bits - 1, ++a)
        if (a >= j0 && a < j0 + kList) to[a - j0] = w * 32 + __ffs(bits) - 1;
      for (uint32_t bits = stays[w] & ~below(w); bits; bits &= bits - 1, ++b)
        if (b >= j0 && b < j0 + kList) from[b - j0] = w * 32 + __ffs(bits) - 1;
    }
    __syncthreads();
    const int m = min(kList, n - j0);
    for (int j = threadIdx.x; j < m; j += NT) {
      p.acc[off + to[j]] = p.acc[off + from[j]];
      p.kept_idx[off + to[j]] = p.kept_idx[off + from[j]];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int pieces = p.rows[t].bytes / PIECE;
      char* base = (char*)p.rows[t].base + off * p.rows[t].bytes;
      for (int x = threadIdx.x; x < m * pieces; x += NT) {
        const int j = x / pieces, at = x % pieces * PIECE;
        char* dst = base + (int64_t)to[j] * p.rows[t].bytes + at;
        const char* src = base + (int64_t)from[j] * p.rows[t].bytes + at;
        if constexpr (PIECE == 16)
          *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
        else
          *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(src);
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) p.kept_len[u] = c;
}

}  // namespace

int launch_evict(const madakv_config& c, int layer, const int32_t* limit, int recent, float* acc, int32_t* kept_idx,
                 const int64_t* seg_off, int32_t* kept_len, int64_t capacity, const RowArray (&rows)[4], cudaStream_t st) {
  EvictParams p = {limit, acc, kept_idx, seg_off, kept_len, capacity, {rows[0], rows[1], rows[2], rows[3]}, recent, c.n_layers, c.n_kv_heads, layer, 0};
  const int n_sel = (layer < 0 ? c.batch * c.n_layers : c.batch) * c.n_kv_heads;
  int64_t longest = c.max_seq_len + (int64_t)c.max_new_tokens;
  if (longest > kMaxRows) return MADAKV_EUNSUPPORTED;
  if (capacity < longest) longest = capacity;
  p.max_rows = (int)longest;
  const size_t smem = (size_t)(longest + 31) / 32 * 4;
  bool wide = true;
  for (const RowArray& r : rows) wide = wide && r.bytes % 16 == 0;
  auto kernel = wide ? evict_kernel<16> : evict_kernel<8>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return MADAKV_ECUDA;
  launch_pdl(kernel, dim3((unsigned)n_sel), dim3(NT), smem, st, p);
  return launch_status();
}

}  // namespace madakv
