// What the kernels of prompt attention and of attention over drafted trees share: the parameters of a call, the work items that
// blocks take, rows and their visible keys, results and their merge where the keys of a row are shared out.
//
// A work item is a tile of rows of one KV head and the stretch of keys that they attend to. Its rows are (query, head of the group)
// pairs, query by query, so that the g heads of a group share every key that is read, whatever g is, and a few queries fill a tile.
#pragma once

#include "common.cuh"

namespace madakv {

constexpr int kAttnSlots = 32;  // shares of a row's keys at most
constexpr int kMaxGroup = 64;

struct AttnParams {
  // queries and results: element strides of (sequence, head, query), and for a tree of the layer
  const void* q;
  void* out;
  madakv_strides sq, so;
  float* lse_out;
  int B, L, Hq, Hkv, g, layer, causal, w;
  int64_t q_rows;  // queries a sequence (padded) or all queries (packed); nodes of a tree
  float scale2;    // softmax scale * log2(e)
  // prompt: keys and values of one layer, where sequences begin (null: sequences have a dimension of their own), their lengths
  const void *k, *v;
  madakv_strides sk, sv;
  int64_t k_rows;
  const int64_t *q_off, *k_off;
  const int32_t *q_len, *seq_len;
  int n_max;
  void* q_win;
  float* lse_win;
  int32_t* win_len;  // null, or: windows keep the rows of earlier queries, and these are the keys up to which they are complete
  // tree: the drafted rows stand in k and v, the ragged cache here
  const void *k_c, *v_c;
  const int64_t* seg_off;
  const int32_t* kept_len;
  int64_t capacity;
  const uint64_t* mask;
  const int32_t* n_nodes;
  int n_sel;  // (sequence, layer, KV head)s of the call
  // shares of the keys: partial results [item, slot, row of the tile, D] and their (max, in the logarithm to base 2, sum) [item, slot, row]
  float* part;
  float2* part_ml;
  int part_rows;       // rows that there is room for
  int slots, least_tiles;
  int tile_keys;       // keys of a tile
  int* order;          // tree, null or: the number of items that have rows, then those items, the longest first
  int tile_q;          // queries of an item
  int tile_rows;       // rows of an item at most
  int g_inverse;       // 2^16 / g, rounded up
  int wide_q, wide_out;  // rows begin on 32-byte boundaries
  int copy_out;          // tensor copies can write whole tiles of results
  int64_t n_items;     // items (without slots) at most; items times slots are fewer than 2^31
  int q_tiles;         // tree: tiles of a unit's rows
  void* ws;
  int hold_copies;        // test of waits that run out: no tile of keys is copied
  long long wait_clocks;  // bound of a wait
};

// One work item. Row r of its tile is query q0 + r / g, head r % g of the group.
struct AttnItem {
  int b, h, q0, n_q;        // sequence, KV head, first query, queries of the sequence
  int n_keys;               // prompt: keys of the sequence; tree: rows of the segment
  int shift;                // prompt: position of query i is i + shift
  int unit;                 // tree
  int nodes;                // tree: nodes of the sequence
  int64_t q_at, out_at;     // elements: query 0, first head of the group
  int64_t lse_at;           // row: the same in lse_out; a head further is q_rows on
  int64_t k_at, v_at;       // elements: prompt: key 0 of the head; tree: node 0 of the head
  int64_t key_row;          // first key: prompt: row of the token dimension; tree: row of the cache
};

// Row r of a tile (fewer than 512) belongs to query r / g: exact, because r times what the inverse is rounded up by stays below 2^16.
__device__ __forceinline__ int group_of(const AttnParams& p, int r) { return r * p.g_inverse >> 16; }

// ---- prompts -------------------------------------------------------------------------------------------------------------
// Keys and queries of sequence b. Lengths outside their range are used as the nearest bound; a stretch of rows that is not one (its
// end before its start, or behind the last row) counts as empty.
__device__ __forceinline__ int stretch(const int64_t* off, int b, int64_t rows, int most) {
  const int64_t a = off[b], e = off[b + 1];
  return a < 0 || e < a || e > rows ? 0 : (int)min(e - a, (int64_t)most);
}
__device__ __forceinline__ int prompt_keys(const AttnParams& p, int b) {
  return p.k_off ? stretch(p.k_off, b, p.k_rows, p.n_max) : max(0, min(p.seq_len[b], (int)min((int64_t)p.n_max, p.k_rows)));
}
__device__ __forceinline__ int prompt_queries(const AttnParams& p, int b, int keys) {
  const int most = (int)min(p.q_rows, (int64_t)p.n_max);
  return p.q_off ? stretch(p.q_off, b, p.q_rows, most) : max(0, min(p.q_len ? p.q_len[b] : keys, most));
}

// Items of a prompt call: tiles of the sequences' queries, the last tiles (those with the most keys under a causal mask) first, so
// that the long items are under way when the short ones fill the gaps. All lanes of a warp call this for item i and get the
// same answer; false: there are no more items. Level t holds the sequences with more than t tiles; at_least(t) counts the tiles of
// level t and above.
__device__ __forceinline__ bool find_prompt_tile(const AttnParams& p, unsigned i, int& b_out, int& tile_out) {
  const int lane = threadIdx.x & 31;
  auto tiles_of = [&](int b) {
    if (b >= p.B) return 0;
    return (prompt_queries(p, b, p.q_off || p.q_len ? 0 : prompt_keys(p, b)) + p.tile_q - 1) / p.tile_q;
  };
  if (p.B == 1) {
    const int n = tiles_of(0);
    b_out = 0;
    tile_out = n - 1 - (int)i;
    return i < (unsigned)n;
  }
  const int first = tiles_of(lane);
  auto at_least = [&](int t) {
    unsigned n = (unsigned)max(0, first - t);
    for (int b = lane + 32; b < p.B; b += 32) n += (unsigned)max(0, tiles_of(b) - t);
    return __reduce_add_sync(0xffffffffu, n);
  };
  if (i >= at_least(0)) return false;
  int lo = 0, hi = ((int)min(p.q_rows, (int64_t)p.n_max) + p.tile_q - 1) / p.tile_q;  // at_least(lo) > i >= at_least(hi) = 0
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (at_least(mid) > i) lo = mid; else hi = mid;
  }
  int r = (int)(i - at_least(lo + 1));
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const unsigned in = __ballot_sync(0xffffffffu, (b0 ? tiles_of(b0 + lane) : first) > lo);
    if (r < __popc(in)) {
      unsigned left = in;
      for (; r > 0; --r) left &= left - 1;
      b_out = b0 + __ffs(left) - 1;
      tile_out = lo;
      return true;
    }
    r -= __popc(in);
  }
  return false;
}

__device__ __forceinline__ bool prompt_item(const AttnParams& p, unsigned i, AttnItem& it) {
  int tile;
  it.h = (int)(i % (unsigned)p.Hkv);
  if (!find_prompt_tile(p, i / (unsigned)p.Hkv, it.b, tile)) return false;
  const int b = it.b;
  it.n_keys = prompt_keys(p, b);
  it.n_q = prompt_queries(p, b, it.n_keys);
  it.q0 = tile * p.tile_q;
  it.shift = it.n_keys - it.n_q;
  const int64_t qb = p.q_off ? 0 : b, kb = p.k_off ? 0 : b, qr = p.q_off ? p.q_off[b] : 0;
  it.key_row = p.k_off ? p.k_off[b] : 0;
  it.q_at = qb * p.sq.batch + (int64_t)it.h * p.g * p.sq.head + qr * p.sq.token;
  it.out_at = qb * p.so.batch + (int64_t)it.h * p.g * p.so.head + qr * p.so.token;
  it.lse_at = ((qb * p.L + p.layer) * p.Hq + (int64_t)it.h * p.g) * p.q_rows + qr;
  it.k_at = kb * p.sk.batch + (int64_t)it.h * p.sk.head + it.key_row * p.sk.token;
  it.v_at = kb * p.sv.batch + (int64_t)it.h * p.sv.head + it.key_row * p.sv.token;
  it.unit = it.nodes = 0;
  return true;
}

// A window without all of its rows, in win_len. (~n: that of a prompt of n keys, which eviction has gone on from.)
constexpr int32_t kNoWindow = INT32_MIN;

// The proxy tokens' rows that are none of the call's queries: log-sum-exp -inf, query 0. `threads` threads of every block. Where windows keep earlier
// rows (win_len) those of sequences with fewer new queries than proxy tokens have been moved by the launch before.
template <int ROW_BYTES>
__device__ __forceinline__ void fill_window(const AttnParams& p, int thread, int threads) {
  if (!p.lse_win && !p.q_win) return;
  for (int x = blockIdx.x; x < p.B * p.Hq; x += gridDim.x) {
    const int b = x / p.Hq, keys = !p.win_len && (p.q_off || p.q_len) ? 0 : prompt_keys(p, b), queries = prompt_queries(p, b, keys);
    int none = max(0, p.w - queries);
    if (p.win_len) {
      const bool whole = queries >= min(p.w, keys);
      if (thread == 0 && x % p.Hq == 0 && (whole || queries > 0)) {
        int32_t* held = p.win_len + b * p.L + p.layer;
        *held = whole || (p.causal && *held == keys - queries) ? keys : kNoWindow;
      }
      if (!whole) none = 0;
    }
    const int64_t row = (((int64_t)b * p.L + p.layer) * p.Hq + x % p.Hq) * p.w;
    if (p.lse_win)
      for (int r = thread; r < none; r += threads) p.lse_win[row + r] = -INFINITY;
    if (p.q_win)
      for (int r = thread; r < none * (ROW_BYTES / 16); r += threads)
        reinterpret_cast<uint4*>((char*)p.q_win + row * ROW_BYTES)[r] = make_uint4(0, 0, 0, 0);
  }
}

// ---- trees ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool tree_item(const AttnParams& p, unsigned i, AttnItem& it) {
  if (i >= (unsigned)p.n_items) return false;
  const int y = (int)(i / (unsigned)p.q_tiles);
  const int u = p.layer < 0 ? y : (y / p.Hkv * p.L + p.layer) * p.Hkv + y % p.Hkv;
  const int bl = u / p.Hkv, b = bl / p.L, l = bl % p.L;
  it.unit = u;
  it.b = b;
  it.h = u % p.Hkv;
  it.q0 = (int)(i % (unsigned)p.q_tiles) * p.tile_q;
  const int T = (int)p.q_rows;
  it.nodes = it.n_q = p.n_nodes ? max(0, min(p.n_nodes[b], T)) : T;
  // a segment that selection refused, or whose length does not fit its slot, counts as empty, as in decode attention
  const int64_t off = p.seg_off[u], end = p.seg_off[u + 1];
  const int len = p.kept_len[u];
  it.n_keys = off < 0 || end < off || end > p.capacity || len < 0 || off + (int64_t)len > end ? 0 : len;
  it.key_row = it.n_keys ? off : 0;
  it.shift = 0;
  const int64_t bq = b, head = (int64_t)it.h * p.g;
  it.q_at = bq * p.sq.batch + l * p.sq.layer + head * p.sq.head;
  it.out_at = bq * p.so.batch + l * p.so.layer + head * p.so.head;
  it.lse_at = ((int64_t)bl * p.Hq + head) * T;
  it.k_at = bq * p.sk.batch + l * p.sk.layer + it.h * p.sk.head;
  it.v_at = bq * p.sv.batch + l * p.sv.layer + it.h * p.sv.head;
  return true;
}
// The nodes that node t of the item's sequence sees.
__device__ __forceinline__ uint64_t node_mask(const AttnParams& p, const AttnItem& it, int t) {
  const uint64_t there = it.nodes >= 64 ? ~0ull : (1ull << it.nodes) - 1;
  return p.mask[(int64_t)it.b * p.q_rows + t] & there;
}

// ---- shares of the keys --------------------------------------------------------------------------------------------------
// Tiles of keys that any row of the item sees; a tree's own nodes are one behind the segment's.
template <bool kTree>
__device__ __forceinline__ int item_tiles(const AttnParams& p, const AttnItem& it) {
  const int seen = kTree || !p.causal ? it.n_keys : max(0, min(it.n_keys, min(it.q0 + p.tile_q, it.n_q) + it.shift));
  return (seen + p.tile_keys - 1) / p.tile_keys + (kTree ? 1 : 0);
}
// Shares of `tiles` tiles of keys that get work, and the tiles of share x: two each at least. Share 0 always takes part.
__device__ __forceinline__ int shares_of(const AttnParams& p, int tiles) { return tiles < p.least_tiles ? 1 : min(p.slots, (tiles + 1) / 2); }
__device__ __forceinline__ void share_tiles(int nb, int tiles, int x, int& begin, int& end) {
  begin = tiles * x / nb;  // (at most 2^25 tiles, 2^5 shares)
  end = tiles * (x + 1) / nb;
}

// Result of a row: o over its sum of weights l; a row without weight gets 0, one whose sum is not a number NaN.
__device__ __forceinline__ float row_factor(float l) { return l > 0.f ? 1.f / l : (l == l ? 0.f : l); }
__device__ __forceinline__ float row_lse(float m2, float l) {
  return l > 0.f ? (m2 + log2f(l)) * 0.6931471805599453f : (l == l ? -INFINITY : l);
}
// Log-sum-exp of query t, head j of the item, to where the caller wants it; true: the query is a proxy token whose row `win` is.
__device__ __forceinline__ bool store_row_lse(const AttnParams& p, const AttnItem& it, int t, int j, float lse, int64_t& win) {
  if (p.lse_out) p.lse_out[it.lse_at + j * p.q_rows + t] = lse;
  const int r = t - it.n_q + p.w;  // row of the window
  if ((!p.lse_win && !p.q_win) || r < 0) return false;
  win = (((int64_t)it.b * p.L + p.layer) * p.Hq + it.h * p.g + j) * p.w + r;
  if (p.lse_win) p.lse_win[win] = lse;
  return p.q_win != nullptr;
}

// ---- host ----------------------------------------------------------------------------------------------------------------
// The items of a call whose tiles have p.tile_q queries. (Packed sequences: a tile more for each than their rows fill.)
inline void attn_items(AttnParams& p, bool tree) {
  if (tree) {
    p.q_tiles = (int)((p.q_rows + p.tile_q - 1) / p.tile_q);
    p.n_items = (int64_t)p.n_sel * p.q_tiles;
    return;
  }
  const int64_t longest = p.q_rows < p.n_max ? p.q_rows : p.n_max, tiles = (longest + p.tile_q - 1) / p.tile_q * p.B;
  const int64_t packed = p.q_rows / p.tile_q + p.B;
  p.n_items = (p.q_off && packed < tiles ? packed : tiles) * p.Hkv;
}
// What a kernel takes, in us: a tile of keys for rows of half an item and of a whole one, an item beside its tiles; and the tiles from
// which it shares out keys.
struct AttnCost {
  float half, whole, item;
  int least;
};
// Shares of the keys: the number that a call should end first with, by the longest sequence or the mean segment, and no more than there is
// room for their results. Blocks go through the shares' items in rounds; shares cost a launch that joins them, and their results are
// written and read in fp32. (28 / 4 heads: 1000 tokens 23.7 us whole and 41.8 in two shares, of which there are more than SMs; 72 tokens on
// 8192 keys 116 us whole, 31 in 8 shares, 39 in 18.)
inline void attn_slots(AttnParams& p, const madakv_config& c, bool tree, int tile_keys, AttnCost cost) {
  constexpr float kJoin = 6.2f, kMegabyte = 0.55f;  // us
  const int64_t units = (int64_t)c.batch * c.n_layers * c.n_kv_heads, longest = (int64_t)c.max_seq_len + c.max_new_tokens;
  const int64_t keys = !tree ? (p.k_rows < p.n_max ? p.k_rows : p.n_max) : p.capacity / units < longest ? p.capacity / units : longest;
  const int64_t queries = p.q_rows < p.n_max ? p.q_rows : p.n_max;
  p.tile_rows = (int)(p.tile_q < p.q_rows ? p.tile_q : p.q_rows) * p.g;
  const float most = (float)(keys / tile_keys + 1), mean = most - (!tree && p.causal ? (float)(queries < keys ? queries : keys) / (2 * tile_keys) : 0.f);
  const float tile = p.q_rows > p.tile_q / 2 ? cost.whole : cost.half;
  const int64_t by_room = p.n_items ? p.part_rows / (p.n_items * p.tile_rows) : 1;
  float best = 0.f;
  p.slots = 1;
  for (int s = 1; s <= kAttnSlots && (s == 1 || (s <= by_room && 2 * s <= most + 1.f && most >= (float)cost.least)); ++s) {
    const float rounds = (float)((p.n_items * s + 147) / 148), one = most / s * tile + cost.item, all = rounds * (mean / s * tile + cost.item);
    const float join = s == 1 ? 0.f : kJoin + kMegabyte * 1e-6f * (float)(p.n_items * s * p.tile_rows) * (float)c.head_dim * 4.f;
    const float t = (one > all ? one : all) + join;
    if (s == 1 || t < best) best = t, p.slots = s;
  }
  p.least_tiles = cost.least;
  p.tile_keys = tile_keys;
  p.part = reinterpret_cast<float*>((char*)p.ws + ws_layout(c).decode_off);
  p.part_ml = reinterpret_cast<float2*>(p.part + (int64_t)p.part_rows * c.head_dim);
}

int launch_window_move(const AttnParams& p, const madakv_config& c, cudaStream_t st);  // ahead of a call whose windows keep earlier rows
int launch_attn_plain(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st);
int launch_attn_join(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st);  // behind a call with shares
int launch_attn_split(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st);
int launch_attn_tc(const AttnParams& p, const madakv_config& c, bool tree, cudaStream_t st);  // -1: its copies cannot take these strides

}  // namespace madakv
