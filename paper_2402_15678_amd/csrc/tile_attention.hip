// Attention of many query rows over the same keys, as tiles of a dense product: whole prompts (packed rows, causal), batches whose
// sequences share a prefix of the paged cache, and rows that see a window of it and its first few tokens.
//
// o_r = sum_j p_rj v_j / sum_j p_rj with p_rj = 2^(c s_rj - m_r), s_rj = q_r . k_j, c = log2(e) / sqrt(head_dim), in one pass over the
// keys with a running reference m_r.  The G query heads of a KV head are stacked: row r of the stack is query head r % G of token
// r / G, so a tile of rows reads the keys of its KV head once for all of them.
//
//  * tile_mfma_kernel   fp16, head_dim 64 or 128, dense rows or pages of 16 tokens: 16x16x32 matrix instructions, keys staged in
//    LDS for all the waves of a workgroup.
//  * tile_f32_kernel    every other type, head_dim and block size: 16x16x4 fp32 matrix instructions.
//  * prefix_plan_kernel, prefix_merge_kernel   the work list of a shared-prefix call, and the sum of its parts.
//  * window_plan_kernel, window_merge_kernel   the same of a windowed call.
#include "launch.h"
#include "tune.h"
#include "../../include/minions_verify.h"

#include <mutex>

namespace mn {

constexpr float LOG2E_T = 1.4426950408889634f;
constexpr int TKEYS = 64;              // ranges of keys begin at multiples of it
constexpr int PAGE = 16;               // tokens per block that it reads
constexpr int NO_LIMIT = 1 << 29;      // an item whose rows all see every key of its range
constexpr float LAZY = 6.f;            // the reference moves when a score exceeds it by 2^6
// From here on the rounding of c s - m alone would be an exponent of the size that the references are there to keep away (half a unit
// at 2^24, 32 at 2^29, where a probability leaves the fp16 range).  Such a row's scores are taken less its reference ahead of the
// exponentials, from the rounded product, so that the largest one is 0, and its reference follows its scores tile by tile.
constexpr float FAR = 0x1p24f;

// One tile of work: stack rows [rbase, R) (as many as a workgroup holds) of the tokens from m0 on against the keys [key0, key_end).
// Row r sees the keys up to ctx + r / G.
struct Item {
  int m0, R, rbase, key0, key_end, ctx, seq, slot;
};

// Division by a number that is mostly a power of two (a uniform branch in place of thirty instructions).
struct Divide {
  int d, shift;
  __device__ __forceinline__ explicit Divide(int d_) : d(d_), shift((d_ & (d_ - 1)) == 0 ? 31 - __clz(d_) : -1) {}
  __device__ __forceinline__ int operator()(int x) const { return shift >= 0 ? x >> shift : (int)((uint32_t)x / (uint32_t)d); }
};

// Sum over the lanes of max(0, n(b) - level) for b < B.
template <typename F>
__device__ __forceinline__ int tiles_from(int level, int B, F n) {
  int s = 0;
  for (int b = threadIdx.x & 63; b < B; b += 64) s += max(0, n(b) - level);
  return __builtin_amdgcn_readfirstlane(wave_sum_i(s));
}

// Tile t of a packed batch whose sequence b has n(b) tiles.  Order: last tiles first (a causal tile's work grows with its number),
// so the longest ones start first and the short ones fill the gaps.  Level `tile` and the sequence are found by counting how
// many tiles lie at or above a level.  0 <= t < the sum of n(b), and n(b) <= max_tiles.
template <typename F>
__device__ __forceinline__ void find_tile(int t, int B, int max_tiles, F n, int& seq, int& tile) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = max_tiles, above = 0;         // tiles at levels >= lo: more than t; >= hi: `above`, t at most
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, c = tiles_from(mid, B, n);
    if (c > t) lo = mid;
    else { hi = mid; above = c; }
  }
  tile = lo;
  int ord = t - above;
  seq = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const bool has = b0 + lane < B && n(b0 + lane) > lo;
    const uint64_t ballot = __ballot(has);
    const int c = __popcll(ballot);
    if (ord < c) {
      seq = b0 + __ffsll((unsigned long long)__ballot(has && __popcll(ballot & ((1ull << lane) - 1)) == ord)) - 1;
      break;
    }
    ord -= c;
  }
}

// The same for up to 64 sequences, lane b holding sequence b's number: 64 levels are counted at once, one per lane.
__device__ __forceinline__ void find_tile_lanes(int t, int B, int max_tiles, int own, int& seq, int& tile) {
  const int lane = threadIdx.x & 63;
  int lo = 0, above = 0, step = 1;
  while ((long)step * 64 < max_tiles) step <<= 6;
  for (;;) {                                     // level lo: more than t tiles at or above it; lo + 64 step: t at most
    const int level = lo + lane * step;
    int c = 0;
    for (int b = 0; b < B; ++b) c += max(0, __builtin_amdgcn_readlane(own, b) - level);
    const int at = 63 - __clzll((unsigned long long)__ballot(c > t));
    lo += at * step;
    if (at < 63) above = __builtin_amdgcn_readlane(c, at + 1);
    if (step == 1) break;
    step >>= 6;
  }
  tile = lo;
  const bool has = own > lo;
  const uint64_t ballot = __ballot(has);
  seq = __ffsll((unsigned long long)__ballot(has && __popcll(ballot & ((1ull << lane) - 1)) == t - above)) - 1;
}

// The prompt's item of this workgroup.  Lengths come from the device; those that do not fit the launch (which the host's sized)
// leave the whole call undone: rows outside the packed ones, another number of tiles, or a sequence longer than the host's longest,
// for which neither the search nor the block table's rows have room.  s_n: room for a number per sequence.
template <int ROWS>
__device__ __forceinline__ bool prompt_item(const TileArgs& a, int t, const Divide& by, int32_t* s_n, Item& it) {
  const int lane = threadIdx.x & 63, G = by.d;
  int r0 = 0, r1 = 0;
  auto tiles = [&](int b) {                      // -1: does not fit
    r0 = a.seq_rows[b];
    r1 = a.seq_rows[b + 1];
    if (r0 < 0 || r1 < r0 || r1 > a.M || r1 - r0 > a.longest) return -1;
    return (int)(((long)(r1 - r0) * G + ROWS - 1) / ROWS);
  };
  int own = 0;
  if (a.B <= 64) {
    if (lane < a.B) own = tiles(lane);
  } else {
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) s_n[b] = tiles(b);
    __syncthreads();
  }
  auto n = [&](int b) { return a.B <= 64 ? own : s_n[b]; };
  bool bad = false;
  for (int b = lane; b < a.B; b += 64) bad |= n(b) < 0;
  const int total = tiles_from(0, a.B, n);
  if (__any(bad) || total != a.n_tiles) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, MN_DEV_SPEC_LEN);
    return false;
  }
  int seq, tile;
  if (a.B <= 64) find_tile_lanes(t, a.B, a.max_tiles, own, seq, tile);
  else find_tile(t, a.B, a.max_tiles, n, seq, tile);
  seq = __builtin_amdgcn_readfirstlane(seq);
  tile = __builtin_amdgcn_readfirstlane(tile);
  int row0, row1;
  if (a.B <= 64) {                               // (the offsets are in the lanes)
    row0 = __builtin_amdgcn_readlane(r0, seq);
    row1 = __builtin_amdgcn_readlane(r1, seq);
  } else {
    row0 = a.seq_rows[seq];
    row1 = a.seq_rows[seq + 1];
  }
  const int len = row1 - row0;
  it.m0 = row0; it.R = len * G; it.rbase = tile * ROWS; it.key0 = 0; it.ctx = 0; it.seq = seq; it.slot = -1;
  it.key_end = min(len, by(min(it.R, it.rbase + ROWS) - 1) + 1);
  return true;
}

// What takes part in a shared-prefix call, for up to 64 sequences: lane b has sequence b's rows, its first row, and the ranges and row
// tiles of its own keys.  Lengths that do not add up to the host's rows, or a run longer than its longest one, disable the batch; a
// context outside [prefix_len, max_ctx) its sequence.  (Larger batches: prefix_plan_kernel.)
struct Share {
  int q, row0, ctx, ranges, tiles, flags;
};
__device__ __forceinline__ Share lane_share(const PrefixBatch& p) {
  const int b = threadIdx.x & 63;
  Share s{0, 0, 0, 0, 0, 0};
  bool off = false;
  if (b < p.B) {
    const int k = p.spec_len[b];
    s.ctx = p.ctx_lens[b];
    off = k < 0 || k >= p.max_q;
    s.q = off ? 0 : k + 1;
  }
  const int incl = wave_scan_i(s.q);
  s.row0 = incl - s.q;
  if (__any(off) || __builtin_amdgcn_readlane(incl, 63) != p.M) {
    s.q = 0;
    s.flags = MN_DEV_SPEC_LEN;
  } else if (s.q > 0) {
    if (s.ctx < p.prefix_len || (long)s.ctx + s.q > p.max_ctx) {
      s.flags = MN_DEV_CTX;
    } else {
      s.ranges = (s.ctx + s.q - p.prefix_len + p.chunk - 1) / p.chunk;
      s.tiles = (p.G * s.q + p.tile_rows - 1) / p.tile_rows;
    }
  }
  return s;
}

// Item t of the sequences' own keys.
__device__ __forceinline__ bool own_item(const TileArgs& a, int t, Item& it) {
  if (a.items) {
    const int4 x = reinterpret_cast<const int4*>(a.items)[2 * t], y = reinterpret_cast<const int4*>(a.items)[2 * t + 1];
    it = Item{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    return it.R > 0;
  }
  const Share s = lane_share(a.batch);
  const int incl = wave_scan_i(s.ranges * s.tiles), first = incl - s.ranges * s.tiles;
  if (t == 0 && threadIdx.x < 64 && (int)blockIdx.x == a.B && s.flags && a.status) atomicOr(a.status, s.flags);
  const uint64_t mine = __ballot(t >= first && t < incl);
  if (mine == 0) return false;
  const int b = __ffsll((unsigned long long)mine) - 1;
  const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
  const int at = t - of(first), ranges = of(s.ranges), rt = at / ranges, k0 = a.batch.prefix_len + (at - rt * ranges) * a.batch.chunk;
  it.ctx = of(s.ctx);
  it.m0 = of(s.row0); it.R = a.batch.G * of(s.q); it.rbase = rt * a.batch.tile_rows; it.key0 = k0;
  it.key_end = min(k0 + a.batch.chunk, it.ctx + of(s.q)); it.seq = b; it.slot = a.prefix_slots + at - rt * ranges;
  return true;
}

// The shared part, as streams.  Its work is a line of units: 64 keys of the prefix for one tile of rows of one KV head, the keys of a tile
// one after the other, the tiles of a KV head one after the other.  Stream s takes the units [s * share, (s + 1) * share), which
// are a piece of one tile or the end of one and the beginning of others; every piece is an item, and leaves its part in the
// slot that counts the streams of its tile.  With as many streams as workgroups fit the chip at once all of them end together,
// whatever the number of tiles: 64 x 9 rows of 64/8 heads behind 8192 keys are 36 tiles x 8 heads for 512 workgroups.
// Consecutive streams run on one XCD (ids are dealt round-robin), so an XCD's L2 holds the keys of few KV heads.
__device__ __forceinline__ int stream_of(const TileArgs& a, int wg) {
  const int per = a.n_streams >> 3;
  return wg < 8 * per ? (wg & 7) * per + (wg >> 3) : wg;
}
__device__ __forceinline__ bool stream_item(const TileArgs& a, int stream, int& unit, int& kvh, Item& it) {
  const int end = min((stream + 1) * a.share, a.n_units);
  if (unit >= end) return false;
  const int tile = unit / a.prefix_units, from = unit - tile * a.prefix_units, n = min(end - unit, a.prefix_units - from);
  unit += n;
  kvh = tile / a.row_tiles;
  it.m0 = 0; it.R = a.H / a.Hkv * a.M; it.rbase = (tile - kvh * a.row_tiles) * a.batch.tile_rows;
  it.key0 = from * TKEYS; it.key_end = min(a.batch.prefix_len, (from + n) * TKEYS);
  it.ctx = NO_LIMIT; it.seq = 0; it.slot = stream - tile * a.prefix_units / a.share;
  return true;
}

typedef __attribute__((address_space(4))) int32_t const_i32;  // (scalar loads)
__device__ __forceinline__ const const_i32* scalar(const int32_t* p) { return reinterpret_cast<const const_i32*>(reinterpret_cast<uintptr_t>(p)); }

// The sequence whose table row names the shared blocks: the first one whose context holds the prefix (slots emptied by then do not).
__device__ __forceinline__ int first_sharer(const TileArgs& a) {
  if (a.items) return scalar(a.seq_bad)[a.B];
  if (scalar(a.batch.ctx_lens)[0] >= a.batch.prefix_len) return 0;
  const int b = threadIdx.x & 63;
  bool has = false;
  if (b < a.B) has = a.batch.ctx_lens[b] >= a.batch.prefix_len;
  const uint64_t all = __ballot(has);
  return all ? __ffsll((unsigned long long)all) - 1 : 0;
}

// Sequence b's table row, looked at by a workgroup of its own (ahead of an item's keys it was 1 to 2 us of that item): every block id in
// range, and the prefix's entries those that the call reads for all of them.  Rows of a sequence that fails are zeros
// (prefix_merge_kernel).
__device__ __forceinline__ void check_table(const TileArgs& a, int b) {
  const int ctx = scalar(a.batch.ctx_lens)[b], k = scalar(a.batch.spec_len)[b];
  if (ctx < a.batch.prefix_len || k < 0 || (long)ctx + k + 1 > a.batch.max_ctx) return;  // (takes no part)
  const int32_t* first = a.kv.block_tables + (size_t)first_sharer(a) * a.kv.max_blocks_per_seq;
  const int32_t* row = a.kv.block_tables + (size_t)b * a.kv.max_blocks_per_seq;
  const int shared = a.batch.prefix_len / a.kv.block_size, all = (ctx + k) / a.kv.block_size + 1;
  bool bad = false;
  for (int i = threadIdx.x; i < all; i += blockDim.x) bad |= (uint32_t)row[i] >= (uint32_t)a.kv.num_blocks || (i < shared && row[i] != first[i]);
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) {
    a.seq_bad[b] = bad;
    if (bad && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
  }
}

// ---- windows: the row at position p sees the keys p - window + 1 .. p and those below `sinks` ----
// A tile's keys in granules of 16 (a page of the fp16 kernel): the first ones, sg of them, then those from sg + jump on, where the window
// of the tile's first row begins.  Entry i of that list is granule at(i); an item takes the entries [i0, i1).
struct Look {
  int sg, jump, i0, i1;
  __device__ __forceinline__ int at(int i) const { return i + (i >= sg ? jump : 0); }
  __device__ __forceinline__ int entry(int granule) const { return granule - (granule >= sg + jump ? jump : 0); }  // (of a visible one)
};
constexpr int GRAIN = 16;
// Negative where the row sees the e-th key from here on: it has `ahead` keys in front of it, `back` of them behind its window, and `sink` first
// ones.  Signs, and no conditions: sixteen of those at once are more than the scalar registers hold.
__device__ __forceinline__ int in_sight(int e, int ahead, int back, int sink) { return ~(ahead - e) & ((back - e) | (e - sink)); }
constexpr int NO_KEY = 1 << 30;        // behind every position

// The list of the tile whose first and last rows are at the positions p0 and p1.
__device__ __forceinline__ Look look_from(const TileArgs& a, int p0, int p1, int& entries) {
  Look k;
  const int lo = max(0, p0 - a.window + 1), first = lo / GRAIN;
  k.sg = min((a.sinks + GRAIN - 1) / GRAIN, first);
  k.jump = first - k.sg;
  entries = k.sg + p1 / GRAIN + 1 - first;
  k.i0 = 0;
  k.i1 = entries;
  return k;
}

// What takes part, for up to 64 sequences: lane b has sequence b's rows, its first row, and its row tiles.  Lengths that do not add up to the
// host's rows and tiles, or a run longer than its longest one, disable the batch (off); a context outside [0, max_ctx) its sequence, whose
// tiles are there all the same: somebody has to write its zeros.
struct WindowShare {
  int q, row0, ctx, tiles, flags;
  bool off;
};
__device__ __forceinline__ bool window_fits(const PrefixBatch& p, int ctx, int q) { return ctx >= 0 && (long)ctx + q <= p.max_ctx; }
__device__ __forceinline__ WindowShare lane_window(const PrefixBatch& p, int n_tiles) {
  const int b = threadIdx.x & 63;
  WindowShare s{0, 0, 0, 0, 0, false};
  bool off = false;
  if (b < p.B) {
    const int k = p.spec_len[b];
    s.ctx = p.ctx_lens[b];
    off = k < 0 || k >= p.max_q;
    s.q = off ? 0 : k + 1;
    s.tiles = (int)(((long)p.G * s.q + p.tile_rows - 1) / p.tile_rows);
    if (!window_fits(p, s.ctx, s.q)) s.flags = MN_DEV_CTX;
  }
  const int incl = wave_scan_i(s.q);
  s.row0 = incl - s.q;
  s.off = __any(off) || __builtin_amdgcn_readlane(incl, 63) != p.M || __builtin_amdgcn_readfirstlane(wave_sum_i(s.tiles)) != n_tiles;
  if (s.off) s.flags = MN_DEV_SPEC_LEN;
  return s;
}

// Tile t of the batch; false: the batch takes no part.  it.R < 0: the sequence does not (|R| rows of zeros).  The last tiles of a sequence
// come first: where the window is longer than the context they have the most keys.
__device__ __forceinline__ bool window_tile(const TileArgs& a, int t, Item& it) {
  if (a.items) {
    const int4 x = reinterpret_cast<const int4*>(a.items)[2 * t], y = reinterpret_cast<const int4*>(a.items)[2 * t + 1];
    it = Item{x.x, x.y, x.z, 0, 0, y.y, y.z, 0};
    return it.R != 0;
  }
  const WindowShare s = lane_window(a.batch, a.n_tiles);
  if ((int)blockIdx.x == a.n_checks && threadIdx.x < 64 && s.flags && a.status) atomicOr(a.status, s.flags);
  if (s.off) return false;
  const int incl = wave_scan_i(s.tiles);
  const int b = __ffsll((unsigned long long)__ballot(t < incl)) - 1;
  const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
  it.m0 = of(s.row0); it.ctx = of(s.ctx); it.seq = b; it.slot = 0; it.key0 = it.key_end = 0;
  it.rbase = (of(incl) - 1 - t) * a.batch.tile_rows;
  it.R = a.batch.G * of(s.q) * (of(s.flags) ? -1 : 1);
  return true;
}

// Zeros for the rows of this workgroup's tile and head (R rows of the stack at most), or, of a batch that takes no part, for its share of all.
template <typename T>
__device__ __forceinline__ void window_zeros(const TileArgs& a, const Item* it, int kvh, int G) {
  struct __attribute__((aligned(4 * sizeof(T)))) Four0 { T x[4]; };
  const int per = a.hd / 4;
  const auto clear = [&](size_t mh, int e) {
    reinterpret_cast<Four0*>(a.out)[mh * per + e] = Four0{};
    if (e == 0 && a.stats) *reinterpret_cast<float2*>(a.stats + 2 * mh) = make_float2(0.f, 0.f);
  };
  if (it) {
    for (int i = threadIdx.x; i < min(-it->R - it->rbase, a.batch.tile_rows) * per; i += blockDim.x) {
      const int r = it->rbase + i / per, j = r / G;
      clear((size_t)(it->m0 + j) * a.H + kvh * G + r - j * G, i % per);
    }
  } else {
    const size_t all = (size_t)a.M * a.H * per;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (size_t)gridDim.x * blockDim.x) clear(i / per, (int)(i % per));
  }
}

// The item of workgroup wg (behind those that look at the table rows, if there are any).
template <typename T>
__device__ __forceinline__ bool window_item(const TileArgs& a, int wg, int G, int& kvh, Item& it, Look& look) {
  kvh = wg % a.Hkv;
  const int at = wg / a.Hkv, t = at / a.ranges, range = at - t * a.ranges;
  if (!window_tile(a, t, it)) {
    if (a.ranges == 1) window_zeros<T>(a, nullptr, kvh, G);
    return false;
  }
  if (it.R < 0) {
    if (a.ranges == 1) window_zeros<T>(a, &it, kvh, G);
    return false;
  }
  const int p1 = it.ctx + (min(it.R, it.rbase + a.batch.tile_rows) - 1) / G;
  int entries;
  look = look_from(a, it.ctx + it.rbase / G, p1, entries);
  look.i0 = range * a.batch.chunk;
  look.i1 = min(entries, look.i0 + a.batch.chunk);
  it.key_end = p1 + 1;
  it.slot = range;
  return look.i0 < look.i1;
}

// Whether an entry of sequence `seq`'s table row that its rows look at is out of range (this thread's share of them).  The last one that it
// looks at is left in `entry`: a caller with something to ask for meanwhile looks at it later.
__device__ __forceinline__ bool window_table_bad(const TileArgs& a, int seq, int ctx, int q, int& entry) {
  const int bs = a.kv.block_size, end = ctx + q, first = max(0, ctx - a.window + 1) / bs, n_first = min(first, (min(a.sinks, end) + bs - 1) / bs);
  const int32_t* row = a.kv.block_tables + (size_t)seq * a.kv.max_blocks_per_seq;
  const int all = n_first + (end - 1) / bs + 1 - first;
  bool bad = false;
  int i = threadIdx.x;
  for (; i + (int)blockDim.x < all; i += blockDim.x) bad |= (uint32_t)row[i < n_first ? i : i - n_first + first] >= (uint32_t)a.kv.num_blocks;
  i = min(i, all - 1);
  entry = row[i < n_first ? i : i - n_first + first];
  return bad;
}
// For the calls whose rows are put together from parts: a workgroup per sequence.
__device__ __forceinline__ void window_check(const TileArgs& a, int b) {
  const int ctx = scalar(a.batch.ctx_lens)[b], k = scalar(a.batch.spec_len)[b];
  if (k < 0 || k >= a.batch.max_q || !window_fits(a.batch, ctx, k + 1)) return;  // (takes no part)
  int entry;
  bool bad = window_table_bad(a, b, ctx, k + 1, entry);
  bad = __syncthreads_or(bad | ((uint32_t)entry >= (uint32_t)a.kv.num_blocks));
  if (threadIdx.x == 0) {
    a.seq_bad[b] = bad;
    if (bad && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
  }
}

// Rows of K and V of the tokens whose first stack row lies in this tile, into the pages (position = token of the sequence).
template <typename T, int ROWS>
__device__ __forceinline__ void append_rows(const TileArgs& a, const Item& it, int G, int kvh) {
  const int j0 = (it.rbase + G - 1) / G, j1 = (min(it.R, it.rbase + ROWS) + G - 1) / G;
  const int hd = a.hd, bs = a.kv.block_size;
  const int32_t* bt = a.kv.block_tables + (size_t)it.seq * a.kv.max_blocks_per_seq;
  bool bad = false;
  // 8 consecutive head-dim elements of one token: 16 bytes (fp32: 32) of a K page, a column of a V page
  for (int i = threadIdx.x; i < (j1 - j0) * (hd / 8); i += blockDim.x) {
    const int j = j0 + i % (j1 - j0), c = i / (j1 - j0);
    const int id = bt[j / bs], off = j % bs;
    if ((uint32_t)id >= (uint32_t)a.kv.num_blocks) {
      bad = true;
      continue;
    }
    struct __attribute__((aligned(16))) Piece { T x[8]; };
    const Piece k = *reinterpret_cast<const Piece*>(static_cast<const T*>(a.k) + (size_t)(it.m0 + j) * a.k_stride + (size_t)kvh * hd + 8 * c);
    const Piece v = *reinterpret_cast<const Piece*>(static_cast<const T*>(a.v) + (size_t)(it.m0 + j) * a.v_stride + (size_t)kvh * hd + 8 * c);
    const size_t page = ((size_t)id * a.Hkv + kvh) * (size_t)(hd * bs);
    *reinterpret_cast<Piece*>(static_cast<T*>(a.kv.k) + page + ((size_t)c * bs + off) * 8) = k;
    T* to = static_cast<T*>(a.kv.v) + page + (size_t)(8 * c) * bs + off;
#pragma unroll
    for (int e = 0; e < 8; ++e) to[(size_t)e * bs] = v.x[e];
  }
  if (bad && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
}

// ------------------------------------------------------------------------------------------
// fp16, head_dim 64 or 128
// ------------------------------------------------------------------------------------------
// A workgroup of NW waves holds 16 * CT * NW stack rows, wave w the rows from 16 * CT * w on, their queries in registers.  Both products
// have the query row as the column index (S^T = K Q^T, O^T = V^T P^T): statistics are per-lane numbers, and with the K rows of a
// half of 32 keys permuted (S^T row 4g + r of half t is key 8g + 4t + r) the probabilities leave the first product in the operand
// order of the second.  Tiles of 32 keys are staged ahead by direct global -> LDS loads of whole rows, or of whole pages, their 16-byte
// pieces in turned places so that the reads of the operands meet every bank; V of dense rows is turned on the way to the registers by
// the transposing LDS read (a page keeps the block's tokens of one head-dim element together already).
//
// Bounds.  Long rows of keys: the matrix pipe.  8192 tokens of 64/8 heads of 128 take 1050 us = 1050 TFLOP/s (a library product of 8192^3
// reaches 1133); without the staging 14 % less, without the exponentials 14 %, without the barriers 3 %.  Two workgroups of 128 rows per
// CU, 251 registers a wave: a tile of 256 rows does not fit them, 64 rows read the stages twice as often (1390 us).  A shared prefix
// behind few rows: HBM; 32000 keys of 8 heads of 128 in 28 us = 4.7 TB/s, lead-in included.
constexpr int TK = 32;                              // keys per stage
template <int HDIM> struct TileStage {
  static constexpr int HS = HDIM / 32, NU = HDIM / 16;
  static constexpr int KP = TK / 16 * HS;           // 1 KB pieces of K in a stage, and as many of V
  static constexpr int FRAGS = 2 * KP;
  static constexpr int BYTES = FRAGS * 1024;
};
constexpr int STAGES = 4;

typedef short s16x4 __attribute__((ext_vector_type(4)));
template <int N> struct PieceC { static constexpr int value = N; };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void pieces(F f) {
  if constexpr (I < N) {
    f(PieceC<I>{});
    pieces<N, I + 1>(f);
  }
}
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// the largest of a lane's eight scores (`maximum` takes a NaN as it is, and so needs no instruction to quiet one first)
__device__ __forceinline__ float top(const f32x4 (&S)[2]) {
  const auto m = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };
  return m(m(m(m(S[0][0], S[0][1]), S[0][2]), m(m(S[0][3], S[1][0]), S[1][1])), m(S[1][2], S[1][3]));
}

template <int HDIM, int CT, int NW, bool PAGED, bool WINDOW>
__global__ void __launch_bounds__(NW * 64, 2) tile_mfma_kernel(TileArgs a) {
  static_assert(PAGED || !WINDOW, "windows are of pages");
  using St = TileStage<HDIM>;
  constexpr int HS = St::HS, NU = St::NU, KP = St::KP, LPW = St::FRAGS / NW, ROWS = 16 * CT * NW;
  static_assert(St::FRAGS % NW == 0, "whole pieces per wave");
  // Tiles asked for ahead of the one at hand.  Four keep two on their way between the hand-overs, where HBM is the bound (64 rows behind
  // pages: 3 x 1 to 3 rows of 64/8 heads behind 32000 tokens 36.9 -> 31.4 us, 16 x 1 of 40 heads 29.3 -> 27.0); with the matrix
  // pipe as the bound three are enough and 1 % faster.
  constexpr int AHEAD = PAGED && CT == 1 ? STAGES : STAGES - 1;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const Divide by(a.H / a.Hkv);                                  // (query heads per KV head)
  const int G = by.d;
  int kvh = 0, stream = 0, unit = 0;
  Item it;
  Look look{};
  bool more = false;
  if constexpr (WINDOW) {
    const int wg = (int)blockIdx.x - a.n_checks;
    if (wg < 0) return window_check(a, blockIdx.x);
    if (!window_item<f16_t>(a, wg, G, kvh, it, look)) return;
  } else if constexpr (PAGED) {
    // a workgroup per table row, those of the sequences' own keys, the streams
    const int own = a.n_tiles * a.Hkv, wg = (int)blockIdx.x - a.B;
    if (wg < 0) return check_table(a, blockIdx.x);
    if (wg < own) {
      kvh = wg % a.Hkv;
      if (!own_item(a, wg / a.Hkv, it)) return;
    } else {
      stream = stream_of(a, wg - own);
      unit = stream * a.share;
      if (!stream_item(a, stream, unit, kvh, it)) return;
      more = true;
    }
  } else {
    kvh = blockIdx.x % a.Hkv;
    if (!prompt_item<ROWS>(a, blockIdx.x / a.Hkv, by, reinterpret_cast<int32_t*>(smem), it)) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  do {
    // this wave's rows, and the keys that its first and last row see
    const int rw0 = it.rbase + wave * CT * 16;
    const bool rows = rw0 < it.R;
    const int min_lim = min(it.key_end - 1, it.ctx + by(rw0));
    const int max_lim = rows ? min(it.key_end - 1, it.ctx + by(min(it.R, rw0 + CT * 16) - 1)) : -1;
    f16x8 qf[CT][HS];
    int lim[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int r = min(rw0 + 16 * ct + l16, it.R - 1), j = by(r);
      lim[ct] = min(it.key_end - 1, it.ctx + j);
      const f16_t* q = static_cast<const f16_t*>(a.q) + (size_t)(it.m0 + j) * a.q_stride + (size_t)(kvh * G + r - j * G) * HDIM;
#pragma unroll
      for (int s = 0; s < HS; ++s) qf[ct][s] = *reinterpret_cast<const f16x8*>(q + 32 * s + 8 * g);
    }
    f32x4 O[CT][NU];
    float run_m[CT], neg_m[CT], thr[CT], L[CT];                    // reference, its negative (0: none yet), scores that move it, sum of this lane
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      run_m[ct] = thr[ct] = -INFINITY;
      neg_m[ct] = L[ct] = 0.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) O[ct][u] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float c = rsqrtf((float)HDIM) * LOG2E_T, inv_c = 1.f / c;

    // ---- staging: waves 0 and 1 fetch K, 2 and 3 V, each the 16 keys (the block) that its parity names, 1 KB of whole rows or of a whole
    // page per load.  The 16-byte chunks of a row, and of a page, change places inside 256 bytes on the way, so that the reads of
    // the operands meet every bank (`turn`). ----
    const int n_tiles = WINDOW ? (look.i1 - look.i0 + 1) / 2 : (it.key_end - it.key0 + TK - 1) / TK;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem);
    const int last_key = it.key_end - 1;
    const bool k_wave = wave < NW / 2;
    const int side = wave & 1;
    const uint32_t to0 = lds0 + (uint32_t)((k_wave ? 0 : KP) + side * LPW) * 1024u;
    // pages
    const const_i32* bt = PAGED ? scalar(a.kv.block_tables + (size_t)it.seq * a.kv.max_blocks_per_seq) : nullptr;
    const uint32_t blk_bytes = PAGED ? (uint32_t)a.Hkv * (HDIM * PAGE) * 2u : 0u;
    int next_id = 0;
    const auto ask_id = [&](int tile) {
      if constexpr (WINDOW) next_id = bt[look.at(min(look.i0 + 2 * tile + side, look.i1 - 1))];
      else next_id = bt[min((it.key0 + min(tile, n_tiles - 1) * TK) / PAGE + side, last_key / PAGE)];
    };
    // dense rows
    constexpr int CH = HDIM / 8, KPP = 64 / CH;                    // 16-byte chunks per row, rows per piece
    const uint32_t stride = (uint32_t)(k_wave ? a.k_stride : a.v_stride) * 2u;
    const int key_lane = 16 * side + lane / CH;                    // the lane's row in its first piece
    // K: the 16 keys of a half in as many places.  V: 32 bytes stay together (the transposing reads take as much of a row)
    const auto turn = [&](int key) {
      if (k_wave) return HDIM == 128 ? ((key >> 1 & 12) | (key & 3)) : ((key >> 2 & 6) | (key >> 1 & 1));
      return HDIM == 128 ? ((key & 3) << 1 | (key & 8)) : ((key & 2) | (key >> 1 & 4));
    };
    const char* base;                                              // of the wave's piece of the next tile (dense), or of its head (pages)
    uint32_t off0, off1 = 0;                                       // the lane's bytes from it, in pieces whose keys agree in bit 3
    if constexpr (PAGED) {
      base = static_cast<const char*>(k_wave ? a.kv.k : a.kv.v) + (size_t)kvh * (HDIM * PAGE * 2);
      off0 = 16u * (uint32_t)(k_wave ? lane ^ (side * 4) : lane ^ (lane >> 4 & 1));
      ask_id(0);
      if (more) {                                                  // (row 0 is mostly the one; its first id is on the way meanwhile)
        const int seq = first_sharer(a);
        if (seq > 0) {
          bt = scalar(a.kv.block_tables + (size_t)seq * a.kv.max_blocks_per_seq);
          ask_id(0);
        }
      }
    } else {
      base = static_cast<const char*>(k_wave ? a.k : a.v) + ((size_t)(it.m0 + it.key0) * stride + (size_t)kvh * HDIM * 2);
      off0 = (uint32_t)key_lane * stride + 16u * (uint32_t)((lane % CH) ^ turn(key_lane));
      off1 = (uint32_t)key_lane * stride + 16u * (uint32_t)((lane % CH) ^ turn(key_lane ^ 8));
    }
    const auto stage = [&](int tile) {
      const uint32_t to = to0 + (uint32_t)(tile & (STAGES - 1)) * St::BYTES;
      if constexpr (PAGED) {
        const char* p = base + (uint64_t)min((uint32_t)next_id, (uint32_t)a.kv.num_blocks - 1u) * blk_bytes;
        // (keys that no other tile of rows reads are not kept in the L2)
        if (WINDOW ? a.keep_keys : (more && a.row_tiles > 1)) pieces<LPW>([&](auto i) { dma16s<i.value * 1024, false>(p, off0, to + i.value * 1024u); });
        else pieces<LPW>([&](auto i) { dma16s<i.value * 1024, true>(p, off0, to + i.value * 1024u); });
        ask_id(tile + 1);
      } else {
        const int k0 = it.key0 + min(tile, n_tiles - 1) * TK;      // (of the first stages, those past the end repeat the last one)
        if (k0 + TK - 1 <= last_key) {
          pieces<LPW>([&](auto i) { dma16s<0, false>(base + i.value * KPP * (uint64_t)stride, (i.value * KPP & 8) ? off1 : off0, to + i.value * 1024u); });
        } else {                                                   // rows past the end repeat the last one
          pieces<LPW>([&](auto i) {
            const int key = key_lane + i.value * KPP;
            dma16s<0, false>(base, (uint32_t)min(key, last_key - k0) * stride + 16u * (uint32_t)((lane % CH) ^ turn(key)), to + i.value * 1024u);
          });
        }
        if (tile + 1 < n_tiles) base += TK * (uint64_t)stride;
      }
    };
    // Operands of the first product: chunk 4s + g of key 8 (l16 >> 2) + 4 half + (l16 & 3).
    uint32_t k_lane;
    {
      const int key = 8 * (l16 >> 2) + (l16 & 3);
      if constexpr (PAGED) k_lane = (uint32_t)((l16 >> 3) * LPW * 1024 + g * 256 + ((key & 15) ^ (l16 >> 3) * 4) * 16);
      else k_lane = (uint32_t)(key * (2 * HDIM) + 16 * (g ^ (HDIM == 128 ? l16 : (l16 >> 2 << 1 | (l16 >> 1 & 1)))));
    }
    // Of the second: 8 tokens of an element of a page, or by transposing reads: lanes 4k .. 4k + 3 of a group of 16 address 32 bytes of key
    // 8g + k, lane i receives column i.
    const uint32_t v_lane = PAGED ? (uint32_t)((g >> 1) * LPW * 1024 + l16 * 32 + ((g & 1) ^ (l16 >> 3)) * 16)
                                  : (uint32_t)((8 * g + (l16 >> 2)) * (2 * HDIM) + (HDIM == 128 ? ((l16 >> 2) | (g & 1) << 2) : ((l16 >> 3) | (g & 1) << 1)) * 32 +
                                               (l16 & 3) * 8);
    const auto slot = [&](int tile) { return smem + (tile & (STAGES - 1)) * St::BYTES; };
    const auto load_k = [&](const unsigned char* st, f16x8 (&kf)[2 * HS]) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int h = 0; h < HS; ++h) {
          const uint32_t at = PAGED ? (k_lane ^ (uint32_t)(half * 64)) + (uint32_t)(h * 1024) : (k_lane ^ (uint32_t)(h * 64)) + (uint32_t)(half * 8 * HDIM);
          kf[half * HS + h] = *reinterpret_cast<const f16x8*>(st + at);
        }
    };
    const auto load_v = [&](const unsigned char* st, f16x8 (&vf)[NU]) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        if constexpr (PAGED) {
          vf[u] = *reinterpret_cast<const f16x8*>(st + v_lane + (KP * 1024 + u * 512));
        } else {
          union { f16x8 v; s16x4 h[2]; } x;
          const uint32_t at = (v_lane ^ (uint32_t)(u * 32)) + (uint32_t)(KP * 1024);
          x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(st + at));
          x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(st + at + 4 * 2 * HDIM));
          vf[u] = x.v;
        }
      }
    };
    const auto scores = [&](const f16x8 (&kf)[2 * HS], f32x4 (&S)[CT][2]) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        S[ct][0] = S[ct][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < HS; ++h) {
          S[ct][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[h], qf[ct][h], S[ct][0], 0, 0, 0);
          S[ct][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[HS + h], qf[ct][h], S[ct][1], 0, 0, 0);
        }
      }
    };

    // One half tile (32 keys) after the other.  Its scores are there when its turn comes (S, their maximum of this lane tm); those of the
    // next one are worked out beside its probabilities (first part), and its second product (second part) runs while the keys of
    // the half behind the next and the values of the next are on their way from the LDS: the matrix pipe and the vector unit both
    // have work, and neither waits for the LDS.
    f16x8 kf[2 * HS], vf[NU], P[CT];
    const auto first = [&](int tile, const unsigned char* next_keys, f32x4 (&S)[CT][2], float (&tm)[CT], f32x4 (&Sn)[CT][2]) {
      int keyg;                                                    // the lane's eight keys
      bool masked;                                                 // (uniform) a key that some row does not see
      if constexpr (WINDOW) {
        const int i = look.i0 + 2 * tile + (g >> 1);
        keyg = i < look.i1 ? look.at(i) * PAGE + 8 * (g & 1) : NO_KEY;
        masked = __any((keyg + 7 > min_lim) | ((keyg <= max_lim - a.window) & (keyg + 7 >= a.sinks)));
      } else {
        const int k0 = it.key0 + tile * TK;
        keyg = k0 + 8 * g;
        masked = k0 + 31 > min_lim;
      }
      if (masked) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if constexpr (WINDOW) {
            const int ahead = lim[ct] - keyg, back = ahead - a.window, sink = a.sinks - keyg;
#pragma unroll
            for (int e = 0; e < 8; ++e) S[ct][e >> 2][e & 3] = in_sight(e, ahead, back, sink) < 0 ? S[ct][e >> 2][e & 3] : -INFINITY;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (keyg + e > lim[ct]) S[ct][e >> 2][e & 3] = -INFINITY;
          }
          tm[ct] = top(S[ct]);
        }
        if constexpr (PAGED) {
          // slots past the last key may hold anything, and 0 times anything has to stay 0
          const int past = keyg + 8 - it.key_end;
          if (past > 0) {
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e >= 8 - past) vf[u][e] = (f16_t)0.f;
          }
        }
      }
      bool move = false;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) move |= tm[ct] > thr[ct];
      if (__any(move)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          uint32_t x, y;
          float t2 = tm[ct];
          lane_pair<16>(__float_as_uint(t2), x, y);
          t2 = __builtin_fmaxf(__uint_as_float(x), __uint_as_float(y));
          lane_pair<32>(__float_as_uint(t2), x, y);
          t2 = __builtin_fmaxf(__uint_as_float(x), __uint_as_float(y)) * c;
          const float nm = __builtin_fmaxf(run_m[ct], t2);
          const float alpha = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(run_m[ct] - nm);
          const bool far = __builtin_fabsf(nm) >= FAR;
          run_m[ct] = nm;
          thr[ct] = far ? -INFINITY : (nm + LAZY) * inv_c;
          neg_m[ct] = far ? 0.f : -nm;
          if (__any(far && nm != -INFINITY)) {
            if (far && nm != -INFINITY) {
#pragma clang fp contract(off)
#pragma unroll
              for (int e = 0; e < 8; ++e) S[ct][e >> 2][e & 3] = (S[ct][e >> 2][e & 3] * c - nm) * inv_c;
            }
          }
#pragma unroll
          for (int u = 0; u < NU; ++u) O[ct][u] *= alpha;
          L[ct] *= alpha;
        }
      }
      if (masked) {
        // Values that are not finite reach the rows that see their key and no other (nor is 0 times them 0): they leave the product, and
        // the rows that see +inf, -inf or NaN (as both) get what the sum would be.
        f16x2 odd = {(f16_t)0.f, (f16_t)0.f};
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd = __builtin_elementwise_fma((f16x2){vf[u][2 * e], vf[u][2 * e + 1]}, (f16x2){(f16_t)0.f, (f16_t)0.f}, odd);
        if (__any(odd[0] != odd[0] || odd[1] != odd[1])) {
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            union { f16x8 v; uint32_t u[4]; } w, at;
            w.v = vf[u];
#pragma unroll
            for (int side = 0; side < 2; ++side) {                 // +inf, -inf; NaN is both
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t x = w.u[e], sign = (side ? x : ~x) >> 15, nan = ((x & 0x03ff03ffu) + 0x03ff03ffu) >> 10;
                at.u[e] = (((x & 0x7fff7fffu) + 0x04000400u) >> 15 & (sign | nan) & 0x00010001u) * 0x3c00u;  // 1.0 there
              }
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) {
                f16x8 sees;
                if constexpr (WINDOW) {
                  // (worked out anew each time: registers)
                  int ahead = lim[ct] - keyg, sink = a.sinks - keyg;
                  asm volatile("" : "+v"(ahead), "+v"(sink));
                  const int back = ahead - a.window;
#pragma unroll
                  for (int e = 0; e < 8; ++e)
                    sees[e] = __builtin_bit_cast(f16_t, (uint16_t)(in_sight(e, ahead, back, sink) >> 31 & 0x3c00));  // 1.0 or 0
                } else {
                  int ahead = lim[ct] - keyg;
                  asm volatile("" : "+v"(ahead));
#pragma unroll
                  for (int e = 0; e < 8; ++e) sees[e] = e <= ahead ? (f16_t)1.f : (f16_t)0.f;
                }
                const f32x4 met = __builtin_amdgcn_mfma_f32_16x16x32_f16(at.v, sees, (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (met[e] > 0.f) O[ct][u][e] += side ? -INFINITY : INFINITY;
                __builtin_amdgcn_sched_barrier(0);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) w.u[e] &= ~((((w.u[e] & 0x7fff7fffu) + 0x04000400u) >> 15 & 0x00010001u) * 0xffffu);
            vf[u] = w.v;
            __builtin_amdgcn_sched_barrier(0);
          }
          load_k(next_keys, kf);                                   // (their registers were needed)
        }
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        union { f16x8 v; uint32_t u[4]; f16x2 h[4]; } pf;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pf.u[e] = pack2h(__builtin_amdgcn_exp2f(fmaf(S[ct][e >> 1][2 * (e & 1)], c, neg_m[ct])),
                           __builtin_amdgcn_exp2f(fmaf(S[ct][e >> 1][2 * (e & 1) + 1], c, neg_m[ct])));
#pragma unroll
        for (int e = 0; e < 4; ++e) L[ct] = __builtin_amdgcn_fdot2(pf.h[e], (f16x2){(f16_t)1.f, (f16_t)1.f}, L[ct], false);
        P[ct] = pf.v;
      }
      scores(kf, Sn);
    };
    const auto second = [&](const unsigned char* k_slot, const unsigned char* v_slot, const f32x4 (&Sn)[CT][2], float (&tn)[CT]) {
      __builtin_amdgcn_sched_barrier(0);
      load_k(k_slot, kf);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int u = 0; u < NU; ++u) O[ct][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[u], P[ct], O[ct][u], 0, 0, 0);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) tn[ct] = top(Sn[ct]);
      __builtin_amdgcn_sched_barrier(0);
      load_v(v_slot, vf);
      __builtin_amdgcn_sched_barrier(0);
    };

    // (what only the end asks for waits in vector registers: of the scalar ones there are not enough)
    const auto aside = [](int v) {
      if constexpr (WINDOW) asm volatile("" : "+v"(v));
      return v;
    };
    const int end_m0 = aside(it.m0), end_seq = aside(it.seq), end_ctx = aside(it.ctx), end_slot = aside(it.slot), end_kvh = aside(kvh);
    // tiles that a row of the wave sees
    const int n_wave = WINDOW ? (rows ? min(n_tiles, max(0, look.entry(max_lim / PAGE) - look.i0 + 2) / 2) : 0) : min(n_tiles, max(0, max_lim + TK - it.key0) / TK);
    bool lost = false;                                             // a damaged table row, looked at while the first tiles are on their way
    int entry = 0;
    if constexpr (WINDOW) {
      if (a.ranges == 1) lost = window_table_bad(a, it.seq, it.ctx, it.R / G, entry);
    }
    __syncthreads();                                               // (the search, or the piece before, is through with the LDS)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (!PAGED || i < n_tiles) stage(i);                         // (dense rows: short ones are rare, and the test cost as much)
    if (!PAGED || n_tiles >= AHEAD) wait_vm<(AHEAD - 2) * LPW>();  // (tiles 0 and 1 are there)
    else wait_vm<0>();
    if constexpr (WINDOW) {
      asm volatile("" : "+v"(entry));
      if (__syncthreads_or(lost | ((uint32_t)entry >= (uint32_t)a.kv.num_blocks))) {
        wait_vm<0>();
        if (tid == 0 && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
        it.R = -it.R;
        window_zeros<f16_t>(a, &it, kvh, G);
        return;
      }
    } else {
      __syncthreads();
    }
    f32x4 Sa[CT][2], Sb[CT][2];
    float ta[CT], tb[CT];
    load_k(slot(0), kf);
    scores(kf, Sa);
    load_k(slot(1), kf);
    load_v(slot(0), vf);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) ta[ct] = top(Sa[ct]);
    // Tile i: its first part, then the hand-over: this wave's share of tile i + 2 has landed, then everybody's; tile i has been read by all
    // (its values are in the registers), and its place, or that of tile i - 1, is filled again.
    const auto tile = [&](int i, f32x4 (&S)[CT][2], float (&tm)[CT], f32x4 (&Sn)[CT][2], float (&tn)[CT]) {
      const bool on = i < n_wave;                                  // (uniform)
      if (on) first(i, slot(i + 1), S, tm, Sn);
      if (AHEAD > 3 && i + 3 < n_tiles) wait_vm<(AHEAD - 3) * LPW>();
      else wait_vm<0>();
      __syncthreads();
      if (i + AHEAD < n_tiles) stage(i + AHEAD);
      if (on) second(slot(i + 2), slot(i + 1), Sn, tn);
    };
    for (int i = 0; i < n_tiles; i += 2) {                         // (behind an odd last tile comes one that no wave works on)
      tile(i, Sa, ta, Sb, tb);
      tile(i + 1, Sb, tb, Sa, ta);
    }
    wait_vm<0>();                                                  // (of a dense item's first stages, any past its end)

    // ---- output: lane holds O^T[16u + 4g + i][row l16], and its row's sum ----
    if constexpr (WINDOW) {
      it.m0 = __builtin_amdgcn_readfirstlane(end_m0); it.seq = __builtin_amdgcn_readfirstlane(end_seq); it.ctx = __builtin_amdgcn_readfirstlane(end_ctx);
      it.slot = __builtin_amdgcn_readfirstlane(end_slot); kvh = __builtin_amdgcn_readfirstlane(end_kvh);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      uint32_t x, y;                                               // the row's sum over the four lane groups
      lane_pair<16>(__float_as_uint(L[ct]), x, y);
      L[ct] = __uint_as_float(x) + __uint_as_float(y);
      lane_pair<32>(__float_as_uint(L[ct]), x, y);
      L[ct] = __uint_as_float(x) + __uint_as_float(y);
      const int r = rw0 + 16 * ct + l16;
      if (r >= it.R) continue;
      const int j = by(r), m = it.m0 + j, h = kvh * G + r - j * G;
      const float l = L[ct];
      if (PAGED && !(WINDOW && a.ranges == 1)) {
        float* o = a.o_part + (((size_t)it.slot * a.M + m) * a.H + h) * HDIM + 4 * g;
#pragma unroll
        for (int u = 0; u < NU; ++u) *reinterpret_cast<f32x4*>(o + 16 * u) = O[ct][u];
        if (g == 0) *reinterpret_cast<float2*>(a.ml_part + (((size_t)it.slot * a.M + m) * a.H + h) * 2) = make_float2(run_m[ct], l);
      } else {
        if (WINDOW && a.stats && g == 0) *reinterpret_cast<float2*>(a.stats + ((size_t)m * a.H + h) * 2) = make_float2(run_m[ct], l);
        const float inv = 1.f / l;
        f16_t* o = static_cast<f16_t*>(a.out) + ((size_t)m * a.H + h) * HDIM + 4 * g;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const f32x4 v = O[ct][u];
          *reinterpret_cast<uint2*>(o + 16 * u) = make_uint2(pack2h(v[0] * inv, v[1] * inv), pack2h(v[2] * inv, v[3] * inv));
        }
      }
    }
    // Rows that enter the cache: those whose first stack row lies in this workgroup's tile, out of the stages.  They are the last keys it
    // read; where they lie in the last tile of keys alone that stage is used as it is, else they are fetched once more (the stages before
    // it are still there as well: nothing is staged past an item's end).  A lane's piece of K is 8 elements of one token, and of V
    // 8 tokens of one element: 16 bytes of a page each way.  7800 rows of 40 KV heads of 128, 161 us without: written as they come
    // by the rows at the start 221 us, by a kernel of its own 253, like this 208 (now 157 and 192), where 160 MB of pages are worth about 35.
    if (!PAGED && a.kv.k) {
      const int put0 = (it.rbase + G - 1) / G, put1 = (min(it.R, it.rbase + ROWS) + G - 1) / G;
      __syncthreads();                                             // (everybody is through with the stages, and the last tile is there)
      if (put0 / TK < n_tiles - 1) {                               // (at most ROWS / TK stages; one more than ROWS / G / TK if that is not whole)
        static_assert(ROWS / TK <= STAGES && ROWS / 2 / TK + 1 <= STAGES, "the rows of a tile fit the stages");
        base = static_cast<const char*>(k_wave ? a.k : a.v) + ((size_t)(it.m0 + put0 / TK * TK) * stride + (size_t)kvh * HDIM * 2);
        for (int i = put0 / TK; i * TK < put1; ++i) stage(i);
        wait_vm<0>();
        __syncthreads();
      }
      bool bad = false;
      for (int i = put0 / TK; i * TK < put1; ++i) {
        const unsigned char* st = slot(i);
        const int in_tile = k_wave ? 16 * side + l16 : 8 * g, key = i * TK + in_tile;
        if (key >= put1 || key + (k_wave ? 0 : 7) < put0) continue;
        const uint32_t id = (uint32_t)a.kv.block_tables[(size_t)it.seq * a.kv.max_blocks_per_seq + key / PAGE];
        if (id >= (uint32_t)a.kv.num_blocks) {
          bad = true;
          continue;
        }
        const size_t page = ((size_t)id * a.Hkv + kvh) * (HDIM * PAGE);
        if (k_wave) {
          f16_t* to = static_cast<f16_t*>(a.kv.k) + page + (key & (PAGE - 1)) * 8;
#pragma unroll
          for (int n = 0; n < CH / 4; ++n)
            *reinterpret_cast<f16x8*>(to + (4 * n + g) * (PAGE * 8)) =
                *reinterpret_cast<const f16x8*>(st + in_tile * (2 * HDIM) + 16 * ((4 * n + g) ^ turn(in_tile)));
        } else {
          f16_t* to = static_cast<f16_t*>(a.kv.v) + page + (16 * side * LPW + l16) * PAGE + (key & (PAGE - 1));
          const bool all = key >= put0 && key + 8 <= put1;
#pragma unroll
          for (int n = 0; n < LPW; ++n) {
            union { f16x8 v; s16x4 h[2]; } x;
            const uint32_t at = (v_lane ^ (uint32_t)((side * LPW + n) * 32)) + (uint32_t)(KP * 1024);
            x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(st + at));
            x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(st + at + 4 * 2 * HDIM));
            if (all) {
              *reinterpret_cast<f16x8*>(to + n * 16 * PAGE) = x.v;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (key + e >= put0 && key + e < put1) to[n * 16 * PAGE + e] = x.v[e];
            }
          }
        }
      }
      if (bad && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
    }
  } while (!WINDOW && more && stream_item(a, stream, unit, kvh, it));
}

// ------------------------------------------------------------------------------------------
// every other type, head_dim and block size
// ------------------------------------------------------------------------------------------
// Products in fp32 on the 16x16x4 instruction, 16 stack rows per wave.  Nothing is staged and the waves never wait for one another: a lane's
// operands are 4 consecutive elements of a row of K (four instructions take one each), and of V 4 elements of one key (dense rows: row i of
// instruction r is element VEC i + r of the group) or 4 tokens of one element (pages), read from memory in that shape and widened;
// 16 rows per workgroup, every fourth 32 keys (heads of 256: 16) to a wave, their parts put together in LDS at the end.  Bound by the round
// trips of a wave through its keys, and beyond by the issue of its instructions (7000 tokens of 4 heads of 64 247 us = 102 TFLOP/s, a
// library product of 8192^3 152; 32 rows per workgroup read half as much and take 283): 4 prompts of 33 to 700 tokens of 4 fp32 heads of 64 11 us (32.6 with 64 rows
// and keys staged for all waves; 27.0 with 64 rows and every wave reading all keys), 4 of 1500 to 2500 127 us = 95 TFLOP/s
// (211, 237), 4 fp16 prompts of 300 to 1500 of 8/2 heads of 256 107 us (245, 260).  HDP: head_dim padded to a multiple of 16.
// Two waves per SIMD are asked for where 256 registers hold a wave (not the pages of heads of 128 and more): left alone the
// compiler takes more, and the last two take 140 and 152 us.
constexpr int FROWS = 16, KW = 4;                                // rows of a workgroup, its waves
template <typename T> struct __attribute__((aligned(4 * sizeof(T)))) Four { T x[4]; };

template <typename T, int HDP, bool PAGED, bool WINDOW>
__global__ void __launch_bounds__(256, PAGED && HDP >= 128 ? 1 : 2) tile_f32_kernel(TileArgs a) {
  constexpr int NU = HDP / 16, LD = HDP + 4, HALVES = HDP == 256 ? 1 : 2;  // (16 keys at a time: registers)
  constexpr int KEYS = 16 * HALVES;
  constexpr int VEC = PAGED ? 1 : (HDP >= 64 ? 4 : HDP / 16);    // consecutive elements of V that a lane takes from a dense row
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const Divide by(a.H / a.Hkv);                                  // (query heads per KV head)
  const int G = by.d;
  int kvh = 0, stream = 0, unit = 0;
  Item it;
  Look look{};
  bool more = false;
  if constexpr (WINDOW) {
    const int wg = (int)blockIdx.x - a.n_checks;
    if (wg < 0) return window_check(a, blockIdx.x);
    if (!window_item<T>(a, wg, G, kvh, it, look)) return;
  } else if constexpr (PAGED) {
    // a workgroup per table row, those of the sequences' own keys, the streams
    const int own = a.n_tiles * a.Hkv, wg = (int)blockIdx.x - a.B;
    if (wg < 0) return check_table(a, blockIdx.x);
    if (wg < own) {
      kvh = wg % a.Hkv;
      if (!own_item(a, wg / a.Hkv, it)) return;
    } else {
      stream = stream_of(a, wg - own);
      unit = stream * a.share;
      if (!stream_item(a, stream, unit, kvh, it)) return;
      more = true;
    }
  } else {
    kvh = blockIdx.x % a.Hkv;
    if (!prompt_item<FROWS>(a, blockIdx.x / a.Hkv, by, reinterpret_cast<int32_t*>(smem), it)) return;
    if (a.kv.k) append_rows<T, FROWS>(a, it, G, kvh);
  }
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int part = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hd = a.hd;
  const float c = rsqrtf((float)hd) * LOG2E_T;
  const int bs = PAGED ? a.kv.block_size : 1;
  do {
    const int r = min(it.rbase + l16, it.R - 1), j = by(r);
    const int lim = min(it.key_end - 1, it.ctx + j);
    const int min_lim = min(it.key_end - 1, it.ctx + by(it.rbase));  // of the rows
    const int max_lim = min(it.key_end - 1, it.ctx + by(min(it.R, it.rbase + FROWS) - 1));
    f32x4 q[NU], O[NU];
    const T* Q = static_cast<const T*>(a.q) + (size_t)(it.m0 + j) * a.q_stride + (size_t)(kvh * G + r - j * G) * hd;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      O[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      q[u] = O[u];
      if (16 * u + 4 * g < hd) {
        const Four<T> x = *reinterpret_cast<const Four<T>*>(Q + 16 * u + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[u][e] = (float)x.x[e] * c;
      }
    }
    float run_m = -INFINITY, run_l = 0.f;
    const int32_t* bt = PAGED ? a.kv.block_tables + (size_t)(more ? first_sharer(a) : it.seq) * a.kv.max_blocks_per_seq : nullptr;
    const bool quads = PAGED && (bs & 3) == 0;                   // four tokens from a multiple of four lie in one block
    const int shift = (bs & (bs - 1)) == 0 ? 31 - __clz(bs) : -1;
    const auto block_of = [&](int key) { return shift >= 0 ? key >> shift : key / bs; };
    const auto page_of = [&](int key) { return ((size_t)min((uint32_t)bt[block_of(key)], (uint32_t)a.kv.num_blocks - 1u) * a.Hkv + kvh) * (size_t)(hd * bs); };
    // (windows: from entry to entry of the list, up to the last that a row sees)
    const int from = WINDOW ? look.i0 + part * HALVES : it.key0 + part * KEYS;
    const int upto = WINDOW ? min(look.i1 - 1, look.entry(max_lim / GRAIN)) : max_lim;
    for (int at = from; at <= upto; at += WINDOW ? KW * HALVES : KW * KEYS) {
      const int last = it.key_end - 1;
      const auto half_key = [&](int h) {                         // the first key of half h
        if constexpr (WINDOW) return at + h < look.i1 ? look.at(at + h) * GRAIN : NO_KEY;
        else return at + 16 * h;
      };
      const auto hidden = [&](int key) {
        if constexpr (WINDOW) return (key > lim) | ((key <= lim - a.window) & (key >= a.sinks));  // (without branches)
        else return key > lim;
      };
      // ---- scores ----
      f32x4 S[HALVES];
      const T* kr[HALVES];
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        S[h] = (f32x4){0.f, 0.f, 0.f, 0.f};
        const int key = min(half_key(h) + l16, last);
        if constexpr (PAGED) kr[h] = static_cast<const T*>(a.kv.k) + page_of(key) + (size_t)(key - block_of(key) * bs) * 8;
        else kr[h] = static_cast<const T*>(a.k) + (size_t)(it.m0 + key) * a.k_stride + (size_t)kvh * hd;
      }
      Four<T> kx[HALVES][NU];
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          const int e0 = HDP == 16 ? min(4 * g, hd - 4) : 16 * u + 4 * g;
          kx[h][u] = *reinterpret_cast<const Four<T>*>(kr[h] + (PAGED ? (e0 >> 3) * (8 * bs) + (e0 & 7) : e0));
          if (HDP == 16 && 4 * g >= hd) kx[h][u] = Four<T>{};    // (heads of 8: zeros, as of the query; 0 times infinity is none)
        }
      // ---- values: asked for ahead of the products ----
      Four<T> vx[HALVES][NU];
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        if constexpr (PAGED) {
          const int key = half_key(h) + 4 * g;
          const size_t page = page_of(min(key, last));
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            const int el = HDP == 16 ? min(l16, hd - 1) : 16 * u + l16;
            const T* v = static_cast<const T*>(a.kv.v) + page + el * bs;
            if (quads) {
              vx[h][u] = *reinterpret_cast<const Four<T>*>(v + (min(key, last & ~3) - block_of(min(key, last)) * bs));
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int ke = min(key + e, last);
                vx[h][u].x[e] = static_cast<const T*>(a.kv.v)[page_of(ke) + (size_t)(el * bs + ke - block_of(ke) * bs)];
              }
            }
            // slots past the last key may hold anything, and 0 times anything has to stay 0
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key + e > last) vx[h][u].x[e] = (T)0.f;
          }
        } else {
          // four keys: four instructions of VEC elements for each of the NU / VEC groups
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const T* v = static_cast<const T*>(a.v) + (size_t)(it.m0 + min(half_key(h) + 4 * g + e, last)) * a.v_stride + (size_t)kvh * hd;
#pragma unroll
            for (int n = 0; n < NU / VEC; ++n) {
              struct __attribute__((aligned(VEC * sizeof(T)))) Some { T x[VEC]; };
              const int el = HDP == 16 ? min(l16, hd - 1) : n * (16 * VEC) + VEC * l16;
              const Some x = *reinterpret_cast<const Some*>(v + el);
#pragma unroll
              for (int i = 0; i < VEC; ++i) vx[h][n * VEC + i].x[e] = x.x[i];
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < HALVES; ++h) S[h] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)kx[h][u].x[e], q[u][e], S[h], 0, 0, 0);
      float tm = -INFINITY;
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          S[h][e] = hidden(half_key(h) + 4 * g + e) ? -INFINITY : S[h][e];
          tm = fmaxf(tm, S[h][e]);
        }
      if (__any(tm > run_m)) {
        uint32_t x, y;
        lane_pair<16>(__float_as_uint(tm), x, y);
        tm = fmaxf(__uint_as_float(x), __uint_as_float(y));
        lane_pair<32>(__float_as_uint(tm), x, y);
        tm = fmaxf(__uint_as_float(x), __uint_as_float(y));
        const float nm = fmaxf(run_m, tm), alpha = nm == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(run_m - nm);
        run_m = nm;
        run_l *= alpha;
#pragma unroll
        for (int u = 0; u < NU; ++u) O[u] *= alpha;
      }
      bool masked;                                               // (uniform) a key that some row does not see
      if constexpr (WINDOW) {
        masked = false;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) masked |= half_key(h) + 15 > min_lim || !(half_key(h) > max_lim - a.window || half_key(h) + 15 < a.sinks);
      } else {
        masked = at + KEYS - 1 > min_lim;
      }
      if (masked) {                                              // values that are not finite, as above
        float odd = 0.f;
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = fmaf((float)vx[h][u].x[e], 0.f, odd);
        if (__any(odd != odd)) {
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float v = (float)vx[h][u].x[e], sees = hidden(half_key(h) + 4 * g + e) ? 0.f : 1.f;
                const bool up = !(v < INFINITY), down = !(v > -INFINITY);
                const f32x4 a = __builtin_amdgcn_mfma_f32_16x16x4f32(up ? 1.f : 0.f, sees, (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                const f32x4 b = __builtin_amdgcn_mfma_f32_16x16x4f32(down ? 1.f : 0.f, sees, (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if (a[i] > 0.f) O[u][i] += INFINITY;
                  if (b[i] > 0.f) O[u][i] -= INFINITY;
                }
                if (up || down) vx[h][u].x[e] = (T)0.f;
                __builtin_amdgcn_sched_barrier(0);
              }
        }
      }
      const float ref = run_m == -INFINITY ? 0.f : run_m;
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(S[h][e] - ref);
          run_l += p;
#pragma unroll
          for (int u = 0; u < NU; ++u) O[u] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)vx[h][u].x[e], p, O[u], 0, 0, 0);
        }
    }
    // the row's sum over the four lane groups
    uint32_t x, y;
    lane_pair<16>(__float_as_uint(run_l), x, y);
    run_l = __uint_as_float(x) + __uint_as_float(y);
    lane_pair<32>(__float_as_uint(run_l), x, y);
    run_l = __uint_as_float(x) + __uint_as_float(y);
    // element of O[u][i] in this lane
    if constexpr (WINDOW) {
      int entry = 0;
      bool lost = false;
      if (a.ranges == 1) lost = window_table_bad(a, it.seq, it.ctx, it.R / G, entry);
      if (__syncthreads_or(lost | ((uint32_t)entry >= (uint32_t)a.kv.num_blocks))) {
        if (tid == 0 && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
        it.R = -it.R;
        window_zeros<T>(a, &it, kvh, G);
        return;
      }
    }
    const auto element = [&](int u, int i) { return u / VEC * (16 * VEC) + VEC * (4 * g + i) + u % VEC; };
    float* s_o = reinterpret_cast<float*>(smem);               // [KW][16][LD]
    float2* s_ml = reinterpret_cast<float2*>(smem + KW * 16 * LD * 4);
    __syncthreads();                                           // (the search, or the piece before, is through with the LDS)
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_o[(part * 16 + l16) * LD + element(u, i)] = O[u][i];
    if (g == 0) s_ml[part * 16 + l16] = make_float2(run_m, run_l);
    __syncthreads();
    for (int i = tid; i < 16 * (HDP / 4); i += 256) {
      const int row = i / (HDP / 4), e0 = i % (HDP / 4) * 4, rr = it.rbase + row;
      if (rr >= it.R || e0 >= hd) continue;
      float top = -INFINITY, l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) top = fmaxf(top, s_ml[w * 16 + row].x);
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 ml = s_ml[w * 16 + row];
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        l += ml.y * f;
        o += *reinterpret_cast<const f32x4*>(s_o + (w * 16 + row) * LD + e0) * f;
      }
      const int jj = by(rr), m = it.m0 + jj, h = kvh * G + rr - jj * G;
      if (PAGED && !(WINDOW && a.ranges == 1)) {
        *reinterpret_cast<f32x4*>(a.o_part + (((size_t)it.slot * a.M + m) * a.H + h) * hd + e0) = o;
        if (e0 == 0) *reinterpret_cast<float2*>(a.ml_part + (((size_t)it.slot * a.M + m) * a.H + h) * 2) = make_float2(top, l);
      } else {
        if (WINDOW && a.stats && e0 == 0) *reinterpret_cast<float2*>(a.stats + ((size_t)m * a.H + h) * 2) = make_float2(top, l);
        Four<T> w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.x[e] = (T)(o[e] / l);
        *reinterpret_cast<Four<T>*>(static_cast<T*>(a.out) + ((size_t)m * a.H + h) * hd + e0) = w;
      }
    }
  } while (!WINDOW && more && stream_item(a, stream, unit, kvh, it));
}

// ------------------------------------------------------------------------------------------
// a batch that shares a prefix
// ------------------------------------------------------------------------------------------
// Every row sees the shared keys [0, P) and its own sequence's from P on.  The shared part is one dense product: all rows of the batch,
// stacked, against keys that are read once per tile of rows (stream_item).  The rest goes sequence by sequence, in ranges of `chunk`
// keys, from a work list.  Each piece leaves an unnormalised output with its reference and sum per row in a slot of its own,
// and a row's slots are put together at the end.
//
// prefix_plan_kernel (one workgroup; more than 64 sequences): the rows' sequences, who takes part, the first sharer, and the list of items.  Up to 64 every
// workgroup finds its item by itself (own_item), and the merge its rows' sequences, which saves a launch, 5 us.
__global__ void __launch_bounds__(1024) prefix_plan_kernel(PrefixPlan p) {
  __shared__ int s_rows[16], s_items[16], s_bad, s_first;
  const PrefixBatch& c = p.batch;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) { s_bad = 0; s_first = c.B; }
  __syncthreads();
  int flags = 0;
  const auto length = [&](int b) {
    const int k = c.spec_len[b];
    return k >= 0 && k < c.max_q ? k + 1 : -1;
  };
  // lengths first: rows that do not add up to the host's, or a run longer than its longest, disable the batch
  int rows = 0;
  bool off = false;
  for (int b = tid; b < c.B; b += 1024) {
    const int q = length(b);
    if (c.ctx_lens[b] >= c.prefix_len) atomicMin(&s_first, b);
    off |= q < 0;
    rows += max(q, 0);
  }
  rows = wave_sum_i(rows);
  if (lane == 0) s_rows[wave] = rows;
  if (off) s_bad = 1;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < 16; ++w) total += s_rows[w];
  if (tid == 0) *p.first = s_first < c.B ? s_first : 0;
  const bool batch = s_bad == 0 && total == c.M;
  if (!batch) flags |= MN_DEV_SPEC_LEN;
  int4* items = reinterpret_cast<int4*>(p.items);
  int row_at = 0, item_at = 0;
  for (int b0 = 0; b0 < c.B; b0 += 1024) {
    const int b = b0 + tid, q = batch && b < c.B ? length(b) : 0;
    int ctx = 0, ranges = 0, rts = 0;
    if (q > 0) {
      ctx = c.ctx_lens[b];
      if (ctx < c.prefix_len || (long)ctx + q > c.max_ctx) {
        flags |= MN_DEV_CTX;
      } else {
        ranges = (ctx + q - c.prefix_len + c.chunk - 1) / c.chunk;
        rts = (c.G * q + c.tile_rows - 1) / c.tile_rows;
      }
    }
    const int rows_incl = wave_scan_i(q), items_incl = wave_scan_i(ranges * rts);
    __syncthreads();
    if (lane == 63) { s_rows[wave] = rows_incl; s_items[wave] = items_incl; }
    __syncthreads();
    int row0 = row_at + rows_incl - q, at = item_at + items_incl - ranges * rts;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) { row0 += s_rows[w]; at += s_items[w]; }
      row_at += s_rows[w];
      item_at += s_items[w];
    }
    for (int j = 0; j < q; ++j) p.row_meta[row0 + j] = make_int2(b, ranges);
    for (int rt = 0; rt < rts; ++rt)
      for (int s = 0; s < ranges; ++s, ++at) {
        const int k0 = c.prefix_len + s * c.chunk;
        items[2 * at] = make_int4(row0, c.G * q, rt * c.tile_rows, k0);
        items[2 * at + 1] = make_int4(min(k0 + c.chunk, ctx + q), ctx, b, p.prefix_slots + s);
      }
  }
  if (!batch)
    for (int m = tid; m < c.M; m += 1024) p.row_meta[m] = make_int2(0, 0);
  for (int i = item_at + tid; i < p.max_items; i += 1024) items[2 * i] = make_int4(0, 0, 0, 0);
  if (flags && p.status) atomicOr(p.status, flags);
}

// Four elements of a row of one head per thread; several slots are asked for at once.  GROUPS threads share them where there are few rows
// and many slots (6 rows of 64 heads, 33 slots: 4.6 us, with one 10).  Bound by
// HBM where there are many rows: 576 rows of 64 heads of 128, 71 MB of parts, 16 us.
constexpr int AT_ONCE = 4;
// The parts of row-head mh in the slots at(0) .. at(n - 1), put together (o, l, top: its output, its sum and their reference).  False: a
// thread of another group than the first, which has no more to do.
template <int GROUPS, typename F>
__device__ __forceinline__ bool sum_slots(const float* o_part, const float* ml_part, size_t heads, int hd, size_t i, size_t mh, int n, F at_slot, f32x4& o,
                                          float& l, float& top) {
  constexpr int WIDE = 256 / GROUPS;
  __shared__ float s_top[GROUPS][WIDE], s_l[GROUPS][WIDE];
  __shared__ f32x4 s_o[GROUPS][WIDE];
  const int group = threadIdx.x / WIDE, lane_at = threadIdx.x % WIDE;
  o = (f32x4){0.f, 0.f, 0.f, 0.f};
  l = 0.f;
  top = -INFINITY;
  for (int s0 = group; s0 < n; s0 += AT_ONCE * GROUPS) {
    float2 ml[AT_ONCE];
    f32x4 v[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int at = at_slot(min(s0 + u * GROUPS, n - 1));
      ml[u] = *reinterpret_cast<const float2*>(ml_part + (at * heads + mh) * 2);
      v[u] = *reinterpret_cast<const f32x4*>(o_part + at * heads * hd + 4 * i);
    }
    float nm = top;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) nm = fmaxf(nm, ml[u].x);
    const float ref = nm == -INFINITY ? 0.f : nm, keep = __builtin_amdgcn_exp2f(top - ref);
    l *= keep;
    o *= keep;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const bool in = s0 + u * GROUPS < n;                       // (what is not finite counts once, and not at all times 0)
      const float w = in ? __builtin_amdgcn_exp2f(ml[u].x - ref) : 0.f;
      l += ml[u].y * w;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += in ? v[u][e] * w : 0.f;
    }
    top = nm;
  }
  if constexpr (GROUPS > 1) {
    s_top[group][lane_at] = top;
    s_l[group][lane_at] = l;
    s_o[group][lane_at] = o;
    __syncthreads();
    if (group > 0) return false;
    float nm = top;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) nm = fmaxf(nm, s_top[g][lane_at]);
    const float ref = nm == -INFINITY ? 0.f : nm, keep = __builtin_amdgcn_exp2f(top - ref);
    l *= keep;
    o *= keep;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) {
      const float w = __builtin_amdgcn_exp2f(s_top[g][lane_at] - ref);
      l += s_l[g][lane_at] * w;
      o += s_o[g][lane_at] * w;
    }
    top = nm;
  }
  return true;
}

template <typename T, int GROUPS>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PrefixMerge p, T* __restrict__ out) {
  constexpr int WIDE = 256 / GROUPS;
  const size_t heads = (size_t)p.M * p.H;
  const int per = p.hd / 4;
  const size_t i = min((size_t)blockIdx.x * WIDE + threadIdx.x % WIDE, heads * per - 1), mh = i / per;  // (past the end: the last ones once more)
  const int m = (int)(mh / p.H), h = (int)(mh - (size_t)m * p.H), G = p.H / p.Hkv, kvh = h / G;
  int2 meta = make_int2(0, 0);                                   // sequence, ranges of its own keys
  if (p.row_meta) {
    meta = p.row_meta[m];
  } else {
    const Share s = lane_share(p.batch);
    // (the rows of the wave, one after the other: few, and one unless a row is very short)
    const int m0 = __builtin_amdgcn_readfirstlane(m), m1 = __builtin_amdgcn_readlane(m, 63);
    for (int r = m0; r <= m1; ++r) {
      const uint64_t has = __ballot(s.q > 0 && r >= s.row0 && r < s.row0 + s.q);
      if (has == 0) continue;
      const int b = __ffsll((unsigned long long)has) - 1, ranges = __builtin_amdgcn_readlane(s.ranges, b);
      if (m == r) meta = make_int2(b, ranges);
    }
  }
  const bool takes_part = meta.y > 0 && !p.seq_bad[meta.x];
  int shared = 0;                                                // streams that met the row's tile
  if (takes_part && p.n_units > 0) {
    const int first = (kvh * p.row_tiles + (m * G + h - kvh * G) / p.batch.tile_rows) * p.prefix_units;
    shared = (first + p.prefix_units - 1) / p.share - first / p.share + 1;
  }
  f32x4 o;
  float l, top;
  if (!sum_slots<GROUPS>(p.o_part, p.ml_part, heads, p.hd, i, mh, takes_part ? shared + meta.y : 0,
                         [&](int s) { return s < shared ? s : p.prefix_slots + s - shared; }, o, l, top))
    return;
  const float inv = takes_part ? 1.f / l : 0.f;                  // (a row whose scores are all -inf is no number, as without a prefix)
#pragma unroll
  for (int e = 0; e < 4; ++e) out[4 * i + e] = (T)(o[e] * inv);
}

// ------------------------------------------------------------------------------------------
// windows
// ------------------------------------------------------------------------------------------
// A row tile's keys are a list of granules (Look), in one range where the tiles fill the chip by themselves: the workgroup then writes
// the rows' outputs, and there is no second launch.  Otherwise in several, whose parts window_merge_kernel puts together.
// One row of 24 sequences behind 4096 tokens of 64/8 heads of 128: 63 us, 385 MB at 6.1 TB/s, and 5 for the merge.  Chunks of 1500 to 2500 tokens
// behind 8192: 1080 us, 1.02 PFLOP/s, the matrix pipe's.  Four prompts of 1500 to 6000 tokens, 40 heads, a window of 1024: 380 us, 0.67 PFLOP/s: the
// tiles' steps are 278 GFLOP for 256 of visible pairs (273 us at the chunks' rate), and 4480 workgroups pay their way in and out for 18 double steps each.
//
// window_plan_kernel (one workgroup; more than 64 sequences): the tiles' records (window_tile), and per row its sequence (-1: takes no part),
// context, rows and first row.  A thread writes its sequence's rows one after the other, and only the merge reads them: 65 prompts of 1000 tokens 44 us
// ahead of 1120 (40 heads of 128), of 200 tokens 11 ahead of 31 (12 of 64).
__global__ void __launch_bounds__(1024) window_plan_kernel(WindowPlan p) {
  __shared__ int s_rows[16], s_tiles[16], s_bad;
  const PrefixBatch& c = p.batch;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  const auto length = [&](int b) {
    const int k = c.spec_len[b];
    return k >= 0 && k < c.max_q ? k + 1 : -1;
  };
  const auto tiles_of = [&](int q) { return (int)(((long)c.G * q + c.tile_rows - 1) / c.tile_rows); };
  // lengths first: rows or tiles that do not add up to the host's, or a run longer than its longest, disable the batch
  int rows = 0, tiles = 0;
  bool off = false;
  for (int b = tid; b < c.B; b += 1024) {
    const int q = length(b);
    off |= q < 0;
    rows += max(q, 0);
    tiles += tiles_of(max(q, 0));
  }
  rows = wave_sum_i(rows);
  tiles = wave_sum_i(tiles);
  if (lane == 0) { s_rows[wave] = rows; s_tiles[wave] = tiles; }
  if (off) s_bad = 1;
  __syncthreads();
  int total = 0, total_tiles = 0;
  for (int w = 0; w < 16; ++w) { total += s_rows[w]; total_tiles += s_tiles[w]; }
  const bool batch = s_bad == 0 && total == c.M && total_tiles == p.n_tiles;
  int flags = batch ? 0 : MN_DEV_SPEC_LEN;
  int4* items = reinterpret_cast<int4*>(p.items);
  if (!batch) {
    for (int m = tid; m < c.M; m += 1024) p.row_meta[m] = make_int4(-1, 0, 0, 0);
    for (int i = tid; i < p.n_tiles; i += 1024) items[2 * i] = items[2 * i + 1] = make_int4(0, 0, 0, 0);
  }
  int row_at = 0, item_at = 0;
  for (int b0 = 0; batch && b0 < c.B; b0 += 1024) {
    const int b = b0 + tid, q = b < c.B ? length(b) : 0, n = tiles_of(q);
    const int rows_incl = wave_scan_i(q), tiles_incl = wave_scan_i(n);
    __syncthreads();
    if (lane == 63) { s_rows[wave] = rows_incl; s_tiles[wave] = tiles_incl; }
    __syncthreads();
    int row0 = row_at + rows_incl - q, at = item_at + tiles_incl - n;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) { row0 += s_rows[w]; at += s_tiles[w]; }
      row_at += s_rows[w];
      item_at += s_tiles[w];
    }
    if (b >= c.B) continue;
    const int ctx = c.ctx_lens[b];
    const bool fits = window_fits(c, ctx, q);
    if (!fits) flags |= MN_DEV_CTX;
    for (int j = 0; j < q; ++j) p.row_meta[row0 + j] = make_int4(fits ? b : -1, ctx, q, row0);
    for (int i = 0; i < n; ++i) {
      items[2 * (at + i)] = make_int4(row0, c.G * q * (fits ? 1 : -1), (n - 1 - i) * c.tile_rows, 0);
      items[2 * (at + i) + 1] = make_int4(0, ctx, b, 0);
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

template <typename T, int GROUPS>
__global__ void __launch_bounds__(256) window_merge_kernel(TileArgs a, const int4* __restrict__ row_meta, T* __restrict__ out) {
  constexpr int WIDE = 256 / GROUPS;
  const size_t heads = (size_t)a.M * a.H;
  const int per = a.hd / 4;
  const size_t i = min((size_t)blockIdx.x * WIDE + threadIdx.x % WIDE, heads * per - 1), mh = i / per;  // (past the end: the last ones once more)
  const int m = (int)(mh / a.H), h = (int)(mh - (size_t)m * a.H), G = a.H / a.Hkv;
  int4 meta = make_int4(-1, 0, 0, 0);                            // sequence, context, rows, first row
  if (row_meta) {
    meta = row_meta[m];
  } else {
    const WindowShare s = lane_window(a.batch, a.n_tiles);
    const int m0 = __builtin_amdgcn_readfirstlane(m), m1 = __builtin_amdgcn_readlane(m, 63);
    for (int r = m0; r <= m1; ++r) {
      const uint64_t has = __ballot(!s.off && s.flags == 0 && r >= s.row0 && r < s.row0 + s.q);
      if (has == 0) continue;
      const int b = __ffsll((unsigned long long)has) - 1;
      const int4 x = make_int4(b, __builtin_amdgcn_readlane(s.ctx, b), __builtin_amdgcn_readlane(s.q, b), __builtin_amdgcn_readlane(s.row0, b));
      if (m == r) meta = x;
    }
  }
  const bool takes_part = meta.x >= 0 && !a.seq_bad[meta.x];
  int ranges = 0;
  if (takes_part) {
    const int R = G * meta.z, rbase = ((m - meta.w) * G + h % G) / a.batch.tile_rows * a.batch.tile_rows;
    int entries;
    look_from(a, meta.y + rbase / G, meta.y + (min(R, rbase + a.batch.tile_rows) - 1) / G, entries);
    ranges = (entries + a.batch.chunk - 1) / a.batch.chunk;
  }
  f32x4 o;
  float l, top;
  if (!sum_slots<GROUPS>(a.o_part, a.ml_part, heads, a.hd, i, mh, ranges, [](int s) { return s; }, o, l, top)) return;
  const float inv = takes_part ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[4 * i + e] = (T)(o[e] * inv);
  if (a.stats && i % per == 0) *reinterpret_cast<float2*>(a.stats + 2 * mh) = takes_part ? make_float2(top, l) : make_float2(0.f, 0.f);
}

// ------------------------------------------------------------------------------------------
// launch
// ------------------------------------------------------------------------------------------
static bool tile_mfma(const TileArgs& a, bool paged) {
  return a.dtype == MN_DT_BF16 && (a.hd == 64 || a.hd == 128) && (!paged || a.kv.block_size == PAGE);
}

// Rows of a workgroup's tile for a call whose longest stack and number of stack rows per KV head are given.
int prompt_tile_rows(const TileArgs& a, long stack_rows) {
  if (!tile_mfma(a, a.kv.k != nullptr)) return FROWS;
  if (const int f = MN_TUNE("MN_TILE", 0)) return f;
  // 128 rows where that fills the chip, 64 otherwise: two workgroups of 128 rows fit a CU, and three with heads of 64, where it pays
  // from five sixths on.  Measured, 128 against 64 rows, heads of 128: 8192 tokens of 64/8 heads 1050 and 1390 us, 8 prompts of
  // 60 to 1500 tokens of 40 heads 155 and 197, 1024 tokens of 64/8 heads (512 workgroups) 33 and 35, of 40 heads (320) 31 and
  // 25.  12 heads of 64: 32 prompts of 1000 95 and 116, 8 of 1000 (750) 28 and 31, 8 of 300 to 1200 (562) 22 and 20, 300
  // tokens 9.3 and 8.0.
  return stack_rows * a.Hkv >= (a.hd == 64 ? 640 : 512) * 128 ? 128 : 64;
}

template <typename K>
static hipError_t allow_lds(K kernel, size_t bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <bool PAGED, bool WINDOW>
static unsigned tile_workgroups(const TileArgs& a) {
  const unsigned tiles = (unsigned)a.n_tiles * (unsigned)a.Hkv;
  return WINDOW ? tiles * (unsigned)a.ranges + (unsigned)a.n_checks : tiles + (PAGED ? (unsigned)(a.n_streams + a.B) : 0u);
}

template <int HDIM, int CT, bool PAGED, bool WINDOW>
static hipError_t launch_mfma_as(const TileArgs& a, hipStream_t st) {
  constexpr size_t lds = STAGES * TileStage<HDIM>::BYTES;
  static std::once_flag once;
  static hipError_t err = hipSuccess;
  std::call_once(once, [] { err = allow_lds(tile_mfma_kernel<HDIM, CT, 4, PAGED, WINDOW>, lds); });
  if (err != hipSuccess) return err;
  tile_mfma_kernel<HDIM, CT, 4, PAGED, WINDOW><<<tile_workgroups<PAGED, WINDOW>(a), 256, lds, st>>>(a);
  return hipSuccess;
}
template <bool PAGED, bool WINDOW = false>
static hipError_t launch_mfma(const TileArgs& a, int tile_rows, hipStream_t st) {
  if (a.hd == 128) return tile_rows == 128 ? launch_mfma_as<128, 2, PAGED, WINDOW>(a, st) : launch_mfma_as<128, 1, PAGED, WINDOW>(a, st);
  return tile_rows == 128 ? launch_mfma_as<64, 2, PAGED, WINDOW>(a, st) : launch_mfma_as<64, 1, PAGED, WINDOW>(a, st);
}

template <typename T, int HDP, bool PAGED, bool WINDOW>
static hipError_t launch_f32(const TileArgs& a, hipStream_t st) {
  constexpr size_t parts = (size_t)KW * 16 * ((HDP + 4) * 4 + 8);
  static std::once_flag once;
  static hipError_t err = hipSuccess;
  std::call_once(once, [] { err = allow_lds(tile_f32_kernel<T, HDP, PAGED, WINDOW>, parts); });
  if (err != hipSuccess) return err;
  const size_t list = PAGED || a.B <= 64 ? 0 : (size_t)a.B * 4;  // (the search's numbers)
  tile_f32_kernel<T, HDP, PAGED, WINDOW><<<tile_workgroups<PAGED, WINDOW>(a), 64 * KW, parts > list ? parts : list, st>>>(a);
  return hipSuccess;
}

template <typename T, bool PAGED, bool WINDOW = false>
static hipError_t launch_f32_hd(const TileArgs& a, hipStream_t st) {
  switch (a.hd) {
    case 8: case 16: return launch_f32<T, 16, PAGED, WINDOW>(a, st);
    case 32: return launch_f32<T, 32, PAGED, WINDOW>(a, st);
    case 64: return launch_f32<T, 64, PAGED, WINDOW>(a, st);
    case 128: return launch_f32<T, 128, PAGED, WINDOW>(a, st);
    default: return launch_f32<T, 256, PAGED, WINDOW>(a, st);
  }
}

hipError_t launch_prompt(const TileArgs& a, hipStream_t st) {
  if (!tile_mfma(a, a.kv.k != nullptr)) return a.dtype == MN_DT_BF16 ? launch_f32_hd<f16_t, false>(a, st) : launch_f32_hd<float, false>(a, st);
  return launch_mfma<false>(a, a.tile_rows, st);
}


// Shape of a shared-prefix launch, from what the host knows.
constexpr int STREAMS = 512;          // two workgroups per CU (64 rows of heads of 64: four)
constexpr int MIN_SHARE = 4;          // units of a stream at least: a workgroup's lead-in is worth about as much
constexpr int MAX_SLOTS = 33;         // of a tile of rows
constexpr int MAX_RANGES = 16;        // of a sequence's own keys
struct PrefixShape {
  int tile_rows, row_tiles, units, n_units, share, n_streams, slots, chunk, ranges;
};
static int prefix_tile_rows(const TileArgs& a, int M, int units) {
  if (!tile_mfma(a, true)) return FROWS;
  if (const int f = MN_TUNE("MN_TILE", 0)) return f;
  // 128 rows where a sequence's run fills most of them, and with heads of 128 where more than 64 rows meet enough of the prefix for
  // seven units per stream; 64 otherwise.  Measured, 128 against 64 rows.  Runs of 17 x 8 rows behind 512 + 1000 keys, 8 sequences
  // 36 and 39 us; of 131 x 8, 2 sequences 52 and 64, 32 sequences without a prefix 335 and 432; of 201 rows of 12 heads of 64, 8
  // sequences 41 and 45; of 9 x 8 behind 2048 + 300, 16 sequences 44 and 41.  One row each, 64 x 8 rows behind 16384 keys
  // 60 and 66; 16 sequences of 5 x 8 rows behind 4096 39 and 35; heads of 64, 128 sequences of 5 rows behind 8192 61 and 54.
  const long G = a.H / a.Hkv;
  if (G * a.batch.max_q >= 96) return 128;
  return a.hd == 128 && M * G > 64 && (M * G + 127) / 128 * a.Hkv * units >= 7 * STREAMS ? 128 : 64;
}
static PrefixShape prefix_shape(const TileArgs& a, int M, int max_ctx) {
  PrefixShape s{};
  const long G = a.H / a.Hkv;
  s.units = (a.batch.prefix_len + TKEYS - 1) / TKEYS;
  s.tile_rows = prefix_tile_rows(a, M, s.units);
  s.row_tiles = (int)((M * G + s.tile_rows - 1) / s.tile_rows);
  s.n_units = s.row_tiles * a.Hkv * s.units;
  const int streams = s.tile_rows == 64 && a.hd == 64 ? 2 * STREAMS : STREAMS;
  s.share = (s.n_units + streams - 1) / streams;
  const int by_slots = (s.units + MAX_SLOTS - 3) / (MAX_SLOTS - 2);
  const int least = s.units < 1 ? 1 : (s.units < MIN_SHARE ? s.units : MIN_SHARE);  // (a stream of several short tiles would only be longer)
  if (s.share < least) s.share = least;
  if (s.share < by_slots) s.share = by_slots;
  s.n_streams = (s.n_units + s.share - 1) / s.share;
  s.slots = s.units > 0 ? (s.units - 1) / s.share + 2 : 0;
  const int rest = max_ctx - a.batch.prefix_len, want = (long)a.B * a.Hkv >= 256 ? 1024 : 256;
  s.ranges = (rest + want - 1) / want;
  if (s.ranges > MAX_RANGES) s.ranges = MAX_RANGES;
  if (s.ranges < 1) s.ranges = 1;
  s.chunk = ((rest + s.ranges - 1) / s.ranges + TKEYS - 1) / TKEYS * TKEYS;
  return s;
}
// Workgroups of a call's largest launch.
long prefix_workgroups(const TileArgs& a) {
  const PrefixShape s = prefix_shape(a, a.M, a.batch.max_ctx);
  const long tiles = ((long)a.M * (a.H / a.Hkv) / s.tile_rows + a.B) * s.ranges * a.Hkv + s.n_streams + a.B, merge = ((long)a.M * a.H * (a.hd / 4) + 255) / 256;
  return tiles > merge ? tiles : merge;
}
struct PrefixLayout {
  size_t meta, bad, items, o_part, ml_part, total;
  size_t max_items, slot_rows;
};
// (everything here grows with B, M and max_ctx: a workspace for the largest batch serves every smaller one)
static PrefixLayout prefix_layout(int B, int M, int H, int Hkv, int hd, int prefix_len, int max_ctx) {
  PrefixLayout L;
  const long G = H / Hkv, ranges = max_ctx - prefix_len > 256 ? MAX_RANGES : 1;
  // slots of a tile: units / share + 2 with share >= row tiles * KV heads * units / streams, and MAX_SLOTS; row tiles >= M G / tile rows, streams * tile rows <= STREAMS * 128
  const long slots_a = (long)MAX_SLOTS * M, slots_b = (long)STREAMS * 128 / H + 3l * M;
  L.slot_rows = (size_t)((slots_a < slots_b ? slots_a : slots_b) + ranges * M);
  L.max_items = (size_t)(((G * M + 15) / 16 + B) * ranges);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 4095) & ~(size_t)4095; return o; };
  L.meta = take((size_t)M * 8); L.bad = take((size_t)(B + 1) * 4); L.items = take(L.max_items * 32);
  L.ml_part = take(L.slot_rows * H * 2 * 4);
  L.o_part = take(L.slot_rows * H * hd * 4);
  L.total = at;
  return L;
}
size_t prefix_workspace_bytes(int B, int M, int H, int Hkv, int hd, int prefix_len, int max_ctx) {
  return prefix_layout(B, M, H, Hkv, hd, prefix_len, max_ctx).total;
}
bool prefix_fits(int M, int H, int Hkv, int prefix_len) {
  return (((long)M * (H / Hkv) + 15) / 16) * Hkv * (((long)prefix_len + TKEYS - 1) / TKEYS) < (1l << 30);
}

template <typename T>
static void launch_prefix_merge(const PrefixMerge& g, T* out, hipStream_t st) {
  const size_t threads = (size_t)g.M * g.H * (g.hd / 4);
  // (8 threads for the slots of a row where that still leaves no more than two workgroups per CU)
  if (g.prefix_slots >= 8 && threads * 8 <= 512 * 256) prefix_merge_kernel<T, 8><<<(unsigned)((threads + 31) / 32), 256, 0, st>>>(g, out);
  else prefix_merge_kernel<T, 1><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(g, out);
}

// a.batch: spec_len, ctx_lens, max_q (the longest run of rows), max_ctx and prefix_len are the caller's
hipError_t launch_prefix(TileArgs a, void* workspace, hipStream_t st) {
  const int max_ctx = a.batch.max_ctx;
  const PrefixLayout L = prefix_layout(a.B, a.M, a.H, a.Hkv, a.hd, a.batch.prefix_len, max_ctx);
  const PrefixShape s = prefix_shape(a, a.M, max_ctx);
  unsigned char* w = static_cast<unsigned char*>(workspace);
  a.batch.B = a.B; a.batch.M = a.M; a.batch.G = a.H / a.Hkv; a.batch.tile_rows = s.tile_rows; a.batch.chunk = s.chunk;
  a.seq_bad = reinterpret_cast<int32_t*>(w + L.bad);
  a.n_tiles = (int)(((long)a.M * a.batch.G / s.tile_rows + a.B) * s.ranges);
  a.prefix_slots = s.slots; a.prefix_units = s.units; a.n_units = s.n_units; a.share = s.share; a.n_streams = s.n_streams;
  a.row_tiles = s.row_tiles; a.tile_rows = s.tile_rows;
  a.o_part = reinterpret_cast<float*>(w + L.o_part); a.ml_part = reinterpret_cast<float*>(w + L.ml_part);
  int2* meta = nullptr;
  if (a.B > 64) {
    meta = reinterpret_cast<int2*>(w + L.meta);
    int32_t* items = reinterpret_cast<int32_t*>(w + L.items);
    a.items = items;
    prefix_plan_kernel<<<1, 1024, 0, st>>>(PrefixPlan{a.batch, s.slots, a.n_tiles, items, meta, a.seq_bad + a.B, a.status});
  }
  hipError_t e;
  if (!tile_mfma(a, true)) e = a.dtype == MN_DT_BF16 ? launch_f32_hd<f16_t, true>(a, st) : launch_f32_hd<float, true>(a, st);
  else e = launch_mfma<true>(a, s.tile_rows, st);
  if (e != hipSuccess) return e;
  const PrefixMerge g{a.o_part, a.ml_part, meta, a.seq_bad, a.batch, a.M, a.H, a.Hkv, a.hd, s.slots, s.units, s.n_units, s.share, s.row_tiles};
  if (a.dtype == MN_DT_BF16) launch_prefix_merge(g, static_cast<f16_t*>(a.out), st);
  else launch_prefix_merge(g, static_cast<float*>(a.out), st);
  return hipSuccess;
}

// Shape of a windowed launch.  Rows of a tile: 128 (each key is staged half as often) where tiles of 64 would be more than the chip holds at
// once.  8 runs of 80 rows behind windows of 1024, 40 heads of 128: 45 us, tiles of 64 62; of 128 rows 52 and 56; but 8 runs of 112 rows behind
// windows of 4096, 64/8 heads: 42 and 38; 2 prompts of 80 rows, 40 heads: 10 and 7.5.  Ranges are as many as workgroups fit: halved, 4 sequences
// of one row behind 4096, 64/8 heads 17.9 -> 19.0, 8 of 96 rows 37 -> 40; quartered 25 and 61.
constexpr int WINDOW_RANGES = 16;      // of a tile's keys at most
constexpr int MIN_GRAINS = 16;         // granules of a range at least
int window_tile_rows(const TileArgs& a) {
  if (!tile_mfma(a, true)) return FROWS;
  if (const int f = MN_TUNE("MN_TILE", 0)) return f;
  const long rows = (long)(a.H / a.Hkv) * a.batch.max_q;
  return rows > 64 && (rows + 63) / 64 * a.B * a.Hkv > STREAMS ? 128 : 64;
}
struct WindowShape {
  int ranges, chunk;
};
static WindowShape window_shape(const TileArgs& a) {
  const long tokens = (a.tile_rows + a.H / a.Hkv - 1) / (a.H / a.Hkv) + 1;
  // granules that the longest tile meets
  long seen = a.window < a.batch.max_ctx ? a.window : a.batch.max_ctx;
  seen = (seen + tokens + a.sinks) / GRAIN + 3;
  const long all = (a.batch.max_ctx + GRAIN - 1) / GRAIN;
  if (seen > all) seen = all;
  const int target = MN_TUNE("MN_WGS", STREAMS);
  long ranges = target / ((long)a.n_tiles * a.Hkv);
  const long by_keys = seen / MIN_GRAINS;
  if (ranges > by_keys) ranges = by_keys;
  if (ranges > WINDOW_RANGES) ranges = WINDOW_RANGES;
  if (ranges < 1) ranges = 1;
  const int chunk = (int)((seen + ranges - 1) / ranges + 1) / 2 * 2;
  return WindowShape{(int)((seen + chunk - 1) / chunk), chunk};
}
struct WindowLayout {
  size_t bad, meta, items, ml_part, o_part, total;
};
// (everything here grows with B and M: a workspace for the largest batch serves every smaller one)
static WindowLayout window_layout(int B, int M, int H, int Hkv, int hd) {
  WindowLayout L;
  const long G = H / Hkv;
  // ranges * tiles * KV heads <= STREAMS where there is more than one, and a tile has 128 rows at most
  const long a = (long)WINDOW_RANGES * M * H, b = (long)STREAMS * 128;
  const size_t rows = (size_t)(a < b ? a : b);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 4095) & ~(size_t)4095; return o; };
  L.bad = take((size_t)B * 4);
  L.meta = take(B > 64 ? (size_t)M * 16 : 0);
  L.items = take(B > 64 ? ((size_t)((G * M + 15) / 16) + B) * 32 : 0);
  L.ml_part = take(rows * 8);
  L.o_part = take(rows * hd * 4);
  L.total = at;
  return L;
}
size_t window_workspace_bytes(int B, int M, int H, int Hkv, int hd) { return window_layout(B, M, H, Hkv, hd).total; }
// Workgroups of a call's largest launch (a.n_tiles, a.tile_rows set).
long window_workgroups(const TileArgs& a) {
  const WindowShape s = window_shape(a);
  const long tiles = (long)a.n_tiles * a.Hkv * s.ranges + a.B, merge = s.ranges > 1 ? ((long)a.M * a.H * (a.hd / 4) + 31) / 32 : 0;
  return tiles > merge ? tiles : merge;
}

template <typename T>
static void launch_window_merge(const TileArgs& a, const int4* meta, hipStream_t st) {
  const size_t threads = (size_t)a.M * a.H * (a.hd / 4);
  if (a.ranges >= 8 && threads * 8 <= 512 * 256) window_merge_kernel<T, 8><<<(unsigned)((threads + 31) / 32), 256, 0, st>>>(a, meta, static_cast<T*>(a.out));
  else window_merge_kernel<T, 1><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(a, meta, static_cast<T*>(a.out));
}

// a.batch: spec_len, ctx_lens, max_q and max_ctx are the caller's, as are tile_rows and n_tiles (by window_tile_rows)
hipError_t launch_window(TileArgs a, void* workspace, hipStream_t st) {
  const WindowLayout L = window_layout(a.B, a.M, a.H, a.Hkv, a.hd);
  const WindowShape s = window_shape(a);
  unsigned char* w = static_cast<unsigned char*>(workspace);
  a.batch.B = a.B; a.batch.M = a.M; a.batch.G = a.H / a.Hkv; a.batch.tile_rows = a.tile_rows; a.batch.chunk = s.chunk;
  a.ranges = s.ranges;
  a.n_checks = s.ranges > 1 ? a.B : 0;
  a.keep_keys = a.n_tiles > a.B;                                 // (other tiles of the sequence read them as well)
  a.seq_bad = reinterpret_cast<int32_t*>(w + L.bad);
  a.o_part = reinterpret_cast<float*>(w + L.o_part); a.ml_part = reinterpret_cast<float*>(w + L.ml_part);
  int4* meta = nullptr;
  if (a.B > 64) {
    meta = reinterpret_cast<int4*>(w + L.meta);
    int32_t* items = reinterpret_cast<int32_t*>(w + L.items);
    a.items = items;
    window_plan_kernel<<<1, 1024, 0, st>>>(WindowPlan{a.batch, a.n_tiles, items, meta, a.status});
  }
  hipError_t e;
  if (!tile_mfma(a, true)) e = a.dtype == MN_DT_BF16 ? launch_f32_hd<f16_t, true, true>(a, st) : launch_f32_hd<float, true, true>(a, st);
  else e = launch_mfma<true, true>(a, a.tile_rows, st);
  if (e != hipSuccess || a.ranges == 1) return e;
  if (a.dtype == MN_DT_BF16) launch_window_merge<f16_t>(a, meta, st);
  else launch_window_merge<float>(a, meta, st);
  return hipSuccess;
}

}  // namespace mn
