// What attention has looked at, and what may go: the weight that every cached token has been given, per layer, sequence and KV head, and
// the eviction of those with the least of it.
//
//   mass[i] += sum over rows r and the query heads of the KV head of p_ri = 2^(c s_ri - m_r) / l_r,
// with the rows' statistics (m_r, l_r) as their attention left them: one product, one exponential, sums along the rows.  A
// token's key may stand in any slot of its sequence, each head's in another, since its rotation is in it and attention asks for no
// order: so a head that loses tokens fills their slots with those that it keeps from behind the new end, and nothing else moves.
//
//  * weigh_mfma_kernel, weigh_stream_kernel  fp16, head_dim 64 or 128, blocks of 16 tokens: many rows, few rows.
//  * weigh_f32_kernel   every other type, head_dim and block size.
//  * evict_plan_kernel  a workgroup per layer, slot and head: who stays, and who goes where.
//  * evict_pages_kernel, evict_move_kernel  the tokens' keys and values (blocks of 16 tokens; others); a workgroup per slot lets the blocks go.
#include "launch.h"
#include "tune.h"
#include "../../include/minions_verify.h"

namespace mn {

constexpr float LOG2E_W = 1.4426950408889634f;
constexpr float FAR_W = 0x1p24f;       // references from here on: see the attention's

// Sequence b's rows: the first one's number among the packed rows, how many count, and the slot of the first.  Lengths that do not add up to
// the host's rows disable the batch.
struct Weighed {
  int row0, count, base;
};
template <int NW>
__device__ __forceinline__ bool weighed_rows(const WeighArgs& a, int b, Weighed& w) {
  __shared__ int s_before[NW], s_all[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0, all = 0;
  bool off = false;
  for (int i = tid; i < a.B; i += 64 * NW) {
    const int k = a.spec_len[i];
    off |= k < 0 || k >= a.max_q;
    if (i < b) before += k + 1;
    all += k + 1;
  }
  before = wave_sum_i(before);
  all = wave_sum_i(all);
  if (lane == 0) { s_before[wave] = before; s_all[wave] = all; }
  off = __syncthreads_or(off);
  w.row0 = all = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) { w.row0 += s_before[i]; all += s_all[i]; }
  if (off || all != a.M) {
    if (tid == 0 && b == 0 && a.status) atomicOr(a.status, MN_DEV_SPEC_LEN);
    return false;
  }
  const int q = a.spec_len[b] + 1, ctx = a.ctx_lens[b];
  w.count = a.n_out ? a.n_out[b] : q;
  w.base = a.n_out ? ctx - w.count : ctx;
  if (w.count <= 0) return false;
  if (w.count > q || w.base < 0 || (long)w.base + w.count > a.max_ctx) {
    if (tid == 0 && a.status) atomicOr(a.status, w.count > q ? MN_DEV_SPEC_LEN : MN_DEV_CTX);
    return false;
  }
  w.row0 = __builtin_amdgcn_readfirstlane(w.row0);
  w.count = __builtin_amdgcn_readfirstlane(w.count);
  w.base = __builtin_amdgcn_readfirstlane(w.base);
  return true;
}

// 1 / l of a row, or 0 for one that is no number.
__device__ __forceinline__ float row_share(float2 st) {
  const bool counts = st.y > 0.f && st.y < INFINITY && __builtin_fabsf(st.x) < INFINITY;
  return counts ? 1.f / st.y : 0.f;
}
__device__ __forceinline__ float weight(float s, float c, float m, float share) {
  float x;
  {
#pragma clang fp contract(off)
    x = s * c - m;                     // (as the attention takes scores of a far reference)
  }
  const float y = __builtin_fabsf(m) >= FAR_W ? x : fmaf(s, c, -m);
  return share > 0.f ? __builtin_amdgcn_exp2f(y) * share : 0.f;
}

// The new weight of slot `key`, and whose it is.
__device__ __forceinline__ void put_weight(const WeighArgs& a, const Weighed& w, int b, int kvh, int key, float sum) {
  if (key >= w.base + w.count) return;
  const size_t at = ((size_t)b * a.Hkv + kvh) * a.width + key;
  if (key < w.base) {
    a.mass[at] += sum;
  } else {
    a.mass[at] = sum;
    a.born[at] = (a.seen ? a.seen[b] : w.base) + key - w.base;
  }
}

constexpr int WPAGE = 16;
// Exponent that a row's scores start from, -(m + log2 l), and whether its weights need more care than 2^(c s + that): statistics that are
// no numbers (its scores may be none either), and references from 2^8 on, whose sum with log2 l is rounded by 2^-16 and more.
__device__ __forceinline__ float row_start(float2 st, bool& careful) {
  careful |= !(st.y >= 0x1p-120f) | !(st.y < INFINITY) | !(__builtin_fabsf(st.x) < 0x1p8f);
  return -st.x - __builtin_amdgcn_logf(st.y);
}

// Many rows (prompts).  The NW waves of a workgroup take the keys of PAGES pages into registers, as they lie there (a page is the operand of
// the product: 16 keys by 8 elements in 256 bytes), and of the rows that see them every NW-th tile of 16 each.  A wave fetches its tiles into
// places of its own in the LDS, two ahead, by direct loads of whole rows: straight into the operands' registers every lane of a load met
// another line, and neither the exponentials nor the products were what it waited for (8000 rows of 40 heads of 128 629 us, without either
// the same, without the loads 418; so 437, 750 TFLOP/s, where a large product reaches 1073: without the exponentials 402, without the fetches
// 361, without the reads from the LDS 438).  16-byte chunks of a row change places, so that the reads of the operands meet every bank.
template <int HDIM, int PAGES, int NW>
__global__ void __launch_bounds__(64 * NW, 2) weigh_mfma_kernel(WeighArgs a) {
  constexpr int HS = HDIM / 32, CH = HDIM / 8, RPL = 64 / CH, LOADS = 16 / RPL;  // 16-byte chunks of a row, rows of a load, loads of a tile
  constexpr int SLOTS = 3, BYTES = 16 * HDIM * 2 + 256;            // a tile: its rows, and their statistics
  __shared__ __attribute__((aligned(1024))) unsigned char s_rows[NW][SLOTS][BYTES];
  __shared__ float s_sum[NW][PAGES * WPAGE];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, b = rest % a.B, chunk = rest / a.B;
  Weighed w;
  if (!weighed_rows<NW>(a, b, w)) return;
  const int end = w.base + w.count, key0 = chunk * (PAGES * WPAGE);
  if (key0 >= end) return;
  const int G = a.H / a.Hkv, R = w.count * G, shift = (G & (G - 1)) == 0 ? 31 - __clz(G) : -1;
  const int32_t* bt = a.kv.block_tables + (size_t)b * a.kv.max_blocks_per_seq;
  f16x8 kf[PAGES][HS];
  bool lost[PAGES];
#pragma unroll
  for (int p = 0; p < PAGES; ++p) {
    const uint32_t id = (uint32_t)bt[min(key0 / WPAGE + p, (end - 1) / WPAGE)];
    lost[p] = id >= (uint32_t)a.kv.num_blocks;
    const f16_t* page = static_cast<const f16_t*>(a.kv.k) + ((size_t)(lost[p] ? 0u : id) * a.Hkv + kvh) * (HDIM * WPAGE);
#pragma unroll
    for (int s = 0; s < HS; ++s) kf[p][s] = *reinterpret_cast<const f16x8*>(page + ((4 * s + g) * WPAGE + l16) * 8);
  }
  f32x4 sum[PAGES];
#pragma unroll
  for (int p = 0; p < PAGES; ++p) sum[p] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const float c = rsqrtf((float)HDIM) * LOG2E_W;
  const auto token_of = [&](int r) { return shift >= 0 ? r >> shift : (int)((uint32_t)r / (uint32_t)G); };
  const auto turn = [](int row) { return HDIM == 128 ? row & 15 : row >> 1 & 7; };

  // ---- fetching.  Where G divides 16 all tiles but the last are the same pattern of rows further on. ----
  const bool regular = shift >= 0 && G <= 16;
  const int last_tile = (R - 1) / 16 * 16;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&s_rows[wave][0][0]);
  const auto place = [&](int i) {                                  // row i from a token's first one on, in rows and heads
    const int j = token_of(i);
    return (uint32_t)(j * a.H + i - j * G);
  };
  const auto offset = [&](int load, int r0, int j0) {              // the lane's bytes of a load of the tile at r0 (past the last row: that one once more)
    const int row = load * RPL + lane / CH;
    return place(min(r0 + row, R - 1) - j0 * G) * (uint32_t)(HDIM * 2) + 16u * (uint32_t)((lane % CH) ^ turn(row));
  };
  const auto stat_offset = [&](int r0, int j0) { return place(min(r0 + (lane >> 1 & 15), R - 1) - j0 * G) * 8u + 4u * (lane & 1); };
  uint32_t off[LOADS], stat_off = stat_offset(0, 0);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) off[i] = offset(i, 0, 0);
  const auto fetch = [&](int r0, int slot) {
    const int rc = min(r0, last_tile), j0 = __builtin_amdgcn_readfirstlane(token_of(rc));
    const size_t mh = (size_t)(w.row0 + j0) * a.H + kvh * G;
    const char* q = reinterpret_cast<const char*>(static_cast<const f16_t*>(a.q) + mh * HDIM);
    const char* stats = reinterpret_cast<const char*>(a.stats + mh * 2);
    const uint32_t to = lds0 + (uint32_t)slot * BYTES;
    const bool same = regular && rc < last_tile;                   // (uniform)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) dma16s<0, false>(q, same ? off[i] : offset(i, rc, j0), to + 1024u * i);
    dma4s(stats, same ? stat_off : stat_offset(rc, j0), to + 16 * HDIM * 2);
  };
  const auto work = [&](int r0, int slot) {
    const unsigned char* st = s_rows[wave][slot];
    f16x8 q[HS];
#pragma unroll
    for (int s = 0; s < HS; ++s) q[s] = *reinterpret_cast<const f16x8*>(st + l16 * (2 * HDIM) + 16 * ((4 * s + g) ^ turn(l16)));
    const float2 stat = *reinterpret_cast<const float2*>(st + 16 * HDIM * 2 + l16 * 8);
    bool careful = r0 + l16 >= R;
    const float start = row_start(stat, careful);
    const bool all = w.base + token_of(r0) >= key0 + PAGES * WPAGE - 1;
    f32x4 S[PAGES];
#pragma unroll
    for (int p = 0; p < PAGES; ++p) S[p] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < HS; ++s)
#pragma unroll
      for (int p = 0; p < PAGES; ++p) S[p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[p][s], q[s], S[p], 0, 0, 0);
    if (all && !__any(careful)) {
#pragma unroll
      for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[p][e] += __builtin_amdgcn_exp2f(fmaf(S[p][e], c, start));
    } else {
      const float share = r0 + l16 < R ? row_share(stat) : 0.f;
      const int lim = w.base + token_of(min(r0 + l16, R - 1));
#pragma unroll
      for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = weight(S[p][e], c, stat.x, share);
          sum[p][e] += key0 + p * WPAGE + 4 * g + e <= lim ? x : 0.f;
        }
    }
  };
  // rows before this key's own see none of them
  constexpr int STEP = 16 * NW;
  int r0 = max(0, key0 - w.base) * G / 16 * 16 + 16 * wave, slot = 0;
  fetch(r0, 0);
  fetch(r0 + STEP, 1);
  for (; r0 < R; r0 += STEP) {
    const int third = slot == 0 ? 2 : slot - 1;
    __builtin_amdgcn_s_waitcnt(0xc07f);                            // lgkmcnt(0): the wave has read that place
    fetch(r0 + 2 * STEP, third);
    wait_vm<2 * (LOADS + 1)>();                                    // (this tile is there; the two behind it may be on their way)
    work(r0, slot);
    slot = slot == SLOTS - 1 ? 0 : slot + 1;
  }
  wait_vm<0>();
#pragma unroll
  for (int p = 0; p < PAGES; ++p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = sum[p][e];
      v += __uint_as_float(lane_swap<LANE_1>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_2>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_4>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_8>(__float_as_uint(v)));
      if (l16 == 0) s_sum[wave][p * WPAGE + 4 * g + e] = v;
    }
  }
  __syncthreads();
  if (wave > 0) return;
  static_assert(PAGES * WPAGE == 64, "a key per lane");
  float v = s_sum[0][lane];
#pragma unroll
  for (int i = 1; i < NW; ++i) v += s_sum[i][lane];
#pragma unroll
  for (int p = 0; p < PAGES; ++p) {
    if (lane >> 4 == p && !lost[p]) put_weight(a, w, b, kvh, key0 + lane, v);
    if (lost[p] && lane == 0 && key0 + p * WPAGE < end && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
  }
}

// Few rows (steps).  The rows of a KV head, STREAM_ROWS at most, wait in the LDS, and the keys go by: a wave takes two pages at a time, the next two on
// their way, the row as the first index of the product (a lane then has one key's weights, of four rows each time).  Bound by HBM: 9 rows of 64/8 heads
// of 128, 32 sequences of 1000 to 8000 tokens 59 us, 4.7 TB/s (a wave that took its keys once and the rows from HBM 103; with a look into the
// table at every step 66; pieces of 128 keys to the workgroups in turn, for the sake of the shorter sequences, nothing).
constexpr int STREAM_ROWS = 160, STREAM_KEYS = 4096;               // rows that fit; keys of a workgroup at most
template <int HDIM>
__global__ void __launch_bounds__(256, 3) weigh_stream_kernel(WeighArgs a) {
  constexpr int HS = HDIM / 32, CH = HDIM / 8;                     // 16-byte chunks of a row
  __shared__ __attribute__((aligned(16))) f16_t s_q[STREAM_ROWS * HDIM];
  __shared__ __attribute__((aligned(16))) float s_start[STREAM_ROWS], s_m[STREAM_ROWS], s_share[STREAM_ROWS];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, b = rest % a.B, range = rest / a.B;
  Weighed w;
  if (!weighed_rows<4>(a, b, w)) return;
  const int end = w.base + w.count, last = min(end, (range + 1) * a.range_keys);
  int key0 = range * a.range_keys + wave * (2 * WPAGE);
  if (range * a.range_keys >= end) return;
  const int G = a.H / a.Hkv, R = w.count * G, tiles = (R + 15) / 16, shift = (G & (G - 1)) == 0 ? 31 - __clz(G) : -1;
  const auto token_of = [&](int r) { return shift >= 0 ? r >> shift : (int)((uint32_t)r / (uint32_t)G); };
  const int32_t* bt = a.kv.block_tables + (size_t)b * a.kv.max_blocks_per_seq;
  const size_t line = ((size_t)b * a.Hkv + kvh) * a.width;
  struct Keys {
    f16x8 k[2][HS];
    float old;                                                     // the weight so far (of the lane's key, lanes 0 .. 31)
    uint32_t id[2];
  };
  // all blocks that the wave will ask for, two of a step to a pair of lanes: looked up step by step, each would be waited for
  constexpr int STEP = 4 * 2 * WPAGE;
  static_assert(STREAM_KEYS <= 32 * STEP, "a lane's block each");
  const int32_t blocks = bt[min((key0 + (lane >> 1) * STEP) / WPAGE + (lane & 1), (end - 1) / WPAGE)];
  const int first = key0;
  const auto load = [&](int key, Keys& t) {
    const int at = min((key - first) / STEP, 31) * 2;              // (past the range: another page of it, that nobody uses)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      t.id[p] = (uint32_t)__builtin_amdgcn_readlane(blocks, at + p);
      const f16_t* page = static_cast<const f16_t*>(a.kv.k) + ((size_t)min(t.id[p], (uint32_t)a.kv.num_blocks - 1u) * a.Hkv + kvh) * (HDIM * WPAGE);
#pragma unroll
      for (int s = 0; s < HS; ++s)
        t.k[p][s] = __builtin_bit_cast(f16x8, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(page + ((4 * s + g) * WPAGE + l16) * 8)));
    }
    t.old = a.mass[line + min(key + (lane & 31), end - 1)];
  };
  Keys ka, kb;
  load(key0, ka);                                                  // (unconditionally: past the end the last page once more, and waits stay counted)
  bool careful = false;
  for (int i = tid; i < tiles * 16 * CH; i += 256) {               // chunks of a row change places, so that 16 rows' meet every bank
    const int r = i / CH, ch = i % CH, at = r * CH + (ch ^ (HDIM == 128 ? r & 15 : (r >> 1 & 7)));
    // (past the last row that one once more, of no weight: zeros for a query would make no number of an infinity in a key)
    const int rr = min(r, R - 1), j = token_of(rr);
    const size_t mh = (size_t)(w.row0 + j) * a.H + kvh * G + rr - j * G;
    const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const f16_t*>(a.q) + mh * HDIM + ch * 8);
    if (ch == 0) {
      if (r < R) {
        const float2 st = *reinterpret_cast<const float2*>(a.stats + mh * 2);
        s_start[r] = row_start(st, careful);
        s_m[r] = st.x;
        s_share[r] = row_share(st);
      } else {
        s_start[r] = -INFINITY;
        s_m[r] = s_share[r] = 0.f;
      }
    }
    *reinterpret_cast<u32x4*>(s_q + at * 8) = x;
  }
  const bool slow = __syncthreads_or(careful);
  const float c = rsqrtf((float)HDIM) * LOG2E_W;
  bool lost = false;
  const auto work = [&](const Keys& t, int key0) {
    float sum[2] = {0.f, 0.f};
    const bool all = key0 + 2 * WPAGE - 1 <= w.base;               // (the first row sees up to its own slot)
    for (int i = 0; i < tiles; ++i) {
      f16x8 q[HS];
#pragma unroll
      for (int s = 0; s < HS; ++s) {
        const int r = 16 * i + l16, ch = 4 * s + g;
        q[s] = *reinterpret_cast<const f16x8*>(s_q + (r * CH + (ch ^ (HDIM == 128 ? r & 15 : (r >> 1 & 7)))) * 8);
      }
      const f32x4 start = *reinterpret_cast<const f32x4*>(s_start + 16 * i + 4 * g);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < HS; ++s) S = __builtin_amdgcn_mfma_f32_16x16x32_f16(q[s], t.k[p][s], S, 0, 0, 0);
        f32x4 x;
        if (!slow) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(S[e], c, start[e]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = weight(S[e], c, s_m[16 * i + 4 * g + e], s_share[16 * i + 4 * g + e]);
        }
        if (!all) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = key0 + p * WPAGE + l16 <= w.base + token_of(16 * i + 4 * g + e) ? x[e] : 0.f;
        }
        sum[p] += (x[0] + x[1]) + (x[2] + x[3]);
      }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {                                  // over the four lane groups
      uint32_t x, y;
      lane_pair<16>(__float_as_uint(sum[p]), x, y);
      sum[p] = __uint_as_float(x) + __uint_as_float(y);
      lane_pair<32>(__float_as_uint(sum[p]), x, y);
      sum[p] = __uint_as_float(x) + __uint_as_float(y);
    }
    const int key = key0 + lane;
    const bool gone = (g & 1 ? t.id[1] : t.id[0]) >= (uint32_t)a.kv.num_blocks;
    lost |= gone && key < end;
    if (lane < 32 && key < end && !gone) {
      const float v = g & 1 ? sum[1] : sum[0];
      a.mass[line + key] = key < w.base ? t.old + v : v;
      if (key >= w.base) a.born[line + key] = (a.seen ? a.seen[b] : w.base) + key - w.base;
    }
  };
  for (; key0 < last; key0 += 2 * STEP) {
    load(key0 + STEP, kb);
    work(ka, key0);
    load(key0 + 2 * STEP, ka);
    if (key0 + STEP < last) work(kb, key0 + STEP);
  }
  if (__any(lost && lane < 32) && lane == 0 && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
}

// A wave takes 16 keys, and the rows that see them in tiles of 16, on the fp32 instruction; ROWS: all waves the same keys and every fourth tile
// (3 prompts of 600 rows of 8/2 heads of 256: 80 us, keys shared out 488).  Products and their order are the attention's own.  Bound by their
// chain, each product waiting for the one before, and by the workgroups of a sequence's first keys, which walk all its rows (the instruction's rate
// alone would be 14 us; 8 prompts of 200 rows of 8/2 fp32 heads of 128 19 and 2); with few rows by the chain and launch.
// The products are those of the attention, factor for factor and in its order (as they are in the fp16 kernels): beyond 2^24 a
// reference is only as good as the very score that it came from.
template <typename T, int HDP, bool ROWS>
__global__ void __launch_bounds__(256) weigh_f32_kernel(WeighArgs a) {
  constexpr int NU = HDP / 16;
  struct __attribute__((aligned(4 * sizeof(T)))) Four { T x[4]; };
  __shared__ float s_sum[4][16];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4, hd = a.hd, bs = a.kv.block_size;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, b = rest % a.B, chunk = rest / a.B;
  Weighed w;
  if (!weighed_rows<4>(a, b, w)) return;
  const int end = w.base + w.count, key0 = (ROWS ? chunk : chunk * 4 + wave) * 16;
  if (key0 >= end) return;
  const int G = a.H / a.Hkv, R = w.count * G;
  const int key = min(key0 + l16, end - 1);
  const uint32_t id = (uint32_t)a.kv.block_tables[(size_t)b * a.kv.max_blocks_per_seq + key / bs];
  const bool lost = id >= (uint32_t)a.kv.num_blocks;
  const T* row = static_cast<const T*>(a.kv.k) + ((size_t)(lost ? 0u : id) * a.Hkv + kvh) * ((size_t)hd * bs) + (size_t)(key % bs) * 8;
  const float c = rsqrtf((float)hd) * LOG2E_W;
  f32x4 k[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    const int e0 = 16 * u + 4 * g;
    k[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (e0 < hd) {
      const Four x = *reinterpret_cast<const Four*>(row + (size_t)(e0 >> 3) * (8 * bs) + (e0 & 7));
#pragma unroll
      for (int e = 0; e < 4; ++e) k[u][e] = (float)x.x[e];
    }
  }
  struct Tile {
    Four q[NU];
    float2 st;
    int lim;
  };
  const auto load = [&](int r0, Tile& t) {                          // (past the last row: that one once more)
    const int r = min(r0 + l16, R - 1), j = (int)((uint32_t)r / (uint32_t)G);
    const size_t mh = (size_t)(w.row0 + j) * a.H + kvh * G + r - j * G;
    const T* q = static_cast<const T*>(a.q) + mh * hd;
#pragma unroll
    for (int u = 0; u < NU; ++u) t.q[u] = *reinterpret_cast<const Four*>(q + (HDP == 16 ? min(4 * g, hd - 4) : 16 * u + 4 * g));  // (heads of 8: keys of zeros behind)
    t.st = *reinterpret_cast<const float2*>(a.stats + mh * 2);
    t.lim = w.base + j;
  };
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const auto work = [&](const Tile& t, int r0) {
    f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_16x16x4f32(k[u][e], HDP == 16 && 4 * g >= hd ? 0.f : (float)t.q[u].x[e] * c, S, 0, 0, 0);
    const float share = r0 + l16 < R ? row_share(t.st) : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = weight(S[e], 1.f, t.st.x, share);
      sum[e] += key0 + 4 * g + e <= t.lim ? x : 0.f;
    }
  };
  constexpr int STEP = ROWS ? 64 : 16;
  int r0 = max(0, key0 - w.base) * G / 16 * 16 + (ROWS ? 16 * wave : 0);
  Tile now, next;
  load(r0, now);
  for (; r0 < R; r0 += 2 * STEP) {
    load(r0 + STEP, next);
    work(now, r0);
    load(r0 + 2 * STEP, now);
    if (r0 + STEP < R) work(next, r0 + STEP);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float v = sum[e];
    v += __uint_as_float(lane_swap<LANE_1>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_2>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_4>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_8>(__float_as_uint(v)));
    if (l16 == 0) s_sum[wave][4 * g + e] = v;
  }
  if constexpr (ROWS) {
    __syncthreads();
    if (wave > 0) return;
  }
  const float v = ROWS ? s_sum[0][l16] + s_sum[1][l16] + s_sum[2][l16] + s_sum[3][l16] : s_sum[wave][l16];
  if (lane < 16 && !lost) put_weight(a, w, b, kvh, key0 + l16, v);
  if (__any(lost) && lane == 0 && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
}

// ------------------------------------------------------------------------------------------
// eviction
// ------------------------------------------------------------------------------------------
// Order of the tokens as 32-bit numbers: the protected ones above all, then by weight, no numbers last.
__device__ __forceinline__ uint32_t rank_of(float mass, bool always) {
  if (always) return 0xffffffffu;
  if (mass != mass) return 0u;
  const uint32_t u = __float_as_uint(mass == 0.f ? 0.f : mass);  // (one zero)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sequence b of the call, of n tokens: whether it loses some, and may (asked by the whole workgroup).
__device__ __forceinline__ bool evicted(const EvictArgs& a, int b, int n, int keep, bool report) {
  const PoolView& p = a.pool;
  if (keep < 0 || n <= keep) return false;
  const int bs = p.block_size, held = p.seq_blocks[b];
  int flags = 0;
  if (n > a.width) flags = MN_DEV_CTX;
  else if (held < 0 || held > p.width || ((long)n + bs - 1) / bs > held) flags = MN_DEV_BLOCK_TABLE;
  bool bad = false, shared = false;
  if (flags == 0) {
    const int32_t* row = p.tables + (size_t)b * p.width;
    const int first = a.sinks / bs, last = (int)(((long)keep + bs - 1) / bs);   // blocks that may be written, if any
    for (int i = threadIdx.x; i < held; i += blockDim.x) {
      const uint32_t id = (uint32_t)row[i];
      if (id >= (uint32_t)p.num_blocks) bad = true;
      else if (i >= first && i < last && p.refs[id] > 1) shared = true;
    }
  }
  if (__syncthreads_or(bad)) flags |= MN_DEV_BLOCK_TABLE;
  if (__syncthreads_or(shared)) flags |= MN_DEV_SHARED;
  if (flags && report && threadIdx.x == 0 && p.status) atomicOr(p.status, flags);
  return flags == 0;
}

// Sums of N numbers of a wave over the workgroup's WAVES waves, and (of the first) over the waves before it.  Two buffers in turn: one
// barrier each.
template <int WAVES, int N>
__device__ __forceinline__ void waves_sum(int (&v)[N], int (*s)[WAVES][4], int& turn, int& before) {
  int (*t)[4] = s[turn ^= 1];
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) t[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0;
  before = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w == (int)(threadIdx.x >> 6)) before = v[0];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += t[w][k];
  }
}

// A wave has a contiguous piece of the slots, a lane every 64th of it: PER of them, as ranks in registers (PER 0: any number, read again each
// time).  The keep-th rank is found digit by digit, counting in the LDS; among the tokens of that very rank the lowest slots stay.
// Then the slots below `keep` that are left, in ascending order, take the tokens that stay from `keep` on, in ascending order: there are
// as many of either.  A workgroup has one head, and what it waits for is one step after the other: 8 layers of 8 heads of 16 sequences of 1000 to
// 4000 tokens 37 us, one sequence of the smallest model 7.
template <int WAVES, int PER>
__global__ void __launch_bounds__(64 * WAVES) evict_plan_kernel(EvictArgs a) {
  __shared__ int s_count[2][WAVES][4], s_bins[4][256], s_digit[2];
  constexpr int THREADS = 64 * WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x, h = row % a.Hkv, b = row / a.Hkv % a.B, layer = row / a.Hkv / a.B;
  const size_t line = (((size_t)layer * a.pool.max_seqs + b) * a.Hkv + h) * a.width;
  float* mass = a.mass + line;
  int32_t* born = a.born + line;
  const int n = a.pool.ctx_lens[b], keep = a.keep[b];
  // (asked for ahead of the table row; a context that is longer than the line is none)
  const int m = n > a.width ? 0 : max(n, 0);
  const int per = (m + THREADS - 1) / THREADS, lo = min(m, wave * per * 64), hi = min(m, lo + per * 64);
  float mine[PER > 0 ? PER : 1];
  int32_t age[PER > 0 ? PER : 1];
  int last = INT32_MIN;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (lo + 64 * i < hi) {                                      // (uniform)
      const int at = min(lo + 64 * i + lane, hi - 1);
      mine[i] = mass[at];
      age[i] = born[at];
    }
  for (int i = tid; i < 4 * 256; i += THREADS) s_bins[0][i] = 0;
  const bool go = evicted(a, b, n, keep, layer == 0 && h == 0);
  if (tid == 0 && layer == 0 && h == 0) a.gone[b] = go ? 1 : 0;
  if (!go) {
    if (tid == 0) a.n_moves[row] = 0;
    return;
  }
  if constexpr (PER > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lo + 64 * i < hi) last = max(last, age[i]);
  } else {
    for (int i = tid; i < n; i += THREADS) last = max(last, born[i]);
  }
  for (int d = 32; d; d >>= 1) last = max(last, __shfl_xor(last, d));
  int turn = 0, before;
  if (lane == 0) s_count[0][wave][0] = last;                     // (the sums' second buffer)
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) last = max(last, s_count[0][w][0]);
  const long young = (long)last - a.recent;                      // born behind it: recent
  uint32_t rank[PER > 0 ? PER : 1];
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (lo + 64 * i < hi) rank[i] = lo + 64 * i + lane < hi ? rank_of(mine[i], lo + 64 * i + lane < a.sinks || age[i] > young) : 0u;
  // f(slot, whether it is one, its rank) over the wave's slots
  const auto each = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lo + 64 * i < hi) f(lo + 64 * i + lane, lo + 64 * i + lane < hi, rank[i]);
    } else {
      for (int i = lo; i < hi; i += 64) {
        const int at = i + lane;
        f(at, at < hi, at < hi ? rank_of(mass[at], at < a.sinks || born[at] > young) : 0u);
      }
    }
  };
  // eight bits at a time, from the top: how many ranks of those that agree with T so far have which digit
  uint32_t T = 0;
  int ties = keep;                                               // of the ranks that agree with T stay
#pragma unroll
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (keep == 0) {                                             // (nobody: no rank is above this one)
      T = ~0u;
      break;
    }
    int* bins = s_bins[shift / 8];
    each([&](int, bool in, uint32_t r) {
      if (in & (shift == 24 || r >> (shift + 8 & 31) == T >> (shift + 8 & 31))) atomicAdd(bins + (r >> shift & 255), 1);
    });
    __syncthreads();
    if (wave == 0) {                                             // lane 0 has the four highest digits
      int c[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += c[k] = bins[255 - 4 * lane - k];
      const int incl = wave_scan_i(sum);
      if (incl >= ties && incl - sum < ties) {
        int above = incl - sum, k = 0;
        while (above + c[k] < ties) above += c[k++];
        s_digit[0] = 255 - 4 * lane - k;
        s_digit[1] = ties - above;
      }
    }
    __syncthreads();
    T |= (uint32_t)s_digit[0] << shift;
    ties = s_digit[1];
  }
  int same[1] = {0}, ties_at;
  each([&](int, bool in, uint32_t r) { same[0] += __popcll(__ballot(in & (r == T))); });
  waves_sum<WAVES>(same, s_count, turn, ties_at);
  const uint64_t below = (1ull << lane) - 1;
  // f(slot, whether it is left for another, whether it moves)
  const auto decide = [&](auto f) {
    int at = ties_at;
    each([&](int i, bool in, uint32_t r) {
      const uint64_t equal = __ballot(in & (r == T));
      const bool stays = in & ((r > T) | ((r == T) & (at + __popcll(equal & below) < ties)));
      at += __popcll(equal);
      f(i, in & !stays & (i < keep), stays & (i >= keep));
    });
  };
  int holes[1] = {0}, movers[1] = {0}, holes_at, movers_at;
  decide([&](int, bool hole, bool mover) {
    holes[0] += __popcll(__ballot(hole));
    movers[0] += __popcll(__ballot(mover));
  });
  waves_sum<WAVES>(holes, s_count, turn, holes_at);
  waves_sum<WAVES>(movers, s_count, turn, movers_at);
  int2* to = a.moves + (size_t)row * a.width;                    // (slot, block) of either side, width / 2 of them at most
  int2* from = to + a.width / 2;
  int32_t* firsts = a.firsts + (size_t)row * (a.width / a.pool.block_size + 2);  // per block, the first of its places in the list
  const int32_t* bt = a.pool.tables + (size_t)b * a.pool.width;
  const int bs = a.pool.block_size, shift = (bs & (bs - 1)) == 0 ? 31 - __clz(bs) : -1;
  const auto block_of = [&](int i) { return shift >= 0 ? i >> shift : i / bs; };
  decide([&](int i, bool hole, bool mover) {
    const uint64_t hb = __ballot(hole), mb = __ballot(mover);
    const int at = holes_at + __popcll(hb & below);
    if (hole) to[at] = make_int2(i, bt[block_of(i)]);
    if (mover) from[movers_at + __popcll(mb & below)] = make_int2(i, bt[block_of(i)]);
    if (i < keep && block_of(i) * bs == i) firsts[block_of(i)] = at;
    holes_at += __popcll(hb);
    movers_at += __popcll(mb);
  });
  __syncthreads();
  for (int i = tid; i < holes[0]; i += THREADS) {
    const int s = from[i].x, d = to[i].x;
    mass[d] = mass[s];
    born[d] = born[s];
  }
  if (tid == 0) {
    a.n_moves[row] = holes[0];
    firsts[(keep + bs - 1) / bs] = holes[0];
  }
}

// The blocks behind the tokens that stay are let go, as when a slot is emptied.
__device__ __forceinline__ void let_go(const EvictArgs& a, int b) {
  if (!a.gone[b]) return;
  const PoolView& p = a.pool;
  const int keep = a.keep[b], held = p.seq_blocks[b], now = (int)(((long)keep + p.block_size - 1) / p.block_size);
  int32_t* row = p.tables + (size_t)b * p.width;
  for (int i = now + threadIdx.x; i < held; i += blockDim.x) {
    const int id = row[i];
    row[i] = -1;
    if (atomicSub(p.refs + id, 1) <= 0) {
      atomicAdd(p.refs + id, 1);
      if (p.status) atomicOr(p.status, MN_DEV_BLOCK_TABLE);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.seq_blocks[b] = now;
    p.ctx_lens[b] = keep;
  }
}

// 16 moves of a row at a time: a K token is pieces of 8 elements in as many places, a V token as many places as it has elements.
template <typename T>
__device__ __forceinline__ void move_tokens(const EvictArgs& a, T* kp, T* vp, int h, const int2* to, const int2* from, int begin, int end) {
  struct __attribute__((aligned(16))) Eight { T x[8]; };
  const int bs = a.pool.block_size, hd = a.hd, nth = threadIdx.x % 16;
  for (int i0 = begin; i0 < end; i0 += 16) {
    if (i0 + nth >= end) continue;
    const int2 d = to[i0 + nth], s = from[i0 + nth];
    const size_t dp = ((size_t)d.y * a.Hkv + h) * ((size_t)hd * bs), sp = ((size_t)s.y * a.Hkv + h) * ((size_t)hd * bs);
    const int dof = d.x % bs, sof = s.x % bs;
    for (int c = threadIdx.x / 16; c < hd / 8; c += 16)
      *reinterpret_cast<Eight*>(kp + dp + ((size_t)c * bs + dof) * 8) = *reinterpret_cast<const Eight*>(kp + sp + ((size_t)c * bs + sof) * 8);
#pragma unroll 8
    for (int e = threadIdx.x / 16; e < hd; e += 16) vp[dp + (size_t)e * bs + dof] = vp[sp + (size_t)e * bs + sof];
  }
}

template <typename T>
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, LayerPages pages, int layer0, int release) {
  const int wg = (int)blockIdx.x - release;
  if (wg < 0) return let_go(a, blockIdx.x);
  const int r = wg / a.splits, split = wg - r * a.splits, per_layer = a.B * a.Hkv;
  const int h = r % a.Hkv, layer = r / per_layer;
  const size_t row = (size_t)layer0 * per_layer + r;
  const int moves = a.n_moves[row];
  const int2* to = a.moves + row * a.width;
  const int each = (moves + 16 * a.splits - 1) / (16 * a.splits) * 16;
  move_tokens(a, static_cast<T*>(pages.k[layer]), static_cast<T*>(pages.v[layer]), h, to, to + a.width / 2, split * each, min(moves, (split + 1) * each));
}

// Blocks of 16 tokens: a wave takes a page at a time, the tokens that stay in it read as well, so that it is written in whole lines.  (Into the
// places alone the writes were parts of lines: 16 sequences of 1000 to 4000 tokens cut to 1024, 8 layers of 8 heads of 128, 505 us; now
// 391.)  A piece of 16 bytes is (part of) one token of K, or PER tokens of one element of V; NU of them per lane.  What is next is looked up
// meanwhile.  Bound by HBM: a page's lines hold pieces of 4 to 8 of its tokens, so nearly every line of the pages that tokens come from and go to
// passes, 1.8 GB at 4.6 TB/s, which is what a copy reaches; the tokens that move alone would be 0.66 GB.  In two turns for pages of 8 KB (2 fp32 heads of 128,
// fp16 of 256): 213 and 218 us, 0.92 GB at 4.3 TB/s.
template <typename T, int NU>
__global__ void __launch_bounds__(256) evict_pages_kernel(EvictArgs a, LayerPages pages, int layer0, int release) {
  constexpr int PER = 16 / sizeof(T), BS = 16, AT_ONCE = NU < 4 ? NU : 4;
  typedef u32x4 Piece;
  __shared__ __attribute__((aligned(16))) T s_pages[4][2][AT_ONCE * 64 * PER];
  const int wg = (int)blockIdx.x - release;
  if (wg < 0) return let_go(a, blockIdx.x);
  const int r = wg / a.splits, split = wg - r * a.splits, per_layer = a.B * a.Hkv;
  const int h = r % a.Hkv, layer = r / per_layer, lane = threadIdx.x & 63, nth = lane & (BS - 1);
  T* image = s_pages[threadIdx.x >> 6][0];
  T* source = s_pages[threadIdx.x >> 6][1];
  const size_t row = (size_t)layer0 * per_layer + r;
  if (a.n_moves[row] == 0) return;
  const int2* to = a.moves + row * a.width;
  const int2* from = to + a.width / 2;
  const int32_t* firsts = a.firsts + row * (a.width / BS + 2);
  T* kp = static_cast<T*>(pages.k[layer]);
  T* vp = static_cast<T*>(pages.v[layer]);
  const int hd = a.hd, page = hd * BS, step = 4 * a.splits;
  const int blocks = (a.keep[r / a.Hkv % a.B] + BS - 1) / BS;
  const auto at = [&](int id) { return ((size_t)id * a.Hkv + h) * page; };
  // places of the block p: [x, y) of the list
  const auto ask = [&](int p) { return p < blocks ? make_int2(firsts[p], firsts[p + 1]) : make_int2(0, 0); };
  int p = split * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int2 now = ask(p);
  for (; p < blocks; p += step) {
    const int2 next = ask(p + step);
    const int n = now.y - now.x;
    if (n > 0) {
      // lane i < 16: the token that slot i gets
      const int2 d = to[now.x + min(nth, n - 1)], s = from[now.x + min(nth, n - 1)];
      const int block = __builtin_amdgcn_readfirstlane(d.y);
      int id = block, off = nth;
#pragma unroll
      for (int i = 0; i < BS; ++i) {
        const int slot = __builtin_amdgcn_readlane(d.x, i) & (BS - 1), sx = __builtin_amdgcn_readlane(s.x, i), sy = __builtin_amdgcn_readlane(s.y, i);
        if (i < n && slot == nth) { id = sy; off = sx & (BS - 1); }
      }
      // K: a lane's pieces are all of one slot
      const int k_slot = lane * PER / 8 & (BS - 1);
      const T* ks = kp + at(__shfl(id, k_slot)) + __shfl(off, k_slot) * 8 + lane * PER % 8;
      T* kd = kp + at(block);
      T* vd = vp + at(block);
#pragma unroll
      for (int u0 = 0; u0 < NU; u0 += AT_ONCE) {
        const auto inside = [&](int u) { return (lane + 64 * (u0 + u)) * PER < page; };
        const auto load = [&](const T* from_page, Piece (&v)[AT_ONCE]) {
#pragma unroll
          for (int u = 0; u < AT_ONCE; ++u)
            if (inside(u)) v[u] = *reinterpret_cast<const Piece*>(from_page + (lane + 64 * (u0 + u)) * PER);
        };
        Piece k[AT_ONCE], v[AT_ONCE], w[AT_ONCE];
        load(vd, v);
        load(vp + at(__builtin_amdgcn_readlane(s.y, 0)), w);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
          if (inside(u)) k[u] = *reinterpret_cast<const Piece*>(ks + (lane + 64 * (u0 + u)) * PER / (8 * BS) * (8 * BS));
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) *reinterpret_cast<Piece*>(image + (lane + 64 * u) * PER) = v[u];
        // V: the tokens that come, source page after source page
        for (int i = 0; i < n;) {
          const int from_block = __builtin_amdgcn_readlane(s.y, i);
#pragma unroll
          for (int u = 0; u < AT_ONCE; ++u) *reinterpret_cast<Piece*>(source + (lane + 64 * u) * PER) = w[u];
          int last = i + 1;
          while (last < n && __builtin_amdgcn_readlane(s.y, last) == from_block) ++last;
          if (last < n) load(vp + at(__builtin_amdgcn_readlane(s.y, last)), w);
          for (; i < last; ++i) {
            const int slot = __builtin_amdgcn_readlane(d.x, i) & (BS - 1), of = __builtin_amdgcn_readlane(s.x, i) & (BS - 1);
#pragma unroll
            for (int e = lane; e < AT_ONCE * 64 * PER / BS; e += 64) image[e * BS + slot] = source[e * BS + of];
          }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
          if (inside(u)) {
            *reinterpret_cast<Piece*>(kd + (lane + 64 * (u0 + u)) * PER) = k[u];
            *reinterpret_cast<Piece*>(vd + (lane + 64 * (u0 + u)) * PER) = *reinterpret_cast<const Piece*>(image + (lane + 64 * u) * PER);
          }
      }
    }
    now = next;
  }
}

// ------------------------------------------------------------------------------------------
// launch
// ------------------------------------------------------------------------------------------
static bool weigh_mfma(const WeighArgs& a) { return a.dtype == MN_DT_BF16 && (a.hd == 64 || a.hd == 128) && a.kv.block_size == WPAGE; }
constexpr int WEIGH_PAGES = 4;
constexpr int WEIGH_WGS = 512;         // to aim for: two a CU.  40 heads, 4 sequences of 2000 tokens, 64 rows: 21.6 us, 1024: 27.2, 2048: 41.9

struct WeighShape {
  int keys;                            // of a workgroup
  bool stream, rows;                   // few rows; many, that the waves share out
  int waves;
};
static WeighShape weigh_shape(const WeighArgs& a) {
  const long heads = (long)a.B * a.Hkv, R = (long)a.max_q * (a.H / a.Hkv);
  if (!weigh_mfma(a)) return R > 64 ? WeighShape{16, false, true, 4} : WeighShape{64, false, false, 4};
  // The rows stay and the keys go by, or the other way round.  Over 64 rows the first pays where keys are many: 128 rows of 64/8 heads, 32
  // sequences of 4000 tokens 63 us (rows going by: 116), of 40 heads, 4 of 2000 tokens 28 (43), 8 of 500 tokens 25 (29); of 64/8 heads, 8 of
  // 2000 tokens 25 (21), their 64 rows 17 (17).
  if (R <= 64 || (R <= STREAM_ROWS && heads * a.max_ctx >= 288 * WEIGH_WGS)) {
    // ranges of 128 keys (two pages for each wave) and more
    long keys = (long)a.max_ctx * heads / WEIGH_WGS / 128 * 128;
    if (keys < 128) keys = 128;
    if (keys > STREAM_KEYS) keys = STREAM_KEYS;
    return WeighShape{(int)keys, true, false, 4};
  }
  const int each = WEIGH_PAGES * WPAGE;
  // Eight waves where workgroups are few (1500 rows of 64/8 heads: 73 us, with four 121; 1000 rows of 40 heads, 640 workgroups: 27, with four
  // 19), two where they are many and each has little to do (8 prompts of 1000 rows of 40 heads 93 us, with four 117, with one 98; 2 of 3000
  // rows 166, with four 161).
  const long wgs = heads * ((a.max_ctx + each - 1) / each);
  return WeighShape{each, false, true, wgs < 512 ? 8 : wgs >= 2048 && R <= 2048 ? 2 : 4};
}
long weigh_workgroups(const WeighArgs& a) {
  const int keys = weigh_shape(a).keys;
  return (long)a.B * a.Hkv * ((a.max_ctx + keys - 1) / keys);
}

template <typename T, int HDP>
static void launch_weigh_f32_as(const WeighArgs& a, bool rows, unsigned wgs, hipStream_t st) {
  if (rows) weigh_f32_kernel<T, HDP, true><<<wgs, 256, 0, st>>>(a);
  else weigh_f32_kernel<T, HDP, false><<<wgs, 256, 0, st>>>(a);
}
template <typename T>
static void launch_weigh_f32(const WeighArgs& a, bool rows, unsigned wgs, hipStream_t st) {
  switch (a.hd) {
    case 8: case 16: launch_weigh_f32_as<T, 16>(a, rows, wgs, st); break;
    case 32: launch_weigh_f32_as<T, 32>(a, rows, wgs, st); break;
    case 64: launch_weigh_f32_as<T, 64>(a, rows, wgs, st); break;
    case 128: launch_weigh_f32_as<T, 128>(a, rows, wgs, st); break;
    default: launch_weigh_f32_as<T, 256>(a, rows, wgs, st); break;
  }
}
template <int HDIM>
static void launch_weigh_mfma(const WeighArgs& a, const WeighShape& s, unsigned wgs, hipStream_t st) {
  if (s.stream) weigh_stream_kernel<HDIM><<<wgs, 256, 0, st>>>(a);
  else if (s.waves == 2) weigh_mfma_kernel<HDIM, WEIGH_PAGES, 2><<<wgs, 128, 0, st>>>(a);
  else if (s.waves == 4) weigh_mfma_kernel<HDIM, WEIGH_PAGES, 4><<<wgs, 256, 0, st>>>(a);
  else weigh_mfma_kernel<HDIM, WEIGH_PAGES, 8><<<wgs, 512, 0, st>>>(a);
}

void launch_weigh(WeighArgs a, hipStream_t st) {
  const unsigned wgs = (unsigned)weigh_workgroups(a);
  const WeighShape s = weigh_shape(a);
  a.range_keys = s.keys;
  if (!weigh_mfma(a)) {
    if (a.dtype == MN_DT_BF16) launch_weigh_f32<f16_t>(a, s.rows, wgs, st);
    else launch_weigh_f32<float>(a, s.rows, wgs, st);
  } else if (a.hd == 128) {
    launch_weigh_mfma<128>(a, s, wgs, st);
  } else {
    launch_weigh_mfma<64>(a, s, wgs, st);
  }
}

template <typename T>
static void launch_pages(const EvictArgs& a, const LayerPages& pages, int l0, int release, unsigned wgs, hipStream_t st) {
  const int pieces = a.hd * (int)sizeof(T);                        // 16 bytes each, of a page of K and of one of V
  if (pieces <= 64) evict_pages_kernel<T, 1><<<wgs, 256, 0, st>>>(a, pages, l0, release);
  else if (pieces <= 128) evict_pages_kernel<T, 2><<<wgs, 256, 0, st>>>(a, pages, l0, release);
  else if (pieces <= 256) evict_pages_kernel<T, 4><<<wgs, 256, 0, st>>>(a, pages, l0, release);
  else if (pieces <= 512) evict_pages_kernel<T, 8><<<wgs, 256, 0, st>>>(a, pages, l0, release);
  else evict_pages_kernel<T, 16><<<wgs, 256, 0, st>>>(a, pages, l0, release);
}

static size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
size_t evict_work_bytes(int B, int n_layers, int Hkv, int width) {
  const size_t rows = (size_t)n_layers * B * Hkv;
  return padded((size_t)B * 4) + padded(rows * 4) + padded(rows * ((size_t)width + 2) * 4) + padded(rows * (size_t)width * 8);
}

void launch_evict(EvictArgs a, void* const* k, void* const* v, int n_layers, void* workspace, hipStream_t st) {
  unsigned char* w = static_cast<unsigned char*>(workspace);
  const size_t rows = (size_t)n_layers * a.B * a.Hkv;
  const auto take = [&](size_t bytes) { unsigned char* p = w; w += padded(bytes); return p; };
  a.gone = reinterpret_cast<int32_t*>(take((size_t)a.B * 4));
  a.n_moves = reinterpret_cast<int32_t*>(take(rows * 4));
  a.firsts = reinterpret_cast<int32_t*>(take(rows * ((size_t)a.width + 2) * 4));
  a.moves = reinterpret_cast<int2*>(take(rows * (size_t)a.width * 8));
  // (ranks per lane: as few as hold the ledger's lines)
  if (a.width <= 256) evict_plan_kernel<4, 1><<<(unsigned)rows, 256, 0, st>>>(a);
  else if (a.width <= 1024) evict_plan_kernel<4, 4><<<(unsigned)rows, 256, 0, st>>>(a);
  else if (a.width <= 4096) evict_plan_kernel<4, 16><<<(unsigned)rows, 256, 0, st>>>(a);
  else if (a.width <= 16384) evict_plan_kernel<16, 16><<<(unsigned)rows, 1024, 0, st>>>(a);
  else evict_plan_kernel<16, 0><<<(unsigned)rows, 1024, 0, st>>>(a);
  for (int l0 = 0; l0 < n_layers; l0 += LAYERS_PER_LAUNCH) {
    LayerPages pages{};
    const int layers = n_layers - l0 < LAYERS_PER_LAUNCH ? n_layers - l0 : LAYERS_PER_LAUNCH;
    for (int l = 0; l < layers; ++l) { pages.k[l] = k[l0 + l]; pages.v[l] = v[l0 + l]; }
    const int release = l0 + layers == n_layers ? a.B : 0;
    const long r = (long)layers * a.B * a.Hkv;
    // 1024, 2048, 4096, 8192, 16384 workgroups: 499, 493, 481, 471, 467 us (16 sequences cut to 1024 tokens, 8 layers of 8 heads, plan included)
    const int want = MN_TUNE("MN_EVICT_WGS", 8192), most = (a.width + 127) / 128;
    a.splits = r >= want ? 1 : (int)((want + r - 1) / r);
    if (a.splits > most) a.splits = most;
    const unsigned wgs = (unsigned)(r * a.splits + release);
    if (a.pool.block_size == 16) {
      if (a.dtype == MN_DT_BF16) launch_pages<f16_t>(a, pages, l0, release, wgs, st);
      else launch_pages<float>(a, pages, l0, release, wgs, st);
    } else if (a.dtype == MN_DT_BF16) {
      evict_move_kernel<f16_t><<<wgs, 256, 0, st>>>(a, pages, l0, release);
    } else {
      evict_move_kernel<float><<<wgs, 256, 0, st>>>(a, pages, l0, release);
    }
  }
}

}  // namespace mn
