// What attention has looked at, and what may go: the weight that every cached token has been given, per layer, sequence and KV head, and
// the eviction of those with the least of it.
//
//   mass[i] += sum over rows r and the query heads of the KV head of p_ri = 2^(c s_ri - m_r) / l_r,
// with the rows' statistics (m_r, l_r) as their attention left them: one product, one exponential, sums along the rows.  A
// token's key may stand in any slot of its sequence, each head's in another, since its rotation is in it and attention asks for no
// order: so a head that loses tokens fills their slots with those that it keeps from behind the new end, and nothing else moves.
//
//  * weigh_mfma_kernel  fp16, head_dim 64 or 128, blocks of 16 tokens.
//  * weigh_f32_kernel   every other type, head_dim and block size.
//  * evict_plan_kernel  a workgroup per layer, slot and head: who stays, and who goes where.
//  * evict_move_kernel  the tokens' keys and values; a workgroup per slot lets the blocks go.
#include "launch.h"
#include "../../include/minions_verify.h"

namespace mn {

constexpr float LOG2E_W = 1.4426950408889634f;
constexpr float FAR_W = 0x1p24f;       // references from here on: see the attention's

// Sequence b's rows: the first one's number among the packed rows, how many count, and the slot of the first.  Lengths that do not add up to
// the host's rows disable the batch.
struct Weighed {
  int row0, count, base;
};
__device__ __forceinline__ bool weighed_rows(const WeighArgs& a, int b, Weighed& w) {
  __shared__ int s_before[4], s_all[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0, all = 0;
  bool off = false;
  for (int i = tid; i < a.B; i += 256) {
    const int k = a.spec_len[i];
    off |= k < 0 || k >= a.max_q;
    if (i < b) before += k + 1;
    all += k + 1;
  }
  before = wave_sum_i(before);
  all = wave_sum_i(all);
  if (lane == 0) { s_before[wave] = before; s_all[wave] = all; }
  off = __syncthreads_or(off);
  w.row0 = s_before[0] + s_before[1] + s_before[2] + s_before[3];
  if (off || s_all[0] + s_all[1] + s_all[2] + s_all[3] != a.M) {
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
// A wave takes the keys of PAGES pages into registers, as they lie there (a page is the operand of the product: 16 keys by 8 elements in
// 256 bytes), and the rows that see them in tiles of 16.
template <int HDIM, int PAGES>
__global__ void __launch_bounds__(256) weigh_mfma_kernel(WeighArgs a) {
  constexpr int HS = HDIM / 32;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, b = rest % a.B, chunk = rest / a.B;
  Weighed w;
  if (!weighed_rows(a, b, w)) return;
  const int end = w.base + w.count, key0 = (chunk * 4 + wave) * (PAGES * WPAGE);
  if (key0 >= end) return;
  const int G = a.H / a.Hkv, R = w.count * G;
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
  // rows before this key's own see none of them
  for (int r0 = max(0, key0 - w.base) * G / 16 * 16; r0 < R; r0 += 16) {
    const int r = min(r0 + l16, R - 1), j = r / G, m = w.row0 + j, h = kvh * G + r - j * G;
    const f16_t* q = static_cast<const f16_t*>(a.q) + ((size_t)m * a.H + h) * HDIM;
    f16x8 qf[HS];
#pragma unroll
    for (int s = 0; s < HS; ++s) qf[s] = *reinterpret_cast<const f16x8*>(q + 32 * s + 8 * g);
    const float2 st = *reinterpret_cast<const float2*>(a.stats + ((size_t)m * a.H + h) * 2);
    const float share = r0 + l16 < R ? row_share(st) : 0.f;
    const int lim = w.base + j;
#pragma unroll
    for (int p = 0; p < PAGES; ++p) {
      f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < HS; ++s) S = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[p][s], qf[s], S, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = weight(S[e], c, st.x, share);
        sum[p][e] += key0 + p * WPAGE + 4 * g + e <= lim ? x : 0.f;
      }
    }
  }
#pragma unroll
  for (int p = 0; p < PAGES; ++p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = sum[p][e];
      v += __uint_as_float(lane_swap<LANE_1>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_2>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_4>(__float_as_uint(v)));
      v += __uint_as_float(lane_swap<LANE_8>(__float_as_uint(v)));
      if (l16 == 0 && !lost[p]) put_weight(a, w, b, kvh, key0 + p * WPAGE + 4 * g + e, v);
    }
    if (lost[p] && lane == 0 && key0 + p * WPAGE < end && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
  }
}

// A wave takes 16 keys, and the rows that see them in tiles of 16, on the fp32 instruction.
template <typename T, int HDP>
__global__ void __launch_bounds__(256) weigh_f32_kernel(WeighArgs a) {
  constexpr int NU = HDP / 16;
  struct __attribute__((aligned(4 * sizeof(T)))) Four { T x[4]; };
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4, hd = a.hd, bs = a.kv.block_size;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, b = rest % a.B, chunk = rest / a.B;
  Weighed w;
  if (!weighed_rows(a, b, w)) return;
  const int end = w.base + w.count, key0 = (chunk * 4 + wave) * 16;
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
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int r0 = max(0, key0 - w.base) * G / 16 * 16; r0 < R; r0 += 16) {
    const int r = min(r0 + l16, R - 1), j = r / G, m = w.row0 + j, h = kvh * G + r - j * G;
    const T* q = static_cast<const T*>(a.q) + ((size_t)m * a.H + h) * hd;
    f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int e0 = 16 * u + 4 * g;
      Four x{};
      if (e0 < hd) x = *reinterpret_cast<const Four*>(q + e0);
#pragma unroll
      for (int e = 0; e < 4; ++e) S = __builtin_amdgcn_mfma_f32_16x16x4f32(k[u][e], (float)x.x[e], S, 0, 0, 0);
    }
    const float2 st = *reinterpret_cast<const float2*>(a.stats + ((size_t)m * a.H + h) * 2);
    const float share = r0 + l16 < R ? row_share(st) : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = weight(S[e], c, st.x, share);
      sum[e] += key0 + 4 * g + e <= w.base + j ? x : 0.f;
    }
  }
  const uint64_t gone = __ballot(lost);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float v = sum[e];
    v += __uint_as_float(lane_swap<LANE_1>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_2>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_4>(__float_as_uint(v)));
    v += __uint_as_float(lane_swap<LANE_8>(__float_as_uint(v)));
    if (l16 == 0 && !(gone >> (4 * g + e) & 1)) put_weight(a, w, b, kvh, key0 + 4 * g + e, v);
  }
  if (gone && lane == 0 && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
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

// Sequence b of the call: whether it loses tokens, and may (asked by the whole workgroup).
__device__ __forceinline__ bool evicted(const EvictArgs& a, int b, int& n, int& keep, bool report) {
  const PoolView& p = a.pool;
  n = p.ctx_lens[b];
  keep = a.keep[b];
  if (keep < 0 || n <= keep) return false;
  const int bs = p.block_size, held = p.seq_blocks[b];
  int flags = 0;
  if (n > a.width) flags = MN_DEV_CTX;
  else if (held < 0 || held > p.width || ((long)n + bs - 1) / bs > held) flags = MN_DEV_BLOCK_TABLE;
  bool bad = false, shared = false;
  if (flags == 0) {
    const int32_t* row = p.tables + (size_t)b * p.width;
    const int first = min(a.sinks, keep) / bs, last = (keep + bs - 1) / bs;   // blocks that may be written
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

constexpr int EVICT_WAVES = 4;
// Sum of a wave's number over the workgroup, and of the waves before it.
__device__ __forceinline__ int waves_sum(int v, int* s, int& before) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  int total = 0;
  before = 0;
  for (int w = 0; w < EVICT_WAVES; ++w) {
    if (w == (int)(threadIdx.x >> 6)) before = total;
    total += s[w];
  }
  return total;
}

// A wave has a contiguous piece of the slots, a lane every 64th of it.  The keep-th rank is found bit by bit, counting by ballots; among
// the tokens of that very rank the lowest slots stay.  Then the slots below `keep` that are left, in ascending order, take the tokens that
// stay from `keep` on, in ascending order: there are as many of either.
__global__ void __launch_bounds__(64 * EVICT_WAVES) evict_plan_kernel(EvictArgs a) {
  __shared__ int s_count[EVICT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x, h = row % a.Hkv, b = row / a.Hkv % a.B, layer = row / a.Hkv / a.B;
  int n, keep;
  const bool go = evicted(a, b, n, keep, layer == 0 && h == 0);
  if (tid == 0 && layer == 0 && h == 0) a.gone[b] = go ? 1 : 0;
  if (!go) {
    if (tid == 0) a.n_moves[row] = 0;
    return;
  }
  const size_t line = (((size_t)layer * a.pool.max_seqs + b) * a.Hkv + h) * a.width;
  float* mass = a.mass + line;
  int32_t* born = a.born + line;
  int last = INT32_MIN;
  for (int i = tid; i < n; i += 64 * EVICT_WAVES) last = max(last, born[i]);
  for (int d = 32; d; d >>= 1) last = max(last, __shfl_xor(last, d));
  __syncthreads();
  if (lane == 0) s_count[wave] = last;
  __syncthreads();
  for (int w = 0; w < EVICT_WAVES; ++w) last = max(last, s_count[w]);
  const long young = (long)last - a.recent;                      // born behind it: recent
  const auto rank = [&](int i) {
    const int o = born[i];
    return rank_of(mass[i], i < a.sinks || o > young);
  };
  const int per = (n + 64 * EVICT_WAVES - 1) / (64 * EVICT_WAVES) * 64, lo = min(n, wave * per), hi = min(n, lo + per);
  const auto count = [&](auto pred) {
    int c = 0;
    for (int i = lo; i < hi; i += 64) c += __popcll(__ballot(i + lane < hi && pred(rank(min(i + lane, n - 1)))));
    return c;
  };
  int before;
  uint32_t T = 0;                                                // the largest number that `keep` ranks reach
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = T | 1u << bit;
    if (waves_sum(count([&](uint32_t r) { return r >= t; }), s_count, before) >= keep) T = t;
  }
  const int above = waves_sum(count([&](uint32_t r) { return r > T; }), s_count, before);
  waves_sum(count([&](uint32_t r) { return r == T; }), s_count, before);
  const int ties = keep - above;                                 // of the rank itself stay
  // f(slot, stays) over the wave's slots
  const auto each = [&](auto f) {
    int at = before;
    for (int i = lo; i < hi; i += 64) {
      const bool in = i + lane < hi;
      const uint32_t r = in ? rank(i + lane) : 0u;
      const uint64_t same = __ballot(in && r == T);
      const bool stays = in && (r > T || (r == T && at + __popcll(same & ((1ull << lane) - 1)) < ties));
      at += __popcll(same);
      f(i + lane, in, stays);
    }
  };
  int holes = 0, movers = 0, holes_at, movers_at;
  each([&](int i, bool in, bool stays) {
    holes += __popcll(__ballot(in && !stays && i < keep));
    movers += __popcll(__ballot(stays && i >= keep));
  });
  const int moves = waves_sum(holes, s_count, holes_at);
  waves_sum(movers, s_count, movers_at);
  int2* to = a.moves + (size_t)row * a.width;                    // (block, offset) of either side, width / 2 of them at most
  int2* from = to + a.width / 2;
  const int32_t* bt = a.pool.tables + (size_t)b * a.pool.width;
  const int bs = a.pool.block_size;
  each([&](int i, bool in, bool stays) {
    const bool hole = in && !stays && i < keep, mover = stays && i >= keep;
    const uint64_t hb = __ballot(hole), mb = __ballot(mover), below = (1ull << lane) - 1;
    if (hole) to[holes_at + __popcll(hb & below)] = make_int2(i, bt[i / bs]);
    if (mover) from[movers_at + __popcll(mb & below)] = make_int2(i, bt[i / bs]);
    holes_at += __popcll(hb);
    movers_at += __popcll(mb);
  });
  __syncthreads();
  for (int i = tid; i < moves; i += 64 * EVICT_WAVES) {
    const int s = from[i].x, d = to[i].x;
    mass[d] = mass[s];
    born[d] = born[s];
  }
  if (tid == 0) a.n_moves[row] = moves;
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
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, LayerPages pages, int layer0, int release) {
  const int wg = (int)blockIdx.x - release;
  if (wg < 0) return let_go(a, blockIdx.x);
  struct __attribute__((aligned(16))) Eight { T x[8]; };
  const int r = wg / a.splits, split = wg - r * a.splits, per_layer = a.B * a.Hkv;
  const int h = r % a.Hkv, layer = r / per_layer;
  const size_t row = (size_t)layer0 * per_layer + r;
  const int moves = a.n_moves[row], bs = a.pool.block_size, hd = a.hd;
  const int2* to = a.moves + row * a.width;
  const int2* from = to + a.width / 2;
  T* kp = static_cast<T*>(pages.k[layer]);
  T* vp = static_cast<T*>(pages.v[layer]);
  for (int i0 = split * 16; i0 < moves; i0 += a.splits * 16) {
    const int m = min(16, moves - i0);
    const int2 d = to[i0 + min((int)threadIdx.x % 16, m - 1)], s = from[i0 + min((int)threadIdx.x % 16, m - 1)];
    if ((int)threadIdx.x % 16 >= m) continue;
    const size_t dp = ((size_t)d.y * a.Hkv + h) * ((size_t)hd * bs), sp = ((size_t)s.y * a.Hkv + h) * ((size_t)hd * bs);
    const int dof = d.x % bs, sof = s.x % bs;
    for (int c = threadIdx.x / 16; c < hd / 8; c += 16)
      *reinterpret_cast<Eight*>(kp + dp + ((size_t)c * bs + dof) * 8) = *reinterpret_cast<const Eight*>(kp + sp + ((size_t)c * bs + sof) * 8);
    for (int e = threadIdx.x / 16; e < hd; e += 16) vp[dp + (size_t)e * bs + dof] = vp[sp + (size_t)e * bs + sof];
  }
}

// ------------------------------------------------------------------------------------------
// launch
// ------------------------------------------------------------------------------------------
static bool weigh_mfma(const WeighArgs& a) { return a.dtype == MN_DT_BF16 && (a.hd == 64 || a.hd == 128) && a.kv.block_size == WPAGE; }
constexpr int WEIGH_PAGES = 4;

static int weigh_keys(const WeighArgs& a) { return weigh_mfma(a) ? 4 * WEIGH_PAGES * WPAGE : 64; }  // of a workgroup
long weigh_workgroups(const WeighArgs& a) { return (long)a.B * a.Hkv * ((a.max_ctx + weigh_keys(a) - 1) / weigh_keys(a)); }

template <typename T>
static void launch_weigh_f32(const WeighArgs& a, unsigned wgs, hipStream_t st) {
  switch (a.hd) {
    case 8: case 16: weigh_f32_kernel<T, 16><<<wgs, 256, 0, st>>>(a); break;
    case 32: weigh_f32_kernel<T, 32><<<wgs, 256, 0, st>>>(a); break;
    case 64: weigh_f32_kernel<T, 64><<<wgs, 256, 0, st>>>(a); break;
    case 128: weigh_f32_kernel<T, 128><<<wgs, 256, 0, st>>>(a); break;
    default: weigh_f32_kernel<T, 256><<<wgs, 256, 0, st>>>(a); break;
  }
}

void launch_weigh(const WeighArgs& a, hipStream_t st) {
  const unsigned wgs = (unsigned)weigh_workgroups(a);
  if (!weigh_mfma(a)) {
    if (a.dtype == MN_DT_BF16) launch_weigh_f32<f16_t>(a, wgs, st);
    else launch_weigh_f32<float>(a, wgs, st);
  } else if (a.hd == 128) {
    weigh_mfma_kernel<128, WEIGH_PAGES><<<wgs, 256, 0, st>>>(a);
  } else {
    weigh_mfma_kernel<64, WEIGH_PAGES><<<wgs, 256, 0, st>>>(a);
  }
}

size_t evict_work_bytes(int B, int n_layers, int Hkv, int width) {
  const size_t rows = (size_t)n_layers * B * Hkv;
  return 4096 + ((size_t)B * 4 + 255) / 256 * 256 + (rows * 4 + 255) / 256 * 256 + rows * (size_t)width * 8;
}

void launch_evict(EvictArgs a, void* const* k, void* const* v, int n_layers, void* workspace, hipStream_t st) {
  unsigned char* w = static_cast<unsigned char*>(workspace);
  const size_t rows = (size_t)n_layers * a.B * a.Hkv;
  a.gone = reinterpret_cast<int32_t*>(w);
  w += ((size_t)a.B * 4 + 255) / 256 * 256;
  a.n_moves = reinterpret_cast<int32_t*>(w);
  w += (rows * 4 + 255) / 256 * 256;
  a.moves = reinterpret_cast<int2*>(w);
  evict_plan_kernel<<<(unsigned)rows, 64 * EVICT_WAVES, 0, st>>>(a);
  for (int l0 = 0; l0 < n_layers; l0 += LAYERS_PER_LAUNCH) {
    LayerPages pages{};
    const int layers = n_layers - l0 < LAYERS_PER_LAUNCH ? n_layers - l0 : LAYERS_PER_LAUNCH;
    for (int l = 0; l < layers; ++l) { pages.k[l] = k[l0 + l]; pages.v[l] = v[l0 + l]; }
    const int release = l0 + layers == n_layers ? a.B : 0;
    const long r = (long)layers * a.B * a.Hkv;
    a.splits = r >= 2048 ? 1 : (int)((2048 + r - 1) / r);
    if (a.splits > (a.width + 31) / 32) a.splits = (a.width + 31) / 32;
    const unsigned wgs = (unsigned)(r * a.splits + release);
    if (a.dtype == MN_DT_BF16) evict_move_kernel<f16_t><<<wgs, 256, 0, st>>>(a, pages, l0, release);
    else evict_move_kernel<float><<<wgs, 256, 0, st>>>(a, pages, l0, release);
  }
}

}  // namespace mn
