// Rows of a projection made ready for the cache: every query and key head normed, turned to its token's position, and rounded once;
// queries to where the attention reads them, keys and values into the pages of their sequences.
//
//   y = g x / sqrt(mean(x^2) + eps) over a head;  pair (i, i + rot / 2) of y is turned by the angle p_a(i) base^(-2i / rot),
// p_a the token's position on the axis that pair i belongs to.  An angle is a fraction of a turn in 64 bits (a far position times a
// frequency has no correct digit of its angle left in 32), its sine and cosine and everything else are 32 bits.
//
// A lane holds eight elements of a head: four, and the four that they are paired with, so that neither the norm's sum (over hd / 8 lanes)
// nor the rotation goes through the LDS.  Elements behind `rot` are paired likewise and turned by nothing.
//  * Queries: a wave takes a row, or a share of its heads where there are few rows; a lane's angles serve all of them.
//  * Keys and values: a workgroup takes the 16 slots of the cache that a page of 16 tokens is, writes them as the page lies into the LDS, and
//    copies whole pieces of 16 bytes out.  Straight from the rows a value is two bytes of a 32-byte sector.
// Bound by HBM where rows are many: prompts of 500 to 3000 tokens of 64/8 heads of 128 70 us, 294 MB at 4.2 TB/s (a copy: 4.6).  9 rows of 64
// sequences (fp32 rows, 35 MB) 14 us: the way in (the batch's lengths, a row's loads, a head's sum) beside the bytes, and work on heads that are not
// kept: a wave asks for and norms as many heads as AT_ONCE loads hold, 16 there, whatever its share is, there 12.  4 rows of 12 heads 6 us, the way in alone.
#include "launch.h"
#include "tune.h"
#include "../../include/minions_verify.h"

namespace mn {

constexpr int SLOTS = 16;              // of a workgroup that fills pages

__device__ __forceinline__ float lanes_sum(float v, int lanes) {  // over groups of a power of two of lanes, up to 32
  if (lanes > 1) v += __uint_as_float(lane_swap<LANE_1>(__float_as_uint(v)));
  if (lanes > 2) v += __uint_as_float(lane_swap<LANE_2>(__float_as_uint(v)));
  if (lanes > 4) v += __uint_as_float(lane_swap<LANE_4>(__float_as_uint(v)));
  if (lanes > 8) v += __uint_as_float(lane_swap<LANE_8>(__float_as_uint(v)));
  if (lanes > 16) {
    uint32_t x, y;
    lane_pair<16>(__float_as_uint(v), x, y);
    v = __uint_as_float(x) + __uint_as_float(y);
  }
  return v;
}

template <typename T> struct __attribute__((aligned(4 * sizeof(T)))) Quad { T x[4]; };

// The lane's place in a head, and its angles there.
struct Place {
  int a, b;                            // its elements a .. a + 3 and b .. b + 3
  int pair;                            // the first of its pairs, or -1: not turned
};
__device__ __forceinline__ Place place_of(int t, int hd, int rot) {
  const int half = rot / 2;
  if (4 * t < half) return Place{4 * t, half + 4 * t, 4 * t};
  const int e = rot + 4 * t - half;
  return Place{e, e + (hd - rot) / 2, -1};
}
__device__ __forceinline__ void angles(const CacheRows& a, int m, int pair, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) { c[e] = 1.f; s[e] = 0.f; }
  if (pair < 0) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = pair + e, axis = (i >= a.axis_end[0]) + (i >= a.axis_end[1]) + (i >= a.axis_end[2]);
    double turns = (double)a.positions[(size_t)axis * a.M + m] * a.freq[i];
    turns -= rint(turns);
    sincospif(2.f * (float)turns, &s[e], &c[e]);
  }
}

// Norm and rotation of the lane's elements x of a head (`lanes` lanes hold one).
__device__ __forceinline__ void ready(float (&x)[8], const float* gain, float eps, int hd, int lanes, const Place& at, const float (&c)[4], const float (&s)[4]) {
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    const float r = 1.f / sqrtf(lanes_sum(ss, lanes) / (float)hd + eps);
    const f32x4 ga = *reinterpret_cast<const f32x4_u*>(gain + at.a), gb = *reinterpret_cast<const f32x4_u*>(gain + at.b);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] *= r * ga[e]; x[4 + e] *= r * gb[e]; }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float u = x[e], v = x[4 + e];
    x[e] = u * c[e] - v * s[e];
    x[4 + e] = v * c[e] + u * s[e];
  }
}
template <typename In>
__device__ __forceinline__ void load8(const In* row, const Place& at, float (&x)[8]) {
  const Quad<In> u = *reinterpret_cast<const Quad<In>*>(row + at.a), v = *reinterpret_cast<const Quad<In>*>(row + at.b);
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[e] = (float)u.x[e]; x[4 + e] = (float)v.x[e]; }
}
template <typename T>
__device__ __forceinline__ Quad<T> round4(const float* x, bool& bad) {
  Quad<T> q;
#pragma unroll
  for (int e = 0; e < 4; ++e) q.x[e] = sizeof(T) == 2 ? (T)sat_h(x[e], bad) : (T)x[e];
  return q;
}

// The sequence of unit u, which of its units that is, its rows and its context: sequence b has (k_b + 1 + 14) / 16 + 1 units, as many pages as
// its rows can touch wherever they begin.  Lengths that do not add up to the host's rows and units are reported, and nothing is written.
struct Unit {
  int seq, nth, row0, q, ctx;
};
__device__ __forceinline__ bool unit_of(const CacheRows& a, int u, Unit& x) {
  __shared__ int s_units[4], s_rows[4], s_hit[5];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  bool off = false;
  const auto length = [&](int b) {
    const int k = a.spec_len[b];
    off |= k < 0 || k >= a.max_q;
    return k < 0 || k >= a.max_q ? 0 : k + 1;
  };
  const auto units_of = [](int n) { return n > 0 ? (n + 14) / SLOTS + 1 : 0; };
  if (a.B <= 64) {                                                 // (every wave by itself)
    int n = 0, ctx = 0;
    if (lane < a.B) { n = length(lane); ctx = a.ctx_lens[lane]; }
    const int units = units_of(n), ui = wave_scan_i(units), ri = wave_scan_i(n);
    off = __any(off) || __builtin_amdgcn_readlane(ui, 63) != a.n_units || __builtin_amdgcn_readlane(ri, 63) != a.M;
    if (!off) {
      const int b = __ffsll((unsigned long long)__ballot(u < ui)) - 1;
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
      x = Unit{b, u - of(ui) + of(units), of(ri) - of(n), of(n), of(ctx)};
      return true;
    }
  } else {
    int units_at = 0, rows_at = 0;
    for (int b0 = 0; b0 < a.B; b0 += 256) {
      const int b = b0 + tid, n = b < a.B ? length(b) : 0, units = units_of(n);
      const int ui = wave_scan_i(units), ri = wave_scan_i(n);
      __syncthreads();
      if (lane == 63) { s_units[wave] = ui; s_rows[wave] = ri; }
      __syncthreads();
      int before = units_at + ui - units, r = rows_at + ri - n;
      for (int w = 0; w < 4; ++w) {
        if (w < wave) { before += s_units[w]; r += s_rows[w]; }
        units_at += s_units[w];
        rows_at += s_rows[w];
      }
      if (u >= before && u < before + units) { s_hit[0] = b; s_hit[1] = u - before; s_hit[2] = r; s_hit[3] = n; s_hit[4] = a.ctx_lens[b]; }
    }
    off = __syncthreads_or(off) || units_at != a.n_units || rows_at != a.M;
    if (!off) {
      x = Unit{s_hit[0], s_hit[1], s_hit[2], s_hit[3], s_hit[4]};
      return true;
    }
  }
  if (tid == 0 && u == 0 && a.status) atomicOr(a.status, MN_DEV_SPEC_LEN);
  return false;
}

template <typename In, typename T>
__global__ void __launch_bounds__(256) cache_rows_kernel(CacheRows a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, hd = a.hd, lanes = hd / 8, t = tid & (lanes - 1);
  const Place at = place_of(t, hd, a.rot);
  bool bad = false;
  const int fills = a.n_units * a.unit_parts * a.unit_splits;
  const bool queries = (int)blockIdx.x >= fills;
  // the row of this thread, and its share of the heads: of queries a wave's, of keys and values the workgroup's
  int m, part, in = 0, from = 0, to = 0, slot0 = 0;
  Unit x{0, 0, 0, a.M, 0};
  bool mine;
  if (queries) {
    const int w = ((int)blockIdx.x - fills) * 4 + (tid >> 6);
    m = w / a.q_splits;
    part = w - m * a.q_splits;
    mine = m < a.M;
    m = min(m, a.M - 1);
  } else {
    const int at_once = min(SLOTS, 256 / lanes);                   // slots side by side (heads of 256: 8)
    const int up = blockIdx.x / a.unit_splits, u = up / a.unit_parts;
    part = blockIdx.x - up * a.unit_splits;
    in = (up - u * a.unit_parts) * at_once + tid / lanes;
    if (a.kv.k) {
      if (!unit_of(a, u, x)) return;
      if (x.ctx < 0 || (long)x.ctx + x.q > (long)a.kv.max_blocks_per_seq * a.kv.block_size) {
        if (tid == 0 && x.nth == 0 && part == 0 && a.status) atomicOr(a.status, MN_DEV_CTX);
        return;
      }
    } else {
      x.nth = u;
    }
    slot0 = (x.ctx / SLOTS + x.nth) * SLOTS;
    from = max(slot0 + (up - u * a.unit_parts) * at_once, x.ctx);
    to = min(slot0 + min(SLOTS, (up - u * a.unit_parts + 1) * at_once), x.ctx + x.q);
    if (from >= to) return;
    mine = slot0 + in >= from && slot0 + in < to;
    m = x.row0 + (mine ? slot0 + in : from) - x.ctx;
  }
  float c[4], s[4];
  if (queries) {
    const int per = 64 / lanes, h0 = part * a.q_heads, h1 = mine ? min(a.H, h0 + a.q_heads) : 0;
    const In* row = static_cast<const In*>(a.q) + (size_t)m * a.q_stride;
    T* out = static_cast<T*>(a.q_out) + (size_t)m * a.H * hd;
    constexpr int AT_ONCE = 4;                                     // heads of a lane asked for together
    for (int hw = h0; hw < h1; hw += AT_ONCE * per) {              // (whole waves: the sums go across lanes)
      float y[AT_ONCE][8];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) load8(row + (size_t)min(hw + u * per + (tid & 63) / lanes, a.H - 1) * hd, at, y[u]);
      if (hw == h0) angles(a, m, at.pair, c, s);
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const int h = hw + u * per + (tid & 63) / lanes;
        ready(y[u], a.q_gain, a.eps, hd, lanes, at, c, s);
        if (h >= h1) continue;
        *reinterpret_cast<Quad<T>*>(out + (size_t)h * hd + at.a) = round4<T>(y[u], bad);
        *reinterpret_cast<Quad<T>*>(out + (size_t)h * hd + at.b) = round4<T>(y[u] + 4, bad);
      }
    }
  } else {
    const int bs = a.kv.block_size, slot = slot0 + in;
    const bool whole = a.kv.k && bs % SLOTS == 0;                  // the slots lie side by side in one block
    const size_t head_page = (size_t)hd * bs;
    bool lost = false;                                             // a block id out of range
    uint32_t id = 0;
    if (a.kv.k) {
      id = (uint32_t)a.kv.block_tables[(size_t)x.seq * a.kv.max_blocks_per_seq + (whole ? slot0 : mine ? slot : from) / bs];
      lost = id >= (uint32_t)a.kv.num_blocks;
    }
    const int off0 = whole ? slot0 % bs : 0, off = a.kv.k ? slot % bs : 0;
    T* img_k = reinterpret_cast<T*>(smem);                         // [hd / 8][16][8], [hd][16]
    T* img_v = img_k + hd * SLOTS;
    const int h0 = part * a.unit_heads, h1 = min(a.Hkv, h0 + a.unit_heads);
    const In* k_row = static_cast<const In*>(a.k) + (size_t)m * a.k_stride;
    const In* v_row = static_cast<const In*>(a.v) + (size_t)m * a.v_stride;
    float kx[8], vx[8];
    load8(k_row + (size_t)h0 * hd, at, kx);
    load8(v_row + (size_t)h0 * hd, at, vx);
    angles(a, m, at.pair, c, s);
    for (int h = h0; h < h1; ++h) {
      Quad<T> k[2], v[2];
      ready(kx, a.k_gain, a.eps, hd, lanes, at, c, s);
      bool over = false;
      k[0] = round4<T>(kx, over); k[1] = round4<T>(kx + 4, over);
      v[0] = round4<T>(vx, over); v[1] = round4<T>(vx + 4, over);
      bad |= over && mine;
      if (h + 1 < h1) {                                            // (the next head's on their way)
        load8(k_row + (size_t)(h + 1) * hd, at, kx);
        load8(v_row + (size_t)(h + 1) * hd, at, vx);
      }
      if (mine) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int el = e ? at.b : at.a;
          if (a.k_out) *reinterpret_cast<Quad<T>*>(static_cast<T*>(a.k_out) + ((size_t)m * a.Hkv + h) * hd + el) = k[e];
          if (a.v_out) *reinterpret_cast<Quad<T>*>(static_cast<T*>(a.v_out) + ((size_t)m * a.Hkv + h) * hd + el) = v[e];
        }
      }
      if (!a.kv.k) continue;
      const size_t page = ((size_t)id * a.Hkv + h) * head_page;
      T* pk = static_cast<T*>(a.kv.k) + page;
      T* pv = static_cast<T*>(a.kv.v) + page;
      if (!whole) {
        if (mine && !lost) {
          int there = off, el_a = at.a, el_b = at.b;
          asm volatile("" : "+v"(there), "+v"(el_a), "+v"(el_b));  // (sixteen addresses worked out anew for every head: registers)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int el = (e < 4 ? el_a : el_b) + (e & 3);
            pk[((size_t)(el >> 3) * bs + there) * 8 + (el & 7)] = k[e >> 2].x[e & 3];
            pv[(size_t)el * bs + there] = v[e >> 2].x[e & 3];
          }
        }
        continue;
      }
      if (h > h0) __syncthreads();                                 // (the head before has left)
      if (mine) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int el = e ? at.b : at.a;
          *reinterpret_cast<Quad<T>*>(img_k + ((el >> 3) * SLOTS + in) * 8 + (el & 7)) = k[e];
#pragma unroll
          for (int i = 0; i < 4; ++i) img_v[(el + i) * SLOTS + in] = v[e].x[i];
        }
      }
      __syncthreads();
      if (lost) continue;
      constexpr int PER = 16 / sizeof(T);                          // elements of a piece
      const int lo = from - slot0, hi = to - slot0;
      for (int i = tid; i < hd * SLOTS / PER; i += 256) {
        const int e = i * PER;
        const int ks = e / 8 % SLOTS;                              // K: a piece is of one token
        if (ks >= lo && ks < hi) *reinterpret_cast<u32x4*>(pk + ((size_t)(e / (8 * SLOTS)) * bs + off0 + ks) * 8 + e % 8) = *reinterpret_cast<const u32x4*>(img_k + e);
        const int vs = e % SLOTS;                                  // V: of several
        T* out = pv + (size_t)(e / SLOTS) * bs + off0 + vs;
        if (vs >= lo && vs + PER <= hi) {
          *reinterpret_cast<u32x4*>(out) = *reinterpret_cast<const u32x4*>(img_v + e);
        } else {
          for (int j = 0; j < PER; ++j)
            if (vs + j >= lo && vs + j < hi) out[j] = img_v[e + j];
        }
      }
    }
    if (lost && mine && a.status) atomicOr(a.status, MN_DEV_BLOCK_TABLE);
  }
  if (sizeof(T) == 2 && bad && a.status) atomicOr(a.status, MN_DEV_RANGE);
}

long cache_row_units(const int32_t* h_spec_len, int B, int M, bool pages) {
  if (!pages) return ((long)M + SLOTS - 1) / SLOTS;
  long n = 0;
  for (int b = 0; b < B; ++b) n += (h_spec_len[b] + 15) / SLOTS + 1;
  return n;
}

// Shares of the heads: whole rows where there are enough of them.  For keys and values 512 workgroups (their angles serve all heads of a page;
// 2048: 76 us for 70 on the prompts above); queries go on until 4096 waves.
static void split_heads(int heads, long items, int least, long want, int& splits, int& each) {
  long n = want / (items > 0 ? items : 1);
  if (n > heads / least) n = heads / least;
  if (n < 1) n = 1;
  each = (int)((heads + n - 1) / n);
  splits = (heads + each - 1) / each;
}

long cache_rows_shape(CacheRows& a) {
  const int lanes = a.hd / 8, per = 64 / lanes;                    // heads that a wave holds at once
  split_heads(a.H, a.M, per, MN_TUNE("MN_ROWS_Q", 4096), a.q_splits, a.q_heads);
  a.q_heads = (a.q_heads + per - 1) / per * per;
  a.q_splits = (a.H + a.q_heads - 1) / a.q_heads;
  a.unit_parts = lanes > 16 ? lanes / 16 : 1;
  split_heads(a.Hkv, (long)a.n_units * a.unit_parts, 1, MN_TUNE("MN_ROWS_KV", 512), a.unit_splits, a.unit_heads);
  return (long)a.n_units * a.unit_parts * a.unit_splits + (a.q_out ? ((long)a.M * a.q_splits + 3) / 4 : 0);
}

hipError_t launch_cache_rows(const CacheRows& a, long workgroups, hipStream_t st) {
  const bool wide = a.rows_f32 != 0;
  const size_t lds = a.kv.k ? (size_t)2 * a.hd * SLOTS * (a.dtype == MN_DT_BF16 ? 2 : 4) : 0;
  if (a.dtype == MN_DT_F32) cache_rows_kernel<float, float><<<(unsigned)workgroups, 256, lds, st>>>(a);
  else if (wide) cache_rows_kernel<float, f16_t><<<(unsigned)workgroups, 256, lds, st>>>(a);
  else cache_rows_kernel<f16_t, f16_t><<<(unsigned)workgroups, 256, lds, st>>>(a);
  return hipSuccess;
}

}  // namespace mn
