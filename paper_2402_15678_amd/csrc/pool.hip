// The pool of cache pages: which sequence holds which physical block, blocks held by several sequences at once, and the
// copies of pages that follow from it (paper section 4: a logical block id and an offset per cached token; the block manager
// behind the table is the caller's in the paper, here its state lives on the device beside the table).
//
// State, all int32 and all the caller's: block_refs[id] = table rows that hold block id (0: free), seq_blocks[s] = blocks that
// slot s holds, its table row's first entries.  Every decision is a function of that state alone: blocks are given out lowest id
// first, in the order of (sequence, position), and nothing depends on the order in which workgroups or atomics run.
//
//  * fork_kernel     one workgroup per pair: the child's row, one more reference per block.  No page is touched.
//  * free_kernel     one workgroup per sequence: one reference less per block.
//  * reserve_plan / compact_plan   one workgroup: who needs how many blocks (a prefix sum over the sequences), which blocks are
//    free (ballots over block_refs, every wave an own range of ids, one scan over the waves), hence who gets which.
//  * copy_pages      the pages of the (from, to) pairs that a plan wrote, in all layers; as many workgroups as fill the chip
//    take chunks by index, so a step without a copy is a short launch.
// A plan is bound by its chain of round trips to memory, a copy by HBM.  16 requests of 100 to 700 tokens that branch into 4 each,
// 64/8 heads of 128, 8 layers: fork 4.2 us, plan 8.6 (half a microsecond less with the counts read once into bit masks), copy 9.2.  16 of 48 sequences
// retired, 12 layers of 12 heads of 64: free 4.8, plan 5.0, copy 92 (4.6 TB/s read and written).
#include "launch.h"
#include "../../include/minions_verify.h"

namespace mn {

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;
constexpr int COPY_UNROLL = 4;                                   // 16-byte pieces of a thread per chunk
constexpr int COPY_CHUNK = 256 * COPY_UNROLL;                    // pieces of a workgroup per chunk (16 KB)

__device__ __forceinline__ void raise(int32_t* status, int bit) {
  if (status) atomicOr(status, bit);
}

__global__ void __launch_bounds__(256) fork_kernel(PoolView p, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = src[i], d = dst[i];
  const bool slots = s >= 0 && s < p.max_seqs && d >= 0 && d < p.max_seqs && s != d;
  // a slot that two pairs would fill goes to the first; a parent that the call itself fills is no parent
  bool taken = false;
  for (int j = tid; j < n; j += 256) {
    const int t = dst[j];
    taken |= (t == d && j < i) || t == s;
  }
  if (__syncthreads_or(taken) || !slots) {
    if (tid == 0) raise(p.status, MN_DEV_SEQ);
    return;
  }
  const int ctx = p.ctx_lens[s], held = p.seq_blocks[s];
  const int nb = ctx > 0 ? (int)(((long)ctx + p.block_size - 1) / p.block_size) : 0;
  if (p.seq_blocks[d] != 0 || p.ctx_lens[d] != 0) {              // (uniform; only this workgroup writes slot d)
    __syncthreads();
    if (tid == 0) raise(p.status, MN_DEV_SEQ);
    return;
  }
  const int32_t* from = p.tables + (size_t)s * p.width;
  int32_t* to = p.tables + (size_t)d * p.width;
  bool bad = ctx < 0 || nb > held || nb > p.width;
  if (!bad)
    for (int k = tid; k < nb; k += 256) bad |= (uint32_t)from[k] >= (uint32_t)p.num_blocks;
  if (__syncthreads_or(bad)) {
    if (tid == 0) raise(p.status, MN_DEV_BLOCK_TABLE);
    return;
  }
  for (int k = tid; k < nb; k += 256) {
    const int id = from[k];
    to[k] = id;
    atomicAdd(p.refs + id, 1);
  }
  if (tid == 0) {
    p.seq_blocks[d] = nb;
    p.ctx_lens[d] = ctx;
  }
}

__global__ void __launch_bounds__(256) free_kernel(PoolView p, const int32_t* __restrict__ seqs) {
  __shared__ int s_held;
  const int s = seqs[blockIdx.x], tid = threadIdx.x;
  if (s < 0 || s >= p.max_seqs) {
    if (tid == 0) raise(p.status, MN_DEV_SEQ);
    return;
  }
  if (tid == 0) {                                                // (listed twice: the second finds nothing)
    s_held = atomicExch(p.seq_blocks + s, 0);
    p.ctx_lens[s] = 0;
  }
  __syncthreads();
  const int nb = min(max(s_held, 0), p.width);
  int32_t* row = p.tables + (size_t)s * p.width;
  bool bad = s_held != nb;
  for (int k = tid; k < nb; k += 256) {
    const int id = row[k];
    row[k] = -1;
    if ((uint32_t)id >= (uint32_t)p.num_blocks) {
      bad = true;
    } else if (atomicSub(p.refs + id, 1) <= 0) {
      atomicAdd(p.refs + id, 1);
      bad = true;
    }
  }
  if (bad) raise(p.status, MN_DEV_BLOCK_TABLE);
}

// Ids [lo, hi) of this wave out of n: whole groups of 64.
__device__ __forceinline__ void wave_range(int n, int& lo, int& hi) {
  const int groups = (n + 63) >> 6, per = (groups + PLAN_WAVES - 1) / PLAN_WAVES, w = threadIdx.x >> 6;
  lo = min(n, w * per * 64);
  hi = min(n, (w + 1) * per * 64);
}

// f(id, refs[id], the wave's ids below this one for which it held, here) over the ids of the wave for which pick(id, refs) holds;
// returns how many there are.  Four loads are on their way at once.
template <typename P, typename F>
__device__ __forceinline__ int for_ids(const int32_t* refs, int lo, int hi, P pick, F f) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int at = lo; at < hi; at += 4 * 64) {
    int r[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = refs[min(at + 64 * u + lane, hi - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int id = at + 64 * u + lane;
      const bool in = id < hi && pick(id, r[u]);
      const uint64_t ballot = __ballot(in);
      if (in) f(id, r[u], count + __popcll(ballot & ((1ull << lane) - 1)));
      count += __popcll(ballot);
    }
  }
  return count;
}

// Exclusive prefix over the waves of a per-wave count, and the total.
__device__ __forceinline__ int wave_offset(int count, int* s_count, int& total) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_count[threadIdx.x >> 6] = count;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < PLAN_WAVES; ++w) {
    if (w == (int)(threadIdx.x >> 6)) before = total;
    total += s_count[w];
  }
  return before;
}

__global__ void __launch_bounds__(PLAN_THREADS) reserve_plan_kernel(PoolView p, const int32_t* __restrict__ tokens, int B, PoolWork w) {
  __shared__ int s_off[MN_MAX_BATCH + 1], s_shared[MN_MAX_BATCH], s_held[MN_MAX_BATCH];
  __shared__ int s_count[PLAN_WAVES], s_pairs, s_end;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bs = p.block_size;
  if (tid == 0) { s_pairs = 0; s_end = 0; }
  // ---- what every sequence needs: shared blocks that would be written, then blocks it does not have yet ----
  int carry = 0;
  for (int b0 = 0; b0 < B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    int need_shared = 0, need_tail = 0;
    if (b < B) {
      const int ctx = p.ctx_lens[b], held = p.seq_blocks[b], t = tokens[b];
      if (t > max(ctx, 0)) {
        const int first = ctx / bs, need = (int)(((long)t + bs - 1) / bs);
        bool bad = ctx < 0 || held < 0 || held > p.width || ((long)ctx + bs - 1) / bs > held || need > p.width;
        const int32_t* row = p.tables + (size_t)b * p.width;
        if (!bad) {
          for (int i = first; i < min(need, held); ++i) {
            const int id = row[i];
            if ((uint32_t)id >= (uint32_t)p.num_blocks) { bad = true; break; }
            need_shared += p.refs[id] > 1 ? 1 : 0;
          }
          need_tail = max(0, need - held);
        }
        if (bad) {
          raise(p.status, MN_DEV_BLOCK_TABLE);
          need_shared = need_tail = 0;
        }
      }
      s_shared[b] = need_shared;
      s_held[b] = held;
    }
    const int incl = wave_scan_i(need_shared + need_tail);
    int total;
    const int before = wave_offset(__builtin_amdgcn_readlane(incl, 63), s_count, total);
    if (b < B) s_off[b + 1] = carry + before + incl;
    carry += total;
  }
  if (tid == 0) s_off[0] = 0;
  // ---- the free blocks ----
  int lo, hi;
  wave_range(p.num_blocks, lo, hi);
  auto is_free = [](int, int r) { return r == 0; };
  int n_free = 0, before = 0;
  if (carry > 0) {                                               // (uniform)
    const int mine = for_ids(p.refs, lo, hi, is_free, [](int, int, int) {});
    before = wave_offset(mine, s_count, n_free);
  }
  __syncthreads();
  // sequences are served in order until the pool runs out
  for (int b = tid; b < B; b += PLAN_THREADS) {
    const int end = s_off[b + 1];
    if (end > s_off[b]) {
      if (end <= n_free) atomicMax(&s_end, end);
      else raise(p.status, MN_DEV_POOL);
    }
  }
  __syncthreads();
  const int end = s_end;
  // free block number e is the e-th that the batch asks for: it belongs to the last sequence whose share starts at or before e
  if (before < end) {
    for_ids(p.refs, lo, hi, is_free, [&](int id, int, int rank) {
      const int e = before + rank;
      if (e >= end) return;
      int a = 0, z = B;                                          // s_off[a] <= e < s_off[z]
      while (z - a > 1) {
        const int mid = (a + z) >> 1;
        if (s_off[mid] <= e) a = mid;
        else z = mid;
      }
      const int r = e - s_off[a];
      p.refs[id] = 1;
      if (r < s_shared[a]) w.list[e] = id;                       // (taken up below)
      else p.tables[(size_t)a * p.width + s_held[a] + r - s_shared[a]] = id;
    });
  }
  __syncthreads();
  for (int b = tid; b < B; b += PLAN_THREADS) {
    int e = s_off[b];
    const int stop = s_off[b + 1];
    if (stop == e || stop > end) continue;
    const int ctx = p.ctx_lens[b], held = s_held[b], first = ctx / bs;
    const int need = (int)(((long)tokens[b] + bs - 1) / bs);
    int32_t* row = p.tables + (size_t)b * p.width;
    int left = s_shared[b];
    for (int i = first; left > 0 && i < min(need, held); ++i) {
      const int id = row[i];
      if (p.refs[id] <= 1) continue;
      const int fresh = w.list[e];
      row[i] = fresh;
      w.list[e++] = id;                                          // (given up behind the barrier: the counts here stay as they were)
      --left;
      if (i == first && ctx % bs != 0) {
        const int at = atomicAdd(&s_pairs, 1);                   // (the order of the copies does not matter)
        w.from[at] = id;
        w.to[at] = fresh;
      }
    }
    p.seq_blocks[b] = max(held, need);
  }
  __syncthreads();
  for (int b = tid; b < B; b += PLAN_THREADS) {
    if (s_off[b + 1] > end) continue;
    for (int r = 0; r < s_shared[b]; ++r) atomicSub(p.refs + w.list[s_off[b] + r], 1);
  }
  if (tid == 0) *w.n_pairs = s_pairs;
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(PoolView p, PoolWork w, int32_t* __restrict__ n_live) {
  __shared__ int s_count[PLAN_WAVES];
  int lo, hi, n, moves, holes;
  wave_range(p.num_blocks, lo, hi);
  const auto nothing = [](int, int, int) {};
  wave_offset(for_ids(p.refs, lo, hi, [](int, int r) { return r > 0; }, nothing), s_count, n);
  // live blocks from id n on, in ascending order, take the free ids below n, in ascending order: there are as many of either
  const auto beyond = [=](int id, int r) { return id >= n && r > 0; };
  const auto hole = [=](int id, int r) { return id < n && !(r > 0); };
  const int from0 = wave_offset(for_ids(p.refs, lo, hi, beyond, nothing), s_count, moves);
  const int to0 = wave_offset(for_ids(p.refs, lo, hi, hole, nothing), s_count, holes);
  for_ids(p.refs, lo, hi, beyond, [&](int id, int, int rank) { w.from[from0 + rank] = id; });
  for_ids(p.refs, lo, hi, hole, [&](int id, int, int rank) { w.to[to0 + rank] = id; });
  for (int id = n + (int)threadIdx.x; id < p.num_blocks; id += PLAN_THREADS) w.map[id] = id;
  __syncthreads();
  for (int i = threadIdx.x; i < moves; i += PLAN_THREADS) {
    const int a = w.from[i], b = w.to[i];
    p.refs[b] = p.refs[a];
    p.refs[a] = 0;
    w.map[a] = b;
  }
  if (threadIdx.x == 0) {
    *w.n_pairs = moves;
    *w.n_live = n;
    if (n_live) *n_live = n;
  }
}

// Pages of the pairs in the layers of `pages`; REMAP (compaction): the first max_seqs workgroups also turn a table row each.
template <bool REMAP>
__global__ void __launch_bounds__(256) copy_pages_kernel(PoolView p, PoolWork w, LayerPages pages, int layers, uint32_t page_pieces) {
  const int tid = threadIdx.x;
  if (REMAP && (int)blockIdx.x < p.max_seqs) {
    const int n = *w.n_live;
    int32_t* row = p.tables + (size_t)blockIdx.x * p.width;
    const int held = min(max(p.seq_blocks[blockIdx.x], 0), p.width);
    for (int i = tid; i < held; i += 256) {
      const int id = row[i];
      if (id >= n && id < p.num_blocks) row[i] = w.map[id];
    }
  }
  const int pairs = *w.n_pairs;
  const uint32_t chunks = (page_pieces + COPY_CHUNK - 1) / COPY_CHUNK;
  const uint32_t per_pair = (uint32_t)layers * 2u * chunks;
  const uint64_t items = (uint64_t)pairs * per_pair;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint32_t pair = (uint32_t)(it / per_pair), rest = (uint32_t)(it % per_pair);
    const uint32_t page = rest / chunks, chunk = rest % chunks;
    char* base = static_cast<char*>((page & 1) ? pages.v[page >> 1] : pages.k[page >> 1]);
    const u32x4* a = reinterpret_cast<const u32x4*>(base + (uint64_t)(uint32_t)w.from[pair] * page_pieces * 16u);
    u32x4* b = reinterpret_cast<u32x4*>(base + (uint64_t)(uint32_t)w.to[pair] * page_pieces * 16u);
    u32x4 x[COPY_UNROLL];
#pragma unroll
    for (int u = 0; u < COPY_UNROLL; ++u) {
      const uint32_t at = chunk * COPY_CHUNK + u * 256 + tid;
      if (at < page_pieces) x[u] = a[at];
    }
#pragma unroll
    for (int u = 0; u < COPY_UNROLL; ++u) {
      const uint32_t at = chunk * COPY_CHUNK + u * 256 + tid;
      if (at < page_pieces) b[at] = x[u];
    }
  }
}

size_t pool_work_bytes(int num_blocks, int max_seqs) {
  const size_t pairs = (size_t)(num_blocks > max_seqs ? num_blocks : max_seqs);
  return 256 + 4 * (3 * pairs + (size_t)num_blocks);
}

static PoolWork pool_work(void* workspace, int num_blocks, int max_seqs) {
  const size_t pairs = (size_t)(num_blocks > max_seqs ? num_blocks : max_seqs);
  int32_t* at = static_cast<int32_t*>(workspace);
  return PoolWork{at, at + 1, at + 64, at + 64 + pairs, at + 64 + 2 * pairs, at + 64 + 3 * pairs};
}

void launch_fork(const PoolView& p, const int32_t* src, const int32_t* dst, int n, hipStream_t st) {
  fork_kernel<<<n, 256, 0, st>>>(p, src, dst, n);
}

void launch_free(const PoolView& p, const int32_t* seqs, int n, hipStream_t st) { free_kernel<<<n, 256, 0, st>>>(p, seqs); }

// Two workgroups of 256 threads per CU and more: enough for HBM, and few enough that they are quick to find nothing to do.
constexpr int COPY_WGS = 2048;

template <bool REMAP>
static void copy_pages(const PoolView& p, const PoolWork& w, void* const* k, void* const* v, int n_layers, size_t page_bytes, hipStream_t st) {
  for (int l0 = 0; l0 < n_layers; l0 += LAYERS_PER_LAUNCH) {
    LayerPages pages{};
    const int layers = n_layers - l0 < LAYERS_PER_LAUNCH ? n_layers - l0 : LAYERS_PER_LAUNCH;
    for (int l = 0; l < layers; ++l) { pages.k[l] = k[l0 + l]; pages.v[l] = v[l0 + l]; }
    if (REMAP && l0 == 0) {
      const int wgs = COPY_WGS > p.max_seqs ? COPY_WGS : p.max_seqs;
      copy_pages_kernel<true><<<wgs, 256, 0, st>>>(p, w, pages, layers, (uint32_t)(page_bytes / 16));
    } else {
      copy_pages_kernel<false><<<COPY_WGS, 256, 0, st>>>(p, w, pages, layers, (uint32_t)(page_bytes / 16));
    }
  }
}

void launch_reserve(const PoolView& p, const int32_t* tokens, int B, void* const* k, void* const* v, int n_layers, size_t page_bytes,
                    void* workspace, hipStream_t st) {
  const PoolWork w = pool_work(workspace, p.num_blocks, p.max_seqs);
  reserve_plan_kernel<<<1, PLAN_THREADS, 0, st>>>(p, tokens, B, w);
  copy_pages<false>(p, w, k, v, n_layers, page_bytes, st);
}

void launch_compact(const PoolView& p, int32_t* n_live, void* const* k, void* const* v, int n_layers, size_t page_bytes, void* workspace,
                    hipStream_t st) {
  const PoolWork w = pool_work(workspace, p.num_blocks, p.max_seqs);
  compact_plan_kernel<<<1, PLAN_THREADS, 0, st>>>(p, w, n_live);
  copy_pages<true>(p, w, k, v, n_layers, page_bytes, st);
}

}  // namespace mn
