// Work plan of attention over packed sequences: from the lengths on the device to a list of workgroups.
//
// Every sequence's query rows (query * group + head in group, so that the heads that share a key head share its
// tiles) are cut into tiles of kPackedTile rows, and a tile's key blocks (64 keys) into pieces where whole tiles
// would leave the GPU unevenly filled: with C key blocks in all, a piece has about C / per_head blocks.  A prefix
// is either part of each tile's key blocks, or, pooled, a pass of its own whose tiles run over the rows of all
// sequences, so its keys are read once per tile of rows and not once per sequence.  Items are listed longest
// first (by 64 classes of length), so the last workgroups to start are the shortest.
//
// One workgroup: three passes over the tiles (cost, classes, emission) between block scans: 6 to 9 us for 4 to 600 tiles
// a head, bound by its barriers and the latency of a few dependent loads.
// A plan never exceeds packed_config's bounds: with pieces of at least C / per_head blocks the cuts come to fewer than
// per_head pieces more than there were tiles, and the tiles that are cut (5 / 4 of a piece or longer) to fewer than
// per_head; a pooled prefix comes to one piece for each of its tiles or to kPrefixPlaces / key heads.
#include <algorithm>

#include "chorus_internal.h"

namespace chorus {

// Blocks of a piece at least.  One query against 16,384 keys, 32 / 8 heads: 33.6 us with 1 or 2, 28.6 with 4, 26.1 with 8
// (the join grows with the pieces); against 2,048: 17.2, 16.7, 17.8, 20.9; eight sequences of 300, 16 / 4 heads, causal:
// 32 with 1 or 2, 19.9 with 4 or more.
constexpr int kMinChunk = 4;
// Pieces of a pooled prefix, over all tiles and key heads at most: one for each CU, as long as the short tiles of the
// sequences' own keys come beside them (96 single tokens behind 16,384 keys, 32 / 8 heads: 57 us, cut by C / per_head as
// the others 60-62; 64 behind 30,000, 40 / 8 heads: 70, 73).
constexpr int kPrefixPlaces = 256;
constexpr int kClasses = 64;

PackedPlan carve_packed_plan(void* plan, int n_seqs, const PackedConfig& c, size_t* bytes) {
  Carver v(plan);
  PackedPlan p;
  p.header = v.take<int32_t>(kPlanHeader);
  p.seqs = v.take<PackedSeq>((size_t)n_seqs + 1);
  p.items = v.take<PackedItem>(c.max_items);
  p.joins = v.take<PackedJoin>(c.max_joins);
  if (bytes) *bytes = align_up(v.used, 256);
  return p;
}

PackedConfig packed_config(const chorus_packed_shape& s) {
  PackedConfig c;
  const int group = s.q_heads / s.kv_heads;
  const int64_t rows = (int64_t)s.total_q * group;
  const int tile = kPackedTile;
  // The prefix is worth a pass of its own when the sequences' own tiles are mostly empty: then a tile of pooled rows
  // replaces several walks over it.  16 sequences x 8,192 rows of prefix, 32 / 8 heads: 4 rows each 26 us (walked by
  // each 63), 64 rows 55 (67), 96 rows 85 (74); 64 x 2,048: 24 (55), 66 (61), 84 (69).
  c.pooled = s.prefix > 0 && s.n_seqs > 1 && 2 * rows <= (int64_t)s.n_seqs * tile;
  // Two workgroups fit a CU.  Single tokens are bound by memory and their join is short, so three pieces for every two
  // places even out the end: 64 caches of up to 16,384 keys 226 -> 214 us.  With full tiles two workgroups of a CU
  // slow each other down and the join is longer: three pieces for four places (40 heads x 1,024: 38 us, 512 pieces 50,
  // 256 39; eight prompts behind a prefix, 16 / 4 heads: 109 + 10 us of join, 117 + 12, 131 + 4).
  c.tokens = s.max_q > 0 && s.max_q * (int64_t)group <= 32;
  c.per_head = ((c.tokens && !c.pooled ? 768 : 384) + s.kv_heads - 1) / s.kv_heads;
  const int64_t tiles = rows / tile + s.n_seqs, pooled_tiles = c.pooled ? rows / tile + 1 : 0;
  const int64_t prefix_cuts = c.pooled ? kPrefixPlaces / s.kv_heads : 0;
  c.max_items = tiles + pooled_tiles + prefix_cuts + c.per_head;
  c.max_slots = pooled_tiles + prefix_cuts + 2 * c.per_head;
  c.max_joins = c.pooled ? tiles : c.per_head;
  c.row_slots = c.pooled ? rows : 0;
  return c;
}

namespace {

constexpr int kMaxThreads = 1024;

struct PlanArgs {
  const int32_t* q_offsets;
  const int32_t* k_offsets;
  const int32_t* k_lens;
  PackedPlan plan;
  int n_seqs, total_q, total_k, prefix, group, kv_heads, causal, tile, pooled, tokens, per_head;
  PackedKey key;
};

// Inclusive scan over the workgroup (every thread takes part); `total` is the last thread's value.
template <class T, class Op>
__device__ inline T block_scan(T v, Op op, T* wave_s, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T u = __shfl_up(v, d);
    if (lane >= d) v = op(u, v);
  }
  __syncthreads();
  if (lane == 63) wave_s[wave] = v;
  __syncthreads();
  T before = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
    if (w == wave && w > 0) v = op(before, v);
    before = w ? op(before, wave_s[w]) : wave_s[0];
  }
  *total = before;
  return v;
}

struct Add {
  template <class T>
  __device__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
  __device__ int operator()(int a, int b) const { return a > b ? a : b; }
};

struct Tile {
  PackedSeq seq;
  int row0, rows, blocks;
};

// Up to this many sequences are kept in LDS, more in the plan buffer.
constexpr int kNear = 1024;

template <class Seqs>
__device__ inline Tile tile_at(const PlanArgs& a, const Seqs& seqs, int t) {
  int lo = 0, hi = a.n_seqs;   // the last sequence whose first tile is at or before t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seqs[mid].tile0 <= t)
      lo = mid;
    else
      hi = mid;
  }
  Tile x;
  x.seq = seqs[lo];
  const int nq = seqs[lo + 1].q0 - x.seq.q0;
  x.rows = nq * a.group;
  x.row0 = (t - x.seq.tile0) * a.tile;
  int seen = x.seq.nk;
  if (a.causal) {
    const int last = (min(x.row0 + a.tile, x.rows) - 1) / a.group;
    seen = min(max(last + 1 + seen - nq, 0), seen);
  }
  x.blocks = (seen + kBlock - 1) / kBlock + (a.pooled ? 0 : (a.prefix + kBlock - 1) / kBlock);
  return x;
}

template <bool NEAR>
__global__ __launch_bounds__(kMaxThreads) void packed_plan_kernel(PlanArgs a) {
  __shared__ int wave_s[kMaxThreads / 64];
  __shared__ unsigned long long cost_s, wave_l[kMaxThreads / 64];
  __shared__ int flags_s, join_rows_s, class_s[kClasses];
  __shared__ PackedSeq near_s[NEAR ? kNear + 1 : 1];
  PackedSeq* far = a.plan.seqs;
  auto seqs = [&]() -> auto& {
    if constexpr (NEAR)
      return near_s;
    else
      return far;
  };
  auto& seq = seqs();
  const int tid = threadIdx.x, threads = blockDim.x, N = a.n_seqs;
  if (tid == 0) {
    cost_s = 0;
    flags_s = 0;
    join_rows_s = 0;
#pragma unroll
    for (int i = 0; i < PackedKey::n; ++i) a.plan.header[kPlanShape + i] = a.key.field[i];
  }
  if (tid < kClasses) class_s[tid] = 0;
  // key rows first: their loads are in flight during the first scan
  int flags = 0;
  for (int i = tid; i < N; i += threads) {
    const int raw0 = a.k_offsets[i];
    const int64_t raw = a.k_lens ? a.k_lens[i] : (int64_t)a.k_offsets[i + 1] - raw0;
    const int k0 = min(max(raw0, 0), a.total_k);
    const int nk = (int)min(max(raw, (int64_t)0), (int64_t)(a.total_k - k0));
    if (k0 != raw0 || nk != raw) flags |= 2;
    seq[i].k0 = k0;
    seq[i].nk = nk;
  }
  int run = 0, total;
  for (int base = 0; base <= N; base += threads) {
    const int i = base + tid;
    const int raw = i <= N ? a.q_offsets[i] : 0;
    const int v = max(run, block_scan(min(max(raw, 0), a.total_q), Max(), wave_s, &total));
    run = max(run, total);
    if (i <= N) {
      seq[i].q0 = v;
      if (v != raw) flags |= 1;
    }
  }
  if (flags) atomicOr(&flags_s, flags);
  __syncthreads();
  run = 0;
  for (int base = 0; base < N; base += threads) {
    const int i = base + tid;
    int tiles = 0;
    if (i < N) {
      const int64_t rows = (int64_t)(seq[i + 1].q0 - seq[i].q0) * a.group;
      tiles = (int)((rows + a.tile - 1) / a.tile);
    }
    const int upto = run + block_scan(tiles, Add(), wave_s, &total);
    run += total;
    if (i < N) seq[i].tile0 = upto - tiles;
  }
  const int n_tiles = run;
  __syncthreads();

  const int first = seq[0].q0;
  const int pooled_rows = (seq[N].q0 - first) * a.group;
  const int pooled_tiles = a.pooled ? (pooled_rows + a.tile - 1) / a.tile : 0;
  const int prefix_blocks = (a.prefix + kBlock - 1) / kBlock;
  // this thread's first tile is kept; most plans have no second
  const Tile mine = tid < n_tiles ? tile_at(a, seq, tid) : Tile{};
  unsigned long long cost = mine.blocks;
  for (int t = tid + threads; t < n_tiles; t += threads) cost += tile_at(a, seq, t).blocks;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) cost += __shfl_xor(cost, d);
  if ((tid & 63) == 0) atomicAdd(&cost_s, cost);
  __syncthreads();
  cost = cost_s + (unsigned long long)pooled_tiles * prefix_blocks;
  // (the quotient in fp32: which blocks make a piece may be off by one in 2^24)
  const int piece = max((int)min((float)cost / (float)a.per_head + 1.f, (float)(1 << 26)), kMinChunk);
  const int longest = piece + piece / 4;
  // A cut saves blocks - blocks / p blocks of a tile's way and costs its rows a join; with more than half the CUs taken
  // by whole tiles that is not worth it for 5 blocks (32 / 8 heads x 700 keys: 24 us whole, 29 cut; 40 x 512: 20 - 24,
  // 26), with fewer it is for any (8 heads x 700 keys, causal: 21 us with every cut, 24 without the short ones).
  const int worth = a.pooled || a.tokens || (int64_t)n_tiles * a.kv_heads <= 128 ? 1 : 6;
  auto pieces = [&](int blocks) {
    const int p = (blocks + piece - 1) / piece;
    return blocks > longest && blocks - (blocks + p - 1) / p >= worth ? p : 1;
  };
  const float per_class = (float)kClasses / (float)(longest + 1);
  // first block of piece i of p
  auto cut = [](int blocks, int p, int i) { return blocks / p * i + min(blocks % p, i); };
  auto class_of = [&](int blocks, int p) {
    return kClasses - 1 - min((int)((float)((blocks + p - 1) / p) * per_class), kClasses - 1);
  };
  const int np =
      pooled_tiles ? max(min(kPrefixPlaces / max(pooled_tiles * a.kv_heads, 1), prefix_blocks / kMinChunk), 1) : 0;

  for (int t = tid; t < n_tiles; t += threads) {
    const int n = t < threads ? mine.blocks : tile_at(a, seq, t).blocks, p = pieces(n);
    if (n > 0 || !a.pooled) atomicAdd(&class_s[class_of(n, p)], p);
  }
  if (tid == 0 && np) atomicAdd(&class_s[class_of(prefix_blocks, np)], pooled_tiles * np);
  __syncthreads();
  if (tid < kClasses) {   // first position of each class
    int v = class_s[tid];
    const int own = v;
#pragma unroll
    for (int d = 1; d < kClasses; d *= 2) {
      const int u = __shfl_up(v, d);
      if (tid >= d) v += u;
    }
    class_s[tid] = v - own;
    if (tid == kClasses - 1) a.plan.header[kPlanItems] = v;
  }
  __syncthreads();

  for (int x = tid; x < pooled_tiles * np; x += threads) {
    const int t = x / np, i = x % np;
    const int at = atomicAdd(&class_s[class_of(prefix_blocks, np)], 1);
    a.plan.items[at] = {first, t * a.tile, pooled_rows, cut(prefix_blocks, np, i),
                        cut(prefix_blocks, np, i + 1), -1, 0, x};
  }
  int slots = pooled_tiles * np, joins = 0, join_rows = 0;
  for (int base = 0; base < n_tiles; base += threads) {
    const int t = base + tid;
    Tile x = {};
    int p = 0, own = 0, joined = 0;
    if (t < n_tiles) {
      x = base ? tile_at(a, seq, t) : mine;
      p = a.pooled && x.blocks == 0 ? 0 : pieces(x.blocks);
      joined = a.pooled || p > 1;
      own = p > 1 ? p : 0;   // a whole tile of a pooled batch leaves its result by row
    }
    unsigned long long both = (unsigned long long)own << 32 | joined, upto;   // slots and joins in one scan
    both = block_scan(both, Add(), wave_l, &upto) - both;
    const int slot = slots + (int)(both >> 32), join = joins + (int)(uint32_t)both;
    slots += (int)(upto >> 32);
    joins += (int)(uint32_t)upto;
    const int first_slot = p > 1 ? slot : joined ? kByRow : kFinished;
    if (p) {
      int at = atomicAdd(&class_s[class_of(x.blocks, p)], p);
      for (int i = 0; i < p; ++i, ++at)
        a.plan.items[at] = {x.seq.q0, x.row0, x.rows, cut(x.blocks, p, i), cut(x.blocks, p, i + 1),
                            x.seq.k0, x.seq.nk, first_slot + i};
    }
    if (joined) {
      join_rows = max(join_rows, min(x.rows - x.row0, a.tile));
      a.plan.joins[join] = {x.seq.q0, x.row0, x.rows, first_slot, p, {0, 0, 0}};
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) join_rows = max(join_rows, __shfl_xor(join_rows, d));
  if ((tid & 63) == 0) atomicMax(&join_rows_s, join_rows);
  __syncthreads();
  if (tid == 0) {
    a.plan.header[kPlanJoinRows] = join_rows_s;
    a.plan.header[kPlanJoins] = joins;
    a.plan.header[kPlanFlags] = flags_s;
    a.plan.header[kPlanPrefixPieces] = np;
    a.plan.header[kPlanFirstRow] = first * a.group;
  }
}

}  // namespace

hipError_t launch_packed_plan(const chorus_packed_shape& s, const PackedConfig& c, const int32_t* q_offsets,
                              const int32_t* k_offsets, const int32_t* k_lens, const PackedPlan& plan, hipStream_t st) {
  const PlanArgs a = {q_offsets, k_offsets, k_lens,   plan,       s.n_seqs, s.total_q,  s.total_k, s.prefix,
                      s.q_heads / s.kv_heads, s.kv_heads, s.causal, kPackedTile, c.pooled, c.tokens, c.per_head, packed_key(s)};
  // a thread for each sequence and tile, as far as a workgroup goes: few threads pass its barriers sooner
  const int most = std::max(s.n_seqs + 1, (int)std::min<int64_t>(c.max_items, kMaxThreads));
  const int threads = std::min((most + 63) / 64 * 64, kMaxThreads);
  if (s.n_seqs <= kNear)
    hipLaunchKernelGGL((packed_plan_kernel<true>), dim3(1), dim3(threads), 0, st, a);
  else
    hipLaunchKernelGGL((packed_plan_kernel<false>), dim3(1), dim3(threads), 0, st, a);
  return hipGetLastError();
}

}  // namespace chorus
