// Attention over packed sequences, f16 / bf16: runs the items of a work plan (packed_plan.hip).
//
// A workgroup takes one item for one key head: a tile of 128 query rows (row = query * group + head in group, so the
// heads that share keys share the tile), four waves of 32 rows, against a run of key blocks of 64.  Key blocks are
// numbered [whole prefix blocks | the sequence's own | the prefix' last, partial one], so the blocks that need a mask
// come last.  Scores are taken transposed, S^T = K Q^T with v_mfma_f32_32x32x16, so a lane holds scores of one query
// (lanes l and l ^ 32 split the keys) and the online softmax is lane-local but for one half-wave exchange; O^T += V^T P^T
// with V^T from the row-major tile through ds_read_b64_tr_b16.  QK^T of block x + 1 is issued beside the softmax of
// block x; K and V go global -> LDS into two buffers each, requested a whole step ahead, one barrier per step; 64 KB, so
// two workgroups share a CU.  Q and the results pass through the second buffers, in whole rows.
//
// Maxima and sums are fp32 in the log2 domain; a row's running maximum moves (and its O is rescaled) only when it grew by
// more than 2^8.  P is rounded to the input's type, as the matrix cores take both factors in 16 bits: half a step for
// each weight, and an error against float64 1.2 to 1.4 times that of a form that rounds O alone; their sum takes the
// weights before the rounding.  O is rounded once at the end.  Rows cut into pieces leave (m, l, O) in fp32 in the
// workspace; packed_join_kernel joins them.
//
// What bounds it and what it measured (bf16 unless said): one causal sequence of 20,280, 40 / 8 heads, 3.7-4.0 ms,
// 1,050-1,140 TFLOP/s, like the dense kernel of one length (matrix cores and the clock under that load); five clips of
// 12 heads in f16 0.83-0.87 ms, 1,000-1,040; ragged prompts, 32 / 8 heads, 0.33-0.34 ms, 840-870 (about 15 blocks a tile,
// with each tile's start and masked end); video tokens attending to 20-512 text tokens 0.11-0.12 ms (tiles of 1 to 8
// blocks: the start of a workgroup, 2-3 us, and the latency of its first loads); 64 caches of up to 16,384 keys 0.21-0.22
// ms, 5.2-5.5 TB/s.  Tried while it was built, on forms that were not kept: eight waves per workgroup 1 % faster on the
// longest case, 10-50 % slower on short ones; one and two waves 1.4 to 4 times slower; several tiles per workgroup with
// the next one's first loads behind the last block 10-20 % slower (registers); the masked blocks' QK^T beside the softmax
// as well 5-25 % slower (registers); the first V and second K tile requested with the first K tile (80 KB of LDS) no
// faster; the next item's Q prefetched into L2 no faster.
#include <cfloat>

#include "attn_common.h"

namespace chorus {
namespace {

constexpr float kRescaleLog2 = 8.f;
constexpr int kTileBytes = kBlock * kHeadDim * 2;

// This wave's LDS reads have returned and its LDS writes are done.
#define CHORUS_WAIT_LDS() asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory")

// 16-byte chunk of row r that holds chunk c: the b128 reads of K and the transposed b64 reads of V then spread over
// all LDS banks.
__device__ inline int k_chunk(int r, int c) { return c ^ (r & 15); }
__device__ inline int v_bits(int r) { return (0xE4A0 >> (4 * (r & 3))) & 15; }   // 0, 10, 4, 14
__device__ inline int v_chunk(int r, int c) { return c ^ v_bits(r); }

template <bool BF16>
struct Type;
template <>
struct Type<true> {
  using vec8 = bf16x8;
  using scalar = __bf16;
  static __device__ inline f32x16 mfma(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ inline vec8 transposed(const char* lo, const char* hi) {
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)lo);
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)hi);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};
template <>
struct Type<false> {
  using vec8 = f16x8;
  using scalar = _Float16;
  static __device__ inline f32x16 mfma(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ inline vec8 transposed(const char* lo, const char* hi) {
    const f16x4 a = __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)lo));
    const f16x4 b = __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)hi));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Key head and item of a workgroup.  Workgroups go round the 8 XCDs; XCD x takes key heads x, x + 8, ..., one
// after the other (blockIdx.y), so the items in flight on it share one head's keys in its L2, and the heads beyond the
// last multiple of 8 are dealt to all XCDs item by item.
__device__ inline bool packed_slot(int Hk, int max_items, int* head, int* item) {
  const int x = blockIdx.x, y = blockIdx.y, rounds = Hk / kNumXcd, rest = Hk % kNumXcd;
  if (y < rounds) {
    *head = kNumXcd * y + x % kNumXcd;
    *item = x / kNumXcd;
  } else {
    *head = kNumXcd * y + x % rest;
    *item = x / rest;
  }
  return *item < max_items;
}
inline dim3 packed_grid(int Hk, int64_t items) {
  const unsigned max_items = (unsigned)items;
  const int rounds = Hk / kNumXcd, rest = Hk % kNumXcd;
  return dim3(rounds ? kNumXcd * max_items : rest * max_items, rounds + (rest > 0));
}

// Was the plan made for the shape of this call?  (A larger one's items would reach past this call's tensors.)
__device__ inline bool plan_fits(const PackedArgs& a, ConstI32* header) {
  int32_t differ = 0;
#pragma unroll
  for (int i = 0; i < PackedKey::n; ++i) differ |= header[kPlanShape + i] ^ a.key.field[i];
  return differ == 0;
}

// 16 bytes per lane from an address per lane to LDS (lane-linear at the wave-uniform byte address lds), as dma16.
__device__ inline void dma16_from(uint32_t lds, const char* from) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(lds), "v"(from)
      : "memory");
}

// row / group
__device__ inline int in_group(const PackedArgs& a, int row) {
  return (int)(((uint64_t)(uint32_t)row * a.group_mul) >> a.group_shift);
}

// The rows of one head in a [rows, heads, 128] tensor, cut into key blocks.
struct Rows {
  const char* base;
  uint32_t ss;         // bytes between rows
  __device__ Rows(const TensorArg& t, int64_t row0, int head)
      : base(static_cast<const char*>(t.data) + 2 * (row0 * t.ss + head * t.sh)), ss((uint32_t)(2 * t.ss)) {}
  __device__ const char* at(int block) const { return base + (int64_t)block * kBlock * ss; }
};

template <bool BF16, bool CAUSAL, bool PREFIX>
__global__ __launch_bounds__(64 * kPackedWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void packed_attn_kernel(PackedArgs a) {
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  using scalar = typename T::scalar;
  constexpr int NW = kPackedWaves, kTile = kPackedTile;
  __shared__ __attribute__((aligned(1024))) char k_s[2][kTileBytes];
  __shared__ __attribute__((aligned(1024))) char v_s[2][kTileBytes];
  __shared__ int again;

  int hk, index;
  if (!packed_slot(a.Hk, a.max_items, &hk, &index)) return;
  // read together, with scalar loads; an item behind the plan's last is within the buffer
  ConstI32* header = as_constant(a.plan.header);
  ConstI32* words = as_constant(reinterpret_cast<const int32_t*>(a.plan.items + index));
  const PackedItem it = {words[0], words[1], words[2], words[3], words[4], words[5], words[6], words[7]};
  if (!plan_fits(a, header) | (index >= header[kPlanItems])) return;
  const int nq = in_group(a, it.rows);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int l32 = lane & 31, hl = lane >> 5;
  const int g = lane >> 4, j16 = lane & 15;

  const int row = it.row0 + wave * 32 + l32;
  const bool valid = row < it.rows;
  // own keys that a row sees: this lane's, and the fewest and most of the tile
  const int shift = it.nk - nq + 1;
  auto sees = [&](int r) { return CAUSAL ? min(max(in_group(a, r) + shift, 0), it.nk) : it.nk; };
  const int seen = valid ? sees(row) : 0;
  const int seen_first = sees(it.row0), seen_last = sees(min(it.row0 + kTile, it.rows) - 1);
  const int prefix = !PREFIX || (a.pooled && it.k0 >= 0) ? 0 : a.prefix;
  const int pw = prefix / kBlock;                                     // whole prefix blocks
  const int own = (seen_last + kBlock - 1) / kBlock;
  const int n = it.j1 - it.j0;
  // leading blocks of this item that every row sees whole
  const int n_full = min(max(pw + seen_first / kBlock - it.j0, 0), n);

  const Rows ko(a.k, it.k0, hk), vo(a.v, it.k0, hk);
  const Rows kp(PREFIX ? a.pk : a.k, 0, hk), vp(PREFIX ? a.pv : a.v, 0, hk);
  const uint32_t klds = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)&k_s[0][0];
  const uint32_t vlds = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)&v_s[0][0];
  // Block x of the item into its buffer: this wave's rows of the tile, 4 per 1 KB load.  Rows past the block's end
  // read its last row again; they are masked.
  const int r0 = 4 * wave + (lane >> 4);
  auto load = [&](bool is_k, int x, int buffer) {
    const int j = it.j0 + x;
    const bool mine = !PREFIX || (j >= pw && j < pw + own);
    const int block = mine ? j - pw : min(j, pw);
    const Rows& t = is_k ? (mine ? ko : kp) : (mine ? vo : vp);
    const int rows = (mine ? it.nk : prefix) - block * kBlock;
    const char* from = t.at(block);
    const uint32_t lds = (is_k ? klds : vlds) + buffer * kTileBytes + wave * 1024;
    // both layouts repeat after 16 rows
    static_assert(4 * NW % 16 == 0, "a lane's chunk is the same in all its rows");
    const uint32_t c = 16 * (is_k ? k_chunk(r0, lane & 15) : v_chunk(r0, lane & 15));
    if (rows >= kBlock) {
#pragma unroll
      for (int u = 0; u < 16 / NW; ++u)
        dma16(lds + NW * u * 1024, from + (int64_t)(4 * NW * u) * t.ss, (uint32_t)r0 * t.ss + c);
    } else {
#pragma unroll
      for (int u = 0; u < 16 / NW; ++u)
        dma16(lds + NW * u * 1024, from, (uint32_t)min(4 * NW * u + r0, rows - 1) * t.ss + c);
    }
  };
  // V rows that no row of the tile sees (past the block's end, or keys of later queries): zeros, by the wave that loaded
  // them, before the barrier that publishes them (a weight of 0 on an infinite value would be NaN).
  auto trim = [&](int x) {
    const int j = it.j0 + x;
    const bool mine = !PREFIX || (j >= pw && j < pw + own);
    const int rows = (mine ? seen_last : prefix) - (mine ? j - pw : min(j, pw)) * kBlock;
    if (rows >= kBlock) return;
    int ln = lane;
    asm volatile("" : "+v"(ln));   // worked out here: kept across the loops the addresses would cost registers
#pragma unroll
    for (int u = 0; u < 16 / NW; ++u)
      if (4 * (NW * u + wave) + (ln >> 4) >= rows)
        *reinterpret_cast<uint4*>(v_s[x & 1] + (NW * u + wave) * 1024 + ln * 16) = make_uint4(0, 0, 0, 0);
  };
  // Address of head dim 0 of tile row r (rows past the last: the last) in q or out.
  auto row_at = [&](const TensorArg& t, int r) {
    const int at = min(it.row0 + r, it.rows - 1), token = in_group(a, at);
    return static_cast<char*>(const_cast<void*>(t.data)) +
           2 * ((int64_t)(it.q0 + token) * t.ss + (int64_t)(hk * a.group + at - token * a.group) * t.sh);
  };
  // This wave's part of the second buffers: its Q rows at first, later its results.  Rows of 256 bytes, as K's.
  char* mine_s = (wave & 2 ? v_s[1] : k_s[1]) + (wave & 1) * (kTileBytes / 2);
  if (n > 0) {
    load(true, 0, 0);
    const uint32_t lds = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)mine_s;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int r = 4 * u + (lane >> 4);
      dma16_from(lds + u * 1024, row_at(a.q, wave * 32 + r) + 16 * k_chunk(r, lane & 15));
    }
    load(false, 0, 0);
    if (CAUSAL && tid == 0) again = 0;
    CHORUS_WAIT_VMCNT(4);   // all but V's
  }
  const int k_row_off = l32 * 256;
  const int k_sw = l32 & 15;
  vec8 qf[8];
#pragma unroll
  for (int d = 0; d < 8; ++d) qf[d] = *reinterpret_cast<const vec8*>(mine_s + k_row_off + (((2 * d + hl) ^ k_sw) << 4));
  CHORUS_WAIT_LDS();   // Q is read before its place is filled
  __syncthreads();
  if (n > 1) load(true, 1, 1);
  if (it.row0 + wave * 32 >= it.rows) {
    // a wave without rows only loads its share
    for (int x = 0; x < n; ++x) {
      CHORUS_WAIT_LDS_TILES();
      if (x >= n_full) trim(x);
      CHORUS_WAIT_LDS();
      __syncthreads();
      if (x + 2 < n) load(true, x + 2, x & 1);
      if (x + 1 < n) load(false, x + 1, (x + 1) & 1);
    }
    if (CAUSAL && n_full < n && seen_first < seen_last) {
      __syncthreads();
      for (int x = 0; again && x < n; ++x) {
        __syncthreads();
        load(true, x, 0);
        load(false, x, 0);
        CHORUS_WAIT_LDS_TILES();
        __syncthreads();
      }
    }
    __syncthreads();
    return;
  }
  const int v_lane_off = (j16 >> 2) * 256 + 8 * (j16 & 1) + 4 * (g >> 1) * 256;
  const int v_c0 = 2 * (g & 1) + ((j16 & 3) >> 1);
  const int v_sw = v_bits(j16 >> 2);

  const float cl2 = a.sm_scale * kLog2e;
  // finite from the start: a block may hold no key that a row sees, and -inf - (-inf) is NaN
  float m_run = -FLT_MAX, l_run = 0.f;
  f32x16 o[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[u][r] = 0.f;

  auto qk = [&](f32x16 (&s)[2], const char* kt) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = T::mfma(*reinterpret_cast<const vec8*>(kt + t * 32 * 256 + k_row_off + (((2 * d + hl) ^ k_sw) << 4)),
                       qf[d], s[t]);
  };
  // keys of block x that this row sees
  auto limit = [&](int x) {
    const int j = it.j0 + x;
    return !PREFIX || (j >= pw && j < pw + own) ? seen - (j - pw) * kBlock : valid ? prefix - min(j, pw) * kBlock : 0;
  };
  auto mask = [&](f32x16 (&s)[2], int lim) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * t + 8 * (r >> 2) + 4 * hl + (r & 3) >= lim) s[t][r] = -INFINITY;
  };
  auto row_max = [&](const f32x16 (&s)[2]) {
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    return pair_max(mx);
  };
  auto rescale = [&](float mx) {
    const float m_new = fmaxf(m_run, mx * cl2);
    const bool grew = m_new > m_run + kRescaleLog2;
    if (__builtin_amdgcn_ballot_w64(grew) != 0) {
      // each row for itself: moved along with another row of the wave, its weights would round by what that one sees
      const float alpha = grew ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      m_run = grew ? m_new : m_run;
      l_run *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[u][r] *= alpha;
    }
  };
  auto probs = [&](const f32x16 (&s)[2], vec8 (&pf)[2][2]) {
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(s[t][r] * cl2 - m_run);
        sum += p;
        pf[t][r >> 3][r & 7] = (scalar)p;
      }
    l_run += sum;
  };
  auto pv = [&](const vec8 (&pf)[2][2], const char* vt) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const char* lo = vt + (32 * t + 16 * hh) * 256 + v_lane_off + (((4 * u + v_c0) ^ v_sw) << 4);
          o[u] = T::mfma(T::transposed(lo, lo + 8 * 256), pf[t][hh], o[u]);
        }
  };

  if (n > 0) {
    f32x16 s0[2], s1[2];
    float mx;
    qk(s0, k_s[0]);
    if (n_full == 0) mask(s0, limit(0));
    mx = row_max(s0);

    // Block x: its softmax beside QK^T of block x + 1, then PV.
    auto fused = [&](int x, int par, f32x16 (&sc)[2], f32x16 (&sn)[2]) {
      CHORUS_WAIT_LDS_TILES();
      __syncthreads();
      if (x + 2 < n) load(true, x + 2, x & 1);
      load(false, x + 1, (x + 1) & 1);
      rescale(mx);
      vec8 pf[2][2];
      qk(sn, k_s[par ^ 1]);
      probs(sc, pf);
      pv(pf, v_s[par]);
      mx = row_max(sn);
    };
    int x = 0;
    for (; x + 2 < n_full; x += 2) {
      fused(x, 0, s0, s1);
      fused(x + 1, 1, s1, s0);
    }
    // the blocks that need a mask, and up to two ahead of them
    for (; x < n; ++x) {
      const int par = x & 1;
      CHORUS_WAIT_LDS_TILES();
      if (x >= n_full) trim(x);
      CHORUS_WAIT_LDS();
      __syncthreads();
      if (x + 2 < n) load(true, x + 2, x & 1);
      if (x + 1 < n) load(false, x + 1, (x + 1) & 1);
      rescale(mx);
      vec8 pf[2][2];
      probs(s0, pf);
      pv(pf, v_s[par]);
      if (x + 1 < n) {
        qk(s0, k_s[par ^ 1]);
        if (x + 1 >= n_full) mask(s0, limit(x + 1));
        mx = row_max(s0);
      }
    }

    // A value that some row of the tile sees and another does not may be infinite or NaN, and a weight of 0 on it NaN.
    // Where that may have happened the item is done again, with the masked blocks' PV key by key for the rows that
    // give the key a weight: slow, in few registers, and rare.
    if (CAUSAL && n_full < n && seen_first < seen_last) {
      float zero = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero += o[u][r] * 0.f;
      if (__builtin_amdgcn_ballot_w64(!(zero == 0.f)) != 0) again = 1;
      __syncthreads();
      if (again) {
        m_run = -FLT_MAX;
        l_run = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[u][r] = 0.f;
        // this wave's weights, [row][key]: the second buffers hold 8 KB for each of up to 4 waves
        float* w_s = reinterpret_cast<float*>(mine_s);
#pragma unroll 1
        for (x = 0; x < n; ++x) {
          __syncthreads();
          load(true, x, 0);
          load(false, x, 0);
          CHORUS_WAIT_LDS_TILES();
          __syncthreads();   // (rows past the end have weight 0 and are passed over)
          qk(s0, k_s[0]);
          if (x >= n_full) mask(s0, limit(x));
          rescale(row_max(s0));
          vec8 pf[2][2];
          probs(s0, pf);
          if (x < n_full) {
            pv(pf, v_s[0]);
            continue;
          }
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) w_s[l32 * kBlock + 32 * t + 8 * (r >> 2) + 4 * hl + (r & 3)] = (float)pf[t][r >> 3][r & 7];
          CHORUS_WAIT_LDS_TILES();
#pragma unroll 1
          for (int key = 0; key < kBlock; ++key) {
            const float w = w_s[l32 * kBlock + key];
            if (!(w == 0.f)) {
#pragma unroll
              for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) {
                  const int d = 32 * u + 8 * rr + 4 * hl;
                  const uint2 v4 = *reinterpret_cast<const uint2*>(v_s[0] + key * 256 + v_chunk(key, d >> 3) * 16 + (d & 4) * 2);
                  scalar v[4];
                  __builtin_memcpy(v, &v4, 8);
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[u][4 * rr + e] += w * (float)v[e];
                }
            }
          }
        }
      }
    }
  }

  const float l_tot = pair_sum(l_run);
  const bool empty = l_tot == 0.f;   // NaN is not
  const float inv_l = empty ? 0.f : 1.f / l_tot;
  CHORUS_WAIT_LDS_TILES();
  __syncthreads();                   // the tiles are done with
  // the rows' places, worked out again: kept across the loops they would cost registers
  int lane2 = tid & 63;
  asm volatile("" : "+v"(lane2));
  const int r32 = lane2 & 31, hl2 = lane2 >> 5;
  const int left = it.rows - it.row0 - wave * 32;   // rows of this wave
  // Results go through LDS, so that each store writes whole rows: written from the accumulators, 16 bytes of each
  // of 32 rows at a time, 25,600 x 24 rows without keys took 98 us, this way 33.
  if (it.slot != kFinished) {
    const int64_t row0 = it.slot == kByRow ? a.by_row + (int64_t)hk * a.total_q * a.group + it.q0 * a.group -
                                                 header[kPlanFirstRow] + it.row0
                                           : ((int64_t)it.slot * a.Hk + hk) * kTile;
    const int64_t at = row0 + wave * 32;
#pragma unroll
    for (int half = 0; half < 2; ++half) {   // 64 of a row's 128 values fit the wave's 8 KB
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const f32x16& v = o[2 * half + u];
          *reinterpret_cast<float4*>(mine_s + r32 * 256 + k_chunk(r32, 8 * u + 2 * rr + hl2) * 16) =
              make_float4(v[4 * rr], v[4 * rr + 1], v[4 * rr + 2], v[4 * rr + 3]);
        }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int r = 4 * u + (lane2 >> 4), c = lane2 & 15;
        const float4 v = *reinterpret_cast<const float4*>(mine_s + r * 256 + k_chunk(r, c) * 16);
        if (r < left) *reinterpret_cast<float4*>(a.part_o + (at + r) * kHeadDim + 64 * half + 4 * c) = v;
      }
    }
    if (hl2 == 0 && r32 < left) *reinterpret_cast<float2*>(a.part_ml + 2 * (at + r32)) = make_float2(m_run, l_tot);
    return;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      scalar v4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v4[e] = (scalar)(o[u][4 * rr + e] * inv_l);
      uint2 packed;
      __builtin_memcpy(&packed, v4, 8);
      *reinterpret_cast<uint2*>(mine_s + r32 * 256 + k_chunk(r32, 4 * u + rr) * 16 + 8 * hl2) = packed;
    }
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const int r = 4 * u + (lane2 >> 4), c = lane2 & 15;
    const uint4 v = *reinterpret_cast<const uint4*>(mine_s + r * 256 + k_chunk(r, c) * 16);
    if (r < left) *reinterpret_cast<uint4*>(row_at(a.o, wave * 32 + r) + 16 * c) = v;
  }
  if (a.lse && hl2 == 0 && r32 < left) {
    const int row = it.row0 + wave * 32 + r32, token = in_group(a, row);
    a.lse[(int64_t)(hk * a.group + row - token * a.group) * a.total_q + it.q0 + token] =
        empty ? -INFINITY : (m_run + __builtin_log2f(l_tot)) * kLn2;
  }
}

// Joins a tile's pieces: with m the largest of their maxima, O = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.
// 32 lanes per row, a workgroup for 8 rows at a time; the maxima of up to 32 pieces are read at once.
template <bool BF16>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
  using scalar = typename Type<BF16>::scalar;
  constexpr int kTile = kPackedTile;
  ConstI32* header = as_constant(a.plan.header);
  if (!plan_fits(a, header)) return;
  const int np = header[kPlanPrefixPieces], first_row = header[kPlanFirstRow];
  const int64_t tiles = (int64_t)header[kPlanJoins] * a.Hk;
  const int64_t units = tiles * ((header[kPlanJoinRows] + 7) / 8);   // eight rows of a tile each
  const int lane = threadIdx.x & 31;
  for (int64_t w = blockIdx.x; w < units; w += gridDim.x) {
    const int r = (int)(w / tiles) * 8 + (threadIdx.x >> 5);
    const int hk = (int)(w % a.Hk);
    const PackedJoin jn = a.plan.joins[w % tiles / a.Hk];
    const int row = jn.row0 + r;
    if (row >= jn.rows) continue;
    const int n = jn.pieces + np;
    const int pooled = jn.q0 * a.group - first_row + row;   // among the rows of all sequences
    auto at = [&](int i) {
      if (jn.slot == kByRow && i < jn.pieces) return a.by_row + (int64_t)hk * a.total_q * a.group + pooled;
      const int64_t slot = i < jn.pieces ? jn.slot + i : pooled / kTile * np + (i - jn.pieces);
      return (slot * a.Hk + hk) * kTile + (i < jn.pieces ? r : pooled % kTile);
    };
    float m = -FLT_MAX;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, a.part_ml[2 * at(i)]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 32));
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int base = 0; base < n; base += 32) {
      const int mine = base + lane;
      float f = 0.f;
      if (mine < n) {
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * at(mine));
        f = __builtin_amdgcn_exp2f(ml.x - m);
        l += f * ml.y;
      }
      const int some = min(n - base, 32);
      for (int i = 0; i < some; i += 4) {   // four loads in flight
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = i + e < some ? *reinterpret_cast<const float4*>(a.part_o + at(base + i + e) * kHeadDim + 4 * lane)
                              : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float fi = __shfl(f, i + e, 32);
          o.x += fi * v[e].x;
          o.y += fi * v[e].y;
          o.z += fi * v[e].z;
          o.w += fi * v[e].w;
        }
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor(l, d, 32);
    const bool empty = l == 0.f;
    const float inv_l = empty ? 0.f : 1.f / l;
    const int token = in_group(a, row), query = jn.q0 + token, qh = hk * a.group + row - token * a.group;
    const scalar v4[4] = {(scalar)(o.x * inv_l), (scalar)(o.y * inv_l), (scalar)(o.z * inv_l), (scalar)(o.w * inv_l)};
    uint2 packed;
    __builtin_memcpy(&packed, v4, 8);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(const_cast<void*>(a.o.data)) + (int64_t)query * a.o.ss +
                              (int64_t)qh * a.o.sh + 4 * lane) = packed;
    if (a.lse && lane == 0)
      a.lse[(int64_t)qh * a.total_q + query] = empty ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
  }
}

template <bool BF16>
void launch_packed(const PackedConfig& c, const PackedArgs& a, hipStream_t st) {
  const dim3 grid = packed_grid(a.Hk, c.max_items), block(64 * kPackedWaves);
  if (a.causal && a.prefix > 0)
    hipLaunchKernelGGL((packed_attn_kernel<BF16, true, true>), grid, block, 0, st, a);
  else if (a.causal)
    hipLaunchKernelGGL((packed_attn_kernel<BF16, true, false>), grid, block, 0, st, a);
  else if (a.prefix > 0)
    hipLaunchKernelGGL((packed_attn_kernel<BF16, false, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((packed_attn_kernel<BF16, false, false>), grid, block, 0, st, a);
  // How many rows there are to join is known on the device alone: 2,048 workgroups go through them (eight prompts behind
  // a prefix 10 us, with 256, 512 or 1,024 29, 18, 12, with 4,096 10); without any they take 4-5 us, as fewer do.
  const int64_t groups = c.max_joins * a.Hk * (kPackedTile / 8);
  hipLaunchKernelGGL((packed_join_kernel<BF16>), dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_packed_attn(chorus_dtype dt, const PackedConfig& c, const PackedArgs& a, hipStream_t st) {
  if (dt == CHORUS_BF16)
    launch_packed<true>(c, a, st);
  else
    launch_packed<false>(c, a, st);
  return hipGetLastError();
}

}  // namespace chorus
