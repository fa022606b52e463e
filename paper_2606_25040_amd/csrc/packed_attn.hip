// Attention over packed sequences, f16 / bf16: runs the items of a work plan (packed_plan.hip).
//
// A workgroup takes one item for one key head: 32 * NW query rows (row = query * group + head in group), a wave 32
// of them, against a run of key blocks of 64.  Key blocks are numbered [whole prefix blocks | the sequence's own |
// the prefix' last, partial one], so the blocks that need a mask come last.  Scores are taken transposed,
// S^T = K Q^T with v_mfma_f32_32x32x16, so a lane holds scores of one query (lanes l and l ^ 32 split the keys) and
// the online softmax is lane-local but for one half-wave exchange; O^T += V^T P^T with V^T from the row-major tile
// through ds_read_b64_tr_b16.  Maxima and sums are fp32 in the log2 domain; P is rounded to the input's type for
// the matrix cores, as O is once at the end; the running maximum moves (and O is rescaled) only when a row's
// grew by more than 2^8.
//
// Rows cut into pieces leave (m, l, O) in fp32 in the workspace; packed_join_kernel joins them.
#include <cfloat>

#include "attn_common.h"

namespace chorus {
namespace {

constexpr float kRescaleLog2 = 8.f;
constexpr int kTileBytes = kBlock * kHeadDim * 2;

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
  static constexpr uint32_t kExp = 0x7f807f80u, kOne = 0x3f80u, kLow = 0x00800080u;   // exponent bits, 1.0
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
  static constexpr uint32_t kExp = 0x7c007c00u, kOne = 0x3c00u, kLow = 0x04000400u;
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
// after the other, so the items in flight on it share one head's keys in its L2, and the heads beyond the last
// multiple of 8 are dealt to all XCDs item by item.
__device__ inline bool packed_slot(int Hk, int max_items, int* head, int* item) {
  const int x = blockIdx.x % kNumXcd, k = blockIdx.x / kNumXcd;
  const int rounds = Hk / kNumXcd, rest = Hk % kNumXcd;
  if (k < rounds * max_items) {
    *head = k / max_items * kNumXcd + x;
    *item = k % max_items;
    return true;
  }
  const int left = (k - rounds * max_items) * kNumXcd + x;
  *head = rounds * kNumXcd + left % rest;
  *item = left / rest;
  return *item < max_items;
}
inline int64_t packed_grid(int Hk, int max_items) {
  const int64_t rest = (int64_t)(Hk % kNumXcd) * max_items;
  return kNumXcd * ((int64_t)(Hk / kNumXcd) * max_items + (rest + kNumXcd - 1) / kNumXcd);
}

// One key block: its first rows and how many there are (>= 1; 64 if more).
struct Block {
  const char* k;
  const char* v;
  uint32_t kss, vss;   // bytes between rows
  int rows;
};

template <bool BF16, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void packed_attn_kernel(PackedArgs a) {
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  using scalar = typename T::scalar;
  __shared__ __attribute__((aligned(1024))) char k_s[kTileBytes];
  __shared__ __attribute__((aligned(1024))) char v_s[kTileBytes];

  int hk, index;
  if (!packed_slot(a.Hk, a.max_items, &hk, &index)) return;
  if (a.plan.header[kPlanKey] != a.key || index >= a.plan.header[kPlanItems]) return;
  const PackedItem it = a.plan.items[index];
  const int nq = it.rows / a.group;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int l32 = lane & 31, hl = lane >> 5;
  const int g = lane >> 4, j16 = lane & 15;

  const int row = it.row0 + wave * 32 + l32;
  const bool valid = row < it.rows;
  const int query = row / a.group, qh = hk * a.group + row % a.group;
  // own keys that this row sees, and the fewest of the tile
  const int shift = it.nk - nq + 1;
  const int seen = !valid ? 0 : a.causal ? min(max(query + shift, 0), it.nk) : it.nk;
  const int seen_first = a.causal ? min(max(it.row0 / a.group + shift, 0), it.nk) : it.nk;
  const int last_row = min(it.row0 + 32 * NW, it.rows) - 1;
  const int seen_last = a.causal ? min(max(last_row / a.group + shift, 0), it.nk) : it.nk;
  const int prefix = a.pooled && it.k0 >= 0 ? 0 : a.prefix;
  const int pw = prefix / kBlock;                                     // whole prefix blocks
  const int own = (seen_last + kBlock - 1) / kBlock;

  auto block = [&](int j) {
    Block x;
    const bool mine = j >= pw && j < pw + own;
    const TensorArg& kt = mine ? a.k : a.pk;
    const TensorArg& vt = mine ? a.v : a.pv;
    const int first = mine ? (j - pw) * kBlock : min(j, pw) * kBlock;
    x.rows = min((mine ? it.nk : prefix) - first, kBlock);
    const int64_t at = (mine ? it.k0 : 0) + (int64_t)first;
    x.k = static_cast<const char*>(kt.data) + 2 * (at * kt.ss + hk * kt.sh);
    x.v = static_cast<const char*>(vt.data) + 2 * (at * vt.ss + hk * vt.sh);
    x.kss = (uint32_t)(2 * kt.ss);
    x.vss = (uint32_t)(2 * vt.ss);
    return x;
  };
  const uint32_t klds = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)&k_s[0];
  const uint32_t vlds = (uint32_t)(size_t)(__attribute__((address_space(3))) char*)&v_s[0];
  // This wave's rows of a tile: 4 rows per 1 KB load.  Rows past the block's end read its last row again: they
  // are masked.
  auto load = [&](uint32_t lds, const char* base, uint32_t ss, int rows, bool is_k) {
#pragma unroll
    for (int u = 0; u < 16 / NW; ++u) {
      const int r = 4 * (NW * u + wave) + (lane >> 4);
      const int c = is_k ? k_chunk(r, lane & 15) : v_chunk(r, lane & 15);
      dma16(lds + (NW * u + wave) * 1024, base, (uint32_t)min(r, rows - 1) * ss + (uint32_t)c * 16);
    }
  };

  vec8 qf[8];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q.data) + (int64_t)(it.q0 + query) * a.q.ss +
                         (int64_t)qh * a.q.sh + 8 * hl;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (valid) {
        qf[s] = *reinterpret_cast<const vec8*>(qp + 16 * s);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) qf[s][e] = (scalar)0.f;
      }
    }
  }
  const int k_row_off = l32 * 256;
  const int k_sw = l32 & 15;
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

  for (int j = it.j0; j < it.j1; ++j) {
    const Block x = block(j);
    const bool mine = j >= pw && j < pw + own;
    const int first = (j - pw) * kBlock;                        // of an own block
    const int lim = mine ? seen - first : valid ? x.rows : 0;   // keys of this block that the row sees
    const bool masked = mine ? first + kBlock > seen_first : x.rows < kBlock;
    __syncthreads();
    load(klds, x.k, x.kss, x.rows, true);
    load(vlds, x.v, x.vss, x.rows, false);
    CHORUS_WAIT_LDS_TILES();
    __syncthreads();
    if (__builtin_amdgcn_ballot_w64(lim > 0) == 0) continue;
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = T::mfma(*reinterpret_cast<const vec8*>(k_s + t * 32 * 256 + k_row_off + (((2 * d + hl) ^ k_sw) << 4)),
                       qf[d], s[t]);
    if (masked) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * t + 8 * (r >> 2) + 4 * hl + (r & 3) >= lim) s[t][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[t][r]);
    const float m_new = fmaxf(m_run, pair_max(mx) * cl2);
    if (__builtin_amdgcn_ballot_w64(m_new > m_run + kRescaleLog2) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[u][r] *= alpha;
    }
    vec8 pf[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(s[t][r] * cl2 - m_run);
        l_run += p;
        pf[t][r >> 3][r & 7] = (scalar)p;
      }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const char* lo = v_s + (32 * t + 16 * hh) * 256 + v_lane_off + (((4 * u + v_c0) ^ v_sw) << 4);
          vec8 vf = T::transposed(lo, lo + 8 * 256);
          if (masked) {
            // A value that some row does not see may be infinite or NaN, and 0 times it is NaN.  Such values are
            // left out of the product, and what they do to the rows that do see them follows from a product
            // with their places: a row with a weight on one gets its infinity or NaN.
            i32x4 w = __builtin_bit_cast(i32x4, vf);
            uint32_t odd = 0, at[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              at[e] = (((uint32_t)w[e] & T::kExp) + T::kLow) & 0x80008000u;
              odd |= at[e];
            }
            if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) {
              i32x4 kind[3];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t full = (at[e] >> 15) * 0xffffu, word = (uint32_t)w[e];
                uint32_t is_nan = 0, is_neg = 0;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  const uint32_t x16 = (word >> (16 * half)) & 0xffffu;
                  if ((x16 & 0x7fffu) > (T::kExp & 0x7fffu)) is_nan |= 0xffffu << (16 * half);
                  if (x16 & 0x8000u) is_neg |= 0xffffu << (16 * half);
                }
                const uint32_t ones = T::kOne * 0x10001u;
                kind[0][e] = (int)(ones & full & ~is_nan & ~is_neg);
                kind[1][e] = (int)(ones & full & ~is_nan & is_neg);
                kind[2][e] = (int)(ones & full & is_nan);
                w[e] = (int)(word & ~full);
              }
              vf = __builtin_bit_cast(vec8, w);
#pragma unroll
              for (int c = 0; c < 3; ++c) {
                const float what = c == 0 ? INFINITY : c == 1 ? -INFINITY : __builtin_nanf("");
                f32x16 hit;
#pragma unroll
                for (int r = 0; r < 16; ++r) hit[r] = 0.f;
                hit = T::mfma(__builtin_bit_cast(vec8, kind[c]), pf[t][hh], hit);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                  if (hit[r] > 0.f) o[u][r] += what;
              }
            }
          }
          o[u] = T::mfma(vf, pf[t][hh], o[u]);
        }
  }

  const float l_tot = pair_sum(l_run);
  if (!valid) return;
  if (it.slot >= 0) {
    const int64_t at = ((int64_t)it.slot * a.Hk + hk) * (32 * NW) + wave * 32 + l32;
    float* po = a.part_o + at * kHeadDim;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        *reinterpret_cast<float4*>(po + 32 * u + 8 * rr + 4 * hl) =
            make_float4(o[u][4 * rr], o[u][4 * rr + 1], o[u][4 * rr + 2], o[u][4 * rr + 3]);
    if (hl == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m_run, l_tot);
    return;
  }
  const bool empty = l_tot == 0.f;   // NaN is not
  const float inv_l = empty ? 0.f : 1.f / l_tot;
  uint16_t* op = static_cast<uint16_t*>(const_cast<void*>(a.o.data)) + (int64_t)(it.q0 + query) * a.o.ss + (int64_t)qh * a.o.sh;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      scalar v4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v4[e] = (scalar)(o[u][4 * rr + e] * inv_l);
      uint2 packed;
      __builtin_memcpy(&packed, v4, 8);
      *reinterpret_cast<uint2*>(op + 32 * u + 8 * rr + 4 * hl) = packed;
    }
  if (a.lse && hl == 0)
    a.lse[(int64_t)qh * a.total_q + it.q0 + query] = empty ? -INFINITY : (m_run + __builtin_log2f(l_tot)) * kLn2;
}

// Joins a tile's pieces: with m the largest of their maxima, O = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i.
// 32 lanes per row.
template <bool BF16, int NW>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
  using scalar = typename Type<BF16>::scalar;
  const int* header = a.plan.header;
  if (header[kPlanKey] != a.key || (int)blockIdx.x >= header[kPlanJoins]) return;
  const PackedJoin jn = a.plan.joins[blockIdx.x];
  const int hk = blockIdx.y, lane = threadIdx.x & 31;
  const int np = header[kPlanPrefixPieces], n = jn.pieces + np;
  constexpr int kTile = 32 * NW;
  for (int r = threadIdx.x >> 5; r < kTile && jn.row0 + r < jn.rows; r += 8) {
    const int row = jn.row0 + r;
    const int pooled = jn.q0 * a.group - header[kPlanFirstRow] + row;   // among the rows of all sequences
    auto at = [&](int i) {
      const int64_t slot = i < jn.pieces ? jn.slot + i : pooled / kTile * np + (i - jn.pieces);
      return (slot * a.Hk + hk) * kTile + (i < jn.pieces ? r : pooled % kTile);
    };
    float m = -FLT_MAX;
    for (int i = 0; i < n; ++i) m = fmaxf(m, a.part_ml[2 * at(i)]);
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < n; ++i) {
      const int64_t p = at(i);
      const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * p] - m);
      const float4 v = *reinterpret_cast<const float4*>(a.part_o + p * kHeadDim + 4 * lane);
      l += f * a.part_ml[2 * p + 1];
      o.x += f * v.x;
      o.y += f * v.y;
      o.z += f * v.z;
      o.w += f * v.w;
    }
    const bool empty = l == 0.f;
    const float inv_l = empty ? 0.f : 1.f / l;
    const int query = jn.q0 + row / a.group, qh = hk * a.group + row % a.group;
    const scalar v4[4] = {(scalar)(o.x * inv_l), (scalar)(o.y * inv_l), (scalar)(o.z * inv_l), (scalar)(o.w * inv_l)};
    uint2 packed;
    __builtin_memcpy(&packed, v4, 8);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(const_cast<void*>(a.o.data)) + (int64_t)query * a.o.ss +
                              (int64_t)qh * a.o.sh + 4 * lane) = packed;
    if (a.lse && lane == 0)
      a.lse[(int64_t)qh * a.total_q + query] = empty ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
  }
}

template <bool BF16, int NW>
void launch_packed(const PackedConfig& c, const PackedArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((packed_attn_kernel<BF16, NW>), dim3((unsigned)packed_grid(a.Hk, c.max_items)), dim3(64 * NW), 0, st,
                     a);
  hipLaunchKernelGGL((packed_join_kernel<BF16, NW>), dim3(c.max_joins, a.Hk), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_packed_attn(chorus_dtype dt, const PackedConfig& c, const PackedArgs& a, hipStream_t st) {
  if (dt == CHORUS_BF16)
    launch_packed<true, 4>(c, a, st);
  else
    launch_packed<false, 4>(c, a, st);
  return hipGetLastError();
}

}  // namespace chorus
