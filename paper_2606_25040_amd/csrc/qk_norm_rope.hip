// Norm and rotation of Q and K in one pass: what a layer does to the projected queries and keys before a mask is
// built from them or attention reads them.
//
// For each token and tensor x [H, 128], in fp32:
//   y = x * rsqrt(mean(x^2) + eps) * w   mean over the head (w [128]) or over the token's H heads (w [H, 128]), or y = x;
//   pair p = 0 .. 63 of a head, the elements (2p, 2p + 1) or (p, p + 64), turned by the angle
//   positions[axis(p)] * freqs[p]: (a, b) -> (a cos - b sin, a sin + b cos);
// and rounded once to x's type (bf16 values whose squares leave the fp32 range are scaled first).  Angles are taken in float64 and reduced to a part of a turn before the fp32
// sine and cosine: in fp32 the angle of position 100,000 would be off by 0.004 rad already.
//
// A lane holds 16 elements of one head, the 16-byte chunks c and c + 8 (c = lane % 8), which hold both elements
// of the lane's pairs in either layout; a head is 8 lanes.  A workgroup holds one token's heads (up to 128) of one
// tensor at a time, its weights in registers.
//
// Memory-bound: at 480p 14B (32,760 tokens x 40 + 40 heads, bf16, norm over the token) 249-266 us, 5.0-5.4 TB/s; at
// 720p 5B (27,280 x 24 + 24, norm per head) 114-123 us, 5.4-5.9 TB/s, the rate of a plain copy.
#include <cfloat>

#include "chorus_internal.h"

namespace chorus {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int kPairs = kHeadDim / 2;
constexpr double kTurnsPerRadian = 0.15915494309189533577;
// bf16 values reach 2^128 and 2^-133, so their squares leave the fp32 range.  A token or head whose sum of squares
// overflows is taken times kDown, and one whose sum is so small that squares may have vanished times kUp, and with it
// eps by the square: any 128 x 128 values then sum to less than 2^126, and the largest square is above 2^-106.  (With
// eps >= kSmall a mean below it does not count beside eps.)
constexpr float kDown = 0x1p-72f, kUp = 0x1p+80f, kSmall = 0x1p-100f;

template <bool BF16>
struct Pack;
template <>
struct Pack<true> {
  static __device__ inline float lo(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ inline float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
  static __device__ inline uint32_t join(float a, float b) {
    const __bf16 v[2] = {(__bf16)a, (__bf16)b};
    uint32_t w;
    __builtin_memcpy(&w, v, 4);
    return w;
  }
};
template <>
struct Pack<false> {
  static __device__ inline float at(uint32_t w, int i) {
    _Float16 v[2];
    __builtin_memcpy(v, &w, 4);
    return (float)v[i];
  }
  static __device__ inline float lo(uint32_t w) { return at(w, 0); }
  static __device__ inline float hi(uint32_t w) { return at(w, 1); }
  static __device__ inline uint32_t join(float a, float b) {
    const _Float16 v[2] = {(_Float16)a, (_Float16)b};
    uint32_t w;
    __builtin_memcpy(&w, v, 4);
    return w;
  }
};

// Sum over the 8 lanes of a head.
__device__ inline float head_sum(float v) {
#pragma unroll
  for (int d = 1; d < 8; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// NORM and the pair layout are template arguments so that each loop carries only its own work.
template <bool BF16, int NORM, int PAIRS>   // PAIRS: 0 no rotation, 1 adjacent, 2 half-split
__global__ __launch_bounds__(1024) void qk_norm_rope_kernel(RopeArgs a) {
  __shared__ float cs[2][2][kPairs];        // [parity][cos, sin][pair]
  __shared__ float sums[2][kMaxTokenHeads / 8];
  const int tensor = blockIdx.y;
  const int H = tensor ? a.Hk : a.Hq;
  const int tid = threadIdx.x, c = tid & 7, h = blockIdx.z * kMaxTokenHeads + (tid >> 3);
  const bool live = h < H;
  const TensorArg& in = tensor ? a.k : a.q;
  const TensorArg& out = tensor ? a.k_out : a.q_out;
  const int tokens = a.B * a.S, step = gridDim.x;

  float w[16];
  if (NORM != CHORUS_NORM_NONE && live) {
    const float* wp = (tensor ? a.k_weight : a.q_weight) + 8 * c + (NORM == CHORUS_NORM_TOKEN ? (int64_t)h * kHeadDim : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(w + 4 * i) = *reinterpret_cast<const float4*>(wp + 4 * (i & 1) + 64 * (i >> 1));
  }
  int axis = 0;
  double turns_per_position = 0.0;
  if (PAIRS && tid < kPairs) {
    for (int p = tid; axis < a.n_axes - 1 && p >= a.pairs[axis]; ++axis) p -= a.pairs[axis];
    turns_per_position = a.freqs[tid] * kTurnsPerRadian;
  }
  auto load = [&](int t, uint32_t (&r)[8], int32_t& pos) {
    const int b = t / a.S, s = t % a.S;
    if (live) {
      const char* row = static_cast<const char*>(in.data) + 2 * (b * in.sb + s * in.ss + h * in.sh) + 16 * c;
      *reinterpret_cast<u32x4*>(r) = *reinterpret_cast<const u32x4*>(row);
      *reinterpret_cast<u32x4*>(r + 4) = *reinterpret_cast<const u32x4*>(row + 128);
    }
    if (PAIRS && tid < kPairs) pos = a.positions[axis * a.pos_axis + b * a.pos_b + s];
  };
  uint32_t r[8] = {}, ahead[8] = {};
  int32_t pos = 0, pos_ahead = 0;
  load(blockIdx.x, r, pos);
  for (int t = blockIdx.x, par = 0; t < tokens; t += step, par ^= 1) {
    if (t + step < tokens) load(t + step, ahead, pos_ahead);
    if (PAIRS && tid < kPairs) {
      const double turns = pos * turns_per_position;
      sincospif(2.f * (float)(turns - rint(turns)), &cs[par][1][tid], &cs[par][0][tid]);
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = Pack<BF16>::lo(r[i]);
      x[2 * i + 1] = Pack<BF16>::hi(r[i]);
    }
    auto squares = [&] {   // of the head, or of the wave's heads and for all waves to add
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
      sum = head_sum(sum);
      if (NORM == CHORUS_NORM_TOKEN) {
#pragma unroll
        for (int d = 8; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if ((tid & 63) == 0) sums[par][tid >> 6] = sum;
      }
      return sum;
    };
    auto of_all_waves = [&] {
      float sum = 0.f;
      for (int i = 0; i < (int)(blockDim.x >> 6); ++i) sum += sums[par][i];
      return sum;
    };
    float total = 0.f;
    if (NORM != CHORUS_NORM_NONE) total = squares();
    // the other parity's values are read before the next barrier, so one per token is enough
    if (PAIRS || NORM == CHORUS_NORM_TOKEN) __syncthreads();
    if (NORM != CHORUS_NORM_NONE) {
      float n = kHeadDim, eps = a.eps;
      if (NORM == CHORUS_NORM_TOKEN) {
        total = of_all_waves();
        n *= H;
      }
      // the same for all lanes of a head, or of the workgroup
      if (BF16 && (!(total <= FLT_MAX) || (total < kSmall && eps < kSmall))) {
        const float scale = total <= FLT_MAX ? kUp : kDown;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= scale;
        eps = eps * scale * scale;
        if (NORM == CHORUS_NORM_TOKEN) __syncthreads();   // the sums are read before they are written again
        total = squares();
        if (NORM == CHORUS_NORM_TOKEN) {
          __syncthreads();
          total = of_all_waves();
        }
      }
      const float f = rsqrtf(total / n + eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= f * w[i];
    }
    if (live) {
      uint32_t y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (PAIRS == 0) {
          y[i] = Pack<BF16>::join(x[2 * i], x[2 * i + 1]);
        } else if (PAIRS == 1) {
          const int p = 4 * c + (i & 3) + 32 * (i >> 2);
          const float co = cs[par][0][p], sn = cs[par][1][p];
          y[i] = Pack<BF16>::join(x[2 * i] * co - x[2 * i + 1] * sn, x[2 * i] * sn + x[2 * i + 1] * co);
        }
      }
      if (PAIRS == 2) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float lo[2], hi[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float co = cs[par][0][8 * c + i + e], sn = cs[par][1][8 * c + i + e];
            lo[e] = x[i + e] * co - x[i + e + 8] * sn;
            hi[e] = x[i + e] * sn + x[i + e + 8] * co;
          }
          y[i / 2] = Pack<BF16>::join(lo[0], lo[1]);
          y[i / 2 + 4] = Pack<BF16>::join(hi[0], hi[1]);
        }
      }
      const int b = t / a.S, s = t % a.S;
      char* row = static_cast<char*>(const_cast<void*>(out.data)) + 2 * (b * out.sb + s * out.ss + h * out.sh) + 16 * c;
      const u32x4 lo = *reinterpret_cast<u32x4*>(y), hi = *reinterpret_cast<u32x4*>(y + 4);
      if (a.streamed) {
        __builtin_nontemporal_store(lo, reinterpret_cast<u32x4*>(row));
        __builtin_nontemporal_store(hi, reinterpret_cast<u32x4*>(row + 128));
      } else {
        *reinterpret_cast<u32x4*>(row) = lo;
        *reinterpret_cast<u32x4*>(row + 128) = hi;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = ahead[i];
    pos = pos_ahead;
  }
}

template <bool BF16, int NORM>
void launch_rope(const RopeArgs& a, dim3 grid, dim3 block, hipStream_t st) {
  if (a.n_axes == 0)
    hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, NORM, 0>), grid, block, 0, st, a);
  else if (a.adjacent)
    hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, NORM, 1>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<BF16, NORM, 2>), grid, block, 0, st, a);
}

template <bool BF16>
void launch_rope(const RopeArgs& a, dim3 grid, dim3 block, hipStream_t st) {
  if (a.norm == CHORUS_NORM_NONE)
    launch_rope<BF16, CHORUS_NORM_NONE>(a, grid, block, st);
  else if (a.norm == CHORUS_NORM_HEAD)
    launch_rope<BF16, CHORUS_NORM_HEAD>(a, grid, block, st);
  else
    launch_rope<BF16, CHORUS_NORM_TOKEN>(a, grid, block, st);
}

}  // namespace

// Waves per CU in a launch, 32 at a time: a workgroup of a long call takes several tokens with one read of its weights
// and with the next token's loads in flight.  480p 14B (norm over the token): 259 us, one token each 313-322 (weights),
// 16 or 32 waves 266-272 (the uneven end); 720p 5B (norm per head) 115-122 with any count from 128 up.
constexpr int64_t kWavesPerCu = 256;
// Outputs beyond this many bytes are stored past the 256 MB cache behind the L2s, which the inputs still to be read
// need: 480p 14B (671 MB) 259 -> 249 us, with a mask built from the outputs 525 -> 498; 720p 5B (335 MB) 122 -> 114 and
// 265 -> 254.  Smaller ones are found there by whoever reads them (84 MB: with the mask 67.5 us, streamed 71).
constexpr int64_t kStreamedBytes = 256 << 20;

hipError_t launch_qk_norm_rope(chorus_dtype dt, RopeArgs a, hipStream_t st) {
  const int H = a.Hk > a.Hq ? a.Hk : a.Hq, tensors = a.Hk > 0 ? 2 : 1;
  const int groups = (H + kMaxTokenHeads - 1) / kMaxTokenHeads;   // one for a norm over the token
  const int waves = ((H < kMaxTokenHeads ? H : kMaxTokenHeads) + 7) / 8;
  const int64_t tokens = (int64_t)a.B * a.S;
  const int64_t full = kWavesPerCu * 256 / (waves * tensors * groups) + 1;
  a.streamed = tokens * (a.Hq + a.Hk) * kHeadDim * 2 > kStreamedBytes;
  const dim3 grid((unsigned)(tokens < full ? tokens : full), tensors, groups), block(64 * waves);
  if (dt == CHORUS_BF16)
    launch_rope<true>(a, grid, block, st);
  else
    launch_rope<false>(a, grid, block, st);
  return hipGetLastError();
}

}  // namespace chorus
