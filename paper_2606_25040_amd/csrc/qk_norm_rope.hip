// Norm and rotation of Q and K in one pass: what a layer does to the projected queries and keys before a mask is
// built from them or attention reads them.
//
// For each token and tensor x [H, 128], in fp32:
//   y = x * rsqrt(mean(x^2) + eps) * w   mean over the head (w [128]) or over the token's H heads (w [H, 128]), or y = x;
//   pair p = 0 .. 63 of a head, the elements (2p, 2p + 1) or (p, p + 64), turned by the angle
//   positions[axis(p)] * freqs[p]: (a, b) -> (a cos - b sin, a sin + b cos);
// and rounded once to x's type.  Angles are taken in float64 and reduced to a part of a turn before the fp32
// sine and cosine: in fp32 the angle of position 100,000 would be off by 0.004 rad already.
//
// A lane holds 16 elements of one head, the 16-byte chunks c and c + 8 (c = lane % 8), which hold both elements
// of the lane's pairs in either layout; a head is 8 lanes.  One workgroup per token and tensor (and 128 heads).
#include "chorus_internal.h"

namespace chorus {
namespace {

constexpr int kPairs = kHeadDim / 2;
constexpr double kTurnsPerRadian = 0.15915494309189533577;

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

template <bool BF16>
__global__ __launch_bounds__(1024) void qk_norm_rope_kernel(RopeArgs a) {
  __shared__ float cs[2][kPairs];
  __shared__ float sums[1024 / 64];
  const int tensor = blockIdx.y;
  const int H = tensor ? a.Hk : a.Hq;
  const int64_t token = blockIdx.x;
  const int b = (int)(token / a.S), s = (int)(token % a.S);
  const int tid = threadIdx.x, c = tid & 7, h = blockIdx.z * kMaxTokenHeads + (tid >> 3);
  if (a.n_axes > 0 && tid < kPairs) {
    int axis = 0;
    for (int p = tid; axis < a.n_axes - 1 && p >= a.pairs[axis]; ++axis) p -= a.pairs[axis];
    const int32_t pos = a.positions[axis * a.pos_axis + b * a.pos_b + s];
    const double turns = pos * a.freqs[tid] * kTurnsPerRadian;
    float sn, co;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &co);
    cs[0][tid] = co;
    cs[1][tid] = sn;
  }
  const TensorArg& in = tensor ? a.k : a.q;
  const TensorArg& out = tensor ? a.k_out : a.q_out;
  const float* w = tensor ? a.k_weight : a.q_weight;
  float x[16];
  if (h < H) {
    const char* row = static_cast<const char*>(in.data) + 2 * (b * in.sb + s * in.ss + h * in.sh) + 16 * c;
    uint32_t r[8];
    *reinterpret_cast<uint4*>(r) = *reinterpret_cast<const uint4*>(row);
    *reinterpret_cast<uint4*>(r + 4) = *reinterpret_cast<const uint4*>(row + 128);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = Pack<BF16>::lo(r[i]);
      x[2 * i + 1] = Pack<BF16>::hi(r[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  }
  float total = 0.f;
  if (a.norm != CHORUS_NORM_NONE) {
#pragma unroll
    for (int i = 0; i < 16; ++i) total += x[i] * x[i];
    total = head_sum(total);
    if (a.norm == CHORUS_NORM_TOKEN) {
#pragma unroll
      for (int d = 8; d < 64; d *= 2) total += __shfl_xor(total, d);
      if ((tid & 63) == 0) sums[tid >> 6] = total;
    }
  }
  __syncthreads();
  if (a.norm != CHORUS_NORM_NONE) {
    int64_t n = kHeadDim;
    const float* wh = w + 8 * c;
    if (a.norm == CHORUS_NORM_TOKEN) {
      total = 0.f;
      for (int i = 0; i < (int)(blockDim.x >> 6); ++i) total += sums[i];
      n *= H;
      wh += (int64_t)h * kHeadDim;
    }
    const float f = rsqrtf(total / (float)n + a.eps);
    if (h < H) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= f * wh[(i & 7) + 64 * (i >> 3)];
    }
  }
  if (h >= H) return;
  float y[16];
  if (a.n_axes == 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
  } else if (a.adjacent) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = 4 * c + (i & 3) + 32 * (i >> 2);
      y[2 * i] = x[2 * i] * cs[0][p] - x[2 * i + 1] * cs[1][p];
      y[2 * i + 1] = x[2 * i] * cs[1][p] + x[2 * i + 1] * cs[0][p];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = 8 * c + i;
      y[i] = x[i] * cs[0][p] - x[i + 8] * cs[1][p];
      y[i + 8] = x[i] * cs[1][p] + x[i + 8] * cs[0][p];
    }
  }
  uint32_t r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = Pack<BF16>::join(y[2 * i], y[2 * i + 1]);
  char* row = static_cast<char*>(const_cast<void*>(out.data)) + 2 * (b * out.sb + s * out.ss + h * out.sh) + 16 * c;
  *reinterpret_cast<uint4*>(row) = *reinterpret_cast<uint4*>(r);
  *reinterpret_cast<uint4*>(row + 128) = *reinterpret_cast<uint4*>(r + 4);
}

}  // namespace

hipError_t launch_qk_norm_rope(chorus_dtype dt, const RopeArgs& a, hipStream_t st) {
  const int H = a.Hk > a.Hq ? a.Hk : a.Hq;
  const int groups = (H + kMaxTokenHeads - 1) / kMaxTokenHeads;   // one for a norm over the token
  const dim3 grid((unsigned)((int64_t)a.B * a.S), a.Hk > 0 ? 2 : 1, groups);
  const dim3 block(64 * (((H < kMaxTokenHeads ? H : kMaxTokenHeads) + 7) / 8));
  if (dt == CHORUS_BF16)
    hipLaunchKernelGGL((qk_norm_rope_kernel<true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace chorus
