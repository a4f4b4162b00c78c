// Norms of the queries and keys of each head and their rotation in one pass.
//
// HBM-bound streaming: every value is read and written once; the norm needs a
// head's sum of squares before its first output, so a head is held in registers.
// A lane owns one unit of 8 channels of a head: of the rotating channels, the 4
// pairs 4u .. 4u + 3 (half pairing: channels 4u .. and rot/2 + 4u ..; interleaved:
// channels 8u .. 8u + 7), so both members of every pair meet in one lane and both
// pairings read the same 4 cosines and sines; of the others, 8 channels in a row.
// The LPH lanes of a head (8, 16 or 32, for head sizes up to 64, 128 and 256) sum
// their squares across lanes.  A wave takes one token, up to U groups of 64 / LPH
// heads of it: table row and weights are read once for all of them, and all of the
// groups' loads are in flight together.
#include "kvb_device.h"
#include "kvb_internal.h"

namespace kvb {
namespace {

// x from the lane chosen by DPP control CTRL
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}

// sum over LPH adjacent lanes; all of them end with the total
template <int LPH>
__device__ __forceinline__ float head_sum(float x) {
  x += dpp<0xB1>(x);                       // quad_perm [1,0,3,2]
  x += dpp<0x4E>(x);                       // quad_perm [2,3,0,1]
  x += dpp<0x141>(x);                      // the other quad of 8 lanes (mirrored)
  if constexpr (LPH >= 16) x += dpp<0x140>(x);  // the other half of 16 lanes (mirrored)
  if constexpr (LPH >= 32) x += __shfl_xor(x, 16, 64);
  return x;
}

// 4 consecutive values as floats
__device__ __forceinline__ void load4(const float* p, float* x) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
}
__device__ __forceinline__ void load4(const uint16_t* p, float* x) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
}
__device__ __forceinline__ void store4(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store4(uint16_t* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}

template <typename T, int LPH, int U>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkNormRope a) {
  constexpr int HPW = 64 / LPH;  // heads of a group
  const int lane = threadIdx.x & 63, u = lane % LPH;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = wave / a.chunks;
  const int g0 = (int)(wave % a.chunks) * U * HPW + lane / LPH;  // first head of this lane
  if (t >= a.n_tokens) return;
  const int heads = a.n_q_heads + a.n_kv_heads;
  const bool in = u * 8 < a.head_dim, turns = u * 8 < a.rot_dim;
  // where the unit's two runs of 4 channels start
  const bool split = turns && a.pairing == KVB_PAIR_HALF;
  const int c0 = split ? 4 * u : 8 * u, c1 = split ? a.rot_dim / 2 + 4 * u : 8 * u + 4;
  float x[U][8];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int h = g0 + k * HPW;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[k][e] = 0.f;
    if (in && h < heads) {
      const T* p = h < a.n_q_heads
                       ? (const T*)a.q + t * a.q_token_stride + h * a.q_head_stride
                       : (const T*)a.k + t * a.k_token_stride + (h - a.n_q_heads) * a.k_head_stride;
      load4(p + c0, x[k]);
      load4(p + c1, x[k] + 4);
    }
  }
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  bool bad = false;
  if (a.rot_dim > 0) {
    const int pos = a.pos[t];
    bad = pos < 0 || pos >= a.table_len;
    if (turns && !bad) {
      load4(a.table_cos + (int64_t)pos * (a.rot_dim / 2) + 4 * u, c);
      load4(a.table_sin + (int64_t)pos * (a.rot_dim / 2) + 4 * u, s);
    }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (in && a.q_weight) load4(a.q_weight + c0, wq), load4(a.q_weight + c1, wq + 4);
  if (in && a.k_weight) load4(a.k_weight + c0, wk), load4(a.k_weight + c1, wk + 4);
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int h = g0 + k * HPW;
    const bool is_q = h < a.n_q_heads;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[k][e], x[k][e], sum);
    sum = head_sum<LPH>(sum);
    if (!in || h >= heads) continue;
    const bool norm = is_q ? a.q_weight != nullptr : a.k_weight != nullptr;
    const float r = norm ? 1.f / sqrtf(sum / (float)a.head_dim + a.eps) : 1.f;
    float y[8], z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = norm ? x[k][e] * r * (is_q ? wq[e] : wk[e]) : x[k][e];
    if (a.pairing == KVB_PAIR_HALF) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i] = __builtin_fmaf(y[i], c[i], -(y[4 + i] * s[i]));
        z[4 + i] = __builtin_fmaf(y[4 + i], c[i], y[i] * s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[2 * i] = __builtin_fmaf(y[2 * i], c[i], -(y[2 * i + 1] * s[i]));
        z[2 * i + 1] = __builtin_fmaf(y[2 * i + 1], c[i], y[2 * i] * s[i]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = bad ? __builtin_nanf("") : turns ? z[e] : y[e];
    T* p = is_q ? (T*)a.q_out + t * a.q_out_token_stride + h * a.q_out_head_stride
                : (T*)a.k_out + t * a.k_out_token_stride + (h - a.n_q_heads) * a.k_out_head_stride;
    store4(p + c0, z);
    store4(p + c1, z + 4);
  }
}

template <typename T, int LPH>
void launch(QkNormRope a, hipStream_t s) {
  constexpr int HPW = 64 / LPH, U = 4;
  const int groups = (a.n_q_heads + a.n_kv_heads + HPW - 1) / HPW;
  a.chunks = (groups + U - 1) / U;
  const int64_t waves = a.n_tokens * a.chunks;
  hipLaunchKernelGGL((qk_norm_rope_kernel<T, LPH, U>), dim3((unsigned)((waves + 3) / 4)), dim3(256),
                     0, s, a);
}

}  // namespace

hipError_t launch_qk_norm_rope(const QkNormRope& a, kvb_dtype dtype, hipStream_t s) {
  if (dtype == KVB_BF16) {
    if (a.head_dim <= 64) launch<uint16_t, 8>(a, s);
    else if (a.head_dim <= 128) launch<uint16_t, 16>(a, s);
    else launch<uint16_t, 32>(a, s);
  } else {
    if (a.head_dim <= 64) launch<float, 8>(a, s);
    else if (a.head_dim <= 128) launch<float, 16>(a, s);
    else launch<float, 32>(a, s);
  }
  return hipGetLastError();
}

}  // namespace kvb
