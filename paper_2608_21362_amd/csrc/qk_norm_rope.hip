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

constexpr int kGroups = 4;  // head groups of a wave where there are many waves

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

// 4 consecutive values, as they are held, and as floats
template <typename T>
struct Four;
template <>
struct Four<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float* x) const { x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w; }
};
template <>
struct Four<uint16_t> {
  uint2 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
  }
};
__device__ __forceinline__ void load4(const float* p, float* x) {
  Four<float> f;
  f.load(p);
  f.get(x);
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
  // what the wave takes, on the scalar unit: a token, and groups of either queries or keys
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const uint32_t chunks = a.q_chunks + a.k_chunks;
  const int64_t t = wave / chunks;
  if (t >= a.n_tokens) return;
  const int chunk = (int)(wave - (uint32_t)t * chunks);
  const bool is_q = chunk < a.q_chunks;
  const int h0 = (is_q ? chunk : chunk - a.q_chunks) * U * HPW, heads = is_q ? a.n_q_heads : a.n_kv_heads;
  const T* from = is_q ? (const T*)a.q + t * a.q_token_stride : (const T*)a.k + t * a.k_token_stride;
  T* to = is_q ? (T*)a.q_out + t * a.q_out_token_stride : (T*)a.k_out + t * a.k_out_token_stride;
  const int64_t from_head = is_q ? a.q_head_stride : a.k_head_stride;
  const int64_t to_head = is_q ? a.q_out_head_stride : a.k_out_head_stride;
  const float* weight = is_q ? a.q_weight : a.k_weight;
  const bool in = u * 8 < a.head_dim, turns = u * 8 < a.rot_dim;
  // where the unit's two runs of 4 channels start
  const bool split = turns && a.pairing == KVB_PAIR_HALF;
  const int c0 = split ? 4 * u : 8 * u, c1 = split ? a.rot_dim / 2 + 4 * u : 8 * u + 4;
  Four<T> x[U][2];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int h = h0 + k * HPW + lane / LPH;
    x[k][0] = x[k][1] = Four<T>{};
    if (in && h < heads) {
      x[k][0].load(from + h * from_head + c0);
      x[k][1].load(from + h * from_head + c1);
    }
  }
  float w[8], c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  if (weight != nullptr && in) load4(weight + c0, w), load4(weight + c1, w + 4);
  bool bad = false;
  if (a.rot_dim > 0) {
    const int pos = a.pos[t];
    bad = pos < 0 || pos >= a.table_len;
    if (turns && !bad) {
      load4(a.table_cos + (int64_t)pos * (a.rot_dim / 2) + 4 * u, c);
      load4(a.table_sin + (int64_t)pos * (a.rot_dim / 2) + 4 * u, s);
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int h = h0 + k * HPW + lane / LPH;
    float y[8], z[8];
    x[k][0].get(y);
    x[k][1].get(y + 4);
    if (weight != nullptr) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
      sum = head_sum<LPH>(sum);
      const float r = 1.f / sqrtf(sum / (float)a.head_dim + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * r * w[e];
    }
    if (!in || h >= heads) continue;
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
    store4(to + h * to_head + c0, z);
    store4(to + h * to_head + c1, z + 4);
  }
}

template <typename T, int LPH>
void launch(QkNormRope a, hipStream_t s) {
  constexpr int HPW = 64 / LPH;
  const int gq = (a.n_q_heads + HPW - 1) / HPW, gk = (a.n_kv_heads + HPW - 1) / HPW;
  // One group a wave where the tensors fit the caches, so that a call's loads spread over the card;
  // more where HBM bounds them, so that each wave has more loads in flight (16 + 2 heads of 128: 8000
  // tokens 18.2 us with 1 and 19.4 with 4, 12000 30.2 and 29.6, 32772 72.3 and 65.8).
  const int u = a.n_tokens * (gq + gk) <= 49152 ? 1 : kGroups;
  a.q_chunks = (gq + u - 1) / u;
  a.k_chunks = (gk + u - 1) / u;
  const int64_t waves = a.n_tokens * (a.q_chunks + a.k_chunks);
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (u == 1) hipLaunchKernelGGL((qk_norm_rope_kernel<T, LPH, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<T, LPH, kGroups>), grid, dim3(256), 0, s, a);
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
