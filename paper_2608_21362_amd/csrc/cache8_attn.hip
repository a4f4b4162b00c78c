// Attention of the last tokens of each sequence over the 8-bit cache.
//
// The G query heads of a kv head and the call's queries of a sequence are its rows
// (row = query * G + head); a tile is 16 * NT rows.  Keys come in steps of 64.  A wave
// computes S^T (64 keys x rows) = K Q^T and O^T (d x rows) += V^T P^T with 16x16x32
// matrix instructions, codes and probabilities as fp16 (8-bit codes are exact there),
// straight from global memory: the contraction index of a product may be permuted if
// both operands agree, so a lane takes 16 consecutive bytes of K (channels) and of the
// channel-major V (keys), and the rows of K are dealt to the four 16-key tiles such that
// the scores a lane holds (keys 16 g .. 16 g + 15, g = lane / 16) are the keys of its V
// operand.  No operand passes through LDS.
//
// Scales: a lane's 16 keys lie in one block (B >= 16), so the scale of K multiplies its
// scores, and that of V its probabilities, relative to the largest scale of the wave's
// chunk of blocks (2^7 at most, so that small blocks keep their bits in fp16).
//
// The waves of a workgroup take runs of steps of their own and meet in LDS; where a call
// has few tiles, several workgroups share a tile's keys and a second launch joins them.
#include <math.h>

#include "kvb_device.h"
#include "kvb_internal.h"

namespace kvb {
namespace {

typedef __attribute__((ext_vector_type(2))) _Float16 half2_t;
typedef __attribute__((ext_vector_type(8))) _Float16 half8_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf8_t;
typedef __attribute__((ext_vector_type(4))) float f4_t;
typedef __attribute__((ext_vector_type(2))) float f2_t;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -1e30f;  // running maximum before the first visible key
constexpr float kSlack = 8.f;     // the running maximum follows once it is off by 2^8
constexpr int kScaleTop = 6;      // weights of V scales stay below 2^(kScaleTop + 1)
constexpr int kWaves = 4;

// four codes -> four fp16 numbers
template <int CODE>
__device__ __forceinline__ void widen4(uint32_t w, half2_t& a, half2_t& b) {
  if constexpr (CODE == KVB_I8) {
    // byte u = code + 128 under the exponent of 1024: the number 1024 + u
    w ^= 0x80808080u;
    const half2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
    a = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    b = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
  } else {
    a = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
    b = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
  }
}
template <int CODE>
__device__ __forceinline__ half8_t widen8(uint32_t w0, uint32_t w1) {
  half2_t r[4];
  widen4<CODE>(w0, r[0], r[1]);
  widen4<CODE>(w1, r[2], r[3]);
  return __builtin_bit_cast(half8_t, r);
}

__device__ __forceinline__ float max4groups(float x) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float sum4groups(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// A sequence as the call sees it.
struct Seq {
  int64_t n_q;   // its queries
  int64_t q0;    // the first of them
  int64_t len;   // its tokens
  int64_t full;  // full blocks
  int64_t keys;  // tokens that can be seen
  bool ok;
};
__device__ __forceinline__ Seq seq_of(const Attn8& a, int b, int B) {
  Seq s;
  s.q0 = a.cu_q[b];
  s.n_q = a.cu_q[b + 1] - s.q0;
  s.ok = s.n_q > 0 && s.q0 >= 0 && s.q0 + s.n_q <= a.n_queries;
  s.len = max(a.c.lens[b], 0);
  s.full = s.len / B;
  s.keys = s.len;
  if (s.full > a.c.max_blocks) s.full = a.c.max_blocks, s.keys = s.full * B;
  return s;
}
// keys that the last row of the tile sees, and the 64-key steps over full blocks that holds
struct Tile {
  int64_t keys, steps;
};
__device__ __forceinline__ Tile tile_of(const Seq& s, int64_t row0, int n_rows, int G, int B) {
  int64_t last = (row0 + n_rows - 1) / G;
  if (last >= s.n_q) last = s.n_q - 1;
  Tile t;
  t.keys = s.len - s.n_q + last + 1;
  if (t.keys > s.keys) t.keys = s.keys;
  if (t.keys < 0) t.keys = 0;
  const int64_t coded = t.keys < s.full * B ? t.keys : s.full * B;
  t.steps = (coded + 63) / 64;
  return t;
}

template <int D, int B, int CODE, int NT, bool WEIGHTS>
__global__ void __launch_bounds__(64 * kWaves, NT == 1 ? 3 : 2)
attn8_kernel(Attn8 a, Attn8Plan plan, float* __restrict__ po, float* __restrict__ ml,
             float* __restrict__ parts) {
  constexpr int KS = D / 32;               // contraction steps of a score
  constexpr int CT = D / 16;               // channel tiles of the output
  constexpr int KP = D / 64;               // 16-byte pieces of a lane's key
  constexpr int PB = B < 64 ? B : 64;      // tokens of a part with a weight of its own
  constexpr int CHUNK = B < 64 ? B : 64;   // steps whose blocks' ids and scales a wave holds
  constexpr int LDO = D + 4;
  __shared__ __align__(16) float part_o[kWaves][16 * NT][LDO];
  __shared__ float part_ml[kWaves][16 * NT][2];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int grp = lane >> 4, col = lane & 15;
  const int z = blockIdx.z, split = blockIdx.x;
  const int b = z / a.c.n_kv_heads, h = z % a.c.n_kv_heads;
  const int G = a.n_q_heads / a.c.n_kv_heads;
  const Seq sq = seq_of(a, b, B);
  const int64_t row0 = (int64_t)blockIdx.y * (16 * NT);
  if (!sq.ok || row0 >= sq.n_q * G) return;
  const Tile tl = tile_of(sq, row0, 16 * NT, G, B);
  int64_t lo = (int64_t)split * plan.span;
  int64_t hi = split == plan.n_splits - 1 ? tl.steps : lo + plan.span;
  if (hi > tl.steps) hi = tl.steps;
  if (split > 0 && lo >= tl.steps) return;
  if (lo > hi) lo = hi;
  const int64_t wlo = lo + (hi - lo) * wave / kWaves, whi = lo + (hi - lo) * (wave + 1) / kWaves;

  // queries: a power of two brings each row's largest value into [0.5, 1), so that fp16 holds
  // a bfloat16 of the row exactly (below 2^-14 of the largest: to 2^-25 of it)
  half8_t q[NT][KS];
  float cq[NT];
  int64_t see[NT];  // keys the row sees
  const uint16_t* qrow[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t r = row0 + n * 16 + col;
    const bool ok = r < sq.n_q * G;
    const int64_t i = ok ? r / G : 0;
    qrow[n] = ok ? a.q + ((sq.q0 + i) * a.n_q_heads + h * G + r % G) * D : nullptr;
    see[n] = ok ? min(sq.len - sq.n_q + i + 1, sq.keys) : 0;
    uint4 w[KS];
    float big = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      w[k] = make_uint4(0, 0, 0, 0);
      if (ok)
        w[k] = *reinterpret_cast<const uint4*>(qrow[n] + 64 * (k / 2) + 16 * grp + 8 * (k % 2));
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) big = fmaxf(big, fmaxf(fabsf(bf16_lo(u[e])), fabsf(bf16_hi(u[e]))));
    }
    big = max4groups(big);
    const int e2 = big > 0.f && big < INFINITY ? __builtin_amdgcn_frexp_expf(big) : 0;
    cq[n] = __builtin_ldexpf(a.softmax_scale * kLog2e, e2);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        q[n][k][2 * e] = (_Float16)__builtin_ldexpf(bf16_lo(u[e]), -e2);
        q[n][k][2 * e + 1] = (_Float16)__builtin_ldexpf(bf16_hi(u[e]), -e2);
      }
    }
  }

  float m[NT], l[NT];
  f4_t o[NT][CT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n] = kNoMax, l[n] = 0.f;
#pragma unroll
    for (int c = 0; c < CT; ++c) o[n][c] = (f4_t){0.f, 0.f, 0.f, 0.f};
  }
  int vexp = -127;  // the outputs are held in units of 2^(vexp - kScaleTop)

  // scores (log2 units) -> probabilities of the step; the running maximum and sums follow
  auto soften = [&](int n, float (&s)[16]) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = max4groups(top);
    if (__any(top > m[n] + kSlack)) {
      const float next = top > m[n] + kSlack ? top : m[n];
      const float f = __builtin_amdgcn_exp2f(m[n] - next);
      l[n] *= f;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] *= f;
      m[n] = next;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - m[n]);
      sum += s[i];
    }
    l[n] += sum;
    return sum;
  };
  // log2 of the weight of this row's tokens among the part's (sum: this lane's 16 tokens)
  auto record = [&](int n, int64_t key, float sum) {
    if constexpr (PB >= 32) sum += __shfl_xor(sum, 16, 64);
    if constexpr (PB >= 64) sum += __shfl_xor(sum, 32, 64);
    const int64_t r = row0 + n * 16 + col, p = key / PB;
    if ((PB == 16 || (PB == 32 && (grp & 1) == 0) || grp == 0) && r < plan.rows && p < plan.n_parts)
      parts[((int64_t)z * plan.n_parts + p) * plan.rows + r] = m[n] + __builtin_amdgcn_logf(sum);
  };

  const int32_t* table = a.c.table + (int64_t)z * a.c.max_blocks;
  for (int64_t c0 = wlo; c0 < whi; c0 += CHUNK) {
    const int64_t c1 = c0 + CHUNK < whi ? c0 + CHUNK : whi;
    const int64_t blk0 = c0 * 64 / B;
    // lane i holds id and scales of block blk0 + i; -1: no block
    int id = -1;
    float ks = 0.f, vs = 0.f;
    if (blk0 + lane < sq.full) {
      id = table[blk0 + lane];
      if (id < 0 || id >= a.c.n_blocks) id = -1;
      if (id >= 0) ks = a.c.k_scale[id], vs = a.c.v_scale[id];
    }
    float big = vs;
    for (int x = 32; x > 0; x >>= 1) big = fmaxf(big, __shfl_xor(big, x, 64));
    if (big > 0.f) {
      const int e = max(__builtin_amdgcn_frexp_expf(big), -100);
      if (e > vexp) {
        const float f = __builtin_ldexpf(1.f, vexp - e);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < CT; ++c) o[n][c] *= f;
        vexp = e;
      }
    }
    const float vw = __builtin_ldexpf(vs, kScaleTop - vexp);

    for (int64_t st = c0; st < c1; ++st) {
      const int64_t key0 = st * 64;
      // the blocks of this lane's K row (keys 16 (col / 4) ..) and of its 16 keys (16 grp ..)
      const int kb = (int)((key0 + 16 * (col >> 2)) / B - blk0);
      const int gb = (int)((key0 + 16 * grp) / B - blk0);
      const int idk = __shfl(id, kb, 64), idg = __shfl(id, gb, 64);
      const float ksg = __shfl(ks, gb, 64), vwg = __shfl(vw, gb, 64);
      const bool have = idg >= 0;
      const uint8_t* kp = a.c.k_codes + (int64_t)max(idk, 0) * (B * D);
      const uint8_t* vp = a.c.v_codes + (int64_t)max(idg, 0) * (B * D);
      const int kr = (int)((key0 + 16 * (col >> 2)) % B) + (col & 3);
      const int vk = (int)((key0 + 16 * grp) % B);
      uint4 kw[4][KP], vr[CT];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int p = 0; p < KP; ++p)
          kw[t][p] = *reinterpret_cast<const uint4*>(kp + (kr + 4 * t) * D + p * 64 + grp * 16);
#pragma unroll
      for (int c = 0; c < CT; ++c)
        vr[c] = *reinterpret_cast<const uint4*>(vp + (c * 16 + col) * B + vk);
      if (!__all(have)) {  // keys past the last full block: no value of V may be a NaN
#pragma unroll
        for (int c = 0; c < CT; ++c)
          if (!have) vr[c] = make_uint4(0, 0, 0, 0);
      }
      float s[NT][16];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f4_t acc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = (f4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < KP; ++p) {
          const half8_t k0 = widen8<CODE>(kw[t][p].x, kw[t][p].y);
          const half8_t k1 = widen8<CODE>(kw[t][p].z, kw[t][p].w);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[n][2 * p], acc[n], 0, 0, 0);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[n][2 * p + 1], acc[n], 0, 0, 0);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[n][4 * t + i] = acc[n][i];
      }
      half8_t pr[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float f = ksg * cq[n];
        const int64_t left = see[n] - (key0 + 16 * grp);  // visible among the lane's 16 keys
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = have && i < left ? s[n][i] * f : -INFINITY;
        const float sum = soften(n, s[n]);
        if constexpr (WEIGHTS) record(n, key0 + 16 * grp, sum);
        const float vwl = left > 0 ? vwg : 0.f;  // a row that sees none of a NaN block stays clean
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          half2_t x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f2_t v = {s[n][8 * j + 2 * e] * vwl, s[n][8 * j + 2 * e + 1] * vwl};
            x[e] = __builtin_convertvector(v, half2_t);
          }
          pr[n][j] = __builtin_bit_cast(half8_t, x);
        }
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const half8_t v0 = widen8<CODE>(vr[c].x, vr[c].y), v1 = widen8<CODE>(vr[c].z, vr[c].w);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pr[n][0], o[n][c], 0, 0, 0);
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pr[n][1], o[n][c], 0, 0, 0);
        }
      }
    }
  }

  // The tail: bfloat16 rows, one step of 64 keys for each wave of the first split (a block
  // has at most two).  Probabilities enter as the sum of two bfloat16, relative to the same
  // unit; rows past the tail's end hold anything, so their values of V are cleared.
  const int64_t t0 = sq.full * B + (int64_t)(kWaves - 1 - wave) * 64;
  if (split == 0 && (kWaves - 1 - wave) * 64 < B && t0 < tl.keys) {
    const int rows = (int)min((int64_t)64, sq.len - t0);  // tail rows of this step
    if (vexp < kScaleTop) {  // a unit of 1 at least: the sums fit a float if the outputs do
      const float f = __builtin_ldexpf(1.f, vexp - kScaleTop);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < CT; ++c) o[n][c] *= f;
      vexp = kScaleTop;
    }
    const int r0 = (kWaves - 1 - wave) * 64;
    const uint16_t* kt = a.c.k_tail + (int64_t)z * B * D;
    const uint16_t* vt = a.c.v_tail + (int64_t)z * B * D;
    float s[NT][16];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f4_t acc[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = (f4_t){0.f, 0.f, 0.f, 0.f};
      const int u = 16 * (col >> 2) + 4 * t + (col & 3);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (u < rows) x = *reinterpret_cast<const uint4*>(kt + (r0 + u) * D + k * 32 + grp * 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint4 y = make_uint4(0, 0, 0, 0);
          if (qrow[n]) y = *reinterpret_cast<const uint4*>(qrow[n] + k * 32 + grp * 8);
          acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, x),
                                                           __builtin_bit_cast(bf8_t, y), acc[n], 0, 0, 0);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][4 * t + i] = acc[n][i];
    }
    bf8_t ph[NT][2], pl[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float f = a.softmax_scale * kLog2e;
      const int64_t left = see[n] - (t0 + 16 * grp);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = i < left ? s[n][i] * f : -INFINITY;
      const float sum = soften(n, s[n]);
      if constexpr (WEIGHTS) record(n, t0 + 16 * grp, sum);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_ldexpf(s[n][8 * j + e], kScaleTop - vexp);
          const __bf16 hi = (__bf16)p;
          ph[n][j][e] = hi;
          pl[n][j][e] = (__bf16)(p - (float)hi);
        }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int u = 16 * grp + 8 * j;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (r0 + u < B) x = *reinterpret_cast<const uint4*>(vt + (c * 16 + col) * B + r0 + u);
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (u + 2 * e >= rows) w[e] = 0;
          else if (u + 2 * e + 1 >= rows) w[e] &= 0xFFFFu;
        }
        // infinities and NaN reach only the rows that see their token: 0 * infinity must not
        bool odd = false;
        uint32_t raw[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          raw[e] = w[e];
          const bool lo = (w[e] & 0x7F80u) == 0x7F80u, hi = (w[e] >> 16 & 0x7F80u) == 0x7F80u;
          odd |= lo || hi;
          w[e] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
        }
        if (__builtin_expect(__any(odd), 0)) {
#pragma unroll 1
          for (int x = 0; x < 32 * 4; ++x) {  // key 16 g + 8 j + e, channel i of this lane's four
            const int g = x >> 5, e = x >> 2 & 7, i = x & 3;
            const uint32_t pair = e < 4 ? (e < 2 ? raw[0] : raw[1]) : (e < 6 ? raw[2] : raw[3]);
            const uint32_t bits = (uint32_t)__shfl((int)(e & 1 ? pair >> 16 : pair & 0xFFFFu),
                                                   g * 16 + grp * 4 + i, 64);
            if ((bits & 0x7F80u) != 0x7F80u) continue;
            const float v = __uint_as_float(bits << 16);
#pragma unroll
            for (int n = 0; n < NT; ++n)
              if (16 * g + 8 * j + e < see[n] - t0) {
                if (i == 0) o[n][c][0] += v;
                if (i == 1) o[n][c][1] += v;
                if (i == 2) o[n][c][2] += v;
                if (i == 3) o[n][c][3] += v;
              }
          }
        }
        const bf8_t v = __builtin_bit_cast(bf8_t, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph[n][j], o[n][c], 0, 0, 0);
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl[n][j], o[n][c], 0, 0, 0);
        }
      }
  }

  // the waves meet
  const float unit = __builtin_ldexpf(1.f, vexp - kScaleTop);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = sum4groups(l[n]);
    if (grp == 0) part_ml[wave][n * 16 + col][0] = m[n], part_ml[wave][n * 16 + col][1] = l[n];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      *reinterpret_cast<f4_t*>(&part_o[wave][n * 16 + col][c * 16 + grp * 4]) = o[n][c] * unit;
  }
  __syncthreads();
  constexpr int LPR = D / 4;  // lanes of a row
  const bool whole = plan.n_splits == 1;
  for (int p = threadIdx.x; p < 16 * NT * LPR; p += 64 * kWaves) {
    const int rr = p / LPR, c = p % LPR * 4;
    const int64_t r = row0 + rr;
    if (r >= sq.n_q * G || r >= plan.rows) continue;
    float top = part_ml[0][rr][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, part_ml[w][rr][0]);
    float sum = 0.f;
    f4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(part_ml[w][rr][0] - top);
      sum += f * part_ml[w][rr][1];
      x += f * *reinterpret_cast<const f4_t*>(&part_o[w][rr][c]);
    }
    const int64_t rec = ((int64_t)z * plan.n_splits + split) * plan.rows + r;
    if (!whole || WEIGHTS) {
      if (c == 0) ml[2 * rec] = top, ml[2 * rec + 1] = sum;
    }
    if (!whole) {
      *reinterpret_cast<f4_t*>(po + rec * D + c) = x;
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int64_t i = sq.q0 + r / G, head = h * G + r % G;
      *reinterpret_cast<uint2*>(a.out + (i * a.n_q_heads + head) * D + c) =
          make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
      if (a.lse && c == 0)
        a.lse[i * a.n_q_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
  }
}

// splits of a row's tile that hold keys
__device__ __forceinline__ int splits_of(const Seq& sq, const Attn8Plan& plan, int64_t r, int G, int B) {
  const int n = 16 * plan.col_tiles;
  const int64_t steps = tile_of(sq, r / n * n, n, G, B).steps;
  const int64_t k = (steps + plan.span - 1) / plan.span;
  return (int)(k < 1 ? 1 : k > plan.n_splits ? plan.n_splits : k);
}

// The splits of a row in order: D / 4 lanes a row, 4 channels each.
template <int D>
__global__ void __launch_bounds__(256) attn8_join_kernel(Attn8 a, Attn8Plan plan, int B,
                                                         const float* __restrict__ po,
                                                         const float* __restrict__ ml) {
  constexpr int LPR = D / 4;
  const int z = blockIdx.y, b = z / a.c.n_kv_heads, h = z % a.c.n_kv_heads;
  const int G = a.n_q_heads / a.c.n_kv_heads;
  const Seq sq = seq_of(a, b, B);
  const int64_t r = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const int c = threadIdx.x % LPR * 4;
  if (!sq.ok || r >= sq.n_q * G || r >= plan.rows) return;
  const int n = splits_of(sq, plan, r, G, B);
  const int64_t rec = (int64_t)z * plan.n_splits * plan.rows + r;
  float top = kNoMax;
  for (int s = 0; s < n; ++s) top = fmaxf(top, ml[2 * (rec + s * plan.rows)]);
  float sum = 0.f;
  f4_t x = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < n; ++s) {
    const int64_t at = rec + s * plan.rows;
    const float f = __builtin_amdgcn_exp2f(ml[2 * at] - top);
    sum += f * ml[2 * at + 1];
    x += f * *reinterpret_cast<const f4_t*>(po + at * D + c);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t i = sq.q0 + r / G, head = h * G + r % G;
  *reinterpret_cast<uint2*>(a.out + (i * a.n_q_heads + head) * D + c) =
      make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
  if (a.lse && c == 0)
    a.lse[i * a.n_q_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// Accumulated weights: 16 lanes a block, each over every 16th row; the rows' log2 sums come
// through LDS, 256 rows at a time.
__global__ void __launch_bounds__(256) attn8_weights_kernel(Attn8 a, Attn8Plan plan, int B,
                                                            const float* __restrict__ ml,
                                                            const float* __restrict__ parts) {
  __shared__ float total[256];  // log2 of a row's sum
  const int z = blockIdx.y, b = z / a.c.n_kv_heads;
  const int G = a.n_q_heads / a.c.n_kv_heads, M = a.c.max_blocks;
  const Seq sq = seq_of(a, b, B);
  const int64_t blk = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
  const int PB = B < 64 ? B : 64, per = B / PB;
  const int64_t rows = sq.ok ? min(sq.n_q * G, plan.rows) : 0;
  float sum = 0.f;
  for (int64_t r0 = 0; r0 < rows; r0 += 256) {
    __syncthreads();
    const int64_t r = r0 + threadIdx.x;
    if (r < rows) {
      const int n = splits_of(sq, plan, r, G, B);
      const int64_t rec = (int64_t)z * plan.n_splits * plan.rows + r;
      float top = kNoMax, t = 0.f;
      for (int s = 0; s < n; ++s) top = fmaxf(top, ml[2 * (rec + s * plan.rows)]);
      for (int s = 0; s < n; ++s) {
        const int64_t at = rec + s * plan.rows;
        t += __builtin_amdgcn_exp2f(ml[2 * at] - top) * ml[2 * at + 1];
      }
      total[threadIdx.x] = t == 0.f ? INFINITY : top + log2f(t);  // nothing seen: no share
    }
    __syncthreads();
    for (int64_t x = r0 + threadIdx.x % 16; x < rows && x < r0 + 256; x += 16) {
      const int64_t see = min(sq.len - sq.n_q + x / G + 1, sq.keys);
      for (int p = 0; p < per; ++p) {
        const int64_t part = blk * per + p;
        if (blk < M && part * PB < see)
          sum += __builtin_amdgcn_exp2f(
              parts[((int64_t)z * plan.n_parts + part) * plan.rows + x] - total[x - r0]);
      }
    }
  }
#pragma unroll
  for (int k = 8; k > 0; k >>= 1) sum += __shfl_xor(sum, k, 64);
  if (blk < M && threadIdx.x % 16 == 0) {
    const int64_t at = (int64_t)z * M + blk;
    a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + sum;
  }
}

}  // namespace

Attn8Plan attn8_plan(int n_kv_heads, int head_dim, int block_len, int max_blocks, int n_q_heads,
                     int n_seqs, int max_queries, int max_len, bool with_weights) {
  Attn8Plan p{};
  p.rows = (int64_t)max_queries * (n_q_heads / n_kv_heads);
  p.col_tiles = p.rows <= 16 ? 1 : 2;
  p.n_tiles = (int)((p.rows + 16 * p.col_tiles - 1) / (16 * p.col_tiles));
  const int64_t heads = (int64_t)n_seqs * n_kv_heads, base = heads * p.n_tiles;
  const int64_t steps = ((int64_t)max_len + 63) / 64;
  // enough workgroups to fill 256 CUs three times, each with two steps a wave at least
  int64_t want = (768 + base - 1) / base, most = steps / 8;
  if (want > most) want = most;
  if (want < 1) want = 1;
  p.span = (int)((steps + want - 1) / want);
  if (p.span < 1) p.span = 1;
  p.n_splits = (int)((steps + p.span - 1) / p.span);
  if (p.n_splits < 1) p.n_splits = 1;
  const int pb = block_len < 64 ? block_len : 64;
  p.n_parts = with_weights ? ((int64_t)max_blocks + 1) * (block_len / pb) : 0;
  const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t records = (size_t)heads * p.n_splits * p.rows;
  p.ml_offset = p.n_splits > 1 ? up(records * head_dim * 4) : 0;
  p.parts_offset = p.ml_offset + (p.n_splits > 1 || with_weights ? up(records * 8) : 0);
  p.workspace = p.parts_offset + up((size_t)heads * p.n_parts * p.rows * 4);
  return p;
}

hipError_t launch_cache8_attn(const Attn8Plan& plan, const Attn8& a, int head_dim, int block_len,
                              int code, void* workspace, hipStream_t s) {
  char* ws = (char*)workspace;
  float *po = (float*)ws, *ml = (float*)(ws + plan.ml_offset), *parts = (float*)(ws + plan.parts_offset);
  const unsigned heads = (unsigned)a.c.n_seqs * a.c.n_kv_heads;
  const dim3 grid((unsigned)plan.n_splits, (unsigned)plan.n_tiles, heads);
#define KVB_ATTN(D, B, C, N, W) \
  hipLaunchKernelGGL((attn8_kernel<D, B, C, N, W>), grid, dim3(64 * kWaves), 0, s, a, plan, po, ml, parts)
#define KVB_ATTN_W(D, B, C, N) \
  do { if (a.weights_out) KVB_ATTN(D, B, C, N, true); else KVB_ATTN(D, B, C, N, false); } while (0)
#define KVB_ATTN_N(D, B, C) \
  do { if (plan.col_tiles == 1) KVB_ATTN_W(D, B, C, 1); else KVB_ATTN_W(D, B, C, 2); } while (0)
#define KVB_ATTN_C(D, B) \
  do { if (code == KVB_I8) KVB_ATTN_N(D, B, KVB_I8); else KVB_ATTN_N(D, B, KVB_E4M3); } while (0)
#define KVB_ATTN_B(D)                        \
  do {                                       \
    if (block_len == 16) KVB_ATTN_C(D, 16);  \
    else if (block_len == 32) KVB_ATTN_C(D, 32); \
    else if (block_len == 64) KVB_ATTN_C(D, 64); \
    else KVB_ATTN_C(D, 128);                 \
  } while (0)
  if (head_dim == 128) KVB_ATTN_B(128);
  else KVB_ATTN_B(64);
  if (hipError_t e = hipGetLastError()) return e;
  if (plan.n_splits > 1) {
    const int per = 256 / (head_dim / 4);
    const dim3 jg((unsigned)((plan.rows + per - 1) / per), heads);
    if (head_dim == 128)
      hipLaunchKernelGGL(attn8_join_kernel<128>, jg, dim3(256), 0, s, a, plan, block_len, po, ml);
    else
      hipLaunchKernelGGL(attn8_join_kernel<64>, jg, dim3(256), 0, s, a, plan, block_len, po, ml);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (a.weights_out)
    hipLaunchKernelGGL(attn8_weights_kernel, dim3((unsigned)((a.c.max_blocks + 15) / 16), heads),
                       dim3(256), 0, s, a, plan, block_len, ml, parts);
  return hipGetLastError();
}

}  // namespace kvb
