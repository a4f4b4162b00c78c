// Attention of the last tokens of each sequence over the 8-bit cache: the kernels.
//
// The G query heads of a kv head and the call's queries of a sequence are its rows
// (row = query * G + head).  Keys come in steps of 64.  A wave computes S^T (64 keys x
// 16 NT rows) = K Q^T and O^T (d x rows) += V^T P^T with 16x16x32 matrix instructions,
// codes and probabilities as fp16 (8-bit codes are exact there).  The contraction index of
// a product may be permuted if both operands agree: the rows of K are dealt to the four
// 16-key tiles of a step such that the scores a lane holds (keys 16 g .. 16 g + 15, g =
// lane / 16) are the keys of its V operand, 16 consecutive bytes of the channel-major V.
// So probabilities never move between lanes.
//
// Scales: a lane's 16 keys lie in one block (B >= 16).  The scale of K goes with the factor
// of the scores; that of V into the exponent of the probabilities, relative to the largest
// of the wave's chunks of blocks so far (2^kScaleTop at most, so that small blocks keep their bits in
// fp16), and out of the sums again by one product a step.  That factor is 2^-40 at least, so sums and
// weights keep their floats' accuracy however small a block's values are; a probability of at most 2^8
// times 2^-40 is 0 in fp16 anyway, so the product with V is the same with any smaller one.
//
// Few rows (attn8_kernel): HBM-bound; the waves of a workgroup take runs of steps of their
// own, operands straight from global memory, and meet in LDS at the end; where a call has
// few tiles, several workgroups share a tile's keys and a second launch joins them.
// Many rows (attn8_tile_kernel): bound by the matrix cores and what feeds them; eight waves of
// 32 rows share each step's keys and values, widened to fp16 once into LDS.
#pragma once
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

template <bool V>
struct Flag {
  static constexpr bool value = V;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -0x1.fffffep127f;  // running maximum before the first visible key: no score is below
constexpr float kSlack = 8.f;     // the running maximum follows once it is off by 2^8
constexpr float kFar = 0x1p20f;   // below it a score's rounding (2^-4 at most) is no matter to 2^score's range
constexpr int kScaleTop = 6;      // weights of V scales stay below 2^kScaleTop
constexpr int kTailTop = 16;      // outputs' unit (log2) over a tail, at least
constexpr int kManyTile = 256;    // rows of a tile of the many-rows kernel

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

// x combined over the lanes l, l ^ 16, l ^ 32 and l ^ 48; all four end with the result
template <typename F>
__device__ __forceinline__ float over4groups(float x, F f) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(f(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max4groups(float x) {
  return over4groups(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum4groups(float x) {
  return over4groups(x, [](float a, float b) { return a + b; });
}

// A sequence as the call sees it (32 bits: lens are int32, keys at most 2^31 - 1).
struct Seq {
  int n_q;   // its queries; 0 when cu_q does not fit the call
  int q0;    // the first of them
  int len;   // its tokens
  int full;  // full blocks
  int keys;  // tokens that can be seen
};
template <int B>
__device__ __forceinline__ Seq seq_of(const Attn8& a, int b) {
  Seq s;
  s.q0 = a.cu_q[b];
  const int64_t end = a.cu_q[b + 1];
  s.n_q = s.q0 >= 0 && end > s.q0 && end <= a.n_queries ? (int)(end - s.q0) : 0;
  s.len = max(a.c.lens[b], 0);
  s.full = s.len / B;
  s.keys = s.len;
  if (s.full > a.c.max_blocks) s.full = a.c.max_blocks, s.keys = s.full * B;
  return s;
}
// keys that query i of the sequence sees
__device__ __forceinline__ int seen_by(const Seq& s, int i) {
  return max(min(s.len - s.n_q + i + 1, s.keys), 0);
}
// the 64-key steps over full blocks that a tile needs; `last`: the tile's last query
template <int B>
__device__ __forceinline__ int steps_of(const Seq& s, int last) {
  const int coded = min(seen_by(s, min(last, s.n_q - 1)), s.full * B);
  return coded / 64 + (coded % 64 != 0);
}

// x of lane i: uniform (on the scalar unit), or a lane's own choice
template <bool UNIFORM>
__device__ __forceinline__ float lane_of(float x, int i) {
  if constexpr (UNIFORM) return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), i));
  return __shfl(x, i, 64);
}
__device__ __forceinline__ float max64(float x) {
#pragma unroll
  for (int k = 1; k < 16; k <<= 1) x = fmaxf(x, __shfl_xor(x, k, 64));
  return max4groups(x);
}

// What a workgroup takes: a split of the keys of a (sequence, kv head) z, and a tile of its rows.
// Workgroups go to the 8 XCDs in turn; with plan.apart, tiles that read the same keys are kXcds apart,
// so that they run side by side on one XCD and share its L2.
constexpr int kXcds = 8;
struct Place {
  int z, split, tile;  // z < 0: none
};
__device__ __forceinline__ Place place(const Attn8& a, const Attn8Plan& plan) {
  if (!plan.apart) return {(int)blockIdx.z, (int)blockIdx.x, (int)blockIdx.y};
  const int group = blockIdx.y * kXcds + blockIdx.x % kXcds, z = group / plan.n_splits;
  return {z < a.c.n_rows ? z : -1, group - z * plan.n_splits, (int)blockIdx.x / kXcds};
}

// Outputs are divided by their sums before they leave a wave, and joined by weights whose sum is 1, so that
// nothing passes the largest value of V (a sum of probabilities, up to 2^8 a key, times V may leave a float).
// A reciprocal within 2^-23 will do (0.08 us less than IEEE quotients of a token's 11.5 over 2000).
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum); }

// One row's result x in bfloat16, and the log of its sum.
__device__ __forceinline__ void write_row(const Attn8& a, int q, int head, int D, int c, f4_t x,
                                          float top, float sum) {
  const int64_t r = (int64_t)q * a.n_q_heads + head;
  *reinterpret_cast<uint2*>(a.out + r * D + c) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  if (a.lse && c == 0) a.lse[r] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// The state of a wave: its rows' queries, running maxima and sums, and outputs O^T in units
// of 2^(vexp - kScaleTop).
template <int D, int B, int NT, bool WEIGHTS>
struct Rows {
  static constexpr int KS = D / 32;           // contraction steps of a score
  static constexpr int CT = D / 16;           // channel tiles of the output
  static constexpr int PB = B < 64 ? B : 64;  // tokens of a part with a weight of its own
  half8_t q[NT][KS];
  float cq[NT];              // score (log2 units) of a product: cq * scale of K
  int see[NT];               // keys the row sees
  float m[NT], l[NT];
  f4_t o[NT][CT];
  int vexp;
  uint64_t far;  // not 0: a running maximum is or was beyond kFar
  float* parts;  // log2 weights of the parts, of plan.rows rows each
  int n_parts;   // the parts below this are written
  int row, rows; // this lane's first row (the others follow 16 apart), rows of a part

  // Queries: a power of two brings each row's largest value into [0.5, 1), so that fp16 holds
  // a bfloat16 of the row exactly (below 2^-14 of the largest: to 2^-25 of it).  They carry the
  // sign of softmax_scale, so that the scores' factors are not negative.
  // where query row r lies; a row past the last one reads the first one (and sees nothing)
  static __device__ __forceinline__ const uint16_t* query(const Attn8& a, const Seq& sq, int h, int G, int r) {
    const int i = (int)((unsigned)r / (unsigned)G);
    const bool ok = i < sq.n_q;
    return a.q + ((int64_t)(sq.q0 + (ok ? i : 0)) * a.n_q_heads + h * G + (ok ? r - i * G : 0)) * D;
  }
  __device__ __forceinline__ void start(const Attn8& a, const Seq& sq, int h, int G, int row0,
                                        int grp, int col) {
    const uint32_t flip = a.softmax_scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = row0 + n * 16 + col, i = (int)((unsigned)r / (unsigned)G);
      const uint16_t* qrow = query(a, sq, h, G, r);
      see[n] = i < sq.n_q ? seen_by(sq, i) : 0;
      uint4 w[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k)
        w[k] = *reinterpret_cast<const uint4*>(qrow + 64 * (k / 2) + 16 * grp + 8 * (k % 2));
      uint32_t big = 0;  // the largest magnitude's bits: integers order like magnitudes
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          big = max(big, max(u[e] << 16 & 0x7FFF0000u, u[e] & 0x7FFF0000u));
      }
      const float top = over4groups(__uint_as_float(big), [](float x, float y) {
        return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y)));
      });
      const int e2 = top > 0.f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
      cq[n] = __builtin_ldexpf(fabsf(a.softmax_scale) * kLog2e, e2);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          q[n][k][2 * e] = (_Float16)__builtin_ldexpf(bf16_lo(u[e] ^ flip), -e2);
          q[n][k][2 * e + 1] = (_Float16)__builtin_ldexpf(bf16_hi(u[e] ^ flip), -e2);
        }
      }
      m[n] = kNoMax, l[n] = 0.f;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] = (f4_t){0.f, 0.f, 0.f, 0.f};
    }
    vexp = -127, far = 0;
  }

  // room for scales of V up to `big`
  __device__ __forceinline__ void fit(float big) {
    if (big > 0.f) {
      const int e = max(__builtin_amdgcn_frexp_expf(big), -100);
      if (e > vexp) unit(e);
    }
  }
  // the weight of a scale of V: its size in the outputs' unit.  Blocks of zeros or NaN have codes 0, any
  // weight will do; the smallest is 2^-40 (a float's reciprocal and its logarithm stay exact enough)
  __device__ __forceinline__ float weight_of(float vs) const {
    return vs > 0.f ? fmaxf(__builtin_ldexpf(vs, kScaleTop - vexp), 0x1p-40f) : 1.f;
  }
  // outputs in units of 2^(e - kScaleTop) from here on
  __device__ __forceinline__ void unit(int e) {
    const float f = __builtin_ldexpf(1.f, vexp - e);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] *= f;
    vexp = e;
  }

  // Raw scores -> probabilities times 2^lv (the scale of V) of the step: exp2(f s - m + lv).  The
  // running maximum, the sums (iv = 2^-lv takes the scale out again) and the part's weight
  // follow.  f >= 0; masked scores are -infinity with f = 1.  key: the first of this lane's 16.
  // Beyond kFar the exact f s and the rounded maximum may be far apart, and lv lost in the maximum: there
  // the rounded products are compared, so that no probability passes 2^kSlack.
  __device__ __forceinline__ void soften(int n, float (&s)[16], float f, float lv, float iv, int key) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = max4groups(top * f);
    float base = m[n];
    if (__builtin_expect((__ballot(top - base > kSlack) | far) != 0, 0)) {
      const float next = top - base > kSlack ? top : base;
      const float g = __builtin_amdgcn_exp2f(base - next);
      l[n] *= g;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] *= g;
      m[n] = base = next;
      far |= __ballot(fabsf(next) > kFar && next != kNoMax);
      if (__builtin_expect(far != 0, 0)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = s[i] * f - next;
        f = 1.f, base = 0.f;
      }
    }
    const float bias = lv - base;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], f, bias));
      sum += s[i];
    }
    sum *= iv;
    l[n] += sum;
    if constexpr (WEIGHTS) {
      if constexpr (PB == 32) {
        const uint32_t u = __float_as_uint(sum);
        const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        sum = __uint_as_float(a[0]) + __uint_as_float(a[1]);
      }
      if constexpr (PB == 64) sum = sum4groups(sum);
      if (key % PB == 0) put_part(n, key / PB, m[n] + __builtin_amdgcn_logf(sum));
    }
  }

  // Scores of a step of coded keys -> the operand of the product with V.  lv, iv: log2 of the weight of
  // the scale of V, and the weight's reciprocal (this lane's block).
  __device__ __forceinline__ void step(float (&s)[NT][16], int key, bool have, float ks, float lv,
                                       float iv, half8_t (&pr)[NT][2]) {
    bool clear = have;
#pragma unroll
    for (int n = 0; n < NT; ++n) clear = clear && see[n] >= key + 16;
    const bool plain = __all(clear);  // every key of the step is seen by every row
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float f = ks * cq[n];
      if (!plain) {
        const int left = have ? see[n] - key : 0;  // visible of the lane's 16 keys
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = i < left ? s[n][i] * f : -INFINITY;
        f = 1.f;
      }
      soften(n, s[n], f, lv, iv, key);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        half2_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f2_t v = {s[n][8 * j + 2 * e], s[n][8 * j + 2 * e + 1]};
          x[e] = __builtin_convertvector(v, half2_t);
        }
        pr[n][j] = __builtin_bit_cast(half8_t, x);
      }
    }
  }
  // A block of V whose scale is a NaN has codes 0: the rows that see of it (keys from `key` on) become
  // NaN, the others stay clean.  The channels of a row lie in the four lanes of its column.
  __device__ __forceinline__ void spoil(bool nan, int key) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float x = sum4groups(nan && see[n] > key ? __builtin_nanf("") : 0.f);
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] += x;
    }
  }
  // One step of 64 keys of the tail, bfloat16 rows from r0 on.  Probabilities enter as the sum of two
  // bfloat16, in the outputs' unit; rows past the tail's end hold anything, so their values of V
  // are cleared.
  __device__ __forceinline__ void tail(const Attn8& a, const Seq& sq, int z, int h, int G, int row0, int r0,
                                       int lane) {
    // up to 128 probabilities of up to 2^kSlack, times bfloat16 values, in a unit of 2^16 fit a float
    if (vexp < kScaleTop + kTailTop) unit(kScaleTop + kTailTop);
    const uint16_t* kt = a.c.k_tail + (int64_t)z * B * D;
    const uint16_t* vt = a.c.v_tail + (int64_t)z * B * D;
    const int grp = lane >> 4, col = lane & 15, t0 = sq.full * B + r0;
    const int rows = min(64, sq.len - t0);  // tail rows of this step
    float s[NT][16];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f4_t acc[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = (f4_t){0.f, 0.f, 0.f, 0.f};
      // rows past the block are read like its last one; they are not seen
      const int u = min(r0 + 16 * (col >> 2) + 4 * t + (col & 3), B - 1);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf8_t x = *reinterpret_cast<const bf8_t*>(kt + u * D + k * 32 + grp * 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bf8_t y = *reinterpret_cast<const bf8_t*>(query(a, sq, h, G, row0 + n * 16 + col) + k * 32 + grp * 8);
          acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[n], 0, 0, 0);
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
      const int left = see[n] - (t0 + 16 * grp);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = i < left ? s[n][i] * f : -INFINITY;
      soften(n, s[n], 1.f, 0.f, 1.f, t0 + 16 * grp);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_ldexpf(s[n][8 * j + e], kScaleTop - vexp);
          const __bf16 top = (__bf16)p;
          ph[n][j][e] = top;
          pl[n][j][e] = (__bf16)(p - (float)top);
        }
    }
    uint32_t odd = 0;  // not 0: an infinity or NaN among the values of V
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int u = 16 * grp + 8 * j, at = min(r0 + u, B - 8);
      uint32_t in[4];  // the halves of each word that are rows of the tail
#pragma unroll
      for (int e = 0; e < 4; ++e)
        in[e] = (u + 2 * e < rows ? 0xFFFFu : 0u) | (u + 2 * e + 1 < rows ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint4 x = *reinterpret_cast<const uint4*>(vt + (c * 16 + col) * B + at);
        uint32_t w[4] = {x.x & in[0], x.y & in[1], x.z & in[2], x.w & in[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bad = ((w[e] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) |
                               ((w[e] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
          odd |= bad;
          w[e] &= ~bad;
        }
        const bf8_t v = __builtin_bit_cast(bf8_t, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph[n][j], o[n][c], 0, 0, 0);
          o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl[n][j], o[n][c], 0, 0, 0);
        }
      }
    }
    // infinities and NaN of V reach only the rows that see their token (0 * infinity must not): they
    // stayed out of the products and are added one by one
    if (__builtin_expect(__any(odd != 0), 0)) {
      for (int u = 0; u < rows; ++u) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bits = vt[(c * 16 + grp * 4 + i) * B + r0 + u];
            const bool bad = (bits & 0x7F80u) == 0x7F80u;
#pragma unroll
            for (int n = 0; n < NT; ++n)
              if (bad && t0 + u < see[n]) o[n][c][i] += __uint_as_float(bits << 16);
          }
      }
    }
  }
  // log2 of the weight of part p
  __device__ __forceinline__ void put_part(int n, int p, float x) {
    if (row + 16 * n < rows && p < n_parts) parts[(int64_t)p * rows + row + 16 * n] = x;
  }
};

template <int D, int B, int CODE, int NT, bool WEIGHTS, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2)
attn8_kernel(Attn8 a, Attn8Plan plan, float* __restrict__ po, float* __restrict__ ml,
             float* __restrict__ parts) {
  typedef Rows<D, B, NT, WEIGHTS> R;
  constexpr int CT = R::CT;
  constexpr int KP = D / 64;              // 16-byte pieces of a lane's key
  constexpr int CHUNK = B < 64 ? B : 64;  // steps whose blocks' ids and scales a wave holds
  constexpr bool ONE = B >= 64;           // a step lies in one block
  constexpr int LDO = D + 4;
  __shared__ __align__(16) float part_o[WAVES][16 * NT][LDO];
  __shared__ float part_ml[WAVES][16 * NT][2];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int grp = lane >> 4, col = lane & 15;
  const Place at = place(a, plan);
  if (at.z < 0) return;
  const int z = at.z, split = at.split;
  const int b = z / a.c.n_kv_heads, h = z - b * a.c.n_kv_heads;
  const int G = plan.group;
  const int row0 = at.tile * (16 * NT);
  const int32_t* table = a.c.table + (int64_t)z * a.c.max_blocks;

  // The wave's steps: the split's, divided evenly; the last split takes what is left over where a
  // sequence is longer than the call was sized for.  The first ids are asked for before the
  // sequence's length is known.
  const int lo = split * plan.span + min(wave * plan.wave_span, plan.span);
  int idn = -1;
  {
    const int blk = (ONE ? lo / (B / 64) : lo * (64 / B)) + lane;
    if (blk < a.c.max_blocks) idn = table[blk];
  }
  const Seq sq = seq_of<B>(a, b);
  if (row0 >= sq.n_q * G) return;
  const int last = (int)((unsigned)(row0 + 16 * NT - 1) / (unsigned)G);
  const int steps = steps_of<B>(sq, last);
  if (split > 0 && split * plan.span >= steps) return;
  int hi = min(min(lo + plan.wave_span, (split + 1) * plan.span), steps);
  if (split == plan.n_splits - 1 && wave == WAVES - 1) hi = steps;

  R r;
  r.start(a, sq, h, G, row0, grp, col);
  if constexpr (WEIGHTS) {
    // parts of the full blocks; the tail's are its own wave's to write
    r.parts = parts + (int64_t)z * plan.n_parts * plan.rows;
    r.n_parts = sq.full * (B / R::PB), r.row = row0 + col, r.rows = plan.rows;
  }

  for (int c0 = lo; c0 < hi; c0 += CHUNK) {
    const int c1 = min(c0 + CHUNK, hi);
    const int blk0 = ONE ? c0 / (B / 64) : c0 * (64 / B);
    // lane i holds id and scales of block blk0 + i
    int id = idn;
    if (c0 != lo) id = blk0 + lane < a.c.max_blocks ? table[blk0 + lane] : -1;
    const uint64_t found = __ballot(blk0 + lane < sq.full && id >= 0 && id < a.c.n_blocks);
    if (found == 0) {  // none of them is a block
      if constexpr (WEIGHTS) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          for (int x = grp; x < (c1 - c0) * (64 / R::PB); x += 4)
            r.put_part(n, c0 * (64 / R::PB) + x, -INFINITY);
      }
      continue;
    }
    // what is no block is read like the first one that is: no value of V may be a NaN
    const bool mine = found >> lane & 1;
    id = mine ? id : __builtin_amdgcn_readlane(id, __builtin_ctzll(found));
    const float ks = a.c.k_scale[id], vs = mine ? a.c.v_scale[id] : 0.f;

    uint4 kw[4][KP], vr[CT];
    // the block of this lane's K row (keys 16 (col / 4) ..) or of its 16 keys (16 grp ..)
    auto id_at = [&](int st, int sub) {
      const int i = ONE ? st / (B / 64) - blk0 : st * (64 / B) + sub / (B / 16) - blk0;
      return ONE ? __builtin_amdgcn_readlane(id, i) : __shfl(id, i, 64);
    };
    auto load_k = [&](int st) {
      const int i = id_at(st, col >> 2);
      const int in = ONE ? st % (B / 64) * 64 + 16 * (col >> 2) : 16 * (col >> 2) % B;
      const uint8_t* p = a.c.k_codes + (int64_t)i * (B * D) + (in + (col & 3)) * D + grp * 16;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < KP; ++x) kw[t][x] = *reinterpret_cast<const uint4*>(p + 4 * t * D + x * 64);
    };
    auto load_v = [&](int st) {
      const int i = id_at(st, grp);
      const int in = ONE ? st % (B / 64) * 64 + 16 * grp : 16 * grp % B;
      const uint8_t* p = a.c.v_codes + (int64_t)i * (B * D) + col * B + in;
#pragma unroll
      for (int c = 0; c < CT; ++c) vr[c] = *reinterpret_cast<const uint4*>(p + c * 16 * B);
    };
    load_k(c0);
    load_v(c0);
    r.fit(max64(vs));
    const float vw = r.weight_of(vs);
    const float lv = __builtin_amdgcn_logf(vw), iv = 1.f / vw;
    const uint64_t nans = __ballot(vs != vs);

#pragma unroll 1
    for (int st = c0; st < c1; ++st) {
      const int key0 = st * 64;
      const int gb = ONE ? st / (B / 64) - blk0 : st * (64 / B) + grp / (B / 16) - blk0;
      const bool have = found >> gb & 1;
      const float ksg = lane_of<ONE>(ks, gb), lvg = lane_of<ONE>(lv, gb), ivg = lane_of<ONE>(iv, gb);
      float s[NT][16];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f4_t acc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = (f4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < KP; ++x) {
          const half8_t k0 = widen8<CODE>(kw[t][x].x, kw[t][x].y);
          const half8_t k1 = widen8<CODE>(kw[t][x].z, kw[t][x].w);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, r.q[n][2 * x], acc[n], 0, 0, 0);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, r.q[n][2 * x + 1], acc[n], 0, 0, 0);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[n][4 * t + i] = acc[n][i];
      }
      if (st + 1 < c1) load_k(st + 1);
      half8_t pr[NT][2];
      r.step(s, key0 + 16 * grp, have, ksg, lvg, ivg, pr);
      if (__builtin_expect(nans != 0, 0)) r.spoil(nans >> gb & 1, key0 + 16 * grp);
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const half8_t v0 = widen8<CODE>(vr[c].x, vr[c].y), v1 = widen8<CODE>(vr[c].z, vr[c].w);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pr[n][0], r.o[n][c], 0, 0, 0);
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pr[n][1], r.o[n][c], 0, 0, 0);
        }
      }
      if (st + 1 < c1) load_v(st + 1);
    }
  }

  // The tail, a step for each of the first split's last waves (a block has at most two)
  const int r0 = (WAVES - 1 - wave) * 64;
  if constexpr (WEIGHTS) r.n_parts += B / R::PB;
  if (split == 0 && r0 < B && sq.full * B + r0 < seen_by(sq, min(last, sq.n_q - 1)))
    r.tail(a, sq, z, h, G, row0, r0, lane);

  // the waves meet
  const float unit = __builtin_ldexpf(1.f, r.vexp - kScaleTop);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    r.l[n] = sum4groups(r.l[n]);
    const float inv = inverse(r.l[n]);
    if (grp == 0) part_ml[wave][n * 16 + col][0] = r.m[n], part_ml[wave][n * 16 + col][1] = r.l[n];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      *reinterpret_cast<f4_t*>(&part_o[wave][n * 16 + col][c * 16 + grp * 4]) = r.o[n][c] * inv * unit;
  }
  __syncthreads();
  constexpr int LPR = D / 4;  // lanes of a row
  const bool whole = plan.n_splits == 1;
#pragma unroll 1
  for (int p = threadIdx.x; p < 16 * NT * LPR; p += 64 * WAVES) {
    const int rr = p / LPR, c = p % LPR * 4;
    const int row = row0 + rr;
    if (row >= sq.n_q * G || row >= plan.rows) continue;
    float top = part_ml[0][rr][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, part_ml[w][rr][0]);
    float sum = 0.f, f[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      f[w] = __builtin_amdgcn_exp2f(part_ml[w][rr][0] - top) * part_ml[w][rr][1];
      sum += f[w];
    }
    const float inv = inverse(sum);
    f4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x += f[w] * inv * *reinterpret_cast<const f4_t*>(&part_o[w][rr][c]);
    const int64_t rec = ((int64_t)z * plan.n_splits + split) * plan.rows + row;
    if ((!whole || WEIGHTS) && c == 0) ml[2 * rec] = top, ml[2 * rec + 1] = sum;
    if (!whole) {
      *reinterpret_cast<f4_t*>(po + rec * D + c) = x;
    } else {
      const int i = (int)((unsigned)row / (unsigned)G);
      write_row(a, sq.q0 + i, h * G + row - i * G, D, c, x, top, sum);
    }
  }
}

// The ids and scales of 64 blocks (or fewer: `steps` 64-key steps from step0 on), one a lane.
template <int B>
struct Chunk {
  static constexpr int STEPS = B < 64 ? B : 64;
  static constexpr bool ONE = B >= 64;  // a step lies in one block
  int id, blk0;
  uint64_t found;  // lanes whose entry is a block; the others read like the first one that is
  __device__ __forceinline__ void load(const Attn8& a, const Seq& sq, const int32_t* table, int step0,
                                       int lane) {
    blk0 = ONE ? step0 / (B / 64) : step0 * (64 / B);
    id = blk0 + lane < a.c.max_blocks ? table[blk0 + lane] : -1;
    found = __ballot(blk0 + lane < sq.full && id >= 0 && id < a.c.n_blocks);
    if (!(found >> lane & 1)) id = found ? __builtin_amdgcn_readlane(id, __builtin_ctzll(found)) : 0;
  }
  // the lane that holds the block of key group g (16 keys) of a step
  __device__ __forceinline__ int lane_of_group(int st, int g) const {
    return ONE ? st / (B / 64) - blk0 : st * (64 / B) + g / (B / 16) - blk0;
  }
};

// Many rows: a workgroup takes 256 rows, 32 a wave, two waves a SIMD.  Each step's codes are read
// once (a thread takes a 512th of it, two steps ahead), widened to fp16 and shared through LDS; K
// lies in rows of keys (in tile order), V in rows of channels, and the 16-byte pieces of a row
// are permuted by the row so that the 16 rows a matrix operand takes lie in all banks.
//
// The matrix cores and the vector unit of a SIMD work for one wave each: a wave's step is a run of
// matrix products, M(i) = the product of step i - 1's probabilities with V, then the scores of step
// i, and a run of vector work, S(i) = the probabilities of step i, codes of K (step i + 2) and of V
// (i + 1) widened into LDS, loads of the next ones; waves 4 to 7 are one run behind waves 0 to 3,
// and a barrier ends every run.  Three slots: a slot is written two runs before it is read and two
// runs after it was.  2048 queries of 16 heads, 32K tokens of 2 (533 GFLOP): 522 to 526 us,
// 1020 TFLOP/s, in a row of such calls (600 to 620 in the first ones after a rest); with 4 waves a
// workgroup, 2 workgroups a CU and every wave free to run, both kinds of work took turns by
// chance: 601 us.  Either kind alone takes 330 to 350 us.
template <int D, int B, int CODE, bool WEIGHTS>
__global__ void __launch_bounds__(512, 2)
attn8_tile_kernel(Attn8 a, Attn8Plan plan, float* __restrict__ po, float* __restrict__ ml,
                  float* __restrict__ parts) {
  constexpr int NT = 2;
  typedef Rows<D, B, NT, WEIGHTS> R;
  typedef Chunk<B> Ids;
  constexpr int KS = R::KS, CT = R::CT;
  constexpr bool ONE = Ids::ONE;
  constexpr int KC = D / 8;          // 16-byte pieces of a key's fp16 row
  constexpr int PIECES = 64 * D / 16;  // 16-byte pieces of codes of a step's K, and of its V
  __shared__ __align__(16) half8_t kl[3][64 * KC], vl[3][D * 8];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = lane >> 4, col = lane & 15;
  const int z = blockIdx.z, split = blockIdx.x;
  const int b = z / a.c.n_kv_heads, h = z - b * a.c.n_kv_heads;
  const int G = plan.group;
  const int row0 = blockIdx.y * kManyTile;
  const int32_t* table = a.c.table + (int64_t)z * a.c.max_blocks;
  const Seq sq = seq_of<B>(a, b);
  if (row0 >= sq.n_q * G) return;
  const int last = min((int)((unsigned)(row0 + kManyTile - 1) / (unsigned)G), sq.n_q - 1);
  const int steps = steps_of<B>(sq, last);
  const int lo = split * plan.span;
  if (split > 0 && lo >= steps) return;
  const int hi = split == plan.n_splits - 1 ? steps : min(lo + plan.span, steps);

  R r;
  const int wrow0 = row0 + 32 * wave;
  r.start(a, sq, h, G, wrow0, grp, col);
  if constexpr (WEIGHTS) {
    r.parts = parts + (int64_t)z * plan.n_parts * plan.rows;
    r.n_parts = sq.full * (B / R::PB), r.row = wrow0 + col, r.rows = plan.rows;
  }

  if (lo < hi) {
    Ids ids[2];  // of the steps' current chunk and the next one
    ids[0].load(a, sq, table, lo, lane);
    ids[1].load(a, sq, table, lo + Ids::STEPS, lane);
    int turn = lo + Ids::STEPS;  // the first step of the next chunk
    float ks = 0.f, lv = 0.f, iv = 1.f;
    uint64_t found = 0, nans = 0;
    auto scales = [&]() __attribute__((always_inline)) {  // of the current chunk
      found = ids[0].found;
      ks = a.c.k_scale[ids[0].id];
      const float vs = found >> lane & 1 ? a.c.v_scale[ids[0].id] : 0.f;
      r.fit(max64(vs));
      const float vw = r.weight_of(vs);
      lv = __builtin_amdgcn_logf(vw), iv = 1.f / vw;
      nans = __ballot(vs != vs);
    };
    scales();

    // A thread's pieces of a step's K and V (head size 64: two threads a piece).  No branches: a step past
    // the last one reads the last one, and lands in a slot that nobody reads.
    uint4 kw[2], vw4[2];  // two steps' codes in flight
    const int p = PIECES >= 512 ? tid : tid & (PIECES - 1);
    const int key = p / (D / 16), kc = p % (D / 16) * 2, ch = p >> 2, vk = (p & 3) * 2;
    const int krow = (key & 12) * 4 + (key >> 4) * 4 + (key & 3);  // tile (key % 16) / 4, row of it
    auto block_of = [&](int st, int group) __attribute__((always_inline)) {
      const bool next = st >= turn;
      const int id = next ? ids[1].id : ids[0].id, blk0 = next ? ids[1].blk0 : ids[0].blk0;
      if constexpr (ONE) return __builtin_amdgcn_readlane(id, st / (B / 64) - blk0);
      else return __shfl(id, st * (64 / B) + group / (B / 16) - blk0, 64);
    };
    auto load_k = [&](int st, uint4& kw) __attribute__((always_inline)) {
      st = min(st, hi - 1);
      const int in = ONE ? st % (B / 64) * 64 + key : key % B;
      kw = *reinterpret_cast<const uint4*>(a.c.k_codes + (int64_t)block_of(st, key >> 4) * (B * D) + in * D + kc * 8);
    };
    auto load_v = [&](int st, uint4& vw4) __attribute__((always_inline)) {
      st = min(st, hi - 1);
      const int in = ONE ? st % (B / 64) * 64 + vk * 8 : vk * 8 % B;
      vw4 = *reinterpret_cast<const uint4*>(a.c.v_codes + (int64_t)block_of(st, p & 3) * (B * D) + ch * B + in);
    };
    const int k0 = krow * KC + (kc ^ (krow & (KC - 1))), k1 = krow * KC + ((kc + 1) ^ (krow & (KC - 1)));
    const int v0 = ch * 8 + ((p & 3) ^ (ch >> 1 & 7)), v1 = ch * 8 + (((p & 3) + 4) ^ (ch >> 1 & 7));
    auto store_k = [&](int slot, const uint4& kw) __attribute__((always_inline)) {
      half8_t* to = kl[0] + slot * (64 * KC);
      to[k0] = widen8<CODE>(kw.x, kw.y);
      to[k1] = widen8<CODE>(kw.z, kw.w);
    };
    auto store_v = [&](int st, int slot, const uint4& vw4) __attribute__((always_inline)) {
      // no block at all in the chunk: no value of V may be a NaN
      const uint32_t some = (st >= turn ? ids[1].found : ids[0].found) ? ~0u : 0u;
      half8_t* to = vl[0] + slot * (D * 8);
      to[v0] = widen8<CODE>(vw4.x & some, vw4.y & some);
      to[v1] = widen8<CODE>(vw4.z & some, vw4.w & some);
    };
    auto run_ends = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_sched_barrier(0);
      __syncthreads();
      __builtin_amdgcn_sched_barrier(0);
    };
    float s[NT][16];
    half8_t pr[NT][2];
    // where this lane's operand pieces lie in a slot: of contraction step k, and of keys 16 grp + 8 j ..
    int ko[KS], vo[2];
#pragma unroll
    for (int k = 0; k < KS; ++k) ko[k] = col * KC + ((8 * (k / 2) + 2 * grp + k % 2) ^ (col & (KC - 1)));
#pragma unroll
    for (int j = 0; j < 2; ++j) vo[j] = col * 8 + ((4 * j + grp) ^ (col >> 1));
    // A run of matrix products: V of the slot before (not for the first), then scores of slot `at`.  The
    // operand pieces are read AHEAD of their products, in this order.
    auto products = [&](int before, int at, bool first) __attribute__((always_inline)) {
      constexpr int AHEAD = 6, NV = 2 * CT, ALL = NV + 4 * KS;
      half8_t x[8];
      f4_t acc[NT][4];
      const half8_t* vp = vl[0] + before * (D * 8);
      const half8_t* kp = kl[0] + at * (64 * KC);
      auto piece = [&](int i) {
        return i < NV ? vp[vo[i / CT] + i % CT * 128] : kp[ko[(i - NV) / 4] + (i - NV) % 4 * 16 * KC];
      };
      const int from = first ? NV : 0;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) x[(from + i) % 8] = piece(from + i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = from; i < ALL; ++i) {
        if (i + AHEAD < ALL) x[(i + AHEAD) % 8] = piece(i + AHEAD);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (i < NV) {
            r.o[n][i % CT] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[i % 8], pr[n][i / CT], r.o[n][i % CT], 0, 0, 0);
          } else {
            const int k = (i - NV) / 4, t = (i - NV) % 4;
            acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                x[i % 8], r.q[n][k], k == 0 ? (f4_t){0.f, 0.f, 0.f, 0.f} : acc[n][t], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[n][e] = acc[n][e / 4][e % 4];
    };

    load_k(lo, kw[0]);
    load_v(lo, vw4[0]);
    load_k(lo + 1, kw[1]);
    store_k(0, kw[0]);
    store_v(lo, 0, vw4[0]);
    load_k(lo + 2, kw[0]);
    load_v(lo + 1, vw4[0]);
    store_k(1, kw[1]);
    load_k(lo + 3, kw[1]);
    load_v(lo + 2, vw4[1]);
    run_ends();
    if (wave >= 4) run_ends();
    int s0 = 0, s1 = 1, s2 = 2;  // slots of steps st, st + 1, st + 2
    auto step = [&](auto busy, int st, uint4& kw, uint4& vw4) __attribute__((always_inline)) {
      const int key = st * 64 + 16 * grp;
      const int gb = ids[0].lane_of_group(st, grp);
      if constexpr (busy.value)
        r.step(s, key, found >> gb & 1, lane_of<ONE>(ks, gb), lane_of<ONE>(lv, gb), lane_of<ONE>(iv, gb), pr);
      if (busy.value && __builtin_expect(nans != 0, 0)) r.spoil(nans >> gb & 1, key);
      store_k(s2, kw);
      store_v(st + 1, s1, vw4);
      load_k(st + 4, kw);
      load_v(st + 3, vw4);
      run_ends();
      __builtin_amdgcn_s_setprio(1);
      if constexpr (busy.value) products(s0, s1, false);  // behind the last step: scores of what the slot holds, for nothing
      __builtin_amdgcn_s_setprio(0);
      if (st + 1 == turn) {  // the next chunk's blocks; st + 4 at most was asked of them so far
        ids[0] = ids[1];
        turn += Ids::STEPS;
        ids[1].load(a, sq, table, turn, lane);
        scales();
      }
      const int x = s0;
      s0 = s1, s1 = s2, s2 = x;
      if (st + 1 < hi || wave < 4) run_ends();
    };
    auto walk = [&](auto busy) __attribute__((always_inline)) {
      if constexpr (busy.value) products(0, 0, true);
      run_ends();
#pragma unroll 1
      for (int st = lo; st < hi; st += 2) {
        step(busy, st, kw[0], vw4[0]);
        if (st + 1 < hi) step(busy, st + 1, kw[1], vw4[1]);
      }
    };
    // a wave without rows only feeds the others
    if (wrow0 < sq.n_q * G) walk(Flag<true>{});
    else walk(Flag<false>{});
  }

  if constexpr (WEIGHTS) r.n_parts += B / R::PB;
  if (split == 0)
    for (int r0 = 0; r0 < B && sq.full * B + r0 < seen_by(sq, last); r0 += 64) r.tail(a, sq, z, h, G, wrow0, r0, lane);

  const float unit = __builtin_ldexpf(1.f, r.vexp - kScaleTop);
  const bool whole = plan.n_splits == 1;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = wrow0 + n * 16 + col;
    const float sum = sum4groups(r.l[n]), inv = inverse(sum);
    if (row >= sq.n_q * G || row >= plan.rows) continue;
    const int64_t rec = ((int64_t)z * plan.n_splits + split) * plan.rows + row;
    if ((!whole || WEIGHTS) && grp == 0) ml[2 * rec] = r.m[n], ml[2 * rec + 1] = sum;
    const int i = (int)((unsigned)row / (unsigned)G);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int ch = c * 16 + grp * 4;
      const f4_t x = r.o[n][c] * inv * unit;
      if (whole) write_row(a, sq.q0 + i, h * G + row - i * G, D, ch, x, r.m[n], sum);
      else *reinterpret_cast<f4_t*>(po + rec * D + ch) = x;
    }
  }
}

template <int D, int B, int CODE>
void launch_kernels(const Attn8Plan& plan, const Attn8& a, float* po, float* ml, float* parts,
                    hipStream_t s) {
  dim3 grid((unsigned)plan.n_splits, (unsigned)plan.n_tiles, (unsigned)a.c.n_rows);
  if (plan.apart)
    grid = dim3((unsigned)(kXcds * plan.n_tiles), (unsigned)((plan.n_splits * a.c.n_rows + kXcds - 1) / kXcds));
  const dim3 block(plan.tile_rows == kManyTile ? 512 : 64 * plan.waves);
#define KVB_ATTN(...) hipLaunchKernelGGL((__VA_ARGS__), grid, block, 0, s, a, plan, po, ml, parts)
  const bool w = a.weights_out != nullptr;
#define KVB_FEW(NT)                                                    \
  do {                                                                 \
    if (plan.waves == 8) {                                             \
      if (w) KVB_ATTN(attn8_kernel<D, B, CODE, NT, true, 8>);          \
      else KVB_ATTN(attn8_kernel<D, B, CODE, NT, false, 8>);           \
    } else {                                                           \
      if (w) KVB_ATTN(attn8_kernel<D, B, CODE, NT, true, 4>);          \
      else KVB_ATTN(attn8_kernel<D, B, CODE, NT, false, 4>);           \
    }                                                                  \
  } while (0)
  if (plan.tile_rows == 16) {
    KVB_FEW(1);
  } else if (plan.tile_rows == 32) {
    KVB_FEW(2);
  } else {
    if (w) KVB_ATTN(attn8_tile_kernel<D, B, CODE, true>);
    else KVB_ATTN(attn8_tile_kernel<D, B, CODE, false>);
  }
#undef KVB_FEW
#undef KVB_ATTN
}

template <int D, int CODE>
void launch_kernels(const Attn8Plan& plan, const Attn8& a, int block_len, float* po, float* ml,
                    float* parts, hipStream_t s) {
  if (block_len == 16) launch_kernels<D, 16, CODE>(plan, a, po, ml, parts, s);
  else if (block_len == 32) launch_kernels<D, 32, CODE>(plan, a, po, ml, parts, s);
  else if (block_len == 64) launch_kernels<D, 64, CODE>(plan, a, po, ml, parts, s);
  else launch_kernels<D, 128, CODE>(plan, a, po, ml, parts, s);
}

}  // namespace
}  // namespace kvb
