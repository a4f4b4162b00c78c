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

// One row's result: x / sum in bfloat16, and the log of the sum.
__device__ __forceinline__ void write_row(const Attn8& a, int q, int head, int D, int c, f4_t x,
                                          float top, float sum) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t r = (int64_t)q * a.n_q_heads + head;
  *reinterpret_cast<uint2*>(a.out + r * D + c) =
      make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
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
  const uint16_t* qrow[NT];
  float m[NT], l[NT];
  f4_t o[NT][CT];
  int vexp;
  float* part[NT];  // the row's place in the weights of part 0
  int part_step;
  int n_parts;  // the parts below this are written

  // Queries: a power of two brings each row's largest value into [0.5, 1), so that fp16 holds
  // a bfloat16 of the row exactly (below 2^-14 of the largest: to 2^-25 of it).
  __device__ __forceinline__ void start(const Attn8& a, const Seq& sq, int h, int G, int row0,
                                        int grp, int col) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = row0 + n * 16 + col, i = (int)((unsigned)r / (unsigned)G);
      const bool ok = i < sq.n_q;  // a row past the last one reads the first one and sees nothing
      qrow[n] = a.q + ((int64_t)(sq.q0 + (ok ? i : 0)) * a.n_q_heads + h * G + (ok ? r - i * G : 0)) * D;
      see[n] = ok ? seen_by(sq, i) : 0;
      uint4 w[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k)
        w[k] = *reinterpret_cast<const uint4*>(qrow[n] + 64 * (k / 2) + 16 * grp + 8 * (k % 2));
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
      m[n] = kNoMax, l[n] = 0.f;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[n][c] = (f4_t){0.f, 0.f, 0.f, 0.f};
    }
    vexp = -127;
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

  // scores (log2 units) -> probabilities of the step; running maximum, sums and the part's
  // weight follow.  key: the first of this lane's 16.
  __device__ __forceinline__ void soften(int n, float (&s)[16], int key, int grp) {
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
  // log2 of the weight of part p
  __device__ __forceinline__ void put_part(int n, int p, float x) {
    if (part[n] && p < n_parts) part[n][(int64_t)p * part_step] = x;
  }
};

template <int D, int B, int CODE, int NT, bool WEIGHTS>
__global__ void __launch_bounds__(64 * kWaves, 2)
attn8_kernel(Attn8 a, Attn8Plan plan, float* __restrict__ po, float* __restrict__ ml,
             float* __restrict__ parts) {
  typedef Rows<D, B, NT, WEIGHTS> R;
  constexpr int KS = R::KS, CT = R::CT;
  constexpr int KP = D / 64;              // 16-byte pieces of a lane's key
  constexpr int CHUNK = B < 64 ? B : 64;  // steps whose blocks' ids and scales a wave holds
  constexpr bool ONE = B >= 64;           // a step lies in one block
  constexpr int LDO = D + 4;
  __shared__ __align__(16) float part_o[kWaves][16 * NT][LDO];
  __shared__ float part_ml[kWaves][16 * NT][2];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int grp = lane >> 4, col = lane & 15;
  const int z = blockIdx.z, split = blockIdx.x;
  const int b = z / a.c.n_kv_heads, h = z - b * a.c.n_kv_heads;
  const int G = plan.group;
  const int row0 = blockIdx.y * (16 * NT);
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
  if (split == plan.n_splits - 1 && wave == kWaves - 1) hi = steps;

  R r;
  r.start(a, sq, h, G, row0, grp, col);
  if constexpr (WEIGHTS) {
    // parts of the full blocks; the tail's are its own wave's to write
    r.part_step = plan.rows, r.n_parts = sq.full * (B / R::PB);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = row0 + n * 16 + col;
      r.part[n] = row < plan.rows ? parts + (int64_t)z * plan.n_parts * plan.rows + row : nullptr;
    }
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
    float big = vs;
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) big = fmaxf(big, __shfl_xor(big, x, 64));
    big = max4groups(big);
    if (big > 0.f) {
      const int e = max(__builtin_amdgcn_frexp_expf(big), -100);
      if (e > r.vexp) r.unit(e);
    }
    const float vw = __builtin_ldexpf(vs, kScaleTop - r.vexp);

#pragma unroll 1
    for (int st = c0; st < c1; ++st) {
      const int key0 = st * 64;
      const int gb = ONE ? st / (B / 64) - blk0 : st * (64 / B) + grp / (B / 16) - blk0;
      const bool have = found >> gb & 1;
      float ksg, vwg;
      if constexpr (ONE) {
        ksg = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks), gb));
        vwg = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vw), gb));
      } else {
        ksg = __shfl(ks, gb, 64), vwg = __shfl(vw, gb, 64);
      }
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
      bool clear = have;
#pragma unroll
      for (int n = 0; n < NT; ++n) clear = clear && r.see[n] >= key0 + 64;
      const bool plain = __all(clear);  // every key of the step is seen by every row
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float f = ksg * r.cq[n];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] *= f;
        const int left = have ? r.see[n] - (key0 + 16 * grp) : 0;  // visible of the lane's 16 keys
        if (!plain) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[n][i] = i < left ? s[n][i] : -INFINITY;
        }
        r.soften(n, s[n], key0 + 16 * grp, grp);
        const float w = left > 0 ? vwg : 0.f;  // a row that sees none of a NaN block stays clean
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          half2_t x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f2_t v = {s[n][8 * j + 2 * e] * w, s[n][8 * j + 2 * e + 1] * w};
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
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pr[n][0], r.o[n][c], 0, 0, 0);
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pr[n][1], r.o[n][c], 0, 0, 0);
        }
      }
      if (st + 1 < c1) load_v(st + 1);
    }
  }

  // The tail: bfloat16 rows, one step of 64 keys for each of the first split's last waves (a block
  // has at most two).  Probabilities enter as the sum of two bfloat16, in the same unit; rows past
  // the tail's end hold anything, so their values of V are cleared.
  const int r0 = (kWaves - 1 - wave) * 64;
  const int t0 = sq.full * B + r0;
  if (split == 0 && r0 < B && t0 < seen_by(sq, min(last, sq.n_q - 1))) {
    const int rows = min(64, sq.len - t0);  // tail rows of this step
    if constexpr (WEIGHTS) r.n_parts += B / R::PB;
    if (r.vexp < kScaleTop) r.unit(kScaleTop);  // 1 at least: the sums fit a float if the outputs do
    const uint16_t* kt = a.c.k_tail + (int64_t)z * B * D;
    const uint16_t* vt = a.c.v_tail + (int64_t)z * B * D;
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
          const bf8_t y = *reinterpret_cast<const bf8_t*>(r.qrow[n] + k * 32 + grp * 8);
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
      const int left = r.see[n] - (t0 + 16 * grp);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = i < left ? s[n][i] * f : -INFINITY;
      r.soften(n, s[n], t0 + 16 * grp, grp);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_ldexpf(s[n][8 * j + e], kScaleTop - r.vexp);
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
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ph[n][j], r.o[n][c], 0, 0, 0);
          r.o[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pl[n][j], r.o[n][c], 0, 0, 0);
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
              if (bad && t0 + u < r.see[n]) r.o[n][c][i] += __uint_as_float(bits << 16);
          }
      }
    }
  }

  // the waves meet
  const float unit = __builtin_ldexpf(1.f, r.vexp - kScaleTop);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    r.l[n] = sum4groups(r.l[n]);
    if (grp == 0) part_ml[wave][n * 16 + col][0] = r.m[n], part_ml[wave][n * 16 + col][1] = r.l[n];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      *reinterpret_cast<f4_t*>(&part_o[wave][n * 16 + col][c * 16 + grp * 4]) = r.o[n][c] * unit;
  }
  __syncthreads();
  constexpr int LPR = D / 4;  // lanes of a row
  const bool whole = plan.n_splits == 1;
#pragma unroll 1
  for (int p = threadIdx.x; p < 16 * NT * LPR; p += 64 * kWaves) {
    const int rr = p / LPR, c = p % LPR * 4;
    const int row = row0 + rr;
    if (row >= sq.n_q * G || row >= plan.rows) continue;
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

// splits of a row's tile that hold keys
template <int B>
__device__ __forceinline__ int splits_of(const Seq& sq, const Attn8Plan& plan, int row) {
  const int n = 16 * plan.col_tiles;
  const int last = (int)((unsigned)(row / n * n + n - 1) / (unsigned)plan.group);
  const int k = (steps_of<B>(sq, last) + plan.span - 1) / plan.span;
  return max(1, min(k, plan.n_splits));
}

// Joins the splits of a row: one workgroup a row.  The sums of the splits are weighed first (a lane
// a split), then D / 4 lanes a split add their outputs, 256 / (D / 4) splits at a time, in an
// order that the sizes fix.
template <int D, int B>
__global__ void __launch_bounds__(256) attn8_join_kernel(Attn8 a, Attn8Plan plan,
                                                         const float* __restrict__ po,
                                                         const float* __restrict__ ml) {
  constexpr int LPR = D / 4, SG = 256 / LPR;  // lanes of a split's row, splits at a time
  __shared__ float weight[256], wave_top[4], wave_sum[4];
  __shared__ f4_t sums[SG][LPR];
  const int z = blockIdx.y, row = blockIdx.x, tid = threadIdx.x;
  const int b = z / a.c.n_kv_heads, h = z - b * a.c.n_kv_heads;
  const Seq sq = seq_of<B>(a, b);
  if (row >= sq.n_q * plan.group) return;
  const int n = splits_of<B>(sq, plan, row);  // at most 256
  const int64_t rec = (int64_t)z * plan.n_splits * plan.rows + row;
  float m = kNoMax, l = 0.f;
  if (tid < n) {
    const float2 x = *reinterpret_cast<const float2*>(ml + 2 * (rec + (int64_t)tid * plan.rows));
    m = x.x, l = x.y;
  }
  float top = m;
  for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
  if ((tid & 63) == 0) wave_top[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
  const float f = tid < n ? __builtin_amdgcn_exp2f(m - top) : 0.f;
  weight[tid] = f;
  float sum = f * l;
  for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k, 64);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
  __syncthreads();
  sum = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
  const int sg = tid / LPR, c = tid % LPR;
  f4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = sg; s < n; s += SG)
    x += weight[s] * *reinterpret_cast<const f4_t*>(po + (rec + (int64_t)s * plan.rows) * D + c * 4);
  sums[sg][c] = x;
  __syncthreads();
  if (tid >= LPR) return;
  for (int s = 1; s < SG; ++s) x += sums[s][c];
  const int i = (int)((unsigned)row / (unsigned)plan.group);
  write_row(a, sq.q0 + i, h * plan.group + row - i * plan.group, D, c * 4, x, top, sum);
}

// Accumulated weights: 16 lanes a block, each over every 16th row; the rows' log2 sums come
// through LDS, 256 rows at a time.
template <int B>
__global__ void __launch_bounds__(256) attn8_weights_kernel(Attn8 a, Attn8Plan plan,
                                                            const float* __restrict__ ml,
                                                            const float* __restrict__ parts) {
  constexpr int PB = B < 64 ? B : 64, PER = B / PB;
  __shared__ float total[256];  // log2 of a row's sum
  const int z = blockIdx.y, b = z / a.c.n_kv_heads;
  const int M = a.c.max_blocks;
  const Seq sq = seq_of<B>(a, b);
  const int blk = blockIdx.x * 16 + threadIdx.x / 16;
  const int rows = min(sq.n_q * plan.group, plan.rows);
  float sum = 0.f;
  for (int r0 = 0; r0 < rows; r0 += 256) {
    __syncthreads();
    const int r = r0 + threadIdx.x;
    if (r < rows) {
      const int n = splits_of<B>(sq, plan, r);
      const int64_t rec = (int64_t)z * plan.n_splits * plan.rows + r;
      float top = kNoMax, t = 0.f;
#pragma unroll 4
      for (int s = 0; s < n; ++s) top = fmaxf(top, ml[2 * (rec + (int64_t)s * plan.rows)]);
#pragma unroll 4
      for (int s = 0; s < n; ++s) {
        const int64_t at = 2 * (rec + (int64_t)s * plan.rows);
        t += __builtin_amdgcn_exp2f(ml[at] - top) * ml[at + 1];
      }
      total[threadIdx.x] = t == 0.f ? INFINITY : top + log2f(t);  // nothing seen: no share
    }
    __syncthreads();
    for (int x = r0 + threadIdx.x % 16; x < min(rows, r0 + 256); x += 16) {
      const int see = seen_by(sq, (int)((unsigned)x / (unsigned)plan.group));
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        const int part = blk * PER + p;
        if (blk < M && part < (see + PB - 1) / PB)
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
  p.rows = max_queries * (n_q_heads / n_kv_heads);
  p.col_tiles = p.rows <= 16 ? 1 : 2;
  p.n_tiles = (int)((p.rows + 16 * p.col_tiles - 1) / (16 * p.col_tiles));
  const int64_t heads = (int64_t)n_seqs * n_kv_heads, base = heads * p.n_tiles;
  const int64_t steps = ((int64_t)max_len + 63) / 64;
  // enough workgroups to fill 256 CUs twice, each with two steps a wave at least
  int64_t want = (512 + base - 1) / base, most = steps / (2 * kWaves);
  if (want > most) want = most;
  if (want < 1) want = 1;
  if (want > 256) want = 256;  // what the join takes
  p.span = (int)((steps + want - 1) / want);
  p.wave_span = (p.span + kWaves - 1) / kWaves;
  p.n_splits = (int)((steps + p.span - 1) / p.span);
  p.group = n_q_heads / n_kv_heads;
  const int pb = block_len < 64 ? block_len : 64;
  p.n_parts = with_weights ? (max_blocks + 1) * (block_len / pb) : 0;
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
#define KVB_FOR_B(F)               \
  do {                             \
    if (block_len == 16) F(16);    \
    else if (block_len == 32) F(32); \
    else if (block_len == 64) F(64); \
    else F(128);                   \
  } while (0)
  if (plan.n_splits > 1) {
    const dim3 jg((unsigned)plan.rows, heads);
#define KVB_JOIN(B)                                                                             \
  do {                                                                                          \
    if (head_dim == 128)                                                                        \
      hipLaunchKernelGGL((attn8_join_kernel<128, B>), jg, dim3(256), 0, s, a, plan, po, ml);    \
    else                                                                                        \
      hipLaunchKernelGGL((attn8_join_kernel<64, B>), jg, dim3(256), 0, s, a, plan, po, ml);     \
  } while (0)
    KVB_FOR_B(KVB_JOIN);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (a.weights_out) {
    const dim3 wg((unsigned)((a.c.max_blocks + 15) / 16), heads);
#define KVB_WEIGHTS(B) \
  hipLaunchKernelGGL(attn8_weights_kernel<B>, wg, dim3(256), 0, s, a, plan, ml, parts)
    KVB_FOR_B(KVB_WEIGHTS);
  }
  return hipGetLastError();
}

}  // namespace kvb
