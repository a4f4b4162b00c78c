// The 8-bit cache: rows in (kvb_cache8_append), rows out (kvb_cache8_read) and the
// eviction of blocks (kvb_cache8_evict).
//
// Append and read stream: bfloat16 in, one byte out (or the reverse), HBM-bound.
// A workgroup takes one block of one (layer, sequence, kv head) and one of K and V.
// It holds the block in registers between the maximum and the codes, so rows are
// read once.  V is turned in registers and LDS, because its blocks are channel-major.
#include "kvb_device.h"
#include "kvb_internal.h"

namespace kvb {
namespace {

// The tokens [first, first + n) of a sequence that a call adds or reads, and the
// blocks they touch.
struct Span {
  int64_t before;  // tokens before the call's rows
  int64_t end;     // tokens after the last of them
  int64_t j0;      // first block touched
  int32_t blocks;  // blocks touched, 0: nothing to do
};
__device__ __forceinline__ Span span_of(const int32_t* cu, const int32_t* lens, int b, int B) {
  Span s;
  const int64_t n = (int64_t)cu[b + 1] - cu[b];
  s.end = lens[b];
  s.before = s.end - n;
  s.j0 = s.before / B;
  s.blocks = n > 0 && s.before >= 0 ? (int32_t)((s.end - 1) / B - s.j0 + 1) : 0;
  return s;
}

// ---- codes ----------------------------------------------------------------

// The scale of a block from its largest magnitude (bf16 bits; 0x7F80 and above: an
// infinity or NaN) and what a value is multiplied with on the way to its code.  The
// quotients of a block whose scale may be subnormal are formed at 2^64 times the size (lift).
struct Scale {
  float scale, lift, s, inv;  // stored; the size; scale * lift; about 1 / s
  int shift;                  // e4m3: code value = x * 2^shift
};
template <int CODE>
__device__ __forceinline__ Scale scale_of(uint32_t amax_bits) {
  Scale r;
  const float amax = __uint_as_float(amax_bits << 16);
  r.lift = 1.f, r.s = 1.f, r.inv = 0.f, r.shift = 0;
  if (amax_bits == 0) {
    r.scale = 0.f;
  } else if (amax_bits >= 0x7F80u) {
    r.scale = __builtin_nanf("");
  } else if constexpr (CODE == KVB_I8) {
    r.scale = amax / 127.0f;
    r.lift = amax < 0x1p-60f ? 0x1p64f : 1.f;
    r.s = r.scale * r.lift;
    r.inv = 1.f / r.s;
  } else {
    const float m = __builtin_amdgcn_frexp_mantf(amax);  // [0.5, 1)
    const int e = __builtin_amdgcn_frexp_expf(amax) - (m <= 0.875f ? 9 : 8);
    r.scale = __builtin_ldexpf(1.f, e);
    r.shift = -e;
  }
  return r;
}

// codes of 8 values, 4 to a word.
// int8: rint(x / scale) of the exact quotient; never past 127, because amax / scale is not.  Adding
// 1.5 * 2^23 rounds to nearest even and leaves the code in the low byte.  t carries two roundings of
// at most 2^-24 of 128, so the code can only be wrong within 2e-5 of a half; there the remainder
// decides: x - c s is exact in one fused operation (both are multiples of the smaller one's last
// bit, and the difference is small).  One branch for the eight, taken by 3 % of the waves.
// e4m3: an exact product with a power of two, then one rounding to nearest even.
template <int CODE>
__device__ __forceinline__ uint2 codes8(const float* x, const Scale& r) {
  if constexpr (CODE == KVB_I8) {
    constexpr float shift = 12582912.f;
    float c[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = x[e] * r.inv;
      c[e] = t + shift;
      far = fmaxf(far, fabsf(t - (c[e] - shift)));
    }
    if (__builtin_expect(far > 0.49997f, 0)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = c[e] - shift, rest = __builtin_fmaf(-n, r.s, x[e]);
        const float over = fabsf(rest) - 0.5f * r.s;  // 0: half way, where the odd code moves
        const float step = __builtin_copysignf(1.f, rest);
        c[e] += over > 0.f || (over == 0.f && (__float_as_uint(c[e]) & 1)) ? step : 0.f;
      }
    }
    uint32_t w[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(c[4 * q + 1]), __float_as_uint(c[4 * q]), 0x0C0C0400u);
      const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(c[4 * q + 3]), __float_as_uint(c[4 * q + 2]), 0x0C0C0400u);
      w[q] = hi << 16 | lo;
    }
    return make_uint2(w[0], w[1]);
  } else {
    uint32_t w[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      int y = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(x[4 * q], r.shift),
                                              __builtin_ldexpf(x[4 * q + 1], r.shift), 0, false);
      w[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_ldexpf(x[4 * q + 2], r.shift),
                                                       __builtin_ldexpf(x[4 * q + 3], r.shift), y, true);
    }
    return make_uint2(w[0], w[1]);
  }
}

// the values of the 4 codes of a word, as code * scale
template <int CODE>
__device__ __forceinline__ void values4(uint32_t w, float scale, float* x) {
  if constexpr (CODE == KVB_I8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i)) * scale;
  } else {
    typedef __attribute__((ext_vector_type(2))) float f2;
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0] * scale, x[1] = a[1] * scale, x[2] = b[0] * scale, x[3] = b[1] * scale;
  }
}

// bytes of 4 words, transposed: byte i of out[j] is byte j of in[i]
__device__ __forceinline__ void turn4(const uint32_t* in, uint32_t* out) {
  const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u);  // in0.0 in1.0 in0.1 in1.1
  const uint32_t b = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u);
  const uint32_t c = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);  // in0.2 in1.2 in0.3 in1.3
  const uint32_t d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// How a workgroup takes a block of B tokens x D channels: a thread owns quads of 4 tokens x 8
// channels, so that the codes of a quad turn into words of 4 tokens in registers and V passes
// through LDS by words.
template <int D, int B>
struct Quads {
  static constexpr int PPR = D / 8;                          // quads across a row
  static constexpr int ALL = PPR * B / 4;
  static constexpr int THREADS = ALL < 64 ? 64 : ALL > 256 ? 256 : ALL;
  static constexpr int N = ALL > THREADS ? ALL / THREADS : 1;  // quads of a thread
  static constexpr int LDT = B + 4;                          // row of the transposed codes in LDS, bytes
};

constexpr int kRowsY = 32768;  // grid rows (K and V of table rows) in y, the others in z

// ---- append ---------------------------------------------------------------

// 16-bit numbers of 2 words of 4 rows, turned: word w of the rows -> words of the 4 rows' low halves
// (lo) and high halves (hi)
__device__ __forceinline__ void turn4x2(const uint32_t* in, uint2& lo, uint2& hi) {
  lo = make_uint2(__builtin_amdgcn_perm(in[1], in[0], 0x05040100u), __builtin_amdgcn_perm(in[3], in[2], 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(in[1], in[0], 0x07060302u), __builtin_amdgcn_perm(in[3], in[2], 0x07060302u));
}
__device__ __forceinline__ uint32_t word_of(const uint4& x, int w) {
  return w == 0 ? x.x : w == 1 ? x.y : w == 2 ? x.z : x.w;
}

// The tail rows [from, to) of a block from the new rows (`rows`: row `from`).  V: a thread takes 4
// tokens x 8 channels, neighbouring lanes neighbouring tokens, so that a wave's stores are runs of
// a channel (one token a thread stored single numbers 2 B apart: 40 us of the 206 above).
template <int D, int B>
__device__ __forceinline__ void write_tail(int is_v, uint16_t* tail, const uint16_t* rows,
                                           int64_t token_stride, int from, int to) {
  constexpr int PPR = D / 8;  // 16-byte pieces of a row
  if (!is_v) {
    for (int i = threadIdx.x; i < (to - from) * PPR; i += blockDim.x) {
      const int u = i / PPR, c = i % PPR * 8;
      *reinterpret_cast<uint4*>(tail + (from + u) * D + c) =
          *reinterpret_cast<const uint4*>(rows + (int64_t)u * token_stride + c);
    }
    return;
  }
  const int q0 = from / 4, quads = (to + 3) / 4 - q0;
  for (int i = threadIdx.x; i < quads * PPR; i += blockDim.x) {
    const int u = (q0 + i % quads) * 4, c = i / quads * 8;
    uint4 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = min(max(u + e, from), to - 1);
      x[e] = *reinterpret_cast<const uint4*>(rows + (int64_t)(t - from) * token_stride + c);
    }
    const bool whole = u >= from && u + 4 <= to;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t in[4] = {word_of(x[0], w), word_of(x[1], w), word_of(x[2], w), word_of(x[3], w)};
      uint2 y[2];
      turn4x2(in, y[0], y[1]);
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        uint16_t* at = tail + (c + 2 * w + z) * B + u;
        if (whole) {
          *reinterpret_cast<uint2*>(at) = y[z];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (u + e >= from && u + e < to) at[e] = (uint16_t)((e < 2 ? y[z].x : y[z].y) >> (16 * (e & 1)));
        }
      }
    }
  }
}

template <int D, int B, int CODE>
__global__ void __launch_bounds__((Quads<D, B>::THREADS))
append_kernel(Cache8 c, const int32_t* __restrict__ cu, const uint16_t* __restrict__ k,
              const uint16_t* __restrict__ v, int64_t layer_stride, int64_t token_stride,
              int64_t head_stride) {
  typedef Quads<D, B> Q;
  constexpr int WAVES = Q::THREADS / 64;
  __shared__ uint32_t wave_max[WAVES];
  __shared__ __align__(16) uint8_t turned[D * Q::LDT];
  const int row = (int)(blockIdx.y + blockIdx.z * kRowsY) >> 1, is_v = blockIdx.y & 1;  // row: (layer, sequence, kv head)
  if (row >= c.n_rows) return;
  const int b = row / c.n_kv_heads % c.n_seqs;
  const Span sp = span_of(cu, c.lens, b, B);
  const int64_t l = row / c.n_kv_heads / c.n_seqs, h = row % c.n_kv_heads;
  const uint16_t* src = (is_v ? v : k) + l * layer_stride + h * head_stride + (int64_t)cu[b] * token_stride;
  uint16_t* tail = (is_v ? c.v_tail : c.k_tail) + (int64_t)row * B * D;
  // tokens of the last block, when it is not full and not past the table
  const int rest = sp.end / B <= c.max_blocks ? (int)(sp.end % B) : 0;
  const bool old = sp.before % B != 0, moves = old && rest != 0 && sp.blocks > 1;
  for (int i = blockIdx.x; i < sp.blocks; i += gridDim.x) {
    const int64_t j = sp.j0 + i, t0 = j * B;
    if (t0 + B <= sp.end) {
      const int32_t id = j < c.max_blocks ? c.table[(int64_t)row * c.max_blocks + j] : -1;
      uint4 x[Q::N][4];  // asked for before the id is known
      const uint16_t* first = src + (t0 - sp.before) * token_stride;  // of the block's token 0
#pragma unroll
      for (int n = 0; n < Q::N; ++n) {
        const int p = threadIdx.x + n * Q::THREADS, cc = p % Q::PPR * 8, u = p / Q::PPR * 4;
        if (Q::ALL < Q::THREADS && p >= Q::ALL) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] = make_uint4(0, 0, 0, 0);
        } else if (t0 >= sp.before) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[n][e] = *reinterpret_cast<const uint4*>(first + (u + e) * token_stride + cc);
        } else {
          for (int e = 0; e < 4; ++e) {
            uint4 y;
            if (t0 + u + e >= sp.before) {
              y = *reinterpret_cast<const uint4*>(first + (u + e) * token_stride + cc);
            } else if (!is_v) {
              y = *reinterpret_cast<const uint4*>(tail + (u + e) * D + cc);
            } else {
              const uint16_t* t = tail + cc * B + u + e;
              y = make_uint4(t[0] | (uint32_t)t[B] << 16, t[2 * B] | (uint32_t)t[3 * B] << 16,
                             t[4 * B] | (uint32_t)t[5 * B] << 16, t[6 * B] | (uint32_t)t[7 * B] << 16);
            }
            x[n][e] = y;
          }
        }
      }
      if (id >= 0 && id < c.n_blocks) {
        // the largest magnitude: bfloat16 bits without the sign order like the magnitudes
        typedef __attribute__((ext_vector_type(2))) uint16_t u2;
        u2 m2 = {0, 0};
#pragma unroll
        for (int n = 0; n < Q::N; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w[4] = {x[n][e].x, x[n][e].y, x[n][e].z, x[n][e].w};
#pragma unroll
            for (int q = 0; q < 4; ++q)
              m2 = __builtin_elementwise_max(m2, __builtin_bit_cast(u2, w[q] & 0x7FFF7FFFu));
          }
        uint32_t mx = m2[0] > m2[1] ? m2[0] : m2[1];
        for (int m = 32; m > 0; m >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, m, 64));
        if constexpr (WAVES > 1) {
          if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = mx;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < WAVES; ++w) mx = max(mx, wave_max[w]);
        }
        const Scale sc = scale_of<CODE>(mx);
        if (threadIdx.x == 0) (is_v ? c.v_scale : c.k_scale)[id] = sc.scale;
        const bool none = mx == 0 || mx >= 0x7F80u;  // every code 0
#pragma unroll
        for (int n = 0; n < Q::N; ++n) {
          const int p = threadIdx.x + n * Q::THREADS, cc = p % Q::PPR * 8, u = p / Q::PPR * 4;
          if (Q::ALL < Q::THREADS && p >= Q::ALL) continue;
          uint32_t q[2][4];  // words of 4 channels, a token each
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w[4] = {x[n][e].x, x[n][e].y, x[n][e].z, x[n][e].w};
            float f[8];
#pragma unroll
            for (int y = 0; y < 4; ++y) f[2 * y] = bf16_lo(w[y]), f[2 * y + 1] = bf16_hi(w[y]);
            if (sc.lift != 1.f) {
#pragma unroll
              for (int y = 0; y < 8; ++y) f[y] *= sc.lift;
            }
            const uint2 code = none ? make_uint2(0, 0) : codes8<CODE>(f, sc);
            q[0][e] = code.x, q[1][e] = code.y;
            if (!is_v) *reinterpret_cast<uint2*>(c.k_codes + (int64_t)id * B * D + (u + e) * D + cc) = code;
          }
          if (is_v) {
            uint32_t y[8];  // words of 4 tokens, a channel each
            turn4(q[0], y);
            turn4(q[1], y + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<uint32_t*>(turned + (cc + e) * Q::LDT + u) = y[e];
          }
        }
        __syncthreads();  // the codes are in LDS, wave_max and the old tail have been read
        if (is_v) {
          uint8_t* dst = c.v_codes + (int64_t)id * B * D;
          for (int p = threadIdx.x; p < D * B / 16; p += Q::THREADS) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(turned + p / (B / 16) * Q::LDT + p % (B / 16) * 16);
            *reinterpret_cast<uint4*>(dst + p * 16) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          __syncthreads();
        }
      }
      // the workgroup that read the old tail is the one that may write the new one
      if (i == 0 && moves) {
        __syncthreads();
        write_tail<D, B>(is_v, tail, src + (sp.end - rest - sp.before) * token_stride, token_stride, 0, rest);
      }
    } else if (rest != 0 && !(moves && i > 0)) {
      const int from = (int)(sp.before > t0 ? sp.before - t0 : 0);
      write_tail<D, B>(is_v, tail, src + (t0 + from - sp.before) * token_stride, token_stride, from, rest);
    }
  }
}

// ---- read -----------------------------------------------------------------

__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                            pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// 8 bfloat16 as they are
__device__ __forceinline__ void store8(uint16_t* p, const uint4& x) { *reinterpret_cast<uint4*>(p) = x; }
__device__ __forceinline__ void store8(float* p, const uint4& x) {
  const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                      bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w)};
  store8(p, f);
}

template <int D, int B, int CODE, typename T>
__global__ void __launch_bounds__((Quads<D, B>::THREADS))
read_kernel(Cache8 c, const int32_t* __restrict__ cu, T* __restrict__ k, T* __restrict__ v,
            int64_t layer_stride, int64_t token_stride, int64_t head_stride) {
  typedef Quads<D, B> Q;
  __shared__ __align__(16) uint8_t turned[D * Q::LDT];
  const int row = (int)(blockIdx.y + blockIdx.z * kRowsY) >> 1, is_v = blockIdx.y & 1;
  if (row >= c.n_rows) return;
  const int b = row / c.n_kv_heads % c.n_seqs;
  const Span sp = span_of(cu, c.lens, b, B);
  const int64_t l = row / c.n_kv_heads / c.n_seqs, h = row % c.n_kv_heads;
  T* dst = (is_v ? v : k) + l * layer_stride + h * head_stride + (int64_t)cu[b] * token_stride;
  const uint16_t* tail = (is_v ? c.v_tail : c.k_tail) + (int64_t)row * B * D;
  for (int i = blockIdx.x; i < sp.blocks; i += gridDim.x) {
    const int64_t j = sp.j0 + i, t0 = j * B;
    const int from = (int)(sp.before > t0 ? sp.before - t0 : 0);
    const int to = (int)(sp.end - t0 < B ? sp.end - t0 : B);
    T* out = dst + (t0 - sp.before) * token_stride;
    if (t0 + B <= sp.end) {
      const int32_t id = j < c.max_blocks ? c.table[(int64_t)row * c.max_blocks + j] : -1;
      if (id < 0 || id >= c.n_blocks) continue;
      const float scale = (is_v ? c.v_scale : c.k_scale)[id];
      const uint8_t* codes = (is_v ? c.v_codes : c.k_codes) + (int64_t)id * B * D;
      uint2 x[Q::N][4];  // 8 channels of 4 tokens
      if (!is_v) {
#pragma unroll
        for (int n = 0; n < Q::N; ++n) {
          const int p = threadIdx.x + n * Q::THREADS, cc = p % Q::PPR * 8, u = p / Q::PPR * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (Q::ALL >= Q::THREADS || p < Q::ALL)
              x[n][e] = *reinterpret_cast<const uint2*>(codes + (u + e) * D + cc);
        }
      } else {
        __syncthreads();  // the previous block has been read
        for (int p = threadIdx.x; p < D * B / 16; p += Q::THREADS) {
          const uint4 q = *reinterpret_cast<const uint4*>(codes + p * 16);
          uint32_t* w = reinterpret_cast<uint32_t*>(turned + p / (B / 16) * Q::LDT + p % (B / 16) * 16);
          w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < Q::N; ++n) {
          const int p = threadIdx.x + n * Q::THREADS, cc = p % Q::PPR * 8, u = p / Q::PPR * 4;
          if (Q::ALL < Q::THREADS && p >= Q::ALL) continue;
          uint32_t y[8], q[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = *reinterpret_cast<const uint32_t*>(turned + (cc + e) * Q::LDT + u);
          turn4(y, q);
          turn4(y + 4, q + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] = make_uint2(q[e], q[4 + e]);
        }
      }
#pragma unroll
      for (int n = 0; n < Q::N; ++n) {
        const int p = threadIdx.x + n * Q::THREADS, cc = p % Q::PPR * 8, u = p / Q::PPR * 4;
        if (Q::ALL < Q::THREADS && p >= Q::ALL) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float f[8];
          values4<CODE>(x[n][e].x, scale, f);
          values4<CODE>(x[n][e].y, scale, f + 4);
          if (u + e >= from) store8(out + (u + e) * token_stride + cc, f);
        }
      }
    } else if (j <= c.max_blocks) {
      if (!is_v) {
        for (int p = threadIdx.x + from * Q::PPR; p < to * Q::PPR; p += Q::THREADS) {
          const int u = p / Q::PPR, cc = p % Q::PPR * 8;
          store8(out + (int64_t)u * token_stride + cc, *reinterpret_cast<const uint4*>(tail + u * D + cc));
        }
      } else {  // as write_tail, the other way
        const int q0 = from / 4, quads = (to + 3) / 4 - q0;
        for (int p = threadIdx.x; p < quads * Q::PPR; p += Q::THREADS) {
          const int u = (q0 + p % quads) * 4, cc = p / quads * 8;
          uint2 y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = *reinterpret_cast<const uint2*>(tail + (cc + e) * B + u);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
              w[q] = __builtin_amdgcn_perm(e < 2 ? y[2 * q + 1].x : y[2 * q + 1].y, e < 2 ? y[2 * q].x : y[2 * q].y,
                                           e & 1 ? 0x07060302u : 0x05040100u);
            if (u + e >= from && u + e < to)
              store8(out + (int64_t)(u + e) * token_stride + cc, make_uint4(w[0], w[1], w[2], w[3]));
          }
        }
      }
    }
  }
}

// ---- evict ----------------------------------------------------------------

// float -> unsigned key of the same order: NaN lowest, -0 equal to +0
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// What a table row keeps: nb full blocks of M entries, `drop` of them leave; the k best of the
// blocks [lo, hi) stay, and all others below nb.
struct Row {
  int nb, drop, lo, hi, k;
};
__device__ __forceinline__ Row row_of(const Evict& a, int b) {
  Row r;
  const int len = max(a.lens[b], 0);
  r.nb = min(len / a.block_len, a.max_blocks);
  r.drop = r.nb > a.budget ? r.nb - a.budget : 0;
  r.lo = a.n_first, r.hi = r.nb - a.n_recent;
  r.k = a.budget - a.n_first - a.n_recent;
  return r;
}

// A wave a row of up to 64 * N entries, all in registers (lane i: entries i, i + 64, ..), so the row
// is read once and nothing waits for another wave.  The k-th largest key is found bit by bit: a
// key set's count is a ballot's population count, and the search ends when it is k.
// (18432 rows of 902 entries, 266 MB: 329 us with a workgroup a row and counts of digits in LDS.)
template <int N>
__global__ void __launch_bounds__(256) evict_wave_kernel(Evict a, int64_t rows) {
  const int lane = threadIdx.x & 63;
  const int64_t row = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (row >= rows) return;
  const int b = (int)((uint32_t)row / (uint32_t)a.n_kv_heads % (uint32_t)a.n_seqs);
  const int M = a.max_blocks;
  const int32_t* table = a.table + row * M;
  const float* weights = a.weights + row * M;
  int32_t* table_out = a.table_out + row * M;
  float* weights_out = a.weights_out + row * M;
  int32_t t[N];
  float w[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = min(j * 64 + lane, M - 1);
    t[j] = table[i];
    w[j] = weights[i];
  }
  const Row r = row_of(a, b);
  if (row < (int64_t)a.n_seqs * a.n_kv_heads && row % a.n_kv_heads == 0 && lane == 0)
    a.lens_out[b] = a.lens[b] - r.drop * a.block_len;
  // the k-th largest key of the competing blocks; the others have key 0, and every candidate is larger
  uint32_t key[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = j * 64 + lane;
    key[j] = i >= r.lo && i < r.hi ? order_key(w[j]) : 0u;
  }
  uint32_t kth = 0;
  int left = 0x7FFFFFFF;  // of the keys equal to kth, this many are kept
  if (r.drop > 0 && r.k > 0) {
    int found = 0;
    for (uint32_t bit = 0x80000000u; bit != 0 && found != r.k; bit >>= 1) {
      const uint32_t candidate = kth | bit;
      int n = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) n += __popcll(__ballot(key[j] >= candidate));
      if (n >= r.k) kth = candidate, found = n;
    }
    if (found != r.k) {  // equal keys on both sides of the cut: the lower indices stay
      int n = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) n += __popcll(__ballot(key[j] > kth));
      left = r.k - n;
    }
  }
  const uint64_t below = (1ull << lane) - 1;
  int kept = 0, ties = 0;  // before this register's entries
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = j * 64 + lane;
    const bool middle = i >= r.lo && i < r.hi;
    int to;
    float x = w[j];
    if (r.drop == 0) {
      to = i;
    } else {
      const bool tie = middle && r.k > 0 && key[j] == kth;
      const uint64_t tm = __ballot(tie);
      const bool keep = i < r.nb && (!middle || (r.k > 0 && (key[j] > kth || (tie && ties + __popcll(tm & below) < left))));
      const uint64_t km = __ballot(keep);
      const int before = kept + __popcll(km & below);
      to = i >= r.nb ? i - r.drop : keep ? before : M - r.drop + (i - before);
      if (!keep && i < r.nb) x = 0.f;
      kept += __popcll(km);
      ties += __popcll(tm);
    }
    if (i < M) table_out[to] = t[j], weights_out[to] = x;
  }
}

// One workgroup per table row of any length.  The k-th largest key of the middle blocks is found
// digit by digit (8 bits) from counts in LDS; the row is then written in order with the ranks of
// kept and dropped entries from ballots.  Counts decide, so the result does not depend on the
// order of the atomics.
constexpr int kEvictWaves = 16;
constexpr int64_t kEvictRows = 1 << 21;  // of a launch: a grid dimension holds less than 2^32 work items
__global__ void __launch_bounds__(64 * kEvictWaves) evict_kernel(Evict a, int first) {
  constexpr int T = 64 * kEvictWaves;
  __shared__ int32_t bins[256], wave_kept[kEvictWaves], wave_ties[kEvictWaves];
  __shared__ uint32_t s_prefix;
  __shared__ int32_t s_left;
  const int64_t row = first + blockIdx.x;
  const int b = (int)((uint32_t)row / (uint32_t)a.n_kv_heads % (uint32_t)a.n_seqs);
  const int M = a.max_blocks, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int32_t* table = a.table + row * M;
  const float* weights = a.weights + row * M;
  int32_t* table_out = a.table_out + row * M;
  float* weights_out = a.weights_out + row * M;
  const Row r = row_of(a, b);
  if (row < (int64_t)a.n_seqs * a.n_kv_heads && row % a.n_kv_heads == 0 && tid == 0)
    a.lens_out[b] = a.lens[b] - r.drop * a.block_len;
  if (r.drop == 0) {
    for (int i = tid; i < M; i += T) table_out[i] = table[i], weights_out[i] = weights[i];
    return;
  }
  uint32_t prefix = 0;
  int left = r.k;  // of the keys that start with prefix, the `left` largest are kept
  if (r.k > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) bins[tid] = 0;
      __syncthreads();
      for (int i = r.lo + tid; i < r.hi; i += T) {
        const uint32_t key = order_key(weights[i]);
        if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8))
          atomicAdd(&bins[key >> shift & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {  // a lane four bins, the largest digits first
        int n[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += n[q] = bins[255 - 4 * lane - q];
        int upto = sum;  // keys in the bins of lanes 0 .. lane
        for (int x = 1; x < 64; x <<= 1) {
          const int y = __shfl_up(upto, x, 64);
          if (lane >= x) upto += y;
        }
        int above = upto - sum;
        if (above < left && upto >= left) {  // one lane: the digit is among its four
          int q = 0;
          while (above + n[q] < left) above += n[q++];
          s_prefix = prefix | (uint32_t)(255 - 4 * lane - q) << shift;
          s_left = left - above;
        }
      }
      __syncthreads();
      prefix = s_prefix;
      left = s_left;
    }
  }
  // kept: forced, above the k-th key, or among the first `left` equal to it
  int kept_before = 0, ties_before = 0;
  for (int base = 0; base < r.nb; base += T) {
    const int i = base + tid;
    const bool in = i < r.nb, middle = in && i >= r.lo && i < r.hi;
    const float w = in ? weights[i] : 0.f;
    const uint32_t key = order_key(w);
    const bool tie = middle && r.k > 0 && key == prefix;
    const uint64_t tm = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) wave_ties[wave] = __popcll(tm);
    __syncthreads();
    int ties = ties_before + __popcll(tm & below);
    for (int q = 0; q < kEvictWaves; ++q) {
      if (q < wave) ties += wave_ties[q];
      ties_before += wave_ties[q];
    }
    const bool keep = in && (!middle || (r.k > 0 && (key > prefix || (tie && ties < left))));
    const uint64_t km = __ballot(keep);
    if (lane == 0) wave_kept[wave] = __popcll(km);
    __syncthreads();
    int kept = kept_before + __popcll(km & below);
    for (int q = 0; q < kEvictWaves; ++q) {
      if (q < wave) kept += wave_kept[q];
      kept_before += wave_kept[q];
    }
    if (in) {
      const int to = keep ? kept : M - r.drop + (i - kept);
      table_out[to] = table[i];
      weights_out[to] = keep ? w : 0.f;
    }
    __syncthreads();
  }
  for (int i = r.nb + tid; i < M; i += T) {
    table_out[i - r.drop] = table[i];
    weights_out[i - r.drop] = weights[i];
  }
}

template <int D, int B>
void append(const Cache8& c, int code, dim3 grid, hipStream_t s, const int32_t* cu, const uint16_t* k,
            const uint16_t* v, int64_t ls, int64_t ts, int64_t hs) {
  if (code == KVB_I8)
    hipLaunchKernelGGL((append_kernel<D, B, KVB_I8>), grid, dim3(Quads<D, B>::THREADS), 0, s, c, cu, k, v, ls, ts, hs);
  else
    hipLaunchKernelGGL((append_kernel<D, B, KVB_E4M3>), grid, dim3(Quads<D, B>::THREADS), 0, s, c, cu, k, v, ls, ts, hs);
}

template <int D, int B>
void read(const Cache8& c, int code, kvb_dtype dtype, dim3 grid, hipStream_t s, const int32_t* cu, void* k,
          void* v, int64_t ls, int64_t ts, int64_t hs) {
#define KVB_READ(C, T)                                                                          \
  hipLaunchKernelGGL((read_kernel<D, B, C, T>), grid, dim3(Quads<D, B>::THREADS), 0, s, c, cu, \
                     (T*)k, (T*)v, ls, ts, hs)
  if (code == KVB_I8) {
    if (dtype == KVB_BF16) KVB_READ(KVB_I8, uint16_t);
    else KVB_READ(KVB_I8, float);
  } else {
    if (dtype == KVB_BF16) KVB_READ(KVB_E4M3, uint16_t);
    else KVB_READ(KVB_E4M3, float);
  }
#undef KVB_READ
}

// The blocks that n consecutive tokens can touch, fastest, so that neighbours in the grid take
// neighbouring rows of one head (36 layers of 2 heads, 7.2K tokens: append and read 242 us with
// the heads fastest, 206 so); then K and V of each row of the table.
dim3 span_grid(const Cache8& c, int B, int n) {
  const int64_t blocks = ((int64_t)n + B - 2) / B + 1, rows = 2 * (int64_t)c.n_rows;
  return dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), (unsigned)(rows < kRowsY ? rows : kRowsY),
              (unsigned)((rows + kRowsY - 1) / kRowsY));
}

}  // namespace

#define KVB_FOR_LAYOUT(F, ...)                     \
  do {                                             \
    if (head_dim == 128) {                         \
      if (block_len == 16) F<128, 16>(__VA_ARGS__); \
      else if (block_len == 32) F<128, 32>(__VA_ARGS__); \
      else if (block_len == 64) F<128, 64>(__VA_ARGS__); \
      else F<128, 128>(__VA_ARGS__);               \
    } else {                                       \
      if (block_len == 16) F<64, 16>(__VA_ARGS__);  \
      else if (block_len == 32) F<64, 32>(__VA_ARGS__); \
      else if (block_len == 64) F<64, 64>(__VA_ARGS__); \
      else F<64, 128>(__VA_ARGS__);                \
    }                                              \
  } while (0)

hipError_t launch_cache8_append(const Cache8& c, int head_dim, int block_len, int code,
                                const int32_t* cu_new, int max_new, const uint16_t* k,
                                const uint16_t* v, int64_t layer_stride, int64_t token_stride,
                                int64_t head_stride, hipStream_t s) {
  const dim3 grid = span_grid(c, block_len, max_new);
  KVB_FOR_LAYOUT(append, c, code, grid, s, cu_new, k, v, layer_stride, token_stride, head_stride);
  return hipGetLastError();
}

hipError_t launch_cache8_read(const Cache8& c, int head_dim, int block_len, int code,
                              const int32_t* cu_out, int max_out, kvb_dtype dtype, void* k, void* v,
                              int64_t layer_stride, int64_t token_stride, int64_t head_stride,
                              hipStream_t s) {
  const dim3 grid = span_grid(c, block_len, max_out);
  KVB_FOR_LAYOUT(read, c, code, dtype, grid, s, cu_out, k, v, layer_stride, token_stride, head_stride);
  return hipGetLastError();
}

hipError_t launch_cache8_evict(const Evict& a, int n_layers, hipStream_t s) {
  const int64_t rows = (int64_t)n_layers * a.n_seqs * a.n_kv_heads;
  const dim3 grid((unsigned)((rows + 3) / 4));
#define KVB_EVICT(N) hipLaunchKernelGGL(evict_wave_kernel<N>, grid, dim3(256), 0, s, a, rows)
  // A workgroup a row where a wave cannot hold it, and where a long row would be one wave's on an
  // empty card (72 rows of 512 / 1024 entries: 9.7 / 17.5 us by waves, 6.8 / 7.2 so; of 256 6.1 and
  // 6.6; 300 rows 10.1 / 18.9 and 11.7 / 12.6; 1200 rows 11.5 / 21.5 and 28.5 / 30.9).
  if (a.max_blocks > 2048 || (a.max_blocks > 256 && rows <= 256)) {
    for (int64_t first = 0; first < rows; first += kEvictRows) {
      const int64_t n = rows - first < kEvictRows ? rows - first : kEvictRows;
      hipLaunchKernelGGL(evict_kernel, dim3((unsigned)n), dim3(64 * kEvictWaves), 0, s, a, (int)first);
    }
  } else if (a.max_blocks <= 256) KVB_EVICT(4);
  else if (a.max_blocks <= 512) KVB_EVICT(8);
  else if (a.max_blocks <= 1024) KVB_EVICT(16);
  else KVB_EVICT(32);
#undef KVB_EVICT
  return hipGetLastError();
}

}  // namespace kvb
