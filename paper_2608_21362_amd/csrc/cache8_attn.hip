// kvb_cache8_attn: how a call is cut, its launches, and the launch that joins what workgroups
// shared (the attention kernels are in cache8_attn_kernels.h).
#include "cache8_attn_kernels.h"

namespace kvb {
namespace {

constexpr int kCus = 256;
// workgroups of a launch that joins and adds weights: a long table takes several (work items of a grid
// dimension past 2^32 are lost)
constexpr int kFinishX = 1 << 22;
// tiles stay small up to this many rows, and may up to this many rows x keys of a call
constexpr int kFewRows = 128;
constexpr int64_t kFewWork = 1 << 25;

// splits of a row's tile that hold keys
template <int B>
__device__ __forceinline__ int splits_of(const Seq& sq, const Attn8Plan& plan, int row) {
  const int n = plan.tile_rows;
  const int last = (int)((unsigned)(row / n * n + n - 1) / (unsigned)plan.group);
  const int k = (steps_of<B>(sq, last) + plan.span - 1) / plan.span;
  return max(1, min(k, plan.n_splits));
}

// Joins the splits of the rows, each divided by its own sum.  MANY: a workgroup a row; the sums of the splits
// are weighed first (a lane a split), then D / 4 lanes a split add their outputs, 256 / (D / 4) splits at a time.
// Otherwise D / 4 lanes a row take its few splits one after another.  Either way the sizes fix the
// order of the sums.
template <int D, int B, bool MANY>
__device__ __forceinline__ void join(const Attn8& a, const Attn8Plan& plan, int z, int wg,
                                     const float* __restrict__ po, const float* __restrict__ ml) {
  constexpr int LPR = D / 4, SG = 256 / LPR;  // lanes of a split's row; rows or splits at a time
  const int tid = threadIdx.x, sg = tid / LPR, c = tid % LPR;
  const int b = z / a.c.n_kv_heads, h = z - b * a.c.n_kv_heads;
  const Seq sq = seq_of<B>(a, b);
  const int row = MANY ? wg : wg * SG + sg;
  const bool in = row < sq.n_q * plan.group && row < plan.rows;
  if (MANY && !in) return;
  const int n = in ? splits_of<B>(sq, plan, row) : 0;  // at most 256
  const int64_t rec = (int64_t)z * plan.n_splits * plan.rows + row;
  float top = kNoMax, sum = 0.f;
  f4_t x = {0.f, 0.f, 0.f, 0.f};
  if constexpr (MANY) {
    __shared__ float weight[256], wave_top[4], wave_sum[4];
    __shared__ f4_t sums[SG][LPR];
    float m = kNoMax, l = 0.f;
    if (tid < n) {
      const float2 y = *reinterpret_cast<const float2*>(ml + 2 * (rec + (int64_t)tid * plan.rows));
      m = y.x, l = y.y;
    }
    top = max64(m);
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    sum = tid < n ? __builtin_amdgcn_exp2f(m - top) * l : 0.f;
    weight[tid] = sum;
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k, 64);
    if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
    __syncthreads();
    sum = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    const float inv = inverse(sum);
#pragma unroll 4
    for (int s = sg; s < n; s += SG)
      x += weight[s] * inv * *reinterpret_cast<const f4_t*>(po + (rec + (int64_t)s * plan.rows) * D + c * 4);
    sums[sg][c] = x;
    __syncthreads();
    if (tid >= LPR) return;
    for (int s = 1; s < SG; ++s) x += sums[s][c];
  } else {
    if (!in) return;
    for (int s = 0; s < n; ++s) {
      const float2 y = *reinterpret_cast<const float2*>(ml + 2 * (rec + (int64_t)s * plan.rows));
      const float next = fmaxf(top, y.x);
      sum = sum * __builtin_amdgcn_exp2f(top - next) + y.y * __builtin_amdgcn_exp2f(y.x - next);
      top = next;
    }
    const float inv = inverse(sum);
    for (int s = 0; s < n; ++s) {
      const int64_t at = rec + (int64_t)s * plan.rows;
      const float f = __builtin_amdgcn_exp2f(ml[2 * at] - top) * ml[2 * at + 1] * inv;
      x += f * *reinterpret_cast<const f4_t*>(po + at * D + c * 4);
    }
  }
  const int i = (int)((unsigned)row / (unsigned)plan.group);
  write_row(a, sq.q0 + i, h * plan.group + row - i * plan.group, D, c * 4, x, top, sum);
}

__device__ __forceinline__ void put_weight(const Attn8& a, int z, int blk, float sum) {
  const int64_t at = (int64_t)z * a.c.max_blocks + blk;
  a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + sum;
}

// Accumulated weights: plan.weight_lanes lanes a block (16 or 64), over the rows in turn; the rows'
// log2 sums come through LDS, 256 rows at a time.
template <int B>
__device__ __forceinline__ void add_weights(const Attn8& a, const Attn8Plan& plan, int z, int wg,
                                            const float* __restrict__ ml, const float* __restrict__ parts) {
  constexpr int PB = B < 64 ? B : 64, PER = B / PB;
  __shared__ float total[256];  // log2 of a row's sum
  const int b = z / a.c.n_kv_heads;
  const int M = a.c.max_blocks, lanes = plan.weight_lanes, tid = threadIdx.x;
  const Seq sq = seq_of<B>(a, b);
  const int blk = wg * (256 / lanes) + tid / lanes;
  const int rows = min(sq.n_q * plan.group, plan.rows);
  float sum = 0.f;
  for (int r0 = 0; r0 < rows; r0 += 256) {
    const int r1 = min(rows, r0 + 256), r = r0 + tid;
    __syncthreads();
    if (r < r1) {
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
      total[tid] = t == 0.f ? INFINITY : top + log2f(t);  // nothing seen: no share
    }
    __syncthreads();
    for (int x = r0 + tid % lanes; x < r1; x += lanes) {
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
  for (int k = lanes / 2; k > 0; k >>= 1) sum += __shfl_xor(sum, k, 64);
  if (blk < M && tid % lanes == 0) put_weight(a, z, blk, sum);
}

// The same with a workgroup a block (plan.weight_lanes 256): a thread takes four rows at a time, from
// the first one that sees the block.
template <int B>
__device__ __forceinline__ void add_weights_of_many(const Attn8& a, const Attn8Plan& plan, int z, int blk,
                                                    const float* __restrict__ ml,
                                                    const float* __restrict__ parts) {
  constexpr int PB = B < 64 ? B : 64, PER = B / PB, U = 4;
  __shared__ float wave_sum[4];
  const Seq sq = seq_of<B>(a, z / a.c.n_kv_heads);
  const int rows = min(sq.n_q * plan.group, plan.rows), tid = threadIdx.x;
  const int64_t before = (int64_t)blk * B - ((int64_t)sq.len - sq.n_q);  // queries that do not see it
  const int64_t from = (before > 0 ? before : 0) * plan.group;
  const float2* records = reinterpret_cast<const float2*>(ml) + (int64_t)z * plan.n_splits * plan.rows;
  const float* part = parts + ((int64_t)z * plan.n_parts + blk * PER) * plan.rows;
  float sum = 0.f;
  for (int64_t x0 = from + tid; x0 < rows; x0 += 256 * U) {
    int x[U], n = 0;
    float top[U], t[U], w[U][PER];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      x[j] = min((int)x0 + 256 * j, rows - 1);  // past the last one: it again, for nothing
      const int see = (int)x0 + 256 * j < rows ? seen_by(sq, (int)((unsigned)x[j] / (unsigned)plan.group)) : 0;
#pragma unroll
      for (int p = 0; p < PER; ++p)
        w[j][p] = (blk * PER + p) * PB < see ? part[(int64_t)p * plan.rows + x[j]] : -INFINITY;
      n = max(n, splits_of<B>(sq, plan, x[j]));
      top[j] = kNoMax, t[j] = 0.f;
    }
    for (int s = 0; s < n; ++s) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (s >= splits_of<B>(sq, plan, x[j])) continue;
        const float2 y = records[(int64_t)s * plan.rows + x[j]];
        const float next = fmaxf(top[j], y.x);
        t[j] = t[j] * __builtin_amdgcn_exp2f(top[j] - next) + y.y * __builtin_amdgcn_exp2f(y.x - next);
        top[j] = next;
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const float total = t[j] == 0.f ? INFINITY : top[j] + log2f(t[j]);  // nothing seen: no share
#pragma unroll
      for (int p = 0; p < PER; ++p) sum += __builtin_amdgcn_exp2f(w[j][p] - total);
    }
  }
  for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k, 64);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) put_weight(a, z, blk, wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3]);
}

// What follows the attention kernel, in one launch: the first join_wgs workgroups of a (sequence, kv
// head) join its rows, the others add the weights of its blocks.
template <int D, int B, bool MANY>
__global__ void __launch_bounds__(256) attn8_finish_kernel(Attn8 a, Attn8Plan plan,
                                                           const float* __restrict__ po,
                                                           const float* __restrict__ ml,
                                                           const float* __restrict__ parts, int first) {
  const int wg = first + blockIdx.x;
  if (wg < plan.join_wgs) join<D, B, MANY>(a, plan, blockIdx.y, wg, po, ml);
  else if (plan.weight_lanes == 256) add_weights_of_many<B>(a, plan, blockIdx.y, wg - plan.join_wgs, ml, parts);
  else add_weights<B>(a, plan, blockIdx.y, wg - plan.join_wgs, ml, parts);
}

// Whether a row's splits are joined one after another: up to 4, and up to 8 of many rows, where a
// workgroup a row costs more (8 splits of 8 rows x 32 heads: 19.5 us so and 18.1 with a workgroup a
// row; of 800 rows 46.1 and 44.7, 1600 47.3 and 47.8, 8192 x 2 159 and 165).
bool few_splits(const Attn8Plan& plan) { return plan.n_splits <= (plan.rows > 1024 ? 8 : 4); }

template <int D, int B>
void finish(const Attn8Plan& plan, const Attn8& a, dim3 grid, int first, const float* po, const float* ml,
            const float* parts, hipStream_t s) {
  if (!few_splits(plan))
    hipLaunchKernelGGL((attn8_finish_kernel<D, B, true>), grid, dim3(256), 0, s, a, plan, po, ml, parts, first);
  else
    hipLaunchKernelGGL((attn8_finish_kernel<D, B, false>), grid, dim3(256), 0, s, a, plan, po, ml, parts, first);
}

template <int D>
void finish(const Attn8Plan& plan, const Attn8& a, int block_len, dim3 grid, int first, const float* po,
            const float* ml, const float* parts, hipStream_t s) {
  if (block_len == 16) finish<D, 16>(plan, a, grid, first, po, ml, parts, s);
  else if (block_len == 32) finish<D, 32>(plan, a, grid, first, po, ml, parts, s);
  else if (block_len == 64) finish<D, 64>(plan, a, grid, first, po, ml, parts, s);
  else finish<D, 128>(plan, a, grid, first, po, ml, parts, s);
}

}  // namespace

Attn8Plan attn8_plan(int n_kv_heads, int head_dim, int block_len, int max_blocks, int n_q_heads,
                     int n_seqs, int max_queries, int max_len, bool with_weights) {
  Attn8Plan p{};
  p.group = n_q_heads / n_kv_heads;
  p.rows = max_queries * p.group;
  // Tiles of 256 rows pay once there are more than 128 rows and work for the whole card (2 heads of 8:
  // 72 / 128 rows over 262K keys 79 us in tiles of 32 and 103 / 101 in one of 256, 160 rows 126 and
  // 101; 400 rows over 1000 keys 13 and 38, 4000 x 4000 43 and 58, 3200 x 16000 70 and 66), or more
  // small tiles than two rounds of workgroups (864 / 1512 of up to 430 keys 28 / 42 us and 34 / 31; with
  // weights 432 / 864 33 / 47 and 35 / 40).
  const int64_t heads = (int64_t)n_seqs * n_kv_heads;
  const bool few = p.rows <= kFewRows || (heads * p.rows <= kFewWork / max_len &&
                                          heads * ((p.rows + 31) / 32) <= (with_weights ? 512 : 1024));
  p.tile_rows = !few ? kManyTile : p.rows <= 16 ? 16 : 32;
  p.n_tiles = (p.rows + p.tile_rows - 1) / p.tile_rows;
  const int64_t base = heads * p.n_tiles;
  const int64_t steps = ((int64_t)max_len + 63) / 64;
  // A CU holds one workgroup of 8 waves, two a SIMD.  Of few rows it takes 4 where heads abound and
  // are short: 512 heads of up to 16 steps take 27 us with 8 and 22 with 4, 600 of up to 47 73 and 77.
  p.waves = few && base > kCus && steps <= 32 ? 4 : 8;
  int64_t want = 1;
  if (few) {
    // As many splits as fit on the card together: HBM-bound, so a part of the CUs keeps the rate up, but
    // workgroups of a second round are late (8192 tokens of 96 heads: 52 us with 2 splits, 59 with 3;
    // of 200 heads: 90 with one, 101 with 2).  Of 4 steps at least (2000 tokens: 12.1 us, of 8 steps
    // 13.7, of 16 15.8), and no split of up to 16 steps where that saves the second launch (500 tokens:
    // 8.5 us and 11.7, 1000: 11.6 and 12.0).
    want = kCus / base;
    if (want > steps / 4) want = steps / 4;
    if (want < 1 || (steps <= 16 && !with_weights)) want = 1;
  } else {
    // Bound by the CUs: a call takes rounds * (steps of a split + 10 for what a workgroup does beside
    // them); the splits that fill 1 to 8 rounds are compared.
    int64_t least = INT64_MAX;
    for (int rounds = 1; rounds <= 8; ++rounds) {
      int64_t n = kCus * rounds / base;
      if (n > steps / 2) n = steps / 2;
      if (n > kCus) n = kCus;
      if (n < 1) n = 1;
      const int64_t cost = (base * n + kCus - 1) / kCus * ((steps + n - 1) / n + 10);
      if (cost < least) least = cost, want = n;
    }
  }
  p.span = (int)((steps + want - 1) / want);
  p.wave_span = (p.span + p.waves - 1) / p.waves;
  p.n_splits = (int)((steps + p.span - 1) / p.span);
  // Tiles that share keys on one XCD, where there are groups of them for all 8 (20 heads of 20K keys, 5
  // tiles of 32 rows 51 -> 46 us; 80 heads, 3 tiles 106 -> 95).
  p.apart = few && p.n_tiles > 1 && heads * p.n_splits >= 32;
  const int pb = block_len < 64 ? block_len : 64;
  p.n_parts = with_weights ? (max_blocks + 1) * (block_len / pb) : 0;
  const int per = 256 / (head_dim / 4);
  if (p.n_splits > 1) p.join_wgs = few_splits(p) ? (p.rows + per - 1) / per : p.rows;
  // Lanes of a block: more rows, more lanes (16 / 64 / 256: 8 rows x 128 heads 21 / 27 / 43 us, 128 rows x
  // 4 heads 40 / 37 / 44, 512 87 / 74 / 86, 64000 rows over 8192 keys 2727 / 1349 / 621).
  p.weight_lanes = p.rows <= 64 ? 16 : p.rows <= 1024 ? 64 : 256;
  const int per_wg = 256 / p.weight_lanes;
  if (with_weights) p.weight_wgs = (max_blocks + per_wg - 1) / per_wg;
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
  const auto kernels = head_dim == 128 ? (code == KVB_I8 ? attn8_d128_i8 : attn8_d128_e4m3)
                                       : (code == KVB_I8 ? attn8_d64_i8 : attn8_d64_e4m3);
  kernels(plan, a, block_len, po, ml, parts, s);
  if (hipError_t e = hipGetLastError()) return e;
  if (plan.join_wgs + plan.weight_wgs == 0) return hipSuccess;
  const int wgs = plan.join_wgs + plan.weight_wgs;
  for (int first = 0; first < wgs; first += kFinishX) {
    const dim3 grid((unsigned)(wgs - first < kFinishX ? wgs - first : kFinishX), (unsigned)(a.c.n_seqs * a.c.n_kv_heads));
    if (head_dim == 128) finish<128>(plan, a, block_len, grid, first, po, ml, parts, s);
    else finish<64>(plan, a, block_len, grid, first, po, ml, parts, s);
  }
  return hipGetLastError();
}

}  // namespace kvb
