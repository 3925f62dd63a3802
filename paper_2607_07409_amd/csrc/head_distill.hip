// Distillation through the vocabulary head: the loss of distill.hip for s = rho W^T, whose rows are never stored.
//
//   p = softmax(rho W^T / T),   d = g / T (M p - q)      (q the teacher's entries, M their mass, g the row's weight)
//   d_rho = d W,                d_W = d^T rho
//
// Two kernels recompute the logits tile by tile on the matrix cores and use each tile at once:
//   k_head_rho  holds 64 rows of rho a wave and streams W: running sum of exponentials and sum_v 2^(y_v - R) W_v
//   k_head_w    holds 64 rows of W a wave and streams rho: p is known by then, d_W is summed over all rows
// so the gradients cost four products of rows x V x r instead of three and no row of logits touches memory.  The
// streamed operand Y passes through LDS in tiles of 32 rows, 16-byte pieces swizzled by row.  The first product is
// S^T = Y X^T (v_mfma_f32_32x32x16_bf16, products exact, sums float32): its result has the held row X in the lane and
// the streamed rows in registers, which is what the second product wants as its left operand, X x d = P^T Y, after
// rounding to bf16; the right operand is the same LDS tile read transposed.  Only that rounding of the
// probabilities (2^-9 relative, each on its own) is below float32, as the gradients' own type is.
//
// The teacher's entries: k_head_finish (one workgroup per row) takes their logits and their part of d_rho from W's
// rows directly, in float32.  Their part of d_W is summed in k_head_w: the entries are put in order of the vocabulary
// tile by a stable counting sort (so the sum's order, and every bit, is the same in every run) and streamed after the
// rows as further tiles of Y, with their coefficients as two bf16 terms.
#include "teacher.hpp"

namespace dls {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kHold = kHeadTile;      // rows of X per workgroup: 64 per wave
constexpr int kTile = 32;             // rows of Y per tile
constexpr float kSlack = 16.f;        // exponents may pass the reference by this before the sums are rescaled

// ------------------------------------------------------------------------------------------
// tiles
// ------------------------------------------------------------------------------------------
// Y tile in LDS: row v of D bf16, its 16-byte piece g at place g ^ (v & swizzle)
template <int D>
struct Tile {
  static constexpr int kPieces = D / 8;                              // per row
  static constexpr int kSwizzle = (kPieces < 16 ? kPieces : 16) - 1;
  static constexpr int kLoads = kTile * kPieces / kThreads;          // per thread
  bf16_t y[kTile * D];
};

// A thread's pieces of a tile, from memory to registers (`row_of(v)` gives the row of Y for tile row v, in range;
// pieces past r are replaced by the row's first: what they meet in X is 0) and from there to LDS.
template <int D, typename RowOf>
__device__ __forceinline__ void tile_load(uint4* reg, const bf16_t* Y, int r, RowOf row_of) {
#pragma unroll
  for (int q = 0; q < Tile<D>::kLoads; ++q) {
    const int p = q * kThreads + threadIdx.x;
    const int v = p / Tile<D>::kPieces, g = (p % Tile<D>::kPieces) ^ (v & Tile<D>::kSwizzle);
    reg[q] = *reinterpret_cast<const uint4*>(Y + (size_t)row_of(v) * r + (g * 8 < r ? g * 8 : 0));
  }
}
template <int D>
__device__ __forceinline__ void tile_store(const uint4* reg, Tile<D>& t) {
#pragma unroll
  for (int q = 0; q < Tile<D>::kLoads; ++q)
    *reinterpret_cast<uint4*>(t.y + (q * kThreads + threadIdx.x) * 8) = reg[q];
}

// the held operand: lane n of tile x has row x0 + 32 x + n, 8 of every 16 columns by its half
template <int D>
__device__ __forceinline__ void hold_load(bf16x8 (&xf)[2][D / 16], const bf16_t* X, int64_t x0, int64_t rows, int r) {
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int64_t row = min(x0 + 32 * x + n, rows - 1);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int c = 16 * k + 8 * h;
      uint4 v = {0, 0, 0, 0};
      if (c < r) v = *reinterpret_cast<const uint4*>(X + (size_t)row * r + c);
      xf[x][k] = __builtin_bit_cast(bf16x8, v);
    }
  }
}

// S^T: tile row m = 8 (i / 4) + 4 half + i % 4 in register i, held row n in the lane
template <int D>
__device__ __forceinline__ void product_s(f32x16 (&s)[2], const Tile<D>& t, const bf16x8 (&xf)[2][D / 16]) {
  const int lane = threadIdx.x & 63, m = lane & 31, h = lane >> 5;
  const char* row = reinterpret_cast<const char*>(t.y) + m * D * 2;
  const int at = (h ^ (m & Tile<D>::kSwizzle)) << 4;
  s[0] = s[1] = f32x16{};
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(row + (at ^ (k << 5)));
    s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, xf[0][k], s[0], 0, 0, 0);
    s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, xf[1][k], s[1], 0, 0, 0);
  }
}

// O[held row][d] += P^T Y.  p[x][j]: the registers 8 j .. 8 j + 7 of S^T's layout, that is tile rows
// 16 j + 8 (e / 4) + 4 half + e % 4; the right operand takes its rows in the same order.
template <int D>
__device__ __forceinline__ void product_o(f32x16 (&o)[2][D / 32], const Tile<D>& t, const bf16x8 (&p)[2][2]) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int v = 4 * h + ((lane & 15) >> 2);                          // + 16 j + 8 e4
  const int g = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);           // + 4 dt
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      union {
        s16x4 q[2];
        bf16x8 b;
      } y;
#pragma unroll
      for (int e4 = 0; e4 < 2; ++e4) {
        const int row = v + 8 * e4;
        const bf16_t* at = t.y + (row + 16 * j) * D + (((g ^ (row & Tile<D>::kSwizzle)) ^ (4 * dt)) << 3) + 4 * (lane & 1);
        y.q[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      }
      o[0][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[0][j], y.b, o[0][dt], 0, 0, 0);
      o[1][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[1][j], y.b, o[1][dt], 0, 0, 0);
    }
  }
}

__device__ __forceinline__ bf16x8 pack8(const float* v) {
  const f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  return __builtin_convertvector(f, bf16x8);
}

// ------------------------------------------------------------------------------------------
// rho held, W streamed
// ------------------------------------------------------------------------------------------
// block (row block, split): split sp of the vocabulary's tiles.  Writes per row and split (R, sum) and, with GRAD,
// sum_v 2^(y_v - R) W_v.
template <int D, bool GRAD>
__global__ __launch_bounds__(kThreads, 1) void k_head_rho(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                          int64_t rows, int V, int r, float c, int splits,
                                                          float2* __restrict__ part_sum, float* __restrict__ part_o) {
  __shared__ Tile<D> tiles[2];
  const int sp = blockIdx.x % splits;
  const int64_t x0 = (int64_t)(blockIdx.x / splits) * kHold + (threadIdx.x >> 6) * 64;
  const int nt = (V + kTile - 1) / kTile;
  const int t0 = (int)((int64_t)nt * sp / splits), t1 = (int)((int64_t)nt * (sp + 1) / splits);
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  auto row_of = [&](int t) { return [=](int v) { return min(t * kTile + v, V - 1); }; };

  bf16x8 xf[2][D / 16];
  hold_load<D>(xf, rho, x0, rows, r);
  f32x16 o[2][GRAD ? D / 32 : 1] = {};
  float ref[2] = {kNoRef, kNoRef}, sum[2] = {0.f, 0.f};
  uint4 reg[Tile<D>::kLoads];
  if (t0 < t1) {
    tile_load<D>(reg, W, r, row_of(t0));
    tile_store<D>(reg, tiles[0]);
  }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const Tile<D>& cur = tiles[(t - t0) & 1];
    tile_load<D>(reg, W, r, row_of(min(t + 1, t1 - 1)));
    f32x16 s[2];
    product_s<D>(s, cur, xf);
    if (t == nt - 1) {   // rows of the last tile past V
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (t * kTile + 8 * (i >> 2) + 4 * h + (i & 3) >= V) s[0][i] = s[1][i] = -INFINITY;
    }
    bf16x8 p[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float top = s[x][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[x][i]);
      top *= c;
      if (__builtin_amdgcn_ballot_w64(top > ref[x] + kSlack)) {   // rare after the first tiles
        const float now = fmaxf(ref[x], fmaxf(top, __shfl_xor(top, 32)));
        const float f = fast_exp2(fmaxf(ref[x] - now, kNoTerm));
        ref[x] = now;
        sum[x] *= f;
        if (GRAD) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float fi = __shfl(f, 8 * (i >> 2) + 4 * h + (i & 3));
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) o[x][GRAD ? dt : 0][i] *= fi;
          }
        }
      }
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        e[i] = fast_exp2(__builtin_fmaf(s[x][i], c, -ref[x]));
        sum[x] += e[i];
      }
      p[x][0] = pack8(e);
      p[x][1] = pack8(e + 8);
    }
    if constexpr (GRAD) product_o<D>(o, cur, p);
    tile_store<D>(reg, tiles[(t - t0 + 1) & 1]);
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float total = sum[x] + __shfl_xor(sum[x], 32);
    const int64_t row = x0 + 32 * x + n;
    if (h == 0 && row < rows) part_sum[(size_t)sp * rows + row] = make_float2(ref[x], total);
    if constexpr (GRAD) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t ro = x0 + 32 * x + 8 * (i >> 2) + 4 * h + (i & 3);
        if (ro >= rows) continue;
        float* out = part_o + ((size_t)sp * rows + ro) * r;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          if (32 * dt + n < r) out[32 * dt + n] = o[x][dt][i];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// a row's results
// ------------------------------------------------------------------------------------------
struct HeadOut {
  float *loss, *lse;       // either may be NULL
  bf16_t* d_rho;           // with gradients: [rows, r]
  float2* row;             //   (R + log2 s, g M / T) of each row
  float* coef;             //   [rows, K]: -g q_k / T of each entry
};

__device__ __forceinline__ float4 widen4(uint2 v) {
  return make_float4(bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y));
}

// one workgroup per row: joins the splits, takes the teacher's logits from W, finishes d_rho
template <bool GRAD>
__global__ __launch_bounds__(kThreads) void k_head_finish(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                          int64_t rows, int V, int r, TeacherArgs te,
                                                          const float* __restrict__ weight, int splits,
                                                          const float2* __restrict__ part_sum,
                                                          const float* __restrict__ part_o, HeadOut o) {
  __shared__ RowShared shr;
  __shared__ TeacherShared sht;
  __shared__ float q[256], log_q[256], scale[256];
  __shared__ int id[256];
  __shared__ float4 acc[kWaves][64];
  __shared__ float loss[kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row = blockIdx.x;
  float mass;
  const TeacherEntry e = teacher_entry(te, row, V, sht, &mass);
  q[t] = e.q;
  log_q[t] = e.log_q;
  id[t] = e.id;
  RowSum a = row_empty();
  if (t < splits) {   // splits <= 256
    const float2 p = part_sum[(size_t)t * rows + row];
    a.R = p.x;
    a.s = p.y;
  }
  const float mine = a.R;
  a = row_block_merge<false>(a, shr);
  const float l2 = fast_log2(a.s), w = (weight ? weight[row] : 1.f) * te.inv_temp;
  scale[t] = t < splits ? w * mass * fast_exp2(fmaxf(mine - a.R, kNoTerm)) / a.s : 0.f;
  __syncthreads();

  const bool on = 4 * lane < r;   // this lane's four columns
  const float4 x = on ? widen4(*reinterpret_cast<const uint2*>(rho + (size_t)row * r + 4 * lane)) : make_float4(0, 0, 0, 0);
  float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
  float term = 0.f;
  for (int k = wave; k < te.k; k += kWaves) {
    if (id[k] < 0) continue;   // the same for the whole wave
    const float4 y = on ? widen4(*reinterpret_cast<const uint2*>(W + (size_t)id[k] * r + 4 * lane)) : make_float4(0, 0, 0, 0);
    const float s = wave_sum(__builtin_fmaf(x.x, y.x, x.y * y.y) + __builtin_fmaf(x.z, y.z, x.w * y.w));
    const TeacherEntry ek = {id[k], q[k], log_q[k]};
    term += teacher_term(ek, __builtin_fmaf(s, te.c, -a.R) - l2);
    if (GRAD) {
      const float f = -w * q[k];
      d.x = __builtin_fmaf(f, y.x, d.x);
      d.y = __builtin_fmaf(f, y.y, d.y);
      d.z = __builtin_fmaf(f, y.z, d.z);
      d.w = __builtin_fmaf(f, y.w, d.w);
    }
  }
  if (GRAD && on) {
    for (int sp = wave; sp < splits; sp += kWaves) {
      const float4 y = *reinterpret_cast<const float4*>(part_o + ((size_t)sp * rows + row) * r + 4 * lane);
      const float f = scale[sp];
      d.x = __builtin_fmaf(f, y.x, d.x);
      d.y = __builtin_fmaf(f, y.y, d.y);
      d.z = __builtin_fmaf(f, y.z, d.z);
      d.w = __builtin_fmaf(f, y.w, d.w);
    }
  }
  if (lane == 0) loss[wave] = term;
  if (GRAD) acc[wave][lane] = d;
  __syncthreads();
  if (t == 0) {
    if (o.loss) o.loss[row] = (loss[0] + loss[1]) + (loss[2] + loss[3]);
    if (o.lse) o.lse[row] = row_lse(a);
    if (GRAD) o.row[row] = make_float2(a.R + l2, w * mass);
  }
  if (GRAD) {
    if (t < te.k) o.coef[(size_t)row * te.k + t] = -w * e.q;
    if (wave == 0 && on) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      typedef float f32x4 __attribute__((ext_vector_type(4)));
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float4 p = acc[k][lane];
        v += f32x4{p.x, p.y, p.z, p.w};
      }
      *reinterpret_cast<bf16x4*>(o.d_rho + (size_t)row * r + 4 * lane) = __builtin_convertvector(v, bf16x4);
    }
  }
}

// ------------------------------------------------------------------------------------------
// the teacher's entries in order of the vocabulary tile: a stable counting sort
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ int entry_tile(const TeacherArgs& te, int64_t e, int64_t n, int V) {
  if (e >= n) return -1;
  const int id = te.ids[e];
  return id >= 0 && id < V && te.values[e] > -INFINITY ? id / kHold : -1;
}

// one wave per chunk of the entries: how many of each tile (tiles <= kMostTiles)
__global__ __launch_bounds__(64) void k_sort_count(TeacherArgs te, int64_t n, int V, int tiles, int chunk,
                                                   uint32_t* __restrict__ counts) {
  __shared__ uint32_t cnt[kHeadMostTiles];
  const int lane = threadIdx.x;
  for (int i = lane; i < tiles; i += 64) cnt[i] = 0;
  __syncthreads();
  const int64_t e0 = (int64_t)blockIdx.x * chunk;
  for (int i = lane; i < chunk; i += 64) {
    const int tile = entry_tile(te, e0 + i, n, V);
    if (tile >= 0) atomicAdd(&cnt[tile], 1u);
  }
  __syncthreads();
  for (int i = lane; i < tiles; i += 64) counts[(size_t)blockIdx.x * tiles + i] = cnt[i];
}

// one workgroup per tile: the chunks' counts become places within the tile; totals[tile]
__global__ __launch_bounds__(kThreads) void k_sort_scan(uint32_t* __restrict__ counts, int chunks, int tiles,
                                                        uint32_t* __restrict__ totals) {
  __shared__ uint32_t wsum[kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t before = 0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + t;
    const uint32_t v = c < chunks ? counts[(size_t)c * tiles + blockIdx.x] : 0;
    uint32_t up = v;   // sum of this and the lower lanes
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(up, d);
      if (lane >= d) up += o;
    }
    if (lane == 63) wsum[wave] = up;
    __syncthreads();
    uint32_t add = before, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) add += wsum[w];
      all += wsum[w];
    }
    if (c < chunks) counts[(size_t)c * tiles + blockIdx.x] = add + up - v;
    before += all;
    __syncthreads();
  }
  if (t == 0) totals[blockIdx.x] = before;
}

// one wave per chunk: entry -> its place, in the order of the entries.  list: (row | place in the tile << 24,
// coefficient).  The first chunk writes where each tile's list begins (begin[tiles] its end).
__global__ __launch_bounds__(64) void k_sort_place(TeacherArgs te, int64_t n, int V, int tiles, int chunk,
                                                   const uint32_t* __restrict__ counts,
                                                   const uint32_t* __restrict__ totals, const float* __restrict__ coef,
                                                   uint32_t* __restrict__ begin, uint2* __restrict__ list) {
  __shared__ uint32_t at[kHeadMostTiles];
  const int lane = threadIdx.x;
  uint32_t before = 0;
  for (int i0 = 0; i0 < tiles; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t v = i < tiles ? totals[i] : 0;
    uint32_t up = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(up, d);
      if (lane >= d) up += o;
    }
    if (i < tiles) {
      at[i] = before + up - v + counts[(size_t)blockIdx.x * tiles + i];
      if (blockIdx.x == 0) begin[i] = before + up - v;
    }
    before += __shfl(up, 63);
  }
  if (blockIdx.x == 0 && lane == 0) begin[tiles] = before;
  __syncthreads();
  const int64_t e0 = (int64_t)blockIdx.x * chunk;
  for (int i = 0; i < chunk; i += 64) {
    const int64_t e = e0 + i + lane;
    const int tile = entry_tile(te, e, n, V);
    // lanes of the same tile
    uint64_t same = __builtin_amdgcn_ballot_w64(tile >= 0);
    if (!same) continue;
#pragma unroll
    for (int b = 0; (1 << b) < kHeadMostTiles; ++b) {
      const bool bit = (tile >> b) & 1;
      const uint64_t set = __builtin_amdgcn_ballot_w64(bit);
      same &= bit ? set : ~set;
    }
    if (tile >= 0) {
      const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
      const uint32_t place = at[tile] + rank;
      list[place] = make_uint2((uint32_t)(e / te.k) | (uint32_t)(te.ids[e] % kHold) << 24, __float_as_uint(coef[e]));
      // (every lane of the tile has read at[tile]: the wave runs in step, and the barrier orders its LDS accesses)
    }
    __syncthreads();
    if (tile >= 0 && (same >> lane) == 1) at[tile] += __popcll(same);   // the last lane of the tile
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------
// W held, rho streamed
// ------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kThreads, 1) void k_head_w(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                        int64_t rows, int V, int r, float c,
                                                        const float2* __restrict__ row_stats,
                                                        const uint32_t* __restrict__ begin,
                                                        const uint2* __restrict__ list, bf16_t* __restrict__ d_w) {
  __shared__ Tile<D> tiles[2];
  __shared__ float rl[2][kTile], ra[2][kTile];   // of a tile's rows: R + log2 s and g M / T; of entries: place, coefficient
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, t = threadIdx.x;
  const int64_t x0 = (int64_t)blockIdx.x * kHold + (t >> 6) * 64;
  const int nt = (int)((rows + kTile - 1) / kTile);
  const uint32_t b0 = begin[blockIdx.x], b1 = begin[blockIdx.x + 1];
  const int ne = (int)((b1 - b0 + kTile - 1) / kTile);
  auto row_of = [&](int tile) { return [=](int v) { return (int)min((int64_t)tile * kTile + v, rows - 1); }; };
  auto entry_of = [&](int tile) {   // (a tile of entries has at least one)
    return [=](int v) { return (int)(list[min(b0 + (uint32_t)tile * kTile + v, b1 - 1)].x & 0xffffffu); };
  };
  auto stats_of = [&](int tile) {
    const int64_t row = (int64_t)tile * kTile + t;
    return t < kTile && row < rows ? row_stats[row] : make_float2(kMostY, 0.f);   // no row: 2^-kMostY times 0
  };

  bf16x8 xf[2][D / 16];
  hold_load<D>(xf, W, x0, V, r);
  f32x16 o[2][D / 32] = {};
  uint4 reg[Tile<D>::kLoads];
  tile_load<D>(reg, rho, r, row_of(0));
  tile_store<D>(reg, tiles[0]);
  if (t < kTile) {
    const float2 st = stats_of(0);
    rl[0][t] = st.x;
    ra[0][t] = st.y;
  }
  __syncthreads();
  for (int k = 0; k < nt; ++k) {
    const Tile<D>& cur = tiles[k & 1];
    const int next = min(k + 1, nt - 1);
    tile_load<D>(reg, rho, r, row_of(next));
    const float2 st = stats_of(next);
    f32x16 s[2];
    product_s<D>(s, cur, xf);
    bf16x8 p[2][2];
    float l[16], a[16];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        l[4 * q + i] = rl[k & 1][8 * q + 4 * h + i];
        a[4 * q + i] = ra[k & 1][8 * q + 4 * h + i];
      }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] = a[i] * fast_exp2(__builtin_fmaf(s[x][i], c, -l[i]));
      p[x][0] = pack8(e);
      p[x][1] = pack8(e + 8);
    }
    product_o<D>(o, cur, p);
    tile_store<D>(reg, tiles[(k + 1) & 1]);
    if (t < kTile) {
      rl[(k + 1) & 1][t] = st.x;
      ra[(k + 1) & 1][t] = st.y;
    }
    __syncthreads();
  }
  // the teacher's entries of this tile
  for (int k = 0; k < ne; ++k) {
    tile_load<D>(reg, rho, r, entry_of(k));
    tile_store<D>(reg, tiles[0]);
    if (t < kTile) {
      const uint32_t i = b0 + (uint32_t)k * kTile + t;
      const uint2 en = i < b1 ? list[i] : make_uint2(0u, 0u);
      rl[0][t] = (float)(en.x >> 24);
      ra[0][t] = __uint_as_float(en.y);
    }
    __syncthreads();
    bf16x8 hi[2][2], lo[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float place = (float)((t >> 6) * 64 + 32 * x + n);
      float e[16], f[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int m = 8 * (i >> 2) + 4 * h + (i & 3);
        e[i] = rl[0][m] == place ? ra[0][m] : 0.f;
        f[i] = e[i] - (float)(__bf16)e[i];
      }
      hi[x][0] = pack8(e);
      hi[x][1] = pack8(e + 8);
      lo[x][0] = pack8(f);
      lo[x][1] = pack8(f + 8);
    }
    product_o<D>(o, tiles[0], hi);
    product_o<D>(o, tiles[0], lo);
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t v = x0 + 32 * x + 8 * (i >> 2) + 4 * h + (i & 3);
      if (v >= V) continue;
      bf16_t* out = d_w + (size_t)v * r;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
        if (32 * dt + n < r) out[32 * dt + n] = __builtin_bit_cast(bf16_t, (__bf16)o[x][dt][i]);
    }
}

__global__ __launch_bounds__(kThreads) void k_zero(uint4* __restrict__ p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) p[i] = make_uint4(0, 0, 0, 0);
}

int head_splits(int64_t rows, int V) {
  // about one workgroup per CU (a wave holds a SIMD's registers), each split at least 8 tiles
  const int64_t blocks = (rows + kHold - 1) / kHold;
  const int64_t cap = std::max<int64_t>(1, V / (8 * kTile));
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(256 / std::max<int64_t>(1, blocks), cap), 256));
}

template <int D>
hipError_t launch_d(const HeadDistillArgs& a, hipStream_t st) {
  const HeadLayout l = head_layout(a.rows, a.V, a.r, a.teacher.k, a.d_rho != nullptr);
  const bf16_t *rho = (const bf16_t*)a.rho, *W = (const bf16_t*)a.w;
  float2* part_sum = (float2*)a.ws;
  float* part_o = (float*)(a.ws + l.off_o);
  const unsigned grid = (unsigned)((a.rows + kHold - 1) / kHold * l.splits);
  HeadOut o = {a.out_loss, a.out_lse, nullptr, nullptr, nullptr};
  hipError_t e;
  if (!a.d_rho) {
    k_head_rho<D, false><<<grid, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher.c, l.splits, part_sum, nullptr);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    k_head_finish<false><<<(unsigned)a.rows, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher, a.weight, l.splits,
                                                                part_sum, nullptr, o);
    return hipGetLastError();
  }
  o.d_rho = (bf16_t*)a.d_rho;
  o.row = (float2*)(a.ws + l.off_row);
  o.coef = (float*)(a.ws + l.off_coef);
  uint32_t *counts = (uint32_t*)(a.ws + l.off_counts), *totals = (uint32_t*)(a.ws + l.off_totals);
  uint32_t* begin = totals + l.tiles;
  uint2* list = (uint2*)(a.ws + l.off_list);
  const int64_t n = a.rows * a.teacher.k;
  k_head_rho<D, true><<<grid, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher.c, l.splits, part_sum, part_o);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_head_finish<true><<<(unsigned)a.rows, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher, a.weight, l.splits,
                                                             part_sum, part_o, o);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_count<<<(unsigned)l.chunks, 64, 0, st>>>(a.teacher, n, a.V, l.tiles, l.chunk, counts);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_scan<<<(unsigned)l.tiles, kThreads, 0, st>>>(counts, l.chunks, l.tiles, totals);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_place<<<(unsigned)l.chunks, 64, 0, st>>>(a.teacher, n, a.V, l.tiles, l.chunk, counts, totals, o.coef, begin, list);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_head_w<D><<<(unsigned)l.tiles, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher.c, o.row, begin, list,
                                                      (bf16_t*)a.d_w);
  return hipGetLastError();
}

}  // namespace

HeadLayout head_layout(int64_t rows, int32_t V, int32_t r, int32_t k, bool grads) {
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  HeadLayout l = {};
  l.splits = head_splits(rows, V);
  l.tiles = (V + kHold - 1) / kHold;
  const int64_t n = rows * k;
  // chunks of at least 512 entries, at most 1,024 of them
  l.chunk = (int)std::max<int64_t>(512, ((n + 1023) / 1024 + 63) / 64 * 64);
  l.chunks = (int)((n + l.chunk - 1) / l.chunk);
  size_t at = up((size_t)l.splits * rows * sizeof(float2));
  if (grads) {
    l.off_o = at;
    at += up((size_t)l.splits * rows * r * sizeof(float));
    l.off_row = at;
    at += up((size_t)rows * sizeof(float2));
    l.off_coef = at;
    at += up((size_t)n * sizeof(float));
    l.off_counts = at;
    at += up((size_t)l.chunks * l.tiles * sizeof(uint32_t));
    l.off_totals = at;
    at += up(((size_t)2 * l.tiles + 1) * sizeof(uint32_t));
    l.off_list = at;
    at += up((size_t)n * sizeof(uint2));
  }
  l.total = at;
  return l;
}

hipError_t launch_head_distill(const HeadDistillArgs& a, hipStream_t st) {
  if (a.rows == 0) {   // with gradients: W's is 0
    const int64_t n = (int64_t)a.V * a.r / 8;
    k_zero<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, st>>>((uint4*)a.d_w, n);
    return hipGetLastError();
  }
  return a.r <= 64 ? launch_d<64>(a, st) : a.r <= 128 ? launch_d<128>(a, st) : launch_d<256>(a, st);
}

}  // namespace dls
