// Distillation through the vocabulary head: the loss of distill.hip for s = rho W^T, whose rows are never stored.
//
//   p = softmax(rho W^T / T),   d = g / T (M p - q)      (q the teacher's entries, M their mass, g the row's weight)
//   d_rho = d W,                d_W = d^T rho
//
// Two kernels recompute the logits tile by tile on the matrix cores and use each tile at once:
//   k_head_rho  holds 64 rows of rho a wave and streams W: running sum of exponentials and sum_v 2^(y_v - R) W_v
//   k_head_w    holds 64 rows of W a wave and streams rho: p is known by then, d_W is summed over all rows
// so the gradients cost four products of rows x V x r instead of three and no row of logits touches memory.  The
// streamed operand Y passes through LDS in tiles of 32 rows (Tile).  The first product is
// S^T = Y X^T (v_mfma_f32_32x32x16_bf16, products exact, sums float32): its result has the held row X in the lane and
// the streamed rows in registers, which is what the second product wants as its left operand, X x d = P^T Y, after
// rounding to bf16; the right operand is the same LDS tile read transposed.  That rounding (2^-9 relative, each
// probability on its own) is below float32, as the gradients' own type is.  It may stand where a probability is all that
// its token has in d; where q is taken from it, and p is near q once the student has learnt, it would be what is left.
//
// The teacher's entries: k_head_finish (one workgroup per row) computes their logits to the bits of the two kernels, so it
// knows what each rounded, and gives an entry the coefficient -g q / T and the lost part of g / T M p: with the dense part
// that makes g / T (M p - q) in float32.  Their part of d_rho is summed there, from W's rows.  Their part of d_W is summed
// in k_head_w: the entries (several of one id as one) are put in order of the vocabulary tile by a stable counting sort (so
// the sum's order, and every bit, is the same in every run) and streamed after the rows as further tiles of Y, with their
// coefficients as two bf16 terms.
//
// Why 64 rows held a wave: every tile of Y read from LDS then meets two tiles of X, which halves the LDS reads for each
// product, and at r = 256 the second product's sums are just the 256 accumulator registers that a lane has.  That is one
// wave a SIMD, so nothing but the wave itself hides its latencies: the streams run three tiles ahead, and the
// exponentials of a tile stand between the matrix instructions of the tile before.
//
// Measured at 6,001 rows, V = 151,936, r = 256, K = 50: 1,641 to 1,777 us a call; in a profile k_head_rho 761 and k_head_w
// 900 (two products of 467 GFLOP each: 1.23 and 1.04 PFLOP/s; a library product of 8192^3 reaches 1.20 to 1.52),
// k_head_finish 49, the sort 51.  At 1,024 rows (K = 64) 411 to 432 us, k_head_rho 149 and k_head_w 224 of them (1.07 and
// 0.71 PFLOP/s), k_head_finish 25; 96 rows of V = 32,003, r = 128: 68 us, of which seven launches and their ramps are
// most.  The loss alone of 256 rows: 34 to 35 us, W read once in 12.
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
constexpr float kMostSum = 0x1p80f;   // of a tile's 16 terms in a lane, above which the reference moves

// ------------------------------------------------------------------------------------------
// tiles
// ------------------------------------------------------------------------------------------
// Y tile in LDS, in 16-byte pieces: four rows together, of each 64 bytes in turn, and within those the four pieces
// permuted by the next two bits of the row.  So one piece of 16 successive rows (a read of the first product) covers 256
// bytes, four pieces of four successive rows (a transposed read of the second) as well, and every read of a tile is at
// a constant distance from one or two addresses of its lane.
template <int D>
struct Tile {
  static constexpr int kPieces = D / 8;                              // per row
  static constexpr int kLoads = kTile * kPieces / kThreads;          // per thread
  static constexpr int kQuad = 4 * D;                                // elements of four rows
  bf16_t y[kTile * D];
  // row and piece at a place
  __device__ __forceinline__ static void at(uint32_t place, uint32_t* row, uint32_t* piece) {
    const uint32_t quad = place / (kQuad / 8), in = place % (kQuad / 8);
    *row = quad * 4 + in / 4 % 4;
    *piece = in / 16 * 4 + ((in ^ quad) & 3);
  }
};
constexpr int kBuffers = 5;   // a tile in the first product, its predecessor in the second, three that arrive
__device__ __forceinline__ int next_buffer(int b) { return b == kBuffers - 1 ? 0 : b + 1; }

// The streams into LDS bypass the registers: 16 (or 4) bytes a lane from base + its own offset to consecutive places
// from a wave's LDS address (in M0) on.  The compiler does not count them, so the waits are written out.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}
// N times 16 bytes a lane, to N successive KiB; offset q is that of the q-th plus (N - 1 - q) KiB.  (An instruction's
// immediate offset counts on both sides; the base is taken N - 1 KiB lower.)
template <int N>
__device__ __forceinline__ void stream_to_lds16(const void* from, const uint32_t (&offset)[N], uint32_t to) {
  static_assert(N == 1 || N == 2 || N == 4, "tiles of rank 64, 128 and 256");
  const char* base = (const char*)from - (N - 1) * 1024;
  uint32_t m0;
  to = __builtin_amdgcn_readfirstlane(to);
  if constexpr (N == 1)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(to), "s"(base), "v"(offset[0]) : "memory");
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\t"
                 "global_load_lds_dwordx4 %4, %2 offset:1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(to), "s"(base), "v"(offset[0]), "v"(offset[1]) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\t"
                 "global_load_lds_dwordx4 %4, %2 offset:1024\n\tglobal_load_lds_dwordx4 %5, %2 offset:2048\n\t"
                 "global_load_lds_dwordx4 %6, %2 offset:3072\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(to), "s"(base), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]) : "memory");
}
__device__ __forceinline__ void stream_to_lds4(const void* base, uint32_t offset, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base) : "memory");
}
// all but this wave's last n streams have arrived
template <int n>
__device__ __forceinline__ void stream_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
}

// byte offset of a row's piece in memory; pieces past r are replaced by the row's first (what they meet in X is 0)
__device__ __forceinline__ uint32_t piece_offset(uint32_t piece, uint32_t r) { return piece * 8 < r ? piece * 16 : 0; }
// Tiles of the rows 0 .. rows - 1 of Y, each wave its share.  The last of several tiles ends with the last row (it begins
// with rows of the one before); a single tile of fewer rows repeats the last one.
template <int D>
struct TileStream {
  static constexpr int N = Tile<D>::kLoads;
  const bf16_t* Y;
  int64_t rows;
  uint32_t r, place;   // bytes from a tile to this wave's share
  uint32_t offset[N];
  __device__ __forceinline__ TileStream(const bf16_t* Y, int64_t rows, uint32_t r) : Y(Y), rows(rows), r(r) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    place = wave * N * 1024;
#pragma unroll
    for (uint32_t q = 0; q < N; ++q) {
      uint32_t v, g;
      Tile<D>::at((wave * N + q) * 64 + lane, &v, &g);
      offset[q] = (uint32_t)min((int64_t)v, rows - 1) * (2 * r) + piece_offset(g, r) + (N - 1 - q) * 1024;
    }
  }
  __device__ __forceinline__ static int count(int64_t rows) { return (int)((rows + kTile - 1) / kTile); }
  // the first row of a tile
  __device__ __forceinline__ static int64_t first(int tile, int64_t rows) {
    return min((int64_t)tile * kTile, max(rows - kTile, (int64_t)0));
  }
  __device__ __forceinline__ void start(const Tile<D>& to, int tile) const {
    stream_to_lds16(Y + (size_t)first(tile, rows) * r, offset, lds_address(to.y) + place);
  }
};

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

// The first product's matrix instructions are written out: their results belong in ordinary registers, where the
// exponentials read them, while the accumulator registers hold nothing but the second product's sums (for r = 256 all
// 256 of them).  The s_nop is the distance of an operand that the vector unit has just written; results_settle the one
// that a result must keep to the instructions that read it.
__device__ __forceinline__ void mfma_first(f32x16& d, bf16x8 a, bf16x8 b) {
  asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_add(f32x16& d, bf16x8 a, bf16x8 b) {
  asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void results_settle(f32x16 (&s)[2]) {
  asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s[0]), "+v"(s[1]));
}

// S^T: tile row m = 8 (i / 4) + 4 half + i % 4 in register i, held row n in the lane.  The tile's first pieces are read
// beforehand (pieces_first), the others as many products ahead.
constexpr int kAhead = 4;
template <int D>
__device__ __forceinline__ bf16x8 piece(const Tile<D>& t, int k) {
  const int lane = threadIdx.x & 63, m = lane & 31, h = lane >> 5;
  const int from = (m / 4) * Tile<D>::kQuad + m % 4 * 32 + ((2 * (k & 1) + h) ^ (m / 4 & 3)) * 8;
  return *reinterpret_cast<const bf16x8*>(t.y + from + (k / 2) * 128);
}
template <int D>
__device__ __forceinline__ void pieces_first(bf16x8 (&a)[kAhead], const Tile<D>& t) {
#pragma unroll
  for (int k = 0; k < kAhead; ++k) a[k] = piece(t, k);
}
template <int D>
__device__ __forceinline__ void product_s(f32x16 (&s)[2], bf16x8 (&a)[kAhead], const Tile<D>& t, const bf16x8 (&xf)[2][D / 16]) {
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    if (k == 0) {
      mfma_first(s[0], a[0], xf[0][0]);
      mfma_first(s[1], a[0], xf[1][0]);
    } else {
      mfma_add(s[0], a[k % kAhead], xf[0][k]);
      mfma_add(s[1], a[k % kAhead], xf[1][k]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (k + kAhead < D / 16) a[k % kAhead] = piece(t, k + kAhead);
  }
  results_settle(s);
}

// O[held row][d] += P^T Y.  p[x][j]: the registers 8 j .. 8 j + 7 of S^T's layout, that is tile rows
// 16 j + 8 (e / 4) + 4 half + e % 4; the right operand takes its rows in the same order.  Step q is the pair of products
// of 32 columns and 16 rows; `beside(q)` follows it, in the time that the products take.
template <int D>
__device__ __forceinline__ bf16x8 columns(const Tile<D>& t, int q) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const int lane = threadIdx.x & 63, h = lane >> 5, dt = q / 2, j = q % 2;
  const int v = (lane & 15) >> 2;                                    // + 4 h + 16 j + 8 e4
  const int g = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);           // + 4 dt
  union {
    s16x4 q[2];
    bf16x8 b;
  } y;
#pragma unroll
  for (int e4 = 0; e4 < 2; ++e4) {
    const bf16_t* from = t.y + h * Tile<D>::kQuad + v * 32 + (g ^ (h + 2 * e4)) * 8 + 4 * (lane & 1);
    const bf16_t* at = from + (4 * j + 2 * e4) * Tile<D>::kQuad + dt * 128;
    y.q[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
  }
  return y.b;
}
template <int D, typename Beside>
__device__ __forceinline__ void product_o(f32x16 (&o)[2][D / 32], const Tile<D>& t, const bf16x8 (&p)[2][2], Beside beside) {
  constexpr int kSteps = D / 16, kEarly = 3;
  bf16x8 y[kEarly];
#pragma unroll
  for (int q = 0; q < kEarly; ++q) y[q] = columns(t, q);
#pragma unroll
  for (int q = 0; q < kSteps; ++q) {
    o[0][q / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[0][q % 2], y[q % kEarly], o[0][q / 2], 0, 0, 0);
    o[1][q / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p[1][q % 2], y[q % kEarly], o[1][q / 2], 0, 0, 0);
    if (q + kEarly < kSteps) y[q % kEarly] = columns(t, q + kEarly);
    beside(q);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The probabilities of a tile from its logits, a few at a step of the tile before's second product: `begin(x, i)` is
// the exponential of register i, `end(x, i, e)` its value, a step later.
template <int D>
struct Exponentials {
  static constexpr int kPer = 256 / D;   // registers a step
  float e[2][16];
  template <typename Begin, typename End>
  __device__ __forceinline__ void step(int q, Begin begin, End end) {
#pragma unroll
    for (int i = q * kPer; i < (q + 1) * kPer; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) e[x][i] = begin(x, i);
    if (q > 0) finish(q - 1, end);
  }
  template <typename End>
  __device__ __forceinline__ void finish(int q, End end) {
#pragma unroll
    for (int i = q * kPer; i < (q + 1) * kPer; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) e[x][i] = end(x, i, e[x][i]);
  }
};

__device__ __forceinline__ bf16x8 pack8(const float* v) {
  const f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  return __builtin_convertvector(f, bf16x8);
}

// this wave's LDS accesses are done: what its lanes wrote is there for the others, and what they read may be overwritten
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// two probabilities as a word of an operand
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
struct Words {
  uint32_t w[2][8];
  __device__ __forceinline__ void operand(bf16x8 (&p)[2][2]) const {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        p[x][j] = __builtin_bit_cast(bf16x8, uint4{w[x][4 * j], w[x][4 * j + 1], w[x][4 * j + 2], w[x][4 * j + 3]});
  }
};

// An accumulator register times f, in place: written out so that the sums stay in the accumulator registers also where
// they are rescaled (the compiler moves all of them out and back in every tile otherwise).  acc_settle covers the
// distance that a matrix instruction's result, and its next addend, must keep to these.
__device__ __forceinline__ float acc_scale(float a, float f) {
  float v;
  asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1" : "+a"(a), "=&v"(v) : "v"(f));
  return a;
}
__device__ __forceinline__ void acc_settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// ------------------------------------------------------------------------------------------
// rho held, W streamed
// ------------------------------------------------------------------------------------------
// block (row block, split): split sp of the vocabulary's tiles.  Writes per row and split (R, sum) and, with GRAD,
// sum_v bf16(2^(y_v - R)) W_v.  R is the largest of the first tile's y_v, and with GRAD all of the split's terms are
// rounded as they stand above the R that is written: k_head_finish takes the roundings of the teacher's entries back.
// Sums of up to 2^80 of what R stands for are as good as others; where one would pass that (55 nats above the first tile's
// largest logit at T = 1), R moves, and the split is done over from the R that it ends with, at most once.  (Logits of
// spread 3, 6,001 rows: 1,777 us at T = 1 and at 0.3, 2,715 at T = 0.1.)
template <int D, bool GRAD>
__global__ __launch_bounds__(kThreads, 1) void k_head_rho(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                          int64_t rows, int V, int r, float c, int splits,
                                                          float2* __restrict__ part_sum, float* __restrict__ part_o) {
  __shared__ Tile<D> tiles[kBuffers];
  const int sp = blockIdx.x % splits;
  const int64_t x0 = (int64_t)(blockIdx.x / splits) * kHold + (threadIdx.x >> 6) * 64;
  const int nt = TileStream<D>::count(V);
  const int t0 = (int)((int64_t)nt * sp / splits), t1 = (int)((int64_t)nt * (sp + 1) / splits);
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;

  bf16x8 xf[2][D / 16];
  hold_load<D>(xf, rho, x0, rows, r);
  f32x16 o[2][GRAD ? D / 32 : 1];
  float ref[2] = {kNoRef, kNoRef}, sum[2];
  constexpr int kLoads = Tile<D>::kLoads;
  const TileStream<D> stream(W, V, r);
  bool over = false;   // a second time
again:
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    sum[x] = 0.f;
#pragma unroll
    for (int dt = 0; dt < (GRAD ? D / 32 : 1); ++dt) o[x][dt] = f32x16{};
  }
  bool moved = false;   // a reference that terms of earlier tiles have been rounded with
  for (int i = 0; i < 3; ++i) stream.start(tiles[i], min(t0 + i, nt - 1));
  stream_wait<2 * kLoads>();
  __syncthreads();
  bf16x8 a[kAhead], p[2][2] = {};   // p: of the tile before, whose second product runs beside this one's exponentials
  pieces_first(a, tiles[0]);
  int at = 0, before = 0;           // t's buffer and the one before it (at first t's own: p is 0)
  for (int t = t0; t < t1; ++t) {
    const Tile<D>&cur = tiles[at], &last = tiles[before];
    const int next = next_buffer(at), free = next_buffer(next_buffer(next));
    f32x16 s[2];
    auto past_v = [&]() {   // what the last tile repeats
      if (t == nt - 1)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int v = (int)TileStream<D>::first(t, V) + 8 * (i >> 2) + 4 * h + (i & 3);
          if (v < t * kTile || v >= V) s[0][i] = s[1][i] = -INFINITY;
        }
    };
    product_s<D>(s, a, cur, xf);
    past_v();
    stream_wait<kLoads>();   // t + 1 has arrived, t + 2 may be on its way
    __syncthreads();         // everybody's share of it, and everybody is done with t - 2: its buffer takes t + 3
    float add[2] = {0.f, 0.f};
    Exponentials<D> ex;
    Words now;
    auto begin = [&](int x, int i) { return fast_exp2(__builtin_fmaf(s[x][i], c, -ref[x])); };
    auto end = [&](int x, int i, float e) {
      add[x] += e;
      if (i % 2) now.w[x][i / 2] = pack2(ex.e[x][i - 1], e);
      return e;
    };
    if constexpr (GRAD) {
      product_o<D>(o, last, p, [&](int q) {
        if (q == 0) stream.start(tiles[free], min(t + 3, nt - 1));
        ex.step(q, begin, end);
      });
    } else {
      stream.start(tiles[free], min(t + 3, nt - 1));
#pragma unroll
      for (int q = 0; q < D / 16; ++q) ex.step(q, begin, end);
    }
    pieces_first(a, tiles[next]);
    ex.finish(D / 16 - 1, end);
    // Entries far above a row's reference (those of the first tile are): a new one, its sums rescaled, the tile again
    if (__builtin_amdgcn_ballot_w64(fmaxf(add[0], add[1]) >= kMostSum)) {
      pieces_first(a, cur);
      product_s<D>(s, a, cur, xf);   // (so that the logits need not be kept)
      past_v();
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = s[x][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[x][i]);
        top *= c;
        const bool far = fmaxf(add[x], __shfl_xor(add[x], 32)) >= kMostSum;
        const float to = fmaxf(ref[x], far ? fmaxf(top, __shfl_xor(top, 32)) : kNoRef);
        const float f = fast_exp2(fmaxf(ref[x] - to, kNoTerm));
        moved |= far && ref[x] > kNoRef;
        ref[x] = to;
        sum[x] *= f;
        add[x] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ex.e[x][i] = end(x, i, begin(x, i));
        if constexpr (GRAD) {
          acc_settle();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float fi = __shfl(f, 8 * (i >> 2) + 4 * h + (i & 3));
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) o[x][dt][i] = acc_scale(o[x][dt][i], fi);
          }
          acc_settle();
        }
      }
      pieces_first(a, tiles[next]);
    }
    sum[0] += add[0];
    sum[1] += add[1];
    if (GRAD) now.operand(p);
    before = at;
    at = next;
  }
  if constexpr (GRAD) {
    if (!over && __syncthreads_or(moved)) {
      over = true;
      stream_wait<0>();
      __syncthreads();
      goto again;
    }
    if (t0 < t1) product_o<D>(o, tiles[before], p, [](int) {});
  }
  stream_wait<0>();
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
// A tile's rows: g M / T p = factor 2^(y - R).  (All in one exponent would leave the row's part of it to the last place of
// R, which is 1/64 where logits of 10 stand at T = 1e-4.)  64 words, one a lane's.
struct RowTile {
  float R[kTile], factor[kTile];
};
static_assert(sizeof(RowTile) == 256, "a word a lane");

struct HeadOut {
  float *loss, *lse;       // either may be NULL
  bf16_t* d_rho;           // with gradients: [rows, r]
  float* row;              //   what k_head_w needs of each row, by tiles (RowTile)
  int32_t* id;             //   [rows, K]: the id of an entry that is its row's first of it, else -1
  float* coef;             //   [rows, K]: what the entry adds to the coefficient that k_head_w gives its token
};

__device__ __forceinline__ void put_row(float* rows, int64_t place, float R, float factor) {
  RowTile* t = reinterpret_cast<RowTile*>(rows) + place / kTile;
  t->R[place % kTile] = R;
  t->factor[place % kTile] = factor;
}

__device__ __forceinline__ float4 widen4(uint2 v) {
  return make_float4(bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y));
}

__device__ __forceinline__ void add4(float4& d, float f, float4 y) {
  d.x = __builtin_fmaf(f, y.x, d.x);
  d.y = __builtin_fmaf(f, y.y, d.y);
  d.z = __builtin_fmaf(f, y.z, d.z);
  d.w = __builtin_fmaf(f, y.w, d.w);
}

// The logits rho . W_id of 32 entries of a row, by a wave on the matrix cores, in steps as those of product_s: a result is
// the same bits wherever its two rows stand in the tiles and whichever of them comes first (checked over 2 x 10^6 results).
// W's rows come by whole lines, eight rows at a load, and turn in LDS, 64 columns at a time (`turn`, 4 KB a wave's).
template <int D>
__device__ __forceinline__ void entry_logits(const uint4* row, const bf16_t* W, int r, const int* id, uint4* turn, float* logit) {
  constexpr int kParts = D / 64, kTogether = kParts < 2 ? kParts : 2;   // (the loads of two parts in flight together)
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, m = lane >> 3, g = lane & 7;
  f32x16 s = {};
#pragma unroll
  for (int part = 0; part < kParts; part += kTogether) {
    uint4 a[kTogether][4];
#pragma unroll
    for (int u = 0; u < kTogether; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 64 * (part + u) + 8 * g;
        a[u][i] = uint4{0, 0, 0, 0};
        if (c < r) a[u][i] = *reinterpret_cast<const uint4*>(W + (size_t)max(id[8 * i + m], 0) * r + c);
      }
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) turn[(8 * i + m) * 8 + (g ^ m)] = a[u][i];
      lds_done();
#pragma unroll
      for (int k = 0; k < 4; ++k)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, turn[n * 8 + ((2 * k + h) ^ (n & 7))]),
                                                    __builtin_bit_cast(bf16x8, row[8 * (part + u) + 2 * k + h]), s, 0, 0, 0);
      lds_done();
    }
  }
  if (n == 0)
#pragma unroll
    for (int i = 0; i < 16; ++i) logit[8 * (i >> 2) + 4 * h + (i & 3)] = s[i];
}
// what rounding to bf16 takes from a value
__device__ __forceinline__ float rounded_off(float v) { return v - (float)(__bf16)v; }

// One workgroup per row: joins the splits, takes the teacher's logits from W, finishes d_rho.  An entry's coefficient is
// -g q / T and what the dense kernels' rounding took from its probability, so that g / T (M p - q) is a difference of
// float32 numbers however near p is to q.
template <int D, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_head_finish(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                          int64_t rows, int V, int r, TeacherArgs te,
                                                          const float* __restrict__ weight, int splits,
                                                          const float2* __restrict__ part_sum,
                                                          const float* __restrict__ part_o, HeadOut o) {
  __shared__ RowShared<> shr;
  __shared__ TeacherShared<kThreads> sht;
  __shared__ float q[256], logit[256], coef[256], ref[kHeadMostSplits], scale[kHeadMostSplits];
  __shared__ __attribute__((aligned(16))) int id[256];
  __shared__ uint4 x[D / 8];   // the row of rho, 0 past r
  __shared__ uint4 turn[kWaves][256];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row = blockIdx.x;
  float mass;
  const TeacherEntry e = teacher_entry<kThreads>(te, teacher_raw(te, row, V), sht, &mass);
  q[t] = e.q;
  id[t] = e.id;
  if (t < D / 8) x[t] = 8 * t < r ? *reinterpret_cast<const uint4*>(rho + (size_t)row * r + 8 * t) : uint4{0, 0, 0, 0};
  RowSum a = row_empty();
  for (int i = t; i < splits; i += kThreads) {   // (at most kHeadMostSplits)
    const float2 p = part_sum[(size_t)i * rows + row];
    ref[i] = p.x;
    a = row_merge<false>(a, RowSum{p.x, p.y, 0.f});
  }
  a = row_block_merge<false>(a, shr);   // (its barrier covers id, q and x)
  const float l2 = fast_log2(a.s), w = (weight ? weight[row] : 1.f) * te.inv_temp;
  for (int i = t; i < splits; i += kThreads) scale[i] = mass * fast_exp2(fmaxf(ref[i] - a.R, kNoTerm)) / a.s;
  for (int k = 32 * wave; k < te.k; k += 32 * kWaves) entry_logits<D>(x, W, r, id + k, turn[wave], logit + k);
  __syncthreads();

  const float loss = block_sum<kThreads>(e.id >= 0 ? teacher_term(e, __builtin_fmaf(logit[t], te.c, -a.R) - l2) : 0.f, sht.red);
  if (t == 0) {
    if (o.loss) o.loss[row] = loss;
    if (o.lse) o.lse[row] = row_lse(a);
  }
  if (!GRAD) return;
  // what k_head_w needs of the row (the log-sum-exp rounded, so that its exponentials are at most about 1, and in the factor
  // what is left); the places of its tile that no row has: 0 2^-kMostY (the last of several tiles ends with the last row)
  const int64_t whole = rows / kTile * kTile, left = rows - whole;
  const float R = a.R + l2, f = w * mass * (fast_exp2(R - a.R) / a.s);
  if (t == 0) put_row(o.row, rows > kTile && row >= whole ? row + kTile - left : row, R, f);
  if (row == rows - 1 && left > 0 && t < kTile - left) put_row(o.row, rows > kTile ? whole + t : rows + t, kMostY, 0.f);
  if (t < te.k) {
    bool first = e.id >= 0;   // several entries of one id are the first one's
    float c_rho = 0.f, c_w = 0.f;
    if (first) {
      uint32_t same = 0;   // how many entries have the id, and how many of them come first
#pragma unroll 4
      for (int j = 0; j < te.k; j += 4) {
        const int4 v = *reinterpret_cast<const int4*>(id + j);
        const int here[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) same += here[u] != e.id ? 0u : j + u < t ? 0x10001u : 1u;
      }
      first = same < 0x10000u;
      float sum = e.q;
      if (same != 1) {
        sum = 0.f;
        for (int j = 0; j < te.k; ++j) sum += id[j] == e.id ? q[j] : 0.f;
      }
      // the split that has the id's tile
      const int nt = TileStream<D>::count(V), sp = (int)(((int64_t)(e.id / kTile + 1) * splits + nt - 1) / nt) - 1;
      c_rho = scale[sp] * rounded_off(fast_exp2(__builtin_fmaf(logit[t], te.c, -ref[sp]))) - sum;
      c_w = rounded_off(f * fast_exp2(__builtin_fmaf(logit[t], te.c, -R))) - w * sum;
    }
    coef[t] = first ? c_rho : 0.f;
    o.id[(size_t)row * te.k + t] = first ? e.id : -1;
    o.coef[(size_t)row * te.k + t] = c_w;
  }
  __syncthreads();

  const bool on = 4 * lane < r;   // this lane's four columns
  float4 d = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    // the wave's splits and entries, four at a time: their loads in flight together
    const float* from = part_o + (size_t)row * r + 4 * lane;
    const size_t step = (size_t)rows * r;
    int sp = wave;
    for (; sp + 3 * kWaves < splits; sp += 4 * kWaves) {
      float4 y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = *reinterpret_cast<const float4*>(from + (sp + u * kWaves) * step);
#pragma unroll
      for (int u = 0; u < 4; ++u) add4(d, scale[sp + u * kWaves], y[u]);
    }
    for (; sp < splits; sp += kWaves) add4(d, scale[sp], *reinterpret_cast<const float4*>(from + sp * step));
    for (int k0 = wave; k0 < te.k; k0 += 4 * kWaves) {
      uint2 y[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = min(k0 + u * kWaves, te.k - 1);
        y[u] = *reinterpret_cast<const uint2*>(W + (size_t)max(id[k], 0) * r + 4 * lane);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = k0 + u * kWaves;
        if (k < te.k && id[k] >= 0) add4(d, coef[k], widen4(y[u]));
      }
    }
  }
  float4* acc = reinterpret_cast<float4*>(turn[0]);   // (turn has served)
  acc[wave * 64 + lane] = d;
  __syncthreads();
  if (wave == 0 && on) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float4 p = acc[k * 64 + lane];
      v += f32x4{p.x, p.y, p.z, p.w};
    }
    v *= w;
    *reinterpret_cast<bf16x4*>(o.d_rho + (size_t)row * r + 4 * lane) = __builtin_convertvector(v, bf16x4);
  }
}

// ------------------------------------------------------------------------------------------
// the teacher's entries in order of the group of 64 vocabulary entries that a wave of k_head_w holds: a stable
// counting sort (keys <= kHeadMostKeys)
// ------------------------------------------------------------------------------------------
extern __shared__ uint32_t key_lds[];   // a word per key

// A wave's entries are taken 512 at a time, eight a lane, whose loads are all in flight together.
constexpr int kSortLoads = 8;
struct SortEntry {
  int id;        // -1: absent, or not its row's first of that id
  float coef;
};
// entries e0 + 64 u + lane below `end`
template <bool COEF>
__device__ __forceinline__ void sort_load(SortEntry (&en)[kSortLoads], const int32_t* ids, const float* coef, int64_t e0,
                                          int64_t end) {
#pragma unroll
  for (int u = 0; u < kSortLoads; ++u) {
    const int64_t e = e0 + u * 64 + (threadIdx.x & 63);
    en[u].id = e < end ? ids[e] : -1;
    if (COEF) en[u].coef = e < end ? coef[e] : 0.f;
  }
}

// one wave per chunk of the entries: how many of each key
__global__ __launch_bounds__(64) void k_sort_count(const int32_t* __restrict__ ids, int64_t n, int keys, int chunk,
                                                   uint32_t* __restrict__ counts) {
  const int lane = threadIdx.x;
  for (int i = lane; i < keys; i += 64) key_lds[i] = 0;
  __syncthreads();
  const int64_t e0 = (int64_t)blockIdx.x * chunk, end = min(e0 + chunk, n);
  for (int64_t e = e0; e < end; e += 64 * kSortLoads) {
    SortEntry en[kSortLoads];
    sort_load<false>(en, ids, nullptr, e, end);
#pragma unroll
    for (int u = 0; u < kSortLoads; ++u)
      if (en[u].id >= 0) atomicAdd(&key_lds[en[u].id / kHeadGroup], 1u);
  }
  __syncthreads();
  for (int i = lane; i < keys; i += 64) counts[(size_t)blockIdx.x * keys + i] = key_lds[i];
}

// exclusive sums of v over a workgroup of NT threads; *all: the total
template <int NT>
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* wsum, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t up = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(up, d);
    if (lane >= d) up += o;
  }
  __syncthreads();
  if (lane == 63) wsum[wave] = up;
  __syncthreads();
  uint32_t add = 0, total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) add += wsum[w];
    total += wsum[w];
  }
  *all = total;
  return add + up - v;
}

// one workgroup per key: the chunks' counts become places within the key; totals[key]
__global__ __launch_bounds__(kThreads) void k_sort_scan(uint32_t* __restrict__ counts, int chunks, int keys,
                                                        uint32_t* __restrict__ totals) {
  __shared__ uint32_t wsum[kThreads / 64];
  uint32_t before = 0, all;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + (int)threadIdx.x;
    const uint32_t v = c < chunks ? counts[(size_t)c * keys + blockIdx.x] : 0;
    const uint32_t at = before + block_before<kThreads>(v, wsum, &all);
    if (c < chunks) counts[(size_t)c * keys + blockIdx.x] = at;
    before += all;
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// where each key's list begins; begin[keys] ends the last
__global__ __launch_bounds__(1024) void k_sort_base(const uint32_t* __restrict__ totals, int keys,
                                                    uint32_t* __restrict__ begin) {
  __shared__ uint32_t wsum[16];
  uint32_t before = 0, all;
  for (int k0 = 0; k0 < keys; k0 += 1024) {
    const int k = k0 + (int)threadIdx.x;
    const uint32_t at = before + block_before<1024>(k < keys ? totals[k] : 0, wsum, &all);
    if (k < keys) begin[k] = at;
    before += all;
  }
  if (threadIdx.x == 0) begin[keys] = before;
}

// one wave per chunk: entry -> its place, in the order of the entries.  list: (row | place in the group << 24,
// coefficient)
__global__ __launch_bounds__(64) void k_sort_place(const int32_t* __restrict__ ids, const float* __restrict__ coef, int per_row,
                                                   int64_t n, int keys, int chunk, const uint32_t* __restrict__ counts,
                                                   const uint32_t* __restrict__ begin, uint2* __restrict__ list) {
  const int lane = threadIdx.x;
  for (int i = lane; i < keys; i += 64) key_lds[i] = begin[i] + counts[(size_t)blockIdx.x * keys + i];
  __syncthreads();
  const int64_t e0 = (int64_t)blockIdx.x * chunk, end = min(e0 + chunk, n);
  for (int64_t e = e0; e < end; e += 64 * kSortLoads) {
    SortEntry en[kSortLoads];
    sort_load<true>(en, ids, coef, e, end);
#pragma unroll
    for (int u = 0; u < kSortLoads; ++u) {
      const int key = en[u].id < 0 ? -1 : en[u].id / kHeadGroup;
      uint64_t same = __builtin_amdgcn_ballot_w64(key >= 0);   // lanes of the same key
      if (!same) continue;
#pragma unroll
      for (int b = 0; (1 << b) < kHeadMostKeys; ++b) {
        const bool bit = (key >> b) & 1;
        const uint64_t set = __builtin_amdgcn_ballot_w64(bit);
        same &= bit ? set : ~set;
      }
      if (key >= 0) {
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        list[key_lds[key] + rank] = make_uint2((uint32_t)((e + u * 64 + lane) / per_row) | (uint32_t)(en[u].id % kHeadGroup) << 24,
                                               __float_as_uint(en[u].coef));
      }
      __syncthreads();
      if (key >= 0 && (same >> lane) == 1) key_lds[key] += __popcll(same);   // the last lane of the key
      __syncthreads();
    }
  }
}

// ------------------------------------------------------------------------------------------
// W held, rho streamed
// ------------------------------------------------------------------------------------------
// A wave's own tile of Y, by itself: lane v has the row of tile row v
template <int D>
__device__ __forceinline__ void wave_tile_stream(const Tile<D>& to, const bf16_t* Y, uint32_t row, uint32_t r) {
  constexpr int N = Tile<D>::kLoads;
  const uint32_t lane = threadIdx.x & 63;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) {
    uint32_t offset[N];
#pragma unroll
    for (uint32_t q = 0; q < N; ++q) {
      uint32_t v, g;
      Tile<D>::at((w * N + q) * 64 + lane, &v, &g);
      offset[q] = (uint32_t)__shfl((int)row, (int)v) * (2 * r) + piece_offset(g, r) + (N - 1 - q) * 1024;
    }
    stream_to_lds16(Y, offset, lds_address(to.y) + w * N * 1024);
  }
}
// O += q^T Y for a tile's coefficients q[tile row][held row] in LDS, as two bf16 terms: their rounded values and the rest's.
// A coefficient is -p + d with p the bf16 number that the rows' tiles have added, so that its first term, the nearest bf16
// number, is within |d| of it: the second is off by at most 2^-8 d (and by 2^-16 of the coefficient).
template <int D>
__device__ __forceinline__ void coefficient_products(f32x16 (&o)[2][D / 32], const Tile<D>& t, const float* q) {
  const int n = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
  bf16x8 p[2][2][2];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float e[8], rest[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = q[(16 * j + 8 * (i >> 2) + 4 * h + (i & 3)) * kHeadGroup + 32 * x + n];
        rest[i] = rounded_off(e[i]);
      }
      p[0][x][j] = pack8(e);
      p[1][x][j] = pack8(rest);
    }
#pragma unroll 1
  for (int term = 0; term < 2; ++term) {
    product_o<D>(o, t, p[0], [](int) {});
#pragma unroll
    for (int x = 0; x < 2; ++x)
      for (int j = 0; j < 2; ++j) p[0][x][j] = p[1][x][j];
  }
}
template <int D>
__global__ __launch_bounds__(kThreads, 1) void k_head_w(const bf16_t* __restrict__ rho, const bf16_t* __restrict__ W,
                                                        int64_t rows, int V, int r, float c,
                                                        const RowTile* __restrict__ row_tiles,
                                                        const uint32_t* __restrict__ begin,
                                                        const uint2* __restrict__ list, int whole, int splits,
                                                        bf16_t* __restrict__ d_w, float* __restrict__ part_w) {
  // the first `whole` workgroups have a tile of W each; the others share theirs, by the rows, with splits - 1 more
  const int shared = (int)blockIdx.x - whole;
  const int tile = shared < 0 ? blockIdx.x : whole + shared / splits;
  const int part = shared < 0 ? 0 : shared % splits, parts = shared < 0 ? 1 : splits;
  // the stream's buffers; after it a tile of each wave
  static_assert(kBuffers >= kWaves, "the stream's buffers hold the waves' own tiles");
  __shared__ Tile<D> tiles[kBuffers];
  __shared__ RowTile stats[kBuffers][kWaves];         // a copy for each wave
  __shared__ float wide[kWaves][kTile * kHeadGroup];  // a tile's coefficients of the teacher's entries
  __shared__ int range[2][kWaves];
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, t = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t x0 = (int64_t)tile * kHold + wave * 64;
  const int all = TileStream<D>::count(rows);
  const int t0 = (int)((int64_t)all * part / parts), nt = (int)((int64_t)all * (part + 1) / parts);
  const TileStream<D> rho_tiles(rho, rows, r);
  auto stream = [&](int tile, int to) {
    stream_to_lds4(row_tiles + tile, 4 * lane, lds_address(&stats[to][wave]));
    rho_tiles.start(tiles[to], tile);
  };

  bf16x8 xf[2][D / 16];
  hold_load<D>(xf, W, x0, V, r);
  f32x16 o[2][D / 32] = {};
  constexpr int kLoads = Tile<D>::kLoads + 1;
  for (int i = 0; i < 3; ++i) stream(min(t0 + i, nt - 1), i);
  stream_wait<2 * kLoads>();
  __syncthreads();
  bf16x8 a[kAhead], p[2][2] = {};   // as in k_head_rho
  pieces_first(a, tiles[0]);
  int at = 0, before = 0;
  for (int k = t0; k < nt; ++k) {
    const int next = next_buffer(at), free = next_buffer(next_buffer(next));
    const RowTile& st = stats[at][wave];
    f32x16 s[2];
    product_s<D>(s, a, tiles[at], xf);
    stream_wait<kLoads>();
    __syncthreads();
    Exponentials<D> ex;
    Words now;
    // four rows' numbers at a time, read while the four before are used (a read just before its use would be waited for,
    // with all the reads of Y before it)
    float4 R[4], factor[4];
    auto rows_of = [&](int g) {
      R[g] = *reinterpret_cast<const float4*>(st.R + 8 * g + 4 * h);
      factor[g] = *reinterpret_cast<const float4*>(st.factor + 8 * g + 4 * h);
    };
    auto of_row = [](const float4 (&f)[4], int i) { return i % 4 == 0 ? f[i / 4].x : i % 4 == 1 ? f[i / 4].y : i % 4 == 2 ? f[i / 4].z : f[i / 4].w; };
    auto begin = [&](int x, int i) { return fast_exp2(__builtin_fmaf(s[x][i], c, -of_row(R, i))); };
    auto end = [&](int x, int i, float e) {
      const float p = of_row(factor, i) * e;
      if (i % 2) now.w[x][i / 2] = pack2(ex.e[x][i - 1], p);
      return p;
    };
    rows_of(0);
    product_o<D>(o, tiles[before], p, [&](int q) {
      constexpr int kPer = Exponentials<D>::kPer;
      if (q == 0) stream(min(k + 3, nt - 1), free);
      if (q * kPer % 4 == 0 && q * kPer / 4 < 3) rows_of(q * kPer / 4 + 1);
      ex.step(q, begin, end);
    });
    pieces_first(a, tiles[next]);
    ex.finish(D / 16 - 1, end);
    now.operand(p);
    before = at;
    at = next;
  }
  product_o<D>(o, tiles[before], p, [](int) {});
  stream_wait<0>();
  __syncthreads();
  // The teacher's entries of this wave's 64 rows of W, in order of the row.  Few of them: 32 entries a tile, each with
  // its own row of rho and one coefficient.  Where any wave has many (frequent tokens): the tiles of rho once more for
  // all four, with every coefficient that a tile's rows have, so that no list takes much longer than the rows did.
  const uint32_t l0 = begin[tile * kWaves + wave], ln = begin[tile * kWaves + wave + 1] - l0;
  const uint32_t b1 = l0 + (uint32_t)((uint64_t)ln * (part + 1) / parts);
  uint32_t b = l0 + (uint32_t)((uint64_t)ln * part / parts);
  float* q = wide[wave];
#pragma unroll
  for (int i = 0; i < kTile * kHeadGroup / 256; ++i) *reinterpret_cast<float4*>(q + (i * 64 + lane) * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
  // (a tile of entries takes about two and a half times as long as one of rows)
  const bool many = __syncthreads_or((b1 - b + kTile - 1) / kTile > (uint32_t)(nt - t0) * 2 / 5);
  const uint32_t end = max(b1, 1u) - 1;
  uint2 en[4];   // many: the next 256 entries; few: 32
#pragma unroll
  for (int u = 0; u < 4; ++u) en[u] = list[min(b + (many ? u * 64 + lane : n), end)];
  int k = 0, last = 0;
  at = 0;
  if (many) {   // (lists are shared by position, rows by tile: a part's entries may begin before and end after its rows)
    if (lane == 0) {
      range[0][wave] = b < b1 ? (int)((list[b].x & 0xffffffu) / kTile) : all;
      range[1][wave] = b < b1 ? (int)((list[b1 - 1].x & 0xffffffu) / kTile) + 1 : 0;
    }
    __syncthreads();
    k = __builtin_amdgcn_readfirstlane(min(min(range[0][0], range[0][1]), min(range[0][2], range[0][3])));
    last = __builtin_amdgcn_readfirstlane(max(max(range[1][0], range[1][1]), max(range[1][2], range[1][3])));
    for (int i = 0; i < 3; ++i) rho_tiles.start(tiles[i], min(k + i, all - 1));
  }
  while (many ? k < last : b < b1) {
    const uint32_t from = b;
    uint32_t batch = b;   // where en, and then old, begins
    uint2 old[4];
    int first = 0;
    if (many) {
      stream_wait<2 * Tile<D>::kLoads>();   // (the loads of entries only make it wait for more)
      __syncthreads();
      rho_tiles.start(tiles[next_buffer(next_buffer(next_buffer(at)))], min(k + 3, all - 1));
      first = (int)TileStream<D>::first(k, rows);
      for (;;) {
        uint32_t found = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t row = en[u].x & 0xffffffu;
          const bool in = b + u * 64 + lane < b1 && (int)(row / kTile) == k;
          if (in) q[(row - first) * kHeadGroup + (en[u].x >> 24)] = __uint_as_float(en[u].y);   // (a place has one entry)
          found += __popcll(__builtin_amdgcn_ballot_w64(in));
        }
        batch = b;
        b += found;
        if (found < 256 || b >= b1) break;
#pragma unroll
        for (int u = 0; u < 4; ++u) en[u] = list[min(b + u * 64 + lane, end)];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        old[u] = en[u];
        en[u] = list[min(b + u * 64 + lane, end)];   // (the next tile's, on their way beside the products)
      }
      ++k;
    } else {
      lds_done();
      wave_tile_stream(tiles[wave], rho, en[0].x & 0xffffffu, r);
      if (h == 0 && b + n < b1) q[n * kHeadGroup + (en[0].x >> 24)] = __uint_as_float(en[0].y);
      b = min(b + kTile, b1);
      en[1] = en[0];
      en[0] = list[min(b + n, end)];   // (the next tile's)
      stream_wait<0>();
    }
    if (b > from) {
      lds_done();
      coefficient_products<D>(o, tiles[many ? at : wave], q);
      if (many) {
        for (uint32_t i = from + lane; i < batch; i += 64) {   // (more than 256 of a tile)
          const uint32_t x = list[i].x;
          q[((x & 0xffffffu) - first) * kHeadGroup + (x >> 24)] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (batch + u * 64 + lane < b) q[((old[u].x & 0xffffffu) - first) * kHeadGroup + (old[u].x >> 24)] = 0.f;
      } else if (h == 0) {
        q[n * kHeadGroup + (en[1].x >> 24)] = 0.f;
      }
    }
    at = next_buffer(at);
  }
  stream_wait<0>();
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int m = 32 * x + 8 * (i >> 2) + 4 * h + (i & 3);
      if (x0 + m >= V) continue;
      if (shared < 0) {
        bf16_t* out = d_w + (size_t)(x0 + m) * r;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          if (32 * dt + n < r) out[32 * dt + n] = __builtin_bit_cast(bf16_t, (__bf16)o[x][dt][i]);
      } else {
        float* out = part_w + ((size_t)shared * kHold + wave * 64 + m) * r;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          if (32 * dt + n < r) out[32 * dt + n] = o[x][dt][i];
      }
    }
}

// the parts of the shared tiles, eight elements a thread
__global__ __launch_bounds__(kThreads) void k_head_join(const float* __restrict__ part_w, int splits, int64_t first,
                                                        int V, int r, bf16_t* __restrict__ d_w) {
  const int64_t per = (int64_t)kHold * r, e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8;
  const int64_t tile = e / per, in = e % per;
  if (first + tile * kHold + in / r >= V) return;
  const float* from = part_w + tile * splits * per + in;
  f32x8 sum = *reinterpret_cast<const f32x8*>(from);
  for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const f32x8*>(from + s * per);
  *reinterpret_cast<bf16x8*>(d_w + first * r + e) = __builtin_convertvector(sum, bf16x8);
}

__global__ __launch_bounds__(kThreads) void k_zero(uint4* __restrict__ p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) p[i] = make_uint4(0, 0, 0, 0);
}

// Workgroups at a time: one per CU, a wave of rank 256 or 128 with gradients holding its SIMD's registers, else two
constexpr int kSlots = 256;
int head_splits(int64_t rows, int V, bool grads) {
  // of the vocabulary, where rho is held: a slot each; every split at least 4 tiles (46 rows at V = 9,176: 77 us a call,
  // with at least 8 tiles 79)
  const int64_t blocks = (rows + kHold - 1) / kHold;
  const int64_t cap = std::max<int64_t>(1, V / (4 * kTile)), slots = grads ? kSlots : 2 * kSlots;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(slots / std::max<int64_t>(1, blocks), cap), kHeadMostSplits));
}

template <int D>
hipError_t launch_d(const HeadDistillArgs& a, hipStream_t st) {
  const HeadLayout l = head_layout(a.rows, a.V, a.r, a.teacher.k, a.d_rho != nullptr);
  const unsigned key_bytes = (unsigned)l.keys * sizeof(uint32_t);
  const bf16_t *rho = (const bf16_t*)a.rho, *W = (const bf16_t*)a.w;
  float2* part_sum = (float2*)a.ws;
  float* part_o = (float*)(a.ws + l.off_o);
  const unsigned grid = (unsigned)((a.rows + kHold - 1) / kHold * l.splits);
  HeadOut o = {a.out_loss, a.out_lse, nullptr, nullptr, nullptr, nullptr};
  hipError_t e;
  if (!a.d_rho) {
    k_head_rho<D, false><<<grid, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher.c, l.splits, part_sum, nullptr);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    k_head_finish<D, false><<<(unsigned)a.rows, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher, a.weight, l.splits,
                                                                part_sum, nullptr, o);
    return hipGetLastError();
  }
  o.d_rho = (bf16_t*)a.d_rho;
  o.row = (float*)(a.ws + l.off_row);
  o.id = (int32_t*)(a.ws + l.off_id);
  o.coef = (float*)(a.ws + l.off_coef);
  uint32_t *counts = (uint32_t*)(a.ws + l.off_counts), *totals = (uint32_t*)(a.ws + l.off_totals);
  uint32_t* begin = totals + l.keys;
  uint2* list = (uint2*)(a.ws + l.off_list);
  const int64_t n = a.rows * a.teacher.k;
  k_head_rho<D, true><<<grid, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher.c, l.splits, part_sum, part_o);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_head_finish<D, true><<<(unsigned)a.rows, kThreads, 0, st>>>(rho, W, a.rows, a.V, a.r, a.teacher, a.weight, l.splits,
                                                             part_sum, part_o, o);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_count<<<(unsigned)l.chunks, 64, key_bytes, st>>>(o.id, n, l.keys, l.chunk, counts);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_scan<<<(unsigned)l.keys, kThreads, 0, st>>>(counts, l.chunks, l.keys, totals);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_base<<<1, 1024, 0, st>>>(totals, l.keys, begin);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_sort_place<<<(unsigned)l.chunks, 64, key_bytes, st>>>(o.id, o.coef, a.teacher.k, n, l.keys, l.chunk, counts, begin, list);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  float* part_w = (float*)(a.ws + l.off_o);   // (the splits' sums are joined by now)
  k_head_w<D><<<(unsigned)(l.whole + (l.tiles - l.whole) * l.row_splits), kThreads, 0, st>>>(
      rho, W, a.rows, a.V, a.r, a.teacher.c, (const RowTile*)o.row, begin, list, l.whole, l.row_splits, (bf16_t*)a.d_w, part_w);
  if ((e = hipGetLastError()) != hipSuccess || l.whole == l.tiles) return e;
  const int64_t elems = (int64_t)(l.tiles - l.whole) * kHold * a.r;
  k_head_join<<<(unsigned)((elems / 8 + kThreads - 1) / kThreads), kThreads, 0, st>>>(part_w, l.row_splits, (int64_t)l.whole * kHold,
                                                                                  a.V, a.r, (bf16_t*)a.d_w);
  return hipGetLastError();
}

}  // namespace

HeadLayout head_layout(int64_t rows, int32_t V, int32_t r, int32_t k, bool grads) {
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  HeadLayout l = {};
  l.splits = head_splits(rows, V, grads);
  l.tiles = (V + kHold - 1) / kHold;
  l.keys = l.tiles * (kHold / kHeadGroup);   // every wave's, also past V
  // the tiles that the last round of workgroups has too few of share a slot's rows: parts of at least 4 tiles of rows
  // (483 rows at V = 10,911: 113 us a call, with at least 8 tiles 139; 1,500 rows at V = 32,003: 230 either way)
  const int left = l.tiles % kSlots;
  l.row_splits = left ? (int)std::max<int64_t>(1, std::min<int64_t>(kSlots / left, rows / (4 * kTile))) : 1;
  l.whole = l.row_splits > 1 ? l.tiles - left : l.tiles;
  const int64_t n = rows * k;
  // chunks of at least 512 entries, at most 1,024 of them
  l.chunk = (int)std::max<int64_t>(512, ((n + 1023) / 1024 + 63) / 64 * 64);
  l.chunks = (int)((n + l.chunk - 1) / l.chunk);
  size_t at = up((size_t)l.splits * rows * sizeof(float2));
  if (grads) {
    l.off_o = at;
    at += up(std::max((size_t)l.splits * rows, (size_t)(l.tiles - l.whole) * l.row_splits * kHold) * r * sizeof(float));
    l.off_row = at;
    at += up((size_t)((rows + kTile - 1) / kTile) * sizeof(RowTile));
    l.off_id = at;
    at += up((size_t)n * sizeof(int32_t));
    l.off_coef = at;
    at += up((size_t)n * sizeof(float));
    l.off_counts = at;
    at += up((size_t)l.chunks * l.keys * sizeof(uint32_t));
    l.off_totals = at;
    at += up(((size_t)2 * l.keys + 1) * sizeof(uint32_t));
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
