// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits.
//
// One pass (row_stream.hpp) gives the log-sum-exp and the entropy.  The alternatives come out of the same pass: eight
// lanes' chunks of an iteration are one stretch of the row, a block (in short parts eight lanes' chunks of one load, so
// that there are many more blocks than k), and of each block the pass keeps the largest entry.
// Ordered by (value, lower block first), the k-th of these block maxima bounds the row's k best entries from below: k
// blocks hold an entry at least as good, so an entry of a block that ranks behind them is behind k others.  Only the k
// best blocks are read again (512 bytes each, 128 in short parts, from the caches), their entries at or above the bound are collected in
// LDS, and the k best of those are put in order.  Nothing in the pass depends on the data, so a row of equal entries
// costs what any other does.  The first selections need not be exact: a few blocks more than k come along where that
// saves a look at their keys.
//
// Keys: a value's bits as an integer of the same order in the upper half, the complement of the index (or block) in
// the lower, so that the larger key is the better entry, ties going to the lower index, and no two are equal.  0 is
// no key.  Masked entries (-inf) and NaN have none.
//
// What bounds it: many rows, the read (1,024 bf16 rows of V = 151,936 with their 20 best: 63 to 64 us a call; only
// reading them takes 55, and 46 at the 6.75 TB/s that one large array is read with).  Few rows, the chain of launch, a part's
// pass, its selection and the merge (16 such rows: 9.1 us the parts, 5.0 the merge; a row with its 5 best: 6.9 and 3.4).
#include "row_stream.hpp"

namespace dls {

namespace {

constexpr int kThreads = kRowThreads;
constexpr int kCand = 1024;       // candidates held in LDS; rows with more are selected from by re-reading them
constexpr int kBlocks = 1024;     // of a part: 32 iterations

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 and 0 are one value
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 key_of(float x, int index) {
  return x > -INFINITY ? ((u64)order_of(x) << 32) | (uint32_t)~(uint32_t)index : 0;
}
__device__ __forceinline__ int index_of(u64 key) { return (int)~(uint32_t)key; }

struct Select {
  uint32_t hist[256], wsum[kThreads / 64];
  uint32_t digit, need, whole;
  int count;
};

// Digit t's keys, and where thread t's digit is the one in which the need-th key from above lies: sh.digit, what is still
// needed of it, and whether all of it may come along (`above` keys are better than any digit).  sh.digit = 256: too few.
__device__ __forceinline__ void find_digit(uint32_t need, uint32_t above, uint32_t most, Select& sh) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t h = sh.hist[t];
  int from = (int)h;   // keys with a digit of at least t: within sixteen lanes, the wave, the workgroup
  from += __builtin_amdgcn_update_dpp(0, from, 0x101, 0xf, 0xf, true);   // lane + 1, 2, 4, 8 of the sixteen
  from += __builtin_amdgcn_update_dpp(0, from, 0x102, 0xf, 0xf, true);
  from += __builtin_amdgcn_update_dpp(0, from, 0x104, 0xf, 0xf, true);
  from += __builtin_amdgcn_update_dpp(0, from, 0x108, 0xf, 0xf, true);
  const int r1 = __builtin_amdgcn_readlane(from, 16), r2 = __builtin_amdgcn_readlane(from, 32),
            r3 = __builtin_amdgcn_readlane(from, 48);
  from += (lane < 16 ? r1 : 0) + (lane < 32 ? r2 : 0) + (lane < 48 ? r3 : 0);
  if (lane == 0) sh.wsum[wave] = (uint32_t)from;
  __syncthreads();
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w)
    if (w > wave) from += (int)sh.wsum[w];
  if ((uint32_t)from >= need && (uint32_t)from - h < need) {
    sh.digit = (uint32_t)t;
    sh.need = need - ((uint32_t)from - h);
    sh.whole = above + (uint32_t)from <= most;
  }
  if (t == 0 && (uint32_t)from < need) sh.digit = 256;
  __syncthreads();
}

// A bound that at least k and at most `most` (>= k) of the workgroup's keys reach, or 1 where there are fewer than k;
// `each(f)` calls f with every key of this thread.  No two keys are equal, so with most = k it is the k-th largest.
// The first look counts the upper sixteen bits of the values from the largest down, 256 of them: two octaves in steps of
// a bf16's last place, which is nearly always enough.  Then, or where the k-th lies lower, digit by digit.
template <typename Each>
__device__ u64 bound_key(Each each, int k, int most, Select& sh) {
  const int t = threadIdx.x;
  uint32_t top = 0;
  each([&](u64 key) { top = max(top, (uint32_t)(key >> 48)); });
  top = (uint32_t)lanes_max((float)top);   // (sixteen bits: exact)
  sh.hist[t] = 0;
  __syncthreads();   // (and nobody reads wsum any more)
  if ((t & 63) == 0) sh.wsum[t >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) top = max(top, sh.wsum[w]);
  each([&](u64 key) {
    if (key) atomicAdd(&sh.hist[255 - min(top - (uint32_t)(key >> 48), 255u)], 1u);
  });
  __syncthreads();
  find_digit((uint32_t)k, 0, (uint32_t)most, sh);
  if (sh.digit == 256) return 1;
  u64 prefix = 0;
  uint32_t need = (uint32_t)k;
  int shift = 56;
  if (sh.digit > 0) {
    prefix = top - (255 - sh.digit);
    need = sh.need;
    if (sh.whole) return prefix << 48;
    shift = 40;
  }
  for (; shift >= 0; shift -= 8) {
    __syncthreads();
    sh.hist[t] = 0;
    __syncthreads();
    each([&](u64 key) {
      if (key && (shift == 56 || (key >> (shift + 8)) == prefix)) atomicAdd(&sh.hist[(key >> shift) & 255], 1u);
    });
    __syncthreads();
    find_digit(need, (uint32_t)k - need, (uint32_t)most, sh);
    prefix = (prefix << 8) | sh.digit;
    need = sh.need;
    if (sh.whole) return prefix << shift;
  }
  return prefix;
}

// a place without a key, as a key below every entry's, no two alike
__device__ __forceinline__ u64 no_key(int place) { return (u64)place + 1; }
__device__ __forceinline__ bool is_entry(u64 key) { return key >> 32; }

// keys list[0 .. n), n <= 256, into out(rank, key), best first, to rank k - 1; missing ones as key 0 (no_key's come last)
template <typename Out>
__device__ __forceinline__ void order_keys(const u64* list, int n, int k, Out out) {
  const int t = threadIdx.x;
  if (t < n) {
    const u64 mine = list[t];
    int rank = 0, j = 0;
#pragma unroll 4
    for (; j + 1 < n; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(list + j);
      rank += two.x > mine;
      rank += two.y > mine;
    }
    if (j < n) rank += list[j] > mine;
    if (rank < k) out(rank, is_entry(mine) ? mine : 0);
  }
  if (t >= n && t < k) out(t, (u64)0);
}

// the k (<= 256) best of the keys that `each` gives, in order; `list` holds 256
template <typename Each, typename Out>
__device__ void best_keys(Each each, int k, u64* list, Select& sh, Out out) {
  const int t = threadIdx.x;
  const u64 bound = bound_key(each, k, min(256, 2 * k + 16), sh);
  __syncthreads();
  if (t == 0) sh.count = 0;
  __syncthreads();
  each([&](u64 key) {
    if (key && key >= bound) list[atomicAdd(&sh.count, 1)] = key;   // at most 256
  });
  __syncthreads();
  order_keys(list, sh.count, k, out);
}
constexpr int kOrderAll = 64;   // so many are put in order without looking for the best of them first

struct RowOut {
  const int32_t* tokens;
  float c, inv_temp;
  int k;
  dls_token_stats* stats;
  int32_t* ids;
  float* logprobs;
};

// log p of an entry: from its distance to the reference, or where that is no float32 number (an entry of the type's
// lowest value in a row of others) from x / T and the log-sum-exp
__device__ __forceinline__ float log_p(const RowOut& o, const RowSum& a, float x, float l2) {
  const float y = above_ref(x, o.c, a.R);
  return y > -kMostY ? kLn2 * (y - l2) : x * o.inv_temp - kLn2 * (a.R + l2);
}

// the results of a row
template <typename T>
__device__ __forceinline__ void put_stats(const RowOut& o, const T* row, int V, int64_t r, const RowSum& a) {
  const bool any = a.s > 0.f;
  const float l2 = fast_log2(a.s), nan = __builtin_nanf("");
  const int32_t tok = o.tokens ? o.tokens[r] : -1;
  dls_token_stats st;
  st.lse = row_lse(a);
  st.entropy = any ? fmaxf(0.f, kLn2 * (l2 - a.t / a.s)) : nan;
  st.logprob = any && tok >= 0 && tok < V ? log_p(o, a, to_f32(row[tok]), l2) : nan;
  o.stats[r] = st;
}
__device__ __forceinline__ void put_best(const RowOut& o, int64_t r, const RowSum& a, int rank, u64 key) {
  const size_t at = (size_t)r * o.k + rank;
  o.ids[at] = key ? index_of(key) : -1;
  o.logprobs[at] = key ? log_p(o, a, value_of(key), fast_log2(a.s)) : -INFINITY;
}

template <typename T, bool TOP, int U, bool FINE>
__global__ __launch_bounds__(kThreads) void k_logprobs_part(const T* __restrict__ L, int V, int64_t stride, RowOut o,
                                                            float4* __restrict__ part_sums,
                                                            u64* __restrict__ part_keys) {
  constexpr int N = Chunk<T>::N, NT = kThreads;
  __shared__ RowShared<> shr;
  __shared__ Select sh;
  __shared__ __attribute__((aligned(16))) u64 blocks[TOP ? kBlocks : 1];
  __shared__ __attribute__((aligned(16))) u64 list[TOP ? kCand : 1];
  __shared__ uint16_t chosen[256];
  const int part = blockIdx.y, parts = gridDim.y, t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const T* row = L + (size_t)r * stride;
  const RowRange g = row_range(row, V, part, parts);
  constexpr int kSub = FINE ? U : 1, kBlockChunks = kBlockLanes * U / kSub, kPerIter = NT / kBlockLanes * kSub;
  const int nblocks = (g.c1 - g.c0 + NT * U - 1) / (NT * U) * kPerIter;   // <= kBlocks

  RowSum a = row_empty();
  float bm[kSub];   // the largest of this thread's chunks of an iteration
#pragma unroll
  for (int i = 0; i < kSub; ++i) bm[i] = -INFINITY;
  row_edges(g, V, part, parts, [&](int v) {
    const float x = to_f32(row[v]);
    row_fold<1, true>(a, &x, x, o.c);
  });
  row_chunks<U>(
      row, g,
      [&](const uint4* raw, auto n, int u0) {
        float x[N * n];
#pragma unroll
        for (int u = 0; u < n; ++u) Chunk<T>::widen(raw[u], x + u * N);
        float cm;
        if (TOP && FINE) {
          cm = -INFINITY;
#pragma unroll
          for (int u = 0; u < n; ++u) {
            bm[(u0 + u) % kSub] = max_of<N>(x + u * N);
            cm = max3(cm, bm[(u0 + u) % kSub], cm);
          }
        } else {
          cm = max_of<N * n>(x);
          bm[0] = max3(bm[0], cm, cm);
        }
        row_fold<N * n, true>(a, x, cm, o.c);
      },
      [&](int it) {
        if (!TOP) return;
#pragma unroll
        for (int i = 0; i < kSub; ++i) {
          const float m = lanes_max<kBlockLanes>(bm[i]);
          const int blk = it * kPerIter + t / kBlockLanes * kSub + i;
          if (t % kBlockLanes == 0) blocks[blk] = key_of(m, blk);
          bm[i] = -INFINITY;
        }
      });
  a = row_block_merge<true>(a, shr);
  if (t == 0) {
    if (parts == 1) put_stats(o, row, V, r, a);
    else part_sums[(size_t)r * parts + part] = make_float4(a.R, a.s, a.t, 0.f);
  }
  if (!TOP) return;

  // the k best blocks, or some more
  const u64 bound = bound_key([&](auto f) {
    for (int i = t; i < nblocks; i += NT) f(blocks[i]);
  }, o.k, min(256, 2 * o.k + 16), sh);
  auto put = [&](int rank, u64 key) {
    if (parts == 1) put_best(o, r, a, rank, key);
    else part_keys[((size_t)r * parts + part) * o.k + rank] = key;
  };
  if (bound == 1) {   // fewer than k blocks hold an entry that is not masked: the k best of all, read again for every digit
    best_keys([&](auto f) {
      row_edges(g, V, part, parts, [&](int v) { f(key_of(to_f32(row[v]), v)); });
      for (int c = g.c0 + t; c < g.c1; c += NT) {
        float x[N];
        Chunk<T>::load(row + g.h0 + (size_t)c * N, x);
#pragma unroll
        for (int i = 0; i < N; ++i) f(key_of(x[i], g.h0 + c * N + i));
      }
    }, o.k, list, sh, put);
    return;
  }
  __syncthreads();
  if (t == 0) sh.count = 0;
  __syncthreads();
  for (int i = t; i < nblocks; i += NT)
    if (blocks[i] && blocks[i] >= bound) chosen[atomicAdd(&sh.count, 1)] = (uint16_t)i;   // at most 256
  __syncthreads();
  const int nb = sh.count;
  // their entries, and the row's edge entries, as keys
  auto entries = [&](auto f) {
    row_edges(g, V, part, parts, [&](int v) { f(key_of(to_f32(row[v]), v)); });
    for (int w = t; w < nb * kBlockChunks; w += NT) {
      const int blk = chosen[w / kBlockChunks], c = g.c0 + blk * kBlockChunks + w % kBlockChunks;
      if (c >= g.c1) continue;
      float x[N];
      Chunk<T>::load(row + g.h0 + (size_t)c * N, x);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (key_of(x[i], blk) >= bound) f(key_of(x[i], g.h0 + c * N + i));
    }
  };
  __syncthreads();
  if (t == 0) sh.count = 0;
  __syncthreads();
  entries([&](u64 key) {
    if (key) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kCand) list[at] = key;
    }
  });
  __syncthreads();
  const int n = sh.count;
  if (n <= kOrderAll) {
    order_keys(list, n, o.k, put);
  } else if (n <= kCand) {
    best_keys([&](auto f) {
      for (int i = t; i < n; i += NT) f(list[i]);
    }, o.k, blocks, sh, put);   // (the blocks have served)
  } else {   // too many at or above the bound (k blocks that hold most of the row's large entries)
    best_keys(entries, o.k, list, sh, put);
  }
}

// rows split into parts: one workgroup per row merges the parts' sums and their k best keys
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprobs_merge(const T* __restrict__ L, int V, int64_t stride, RowOut o,
                                                             int parts, const float4* __restrict__ part_sums,
                                                             const u64* __restrict__ part_keys) {
  __shared__ RowShared<> shr;
  __shared__ Select sh;
  __shared__ __attribute__((aligned(16))) u64 list[TOP ? 256 : 1];
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const u64* keys = part_keys + (size_t)r * parts * o.k;
  const int n = parts * o.k;
  if (TOP && n <= kOrderAll && t < n) {   // (row_block_merge's barrier comes before it is read)
    const u64 key = keys[t];
    list[t] = key ? key : no_key(t);
  }
  RowSum a = row_empty();
  if (t < parts) {   // parts <= 256
    const float4 p = part_sums[(size_t)r * parts + t];
    a = RowSum{p.x, p.y, p.z};
  }
  a = row_block_merge<true>(a, shr);
  if (t == 0) put_stats(o, L + (size_t)r * stride, V, r, a);
  if (!TOP) return;
  auto put = [&](int rank, u64 key) { put_best(o, r, a, rank, key); };
  if (n <= kOrderAll)
    order_keys(list, n, o.k, put);
  else
    best_keys([&](auto f) {
      for (int i = t; i < n; i += kThreads) f(keys[i]);
    }, o.k, list, sh, put);
}

// With alternatives wanted, a part has at least 256 k entries (so that the k best blocks are few of its blocks), and at
// most kBlocks blocks of four chunks a lane.  (300 float32 rows of V = 32,003, the 64 best: 22.1 us a call; with at least
// 128 k entries 26.4, with 64 k 27.8.)
int logprobs_parts(int64_t rows, int32_t V, int elem_bytes, int k) {
  const int p = row_parts(rows, V, elem_bytes);
  if (k == 0) return p;
  const int most = kBlocks * kBlockLanes * 4 * (16 / elem_bytes);
  return std::max(std::max(1, std::min(p, V / (256 * k))), (V + most - 1) / most);
}

template <typename T>
hipError_t launch_t(const LogprobsArgs& a, hipStream_t st) {
  const int parts = logprobs_parts(a.rows, a.V, (int)sizeof(T), a.k);
  const dim3 grid((unsigned)a.rows, (unsigned)parts);
  const RowOut o = {a.tokens, kLog2e / a.temperature, 1.f / a.temperature, a.k, a.out, a.top_ids, a.top_logprobs};
  const LogprobsLayout l = logprobs_layout(a.rows, a.V, (int)sizeof(T), a.k);
  float4* sums = (float4*)a.ws;
  u64* keys = (u64*)(a.ws + l.off_keys);
  const T* L = (const T*)a.logits;
  // Long parts: four loads a thread in flight and, with alternatives, blocks of all four, so that they fit LDS.  Short
  // ones: two (300 rows of V = 32,003: 17.1 us, with four 17.9).  Fine blocks where they fit (1,024 rows of V = 32,003:
  // 24.0 us, else 24.6; 300 float32 rows with the 64 best: 22.0, else 22.6).
  const int64_t chunks = (a.V / Chunk<T>::N + parts - 1) / parts;
  const bool four = a.V / parts > 16384;
  const bool fine = (chunks + 1023) / 1024 * 1024 <= kBlocks * kBlockLanes;
  const auto part = a.k == 0 ? (four ? k_logprobs_part<T, false, 4, false> : k_logprobs_part<T, false, 2, false>)
                    : four   ? (fine ? k_logprobs_part<T, true, 4, true> : k_logprobs_part<T, true, 4, false>)
                             : k_logprobs_part<T, true, 2, true>;
  part<<<grid, kThreads, 0, st>>>(L, a.V, a.stride, o, sums, keys);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  if (a.k > 0) k_logprobs_merge<T, true><<<(unsigned)a.rows, kThreads, 0, st>>>(L, a.V, a.stride, o, parts, sums, keys);
  else k_logprobs_merge<T, false><<<(unsigned)a.rows, kThreads, 0, st>>>(L, a.V, a.stride, o, parts, sums, keys);
  return hipGetLastError();
}

}  // namespace

LogprobsLayout logprobs_layout(int64_t rows, int32_t V, int elem_bytes, int k) {
  const int parts = logprobs_parts(rows, V, elem_bytes, k);
  LogprobsLayout l = {0, 0};
  if (parts > 1) {
    l.off_keys = (size_t)rows * parts * sizeof(float4);
    l.total = l.off_keys + (size_t)rows * parts * k * sizeof(u64);
  }
  return l;
}

hipError_t launch_logprobs(const LogprobsArgs& a, hipStream_t st) {
  return a.dtype == DLS_BF16 ? launch_t<bf16_t>(a, st) : launch_t<float>(a, st);
}

}  // namespace dls
