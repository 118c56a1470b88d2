// Rows of a table by token (attr_embed), and the table's gradient (attr_embed_backward).
//
//     out[row] = scale table[token]          dtable[v] (+)= scale sum of dout[row], token = v
//
// Both are HBM-bound: a row is read and written once (13000 rows of 2048, fp32 to bf16: 37.7 us, 34 at
// the rate of a large copy).  The gradient sorts the batch's (token, row) pairs by token, stably, and
// adds up each token's rows in that order in fp32: no atomic additions of values, the same bits every
// time.  The sort is a chain of short launches, which write the gradient's zeros meanwhile; the sums read
// dout once, a wave a run of neighbours.
#include "rows.h"

namespace attr {
namespace {

// U vectors of a lane: 64 U N columns of a row.
template <typename T, typename O, int N>
__device__ inline void embed_row(const RowsArgs& r, const EmbedArgs& a, uint32_t slot, uint32_t cut) {
  const RowSlot s = row_slot(r, slot);
  if (!s.written) return;
  const int64_t v = s.inside ? a.token[s.row] : -1;
  const bool there = v >= 0 && v < a.V;
  const T* const from = (const T*)a.table + (there ? v : 0) * a.ldt;
  O* const out = (O*)a.out + s.row * a.ldo;
  constexpr int U = 4;
  const int c0 = (int)(cut * U * 64 + (threadIdx.x & 63)) * N;
  Raw<T, N> in[U];
  if (there) {
#pragma unroll
    for (int u = 0; u < U; ++u) in[u].load(from + Cols<N>(c0 + u * 64 * N, a.d).at);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[N];
    in[u].get(x);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = there ? x[e] * a.scale : 0.f;
    store_n<O, N>(out, Cols<N>(c0 + u * 64 * N, a.d), x);
  }
}
template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_kernel(RowsArgs r, EmbedArgs a, uint32_t cuts) {
  for (uint64_t unit = (uint64_t)blockIdx.x * 4 + wave_uniform(threadIdx.x >> 6); unit < (uint64_t)r.n_slots * cuts;
       unit += (uint64_t)gridDim.x * 4)
    embed_row<T, O, N>(r, a, (uint32_t)(unit / cuts), (uint32_t)(unit % cuts));
}

// ----------------------------------------------------------------------------
// zeros of a gradient
// ----------------------------------------------------------------------------
// n bytes from p on, by `threads` threads: whole 16-byte pieces, bytes before and behind them.
__device__ inline void zero_span(char* p, int64_t n, int thread, int threads) {
  const int64_t lead = (int64_t)(-reinterpret_cast<uintptr_t>(p) & 15), head = lead < n ? lead : n;
  if (thread < head) p[thread] = 0;
  i32x4* const q = reinterpret_cast<i32x4*>(p + head);
  const int64_t whole = (n - head) / 16;
#pragma unroll 4
  for (int64_t k = thread; k < whole; k += threads) q[k] = i32x4{0, 0, 0, 0};
  if (head + whole * 16 + thread < n) p[head + whole * 16 + thread] = 0;
}
// Share `share` of the table's rows, by a workgroup of the sort's launches.
__device__ inline void zero_share(const EmbedZero& z, uint32_t share) {
  const int64_t each = (z.rows + z.shares - 1) / z.shares, from = share * each, to = from + each < z.rows ? from + each : z.rows;
  if (from >= to) return;
  if (z.row == z.ld) {  // rows without gaps are one span
    zero_span(z.to + from * z.ld, (to - from) * z.row, threadIdx.x, blockDim.x);
    return;
  }
  const int wave = (int)(threadIdx.x >> 6), waves = (int)(blockDim.x >> 6);
  for (int64_t r = from + wave; r < to; r += waves) zero_span(z.to + r * z.ld, z.row, threadIdx.x & 63, 64);
}

// ----------------------------------------------------------------------------
// the sort: least significant digits first, each pass stable
// ----------------------------------------------------------------------------
struct Pair {
  uint32_t key, row;
};

// A lane's pairs of a wave's share: K rounds from `from` on, all loads in flight.
template <int K>
__device__ inline void load_pairs(const uint32_t* key, const uint32_t* row, uint32_t from, uint32_t to, Pair (&p)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t i = from + k * 64 + (threadIdx.x & 63), j = i < to ? i : from;
    p[k] = {key[j], row[j]};
  }
}
// The same of the batch itself: tokens outside [0, V) and slots that are not inside have the key V.
template <int K>
__device__ inline void load_tokens(const RowsArgs& r, const int64_t* token, int64_t V, uint32_t from, uint32_t to, Pair (&p)[K]) {
  RowSlot s[K];
  int64_t v[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t i = from + k * 64 + (threadIdx.x & 63);
    s[k] = row_slot(r, i < to ? i : from);
  }
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = s[k].inside ? token[s[k].row] : -1;
#pragma unroll
  for (int k = 0; k < K; ++k) p[k] = {v[k] >= 0 && v[k] < V ? (uint32_t)v[k] : (uint32_t)V, (uint32_t)s[k].row};
}

// Where each of a wave's lanes puts its pair: base[digit] and the lanes before it with the
// same digit; the last of them moves base on.
__device__ inline uint32_t place(uint32_t* base, uint32_t digit, int bits, bool live) {
  uint64_t same = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((digit >> b) & 1);
    same &= (digit >> b) & 1 ? set : ~set;
  }
  const int lane = threadIdx.x & 63;
  const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
  uint32_t at = 0;
  if (live) {
    at = base[digit] + before;
    if ((same >> lane) == 1) base[digit] = at + 1;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the next call's reads stay behind this one's writes
  return at;
}

// Exclusive sum over the workgroup's threads (NW waves); `total` gets the whole.
template <int NW>
__device__ inline uint32_t block_before(uint32_t v, uint32_t* sm, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t o = __shfl_up(x, off, kWave);
    if (lane >= off) x += o;
  }
  __syncthreads();
  if (lane == 63) sm[wave] = x;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    if (w < wave) before += sm[w];
    total += sm[w];
  }
  return before + x - v;
}

constexpr int kBinsMost = 1 << kSortBits;

// Adds a wave's pairs to the counts of their digits; then, the counts turned into first places,
// puts the pairs there.
template <int K>
__device__ inline void count_pairs(uint32_t* count, const Pair (&p)[K], uint32_t from, uint32_t to, int shift, uint32_t bins) {
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (from + k * 64 + (threadIdx.x & 63) < to) atomicAdd(&count[(p[k].key >> shift) & (bins - 1)], 1u);
}
template <int K, typename F>
__device__ inline void place_pairs(uint32_t* base, const EmbedSort& e, int pass, const Pair (&p)[K], uint32_t from, uint32_t to,
                                   F placed) {
  uint32_t* const key = e.key[(pass + 1) & 1];
  uint32_t* const row = e.row[(pass + 1) & 1];
  const uint32_t bins = 1u << e.bits;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (from + k * 64 >= to) break;
    const bool live = from + k * 64 + (threadIdx.x & 63) < to;
    const uint32_t at = place(base, (p[k].key >> (pass * e.bits)) & (bins - 1), e.bits, live);
    if (live) {
      key[at] = p[k].key;
      row[at] = p[k].row;
      placed(p[k].key, at);
    }
  }
}
// Counts of a workgroup's waves to the first places of their pairs of one digit.
template <int NW>
__device__ inline void wave_places(uint32_t (&base)[NW][kBinsMost], uint32_t bin, uint32_t at) {
  uint32_t c[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) c[w] = base[w][bin];
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    base[w][bin] = at;
    at += c[w];
  }
}
// A wave's share of a workgroup's kSortKeys pairs.
constexpr int kSortWaves = 8, kSortThreads = 64 * kSortWaves, kSortRounds = kSortKeys / kSortThreads;
static_assert(kBinsMost <= kSortThreads, "a thread for each digit");
struct Share {
  uint32_t from, to;
  __device__ inline Share(uint32_t n, uint32_t wave, uint32_t each) {
    const uint32_t first = blockIdx.x * kSortKeys + wave * each;
    from = first < n ? first : n;
    to = n - from < each ? n : from + each;
  }
};

// Every pass of a short batch (up to 1024 K pairs) in one workgroup; the others of this launch, and
// of those below, write the gradient's zeros meanwhile.
template <int K>
__global__ __launch_bounds__(1024) void embed_sort_one_kernel(RowsArgs r, const int64_t* token, int64_t V, EmbedSort e, EmbedZero z) {
  __shared__ uint32_t base[16][kBinsMost];
  __shared__ uint32_t sm[16];
  if (blockIdx.x > 0) return zero_share(z, blockIdx.x - 1);
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  const Share w(r.n_slots, wave, ((r.n_slots + 1023) / 1024) * 64);
  const uint32_t bins = 1u << e.bits;
  for (int pass = 0; pass < e.passes; ++pass) {
    Pair p[K];
    if (w.from < w.to) {
      if (pass == 0) load_tokens<K>(r, token, V, w.from, w.to, p);
      else load_pairs<K>(e.key[pass & 1], e.row[pass & 1], w.from, w.to, p);
    }
    for (uint32_t b = lane; b < bins; b += 64) base[wave][b] = 0;
    __syncthreads();
    count_pairs<K>(base[wave], p, w.from, w.to, pass * e.bits, bins);
    __syncthreads();
    uint32_t mine = 0, total;
    const uint32_t b = threadIdx.x;
    if (b < bins) {
#pragma unroll
      for (int k = 0; k < 16; ++k) mine += base[k][b];
    }
    const uint32_t at = block_before<16>(mine, sm, total);
    if (b < bins) wave_places(base, b, at);
    __syncthreads();
    place_pairs<K>(base[wave], e, pass, p, w.from, w.to, [](uint32_t, uint32_t) {});
    __threadfence_block();
    __syncthreads();
  }
}

// Longer ones, pass by pass: each workgroup counts its pairs' digits (the first pass leaves the
// pairs themselves behind), the counts are added up, and each workgroup puts its pairs in their places.
// Two passes over few workgroups (kNextMost counts) take three launches: the first placing counts the
// second pass's digits where the pairs went, in LDS first.
constexpr uint32_t kNextMost = 8192;
__host__ __device__ inline bool counts_next(const EmbedSort& e) {
  return e.passes == 2 && e.blocks <= 32 && (e.blocks << e.bits) <= kNextMost;
}
__device__ inline uint32_t* counts_of(const EmbedSort& e, int pass) {
  return e.count + (pass && counts_next(e) ? e.blocks << e.bits : 0u);
}
template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(RowsArgs r, const int64_t* token, int64_t V, EmbedSort e, EmbedZero z, int pass) {
  __shared__ uint32_t count[kBinsMost];
  if (blockIdx.x >= e.blocks) return zero_share(z, 2 * pass * z.blocks + blockIdx.x - e.blocks);
  const uint32_t bins = 1u << e.bits;
  for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  const Share w(r.n_slots, wave_uniform(threadIdx.x >> 6), kSortKeys / kSortWaves);
  Pair p[kSortRounds];
  if (w.from < w.to) {
    if (FIRST) load_tokens<kSortRounds>(r, token, V, w.from, w.to, p);
    else load_pairs<kSortRounds>(e.key[pass & 1], e.row[pass & 1], w.from, w.to, p);
  }
  __syncthreads();
  count_pairs<kSortRounds>(count, p, w.from, w.to, pass * e.bits, bins);
  if (FIRST) {
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
      const uint32_t i = w.from + k * 64 + (threadIdx.x & 63);
      if (i < w.to) {
        e.key[0][i] = p[k].key;
        e.row[0][i] = p[k].row;
      }
    }
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) {
    counts_of(e, pass)[(uint64_t)b * e.blocks + blockIdx.x] = count[b];
    if (FIRST && counts_next(e)) counts_of(e, 1)[(uint64_t)b * e.blocks + blockIdx.x] = 0;
  }
}
// Counts of many workgroups to first places, by one.
__global__ __launch_bounds__(1024) void embed_scan_kernel(EmbedSort e) {
  __shared__ uint32_t sm[16];
  const uint32_t n = e.blocks << e.bits;
  uint32_t run = 0;
  for (uint32_t i0 = 0; i0 < n; i0 += 4096) {
    uint32_t c[4], sum = 0, total;
    const uint32_t i = i0 + threadIdx.x * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[k] = i + k < n ? e.count[i + k] : 0u;
      sum += c[k];
    }
    uint32_t at = run + block_before<16>(sum, sm, total);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i + k < n) e.count[i + k] = at;
      at += c[k];
    }
    run += total;
  }
}
// SCAN: the counts are those of few workgroups, and each adds them up by itself.
template <bool SCAN>
__global__ __launch_bounds__(kSortThreads) void embed_place_kernel(EmbedSort e, EmbedZero z, uint32_t n, int pass) {
  __shared__ uint32_t base[kSortWaves][kBinsMost];
  __shared__ uint32_t sm[16];
  __shared__ uint32_t next[SCAN ? kNextMost : 1];  // counts of the next pass, as its table has them
  if (blockIdx.x >= e.blocks) return zero_share(z, (2 * pass + 1 - (pass && counts_next(e) ? 1 : 0)) * z.blocks + blockIdx.x - e.blocks);
  const bool ahead = SCAN && pass == 0 && counts_next(e);
  if (ahead)
    for (uint32_t k = threadIdx.x; k < e.blocks << e.bits; k += kSortThreads) next[k] = 0;
  const int lane = threadIdx.x & 63;
  const uint32_t wave = wave_uniform(threadIdx.x >> 6), bins = 1u << e.bits, b = threadIdx.x;
  const Share w(n, wave, kSortKeys / kSortWaves);
  Pair p[kSortRounds];
  if (w.from < w.to) load_pairs<kSortRounds>(e.key[pass & 1], e.row[pass & 1], w.from, w.to, p);
  uint32_t at = 0;
  if (SCAN) {
    uint32_t mine = 0, before = 0, total;
    if (b < bins)
      for (uint32_t k0 = 0; k0 < e.blocks; k0 += 8) {
        uint32_t c[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) c[k] = counts_of(e, pass)[(uint64_t)b * e.blocks + (k0 + k < e.blocks ? k0 + k : k0)];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
          if (k0 + k >= e.blocks) c[k] = 0;
          mine += c[k];
          if (k0 + k < blockIdx.x) before += c[k];
        }
      }
    at = block_before<kSortWaves>(mine, sm, total) + before;
  } else if (b < bins) {
    at = counts_of(e, pass)[(uint64_t)b * e.blocks + blockIdx.x];
  }
  for (uint32_t k = lane; k < bins; k += 64) base[wave][k] = 0;
  __syncthreads();
  count_pairs<kSortRounds>(base[wave], p, w.from, w.to, pass * e.bits, bins);
  __syncthreads();
  if (b < bins) wave_places(base, b, at);
  __syncthreads();
  place_pairs<kSortRounds>(base[wave], e, pass, p, w.from, w.to, [&](uint32_t key, uint32_t to) {
    if (ahead) atomicAdd(&next[((key >> e.bits) & (bins - 1)) * e.blocks + to / kSortKeys], 1u);
  });
  if (!ahead) return;
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < e.blocks << e.bits; k += kSortThreads)
    if (next[k]) atomicAdd(&counts_of(e, 1)[k], next[k]);
}

// ----------------------------------------------------------------------------
// sums of a token's rows
// ----------------------------------------------------------------------------
// The first place of the sorted keys whose key is above `key`.
__device__ inline uint32_t end_of(const uint32_t* keys, uint32_t n, uint32_t key) {
  uint32_t lo = 0, hi = n;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) >> 1;
    if (keys[mid] <= key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

template <typename T, int N>
__device__ inline void put_sum(const EmbedGradArgs& a, uint32_t v, Cols<N> c, float (&sum)[N]) {
  T* const out = (T*)a.dtable + (int64_t)v * a.ldt;
  if (a.accumulate) {
    float was[N];
    load_n<T, N>(out, c, was);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = sum[e] * a.scale + was[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] *= a.scale;
  }
  store_n<T, N>(out, c, sum);
}

// A wave takes 64 N columns of a part of the sorted pairs.
template <typename G, typename T, int N>
__device__ inline void embed_sum(const EmbedGradArgs& a, uint32_t cuts, uint64_t unit) {
  const int lane = threadIdx.x & 63;
  const uint32_t part = (uint32_t)(unit / cuts), cut = (uint32_t)(unit % cuts);
  const Cols<N> c((int)(cut * 64 + lane) * N, a.d);
  const uint32_t from = part * a.each, to = a.n - from < a.each ? a.n : from + a.each;
  const uint32_t V = (uint32_t)a.V;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  // the part's pairs, and the keys on both sides of it, in the wave's lanes
  const uint32_t j = from + (lane & (a.each - 1)), jj = j < to ? j : to - 1;
  const uint32_t keys = a.key[jj], rows = a.row[jj];
  const uint32_t sides = a.key[lane ? (to < a.n ? to : a.n - 1) : (from > 0 ? from - 1 : 0)];
  const auto lane_of = [](uint32_t x, uint32_t k) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)k); };
  uint32_t cur = lane_of(keys, 0);
  if (cur == V) return;
  bool before = from > 0 && lane_of(sides, 0) == cur;  // cur's rows began in an earlier part
  constexpr int U = N == 1 ? 32 : N == 4 ? 16 : 8;  // rows in flight
  const uint32_t count = to - from;
  for (uint32_t i = 0; i < count; i += U) {
    Raw<G, N> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t k = i + u < count ? i + u : 0;  // the first one is there, and has a row
      x[u].load((const G*)a.dout + (int64_t)(lane_of(keys, k) != V ? lane_of(rows, k) : lane_of(rows, 0)) * a.ldd + c.at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= count) break;
      const uint32_t key = lane_of(keys, i + u);
      if (key != cur) {
        if (before) store_n<float, N>(a.part + (int64_t)part * 2 * a.d, c, sum);
        else put_sum<T, N>(a, cur, c, sum);
        before = false;
        cur = key;
        if (cur == V) return;
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.f;
      }
      float f[N];
      x[u].get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += f[e];
    }
  }
  const bool on = to < a.n && lane_of(sides, 1) == cur;
  if (!before && !on) put_sum<T, N>(a, cur, c, sum);
  else store_n<float, N>(a.part + ((int64_t)part * 2 + (before ? 0 : 1)) * a.d, c, sum);
}
template <typename G, typename T, int N>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a, uint32_t cuts, uint64_t units) {
  for (uint64_t unit = (uint64_t)blockIdx.x * 4 + wave_uniform(threadIdx.x >> 6); unit < units; unit += (uint64_t)gridDim.x * 4)
    embed_sum<G, T, N>(a, cuts, unit);
}

// Joins the sums of a token that begins in a part and goes on behind it: each of the four
// waves an equal share of the following parts, in fp64.  Bound by latency: most workgroups only read the
// keys at a part's end (65536 slots of 1024: 9 us; of one token, whose parts one workgroup a cut adds up: 45).
template <typename T, int N>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a, uint32_t parts, uint32_t cuts) {
  __shared__ double sm[3][N][64];
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  for (uint64_t block = blockIdx.x; block < (uint64_t)(parts - 1) * cuts; block += gridDim.x) {
    const uint32_t part = (uint32_t)(block / cuts), cut = (uint32_t)(block % cuts);
    const uint32_t to = (part + 1) * a.each;  // not the last part: it has nothing behind it
    const uint32_t cur = wave_uniform(a.key[to - 1]);
    if (cur == (uint32_t)a.V || wave_uniform(a.key[to]) != cur) continue;
    const uint32_t from = part * a.each;
    if (wave_uniform(a.key[from]) == cur && from > 0 && wave_uniform(a.key[from - 1]) == cur) continue;
    const uint32_t last = (end_of(a.key, a.n, cur) - 1) / a.each;  // the part that holds its last row
    const Cols<N> c((int)(cut * 64 + lane) * N, a.d);
    const uint32_t each = (last - part + 3) / 4;
    const uint32_t k0 = part + 1 + wave * each, k1 = k0 + each < last + 1 ? k0 + each : last + 1;
    double sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0;
    if (wave == 0) {
      float x[N];
      load_n<float, N>(a.part + ((int64_t)part * 2 + 1) * a.d, c, x);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] = x[e];
    }
#pragma unroll 4
    for (uint32_t k = k0; k < k1; ++k) {
      float x[N];
      load_n<float, N>(a.part + (int64_t)k * 2 * a.d, c, x);
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += x[e];
    }
    __syncthreads();
    if (wave > 0) {
#pragma unroll
      for (int e = 0; e < N; ++e) sm[wave - 1][e][lane] = sum[e];
    }
    __syncthreads();
    if (wave > 0) continue;
    float out[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      for (int w = 0; w < 3; ++w) sum[e] += sm[w][e][lane];
      out[e] = (float)sum[e];
    }
    put_sum<T, N>(a, cur, c, out);
  }
}

// A batch of up to 64 K slots, without a sort: a wave looks through its tokens for those of `each` rows of
// the table, and adds up their rows in the order of their slots.  A token of more than kEmbedLong rows
// takes a workgroup, a quarter of its rows each wave (512 slots of one token: 39.5 us, by one wave 151).
constexpr int kEmbedLong = 64;
struct Found {
  uint32_t count;  // the tokens' slots that have the token
  template <int K>
  __device__ inline Found(const Pair (&p)[K], uint32_t v, uint32_t* list) : count(0) {
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < K; ++k) {  // their rows, in their order
      const bool mine = p[k].key == v;
      const uint64_t has = __ballot(mine);
      if (mine) list[count + (uint32_t)__popcll(has & ((1ull << lane) - 1))] = p[k].row;
      count += (uint32_t)__popcll(has);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
};
// Adds up rows [from, to) of a list, eight of them in flight (16 take the kernel 178 registers: 400 slots of
// 1024 in 21.5 us, where they take 12).
template <typename G, int N>
__device__ inline void sum_list(const EmbedGradArgs& a, const uint32_t* list, uint32_t from, uint32_t to, Cols<N> c, float (&sum)[N]) {
  constexpr int U = 8;
  const uint32_t lane = threadIdx.x & 63;
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  for (uint32_t i0 = from; i0 < to; i0 += U) {
    const uint32_t rows = list[i0 + (lane & (U - 1)) < to ? i0 + (lane & (U - 1)) : i0];
    Raw<G, N> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u].load((const G*)a.dout + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)rows, u) * a.ldd + c.at);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u < to) {
        float f[N];
        x[u].get(f);
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += f[e];
      }
    }
  }
}
template <typename G, typename T, int N, int K>
__global__ __launch_bounds__(256) void embed_small_kernel(RowsArgs r, const int64_t* token, EmbedGradArgs a, uint32_t each,
                                                          uint32_t cuts, uint64_t units) {
  __shared__ uint32_t lists[4][64 * K];
  __shared__ uint32_t longs[4][8], n_long[4];  // each wave's tokens of many rows
  __shared__ float quarter[3][N][64];
  const uint32_t lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  uint32_t* const list = lists[wave];
  Pair p[K];
  load_tokens<K>(r, token, a.V, 0, r.n_slots, p);
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (k * 64 + lane >= r.n_slots) p[k].key = (uint32_t)a.V;
  for (uint64_t first = (uint64_t)blockIdx.x * 4; first < units; first += (uint64_t)gridDim.x * 4) {
    const uint64_t unit = first + wave;
    uint32_t longer = 0;
    if (unit < units) {
      const int64_t v0 = (int64_t)(unit / cuts) * each, v1 = v0 + each < a.V ? v0 + each : a.V;
      const Cols<N> c((int)(((uint32_t)(unit % cuts)) * 64 + lane) * N, a.d);
      for (int64_t v = v0; v < v1; ++v) {
        const Found f(p, (uint32_t)v, list);
        if (a.accumulate && f.count == 0) continue;
        if (f.count > kEmbedLong) {
          longs[wave][longer++] = (uint32_t)v;
          continue;
        }
        float sum[N];
        sum_list<G, N>(a, list, 0, f.count, c, sum);
        put_sum<T, N>(a, (uint32_t)v, c, sum);
      }
    }
    if constexpr (K == 1) continue;
    if (lane == 0) n_long[wave] = longer;
    __syncthreads();
    for (uint32_t w = 0; w < 4; ++w) {
      const Cols<N> c((int)(((uint32_t)((first + w) % cuts)) * 64 + lane) * N, a.d);
      for (uint32_t k = 0; k < n_long[w]; ++k) {
        const uint32_t v = longs[w][k];
        const Found f(p, v, list);
        const uint32_t share = (f.count + 3) / 4, from = wave * share, to = from + share < f.count ? from + share : f.count;
        float sum[N];
        sum_list<G, N>(a, list, from, to, c, sum);
        if (wave > 0) {
#pragma unroll
          for (int e = 0; e < N; ++e) quarter[wave - 1][e][lane] = sum[e];
        }
        __syncthreads();
        if (wave == 0) {
#pragma unroll
          for (int e = 0; e < N; ++e)
            sum[e] = (float)((double)sum[e] + quarter[0][e][lane] + quarter[1][e][lane] + quarter[2][e][lane]);
          put_sum<T, N>(a, v, c, sum);
        }
        __syncthreads();
      }
    }
    __syncthreads();  // n_long is read until here
  }
}

template <typename T, typename O, int N>
hipError_t embed_rows(const RowsArgs& r, const EmbedArgs& a, hipStream_t s) {
  const uint32_t cuts = (uint32_t)((a.d + 256 * N - 1) / (256 * N));
  const uint64_t units = (uint64_t)r.n_slots * cuts;
  hipLaunchKernelGGL((embed_kernel<T, O, N>), dim3(grid_of((units + 3) / 4)), dim3(256), 0, s, r, a, cuts);
  return hipGetLastError();
}
template <typename G, typename T, int N>
hipError_t embed_small(const RowsArgs& r, const int64_t* token, const EmbedGradArgs& a, hipStream_t s) {
  const uint32_t cuts = embed_small_cuts(a.d);
  // a small table: a wave for each row; a large one: fewer searches of the tokens (256 slots of 1024,
  // 50257 rows: 36.3 us, a wave for each row 45.0; 2048 rows: 5.2 and 5.5)
  const uint32_t each = a.V <= 8192 ? 1 : 8;
  const uint64_t units = ((uint64_t)a.V + each - 1) / each * cuts;
  const dim3 grid(grid_of((units + 3) / 4));
  if (r.n_slots <= 64) hipLaunchKernelGGL((embed_small_kernel<G, T, N, 1>), grid, dim3(256), 0, s, r, token, a, each, cuts, units);
  else if (r.n_slots <= 256) hipLaunchKernelGGL((embed_small_kernel<G, T, N, 4>), grid, dim3(256), 0, s, r, token, a, each, cuts, units);
  else hipLaunchKernelGGL((embed_small_kernel<G, T, N, kEmbedSmall / 64>), grid, dim3(256), 0, s, r, token, a, each, cuts, units);
  return hipGetLastError();
}
template <typename G, typename T, int N>
hipError_t embed_sums(const EmbedGradArgs& a, hipStream_t s) {
  const uint32_t parts = (a.n + a.each - 1) / a.each, cuts = embed_cuts(a.d);
  const uint64_t units = (uint64_t)parts * cuts;
  hipLaunchKernelGGL((embed_sum_kernel<G, T, N>), dim3(grid_of((units + 3) / 4)), dim3(256), 0, s, a, cuts, units);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts < 2) return e;
  hipLaunchKernelGGL((embed_join_kernel<T, N>), dim3(grid_of((uint64_t)(parts - 1) * cuts)), dim3(256), 0, s, a, parts, cuts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int table_dtype, int out_dtype, const RowsArgs& r, const EmbedArgs& a, hipStream_t s) {
  return with_type(table_dtype, [&](auto t) {
    return with_type(out_dtype, [&](auto o) {
      if (a.d > 512) return embed_rows<decltype(t), decltype(o), 8>(r, a, s);
      if (a.d >= 64) return embed_rows<decltype(t), decltype(o), 2>(r, a, s);
      return embed_rows<decltype(t), decltype(o), 1>(r, a, s);
    });
  });
}

hipError_t launch_embed_sort(const RowsArgs& r, const int64_t* token, int64_t V, const EmbedSort& e, EmbedZero z, hipStream_t s) {
  // 64 KB and more of zeros a workgroup, spread over the launches
  const bool skip = counts_next(e);  // the second pass's count
  const uint32_t launches = r.n_slots <= kSortOne ? 1 : 2 * (uint32_t)e.passes - (skip ? 1 : 0);
  const uint64_t bytes = (uint64_t)z.rows * (uint64_t)z.row, want = (bytes + 65535) / 65536;
  z.blocks = (uint32_t)((want + launches - 1) / launches < 512 ? (want + launches - 1) / launches : 512);
  z.shares = z.blocks * launches;
  if (r.n_slots <= 1024) {
    hipLaunchKernelGGL(embed_sort_one_kernel<1>, dim3(1 + z.blocks), dim3(1024), 0, s, r, token, V, e, z);
    return hipGetLastError();
  }
  if (r.n_slots <= kSortOne) {
    hipLaunchKernelGGL(embed_sort_one_kernel<kSortOne / 1024>, dim3(1 + z.blocks), dim3(1024), 0, s, r, token, V, e, z);
    return hipGetLastError();
  }
  const dim3 grid(e.blocks + z.blocks);
  for (int pass = 0; pass < e.passes; ++pass) {
    if (pass == 0) hipLaunchKernelGGL(embed_count_kernel<true>, grid, dim3(kSortThreads), 0, s, r, token, V, e, z, pass);
    else if (!skip) hipLaunchKernelGGL(embed_count_kernel<false>, grid, dim3(kSortThreads), 0, s, r, token, V, e, z, pass);
    if (e.blocks <= 32) {
      hipLaunchKernelGGL(embed_place_kernel<true>, grid, dim3(kSortThreads), 0, s, e, z, r.n_slots, pass);
    } else {
      hipLaunchKernelGGL(embed_scan_kernel, dim3(1), dim3(1024), 0, s, e);
      hipLaunchKernelGGL(embed_place_kernel<false>, grid, dim3(kSortThreads), 0, s, e, z, r.n_slots, pass);
    }
  }
  return hipGetLastError();
}

hipError_t launch_embed_grad(int dout_dtype, int table_dtype, const EmbedGradArgs& a, hipStream_t s) {
  return with_type(dout_dtype, [&](auto g) {
    return with_type(table_dtype, [&](auto t) {
      if (embed_lane(a.d) == 8) return embed_sums<decltype(g), decltype(t), 8>(a, s);
      if (embed_lane(a.d) == 4) return embed_sums<decltype(g), decltype(t), 4>(a, s);
      return embed_sums<decltype(g), decltype(t), 1>(a, s);
    });
  });
}

hipError_t launch_embed_small(int dout_dtype, int table_dtype, const RowsArgs& r, const int64_t* token, const EmbedGradArgs& a,
                              hipStream_t s) {
  return with_type(dout_dtype, [&](auto g) {
    return with_type(table_dtype, [&](auto t) {
      if (embed_small_lane(a.d) == 8) return embed_small<decltype(g), decltype(t), 8>(r, token, a, s);
      if (embed_small_lane(a.d) == 4) return embed_small<decltype(g), decltype(t), 4>(r, token, a, s);
      return embed_small<decltype(g), decltype(t), 1>(r, token, a, s);
    });
  });
}

}  // namespace attr
