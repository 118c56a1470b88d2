// Rows of a table by token (attr_embed), and the table's gradient (attr_embed_backward).
//
//     out[row] = scale table[token]          dtable[v] (+)= scale sum of dout[row], token = v
//
// Both are HBM-bound.  The gradient sorts the batch's (token, row) pairs by token, stably, and
// adds up each token's rows in that order in fp32: no atomic additions, the same bits every time.
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
  float x[U][N];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 64 * N;
    load_n<T, N>(from + c, there ? a.d - c : 0, x[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * 64 * N;
#pragma unroll
    for (int e = 0; e < N; ++e) x[u][e] = there ? x[u][e] * a.scale : 0.f;
    store_n<O, N>(out + c, a.d - c, x[u]);
  }
}
template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_kernel(RowsArgs r, EmbedArgs a, uint32_t cuts) {
  for (uint64_t unit = (uint64_t)blockIdx.x * 4 + wave_uniform(threadIdx.x >> 6); unit < (uint64_t)r.n_slots * cuts;
       unit += (uint64_t)gridDim.x * 4)
    embed_row<T, O, N>(r, a, (uint32_t)(unit / cuts), (uint32_t)(unit % cuts));
}

// ----------------------------------------------------------------------------
// the sort: least significant digits first, each pass stable
// ----------------------------------------------------------------------------
struct Pair {
  uint32_t key, row;
};
__device__ inline Pair first_pair(const RowsArgs& r, const int64_t* token, int64_t V, uint32_t slot) {
  const RowSlot s = row_slot(r, slot);
  const int64_t v = s.inside ? token[s.row] : -1;
  return {v >= 0 && v < V ? (uint32_t)v : (uint32_t)V, (uint32_t)s.row};
}
__device__ inline Pair pair_of(const RowsArgs& r, const int64_t* token, int64_t V, const EmbedSort& e, int pass, uint32_t i) {
  if (pass == 0) return first_pair(r, token, V, i);
  return {e.key[pass & 1][i], e.row[pass & 1][i]};
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

// Every pass of a short batch in one workgroup; a wave takes a contiguous share of the pairs.
__global__ __launch_bounds__(1024) void embed_sort_one_kernel(RowsArgs r, const int64_t* token, int64_t V, EmbedSort e) {
  __shared__ uint32_t base[16][kBinsMost];
  __shared__ uint32_t sm[16];
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  const uint32_t n = r.n_slots, share = ((n + 1023) / 1024) * 64;
  const uint32_t from = wave * share, to = from + share < n ? from + share : n;
  const uint32_t bins = 1u << e.bits;
  for (int pass = 0; pass < e.passes; ++pass) {
    const int shift = pass * e.bits;
    for (uint32_t b = lane; b < bins; b += 64) base[wave][b] = 0;
    __syncthreads();
    for (uint32_t i = from + lane; i < to; i += 64) {
      const Pair p = pair_of(r, token, V, e, pass, i);
      atomicAdd(&base[wave][(p.key >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    // counts to first places: over the bins, and over a bin's waves
    uint32_t mine = 0, total;
    const uint32_t b = threadIdx.x;
    if (b < bins)
      for (int w = 0; w < 16; ++w) mine += base[w][b];
    uint32_t at = block_before<16>(mine, sm, total);
    if (b < bins)
      for (int w = 0; w < 16; ++w) {
        const uint32_t c = base[w][b];
        base[w][b] = at;
        at += c;
      }
    __syncthreads();
    uint32_t* const key = e.key[(pass + 1) & 1];
    uint32_t* const row = e.row[(pass + 1) & 1];
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
      const bool live = i0 + lane < to;
      Pair p{0, 0};
      if (live) p = pair_of(r, token, V, e, pass, i0 + lane);
      const uint32_t at = place(base[wave], (p.key >> shift) & (bins - 1), e.bits, live);
      if (live) {
        key[at] = p.key;
        row[at] = p.row;
      }
    }
    __threadfence_block();
    __syncthreads();
  }
}

// Long batches: each workgroup counts its pairs' digits, one adds the counts up, and each
// puts its pairs in their places.
__global__ __launch_bounds__(256) void embed_count_kernel(RowsArgs r, const int64_t* token, int64_t V, EmbedSort e, int pass) {
  __shared__ uint32_t count[kBinsMost];
  const uint32_t bins = 1u << e.bits;
  for (uint32_t b = threadIdx.x; b < bins; b += 256) count[b] = 0;
  __syncthreads();
  const uint32_t from = blockIdx.x * kSortKeys, to = r.n_slots - from < kSortKeys ? r.n_slots : from + kSortKeys;
  for (uint32_t i = from + threadIdx.x; i < to; i += 256)
    atomicAdd(&count[(pair_of(r, token, V, e, pass, i).key >> (pass * e.bits)) & (bins - 1)], 1u);
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += 256) e.count[(uint64_t)b * e.blocks + blockIdx.x] = count[b];
}
__global__ __launch_bounds__(1024) void embed_scan_kernel(EmbedSort e) {
  __shared__ uint32_t sm[16];
  const uint32_t n = (1u << e.bits) * e.blocks;
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
__global__ __launch_bounds__(256) void embed_place_kernel(RowsArgs r, const int64_t* token, int64_t V, EmbedSort e, int pass) {
  __shared__ uint32_t base[4][kBinsMost];
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6), shift = pass * e.bits;
  const uint32_t bins = 1u << e.bits;
  const uint32_t end = r.n_slots, first = blockIdx.x * kSortKeys + wave * (kSortKeys / 4);
  const uint32_t from = first < end ? first : end, to = end - from < kSortKeys / 4 ? end : from + kSortKeys / 4;
  for (uint32_t b = lane; b < bins; b += 64) base[wave][b] = 0;
  __syncthreads();
  for (uint32_t i = from + lane; i < to; i += 64)
    atomicAdd(&base[wave][(pair_of(r, token, V, e, pass, i).key >> shift) & (bins - 1)], 1u);
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += 256) {
    uint32_t at = e.count[(uint64_t)b * e.blocks + blockIdx.x];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t c = base[w][b];
      base[w][b] = at;
      at += c;
    }
  }
  __syncthreads();
  uint32_t* const key = e.key[(pass + 1) & 1];
  uint32_t* const row = e.row[(pass + 1) & 1];
  for (uint32_t i0 = from; i0 < to; i0 += 64) {
    const bool live = i0 + lane < to;
    Pair p{0, 0};
    if (live) p = pair_of(r, token, V, e, pass, i0 + lane);
    const uint32_t at = place(base[wave], (p.key >> shift) & (bins - 1), e.bits, live);
    if (live) {
      key[at] = p.key;
      row[at] = p.row;
    }
  }
}

// ----------------------------------------------------------------------------
// sums of a token's rows
// ----------------------------------------------------------------------------
// First of the sorted keys that is not below (or, ABOVE, that is above) `key`.
template <bool ABOVE>
__device__ inline uint32_t bound_of(const uint32_t* keys, uint32_t n, uint32_t key) {
  uint32_t lo = 0, hi = n;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) >> 1;
    if (ABOVE ? keys[mid] <= key : keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

template <typename T, int N>
__device__ inline void put_sum(const EmbedGradArgs& a, uint32_t v, int c, float (&sum)[N]) {
  T* const out = (T*)a.dtable + (int64_t)v * a.ldt + c;
  if (a.accumulate) {
    float was[N];
    load_n<T, N>(out, a.d - c, was);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = sum[e] * a.scale + was[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] *= a.scale;
  }
  store_n<T, N>(out, a.d - c, sum);
}

// A wave takes 64 N columns of a part of the sorted pairs, or zeroes rows of tokens that the
// batch does not hold.
constexpr uint32_t kZeroRows = 16;
template <typename G, typename T, int N>
__device__ inline void embed_sum(const EmbedGradArgs& a, uint32_t parts, uint32_t cuts, uint64_t unit) {
  const int lane = threadIdx.x & 63;
  if (unit >= (uint64_t)parts * cuts) {
    const int64_t v0 = (int64_t)(unit - (uint64_t)parts * cuts) * kZeroRows;
    bool absent = false;
    if (lane < (int)kZeroRows && v0 + lane < a.V) {
      const uint32_t v = (uint32_t)(v0 + lane), at = bound_of<false>(a.key, a.n, v);
      absent = at == a.n || a.key[at] != v;
    }
    const uint64_t rows = __ballot(absent);
    const float zero[N] = {};
    for (uint32_t k = 0; k < kZeroRows; ++k) {
      if (!((rows >> k) & 1)) continue;
      T* const out = (T*)a.dtable + (v0 + k) * a.ldt;
      for (int c = lane * N; c < a.d; c += 64 * N) store_n<T, N>(out + c, a.d - c, zero);
    }
    return;
  }
  const uint32_t part = (uint32_t)(unit / cuts), cut = (uint32_t)(unit % cuts);
  const int c = (int)(cut * 64 + lane) * N;
  const uint32_t from = part * kEmbedPart, to = a.n - from < kEmbedPart ? a.n : from + kEmbedPart;
  const uint32_t V = (uint32_t)a.V;
  const int n = a.d - c > 0 ? a.d - c : 0;
  float sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0.f;
  uint32_t cur = wave_uniform(a.key[from]);
  if (cur == V) return;
  bool before = from > 0 && wave_uniform(a.key[from - 1]) == cur;  // cur's rows began in an earlier part
  constexpr int U = 4;
  for (uint32_t i = from; i < to; i += U) {
    float x[U][N];
    uint32_t key[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t j = i + u < to ? i + u : to - 1;
      key[u] = i + u < to ? wave_uniform(a.key[j]) : V;
      const bool there = key[u] != V;
      load_n<G, N>((const G*)a.dout + (int64_t)(there ? wave_uniform(a.row[j]) : 0u) * a.ldd + c, there ? n : 0, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u < to && key[u] != cur) {
        if (before) store_n<float, N>(a.part + (int64_t)part * 2 * a.d + c, n, sum);
        else put_sum<T, N>(a, cur, c, sum);
        before = false;
        cur = key[u];
        if (cur == V) return;
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] += x[u][e];
    }
  }
  const bool on = to < a.n && wave_uniform(a.key[to]) == cur;
  if (!before && !on) put_sum<T, N>(a, cur, c, sum);
  else store_n<float, N>(a.part + ((int64_t)part * 2 + (before ? 0 : 1)) * a.d + c, n, sum);
}
template <typename G, typename T, int N>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a, uint32_t parts, uint32_t cuts, uint64_t units) {
  for (uint64_t unit = (uint64_t)blockIdx.x * 4 + wave_uniform(threadIdx.x >> 6); unit < units; unit += (uint64_t)gridDim.x * 4)
    embed_sum<G, T, N>(a, parts, cuts, unit);
}

// Joins the sums of a token that begins in a part and goes on behind it: each of the four
// waves an equal share of the following parts, in fp64.
template <typename T, int N>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a, uint32_t parts, uint32_t cuts) {
  __shared__ double sm[3][N][64];
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  for (uint64_t block = blockIdx.x; block < (uint64_t)(parts - 1) * cuts; block += gridDim.x) {
  const uint32_t part = (uint32_t)(block / cuts), cut = (uint32_t)(block % cuts);
  const uint32_t to = (part + 1) * kEmbedPart;  // not the last part: it has nothing behind it
  const uint32_t cur = wave_uniform(a.key[to - 1]);
  if (cur == (uint32_t)a.V || wave_uniform(a.key[to]) != cur) continue;
  const uint32_t from = part * kEmbedPart;
  if (wave_uniform(a.key[from]) == cur && from > 0 && wave_uniform(a.key[from - 1]) == cur) continue;
  const uint32_t last = (bound_of<true>(a.key, a.n, cur) - 1) / kEmbedPart;  // the part that holds its last row
  const int c = (int)(cut * 64 + lane) * N;
  const int n = a.d - c > 0 ? a.d - c : 0;
  const uint32_t each = (last - part + 3) / 4;
  const uint32_t k0 = part + 1 + wave * each, k1 = k0 + each < last + 1 ? k0 + each : last + 1;
  double sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) sum[e] = 0;
  if (wave == 0) {
    float x[N];
    load_n<float, N>(a.part + ((int64_t)part * 2 + 1) * a.d + c, n, x);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = x[e];
  }
#pragma unroll 4
  for (uint32_t k = k0; k < k1; ++k) {
    float x[N];
    load_n<float, N>(a.part + (int64_t)k * 2 * a.d + c, n, x);
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

template <typename T, typename O, int N>
hipError_t embed_rows(const RowsArgs& r, const EmbedArgs& a, hipStream_t s) {
  const uint32_t cuts = (uint32_t)((a.d + 256 * N - 1) / (256 * N));
  const uint64_t units = (uint64_t)r.n_slots * cuts;
  hipLaunchKernelGGL((embed_kernel<T, O, N>), dim3(grid_of((units + 3) / 4)), dim3(256), 0, s, r, a, cuts);
  return hipGetLastError();
}
template <typename G, typename T, int N>
hipError_t embed_sums(const EmbedGradArgs& a, hipStream_t s) {
  const uint32_t parts = (a.n + kEmbedPart - 1) / kEmbedPart, cuts = (uint32_t)((a.d + 64 * N - 1) / (64 * N));
  const uint64_t zero = a.accumulate ? 0 : ((uint64_t)a.V + kZeroRows - 1) / kZeroRows;
  const uint64_t units = (uint64_t)parts * cuts + zero;
  hipLaunchKernelGGL((embed_sum_kernel<G, T, N>), dim3(grid_of((units + 3) / 4)), dim3(256), 0, s, a, parts, cuts, units);
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
      return embed_rows<decltype(t), decltype(o), 2>(r, a, s);
    });
  });
}

hipError_t launch_embed_sort(const RowsArgs& r, const int64_t* token, int64_t V, const EmbedSort& e, hipStream_t s) {
  if (r.n_slots <= kSortOneMost) {
    hipLaunchKernelGGL(embed_sort_one_kernel, dim3(1), dim3(1024), 0, s, r, token, V, e);
    return hipGetLastError();
  }
  for (int pass = 0; pass < e.passes; ++pass) {
    hipLaunchKernelGGL(embed_count_kernel, dim3(e.blocks), dim3(256), 0, s, r, token, V, e, pass);
    hipLaunchKernelGGL(embed_scan_kernel, dim3(1), dim3(1024), 0, s, e);
    hipLaunchKernelGGL(embed_place_kernel, dim3(e.blocks), dim3(256), 0, s, r, token, V, e, pass);
    const hipError_t st = hipGetLastError();
    if (st != hipSuccess) return st;
  }
  return hipSuccess;
}

hipError_t launch_embed_grad(int dout_dtype, int table_dtype, const EmbedGradArgs& a, hipStream_t s) {
  return with_type(dout_dtype, [&](auto g) {
    return with_type(table_dtype, [&](auto t) {
      if (a.d > 256) return embed_sums<decltype(g), decltype(t), 8>(a, s);
      if (a.d > 64) return embed_sums<decltype(g), decltype(t), 4>(a, s);
      return embed_sums<decltype(g), decltype(t), 1>(a, s);
    });
  });
}

}  // namespace attr
