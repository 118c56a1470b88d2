// C-ABI layer of libattr: argument validation, workspace layout and kernel
// dispatch.  Every check runs on the host before anything is enqueued, so a
// rejected call leaves all outputs untouched.  See include/attr.h for the
// contract of each entry point.
#include "attr.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <exception>
#include <numeric>
#include <string>
#include <map>
#include <tuple>
#include <vector>

#include "kernels.h"
#include "project_plan.h"
#include "syrk_plan.h"

namespace {

thread_local std::string g_err;

attr_status fail(attr_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_err = buf;
  return st;
}

attr_status device_fail(hipError_t e, const char* what) {
  return fail(ATTR_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

int dtype_bytes(attr_dtype d) { return d == ATTR_F32 ? 4 : 2; }

bool valid_dtype(attr_dtype d) { return d == ATTR_F32 || d == ATTR_BF16 || d == ATTR_F16; }

// Byte range [lo, hi) spanned by a row-major [rows, width] matrix with stride ld.
struct Span {
  uintptr_t lo, hi;
};
Span span_of(const void* p, int64_t rows, int64_t width, int64_t ld, int eb) {
  uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  if (rows <= 0 || width <= 0) return {lo, lo};
  return {lo, lo + (uintptr_t)(((rows - 1) * ld + width) * eb)};
}
bool overlap(Span a, Span b) { return a.lo < b.hi && b.lo < a.hi; }

// ---------------------------------------------------------------------------
// projection
// ---------------------------------------------------------------------------
struct ProjLayout {
  size_t off_tab, off_gtab, off_wl, off_pk, off_part, total;
  attr::ProjFewPlan few;  // ct = 0: the general kernel
  size_t query;           // bytes that the workspace query returns
  std::vector<int> order;       // slot -> module index
  std::vector<size_t> pk_off;   // per slot, relative to off_pk
  std::vector<int> slot_grp;    // slot -> group
  std::vector<int> lead_ms;     // slot -> group size if the group's first slot, else 0
  int n_groups;
  int n_chunks;
};

ProjLayout project_layout(const attr_module* mods, int32_t n_mods, int eb, int64_t n_ex,
                          int64_t T, int k, bool tok = false, bool ragged = false) {
  ProjLayout L;
  const int nk = k / 16;
  // Modules that read the same input rows (same a, lda and d_in: q/k/v or
  // gate/up of a transformer layer) form groups of up to kProjGroupMax,
  // projected together so that a is read once.  Groups are ordered by their
  // work per token (the row elements they read), largest first, so that the
  // one main launch starts the longest items first and ends on the
  // shortest; a group's members take consecutive slots.
  // (three members at k = 64 would need more than the 512 registers of a wave
  // that has its SIMD alone, so groups stop at two there; per-token blocks keep
  // one module per item: their row-writing code would pass the 256 of two waves)
  const size_t gmax = tok ? 1 : (nk >= 4 ? 2 : (size_t)attr::kProjGroupMax);
  std::vector<std::vector<int>> groups;
  std::map<std::tuple<const void*, int64_t, int64_t>, size_t> open;
  for (int x = 0; x < n_mods; ++x) {
    const auto key = std::make_tuple(mods[x].a, (int64_t)mods[x].lda, (int64_t)mods[x].d_in);
    auto it = open.find(key);
    if (it != open.end() && groups[it->second].size() < gmax) {
      groups[it->second].push_back(x);
    } else {
      open[key] = groups.size();
      groups.push_back({x});
    }
  }
  auto cost = [&](const std::vector<int>& gm) {
    int64_t c = mods[gm[0]].d_in;
    for (int x : gm) c += mods[x].d_out;
    return c;
  };
  std::stable_sort(groups.begin(), groups.end(),
                   [&](const std::vector<int>& x, const std::vector<int>& y) {
                     return cost(x) > cost(y);
                   });
  L.n_groups = (int)groups.size();
  for (int gi = 0; gi < L.n_groups; ++gi) {
    const auto& gm = groups[gi];
    for (size_t u = 0; u < gm.size(); ++u) {
      L.order.push_back(gm[u]);
      L.slot_grp.push_back(gi);
      L.lead_ms.push_back(u == 0 ? (int)gm.size() : 0);
    }
  }
  const int CT = attr::project_chunk_tokens(nk, tok);
  L.n_chunks = (int)((T + CT - 1) / CT);
  L.off_tab = 0;
  size_t off = align_up(sizeof(attr::ProjTab) * (size_t)n_mods);
  L.off_gtab = off;
  off += align_up(sizeof(attr::ProjGroup) * (size_t)L.n_groups);
  // work list (examples by chunk count, chunk-row offsets), whether or not
  // the call passes lengths: the query has no lengths to look at
  L.off_wl = off;
  if (n_ex <= attr::kWorklistMaxExamples && L.n_chunks <= attr::kWorklistMaxChunks)
    off += align_up(4 * (size_t)n_ex) + align_up(4 * ((size_t)L.n_chunks + 1));
  L.off_pk = off;
  size_t pk = 0;
  L.pk_off.resize(n_mods);
  for (int sl = 0; sl < n_mods; ++sl) {
    const attr_module& m = mods[L.order[sl]];
    L.pk_off[sl] = pk;
    pk += align_up(attr::project_packed_bytes(m.d_in, m.d_out, k, eb));
  }
  off += pk;
  L.off_part = off;
  // per-token blocks have no partials; without them the ungrouped call's larger
  // group table fits what the query (which does not know the call) returns
  if (!tok) off += align_up((size_t)n_mods * (size_t)L.n_chunks * (size_t)n_ex * (size_t)k * k * 4);
  L.total = off;
  int64_t slot_cost = 0, longest = 0;
  for (int x = 0; x < n_mods; ++x) {
    slot_cost += mods[x].d_in + mods[x].d_out;
    longest = std::max(longest, mods[x].d_in + mods[x].d_out);
  }
  // the plan of this call, and the bytes of the larger of the plans with and
  // without lengths: the query does not know which the call will have
  L.query = L.total;
  for (const bool r : {!ragged, ragged}) {
    L.few = attr::plan_project_few(eb == 2, nk, tok, slot_cost, longest, n_mods, n_ex, T, r);
    size_t few_total = L.off_part;  // the few-item plan's partials are there too
    if (L.few.ct && L.few.n_chunks > 1 && !tok && n_ex > 0)
      few_total += align_up(attr::project_few_query(L.few, (size_t)n_mods * (size_t)n_ex * (size_t)k * k * 4));
    L.query = std::max(L.query, few_total);
  }
  return L;
}

attr_status project_validate(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                             int32_t k, int64_t n_ex, int64_t T, float* out, int64_t ldo) {
  if (n_mods < 1 || n_mods > 4096) return fail(ATTR_ERR_INVALID_ARG, "n_mods=%d must be in [1, 4096]", n_mods);
  if (!mods) return fail(ATTR_ERR_INVALID_ARG, "mods is NULL");
  if (in_dtype != ATTR_BF16 && in_dtype != ATTR_F32)
    return fail(ATTR_ERR_UNSUPPORTED, "attr_project: in_dtype must be ATTR_BF16 or ATTR_F32");
  if (k != 16 && k != 32 && k != 64) return fail(ATTR_ERR_UNSUPPORTED, "k=%d must be 16, 32 or 64", k);
  if (n_ex < 0) return fail(ATTR_ERR_INVALID_ARG, "n_examples=%lld is negative", (long long)n_ex);
  if (T < 1) return fail(ATTR_ERR_INVALID_ARG, "T=%lld must be >= 1", (long long)T);
  if (T > (1ll << 24)) return fail(ATTR_ERR_UNSUPPORTED, "T=%lld exceeds 2^24", (long long)T);
  if (n_ex > 0 && !out) return fail(ATTR_ERR_INVALID_ARG, "out is NULL");
  if (!aligned16(out)) return fail(ATTR_ERR_ALIGNMENT, "out must be 16-byte aligned");
  const int eb = dtype_bytes(in_dtype);
  // Rows are streamed in 128-byte groups: 64 bf16 or 32 fp32 values.
  const int KS = in_dtype == ATTR_BF16 ? 64 : 32;
  const int ld_mult = 16 / eb;
  const int64_t kk = (int64_t)k * k;
  if (ldo < kk) return fail(ATTR_ERR_INVALID_ARG, "ldo=%lld < k*k", (long long)ldo);
  std::vector<std::pair<int64_t, int>> cols;
  for (int j = 0; j < n_mods; ++j) {
    const attr_module& m = mods[j];
    if (!m.a || !m.g || !m.R || !m.S) return fail(ATTR_ERR_INVALID_ARG, "module %d: NULL pointer", j);
    if (m.d_in <= 0 || m.d_out <= 0 || m.d_in > 65536 || m.d_out > 65536)
      return fail(ATTR_ERR_INVALID_ARG, "module %d: d_in=%lld d_out=%lld must be in [1, 65536]", j,
                  (long long)m.d_in, (long long)m.d_out);
    if (m.d_in % KS || m.d_out % KS)
      return fail(ATTR_ERR_ALIGNMENT, "module %d: d_in=%lld d_out=%lld must be multiples of %d", j,
                  (long long)m.d_in, (long long)m.d_out, KS);
    if (m.lda < m.d_in || m.ldg < m.d_out)
      return fail(ATTR_ERR_INVALID_ARG, "module %d: lda/ldg smaller than the row width", j);
    if (m.lda % ld_mult || m.ldg % ld_mult)
      return fail(ATTR_ERR_ALIGNMENT, "module %d: lda/ldg must be multiples of %d elements", j, ld_mult);
    if (!aligned16(m.a) || !aligned16(m.g) || !aligned16(m.R) || !aligned16(m.S))
      return fail(ATTR_ERR_ALIGNMENT, "module %d: pointers must be 16-byte aligned", j);
    if ((m.v_out == nullptr) != (m.v_in == nullptr))
      return fail(ATTR_ERR_INVALID_ARG, "module %d: v_out and v_in must both be set or both NULL", j);
    if ((reinterpret_cast<uintptr_t>(m.v_out) | reinterpret_cast<uintptr_t>(m.v_in)) & 3u)
      return fail(ATTR_ERR_ALIGNMENT, "module %d: v_out / v_in must be 4-byte aligned", j);
    if (m.lda * 256 * eb >= (1ll << 31) || m.ldg * 256 * eb >= (1ll << 31))
      return fail(ATTR_ERR_UNSUPPORTED, "module %d: row stride too large", j);
    if (m.out_col < 0 || m.out_col + kk > ldo)
      return fail(ATTR_ERR_INVALID_ARG, "module %d: out_col=%lld + k*k exceeds ldo=%lld", j,
                  (long long)m.out_col, (long long)ldo);
    cols.push_back({m.out_col, j});
  }
  std::sort(cols.begin(), cols.end());
  for (size_t j = 1; j < cols.size(); ++j)
    if (cols[j].first < cols[j - 1].first + kk)
      return fail(ATTR_ERR_INVALID_ARG, "modules %d and %d write overlapping output columns",
                  cols[j - 1].second, cols[j].second);
  return ATTR_OK;
}

}  // namespace

extern "C" {

const char* attr_last_error(void) { return g_err.c_str(); }

const char* attr_status_string(attr_status st) {
  switch (st) {
    case ATTR_OK: return "ATTR_OK";
    case ATTR_ERR_INVALID_ARG: return "ATTR_ERR_INVALID_ARG";
    case ATTR_ERR_UNSUPPORTED: return "ATTR_ERR_UNSUPPORTED";
    case ATTR_ERR_ALIGNMENT: return "ATTR_ERR_ALIGNMENT";
    case ATTR_ERR_WORKSPACE: return "ATTR_ERR_WORKSPACE";
    case ATTR_ERR_DEVICE: return "ATTR_ERR_DEVICE";
  }
  return "ATTR_UNKNOWN_STATUS";
}

int attr_abi_version(void) { return ATTR_ABI_VERSION; }

// ---------------------------------------------------------------------------
size_t attr_project_workspace_size(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                   int64_t n_examples, int64_t T, int32_t k) {
  try {
    if (!mods || n_mods < 1 || n_mods > 4096 || (k != 16 && k != 32 && k != 64) || T < 1 ||
        n_examples < 0 || (in_dtype != ATTR_BF16 && in_dtype != ATTR_F32))
      return 0;
    return project_layout(mods, n_mods, dtype_bytes(in_dtype), n_examples, T, k).query;
  } catch (...) {
    return 0;
  }
}

// tok: per-token blocks into out rows [0, n_rows) (attr_project_tokens),
// else per-example rows (attr_project).
static attr_status project_impl(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                int32_t k, int64_t n_examples, int64_t T,
                                const int64_t* row_offset, const int32_t* length, float* out,
                                int64_t ldo, void* ws, size_t ws_bytes, void* stream, bool tok,
                                int64_t n_rows) {
  try {
    g_err.clear();
    attr_status st = project_validate(mods, n_mods, in_dtype, k, n_examples, T, out, ldo);
    if (st != ATTR_OK) return st;
    if (tok && n_rows < 0) return fail(ATTR_ERR_INVALID_ARG, "n_rows=%lld is negative", (long long)n_rows);
    if (n_examples == 0) return ATTR_OK;
    const int eb = dtype_bytes(in_dtype);
    ProjLayout L = project_layout(mods, n_mods, eb, n_examples, T, k, tok, length != nullptr);
    if (!ws || ws_bytes < L.total)
      return fail(ATTR_ERR_WORKSPACE, "attr_project needs %zu workspace bytes, got %zu", L.total,
                  ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u)
      return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    const int64_t nblk = (int64_t)n_mods * L.n_chunks * n_examples;
    if (nblk > (1ll << 24))
      return fail(ATTR_ERR_UNSUPPORTED, "attr_project: %lld work items exceed one launch; split the batch",
                  (long long)nblk);
    // The few-item plan's chunks come in rounds of as many as a launch takes and
    // a workspace below the queried size holds partials for: the same bits.
    const bool few_parts = !tok && L.few.n_chunks > 1;
    const int64_t items = (int64_t)n_mods * n_examples;
    const int round = attr::project_few_round(L.few, items, ws_bytes - L.off_part,
                                              few_parts ? (size_t)items * (size_t)k * k * 4 : 0);
    if (L.few.ct ? round < 1 : std::max(items, (int64_t)L.n_groups * L.n_chunks * n_examples) > attr::kProjectMaxBlocks)
      return fail(ATTR_ERR_UNSUPPORTED, "attr_project: %lld modules x examples exceed one launch; split the batch",
                  (long long)items);
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* base = static_cast<char*>(ws);
    attr::ProjTab* tab = reinterpret_cast<attr::ProjTab*>(base + L.off_tab);
    attr::ProjGroup* gtab = reinterpret_cast<attr::ProjGroup*>(base + L.off_gtab);
    char* pk = base + L.off_pk;
    float* part = reinterpret_cast<float*>(base + L.off_part);
    const bool bf16 = in_dtype == ATTR_BF16;
    const int nk = k / 16;
    for (int s0 = 0; s0 < n_mods; s0 += attr::kPackMax) {
      attr::PackArgs pa;
      std::memset(&pa, 0, sizeof(pa));
      pa.n = std::min(attr::kPackMax, n_mods - s0);
      pa.slot0 = s0;
      for (int j = 0; j < pa.n; ++j) {
        const attr_module& m = mods[L.order[s0 + j]];
        attr::PackEntry& e = pa.e[j];
        e.a = m.a;
        e.g = m.g;
        e.R = m.R;
        e.S = m.S;
        e.lda = (int32_t)m.lda;
        e.ldg = (int32_t)m.ldg;
        e.out_col = m.out_col;
        e.pk_off = (uint32_t)(L.pk_off[s0 + j] / 256);  // module fragments are 256-byte aligned
        e.d_in = (int32_t)m.d_in;
        e.d_out = (int32_t)m.d_out;
        e.v_out = m.v_out;
        e.v_in = m.v_in;
        e.grp = (int16_t)L.slot_grp[s0 + j];
        e.lead_ms = (int16_t)L.lead_ms[s0 + j];
      }
      hipError_t e = attr::launch_project_pack(bf16, nk, pa, tab, gtab, pk, s);
      if (e != hipSuccess) return device_fail(e, "attr_project pack launch");
    }
    hipError_t e;
    if (L.few.ct) {
      for (int c0 = 0; c0 < L.few.n_chunks; c0 += round) {
        const int nc = std::min(round, L.few.n_chunks - c0);
        e = attr::launch_project_few(bf16, nk, L.few, c0, nc, tab, n_mods, n_examples, T, row_offset, length,
                                     few_parts ? part : out, tok, ldo, n_rows, s);
        if (e != hipSuccess) return device_fail(e, "attr_project main launch");
        if (!few_parts) continue;
        e = attr::launch_project_reduce(nk, L.few.ct, c0, nc, tab, n_mods, n_examples, T, length, part, out,
                                        ldo, s);
        if (e != hipSuccess) return device_fail(e, "attr_project reduce launch");
      }
      return ATTR_OK;
    }
    int32_t* wl_perm = nullptr;
    int32_t* wl_off = nullptr;
    if (attr::project_uses_worklist(length, n_examples, L.n_chunks)) {
      wl_perm = reinterpret_cast<int32_t*>(base + L.off_wl);
      wl_off = reinterpret_cast<int32_t*>(base + L.off_wl + align_up(4 * (size_t)n_examples));
    }
    e = attr::launch_project_main(bf16, nk, tab, gtab, L.n_groups, L.n_chunks, n_examples, T,
                                  row_offset, length, wl_perm, wl_off, tok ? out : part, s, tok, ldo,
                                  n_rows);
    if (e != hipSuccess) return device_fail(e, "attr_project main launch");
    if (tok) return ATTR_OK;
    e = attr::launch_project_reduce(nk, attr::project_chunk_tokens(nk, false), 0, L.n_chunks, tab, n_mods, n_examples, T, length,
                                    part, out, ldo, s);
    if (e != hipSuccess) return device_fail(e, "attr_project reduce launch");
    return ATTR_OK;
  } catch (const std::exception& ex) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_project: host exception: %s", ex.what());
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_project: unknown host exception");
  }
}

attr_status attr_project(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype, int32_t k,
                         int64_t n_examples, int64_t T, const int64_t* row_offset,
                         const int32_t* length, float* out, int64_t ldo, void* ws,
                         size_t ws_bytes, void* stream) {
  return project_impl(mods, n_mods, in_dtype, k, n_examples, T, row_offset, length, out, ldo, ws,
                      ws_bytes, stream, false, 0);
}

attr_status attr_project_tokens(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                int32_t k, int64_t n_examples, int64_t T,
                                const int64_t* row_offset, const int32_t* length, float* out,
                                int64_t ldo, int64_t n_rows, void* ws, size_t ws_bytes,
                                void* stream) {
  return project_impl(mods, n_mods, in_dtype, k, n_examples, T, row_offset, length, out, ldo, ws,
                      ws_bytes, stream, true, n_rows);
}

attr_status attr_project_noalloc(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                 int32_t k, int64_t n_examples, int64_t T,
                                 const int64_t* row_offset, const int32_t* length, float* out,
                                 int64_t ldo, void* stream) {
  try {
    g_err.clear();
    attr_status st = project_validate(mods, n_mods, in_dtype, k, n_examples, T, out, ldo);
    if (st != ATTR_OK) return st;
    if (n_examples == 0) return ATTR_OK;
    // the size check comes first: a call that cannot fit touches no device state
    const size_t need = project_layout(mods, n_mods, dtype_bytes(in_dtype), n_examples, T, k).total;
    if (need > attr::kProjectScratchBytes)
      return fail(ATTR_ERR_WORKSPACE,
                  "attr_project_noalloc: the call needs %zu bytes of scratch, the static buffer "
                  "holds %zu; split the batch or call attr_project with a workspace",
                  need, attr::kProjectScratchBytes);
    void* scratch = nullptr;
    const hipError_t e = attr::project_scratch(&scratch);
    if (e != hipSuccess) return device_fail(e, "attr_project_noalloc: static scratch address");
    return project_impl(mods, n_mods, in_dtype, k, n_examples, T, row_offset, length, out, ldo,
                        scratch, attr::kProjectScratchBytes, stream, false, 0);
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_project_noalloc: host exception");
  }
}

// ---------------------------------------------------------------------------
size_t attr_precond_accumulate_workspace_size(int64_t n_rows, int64_t D, attr_dtype x_dtype,
                                              attr_precond mode) {
  (void)x_dtype;
  if (n_rows <= 0 || D < 1) return 0;
  if (mode == ATTR_PRECOND_DIAG)
    return align_up((size_t)attr::colsumsq_panels(n_rows, D) * (size_t)D * sizeof(double));
  if (mode == ATTR_PRECOND_FULL) {
    const attr::SyrkPlan P = attr::plan_syrk(n_rows, D, 0);  // any stride's plan fits in it
    return align_up(P.part_bytes) + align_up(P.h64_bytes);
  }
  return 0;
}

attr_status attr_precond_accumulate(const void* X, attr_dtype x_dtype, int64_t n_rows, int64_t D,
                                    int64_t ldx, attr_precond mode, float* H, void* ws,
                                    size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    if (mode != ATTR_PRECOND_DIAG && mode != ATTR_PRECOND_FULL)
      return fail(ATTR_ERR_UNSUPPORTED, "attr_precond_accumulate: mode must be DIAG or FULL");
    if (!valid_dtype(x_dtype)) return fail(ATTR_ERR_UNSUPPORTED, "unknown x_dtype");
    const bool full = mode == ATTR_PRECOND_FULL;
    if (full && x_dtype == ATTR_F32)
      return fail(ATTR_ERR_UNSUPPORTED, "attr_precond_accumulate: FULL takes ATTR_F16 or ATTR_BF16 rows");
    if (n_rows < 0) return fail(ATTR_ERR_INVALID_ARG, "n_rows is negative");
    if (D < 1) return fail(ATTR_ERR_INVALID_ARG, "D must be >= 1");
    if (D % 8) return fail(ATTR_ERR_ALIGNMENT, "D=%lld must be a multiple of 8", (long long)D);
    if (ldx < D) return fail(ATTR_ERR_INVALID_ARG, "ldx < D");
    const int eb = dtype_bytes(x_dtype);
    if (ldx % (16 / eb)) return fail(ATTR_ERR_ALIGNMENT, "ldx must keep rows 16-byte aligned");
    if (!H) return fail(ATTR_ERR_INVALID_ARG, "H is NULL");
    if (n_rows > 0 && !X) return fail(ATTR_ERR_INVALID_ARG, "X is NULL");
    if (!aligned16(X) || !aligned16(H)) return fail(ATTR_ERR_ALIGNMENT, "X and H must be 16-byte aligned");
    if (full && D % 64) return fail(ATTR_ERR_ALIGNMENT, "FULL needs D a multiple of 64");
    if (full && D > 32768) return fail(ATTR_ERR_UNSUPPORTED, "FULL needs D <= 32768");
    if (full && ldx > 65536)
      return fail(ATTR_ERR_UNSUPPORTED, "FULL needs ldx <= 65536 (64-row stages of K-slices of at "
                  "least 16384 rows, each slice spanning at most 2 GiB)");
    if (overlap(span_of(X, n_rows, D, ldx, eb), span_of(H, full ? D : 1, D, D, 4)))
      return fail(ATTR_ERR_INVALID_ARG, "X and H overlap");
    if (n_rows == 0) return ATTR_OK;
    const size_t need = attr_precond_accumulate_workspace_size(n_rows, D, x_dtype, mode);
    if (!ws || ws_bytes < need)
      return fail(ATTR_ERR_WORKSPACE, "attr_precond_accumulate needs %zu workspace bytes", need);
    if (reinterpret_cast<uintptr_t>(ws) & 255u)
      return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    if (n_rows > (1ll << 40)) return fail(ATTR_ERR_UNSUPPORTED, "n_rows too large");
    hipError_t e;
    if (full) {
      const attr::SyrkPlan P = attr::plan_syrk(n_rows, D, ldx);
      if (P.Cs * ldx * 2 > (1ll << 31))
        return fail(ATTR_ERR_UNSUPPORTED, "internal: SYRK slice of %lld rows spans more than 2 GiB",
                    (long long)P.Cs);
      char* part = static_cast<char*>(ws);
      char* h64 = part + align_up(P.part_bytes);
      e = attr::launch_syrk(x_dtype == ATTR_BF16, X, ldx, n_rows, D, H, P, part, h64,
                            static_cast<hipStream_t>(stream));
    } else {
      e = attr::launch_colsumsq((int)x_dtype, X, ldx, n_rows, D, H, static_cast<double*>(ws),
                                static_cast<hipStream_t>(stream));
    }
    if (e != hipSuccess) return device_fail(e, "attr_precond_accumulate launch");
    return ATTR_OK;
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_precond_accumulate: host exception");
  }
}

// ---------------------------------------------------------------------------
size_t attr_precond_apply_workspace_size(int64_t n_rows, int64_t D, attr_precond mode) {
  if (mode != ATTR_PRECOND_FULL || n_rows <= 0 || D < 1) return 0;
  return attr::apply_full_workspace(n_rows, D, 1);  // the few-row path fits in it
}

attr_status attr_precond_apply(const void* X, attr_dtype x_dtype, int64_t n_rows, int64_t D,
                               int64_t ldx, attr_precond mode, const float* M,
                               int32_t unit_normalize, void* Y, attr_dtype y_dtype, int64_t ldy,
                               void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    if (mode != ATTR_PRECOND_NONE && mode != ATTR_PRECOND_DIAG && mode != ATTR_PRECOND_FULL)
      return fail(ATTR_ERR_UNSUPPORTED, "unknown preconditioner mode");
    if ((x_dtype != ATTR_F32 && x_dtype != ATTR_F16) || (y_dtype != ATTR_F32 && y_dtype != ATTR_F16))
      return fail(ATTR_ERR_UNSUPPORTED, "attr_precond_apply: dtypes must be ATTR_F32 or ATTR_F16");
    const bool full = mode == ATTR_PRECOND_FULL;
    if (full && x_dtype != ATTR_F16)
      return fail(ATTR_ERR_UNSUPPORTED, "attr_precond_apply: FULL takes ATTR_F16 rows");
    if (n_rows < 0) return fail(ATTR_ERR_INVALID_ARG, "n_rows is negative");
    if (D < 1) return fail(ATTR_ERR_INVALID_ARG, "D must be >= 1");
    if (D % 8) return fail(ATTR_ERR_ALIGNMENT, "D=%lld must be a multiple of 8", (long long)D);
    if (ldx < D || ldy < D) return fail(ATTR_ERR_INVALID_ARG, "ldx/ldy < D");
    const int xb = dtype_bytes(x_dtype), yb = dtype_bytes(y_dtype);
    if (ldx % (16 / xb) || ldy % (16 / yb))
      return fail(ATTR_ERR_ALIGNMENT, "ldx/ldy must keep rows 16-byte aligned");
    if (n_rows > 0 && (!X || !Y)) return fail(ATTR_ERR_INVALID_ARG, "X or Y is NULL");
    if (mode == ATTR_PRECOND_DIAG && !M) return fail(ATTR_ERR_INVALID_ARG, "DIAG needs M");
    if (full && !M) return fail(ATTR_ERR_INVALID_ARG, "FULL needs M");
    if (full && D % 64) return fail(ATTR_ERR_ALIGNMENT, "FULL needs D a multiple of 64");
    if (mode == ATTR_PRECOND_NONE && M) return fail(ATTR_ERR_INVALID_ARG, "NONE takes M = NULL");
    if (!aligned16(X) || !aligned16(Y) || !aligned16(M))
      return fail(ATTR_ERR_ALIGNMENT, "X, Y and M must be 16-byte aligned");
    const Span sx = span_of(X, n_rows, D, ldx, xb), sy = span_of(Y, n_rows, D, ldy, yb);
    const bool inplace = X == Y && x_dtype == y_dtype && ldx == ldy;
    if (!inplace && overlap(sx, sy)) return fail(ATTR_ERR_INVALID_ARG, "X and Y overlap");
    if (full && overlap(sx, sy)) return fail(ATTR_ERR_INVALID_ARG, "FULL cannot run in place");
    if (M && overlap(span_of(M, full ? D : 1, D, D, 4), sy))
      return fail(ATTR_ERR_INVALID_ARG, "M and Y overlap");
    if (n_rows == 0) return ATTR_OK;
    if (n_rows > (1ll << 31) - 1) return fail(ATTR_ERR_UNSUPPORTED, "n_rows exceeds one launch");
    if (full) {
      if (ldx * 256 * 2 >= (1ll << 31)) return fail(ATTR_ERR_UNSUPPORTED, "row stride too large");
      const size_t need = attr::apply_full_workspace(n_rows, D, unit_normalize ? 1 : 0);
      if (!ws || ws_bytes < need)
        return fail(ATTR_ERR_WORKSPACE, "attr_precond_apply (FULL) needs %zu workspace bytes", need);
      if (reinterpret_cast<uintptr_t>(ws) & 255u)
        return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
      const hipStream_t st = static_cast<hipStream_t>(stream);
      const attr::ApplyFewPlan few = attr::plan_apply_few(n_rows, D);
      hipError_t e = few.use ? attr::launch_apply_few(few, X, n_rows, ldx, D, M, (int)y_dtype, Y, ldy,
                                                      unit_normalize ? 1 : 0, ws, st)
                             : attr::launch_apply_full(X, n_rows, ldx, D, M, (int)y_dtype, Y, ldy,
                                                       unit_normalize ? 1 : 0, ws, st);
      if (e != hipSuccess) return device_fail(e, "attr_precond_apply (FULL) launch");
      return ATTR_OK;
    }
    hipError_t e = attr::launch_rowscale((int)x_dtype, (int)y_dtype, X, ldx, n_rows, D,
                                         mode == ATTR_PRECOND_DIAG ? M : nullptr, unit_normalize ? 1 : 0,
                                         nullptr, nullptr, 0, Y, ldy, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return device_fail(e, "attr_precond_apply launch");
    return ATTR_OK;
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_precond_apply: host exception");
  }
}

// ---------------------------------------------------------------------------
struct ScoreLayout {
  attr::ScorePlan plan;
  size_t off_s, off_i, off_p, total;
};

static ScoreLayout score_layout(int64_t n_q, int64_t n_g, int64_t D, int32_t k, int eb,
                                bool fewest_bytes = false) {
  ScoreLayout L{};
  L.plan = attr::plan_score(n_q, n_g, D, k, eb, fewest_bytes);
  if (n_q <= 0 || n_g <= 0) return L;
  const size_t n = L.plan.list_entries;
  L.off_s = 0;
  L.off_i = align_up(n * sizeof(float));
  L.off_p = L.off_i + align_up(n * sizeof(int64_t));
  L.total = L.off_p + align_up(L.plan.spart_bytes);
  return L;
}

size_t attr_score_topk_workspace_size(int64_t n_q, int64_t n_g, int64_t D, int32_t k) {
  if (n_q < 0 || n_g < 0 || k < 1 || k > 128 || D < 1) return 0;
  size_t total = 0;
  for (const int eb : {2, 4})
    for (const bool fewest : {false, true})
      total = std::max(total, score_layout(n_q, n_g, D, k, eb, fewest).total);
  return total;
}

attr_status attr_score_topk(const void* Q, int64_t n_q, int64_t ldq, const void* G, int64_t n_g,
                            int64_t ldg, attr_dtype dtype, int64_t D, int32_t k, int64_t index_base,
                            int32_t merge, float* top_score, int64_t* top_index, void* ws,
                            size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    if (dtype != ATTR_F16 && dtype != ATTR_F32)
      return fail(ATTR_ERR_UNSUPPORTED, "attr_score_topk: dtype must be ATTR_F16 or ATTR_F32");
    if (k < 1 || k > 128) return fail(ATTR_ERR_UNSUPPORTED, "attr_score_topk: k=%d must be in [1, 128]", k);
    if (n_q < 0 || n_g < 0) return fail(ATTR_ERR_INVALID_ARG, "n_q / n_g is negative");
    if (n_q > (1ll << 31) - 1 || n_g > (1ll << 31) - 1)
      return fail(ATTR_ERR_UNSUPPORTED, "n_q and n_g must be below 2^31 per call");
    if (D < 1) return fail(ATTR_ERR_INVALID_ARG, "D must be >= 1");
    const int eb = dtype_bytes(dtype);
    const int grp = dtype == ATTR_F16 ? 64 : 32;
    if (D % grp) return fail(ATTR_ERR_ALIGNMENT, "D=%lld must be a multiple of %d", (long long)D, grp);
    if (ldq < D || ldg < D) return fail(ATTR_ERR_INVALID_ARG, "ldq/ldg < D");
    if (ldq % (16 / eb) || ldg % (16 / eb))
      return fail(ATTR_ERR_ALIGNMENT, "ldq/ldg must keep rows 16-byte aligned");
    if (ldq * 256 * eb >= (1ll << 31) || ldg * 256 * eb >= (1ll << 31))
      return fail(ATTR_ERR_UNSUPPORTED, "row stride too large (256 rows must span < 2 GiB)");
    if (merge != 0 && merge != 1) return fail(ATTR_ERR_INVALID_ARG, "merge must be 0 or 1");
    if (index_base < 0 || index_base > (1ll << 62))
      return fail(ATTR_ERR_INVALID_ARG, "index_base must be in [0, 2^62]");
    if (n_q > 0 && (!Q || !top_score || !top_index))
      return fail(ATTR_ERR_INVALID_ARG, "Q / top_score / top_index is NULL");
    if (n_g > 0 && !G) return fail(ATTR_ERR_INVALID_ARG, "G is NULL");
    if (!aligned16(Q) || !aligned16(G) || !aligned16(top_score) || !aligned16(top_index))
      return fail(ATTR_ERR_ALIGNMENT, "Q, G, top_score and top_index must be 16-byte aligned");
    const Span ss = span_of(top_score, n_q, k, k, 4), si = span_of(top_index, n_q, k, k, 8);
    const Span sq = span_of(Q, n_q, D, ldq, eb), sg = span_of(G, n_g, D, ldg, eb);
    if (overlap(ss, si) || overlap(ss, sq) || overlap(ss, sg) || overlap(si, sq) || overlap(si, sg))
      return fail(ATTR_ERR_INVALID_ARG, "top_score / top_index overlap each other or the inputs");
    if (n_q == 0) return ATTR_OK;
    if (n_g == 0 && merge) return ATTR_OK;
    ScoreLayout L = score_layout(n_q, n_g, D, k, eb);
    if (L.total > (ws ? ws_bytes : 0)) L = score_layout(n_q, n_g, D, k, eb, true);
    if (L.total > 0 && (!ws || ws_bytes < L.total))
      return fail(ATTR_ERR_WORKSPACE, "attr_score_topk needs %zu workspace bytes", L.total);
    if (reinterpret_cast<uintptr_t>(ws) & 255u)
      return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    char* base = static_cast<char*>(ws);
    hipError_t e = attr::launch_score_topk(
        dtype == ATTR_F16, L.plan, Q, n_q, ldq, G, n_g, ldg, k, index_base, merge, top_score,
        top_index, base ? reinterpret_cast<float*>(base + L.off_s) : nullptr,
        base ? reinterpret_cast<int64_t*>(base + L.off_i) : nullptr,
        base ? reinterpret_cast<float*>(base + L.off_p) : nullptr, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return device_fail(e, "attr_score_topk launch");
    return ATTR_OK;
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_score_topk: host exception");
  }
}

// ---------------------------------------------------------------------------
// losses over token log-probabilities
// ---------------------------------------------------------------------------
namespace {

static_assert(sizeof(attr_token_rows) == 96 && sizeof(attr_adamw_tensor) == 72, "layouts that the binding mirrors");

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

attr_status token_validate(const attr_token_rows* r, const char* who) {
  if (!r) return fail(ATTR_ERR_INVALID_ARG, "%s: rows is NULL", who);
  if (r->dtype != ATTR_F32 && r->dtype != ATTR_BF16 && r->dtype != ATTR_F16)
    return fail(ATTR_ERR_UNSUPPORTED, "%s: logits must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
  if (r->V < 1 || r->V > (1ll << 28))
    return fail(ATTR_ERR_INVALID_ARG, "%s: V=%lld must be in [1, 2^28]", who, (long long)r->V);
  if (r->n_rows < 0 || r->n_examples < 0 || r->T < 1)
    return fail(ATTR_ERR_INVALID_ARG, "%s: n_rows and n_examples must be >= 0, T >= 1", who);
  if (r->T >= (1ll << 31) || r->n_examples >= (1ll << 31) || r->n_examples * r->T >= (1ll << 31))
    return fail(ATTR_ERR_UNSUPPORTED, "%s: n_examples * T must be below 2^31; split the batch", who);
  if (r->ldl < r->V || r->ldl > (1ll << 40))
    return fail(ATTR_ERR_INVALID_ARG, "%s: ldl=%lld must be in [V, 2^40]", who, (long long)r->ldl);
  if (r->n_rows > (1ll << 40) / r->ldl * (1ll << 20))
    return fail(ATTR_ERR_INVALID_ARG, "%s: n_rows=%lld is too large", who, (long long)r->n_rows);
  if (!(r->logit_scale > 0.f) || r->logit_scale > 2.0e38f)  // times log2 e it is finite
    return fail(ATTR_ERR_INVALID_ARG, "%s: logit_scale must be positive and at most 2e38", who);
  if (!r->row_offset && r->n_rows < r->n_examples * r->T)
    return fail(ATTR_ERR_INVALID_ARG, "%s: %lld rows, %lld examples of %lld tokens need more", who,
                (long long)r->n_rows, (long long)r->n_examples, (long long)r->T);
  if (r->n_examples > 0 && r->n_rows > 0 && (!r->logits || !r->target))
    return fail(ATTR_ERR_INVALID_ARG, "%s: logits or target is NULL", who);
  if (!aligned_to(r->logits, (size_t)dtype_bytes(r->dtype)) || !aligned_to(r->target, 8) ||
      !aligned_to(r->weight, 4) || !aligned_to(r->row_offset, 8) || !aligned_to(r->length, 4))
    return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
  return ATTR_OK;
}

// Checks of the gradient's buffer: its stride, and no overlap with the logits
// but the same rows.
attr_status dlogits_validate(const attr_token_rows* r, void* dlogits, int64_t ldd, const char* who) {
  if (!dlogits) return ATTR_OK;
  const int eb = dtype_bytes(r->dtype);
  if (ldd < r->V || ldd > (1ll << 40))
    return fail(ATTR_ERR_INVALID_ARG, "%s: ldd=%lld must be in [V, 2^40]", who, (long long)ldd);
  if (r->n_rows > (1ll << 40) / ldd * (1ll << 20))
    return fail(ATTR_ERR_INVALID_ARG, "%s: n_rows=%lld is too large", who, (long long)r->n_rows);
  if (!aligned_to(dlogits, (size_t)eb))
    return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
  if (dlogits == r->logits && ldd == r->ldl) return ATTR_OK;
  if (overlap(span_of(dlogits, r->n_rows, r->V, ldd, eb), span_of(r->logits, r->n_rows, r->V, r->ldl, eb)))
    return fail(ATTR_ERR_INVALID_ARG, "%s: dlogits overlaps the logits", who);
  return ATTR_OK;
}

// Outputs overlap neither each other nor an input: workgroups of one row read its loss's
// inputs while another of them writes (dlogits and the logits: dlogits_validate).
class TokenSpans {
 public:
  explicit TokenSpans(const attr_token_rows* r) : n_rows_(r->n_rows) {
    input(r->target, r->n_rows, 8);
    input(r->weight, r->n_rows, 4);
    input(r->row_offset, r->n_examples, 8);
    input(r->length, r->n_examples, 4);
  }
  void input(const void* p, int64_t n, int eb) {
    if (p && n > 0) in_[n_in_++] = span_of(p, 1, n, n, eb);
  }
  void output(const void* p, int64_t n, int eb = 4) {
    if (p && n > 0) out_[n_out_++] = span_of(p, 1, n, n, eb);
  }
  // `r`'s logits are an input of every output but dlogits.
  attr_status check(const attr_token_rows* r, const void* dlogits, int64_t ldd, const char* who) {
    const int eb = dtype_bytes(r->dtype);
    const Span logits = span_of(r->logits, n_rows_, r->V, r->ldl, eb);
    bool bad = false;
    for (int i = 0; i < n_out_; ++i) {
      bad |= n_rows_ > 0 && overlap(out_[i], logits);
      for (int j = 0; j < i; ++j) bad |= overlap(out_[i], out_[j]);
    }
    if (dlogits && n_rows_ > 0) {
      const Span d = span_of(dlogits, n_rows_, r->V, ldd, eb);
      for (int i = 0; i < n_out_; ++i) bad |= overlap(d, out_[i]);
      out_[n_out_++] = d;
    }
    for (int i = 0; i < n_out_; ++i)
      for (int j = 0; j < n_in_; ++j) bad |= overlap(out_[i], in_[j]);
    return bad ? fail(ATTR_ERR_INVALID_ARG, "%s: outputs overlap each other or the inputs", who) : ATTR_OK;
  }

 private:
  Span in_[8], out_[4];  // four of the rows and up to three of the loss; three vectors and dlogits
  int n_in_ = 0, n_out_ = 0;
  int64_t n_rows_;
};

// Workspace of the three calls: what each keeps per token slot, per pair and per part
// of a row.
struct TokenLayout {
  size_t off_stats, off_part, off_coef, off_parts, off_zy, total;
  int n_parts;
};
TokenLayout token_layout(const attr_token_rows* r, int mode) {
  TokenLayout L{0, 0, 0, 0, 0, 0, 1};
  const int64_t n = r->n_examples * r->T;
  const size_t slots = (size_t)n;
  if (mode == attr::kTokenPolicy) L.total = align_up(4 * slots);
  if (mode == attr::kTokenPref) {
    L.off_part = align_up(8 * slots);
    L.off_coef = L.off_part + align_up(8 * slots);
    L.total = L.off_coef + align_up(4 * (size_t)(r->n_examples / 2));
  }
  L.n_parts = attr::token_parts(mode, n, r->V * dtype_bytes(r->dtype));
  if (L.n_parts > 1) {
    L.off_parts = L.total;
    L.off_zy = L.off_parts + align_up(8 * slots * (size_t)L.n_parts);
    L.total = L.off_zy + align_up(4 * slots);
  }
  return L;
}

attr::TokenArgs token_args(const attr_token_rows* r, const TokenLayout& L, float* logp, void* dlogits, int64_t ldd,
                           void* ws) {
  attr::TokenArgs a;
  std::memset(&a, 0, sizeof(a));
  a.logits = r->logits;
  a.target = r->target;
  a.weight = r->weight;
  a.row_offset = r->row_offset;
  a.length = r->length;
  a.logp = logp;
  a.dlogits = dlogits;
  a.n_rows = r->n_rows;
  a.ldl = r->ldl;
  a.ldd = ldd;
  a.n_slots = (uint32_t)(r->n_examples * r->T);
  a.T = (uint32_t)r->T;
  a.V = (int32_t)r->V;
  a.scale = r->logit_scale;
  // parts start at multiples of 64 elements, so that they cut no vector of an aligned row
  a.part_len = (int32_t)(L.n_parts > 1 ? ((r->V + L.n_parts - 1) / L.n_parts + 63) & ~63ll : r->V);
  a.n_parts = (int32_t)((r->V + a.part_len - 1) / a.part_len);
  if (L.n_parts > 1) {
    a.parts = reinterpret_cast<float2*>(static_cast<char*>(ws) + L.off_parts);
    a.zy = reinterpret_cast<float*>(static_cast<char*>(ws) + L.off_zy);
  }
  return a;
}

attr_status token_workspace(const TokenLayout& L, void* ws, size_t ws_bytes, const char* who) {
  if (L.total > 0 && (!ws || ws_bytes < L.total))
    return fail(ATTR_ERR_WORKSPACE, "%s needs %zu workspace bytes, got %zu", who, L.total,
                ws ? ws_bytes : (size_t)0);
  if (reinterpret_cast<uintptr_t>(ws) & 255u)
    return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
  return ATTR_OK;
}

size_t token_query(const attr_token_rows* r, int mode) {
  if (!r || !valid_dtype(r->dtype) || r->V < 1 || r->V > (1ll << 28) || r->n_examples < 0 || r->T < 1 ||
      r->T >= (1ll << 31) || r->n_examples >= (1ll << 31) || r->n_examples * r->T >= (1ll << 31))
    return 0;
  return token_layout(r, mode).total;
}

}  // namespace

size_t attr_token_logp_workspace_size(const attr_token_rows* rows) { return token_query(rows, attr::kTokenLogp); }
size_t attr_policy_loss_workspace_size(const attr_token_rows* rows) { return token_query(rows, attr::kTokenPolicy); }
size_t attr_preference_loss_workspace_size(const attr_token_rows* rows) { return token_query(rows, attr::kTokenPref); }

attr_status attr_token_logp(const attr_token_rows* rows, float* logp, void* ws, size_t ws_bytes,
                            void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_token_logp";
    attr_status st = token_validate(rows, who);
    if (st != ATTR_OK) return st;
    if (rows->n_examples == 0 || rows->n_rows == 0) return ATTR_OK;
    if (!logp) return fail(ATTR_ERR_INVALID_ARG, "%s: logp is NULL", who);
    if (!aligned_to(logp, 4)) return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
    TokenSpans spans(rows);
    spans.output(logp, rows->n_rows);
    st = spans.check(rows, nullptr, 0, who);
    if (st != ATTR_OK) return st;
    const TokenLayout L = token_layout(rows, attr::kTokenLogp);
    st = token_workspace(L, ws, ws_bytes, who);
    if (st != ATTR_OK) return st;
    const attr::TokenArgs a = token_args(rows, L, logp, nullptr, 0, ws);
    const hipError_t e = attr::launch_token_logp((int)rows->dtype, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_token_logp launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_token_logp: host exception");
  }
}

attr_status attr_policy_loss(const attr_token_rows* rows, const float* advantage, int32_t per_token,
                             const float* logp_old, const float* logp_ref, float clip_low,
                             float clip_high, float beta, float* loss, float* logp, void* dlogits,
                             int64_t ldd, void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_policy_loss";
    attr_status st = token_validate(rows, who);
    if (st == ATTR_OK) st = dlogits_validate(rows, dlogits, ldd, who);
    if (st != ATTR_OK) return st;
    if (!(clip_low >= 0.f) || !(clip_high >= 0.f))
      return fail(ATTR_ERR_INVALID_ARG, "%s: clip_low and clip_high must be >= 0", who);
    if (!(beta >= 0.f) || beta > 3.0e38f)
      return fail(ATTR_ERR_INVALID_ARG, "%s: beta must be finite and >= 0", who);
    if (per_token != 0 && per_token != 1) return fail(ATTR_ERR_INVALID_ARG, "%s: per_token must be 0 or 1", who);
    if (rows->n_examples == 0) return ATTR_OK;
    if (!loss || !advantage) return fail(ATTR_ERR_INVALID_ARG, "%s: loss or advantage is NULL", who);
    if (beta != 0.f && !logp_ref) return fail(ATTR_ERR_INVALID_ARG, "%s: a KL term needs logp_ref", who);
    if (!aligned_to(advantage, 4) || !aligned_to(logp_old, 4) || !aligned_to(logp_ref, 4) || !aligned_to(loss, 4) ||
        !aligned_to(logp, 4))
      return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
    TokenSpans spans(rows);
    spans.input(advantage, per_token ? rows->n_rows : rows->n_examples, 4);
    spans.input(logp_old, rows->n_rows, 4);
    spans.input(beta != 0.f ? logp_ref : nullptr, rows->n_rows, 4);
    spans.output(loss, rows->n_examples);
    spans.output(logp, rows->n_rows);
    st = spans.check(rows, dlogits, ldd, who);
    if (st != ATTR_OK) return st;
    const TokenLayout L = token_layout(rows, attr::kTokenPolicy);
    st = token_workspace(L, ws, ws_bytes, who);
    if (st != ATTR_OK) return st;
    const attr::TokenArgs a = token_args(rows, L, logp, dlogits, ldd, ws);
    attr::PolicyArgs p;
    std::memset(&p, 0, sizeof(p));
    p.advantage = advantage;
    p.per_token = per_token;
    p.logp_old = logp_old;
    p.logp_ref = logp_ref;
    p.lo = 1.f - clip_low;
    p.hi = 1.f + clip_high;
    p.beta = beta;
    p.token_loss = static_cast<float*>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (attr::policy_by_example(rows->V * dtype_bytes(rows->dtype), rows->T, rows->n_examples)) {
      const hipError_t e =
          attr::launch_policy_examples((int)rows->dtype, a, p, (uint32_t)rows->n_examples, loss, s);
      return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_policy_loss launch");
    }
    if (rows->T == 1) p.token_loss = loss;  // an example is its token
    hipError_t e = attr::launch_policy_rows((int)rows->dtype, a, p, s);
    if (e != hipSuccess) return device_fail(e, "attr_policy_loss launch");
    if (rows->T == 1) return ATTR_OK;
    e = attr::launch_example_sum(p.token_loss, a.T, (uint32_t)rows->n_examples, loss, s);
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_policy_loss sum launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_policy_loss: host exception");
  }
}

attr_status attr_preference_loss(const attr_token_rows* rows, const float* logp_ref,
                                 const float* pair_weight, float beta, float margin,
                                 float label_smoothing, float* loss, float* log_ratio, float* logp,
                                 void* dlogits, int64_t ldd, void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_preference_loss";
    attr_status st = token_validate(rows, who);
    if (st == ATTR_OK) st = dlogits_validate(rows, dlogits, ldd, who);
    if (st != ATTR_OK) return st;
    if (rows->n_examples % 2)
      return fail(ATTR_ERR_INVALID_ARG, "%s: n_examples=%lld must be even (chosen, then rejected)", who,
                  (long long)rows->n_examples);
    if (!(beta >= -3.0e38f && beta <= 3.0e38f) || !(margin >= -3.0e38f && margin <= 3.0e38f))
      return fail(ATTR_ERR_INVALID_ARG, "%s: beta and margin must be finite", who);
    if (!(label_smoothing >= 0.f && label_smoothing <= 1.f))
      return fail(ATTR_ERR_INVALID_ARG, "%s: label_smoothing must be in [0, 1]", who);
    if (rows->n_examples == 0) return ATTR_OK;
    if (!loss) return fail(ATTR_ERR_INVALID_ARG, "%s: loss is NULL", who);
    if (!aligned_to(logp_ref, 4) || !aligned_to(pair_weight, 4) || !aligned_to(loss, 4) ||
        !aligned_to(log_ratio, 4) || !aligned_to(logp, 4))
      return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
    TokenSpans spans(rows);
    spans.input(logp_ref, rows->n_rows, 4);
    spans.input(pair_weight, rows->n_examples / 2, 4);
    spans.output(loss, rows->n_examples / 2);
    spans.output(log_ratio, rows->n_examples);
    spans.output(logp, rows->n_rows);
    st = spans.check(rows, dlogits, ldd, who);
    if (st != ATTR_OK) return st;
    const TokenLayout L = token_layout(rows, attr::kTokenPref);
    st = token_workspace(L, ws, ws_bytes, who);
    if (st != ATTR_OK) return st;
    char* base = static_cast<char*>(ws);
    attr::TokenArgs a = token_args(rows, L, logp, dlogits, ldd, ws);
    a.stats = reinterpret_cast<float2*>(base + L.off_stats);
    a.part = reinterpret_cast<double*>(base + L.off_part);
    attr::PrefArgs p;
    std::memset(&p, 0, sizeof(p));
    p.logp_ref = logp_ref;
    p.pair_weight = pair_weight;
    p.loss = loss;
    p.log_ratio = log_ratio;
    p.coef = reinterpret_cast<float*>(base + L.off_coef);
    p.n_pairs = (uint32_t)(rows->n_examples / 2);
    p.beta = beta;
    p.margin = margin;
    p.smoothing = label_smoothing;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (attr::pref_by_pair(rows->V * dtype_bytes(rows->dtype), rows->T, p.n_pairs)) {
      const hipError_t e = attr::launch_pref_pairs((int)rows->dtype, a, p, s);
      return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_preference_loss launch");
    }
    hipError_t e = attr::launch_pref_stats((int)rows->dtype, a, p, s);
    if (e != hipSuccess) return device_fail(e, "attr_preference_loss launch");
    const bool pair = dlogits && attr::pref_pairs_within(rows->V * dtype_bytes(rows->dtype), rows->T, a.n_slots);
    if (!pair) e = attr::launch_pairs(a, p, s);
    if (e != hipSuccess) return device_fail(e, "attr_preference_loss pair launch");
    if (!dlogits) return ATTR_OK;
    e = attr::launch_pref_grad((int)rows->dtype, pair, a, p, s);
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_preference_loss gradient launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_preference_loss: host exception");
  }
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
namespace {

// Gathers tensors into launches.
struct AdamwLaunch {
  int p_dtype, g_dtype;
  bool eight;
  int runs;
  attr::AdamwStep step;
  hipStream_t stream;
  bool master = false;  // of the launch being filled
  uint32_t blocks = 0;
  attr::AdamwPlain plain = {};
  attr::AdamwFull full = {};

  hipError_t add(attr::AdamwEntry e, const attr::AdamwExtra& x) {
    const uint32_t chunk = 4 * (uint32_t)runs * attr::kAdamwRun, lead = eight ? 0 : attr::adamw_lead(e.m),
                   need = (uint32_t)(((uint64_t)e.n + lead + chunk - 1) / chunk);
    const int most = eight || x.master ? attr::kAdamwMostExtra : attr::kAdamwMost;
    // below 2^32 threads a launch
    if (step.n >= most || blocks + need > (1u << 23) || master != (x.master != nullptr)) {
      const hipError_t r = flush();
      if (r != hipSuccess) return r;
    }
    master = x.master != nullptr;
    e.chunk0 = blocks;
    if (eight || master) {
      full.e[step.n] = e;
      full.x[step.n] = x;
    } else {
      plain.e[step.n] = e;
    }
    ++step.n;
    blocks += need;
    return hipSuccess;
  }
  hipError_t flush() {
    if (step.n == 0) return hipSuccess;
    hipError_t r;
    if (eight || master) {
      full.step = step;
      r = attr::launch_adamw(p_dtype, g_dtype, eight, master, runs, blocks, full, stream);
    } else {
      plain.step = step;
      r = attr::launch_adamw(p_dtype, g_dtype, runs, blocks, plain, stream);
    }
    step.n = 0;
    blocks = 0;
    return r;
  }
};

}  // namespace

attr_status attr_adamw_step(const attr_adamw_tensor* tensors, int32_t n_tensors, attr_dtype p_dtype,
                            attr_dtype g_dtype, attr_dtype state_dtype, int64_t step, double lr,
                            double beta1, double beta2, double eps, double eps_root,
                            const float* grad_scale, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_adamw_step";
    if (n_tensors < 0 || (n_tensors > 0 && !tensors))
      return fail(ATTR_ERR_INVALID_ARG, "%s: n_tensors is negative or tensors NULL", who);
    if (!valid_dtype(p_dtype) || !valid_dtype(g_dtype))
      return fail(ATTR_ERR_UNSUPPORTED, "%s: weights and gradients must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
    if (state_dtype != ATTR_F32 && state_dtype != ATTR_E4M3)
      return fail(ATTR_ERR_UNSUPPORTED, "%s: states must be ATTR_F32 or ATTR_E4M3", who);
    if (step < 1) return fail(ATTR_ERR_INVALID_ARG, "%s: step=%lld must be >= 1", who, (long long)step);
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
      return fail(ATTR_ERR_INVALID_ARG, "%s: beta1 and beta2 must be in [0, 1)", who);
    if (!(eps >= 0.0 && eps <= 3.0e38) || !(eps_root >= 0.0 && eps_root <= 3.0e38) || !(std::fabs(lr) <= 3.0e38))
      return fail(ATTR_ERR_INVALID_ARG, "%s: lr, eps and eps_root must be finite, eps and eps_root >= 0", who);
    // The step divides by sqrt(v + eps_root) + eps through fp32 reciprocals: an eps that fp32
    // holds as a subnormal number or as 0 would make 0 / eps of an untouched weight NaN, and
    // so would an eps_root that it holds as 0.
    if ((eps > 0.0 && eps < 0x1p-126) || (eps_root > 0.0 && eps_root < 0x1p-149))
      return fail(ATTR_ERR_INVALID_ARG, "%s: eps must be 0 or at least 2^-126, eps_root 0 or at least 2^-149", who);
    if (!aligned_to(grad_scale, 4)) return fail(ATTR_ERR_ALIGNMENT, "%s: grad_scale must be 4-byte aligned", who);
    const bool eight = state_dtype == ATTR_E4M3;
    const size_t pb = (size_t)dtype_bytes(p_dtype), gb = (size_t)dtype_bytes(g_dtype), sb = eight ? 1 : 4;
    for (int32_t j = 0; j < n_tensors; ++j) {
      const attr_adamw_tensor& t = tensors[j];
      if (t.n < 0 || t.n >= (1ll << 40)) return fail(ATTR_ERR_INVALID_ARG, "%s: tensor %d: n=%lld", who, j, (long long)t.n);
      if (!(std::fabs(t.lr_scale) <= 3.0e38f) || !(std::fabs(t.weight_decay) <= 3.0e38f))
        return fail(ATTR_ERR_INVALID_ARG, "%s: tensor %d: lr_scale and weight_decay must be finite", who, j);
      if (t.n == 0) continue;
      if (!t.p || !t.g || !t.m || !t.v) return fail(ATTR_ERR_INVALID_ARG, "%s: tensor %d: NULL pointer", who, j);
      if (eight != (t.m_scale != nullptr) || eight != (t.v_scale != nullptr))
        return fail(ATTR_ERR_INVALID_ARG, "%s: tensor %d: m_scale and v_scale go with 8-bit states", who, j);
      if (!aligned_to(t.p, pb) || !aligned_to(t.g, gb) || !aligned_to(t.m, sb) || !aligned_to(t.v, sb) ||
          !aligned_to(t.master, 4) || !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))
        return fail(ATTR_ERR_ALIGNMENT, "%s: tensor %d: pointers must be aligned to their elements", who, j);
    }
    attr::AdamwStep h;
    std::memset(&h, 0, sizeof(h));
    h.grad_scale = grad_scale;
    h.beta1 = (float)beta1;
    h.one_beta1 = (float)(1.0 - beta1);
    h.beta2 = (float)beta2;
    h.one_beta2 = (float)(1.0 - beta2);
    const double corr1 = 1.0 / (1.0 - std::pow(beta1, (double)step));
    h.corr2 = (float)(1.0 / (1.0 - std::pow(beta2, (double)step)));
    h.eps = (float)eps;
    h.eps_root = (float)eps_root;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int64_t total = 0;
    for (int32_t j = 0; j < n_tensors; ++j) total = std::min(total + tensors[j].n, (int64_t)1 << 40);
    AdamwLaunch L{(int)p_dtype, (int)g_dtype, eight, attr::adamw_runs_per_wave(total, eight), h, s};
    // The neighbour of a tensor in every buffer, with the same rates, is one tensor with
    // it: a model in flat buffers takes one launch (168 adapters: two, and 20.7 us
    // against 15.6).
    const auto joins = [&](const attr_adamw_tensor& t, const attr_adamw_tensor& u) {
      const auto after = [&](const void* x, const void* y, size_t each) {
        return x ? y == static_cast<const char*>(x) + (size_t)t.n * each : !y;
      };
      return (!eight || (t.n % attr::kAdamwRun == 0 && u.m_scale == t.m_scale + t.n / attr::kAdamwRun &&
                         u.v_scale == t.v_scale + t.n / attr::kAdamwRun)) &&
             after(t.p, u.p, pb) && after(t.g, u.g, gb) && after(t.m, u.m, sb) && after(t.v, u.v, sb) &&
             after(t.master, u.master, 4) && t.lr_scale == u.lr_scale && t.weight_decay == u.weight_decay;
    };
    for (int32_t j = 0; j < n_tensors; ++j) {
      attr_adamw_tensor t = tensors[j];
      if (t.n == 0) continue;
      while (j + 1 < n_tensors && tensors[j + 1].n > 0 && joins(t, tensors[j + 1])) t.n += tensors[++j].n;
      // pieces of whole blocks whose sizes fit 32 bits
      constexpr int64_t kMost = 1ll << 31;
      for (int64_t at = 0; at < t.n; at += kMost) {
        attr::AdamwEntry e;
        e.p = static_cast<char*>(t.p) + (size_t)at * pb;
        e.g = static_cast<const char*>(t.g) + (size_t)at * gb;
        e.m = static_cast<char*>(t.m) + (size_t)at * sb;
        e.v = static_cast<char*>(t.v) + (size_t)at * sb;
        e.lr = (float)(lr * (double)t.lr_scale * corr1);
        e.lr_wd = (float)(lr * (double)t.lr_scale * (double)t.weight_decay);
        e.n = (uint32_t)std::min(t.n - at, kMost);
        e.chunk0 = 0;
        const attr::AdamwExtra x{t.master ? t.master + at : nullptr, t.m_scale ? t.m_scale + at / 256 : nullptr,
                                 t.v_scale ? t.v_scale + at / 256 : nullptr};
        const hipError_t r = L.add(e, x);
        if (r != hipSuccess) return device_fail(r, "attr_adamw_step launch");
      }
    }
    const hipError_t r = L.flush();
    return r == hipSuccess ? ATTR_OK : device_fail(r, "attr_adamw_step launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_adamw_step: host exception");
  }
}

// ---------------------------------------------------------------------------
// Muon
// ---------------------------------------------------------------------------
namespace {

static_assert(sizeof(attr_muon_matrix) == 56 && sizeof(attr_rows) == 40, "layouts that the binding mirrors");

// Matrices that are worked on together: those of one shape side by side.
struct MuonRound {
  int kind;                    // sixteens of the shorter sides, all at most kThinMost; or kTiles, kBigTiles
  std::vector<int32_t> order;  // the matrices, group by group
  attr::MuonArgs args;         // but for the table and the workspace's address
  uint32_t sym, full, flat, turn, gram;  // workgroups
  bool split;                  // some group's rows are divided
  size_t bytes;                // of workspace behind the table
};
struct MuonPlan {
  std::vector<MuonRound> rounds;
  size_t table, total;  // bytes
};

bool muon_fits(const attr_muon_matrix& t) {
  if (t.rows < 0 || t.cols < 0 || t.rows > (1ll << 20) || t.cols > (1ll << 20)) return false;
  return std::max(t.rows, t.cols) * ((std::min(t.rows, t.cols) + 63) / 64 * 64) < (1ll << 30);
}

// Workspace of one matrix, and the workgroups that its launches take.
attr::MuonGroup muon_group(int64_t rows, int64_t cols, bool pairs, bool big) {
  attr::MuonGroup q;
  std::memset(&q, 0, sizeof(q));
  q.rows = (int32_t)rows;
  q.cols = (int32_t)cols;
  q.L = (int32_t)std::max(rows, cols);
  q.S = (int32_t)std::min(rows, cols);
  q.ld = (q.S + 63) / 64 * 64;
  const int64_t y = (int64_t)align_up((size_t)q.L * q.ld * 2), s = (int64_t)align_up((size_t)q.S * q.ld * 2);
  const int64_t many = pairs ? 2 : 1;
  q.lo_y = y;
  q.lo_s = s;
  q.y[0] = 0;
  q.y[1] = many * y;
  q.gram = 2 * many * y;
  q.poly = q.gram + many * s;
  q.norm = q.poly + many * s;
  q.stride = q.norm + (int64_t)align_up(8 * attr::kMuonFlatMost);
  const int32_t tile = big ? 2 * attr::kMuonTile : attr::kMuonTile;
  const uint32_t ts = (uint32_t)((q.S + tile - 1) / tile), tl = (uint32_t)((q.L + tile - 1) / tile);
  q.n_sym = ts * (ts + 1) / 2;
  q.n_full = ts * tl;
  q.n_flat = (uint32_t)std::min<int64_t>((rows * cols + attr::kMuonFlat - 1) / attr::kMuonFlat, attr::kMuonFlatMost);
  q.n_turn = (uint32_t)((q.L + 63) / 64) * (uint32_t)(q.ld / 64);
  return q;
}

// The same of a thin one.
attr::MuonGroup thin_group(int64_t rows, int64_t cols) {
  attr::MuonGroup q;
  std::memset(&q, 0, sizeof(q));
  q.rows = (int32_t)rows;
  q.cols = (int32_t)cols;
  q.L = (int32_t)std::max(rows, cols);
  q.S = (int32_t)std::min(rows, cols);
  const int64_t t = (q.S + 15) / 16;
  q.n_flat = (uint32_t)((q.L + attr::kThinRows - 1) / attr::kThinRows);
  q.poly = (int64_t)q.n_flat * (t * (t + 1) / 2 * 256 * 8);
  q.stride = q.poly + t * t * 256 * 8;
  return q;
}

constexpr int kTiles = 8, kBigTiles = 9;
// Tiles of 256 x 256 for shorter sides from 1024 on, where the call has enough of them: 128 and more
// for the products A, which have the fewest (us, 128 x 128 in brackets; bf16 weights: 4 of 2048 x 8192, 144
// tiles, 2665 (2982); 24 of 1024 x 4096, 240 tiles, 2251 (2810); 4 of them, 40 tiles, 844 (540)).  The line is a
// middle one: fp32 weights, fp16 operands, 3 of 4096 x 4096, 408 tiles, 3930 (4971), but 14 of 1024 x 4096, 140
// tiles, 1665 (1457).  With pairs, whose three products share no fragments there, it lies further up:
// 4 of 2048 x 8192 6681 (7331), 3 of 4096 x 4096 11217 (13184), but 16 of 2048 x 2048, 576 tiles, 10396 (9217) and
// 28 of 1024 x 4096, 280 tiles, 7605 (7070).
constexpr int64_t kMuonBigSide = 1024, kMuonBigTiles = 128;
bool muon_big(const attr_muon_matrix* mats, int32_t n) {
  int64_t tiles = 0;
  for (int32_t j = 0; j < n; ++j) {
    const int64_t s = std::min(mats[j].rows, mats[j].cols), t = (s + 255) / 256;
    if (s >= kMuonBigSide) tiles += t * (t + 1) / 2;
  }
  return tiles >= kMuonBigTiles;
}
int muon_kind(const attr_muon_matrix& t, bool big) {
  const int64_t s = std::min(t.rows, t.cols);
  if (s <= attr::kThinMost) return (int)((s + 15) / 16);
  return big && s >= kMuonBigSide ? kBigTiles : kTiles;
}

// A round ends where its launches fill the GPU some times over: its buffers then stay
// small, and nearer to the caches.
constexpr uint32_t kMuonRoundTiles = 4096;
constexpr uint32_t kMuonRoundFlat = 1u << 20;
constexpr size_t kMuonRoundBytes = (size_t)1 << 30;

MuonPlan muon_plan(const attr_muon_matrix* mats, int32_t n, bool pairs) {
  MuonPlan P;
  const bool big = muon_big(mats, n);
  // by kind, and by shape
  std::map<std::tuple<int, int64_t, int64_t>, std::vector<int32_t>> shapes;
  for (int32_t j = 0; j < n; ++j) {
    if (mats[j].rows > 0 && mats[j].cols > 0) shapes[{muon_kind(mats[j], big), mats[j].rows, mats[j].cols}].push_back(j);
  }
  MuonRound R;
  const auto clear = [&] {
    R.order.clear();
    std::memset(&R.args, 0, sizeof(R.args));
    R.sym = R.full = R.flat = R.turn = R.gram = 0;
    R.split = false;
    R.bytes = 0;
  };
  size_t most = 0, matrices = 0;
  const auto end = [&] {
    if (R.order.empty()) return;
    uint32_t tiles = 0;
    for (int k = 0; k < R.args.n_groups; ++k) tiles += R.args.g[k].n_sym * R.args.g[k].count;
    const uint32_t slots = R.kind == kBigTiles ? 256 : 512;  // workgroups that the GPU holds at once
    for (int k = 0; k < R.args.n_groups; ++k) {
      attr::MuonGroup& q = R.args.g[k];
      q.tile_sym = R.sym;
      q.tile_full = R.full;
      R.sym += attr::muon_tiles(q.n_sym * q.count);
      R.full += attr::muon_tiles(q.n_full * q.count);
      q.splits = 1;
      if (R.kind < kTiles) {
        R.split |= q.n_flat > attr::kThinParts;
        continue;
      }
      const int32_t want = std::min({(int32_t)(slots / tiles), q.L / attr::kMuonSplitRows, attr::kMuonSplits});
      if (want > 1) {
        q.split_rows = ((q.L + want - 1) / want + 63) / 64 * 64;
        q.splits = (uint32_t)((q.L + q.split_rows - 1) / q.split_rows);
      } else {
        q.split_rows = q.L;
      }
      q.tile_gram = R.gram;
      R.gram += attr::muon_tiles(q.n_sym * q.count * q.splits);
      if (q.splits > 1) {
        const size_t side = R.kind == kBigTiles ? 2 * attr::kMuonTile : attr::kMuonTile;
        q.part = reinterpret_cast<char*>(R.bytes);
        R.bytes += (size_t)q.n_sym * q.count * q.splits * side * side * 4;
        R.split = true;
      }
    }
    most = std::max(most, R.bytes);
    matrices = std::max(matrices, R.order.size());
    P.rounds.push_back(R);
    clear();
  };
  clear();
  // the workgroups of the tile kinds' launches, from their groups' numbers of matrices
  const auto tiles = [](const MuonRound& r, uint32_t attr::MuonGroup::*each) {
    uint32_t n = 0;
    for (int k = 0; k < r.args.n_groups; ++k) n += attr::muon_tiles(r.args.g[k].*each * r.args.g[k].count);
    return n;
  };
  // long products first: what is left at a launch's end is short
  std::vector<const std::pair<const std::tuple<int, int64_t, int64_t>, std::vector<int32_t>>*> order;
  for (const auto& sh : shapes) order.push_back(&sh);
  std::stable_sort(order.begin(), order.end(), [](const auto* x, const auto* y) {
    const auto side = [](const auto* s) { return std::max(std::get<1>(s->first), std::get<2>(s->first)); };
    return std::make_tuple(std::get<0>(x->first), -side(x)) < std::make_tuple(std::get<0>(y->first), -side(y));
  });
  for (const auto* sh : order) {
    const int kind = std::get<0>(sh->first);
    attr::MuonGroup q = kind < kTiles ? thin_group(std::get<1>(sh->first), std::get<2>(sh->first))
                                      : muon_group(std::get<1>(sh->first), std::get<2>(sh->first), pairs, kind == kBigTiles);
    if (!R.order.empty() && R.kind != kind) end();
    bool open = false;
    for (int32_t j : sh->second) {
      if (!R.order.empty() && (tiles(R, &attr::MuonGroup::n_full) > kMuonRoundTiles || R.flat + q.n_flat > kMuonRoundFlat ||
                               R.bytes + (size_t)q.stride > kMuonRoundBytes ||
                               (!open && R.args.n_groups == attr::kMuonGroups))) {
        end();
        open = false;
      }
      R.kind = kind;
      if (!open) {
        q.base = reinterpret_cast<char*>(R.bytes);  // behind the table
        q.tile_flat = R.flat;
        q.tile_turn = R.turn;
        q.entry = (uint32_t)R.order.size();
        R.args.g[R.args.n_groups++] = q;
        open = true;
      }
      ++R.args.g[R.args.n_groups - 1].count;
      R.order.push_back(j);
      R.flat += q.n_flat;
      R.turn += q.n_turn;
      R.bytes += (size_t)q.stride;
    }
  }
  end();
  P.table = align_up(matrices * sizeof(attr::MuonEntry));
  P.total = P.rounds.empty() ? 0 : P.table + most;
  return P;
}

}  // namespace

size_t attr_muon_step_workspace_size(const attr_muon_matrix* mats, int32_t n_mats, int32_t pairs) {
  try {
    if (n_mats <= 0 || !mats || (pairs != 0 && pairs != 1)) return 0;
    for (int32_t j = 0; j < n_mats; ++j)
      if (!muon_fits(mats[j])) return 0;
    return muon_plan(mats, n_mats, pairs != 0).total;
  } catch (...) {
    return 0;
  }
}

attr_status attr_muon_step(const attr_muon_matrix* mats, int32_t n_mats, attr_dtype p_dtype, attr_dtype g_dtype,
                           double lr, double momentum, int32_t nesterov, int32_t steps, int32_t pairs,
                           const float* grad_scale, void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_muon_step";
    if (n_mats < 0 || (n_mats > 0 && !mats))
      return fail(ATTR_ERR_INVALID_ARG, "%s: n_mats is negative or mats NULL", who);
    if (!valid_dtype(p_dtype) || !valid_dtype(g_dtype))
      return fail(ATTR_ERR_UNSUPPORTED, "%s: weights and gradients must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
    if (!(std::fabs(lr) <= 3.0e38)) return fail(ATTR_ERR_INVALID_ARG, "%s: lr must be finite", who);
    if (!(momentum >= 0.0 && momentum < 1.0)) return fail(ATTR_ERR_INVALID_ARG, "%s: momentum must be in [0, 1)", who);
    if ((nesterov != 0 && nesterov != 1) || (pairs != 0 && pairs != 1))
      return fail(ATTR_ERR_INVALID_ARG, "%s: nesterov and pairs must be 0 or 1", who);
    if (steps < 1 || steps > 16) return fail(ATTR_ERR_INVALID_ARG, "%s: steps=%d must be in [1, 16]", who, (int)steps);
    if (!aligned_to(grad_scale, 4)) return fail(ATTR_ERR_ALIGNMENT, "%s: grad_scale must be 4-byte aligned", who);
    const size_t pb = (size_t)dtype_bytes(p_dtype), gb = (size_t)dtype_bytes(g_dtype);
    bool master = false, plain = false;
    for (int32_t j = 0; j < n_mats; ++j) {
      const attr_muon_matrix& t = mats[j];
      if (t.rows < 0 || t.cols < 0)
        return fail(ATTR_ERR_INVALID_ARG, "%s: matrix %d: %lld x %lld", who, j, (long long)t.rows, (long long)t.cols);
      if (!muon_fits(t))
        return fail(ATTR_ERR_UNSUPPORTED, "%s: matrix %d: %lld x %lld is too large", who, j, (long long)t.rows,
                    (long long)t.cols);
      if (!(std::fabs(t.lr_scale) <= 3.0e38f) || !(std::fabs(t.weight_decay) <= 3.0e38f))
        return fail(ATTR_ERR_INVALID_ARG, "%s: matrix %d: lr_scale and weight_decay must be finite", who, j);
      if (t.rows == 0 || t.cols == 0) continue;
      if (!t.p || !t.g || !t.m) return fail(ATTR_ERR_INVALID_ARG, "%s: matrix %d: NULL pointer", who, j);
      if (!aligned_to(t.p, pb) || !aligned_to(t.g, gb) || !aligned_to(t.m, 4) || !aligned_to(t.master, 4))
        return fail(ATTR_ERR_ALIGNMENT, "%s: matrix %d: pointers must be aligned to their elements", who, j);
      (t.master ? master : plain) = true;
    }
    if (master && plain)
      return fail(ATTR_ERR_INVALID_ARG, "%s: either every matrix has a master, or none has", who);
    const MuonPlan P = muon_plan(mats, n_mats, pairs != 0);
    if (P.rounds.empty()) return ATTR_OK;
    if (!ws || ws_bytes < P.total)
      return fail(ATTR_ERR_WORKSPACE, "%s needs %zu workspace bytes, got %zu", who, P.total, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* const base = static_cast<char*>(ws);
    const auto launch = [&](const MuonRound& R) -> hipError_t {
      attr::MuonTable T;
      for (size_t at = 0; at < R.order.size(); at += attr::kMuonTable) {
        std::memset(&T, 0, sizeof(T));
        T.n = (int32_t)std::min<size_t>(attr::kMuonTable, R.order.size() - at);
        T.to = reinterpret_cast<attr::MuonEntry*>(base) + at;
        for (int32_t k = 0; k < T.n; ++k) {
          const attr_muon_matrix& t = mats[R.order[at + (size_t)k]];
          const double rate = lr * (double)t.lr_scale;
          T.e[k] = {t.p, t.g, t.m, t.master, (float)rate, (float)(rate * (double)t.weight_decay)};
        }
        const hipError_t e = attr::launch_muon_table(T, s);
        if (e != hipSuccess) return e;
      }
      attr::MuonArgs a = R.args;
      for (int k = 0; k < a.n_groups; ++k) {
        a.g[k].base = base + P.table + reinterpret_cast<uintptr_t>(a.g[k].base);
        a.g[k].part = base + P.table + reinterpret_cast<uintptr_t>(a.g[k].part);
      }
      a.table = reinterpret_cast<const attr::MuonEntry*>(base);
      a.grad_scale = grad_scale;
      a.momentum = (float)momentum;
      a.one_momentum = (float)(1.0 - momentum);
      a.nesterov = nesterov;
      if (R.kind < kTiles) {
        hipError_t e = attr::launch_muon_thin_gram((int)g_dtype, R.kind, a, R.flat, s);
        if (e == hipSuccess && R.split) e = attr::launch_muon_thin_sum(R.kind, a, (uint32_t)R.order.size(), s);
        if (e == hipSuccess) e = attr::launch_muon_thin_poly(R.kind, steps, a, (uint32_t)R.order.size(), s);
        if (e == hipSuccess) e = attr::launch_muon_thin_apply((int)p_dtype, (int)g_dtype, master, R.kind, a, R.flat, s);
        return e;
      }
      const bool big = R.kind == kBigTiles;
      hipError_t e = attr::launch_muon_momentum((int)g_dtype, a, R.flat, s);
      if (e == hipSuccess) e = attr::launch_muon_split((int)g_dtype, pairs != 0, a, R.turn, s);
      for (int32_t k = 0; k < steps && e == hipSuccess; ++k) {
        const int from = k & 1;
        e = attr::launch_muon_gram(big, pairs != 0, from, a, R.gram, s);
        if (e == hipSuccess && R.split) e = attr::launch_muon_join(big, pairs != 0, a, R.sym, s);
        if (e == hipSuccess) e = attr::launch_muon_poly(big, pairs != 0, a, R.sym, s);
        if (e != hipSuccess) break;
        e = k + 1 < steps ? attr::launch_muon_apply(big, pairs != 0, from, a, R.full, s)
                          : attr::launch_muon_last(big, pairs != 0, (int)p_dtype, master, from, a, R.full, s);
      }
      return e;
    };
    for (const MuonRound& R : P.rounds) {
      const hipError_t e = launch(R);
      if (e != hipSuccess) return device_fail(e, "attr_muon_step launch");
    }
    return ATTR_OK;
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_muon_step: host exception");
  }
}

// ---------------------------------------------------------------------------
// embedding and layer norm over token rows
// ---------------------------------------------------------------------------
namespace {

bool rows_sizes_ok(const attr_rows* r) {
  return r && r->n_rows >= 0 && r->n_examples >= 0 && r->T >= 1 && r->T < (1ll << 31) &&
         r->n_examples < (1ll << 31) && r->n_examples * r->T < (1ll << 31);
}

attr_status rows_validate(const attr_rows* r, const char* who) {
  if (!r) return fail(ATTR_ERR_INVALID_ARG, "%s: rows is NULL", who);
  if (r->n_rows < 0 || r->n_examples < 0 || r->T < 1)
    return fail(ATTR_ERR_INVALID_ARG, "%s: n_rows and n_examples must be >= 0, T >= 1", who);
  if (!rows_sizes_ok(r)) return fail(ATTR_ERR_UNSUPPORTED, "%s: n_examples * T must be below 2^31; split the batch", who);
  if (!r->row_offset && r->n_rows < r->n_examples * r->T)
    return fail(ATTR_ERR_INVALID_ARG, "%s: %lld rows, %lld examples of %lld tokens need more", who, (long long)r->n_rows,
                (long long)r->n_examples, (long long)r->T);
  if (!aligned_to(r->row_offset, 8) || !aligned_to(r->length, 4))
    return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
  return ATTR_OK;
}

// A matrix of a call: its type, stride, size and alignment.
attr_status matrix_validate(const void* p, attr_dtype t, int64_t rows, int64_t d, int64_t ld, const char* name,
                            const char* who) {
  if (!valid_dtype(t)) return fail(ATTR_ERR_UNSUPPORTED, "%s: %s must be ATTR_F32, ATTR_BF16 or ATTR_F16", who, name);
  if (ld < d || ld > (1ll << 40)) return fail(ATTR_ERR_INVALID_ARG, "%s: %s's row stride %lld must be in [d, 2^40]", who, name, (long long)ld);
  if (rows > (1ll << 40) / ld * (1ll << 20)) return fail(ATTR_ERR_INVALID_ARG, "%s: %s has too many rows", who, name);
  if (!p) return fail(ATTR_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  if (!aligned_to(p, (size_t)dtype_bytes(t))) return fail(ATTR_ERR_ALIGNMENT, "%s: %s must be aligned to its elements", who, name);
  return ATTR_OK;
}

attr::RowsArgs rows_args(const attr_rows* r) {
  attr::RowsArgs a;
  a.row_offset = r->row_offset;
  a.length = r->length;
  a.n_rows = r->n_rows;
  a.n_slots = (uint32_t)(r->n_examples * r->T);
  a.T = (uint32_t)r->T;
  return a;
}

// Spans of a call's buffers: no output overlaps an input or another output.
class RowSpans {
 public:
  explicit RowSpans(const attr_rows* r) {
    input(span_of(r->row_offset, 1, r->row_offset ? r->n_examples : 0, r->n_examples, 8));
    input(span_of(r->length, 1, r->length ? r->n_examples : 0, r->n_examples, 4));
  }
  void input(Span x) { in_.push_back(x); }
  // between: its rows lie between those of the output before it, and are known not to touch them
  void output(Span x, bool between = false) {
    for (size_t j = 0; j + (between ? 1 : 0) < out_.size(); ++j) clash_ |= touches(x, out_[j]);
    out_.push_back(x);
  }
  bool clash() const {
    bool bad = clash_;
    for (const Span& o : out_)
      for (const Span& x : in_) bad |= touches(o, x);
    return bad;
  }

 private:
  static bool touches(Span a, Span b) { return a.lo < a.hi && b.lo < b.hi && overlap(a, b); }
  std::vector<Span> in_, out_;
  bool clash_ = false;
};
Span vector_span(const void* p, int64_t n, int eb) { return span_of(p, 1, p ? n : 0, n, eb); }
attr_status overlap_fail(const char* who) {
  return fail(ATTR_ERR_INVALID_ARG, "%s: outputs overlap each other or the inputs", who);
}

attr_status table_validate(int64_t V, int64_t d, const char* who) {
  if (V < 1 || V > (1ll << 28)) return fail(ATTR_ERR_INVALID_ARG, "%s: V=%lld must be in [1, 2^28]", who, (long long)V);
  if (d < 1 || d > 65536) return fail(ATTR_ERR_INVALID_ARG, "%s: d=%lld must be in [1, 65536]", who, (long long)d);
  return ATTR_OK;
}

struct EmbedLayout {
  size_t key[2], row[2], count, part, total;
};
EmbedLayout embed_layout(const attr_rows* r, int64_t V, int64_t d) {
  EmbedLayout L;
  std::memset(&L, 0, sizeof(L));
  const size_t n = (size_t)(r->n_examples * r->T), each = align_up(4 * n);
  if (attr::embed_searches(n, V, d)) return L;
  L.key[0] = 0;
  L.key[1] = each;
  L.row[0] = 2 * each;
  L.row[1] = 3 * each;
  L.count = 4 * each;
  const size_t blocks = (n + attr::kSortKeys - 1) / attr::kSortKeys;
  L.part = L.count + (n > attr::kSortOne ? align_up((blocks << attr::sort_bits(V)) * 8) : 0);
  const size_t each_part = attr::embed_part(n, d), parts = (n + each_part - 1) / each_part;
  L.total = L.part + align_up(parts * 2 * (size_t)d * 4);
  return L;
}

}  // namespace

attr_status attr_embed(const attr_rows* rows, const int64_t* token, const void* table, attr_dtype table_dtype, int64_t V,
                       int64_t d, int64_t ldt, float scale, void* out, attr_dtype out_dtype, int64_t ldo, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_embed";
    attr_status st = rows_validate(rows, who);
    if (st == ATTR_OK) st = table_validate(V, d, who);
    if (st != ATTR_OK) return st;
    if (!(std::fabs(scale) <= 3.0e38f)) return fail(ATTR_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (rows->n_examples == 0 || rows->n_rows == 0) return ATTR_OK;
    st = matrix_validate(table, table_dtype, V, d, ldt, "table", who);
    if (st == ATTR_OK) st = matrix_validate(out, out_dtype, rows->n_rows, d, ldo, "out", who);
    if (st != ATTR_OK) return st;
    if (!token) return fail(ATTR_ERR_INVALID_ARG, "%s: token is NULL", who);
    if (!aligned_to(token, 8)) return fail(ATTR_ERR_ALIGNMENT, "%s: token must be aligned to its elements", who);
    RowSpans spans(rows);
    spans.input(vector_span(token, rows->n_rows, 8));
    spans.input(span_of(table, V, d, ldt, dtype_bytes(table_dtype)));
    spans.output(span_of(out, rows->n_rows, d, ldo, dtype_bytes(out_dtype)));
    if (spans.clash()) return overlap_fail(who);
    const attr::EmbedArgs a{token, table, out, V, ldt, ldo, (int32_t)d, scale};
    const hipError_t e = attr::launch_embed((int)table_dtype, (int)out_dtype, rows_args(rows), a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_embed launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_embed: host exception");
  }
}

size_t attr_embed_backward_workspace_size(const attr_rows* rows, int64_t V, int64_t d) {
  if (!rows_sizes_ok(rows) || V < 1 || V > (1ll << 28) || d < 1 || d > 65536) return 0;
  return embed_layout(rows, V, d).total;
}

attr_status attr_embed_backward(const attr_rows* rows, const int64_t* token, const void* dout, attr_dtype dout_dtype,
                                int64_t ldd, int64_t V, int64_t d, float scale, void* dtable, attr_dtype dtable_dtype,
                                int64_t ldt, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_embed_backward";
    attr_status st = rows_validate(rows, who);
    if (st == ATTR_OK) st = table_validate(V, d, who);
    if (st != ATTR_OK) return st;
    if (!(std::fabs(scale) <= 3.0e38f)) return fail(ATTR_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (accumulate != 0 && accumulate != 1) return fail(ATTR_ERR_INVALID_ARG, "%s: accumulate must be 0 or 1", who);
    if (rows->n_rows >= (1ll << 32)) return fail(ATTR_ERR_UNSUPPORTED, "%s: n_rows must be below 2^32; split the batch", who);
    const bool none = rows->n_examples == 0 || rows->n_rows == 0;
    if (none && accumulate) return ATTR_OK;
    st = matrix_validate(dtable, dtable_dtype, V, d, ldt, "dtable", who);
    if (st == ATTR_OK && !none) st = matrix_validate(dout, dout_dtype, rows->n_rows, d, ldd, "dout", who);
    if (st != ATTR_OK) return st;
    if (!valid_dtype(dout_dtype)) return fail(ATTR_ERR_UNSUPPORTED, "%s: dout must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
    if (!none && !token) return fail(ATTR_ERR_INVALID_ARG, "%s: token is NULL", who);
    if (!aligned_to(token, 8)) return fail(ATTR_ERR_ALIGNMENT, "%s: token must be aligned to its elements", who);
    RowSpans spans(rows);
    spans.input(vector_span(token, rows->n_rows, 8));
    if (!none) spans.input(span_of(dout, rows->n_rows, d, ldd, dtype_bytes(dout_dtype)));
    spans.output(span_of(dtable, V, d, ldt, dtype_bytes(dtable_dtype)));
    if (spans.clash()) return overlap_fail(who);
    hipStream_t s = static_cast<hipStream_t>(stream);
    attr::EmbedGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.dout = dout;
    a.dtable = dtable;
    a.V = V;
    a.ldd = ldd;
    a.ldt = ldt;
    a.d = (int32_t)d;
    a.accumulate = accumulate;
    a.scale = scale;
    const attr::RowsArgs r = none ? attr::RowsArgs{nullptr, nullptr, 0, 0, 1} : rows_args(rows);
    if (attr::embed_searches(r.n_slots, V, d)) {
      const hipError_t e = attr::launch_embed_small((int)dout_dtype, (int)dtable_dtype, r, token, a, s);
      return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_embed_backward launch");
    }
    const EmbedLayout L = embed_layout(rows, V, d);
    if (!ws || ws_bytes < L.total)
      return fail(ATTR_ERR_WORKSPACE, "%s needs %zu workspace bytes, got %zu", who, L.total, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
    char* const base = static_cast<char*>(ws);
    attr::EmbedSort sort;
    for (int k = 0; k < 2; ++k) {
      sort.key[k] = reinterpret_cast<uint32_t*>(base + L.key[k]);
      sort.row[k] = reinterpret_cast<uint32_t*>(base + L.row[k]);
    }
    sort.count = reinterpret_cast<uint32_t*>(base + L.count);
    sort.passes = attr::sort_passes(V);
    sort.bits = attr::sort_bits(V);
    sort.blocks = (r.n_slots + attr::kSortKeys - 1) / attr::kSortKeys;
    const int eb = dtype_bytes(dtable_dtype);
    const attr::EmbedZero z{static_cast<char*>(dtable), accumulate ? 0 : V, d * eb, ldt * eb, 0, 0};
    hipError_t e = attr::launch_embed_sort(r, token, V, sort, z, s);
    if (e != hipSuccess) return device_fail(e, "attr_embed_backward sort launch");
    a.key = sort.key[sort.passes & 1];
    a.row = sort.row[sort.passes & 1];
    a.part = reinterpret_cast<float*>(base + L.part);
    a.n = r.n_slots;
    a.each = attr::embed_part(a.n, d);
    e = attr::launch_embed_grad((int)dout_dtype, (int)dtable_dtype, a, s);
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_embed_backward launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_embed_backward: host exception");
  }
}

namespace {

attr_status norm_validate(const attr_rows* r, int64_t d, const void* weight, const void* bias, attr_dtype w_dtype,
                          const char* who) {
  const attr_status st = rows_validate(r, who);
  if (st != ATTR_OK) return st;
  if (d < 1 || d > attr::kNormWidest)
    return fail(ATTR_ERR_INVALID_ARG, "%s: d=%lld must be in [1, %d]", who, (long long)d, (int)attr::kNormWidest);
  if ((weight || bias) && !valid_dtype(w_dtype))
    return fail(ATTR_ERR_UNSUPPORTED, "%s: weights must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
  const size_t wb = weight || bias ? (size_t)dtype_bytes(w_dtype) : 1;
  if (!aligned_to(weight, wb) || !aligned_to(bias, wb))
    return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
  return ATTR_OK;
}

// Whether d columns from p and d from q of matrices with row stride ld are columns of one matrix
// that do not touch.
bool columns_apart(const float* p, const float* q, int64_t d, int64_t ld) {
  const int64_t at = (int64_t)(reinterpret_cast<uintptr_t>(q) / 4) - (int64_t)(reinterpret_cast<uintptr_t>(p) / 4);
  const int64_t c = (at % ld + ld) % ld;
  return c >= d && c + d <= ld;
}

// (unit, units, chunks) of a gradient call.
void norm_split(const attr_rows* r, int64_t d, int32_t per_example, attr::NormGradArgs& a) {
  a.unit = (uint32_t)(per_example ? r->T : r->n_examples * r->T);
  a.units = (uint32_t)(per_example ? r->n_examples : 1);
  a.chunks = attr::norm_chunks(a.unit, a.units, (int32_t)d);
}
size_t norm_bytes(const attr::NormGradArgs& a, int64_t d) {
  return a.chunks > 1 ? align_up((size_t)a.units * a.chunks * 2 * (size_t)d * 4) : 0;
}

}  // namespace

attr_status attr_layer_norm(const attr_rows* rows, const void* x, attr_dtype x_dtype, int64_t d, int64_t ldx,
                            const void* weight, const void* bias, attr_dtype w_dtype, float eps, void* y,
                            attr_dtype y_dtype, int64_t ldy, float* mean, float* rstd, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_layer_norm";
    attr_status st = norm_validate(rows, d, weight, bias, w_dtype, who);
    if (st != ATTR_OK) return st;
    if (!(eps >= 0.f && eps <= 3.0e38f)) return fail(ATTR_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", who);
    if (rows->n_examples == 0 || rows->n_rows == 0) return ATTR_OK;
    st = matrix_validate(x, x_dtype, rows->n_rows, d, ldx, "x", who);
    if (st == ATTR_OK) st = matrix_validate(y, y_dtype, rows->n_rows, d, ldy, "y", who);
    if (st != ATTR_OK) return st;
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4))
      return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
    RowSpans spans(rows);
    if (!(y == x && y_dtype == x_dtype && ldy == ldx)) spans.input(span_of(x, rows->n_rows, d, ldx, dtype_bytes(x_dtype)));
    if (weight) spans.input(vector_span(weight, d, dtype_bytes(w_dtype)));
    if (bias) spans.input(vector_span(bias, d, dtype_bytes(w_dtype)));
    spans.output(span_of(y, rows->n_rows, d, ldy, dtype_bytes(y_dtype)));
    spans.output(vector_span(mean, rows->n_rows, 4));
    spans.output(vector_span(rstd, rows->n_rows, 4));
    if (spans.clash()) return overlap_fail(who);
    const attr::NormArgs a{x, weight, bias, y, mean, rstd, ldx, ldy, (int32_t)d, (int32_t)w_dtype, eps};
    const hipError_t e = attr::launch_layer_norm((int)x_dtype, (int)y_dtype, rows_args(rows), a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_layer_norm launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_layer_norm: host exception");
  }
}

size_t attr_layer_norm_backward_workspace_size(const attr_rows* rows, int64_t d, int32_t per_example) {
  if (!rows_sizes_ok(rows) || d < 1 || d > attr::kNormWidest || (per_example != 0 && per_example != 1) ||
      rows->n_examples == 0)
    return 0;
  attr::NormGradArgs a;
  norm_split(rows, d, per_example, a);
  return norm_bytes(a, d);
}

attr_status attr_layer_norm_backward(const attr_rows* rows, const void* dy, attr_dtype dy_dtype, int64_t lddy,
                                     const void* x, attr_dtype x_dtype, int64_t d, int64_t ldx, const float* mean,
                                     const float* rstd, const void* weight, attr_dtype w_dtype, void* dx, int64_t lddx,
                                     float* dweight, int64_t ldw, float* dbias, int64_t ldb, int32_t per_example,
                                     int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  try {
    g_err.clear();
    const char* who = "attr_layer_norm_backward";
    attr_status st = norm_validate(rows, d, weight, nullptr, w_dtype, who);
    if (st != ATTR_OK) return st;
    if ((per_example != 0 && per_example != 1) || (accumulate != 0 && accumulate != 1))
      return fail(ATTR_ERR_INVALID_ARG, "%s: per_example and accumulate must be 0 or 1", who);
    const int64_t units = per_example ? rows->n_examples : 1;
    if (dweight && (st = matrix_validate(dweight, ATTR_F32, units, d, per_example ? ldw : d, "dweight", who)) != ATTR_OK) return st;
    if (dbias && (st = matrix_validate(dbias, ATTR_F32, units, d, per_example ? ldb : d, "dbias", who)) != ATTR_OK) return st;
    if (rows->n_examples == 0 && (per_example || accumulate)) return ATTR_OK;
    const bool none = rows->n_examples == 0 || rows->n_rows == 0;
    if (!none) {
      st = matrix_validate(x, x_dtype, rows->n_rows, d, ldx, "x", who);
      if (st == ATTR_OK) st = matrix_validate(dy, dy_dtype, rows->n_rows, d, lddy, "dy", who);
      if (st == ATTR_OK && dx) st = matrix_validate(dx, x_dtype, rows->n_rows, d, lddx, "dx", who);
      if (st != ATTR_OK) return st;
      if (!mean || !rstd) return fail(ATTR_ERR_INVALID_ARG, "%s: mean or rstd is NULL", who);
      if (!aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return fail(ATTR_ERR_ALIGNMENT, "%s: pointers must be aligned to their elements", who);
    }
    if (!valid_dtype(x_dtype) || !valid_dtype(dy_dtype))
      return fail(ATTR_ERR_UNSUPPORTED, "%s: x and dy must be ATTR_F32, ATTR_BF16 or ATTR_F16", who);
    RowSpans spans(rows);
    if (!none) {
      if (!(dx == x && lddx == ldx)) spans.input(span_of(x, rows->n_rows, d, ldx, dtype_bytes(x_dtype)));
      if (!(dx == dy && dy_dtype == x_dtype && lddx == lddy)) spans.input(span_of(dy, rows->n_rows, d, lddy, dtype_bytes(dy_dtype)));
      if (weight) spans.input(vector_span(weight, d, dtype_bytes(w_dtype)));
      spans.input(vector_span(mean, rows->n_rows, 4));
      spans.input(vector_span(rstd, rows->n_rows, 4));
      if (dx) spans.output(span_of(dx, rows->n_rows, d, lddx, dtype_bytes(x_dtype)));
    }
    if (dweight) spans.output(span_of(dweight, units, d, per_example ? ldw : d, 4));
    if (dbias)
      spans.output(span_of(dbias, units, d, per_example ? ldb : d, 4),
                   dweight && per_example && ldw == ldb && columns_apart(dweight, dbias, d, ldw));
    if (spans.clash()) return overlap_fail(who);
    if (!dx && !dweight && !dbias) return ATTR_OK;
    attr::NormGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = x;
    a.dy = dy;
    a.weight = weight;
    a.mean = mean;
    a.rstd = rstd;
    a.dx = dx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.ldx = ldx;
    a.lddy = lddy;
    a.lddx = lddx;
    a.ldw = ldw;
    a.ldb = ldb;
    a.d = (int32_t)d;
    a.w_dtype = (int32_t)w_dtype;
    a.accumulate = accumulate;
    attr::RowsArgs r = rows_args(rows);
    if (none) {  // sums of no rows: one empty unit, or one for each example
      a.unit = a.chunks = 1;
      a.units = (uint32_t)units;
      r = attr::RowsArgs{nullptr, nullptr, 0, (uint32_t)units, 1};
    } else {
      norm_split(rows, d, per_example, a);
      const size_t need = norm_bytes(a, d);
      if (need && (!ws || ws_bytes < need))
        return fail(ATTR_ERR_WORKSPACE, "%s needs %zu workspace bytes, got %zu", who, need, ws ? ws_bytes : (size_t)0);
      if (reinterpret_cast<uintptr_t>(ws) & 255u) return fail(ATTR_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
      a.part = need ? static_cast<float*>(ws) : nullptr;
    }
    const hipError_t e = attr::launch_layer_norm_grad((int)x_dtype, (int)dy_dtype, r, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_layer_norm_backward launch");
  } catch (...) {
    return fail(ATTR_ERR_INVALID_ARG, "attr_layer_norm_backward: host exception");
  }
}

// ---------------------------------------------------------------------------
attr_status attr_probe_read(const void* x, size_t bytes, void* sink, void* stream) {
  g_err.clear();
  if (bytes == 0) return ATTR_OK;
  if (!x || !sink) return fail(ATTR_ERR_INVALID_ARG, "attr_probe_read: NULL pointer");
  if (!aligned16(x) || bytes % 16) return fail(ATTR_ERR_ALIGNMENT, "attr_probe_read: x and bytes must be 16-byte multiples");
  const hipError_t e = attr::launch_probe_read(x, bytes, sink, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_probe_read launch");
}

attr_status attr_probe_mfma(int64_t n_mfma, void* sink, void* stream) {
  g_err.clear();
  if (n_mfma <= 0 || n_mfma % 8) return fail(ATTR_ERR_INVALID_ARG, "attr_probe_mfma: n_mfma must be a positive multiple of 8");
  if (!sink) return fail(ATTR_ERR_INVALID_ARG, "attr_probe_mfma: NULL sink");
  const hipError_t e = attr::launch_probe_mfma(n_mfma, sink, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ATTR_OK : device_fail(e, "attr_probe_mfma launch");
}

}  // extern "C"
