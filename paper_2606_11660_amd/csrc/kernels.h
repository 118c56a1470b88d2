// Internal interface between the C-ABI layer (api.cpp) and the HIP kernels.
// Nothing here is exported from the shared library.
#pragma once

#include <hip/hip_runtime_api.h>
#include <hip/hip_vector_types.h>
#include <stddef.h>
#include <stdint.h>

namespace attr {

// ---------------------------------------------------------------------------
// projection
// ---------------------------------------------------------------------------
// One module slot of the projection's device-side table (slots are in
// launch order, largest modules first).
struct ProjTab {
  const void* a;
  const void* g;
  const void* pk;     // packed S fragments, then packed R fragments
  int64_t lda, ldg, out_col;
  int32_t d_in, d_out;
};

// One work group of the projection: ms consecutive slots from slot0 whose
// modules share their input rows (ms = 1 for a module on its own).
struct ProjGroup {
  int32_t slot0, ms;
};

// Host -> device upload of module descriptors travels in kernel arguments (4096
// bytes in all).  80 bytes an entry: the 48 modules of a GPT-2-shaped model go in
// one launch (at 24 entries a launch, a 389-token query's call took 45.4 us, now
// 41.7).
struct PackEntry {
  const void* a;
  const void* g;
  const void* R;
  const void* S;
  const float* v_out;  // optional factored second moment (both or neither)
  const float* v_in;
  int64_t out_col;
  int32_t lda, ldg;    // 256 rows span less than 2^31 bytes
  uint32_t pk_off;     // in 256-byte units
  int32_t d_in, d_out;
  int16_t grp;      // group of this slot
  int16_t lead_ms;  // group size if this slot is the group's first, else 0
};
static_assert(sizeof(PackEntry) == 80, "entries per launch");
constexpr int kPackMax = 48;
struct PackArgs {
  PackEntry e[kPackMax];
  int32_t n;
  int32_t slot0;
};

// Tokens handled by one workgroup of the general projection kernel for fragment
// width nk (k = 16 nk); per-token calls (tok) take fewer at k = 32 and 64.
constexpr int project_chunk_tokens(int nk, bool tok) { return tok ? 256 / nk : 256; }
// Bytes of packed S and R for one module.
size_t project_packed_bytes(int64_t d_in, int64_t d_out, int k, int elem_bytes);

// Static device scratch of attr_project_noalloc (per GPU, 256-byte aligned):
// its device address on the current device, resolved once per device.
constexpr size_t kProjectScratchBytes = (size_t)64 << 20;
hipError_t project_scratch(void** ptr);

hipError_t launch_project_pack(bool bf16, int nk, const PackArgs& args, ProjTab* tab,
                               ProjGroup* gtab, char* pk_base, hipStream_t s);
// Modules sharing their input rows (same a, lda, d_in) are projected in
// groups of up to kProjGroupMax consecutive slots (one read of a per group).
// One launch covers every (group, token chunk, example) item, groups in
// table order (largest work first).
constexpr int kProjGroupMax = 3;
// Work list of a call with per-example lengths (device-built): examples
// sorted by chunk count, longest first, and the item offset of each chunk
// row.  Built when length is given, n_chunks <= kWorklistMaxChunks and
// n_examples <= kWorklistMaxExamples; otherwise the main kernel decodes its
// block index densely.
constexpr int kWorklistMaxChunks = 2048;
constexpr int64_t kWorklistMaxExamples = 1 << 20;
inline bool project_uses_worklist(const int32_t* length, int64_t n_ex, int n_chunks) {
  return length && n_chunks <= kWorklistMaxChunks && n_ex <= kWorklistMaxExamples;
}
// tok: per-token blocks written straight into `partial` = the output [n_rows, ldo]
// wl_perm / wl_off: the work list (both NULL for the dense decode).
hipError_t launch_project_main(bool bf16, int nk, const ProjTab* tab, const ProjGroup* gtab,
                               int n_groups, int n_chunks, int64_t n_ex, int64_t T,
                               const int64_t* row_offset, const int32_t* length,
                               int32_t* wl_perm, int32_t* wl_off,
                               float* partial, hipStream_t s, bool tok = false, int64_t ldo = 0,
                               int64_t n_rows = 0);
// Calls with few items: chunks of ct tokens, the contraction split over the
// waves of a workgroup (ct = 0: the call takes the general kernel).  The rule
// is plan_project_few in project_plan.h (host only).
struct ProjFewPlan {
  int ct, n_chunks;
};
// Chunks [c0, c0 + nc) of every (slot, example).  dst: the output (tok, or a
// single chunk per example) or the partials [slot][chunk - c0][example][k k].
hipError_t launch_project_few(bool bf16, int nk, const ProjFewPlan& P, int c0, int nc, const ProjTab* tab,
                              int n_slots, int64_t n_ex, int64_t T, const int64_t* row_offset,
                              const int32_t* length, float* dst, bool tok, int64_t ldo, int64_t n_rows,
                              hipStream_t s);
// Adds the partials of chunks [c0, c0 + nc) (CT tokens each) to the rows of the
// chunks before, in chunk order: the same bits whether the chunks of a call come
// in one round or in several.
hipError_t launch_project_reduce(int nk, int CT, int c0, int nc, const ProjTab* tab, int n_slots,
                                 int64_t n_ex, int64_t T, const int32_t* length, const float* partial,
                                 float* out, int64_t ldo, hipStream_t s);

// ---------------------------------------------------------------------------
// row-wise preconditioning / normalisation (NONE and DIAG)
// ---------------------------------------------------------------------------
// x_dtype / y_dtype: 0 = fp32, 2 = fp16 (attr_dtype values).
// row_ss (optional): n_ss partial sums of squares per row that give the
// norm; seg_e (optional, with row_ss): per row, the exponent e of each
// 128-column segment of X, which holds y 2^-e (y = X 2^e is normalised).
hipError_t launch_rowscale(int x_dtype, int y_dtype, const void* X, int64_t ldx,
                           int64_t n_rows, int64_t D, const float* m, int unit,
                           const float* row_ss, const int8_t* seg_e, int64_t n_ss, void* Y,
                           int64_t ldy, hipStream_t s);

// ---------------------------------------------------------------------------
// diagonal accumulate
// ---------------------------------------------------------------------------
int colsumsq_panels(int64_t n_rows, int64_t D);
hipError_t launch_colsumsq(int x_dtype, const void* X, int64_t ldx, int64_t n_rows,
                           int64_t D, float* H, double* part, hipStream_t s);

// ---------------------------------------------------------------------------
// scoring
// ---------------------------------------------------------------------------
struct ScorePlan {
  int n_qb;              // query blocks of 64 queries
  int n_grp;             // 128-byte K-groups per row
  int split_plan;        // split-K plan (else: streaming or GEMM)
  int split;             // its D-slices
  int n_tiles;           // 128-row tiles (split-K plan)
  int n_parts;           // row partitions, one sorted list each per query
  int64_t rows_per_part;
  size_t spart_bytes;    // split-K partial scores / GEMM-plan score chunk
  size_t list_entries;   // n_q * n_parts * k
  int gemm;              // GEMM plan (1: 256 x 256 tiles, 2: 128 x 256 ring): row chunks of `chunk` rows, one list per chunk
  int64_t chunk;
  int64_t D;
  int64_t bound_rows;    // streaming plan: rows of the prefix scan that bounds the k-th best (0: none)
};
// fewest_bytes: no plan that takes more workspace for speed
ScorePlan plan_score(int64_t n_q, int64_t n_g, int64_t D, int k, int elem_bytes, bool fewest_bytes);
hipError_t launch_score_topk(bool f16, const ScorePlan& plan, const void* Q, int64_t n_q,
                             int64_t ldq, const void* G, int64_t n_g, int64_t ldg, int k,
                             int64_t index_base, int merge, float* top_s, int64_t* top_i,
                             float* part_s, int64_t* part_i, float* spart, hipStream_t s);

// ---------------------------------------------------------------------------
// full second moment: accumulate (SYRK) and apply
// ---------------------------------------------------------------------------
struct SyrkPlan {
  int nt;          // 256-wide tiles per side
  int n_up;        // upper-triangle tiles
  int J;           // K-slices per chunk
  int64_t Cs;      // rows per slice
  int64_t C;       // rows per chunk (J * Cs)
  size_t part_bytes, h64_bytes;
};
// plan_syrk(n_rows, D, ldx) is in syrk_plan.h (host only).
hipError_t launch_syrk(bool bf16, const void* X, int64_t ldx, int64_t n_rows, int64_t D, float* H,
                       const SyrkPlan& P, void* part, void* h64, hipStream_t s);

int apply_full_nss(int64_t D);
size_t apply_full_workspace(int64_t n_rows, int64_t D, int unit);
hipError_t launch_apply_full(const void* X, int64_t n_rows, int64_t ldx, int64_t D, const float* M,
                             int y_dtype, void* Y, int64_t ldy, int unit, void* ws,
                             hipStream_t s);

// FULL apply on few rows (apply_few.hip): M read once straight from the
// caller, fp32 partials per K-slice in the workspace.  use: this row count
// takes that path (the rule and its measurements are at plan_apply_few).
struct ApplyFewPlan {
  bool use;
  int xt;                 // 16-row tiles of X per wave
  int n_ct, n_sl, n_rb;   // column tiles, K-slices, row blocks
  size_t part_bytes;      // fp32 partials, then
  size_t pack_bytes;      // X in fragment order (0: read in place)
};
ApplyFewPlan plan_apply_few(int64_t n_rows, int64_t D);
hipError_t launch_apply_few(const ApplyFewPlan& P, const void* X, int64_t n_rows, int64_t ldx,
                            int64_t D, const float* M, int y_dtype, void* Y, int64_t ldy, int unit,
                            void* ws, hipStream_t s);

// ---------------------------------------------------------------------------
// losses over token log-probabilities
// ---------------------------------------------------------------------------
constexpr int kTokenLogp = 0, kTokenPolicy = 1, kTokenPref = 2;  // the three calls
struct TokenArgs {
  const void* logits;
  const int64_t* target;
  const float* weight;         // or null
  const int64_t* row_offset;   // or null
  const int32_t* length;       // or null
  float* logp;                 // or null
  void* dlogits;               // or null
  float2* stats;               // per slot: a row's offset and sum (preference loss)
  double* part;                // per slot: its share of the log ratio (preference loss)
  float2* parts;               // per slot and part of its row: maximum and sum (n_parts > 1)
  float* zy;                   // per slot: the target's logit (n_parts > 1)
  int64_t n_rows, ldl, ldd;
  uint32_t n_slots, T;         // slot = example * T + token
  uint32_t slot0;              // of a launch
  int32_t V;
  int32_t n_parts, part_len;   // a row's parts and their elements (1 and V: whole rows)
  float scale;
};
struct PolicyArgs {
  const float* advantage;
  const float* logp_old;       // or null
  const float* logp_ref;       // null only with beta 0
  float* token_loss;           // per slot
  float lo, hi, beta;          // ratio bounds
  int32_t per_token;
};
struct PrefArgs {
  const float* logp_ref;       // or null
  const float* pair_weight;    // or null
  float* loss;
  float* log_ratio;            // or null
  float* coef;                 // per pair: dloss/dlogp of a chosen token of weight 1
  uint32_t n_pairs;
  float beta, margin, smoothing;
};
int token_parts(int mode, int64_t n_slots, int64_t row_bytes);
hipError_t launch_token_logp(int dtype, const TokenArgs& a, hipStream_t s);
// Policy loss: token losses of every slot, then their sums; or both at once.
hipError_t launch_policy_rows(int dtype, const TokenArgs& a, const PolicyArgs& p, hipStream_t s);
hipError_t launch_example_sum(const float* token_loss, uint32_t T, uint32_t n, float* loss, hipStream_t s);
constexpr uint32_t kPolicyExampleMost = 32;  // tokens of an example
bool policy_by_example(int64_t row_bytes, int64_t T, int64_t n_examples);
hipError_t launch_policy_examples(int dtype, const TokenArgs& a, const PolicyArgs& p, uint32_t n, float* loss,
                                  hipStream_t s);
// Preference loss: all of it at once; or a row's sums and its share of the log ratio,
// the pairs, and the gradient, with the pairs (pair) or after them.
constexpr uint32_t kPrefPairMost = 16;  // tokens of a sequence
bool pref_by_pair(int64_t row_bytes, int64_t T, int64_t n_pairs);
bool pref_pairs_within(int64_t row_bytes, int64_t T, int64_t n_slots);
hipError_t launch_pref_pairs(int dtype, const TokenArgs& a, const PrefArgs& p, hipStream_t s);
hipError_t launch_pref_stats(int dtype, const TokenArgs& a, const PrefArgs& p, hipStream_t s);
hipError_t launch_pairs(const TokenArgs& a, const PrefArgs& p, hipStream_t s);
hipError_t launch_pref_grad(int dtype, bool pair, const TokenArgs& a, const PrefArgs& p, hipStream_t s);

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
// One tensor, or a piece of one, of a launch; descriptors travel in kernel arguments
// (4096 bytes).  What only masters and 8-bit states need is apart: 84 tensors a launch
// without it, 55 with it.
struct AdamwEntry {
  void* p;
  const void* g;
  void* m;
  void* v;
  float lr, lr_wd;  // of the corrected first moment, of the weight
  uint32_t n;       // elements
  uint32_t chunk0;  // first workgroup
};
struct AdamwExtra {
  float* master;
  float* m_scale;
  float* v_scale;
};
constexpr int kAdamwMost = 84, kAdamwMostExtra = 55;
struct AdamwStep {
  const float* grad_scale;  // or null
  float beta1, one_beta1, beta2, one_beta2, corr2, eps, eps_root;
  int32_t n;
};
struct AdamwPlain {
  AdamwStep step;
  AdamwEntry e[kAdamwMost];
};
struct AdamwFull {
  AdamwStep step;
  AdamwEntry e[kAdamwMostExtra];
  AdamwExtra x[kAdamwMostExtra];
};
static_assert(sizeof(AdamwPlain) <= 4096 && sizeof(AdamwFull) <= 4096, "kernel arguments");
// A wave takes runs of 256 elements (a block of the 8-bit states), a workgroup four
// waves' chunk of them.
constexpr int kAdamwRun = 256;
int adamw_runs_per_wave(int64_t elements, bool eight);
// 32-bit states: elements of the first run that would be before the tensor's start, so
// that every run starts at a 128-byte line of the first moment.
#ifdef __HIPCC__
__host__ __device__
#endif
inline int adamw_lead(const void* m) { return (int)(reinterpret_cast<uintptr_t>(m) & 127) >> 2; }
// Every tensor of a launch has a master, or none has.  AdamwPlain: no masters, 32-bit
// states.
hipError_t launch_adamw(int p_dtype, int g_dtype, int runs, uint32_t blocks, const AdamwPlain& a, hipStream_t s);
hipError_t launch_adamw(int p_dtype, int g_dtype, bool eight, bool master, int runs, uint32_t blocks,
                        const AdamwFull& a, hipStream_t s);

// ---------------------------------------------------------------------------
// calibration
// ---------------------------------------------------------------------------
hipError_t launch_probe_read(const void* x, size_t bytes, void* sink, hipStream_t s);
hipError_t launch_probe_mfma(int64_t n_mfma, void* sink, hipStream_t s);

}  // namespace attr
