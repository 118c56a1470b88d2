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
// embedding and layer norm over token rows
// ---------------------------------------------------------------------------
struct RowsArgs {
  const int64_t* row_offset;  // or null
  const int32_t* length;      // or null
  int64_t n_rows;
  uint32_t n_slots, T;
};
struct EmbedArgs {
  const int64_t* token;
  const void* table;
  void* out;
  int64_t V, ldt, ldo;
  int32_t d;
  float scale;
};
hipError_t launch_embed(int table_dtype, int out_dtype, const RowsArgs& r, const EmbedArgs& a, hipStream_t s);

// The gradient of a table: the batch's (token, row) pairs in the order of their tokens,
// rows of one token in the order of their slots; slots without a token have the key V.
struct EmbedSort {
  uint32_t* key[2];   // [n_slots] each; the sorted pairs are in [passes & 1]
  uint32_t* row[2];
  uint32_t* count;    // two of [bins][blocks], one workgroup's sort needs none
  int passes, bits;   // bits of a pass's digit
  uint32_t blocks;
};
constexpr uint32_t kSortOne = 4096;   // keys that one workgroup sorts alone
constexpr uint32_t kSortKeys = 2048;  // keys of each of several
constexpr int kSortBits = 9;          // of a digit, at most
inline int sort_passes(int64_t V) {
  int bits = 1;
  while ((V >> bits) != 0) ++bits;  // of the key V
  return (bits + kSortBits - 1) / kSortBits;
}
inline int sort_bits(int64_t V) {
  int bits = 1;
  while ((V >> bits) != 0) ++bits;
  const int passes = sort_passes(V);
  return (bits + passes - 1) / passes;
}
// The rows of a gradient that the sort's launches write zeros to, beside the sort (0 rows: none).
struct EmbedZero {
  char* to;
  int64_t rows, row, ld;    // row and stride in bytes
  uint32_t blocks, shares;  // workgroups of a launch, and of all; set by the launch
};
hipError_t launch_embed_sort(const RowsArgs& r, const int64_t* token, int64_t V, const EmbedSort& e, EmbedZero z, hipStream_t s);
// A wave adds up 64 N columns, N = embed_lane(d), of the rows of a part of neighbours in that order: of 32,
// or of 64 where those leave 16 waves a CU (65536 slots of 1024, 4096 waves: 89.0 us with parts of 32, 82.0 of
// 64; 32768 of 2048, 2048 waves: 99 and 115).  A token whose rows reach past a part leaves sums to be joined.
inline int embed_lane(int64_t d) { return d > 1024 ? 8 : d > 64 ? 4 : 1; }
inline uint32_t embed_cuts(int64_t d) { return (uint32_t)((d + 64 * embed_lane(d) - 1) / (64 * embed_lane(d))); }
inline uint32_t embed_part(uint64_t n, int64_t d) { return n / 64 * embed_cuts(d) >= 4096 ? 64 : 32; }
struct EmbedGradArgs {
  const uint32_t* key;
  const uint32_t* row;
  const void* dout;
  void* dtable;
  float* part;        // [parts][2][d]: of the token that began before, of the one that goes on
  int64_t V, ldd, ldt;
  uint32_t n;         // pairs, those without a token last
  uint32_t each;      // pairs of a part
  int32_t d, accumulate;
  float scale;
};
// Whether a batch needs no sort: up to kEmbedSmall slots, searched for every row of the table (400 slots, a
// table of 8192 x 1024: 13.3 us without a sort, 24.2 with it), unless these searches are many (256 slots and
// 128256 x 2048, added to, 2.1M searches of 64 slots: 36.9 us and 25.5).
constexpr uint32_t kEmbedSmall = 512;
inline int embed_small_lane(int64_t d) { return d > 256 ? 8 : d > 64 ? 4 : 1; }
inline uint32_t embed_small_cuts(int64_t d) { return (uint32_t)((d + 64 * embed_small_lane(d) - 1) / (64 * embed_small_lane(d))); }
inline bool embed_searches(uint64_t n, int64_t V, int64_t d) {
  return n <= kEmbedSmall && (n + 63) / 64 * (uint64_t)V * embed_small_cuts(d) <= (1u << 20);
}
hipError_t launch_embed_small(int dout_dtype, int table_dtype, const RowsArgs& r, const int64_t* token, const EmbedGradArgs& a,
                              hipStream_t s);
hipError_t launch_embed_grad(int dout_dtype, int table_dtype, const EmbedGradArgs& a, hipStream_t s);

struct NormArgs {
  const void* x;
  const void* weight;  // or null: 1
  const void* bias;    // or null: 0
  void* y;
  float* mean;         // or null
  float* rstd;         // or null
  int64_t ldx, ldy;
  int32_t d, w_dtype;
  float eps;
};
hipError_t launch_layer_norm(int x_dtype, int y_dtype, const RowsArgs& r, const NormArgs& a, hipStream_t s);

// A unit is what the weights' gradients are summed over: an example's slots, or all of
// them; a workgroup sums a share of a unit's slots.
struct NormGradArgs {
  const void* x;
  const void* dy;
  const void* weight;  // or null: 1
  const float* mean;
  const float* rstd;
  void* dx;            // or null
  float* dweight;      // or null
  float* dbias;        // or null
  float* part;         // [units * chunks][2][d], or null: a unit is one share
  int64_t ldx, lddy, lddx, ldw, ldb;
  int32_t d, w_dtype, accumulate;
  uint32_t unit;       // slots of a unit
  uint32_t chunks;     // shares of a unit
  uint32_t units;
};
uint32_t norm_chunks(uint32_t unit, uint32_t units, int32_t d);
hipError_t launch_layer_norm_grad(int x_dtype, int dy_dtype, const RowsArgs& r, const NormGradArgs& a, hipStream_t s);
constexpr int32_t kNormWidest = 32768;

// ---------------------------------------------------------------------------
// Muon
// ---------------------------------------------------------------------------
struct MuonEntry {
  void* p;
  const void* g;
  float* m;
  float* master;
  float lr, lr_wd;
};
constexpr int kMuonTable = 96;  // entries that travel in one launch's arguments
struct MuonTable {
  MuonEntry* to;
  int32_t n, pad;
  MuonEntry e[kMuonTable];
};
static_assert(sizeof(MuonTable) <= 4096, "kernel arguments");
// Matrices of one shape.  Y is the update with its longer side first, [L][S] with rows of ld
// halves; each is held as 16-bit values, and with pairs as two (the second `lo` bytes after the
// first).
struct MuonGroup {
  char* base;             // of the first matrix's buffers
  int64_t stride;         // bytes from a matrix's to the next one's
  int64_t y[2], gram, poly, norm;  // byte offsets in a matrix's buffers
  int64_t lo_y, lo_s;     // from the first halves to the second: of Y; of gram and poly
  uint32_t tile_sym, tile_full, tile_flat, tile_turn;  // first workgroup of the group in each launch
  uint32_t n_sym, n_full, n_flat, n_turn;              // workgroups of a matrix
  uint32_t entry, count;  // first matrix in the table, matrices
  char* part;             // the partial sums of A's tiles, [count][splits][n_sym] tiles of fp32; with one split none
  uint32_t tile_gram, splits;  // first workgroup of A's launch; parts of Y's rows (of split_rows), one a workgroup
  int32_t split_rows, pad;
  int32_t rows, cols, L, S, ld;
};
// Workgroups of a group's n tiles: an eighth for each die.
inline uint32_t muon_tiles(uint32_t n) { return (n + 7) / 8 * 8; }
constexpr int kMuonGroups = 16;
struct MuonArgs {
  const MuonEntry* table;
  const float* grad_scale;
  float momentum, one_momentum;
  int32_t nesterov, n_groups;
  MuonGroup g[kMuonGroups];
};
static_assert(sizeof(MuonArgs) <= 4096, "kernel arguments");
// Shorter sides up to kThinMost: the iteration on their products (t: their sixteens); a workgroup takes
// kThinRows of the longer side.  A group's workgroups are its tile_flat and n_flat; gram is its parts'
// place, poly that of what u is multiplied by.
constexpr int kThinMost = 64, kThinRows = 256;
constexpr uint32_t kThinParts = 32;  // more parts of a matrix are added up by a launch of their own
hipError_t launch_muon_thin_gram(int g_dtype, int t, const MuonArgs& a, uint32_t blocks, hipStream_t s);
hipError_t launch_muon_thin_sum(int t, const MuonArgs& a, uint32_t matrices, hipStream_t s);
hipError_t launch_muon_thin_poly(int t, int steps, const MuonArgs& a, uint32_t matrices, hipStream_t s);
hipError_t launch_muon_thin_apply(int p_dtype, int g_dtype, bool master, int t, const MuonArgs& a, uint32_t blocks, hipStream_t s);
constexpr int kMuonTile = 128;
// A launch of few of A's tiles divides Y's rows: into parts of kMuonSplitRows rows or more, kMuonSplits
// at most, one workgroup for each slot of the GPU.
constexpr int kMuonSplitRows = 512, kMuonSplits = 32;
constexpr int64_t kMuonFlat = 16384;   // elements of a workgroup of the momentum's launch, at least
constexpr uint32_t kMuonFlatMost = 256;  // such workgroups of a matrix
hipError_t launch_muon_table(const MuonTable& t, hipStream_t s);
hipError_t launch_muon_momentum(int g_dtype, const MuonArgs& a, uint32_t blocks, hipStream_t s);
hipError_t launch_muon_split(int g_dtype, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s);
// big: tiles of 256 x 256, whose numbers the groups then hold
hipError_t launch_muon_gram(bool big, bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s);
// A from the parts' sums, of the groups with more than one; blocks as for the polynomial
hipError_t launch_muon_join(bool big, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s);
hipError_t launch_muon_poly(bool big, bool pairs, const MuonArgs& a, uint32_t blocks, hipStream_t s);
hipError_t launch_muon_apply(bool big, bool pairs, int from, const MuonArgs& a, uint32_t blocks, hipStream_t s);
hipError_t launch_muon_last(bool big, bool pairs, int p_dtype, bool master, int from, const MuonArgs& a, uint32_t blocks,
                            hipStream_t s);

// ---------------------------------------------------------------------------
// calibration
// ---------------------------------------------------------------------------
hipError_t launch_probe_read(const void* x, size_t bytes, void* sink, hipStream_t s);
hipError_t launch_probe_mfma(int64_t n_mfma, void* sink, hipStream_t s);

}  // namespace attr
