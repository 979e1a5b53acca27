// Internal launch interface between the C ABI (api.cpp) and the HIP kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dpg {

enum { DT_F32 = 0, DT_BF16 = 1 };  // element type of the float operands

// ----------------------------------------------------------------- Gram norm
constexpr int GR_TM = 128;          // rows of one T-tile
constexpr int GR_MAX_LAYERS = 52;   // layers per launch (kernel arguments stay < 4 KiB)
// bf16 launches with aligned rows and 128 < T <= 256 reduce each example's
// whole 256 x 256 Gram in one work item (one partial slot per chunk) instead
// of one item per T-tile pair.
inline bool gram_whole(int dt, bool vec, int T) {
  return dt == DT_BF16 && vec && T > GR_TM && T <= 2 * GR_TM;
}
// Gram workgroups resident per CU: two for the single-tile kernels (T <= 128),
// one for the others.
inline int gram_groups_per_cu(int T) { return T <= GR_TM ? 2 : 1; }
// Gram launches that can fuse a layer's bias gradient (every example row of
// a stage is in LDS at once).
inline bool gram_fuses_bias(int dt, bool vec, int T) {
  return dt == DT_BF16 && vec && T <= 2 * GR_TM;
}

struct GramLayer {
  const void* A;        // [B*T rows, lda] activations
  const void* G;        // [B*T rows, ldg] output grads
  int64_t lda, ldg;
  int32_t d_in;         // A features
  int32_t g0, g1;       // G feature range of this entry
  int32_t kg;           // G features per chunk
  int32_t nc;           // number of G chunks
  uint32_t item_begin;  // first work item of this layer among an example's items
  int32_t slot_begin;   // first partial slot of this layer in an example's row
  // The layer's bias gradient, fused (bf16, 16-byte rows, T <= 256 only):
  // row b of [B, g1] gets sum_t G[b,t,:], and its squared norm joins the
  // example's partial sums. Null: no bias.
  float* bias;
};

// Work items are numbered example-major: example b owns items
// [b * per_ex, (b + 1) * per_ex), one per (layer, T-tile pair, G chunk), so
// that the contiguous item range each XCD walks holds whole examples (equal
// work per XCD, and an example's G chunks share its A rows in one L2).
struct GramArgs {
  GramLayer L[GR_MAX_LAYERS];
  int32_t n_layers;
  int32_t B, T, n_t, P;   // T-tiles per side, upper-triangle tile pairs
  int32_t slots;          // partial slots per example
  uint32_t per_ex;        // work items per example
  uint32_t n_items;
  float* ws;              // [B, slots]
};

static_assert(sizeof(GramArgs) <= 4096, "kernel arguments must stay within 4 KiB");
hipError_t launch_gram_norm(const GramArgs& a, int dt, bool vec, hipStream_t s);

// Tied cross term: sum_{t,s} Gz[s, ids[t]] <dE_t, H_s>, all T-tile pairs.
constexpr int CR_FCHUNK = 128;  // features per cross-term work item
constexpr int CR_DL_ROWS = 64;  // row block of the direct-load cross kernel
constexpr int CR_RX_ROWS = 32;  // token and row blocks of the register-direct cross kernel
constexpr int CX_ROWS_T = 128;  // longest example given to it (measured: at T = 256 its
                                // 32-row blocks re-read E and H more than dl_cross's 64-row ones)
// Cross-term kernel of a call: the register-staged tied_cross_kernel (fp32 or
// unaligned rows), the register-direct cross_rows_kernel (bf16, aligned rows,
// T <= CX_ROWS_T) or the direct-load dl_cross_kernel (bf16, aligned, longer T).
enum { CROSS_STAGED = 0, CROSS_DL = 1, CROSS_ROWS = 2 };
inline int cross_kind(int dt, bool vec, int T) {
  if (dt != DT_BF16 || !vec) return CROSS_STAGED;
  return T <= CX_ROWS_T ? CROSS_ROWS : CROSS_DL;
}

struct CrossArgs {
  const int32_t* ids;   // [B,T]
  const void* E;        // dE [B*T, lde]
  const void* H;        // [B*T, ldh]
  const void* Gz;       // [B*T, ldz]
  int64_t lde, ldh, ldz;
  int32_t B, T, V, d, n_t;  // n_t: row blocks per example (128, 64 or 32 rows by kernel)
  int32_t n_fc;         // feature chunks (1 for bf16 aligned: all features per item)
  int32_t kind;         // CROSS_STAGED, CROSS_DL or CROSS_ROWS
  int32_t slots;        // n_t * n_t * n_fc
  float* ws;            // [B, slots]
};
hipError_t launch_tied_cross(const CrossArgs& a, int dt, bool vec, hipStream_t s);

// out[b] = (acc ? out[b] : 0) + scale * sum_j ws[b*slots + j], fixed order.
hipError_t launch_finish_rows(const float* ws, int B, int slots, float* out, int accumulate,
                              float scale, hipStream_t s);

// ------------------------------------------------------- K-major GEMM family
constexpr int GM_BM = 256, GM_BN = 256;
constexpr int GM_MAX_LAYERS = 52;   // layers per launch (kernel arguments stay < 4 KiB)

struct GemmLayer {
  const void* X;        // [K rows, ldx]
  const void* Y;        // [K rows, ldy]
  float* out;           // clipped sum: [M, ldo] (from a gradient store also transposed, [N, ldo])
  union {
    int64_t ldx;          // row stride of X in elements
    int64_t store_slot;   // sum from a gradient store (X, Y unread): first tile slot
  };
  union {
    int64_t ldy;          // row stride of Y in elements
    int64_t store_transpose;  // sum from a gradient store: 1 = output [N, ldo]
  };
  int64_t ldo;          // row stride of out in elements
  int32_t M, N;         // X columns (output rows) and Y columns (output columns)
  uint16_t tm, tn;      // 256-wide tiles along M and N
  uint32_t tile_begin;  // first work item of this entry
  union {
    int32_t slot_begin;   // direct norm: first partial slot in an example's row
    uint32_t tensor_id;   // clipped sum with noise: the tensor's generator id
  };
  int32_t accumulate;   // clipped sum: out += (else out =)
};

struct GemmArgs {
  GemmLayer L[GM_MAX_LAYERS];
  int32_t n_layers;
  int32_t B, T;
  uint32_t n_items;
  const float* c;       // clipped sum: per-example scale [B]
  float* ws;            // direct norm: [B, slots]
  int32_t slots;
  // Gaussian mechanism fused into the clipped sum's store (noise != 0):
  // out = (prior + sum + sigma_c * z) * inv_b, z from Philox (seed, tensor_id,
  // step) at the element's row-major index in the output tensor.
  int32_t noise;
  float sigma_c, inv_b;
  uint32_t step;
  uint64_t seed;
  // Tail split of the clipped sum: tiles [0, n_full) are
  // whole work items; each of the n_split tiles after them is ksplit items
  // over consecutive K ranges, whose fp32 partial tiles (256 x 256, row-major)
  // go to part and are added by the fixup kernel. n_full = n_items, ksplit = 1
  // when nothing is split.
  uint32_t n_full, n_split;
  int32_t ksplit;
  float* part;
  int32_t big;          // some operand spans 4 GiB or more (direct-load kernel rebases per stage)
  // Direct norm, direct-load kernel: examples per work item (a tile over eg
  // consecutive examples; items of one layer are group-major). 1 elsewhere.
  int32_t eg;
  // Per-example gradient store: the direct norm (direct-load kernel) also
  // writes each example's fp32 tile there; store_sum_kernel reads it back.
  // Tile slot q of example e is the 65536 floats at ((q * B + e) << 16), in
  // the register order of the 8 waves (GRAD_STORE layout below).
  float* store;
};

static_assert(sizeof(GemmArgs) <= 4096, "kernel arguments must stay within 4 KiB");

// Forms of the bf16 GEMM's stages (32 rows each).
//  PLAIN:  16-byte rows, T a multiple of 32, loaded straight into LDS.
//  BIG:    the same with an operand of 4 GiB or more.
//  RAGGED: 16-byte rows, any T: an example's last stage may be short; its
//          missing rows read as zeros.
//  STAGED: rows of any alignment, any T, loaded through registers.
//  SCALED, ROWS: (clipped sum) stages run over the batch's rows without regard to
//          examples, and one operand's rows are scaled by their examples' factors, which
//          rounds c_i A (or c_i G) to bf16: SCALED (16-byte rows) loads like PLAIN
//          and scales the fragments, ROWS loads like STAGED and scales what it stages. For
//          short examples, whose padding to whole stages would cost more than ROWS_NUM /
//          ROWS_DEN of their rows. By time alone they would pay earlier; the line is where it is
//          because the other forms scale in fp32 (error 3e-7 where these have 1.3e-3). Twelve
//          layers 768 -> 3072, 3072 tokens, us: T = 21: 217 SCALED, 353 RAGGED; 404 ROWS,
//          592 STAGED (unaligned); T = 22: 217, 337; 404, 565; T = 42: 217, 271; 404,
//          489; T = 43: 217, 255; 404, 477.
//  FP32:   the fp32 kernel (split_gemm_kernel).
enum GemmForm { FORM_PLAIN = 0, FORM_BIG, FORM_RAGGED, FORM_STAGED, FORM_ROWS, FORM_SCALED, FORM_FP32 };
constexpr int DL_SUM_BK = 32;
constexpr int DL_SUM_MAXB = 4096;  // clip factors held in LDS
constexpr int ROWS_NUM = 3, ROWS_DEN = 2;
inline int sum_form(int dt, bool vec, int T, int B) {
  if (dt != DT_BF16) return FORM_FP32;
  if (T % DL_SUM_BK == 0) return !vec ? FORM_STAGED : B <= DL_SUM_MAXB ? FORM_PLAIN : FORM_RAGGED;
  const int64_t padded = (int64_t)((T + DL_SUM_BK - 1) / DL_SUM_BK) * DL_SUM_BK;
  if (padded * ROWS_DEN > (int64_t)T * ROWS_NUM) return vec ? FORM_SCALED : FORM_ROWS;
  return vec ? FORM_RAGGED : FORM_STAGED;
}
inline int norm_form(bool vec, int T) {
  return !vec ? FORM_STAGED : T % DL_SUM_BK == 0 ? FORM_PLAIN : FORM_RAGGED;
}
// The launches whose operands may span 4 GiB or more.
inline bool dl_sum_applies(int dt, bool vec, int T, int B) {
  return dt == DT_BF16 && vec && T % DL_SUM_BK == 0 && B <= DL_SUM_MAXB;
}

constexpr int SP_BK = 16;          // K rows per stage of the fp32 kernel
// K stages of a clipped sum's launch.
inline int sum_stages(int form, int T, int B) {
  const int64_t K = (int64_t)B * T;
  if (form == FORM_FP32) return (int)((K + SP_BK - 1) / SP_BK);
  if (form == FORM_ROWS || form == FORM_SCALED) return (int)((K + DL_SUM_BK - 1) / DL_SUM_BK);
  return (int)((int64_t)B * ((T + DL_SUM_BK - 1) / DL_SUM_BK));
}

// The last round of a launch of n_tiles equal tiles on `cus` CUs holds
// r = n_tiles mod cus of them (all of them if n_tiles < cus). When r is at most
// half the CUs, each of those tiles may be split into ks consecutive K ranges of at
// least 4 stages (ks <= 8, r * ks <= cus). The round then takes about 1/ks of a
// tile's time, plus the fix-up launch (SPLIT_US) and the partial tiles' way to memory and
// back (SPLIT_PART_US each: 512 KB at about 6 TB/s); where noise is drawn, the fix-up
// spreads that over the chip too, which takes a whole tile SPLIT_NOISE_US. The largest ks
// that gains by this is taken (shorter ranges round less), 1 where none does. Measured, whole
// and split: norm and plain sum of one 768 -> 3072 layer at K = 3072 (36 tiles) 84 and 62 us; plain
// sums of four layers 768 -> 2304, 768, 3072 and 3072 -> 768 at K = 256 (108 tiles) 14 and 32,
// with noise 29 and 38; of one tile at K = 256 with noise 30 and 17.
constexpr double SPLIT_US = 3.0, SPLIT_PART_US = 0.0875, SPLIT_NOISE_US = 13.0;
// Time of one K stage of a tile (us) on a chip with few tiles, by the form of the sum.
inline double stage_us(int form) {
  switch (form) {
    case FORM_PLAIN: return 0.66;
    case FORM_SCALED: return 0.8;
    case FORM_RAGGED: return 1.1;
    case FORM_FP32: return 2.4;
    default: return 1.9;
  }
}
struct TailSplit {
  uint32_t n_full, n_split;
  int32_t ks;
};
inline TailSplit tail_split(uint64_t n_tiles, int k_stages, int form, bool noised, int cus) {
  TailSplit t{(uint32_t)n_tiles, 0u, 1};
  if (cus <= 0 || n_tiles == 0) return t;
  const uint64_t r = n_tiles % (uint64_t)cus;
  if (r == 0 || 2 * r > (uint64_t)cus) return t;
  const int top = (int)((uint64_t)cus / r);
  int ks = top < 8 ? top : 8;
  ks = ks < k_stages / 4 ? ks : k_stages / 4;
  const double whole = k_stages * stage_us(form) + (noised ? SPLIT_NOISE_US : 0.0);
  auto gains = [&](int n) {
    return (k_stages + n - 1) / n * stage_us(form) + SPLIT_US + (double)r * n * SPLIT_PART_US < whole;
  };
  while (ks >= 2 && !gains(ks)) --ks;
  if (ks < 2) return t;
  t.ks = ks;
  t.n_full = (uint32_t)(n_tiles - r);
  t.n_split = (uint32_t)r;
  return t;
}
constexpr size_t SPLIT_TILE_BYTES = (size_t)GM_BM * GM_BN * 4;  // one fp32 partial tile

// Direct norm on the direct-load kernel: the number of consecutive examples
// one work item covers. An item streams its examples' K stages without a gap
// and pays the ring's fill and drain once (about NG_OVERHEAD stages), so
// longer items cost less per stage, while fewer, longer items leave more of
// the chip idle in the last round. The choice minimises
// rounds(items) * (eg * stages per example + NG_OVERHEAD) over 1 <= eg <= B
// (eg <= NG_MAX: the item keeps a partial per example and wave in LDS).
constexpr int NG_OVERHEAD = 6;
constexpr int NG_MAX = 512;
inline int norm_group(uint64_t n_tiles, int B, int spe, int cus) {
  if (n_tiles == 0 || B <= 1 || cus <= 0) return 1;
  int best = 1;
  uint64_t best_cost = ~0ull;
  const int top = B < NG_MAX ? B : NG_MAX;
  for (int eg = 1; eg <= top; ++eg) {
    const uint64_t items = n_tiles * (uint64_t)((B + eg - 1) / eg);
    const uint64_t rounds = (items + (uint64_t)cus - 1) / (uint64_t)cus;
    const uint64_t cost = rounds * (uint64_t)(eg * spe + NG_OVERHEAD);
    if (cost < best_cost) { best_cost = cost; best = eg; }
  }
  return best;
}

// Clipped sum: out (+)= sum_i c_i X_i^T Y_i over all B*T rows (K = B*T).
// With a.part set (and room for the split that tail_split gives on `cus` CUs),
// the last round is split and a fixup kernel follows.
hipError_t launch_clipped_sum(const GemmArgs& a, int dt, bool vec, int cus, size_t part_bytes,
                              hipStream_t s);
// Direct norm: ws[b, slot] = ||tile of X_b^T Y_b||_F^2 for every output tile.
hipError_t launch_direct_norm(const GemmArgs& a, int dt, bool vec, hipStream_t s);
// Clipped sum from a gradient store: for every tile of every layer,
// out (+)= sum_e c_e * tile_e (then the fused noise and 1/B), one workgroup
// per tile; the layers' store_slot give each layer's first tile slot.
hipError_t launch_store_sum(const GemmArgs& a, hipStream_t s);
constexpr size_t STORE_TILE_FLOATS = (size_t)GM_BM * GM_BN;

// --------------------------------------------------------- embedding / ids
struct EmbedNormArgs {
  const int32_t* ids;   // [B,T]
  const void* E;        // dE [B*T, lde]
  int64_t lde;
  int32_t B, T, V, d;
  int32_t pbits;        // bits for a position in a sort key
  int32_t n_chunks;     // partials per example: feature chunks of 64, or (runs) position ranges
  int32_t runs;         // 1: embed_norm_runs_kernel (rows read EN_VB bytes per lane)
  int32_t gram;         // embed_norm_gram_kernel (bf16, 16-byte rows, T <= EN_G_T): n_chunks
                        // feature chunks; 2 (set at launch): workgroup row 0 ranks the ids
  int32_t* seg_id;      // nullable [B,T]
  int32_t* n_unique;    // nullable [B]
  float* ws;            // [B, n_chunks]
  // T > EN_MAX_T (runs only): each example sorted and ranked by the
  // workspace radix sort (keys [B*T] and their second buffer, digit counts
  // [B, 256, blocks per example], block run counts [B * blocks], run index of
  // every sorted position [B*T], run starts [B, T+1], run counts [B]).
  uint32_t *gkeys, *gkeys2;
  int32_t *ghist, *gruns, *grank, *gseg, *gnseg;
};
hipError_t launch_embed_norm(const EmbedNormArgs& a, int dt, hipStream_t s);

constexpr int EN_MAX_T = 4096;   // tokens per example sorted in LDS (bucketing)
constexpr int EN_CT_T = 256;     // up to this T the norm ranks keys by counting (one per thread)
constexpr int EN_P = 32;         // sorted positions whose runs one workgroup of the norm owns
constexpr int EN_VB = 8;         // bytes per lane load of the run-walking norm
constexpr int EN_BATCH = 32;     // row loads a lane has in flight (EN_P: one batch per range)
constexpr int EN_G_T = 128;      // up to this T (bf16) the norm takes the pairwise (Gram) form
constexpr int EN_GF = 96;        // features per workgroup of the pairwise form
constexpr int ES_MAX_K = 16384;  // tokens per batch sorted in LDS (embedding sum)
constexpr int ES_BLOCK = 32;     // sorted tokens per reduction block
constexpr int GS_KB = 4096;      // keys per block of the workspace radix sort (more than ES_MAX_K keys)

struct EmbedSumArgs {
  const int32_t* ids;   // [K] flattened B*T
  const void* E;        // [K, lde]
  int64_t lde;
  const float* c;       // [B]
  int32_t B, K, T, V, d;
  int32_t pbits;        // bits for a token index in a sort key
  uint32_t* keys;       // workspace [K] sorted keys
  float* head;          // workspace [n_blocks, d] partial of the run a block starts inside
  float* tail;          // workspace [n_blocks, d] partial of the run a block ends inside
  float* out;           // [V, ldo] or transposed [d, ldo]; accumulated into
  int64_t ldo;
  int32_t transpose;
  // Compact form: each run of equal ids gets one row of `rows` (its index is
  // the run's rank among the batch's runs), written once, instead of being
  // added onto out[id]; a later scatter adds the rows onto out.
  int32_t* rank;        // workspace [K] run index of every sorted position
  int32_t* seg;         // workspace [K + 1] first sorted position of every run
  int32_t* n_runs;      // workspace [1] number of runs
  float* rows;          // workspace [K, d] run sums
  // More than ES_MAX_K keys: the workspace radix sort in segments of gs_seg
  // keys (here one: the batch), gs_nbs blocks of GS_KB keys each, gs_blocks
  // in all (keys2: the other key buffer; hist: [segments, 256, gs_nbs]
  // digit counts, then offsets; gs_runs: [gs_blocks] run counts, then bases).
  int32_t gs_blocks, gs_nbs, gs_seg;
  uint32_t* keys2;
  int32_t* hist;
  int32_t* gs_runs;
};
hipError_t launch_embed_sum(const EmbedSumArgs& a, int dt, hipStream_t s);
// The compact form: sort, ranks, run sums into a.rows.
hipError_t launch_embed_rows(const EmbedSumArgs& a, int dt, hipStream_t s);
// out[id of run r] (+)= rows[r] for every run (reads a.keys, a.seg, a.n_runs).
hipError_t launch_embed_scatter(const EmbedSumArgs& a, hipStream_t s);
hipError_t launch_fill_zero(float* p, int64_t n, hipStream_t s);

// ------------------------------------- vector parameters and position table
enum { VEC_GRAD = 0, VEC_SQ = 1 };
constexpr int VR_MAX_PARAMS = 44;   // entries per reduce launch (kernel arguments < 4 KiB)
constexpr int VS_MAX_PARAMS = 64;   // entries per clipped-sum launch
static_assert(GR_MAX_LAYERS <= 64 && GM_MAX_LAYERS <= 64 && VR_MAX_PARAMS <= 64,
              "a wave finds a work item's table entry with one lane per entry");

struct VecParam {
  const void* X;        // [B*T rows, ldx] elementwise factor, or null (a plain sum)
  const void* G;        // [B*T rows, ldg]
  int64_t ldx, ldg;
  int32_t d;            // features
  int32_t mode;         // VEC_GRAD: per-example gradient; VEC_SQ: sum of squares only
  float* grad;          // VEC_GRAD: [B, d] per-example gradients (of X * G, or of G)
  float* grad2;         // VEC_GRAD with X: [B, d] sums of G as well (a LayerNorm bias), or null
  int32_t tsplit;       // row ranges per feature chunk (VEC_SQ; 1 for VEC_GRAD)
  int32_t trows;        // rows per range
  uint32_t item_begin;  // first item of this entry among an example's items
  int32_t slot_begin;   // first partial slot of this entry in an example's row
};

// Items example-major: example b owns [b * per_ex, (b + 1) * per_ex), one per
// (entry, feature chunk of 64 lanes x 16 bytes, row range).
struct VecArgs {
  VecParam P[VR_MAX_PARAMS];
  int32_t n_params;
  int32_t B, T;
  int32_t slots;        // partial slots per example
  uint32_t per_ex;
  uint32_t n_items;
  float* ws;            // [B, slots]
};
static_assert(sizeof(VecArgs) <= 4096, "kernel arguments must stay within 4 KiB");
hipError_t launch_vec_reduce(const VecArgs& a, int dt, bool vec, hipStream_t s);

struct VecSumParam {
  const float* grad;    // [B, d]
  float* out;           // [d]
  int64_t d;
  uint32_t quad_begin;  // first 4-feature group of this entry
  uint32_t tensor_id;
  int32_t accumulate;
};
struct VecSumArgs {
  VecSumParam P[VS_MAX_PARAMS];
  int32_t n_params, B;
  uint32_t n_quads;
  const float* c;       // [B]
  int32_t noise;
  float sigma_c, inv_b;
  uint32_t step;
  uint64_t seed;
};
static_assert(sizeof(VecSumArgs) <= 4096, "kernel arguments must stay within 4 KiB");
hipError_t launch_vec_sum(const VecSumArgs& a, hipStream_t s);

struct PosSumArgs {
  const void* E;        // dE [B*T, lde]
  int64_t lde;
  const float* c;       // [B]
  float* out;           // [n_pos, ldo]
  int64_t ldo;
  int32_t B, T, d, n_pos;
  int32_t accumulate, noise;
  float sigma_c, inv_b;
  uint32_t tensor_id, step;
  uint64_t seed;
};
hipError_t launch_pos_sum(const PosSumArgs& a, int dt, hipStream_t s);

// A launch counts its threads in 32 bits; the row-wise kernels below are launched for at
// most this many workgroups of up to 1024 threads at a time.
constexpr int64_t MAX_GROUPS = (int64_t)1 << 21;

// ---------------------------------------------------------------- LayerNorm
constexpr int LN_MAX_D = 32768;     // a row is held in the registers of at most 16 waves
struct LnForwardArgs {
  const void* x;        // [rows, ldx]
  const void* gain;     // [d] of param_dt, or null (1)
  const void* bias;     // [d] of param_dt, or null (0)
  void* y;              // [rows, ldy]
  float* mean;          // nullable [rows]
  float* rstd;          // nullable [rows]
  int64_t ldx, ldy, rows;
  int32_t d, param_dt;
  float eps;
};
hipError_t launch_ln_forward(const LnForwardArgs& a, int dt, hipStream_t s);

struct LnBackwardArgs {
  const void* gy;       // [B*T rows, ldgy]
  const void* x;        // [B*T rows, ldx]
  const void* gain;     // [d] of param_dt, or null (1)
  const float* mean;    // [B*T]
  const float* rstd;    // [B*T]
  void* dx;             // nullable [B*T rows, lddx]
  float* dgain;         // nullable [B, d]
  float* dbias;         // nullable [B, d]
  float* norm2;         // nullable [B]
  float* ws;            // [B, ranges, 2, d] partial sums (ranges > 1)
  float* sq;            // [B, chunks] partial squares (ranges > 1)
  int64_t ldgy, ldx, lddx;
  int32_t B, T, d, param_dt;
  int32_t b0;           // first example of the launch
  int32_t ranges, span; // an example's rows are cut into `ranges` of `span`
  int32_t chunks;       // workgroups per example of the second launch
  int32_t accumulate_dx, accumulate;
};
hipError_t launch_ln_backward(const LnBackwardArgs& a, int dt, hipStream_t s);

// How the backward pass cuts an example's T rows: about LN_GROUPS workgroups in
// all, but about `least` rows each at least, beside whose operands (3 d elements a row) the partial
// sums' way to memory and back (16 d bytes a range) stays small: a sixth in bf16 up to 2048 features, a third above,
// half of that in fp32; up to twice that where T is little more than `least`, as T / least is rounded up.
constexpr int LN_GROUPS = 512, LN_FEW = 32;
struct LnPlan {
  int32_t ranges, span, chunks;
};
inline LnPlan ln_plan(int B, int T, int d, bool grads) {
  const int teams = d <= 2048 ? 8 : 1;
  const int least = grads ? (teams > 1 ? 2 * teams : 8) : teams;
  const int groups = d <= 2048 ? LN_GROUPS : d <= 4096 ? 4 * LN_GROUPS : LN_GROUPS;
  int64_t ranges = ((int64_t)groups + B - 1) / B, most = ((int64_t)T + least - 1) / least;
  if (ranges > most) ranges = most;
  LnPlan p;
  p.span = (int32_t)((T + ranges - 1) / ranges);
  p.ranges = (int32_t)(((int64_t)T + p.span - 1) / p.span);
  // One workgroup per example adds few ranges (a chain of loads each); more are added by
  // chunks of 64 features, and the norms of more than one chunk by a third launch.
  p.chunks = p.ranges <= LN_FEW ? 1 : (d + 63) / 64;
  return p;
}

// ------------------------------------------------------------------- losses
struct RowStat {
  float top, scale;     // largest logit; 1 / sum exp(z - top), 0 for a row without any
};
struct LossArgs {
  const void* Z;        // [rows, ldz] logits
  void* Gz;             // [rows, ldg] their gradient (may be Z)
  const int32_t* targets;  // [rows]; outside [0, V): ignored
  const float* w;       // [rows] weights (cross-entropy), or [B] (preference)
  float* logp;          // nullable [rows]
  float* lse;           // nullable [rows]
  double* logp64;       // nullable [rows] (preference)
  RowStat* stat;        // nullable [rows] (preference)
  int64_t ldz, ldg, rows, row0;
  int32_t V, T, split;  // split: tokens before it are the chosen answer's (preference)
};
// log p and its logarithmic sum of every row; with a.stat also what the backward pass needs.
hipError_t launch_token_logprobs(const LossArgs& a, int dt, hipStream_t s);
// log p and the weighted gradient in one pass over the logits.
hipError_t launch_cross_entropy(const LossArgs& a, int dt, hipStream_t s);
// The gradient from saved row statistics.
hipError_t launch_logit_grads(const LossArgs& a, int dt, hipStream_t s);

struct PreferenceArgs {
  const int32_t* targets;  // [B, T]
  const double* logp;   // [B, T]
  const float* ref;     // nullable [B, T]
  float* loss;          // [B]
  float* rewards;       // nullable [B, 2]
  float* slope;         // [B] -d loss / d log p of a chosen answer's token
  int32_t T, V, split, b0;  // b0: first pair of the launch
  float beta, smoothing;
};
hipError_t launch_preference(PreferenceArgs a, int B, hipStream_t s);

// ---------------------------------------------------- orthogonalised updates
constexpr int NS_TILE = 128;        // rows and columns of an output tile; sizes are padded to it
constexpr int NS_MAX_MATS = 48;     // matrices per launch (kernel arguments stay < 4 KiB)
constexpr int NS_MAX_SIDE = 65536;
constexpr int64_t NS_MAX_SIZE = (int64_t)1 << 30;   // padded elements: a plane spans less than 2 GiB
constexpr int NS_MAX_STEPS = 64;
enum { NS_GRAM = 0, NS_POLY = 1, NS_UPDATE = 2, NS_LAST = 3 };       // the products of a step
enum { NS_Y0 = 0, NS_Y1 = 1, NS_A = 2, NS_P = 3 };                   // a matrix's buffers

struct NsMat {
  const void* G;        // [rows, ldg]
  void* out;            // [rows, ldo]
  char* ws;             // partial sums of squares, then the buffers
  int64_t ldg, ldo;
  int32_t rows, cols;
  int32_t mp, np;       // shorter and longer side, padded
  float scale;
  uint32_t item_begin;  // first work item of this matrix in a launch
};
struct NsArgs {
  NsMat M[NS_MAX_MATS];
  int32_t n;
  int32_t out_dt, accumulate;
  int32_t step, last;
  float coef[3];          // of I, A and A^2 in P
  float own;              // X goes into the update by itself, times this (P then has no I)
  int32_t fine_next;      // one plane: the next X's second plane is written too
  float eps;
  uint32_t xcd_begin[9];  // items of XCD x: [xcd_begin[x], xcd_begin[x + 1])
  int32_t ks;             // ranges of k of a symmetric product's tile
  float* part;            // their sums, 64 KB each
  int32_t steps;          // small matrices: all of them
};
constexpr int NS_COEFS = 3 * NS_MAX_STEPS;
struct NsCoefs {
  float c[NS_COEFS];
};
static_assert(sizeof(NsArgs) + 4 * 3 * NS_MAX_STEPS <= 4096, "kernel arguments must stay within 4 KiB");
static_assert(NS_MAX_MATS <= 64, "a wave finds a work item's matrix with one lane per entry");

constexpr int NS_PARTS = 128;       // most partial sums of squares of a matrix
constexpr size_t NS_HEAD = NS_PARTS * 8;
#define DPG_HD __host__ __device__
// Workgroups that sum a matrix's squares: 32768 elements each, or NS_PARTS of them.
DPG_HD inline int ns_parts(int rows, int cols) {
  const int64_t p = ((int64_t)rows * cols + 32767) / 32768;
  return p < 1 ? 1 : p > NS_PARTS ? NS_PARTS : (int)p;
}
// Offset of plane `plane` of buffer `which`: X^T [np, mp] twice, two planes each, A and P [mp, mp]
// of pl planes.
DPG_HD inline size_t ns_offset(int mp, int np, int which, int plane, int pl) {
  const size_t y = (size_t)mp * np * 2, q = (size_t)mp * mp * 2;
  const size_t at = which <= NS_A ? (size_t)which * 2 * y : 4 * y + (size_t)pl * q;
  return NS_HEAD + at + (size_t)plane * (which < NS_A ? y : q);
}
// Whether X goes into step k's update by itself, from two planes whatever the products have.
DPG_HD inline bool ns_fine(int k, int steps, int pl) { return k < steps - (pl == 1 ? 2 : 1); }
DPG_HD inline size_t ns_bytes(int mp, int np, int pl) {
  return ns_offset(mp, np, NS_P, 0, pl) + (size_t)pl * mp * mp * 2;
}
#undef DPG_HD
// How a product is launched: 64 x 64 tiles (small), or large ones, those of a symmetric
// product perhaps in ks ranges of k.
//
// One workgroup with a large tile keeps a CU's matrix cores as busy as two do (a second one
// only fills the first's gaps), so a launch runs 256 items at a time, each for about its k and
// 600 more, US_K us per k; joining ranges is another launch. Ranges are cut where a launch fills
// at most half a round and that pays. (1601 x 6397, two planes, us: X X^T 103 whole and 67 + 9 in
// 5 ranges, A^2 35 and 20 + 8 in 2; 2048 x 8192, one plane, 136 tiles: 75 whole, 58 + 13 in 3.)
// Small tiles cost more LDS reads and loads per product, but a launch of few of them ends
// sooner: 6 us and US_K_SMALL per k, 512 at a time with one plane and 256 with two (their rings). All five
// steps, us, large and small: 600 x 600 fp32 results 251, 153; bf16 188, 116; 1536 x 1536 bf16 350, 269;
// and 100 x 3000 fp32, X X^T alone small: 144, 210; 1536 x 1536 fp32, updates alone: 419, 451.
// Updates and X X^T with one plane that fill a round with 256 x 256 tiles take those: fewer LDS reads and
// loads per product (us, such tiles and the others: updates 4096 x 4096 120, 131; 24 x (1024 x 1024, 1024 x
// 4096) 281, 312; their X X^T 167, 184). A^2, whose other operand needs registers too, does not: 115, 95;
// nor do updates that X goes into by itself (see ns_step).
struct NsPlan {
  int ks;
  bool small, wide;       // 64 x 64 tiles; 256 x 256 tiles
};
constexpr double NS_JOIN_US = 8.0;
inline NsPlan ns_plan(const NsArgs& a, int kind, int pl) {
  const bool sym = kind == NS_GRAM || kind == NS_POLY;
  const double us_k = pl == 2 ? 0.0136 : sym ? 0.008 : 0.0139, us_k_small = pl == 2 ? 0.0067 : 0.0045;
  const double us_k_wide = 0.0256;
  const int64_t at_once = pl == 2 ? 256 : 512;
  int64_t tiles = 0, few = 0, wide = 0, k_most = 0, k_least = 1 << 30;   // few: large tiles
  double few_k = 0.0, wide_k = 0.0;                                     // and the sum of their costs in k
  for (int l = 0; l < a.n; ++l) {
    const int64_t m = a.M[l].mp / 64, n = a.M[l].np / 64, k = kind == NS_GRAM ? a.M[l].np : a.M[l].mp;
    const int64_t mw = (m + 3) / 4, nw = (n + 3) / 4;
    const int64_t f = sym ? m / 2 * (m / 2 + 1) / 2 : m / 2 * ((n / 2 + 2 - pl) / (3 - pl));
    const int64_t w = sym ? mw * (mw + 1) / 2 : mw * nw;
    tiles += sym ? m * (m + 1) / 2 : m * n;
    few += f;
    wide += w;
    few_k += (double)f * (double)(k + 600);
    wide_k += (double)w * (double)(k + 600);
    k_most = k > k_most ? k : k_most;
    k_least = k < k_least ? k : k_least;
  }
  // Items of one length end in whole rounds; longer ones first, shorter ones fill the last.
  auto rounds_k = [&](int64_t items, double sum) {
    if (k_most == k_least) return (double)((items + 255) / 256) * (double)(k_most + 600);
    return sum / 256 > (double)(k_most + 600) ? sum / 256 : (double)(k_most + 600);
  };
  NsPlan best{1, false, false};
  double best_us = rounds_k(few, few_k) * us_k;
  if (sym && few <= 128)
    for (int ks = 2; ks <= 16 && ks * 128 <= k_least; ++ks) {
      const double us = (double)((few * ks + 255) / 256) * ((double)k_most / ks + 600) * us_k + NS_JOIN_US;
      if (us < 0.95 * best_us) { best_us = us; best.ks = ks; }
    }
  const int64_t rounds = (tiles + at_once - 1) / at_once;
  if (rounds <= 2 && 6.0 + (double)rounds * (double)k_most * us_k_small < 1.1 * best_us) return NsPlan{1, true, false};
  if (pl == 1 && (kind == NS_GRAM || kind == NS_UPDATE) && wide >= 256 && rounds_k(wide, wide_k) * us_k_wide < 1.02 * best_us)
    return NsPlan{1, false, true};
  return best;
}
inline size_t ns_part_bytes(const NsArgs& a, int pl) {
  size_t most = 0;
  for (int kind = NS_GRAM; kind <= NS_POLY; ++kind) {
    const int ks = ns_plan(a, kind, pl).ks;
    if (ks == 1) continue;
    size_t tiles = 0;
    for (int l = 0; l < a.n; ++l) {
      const size_t t = (size_t)(a.M[l].mp + NS_TILE - 1) / NS_TILE;
      tiles += t * (t + 1) / 2;
    }
    const size_t n = tiles * ks * NS_TILE * NS_TILE * 4;
    most = n > most ? n : most;
  }
  return most;
}

// Reorders the matrices so that 8 bins, one per XCD, of consecutive ones have nearly equal
// work, the longest sums first in each (longest first, each to the emptiest bin).
struct NsBins {
  int begin[9];
};
inline NsBins ns_order(NsArgs& a) {
  int by[NS_MAX_MATS], bin[NS_MAX_MATS];
  double load[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto work = [&](int l) { return (double)a.M[l].mp * a.M[l].mp * a.M[l].np; };
  for (int l = 0; l < a.n; ++l) {   // insertion sort: stable, and short
    int k = l;
    while (k > 0 && work(by[k - 1]) < work(l)) { by[k] = by[k - 1]; --k; }
    by[k] = l;
  }
  for (int k = 0; k < a.n; ++k) {
    int x = 0;
    for (int q = 1; q < 8; ++q) x = load[q] < load[x] ? q : x;
    bin[k] = x;
    load[x] += work(by[k]);
  }
  NsBins b;
  NsMat sorted[NS_MAX_MATS];
  int n = 0;
  for (int x = 0; x < 8; ++x) {
    b.begin[x] = n;
    for (int k = 0; k < a.n; ++k)
      if (bin[k] == x) sorted[n++] = a.M[by[k]];
  }
  b.begin[8] = n;
  for (int l = 0; l < n; ++l) a.M[l] = sorted[l];
  return b;
}
// Matrices small enough for one workgroup to keep X, A and P in its LDS take all their
// steps there (mp, np: sides padded to 32; no workspace).
constexpr int NS_SMALL_WAVES = 8, NS_SMALL_BLOCKS = 4;   // waves; most 32 x 32 blocks of X per wave
constexpr int NS_SMALL_LDS = 160 * 1024 - NS_SMALL_WAVES * 32 * 36 * 4 - 256;
inline bool ns_small(int rows, int cols, int pl) {
  const int64_t r = (rows + 31) / 32 * 32, c = (cols + 31) / 32 * 32, m = r < c ? r : c, n = r < c ? c : r;
  return 2 * pl * (n * m + 2 * m * m) <= NS_SMALL_LDS && n * m <= 1024 * NS_SMALL_WAVES * NS_SMALL_BLOCKS;
}
hipError_t launch_orthogonalize_small(const NsArgs& a, int dt, int planes, const float* coef, int steps,
                                      hipStream_t s);
hipError_t launch_orthogonalize(const NsArgs& a, int dt, int planes, const float* coef, int steps,
                                hipStream_t s);

// ----------------------------------------------------------- clip and noise
// c (nullable) = clip factors; cs (nullable) = scale * clip factors; the
// squared norm is norm2 (+ norm2_b when not null).
hipError_t launch_clip_factors(const float* norm2, const float* norm2_b, int B, float C,
                               float scale, float* c, float* cs, hipStream_t s);
// accumulate: g = (g + sigma_c z) inv_b; else g = sigma_c z inv_b (g not read).
hipError_t launch_add_noise(float* g, int64_t n, float sigma_c, float inv_b, uint64_t seed,
                            uint32_t tensor_id, uint32_t step, bool accumulate, hipStream_t s);

}  // namespace dpg
