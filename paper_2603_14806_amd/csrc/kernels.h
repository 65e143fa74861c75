// Host-side launchers of the triangle-multiplication kernels.  Each returns
// hipSuccess or the error hipGetLastError() reported right after the launch.
// Shapes are validated by the C-ABI layer before these are called.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace trimul {

// Repacked, device-resident layer parameters (owned by the handle).
struct DeviceWeights {
    // fp32 LayerNorm parameters (both storage types)
    float* ln_in_w = nullptr;   // [c_z]
    float* ln_in_b = nullptr;   // [c_z]
    float* ln_out_w = nullptr;  // [c]
    float* ln_out_b = nullptr;  // [c]
    // fp32 MFMA operands (fp32 storage only): blocks of 32 weight rows, [block][16 k groups][64 lanes][4]
    // with row l % 32 and k = 8 q + 4 (l / 32) + e at lane l, element e of k group q
    float* proj_f = nullptr;    // 8 gated groups (a's four 32-channel groups, then b's) x (value, gate) blocks
    float* epi_f = nullptr;     // 4 groups of 32 output channels x (W_o, W_g) blocks
    // bf16 copies used by the MFMA kernels (bf16 storage only)
    uint16_t* proj_bf = nullptr;  // [4*c][c_z]: rows ordered per 32-channel group g:
                                  // W_a[g], W_ga[g], W_b[g], W_gb[g] (32 rows each)
    uint16_t* epi_bf = nullptr;   // [2*c_z][128]: W_o rows then W_g rows
    uint16_t* epit_bf = nullptr;  // [2*128][c_z]: W_o^T rows then W_g^T rows (backward)
    uint16_t* projt_bf = nullptr; // [c_z][4*c]: row d = W_a[:, d], W_ga[:, d], W_b[:, d], W_gb[:, d] (backward)
    // fp16 copies for the bf16-path projection (K1), each matrix scaled by a
    // power of two 2^s_m and the LayerNorm gain and bias by 2^s_x, so that
    // the largest possible |W x| operand lies in [2^14, 2^15]; the gating
    // undoes the scales (K1Scales).
    uint16_t* proj_h = nullptr;   // [4*c][c_z] fp16 bits, rows as proj_bf, W_m * 2^s_m
    float* ln_in_w_h = nullptr;   // [c_z] gamma * 2^s_x
    float* ln_in_b_h = nullptr;   // [c_z] beta * 2^s_x
    struct K1Scales {
        // a = v * sigmoid(g) from accumulators v' = 2^Sv v, g' = 2^Sg g:
        // a = v' / (2^Sv + 2^(Sv - g log2 e)) = v' * rcp(kv + exp2(g' * cg + Sv))
        float kv_a, cg_a, sv_a;   // 2^Sv, -log2(e) 2^-Sg, Sv of a
        float kv_b, cg_b, sv_b;   // the same for b
    } k1s{};
    float eps = 1e-5f;
    int cus = 256;                // compute units of the device (persistent grids)
    uint8_t* kmask_pad = nullptr; // 0/1 staging of a k-panel's token mask, kMaskStageBytes
};

constexpr int64_t kMaxKPanel = 65536;   // longest k-panel of one block call
constexpr int64_t kMaskStageBytes = kMaxKPanel + 128;   // size of DeviceWeights::kmask_pad

// Copies mask[0, klen) into dst as 0/1 bytes (mask NULL: all ones) and zero-fills dst up to the next
// multiple of 32 (so the contraction can read whole 4-byte words of it).
hipError_t launch_stage_kmask(const uint8_t* mask, int64_t klen, uint8_t* dst, hipStream_t s);
// Row-major bf16 panel [nch][rows][ld] -> blocked [nch][ceil(rows/256)][ceil(klen/32)][256][32],
// staged k-mask applied, padding zero.
hipError_t launch_panel_block(const void* P, int64_t rows, int64_t ld, int64_t klen, int nch, const uint8_t* kst,
                              void* dst, hipStream_t s);
// bf16 contraction of blocked operands into a row-major fp32 C [batch][M][N].
hipError_t launch_contract_blocked_rowc(const void* A, const void* B, float* C, int64_t M, int64_t N, int64_t K,
                                        int batch, int accumulate, int cus, hipStream_t s);
// bf16 contraction of blocked operands into the pair-blocked fp32 result layout over (M, N) (a device
// tile's packed accumulator), overwritten or accumulated into.
hipError_t launch_contract_blocked_packed(const void* A, const void* B, float* C, int64_t M, int64_t N, int64_t K,
                                          int batch, int accumulate, int cus, hipStream_t s);
// bf16 contraction of blocked operands, either given as its transpose in the
// panel layout (ta: A[c][i][k] = X[c][k][i], X with K rows and M columns; tb
// likewise with N columns), into the pair-blocked fp32 result layout.
// Supported: (ta, tb) = (0, 1), (1, 1) and (1, 0); accumulate adds into C.
hipError_t launch_contract_transposed(int ta, int tb, const void* A, const void* B, float* C, int64_t M, int64_t N,
                                      int64_t K, int batch, int cus, hipStream_t s, int accumulate = 0);

// Host-side check of the contraction kernel's loads (contract.hip): counts of
// tiles, loads and needed elements visited, and of violations.
struct K2CheckCounts {
    int64_t tiles = 0, loads = 0, elems = 0;
    int64_t bad_tiles = 0;   // tiles taken by no or several (work-group, round) pairs
    int64_t bad_desc = 0;    // loads whose descriptor reaches outside the operand
    int64_t bad_elem = 0;    // needed elements read from the wrong address or not at all
};
// a_mode / b_mode: 0 blocked panel, 1 row-major [batch][rows][ld] (channel stride sA / sB), 2 transposed
// (the operand given as X[k][row] in the panel layout of K rows).  a_bytes / b_bytes: allocation sizes.
void k2_check_loads(int a_mode, int b_mode, int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb, int64_t sA,
                    int64_t sB, int batch, uint64_t a_bytes, uint64_t b_bytes, int grid, int all_channels,
                    K2CheckCounts& n);
// The same for the accesses to a pair-blocked C of M rows, N columns and `batch` channels (the result layout,
// c_bytes allocated): every load / store descriptor inside the allocation, every accessed element at the
// layout's address, every element (row < M, column < N) accessed exactly once (loads counts the 64-lane
// register groups visited).
void k2_check_c(int64_t M, int64_t N, int batch, uint64_t c_bytes, int all_channels, K2CheckCounts& n);

struct EpilogueArgs {
    const float* C;      // fp32 contraction result: pair-blocked (cblocked) or [c][rows][ldc]
    int cblocked;        // C in the pair-blocked result layout (common.h)
    int64_t ldc;         // row stride of C (elements), row-major C only
    int64_t sc;          // channel stride of C (elements), row-major C only
    const void* z;       // [rows][cols][c_z] pair tensor (same tile as C)
    const uint8_t* mask; // token mask over global indices, or null
    int64_t row0, col0;  // global token index of tile row 0 / column 0
    int64_t rows, cols;
    void* out;           // [rows][cols][c_z]
};

// K1: LN_in + gated projections + pair mask -> channel-major operands A, B in
// the blocked panel layout (common.h) of N rows and K = N.  Padding rows are
// left untouched; the k padding of a row's last k-step is written with zeros by
// the bf16 projection and left untouched by the fp32 one (both contractions
// drop it themselves).
// The bf16 projection of an M x K operand pair (A, B in the blocked layout of
// panel_geom(M, K)): operand row i, contraction index k is pair (i, k) of z
// (outgoing) or (k, i) (incoming), z rows ldz pairs apart; mask: token mask
// over global indices or null, operand row i's byte at m0 + i, k's at k0 + k.
hipError_t launch_project_mfma(const DeviceWeights& w, const void* z, int64_t ldz, const uint8_t* mask, int64_t m0,
                               int64_t k0, int64_t M, int64_t K, int incoming, void* A, void* B, hipStream_t s);
hipError_t launch_project(int dtype, const DeviceWeights& w, const void* z, const uint8_t* mask,
                          int64_t N, int incoming, void* A, void* B, hipStream_t s);

// K2: C[b] (+)= A[b] * diag(kmask) * B[b]^T for b < batch.
// blocked != 0: A, B in the blocked panel layout of M (N) rows and K columns
// (lda, ldb, sA, sB unused) and C in the pair-blocked result layout (ldc, sC
// unused); blocked == 0: A [b][M][lda], B [b][N][ldb], C [b][M][ldc] (stride sC).
hipError_t launch_contract(int dtype, int blocked, const void* A, const void* B, float* C, int64_t M,
                           int64_t N, int64_t K, int64_t lda, int64_t ldb, int64_t ldc, int64_t sA,
                           int64_t sB, int64_t sC, int batch, int accumulate, const uint8_t* kmask, int cus,
                           hipStream_t s);

// Side of the output tiles of the fp32 contraction: 64 or 128.
int contract_f32_tile(int64_t M, int64_t N, int batch, int cus);

// K3: LN_out + output projection + sigmoid gate + pair mask -> out [rows][cols][c_z].
hipError_t launch_epilogue(int dtype, int out_dtype, const DeviceWeights& w, const EpilogueArgs& a,
                           hipStream_t s);

// Backward of the contraction: the fp32 result layout -> a panel (dtype
// elements), and the per-channel panel transpose X_c[i][k] -> X_c[k][i].
hipError_t launch_result_to_panel(int dtype, const float* R, void* P, int64_t N, int cus, hipStream_t s);
hipError_t launch_panel_transpose(int dtype, const void* X, void* Y, int64_t N, int cus, hipStream_t s);

// Layer backward (bf16 storage).  Unit blocks: per unit of 32 pairs a bf16
// [128][32] block of one per-pair quantity (see backward.hip).
struct BackwardBlocks {
    bf16_t *dpa, *dga, *dpb, *dgb, *xp;   // from the projection backward
};
// Persistent grid: min(units, per_cu * compute units).
int backward_grid(int64_t units, int cus, int per_cu);
hipError_t launch_epilogue_backward(int out_dtype, const DeviceWeights& w, const float* C, const void* z,
                                    const uint8_t* mask, const void* dout, int64_t N, void* dCp, float* dxg,
                                    float* wpart, float* partial, int grid, hipStream_t s);
hipError_t launch_projection_backward(const DeviceWeights& w, const void* z, const uint8_t* mask, int64_t N,
                                      int incoming, const float* dA, const float* dB, const float* dxg, void* dz,
                                      const BackwardBlocks& bb, float* partial, int grid, hipStream_t s);
// Four weight gradients sharing V: partial[o][grid][128][128] for U[o] V^T, o = 0..3.
hipError_t launch_wgrad4(const bf16_t* const U[4], const bf16_t* V, int64_t N, float* partial, int grid,
                         hipStream_t s);
// Sums of partials, several in one launch: out[i] = sum over g < parts of in[g * stride + i], i < n (n a
// multiple of 32; in and stride 16-byte aligned).  block0 is filled in by the launcher.
struct SumTask {
    const float* in;
    float* out;
    int parts, stride, n, block0;
};
constexpr int kMaxSumTasks = 10;
struct SumTasks {
    SumTask task[kMaxSumTasks];
    int count;
};
hipError_t launch_sum_parts(const SumTask* tasks, int count, hipStream_t s);

// Outer product mean (opm.hip).  Pack: tokens [row0, row0 + rows) of a and
// [col0, col0 + cols) of b, sequences [s0, s0 + slen) of [S][n_total][32] bf16
// tensors, masked, into the transposed operands of the sums -- the blocked
// panels of slen rows and tokens * 32 columns, X[s][token * 32 + c] -- and the
// mask into words of 32 sequences, bits[s / 32][token] (8 * ceil(slen / 256)
// words per token).  Count: the pairs' common sequences from those words into
// [rows][32 * ceil(cols / 32)] floats.  Epilogue: out[rows][cols][128] from the
// sums O (result layout, [rows * 32][cols * 32]) and the counts.
hipError_t launch_opm_pack(const void* a, const void* b, const uint8_t* mask, int64_t n_total, int64_t row0,
                           int64_t rows, int64_t col0, int64_t cols, int64_t s0, int64_t slen, void* PA, void* PB,
                           uint32_t* abits, uint32_t* bbits, hipStream_t s);
hipError_t launch_opm_count(const uint32_t* abits, const uint32_t* bbits, int64_t rows, int64_t cols, int64_t slen,
                            int accumulate, float* cnt, hipStream_t s);
hipError_t launch_opm_epilogue(int out_dtype, const float* O, const float* cnt, int64_t rows, int64_t cols,
                               const uint16_t* wo, const float* bo, void* out, int cus, hipStream_t s);

// Triangle attention core (triattn.hip): rows x heads x ceil(N / 128)
// work-groups over keys [k0, kend); q, k, v [rows][N][H][32] bf16, bias
// [H][N][ldb] bf16 (ldb % 8 == 0, k0 % 8 == 0), mask [N] or null.  State
// (A [rows][N][H][32], M and L [rows][H][N], fp32) is read when load_state and
// written unless finish; finish writes out [rows][N][H][32] (fp32 or bf16).
hipError_t launch_triattn(int out_dtype, const void* q, const void* k, const void* v, const void* bias,
                          const uint8_t* mask, int64_t rows, int64_t N, int H, int64_t ldb, int64_t k0, int64_t kend,
                          float* stA, float* stM, float* stL, int load_state, int finish, void* out, hipStream_t s);

// Attention of queries over keys of another length (crossattn.hip,
// crossattn_backward.hip).  The queries of one key head are taken together
// as "columns": column c of key head hk is query c / group of head
// hk * group + c % group, so that the heads that share K and V read them once.
struct CrossTensor {
    void* data;
    int64_t batch, token, head;   // strides in elements
};
struct CrossBias {
    void* data;                   // null: none
    int64_t batch, head, row;     // strides in elements; 0 along a shared axis (batch, head)
};
struct CrossArgs {
    CrossTensor q, k, v, out, dout, dq, dk, dv;
    CrossBias bias, dbias;
    const uint8_t* mask;
    int64_t mask_batch;
    float* stats;      // [2][batch][heads][nq]: maximum, sum
    void* rest;        // [batch][heads][nq][d] bf16: out before its rounding less out (bf16 storage)
    float* rows;       // [batch][heads][nq][4]: statistics and dout . out (written by the query pass, read by the other two)
    float* part;       // partial results of split calls
    int64_t batch;
    int nq, nk, heads, kv_heads, group, d;
    int key_div;       // key head of kv_heads' hk: hk / key_div (1, unless query heads that share one are taken singly)
    float scale;
    int direct_bias;          // the query pass writes dbias: no other entry or head shares it
    int splits, split_keys;   // forward: key ranges [s * split_keys, ...); dbias: splits of the shared entries
};
// How a forward call is laid out: columns per work-group (32: the four waves
// take different keys; 128: 32 columns a wave), and the split of the keys.
constexpr int kCrossMaxSplits = 64;   // one lane of the join each
struct CrossPlan {
    int cols, splits, split_keys;
    bool solo;   // a wave to each key head (32 columns at most)
};
// Whether tiles of 128 columns (or keys) are too few: below one for each of the
// 256 compute units.  (16 heads of d = 24 with bias: 2600 columns, 336 tiles, 31 us
// in tiles of 128 and 47 in tiles of 32; 1300, 176 tiles, 28 and 27.)
inline bool cross_few(int64_t heads, int64_t n) { return heads * ((n + 127) / 128) < 256; }
// Whether the key heads have so few columns, and are so many (four waves for each
// compute unit), that a wave takes one alone.  (1500 windows of 32 queries and 128
// keys, 4 heads: forward 25.6 us, dq 24.9; as 128-column tiles with three waves
// idle 30.4 and 39.9.  256 x 8 single queries over 2000 keys, d = 128: 359 and 374 us.  At the edge, 1024 key
// heads, one wave a SIMD: single queries over 256 keys of d = 64 13.6 and 17.5, over 8000 354 and 438; 32 queries and
// 128 keys of d = 32 6.2 and 7.0; but 32 queries and 2000 keys of d = 32 54.7 and 45.0.)
inline bool cross_solo(int64_t heads, int64_t cols) { return cols <= 32 && heads >= 1024; }
CrossPlan cross_plan(int64_t batch, int kv_heads, int64_t cols, int64_t nk);
size_t cross_part_floats(const CrossPlan& p, int64_t batch, int64_t nq, int heads, int d);
// How the key pass of a backward is laid out: 32 keys to a work-group (its waves on different queries) or 128, and
// the split of the queries.
struct CrossKvPlan {
    bool few;
    int ktiles, splits;
};
CrossKvPlan cross_kv_plan(int dtype, int d, int64_t heads, int64_t nk, int64_t per_head, int64_t group);
size_t cross_kv_part_floats(const CrossKvPlan& p, int64_t heads, int64_t nk, int d);
// Splits of the dbias pass over `shared` entries and heads per bias.
int cross_dbias_splits(int dtype, int d, int64_t slots, int64_t shared, int64_t nq, int64_t nk);
size_t cross_dbias_part_floats(int dtype, int splits, int64_t slots, int64_t nq, int64_t nk);
hipError_t launch_cross_forward(int dtype, const CrossArgs& a, const CrossPlan& p, hipStream_t s);
// Whether the query pass and the key pass run in one launch (launch_cross_backward_both, for the two).
bool cross_both(const CrossArgs& a, const CrossKvPlan& p);
hipError_t launch_cross_backward_both(int dtype, const CrossArgs& a, const CrossKvPlan& p, hipStream_t s);
hipError_t launch_cross_backward_q(int dtype, const CrossArgs& a, hipStream_t s);
hipError_t launch_cross_backward_kv(int dtype, const CrossArgs& a, const CrossKvPlan& p, hipStream_t s);
hipError_t launch_cross_backward_bias(int dtype, const CrossArgs& a, hipStream_t s);

// Residual addition with dropout (dropout.hip): out = res + kept x scale over
// [rows][cols][channels], res null for 0; share 0: a mask value per element,
// 1: all rows share one, 2: all columns do.
struct DropoutArgs {
    int64_t rows, cols, channels, row0, col0, n_cols, ld_in, ld_res, ld_res_out;   // row strides: x, res, out
    uint64_t seed, offset;
    uint32_t threshold;   // dropped below it
    uint32_t any;         // ~0; 0 where the threshold is 2^32, which no word reaches: nothing is kept
    float scale;
    int64_t loop;                    // filled in by the launcher, as are the next
    int blocks, lanes, span;
};
hipError_t launch_pair_dropout(int in_dtype, int out_dtype, int share, const DropoutArgs& a, const void* x,
                               const void* res, void* out, hipStream_t s);

// Activations in 8 bits (checkpoint8.hip): x to codes and powers (pack), or codes and powers to x.
struct CheckpointArgs {
    int64_t rows, n, ld;      // ld: elements from one row of x to the next
    int group;
    int wide;                 // filled in by the launcher, as are the next: every group allows vectors of eight
    int64_t groups, slots;    // groups of a row, and of all
};
int64_t checkpoint8_work_groups(CheckpointArgs a);
hipError_t launch_checkpoint8(int dtype, bool pack, CheckpointArgs a, const void* from, const uint8_t* powers, void* to, hipStream_t s);

// Relative position bias by buckets (relative.hip).  The pair form takes its channels as heads, and of base and out the
// data and the row stride.
struct RelativeArgs {
    int64_t batch, nq, nk;
    int heads, buckets, reach, table_bf16;
    const uint8_t* lut;
    const int32_t *pos_q, *pos_k, *seg_q, *seg_k;                       // seg_q null: one segment
    int64_t pos_q_batch, pos_k_batch, seg_q_batch, seg_k_batch;
    const void* table;
    CrossBias base, out;      // out: dout in the backward
    float *dtable, *part;     // part: partial sums (workspace)
    uint32_t* masks;          // which of them are there; filled in by the launcher, as are the next
    int wide, wide_keys;      // vectors of eight fit the tensors, and the keys' positions and segments
    int hb, tx, cwidth, cblocks, hblocks, waves, splits;
    int64_t loop, rblocks, span;
};
int64_t relative_bias_plan(RelativeArgs& a);                            // work-groups
int64_t relative_bias_backward_plan(RelativeArgs& a);
int64_t relative_pair_groups(RelativeArgs a);
size_t relative_bias_part_floats(RelativeArgs a);
size_t relative_pair_part_floats(RelativeArgs a);
hipError_t launch_relative_bias(int dtype, RelativeArgs a, hipStream_t s);
hipError_t launch_relative_bias_backward(int dtype, RelativeArgs a, hipStream_t s);
hipError_t launch_relative_pair(int dtype, RelativeArgs a, hipStream_t s);
hipError_t launch_relative_pair_backward(int dtype, RelativeArgs a, hipStream_t s);

// Norms of queries and keys by head with the position rotation (normrotate.hip).
struct NormSide {
    int heads;                // 0: this side is missing
    CrossTensor x, y, dx;     // y: dy in the backward
    const void *gain, *shift;
    int8_t* codes;
    uint8_t* powers;
    float *dgain, *dshift;
    int slots, steps;         // filled in by the launcher, as are the next: heads of a token that a wave takes at once, and
                              // the steps that all of them take
    int groups;                                       // work-groups
    int64_t tiles, chunk, chunks;                     // token tiles, entries of an item, chunks of entries
    int64_t step_tile, step_chunk;                    // what lies between two items of one wave
};
struct NormArgs {
    int64_t batch, n;
    int d, rot, weight_bf16, layer;
    float eps, inv_d;
    const int32_t* positions;
    int64_t positions_batch;
    const double* freqs;
    NormSide side[2];
    float* part;              // [work-groups][2][d]: dgain and dshift
    int ragged;               // filled in by the launcher: a row has fewer eighths than lanes
};
int64_t norm_rotate_backward_groups(NormArgs a, int dtype);             // its work-groups
hipError_t launch_norm_rotate(int dtype, bool adjacent, bool backward, NormArgs a, hipStream_t s);

}  // namespace trimul
