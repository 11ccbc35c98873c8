// Internal launch interface between the C-ABI layer (api.cpp) and the HIP
// kernels.  Nothing here is exported.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace isam {

enum Dtype : int { kF32 = 0, kBF16 = 1 };

// One GEMM launch: C[M][N] (+)= op(A)[M][K] . op(B)[K][N].
struct GemmArgs {
    const void* A;
    const void* B;
    void* C;
    float* partial;        // split-K partial sums [k_splits][M][N] fp32 (k_splits > 1)
    const float* bias;     // optional per-column bias added in the epilogue (fp32, length N)
    int64_t M, N, K;
    int64_t lda, ldb, ldc;
    int trans_a, trans_b;
    int ab_type;           // kF32 / kBF16
    int c_type;            // kF32 / kBF16
    int accumulate;        // C += instead of C =
    // Strided batch (grid z): problem z uses A, B, C offset by z times these
    // byte strides.  batch == 1 for a single product; batched launches never
    // split K and never take the skinny kernels.
    int64_t batch;
    int64_t stride_a, stride_b, stride_c;
};

// Tile configurations of the MFMA tile kernel (see gemm.hip).
enum TileCfg : int {
    kTile256x256 = 0,  // 4 waves, 128x128 per wave
    kTile256x128 = 1,  // 4 waves, 128x64 per wave
    kTile128x128 = 2,  // 4 waves, 64x64 per wave
    kTile128x64 = 3,   // 4 waves, 64x32 per wave
    kTile64x64 = 4,    // 4 waves, 32x32 per wave
    kTile128x32 = 5,   // 4 waves, 32x32 per wave (tall-skinny)
    kTileCount
};

struct GemmPlan {
    int tile;        // TileCfg
    int vec;         // 1: 16-byte vector loads (needs alignment); 0: element loads
    int k_splits;    // >= 1
    int64_t k_per_split;  // multiple of the tile K depth
    int group_m;     // tile-row group size of the rasterisation
    int xcd_remap;   // spread consecutive tiles of one group over one XCD
    int dma;         // 1: direct-to-LDS kernel where it applies (bf16, A K-contiguous, vec)
    int dma_waves;   // 4 or 8 waves per workgroup for the direct-to-LDS kernel
    int fixup;       // 1: a two-slice split on 256x256 tiles may sum its slices inside the kernel
                     // 2: the same, each slice finishing half of the tile (whole grid resident)
    int skinny;      // 1: streaming kernel for N <= 32 (k_splits = K slices of skinny_k_slice);
                     // 2: bf16 row-streaming kernel (16 rows per workgroup, whole K, no split);
                     // 4: narrow dot-product kernel (N < 8, not a multiple of the vector width)
    int small;       // 1: small-product kernel (one 32x32 tile per workgroup, waves split K)
    int sk;          // 1: stream-K schedule of the direct-to-LDS kernel (persistent grid of
                     //    sk_grid workgroups sharing the (tile, K tile) units evenly)
    int sk_grid;
    int sk_keep;     // whole rounds left to the stream-K shares (0 or 1)
};
// Stream-K schedule: persistent grid size for a tile shape (one workgroup per
// CU; two for 128x128 tiles, whose ring takes half the LDS) and its workspace
// (one fp32 partial-sum tile and one 128-byte flag line per workgroup).
int gemm_sk_grid(int tile, int cus);
size_t gemm_sk_ws_bytes(int tile, int grid);
bool gemm_sk_tile(int tile);
// Mid-size bf16 products (gemm_ring.hpp), any operand layout with 16-byte
// aligned rows: instance (0: none, 1: 128x128 tiles, 2: 64x64 tiles, 3: 128x64 tiles, fp32 only) and K
// slices per tile, summed in the kernel through the workspace (a.partial).
struct RingPlan {
    int ring, splits;
    int mixed;  // 1: treat every tile's slices as spread over XCDs (test hook)
};
// Rows are readable to ld values each (operands packed by the library): the
// last row's 16-byte pieces may then pass the row's last value.
struct RingPadded {
    bool a, b;
};
void gemm_ring_dims(int ring, int* bm, int* bn);
size_t gemm_ring_ws_bytes(const RingPlan& r, int64_t M, int64_t N);
hipError_t launch_gemm_ring(const GemmArgs& a, const RingPlan& r, const RingPadded& pad, int cus, hipStream_t s);
// fp32 products on bf16 terms formed in registers (gemm_f32x.hpp): the same
// tiles, K slices and workspace.
hipError_t launch_gemm_f32x(const GemmArgs& a, const RingPlan& r, const RingPadded& pad, int cus, hipStream_t s);
// One value per launch for flags that stale workspace contents must not match
// (random 64-bit start).
uint64_t next_fixup_epoch();
// Small products: at most kSmallMaxTiles output tiles of 32x32 and K <= kSmallMaxK
// (A K-contiguous, 16-byte aligned operands, batch 1: checked by the caller).
constexpr int64_t kSmallMaxTiles = 64;
constexpr int64_t kSmallMaxK = 1024;
bool gemm_small_fits(int64_t M, int64_t N, int64_t K);
// Very shallow products (rows of A up to 512 bytes, N <= 256, NN): B in registers, A streamed.
constexpr int64_t gemm_stream_max_k(int ab_type) { return ab_type == kF32 ? 128 : 256; }
bool gemm_stream_fits(const GemmArgs& a);
hipError_t launch_gemm_stream(const GemmArgs& a, int cus, hipStream_t s);
hipError_t launch_gemm_small(const GemmArgs& a, hipStream_t s);
int64_t skinny_k_slice(int ab_type);
int skinny_rows_per_wg(int ab_type);
hipError_t launch_skinny(const GemmArgs& a, int splits, hipStream_t s);
int skinny_stream_rows();
hipError_t launch_skinny_rows(const GemmArgs& a, hipStream_t s);
// Narrow product (N < 8): dot-product kernel streaming A once (NN, A rows
// 16-byte aligned, any ldb).
hipError_t launch_narrow(const GemmArgs& a, hipStream_t s);

void tile_dims(int tile, int ab_type, int* bm, int* bn, int* bk);

// Launch facts cached per device and kernel (launch_cache.cpp): raise a
// kernel's dynamic-LDS limit to at least `lds` bytes, and its resident
// workgroups per CU at `threads` threads and `lds` dynamic LDS bytes (0 when
// the runtime cannot say).
hipError_t ensure_dynamic_lds(const void* fn, size_t lds);
int resident_per_cu(const void* fn, int threads, size_t lds);
hipError_t launch_gemm(const GemmArgs& a, const GemmPlan& p, hipStream_t s);
// Copies src[s_rows][s_cols] (leading dimension ld, elements of esize = 2 or 4
// bytes) into the dense dst[d_rows][d_cols] -- transposed (dst[i][j] =
// src[j][i]) if asked -- with zeros outside the source; d_cols * esize must
// be a multiple of 16 and dst 16-byte aligned for the plain copy.
// fp32 operand split into six bf16 K blocks of kp values (terms by the 2-bit
// fields of pattern: 0 = h, 1 = m, 2 = l).  k_rows = false: src [s_rows][K],
// dst [d_rows][6 kp] (d_cols = kp); k_rows = true: src [K][s_cols], dst
// [6 kp][d_cols] (d_rows = kp).  d_cols a multiple of 8, dst 16-byte aligned.
hipError_t launch_split6(const float* src, int64_t s_rows, int64_t s_cols, int64_t ld, uint16_t* dst,
                         int64_t d_rows, int64_t d_cols, int64_t kp, bool k_rows, uint32_t pattern, int cus,
                         hipStream_t s);
hipError_t launch_pack(const void* src, int64_t s_rows, int64_t s_cols, int64_t ld, void* dst, int64_t d_rows,
                       int64_t d_cols, int esize, bool transpose, int cus, hipStream_t s);

// bf16 rows src[rows][s_cols] (leading dimension ld) into dense 16-byte aligned
// rows dst[rows][d_cols], zeros past s_cols (d_cols a multiple of 8); rows = 0: nothing.
struct PackRows {
    const uint16_t* src;
    int64_t rows, s_cols, ld;
    uint16_t* dst;
    int64_t d_cols;
};
hipError_t launch_pack_rows(const PackRows& a, const PackRows& b, int cus, hipStream_t s);

// Depthwise kh x kw convolution, NHWC.  Y is [batch][Ho][Wo][C*cm] in y_type.
struct DwArgs {
    const void* x;
    const void* w;  // [kh][kw][C][cm]
    void* y;
    int64_t batch, H, W, C, cm, kh, kw, stride, pad, Ho, Wo;
    int in_type, y_type;
};
hipError_t launch_depthwise(const DwArgs& a, hipStream_t s);
// Fused depthwise + pointwise (bf16 input): rows per tile, 0 if not applicable.
int dwsep_fused_rows(const DwArgs& d, int64_t C_out, int lds_max);
hipError_t launch_dwsep_fused(const DwArgs& d, const void* pw, void* out, int64_t C_out, int out_type, int lds_max,
                              int cus, hipStream_t s);
// Fused depthwise + pointwise, fp32 in and out (fp32 MFMA).
bool dwsep_fused_f32_ok(const DwArgs& d, int64_t C_out, int lds_max);
hipError_t launch_dwsep_fused_f32(const DwArgs& d, const void* pw, void* out, int64_t C_out, int cus, hipStream_t s);

// GRU recurrence (the input projection is a GemmArgs launch done before).
struct GruArgs {
    int64_t T, batch, I, H;
    int w_type;
    const float* gx;        // [T*batch][3H] fp32: x W^T (no bias)
    const float* h0;        // [batch][H] fp32 or null
    const void* U;          // [3H][H]
    const float* bias;      // [3H] or null
    const float* bias_hn;   // [H] or null
    float* h_seq;           // [T][batch][H] or null
    float* h_T;             // [batch][H] or null
    void* hbuf;             // [T+1] slots of `slot` elements in w_type: ring of per-step MFMA
                            // copies of h, slot t holding h_{t-1} as [batch][H]
    int64_t slot;           // elements per ring slot: batch*H rounded up to a multiple of 256 bytes
    unsigned* sync;         // barrier counters and error word (kGruSyncBytes, zeroed by the launch)
    uint64_t timeout_ticks; // bound on one barrier wait, in ticks of the 100 MHz constant clock
    int stall;              // 1: barrier targets one arrival beyond the grid (never met), so every
                            // wait runs into the bound; exercises the timeout path
    int units_per_wg;       // J
    int batch_per_wg;       // BB
    int n_wg;
    int barrier_group;      // workgroups per first-level barrier counter
    int groups;             // batch-group schedule: barrier domains (batch groups); 0 otherwise
    int device_scope;       // batch-group schedule: 1 = exchange through device scope even when a
                            // domain sits on one XCD
    int xcds;               // batch-group schedule: width of the round-robin dispatch over XCDs
};
// Barrier layout of the GRU kernel: per batch group a domain of 512 words
// holds the domain counter and up to 31 first-level group counters (64
// bytes apart).
constexpr int kGruMaxGroupsPerDomain = 31;
size_t gru_lds_bytes(int w_type, int64_t H, int J);
// Resident workgroups of the recurrent kernel per compute unit at this LDS size.
int gru_blocks_per_cu(int w_type, size_t lds);
// Barrier area of the GRU workspace: the domain counters of the grid barrier
// in the first 32 KiB, then per-domain flag words (64 per domain) and the XCC
// id of every workgroup (batch-group schedule).
constexpr int kGruBarrierBytes = 32768;
constexpr int kGruSyncBytes = 65536;
constexpr int kGruFlagWord = 8192;    // flags of domain d: words kGruFlagWord + 64 d ..
constexpr int kGruXccWord = 12288;    // XCC id of workgroup b: word kGruXccWord + b
constexpr int kGruMaxWgs = 4096;
// Ring slot stride in elements: whole 256-byte blocks, so no cache line holds
// parts of two slots.
inline int64_t gru_slot_elems(int64_t batch, int64_t H, int64_t es) { return (batch * H * es + 255) / 256 * 256 / es; }
hipError_t launch_gru_recurrent(const GruArgs& a, hipStream_t s);
// Batch-group persistent recurrence (bf16): `groups` independent barrier
// domains, each a set of n_wg / groups workgroups that own kGruGroupUnits
// hidden units apiece with their rows of U held in registers, and each a
// contiguous slice of the batch.  Needs H = 256 * KS (KS in 1..4), at most 16
// batch columns per group and every workgroup resident.
constexpr int kGruGroupUnits = 32;
bool gru_group_supported(int64_t H);
size_t gru_group_lds_bytes();
hipError_t launch_gru_group(const GruArgs& a, hipStream_t s);
// Resident workgroups of the batch-group kernel per compute unit (0: none).
int gru_group_blocks_per_cu(int64_t H);
// NaN into h_seq and h_T if the recurrence's sticky error word is set.
hipError_t launch_gru_error_fill(const GruArgs& a, hipStream_t s);
// Bound on one barrier wait of the persistent recurrence (2 s at 100 MHz).
constexpr uint64_t kGruTimeoutTicks = 200000000ull;
// Bounded wait of a GEMM tile's second K slice for the first (100 MHz ticks).
constexpr uint64_t kFixupTimeoutTicks = 200000000ull;
// Workspace of a two-slice split summed inside the kernel: one 256x256 fp32
// tile of partial sums per output tile, then one 128-byte flag line per tile.
size_t gemm_fixup_ws_bytes(int64_t M, int64_t N);
// Stepwise recurrence (state init + one kernel per step, launched in order);
// hstate is a [2][batch][H] fp32 workspace.
hipError_t launch_gru_steps(const GruArgs& a, float* hstate, hipStream_t s);
// Static scratch of the allocation-free GRU entry point: its device address on
// the current device (looked up once per device).
constexpr size_t kGruScratchBytes = size_t(64) << 20;
hipError_t gru_scratch(void** ptr);
// T == 0: h_T = h0 (or zeros when h0 is null).
hipError_t launch_gru_copy_state(const float* h0, float* h_T, int64_t n, hipStream_t s);


// Linear GRU (linear_gru.hip).  Strides in elements; rows are [2H] (gx, dgx) or [H].
constexpr int64_t kLinGruChunk = 128;  // steps between two rows of `states`
constexpr int kLinGruFew = 8;                                // steps forward up to which no tile is formed (64-bit offsets)
constexpr int kLinGruSteps = 8;                              // steps of a group, four groups to a wave
constexpr int kLinGruFwdWaves = 8, kLinGruBwdWaves = 4;      // waves of a tile
constexpr int kLinGruLooks = 1 << 22;                    // bound of a wait for an earlier tile, a microsecond or more each
struct LinGruArgs {
    int64_t T, batch, H;
    int type;                // of gx, h_seq, dh_seq and dgx
    int candidate;           // 1: tanh, 0: linear
    const void* gx;
    int64_t gx_t, gx_b;
    const float* bias;       // [2H] or null
    const float* h0;         // [batch][H] or null
    const uint8_t* reset;    // nonzero: the step starts from a zero state; or null
    int64_t rs_t, rs_b;
    void* h_seq;             // or null
    int64_t h_t, h_b;
    float* h_T;              // [batch][H] or null
    float* states;           // [ceil(T / 128)][batch][H]: state before steps 0, 128, ...; or null (forward)
    // backward
    const void* dh_seq;      // or null
    int64_t dh_t, dh_b;
    const float* dh_T;       // [batch][H] or null
    void* dgx;
    int64_t dg_t, dg_b;
    float* dh0;              // [batch][H] or null
    float* dbias;            // [2H] or null
    uint64_t* chain;         // lingru_chain_bytes: counter, then the tiles' words; or null (a single tile)
    float* bias_part;        // [tiles][batch][2H] (dbias)
};
// Tiles of one column of channels, and the bytes of their chain.
int64_t lingru_tiles(int64_t T, bool backward);
bool lingru_strides(int64_t stride_t, int64_t width, int64_t es);
size_t lingru_chain_bytes(int64_t T, int64_t batch, int64_t H, bool backward);
hipError_t launch_lingru_forward(const LinGruArgs& a, hipStream_t s);
hipError_t launch_lingru_backward(const LinGruArgs& a, hipStream_t s);

// Gated residual norm (norm_residual.hip): rows of D values at their own leading
// dimensions, gate and dgate dense [gates][D], rows / gates rows to a gate row.
constexpr int64_t kNormMaxD = 16384;
struct NormArgs {
    int64_t rows, D;
    int type;                       // of every matrix
    int64_t gates, rows_per_gate;   // 1 and all rows without a gate
    const void* x;                  // or null: r_out = r
    const void* r;                  // backward: r_out of the forward pass
    const void* gate;               // or null
    int64_t ld_x, ld_r;
    const float* w_post;            // or null: no norm after the block
    const float* w_pre;
    float scale, eps;
    void* r_out;
    void* y;
    int64_t ld_ro, ld_y;
    // backward
    const void* dy;
    const void* dr_out;             // or null
    void* dx;
    void* dr;
    int64_t ld_dy, ld_dro, ld_dx, ld_dr;
    void* dgate;                    // or null
    float* dw_post;                 // or null
    float* dw_pre;                  // or null
    int parts;                      // workgroups of a gate row; 0: row groups own whole gate rows
    float* partial;                 // [3][grid][D]: sums for w_pre, w_post and the gate
};
// Grid and a.parts of the backward pass; the pointers and leading dimensions count by their
// alignment (none given: aligned).
void norm_bwd_grid(const NormArgs& a, int cus, int64_t* grid, int* parts);
// Most workgroups it takes at any alignment.
int64_t norm_bwd_most(const NormArgs& a, int cus);
hipError_t launch_norm_forward(const NormArgs& a, int cus, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, int64_t grid, hipStream_t s);

// Gated feed-forward block (gated_ffn.hpp): bf16 tiles over 16-byte aligned rows,
// a kernel for up to kGatedTokens rows of x (either type, any alignment), and the
// element-wise step behind fp32 products.
constexpr int64_t kGatedTokens = 16;
constexpr int64_t kGatedRows = 16;   // rows of a workgroup of the element-wise step
constexpr int64_t kGatedF32Tile = 32;  // rows and values of f of a tile of the fp32 kernel
enum GatedTile : int { kGated256 = 0, kGated128 = 1, kGated64 = 2 };
struct GatedArgs {
    int64_t M, K, F;
    int act;                  // 0 sigmoid, 1 silu, 2 gelu
    const void* x;            // [M][K]
    const void* W;            // [2F][K]: gate rows, then up rows
    const float* bias;        // [2F] or null
    int64_t ld_x, ld_w;
    void* out;                // p [M][F]; backward: [dG dU], [M][2F]
    int64_t ld_out;
    const void* dout;         // backward: dp [M][F]
    int64_t ld_dout;
    float* bias_part;         // backward: partial sums [rows][2F], or null
    int whole;                // rows of out and dout on 4 bytes, F a multiple of 8 (set by the launch)
    float* gu;                // element-wise step: G and U, [M][2F]
};
int gated_tile(int64_t M, int64_t F, int cus);
int64_t gated_bias_rows(int tile, int64_t M);
hipError_t launch_gated_tiles(const GatedArgs& a, int tile, bool backward, hipStream_t s);
hipError_t launch_gated_tokens(const GatedArgs& a, int type, bool backward, hipStream_t s);
// The sum of two [M][K] fp32 matrices at a.gu, as bf16 at a.out.
hipError_t launch_gated_join(const GatedArgs& a, hipStream_t s);
// fp32 without the library's product: whether it is taken, and its launch.
bool gated_f32_direct(int64_t M, int64_t K, int64_t F, int cus);
hipError_t launch_gated_f32(const GatedArgs& a, bool backward, hipStream_t s);
hipError_t launch_gated_pairs(const GatedArgs& a, bool backward, hipStream_t s);

// Projection with its epilogue (linear.hip): bf16 tiles over 16-byte aligned rows (GatedTile's, each as wide as
// high), up to kLinearFew rows of x (backward kGatedTokens) and fp32 grids of few tiles at any alignment, and the
// element-wise pass.
constexpr int64_t kLinearRows = 32;  // rows of a workgroup of the element-wise pass
constexpr int64_t kLinearFew = 64;   // most rows of the kernel for a few of them
struct LinearArgs {
    int64_t M, K, N;
    int act;                  // 0 sigmoid, 1 silu, 2 gelu, 3 none
    const void* x;            // [M][K]
    const void* W;            // [N][K]
    const float* bias;        // [N] or null
    int64_t ld_x, ld_w;
    const void* side;         // residual [M][N] or null; backward: dout
    int64_t ld_side;
    void* out;                // [M][N]; backward: dP
    int64_t ld_out;
    float* bias_part;         // backward: partial sums [rows][N], or null
    int whole;                // rows of out and side on 4 bytes, N a multiple of 8 (set by the launch)
    const float* pre;         // the pass: P, [M][ld_pre]; null: column sums of side alone
    int64_t ld_pre;
};
hipError_t launch_linear_tiles(const LinearArgs& a, int tile, bool backward, hipStream_t s);
hipError_t launch_linear_tokens(const LinearArgs& a, int type, bool backward, hipStream_t s);
hipError_t launch_linear_f32(const LinearArgs& a, bool backward, hipStream_t s);
hipError_t launch_linear_pass(const LinearArgs& a, int type, bool backward, hipStream_t s);

// Selective scan (selective_scan.hpp).  Rows of a [T][batch] tensor, strides in elements.
struct ScanRows {
    const void* p;  // or null
    int64_t st, sb;
};
// Tokens between two rows of `states`: what the backward pass holds of them in registers.
constexpr int scan_chunk(int64_t N) { return N > 32 ? 8 : 16; }
constexpr int kScanFew = 8;           // tokens forward up to which no tile is formed (64-bit offsets)
constexpr int64_t kScanMaxN = 64;
constexpr int64_t kScanMaxSegments = 64;
struct ScanArgs {
    int64_t T, batch, D, N;
    int type;                 // of the rows
    ScanRows x, dt, z, B, C, y;
    const float* A;           // [D][N]
    const float* skip;        // [D] or null
    const float* dt_bias;     // [D] or null
    const float* h0;          // [batch][D][N] or null
    const uint8_t* reset;     // or null
    int64_t rs_t, rs_b;
    float* h_T;               // [batch][D][N] or null
    float* states;            // [ceil(T / scan_chunk)][batch][D][N]: state before tokens 0, 16, ...; or null (forward)
    int64_t segs, seg_len;    // segments of time, tokens of each (a multiple of the tile)
    float* seg_sum;           // [segs][batch][D]
    float* seg_end;           // [segs][batch][D][N]
    // backward
    ScanRows dy, dx, ddt, dz, dB, dC;
    const float* dh_T;        // [batch][D][N] or null
    float* dA;                // [D][N] or null
    float* dskip;             // [D] or null
    float* ddt_bias;          // [D] or null
    float* dh0;               // [batch][D][N] or null
    float* bc_part;           // [blocks][T][batch][2N]: dB and dC of a workgroup's channels
    float* par_part;          // [segs][batch][D N + 2 D]: dA, dskip, ddt_bias
};
int64_t scan_channels(int64_t N);     // of a workgroup
int64_t scan_segments(int64_t T, int64_t batch, int64_t D, int64_t N, int cus);
int64_t scan_segment_length(int64_t T, int64_t segs);
bool scan_pieces(const ScanRows& r, int64_t D, int64_t N, int type);
hipError_t launch_scan_copy(const float* src, float* dst, int64_t n, hipStream_t s);
hipError_t launch_scan_forward(const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_backward(const ScanArgs& a, hipStream_t s);

// Causal convolution (causal_conv.hip): K taps over time, channels independent.
constexpr int64_t kConvMaxK = 6;
constexpr int64_t kConvFew = 8;   // tokens up to which one thread owns a channel's whole sequence
struct ConvArgs {
    int64_t T, batch, C, K;
    int type;                 // of the rows and states
    int act;                  // 0 none, 1 silu
    ScanRows x, y;
    const float* w;           // [K][C], the last row for the token itself
    const float* bias;        // [C] or null
    const void* state;        // [K-1][batch][C]: the inputs before the first token; or null
    const uint8_t* reset;     // or null
    int64_t rs_t, rs_b;
    void* state_T;            // or null
    // backward
    ScanRows dy, dx;
    const void* dstate_T;     // or null
    void* dstate;             // or null
    float* dw;                // [K][C] or null
    float* dbias;             // [C] or null
    float* part;              // [rows][K C], then [rows][C]
    bool packed;              // a wave may have several sequences
    // set by conv_plan
    int64_t run, rows;        // tokens of a wave, rows of partial sums
};
bool conv_packs(const ScanRows& r, int64_t C, int type);
void conv_plan(ConvArgs& a, int cus);
hipError_t launch_causal_conv(const ConvArgs& a, bool backward, hipStream_t s);

// Beam search (beam.hip): rows of V logits, `beams` to a text, of which `width` candidates go on.
constexpr int64_t kBeamMax = 64;        // beams and width
constexpr int64_t kBeamPart = 4096;     // logits of a workgroup
struct BeamArgs {
    int64_t batch, beams, V, width;
    int type;                  // of the logits
    const void* logits;
    int64_t lg_b, lg_n;        // strides of a text and of a beam, in elements
    const float* scores;       // [batch][beams]
    const uint8_t* finished;   // [batch][beams] or null
    int64_t end;               // the token that ends a text; negative: none
    float* scores_out;         // [batch][width]
    int32_t* parent;
    int32_t* token;
    uint8_t* finished_out;     // or null
    int64_t parts;             // workgroups of a row
    double2* sums;             // [batch][beams][parts]: largest logit, sum of exponentials from it
    uint64_t* best;            // [batch][beams][parts][width]: order of the logit, then of the token
};
hipError_t launch_beam_step(const BeamArgs& a, hipStream_t s);
struct ReorderArgs {
    int64_t outer, batch, beams, width, bytes;   // of a row
    const void* src;           // [outer][batch][beams] rows
    const int32_t* parent;     // [batch][width]
    void* dst;                 // [outer][batch][width] rows
};
hipError_t launch_beam_reorder(const ReorderArgs& a, hipStream_t s);

// out[g][c] = sum over r of part[g][r][c] (rows may be 0: zeros), up to three such
// sums in one launch.
struct ColSum {
    const float* part;
    void* out;
    int64_t rows, cols, groups;
    int type;  // of out
};
hipError_t launch_colsum(const ColSum* sums, int count, hipStream_t s);

}  // namespace isam
