/*
 * moe.h -- C ABI of the MI355X (gfx950) MoE-layer library.
 *
 * One GPU's share of an expert-parallel MoE layer (paper section 2.1, Fig 3):
 * top-k routing, dispatch of token rows into expert-contiguous buffers, a
 * per-expert SwiGLU grouped GEMM (GEMM0 = gate and up projection, SiLU times
 * up, GEMM1 = down projection) and the weighted combine.  The forward pass is
 * one persistent megakernel whose workers are split at run time into
 * data-movement workers (dispatch and combine) and MFMA compute workers
 * (section 3, section 4); an in-kernel cost model (Eq 1-16) picks the split c,
 * the chunk count K and the steal count from the routing histogram.
 *
 * On one GPU the cross-GPU dispatch and combine become HBM-to-HBM copies:
 * rows of source rank r live in the staging region x[r*Tr .. (r+1)*Tr) and
 * their outputs go to y[r*Tr .. (r+1)*Tr).  This GPU is EP rank 0 and holds
 * the local experts [first_local_expert, first_local_expert + n_local_experts).
 *
 * Conventions for every entry point
 *  - bf16 tensors are passed as uint16_t bit patterns, row-major, densely
 *    packed (no strides), in device memory.
 *  - Every pointer argument is a device pointer unless marked "host".
 *  - The caller owns all memory: inputs, outputs, packed weights and the
 *    workspace.  The library never allocates or frees device memory; the
 *    handle holds host state only.
 *  - Streams are hipStream_t passed as void* (NULL = the null stream).  Calls
 *    are asynchronous on that stream unless documented to synchronise.
 *  - A handle is used from one host thread and one stream at a time.
 *  - Argument errors are detected on the host before anything is launched
 *    and return MOE_ERR_INVALID_ARG (nothing is enqueued).  Errors detected on
 *    the device (out-of-range routing ids, a wait that timed out) are latched
 *    in a device error word and returned by moe_sync_status and by the next
 *    synchronising call.
 *  - moe_last_error() returns a thread-local message for the last failure.
 */
#ifndef MOE_H
#define MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct moe_handle moe_handle;

typedef enum {
  MOE_OK = 0,
  MOE_ERR_INVALID_ARG = -1, /* bad argument, detected on the host */
  MOE_ERR_UNSUPPORTED = -2, /* valid but outside what the kernels support */
  MOE_ERR_HIP = -3,         /* a HIP runtime call failed */
  MOE_ERR_TIMEOUT = -4,     /* a device-side wait exceeded its time limit */
  MOE_ERR_ROUTING = -5,     /* routing ids out of range or repeated in a row */
  MOE_ERR_STATE = -6        /* call order violated (e.g. forward before tables) */
} moe_status;

typedef enum {
  MOE_MODE_DYNAMIC = 0, /* megakernel, plan from the in-kernel cost model */
  MOE_MODE_STATIC = 1,  /* megakernel, fixed split c = static_c, K = 1, no steal,
                           combine by movement workers only */
  MOE_MODE_SERIAL = 2   /* four kernels in sequence, each on every CU:
                           dispatch, GEMM0 + SiLU*up, GEMM1, combine */
} moe_mode;

/* Problem shape (section 3.1 notation: H hidden, I = ffn, E experts, top-k). */
typedef struct {
  int32_t n_src_ranks;        /* R >= 1 source ranks (staging regions) */
  int32_t tokens_per_rank;    /* Tr >= 1; T = R*Tr tokens in total */
  int32_t hidden;             /* H, multiple of 64, <= 16384 */
  int32_t ffn;                /* I (F), multiple of 64, <= 32768 */
  int32_t n_experts;          /* E, 1..512 */
  int32_t top_k;              /* k, 1..min(E, 8) */
  int32_t n_local_experts;    /* E_l, 1..64 */
  int32_t first_local_expert; /* e0, 0 <= e0 <= E - E_l */
  int32_t n_shared_experts;   /* S, 0..8, always-on experts applied to rank-0 tokens */
  int32_t n_workers;          /* persistent workgroups N; 0 = one per CU */
  int32_t gemm1_split;        /* split-K factor of GEMM1 (K = F): 1, 2, 4 or 8; 0 = chosen from F/H */
} moe_config;

#define MOE_CALIB_MAX_C 32
#define MOE_CALIB_MAX_K 4

/* Which movement work the bubble-steal window of Eq 11 holds (section
 * 3.2.2 leaves its W_comm undefined). */
typedef enum {
  MOE_WINDOW_PLAIN = 0,        /* W_dispatch + W_combine, the volume of Eq 5 */
  MOE_WINDOW_MOVE_STEAL = 1,   /* (W_dispatch + W_combine)(K-1)/K: compute workers
                                  whose GEMM0 rows are not dispatched yet copy rows
                                  themselves, so the first chunk's dispatch runs on
                                  all N workers before any GEMM tile starts, and the
                                  last chunk's combine runs on all N workers after
                                  the GEMMs (section 4); the default */
  MOE_WINDOW_LAST_COMBINE = 2  /* W_dispatch + W_combine (K-1)/K: only the last
                                  chunk's combine is outside the window */
} moe_steal_window;

/* Hardware input of the cost model (section 3, Fig 4a/b, Fig 7a).
 * For grid point i: c[i] movement workers move bw_bytes_per_s[i] payload
 * bytes/s (BW(c)) while N - c[i] compute workers reach comp_flop_per_s[i]
 * (TFLOPS(N - c)).  eff_chunk[j] is the chunked/unchunked GEMM throughput
 * ratio at k_chunks[j] chunks; alpha is the tile-level overlap ratio (Eq 6).
 * literal_volumes = 1 uses the printed remote-only volumes of Eq 2-3;
 * 0 (default) counts every moved row, since on one GPU rank 0's rows also go
 * through the movement workers.  bw_all_bytes_per_s is the rate of all N
 * workers moving together: the last chunk's combine runs on every worker
 * (section 4), so the exposed tail of Eq 6/10 moves at that rate; 0 takes the
 * printed BW(c) instead.  steal_window selects the window of Eq 11 (a
 * moe_steal_window); steal_ceil = 1 (the default) rounds Eq 14's share
 * W_steal / (N W_tile) up to whole tiles, 0 takes its whole part.  With
 * literal_volumes = 1, bw_all = 0, MOE_WINDOW_PLAIN and steal_ceil = 0 the
 * model is the printed equations as they stand. */
typedef struct {
  int32_t n_c;
  int32_t c[MOE_CALIB_MAX_C];            /* ascending, 1 <= c < N */
  double bw_bytes_per_s[MOE_CALIB_MAX_C];
  double comp_flop_per_s[MOE_CALIB_MAX_C];
  int32_t n_k;
  int32_t k_chunks[MOE_CALIB_MAX_K];     /* ascending, each in {1,2,4,8} */
  double eff_chunk[MOE_CALIB_MAX_K];     /* in (0, 1] */
  double alpha;                          /* in [0, 1] */
  int32_t literal_volumes;
  int32_t static_c;                      /* split used by MOE_MODE_STATIC */
  double bw_all_bytes_per_s;             /* >= 0; 0: tail at BW(c) */
  int32_t steal_window;                  /* a moe_steal_window */
  int32_t steal_ceil;                    /* 0 or 1 */
} moe_calib;

/* Execution plan (section 3.3): the split, the chunk count and the steal count. */
typedef struct {
  int32_t c;          /* movement workers (section 3.1) */
  int32_t K;          /* chunk count of the chunk pipeline (section 3.2.1) */
  int32_t n_steal;    /* GEMM tiles each movement worker steals (Eq 14) */
  int32_t final_all;  /* 1: every worker joins the combine once the compute
                         queue is empty (section 4); 0: movement workers only */
  double t_pred_s;    /* T_total(c, K) predicted by Eq 15; 0 for forced plans */
} moe_plan;

/* Byte offsets of the workspace regions (for inspection by tests). */
typedef struct {
  size_t total;
  size_t slot;        /* int32 [T*k]: slot of pair (g,j) or -1 */
  size_t inv;         /* int32 [T*min(k,E_l)]: g*k+j of each slot */
  size_t first_slot;  /* int32 [T] */
  size_t off;         /* int32 [E_l+1] */
  size_t sub_off;     /* int32 [4][E_l][9]: chunk offsets for K = 1,2,4,8:
                         entry q of (K option, expert) is the first slot of
                         chunk q, entry K the expert's end */
  size_t row_off;     /* int32 [4][E_l+S][9]: the row map of A, Hbuf and O
                         for K = 1,2,4,8: entry q < K of (K option, segment)
                         is the first row of chunk q of that segment (local
                         experts, then shared experts).  The (segment,
                         chunk) pairs follow each other in segment-major
                         order, each rounded up to a multiple of 32 rows, so
                         every one starts on a 32-row group; within one, rows
                         follow the slots (local experts) or the tokens
                         (shared experts).  Entries q >= K are 0. */
  size_t cnt_rank;    /* int32 [E_l][R] */
  size_t uniq;        /* int32 [R] */
  size_t stats;       /* int32 [16]: X, X_local, X_in, U_local, U_in, bad ids (0-5);
                         gate candidates (8): the experts whose logits the
                         filtering gate evaluated, T*k where the gate
                         evaluates every logit; GEMM tiles of the layer at
                         K = 1, 2, 4, 8 chunks (10-13), written by the table
                         builder for the cost model (section 3.2, Eq 14) */
  size_t plan;        /* moe_plan of the last megakernel launch */
  size_t err;         /* int32 device error word */
  size_t A;           /* bf16 [X_max + 256 E_l + 256][H] (X_max = T*min(k, E_l)):
                         dispatched rows at the rows of the row map of the
                         launch's chunk count, group-tiled: row r, column j
                         at element ((r/32)*(H/32) + j/32)*1024 + (r%32)*32 + j%32 */
  size_t Hbuf;        /* bf16 [rows of A + S*(Tr + 256)][F]: SiLU(gate)*up,
                         the same row map, group-tiled like A (F in place of H) */
  size_t O;           /* bf16 [rows of Hbuf][H]: expert outputs, the same row
                         map, row-major */
} moe_ws_layout;

/* Creates a handle.  cfg (host) is copied; calib (host) may be NULL for the
 * built-in MI355X calibration.  Validates the shape; does not touch the GPU
 * beyond querying the current device's CU count.  *out receives the handle. */
moe_status moe_init(const moe_config* cfg, const moe_calib* calib, moe_handle** out);

/* Releases the handle (host memory only).  NULL is accepted. */
moe_status moe_destroy(moe_handle* h);

/* Thread-local text of the last error returned on this thread ("" if none). */
const char* moe_last_error(void);

/* Replaces the calibration table (host struct, copied; validated against N).
 * The table lives in the workspace: if one is bound it is updated with a
 * synchronous copy, so call this between launches, not while one runs. */
moe_status moe_set_calib(moe_handle* h, const moe_calib* calib);
moe_status moe_get_calib(const moe_handle* h, moe_calib* out);

/* Time limit of every device-side wait of the megakernel (a wait for
 * dispatched rows, finished GEMM tiles or a finished chunk).  When a wait
 * exceeds it the workgroup latches MOE_ERR_TIMEOUT, raises an abort word that
 * makes every other wait give up, and the launch drains and exits.
 * inject_stall != 0 is a test hook that makes every wait target unreachable,
 * so the next megakernel launch exercises this path and exits after ~ms.
 * Default: 2000 ms, no injection. */
moe_status moe_set_timeout_ms(moe_handle* h, double ms, int32_t inject_stall);

/* Test hook for section 4's claim that dynamic claiming tolerates CUs that
 * run at different speeds: with max_sleeps > 0, every workgroup of the
 * megakernel waits a pseudo-random 0..max_sleeps times 64 cycles before
 * taking its arrival ticket and before each GEMM tile, and every wavefront
 * before each dispatch and combine unit it claims.  The counts are drawn
 * from (seed, workgroup, wavefront, event).  Results must not change.
 * max_sleeps in [0, 4096]; 0 (the default) turns it off. */
moe_status moe_set_jitter(moe_handle* h, uint32_t seed, int32_t max_sleeps);

/* Timeline trace of the megakernel (a measurement aid for the schedule of
 * sections 3-4: worker roles, tile waits, movement phases).  buf is caller-
 * owned device memory of `bytes` bytes, or NULL to turn tracing off.  Each
 * later moe_forward in a non-serial mode writes, per wavefront of the launch
 * (S = n_workers * 8 wavefronts, segment b * 8 + w for wavefront w of
 * workgroup b), up to R records into that wavefront's own segment:
 *   bytes 0-63: int32 header: magic 0x31435254, S, R, the int64 word offset
 *     of segment 0
 *   bytes 64..: int32 record count of each segment (S of them), padded to
 *     a multiple of 64 bytes
 *   then S segments of R records of 32 bytes:
 *     int64 word 0: kind | ticket << 8 | xcd << 20 | id << 32
 *     int64 words 1-3: times t0, t1, t2 from the 100 MHz device clock
 * (ticket: the recording workgroup's arrival ticket, which fixes its role:
 * tickets below the plan's c are movement workers; xcd: the XCD it runs on)
 * kind 1 workgroup (id 1 = movement worker): entry, plan + schedule built, exit
 * kind 2 compute tile (id = tile code: stage << 24 | XCD class << 21 |
 *        index): claimed, inputs ready, finished
 * kind 3 dispatch by one movement worker: start, end
 * kind 4 combine unit of one wavefront (id = unit | wave << 24): claimed,
 *        inputs ready (its GEMM1 row tiles done), end
 * kind 5 dispatch unit of one wavefront (id = unit | wave << 24): start,
 *        rows stored and drained, readiness counted
 * R = (bytes - header and counts) / 32 / S; records past R are dropped.  A
 * wavefront appends with a counter of its own (no global atomics).  The
 * counts and header are written at the end of the launch.  The layout of a
 * trace follows the handle's current plan; it changes nothing else.
 * Errors: MOE_ERR_INVALID_ARG for a non-NULL buf too small for one record per
 * wavefront. */
moe_status moe_set_trace(moe_handle* h, void* buf, int64_t bytes);

/* Workspace size in bytes and its region offsets (host out-parameters). */
moe_status moe_workspace_size(const moe_handle* h, size_t* bytes);
moe_status moe_workspace_layout(const moe_handle* h, moe_ws_layout* out);

/* Binds a caller-owned device workspace of at least moe_workspace_size bytes,
 * 256-byte aligned, and initialises its control words on `stream`.  The
 * workspace must stay alive and unused by others while the handle uses it. */
moe_status moe_set_workspace(moe_handle* h, void* ws, size_t bytes, void* stream);

/* Size of the packed expert weights: (E_l + S) * (R(2F) * H + R(H) * F) * 2
 * bytes, R(n) = n rounded up to a multiple of 256 (the operand slabs of the
 * GEMM tiles are padded to 256 rows). */
moe_status moe_packed_weights_size(const moe_handle* h, size_t* bytes);

/* Packs the expert weights into the GEMM operand layout (not part of the
 * layer; done once): each matrix is transposed to k-contiguous rows and
 * stored as strips of 64 rows, one 64 x 32 block per 32-deep k-step, so that
 * the GEMM tiles stream whole blocks.  The layout is internal to the
 * library: a packed buffer is for the build that wrote it.  w1, w3: bf16 [E_l][H][F] (gate, up), w2: bf16
 * [E_l][F][H] (down); ws1, ws3, ws2 the same for the S shared experts (NULL
 * when S = 0).  packed: device buffer of moe_packed_weights_size bytes. */
moe_status moe_pack_weights(moe_handle* h, const uint16_t* w1, const uint16_t* w3,
                            const uint16_t* w2, const uint16_t* ws1, const uint16_t* ws3,
                            const uint16_t* ws2, void* packed, void* stream);

/* Top-k routing (the routing that precedes the layer, section 4) followed by
 * moe_build_tables.  x: bf16 [T][H] (rank r's rows at r*Tr); wg: bf16 [H][E];
 * logit_bias: fp32 [E] added to the logits, or NULL.  Logits are accumulated
 * in fp32 over ascending h (one accumulator per (token, expert)); the top_k
 * largest logits are selected (ties -> smaller expert id), written in
 * descending order to topk_idx int32 [T][k]; topk_w fp32 [T][k] receives the
 * selected softmax probabilities divided by their sum.  A NaN logit is never
 * selected; a token with fewer than k others gets id 2^30 for the rest, which
 * latches MOE_ERR_ROUTING.  top_k must equal the configured k.  x and wg may
 * start at any bf16 value; off a 16-byte boundary they are copied first (x
 * into the workspace's A). */
moe_status moe_route(moe_handle* h, const uint16_t* x, const uint16_t* wg,
                     const float* logit_bias, int32_t top_k, int32_t* topk_idx,
                     float* topk_w, void* stream);

/* Size of the device scratch of moe_route_topk_static: 96 MiB. */
#define MOE_ROUTE_STATIC_SCRATCH_BYTES (96u << 20)

/* The top-k routing of moe_route (gate logits, softmax, top-k,
 * renormalisation; the same kernels and the same results) without a handle
 * and without allocating anything, for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that
 * forbid allocation.  It builds no routing tables (moe_build_tables does).
 * x: bf16 [T][H], wg: bf16 [H][E], logit_bias: fp32 [E] or NULL; writes
 * topk_idx int32 [T][top_k] and topk_w fp32 [T][top_k] as moe_route does.
 * The gate's scratch (a copy of wg where E is no multiple of 4, and of wg or
 * x where they start off a 16-byte boundary; for large batches of more than 32
 * experts, intermediate logits, norms and candidate chains) lives in a static
 * device array of MOE_ROUTE_STATIC_SCRATCH_BYTES that each GPU the library
 * runs on holds until the process ends; problems of more than about
 * E*H*2 + 16*T*E + 16*T = 96 MiB are refused with MOE_ERR_UNSUPPORTED (nothing
 * is launched).  Every call on a GPU shares that
 * GPU's array and leaves its contents behind: calls that overlap on one GPU
 * (other streams, other threads) race, so serialise them.  H must be a
 * multiple of 64 in [64, 16384], E in [1, 512], top_k in [1, min(E, 8)]. */
moe_status moe_route_topk_static(int32_t T, int32_t H, int32_t E, int32_t top_k, const uint16_t* x,
                                 const uint16_t* wg, const float* logit_bias, int32_t* topk_idx, float* topk_w,
                                 void* stream);

/* Builds the routing tables of this GPU's share from topk_idx int32 [T][k]
 * (section 3.1 descriptors and the dispatch permutation): per-(expert, rank)
 * counts, unique-token counts, expert offsets, the slot of each local pair
 * (slots ordered by local expert, then token), its inverse, each token's
 * first slot and the chunk offsets for K = 1, 2, 4, 8.  Ids outside [0, E) or
 * repeated within a row latch MOE_ERR_ROUTING and are treated as non-local. */
moe_status moe_build_tables(moe_handle* h, const int32_t* topk_idx, void* stream);

/* The MoE layer (section 2.1 stages 1-5) on the tables built from topk_idx.
 * x: bf16 [T][H] staging regions (16-byte aligned where the layer has shared
 * experts); topk_idx/topk_w: the routing result
 * (topk_idx must be the array the current tables were built from: checked by
 * address); packed: from moe_pack_weights; y: bf16 [T][H] output staging
 * regions, y[g] = sum over local j of topk_w[g,j] * FFN(x[g]) (+ the shared
 * experts for rank-0 tokens), 0 for tokens with no local expert.
 * mode: a moe_mode.  forced: host plan overriding the cost model (c, K,
 * n_steal, final_all) in the megakernel modes, or NULL.
 * The megakernel modes launch one persistent kernel of n_workers workgroups
 * that wait on each other, as an ordinary launch on `stream`: all of them
 * must be resident at once (the first call checks that the GPU holds them:
 * else MOE_ERR_UNSUPPORTED), and work on other streams that holds CUs while
 * it runs can keep workers from starting; the waiting ones then stop at the
 * timeout (moe_set_timeout_ms) with MOE_ERR_TIMEOUT. */
moe_status moe_forward(moe_handle* h, const uint16_t* x, const int32_t* topk_idx,
                       const float* topk_w, const void* packed, uint16_t* y,
                       int32_t mode, const moe_plan* forced, void* stream);

#define MOE_STACK_MAX 12

/* Several MoE layers in one persistent megakernel launch (a stack of
 * independent layers that share the tokens x but not their outputs, as the
 * layers of one GPU's expert-parallel share are when each takes its own
 * routing of the same batch).  layers[l]: the handle of layer l (each with its
 * own workspace, tables built from topk_idx[l], and n_workers equal to layer
 * 0's); packed[l], topk_idx[l], topk_w[l], y[l]: as in moe_forward for that
 * layer (host arrays of device pointers).  Each layer's plan comes from its
 * own prologue (section 3.3), or is `forced` (host, the same for every layer).
 * A workgroup moves on to layer l + 1 as soon as it finds no more work to
 * claim in layer l (section 4's dynamic claiming, across layers), so layer
 * l + 1's dispatch and first GEMM tiles overlap layer l's last tiles and its
 * combine; in every layer but the last, the final combine is left to that
 * layer's movement workers while the compute workers go on to the next
 * layer.  In dynamic mode those movement workers first claim layer l + 1's
 * dispatch units, beside layer l's GEMMs, when layer l + 1's prologue will
 * take a plan known before it runs (forced, or stored with its tables under
 * the current calibration).  Results are those of moe_forward on each layer,
 * bit for bit.
 * mode: MOE_MODE_DYNAMIC or MOE_MODE_STATIC.  1 <= n_layers <= MOE_STACK_MAX,
 * no handle twice.  The timeline trace is not recorded in a stacked launch.
 * Errors: as moe_forward, per layer (device errors latch in each layer's
 * error word). */
moe_status moe_forward_stack(moe_handle* const* layers, int32_t n_layers, const uint16_t* x,
                             const int32_t* const* topk_idx, const float* const* topk_w, const void* const* packed,
                             uint16_t* const* y, int32_t mode, const moe_plan* forced, void* stream);

/* Calibration of the cost model's hardware curves (BW(c), TFLOPS(N-c),
 * eff_chunk(K); Fig 4a/b, Fig 7a): runs the selected stages of the layer as
 * separate kernels on n_workers workgroups.  stages: bit 0 dispatch, bit 1
 * GEMM0 + SiLU*up, bit 2 GEMM1, bit 3 combine; the GEMMs use the tiling of K
 * chunks.  A stage reads what the earlier stages wrote, so a partial mask is
 * meant for timing (after a full run), not for producing y.  Same arguments
 * and table requirement as moe_forward. */
moe_status moe_run_stages(moe_handle* h, const uint16_t* x, const int32_t* topk_idx,
                          const float* topk_w, const void* packed, uint16_t* y,
                          int32_t stages, int32_t n_workers, int32_t K, void* stream);

/* Copies the plan of the last megakernel launch to *out (host).  Synchronises
 * the stream. */
moe_status moe_get_plan(moe_handle* h, moe_plan* out, void* stream);

/* Reads and clears the device error word; synchronises the stream. */
moe_status moe_sync_status(moe_handle* h, void* stream);

/* The cost model alone, on the host, for given routing volumes (fp64, same
 * operation order as the in-kernel prologue).  n_tiles[j]: GEMM tiles at
 * k_chunks[j]. */
moe_status moe_plan_host(const moe_handle* h, double w_comp, double w_dispatch,
                         double w_combine, const int64_t* n_tiles, moe_plan* out);

/* Tile geometry of the grouped GEMM for this shape: rows per tile (bm), GEMM0
 * tiles per row tile (nt0: column tiles over 2F) and GEMM1 tiles per row tile
 * (nt1: column tiles over H times the split-K factor of GEMM1), in whole slabs
 * of 256 columns, as the cost model counts them (layers of few rows may run
 * narrower tiles). */
moe_status moe_tile_geometry(const moe_handle* h, int32_t* bm, int32_t* nt0, int32_t* nt1);

/* ---- feed-forward blocks over row groups ------------------------------------
 *
 * The block of section 2.1 (gate and up projection, activation times up, down
 * projection) on rows that are already ordered by group, with the weights as
 * they are (not packed: in training they change every step), its backward
 * pass, and the same products in 8-bit integers for serving.  A group is an
 * expert (rows in the order of the layer's slots: group_off is then the `off`
 * region of moe_ws_layout), or the one block of a dense layer.
 *
 * group_off: int32 [n_groups + 1]; group g has rows [group_off[g],
 * group_off[g + 1]).  NULL where n_groups = 1: every row.  Offsets ascend in
 * [0, rows]; groups may be empty, and rows before the first or behind the last
 * group are neither read nor written.  (An offset outside that range or below
 * an earlier one counts as the nearest that is not: no row has two groups and
 * nothing outside the tensors is touched.)
 *
 * These calls need no handle.  They run on the current device, whose memory
 * every argument is; pointers start on 16-byte boundaries (group_off on its
 * values', the workspace on 256 bytes), else MOE_ERR_INVALID_ARG.  A workspace
 * holds scratch only: it needs no initialisation, keeps nothing from one call
 * for the next, and may serve any calls that run one after the other, but not
 * two that overlap.  No call allocates, waits, or adds in an order that changes
 * from run to run, and all can be captured into a graph.  Outputs must not
 * overlap inputs or each other.
 *
 * No value of another row enters a row's results, and none of another group a
 * weight's gradient.  The tiles, and the parts of a sum and their order, follow
 * from the config alone (moe_ffn_plan_host): under one config a row's results
 * are the same bits wherever it lies in its group, whatever the offsets and the
 * other rows are, and a weight's gradient depends on its group's rows in their
 * order alone.  Other rows, n_groups or widths in the config may change the last
 * bits of fp32 sums (a token alone and in a batch).  8-bit sums are exact, so
 * moe_gemm_i8 and the quantisers give a row the same bits under any config.
 */
typedef enum {
  MOE_ACT_NONE = 0,
  MOE_ACT_SILU = 1, /* v / (1 + e^-v) */
  MOE_ACT_GELU = 2  /* tanh form: v (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))) / 2 */
} moe_act;

#define MOE_MAX_GROUPS 512

typedef struct {
  int32_t rows;     /* T, 0..2^22 */
  int32_t hidden;   /* H, multiple of 64, <= 16384 */
  int32_t ffn;      /* F, multiple of 64, <= 32768 */
  int32_t n_groups; /* G, 1..MOE_MAX_GROUPS */
  int32_t act;      /* MOE_ACT_SILU or MOE_ACT_GELU */
} moe_ffn_config;

/* Workspace of moe_ffn_forward (backward = 0) or moe_ffn_backward (1). */
moe_status moe_ffn_workspace_size(const moe_ffn_config* cfg, int32_t backward, size_t* bytes);

/* y = (act(x W1) * (x W3)) W2 for the rows of each group.  x, y: bf16 [T][H];
 * w1, w3: bf16 [G][H][F] (gate, up); w2: bf16 [G][F][H] (down).  gate, up:
 * bf16 [T][F], x W1 and x W3 for moe_ffn_backward, or both NULL.  Products are
 * summed in fp32; act(.) * up is rounded to bf16 once, for the second product. */
moe_status moe_ffn_forward(const moe_ffn_config* cfg, const uint16_t* x, const int32_t* group_off,
                           const uint16_t* w1, const uint16_t* w3, const uint16_t* w2, uint16_t* gate, uint16_t* up,
                           uint16_t* y, void* ws, size_t ws_bytes, void* stream);

/* The gradients of moe_ffn_forward from dy (bf16 [T][H]), its inputs and the
 * gate and up it kept: dx bf16 [T][H] (NULL: not wanted), dw1, dw3 bf16
 * [G][H][F] and dw2 bf16 [G][F][H] (all, or all NULL).  The gradients of an
 * empty group's weights are 0.  Sums are in fp32; the gradients of gate and up
 * and act(gate) * up are rounded to bf16 once, for the products that take them. */
moe_status moe_ffn_backward(const moe_ffn_config* cfg, const uint16_t* dy, const uint16_t* x,
                            const int32_t* group_off, const uint16_t* w1, const uint16_t* w3, const uint16_t* w2,
                            const uint16_t* gate, const uint16_t* up, uint16_t* dx, uint16_t* dw1, uint16_t* dw3,
                            uint16_t* dw2, void* ws, size_t ws_bytes, void* stream);

/* Which tiles a product over row groups is computed by, and in how many parts
 * its depth is split (on the host; no device is touched). */
typedef enum {
  MOE_TILES_FEW4 = 0,  /* 32 rows x 64 columns, 4 waves that share the depth */
  MOE_TILES_FEW8 = 1,  /* the same, 8 waves */
  MOE_TILES_SMALL = 2, /* 128 x 128 */
  MOE_TILES_WIDE = 3,  /* 256 x 256 */
  /* of the gate's products alone: */
  MOE_TILES_RING = 4,  /* 128 x 128, a ring of four stages */
  MOE_TILES_BROAD = 5, /* 128 x 256, a ring of three */
  MOE_TILES_STRIPS = 6 /* 64 rows at a time x 256 columns, whose gate stays in registers */
} moe_tiles;

typedef struct {
  int32_t tiles; /* moe_tiles */
  int32_t split; /* parts of the depth, 1: whole */
} moe_product_plan;

typedef struct {
  moe_product_plan up, down; /* forward: both projections of x, and of the hidden rows */
  moe_product_plan dh;       /* backward: the hidden rows' gradients */
  moe_product_plan dx, dw;   /* and those of x and of the weights, in one launch of the same tiles */
} moe_ffn_plan;

moe_status moe_ffn_plan_host(const moe_ffn_config* cfg, moe_ffn_plan* out);

/* Rows in 8 bits: scale[t] = max |x[t][.]| / 127 in fp32, q[t][c] = x[t][c] /
 * scale[t] in fp32, rounded to the nearest whole number (halves to even), in
 * [-127, 127].  A row of zeros has scale 0 and q = 0.  A row that holds an
 * infinity or a NaN has scale NaN and q = 0, so that its products are NaN.
 * x: bf16 [rows][cols], q: int8 [rows][cols], scale: fp32 [rows]; rows in
 * [0, 2^22], cols a multiple of 64 up to 32768. */
moe_status moe_quantize_rows_i8(int32_t rows, int32_t cols, const uint16_t* x, int8_t* q, float* scale, void* stream);

/* Weights in 8 bits, a scale for each output channel: w bf16
 * [n_groups][depth][channels] (the layout of w1, w3 and w2) becomes wq int8
 * [n_groups][q_channels][depth], of which rows [first, first + channels) are
 * written, and scale fp32 [n_groups][q_channels]; scales and rounding as
 * moe_quantize_rows_i8's along the depth.  Two calls with q_channels = 2 F,
 * first = 0 and F put gate and up into one operand.  depth and channels:
 * multiples of 64, depth up to 32768, q_channels up to 65536. */
moe_status moe_quantize_weights_i8(int32_t n_groups, int32_t depth, int32_t channels, int32_t q_channels,
                                   int32_t first, const uint16_t* w, int8_t* wq, float* scale, void* stream);

typedef struct {
  int32_t rows;     /* T, 0..2^22 */
  int32_t depth;    /* K, multiple of 64, <= 32768 */
  int32_t channels; /* N, multiple of 8 (gated: of 16), <= 65536 */
  int32_t n_groups; /* G, 1..MOE_MAX_GROUPS */
  int32_t act;      /* MOE_ACT_NONE, or the activation of a gated product */
} moe_gemm_i8_config;

moe_status moe_gemm_i8_workspace_size(const moe_gemm_i8_config* cfg, size_t* bytes);
moe_status moe_gemm_i8_plan_host(const moe_gemm_i8_config* cfg, moe_product_plan* out);

/* v[t][n] = (sum_k xq[t][k] wq[g][n][k]) * x_scale[t] * w_scale[g][n] for the
 * rows t of group g: the sum exact in 32-bit integers (any int8 values), the
 * scales fp32 (neither their product nor the sum's with one of them has to be
 * within fp32's range).  act = MOE_ACT_NONE: y bf16 [T][N] is v.  Else channels
 * [0, N/2) are gates and the rest their ups: y bf16 [T][N/2] = act(v[t][f]) *
 * v[t][N/2 + f], v unrounded.  xq: int8 [T][K], x_scale: fp32 [T], wq: int8
 * [G][N][K], w_scale: fp32 [G][N]. */
moe_status moe_gemm_i8(const moe_gemm_i8_config* cfg, const int8_t* xq, const float* x_scale,
                       const int32_t* group_off, const int8_t* wq, const float* w_scale, uint16_t* y, void* ws,
                       size_t ws_bytes, void* stream);

/* ---- a training step around the products -------------------------------------
 *
 * What the layer and the blocks above leave to their user in a training step (and
 * in serving, the norm): the norm before the layer, the gate's logits and
 * gradients, the routing's losses, and the optimizer's step.
 *
 * Conventions are those of the calls over row groups: no handle, the current
 * device, pointers on 16-byte boundaries (seq_off on its values', the workspace
 * on 256 bytes), scratch workspaces without state, no allocation, wait or
 * addition whose order changes from run to run, and capture into graphs.  Outputs
 * must not overlap inputs or each other but where a call says so.
 */

/* ---- root-mean-square norm with the residual's addition ---- */
typedef struct {
  int32_t rows;   /* T, 0..2^22 (above H = 8192: below 2^22) */
  int32_t hidden; /* H, multiple of 8, 8..16384 */
  float eps;      /* > 0, added to the mean square */
} moe_rms_norm_config;

/* s = x + residual, rounded to bf16 (x where residual is NULL), r = 1 /
 * sqrt(mean_h(s^2) + eps) and y = s weight r, the norm of the rounded s.
 * x, residual: bf16 [T][H]; weight: bf16 [H].  Outputs, each NULL if not wanted,
 * but y or q has to be:
 *   sum    bf16 [T][H]  s
 *   rstd   fp32 [T]     r, for the backward pass
 *   y      bf16 [T][H]
 *   q      int8 [T][H] and scale fp32 [T] (both or neither): y in 8 bits as
 *          moe_quantize_rows_i8 would have it, from y in fp32
 * sum may be x or residual, and y may be x (the same address): a row is read
 * before it is written.  Sums are fp32: a row whose squares add up to more than
 * fp32 holds (magnitudes above 2^56 may) has r = 0, y = 0 and scale = 0, but NaN where
 * s weight passes fp32 too; one with an infinity or a NaN has y = NaN wherever r or s
 * is not finite, q = 0 and scale = NaN.  A row's results have the same bits in any
 * batch. */
moe_status moe_rms_norm_forward(const moe_rms_norm_config* cfg, const uint16_t* x, const uint16_t* residual,
                                const uint16_t* weight, uint16_t* sum, float* rstd, uint16_t* y, int8_t* q,
                                float* scale, void* stream);

/* Workspace of moe_rms_norm_backward. */
moe_status moe_rms_norm_workspace_size(const moe_rms_norm_config* cfg, size_t* bytes);

/* The gradients of moe_rms_norm_forward from dy (bf16 [T][H]), the s it kept (sum,
 * or x where there was no residual), weight and rstd:
 *   dx[t] = r (g - n mean_h(g n)) + dsum[t],  n = s r,  g = weight dy
 * the gradient of x and of residual alike; dsum: bf16 [T][H], the gradient that
 * reaches sum from elsewhere, or NULL.  dweight: fp32 [H], sum_t dy n (zeros where
 * T = 0).  dx (bf16 [T][H]) or dweight may be NULL.  dx may be dy, dsum or sum.
 * A row of dx has the same bits in any batch. */
moe_status moe_rms_norm_backward(const moe_rms_norm_config* cfg, const uint16_t* dy, const uint16_t* dsum,
                                 const uint16_t* sum, const uint16_t* weight, const float* rstd, uint16_t* dx,
                                 float* dweight, void* ws, size_t ws_bytes, void* stream);

/* ---- the gate and the routing's losses in training ----
 *
 * moe_route chooses experts and gives their weights; these calls give what its
 * training needs: the logits, losses on them, and gradients back to the tokens
 * and to the gate.
 *
 * seq_off: int32 [n_seqs + 1]; sequence s has rows [seq_off[s], seq_off[s + 1]),
 * under the rules of group_off: NULL where n_seqs = 1 (every row), ascending
 * offsets in [0, rows], any of them empty, and rows before the first or behind the
 * last sequence are neither read nor written. */
typedef struct {
  int32_t rows;      /* T, 0..2^22 */
  int32_t hidden;    /* H, multiple of 64, 64..16384 */
  int32_t n_experts; /* E, 1..512 */
  int32_t top_k;     /* k, 1..min(E, 8) */
  int32_t n_seqs;    /* S, 1..MOE_MAX_GROUPS */
} moe_router_config;

/* Workspace of moe_gate_logits (backward = 0) or moe_gate_backward (1). */
moe_status moe_gate_workspace_size(const moe_router_config* cfg, int32_t backward, size_t* bytes);

/* Which tiles the gate's products are computed by (on the host; no device is
 * touched): logits in parts of the depth H, dwg in parts of the rows, dx (with dwg
 * wanted too) in parts that strips of rows are dealt to, whole where it takes tiles. */
typedef struct {
  moe_product_plan logits, dx, dwg;
} moe_gate_plan;

moe_status moe_gate_plan_host(const moe_router_config* cfg, moe_gate_plan* out);

/* logits[t][e] = sum_h x[t][h] wg[h][e] + logit_bias[e]: x bf16 [T][H], wg bf16
 * [H][E], logit_bias fp32 [E] or NULL, logits fp32 [T][E].  The sum is fp32, in
 * another order than moe_route's, and in longer batches in one that depends on the
 * row's place, so the last bits may differ from the logits that moe_route compares.
 * top_k is not read. */
moe_status moe_gate_logits(const moe_router_config* cfg, const uint16_t* x, const uint16_t* wg,
                           const float* logit_bias, const int32_t* seq_off, float* logits, void* ws, size_t ws_bytes,
                           void* stream);

/* The gradients of moe_gate_logits from dlogits (fp32 [T][E]): dx bf16 [T][H] =
 * dlogits wg^T, dwg bf16 [H][E] = x^T dlogits, dbias fp32 [E] = sum_t dlogits; each
 * may be NULL.  dlogits are rounded to bf16 once for the two products, as every
 * operand of the matrix instructions is, so each of their terms is off by up to 2^-8 of
 * itself (dbias adds them unrounded); sums are fp32.  Where terms cancel and that is
 * too much, two calls have the products of dlogits to 2^-16 of a term: of dlogits
 * rounded to bf16 and of what that left, their results added in fp32.  Without rows
 * dwg and dbias are 0. */
moe_status moe_gate_backward(const moe_router_config* cfg, const float* dlogits, const uint16_t* x,
                             const uint16_t* wg, const int32_t* seq_off, uint16_t* dx, uint16_t* dwg, float* dbias,
                             void* ws, size_t ws_bytes, void* stream);

/* Workspace of moe_route_loss. */
moe_status moe_route_loss_workspace_size(const moe_router_config* cfg, size_t* bytes);

/* The losses of a routing: logits fp32 [T][E], topk_idx int32 [T][k].
 *   counts int32 [S][E]: how often each expert is chosen in each sequence (ids
 *          outside [0, E) count nowhere, repeated ones each time)
 *   lse    fp32 [T]: log sum_e exp(logits)
 *   loss   fp32 [2]: loss[0], balance: the mean over sequences that have rows of
 *          E / (k n^2) sum_e counts[s][e] P[s][e], n the sequence's rows and P the
 *          sums of their softmax over all experts (1 where both are even);
 *          loss[1], z: the mean of lse^2 over the rows of all sequences.
 * Without any rows both are 0.  A logit of -inf has probability 0 (moe_route selects
 * one only where fewer than k others are left, with weight 0; counts count it like any
 * other); a row of nothing else has lse = -inf and adds 0 to both sums.  A row with a
 * NaN or +inf has lse = NaN, and so have the losses it enters.  hidden is not read. */
moe_status moe_route_loss(const moe_router_config* cfg, const float* logits, const int32_t* topk_idx,
                          const int32_t* seq_off, int32_t* counts, float* lse, float* loss, void* ws, size_t ws_bytes,
                          void* stream);

/* dlogits fp32 [T][E] from the losses' gradients dloss (fp32 [2], device: the
 * coefficients times whatever the losses are scaled by; NULL: zeros) and from the
 * gradient dtopk_w (fp32 [T][k]) of moe_route's topk_w (fp32 [T][k]; both or
 * neither).  With p = exp(logits - lse), c = counts of the row's sequence, of n rows,
 * S' sequences and N rows in all:
 *   dloss[0] E / (k n^2 S') p_e (c_e - sum_i c_i p_i) + dloss[1] 2 / N lse p_e
 *   + sum over j with topk_idx[j] = e of w_j (dw_j - sum_i w_i dw_i)
 * (the counts are constants; the weights are the softmax over the chosen logits).
 * counts and lse as moe_route_loss gave them.  A row of -inf alone (lse = -inf) has
 * gradient 0 whatever its ids and weights are (moe_route's are the k smallest and NaN).
 * dlogits may be logits (the same address). */
moe_status moe_route_loss_backward(const moe_router_config* cfg, const float* logits, const int32_t* topk_idx,
                                   const float* topk_w, const int32_t* seq_off, const int32_t* counts,
                                   const float* lse, const float* dloss, const float* dtopk_w, float* dlogits,
                                   void* stream);

/* ---- AdamW over many tensors ---- */
typedef struct {
  double lr, beta1, beta2, eps; /* lr >= 0, betas in [0, 1), eps >= 1e-15 */
  double grad_scale;            /* gradients are multiplied by it */
  int32_t step;                 /* t, counted from 1 */
  uint32_t seed;                /* of what is rounded at random */
  int32_t state_bits;           /* 32 or 8 */
} moe_adamw_config;

#define MOE_ADAMW_BLOCK 256

/* One tensor of n values.  param: bf16, or NULL; master: the same weights in fp32,
 * or NULL (param alone is stepped then); at least one of them.  grad: bf16, or fp32
 * where grad_fp32 = 1.  m, v: fp32, or 8 bits each: m in e4m3, v in e5m2 (OCP), times
 * a scale for every MOE_ADAMW_BLOCK consecutive values, m_scale and v_scale: fp32
 * [ceil(n / 256)], on their values' alignment (NULL with 32 bits).  All zeros is the
 * state before the first step. */
typedef struct {
  int64_t n; /* 0..2^36 - 4096 */
  uint16_t* param;
  float* master;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  float weight_decay; /* >= 0 */
  int32_t grad_fp32;  /* 0 or 1 */
} moe_adamw_tensor;

/* One step for every tensor (host array of n_tensors, copied before the call
 * returns), in place:
 *   g = grad_scale grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   w -= lr (weight_decay w + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
 * in fp32, from m and v before they are rounded.  now: NULL, or device memory with
 * three fp32 values, lr, grad_scale and step, in place of the config's (a captured
 * step reads them at each replay; a step below 1 counts as 1, and above 2^24 fp32
 * holds no more every step: steps there share random bits, and adding 1 stands still).
 * A grad_scale there that is NaN leaves every tensor as it was: a step to be skipped.
 *
 * master's rounded value goes to param; param alone, and states in 8 bits, are
 * rounded up or down at random, with the probabilities that keep their means (to
 * the nearest, an average that moves by less than half a step would stand still).
 * The random bits are a function of (seed, step, the tensor's place in the list, the
 * value's place in it), so a step gives the same bits wherever it runs.  An 8-bit
 * block's scale is its largest magnitude / 448 (m) or / 57344 (v); a block below
 * 2^-110 is 0; a v above 0 stays above 0; a block that holds an infinity or a NaN
 * gets scale NaN, so that it stays NaN.  A tensor must not be in the list twice. */
moe_status moe_adamw(const moe_adamw_config* cfg, const moe_adamw_tensor* tensors, int32_t n_tensors, const float* now,
                     void* stream);

#ifdef __cplusplus
}
#endif
#endif
