/*
 * goldy.h — C ABI of the concurrent-GEMM library (GO-Kernels + dynamic logic)
 * for one GB300 (sm_103a).
 *
 * The paper's problem (Sec. 4.1, Sec. 4.4): a set of independent GEMMs is
 * queued at once; the system picks how many run concurrently (the
 * concurrency degree, CD) and, for each GEMM, a kernel tuned for the
 * resources it will share at that CD (a "GO-Kernel"), then launches them.
 * This header splits that into
 *
 *   goldy_plan()  host only, integer work, no CUDA call: GEMM descriptors +
 *                 lookup table -> schedule (groups run one after another; in
 *                 a group, CD streams; per GEMM a kernel variant and a stream
 *                 slot).  The dynamic logic of Sec. 4.3 / Sec. 4.4.
 *   goldy_run()   asynchronous launch of a schedule on caller-owned streams
 *                 and caller-owned device buffers.  No allocation, no
 *                 synchronisation.  The GO-Kernels themselves (Sec. 4.2).
 *
 * Conventions for every entry point:
 *   - Return a goldy_status; nothing is thrown across the ABI.  On error the
 *     thread-local text of goldy_last_error() says why.
 *   - Pointers the caller passes stay owned by the caller.  Objects the
 *     library returns (goldy_lut, goldy_schedule, goldy_graph) are owned by
 *     the library and released with the matching *_free function.
 *   - Device pointers are plain CUDA device addresses on the current device;
 *     streams are cudaStream_t values passed as void*.
 *
 * Matrix layout (Sec. 2.1.2; transposes T1 = T2 = 0 in the K x N sense):
 *   A: M x K, row-major, element (i, k) at A[i*lda + k], bf16
 *   B: K x N, row-major, element (k, j) at B[k*ldb + j], bf16
 *   C: M x N, row-major, element (i, j) at C[i*ldc + j], fp32 or bf16
 *   C = A * B with fp32 accumulation; bf16 output is rounded to nearest even.
 */
#ifndef GOLDY_H_
#define GOLDY_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GOLDY_ABI_VERSION 2

typedef enum goldy_status {
  GOLDY_OK = 0,
  GOLDY_ERR_INVALID_ARG = 1,   /* null pointer, bad size, bad stride, bad flags */
  GOLDY_ERR_UNSUPPORTED = 2,   /* valid request this build does not implement */
  GOLDY_ERR_LUT = 3,           /* lookup table missing, malformed or empty */
  GOLDY_ERR_CUDA = 4,          /* a CUDA runtime/driver call failed */
  GOLDY_ERR_TIMEOUT = 5,       /* a kernel gave up a bounded wait (see goldy_device_error) */
  GOLDY_ERR_NOMEM = 6          /* host allocation failed, or a caller buffer is too small */
} goldy_status;

typedef enum goldy_dtype { GOLDY_BF16 = 0, GOLDY_F32 = 1 } goldy_dtype;

/* One GEMM (Sec. 2.1.2), or a strided batch of equal-sized GEMMs (the
 * paper's B-GEMMs, Sec. 6.7): entry i computes C + i*stride_c = (A +
 * i*stride_a)(B + i*stride_b).  Sizes, leading dimensions and strides are in
 * elements.  Supported now: trans_a = trans_b = 0, a = b = GOLDY_BF16, c =
 * BF16 or F32, M, N, K >= 0, lda >= K, ldb >= N, ldc >= N, lda and ldb
 * multiples of 8 (16-byte rows for the tensor-memory-accelerator copies);
 * batch >= 1 (1: a plain GEMM, strides ignored); for batch > 1 the entries
 * do not overlap — stride_a >= M*lda, stride_b >= K*ldb, stride_c >= M*ldc —
 * and stride_a, stride_b are multiples of 8. */
typedef struct goldy_gemm_desc {
  int64_t M, N, K;
  int64_t lda, ldb, ldc;
  int32_t trans_a, trans_b;    /* the paper's T1, T2; only 0, 0 is supported */
  int32_t a_dtype, b_dtype, c_dtype;
  int32_t reserved;            /* must be 0 */
  int64_t batch;               /* strided batch entries, >= 1 */
  int64_t stride_a, stride_b, stride_c;
} goldy_gemm_desc;

typedef struct goldy_lut goldy_lut;
typedef struct goldy_schedule goldy_schedule;
typedef struct goldy_graph goldy_graph;

/* ---- planning policies (goldy_plan flags) -------------------------------
 * The comparison configurations of Sec. 5.5 through one schedule type:
 *   AUTO        the dynamic logic: preferred CD from the table, min(CD,
 *               available), heterogeneous grouping (Sec. 4.3, Sec. 6.7);
 *               then, in each wave (a group's members taken CD at a time,
 *               in launch order), a GEMM takes the kernel kind of the
 *               wave's largest GEMM (no K split, that kernel's grid cap)
 *               when the kind suits it — same C dtype, K no longer than the
 *               largest's, M >= 128 for a CTA-pair kind, M <= 2 x the tile
 *               rows for a transposed skinny-M kind, M >= 64 otherwise —
 *               so that a fused wave runs as fewer launches
 *   SEQUENTIAL  isolation-tuned kernels one after another ("sequential")
 *   DEFAULT     isolation-tuned kernels, every GEMM at once on its own stream
 *               ("default", the naive all-streams launch)
 *   GO          GO-Kernels for CD = n, every GEMM at once ("GO-Kernels")
 *   FORCE_CD    GO-Kernels at a fixed CD; put the CD in bits 8..15
 *               (GOLDY_PLAN_FORCE_CD | (cd << 8)) */
#define GOLDY_PLAN_AUTO 0
#define GOLDY_PLAN_SEQUENTIAL 1
#define GOLDY_PLAN_DEFAULT 2
#define GOLDY_PLAN_GO 3
#define GOLDY_PLAN_FORCE_CD 4
/* Launch-mode bit, combinable with any policy above.  FUSED: within each
 * group, the GEMMs that run at the same time (a "wave" of CD members) and
 * share a kernel kind and output dtype go into ONE persistent launch over the
 * concatenation of their tiles (at most 16 GEMMs per launch); its grid cap is
 * the sum of the members' caps.  A wave's launches carry launch priorities
 * ranked by their FLOPs, and the first wave's largest launch goes out first
 * (outside a stream capture the other streams also wait until all of its
 * CTAs have begun).  Groups are not separated by a join: the run forks once
 * and joins once, and a later group's launches take lower priorities, so they
 * fill the SMs an earlier group frees.  A fused run with
 * goldy_run_opts.inputs_ready = 1 goes out on streams[0] alone
 * instead, each wave's largest launch first, every launch overlapping the
 * previous one's tail (no fork, no join).  Without FUSED every GEMM is its own
 * launch on its slot's stream and the groups run one after another.  The plan
 * (groups, CDs, variants, slots) is the same, and so are the results, byte
 * for byte. */
#define GOLDY_PLAN_FUSED 0x10

#define GOLDY_MAX_GEMMS 64      /* GEMMs per plan */
#define GOLDY_MAX_STREAMS 16    /* concurrency degrees 1, 2, 4, 8, 16 (Sec. 4.3) */

/* ---- version / device ---------------------------------------------------- */

/* GOLDY_ABI_VERSION of the loaded library. */
int goldy_abi_version(void);

/* Text of the last error on this thread ("" if none).  Valid until the next
 * call into the library from the same thread. */
const char* goldy_last_error(void);

/* ---- kernel variant registry --------------------------------------------
 * A variant is one GO-Kernel configuration (Sec. 4.2): a tile shape and
 * shared-memory/tensor-memory footprint (kind), a split of the K loop, and a
 * resource constraint (RC) capping the persistent grid at the whole GPU, half
 * or a quarter of it (Sec. 4.2.1's GPU, GPU/2, GPU/4).  With a split S > 1
 * the S K-ranges of a tile are summed in split order 0 .. S-1 (in a cluster
 * of S CTAs, or by the last split to arrive, through the workspace; a CTA-pair
 * kind always through the workspace). */
typedef struct goldy_variant_info {
  int32_t id;
  int32_t kind;           /* tile/footprint family, 0 .. n_kinds-1 */
  int32_t mma_m;          /* rows of the tensor-core tile (128) */
  int32_t mma_n;          /* columns of the tensor-core tile */
  int32_t swap_ab;        /* 1: computes C^T = B^T A^T tiles (skinny M) */
  int32_t stages;         /* shared-memory pipeline depth */
  int32_t acc_stages;     /* accumulators held in tensor memory */
  int32_t tmem_cols;      /* tensor-memory columns allocated per CTA */
  int32_t smem_bytes;     /* dynamic shared memory per CTA */
  int32_t split_k;        /* K-loop split factor (1, 2, 4, 8) */
  int32_t rc_div;         /* grid cap = resident CTAs per SM * SMs / rc_div */
  int32_t ctas_per_sm;    /* CTAs per SM the footprint is sized for */
  int32_t cta_pair;       /* 2: tiles of 2 x 128 rows computed by a pair of CTAs
                             (one tcgen05 MMA across both SMs), else 1 */
  char name[32];
} goldy_variant_info;

/* Number of variant ids (ids are 0 .. count-1). */
int goldy_variant_count(void);

/* Describe variant `id`.  GOLDY_ERR_INVALID_ARG if id is out of range or out
 * is null. */
goldy_status goldy_variant_info_get(int id, goldy_variant_info* out);

/* ---- lookup table (the dynamic logic's profiled data, Sec. 4.3) ---------
 * File format (little-endian): magic "GOLDYLUT", u32 version = 1, u32 entry
 * count, u32 variant-id bound, u32 SM count of the profiling GPU, 8 zero
 * bytes; then 16-byte entries {u8 lm, ln, lk, out_dtype; u8 pref_cd; u8 flags;
 * u16 variant[5]} strictly sorted by (lm, ln, lk, out_dtype), where lm, ln,
 * lk are floor(log2) of M, N, K and variant[c] is the GO-Kernel for CD class
 * c in {1, 2, 4, 8, 16}; flags: how the bucket's GEMM runs with an
 * element-wise op of its output size (see goldy_corun_plan) — bit 0: at once
 * (else one after the other), bit 1: with the CD-2 GO-Kernel (else the CD-1
 * kernel), bits 2-3: the op's grid-cap divisor 1, 2 or 4 as 0, 1, 2; other
 * bits 0.  GOLDY_ERR_LUT if the data is malformed or empty. */
goldy_status goldy_lut_load(const char* path, goldy_lut** out);
goldy_status goldy_lut_from_memory(const void* data, size_t bytes, goldy_lut** out);
void goldy_lut_free(goldy_lut* lut);

/* Bucket key of one GEMM: (lm << 24) | (ln << 16) | (lk << 8) | c_dtype,
 * each log2 floored (0 for a size of 0) and clamped to 255; a batched GEMM
 * is bucketed by its rows over all entries (lm = floor log2(M * batch)). */
goldy_status goldy_bucket_key(const goldy_gemm_desc* d, uint32_t* key);

/* ---- planning (host only; makes no CUDA call) ---------------------------
 * Plan n (1 .. GOLDY_MAX_GEMMS) GEMMs with the policy in `flags`.
 * Deterministic: the schedule is a pure function of (descs, lut, flags).
 * GOLDY_ERR_INVALID_ARG for null pointers, n out of range, bad flags or a
 * descriptor violating the layout rules above; GOLDY_ERR_UNSUPPORTED for a
 * transposed operand or unsupported dtype. */
goldy_status goldy_plan(const goldy_gemm_desc* descs, int n, const goldy_lut* lut,
                        int flags, goldy_schedule** out);

/* ---- logistic-regression CD predictor (Sec. 4.3, Eq. 1) -----------------
 * The paper predicts each GEMM's preferred CD with a multi-class logistic
 * regression trained offline once per GPU.  Features (GOLDY_LR_FEATURES, in
 * this order): M (times the batch), N, K, then for each CD class c in (1, 2,
 * 4, 8, 16) three numbers of the table's GO-Kernel for the GEMM's bucket at
 * c: its CTAs of work (output tiles of all batch entries x split-K slices;
 * two CTAs per tile for a CTA-pair kernel), its CTAs resident per SM, and its waves (CTAs of work over
 * CTAs/SM x sm_count / grid-cap divisor, rounded up).  The model min-max
 * normalises them ((x - lo) / (hi - lo), 0 where hi == lo), scores each
 * class s_c = b_c + sum_j W[c][j] x_j (in j order, doubles, no fused
 * multiply-add), and predicts the class of largest score (= largest Eq. 1
 * probability; ties to the smaller CD).
 * Model file (little-endian): magic "GOLDYLRM", u32 version = 1, u32 feature
 * count = 18, u32 class count = 5, u32 SM count (> 0), 8 zero bytes; then
 * f64 lo[18], hi[18], W[5][18] (class-major), b[5]; all finite, hi >= lo.
 * GOLDY_ERR_LUT if malformed.  The library owns the object. */
#define GOLDY_LR_FEATURES 18
typedef struct goldy_predictor goldy_predictor;
goldy_status goldy_predictor_load(const char* path, goldy_predictor** out);
goldy_status goldy_predictor_from_memory(const void* data, size_t bytes, goldy_predictor** out);
void goldy_predictor_free(goldy_predictor* p);

/* The table entry a GEMM plans with (its bucket, or the nearest stored one):
 * preferred CD and the variant per CD class. */
goldy_status goldy_lut_lookup(const goldy_lut* lut, const goldy_gemm_desc* d, int* pref_cd, int variants[5]);

/* The predictor's raw (unnormalised) features of one GEMM against a table,
 * for an SM count (> 0).  Used to build the training set. */
goldy_status goldy_lr_features(const goldy_gemm_desc* d, const goldy_lut* lut, int sm_count,
                               double out[GOLDY_LR_FEATURES]);

/* Predicted preferred CD (1, 2, 4, 8 or 16) of one GEMM; probs (may be null)
 * receives Eq. 1's probability per CD class. */
goldy_status goldy_predict_cd(const goldy_predictor* p, const goldy_lut* lut, const goldy_gemm_desc* d,
                              int* cd, double probs[5]);

/* goldy_plan with the predictor (may be null: same as goldy_plan) supplying
 * the preferred CDs under GOLDY_PLAN_AUTO: a bucket's preference is the
 * smallest prediction over its GEMMs, and the CD run is still
 * min(preference, GEMMs available).  Kernels still come from the table.  The
 * forced policies ignore the predictor. */
goldy_status goldy_plan_ex(const goldy_gemm_desc* descs, int n, const goldy_lut* lut,
                           const goldy_predictor* predictor, int flags, goldy_schedule** out);

/* Explicit schedule (used by the offline profiler and for measuring any
 * chosen schedule): GEMM i runs in group group_of[i] (groups are run in
 * increasing order, ids 0 .. n_groups-1 all used), with variant
 * variant_of[i], on stream slot slot_of[i] (< GOLDY_MAX_STREAMS).  A group's
 * CD is its number of distinct slots.  flags: 0 or GOLDY_PLAN_FUSED (waves are
 * then the group's members taken CD at a time, in GEMM index order). */
goldy_status goldy_schedule_build(const goldy_gemm_desc* descs, int n, const int* group_of,
                                  const int* variant_of, const int* slot_of, int flags,
                                  goldy_schedule** out);

/* Sizes of a schedule.  workspace_bytes is the device workspace goldy_run
 * needs (split-K partial tiles and arrival counters, and for GOLDY_PLAN_FUSED
 * schedules of several GEMMs 8 bytes of unit counters per GEMM; 0 if none). */
goldy_status goldy_schedule_query(const goldy_schedule* s, int* n_gemms, int* n_groups,
                                  int* max_streams, size_t* workspace_bytes);

/* Placement of GEMM `gemm`: its group, variant, stream slot and its group's CD. */
goldy_status goldy_schedule_entry(const goldy_schedule* s, int gemm, int* group,
                                  int* variant, int* slot, int* cd);

/* Canonical bytes of the plan (little-endian u32 words): "GSCH", version 1,
 * n_gemms, n_groups, max_streams, flags; per group: cd, size, members in
 * launch order; per GEMM: group, variant, slot.  Writes at most `cap` bytes;
 * *size gets the full length (GOLDY_ERR_NOMEM if cap is too small). */
goldy_status goldy_schedule_serialize(const goldy_schedule* s, void* buf, size_t cap,
                                      size_t* size);

void goldy_schedule_free(goldy_schedule* s);

/* ---- execution ----------------------------------------------------------
 * Launch schedule `s`: A[i], B[i], C[i] are device pointers of GEMM i;
 * `workspace` is a device buffer of at least goldy_schedule_query's
 * workspace_bytes (may be null when that is 0), zero-filled by the caller
 * before its first use — the kernels leave it zero-filled after every
 * complete run; streams[0 .. n_streams-1] are CUDA streams with n_streams >=
 * max_streams.  Groups run in order (in GOLDY_PLAN_FUSED mode by launch
 * priority, see there); the run forks from streams[0] and joins back to it,
 * so work queued on streams[0] before the call happens before every GEMM and
 * work queued on streams[0] after it happens after all of them.  Slot k runs on streams[k].  Asynchronous: returns after launching;
 * no allocation, no synchronisation.  Errors: GOLDY_ERR_INVALID_ARG (null or
 * misaligned pointers, too few streams, workspace too small),
 * GOLDY_ERR_CUDA (launch failure).  A kernel that gave up a bounded wait
 * shows up later through goldy_device_error(); the outputs of that run are
 * then incomplete, and its workspace may hold non-zero split-K arrival or
 * unit counters: zero-fill the workspace again before the next run that uses
 * it. */
goldy_status goldy_run(const goldy_schedule* s, const void* const* A, const void* const* B,
                       void* const* C, void* workspace, size_t workspace_bytes,
                       void* const* streams, int n_streams);

/* Options of goldy_run_ex / goldy_graph_create_ex (all fields may be null).
 * ev_begin[i] / ev_end[i] (cudaEvent_t as void*, caller-created, one pair per
 * GEMM) are recorded on GEMM i's stream right before and right after its
 * kernel launch, so the caller can time each launch on the stream it runs on.
 * Inside a graph capture they become event-record nodes of the graph. */
typedef struct goldy_run_opts {
  void* const* ev_begin;
  void* const* ev_end;
  /* Optional device buffer of unsigned 64-bit words for a phase trace: every
   * CTA of every GO-Kernel launch writes 16 words at trace[cta * 16 + k]
   * (k: 0 entry, 1 set-up done and the epilogue past the wait for the
   * previous kernel, 2 first TMA load, 3 first full stage seen by
   * the MMA thread, 4 first accumulator committed, 5 first accumulator seen
   * by the epilogue, 6 split-K partial stored, 7 split-K arrival counted,
   * 8 first unit stored, 9 exit, 10 set-up done before waiting for the
   * previous kernel on the stream, 11 producer started — %globaltimer
   * nanoseconds; 12 the launch's grid size; 13 the CTA's index in its launch;
   * 14 units this CTA processed; 15 SM id).  The launches of one run use
   * consecutive regions in launch order (launch j starts after the CTAs of
   * launches 0 .. j-1); a launch that does not fit in the trace_ctas CTAs
   * left is not traced.  Null: no tracing. */
  void* trace;
  size_t trace_ctas;
  /* 0 (default): each GO-Kernel launch may begin its set-up (barriers, tensor
   * memory, descriptor prefetch) while the previous kernel on its stream is
   * still running — programmatic dependent launch; the kernel waits for that
   * kernel to complete before it touches global memory, so results and
   * stream order are unchanged.  1: plain serialised launches. */
  int32_t serial_launch;
  /* 0 (default): as above.  1: the caller asserts that no kernel enqueued
   * before this run (on its streams) writes any A or B of the run.  Each
   * GO-Kernel's load and MMA roles then start as soon as its CTAs are
   * resident, while the previous kernel on the stream may still be running
   * (reading A and B, filling shared and tensor memory); the epilogue still
   * waits for that kernel to complete before it writes C or the workspace.
   * Results are unchanged when the assertion holds; a violated assertion
   * (an earlier kernel producing A or B) gives wrong results.  The bounded
   * waits of the load and MMA roles then also cover the previous kernel's
   * remaining time.  No effect with serial_launch = 1. */
  int32_t inputs_ready;
  /* Limit of every bounded wait inside the GO-Kernels, in microseconds
   * (0: the default of 2 seconds).  A wait that runs out sets the error word
   * (goldy_device_error) and the kernel returns. */
  uint32_t wait_limit_us;
  /* Test hook, 0 in normal use.  1: in the run's first GO-Kernel launch, CTA
   * 0 never fills its first shared-memory stage (no copy is issued), so that
   * the MMA thread's bounded wait for it runs out: the launch returns with
   * the error word set to 2 (an MMA-thread wait gave up) and the outputs of
   * that launch are incomplete.  Used with a short wait_limit_us to test the
   * timeout path without faulting anything. */
  int32_t test_stall_first_stage;
} goldy_run_opts;

/* goldy_run with options; opts may be null (then identical to goldy_run). */
goldy_status goldy_run_ex(const goldy_schedule* s, const void* const* A, const void* const* B,
                          void* const* C, void* workspace, size_t workspace_bytes,
                          void* const* streams, int n_streams, const goldy_run_opts* opts);

/* Prepared run: record goldy_run_ex(...) with these exact pointers and
 * streams once — tensor maps encoded, kernel parameter blocks built, grids and
 * cluster shapes fixed, fork/join events owned by the object — so that
 * goldy_exec_launch replays it with plain launch calls on the same streams.
 * On this platform a replay costs about half of a one-kernel CUDA graph
 * launch.  Nothing is launched by goldy_exec_create; the buffers and streams
 * must outlive the object.  Not thread-safe per object. */
typedef struct goldy_exec goldy_exec;
goldy_status goldy_exec_create(const goldy_schedule* s, const void* const* A, const void* const* B,
                               void* const* C, void* workspace, size_t workspace_bytes,
                               void* const* streams, int n_streams, const goldy_run_opts* opts,
                               goldy_exec** out);
/* Enqueue a prepared run (asynchronous, no allocation). */
goldy_status goldy_exec_launch(const goldy_exec* e);
void goldy_exec_free(goldy_exec* e);

/* Device time of prepared runs replayed back to back: `warmup` untimed
 * replays, then `reps` replays timed by CUDA events on the first stream
 * (replay k uses execs[k % n]: rotate copies of the inputs past the L2).  All
 * n runs must share their first stream and partition.  Synchronises on the
 * end event; *ms_per_rep = elapsed / reps.  Events live in the runs'
 * partition, so this also times work inside an SM partition. */
goldy_status goldy_exec_time(const goldy_exec* const* execs, int n, int warmup, int reps, float* ms_per_rep);

/* ---- a GEMM co-scheduled with a non-GEMM kernel (Sec. 7.1) --------------
 * The paper co-runs a GEMM with an element-wise add of the GEMM's output size
 * (2 kernels at once) and finds concurrency worth restricting for
 * memory-bound GEMMs.  The non-GEMM here is Z = X + Y over n contiguous
 * elements of `dtype` (bf16: each element widened to fp32, added in IEEE
 * fp32 with round-to-nearest-even, rounded back to bf16 RNE; fp32: one IEEE
 * fp32 addition), by a persistent grid-stride kernel whose grid is capped at
 * 8 CTAs/SM x SMs / rc_div (rc_div 1, 2 or 4: GPU, GPU/2, GPU/4).
 *
 * Policies (goldy_corun_plan):
 *   GOLDY_PLAN_SEQUENTIAL  isolation-tuned GEMM kernel, then the add, one stream
 *   GOLDY_PLAN_DEFAULT     isolation-tuned GEMM kernel and the add (whole-GPU
 *                          grid) at once on two streams
 *   GOLDY_PLAN_GO          the table's CD-2 GO-Kernel and the add capped at
 *                          GPU/2, at once
 *   GOLDY_PLAN_AUTO        the configuration the table entry's flags record
 *                          (profiled: the fastest of running at once with the
 *                          CD-1 or CD-2 kernel and the op capped at GPU,
 *                          GPU/2 or GPU/4, taken only when it beats one after
 *                          the other by >= 5%), else SEQUENTIAL — concurrency
 *                          restricted where it does not pay.
 * The table's kernels are those of the GEMM's bucket (see goldy_lut_lookup). */
typedef struct goldy_ewise_desc {
  int64_t n;        /* elements (>= 0) */
  int32_t dtype;    /* GOLDY_BF16 or GOLDY_F32, for X, Y and Z */
  int32_t reserved; /* must be 0 */
} goldy_ewise_desc;
typedef struct goldy_corun goldy_corun;
goldy_status goldy_corun_plan(const goldy_gemm_desc* gemm, const goldy_ewise_desc* ew, const goldy_lut* lut,
                              int policy, goldy_corun** out);
/* concurrent: 1 if the two kernels run at once (needs 2 streams); the GEMM's
 * variant; the add's grid-cap divisor; device workspace bytes (split-K). */
goldy_status goldy_corun_query(const goldy_corun* c, int* concurrent, int* gemm_variant, int* add_rc_div,
                               size_t* workspace_bytes);
/* Enqueue: the GEMM C = A B on streams[0]; the add on streams[1] (forked
 * from and joined back into streams[0]) when concurrent, else on streams[0]
 * after the GEMM.  X, Y, Z: device arrays of n elements; the vector path
 * needs them 16-byte aligned (others take a scalar path).  Asynchronous. */
goldy_status goldy_corun_run(const goldy_corun* c, const void* A, const void* B, void* C, void* workspace,
                             size_t workspace_bytes, const void* X, const void* Y, void* Z, void* const* streams,
                             int n_streams);
/* The same, recorded once as a prepared run (see goldy_exec_create). */
goldy_status goldy_corun_exec_create(const goldy_corun* c, const void* A, const void* B, void* C, void* workspace,
                                     size_t workspace_bytes, const void* X, const void* Y, void* Z,
                                     void* const* streams, int n_streams, goldy_exec** out);
void goldy_corun_free(goldy_corun* c);

/* The element-wise add alone on one stream (rc_div 1, 2 or 4). */
goldy_status goldy_ewise_add(const void* X, const void* Y, void* Z, int64_t n, int dtype, int rc_div, void* stream);

/* ---- SM partitions (CU-Partition, Sec. 6.9; GPU-Quarter/Half, Sec. 7.4) -----------
 * A partition is a CUDA green context owning a subset of the GPU's SMs plus
 * n_streams (1 .. GOLDY_MAX_STREAMS) non-blocking streams in it; kernels
 * enqueued on those streams run on the partition's SMs only.  min_sms <= 0
 * or >= the device's SMs gives the whole device as a partition; otherwise the
 * driver rounds min_sms up to its partition granularity (query the actual
 * count).  Passing a partition's streams to goldy_run / goldy_run_ex /
 * goldy_exec_create / goldy_graph_create(_ex) / goldy_graph_launch runs the
 * schedule inside the partition: grid caps are computed from the partition's
 * SM count, and the library makes the partition's context current on the
 * calling thread for the duration of each call (device memory of the
 * device's primary context stays valid).  GOLDY_ERR_UNSUPPORTED if the
 * driver has no green contexts or cannot split off such a partition.  Free
 * every exec and graph that uses a partition before the partition. */
typedef struct goldy_partition goldy_partition;
goldy_status goldy_partition_create(int min_sms, int n_streams, goldy_partition** out);
/* SM count, and the first n (<= n_streams) streams (CUstream handles). */
goldy_status goldy_partition_query(const goldy_partition* p, int* sm_count, void** streams, int n);
void goldy_partition_free(goldy_partition* p);

/* Capture goldy_run(...) with these exact pointers into a CUDA graph, for
 * replay with one launch (the closest host-side analogue of the command
 * processor dispatching a whole set).  The streams must be idle.  The graph
 * owns copies of all launch parameters; the buffers must outlive it. */
goldy_status goldy_graph_create(const goldy_schedule* s, const void* const* A,
                                const void* const* B, void* const* C, void* workspace,
                                size_t workspace_bytes, void* const* streams, int n_streams,
                                goldy_graph** out);
/* goldy_graph_create with run options (event hooks captured into the graph). */
goldy_status goldy_graph_create_ex(const goldy_schedule* s, const void* const* A,
                                   const void* const* B, void* const* C, void* workspace,
                                   size_t workspace_bytes, void* const* streams, int n_streams,
                                   const goldy_run_opts* opts, goldy_graph** out);
/* Launch a captured graph on `stream` (asynchronous). */
goldy_status goldy_graph_launch(const goldy_graph* g, void* stream);
void goldy_graph_free(goldy_graph* g);

/* One GEMM with GO-Kernel variant `variant`, for callers that cannot allocate
 * device memory (the paper has no counterpart; this is a service of this
 * library).  goldy_run needs a caller workspace for split-K variants; callers
 * held to a fixed memory budget, plugins inside a framework that owns all
 * device allocations, and paths where cudaMalloc's implicit synchronisation
 * is unacceptable cannot provide one.  Here the split-K scratch is a fixed
 * 32 MiB device array compiled into the library (one per GPU that loads it,
 * held until exit); nothing is allocated.  Launches on `stream`
 * (cudaStream_t as void*, may be null; a stream of an SM partition runs the
 * GEMM inside the partition, as goldy_run does) and returns without
 * synchronising.  A, B, C, desc: as for goldy_run (16-byte aligned A and B).
 * Errors: GOLDY_ERR_INVALID_ARG for a bad descriptor, variant or pointer, or
 * when the GEMM would need more than the 32 MiB scratch (the message gives the
 * size); GOLDY_ERR_CUDA for a failed launch.  The first call on a device looks
 * up the scratch's device address (cudaGetSymbolAddress, which may load
 * device code) and keeps it for the life of the process: make that call
 * before any stream capture, and do not call this entry point on a device
 * after cudaDeviceReset.  All calls share the scratch: calls whose kernels
 * overlap on the GPU race and give wrong results, so serialise them (one
 * stream, or events). */
goldy_status goldy_gemm_noalloc(const goldy_gemm_desc* desc, int variant, const void* A,
                                const void* B, void* C, void* stream);

/* ---- a linear layer, plain or grouped by expert ---------------------------
 * The products of Y = act(X W + b) + R and of its backward pass, each one
 * kernel with the work around the product in its epilogue.  X is rows x in, W
 * is in x out, Y is rows x out, row-major; X, W and dY are bf16, products are
 * accumulated in fp32, and every result is rounded once, to nearest even.
 * (The tensor cores' fp32 accumulators truncate: about 1e-9 of the sum per
 * reduction element.  An accumulator takes at most 768 elements of an fp32
 * result and 8192 rows of a bf16 weight gradient over more than 65536; other
 * bf16 results keep the whole reduction in one.)
 *
 * groups = 0: one W for all rows.  groups = E >= 1: E experts with weights
 * W + e * stride_w and packed biases b + e * out; rows offsets[e] ..
 * offsets[e+1] - 1 belong to expert e.  offsets: E + 1 non-decreasing 32-bit
 * integers in device memory, read by the kernels (so they may be written by
 * an earlier kernel of the stream, and no host copy is needed).  Experts may
 * be empty; rows before offsets[0] and from offsets[E] on belong to none and
 * their results are left as they are.  Offsets are clamped to [0, rows], and
 * where they decrease the rows concerned are assigned in an unspecified way
 * (nothing outside the arrays is touched).
 *
 * Row strides are in elements; 0 stands for dense rows, which for bf16 are
 * padded to a multiple of 8 elements (16 bytes) and for fp32 are packed.
 * ldx: X; lddx: dX; ldw: W and dW; ldy: Y, dY and dZ; ldz: Z; ldr: R.  A
 * product reads X, W and dY in place where their row strides (and stride_w)
 * are multiples of 8, and they then start on 16-byte boundaries; other strides
 * cost a padded copy in the workspace.  Results, R, Z and biases need their
 * element's alignment only (bf16: faster accesses where base and row stride
 * are multiples of 4 bytes).  in, out and rows are arbitrary, 0 included (an empty
 * sum is 0).
 *
 * Results must not overlap inputs, except that R may be the result itself
 * (Y += ..., same stride). */
typedef enum goldy_act {
  GOLDY_ACT_NONE = 0,
  GOLDY_ACT_RELU = 1,       /* max(z, 0); slope 0 at 0 */
  GOLDY_ACT_GELU = 2,       /* z (1 + erf(z / sqrt 2)) / 2 */
  GOLDY_ACT_GELU_TANH = 3,  /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
  GOLDY_ACT_SILU = 4        /* z / (1 + exp(-z)) */
} goldy_act;

#define GOLDY_MAX_GROUPS 4096

typedef struct goldy_linear_desc {
  int64_t rows, in, out;
  int64_t ldx, lddx, ldw, ldy, ldz, ldr;
  int64_t stride_w;         /* elements between two experts' W (and dW); 0: in * ldw */
  int32_t groups;           /* 0, or experts 1 .. GOLDY_MAX_GROUPS */
  int32_t act;              /* goldy_act of this layer (forward, bias gradient) */
  int32_t act_x;            /* goldy_act that made X (input gradient) */
  int32_t y_dtype, dx_dtype, dw_dtype;   /* of Y, dX, dW (and of the R added to them) */
  int32_t bias_dtype;
  int32_t reserved;         /* must be 0 */
} goldy_linear_desc;

/* Device workspace that covers every call with this descriptor (host only; 0
 * if none is needed).  A workspace is 256-byte aligned and zero-filled by the
 * caller before its first use; its first 64 KiB are zero again after every
 * complete call.  One workspace of the largest size serves all layer
 * operators (these, goldy_layernorm_backward) of one stream; calls that may
 * overlap on the GPU need one each. */
goldy_status goldy_linear_query(const goldy_linear_desc* desc, size_t* workspace_bytes);

/* Y = act(X W + bias) + R.  bias and R may be null; Z (bf16, rows x out), if
 * not null, receives X W + bias for the backward pass (act uses the unrounded
 * value).  Asynchronous on `stream`, like all calls below: no allocation, no
 * synchronisation.  A stream of an SM partition runs the call inside the
 * partition.  Errors: GOLDY_ERR_INVALID_ARG, GOLDY_ERR_UNSUPPORTED (types),
 * GOLDY_ERR_NOMEM (workspace smaller than this call needs), GOLDY_ERR_CUDA; a
 * kernel that gave up a bounded wait shows up in goldy_device_error(), and
 * the workspace is then to be zero-filled again. */
goldy_status goldy_linear_forward(const goldy_linear_desc* desc, const int32_t* offsets, const void* X, const void* W,
                                  const void* bias, const void* R, void* Z, void* Y, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* dX = (dY W^T) * act_x'(Z) + R: the gradient of this layer's input, carried
 * through the activation that made X (X = act_x(Z); Z is bf16, rows x in, and
 * null exactly when act_x is GOLDY_ACT_NONE).  R (may be null) is a gradient
 * that reaches X another way. */
goldy_status goldy_linear_input_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* dY,
                                     const void* W, const void* Z, const void* R, void* dX, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* dW = X^T dY (per expert over its rows; 0 for an empty expert), added to
 * what dW holds when accumulate is 1. */
goldy_status goldy_linear_weight_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* X,
                                      const void* dY, void* dW, int accumulate, void* workspace,
                                      size_t workspace_bytes, void* stream);

/* db = sum of dZ over the rows (per expert; fp32, packed), dZ = dY * act'(Z).
 * Z null: dZ = dY and dZ is null too; otherwise dZ (bf16, stride ldy; may be
 * dY itself) is written: the gradient the other two calls take as their dY
 * when the layer has an activation that no later layer's input gradient has
 * gone through.  The sum takes dZ before it is rounded. */
goldy_status goldy_linear_bias_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* dY,
                                    const void* Z, void* dZ, float* db, int accumulate, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* ---- layer norm -------------------------------------------------------------
 * y = (x - mean) * rstd * gamma + beta per row of n elements, mean = sum(x) /
 * n, rstd = 1 / sqrt(sum((x - mean)^2) / n + eps), in fp32.  X, Y, dX and dY
 * share `dtype` (any row strides >= n, element alignment; ldx: X and dX, ldy:
 * Y and dY); gamma and beta have param_dtype and may be null (1 and 0).  The
 * aligned 16-byte blocks that a row begins and ends in may be read whole; only
 * rows are written. */
typedef struct goldy_layernorm_desc {
  int64_t rows, n;
  int64_t ldx, ldy;
  int32_t dtype;            /* GOLDY_BF16 or GOLDY_F32 */
  int32_t param_dtype;
  float eps;                /* >= 0 */
  int32_t reserved;         /* must be 0 */
} goldy_layernorm_desc;

/* Device workspace of the backward call (see goldy_linear_query; the forward
 * call needs none). */
goldy_status goldy_layernorm_query(const goldy_layernorm_desc* desc, size_t* workspace_bytes);

/* mean and rstd (fp32, one per row) may be null when no backward pass needs
 * them.  Y may be X itself. */
goldy_status goldy_layernorm_forward(const goldy_layernorm_desc* desc, const void* X, const void* gamma,
                                     const void* beta, void* Y, float* mean, float* rstd, void* stream);

/* dX; and dgamma, dbeta (fp32, n each, either may be null), added to what
 * they hold when accumulate is 1.  dX may be dY or X itself (same stride). */
goldy_status goldy_layernorm_backward(const goldy_layernorm_desc* desc, const void* dY, const void* X,
                                      const void* gamma, const float* mean, const float* rstd, void* dX,
                                      float* dgamma, float* dbeta, int accumulate, void* workspace,
                                      size_t workspace_bytes, void* stream);

/* ---- a router: experts and weights of each token ---------------------------
 * Of each row of `experts` logits the k largest are chosen, ties to the lowest
 * index (NaN counts as larger than any number, as it does in sorts).  An expert
 * whose logit is -infinity is closed to the row and never chosen; a slot for
 * which no open expert is left has id -1 and weight 0.  The weight of a chosen
 * expert e is
 *   GOLDY_ROUTER_ALL     scale * exp(l_e) / sum of exp(l) over all experts
 *   GOLDY_ROUTER_CHOSEN  scale * exp(l_e) / sum of exp(l) over the chosen ones
 * computed in fp32 from the logits less their largest; a row's results are the same
 * bits whatever the other rows hold.  Logits and dlogits have
 * `dtype`, any row strides >= experts, element alignment; ids (int32) and
 * weights (fp32) are packed rows x k.  Results must not overlap inputs unless
 * stated. */
typedef enum goldy_router_over { GOLDY_ROUTER_ALL = 0, GOLDY_ROUTER_CHOSEN = 1 } goldy_router_over;

#define GOLDY_MAX_SLOTS 32      /* experts per token */

typedef struct goldy_router_desc {
  int64_t rows;
  int64_t ld, ldd;          /* row strides of the logits and of dlogits */
  int32_t experts;          /* 1 .. GOLDY_MAX_GROUPS */
  int32_t k;                /* 1 .. min(experts, GOLDY_MAX_SLOTS) */
  int32_t dtype;            /* GOLDY_BF16 or GOLDY_F32 */
  int32_t over;             /* goldy_router_over */
  float scale;              /* finite */
  int32_t reserved;         /* must be 0 */
} goldy_router_desc;

/* ids and weights of every row, in falling order of the logits. */
goldy_status goldy_router_forward(const goldy_router_desc* desc, const void* logits, int32_t* ids, float* weights,
                                  void* stream);

/* dlogits (all of them; 0 for closed experts, and for all that were not chosen
 * under GOLDY_ROUTER_CHOSEN) from the gradient of the weights.  ids: as the
 * forward call gave them; a slot with an id out of range adds nothing, and an
 * expert that a row names twice takes both slots' gradients.  dlogits may be
 * the logits themselves (ldd = ld). */
goldy_status goldy_router_backward(const goldy_router_desc* desc, const void* logits, const int32_t* ids,
                                   const float* dweights, void* dlogits, void* stream);

/* ---- tokens sorted by expert, and back --------------------------------------
 * Token t has k slots, slot t * k + j with the expert ids[t * k + j].  Sorted by
 * expert (a slot's order within its expert is that of the slots), a slot's row
 * among the experts' rows is its place; the grouped products take the experts'
 * row ranges from the same offsets (goldy_linear_desc with rows = rows * k).  A
 * slot whose id is not in 0 .. groups - 1 belongs to no expert: its place is -1,
 * nothing is copied for it and it adds nothing.  Experts' rows from
 * offsets[groups] on are never read or written.
 *
 * Tokens' rows (X, Y, R, dY) and experts' rows (E, dE) have `dtype` and `width`
 * elements, any row strides >= width, element alignment; the aligned 16-byte
 * blocks that a row begins and ends in may be read whole, only rows are
 * written.  rows * k < 2^31.  A place that is not in 0 .. rows * k - 1 counts as -1; places
 * must otherwise differ.  Results must not overlap inputs unless stated. */
typedef struct goldy_route_desc {
  int64_t rows, width;
  int64_t ldx, lde, ldr;    /* row strides of tokens' rows (X, Y, dY), of experts' rows (E, dE), of R */
  int32_t k;                /* slots per token, 1 .. GOLDY_MAX_SLOTS */
  int32_t groups;           /* experts, 1 .. GOLDY_MAX_GROUPS */
  int32_t dtype;            /* GOLDY_BF16 or GOLDY_F32 */
  int32_t reserved;         /* must be 0 */
} goldy_route_desc;

/* Device workspace of goldy_route_sort (see goldy_linear_query; the other calls
 * need none). */
goldy_status goldy_route_query(const goldy_route_desc* desc, size_t* workspace_bytes);

/* offsets (groups + 1), place (rows * k) and, if not null, source (rows * k: the
 * slot whose place this is, -1 from offsets[groups] on).  All int32. */
goldy_status goldy_route_sort(const goldy_route_desc* desc, const int32_t* ids, int32_t* offsets, int32_t* place,
                              int32_t* source, void* workspace, size_t workspace_bytes, void* stream);

/* E[place of slot (t, j)] = X[t].  Its gradient is goldy_route_combine of dE
 * without weights. */
goldy_status goldy_route_dispatch(const goldy_route_desc* desc, const void* X, const int32_t* place, void* E,
                                  void* stream);

/* Y[t] = R[t] + sum over j of weights[t, j] * E[place of slot (t, j)], summed in
 * fp32 in the slots' order, R last.  weights (fp32, packed) and R may be null (1
 * and 0).  Y may be R (ldx = ldr). */
goldy_status goldy_route_combine(const goldy_route_desc* desc, const void* E, const int32_t* place,
                                 const float* weights, const void* R, void* Y, void* stream);

/* dE[place of slot (t, j)] = weights[t, j] * dY[t], dweights[t, j] = the dot
 * product of dY[t] and that row of E (0 for a slot without an expert).  dE may
 * be E.  dweights may be null (E is then not read and may be null), weights too
 * (1). */
goldy_status goldy_route_combine_grad(const goldy_route_desc* desc, const void* dY, const void* E,
                                      const int32_t* place, const float* weights, void* dE, float* dweights,
                                      void* stream);

/* ---- norms before and after a block ------------------------------------------
 * A block's output F joins the residual stream X through a norm of its own, a
 * gate and the stream's scale, and the next block's norm follows at once:
 *   S = alpha * X + gate * N_f(F),   Y = N_y(S)
 * with N(v) = (v - mean) * rstd * gamma + beta per row of n elements:
 *   GOLDY_NORM_NONE   N(v) = v
 *   GOLDY_NORM_LAYER  mean = sum(v) / n, rstd = 1 / sqrt(sum((v - mean)^2) / n + eps)
 *   GOLDY_NORM_RMS    mean = 0, rstd = 1 / sqrt(sum(v^2) / n + eps)
 * in fp32; Y is the norm of S before S is rounded.  X, F, S, Y and their
 * gradients share `dtype`, any row strides >= n, element alignment (the aligned
 * 16-byte blocks that a row begins and ends in may be read whole; only rows are
 * written).  gate, gamma and beta (n elements each) have param_dtype and may be
 * null (1, 1 and 0); those of a norm that is GOLDY_NORM_NONE must be. */
typedef enum goldy_norm_kind { GOLDY_NORM_NONE = 0, GOLDY_NORM_LAYER = 1, GOLDY_NORM_RMS = 2 } goldy_norm_kind;

typedef struct goldy_residual_norm_desc {
  int64_t rows, n;
  int64_t ldx, ldf, lds, ldy;   /* row strides: X and dX; F and dF; S and dS; Y and dY */
  int32_t dtype;                /* GOLDY_BF16 or GOLDY_F32 */
  int32_t param_dtype;
  int32_t norm_f, norm_y;       /* goldy_norm_kind */
  float eps;                    /* >= 0 */
  float alpha;                  /* finite */
  int32_t reserved;             /* must be 0 */
} goldy_residual_norm_desc;

/* Device pointers of the parameters (forward and backward), or of their
 * gradients (fp32; null: not wanted). */
typedef struct goldy_residual_norm_params {
  void* gate;
  void* gamma_f;
  void* beta_f;
  void* gamma_y;
  void* beta_y;
} goldy_residual_norm_params;

/* Device workspace of the backward call (see goldy_linear_query; the forward
 * call needs none). */
goldy_status goldy_residual_norm_query(const goldy_residual_norm_desc* desc, size_t* workspace_bytes);

/* params may be null (all absent).  Y is null exactly when norm_y is
 * GOLDY_NORM_NONE.  stats (fp32, 4 x rows: mean and rstd of N_f, mean and rstd of
 * N_y; those that a norm does not have are left as they are) may be null when no
 * backward pass needs them.  S and Y may each be X or F (same stride). */
goldy_status goldy_residual_norm_forward(const goldy_residual_norm_desc* desc, const goldy_residual_norm_params* params,
                                         const void* X, const void* F, void* S, void* Y, float* stats, void* stream);

/* dX and dF from dY (null exactly when norm_y is GOLDY_NORM_NONE) and dS, the
 * gradient that reaches S past N_y (may be null unless dY is); S and F as the
 * forward call read and left them.  grads (may be null): the parameters'
 * gradients, fp32, added to what they hold when accumulate is 1; a parameter
 * that is absent because it is 1 or 0 has one all the same.  dX and dF may each
 * be any of the four inputs (same stride).  The workspace is needed for grads. */
goldy_status goldy_residual_norm_backward(const goldy_residual_norm_desc* desc,
                                          const goldy_residual_norm_params* params, const void* dY, const void* dS,
                                          const void* F, const void* S, const float* stats, void* dX, void* dF,
                                          const goldy_residual_norm_params* grads, int accumulate, void* workspace,
                                          size_t workspace_bytes, void* stream);

/* ---- pre-activations kept in 8 bits --------------------------------------------
 * What a layer's backward pass needs of its pre-activation Z, in half the bytes
 * of bf16: each block of GOLDY_KEEP8_BLOCK elements of a row (the last one of a
 * row may be shorter) is held as e4m3 numbers q times a power of two 2^e, the
 * smallest that keeps the block's largest finite |z| within 448 * 2^e, at least
 * 2^-127; q = z / 2^e rounded to nearest even (relative error at most 2^-4 from
 * |z| = 2^(e-6) on, absolute error at most 2^(e-10) below).  An infinity or NaN
 * is held as NaN.  Q holds the blocks of a row one after another, each of
 * GOLDY_KEEP8_BLOCK bytes (zeros behind the row's end), rows packed: rows * blocks *
 * GOLDY_KEEP8_BLOCK bytes, 16-byte aligned; scales holds e + 127 per block, one
 * byte each, packed.  The aligned 16-byte blocks that a row of Z begins and ends in
 * may be read whole; of Z and H only rows are written.  No array may overlap another. */
#define GOLDY_KEEP8_BLOCK 32

typedef struct goldy_keep8_desc {
  int64_t rows, n;
  int64_t ldz, ldh;         /* row strides of Z and H, >= n */
  int32_t dtype;            /* of Z and H: GOLDY_BF16 or GOLDY_F32 (element alignment) */
  int32_t act;              /* goldy_act of H */
  int32_t reserved;         /* must be 0 */
} goldy_keep8_desc;

/* Bytes of Q and of scales (host only). */
goldy_status goldy_keep8_query(const goldy_keep8_desc* desc, size_t* q_bytes, size_t* scale_bytes);

/* Q and scales from Z. */
goldy_status goldy_keep8_pack(const goldy_keep8_desc* desc, const void* Z, void* Q, void* scales, void* stream);

/* Z = q * 2^e (exact but for a bf16 or fp32 underflow) and H = act(Z), of the
 * value before any rounding; either may be null: the backward pass takes Z for
 * the activation's gradient (goldy_linear_input_grad) and H for the weight
 * gradient of the layer that read it. */
goldy_status goldy_keep8_unpack(const goldy_keep8_desc* desc, const void* Q, const void* scales, void* Z, void* H,
                                void* stream);

/* Error word the kernels set when a bounded wait gives up (0 = none; the
 * first failure wins): 1 a load-role wait, 2 an MMA-thread wait, 3 an
 * epilogue wait, 4 a split-K cluster-exchange wait.  Reads it synchronously
 * on the current device and, if `clear`, resets it.  After a non-zero code,
 * zero-fill the workspace of the failed run before reusing it (goldy_run). */
goldy_status goldy_device_error(int* code, int clear);

/* SM count and CTAs of variant `variant_id` resident per SM on the current
 * device (occupancy query, no launch). */
goldy_status goldy_device_info(int variant_id, int* sm_count, int* ctas_per_sm);

#ifdef __cplusplus
}
#endif

#endif /* GOLDY_H_ */
