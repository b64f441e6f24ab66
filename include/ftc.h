/*
 * ftc.h -- C ABI of the batched executor for the correction-based fault-tolerant
 * reduce and allreduce (Kuettler & Haertig, "Fault-tolerant Reduce and Allreduce
 * operations based on correction").
 *
 * The library plays the paper's message schedule for S independent scenarios at once
 * on one NVIDIA B200 (sm_100a). A scenario is one input vector of k elements for each
 * of P logical processes plus a failure pattern; the result is the value the root
 * (reduce) or every surviving process (allreduce) ends up with, and a status record.
 *
 * Conventions for every entry point
 *   - plain C linkage, no exceptions, no global state (except where an entry point
 *     says otherwise); pointers named d_* are DEVICE pointers, h_* HOST pointers;
 *   - the caller owns every buffer and the stream; inputs are read-only; the library
 *     allocates nothing and never synchronises the host unless stated;
 *   - work is enqueued on `cuda_stream` (a cudaStream_t passed as void*, NULL = the
 *     default stream) and is complete when that stream has drained;
 *   - the return value reports call-level errors only (0 = FTC_OK, negative = error,
 *     see ftc_strerror). What happens inside a scenario (failed root, no failure-free
 *     subtree, ...) is not an error: it is written to that scenario's status record.
 *
 * Readings of the paper that fix the schedule (the paper leaves them open):
 *   - the root swaps numbers with process 0 (section "Reduce"); all rules below apply
 *     to the renumbered ranks v;
 *   - up-correction group of v >= 1 is floor((v-1)/(f+1)); the root joins the last
 *     group iff that group is short (section "Up-Correction"); partners are visited in
 *     ascending rank, the root first;
 *   - v >= 1 lies below root child s = (v-1) mod (f+1) (proof of the first theorem of
 *     section "Properties"); within a subtree the nodes j = floor((v-1)/(f+1)) form a
 *     heap, binary unless FTC_TREE_ARITY(a) in the flags asks for a children per node: children a*j+1 .. a*j+a,
 *     received in that order, accumulator on the left (the paper's I(f)-tree fixes only the root's f+1 children
 *     and their subtree sizes; heaps of other arities and binomial trees run on the level kernel in shared memory
 *     where their shape fits it, else on the general kernel, which needs its workspace);
 *   - failure information is the single failed bit (third scheme of section "Failure
 *     information"); the root takes the lowest-numbered child that delivered with the
 *     bit clear (Algorithm "reduce_root");
 *   - rounds: up-correction iteration i is round i (0..f-1); a node at depth d sends up
 *     the tree in round f+H-d, H = 1+floor(log2(ceil((P-1)/(f+1)))); one reduce has
 *     f+H rounds. The broadcast of the allreduce sends down the same tree (depth d in
 *     round f+H+d) and then lets every process the tree reached send the value to its
 *     up-correction partners (iteration i in round f+2H+i); one allreduce attempt has
 *     2(f+H) rounds and attempt a starts at round a*2(f+H). A process with failure
 *     round t performs exactly the sends scheduled in rounds < t;
 *   - allreduce root candidates are first, first+1, ... (mod P), f+1 of them
 *     (Algorithm "Allreduce"; "at least f+1 processes must eventually be tried").
 */
#ifndef FTC_H
#define FTC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define FTC_API __attribute__((visibility("default")))
#else
#define FTC_API
#endif

#define FTC_VERSION 0x00010000u

/* element types and reduction functions (section "Reduce": associative and commutative) */
enum { FTC_I32 = 0, FTC_I64 = 1, FTC_U64 = 2, FTC_F32 = 3,
       FTC_BF16 = 4, FTC_F16 = 5 };           /* the training operators below only; the batch calls refuse them */
enum { FTC_SUM = 0, FTC_MAX = 1, FTC_XOR = 2 };   /* integer sums wrap; FTC_F32 supports FTC_SUM only */

/* call-level return codes */
enum {
    FTC_OK = 0,
    FTC_EINVAL = -1,        /* P < f+2, k = 0, root >= P, NULL or misaligned required pointer, f > 31, max_inop > 32, tree arity 1 or > 32 */
    FTC_EUNSUPPORTED = -2,  /* unknown dtype/op, xor or max on f32, expanded output for so many processes that its bitmasks
                               exceed shared memory */
    FTC_EWORKSPACE = -3,    /* workspace missing or smaller than ftc_workspace_bytes() */
    FTC_ECUDA = -4,         /* a CUDA call or launch failed */
    FTC_ETOOLARGE = -5      /* ftc_reduce_batch_noalloc: the shape does not fit the built-in scratch */
};

/* per-scenario outcome, low byte of status word 0 */
enum {
    FTC_ST_OK = 0,
    FTC_ST_ROOT_FAILED = 1,             /* reduce to a failed root is a no-op (section "Semantics") */
    FTC_ST_NO_CLEAN_SUBTREE = 2,        /* Algorithm "reduce_root": "No failure-free subtree" (needs > f failures) */
    FTC_ST_NO_LIVE_ROOT_CANDIDATE = 3,  /* allreduce: all f+1 candidates had failed before the operation */
    FTC_ST_PRECONDITION_INOP_ROOT = 4,  /* allreduce: a root candidate is listed as failing in-operation */
    FTC_ST_BAD_ROOT = 5,                /* d_roots[s] >= P */
    FTC_ST_INTERNAL_TIMEOUT = 6         /* a bounded wait for a copy inside the kernel ran out: this scenario and every later one
                                           that the same thread block plays report this outcome; results are zero bytes */
};

/*
 * Status record, FTC_STATUS_WORDS uint32 per scenario:
 *   word 0: outcome | selected root child (0..f, 0xFF none) << 8 | attempts used << 16
 *   word 1: number of processes whose input is included in the result
 *   word 2: bit i set = the victim of in-operation slot i is included in the result
 *   word 3: allreduce: processes that are alive at the end and hold the result; reduce: 0
 * When the outcome is not FTC_ST_OK words 1..3 are 0 and the result is all zero bytes.
 */
#define FTC_STATUS_WORDS 4

/* An in-operation failure: `victim` performs exactly the sends scheduled in rounds < `round`.
 * victim = FTC_INOP_UNUSED marks an empty slot; a victim that is also pre-failed counts as pre-failed;
 * round 0 is the same as a pre-operation failure. (Sections "Introduction", "Failures".) */
typedef struct { uint32_t victim; uint32_t round; } ftc_inop_t;
#define FTC_INOP_UNUSED 0xFFFFFFFFu
#define FTC_MAX_INOP 32u
#define FTC_MAX_F 31u

/* flags */
#define FTC_OUT_EXPANDED   0x1u   /* allreduce: d_out is [S][P][k], zeros for processes that do not hold the result */
#define FTC_TREE_ARITY(a)  (((uint32_t)(a) & 0xFFu) << 16)  /* subtrees below the root's children are a-ary heaps, 2 <= a <= FTC_MAX_ARITY (not given: binary) */
#define FTC_MAX_ARITY 32u
#define FTC_TREE_BINOMIAL   0x1000000u /* subtrees below the root's children are binomial trees on the local index j: parent of j =
                                         j without its lowest set bit, children in ascending order, depth = 1 + set bits of j
                                         (not together with FTC_TREE_ARITY) */
#define FTC_PARTNERS_DESCENDING 0x2000000u /* up-correction (and the broadcast's correction) visits the group partners in descending
                                            rank, the root last, instead of ascending with the root first: the algorithm leaves the
                                            order open (every kernel plays it) */
#define FTC_KERNEL_GENERIC 0x100u /* force the general level-by-level kernel (needs the workspace) */
#define FTC_KERNEL_LEVELS  0x400u /* binary heaps: take the level kernel (shared-memory tiles evaluated level by level), which heaps of
                                     arity 3 and more and binomial trees use by default, where the shape allows it */
#define FTC_KERNEL_DIRECT  0x200u /* force the register-tiled kernel (direct global loads) where the shape allows it */
#define FTC_DEBUG_ONE_POLL 0x4000000u /* testing aid: the kernel's bounded waits for its asynchronous copies look once instead of
                                         polling, so most of them give up and the give-up path runs: affected scenarios report
                                         FTC_ST_INTERNAL_TIMEOUT with zero bytes, nothing waits without a limit and nothing is read
                                         or written out of bounds. Never set it in production calls */

typedef struct {
    uint32_t P;         /* processes, P >= f+2 (the root needs f+1 children: definition of the I(f)-tree) */
    uint32_t f;         /* failures to tolerate, 0..31; up-correction groups have f+1 members */
    uint32_t k;         /* elements per process */
    uint32_t dtype;     /* FTC_I32 ... */
    uint32_t op;        /* FTC_SUM ... */
    int32_t  root;      /* >= 0: root (reduce) / first root candidate (allreduce) of every scenario; -1: d_roots[s] */
    uint32_t max_inop;  /* in-operation slots per scenario in d_inop, 0..32 */
    uint32_t flags;
} ftc_desc_t;

/* Schedule constants under the readings above and the failure-free message counts of the theorem on the
 * number of messages (section "Properties"). */
typedef struct {
    uint32_t q, r;              /* full groups, size of the short last group without the root: P-1 = q(f+1)+r */
    uint32_t H;                 /* depth of the deepest node */
    uint32_t rounds_reduce;     /* f+H */
    uint32_t rounds_attempt;    /* 2(f+H): reduce plus broadcast */
    uint64_t msgs_upcorrection; /* f(f+1)q + a(a-1), a = r+1 */
    uint64_t msgs_tree;         /* P-1 */
} ftc_sched_t;

/*
 * Corrected reduce (Algorithms "Up-correction", "reduce_root", "reduce_non_root", "reduce") for S scenarios.
 *   d_in      [S][P][k] elements of desc->dtype, process order as the caller numbers them; 16-byte aligned
 *   d_prefail [S][ceil(P/32)] uint32, bit p of a scenario's words set = process p failed before the operation
 *   d_inop    [S][max_inop] or NULL when max_inop = 0
 *   d_roots   [S] or NULL; read only when desc->root < 0
 *   d_out     [S][k]: the value delivered at the root (zeros unless the outcome is FTC_ST_OK); 16-byte aligned
 *   d_status  [S][FTC_STATUS_WORDS] uint32; 16-byte aligned (one record is stored as one 16-byte word)
 *   d_workspace, workspace_bytes: scratch of at least ftc_workspace_bytes(desc, S, 0) bytes (may be NULL if that is 0),
 *             16-byte aligned; contents are undefined afterwards; calls that share a workspace must not overlap on
 *             the device. Shapes that run on the shared-memory kernels also run with less or none (large process
 *             counts with wide vectors then more slowly); shapes that need the general kernel get FTC_EWORKSPACE
 * S = 0 is valid and does nothing. Returns FTC_OK or an error before anything is enqueued.
 */
FTC_API int ftc_reduce_batch(const ftc_desc_t* desc, uint64_t S, const void* d_in, const uint32_t* d_prefail,
                     const ftc_inop_t* d_inop, const uint32_t* d_roots, void* d_out, uint32_t* d_status,
                     void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Corrected allreduce (Algorithm "Allreduce": reduce to a root candidate, broadcast from it, next candidate if
 * it had failed before the operation). Arguments as for ftc_reduce_batch; desc->root / d_roots give the first
 * candidate. d_out is [S][k] (the value every holder has) or, with FTC_OUT_EXPANDED, [S][P][k]: the value in the
 * slot of every process that is alive at the end and holds it, zero bytes in all other slots. The expanded form
 * needs ftc_workspace_bytes() of 256-byte aligned workspace (the compact results pass through it); the host-buffer
 * variants and ftc_reduce_batch do not offer it (FTC_EUNSUPPORTED).
 */
FTC_API int ftc_allreduce_batch(const ftc_desc_t* desc, uint64_t S, const void* d_in, const uint32_t* d_prefail,
                        const ftc_inop_t* d_inop, const uint32_t* d_roots, void* d_out, uint32_t* d_status,
                        void* d_workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Corrected reduce for callers that cannot give the library any scratch memory and cannot allocate it either.
 * (The paper has no counterpart to this entry point: it exists for the sake of the host program, not the method.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- inside a latency-critical loop, where an
 * allocation's implicit device-wide synchronisation would stall unrelated streams; inside a plug-in or callback
 * of another framework that owns the memory budget and hands out no allocator; or after start-up in a service
 * whose device memory is fully accounted for. ftc_reduce_batch wants a caller-provided workspace for shapes that
 * run on the general kernel; this variant needs none.
 *
 * How: the general kernel's per-block node values go to an array of FTC_NOALLOC_SCRATCH_BYTES bytes that is part
 * of the library image. Every GPU that loads the library holds that array until the process exits. The call
 * allocates nothing (no cudaMalloc, cudaFree or allocating library routine), results and status records are
 * identical to ftc_reduce_batch's, and it is slower when fewer blocks than usual fit into the array.
 *   - Limit: one block's slice, ceil((P-1)/(f+1)) * k * element size bytes, must fit the array; otherwise
 *     FTC_ETOOLARGE is returned and nothing is enqueued.
 *   - The first call on each device looks the array's device address up (one runtime query, with that device
 *     current) and keeps it for the life of the process. Make that first call before starting any stream capture
 *     on that device. The address belongs to the device's primary context: a host program that destroys that
 *     context (cudaDeviceReset) must not call this entry point on that device afterwards.
 *   - All calls on a device share the one array, which keeps whatever the previous call left in it. Nothing in it
 *     needs clearing: within a scenario every slot is written before it is read. But two calls whose kernels can
 *     overlap on the same GPU (different streams, or different host threads) race on it: serialise them.
 * Arguments and all other rules as for ftc_reduce_batch, without the workspace pair. The always-general kernel
 * is used whatever the shape.
 */
#define FTC_NOALLOC_SCRATCH_BYTES (8u << 20)
FTC_API int ftc_reduce_batch_noalloc(const ftc_desc_t* desc, uint64_t S, const void* d_in, const uint32_t* d_prefail,
                                     const ftc_inop_t* d_inop, const uint32_t* d_roots, void* d_out,
                                     uint32_t* d_status, void* cuda_stream);

/*
 * What the root receives from each of its f+1 children (Algorithm "reduce_root": "receive from any child (data,
 * failure information)"; section "Failure information", second and third scheme), for S scenarios. The batch calls
 * above evaluate only the child the root selects; this call plays all f+1 subtrees, nodes that deliver nothing
 * included. is_allreduce != 0: the reduce of the allreduce attempt that counts (the last one if no candidate is alive).
 *   d_cand      [S][f+1][k]: the value child s delivers (zeros if it delivers nothing); 16-byte aligned
 *   d_cand_info [S][f+1][2] uint32: [0] 0 = delivered with the failed bit clear, 1 = delivered with the failed bit set,
 *               2 = nothing delivered, 3 = a bounded wait inside the kernel ran out (no value; as FTC_ST_INTERNAL_TIMEOUT);
 *               [1] size of the list of failed processes that came with the value
 *   workspace of at least ftc_candidates_workspace_bytes(desc, S) bytes, 256-byte aligned
 * Other arguments as for ftc_reduce_batch. Scenarios whose root is invalid or violates the allreduce precondition
 * play no attempt: zeros and "nothing delivered".
 * Two kernels (ftc_candidates_kernel_name): "staged" on binary heaps with vectors of 16..512 bytes (a power-of-two number of
 * 16-byte chunks) and scenarios above 12 KB -- one pass over the inputs on the tiles of the shared-memory kernel; for the
 * exactly associative operations (integer sum, max, xor) a group without a failed member is folded once for all children,
 * for float32 every child's member folds in its own order from the staged copy; "generic" (any k, other subtree shapes,
 * FTC_KERNEL_GENERIC) plays child after child.
 */
FTC_API int ftc_candidates_batch(const ftc_desc_t* desc, uint64_t S, int is_allreduce, const void* d_in,
                                 const uint32_t* d_prefail, const ftc_inop_t* d_inop, const uint32_t* d_roots,
                                 void* d_cand, uint32_t* d_cand_info, void* d_workspace, size_t workspace_bytes,
                                 void* cuda_stream);
FTC_API size_t ftc_candidates_workspace_bytes(const ftc_desc_t* desc, uint64_t S);
FTC_API const char* ftc_candidates_kernel_name(const ftc_desc_t* desc);

/*
 * The list of failed processes that the root holds when it delivers (section "Failure information", first scheme:
 * in the up-correction phase and in the tree phase every process appends the ids of the processes it could not
 * receive a value from; the lists travel up the tree with the values; "the root receives a complete list of failed
 * processes from each child ... that does not contain a failed process in the subtree spanned by it"). It is the list
 * that came with the value of the child the root selected, plus, when that child's subtree holds no member of the
 * root's own up-correction group, what the root noted itself. Under in-operation failures it lists exactly the
 * processes whose input is not part of the delivered result. is_allreduce != 0: the reduce of the attempt that counts.
 *   d_failed [S][ceil(P/32)] uint32: bit p of a scenario's words set = process p (the caller's numbering) is on the list
 *   d_nfail  [S] uint32: the size of the list (the second scheme sends only this); equals the number of set bits,
 *            since concatenated lists come from disjoint sets
 * Scenarios whose outcome is not FTC_ST_OK deliver nothing: all zero. Only the failure pattern is read; desc->k, dtype
 * and op must be valid but do not matter. Other arguments as for ftc_reduce_batch. No workspace.
 */
FTC_API int ftc_failed_list_batch(const ftc_desc_t* desc, uint64_t S, int is_allreduce, const uint32_t* d_prefail,
                                  const ftc_inop_t* d_inop, const uint32_t* d_roots, uint32_t* d_failed, uint32_t* d_nfail,
                                  void* cuda_stream);

/*
 * Messages sent in each scenario (theorem on the number of messages of the reduce and theorem on the messages of
 * the allreduce, section "Properties": failure-free f(f+1)q + a(a-1) up-correction and P-1 tree messages; no
 * process sends more when processes fail; an allreduce whose first candidates had failed repeats the reduce).
 * A message counts when its sender performs the send, whether or not the receiver is alive (section "Failures":
 * a send to a failed process completes). Only the failure pattern is read; desc->k, dtype and op must be valid
 * but do not matter.
 *   d_msgs [S][FTC_MSG_WORDS] uint64, 8-byte aligned:
 *     [0..3] over all attempts that are played: up-correction, tree, tree-down (broadcast), correction (broadcast)
 *     [4..7] the same four for the last attempt alone
 *   A reduce plays one attempt and has no broadcast ([2], [3], [6], [7] are 0), also when its root has failed
 *   (the others still send). An allreduce plays one attempt per root candidate up to the first one that had not
 *   failed before the operation; only that candidate broadcasts, and only if it found a failure-free subtree.
 *   Scenarios with outcome FTC_ST_BAD_ROOT or FTC_ST_PRECONDITION_INOP_ROOT play nothing: all zero.
 *   The broadcast numbers rest on this library's reading of the broadcast (see the top of this file), which the
 *   paper does not define.
 * Other arguments as for ftc_reduce_batch. No workspace.
 */
#define FTC_MSG_WORDS 8
FTC_API int ftc_message_counts_batch(const ftc_desc_t* desc, uint64_t S, int is_allreduce, const uint32_t* d_prefail,
                                     const ftc_inop_t* d_inop, const uint32_t* d_roots, uint64_t* d_msgs,
                                     void* cuda_stream);

/* Scratch bytes ftc_reduce_batch / ftc_allreduce_batch want for this descriptor and batch size: the general kernel's
 * node values, the compact results of the expanded output, and for many processes with wide vectors the shared-memory
 * kernel's array of tile results (0 otherwise). Returns 0 for an invalid descriptor as well; the batch calls report that. */
FTC_API size_t ftc_workspace_bytes(const ftc_desc_t* desc, uint64_t S, int is_allreduce);

/*
 * Same operations with HOST buffers (h_* as the d_* above): copies the inputs to the device in chunks, runs the
 * kernels, copies results and status back, all on `cuda_stream`, then synchronises that stream before returning.
 * d_staging is device scratch of at least ftc_host_staging_bytes(desc, 1) bytes; larger staging means larger
 * chunks. Pinned host memory makes the copies asynchronous but is not required.
 */
FTC_API int ftc_reduce_batch_host(const ftc_desc_t* desc, uint64_t S, const void* h_in, const uint32_t* h_prefail,
                          const ftc_inop_t* h_inop, const uint32_t* h_roots, void* h_out, uint32_t* h_status,
                          void* d_staging, size_t staging_bytes, void* cuda_stream);
FTC_API int ftc_allreduce_batch_host(const ftc_desc_t* desc, uint64_t S, const void* h_in, const uint32_t* h_prefail,
                             const ftc_inop_t* h_inop, const uint32_t* h_roots, void* h_out, uint32_t* h_status,
                             void* d_staging, size_t staging_bytes, void* cuda_stream);
/* Device staging bytes for chunks of `chunk_scenarios` scenarios (inputs, masks, outputs and workspace). */
FTC_API size_t ftc_host_staging_bytes(const ftc_desc_t* desc, uint64_t chunk_scenarios);

/* Schedule constants and failure-free message counts for (P, f) of the descriptor. FTC_EINVAL if P < f+2. */
FTC_API int ftc_schedule_info(const ftc_desc_t* desc, ftc_sched_t* out);

/*
 * Synthetic scenario inputs on the device (not part of the paper's method): element (s, p, e) of scenario
 * first_scenario+s is a function of (seed, scenario, p, e) only -- the splitmix64 output function applied to
 * seed + 0x9E3779B97F4A7C15 * (counter+1) -- mapped to one of the value kinds
 *   0 int32 in [-2^20, 2^20]   1 int64 in [-2^40, 2^40]   2 float32, sum of twelve 32-bit uniforms (six counters per
 *   element) centred, rounded to float32 once and scaled to unit variance: close to N(0,1), full mantissas
 *   3 int32 full range         4 uint64 full range
 * d_out is [S][P][k] of the kind's type. Returns FTC_OK, FTC_EINVAL (unknown kind, NULL) or FTC_ECUDA.
 */
FTC_API int ftc_fill_inputs(uint32_t kind, uint64_t seed, uint64_t first_scenario, uint64_t S, uint32_t P, uint32_t k,
                    void* d_out, void* cuda_stream);

/*
 * Measurement aid (not part of the paper's method): reads `bytes` bytes (a multiple of 16 KiB) at d_buf (16-byte
 * aligned) once and does nothing else. mode 0: 128-bit loads folded with xor in registers; mode 1: asynchronous bulk
 * copies into shared memory, the way the batch kernels stage their inputs. Timed over the buffer a batch call reads,
 * it gives the bandwidth a read-only kernel can reach on this GPU (a copy benchmark reads and writes).
 * d_sink: two uint64 words, zeroed by the caller; word 1 counts warps whose bounded wait for a copy gave up (0 in a valid run).
 */
FTC_API int ftc_read_bandwidth_probe(uint32_t mode, const void* d_buf, uint64_t bytes, uint64_t* d_sink, void* cuda_stream);

/* Name of the kernel family the batch calls would use for this descriptor: "staged", "tiled" or "generic". */
FTC_API const char* ftc_kernel_name(const ftc_desc_t* desc, int is_allreduce);

/* The same, down to the instantiation of the shared-memory kernel: "staged/warp" (scenarios of a few KB: one warp per
 * scenario), "staged/warp-pair" (two scenarios per warp, half a warp each), "staged/whole" (scenario staged by one copy),
 * "staged/lean" (blocks of one or two warps), "staged/large" (4-8 warps), "staged/batched-lean" (4-8 warps, groups of at
 * most 128 bytes, exact operations), "staged/lean-swz" and "staged/batched-swz" (float32 vectors of 16 or 32 bytes, tiles
 * by swizzled tensor copies), "staged/whole-large", "tiled", "generic"; assuming the workspace ftc_workspace_bytes() asks for. */
FTC_API const char* ftc_kernel_variant(const ftc_desc_t* desc, int is_allreduce);

/* Thread blocks the batch calls would launch for S scenarios on the current device (given the workspace
 * ftc_workspace_bytes() asks for). Block b plays scenarios b, b + blocks, b + 2*blocks, ... one after the other (the warp
 * kernel for scenarios of a few KB hands out short runs of consecutive scenarios the same way); a batch keeps the whole
 * GPU busy when S is a few times this number. Needs a device. Launches nothing. */
FTC_API int ftc_launch_blocks(const ftc_desc_t* desc, uint64_t S, int is_allreduce, uint32_t* blocks);

/*
 * Training operators around the collectives (not part of the paper's method): the operators of a data-parallel training
 * step that make the messages a corrected allreduce sends, and that consume what it delivers together with the status
 * records. All arithmetic is in float32 whatever the element types; sums over long axes keep float32 or float64 partial
 * sums in a fixed order (no atomic additions: the same call on the same GPU model gives the same bits).
 *
 * Layer norm over rows of H elements, as P processes of a data-parallel job see it.
 */
typedef struct {
    uint32_t H;         /* elements of a row, 1 .. 2^24 */
    uint32_t P;         /* processes the rows are divided over (backward), 1 .. 2^20; 1: the ordinary weight gradient */
    uint32_t k;         /* elements of a message (backward), 1 .. 2^24: the weight gradients are [ceil(H/k)][P][k]; k = H and P = 1:
                           [H]; (H + k) * P at most 2^35 */
    uint32_t dtype;     /* x, y, dy, dx: FTC_F32, FTC_BF16 or FTC_F16 */
    uint32_t wdtype;    /* gamma, beta: FTC_F32 or dtype */
    float    eps;       /* >= 0 */
} ftc_norm_t;

/*
 * y = (x - mean) * rstd * gamma + beta with mean = sum(x) / H, rstd = 1 / sqrt(sum((x - mean)^2) / H + eps), for each row.
 *   d_x     [rows] rows of H elements, row r at element r * x_stride; d_y likewise (x_stride, y_stride >= H); d_y may be d_x
 *           (with the same stride)
 *   d_gamma, d_beta  [H] of wdtype; NULL: ones, zeros
 *   d_mean, d_rstd   [rows] float32 for the backward pass; either may be NULL
 * rows is at most 2^31. Pointers are aligned to their element size; rows that begin on 16-byte boundaries (pointer and stride) with H a multiple
 * of 16 bytes are the fast case. rows = 0 is valid and does nothing. FTC_EUNSUPPORTED: another dtype or wdtype.
 */
FTC_API int ftc_layernorm_forward(const ftc_norm_t* desc, uint64_t rows, const void* d_x, uint64_t x_stride, const void* d_gamma,
                                  const void* d_beta, void* d_y, uint64_t y_stride, float* d_mean, float* d_rstd, void* cuda_stream);

/*
 * Gradients of the above. With xh = (x - mean) * rstd and a = dy * gamma:
 *   dx = rstd * (a - sum(a)/H - xh * sum(a * xh)/H) for each row, dgamma = sum of dy * xh and dbeta = sum of dy over the rows
 *   that a process holds.
 *   d_mean, d_rstd  [rows], as the forward pass left them
 *   d_row_splits    [P+1] uint64, ascending: process p holds rows d_row_splits[p] .. d_row_splits[p+1]-1 (values beyond `rows`
 *                   count as `rows`; none: its gradients are zero). NULL: process p holds rows p*rows/P .. (p+1)*rows/P-1
 *   d_dx            rows of H elements, or NULL; may be d_dy or d_x (with the same stride)
 *   d_dgamma, d_dbeta  float32 [ceil(H/k)][P][k] -- the inputs of ceil(H/k) scenarios for ftc_allreduce_batch (FTC_F32, FTC_SUM):
 *                   column h of process p is element h % k of message h / k; the last message is filled up with zeros; NULL: not
 *                   computed
 *   d_workspace     ftc_layernorm_workspace_bytes(desc, rows) bytes (may be NULL when neither weight gradient is wanted), 16-byte
 *                   aligned; contents are undefined afterwards; calls that share a workspace must not overlap on the device
 * rows = 0 writes zeros to the weight gradients.
 */
FTC_API int ftc_layernorm_backward(const ftc_norm_t* desc, uint64_t rows, const void* d_dy, uint64_t dy_stride, const void* d_x,
                                   uint64_t x_stride, const void* d_gamma, const float* d_mean, const float* d_rstd,
                                   const uint64_t* d_row_splits, void* d_dx, uint64_t dx_stride, float* d_dgamma, float* d_dbeta,
                                   void* d_workspace, size_t workspace_bytes, void* cuda_stream);
FTC_API size_t ftc_layernorm_workspace_bytes(const ftc_norm_t* desc, uint64_t rows);   /* 0 for an invalid descriptor */

/*
 * Many tensors at once: a table of a model's tensors, built on the host, kept by the caller on the host and (a copy) on the
 * device, and given to the calls below. Each call is one pass over all tensors.
 */
typedef struct {
    void* param;                /* [n] of param_dtype: the weights (may be NULL in tables that only ftc_grad_norm gets) */
    float* master;              /* [n]: the weights in 32 bits, which the update works on; param is then the rounded copy, written
                                   only. NULL: param itself is updated (rounded to nearest) */
    const void* grad;           /* [n] of grad_dtype: the gradient, or (with status) the sums that an allreduce delivered, its d_out
                                   [ceil(n/k)][k] of which the first n elements count */
    const uint32_t* status;     /* [ceil(n/k)][FTC_STATUS_WORDS]: the status records of those messages, 16-byte aligned. The gradient
                                   is the sum divided by the processes included in it; a message with another outcome than FTC_ST_OK
                                   (or nobody included) was not delivered: its elements keep their weights and 32-bit states and count
                                   nothing in the norm. NULL: the gradient is taken as it is */
    uint64_t n;                 /* elements, 0 .. 2^40 */
    uint32_t k;                 /* elements of a message, 1 .. 2^30; read only with status */
    uint32_t param_dtype;       /* FTC_F32, FTC_BF16, FTC_F16 */
    uint32_t grad_dtype;
    float    lr_scale;          /* this tensor's learning rate is lr * lr_scale */
    float    weight_decay;
    uint32_t reserved;          /* 0 */
} ftc_param_t;

#define FTC_STATE_BLOCK 256u    /* the optimizer states are laid out in blocks of so many elements of one tensor: tensor i begins at
                                   the sum of ceil(n/256) over the tensors before it (in blocks), its last block filled up */

FTC_API size_t ftc_param_table_bytes(const ftc_param_t* h_params, uint32_t n_params);  /* 0 for invalid entries */
/* Checks the entries and writes the table to h_table (8-byte aligned host memory of that many bytes). The caller copies it to
 * the device as it is (256-byte aligned); it holds the tensors' addresses, so tensors that move need a new table.
 * FTC_EINVAL: NULL grad with n > 0, misaligned pointers (element size), k = 0 with status, n or n_params out of range. */
FTC_API int ftc_param_table_build(const ftc_param_t* h_params, uint32_t n_params, void* h_table, size_t table_bytes);
/* Blocks of FTC_STATE_BLOCK elements that the table's tensors take up; 0 for anything that is no table. */
FTC_API uint64_t ftc_param_table_blocks(const void* h_table);

/*
 * The 2-norm of all gradients together, the factor that clips it, and the norm of each tensor's gradient.
 *   d_norm   [2] float32: the norm over all tensors; max_norm / norm where the norm exceeds max_norm, else 1, NaN where the norm is
 *            not finite (which makes ftc_adamw_step do nothing)
 *   d_norms  [n_params] float32: each tensor's norm, or NULL
 *   d_workspace  ftc_grad_norm_workspace_bytes(h_table) bytes, 16-byte aligned; as for ftc_layernorm_backward
 * Squares of eight elements are added in float32 (in float64 where that would overflow or lose small ones), their sums in float64.
 * max_norm > 0 (infinity: no clipping).
 */
FTC_API int ftc_grad_norm(const void* h_table, const void* d_table, float max_norm, float* d_norm, float* d_norms,
                          void* d_workspace, size_t workspace_bytes, void* cuda_stream);
FTC_API size_t ftc_grad_norm_workspace_bytes(const void* h_table);

/* One AdamW step (decoupled weight decay). */
typedef struct {
    double lr, beta1, beta2, eps;   /* lr >= 0, 0 <= beta < 1, eps >= 1e-30; lr finite and the betas below 1 as float32 too. A beta near
                                       1 and its state in float32 leave the state within about 1e-7 / (1 - beta) of itself: 0.01 %
                                       at 0.999, 1 % at 0.99999 */
    uint64_t step;                  /* 1 for the first step (bias corrections 1 - beta^step). lr and step are numbers of the call: a captured
                                       graph replays those that it was captured with */
    uint32_t state_bits;            /* 32 or 8 */
    uint32_t reserved;              /* 0 */
} ftc_adamw_t;

/*
 * For every element, in float32, with c1 = 1/(1-beta1^step), c2 = 1/sqrt(1-beta2^step), l = lr * lr_scale:
 *   g = grad * (1 / included) * *d_grad_scale;  m = m*beta1 + g*(1-beta1);  v = v*beta2 + (g*g)*(1-beta2)
 *   p = p * (1 - l*weight_decay) - (m / (sqrt(v)*c2 + eps)) * (l*c1)
 * Each operation of g, m and v is rounded (no fused multiply-add). The move of p has an approximate root and quotient (2^-23 each) and ends in a
 * multiply-add: it is good to 16 half units in its last place.
 *   d_m, d_v  states of ftc_param_table_blocks() blocks of FTC_STATE_BLOCK elements: float32, or with state_bits = 8 int8 and
 *             uint8; zero bytes before the first step; 32-byte aligned
 *   d_m_scale, d_v_scale  float32, one for each block (state_bits = 8; else NULL); zeros before the first step
 *   d_grad_scale  one float32 (d_norm + 1 of ftc_grad_norm), or NULL for 1; where it is not finite the call changes nothing
 * States in 8 bits: with s = max |m| of the block (at least 2^-126), m is held as the whole number c nearest to 127*sqrt(|m|/s),
 * signed, and stands for c*|c|*s/127^2. v is held through its root r = sqrt(v): s = max r, c nearest to 255*sqrt(r/s) and at
 * least 1 where r > 0; it stands for (c^2*s/255^2)^2. A state whose beta exceeds 31/32 changes too little in a step for the nearest code
 * to follow: its code is the one below or the one above, the upper one where what the state stands for lies more than u of the way
 * from the lower code's value to the upper's, with u = (e*0x6A09E667 + step*0x9E3779B9) mod 2^32 / 2^32 (its upper 23 bits) for
 * element e of d_m and d_v. Over the steps u is spread evenly, so the states' mean is kept, while single ones spread around the 32-bit
 * state (v's root by a tenth or two). Steps have to be numbered one after the other for that. With a beta up to 31/32 codes are the
 * nearest ones, and a state whose gradients vanish falls no further than about code 2/(1-beta2) of 255 (v; 40 at 0.95, 2.5 % of the
 * block's largest root) and 1/(1-beta1) of 127 (m; 10 at 0.9, 0.6 % of the largest). The update itself uses the new m and v before they
 * are rounded. A block of which no element's message was delivered stays as it is; in a block of which some were, the others' m and v are
 * rounded again under the block's new scales. A block whose m or v meets NaN or an infinity has NaN in its place afterwards.
 * param must not be NULL for tensors with n > 0 (FTC_EINVAL).
 */
FTC_API int ftc_adamw_step(const ftc_adamw_t* hyper, const void* h_table, const void* d_table, void* d_m, void* d_v,
                           float* d_m_scale, float* d_v_scale, const float* d_grad_scale, void* cuda_stream);

/* What states in 8 bits stand for, in the same layout: d_m_out, d_v_out float32 [blocks][FTC_STATE_BLOCK], 32-byte aligned (for
 * checkpoints, inspection, or going on in 32 bits). `blocks` blocks of d_m, d_v and the scales are read. */
FTC_API int ftc_adamw_states(uint64_t blocks, const void* d_m, const void* d_v, const float* d_m_scale, const float* d_v_scale,
                             float* d_m_out, float* d_v_out, void* cuda_stream);

/*
 * The two ends of a language model, and the update of its matrices. As above: float32 arithmetic whatever the element types, sums in a
 * fixed order, status records read as the allreduce leaves them.
 *
 * Embedding lookup: rows of a table of V rows of H elements.
 */
typedef struct {
    uint32_t V;          /* rows of the table, 1 .. 2^30 */
    uint32_t H;          /* elements of a row, 1 .. 2^24; V * H at most 2^40 */
    uint32_t P;          /* processes the tokens are divided over (backward), 1 .. 2^20 */
    uint32_t k;          /* elements of a message (backward), 1 .. 2^24: the gradient is [ceil(V*H/k)][P][k]; with P = 1 that is [V][H] (and
                            the last message's fill) whatever k; (V * H + k) * P at most 2^40 */
    uint32_t dtype;      /* y, dy: FTC_F32, FTC_BF16 or FTC_F16 */
    uint32_t wdtype;     /* the table: FTC_F32 or dtype */
    uint32_t token_bits; /* tokens are int64 or int32: 64 or 32 */
    float    scale;      /* finite */
} ftc_embed_t;

/*
 * y[t] = scale * table[token t], rounded once; zeros where the token is not in 0 .. V-1 (padding, positions without a token).
 *   d_tokens  [n] of token_bits, n at most 2^31
 *   d_table   row v at element v * table_stride; d_y: row t at element t * y_stride (strides >= H)
 * Pointers are aligned to their element size; rows on 16-byte boundaries are the fast case. n = 0 is valid and does nothing.
 */
FTC_API int ftc_embedding_forward(const ftc_embed_t* desc, uint64_t n, const void* d_tokens, const void* d_table, uint64_t table_stride,
                                  void* d_y, uint64_t y_stride, void* cuda_stream);

/*
 * The table's gradient, for each process: row v of process p is scale * the sum of dy[t] over its tokens t of value v (in a fixed order:
 * by stretches of the sorted list of tokens, FTC_EMBED_RUN long, or, of few tokens, of the tokens themselves).
 *   d_row_splits  as for ftc_layernorm_backward, of tokens
 *   d_dtable      float32 [ceil(V*H/k)][P][k], the inputs of ceil(V*H/k) scenarios for ftc_allreduce_batch: element e = v*H + h of
 *                 process p is element e % k of message e / k; the last message is filled up with zeros. Written whole.
 *   d_workspace   ftc_embedding_workspace_bytes(desc, n) bytes, 16-byte aligned; as for ftc_layernorm_backward. NULL with n = 0
 */
FTC_API int ftc_embedding_backward(const ftc_embed_t* desc, uint64_t n, const void* d_tokens, const void* d_dy, uint64_t dy_stride,
                                   const uint64_t* d_row_splits, float* d_dtable, void* d_workspace, size_t workspace_bytes,
                                   void* cuda_stream);
FTC_API size_t ftc_embedding_workspace_bytes(const ftc_embed_t* desc, uint64_t n);   /* 0 for an invalid descriptor, and for n = 0 */
#define FTC_EMBED_RUN 32u

/* Log probabilities of given tokens under rows of logits. */
typedef struct {
    uint32_t V;          /* logits of a row, 1 .. 2^30 */
    uint32_t dtype;      /* logits and their gradient: FTC_F32, FTC_BF16 or FTC_F16 */
    uint32_t token_bits; /* tokens are int64 or int32: 64 or 32 */
    uint32_t top;        /* the most likely tokens that are listed, 0 .. 32 and at most V */
    float    scale;      /* z = scale * logit (1 / temperature), 1e-6 .. 1e6 */
} ftc_logprob_t;

/*
 * For each row, with z = scale * logits: lse = log(sum(exp(z))), logprob = z[token] - lse, entropy = -sum(p * log p) with p = exp(z - lse),
 * and the `top` largest logits' log probabilities and tokens, largest first, the lower token first where logits are the same.
 *   d_logits  [rows] rows of V elements, row r at element r * stride (stride >= V); fewer than 2^31 rows
 *   d_tokens  [rows] of token_bits, or NULL (with d_logprob NULL). A token outside 0 .. V-1: logprob 0
 *   d_logprob, d_entropy, d_lse  [rows] float32; each may be NULL
 *   d_top_logprob [rows][top] float32, d_top_token [rows][top] int32: both given with top > 0, both NULL otherwise
 * Logits of -infinity are tokens that cannot come: p = 0. A row of nothing else has lse = logprob = top_logprob = -infinity and entropy 0. Any other
 * row's lse is held within float32's finite numbers (scale * logits may leave them; the rest is right all the same). A row that holds +infinity
 * or NaN has NaN for logprob (of a token), entropy, lse and top_logprob; its top_token are unspecified.
 * rows = 0 is valid and does nothing.
 */
FTC_API int ftc_token_logprobs(const ftc_logprob_t* desc, uint64_t rows, const void* d_logits, uint64_t stride, const void* d_tokens,
                               float* d_logprob, float* d_entropy, float* d_lse, float* d_top_logprob, int32_t* d_top_token,
                               void* cuda_stream);

/*
 * The gradient of the logits: scale * (dlogprob * ([j = token] - p_j) - dentropy * p_j * (log p_j + entropy)).
 *   d_lse, d_entropy       [rows], as the forward pass left them (d_entropy may be NULL without d_dentropy)
 *   d_dlogprob, d_dentropy [rows] float32; either may be NULL: 0. Where the token is outside 0 .. V-1 its dlogprob is not read into the result
 *   d_dlogits  rows of V elements, row r at element r * dstride; may be d_logits (with the same stride)
 * Rows with lse = -infinity get zeros. Where lse is finite but its size (2^7 or more in float32, 2^11 in float16, 2^14 in bfloat16) leaves p too few bits,
 * p is found from the logits again, in two more passes over the row.
 */
FTC_API int ftc_token_logprobs_backward(const ftc_logprob_t* desc, uint64_t rows, const void* d_logits, uint64_t stride, const void* d_tokens,
                                        const float* d_lse, const float* d_entropy, const float* d_dlogprob, const float* d_dentropy,
                                        void* d_dlogits, uint64_t dstride, void* cuda_stream);

/*
 * Orthogonalised updates of many matrices at once (momentum, then Newton-Schulz products, as the Muon optimiser does). A plan of the
 * matrices is built on the host and kept by the caller on the host and (a copy) on the device, as the table of tensors is.
 */
typedef struct {
    ftc_param_t tensor;      /* n = rows * cols elements, contiguous, row by row; as in the table of tensors */
    uint32_t rows, cols;     /* each 1 .. 2^20, the smaller at most 2^14; rows * cols at most 2^31 */
} ftc_matrix_t;

FTC_API size_t ftc_muon_plan_bytes(const ftc_matrix_t* h_matrices, uint32_t n);      /* 0 for invalid entries */
/* Checks the entries and writes the plan to h_plan (8-byte aligned host memory). FTC_EINVAL: what ftc_param_table_build refuses, NULL
 * param, tensor.n other than rows * cols, sizes out of range. */
FTC_API int ftc_muon_plan_build(const ftc_matrix_t* h_matrices, uint32_t n, void* h_plan, size_t plan_bytes);
FTC_API uint64_t ftc_muon_plan_blocks(const void* h_plan);                           /* blocks of FTC_STATE_BLOCK elements of momentum */
FTC_API size_t ftc_muon_workspace_bytes(const void* h_plan, uint32_t products);      /* 0 for anything that is no plan */

typedef struct {
    double lr, momentum, eps;    /* lr >= 0 and finite, 0 <= momentum < 1, eps >= 1e-30, all of them as float32 */
    uint32_t steps;              /* Newton-Schulz steps, 1 .. 16 (5 is usual) */
    uint32_t nesterov;           /* 1 or 0 */
    uint32_t products;           /* 16: the operands of products are rounded to float16 (of numbers up to 1.3, held times 2^14): the update X is
                                    good to 1e-3 of its norm where the momentum is well conditioned (6e-4 for wide ones). 32: operands are
                                    held as two float16 numbers each, three products for one: 2e-6 with sums of 256 terms, 5e-6 with 1000,
                                    1.5e-5 with 2000, 3e-5 with 4096 */
    uint32_t reserved;           /* 0 */
} ftc_muon_t;

/*
 * For each matrix, with l = lr * lr_scale:
 *   g = grad * (1 / included) * *d_grad_scale;  M = M*momentum + g;  U = nesterov ? g + M*momentum : M
 *   X = U / (|U| + eps) with the root of the sum of squares |U|, transposed if it has more rows than columns; then, `steps` times,
 *   A = X X^T, X = 3.4445 X + (-4.775 A + 2.0315 A A) X
 *   p = p * (1 - l*weight_decay) - l * X
 * X has singular values between 0.68 and 1.21 but where U's are tiny; a matrix's elements then move by about l / sqrt(max(rows, cols))
 * (lr_scale = 0.2 * sqrt(max(rows, cols)) makes it 0.2 l as with AdamW).
 *   d_momentum    float32, ftc_muon_plan_blocks() blocks of FTC_STATE_BLOCK elements laid out as AdamW's states; zeros before the first step; 32-byte aligned
 *   d_grad_scale  as for ftc_adamw_step
 *   d_workspace   ftc_muon_workspace_bytes(h_plan, products) bytes, 256-byte aligned; as for ftc_layernorm_backward
 * An element of a message that was not delivered keeps its momentum, which is its U; a matrix of which nothing was delivered (with n > 0) stays as it is.
 * A matrix that meets NaN or an infinity has NaN in its weights afterwards. d_workspace's first 32-bit word is 0 once the call's work is done; were a
 * wait inside a kernel ever to give up, it is not, and no weights were changed, but d_momentum has moved: the step is not to be called again
 * with the same gradients unless d_momentum is put back. FTC_ECUDA: the GPU cannot run the kernels (nothing was changed), or a launch failed on the
 * way (d_momentum may have moved).
 */
FTC_API int ftc_muon_step(const ftc_muon_t* hyper, const void* h_plan, const void* d_plan, float* d_momentum, const float* d_grad_scale,
                          void* d_workspace, size_t workspace_bytes, void* cuda_stream);

FTC_API const char* ftc_strerror(int code);
FTC_API uint32_t ftc_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FTC_H */
