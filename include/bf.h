/*
 * bf.h -- C ABI of the brute-force optimal device-mapping search (libbf.so).
 *
 * The problem (§2.1 of "Agentic CPU-GPU Scheduling for Heterogeneous AI
 * Workloads"): a workflow is a DAG G=(V,E) of N tool invocations; each tool v
 * is mapped to a mode a_v in {cpu, gpu_now, gpu_queue}; a mapping is feasible
 * only if the VRAM of the GPU tools running at any instant stays within the
 * budget M; its end-to-end latency T_e2e is the largest completion time over
 * the sinks.  The brute-force oracle the paper grades its scheduler against
 * (§2.3, §4.1) is the feasible mapping of lowest T_e2e among all 3^N.
 *
 * The paper measures T_e2e on hardware.  This library evaluates it under a
 * fixed integer latency model (version 1), exact to the microsecond:
 *
 *   - Times are integer microseconds.  GPU progress is a virtual clock V in
 *     1/1024 isolated-microsecond units; a GPU tool of isolated time w that
 *     starts at V ends when V reaches V + 1024*w.
 *   - GPU contention (Factor A, §2.3): while k GPU tools run, each runs at
 *     1024/f[k] of its isolated speed (processor sharing).  CPU tools are
 *     unaffected; CPU cores are unlimited.
 *   - cpu: duration c.  gpu_now: isolated work g + x (Table 1's GPU time
 *     includes PCIe transfer), starts when its predecessors are done, holds
 *     its VRAM m while running; a start that brings live VRAM above M makes
 *     the mapping infeasible (out of memory, Factor B).  gpu_queue: waits in
 *     one serialised FIFO queue (ready time, then index) without holding VRAM;
 *     the head starts when no queued tool is running and live VRAM + m <= M;
 *     isolated work l + g + x (Table 1's gpu_queue column = GPU + Load).  A
 *     queued tool with m > M can never start: infeasible.  No bypass.
 *   - Event loop: next CPU completion vs next GPU completion
 *     T + ceil((Vmin - V) * f[k] / 2^20); if a CPU tool ends first, V advances
 *     by floor((t_cpu - T) * 2^20 / f[k]).  At each event every tool ending at
 *     that instant retires (freeing VRAM), then newly ready tools start in
 *     index order, then the queue head is tried.  Makespan = time of the last
 *     retirement; infeasible mappings have makespan 0xFFFFFFFF.
 *
 * Mapping index: idx = sum_i a_i * 3^i, a_i in {0=cpu, 1=gpu_now,
 * 2=gpu_queue}; tool 0 is the least-significant digit.  Searches return the
 * feasible mapping of lowest makespan, ties to the lowest index.  The all-cpu
 * mapping (index 0) is always feasible, so a full search always succeeds.
 *
 * Conventions for every entry point:
 *   - Return 0 (BF_OK) or a BF_E* status; bf_last_error() then describes the
 *     failure (thread-local string owned by the library, valid until the next
 *     call on that thread).  Outputs are written only on BF_OK.
 *   - Host pointers are caller-owned and only read during the call (inputs are
 *     copied).  Device pointers are caller-owned CUDA device memory on the
 *     current device.  `cuda_stream` is a cudaStream_t (NULL = legacy default
 *     stream); work is ordered on it.
 *   - A handle's scratch (search key, what-if list) is shared by the calls that
 *     use it: calls on one handle must not overlap in time.  A handle belongs
 *     to the device that was current when it was created; calls on it with
 *     another device current return BF_EINVAL.
 *   - Blocking calls wait with a time limit (bf_set_wait_timeout_ms) and
 *     return BF_ETIMEOUT if it passes; the GPU work is then still in flight,
 *     and the scenario must not be destroyed until the stream has finished.
 */
#ifndef BF_H_
#define BF_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Entry points are the library's only exported symbols (it is built with
 * hidden visibility). */
#if defined(__GNUC__)
#define BF_API __attribute__((visibility("default")))
#else
#define BF_API
#endif

#define BF_MAX_TOOLS 32       /* largest scenario (32-bit tool masks) */
#define BF_MAX_TOOLS_ENUM 20  /* largest scenario of the full-enumeration entry points
                                 (bf_eval_mappings, bf_search_best, bf_search_range,
                                 bf_search_pruned, bf_search_batch*): 3^20 < 2^32 */

enum bf_status {
  BF_OK = 0,
  BF_EINVAL = 1,    /* invalid argument or scenario */
  BF_ERANGE = 2,    /* index range outside [0, 3^n) */
  BF_ENOMEM = 3,    /* device or pinned-host allocation failed */
  BF_ECUDA = 4,     /* a CUDA runtime call failed (message names it) */
  BF_ETIMEOUT = 5   /* a blocking wait exceeded its time limit */
};

enum bf_mode { BF_MODE_CPU = 0, BF_MODE_GPU_NOW = 1, BF_MODE_GPU_QUEUE = 2 };

/*
 * One workflow (§2.1) with the per-tool profile of Table 1 / §3.1 plus a
 * transfer time.  Tools are numbered 0..n-1 in a topological order.
 * Validity (checked by every entry point that takes a desc):
 *   1 <= n <= 32 (the full-enumeration entry points take n <= 20 and return
 *   BF_EINVAL above); pred_mask[v] has bits only below v (u < v);
 *   cpu_us >= 1, gpu_us >= 1; load_us + gpu_us + xfer_us < 2^22;
 *   vram_mib <= 2^27, vram_budget_mib <= 2^31;
 *   slowdown_q10[1] == 1024, slowdown_q10[k] non-decreasing and <= 65536 for
 *   k = 1..n (entries 0 and > n are ignored);
 *   the makespan bound sum_i max(c_i, floor((l_i+g_i+x_i)*f[n]/1024) + n + 1)
 *   is <= 0xFFFFFFFD, so every makespan fits in 32 bits.
 * Entries at index >= n are ignored.
 */
typedef struct bf_scenario_desc {
  uint32_t n;                               /* number of tools, 1..32 */
  uint32_t pred_mask[BF_MAX_TOOLS];         /* bit u of pred_mask[v] <=> edge u->v */
  uint32_t cpu_us[BF_MAX_TOOLS];            /* c_i: CPU latency, us */
  uint32_t gpu_us[BF_MAX_TOOLS];            /* g_i: isolated GPU latency, us */
  uint32_t xfer_us[BF_MAX_TOOLS];           /* x_i: host<->device transfer, us (GPU modes only) */
  uint32_t load_us[BF_MAX_TOOLS];           /* l_i: gpu_queue load-in, us */
  uint32_t vram_mib[BF_MAX_TOOLS];          /* m_i: VRAM footprint, MiB */
  uint32_t vram_budget_mib;                 /* M */
  uint32_t slowdown_q10[BF_MAX_TOOLS + 1];  /* f[k], k=1..n, 1024 = isolated speed */
} bf_scenario_desc;

/* Result of a search: the argmin mapping and its makespan. */
typedef struct bf_result {
  uint64_t index;                  /* canonical mapping index */
  uint32_t makespan_us;            /* 0xFFFFFFFF if feasible == 0 */
  uint32_t feasible;               /* 1 if a feasible mapping was found in the searched range */
  uint8_t mode[BF_MAX_TOOLS];      /* decoded digits of `index` (bf_mode), 0 beyond n */
} bf_result;

/* Opaque handle: validated scenario, its device-format tables and a small
 * device/pinned scratch area.  Owned by the library. */
typedef struct bf_scenario bf_scenario;

/* Validate a desc without touching the GPU.  BF_OK or BF_EINVAL. */
BF_API int bf_validate_desc(const bf_scenario_desc* desc);

/* The problem instance of §2.1 -- the tool DAG G=(V,E), each tool's profile
 * (Table 1 / §3.1: CPU and GPU latency, load-in, VRAM) plus its transfer time,
 * the VRAM budget M -- with the contention table of §2.3 Factor A.
 * Validate `desc`, copy it, allocate the handle's scratch (8-byte device key,
 * 8-byte pinned host key) on the current device and return it in *out.
 * The caller releases it with bf_destroy_scenario.  BF_EINVAL, BF_ENOMEM,
 * BF_ECUDA. */
BF_API int bf_create_scenario(const bf_scenario_desc* desc, bf_scenario** out);

/* Release a handle (NULL is accepted).  Synchronises with nothing: the caller
 * must make sure no work using it is still in flight. */
BF_API int bf_destroy_scenario(bf_scenario* scn);

/* Evaluate mappings [first, first+count) (§2.1's T_e2e under the model):
 * d_makespan[j] = makespan of mapping first+j (0xFFFFFFFF if infeasible),
 * d_feasible[j] = 1/0.  Both are caller-owned device arrays of >= count
 * elements.  Asynchronous on `cuda_stream`.  count == 0 is a no-op.
 * BF_ERANGE if first+count > 3^n; BF_EINVAL on NULL pointers.
 * A scenario whose DAG has barriers (every tool >= c waits for every tool < c)
 * is a row of independent segments: a large evaluation simulates each
 * segment's mappings into tables in the handle and writes every mapping's
 * makespan as the sum of its segments'.  Such evaluations of one handle may
 * overlap each other; a captured one never uses the tables. */
BF_API int bf_eval_mappings(const bf_scenario* scn, uint64_t first, uint64_t count,
                     uint32_t* d_makespan, uint8_t* d_feasible, void* cuda_stream);

/* Brute-force oracle of §2.3/§4.1 under the model: the feasible mapping of
 * lowest makespan over all 3^n, ties to the lowest index.  Blocks until the
 * result is on the host (bounded wait).  Writes *out on BF_OK. */
BF_API int bf_search_best(const bf_scenario* scn, bf_result* out, void* cuda_stream);

/* As bf_search_best over mappings [first, first+count) only; out->feasible is
 * 0 (and index = first) when no mapping in the range is feasible.  Range
 * searches compose: the best of the parts' results (lowest makespan, then
 * lowest index) is the result of their union -- used to split one search
 * across devices or to resume it piecewise.  BF_ERANGE if outside [0, 3^n);
 * count == 0 gives feasible = 0. */
BF_API int bf_search_range(const bf_scenario* scn, uint64_t first, uint64_t count,
                    bf_result* out, void* cuda_stream);

/* Full search of `count` independent scenarios in one call (one launch per
 * group of scenarios of similar size, four at most): out[i] is the
 * brute-force oracle of §2.3/§4.1 (as bf_search_best) for descs[i].  The paper
 * searches one workflow at a time; running many per launch is this library's
 * addition, for callers that score many workflows or many candidate
 * contention tables (the calibration of Table 2's S5 latencies) together.  All descs are validated
 * before any GPU work; the first invalid one (lowest position) fails the call with BF_EINVAL naming
 * its position.  Allocates its device scratch (packed tables + one key per scenario) from the
 * device's default stream-ordered memory pool on cuda_stream and frees it there after its kernels,
 * also when the wait times out (BF_ETIMEOUT).  A large batch launches part of its work on a stream
 * the call creates and destroys; that work starts after the work already enqueued on cuda_stream,
 * and work enqueued on cuda_stream after the call starts after it.  Blocks until the results are
 * on the host. */
BF_API int bf_search_batch(const bf_scenario_desc* descs, uint32_t count, bf_result* out,
                    void* cuda_stream);

/* Same result as bf_search_best (the feasible mapping of lowest makespan over
 * all 3^n, ties to the lowest index), found by branch and bound instead of
 * full enumeration.  An incumbent is taken from a few mappings (hint_index if
 * < 3^n, all-cpu, all-gpu_now, all-gpu_queue, each tool on its isolated-faster
 * device); a prefix (or a mid combination) is skipped when the time at which
 * its remaining tools can first start, plus the longest path through them in
 * minimum isolated durations min(c, g + x), exceeds the incumbent's makespan
 * -- no mode, contention or queueing makes a tool faster than that.  When
 * that first pass keeps more than 1/64 of the prefixes (a DAG without cut
 * points), the call continues as bf_search_tree over the full space, whose
 * bound is stronger.  Exact either way: the optimum and all its ties are
 * never skipped.  Allocates a 4-byte-per-prefix buffer (and, when it hands
 * over, the tree search's level buffers) in the handle on first use.  Blocks
 * until the result is on the host. */
BF_API int bf_search_pruned(const bf_scenario* scn, uint64_t hint_index, bf_result* out, void* cuda_stream);

/* Decision spaces of bf_search_tree: the full space (each tool on cpu,
 * gpu_now or gpu_queue; 3^n mappings) or the binary space the paper's S1-S10
 * use (§4.1: each tool on the CPU or the GPU, i.e. cpu or gpu_now; 2^n
 * mappings).  The value is the number of modes per tool. */
#define BF_SPACE_BINARY 2u
#define BF_SPACE_FULL 3u
/* bf_search_tree flag: simulate every mapping of the space (no pruning). */
#define BF_TREE_NO_PRUNE 1u

/* What a tree search did (bf_search_tree, optional). */
typedef struct bf_tree_stats {
  uint64_t nodes;         /* prefix nodes created (tools assigned in the search's order), root included */
  uint64_t leaf_nodes;    /* nodes whose last leaf_depth tools were enumerated */
  uint64_t leaves;        /* mappings simulated: to the end, or when pruning until past the best makespan known
                             (at most leaf_nodes * modes^leaf_depth) */
  uint32_t launches;      /* kernel launches */
  uint32_t leaf_depth;    /* tools enumerated below each leaf node */
  uint32_t incumbent_us;  /* the starting bound (0xFFFFFFFF with BF_TREE_NO_PRUNE) */
  uint32_t pad;
} bf_tree_stats;

/* The optimum of a decision space -- the feasible mapping of lowest makespan,
 * ties to the lowest canonical index, exactly as full enumeration would give
 * it -- for scenarios of up to 32 tools (3^32 ~ 1.9e15 mappings), by depth-
 * first branch and bound over the modes of the tools in a topological order:
 * the sources (tools without predecessors) first, then the others, each group
 * in index order (the model's results do not depend on that order; the index
 * returned is the canonical one).  A node (the modes of the first d tools of
 * that order) carries the simulation state at the first instant a later tool
 * could become ready, shared by all its mappings.
 * A node is dropped when a lower bound on all of its mappings' makespans
 * exceeds the best makespan known (strictly, so the optimum and its ties
 * survive): running tools end no earlier than their remaining work at
 * isolated speed allows, every other tool ends no earlier than the latest of
 * the node's time and its predecessors' earliest ends plus its duration in
 * its mode (or min(c, g + x) if open), and queued tools run one at a time.
 * The first bound is the best of a few mappings of the space (hint_index if
 * it lies in it, all-cpu, all-gpu_now, each tool on its isolated-faster
 * device, all-gpu_queue); when the tree is large, two narrow dives to the leaves
 * (256, then 2048 nodes per level) tighten it before the search restarts from the
 * root; at the leaves, modes in which a tool would end too late for the bound are
 * not enumerated; better bounds are found as the search proceeds.  space: BF_SPACE_FULL or
 * BF_SPACE_BINARY.
 * flags: 0 or BF_TREE_NO_PRUNE (every mapping of the space is simulated to
 * its end: full enumeration).  `stats` may be NULL.  Allocates level buffers in the
 * handle on first use (about 1.7 GB for 32 tools in the full space).  Blocks
 * until the result is on the host.  A pruned search of a scenario cut by
 * barriers into segments of at most 13 tools (see bf_eval_mappings) enumerates
 * each segment on its own instead, in one launch, and adds their optima up
 * (bf_search_pruned does the same); its stats count the segments as nodes and
 * their mappings as leaves.  The whole search, not only each wait, is held to the wait limit (bf_set_wait_timeout_ms): past it the call
 * returns BF_ETIMEOUT (an unpruned full space of 28 or more tools takes
 * hours). */
BF_API int bf_search_tree(const bf_scenario* scn, uint32_t space, uint32_t flags, uint64_t hint_index,
                   bf_result* out, bf_tree_stats* stats, void* cuda_stream);

/* Makespans and feasibility of an arbitrary list of mappings: d_makespan[j] and
 * d_feasible[j] for mapping d_indices[j] (all three caller-owned device arrays
 * of >= count elements).  An index >= 3^n yields makespan 0xFFFFFFFF and
 * d_feasible = 0xFF.  Asynchronous on `cuda_stream`; count == 0 is a no-op.
 * Used to score neighbourhoods of a mapping (bf_whatif) or any caller-chosen
 * candidate set. */
BF_API int bf_eval_indices(const bf_scenario* scn, const uint64_t* d_indices, uint64_t count,
                    uint32_t* d_makespan, uint8_t* d_feasible, void* cuda_stream);

/* One probe of the runtime monitor's bounded what-if exploration. */
typedef struct bf_probe {
  uint64_t index;        /* canonical index of the probed mapping */
  uint32_t makespan_us;  /* 0xFFFFFFFF if infeasible */
  uint32_t feasible;     /* 0 = exceeds the VRAM budget ("exceed") */
  uint8_t kind;          /* 0 = single-tool reprobe, 1 = swap reprobe */
  uint8_t tool;          /* i: the tool moved (swap: the tool moved to gpu_now) */
  uint8_t mode;          /* the new mode of tool i (bf_mode) */
  uint8_t other;         /* swap: j, the gpu_now tool moved to gpu_queue; single: 0xFF */
} bf_probe;

#define BF_MAX_PROBES (2 * BF_MAX_TOOLS + BF_MAX_TOOLS * BF_MAX_TOOLS)

/* The what-if probes of Algorithm 1's exploration step (§3.2) around mapping
 * base_index, scored on the model in one launch: for each tool i in index
 * order and each alternative mode a != d_i (in the order cpu, gpu_now,
 * gpu_queue), the single-tool reprobe d[i := a]; when that reprobe moves i to
 * gpu_now and exceeds the budget (infeasible), then for each tool j on
 * gpu_now in d (index order) the swap reprobe d[i := gpu_now, j := gpu_queue].
 * Writes the probes in that order to out[0 .. *count) (at most
 * BF_MAX_PROBES); BF_EINVAL if capacity is smaller than the number of probes,
 * BF_ERANGE if base_index >= 3^n.  Blocks until the results are on the host. */
BF_API int bf_whatif(const bf_scenario* scn, uint64_t base_index, bf_probe* out, uint32_t capacity,
              uint32_t* count, void* cuda_stream);

/* Largest batch bf_search_batch_noalloc accepts. */
#define BF_NOALLOC_MAX_SCENARIOS 1024

/* The batched search of bf_search_batch without any memory allocation.  The
 * paper has no counterpart: this exists for callers that cannot allocate
 * device memory at the moment they search -- e.g. a scheduler loop whose
 * process has handed all GPU memory to another allocator's pool, or one that
 * must not let cudaMalloc/cudaFree synchronise the device between rounds.
 * The caller passes the inputs (descs) and outputs (out) as for
 * bf_search_batch; the scratch (packed scenario records and one key per
 * scenario, about 0.84 MiB for BF_NOALLOC_MAX_SCENARIOS) is a fixed array in
 * the library's device image, held on every GPU that loads the library until
 * the process exits.  count > BF_NOALLOC_MAX_SCENARIOS fails with BF_EINVAL.
 * The first call on a device (and the first after a device reset) resolves
 * that array's device address; make it before any stream capture.
 * All calls share the one array, which keeps the last call's contents (each
 * call resets its keys), so two calls whose GPU work overlapped would race.
 * The library prevents that: calls on one device are serialised by a host
 * lock, and after a call returns BF_ETIMEOUT its kernel may still be using
 * the array, so the next call first waits (bounded) for that call's stream to
 * finish and returns BF_ETIMEOUT if it does not; keep that stream alive until
 * then.  Blocks until the results are on the host. */
BF_API int bf_search_batch_noalloc(const bf_scenario_desc* descs, uint32_t count, bf_result* out,
                            void* cuda_stream);

/* ---- Learning from makespans ----------------------------------------------
 *
 * The searches and evaluations above grade the mappings a scheduling model
 * answers with; these entry points turn such grades into gradients.  The paper
 * prompts its scheduler (§3.3) and trains nothing: they are this library's
 * addition, for callers that fit a policy to the makespans of the mappings it
 * samples.
 *
 * All of them are asynchronous on `cuda_stream`, allocate nothing and can be
 * captured; a workspace is the caller's, of the size its *_workspace function
 * gives and aligned to 256 bytes, holds nothing between calls, and must not be
 * used by two calls whose work overlaps.  Values are computed in 32 bits
 * whatever the matrices' types, sums in an order that does not depend on when
 * blocks run (the same call gives the same bits), and rounded once.
 *
 * A row t of logits x (vocab columns) goes with token y = tokens[t].  With
 * temperature tau, z = x / tau, p = softmax(z), lp = ln p_y, H = -sum p ln p.
 * A token below 0 marks a row that is not scored (a prompt, padding): its
 * logits are not used, its log-probability and entropy are 0 and its gradient
 * is 0.  A token >= vocab makes its row's values NaN (log-probability,
 * entropy, gradient, terms of a loss), whatever the row's logits.  Logits may
 * be -inf (banned tokens); a row with none above -inf has log-probability
 * -inf, entropy 0, gradient 0, and terms of 0 in the policy loss.  A probability
 * below 2^-126 of its row's largest counts as 0.
 */
enum bf_dtype { BF_F32 = 0, BF_BF16 = 1, BF_F16 = 2 };

/* A matrix in device memory: element (i, j) is data[i * row_stride + j], at any
 * address its type allows.  At most 2^31 - 1 rows and 2^30 columns, row_stride
 * >= cols.  What lies between its rows may be read and is never written. */
typedef struct bf_matrix {
  void* data;
  uint64_t rows, cols;
  uint64_t row_stride;  /* in elements */
  uint32_t dtype;       /* bf_dtype */
  uint32_t pad;
} bf_matrix;

/* Log-probabilities d_logprob[t] = lp and, unless d_entropy is NULL, entropies
 * d_entropy[t] = H of the rows of `logits`.  1e-18 <= temperature <= 1e18. */
BF_API int bf_token_logprobs(const bf_matrix* logits, const int64_t* d_tokens, float temperature, float* d_logprob,
                             float* d_entropy, void* cuda_stream);

/* The gradient in the logits of sum_t d_grad_logprob[t] lp_t +
 * d_grad_entropy[t] H_t (d_grad_entropy may be NULL):
 *   dx_j = (g ([j = y] - p_j) - h p_j (ln p_j + H)) / tau.
 * `grad` has the shape and type of `logits`; it may be `logits` itself (same
 * data and stride), else the two must not overlap. */
BF_API int bf_token_logprobs_grad(const bf_matrix* logits, const int64_t* d_tokens, float temperature,
                                  const float* d_grad_logprob, const float* d_grad_entropy, const bf_matrix* grad,
                                  void* cuda_stream);

/* How the policy loss weighs its rows: w = 1 / (scored rows); w = 1 / (scored
 * rows of the row's sequence * sequences with a scored row); w = 1. */
enum bf_reduction { BF_MEAN_TOKENS = 0, BF_MEAN_SEQUENCES = 1, BF_SUM = 2 };

/* Sequence s is rows [offsets[s], offsets[s+1]); offsets ascend.  Rows outside
 * every sequence are not scored. */
typedef struct bf_policy_args {
  const int64_t* tokens;       /* device, one per row */
  const int64_t* offsets;      /* device, sequences + 1 */
  const float* old_logprob;    /* device, one per row: under the policy that sampled the tokens */
  const float* ref_logprob;    /* device, one per row: under the reference policy; NULL without a KL term */
  const float* advantage;      /* device, one per sequence, or per row with advantage_per_token */
  uint64_t sequences;
  uint32_t advantage_per_token;
  uint32_t reduction;          /* bf_reduction */
  float clip_low, clip_high;   /* the ratio is held to [1 - clip_low, 1 + clip_high]; >= 0 */
  float kl_coef;               /* >= 0 */
  float entropy_coef;
  float temperature;           /* 1e-18 to 1e18 */
  float grad_scale;            /* factor of the gradient (loss scaling), 1 for none */
} bf_policy_args;

#define BF_POLICY_STATS 6

/* The clipped policy loss with a KL term and its gradient in the logits.  With
 * r = e^(lp - old), advantage A and u = ref - lp, a scored row's term is
 *   l = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *       + kl_coef (e^u - u - 1) - entropy_coef H
 * and the loss is sum w l; with kl_coef = 0 a reference is only watched, and
 * nothing of it gets into the loss or the gradient.  d_stats: the loss, then
 * the weighted sums of -min(...), of e^u - u - 1 (0 without ref_logprob), of H,
 * of the rows whose clip stops the gradient, and of r.  d_logprob (may be
 * NULL): lp of each row.
 * `grad` (may be NULL: loss only) as for bf_token_logprobs_grad. */
BF_API int bf_policy_loss(const bf_matrix* logits, const bf_policy_args* args, float* d_stats, float* d_logprob,
                          const bf_matrix* grad, void* d_workspace, uint64_t workspace_bytes, void* cuda_stream);
BF_API int bf_policy_loss_workspace(uint64_t rows, uint64_t sequences, uint64_t* bytes);

/* Pair p: sequence 2p is the preferred answer (the faster mapping), 2p + 1 the
 * other. */
typedef struct bf_preference_args {
  const int64_t* tokens;       /* device, one per row */
  const int64_t* offsets;      /* device, 2 * pairs + 1 */
  const float* ref_logprob;    /* device, one per row; NULL for no reference policy */
  uint64_t pairs;
  uint32_t average;            /* rewards from the mean over a sequence's scored rows instead of the sum */
  float beta;                  /* > 0 */
  float label_smoothing;       /* eps: in [0, 1) */
  float margin;
  float temperature;           /* 1e-18 to 1e18 */
  float grad_scale;            /* factor of the gradient (loss scaling), 1 for none */
} bf_preference_args;

#define BF_PREFERENCE_STATS 4

/* The preference loss and its gradient in the logits.  A sequence's reward is
 * beta sum (lp - ref) over its scored rows (beta times their mean with
 * `average`; 0 without scored rows); with h = reward_2p - reward_2p+1 - margin
 * a pair's loss is -(1 - eps) ln sigma(h) - eps ln sigma(-h), and the loss the
 * mean over the pairs.  d_stats: the loss, the share of pairs with reward_2p >
 * reward_2p+1, the mean reward of the preferred and of the other answers.
 * d_rewards: 2 * pairs.  d_logprob (may be NULL) and `grad` (may be NULL) as
 * for bf_policy_loss. */
BF_API int bf_preference_loss(const bf_matrix* logits, const bf_preference_args* args, float* d_stats,
                              float* d_rewards, float* d_logprob, const bf_matrix* grad, void* d_workspace,
                              uint64_t workspace_bytes, void* cuda_stream);
BF_API int bf_preference_loss_workspace(uint64_t rows, uint64_t pairs, uint64_t* bytes);

/* Token embedding: row t of `out` is scale * table[tokens[t]], 0 for a token
 * below 0 and NaN for one >= table->rows.  `out` has one row per token and the
 * table's width and type, and does not overlap it. */
BF_API int bf_embed(const bf_matrix* table, const int64_t* d_tokens, float scale, const bf_matrix* out,
                    void* cuda_stream);

/* Its gradient: grad_table[v] = scale * sum over t with tokens[t] = v, in
 * ascending t, of grad_out[t] (added to what grad_table holds with
 * `accumulate`; else every row is written, 0 where no token occurs).  Tokens
 * outside the table are left out.  The types may differ; the matrices do not
 * overlap. */
BF_API int bf_embed_grad(const bf_matrix* grad_out, const int64_t* d_tokens, float scale, uint32_t accumulate,
                         const bf_matrix* grad_table, void* d_workspace, uint64_t workspace_bytes, void* cuda_stream);
BF_API int bf_embed_grad_workspace(uint64_t rows, uint64_t width, uint64_t* bytes);

/* ---- Answering --------------------------------------------------------------
 *
 * A decoding step of a scheduling model that answers a workflow's prompt with
 * many candidate mappings: beams, or samples that are graded against each
 * other.  The paper's scheduler (§3.3) answers once and by a prompted model;
 * these entry points are this library's addition, beside the learning ones and
 * under the same conventions: asynchronous on `cuda_stream`, no allocation, can be
 * captured, a workspace (aligned to 256 bytes) that holds nothing between
 * calls and serves one call at a time, values in 32 bits or more, the same
 * bits for the same call.
 */

/* Vectors of many sequences in device memory: element (b, t, h, d) is
 * data[b * batch_stride + t * token_stride + h * head_stride + d] (strides in
 * elements), at any address its type allows.  At most 2^31 - 1 sequences and
 * tokens, 65,536 heads, 256 dimensions, 2^42 elements from first to last. */
typedef struct bf_cache {
  void* data;
  uint64_t batch, tokens, heads, dim;
  uint64_t batch_stride, token_stride, head_stride;
  uint32_t dtype;  /* bf_dtype */
  uint32_t pad;
} bf_cache;

typedef struct bf_attention_args {
  const int64_t* prefix_lengths;  /* device, one per prompt; NULL: prefix_k->tokens each */
  const int64_t* suffix_lengths;  /* device, one per answer; NULL: suffix_k->tokens each */
  float scale;                    /* of the scores, 1 / sqrt(dim) as a rule; up to 1e30 in size */
  uint32_t pad;
} bf_attention_args;

/* Attention of one token of each answer to its prompt, whose keys the answers
 * share and which is read once for all of them, and to the answer's own keys.
 * With `prompts` = prefix_k->batch prompts and w = q->batch / prompts answers to
 * each, answer a belongs to prompt a / w; query head h reads key head
 * h / (q->heads / prefix_k->heads).  Over the prompt's first
 * prefix_lengths[a / w] tokens and the answer's first suffix_lengths[a]:
 *   s_t = scale q . k_t, out = sum e^(s_t) v_t / sum e^(s_t), lse = ln sum e^(s_t).
 * q and out have one token per answer; all types are the same.  suffix_k and
 * suffix_v may both be NULL (the prompt alone); d_lse (answers x heads) may be
 * NULL.  What lies behind a length is not used, whatever it holds.  With nothing
 * to attend to (lengths 0, or every score -inf) out is 0 and lse -inf; a length
 * outside 0..tokens makes its answers' out and lse NaN, and so does a score that is NaN or above
 * 32-bit numbers.  For 16-bit types the
 * weights e^(s_t - max) are rounded to the type before the second product (by at most 2^-8 of
 * themselves for bf16; for f16 2^-11, or 2^-32 of the largest).  Neither out nor lse overlaps an input (the lengths among them) or the other. */
BF_API int bf_prefix_attention(const bf_cache* q, const bf_cache* prefix_k, const bf_cache* prefix_v,
                               const bf_cache* suffix_k, const bf_cache* suffix_v, const bf_attention_args* args,
                               const bf_cache* out, float* d_lse, void* d_workspace, uint64_t workspace_bytes,
                               void* cuda_stream);
BF_API int bf_prefix_attention_workspace(const bf_cache* q, const bf_cache* prefix_k, const bf_cache* suffix_k,
                                         uint64_t* bytes);

#define BF_MAX_BEAMS 256

typedef struct bf_beam_args {
  const float* scores;      /* device, one per beam: log-probability so far; -inf for a beam that is not alive */
  const uint8_t* finished;  /* device, one per beam, 0 or 1; NULL: none is */
  const int64_t* lengths;   /* device, one per beam: tokens so far; NULL without a length penalty */
  uint64_t groups;          /* prompts; the logits have groups * beams rows */
  uint32_t beams;           /* per group, 1 to BF_MAX_BEAMS */
  uint32_t keep;            /* continuations kept per group, 1 to BF_MAX_BEAMS */
  int64_t end_token;        /* the token that finishes a beam; -1: none */
  float length_penalty;     /* 0 to 65536 */
  float temperature;        /* 1e-18 to 1e18 */
} bf_beam_args;

/* The best continuations of each group's beams.  A beam that is alive continues
 * with every token v of its row of logits, at the total score + ln softmax(logits
 * / temperature)_v; one that is finished stays as it is, as the one continuation
 * end_token at its own score (its logits are not used).  A continuation of n
 * tokens has rank total / max(1, n)^length_penalty.  The `keep` of highest rank
 * of each group, ties to the lower beam, then the lower token, are written in
 * that order: d_scores (the total), d_tokens, d_parents (the row of the beam
 * continued), d_finished (may be NULL: 1 where the beam was finished or the
 * token is end_token) and d_lengths (may be NULL: n), groups * keep of each.
 * Tokens of logit -inf are no continuations.  Where a group has fewer than
 * `keep`, the rest has score -inf, token -1, finished 0, length 0 and as parent j
 * the group's beam j modulo beams.  A logit of NaN or +inf, a score of NaN or
 * +inf makes its group's scores NaN and the rest as if nothing could continue
 * (a finished beam's logits do not matter).  At most 2^23 - 1 groups and a
 * vocabulary of 2^24.  No output overlaps an input or another output.  Where the
 * workspace has 0 bytes it may be NULL. */
BF_API int bf_beam_step(const bf_matrix* logits, const bf_beam_args* args, float* d_scores, int64_t* d_tokens,
                        int64_t* d_parents, uint8_t* d_finished, int64_t* d_lengths, void* d_workspace,
                        uint64_t workspace_bytes, void* cuda_stream);
BF_API int bf_beam_step_workspace(uint64_t groups, uint32_t beams, uint64_t vocab, uint32_t keep, uint64_t* bytes);

/* The states of beams: `count` arrays of the same layout, `rows` rows of up to
 * `tokens` tokens of `heads` runs of `width` bytes. */
typedef struct bf_states {
  uint64_t rows, tokens, heads, width;
  uint64_t row_stride, token_stride, head_stride;  /* in bytes */
} bf_states;

#define BF_MAX_STATES 128

/* Row i of each array takes row d_parents[i]'s first d_lengths[d_parents[i]]
 * tokens (all of them where d_lengths is NULL); what is behind them in row i
 * stays as it was.  Groups are runs of `beams` rows, and a parent is in its
 * row's group: a row whose parent is not stays as it was, and so does one whose
 * parent's length is negative; a length above `tokens` counts as `tokens`.
 * `from` and `to` are host arrays of `count` (at most BF_MAX_STATES) device
 * addresses; to[k] == from[k] with the same layout reorders in place (rows that
 * are their own parent cost nothing), otherwise no array overlaps another.  No array of `to`
 * overlaps d_parents or d_lengths, which are not reordered.  On a GPU whose copies no longer
 * come in, the parts of rows that could not be moved hold bytes of 255 (NaN, or -1). */
BF_API int bf_beam_reorder(void* const* from, const bf_states* from_layout, void* const* to,
                           const bf_states* to_layout, uint32_t count, const int64_t* d_parents, uint32_t beams,
                           const int64_t* d_lengths, void* cuda_stream);

/* Time limit of blocking waits, in milliseconds (default 600000; 0 = none).
 * Process-wide. */
BF_API void bf_set_wait_timeout_ms(uint32_t ms);

/* Description of the last failure on this thread ("" if none). */
BF_API const char* bf_last_error(void);

/* Library version string, e.g. "bf 1.0 (model v1)". */
BF_API const char* bf_version(void);

#ifdef __cplusplus
}
#endif

#endif /* BF_H_ */
