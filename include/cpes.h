/*
 * cpes.h -- C ABI of the CoPES parameter-space hot path for AMD Instinct
 * MI355X (gfx950).
 *
 * CoPES ("Cooperative Coevolution for Resource-Constrained Agentic LLM
 * Post-Training", arXiv 2608.02391) is an evolution strategy over all
 * parameters of a model.  One step (Alg. 1) partitions the d parameters into K
 * disjoint subspaces (Eq. 7), evaluates seed-defined Gaussian perturbations of
 * one subspace at a time (Eq. 8, scale sigma_k of Eq. 11), standardises the
 * rewards of all members jointly (Eq. 12) and adds the reward-weighted noise
 * back to the parameters (Eq. 13; Eq. 6 for standard ES).  Noise is never
 * stored: every call regenerates it from the member's seed (Sec. 3.3 and
 * Supp. A.8, "Seed Replay and Chunking"), and the pre-perturbation weights are
 * restored from a backup rather than by subtraction ("CPU Weight Backup").
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Pointers named *_dev are device pointers (e.g. a torch tensor's data_ptr());
 * pointers named *_host are host pointers.  The caller owns every buffer; the
 * library keeps no pointer and no state between calls besides a thread-local
 * error string.  `stream` is a hipStream_t passed as void* (NULL = the null
 * stream).  Every call only enqueues work on `stream` and returns without
 * synchronising; a kernel failure surfaces at the caller's next
 * synchronisation.  Arguments are validated on the host before anything is
 * enqueued, so a call that returns an error has had no effect.  No call
 * allocates device memory; scratch space comes in through `workspace`.
 * Results depend only on the arguments (not on the stream, launch geometry or
 * run).
 *
 * Weights are a flat buffer of `numel` elements of dtype CPES_BF16 or
 * CPES_F32.  A subspace (cpes_subspace) lists `length` positions j = 0 ..
 * length-1 -- the embedding P_k of Eq. 8.  Position j is parameter
 *   offset + j                                  (index == NULL),
 *   index[offset + j]                           (index != NULL, chunk == 0), or
 *   index[offset + j / chunk] * chunk + j % chunk
 *                                               (index != NULL, chunk > 0:
 *                                                the map names chunks of `chunk`
 *                                                consecutive parameters),
 * index being a device array of int64; an element map may instead be a
 * uint32 array (index32, models of at most 2^32 parameters).  Entries that
 * would address outside [0, numel) are skipped.
 *
 * Noise.  Position j of a subspace draws noise index i = noise_offset + j
 * (noise_offset = 0 for a whole subspace; a shard of one passes its start).
 * Noise index i of a member with seed s is
 *   eps_i = BoxMuller(Philox4x32-10(counter = (lo32 q, hi32 q, 0, 0),
 *                                   key = (lo32 s, hi32 s)), i mod 4),
 * q = i / 4: words (x0, x1) give indices 4q and 4q+1, words (x2, x3) give
 * 4q+2 and 4q+3; radius sqrt(-2 ln U(a)), angle 2 pi U(b), U(x) = ((x >> 8) +
 * 1) 2^-24; cosine for the even index, sine for the odd one; evaluated in
 * fp64 and rounded once to fp32.
 */
#ifndef CPES_H
#define CPES_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Raised when a call or a struct that was there changes; calls can be added without
 * (the ones that evaluate a member were): a program that may meet a library without
 * them looks the symbol up. */
#define CPES_ABI_VERSION 8

/* Exported symbols (the library is built with hidden default visibility). */
#define CPES_API __attribute__((visibility("default")))

/* Status codes returned by every int-valued entry point. */
enum cpes_status {
    CPES_OK = 0,
    CPES_ERR_INVALID_ARGUMENT = -1, /* a null, out-of-range or inconsistent argument */
    CPES_ERR_UNSUPPORTED = -2,      /* valid but beyond the library's limits (see each call) */
    CPES_ERR_WORKSPACE = -3,        /* workspace missing or smaller than required */
    CPES_ERR_HIP = -4,              /* the HIP runtime reported an error while enqueueing */
};

enum cpes_dtype { CPES_BF16 = 0, CPES_F32 = 1 };
enum cpes_partition_mode { CPES_PART_CONTIGUOUS = 0, CPES_PART_PERMUTATION = 1 };
enum cpes_aux_mode { CPES_AUX_NONE = 0, CPES_AUX_SNAPSHOT = 1, CPES_AUX_MASTER = 2, CPES_AUX_BACKUP = 3 };
enum cpes_norm_mode { CPES_NORM_Z = 0, CPES_NORM_RANK = 1 };
enum cpes_scale_mode { CPES_SCALE_ALPHA_OVER_N_SIGMA = 0, CPES_SCALE_ALPHA_OVER_N = 1 };

/* Limits of the library. */
#define CPES_MAX_MEMBERS 256         /* members per cpes_update call */
#define CPES_MAX_REWARDS 4096        /* rewards per cpes_normalize_rewards call */
#define CPES_MAX_GROUPS 1024         /* reward groups per cpes_normalize_rewards call */
#define CPES_MAX_PERMUTATION_K 256   /* subspaces of a CPES_PART_PERMUTATION partition */
#define CPES_MAX_STEP_SUBSPACES 32   /* subspaces per cpes_update_step call */
#define CPES_STATIC_MAX_CHUNKS (1 << 20) /* chunks per cpes_partition_chunks_static call */
#define CPES_MAX_HEAD_DIM 256        /* head dimension of a cpes_cache */
#define CPES_MAX_HEADS 65536         /* key-value heads of a cpes_cache, query heads of cpes_attend */
#define CPES_MAX_ALTERNATIVES 64     /* most likely tokens cpes_logprobs lists per row */
#define CPES_MAX_SEQUENCES (1 << 20) /* sequences listed per cpes_pages_* call, rows per cpes_attend call */
#define CPES_MAX_TREE 256            /* drafted tokens of one sequence in a tree (chains of cpes_attend_tree: any) */

typedef struct cpes_subspace {
    int64_t offset;          /* first parameter (no map) or first map entry */
    int64_t length;          /* number of positions d_k, >= 0 */
    const int64_t* index;    /* NULL, or device int64 map (parameters or chunk ids) */
    int64_t chunk;           /* 0, or a power of two >= 8: index entries name chunks of this size */
    const uint32_t* index32; /* NULL, or device uint32 map of parameters (half the map traffic
                                of `index`; models of at most 2^32 parameters); at most one of
                                index / index32, and chunk = 0 with index32 */
    int64_t noise_offset;    /* 0, or a multiple of 8: position j draws noise index
                                noise_offset + j.  A shard [a, b) of a subspace is
                                {offset + a (or the map entry a), b - a, ..., noise_offset = a}
                                and gets exactly the noise, and the results, of those positions
                                of the whole subspace (a sharded update across GPUs). */
    int64_t flags;           /* 0, or CPES_SUB_ASCENDING (below) */
} cpes_subspace;

/* cpes_subspace.flags.  CPES_SUB_ASCENDING: the element map (index or
 * index32) is strictly ascending over the subspace's positions, as the maps
 * of cpes_partition and cpes_partition32 are.  With bf16 weights the
 * perturbations (cpes_perturb, every aux mode) and the restores (cpes_restore
 * from a backup or a master, cpes_restore_from_host) may then read and write
 * whole 128-byte lines of the weights around the subspace's entries (once
 * each), writing the other parameters of those lines back with the values
 * just read, instead of storing the entries one by one: on a dense subspace
 * almost every line is then written in full rather than partially.  Results
 * are those of the entry-by-entry path, provided nothing else writes the same
 * weights while the call runs; with a map that is not strictly ascending they
 * are undefined (every access stays within w, the map and the side buffer).
 * Ignored for other calls, contiguous and chunked subspaces and fp32
 * weights. */
#define CPES_SUB_ASCENDING 1

/*
 * cpes_partition -- subspaces of Eq. (7): disjoint, covering all d indices,
 * sizes d/K (differing by at most one when K does not divide d).  The paper
 * resamples the partition every step from a stored seed and replays it
 * (Sec. 3.3, Supp. A.8 "Partition Replay").
 *
 * mode CPES_PART_CONTIGUOUS: offsets_host[k] = bounds_host[k] (K+1 values,
 *   non-decreasing from 0 to d) or, with bounds_host == NULL, floor(k d / K).
 *   Subspace k is the parameter range [offsets[k], offsets[k+1]).  Host only:
 *   nothing is enqueued, index_dev / workspace may be NULL.
 * mode CPES_PART_PERMUTATION: element i belongs to subspace
 *   floor(E(i) K / d), where E is a keyed pseudo-random permutation of [0, d):
 *   an 8-round balanced Feistel network on b = max(2, ceil(log2 d)) (rounded
 *   up to even) bits whose round r function is word 0 of the Philox block
 *   (counter (R, r, 3, 0), key seed) masked to b/2 bits, restricted to [0, d)
 *   by cycle-walking.  index_dev (device int64[d]) receives, for each k, the
 *   members of subspace k in ascending order at [offsets[k], offsets[k+1]),
 *   and offsets_host[k] = ceil(k d / K) (exact because E is a bijection).
 *   While the call runs the map's memory also holds intermediate tables, so
 *   its entries are undefined until it ends, also where the same map is replayed.
 *   Requires 1 <= K <= CPES_MAX_PERMUTATION_K, d < 2^55 and a device workspace of
 *   cpes_partition_workspace_bytes() bytes (16-byte aligned).
 * status_dev: NULL, or a device int32 set to 0, or to 1 if a cycle walk
 *   exceeded its bound (cannot happen for a bijection; a safety net).
 * Errors: d < 1 or d >= 2^62, K < 1 or K > d, bad bounds, mode unknown,
 *   index_dev NULL for PERMUTATION -> CPES_ERR_INVALID_ARGUMENT; K above the
 *   limit -> CPES_ERR_UNSUPPORTED; workspace too small -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_partition(int mode, int64_t d, int32_t K, uint64_t seed, const int64_t* bounds_host,
                   int64_t* offsets_host, int64_t* index_dev, void* workspace_dev,
                   size_t workspace_bytes, int32_t* status_dev, void* stream);

/*
 * cpes_partition32 -- the CPES_PART_PERMUTATION partition of cpes_partition
 * written as a uint32 map (index_dev: device uint32[d]) for d <= 2^32: half
 * the memory and half the map traffic of the int64 map, same entries.  Use it
 * through cpes_subspace.index32.  Workspace as
 * cpes_partition_workspace_bytes(CPES_PART_PERMUTATION, d, K).
 * Errors: d < 1 or d > 2^32, K < 1 or K > d, null pointers ->
 *   CPES_ERR_INVALID_ARGUMENT; otherwise as cpes_partition.
 */
CPES_API int cpes_partition32(int64_t d, int32_t K, uint64_t seed, int64_t* offsets_host, uint32_t* index_dev,
                     void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream);

/* Workspace bytes cpes_partition needs (0 for CONTIGUOUS); 0 for invalid arguments. */
CPES_API size_t cpes_partition_workspace_bytes(int mode, int64_t d, int32_t K);

/*
 * cpes_partition_chunks -- the chunk-granular random partition the paper runs
 * (Sec. 3.3; Supp. A.8 "Partition Replay": the assignment of chunks to
 * subspaces is replayed from a stored seed).  The d parameters form n_chunks = ceil(d /
 * chunk) chunks of `chunk` consecutive parameters (the last may be shorter);
 * chunk c belongs to subspace floor(E(c) K / n_chunks), E being the keyed
 * permutation of cpes_partition (CPES_PART_PERMUTATION) on [0, n_chunks).
 *   chunks_dev (device int64[n_chunks]) receives the chunk ids of each
 *   subspace, ascending, at [list_offsets[k], list_offsets[k+1]);
 *   list_offsets_host[k] = ceil(k n_chunks / K) (host, K+1);
 *   lengths_host[k] = parameters in subspace k (host, K; they sum to d).
 * Subspace k is then cpes_subspace{list_offsets[k], lengths[k], chunks_dev,
 * chunk}: every 16-byte unit is contiguous, so kernels stream it at full
 * bandwidth.  chunk must be a power of two, 8 <= chunk <= 2^30; 1 <= K <=
 * min(n_chunks, CPES_MAX_PERMUTATION_K); workspace as
 * cpes_partition_chunks_workspace_bytes(); status_dev as cpes_partition.
 */
CPES_API int cpes_partition_chunks(int64_t d, int64_t chunk, int32_t K, uint64_t seed,
                                   int64_t* list_offsets_host, int64_t* lengths_host, int64_t* chunks_dev,
                                   void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                                   void* stream);

/*
 * cpes_partition_chunks_static -- cpes_partition_chunks with no workspace
 * argument and no allocation of any kind, for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Its scratch space is a file-scope device array of
 * the library (2,621,696 bytes: room for n_chunks <= CPES_STATIC_MAX_CHUNKS
 * and K <= CPES_MAX_PERMUTATION_K), which every GPU the library runs on holds
 * until the process ends.  The first call on a device looks up that device's
 * copy (hipGetSymbolAddress; not a stream operation, so make that first call
 * outside a graph capture).  All calls on one GPU share the array and each
 * leaves its contents behind: calls that overlap in time on one GPU (other
 * streams or threads) race and must be serialised by the caller.  Nothing in
 * it needs to start at zero: every call writes each scratch entry before
 * reading it.
 * Arguments, outputs and results as cpes_partition_chunks (bit-identical).
 * Errors: as cpes_partition_chunks; more than CPES_STATIC_MAX_CHUNKS chunks
 *   -> CPES_ERR_UNSUPPORTED; the address lookup failing -> CPES_ERR_HIP.
 */
CPES_API int cpes_partition_chunks_static(int64_t d, int64_t chunk, int32_t K, uint64_t seed,
                                          int64_t* list_offsets_host, int64_t* lengths_host, int64_t* chunks_dev,
                                          int32_t* status_dev, void* stream);

/* Workspace bytes cpes_partition_chunks needs; 0 for invalid arguments. */
CPES_API size_t cpes_partition_chunks_workspace_bytes(int64_t d, int64_t chunk, int32_t K);

/*
 * cpes_perturb -- theta_{k,i} = theta + sigma_k P_k eps_{k,i} (Eq. 8, Alg. 1),
 * in place on the subspace `s` of w (numel elements of `dtype`):
 *   w[p(j)] = cast(fmaf(sign * sigma, eps_j(seed), src_j)),  j < s->length,
 * one fp32 fused multiply-add, then round-to-nearest-even for bf16.
 * sigma is the effective scale sigma_k = sigma sqrt(d / d_k) (Eq. 11);
 * sign is +1 or -1 (mirrored pairs).
 *   aux_mode CPES_AUX_NONE:     src_j = w[p(j)]; aux ignored.
 *   aux_mode CPES_AUX_SNAPSHOT: src_j = w[p(j)], and aux (device, dtype of w,
 *                               s->length elements) receives aux[j] = w[p(j)]
 *                               before the change: the weight backup.
 *   aux_mode CPES_AUX_MASTER:   src_j = ((const float*)aux)[j], an fp32 master
 *                               of the subspace (CPES_BF16 weights only).
 *   aux_mode CPES_AUX_BACKUP:   src_j = aux[j], an existing backup (dtype of w)
 *                               of the unperturbed subspace, read only; w is
 *                               not read.  Equal to restoring from the backup
 *                               and then perturbing, in one pass.  Every member
 *                               of a step perturbs the same pre-update weights,
 *                               so one backup serves all of them.
 * Parameters outside the subspace keep their values (through a map flagged
 * CPES_SUB_ASCENDING, bf16 lines around the entries are rewritten with the
 * values just read; see cpes_subspace.flags).
 * Errors: w NULL, s NULL, length < 0, contiguous range beyond numel, dtype /
 *   aux_mode unknown, aux NULL when needed, sign not +-1, sigma negative or
 *   not finite, MASTER with fp32 weights -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_perturb(void* w_dev, int64_t numel, int dtype, const cpes_subspace* s, float sigma,
                 uint64_t seed, int32_t sign, void* aux_dev, int aux_mode, void* stream);

/*
 * cpes_restore -- undo a perturbation (Sec. 3.3):
 *   CPES_AUX_SNAPSHOT: w[p(j)] = aux[j] (bit copy; exact).
 *   CPES_AUX_MASTER:   w[p(j)] = rne_bf16(((const float*)aux)[j]) (exact when
 *                      the master was staged from w).
 *   CPES_AUX_NONE:     replay: w[p(j)] = cast(fmaf(-sign * sigma, eps_j, w[p(j)])).
 *                      Not an identity in floating point; the paper's reason for
 *                      keeping a backup.  Differs by at most one fp32 ulp (more
 *                      after bf16 rounding).
 * Arguments and errors as cpes_perturb (sigma, seed, sign only used by NONE).
 */
CPES_API int cpes_restore(void* w_dev, int64_t numel, int dtype, const cpes_subspace* s, float sigma,
                 uint64_t seed, int32_t sign, const void* aux_dev, int aux_mode, void* stream);

/*
 * cpes_backup_to_host -- backup_host[j] = w[p(j)] (bit copy), the weight
 * backup in host memory (Sec. 3.3; Supp. A.8, CPU weight backup): the
 * pre-perturbation weights of the subspace leave the GPU, so the backup adds
 * no device-resident copy.
 * cpes_restore_from_host -- w[p(j)] = backup_host[j] (bit copy), the restore
 * after each perturbed-model evaluation.
 *   backup_host: s->length elements of `dtype`, PINNED host memory the device
 *                can address (hipHostMalloc, or a torch tensor made with
 *                pin_memory=True); owned by the caller, who keeps it alive and
 *                unmodified until the work on `stream` has finished.
 * A contiguous subspace moves as one DMA copy on `stream`; an index-map or
 * chunked subspace is gathered / scattered by a kernel that reads or writes
 * the pinned buffer over the host link.  Both are asynchronous on `stream`.
 * Errors: as cpes_perturb for w and s; backup_host NULL or not pinned host
 *   memory (pageable, or device memory) -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_backup_to_host(const void* w_dev, int64_t numel, int dtype, const cpes_subspace* s,
                        void* backup_host, void* stream);
CPES_API int cpes_restore_from_host(void* w_dev, int64_t numel, int dtype, const cpes_subspace* s,
                           const void* backup_host, void* stream);

/*
 * cpes_backup -- backup_dev[j] = w[p(j)] (bit copy), the weight backup of
 * Sec. 3.3 taken on its own, in device memory: for a subspace whose members
 * are perturbed from another source (an fp32 master) but restored from a copy
 * of the weights.  (A member's perturbation can also take the backup itself:
 * cpes_perturb with CPES_AUX_SNAPSHOT.)
 *   backup_dev: s->length elements of `dtype` in device memory, caller-owned;
 *               it must not overlap w.
 * Errors: as cpes_perturb for w and s; backup_dev NULL -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_backup(const void* w_dev, int64_t numel, int dtype, const cpes_subspace* s, void* backup_dev,
                void* stream);

/*
 * cpes_stage_master -- master_dev[j] = fp32 value of w[p(j)] (exact), the fp32
 * master copy of the active subspace kept while its bf16 weights are
 * perturbed and updated.  Errors as cpes_perturb.
 */
CPES_API int cpes_stage_master(const void* w_dev, int64_t numel, int dtype, const cpes_subspace* s,
                      float* master_dev, void* stream);

/*
 * cpes_normalize_rewards -- reward standardisation.
 *   CPES_NORM_Z:    Eq. (5) / Eq. (12): mu = sum r / n, s = sqrt(sum (r - mu)^2 / n)
 *                   (population std, sums in fp64 in a fixed order);
 *                   out = (r - mu) / s, or 0 for every member when s == 0.
 *   CPES_NORM_RANK: centred average rank a / (n - 1) - 1/2 with a the 0-based
 *                   rank and ties sharing the mean of their ranks; 0 when n == 1.
 * group_dev == NULL standardises all n rewards jointly (Eq. 12).  Otherwise
 * group_dev (device int32[n], values in [0, n_groups)) standardises each group
 * on its own (independent standardisation, the ablation of Sec. 4.4).
 * r_dev and out_dev are device float32[n] and may alias.  status_dev (NULL or
 * device int32) receives 0, 1 if a reward is not finite, or 2 if a group id is
 * out of range; in both failure cases every output is 0 (so an update leaves
 * the weights unchanged).
 * Errors: NULL r_dev / out_dev, n outside [1, CPES_MAX_REWARDS], unknown mode,
 *   n_groups outside [1, n] with group_dev given -> CPES_ERR_INVALID_ARGUMENT;
 *   n_groups above CPES_MAX_GROUPS -> CPES_ERR_UNSUPPORTED.
 */
CPES_API int cpes_normalize_rewards(const float* r_dev, int32_t n, int mode, const int32_t* group_dev,
                           int32_t n_groups, float* out_dev, int32_t* status_dev, void* stream);

/*
 * cpes_update -- seed-replayed ES update of one subspace (Eq. 6 / Eq. 13;
 * Sec. 3.3):  theta_S += step * sum_i sign_i * rnorm_i * eps(seed_i),
 *   step = alpha / (n * sigma)   (CPES_SCALE_ALPHA_OVER_N_SIGMA, OpenAI-ES form)
 *   step = alpha / n             (CPES_SCALE_ALPHA_OVER_N, the paper's form with
 *                                 n = N_k members of this subspace).
 * seeds_host / signs_host (host, n entries; signs +-1) describe the members in
 * the order their rewards appear in rnorm_dev (device float32[n], typically
 * the output of cpes_normalize_rewards).  Members sharing a seed (mirrored
 * pairs) share one noise vector, which is generated once with coefficient
 * sum(sign * rnorm).  Each weight is read once and written once; the weighted
 * noise sum is accumulated in fp64 in order of first appearance of each seed
 * and rounded once to fp32.
 *   master_dev == NULL: w[p(j)] = cast(fmaf(step, acc_j, w[p(j)])).
 *   master_dev != NULL: master[j] = fmaf(step, acc_j, master[j]) and
 *                       w[p(j)] = cast(master[j]) (device float32[length]).
 * Errors: NULL pointers, n outside [1, CPES_MAX_MEMBERS] (UNSUPPORTED above),
 *   a sign not +-1, alpha or sigma not finite, sigma <= 0 with the
 *   OVER_N_SIGMA scale, dtype / scale_mode unknown, contiguous range beyond
 *   numel -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_update(void* w_dev, int64_t numel, int dtype, const cpes_subspace* s, float* master_dev,
                int32_t n, const uint64_t* seeds_host, const int8_t* signs_host,
                const float* rnorm_dev, float alpha, float sigma, int scale_mode, void* stream);

/*
 * cpes_update_step -- the whole CoPES update of one step in one launch
 * (Eq. 13; Alg. 1, after joint standardisation): for every subspace k of a
 * partition,  theta_{S_k} += step_k * sum_{i in members of k} sign_i rnorm_i eps(seed_i),
 *   step_k = alpha / (n_k sigma_k)  (CPES_SCALE_ALPHA_OVER_N_SIGMA) or
 *   step_k = alpha / n_k            (CPES_SCALE_ALPHA_OVER_N; Eq. 13 with n_k = N_k),
 * where n_k counts the members of subspace k.  With K = 1 and alpha / N this
 * is the standard ES update of Eq. 6.  Subspaces are disjoint, so the result
 * equals K cpes_update calls in any order.
 * offsets_host (K+1, non-decreasing): subspace k is positions [offsets[k],
 *   offsets[k+1]) -- parameters themselves (index_dev == NULL; offsets[K] <=
 *   numel) or entries of the int64 device map index_dev (e.g. the output of
 *   cpes_partition; a uint32 map goes to cpes_update_step32).  Noise
 *   position j is counted from offsets[k].
 *   With chunk > 0, index_dev holds chunk ids (cpes_partition_chunks),
 *   subspace k is cpes_subspace{offsets[k], lengths_host[k], index_dev, chunk}
 *   and lengths_host (host, K) is required; otherwise lengths_host is ignored.
 * seeds_host / signs_host / subspace_host (host, n entries): member i has seed,
 *   sign +-1 and the subspace it perturbed; rnorm_dev (device float32[n]) its
 *   standardised reward (joint or per group, cpes_normalize_rewards).
 *   Members of one subspace sharing a seed share one noise stream.
 * sigma_host (host, K): the effective sigma_k each subspace was perturbed with.
 * Subspaces without members are left unchanged.  Each weight is read and
 * written once; accumulation in fp64 as in cpes_update.
 * Errors: NULL pointers, K < 1, n < 1, a sign not +-1, a member's subspace
 *   outside [0, K), decreasing offsets, contiguous range beyond numel, alpha
 *   not finite, sigma_k <= 0 for a subspace with members under the
 *   OVER_N_SIGMA scale -> CPES_ERR_INVALID_ARGUMENT; K above
 *   CPES_MAX_STEP_SUBSPACES or n above CPES_MAX_MEMBERS -> CPES_ERR_UNSUPPORTED.
 */
CPES_API int cpes_update_step(void* w_dev, int64_t numel, int dtype, int32_t K, const int64_t* offsets_host,
                              const int64_t* index_dev, int64_t chunk, const int64_t* lengths_host,
                              int32_t n, const uint64_t* seeds_host,
                              const int8_t* signs_host, const int32_t* subspace_host, const float* rnorm_dev,
                              float alpha, const float* sigma_host, int scale_mode, void* stream);

/*
 * cpes_update_step32 -- cpes_update_step over a uint32 element map
 * (index32_dev, e.g. the output of cpes_partition32; models of at most 2^32
 * parameters): subspace k is entries [offsets[k], offsets[k+1]) of the map.
 * Half the map traffic of the int64 map, same result.  No chunk lists.
 * Arguments and errors otherwise as cpes_update_step; index32_dev NULL ->
 * CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_update_step32(void* w_dev, int64_t numel, int dtype, int32_t K, const int64_t* offsets_host,
                                const uint32_t* index32_dev, int32_t n, const uint64_t* seeds_host,
                                const int8_t* signs_host, const int32_t* subspace_host, const float* rnorm_dev,
                                float alpha, const float* sigma_host, int scale_mode, void* stream);

/* ---------------- evaluating a member ----------------------------------- *
 *
 * Between a member's perturbation and its restore the perturbed model is
 * evaluated: rollouts are generated token by token and their tokens scored.
 * The calls below are that evaluation's operators next to the model's plain
 * matrix products.  The conventions are those above; in addition:
 *   - sequence lengths, page tables and reference counts live in device
 *     memory and are read there when the work runs, so a captured graph can be
 *     replayed as sequences grow.  Nothing on the device is trusted to address
 *     memory: page ids outside [0, pages), sequence ids outside [0, sequences)
 *     and lengths beyond the table are caught there, as each call says.
 *   - calls that change one pool or cache, or read what another changes, must not
 *     overlap in time (one stream, or events between streams).
 *   - tensors start at any element; only cpes_cache has a rule for its rows. */

/*
 * Keys and values of `layers` layers in pages of `page_size` tokens.  Element d
 * of token t of head h in page p of layer l is at
 *   l * layer_stride + p * page_stride + h * head_stride + t * token_stride + d
 * (in elements, the same for keys and values), so pages may be head-major,
 * token-major or hold keys beside values.  head_dim: a multiple of 8 up to
 * CPES_MAX_HEAD_DIM; strides not negative.  Different (l, p, h, t) must not
 * overlap.
 */
typedef struct cpes_cache {
    void* k_dev;
    void* v_dev;
    int64_t layer_stride;
    int64_t page_stride;
    int64_t head_stride;
    int64_t token_stride;
    int32_t layers;
    int32_t pages;
    int32_t heads;          /* key-value heads */
    int32_t page_size;      /* tokens per page, any number >= 1 */
    int32_t head_dim;
    int32_t dtype;          /* CPES_BF16 or CPES_F32 */
} cpes_cache;

/*
 * The pages of `sequences` sequences: token j of sequence s lies in slot j %
 * page_size of page table[s * table_stride + j / page_size], j < lengths[s].
 * refs[p] counts the sequences that hold page p; a page is free while it is
 * not positive.  Entries of the table behind a sequence's last page mean
 * nothing.  A page held by several sequences is full: only the last, partly
 * filled page of a sequence is ever written to, and cpes_pages_fork copies it.
 */
typedef struct cpes_pool {
    int32_t* table_dev;     /* int32[sequences * table_stride] */
    int32_t* lengths_dev;   /* int32[sequences] */
    int32_t* refs_dev;      /* int32[pages]; NULL for calls that only read the cache through the table */
    int64_t table_stride;   /* >= width */
    int32_t sequences;
    int32_t width;          /* pages a sequence can hold */
    int32_t pages;
    int32_t page_size;
} cpes_pool;

/* What the page calls report in status_dev (NULL, or a device int32).  A call
 * overwrites it: where several run before it is looked at, each has its own, or
 * the largest is kept. */
enum cpes_pages_status {
    CPES_PAGES_OK = 0,
    CPES_PAGES_SHORT = 1,       /* not enough free pages: nothing was changed */
    CPES_PAGES_BAD_SEQUENCE = 2 /* a sequence id, length or state the call does not allow: nothing was changed */
};

/* Workspace bytes of cpes_pages_reserve, cpes_pages_fork and cpes_pages_compact
 * on a pool of `pages` pages; 0 for pages < 1. */
CPES_API size_t cpes_pages_workspace_bytes(int32_t pages);

/*
 * cpes_pages_reserve -- room for the next tokens: sequence seqs[i] grows to
 * new_lengths[i] tokens (device int32[n] each).  The pages it lacks are the
 * free pages of lowest id, handed out in the order of the list; a length not
 * above the present one leaves the sequence as it is.  All or nothing: too few
 * free pages give status CPES_PAGES_SHORT, a sequence id out of range or listed
 * twice, or a length that is negative or beyond the table's width,
 * CPES_PAGES_BAD_SEQUENCE, and then nothing has changed.
 * Errors: null pointers, n < 0, n > sequences -> CPES_ERR_INVALID_ARGUMENT; n above
 *   CPES_MAX_SEQUENCES -> CPES_ERR_UNSUPPORTED; workspace too small or not 16-byte
 *   aligned -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_pages_reserve(const cpes_pool* pool, int32_t n, const int32_t* seqs_dev,
                                const int32_t* new_lengths_dev, void* workspace_dev, size_t workspace_bytes,
                                int32_t* status_dev, void* stream);

/*
 * cpes_pages_fork -- children[i], an empty sequence (length 0), becomes a copy of
 * parents[i] (device int32[n] each; a parent may occur many times): full pages
 * are shared and their reference counts raised, a partly filled last page is
 * copied, in every layer of the cache, to the free page of lowest id, handed
 * out in the order of the list.  All or nothing, as cpes_pages_reserve: a child
 * that is not empty or listed twice, or an id out of range, gives
 * CPES_PAGES_BAD_SEQUENCE.  A listed child is no parent in the same call (it
 * counts as empty).
 * Errors: as cpes_pages_reserve; a cache that does not fit the pool (pages,
 *   page size) or breaks the rules of cpes_cache -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_pages_fork(const cpes_cache* cache, const cpes_pool* pool, int32_t n, const int32_t* parents_dev,
                             const int32_t* children_dev, void* workspace_dev, size_t workspace_bytes,
                             int32_t* status_dev, void* stream);

/*
 * cpes_pages_free -- sequences seqs[i] (device int32[n]) give their pages up: each
 * page's reference count falls by one, their table entries become -1, their
 * lengths 0.  A sequence listed twice is freed once; ids out of range are
 * skipped and give CPES_PAGES_BAD_SEQUENCE.
 * Errors: null pointers, n < 0 -> CPES_ERR_INVALID_ARGUMENT; n above
 *   CPES_MAX_SEQUENCES -> CPES_ERR_UNSUPPORTED.
 */
CPES_API int cpes_pages_free(const cpes_pool* pool, int32_t n, const int32_t* seqs_dev, int32_t* status_dev,
                             void* stream);

/*
 * cpes_pages_copy -- page dst[i] of every layer becomes a copy of page src[i]
 * (device int32[n] each).  Pairs with an id outside [0, pages) are skipped; a
 * page that is both a source and a destination, or a destination twice, has
 * undefined contents.
 * Errors: null pointers, n < 0, a bad cache -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_pages_copy(const cpes_cache* cache, int32_t n, const int32_t* src_dev, const int32_t* dst_dev,
                             void* stream);

/*
 * cpes_pages_compact -- the L live pages (refs > 0) move to page ids below L, so
 * that the rest of the cache can be used for something else (the next weight
 * backup).  Live pages with ids >= L move, in ascending order, into the free
 * ids below L in ascending order; all others stay.  `packed` receives the
 * table, lengths and reference counts with the new ids; its tensors may be
 * those of `pool` (in place).  moved_dev: NULL, or a device int32 that receives
 * the number of pages moved.
 * Errors: null pointers, `packed` of another shape than `pool`, a cache that
 *   does not fit -> CPES_ERR_INVALID_ARGUMENT; workspace as cpes_pages_reserve.
 */
CPES_API int cpes_pages_compact(const cpes_cache* cache, const cpes_pool* pool, const cpes_pool* packed,
                                void* workspace_dev, size_t workspace_bytes, int32_t* moved_dev, void* stream);

/* Workspace bytes of cpes_pages_keep on up to `n` sequences with up to `longest`
 * drafted tokens each; 0 for n < 0 or a `longest` outside [1, CPES_MAX_TREE]. */
CPES_API size_t cpes_pages_keep_workspace_bytes(int32_t n, int32_t longest);

/*
 * cpes_pages_keep -- drafted tokens that were not confirmed leave the cache.  The
 * newest T = starts[i + 1] - starts[i] tokens of sequence seqs[i] (device int32[n];
 * NULL: i) are drafted ones, in the order in which they entered the cache; the
 * first kept[i] entries of path[i * longest ..] (device int32[n * longest], as
 * cpes_tree_accept leaves them) are the ones that stay, ascending in [0, T).  Their
 * keys and values move together, in every layer, behind the tokens in front of the
 * drafted ones; the sequence's length falls by T - kept[i], and the pages it then
 * no longer needs are given back (table entries -1, reference counts one lower).
 * All or nothing: a sequence id out of range or listed twice, starts (device
 * int32[n + 1]) that fall or lie more than `longest` apart, a sequence shorter than
 * its drafted tokens or of a length that is negative or beyond its table, kept outside
 * [0, T] or a path that does not ascend in [0, T) give CPES_PAGES_BAD_SEQUENCE, and then
 * nothing has changed.  A token whose table entry names no page moves nowhere.
 * Pages with drafted tokens belong to one sequence: a fork in between shares them,
 * and leaves either's contents undefined.
 * Errors: as cpes_pages_fork; null pointers, longest < 1 -> CPES_ERR_INVALID_ARGUMENT;
 *   longest above CPES_MAX_TREE -> CPES_ERR_UNSUPPORTED; workspace, as
 *   cpes_pages_keep_workspace_bytes, too small or not 16-byte aligned -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_pages_keep(const cpes_cache* cache, const cpes_pool* pool, int32_t n, const int32_t* seqs_dev,
                             const int32_t* starts_dev, int32_t longest, const int32_t* kept_dev,
                             const int32_t* path_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                             void* stream);

/*
 * cpes_cache_append -- the keys and values of n new tokens enter their pages in
 * one layer: token i belongs to sequence seqs[i] (device int32[n]; NULL: i) and
 * position positions[i] (device int32[n]); element d of head h of token i is
 * k_new[i * new_stride + h * new_head_stride + d], and the same of v_new.  Bit
 * copies.  Tokens whose sequence or position is outside the table, or whose table
 * entry names no page, are skipped.  The table alone decides, not the length: a
 * table that was filled with -1 has no page for a token whose reservation failed.
 * Two tokens at one place leave parts of either.
 * Errors: null pointers, n < 0, a layer out of range, negative strides, a bad
 *   cache or a pool that does not fit it -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_cache_append(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t n,
                               const int32_t* seqs_dev, const int32_t* positions_dev, const void* k_new_dev,
                               const void* v_new_dev, int64_t new_stride, int64_t new_head_stride, void* stream);

/* Workspace bytes of cpes_attend on up to `rows` rows (0 for invalid arguments). */
CPES_API size_t cpes_attend_workspace_bytes(int32_t rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim);

/*
 * cpes_attend -- attention of one new token per row over the paged cache of one
 * layer.  Row r asks for sequence s = seqs[r] (device int32[rows]; NULL: r),
 * whose newest token, at position n - 1 with n = lengths[s], is the one asking
 * (its own key and value are in the cache).  It sees the positions
 *   j < n,  and with window > 0 only  j >= n - window  or  j < sinks.
 * Query head i of key-value head h = i / (q_heads / heads), q at
 * q[r * q_stride + i * q_head_stride + d]:
 *   x_j = scale * sum_d q_d k_j,d;  out_d = sum_j e^(x_j) v_j,d / sum_j e^(x_j);
 *   lse = ln sum_j e^(x_j)  (lse_dev: NULL, or device float32[rows * q_heads]).
 * One pass over the keys and values with a running maximum; the maximum, the
 * sums and the output are held in fp32, and the weights of bf16 values carry 16
 * bits of mantissa into the matrix instructions.  out has the cache's dtype:
 * element d of head i of row r at out[r * out_stride + i * out_head_stride + d].
 * Of a sequence the first 2^31 - 65 positions count.  A row that sees nothing (an
 * empty sequence, an id out of range) gets out = 0 and lse = -inf, as does one
 * whose scores are all -inf; positions whose table entry names no page are not
 * seen.  The result does not depend on the contents of unseen positions, nor on
 * the run.  Where a value that is seen is infinite, its dim of out is that infinity or, of
 * a bf16 cache (whose weights go in as two numbers, the second of any sign), NaN.
 * workspace: as cpes_attend_workspace_bytes, 16-byte aligned; needs no
 * particular contents, and calls that overlap in time need their own.
 * Errors: null pointers, rows < 0, q_heads not a positive multiple of the
 *   cache's heads, a layer out of range, window or sinks negative, scale not
 *   finite, negative strides, a bad cache or a pool that does not fit it ->
 *   CPES_ERR_INVALID_ARGUMENT; rows above CPES_MAX_SEQUENCES ->
 *   CPES_ERR_UNSUPPORTED; workspace -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_attend(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t rows,
                         const int32_t* seqs_dev, const void* q_dev, int64_t q_stride, int64_t q_head_stride,
                         int32_t q_heads, float scale, int32_t window, int32_t sinks, void* out_dev,
                         int64_t out_stride, int64_t out_head_stride, float* lse_dev, void* workspace_dev,
                         size_t workspace_bytes, void* stream);

/* Workspace bytes of cpes_attend_tree on up to `rows` sequences with up to `tokens` new
 * tokens in all and `longest` each (0 for invalid arguments). */
CPES_API size_t cpes_attend_tree_workspace_bytes(int32_t rows, int32_t tokens, int32_t longest, int32_t q_heads,
                                                 int32_t kv_heads, int32_t head_dim);

/*
 * cpes_attend_tree -- attention of several new tokens per sequence over the paged
 * cache of one layer: a tree of drafted tokens, or a chain of them (a prompt, or a
 * piece of one).  Row r asks for sequence s = seqs[r] (device int32[rows]; NULL: r);
 * its new tokens are rows starts[r] .. starts[r + 1] - 1 of q and out (starts: device
 * int32[rows + 1]), T of them, and the newest T of the n = lengths[s] tokens in the
 * cache, in the same order (their keys and values are there).  Token i of a row
 * hangs from token parents[starts[r] + i] of it, one before it, or with -1 from the
 * b = n - T tokens in front of them (device int32[tokens]; any other number counts as
 * -1; NULL: from token i - 1).  With depth_i its number of ancestors in the tree, it
 * stands at position b + depth_i of its text and sees the b tokens in front, its
 * ancestors and itself; with window > 0 only those at positions p of that text with
 *   p > b + depth_i - window  or  p < sinks.
 * Scores, sums and outputs are those of cpes_attend (out, and lse: NULL, or device
 * float32[tokens * q_heads]), to which it gives the same results for trees of one
 * token up to roundings.  Of a sequence the first 2^31 - 65 positions count.  The
 * tokens of a sequence that has fewer than T, or of an id out of range, get out = 0
 * and lse = -inf; positions whose table entry names no page are not seen.  A row
 * whose starts fall, lie outside [0, tokens] or more than `longest` apart is left out;
 * where starts fall, tokens of other rows may be left out too, and tokens of two rows
 * get either's result.  What no row covers is left as it was.
 * The result of a token does not depend on the contents of positions it does not see
 * (other branches, too), nor on the run.  Infinite values that it sees make their dims
 * infinite or NaN, as in cpes_attend; which of them depends on the number of queries and
 * the place in a tile, the other dims and lse on neither.  Sums are of weights of up to
 * 2^4 before they are divided: of n positions seen, values above 2^124 / n may come out
 * infinite.
 * Any alignment of the cache and any finite scale will do; more than 32 queries of a row
 * and KV head are fastest where its keys and values, and their strides, lie at multiples
 * of 16 bytes, and |scale| in [1e-30, 1e30].
 * workspace: as cpes_attend_tree_workspace_bytes, 16-byte aligned; needs no
 * particular contents, and calls that overlap in time need their own.
 * Errors: as cpes_attend; tokens < 0, longest outside [1, tokens] with tokens > 0 ->
 *   CPES_ERR_INVALID_ARGUMENT; rows above CPES_MAX_SEQUENCES, longest above
 *   CPES_MAX_TREE with parents -> CPES_ERR_UNSUPPORTED.
 */
CPES_API int cpes_attend_tree(const cpes_cache* cache, int32_t layer, const cpes_pool* pool, int32_t rows,
                              const int32_t* seqs_dev, const int32_t* starts_dev, int32_t tokens, int32_t longest,
                              const int32_t* parents_dev, const void* q_dev, int64_t q_stride, int64_t q_head_stride,
                              int32_t q_heads, float scale, int32_t window, int32_t sinks, void* out_dev,
                              int64_t out_stride, int64_t out_head_stride, float* lse_dev, void* workspace_dev,
                              size_t workspace_bytes, void* stream);

/*
 * cpes_tree_accept -- which drafted tokens the model confirms.  Row r's tree is
 * tokens starts[r] .. starts[r + 1] - 1 of drafted and sampled (device int64[tokens]),
 * with parents as in cpes_attend_tree.  Token 0 of a row is no guess (the last step
 * sampled it) and always stays; from a token that stays the walk goes on to the lowest
 * one that hangs from it and is the token sampled behind it, drafted[j] == sampled[i],
 * and ends where there is none.
 *   kept_dev (device int32[rows]): tokens that stay; path_dev (device int32[rows *
 *   longest]): which, ascending, then -1; next_dev (device int64[rows]): the token
 *   sampled behind the last of them, the next step's token 0.
 * Where each sampled token comes from the model's own distribution behind its branch
 * (cpes_sample), the text is distributed as if nothing had been drafted.  Rows without
 * tokens, and rows whose starts fall, lie outside [0, tokens] or more than `longest`
 * apart, get kept = 0 and next = -1.
 * Errors: null pointers, rows < 0, tokens < 0, longest < 1 -> CPES_ERR_INVALID_ARGUMENT;
 *   rows above CPES_MAX_SEQUENCES, longest above CPES_MAX_TREE -> CPES_ERR_UNSUPPORTED.
 */
CPES_API int cpes_tree_accept(int32_t rows, const int32_t* starts_dev, int32_t tokens, int32_t longest,
                              const int32_t* parents_dev, const int64_t* drafted_dev, const int64_t* sampled_dev,
                              int32_t* kept_dev, int32_t* path_dev, int64_t* next_dev, void* stream);

/* Workspace bytes of cpes_logprobs on up to `rows` rows with up to `top`
 * alternatives, in either type: one sized for the largest batch serves it as its
 * rows end (0 for invalid arguments, or where none is needed). */
CPES_API size_t cpes_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top);

/*
 * cpes_logprobs -- scores of given tokens under rows of logits x (`dtype`, row r
 * at x + r * stride, `vocab` entries), with z = scale * x (scale = 1 /
 * temperature):
 *   lse = ln sum_v e^(z_v);  logp = z_target - lse;  entropy = -sum_v p_v ln p_v,
 *   p_v = e^(z_v - lse);
 *   alternatives: the `top` tokens of largest x in descending order, ties by the
 *   lowest token, and their log probabilities.
 * targets_dev: device int64[rows]; a target outside [0, vocab) scores 0, in any row.
 * logp_dev, entropy_dev, lse_dev: NULL, or device float32[rows].
 * stats_dev: NULL, or device float32[2 * rows]: max x and ln sum_v e^(z_v - scale
 *   max x), what cpes_logprobs_backward needs.
 * top_logp_dev / top_ids_dev: device float32 / int64[rows * top] (NULL with top
 *   = 0); entries behind the vocabulary's end are -inf and -1.
 * Each logit is read once.  Sums are fp32 within a thread and a workgroup.
 * Logits of -inf have probability 0; a row of nothing but -inf has lse = -inf,
 * entropy 0 and log probabilities -inf.  A NaN or +inf, whatever stands beside it,
 * makes the row's numbers NaN and its alternatives -1.
 * Errors: x NULL, rows < 0, vocab < 1, stride < vocab with more than one row,
 *   scale not positive or above FLT_MAX / 2, logp without targets, top outside [0,
 *   CPES_MAX_ALTERNATIVES] or without both outputs -> CPES_ERR_INVALID_ARGUMENT;
 *   workspace -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_logprobs(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale,
                           const int64_t* targets_dev, float* logp_dev, float* entropy_dev, float* lse_dev,
                           float* stats_dev, int32_t top, float* top_logp_dev, int64_t* top_ids_dev,
                           void* workspace_dev, size_t workspace_bytes, void* stream);

/*
 * cpes_logprobs_backward -- the gradient of cpes_logprobs' logp and entropy with
 * respect to the logits:
 *   dx_v = scale * (d_logp * ([v = target] - p_v) - d_entropy * p_v (ln p_v + entropy)),
 * from the forward call's stats and entropy and the upstream gradients d_logp,
 * d_entropy (device float32[rows]; either may be NULL, for zero).  dx has the
 * dtype of x, row r at dx + r * dx_stride, and may be x itself.  The targets
 * of rows outside [0, vocab) give no gradient of logp, a row of nothing but -inf
 * gives 0.  Computed in fp32, rounded once.
 * Errors: null pointers (targets needed with d_logp, entropy with d_entropy),
 *   sizes and scale as cpes_logprobs -> CPES_ERR_INVALID_ARGUMENT.
 */
CPES_API int cpes_logprobs_backward(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride,
                                    float scale, const int64_t* targets_dev, const float* stats_dev,
                                    const float* entropy_dev, const float* d_logp_dev, const float* d_entropy_dev,
                                    void* dx_dev, int64_t dx_stride, void* stream);

/* Workspace bytes of cpes_sample on up to `rows` rows in either type (0 for invalid
 * arguments, or where none is needed). */
CPES_API size_t cpes_sample_workspace_bytes(int32_t rows, int32_t vocab);

/*
 * cpes_sample -- a token for each row of logits x (`dtype`, row r at x + r * stride,
 * `vocab` entries) from a given number u = uniforms[r] (device float32[rows], in [0,
 * 1)).  With z = scale * x (scale = 1 / temperature) and w_v = e^(z_v - max z), in
 * the order of descending x, ties by the lowest token:
 *   top_k > 0:  only the first top_k tokens stay;
 *   top_p < 1:  of these only the ones in front of which less than top_p of their
 *               weight lies (the fewest that reach it, one at least);
 *   min_p > 0:  of these only the ones with ln w_v >= ln min_p.
 * token = the lowest v of those that stay with sum_{v' <= v} w_v' > u sum w, and
 * logp = ln(w_token / sum w), both sums over those that stay.  Weights and sums are in
 * 64 bits (of 37 bits and more; below 2^-52 of the largest one a weight counts as 0): a
 * token is off its place only where u is within their roundings of a border.  top_k = 1
 * takes the most likely token.  A u below 0 or NaN counts as 0, one of 1 or more takes
 * the last token that has a weight.
 * tokens_dev: device int64[rows]; logp_dev: NULL, or device float32[rows].
 * Logits of -inf are never chosen; a row of nothing but -inf has token -1 and logp
 * -inf, one with a NaN or +inf token -1 and logp NaN.
 * workspace: 16-byte aligned; needs no particular contents, and calls that overlap in
 * time need their own.
 * Errors: x, uniforms or tokens NULL, rows < 0, vocab < 1, stride < vocab with more than
 *   one row, scale not positive or above FLT_MAX / 2, top_k < 0, top_p outside (0, 1],
 *   min_p outside [0, 1] -> CPES_ERR_INVALID_ARGUMENT; workspace -> CPES_ERR_WORKSPACE.
 */
CPES_API int cpes_sample(const void* x_dev, int dtype, int32_t rows, int32_t vocab, int64_t stride, float scale,
                         int32_t top_k, float top_p, float min_p, const float* uniforms_dev, int64_t* tokens_dev,
                         float* logp_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

/* ---------------- test hooks and measurement utilities ------------------ */

/* out_dev[4 b + t] = word t of the Philox block q0 + b of stream (seed, domain),
 * b < nblocks.  Errors: out_dev NULL, nblocks < 0. */
CPES_API int cpes_debug_philox(uint64_t seed, uint32_t domain, uint64_t q0, int64_t nblocks,
                      uint32_t* out_dev, void* stream);

/* out_dev[k] = eps_{j0 + k}(seed) for k < n (the noise perturb/update use). */
CPES_API int cpes_debug_normals(uint64_t seed, int64_t j0, int64_t n, float* out_dev, void* stream);

/* The two halves of the normal transform on the grid m = m0 + k, k < n,
 * 1 <= m <= 2^24 (word (m - 1) << 8): rho_dev[k] = sqrt(-2 ln(m 2^-24)),
 * (cos_dev[k], sin_dev[k]) = (cos, sin)(pi m 2^-23), all fp64 (any may be
 * NULL), as the kernels evaluate them.  At m = 2^24 the radius comes out as
 * about 2^-200 instead of 0, which still gives a zero normal in fp32. */
CPES_API int cpes_debug_bm_grid(uint32_t m0, int64_t n, double* rho_dev, double* cos_dev,
                       double* sin_dev, void* stream);

/* The partition permutation of cpes_partition on i = i0 + k, k < n:
 * perm_dev[k] = E(i) (may be NULL), bucket_dev[k] = floor(E(i) K / d) (may be NULL). */
CPES_API int cpes_debug_prp(uint64_t seed, int64_t d, int32_t K, int64_t i0, int64_t n,
                   int64_t* perm_dev, int32_t* bucket_dev, void* stream);

/* RNG-only throughput probe: generates n normals (rounded up to a multiple
 * of 128) -- positions 0 .. n/16 - 1 of each of the 16 streams seed ..
 * seed + 15, the 16 streams of a position together, scaled and summed in
 * fp64 as the update does with its members' noise -- and folds the sums into
 * sink_dev[0] (one uint32, overwritten) without other memory traffic: the
 * update's throughput when nothing else runs.  Perturbations round each
 * normal to fp32, a few instructions more. */
CPES_API int cpes_rng_probe(uint64_t seed, int64_t n, uint32_t* sink_dev, void* stream);

/* Measurement references for the map and copy kernels: the same memory
 * traffic with nothing else, timed beside them.
 * cpes_probe_map_copy: the plainest gather (direction 0: buf[j] = w[p(j)])
 *   or scatter (direction 1: w[p(j)] = buf[j]) through the element map of
 *   `s` (index or index32; no chunk lists), one position per thread.  buf_dev:
 *   s->length elements of `dtype`, device memory.  Entries outside
 *   [0, numel) are skipped.
 * cpes_probe_copy: dst[i] = src[i] over `bytes` bytes (a multiple of 16; both
 *   pointers 16-byte aligned device memory), one 16-byte vector per thread;
 *   nontemporal != 0 takes non-temporal loads and stores (streaming past the
 *   caches, as the library's large copies do).
 * Errors: null pointers, a subspace without an element map, direction not 0
 *   or 1, bytes negative or not a multiple of 16, misaligned pointers ->
 *   CPES_ERR_INVALID_ARGUMENT. */
CPES_API int cpes_probe_map_copy(void* w_dev, int64_t numel, int dtype, const cpes_subspace* s, void* buf_dev,
                                 int direction, void* stream);
CPES_API int cpes_probe_copy(const void* src_dev, void* dst_dev, int64_t bytes, int nontemporal, void* stream);

/* Message of the last error on the calling thread ("" if none). */
CPES_API const char* cpes_last_error(void);

/*
 * cpes_fill_normal -- w[j] = cast(stddev * z_j) for j < n, where z_j is the
 * normal of position j in stream (seed, domain): the Philox4x32-10 words of
 * counter (lo32 q, hi32 q, domain, 0), q = j / 4, through the Box-Muller
 * transform of the perturbation noise (domain 0 is the noise itself; domain
 * 1 is meant for synthetic weight initialisation).  One fp32 multiply, then
 * round-to-nearest-even for bf16.  A utility for seeded inputs; not on the
 * training path.
 *   w_dev: n elements of `dtype` (any alignment), owned by the caller.
 * Errors: dtype unknown, n < 0, stddev negative or not finite, w NULL with
 *   n > 0 -> CPES_ERR_INVALID_ARGUMENT.  n = 0 does nothing.
 */
CPES_API int cpes_fill_normal(void* w_dev, int64_t n, int dtype, uint64_t seed, uint32_t domain, float stddev,
                     void* stream);

/* CPES_ABI_VERSION of the built library. */
CPES_API int cpes_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* CPES_H */
