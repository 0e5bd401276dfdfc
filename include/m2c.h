/*
 * m2c.h -- C ABI of the MI355X (gfx950) dynamic sparse mixed-precision FFN
 * with a neuron-level HBM slot cache (M2Cache, arXiv 2410.14740).
 *
 * One decode step of one FFN layer is four calls, in this order:
 *
 *   m2c_predict_rank  score every FFN neuron with the layer's low-rank
 *                     predictor, take the top-k, split them into FP16 / INT8 /
 *                     INT4 tiers by score rank            (Sec. 1 "Active Neuron
 *                     Identification" and "Active Score-based Quantization";
 *                     Sec. 5.2, Fig. 3)
 *   m2c_cache_plan    resolve the active neurons against the layer's HBM slot
 *                     cache: hit / refill / new / bypass, LRU victims, slot
 *                     table update                        (Sec. 5.3 "Overall
 *                     architecture" and "Cache Policy"; Sec. 1 LRU cache)
 *   m2c_cache_fill    copy every missing neuron record, at its tier, from the
 *                     pinned host-DRAM neuron store into its slot (Sec. 1
 *                     "Selective Loading into GPU"; Sec. 6.1 dedicated streams)
 *   m2c_sparse_ffn    gated FFN over only the active neurons, each read from
 *                     its slot and dequantized at its tier (Sec. 1, Sec. 5.2)
 *
 * Conventions shared by every call
 * --------------------------------
 * - All functions return an m2c_status. On an error detected on the host
 *   nothing is enqueued, the layer is unchanged and m2c_last_error() returns
 *   a message (thread-local). Nothing throws across the ABI.
 * - "dev" pointers are device memory of the layer's device; "host" pointers
 *   are ordinary host memory. The caller owns every pointer it passes.
 * - Streams are hipStream_t values passed as void*; NULL is the null stream.
 *   Asynchronous calls only enqueue work on the given stream and return.
 *   Ordering between streams (for example the fill stream and the FFN
 *   stream) is the caller's job, with events.
 * - fp16 values are passed as their IEEE binary16 bit patterns (uint16_t).
 *
 * Neuron and tiers (Sec. 1 footnote, Sec. 5.2)
 * --------------------------------------------
 * Neuron i of a SwiGLU FFN with W_gate, W_up [d_ff][d_model] and
 * W_down [d_model][d_ff] is row i of W_gate, row i of W_up and column i of
 * W_down. Tier codes: 0 inactive, 1 INT4, 2 INT8, 3 FP16 (higher score ->
 * higher precision, Sec. 5.2).
 *
 * Neuron records (the unit that is stored, copied and cached)
 * ----------------------------------------------------------
 * d = d_model, G = d / 128 (quantization group of 128 consecutive elements).
 *   FP16 record (tier 3), 6d bytes:
 *     gate[d] fp16 | up[d] fp16 | down[d] fp16
 *   INT8 record (tier 2), 3d + 6G bytes:
 *     gate[d] int8 | up[d] int8 | down[d] int8 |
 *     gate_scale[G] fp16 | up_scale[G] fp16 | down_scale[G] fp16
 *   INT4 record (tier 1), 1.5d + 6G bytes:
 *     gate[d/2] | up[d/2] | down[d/2] | gate_scale[G] | up_scale[G] | down_scale[G]
 *     byte m of a vector holds element 2m in bits 0-3 and element 2m+1 in
 *     bits 4-7, each a two's-complement nibble.
 * Quantization (symmetric, per group g of one vector, qmax = 127 or 7):
 *     amax = max |w| over the group (w are the fp16 weights),
 *     s    = fp16_rne( fp32(amax) / qmax )        (IEEE fp32 division),
 *     q    = clamp( rne( fp32(w) / fp32(s) ), -qmax, qmax ), q = 0 if s == 0,
 *     dequantized weight = q * s (exact in fp32).
 * Records of tier t are stored back to back with a stride of
 * record_stride[t] = record_bytes[t] rounded up to 16 bytes.
 *
 * Predictor scores (Sec. 5.2; low-rank predictor of Sec. 1)
 * ---------------------------------------------------------
 *   z = A x  (A [r][d] fp16),   s = B z + bias  (B [d_ff][r] fp16, bias fp32).
 * Every dot product is evaluated in fp32 in one fixed order, so that scores
 * (and therefore the selected ids) are reproducible bit for bit:
 *   n-element dot product, n % 8 == 0: split into chunks of 8 consecutive
 *   elements; L = min(64, largest power of two <= n/8) partial sums; chunk c
 *   belongs to partial c % L; each partial starts at +0.0f and takes
 *   acc = fmaf(a_j, b_j, acc) over its chunks in ascending order, elements in
 *   ascending order inside a chunk; then for off = L/2, L/4, ..., 1 every
 *   partial p becomes p[l] + p[l ^ off]; the result is p[0]. z stays fp32;
 *   the bias, when present, is one fp32 addition after the dot product.
 *
 * Selection and tiers (Sec. 5.2)
 * ------------------------------
 * Neurons are ranked by score descending, ties by id ascending; scores are
 * compared as order-preserving unsigned keys of their fp32 bit patterns
 * (so -0.0 ranks below +0.0). Rank rho < n_fp16 -> tier 3;
 * rho < n_fp16 + n_int8 -> tier 2; rho < k -> tier 1; else tier 0.
 *
 * Cache policy (Sec. 5.3; LRU of Sec. 1 and Sec. 6.4)
 * ---------------------------------------------------
 * One cache unit per layer: C resident slots plus S staging slots, each
 * slot_bytes = 6d bytes (an FP16 record). The required set R of a step is
 * every neuron with tier > 0 in some batch row, taken at the highest tier any
 * row asks for. The step is atomic: for i in R (ascending id)
 *   HIT     i is resident at the requested tier (with M2C_FLAG_DOMINANT_HITS:
 *           at the requested tier or above; the step then uses the resident
 *           tier);
 *   REFILL  i is resident at another tier (with M2C_FLAG_DOMINANT_HITS: a
 *           lower one): it is refilled in its own slot;
 *   NEW     i is not resident.
 * Victims are the slots holding no neuron of R, ordered by (last use
 * ascending, slot ascending); never-used slots count as last use -1. The j-th
 * NEW neuron in ascending id takes the j-th victim and evicts its previous
 * neuron. NEW neurons beyond the number of victims are BYPASS: they are
 * filled into staging slot C + j' (j' counts bypasses in ascending id) and
 * are not retained. Every slot of R gets last use = step. With C = k and a
 * single tier this reduces to the paper's Adjacent Token Update policy.
 */
#ifndef M2C_H
#define M2C_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  M2C_OK = 0,
  M2C_ERR_INVALID_ARG = 1,  /* bad pointer, size, count or descriptor        */
  M2C_ERR_OUT_OF_MEMORY = 2,/* device or pinned host allocation failed       */
  M2C_ERR_HIP = 3,          /* a HIP runtime call failed (message has detail)*/
  M2C_ERR_CAPACITY = 4,     /* a size beyond what the layer was created for  */
  M2C_ERR_STATE = 5         /* call out of order (e.g. step not increasing)  */
} m2c_status;

typedef struct m2c_layer m2c_layer; /* opaque; one per FFN layer */

enum { M2C_TIER_NONE = 0, M2C_TIER_INT4 = 1, M2C_TIER_INT8 = 2, M2C_TIER_FP16 = 3 };

/* Layer descriptor. All fields are required. */
typedef struct {
  int32_t d_model;       /* d: multiple of 128, 128..16384                      */
  int32_t d_ff;          /* neurons: 1..262144                                  */
  int32_t pred_rank;     /* r: multiple of 8, 8..1024                           */
  int32_t group;         /* quantization group; must be 128                     */
  int32_t k_max;         /* largest k any call will use: 0..d_ff                */
  int32_t max_batch;     /* largest batch any call will use: 1..32              */
  int32_t cache_slots;   /* C: resident slots, 0..d_ff                          */
  int32_t staging_slots; /* S: bypass slots; -1 = the minimum that can never
                            overflow, max(0, min(d_ff, max_batch*k_max) - C);
                            smaller explicit values are rejected               */
  int32_t device;        /* HIP device ordinal                                  */
  int32_t flags;         /* M2C_FLAG_* bits, 0 for the defaults                 */
  int32_t tier_slots[4]; /* with M2C_FLAG_TIER_POOLS: resident slots of the INT4
                            [1], INT8 [2] and FP16 [3] pools, summing to
                            cache_slots ([0] unused); otherwise ignored        */
} m2c_layer_desc;

/* m2c_layer_desc.flags */
enum {
  /* Sparse FFN at batch 1 by three kernels (up, down by column slices, ordered
     reduce) whose output is the same bit pattern on every run. By default, and
     with more rows, groups of neurons are added into y with fp32 atomics, so the
     summation order, and the last bits of y, vary from run to run. */
  M2C_FLAG_DETERMINISTIC_FFN = 1,
  /* Cache policy variant (Sec. 5.3 "Cache Policy"): a neuron resident at a
     tier at or above the requested one is a HIT and the step uses it at its
     resident tier (req_tier and the FFN then carry the resident tier); only
     a resident tier below the requested one is a REFILL. The default is the
     exact-tier policy: any other resident tier is a REFILL. With dominance
     hits the output depends on the cache history, not only on the step. */
  M2C_FLAG_DOMINANT_HITS = 2,
  /* Per-tier record arena: the cache unit is split into one pool per tier,
     pool t with tier_slots[t] resident slots of record_stride[t] bytes (an
     INT4 neuron no longer takes an FP16-sized slot, so the same HBM holds
     more neurons). Each pool is its own step-atomic LRU cache over the
     neurons whose step tier is t: HIT if resident in that pool, else NEW
     there (victims from that pool, BYPASS into that pool's staging slots,
     max(0, plan_capacity - tier_slots[t]) of them). A neuron may be resident
     in several pools; there are no REFILLs. Global slot ids are numbered in
     tier blocks, FP16 first (see m2c_layer_info.pool_first). With
     M2C_FLAG_DOMINANT_HITS a neuron required at tier t that is not resident
     in pool t but is resident (at the start of the step) in a pool of higher
     precision is served by the lowest such pool, a HIT at that pool's tier
     (req_tier and the FFN carry it). Needs max_batch == 1, d_model <= 8192,
     d_ff <= 32768, staging_slots == -1, and not M2C_FLAG_DETERMINISTIC_FFN. */
  M2C_FLAG_TIER_POOLS = 4
};

/* Sizes that follow from a descriptor. */
typedef struct {
  int32_t record_bytes[4];  /* by tier; [0] = 0                               */
  int32_t record_stride[4]; /* host store stride by tier; [0] = 0             */
  int32_t slot_bytes;       /* 6 * d_model                                    */
  int32_t cache_slots;      /* C                                              */
  int32_t staging_slots;    /* S (resolved)                                   */
  int32_t plan_capacity;    /* entries of every plan list: min(d_ff, max_batch*k_max) */
  int64_t plan_bytes;       /* size of one plan buffer                        */
  int64_t host_store_bytes; /* pinned host neuron store (all three tiers)     */
  int64_t device_bytes;     /* device memory the layer owns                   */
  /* Slots of the tier-t records, by tier [1..3]: global slot ids
     [pool_first[t], pool_first[t] + pool_slots[t]), resident ones first,
     each pool_stride[t] bytes. Without M2C_FLAG_TIER_POOLS every tier shares
     one pool: pool_first 0, pool_slots C + S, pool_stride slot_bytes. */
  int32_t pool_first[4];
  int32_t pool_slots[4];
  int32_t pool_resident[4]; /* resident slots of the pool (the rest stage)    */
  int32_t pool_stride[4];
  int64_t slot_arena_bytes; /* every pool plus the all-zero padding slot      */
} m2c_layer_info;

/* A plan is one caller-allocated device buffer of info.plan_bytes bytes,
 * 256-byte aligned. These are the byte offsets of its arrays; every list has
 * plan_capacity entries of which counts[...] are valid. */
enum {
  M2C_CNT_REQ = 0,     /* |R|                                                 */
  M2C_CNT_HIT = 1,
  M2C_CNT_REFILL = 2,
  M2C_CNT_NEW = 3,     /* NEW that got a resident victim slot                 */
  M2C_CNT_BYPASS = 4,  /* NEW that went to a staging slot                     */
  M2C_CNT_EVICT = 5,   /* victims that held a neuron                          */
  M2C_CNT_FILL = 6,    /* REFILL + NEW + BYPASS                               */
  M2C_CNT_REQ_FP16 = 7,/* |R| by tier                                         */
  M2C_CNT_REQ_INT8 = 8,
  M2C_CNT_REQ_INT4 = 9,
  M2C_CNT_FILL_FP16 = 10, /* fills by tier                                    */
  M2C_CNT_FILL_INT8 = 11,
  M2C_CNT_FILL_INT4 = 12,
  M2C_CNT_FILL_DERIVED = 13, /* INT8 / INT4 fills of a neuron whose slot held its
                             FP16 record: made on the GPU from that record,
                             no host read (fill_from == 3)                     */
  M2C_NCOUNTS = 16
};
typedef struct {
  int64_t counts;      /* int32 [M2C_NCOUNTS]                                 */
  int64_t req_ids;     /* int32 [cap] R in ascending neuron id                */
  int64_t req_tier;    /* uint8 [cap] tier taken for the step (max over rows) */
  int64_t req_hit;     /* uint8 [cap] 0 NEW, 1 HIT, 2 REFILL, 3 BYPASS        */
  int64_t req_slot;    /* int32 [cap] slot read by the FFN                    */
  int64_t req_mask;    /* uint32[cap] bit b set if batch row b selected it    */
  int64_t fill_ids;    /* int32 [cap] misses in ascending neuron id           */
  int64_t fill_tier;   /* uint8 [cap]                                         */
  int64_t fill_slot;   /* int32 [cap]                                         */
  int64_t fill_from;   /* uint8 [cap] REFILL: tier of the record the slot held
                          for the neuron before the step; NEW / BYPASS: 0     */
  int64_t evicted_ids; /* int32 [cap] evicted neurons in victim order         */
  int64_t work_slot;   /* int32 [cap] R regrouped tier-major (FP16, INT8,
                          INT4), ascending id inside a tier: FFN work order;
                          512 spare entries follow (read, never used)         */
  int64_t work_mask;   /* uint32[cap] row masks in work order                 */
  int64_t ffn_tasks;   /* the batch-1 FFN kernel's per-workgroup task table:
                          library-internal format, written by m2c_cache_plan
                          (empty for layers whose FFN does not use it)       */
  int64_t total_bytes;
} m2c_plan_layout;

/* Cumulative per-layer counters since creation or the last cache reset. */
typedef struct {
  int64_t plans;
  int64_t req, hit, refill, new_, bypass, evict;
  int64_t fill[4];        /* fills by tier                                    */
  int64_t fill_bytes;     /* sum of record_bytes over fills                   */
  int64_t derived[4];     /* fills by tier made from the resident FP16 record */
  int64_t host_bytes;     /* sum of record_bytes over fills read from the host
                             store: fill_bytes minus the derived fills'       */
  int64_t req_tier[4];    /* required neurons by step tier                    */
  int64_t req_bytes;      /* sum of record_bytes over required neurons: what
                             the sparse FFN reads from the slots              */
} m2c_stats;

/* Bytes of one neuron record of `tier` (1..3) for d_model d, or -1. */
int64_t m2c_record_bytes(int32_t d_model, int32_t tier);

/* Create a layer (Sec. 5.3 isolated cache unit + the layer's share of the
 * host-DRAM neuron store). Host inputs, copied; may be freed on return:
 *   w_gate, w_up  [d_ff][d_model] fp16; w_down [d_model][d_ff] fp16;
 *   pred_a [pred_rank][d_model] fp16;  pred_b [d_ff][pred_rank] fp16;
 *   score_bias [d_ff] fp32 or NULL (no addition).
 * Quantizes every neuron to the INT8 and INT4 records on the device and keeps
 * all three records in pinned host memory; the cache starts cold.
 * Synchronous. */
m2c_status m2c_layer_create(const m2c_layer_desc* desc, const uint16_t* w_gate,
                            const uint16_t* w_up, const uint16_t* w_down,
                            const uint16_t* pred_a, const uint16_t* pred_b,
                            const float* score_bias, m2c_layer** out);

/* Create a layer that reads its neuron records from the host store of
 * `weights_of` (same d_model, d_ff and device) instead of owning a copy; it
 * has its own predictor, slot cache and tables. The store lives until every
 * layer using it is destroyed. Synchronous. */
m2c_status m2c_layer_create_shared(const m2c_layer_desc* desc, const m2c_layer* weights_of,
                                   const uint16_t* pred_a, const uint16_t* pred_b,
                                   const float* score_bias, m2c_layer** out);

/* Wait for the device, then free everything the layer owns. NULL is a no-op. */
m2c_status m2c_layer_destroy(m2c_layer* layer);

m2c_status m2c_layer_get_info(const m2c_layer* layer, m2c_layer_info* out);
m2c_status m2c_plan_get_layout(const m2c_layer* layer, m2c_plan_layout* out);

/* Scores and tiers for `batch` tokens.
 *   x        dev fp16 [batch][d_model]
 *   scores   dev fp32 [batch][d_ff] output, or NULL (kept internally)
 *   tier_map dev uint8 [batch][d_ff] output, tier of every neuron
 * 0 <= n_fp16, 0 <= n_int8, n_fp16 + n_int8 <= k <= k_max, 1 <= batch <= max_batch. */
m2c_status m2c_predict_rank(m2c_layer* layer, const uint16_t* x, int32_t batch, int32_t k,
                            int32_t n_fp16, int32_t n_int8, float* scores, uint8_t* tier_map,
                            void* stream);

/* Bytes of the fixed device scratch array of m2c_predict_rank_noalloc. */
#define M2C_NOALLOC_SCRATCH_BYTES (4u << 20)

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the same
 * scores and tier map as m2c_predict_rank, bit for bit, with the call's
 * scratch -- z [batch][pred_rank] fp32 and, when `scores` is NULL, the scores
 * [batch][d_ff] fp32 -- in one fixed device array of M2C_NOALLOC_SCRATCH_BYTES
 * that the library keeps on every GPU it runs on until the process ends,
 * instead of the layer's own buffers. Allocates nothing: no hipMalloc, no
 * hipFree, no allocating library call.
 * Limit: round_up(4 * batch * pred_rank, 256) + (scores ? 0 : 4 * batch *
 * d_ff) <= M2C_NOALLOC_SCRATCH_BYTES, else M2C_ERR_CAPACITY with nothing
 * enqueued. Every call on one GPU, from any layer, shares that GPU's array:
 * calls that can run at the same time on one GPU (streams not ordered with
 * each other, or other threads) race and give wrong results; calls ordered
 * on one stream are safe. The array is fully written before it is read, so
 * what an earlier call left in it never matters. */
m2c_status m2c_predict_rank_noalloc(m2c_layer* layer, const uint16_t* x, int32_t batch, int32_t k,
                                    int32_t n_fp16, int32_t n_int8, float* scores,
                                    uint8_t* tier_map, void* stream);

/* Resolve tier_map (dev uint8 [batch][d_ff]) against the slot cache for
 * decode step `step`, write the plan into `plan` (dev, plan_bytes) and update
 * the slot tables. `step` must be >= 0, < 2^31 and strictly greater than the
 * previous step given to this layer (M2C_ERR_STATE otherwise). The plan must
 * not be reused until every fill and FFN that reads it has completed. */
m2c_status m2c_cache_plan(m2c_layer* layer, const uint8_t* tier_map, int32_t batch, int64_t step,
                          void* plan, void* stream);

/* Copy every fill of `plan` from the pinned host store into its slot, on
 * `stream`, by a device gather kernel that reads host memory over the host
 * link. A fill to INT8 / INT4 whose slot holds the neuron's FP16 record
 * (fill_from == 3) is instead quantized in place from that record, which
 * gives the bytes of the store's record (both are the group-128 quantization
 * of the same fp16 values); the layer tracks which slots hold FP16 bytes, so
 * running the fill of a plan again copies instead and gives the same slots.
 * Must run after the plan on the same stream or behind an event, and before
 * the FFN that reads the plan. No host synchronization. */
m2c_status m2c_cache_fill(m2c_layer* layer, const void* plan, void* stream);

/* y += sum over i in R of silu(<g_i, x>) * <u_i, x> * d_i, per batch row b
 * over the neurons whose req_mask has bit b, every vector dequantized at the
 * neuron's step tier; fp32 accumulation. The result is ADDED to y (a residual
 * stream); zero y first for the plain FFN output.
 *   x dev fp16 [batch][d_model];  y dev fp32 [batch][d_model], in/out.
 * `batch` (1..max_batch) must equal the batch given to the plan. Batch 1 is a
 * gather-dequant GEMV; larger batches run both contractions on the matrix
 * cores with fp32 accumulation: gate / up with the codes (exact as fp16) and
 * x, group scales applied in fp32; down with the codes and h times the group
 * scale, the latter split into an fp16 high and low part. They are never
 * bit-deterministic (the deterministic flag applies to batch 1). */
m2c_status m2c_sparse_ffn(m2c_layer* layer, const uint16_t* x, int32_t batch, const void* plan,
                          float* y, void* stream);

/* Make the cache cold again (all slots empty, stats zeroed, step history
 * cleared), on `stream`. */
m2c_status m2c_layer_reset_cache(m2c_layer* layer, void* stream);

/* Synchronizes the device, then reads the cumulative counters. Returns
 * M2C_ERR_CAPACITY (and clears the condition) if a cache plan since the last
 * call received a tier map with more active neurons than the layer's plan
 * capacity, min(d_ff, max_batch * k_max): such a plan is left empty and the
 * cache unchanged. Returns M2C_ERR_STATE (and clears the condition) if a
 * batch-1 sparse FFN gave up waiting for one of its own h values (its
 * workgroups could not all run, for instance because another kernel held the
 * GPU for a long time); that call's output is wrong. */
m2c_status m2c_layer_stats(const m2c_layer* layer, m2c_stats* out);

/* ------------------------------------------------------------------------
 * SSD -> DRAM tier (Sec. 5.4 "Pattern-Aware Preloading for SSD", Fig. 8)
 * ------------------------------------------------------------------------
 * Every layer's neuron records live in a file (the SSD). A two-level DRAM
 * cache holds the first `fixed_layers` layers in a fixed area, read once at
 * creation and never evicted (a new token does not reload them), and the
 * other layers in a dynamic area of `dynamic_slots` layer-sized buffers. A
 * loader thread reads whole layers ahead of use. When layer l is acquired,
 * the window l, l+1, ..., l+lookahead (mod n_layers) is made resident in
 * that order (the caller waits only for l); a missing layer takes the lowest
 * empty slot, else the slot of the loaded, unheld layer outside the window
 * whose next use in the cyclic layer order is furthest away (largest
 * (layer - l) mod n_layers); a look-ahead load with no slot to give up is
 * skipped. These decisions depend only on the order of acquires.
 *
 * File layout of one layer (what m2c_layer_write_store writes): the FP16,
 * INT8 and INT4 record arrays back to back (d_ff * record_stride[t] bytes
 * each), zero-padded to a multiple of 4096 bytes; layer_bytes is the
 * unpadded size. Layer offsets in the file are multiples of 4096. */
enum {
  M2C_DRAM_HOST_MEMORY = 1, /* plain host memory (no HIP calls; CPU-side use
                               and tests); default: pinned (hipHostMalloc) so
                               that the GPU fill reads it over the host link */
  M2C_DRAM_DIRECT_IO = 2    /* read with O_DIRECT (bypass the page cache);
                               falls back to buffered reads if the file system
                               refuses it (m2c_dram_stats.direct_io says) */
};
typedef struct {
  int32_t n_layers;      /* layers in the file                                 */
  int32_t fixed_layers;  /* fixed area: layers 0 .. fixed_layers-1             */
  int32_t dynamic_slots; /* dynamic area: >= lookahead + 1 unless every layer
                            is fixed                                          */
  int32_t lookahead;     /* layers loaded ahead of the one in use, >= 1        */
  int64_t layer_bytes;   /* bytes of one layer's records (unpadded)            */
  int32_t flags;         /* M2C_DRAM_*                                         */
  int32_t device;        /* device whose fills read the pinned buffers         */
} m2c_dram_desc;
typedef struct {
  int64_t acquires, hits;  /* hits: the layer was already in DRAM             */
  int64_t loads, evictions;
  int64_t bytes_read;      /* layer_bytes per load from the file              */
  int64_t fixed_bytes;     /* bytes of the fixed area                         */
  double read_seconds;     /* time the loader spent reading                   */
  double wait_seconds;     /* time acquires spent waiting for their layer     */
  int32_t direct_io;       /* 1 if reads bypass the page cache                */
} m2c_dram_stats;
typedef struct m2c_dram m2c_dram; /* opaque */

/* Write the layer's host store into `path` (created if missing) at `offset`
 * (a multiple of 4096), in the file layout above; *padded_bytes gets the
 * bytes written (layer_bytes rounded up to 4096). Synchronous. */
m2c_status m2c_layer_write_store(const m2c_layer* layer, const char* path, int64_t offset,
                                 int64_t* padded_bytes);

/* Open the cache over `path`; offsets[l] is layer l's offset. Reads the fixed
 * area before returning and starts the loader thread. */
m2c_status m2c_dram_create(const m2c_dram_desc* desc, const char* path, const int64_t* offsets,
                           m2c_dram** out);
/* Stops the loader, waits for the GPU readers of the buffers, frees them.
 * M2C_ERR_STATE while layers created on the cache still exist. */
m2c_status m2c_dram_destroy(m2c_dram* dram);
/* Host-side use: wait until `layer` is in DRAM, hold it, return its bytes. */
m2c_status m2c_dram_acquire(m2c_dram* dram, int32_t layer, const uint8_t** data);
/* Give up a hold taken by m2c_dram_acquire. */
m2c_status m2c_dram_release(m2c_dram* dram, int32_t layer);
m2c_status m2c_dram_get_stats(m2c_dram* dram, m2c_dram_stats* out);
/* Test support: the loads decided so far, in order (layer loaded, layer
 * evicted or -1); *count gets the total, at most `capacity` are copied. */
m2c_status m2c_dram_get_log(m2c_dram* dram, int32_t* loaded, int32_t* evicted, int32_t capacity,
                            int32_t* count);

/* Create a layer whose neuron records are layer `index` of a pinned DRAM
 * cache (same d_model / d_ff and device; dram layer_bytes must equal the
 * layer's record arrays). Its own predictor, slot cache and tables; each
 * m2c_cache_fill acquires the layer from the cache (waiting for the loader
 * if needed), enqueues the gather from those buffers and releases them
 * behind a HIP event, so the loader never overwrites bytes a fill still
 * reads. Fills of layers of one cache should be issued in layer order (the
 * cyclic order the look-ahead assumes). The cache must outlive the layer. */
m2c_status m2c_layer_create_from_dram(const m2c_layer_desc* desc, m2c_dram* dram, int32_t index,
                                      const uint16_t* pred_a, const uint16_t* pred_b,
                                      const float* score_bias, m2c_layer** out);

/* Offline neuron-ratio search (Sec. 5.2 "Offline Neuron Ratio Search",
 * Algorithm 1) on an FFN-error proxy of the paper's entropy estimate, which
 * needs a trained language model. Candidate i = 1, 2, ... has
 * n_high = i * step FP16 neurons and n_low = n_low0 - i * step * bit_ratio
 * low-precision ones (INT4 for bit_ratio 4, INT8 for bit_ratio 2), while
 * n_low >= 0: the bytes of the active neurons stay the same. Its score is
 *   uq = sum_t |y_t - y*_t|^2 / sum_t |y*_t|^2
 * over the T calibration tokens x (dev fp16 [T][d_model]): y_t is this
 * layer's sparse FFN with the top n_high + n_low neurons by predictor score,
 * the n_high best at FP16, the rest at the low tier; y*_t the FFN with every
 * neuron at FP16. Each FFN runs through the layer's predict, plan, fill and
 * FFN kernels on `stream`. The chosen candidate is the one with the lowest
 * score, a later one winning ties (the comparison UQ_best >= UQ_score).
 * Needs k_max == d_ff (the all-FP16 reference). Outputs (host, room for
 * max_candidates): n_high, n_low, uq per candidate, *count candidates,
 * *best the chosen index (-1 if none). Synchronous; allocates its buffers;
 * leaves the layer's cache cold (reset). */
m2c_status m2c_ratio_search(m2c_layer* layer, const uint16_t* x, int32_t T, int32_t n_low0,
                            int32_t step, int32_t bit_ratio, int32_t max_candidates,
                            int32_t* n_high, int32_t* n_low, double* uq, int32_t* count,
                            int32_t* best, void* stream);

/* ------------------------------------------------------------------------
 * Attention next to the sparse FFN: whole prompts, and single tokens over a
 * key/value cache held in 8 bits
 * ------------------------------------------------------------------------
 * These calls keep no state in the library: every buffer is the caller's, and
 * a call only enqueues kernels (m2c_kv_status excepted). Nothing allocates, so
 * all of them may be captured into a HIP graph.
 *
 * Head layout: n_heads query heads over n_kv_heads key/value heads, n_heads a
 * multiple of n_kv_heads; with G = n_heads / n_kv_heads query head h reads
 * key/value head h / G. Rows of queries, keys, values and outputs are given by
 * two strides in elements, between tokens (head_dim .. 2^24) and between heads
 * (0 for rows that heads share; rows that are written must not overlap); the
 * head_dim elements of a head are contiguous, and pointers and strides are
 * multiples of 16 bytes (8 elements).
 *
 * Softmax statistics and sums are fp32; weights of the value product are
 * rounded to the 16-bit type of the matrix instruction that takes them. A
 * masked key contributes nothing, whatever its key and value hold. A query
 * without any key has a zero output and the log-sum-exp -infinity. */
enum { M2C_DTYPE_FP16 = 0, M2C_DTYPE_BF16 = 1,
       M2C_DTYPE_FP32 = 2 /* m2c_residual_norm only */ };

typedef struct {
  int32_t dtype;         /* M2C_DTYPE_* of q, k, v and out                      */
  int32_t n_heads;       /* query heads, 1..1024                                */
  int32_t n_kv_heads;    /* divides n_heads                                     */
  int32_t head_dim;      /* 64 or 128                                           */
  int32_t causal;        /* 1: query i of a sequence with lq queries and lk keys
                            sees its keys 0 .. lk - lq + i (the last query sees
                            them all); 0: every key of its sequence             */
  int32_t device;        /* HIP device ordinal of every pointer                 */
  float scale;           /* factor of <q, k>; 0 = 1 / sqrt(head_dim)            */
  int32_t max_q;         /* longest query sequence, or 0 if not known: only
                            helps to choose whether rows are split along their
                            keys, never what is computed                        */
  int64_t q_stride[2], k_stride[2], v_stride[2], out_stride[2]; /* token, head  */
  void* workspace;       /* dev, 256-byte aligned, not shared with a call that
                            may run at the same time, or NULL: no row of
                            queries is then split along its keys                */
  int64_t workspace_bytes;
} m2c_attn_desc;

/* Bytes of the workspace with which a call with these arguments splits the
 * queries that see many more keys than the others along them (0 where it would
 * split none), or -1. cu_q and cu_k are compared, not read. */
int64_t m2c_prompt_attention_workspace(const m2c_attn_desc* desc, const int32_t* cu_q,
                                       const int32_t* cu_k, int32_t n_seqs, int64_t total_q,
                                       int64_t total_k);

/* Attention of packed sequences: rows cu_q[b] .. cu_q[b + 1] - 1 of q and out
 * and rows cu_k[b] .. cu_k[b + 1] - 1 of k and v are sequence b.
 *   cu_q, cu_k  dev int32 [n_seqs + 1], ascending, within [0, total_q] and
 *               [0, total_k]; they may be the same array
 *   q, out      dev [total_q] rows;  k, v  dev [total_k] rows
 *   lse         dev fp32 [total_q][n_heads], ln sum exp(scale <q, k>), or NULL
 * Output rows of no sequence are not written. With starts that do not ascend
 * nothing outside the arrays is touched, but which rows are computed is not
 * defined. Results are the same bits on every run with the same arguments. */
m2c_status m2c_prompt_attention(const m2c_attn_desc* desc, const void* q, const void* k,
                                const void* v, const int32_t* cu_q, const int32_t* cu_k,
                                int32_t n_seqs, int64_t total_q, int64_t total_k, void* out,
                                float* lse, void* stream);

/* Rotation of queries and keys by their positions. A pair (a, b) of a head's
 * first rot_dim elements becomes
 *     scale (a cos w - b sin w),  scale (b cos w + a sin w),
 *     w = position * freq[pair],
 * the other elements stay as they are. A position has n_axes coordinates (time,
 * height and width, for example); the first section[0] pairs turn by the first,
 * the next section[1] by the second, and so on. The angle is exact to 2^-51 of
 * itself, so that far positions turn as near ones do. */
typedef struct {
  int32_t rot_dim;       /* a multiple of 16, 16 .. head_dim                    */
  int32_t interleaved;   /* 1: pair i is elements 2i, 2i + 1; 0: elements i,
                            i + rot_dim / 2                                     */
  int32_t n_axes;        /* 1..4                                                */
  int32_t section[4];    /* pairs of each axis, >= 0 (those past n_axes 0); all
                            together rot_dim / 2                                */
  float scale;           /* finite; 0 = 1                                       */
  const float* freq;     /* dev [rot_dim / 2], radians per position             */
} m2c_rotary;

/* Rows of queries and keys turned: q_out gets q's [total] rows, k_out k's.
 *   positions  dev int32, row i's coordinate a at positions[a * pos_stride + i]
 *   q, k       with their strides (tokens, heads); k NULL: queries alone (n_kv_heads 0)
 *   q_out may be q with its strides, and k_out k; otherwise what is written must
 *   not overlap what is read. head_dim 64 or 128. */
m2c_status m2c_rotate(const m2c_rotary* rotary, int32_t dtype, int32_t head_dim, int32_t device,
                      int64_t total, const int32_t* positions, int64_t pos_stride, int32_t n_heads,
                      const void* q, const int64_t q_stride[2], void* q_out,
                      const int64_t q_out_stride[2], int32_t n_kv_heads, const void* k,
                      const int64_t k_stride[2], void* k_out, const int64_t k_out_stride[2],
                      void* stream);

/* Key/value cache. The tokens of a sequence are cut into blocks of
 * block_tokens. A block of one key/value head lies in a page:
 *     amax = max |x| over the block (its keys, and apart its values),
 *     s    = fp32(amax) / 127                        (IEEE fp32 division),
 *     code = clamp( rne( fp32(x) / s ), -127, 127 ), 0 if s == 0,
 *     it stands for code * s.
 * A block that holds an infinity or a NaN has a scale that is not finite and
 * codes 0: it reads back as NaN.
 * The last block of a sequence (the one that holds token len - 1) also keeps
 * its tokens in their 16-bit type in tail_k / tail_v; they are attended from
 * there until the block is full, and quantized once, when it is. So what the
 * cache holds depends on the tokens alone, not on how many came per call.
 * Every array is the caller's, contiguous device memory of one device: */
typedef struct {
  int32_t dtype;         /* M2C_DTYPE_* of the tokens and tails                 */
  int32_t n_seqs;        /* sequences, 1..65535                                 */
  int32_t n_kv_heads;    /* 1..1024                                             */
  int32_t head_dim;      /* 64 or 128                                           */
  int32_t block_tokens;  /* 32, 64 or 128                                       */
  int32_t max_blocks;    /* blocks of a sequence, 1..16384                      */
  int32_t device;
  int32_t reserved;      /* 0                                                   */
  int64_t n_pages;       /* pages, 1..2^31 - 1                                  */
  int8_t* k_codes;       /* [n_pages][block_tokens][head_dim]                   */
  int8_t* v_codes;
  float* k_scale;        /* [n_pages]                                           */
  float* v_scale;
  void* tail_k;          /* [n_seqs][n_kv_heads][block_tokens][head_dim]        */
  void* tail_v;
  int32_t* table;        /* [n_seqs][n_kv_heads][max_blocks] page of each block;
                            set by the caller for every block that may fill.
                            Pages that no append fills may be shared            */
  int32_t* len;          /* [n_seqs] tokens held                                */
  float* weight;         /* [n_seqs][n_kv_heads][max_blocks] accumulated
                            attention weight of each block                      */
  int32_t* arrive;       /* [n_seqs] zeroed once by the caller; library's own   */
  int32_t* status;       /* [1] zeroed once by the caller; see m2c_kv_status    */
} m2c_kv_cache;

/* seqs (in the calls below): dev int32 [n], the sequence of each row of the
 * call, no sequence twice; NULL means sequences 0 .. n - 1. What a call finds
 * wrong on the device sets a bit that m2c_kv_status reports, and nothing out of
 * range is touched: of a sequence out of range nothing is written but attend's
 * zero row; an append that is refused leaves its sequence as it was; a block
 * whose page is out of range is not stored, and is read and attended as zeros.
 * Row starts that do not ascend are reported and touch nothing out of range, but
 * which rows the sequences of the call then get is not defined. */

/* Forget the tokens of n sequences. */
m2c_status m2c_kv_reset(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, void* stream);

/* Append tokens. Sequence seqs[b] gets rows cu[b] .. cu[b + 1] - 1 of k and v
 * (cu dev int32 [n + 1], ascending, within [0, total]); cu NULL: row b, one
 * token each (total == n).
 *   pos       dev int32 [n], the place of the first new token, or NULL: at the
 *             end. A place before the end writes over the tokens from there on
 *             and ends the sequence after the new ones; it must be the start
 *             of a block or lie in the last block (M2C_ERR_STATE otherwise)
 *   k_stride, v_stride  token and head strides in elements
 * The weight of every block that gets its first token is set to 0. A sequence
 * that gets no rows stays as it is, wherever its pos lies. A sequence
 * that would pass max_blocks * block_tokens tokens is M2C_ERR_CAPACITY. */
m2c_status m2c_kv_append(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n,
                         const int32_t* cu, int64_t total, const int32_t* pos, const void* k,
                         const void* v, const int64_t k_stride[2], const int64_t v_stride[2],
                         void* stream);

/* m2c_kv_append with keys that are turned by their positions on the way, rounded
 * once to the cache's 16-bit type: what the cache holds is to the bit what
 * m2c_rotate and m2c_kv_append would leave. In the same launch:
 *   q, q_out   dev [total] rows of n_heads heads, the queries of the same tokens,
 *              turned as well (q_out may be q with its strides), or NULL
 *              (n_heads 0)
 *   k_out      dev [total] rows that get the turned keys too, not k, or NULL
 * positions and pos_stride are m2c_rotate's; pos is the place in the cache, as in
 * m2c_kv_append. Queries of every row of a sequence are turned, whatever becomes
 * of its append; keys of a sequence whose append is refused are not written to
 * k_out. Rows of no sequence are not written. */
m2c_status m2c_kv_append_rotated(const m2c_kv_cache* cache, const m2c_rotary* rotary,
                                 const int32_t* seqs, int32_t n, const int32_t* cu, int64_t total,
                                 const int32_t* pos, const int32_t* positions, int64_t pos_stride,
                                 const void* k, const void* v, const int64_t k_stride[2],
                                 const int64_t v_stride[2], void* k_out,
                                 const int64_t k_out_stride[2], int32_t n_heads, const void* q,
                                 const int64_t q_stride[2], void* q_out,
                                 const int64_t q_out_stride[2], void* stream);

/* Read tokens back in the cache's 16-bit type (code * s rounded once; tokens
 * of the open block as they came): rows cu[b] .. cu[b + 1] - 1 of k and v get
 * tokens 0, 1, .. of sequence seqs[b], as many as there are; rows past its
 * length are not written. cu dev int32 [n + 1], ascending, within [0, total]. */
m2c_status m2c_kv_read(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n,
                       const int32_t* cu, int64_t total, void* k, void* v,
                       const int64_t k_stride[2], const int64_t v_stride[2], void* stream);

/* Bytes of the workspace of m2c_kv_attend with the same arguments, or -1. */
int64_t m2c_kv_attend_workspace(const m2c_kv_cache* cache, int32_t n, int32_t n_heads,
                                int32_t track, int32_t max_len);

/* Attention of one query token per sequence over everything its sequence
 * holds.
 *   q, out     dev [n] rows of n_heads heads, with their strides
 *   scale      factor of <q, k>; 0 = 1 / sqrt(head_dim)
 *   lse        dev fp32 [n][n_heads] or NULL
 *   track      1: adds to weight[s][h][block] the attention weights of the
 *              block's tokens, summed over the tokens and the query heads of h
 *   max_len    longest sequence of the call, or 0 if not known (the capacity):
 *              how far a sequence is split; a longer one is still computed
 *   workspace  dev, m2c_kv_attend_workspace bytes, 256-byte aligned; not shared
 *              with a call that may run at the same time
 * Results are the same bits on every run with the same max_len and n. */
m2c_status m2c_kv_attend(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n,
                         int32_t n_heads, float scale, const void* q, const int64_t q_stride[2],
                         void* out, const int64_t out_stride[2], float* lse, int32_t track,
                         int32_t max_len, void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of the workspace with which m2c_kv_attend_chunk with the same arguments
 * splits the queries that see many more keys than the others along them (0 where
 * it would split none: always for n > 64, where a chunk's few rows on a sequence far
 * longer than the others take as long as that sequence alone), or -1. */
int64_t m2c_kv_attend_chunk_workspace(const m2c_kv_cache* cache, int32_t n, int64_t total,
                                      int32_t n_heads, int32_t max_q, int32_t max_len);

/* Attention of chunks of tokens: rows cu[b] .. cu[b + 1] - 1 of q and out are
 * sequence seqs[b]'s (which may be listed twice). Its keys are the tokens that the
 * cache holds and then, where k and v are given, the same rows of k and v: the
 * chunk's own, which are not in the cache yet (append them afterwards). With k and
 * v NULL the cache holds the chunk already. Of nk keys in all, query i of lq sees
 * keys 0 .. nk - lq + i. The cache is not changed.
 *   cu         dev int32 [n + 1], ascending, within [0, total]; rows of no sequence
 *              are not written
 *   q, out     dev [total] rows of n_heads heads, with their strides
 *   k, v       dev [total] rows of the cache's heads, with their strides, or both NULL
 *   scale      factor of <q, k>; 0 = 1 / sqrt(head_dim)
 *   lse        dev fp32 [total][n_heads] or NULL
 *   max_q, max_len  longest chunk, and most tokens that a sequence of the call
 *              holds in the cache, or 0 if not known: only help to choose whether
 *              rows are split along their keys
 *   workspace  dev, 256-byte aligned, not shared with a call that may run at the
 *              same time, or NULL: no row is split
 * A sequence id out of range is reported, its rows become zeros (lse -infinity);
 * row starts that do not ascend are reported and touch nothing out of range.
 * bf16 caches: blocks of values whose scale is below 2^-80 of another's, or of the
 * 16-bit values', may count as larger, up to that; values near the type's largest,
 * whose sum over a row's keys times 2^14 leaves fp32, may give infinities. Results are the same bits on every run with the same arguments. */
m2c_status m2c_kv_attend_chunk(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n,
                               const int32_t* cu, int64_t total, int32_t n_heads, float scale,
                               const void* q, const int64_t q_stride[2], const void* k,
                               const int64_t k_stride[2], const void* v, const int64_t v_stride[2],
                               void* out, const int64_t out_stride[2], float* lse, int32_t max_q,
                               int32_t max_len, void* workspace, int64_t workspace_bytes,
                               void* stream);

/* Evict blocks by accumulated weight. The last block of a sequence always
 * stays; of the m blocks before it every key/value head keeps
 * `keep` if m > keep (all of them otherwise): the first `first`, the last
 * `recent`, and of the others the heaviest, ties to the lowest index (weights
 * compare as the keys of m2c_predict_rank's scores). The entries of the head's
 * table and weight rows move together: kept blocks in order, then the last
 * block and the unused entries in order, then the evicted blocks in order with
 * weight 0 (their pages are the next to be used, or the caller's to take). The
 * length falls by block_tokens per evicted block.
 * 0 <= first, 0 <= recent, first + recent <= keep.
 * table_out, weight_out, len_out: arrays like the cache's that get the rows of
 * the listed sequences instead, the cache unchanged; all three or none (NULL). */
m2c_status m2c_kv_evict(const m2c_kv_cache* cache, const int32_t* seqs, int32_t n, int32_t keep,
                        int32_t first, int32_t recent, int32_t* table_out, float* weight_out,
                        int32_t* len_out, void* stream);

/* Waits for `stream`, then reports and clears what the calls above found on
 * the device since the last check: M2C_ERR_INVALID_ARG (a sequence or page out
 * of range, row starts that do not ascend), M2C_ERR_CAPACITY, M2C_ERR_STATE, or M2C_OK. */
m2c_status m2c_kv_status(const m2c_kv_cache* cache, void* stream);

/* ------------------------------------------------------------------------
 * Between a layer's blocks: the residual stream and its norms
 * ------------------------------------------------------------------------
 * Per row of d elements, x the residual stream, y a block's output:
 *     t   = N(y) post_weight + post_bias if post, y otherwise
 *     r   = x + scale gate t                                    (x_out)
 *     out = N(r) weight + bias                                  (the next block's input)
 *     N(z) = (z - mean z) / sqrt(mean (z - mean z)^2 + eps), mean z taken as 0
 *            for M2C_NORM_RMS
 * All of it in fp32 (sums that leave its range in 64 bits, the row brought near 1 by
 * a power of two then), each output rounded once: out is of r, not of what x_out's type keeps of it. */
enum { M2C_NORM_RMS = 0, M2C_NORM_LAYER = 1 };

typedef struct {
  int32_t kind;          /* M2C_NORM_*, of both norms                           */
  int32_t post;          /* 1: y is normed before it is added                   */
  int32_t d;             /* elements of a row, 1..65536                         */
  int32_t device;        /* HIP device ordinal of every pointer                 */
  int32_t x_dtype;       /* of x and x_out: M2C_DTYPE_FP32, or the one 16-bit   */
  int32_t y_dtype;       /* type that the call uses; so are the others          */
  int32_t out_dtype;
  int32_t weight_dtype;  /* of weights, biases and gate                         */
  float eps;             /* >= 0 and finite                                     */
  float scale;           /* finite                                              */
  int64_t x_stride, y_stride, x_out_stride, out_stride; /* elements between rows,
                            0 .. 2^40; rows that are written must not overlap   */
  int64_t gate_stride;   /* between the rows of gate; 0: one for all            */
  const void *weight, *bias;           /* dev [d], or NULL: 1 and 0             */
  const void *post_weight, *post_bias; /* the same; NULL unless post            */
  const void* gate;      /* dev, or NULL: 1                                     */
} m2c_norm_desc;

/* One pass over `rows` rows (up to 2^30). y NULL: r = x (no post, gate). x_out
 * may be x, with its strides, or NULL; out may be NULL; otherwise what is written
 * must not overlap what is read. Any alignment of whole elements; rows of 16-byte
 * aligned starts whose length divides by 8 are faster. Results are the same bits
 * on every run. Only enqueues; keeps no state. */
m2c_status m2c_residual_norm(const m2c_norm_desc* desc, const void* x, const void* y, int64_t rows,
                             void* x_out, void* out, void* stream);

/* Test support. Copies one record of the host store (no device work). */
m2c_status m2c_debug_read_record(const m2c_layer* layer, int32_t tier, int32_t neuron, void* out,
                                 size_t bytes);
/* Test support. Synchronizes the device, then copies slot `slot` (0..C+S-1;
 * at most its pool's stride with M2C_FLAG_TIER_POOLS). */
m2c_status m2c_debug_read_slot(const m2c_layer* layer, int32_t slot, void* out, size_t bytes);
/* Test support. Synchronizes the device, then copies the tables of tier
 * `tier`'s pool (M2C_FLAG_TIER_POOLS): slot_of int32 [d_ff] (pool-local
 * resident slot or -1), slot_key int32 [tier_slots[tier]], slot_last int32
 * [tier_slots[tier]]; any pointer may be NULL. */
m2c_status m2c_debug_read_pool_tables(const m2c_layer* layer, int32_t tier, int32_t* slot_of,
                                      int32_t* slot_key, int32_t* slot_last);

/* Test support. Synchronizes the device, then copies the slot tables; any
 * pointer may be NULL. slot_of int32 [d_ff] (-1 = not resident);
 * slot_key int32 [C] (-1 = empty); slot_tier uint8 [C]; slot_last int32 [C]. */
m2c_status m2c_debug_read_tables(const m2c_layer* layer, int32_t* slot_of, int32_t* slot_key,
                                 uint8_t* slot_tier, int32_t* slot_last);

/* Test support. Enqueues on `stream` a kernel that overwrites with 0xFF
 * bytes every slot the fill of `plan` writes (slot_bytes each), except the
 * slots whose INT8 / INT4 record the fill may make from the FP16 bytes
 * already there (fill_from == 3). Enqueued right before m2c_cache_fill on the
 * same stream, it makes ordering mistakes visible: an FFN that reads a slot
 * before its fill completes reads 0xFF bytes (NaN as fp16, code -1 as
 * INT8 / INT4 with a NaN scale), and a fill that starts while an earlier FFN
 * still reads the slot corrupts that FFN's output. */
m2c_status m2c_debug_poison_fill_slots(m2c_layer* layer, const void* plan, void* stream);

/* Test support. polls > 0: the layer's one-launch batch-1 sparse FFN (d_model
 * <= 8192, not deterministic) stops publishing its h values and its down
 * tasks give up after `polls` polls, so that every later call takes the
 * bounded-wait give-up path (h = 0, status word set, M2C_ERR_STATE from the
 * next m2c_layer_stats) while every kernel still exits normally. polls == 0
 * restores the normal behaviour. Host-side setting; affects launches made
 * after the call. */
m2c_status m2c_debug_ffn_withhold_h(m2c_layer* layer, int32_t polls);

/* Message of the last error on this thread ("" if none). */
const char* m2c_last_error(void);

/* Identifier of the sources the library was built from (16 hex digits of a
 * SHA-256 over the kernel sources and this header), so that a loader can
 * refuse a library built from other sources. Static string, never NULL. */
const char* m2c_build_id(void);

#ifdef __cplusplus
}
#endif
#endif /* M2C_H */
