/*
 * hisparse.h -- C ABI of the HiSparse decode hot path on AMD Instinct MI355X (gfx950).
 *
 * HiSparse ("Scaling Sparse-Attention Decoding with Hierarchical KV Cache Management") keeps
 * every request's full KV history in pinned host memory and gives each (request, layer) a
 * small fixed-size GPU cache of B record slots (Section 3.2). Each decode step, the sparse
 * indexer emits k selected logical records per request and layer; the library resolves them
 * against the cache -- hit detection, LRU victim choice among the slots this step does not
 * reference, fetch of the misses from pinned host memory into the freed HBM slots, and
 * emission of the physical slot of every selected record in the selection's order
 * (Section 3.4, phases 1-5) -- and then runs sparse decode attention over the k gathered
 * records. For models whose layers share one indexer's selection, the anchor layer's miss
 * plan is replayed into every shared layer's cache (Section 3.5, exact prefetch).
 *
 * Terms used below
 *   unit   one independent cache: a (request, layer) for token-level selection, or a
 *          (request, layer, kv head) for block/page selection. Unit u of a layer call is
 *          request * units_per_request + head.
 *   L      logical records per unit (tokens, blocks or pages), positions 0 .. L-1.
 *   R      bytes per record.   k  selected records per unit per step.   B  slots per unit.
 *
 * Conventions
 *   - Pointers prefixed d_ are device (HBM) pointers owned by the caller; the library reads or
 *     writes them on the given stream and keeps no reference after the call returns.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *   - Calls marked [async] enqueue GPU work on `stream`, never synchronise the host, allocate
 *     nothing and can be captured in a HIP graph (with HISPARSE_FETCH_SDMA or
 *     HISPARSE_FETCH_STAGED, the calls that fetch synchronise `stream` once to read the miss
 *     plan back, and cannot be captured).
 *     Calls marked [sync] block the host.
 *   - Every call returns HISPARSE_OK or a negative hisparse_status_t; an argument error is
 *     reported before any work is enqueued, and leaves all state untouched.
 *   - Data errors found on the device (a selection entry >= L, or a repeated entry within one
 *     unit's selection) do not fail the enqueueing call: that unit's state is left unchanged,
 *     its k output slots are -1, its counts are (0, 0), and the error is latched for
 *     hisparse_check_errors. Negative selection entries are padding: output slot -1, not
 *     counted, never fetched.
 *   - One handle must not be used by two host threads at once; calls on one handle that touch
 *     the same layer must be ordered by the caller's streams.
 */
#ifndef HISPARSE_H
#define HISPARSE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hisparse_cache* hisparse_cache_t;

typedef enum {
  HISPARSE_OK = 0,
  HISPARSE_ERR_INVALID_ARG = -1,   /* bad descriptor, layer index, pointer or size */
  HISPARSE_ERR_OOM = -2,           /* device or pinned host allocation failed */
  HISPARSE_ERR_HIP = -3,           /* a HIP runtime call failed */
  HISPARSE_ERR_UNSUPPORTED = -4,   /* valid request the library does not implement */
  HISPARSE_ERR_BAD_SELECTION = -5, /* latched device-side selection error (see above) */
  HISPARSE_ERR_FULL = -6           /* every request slot is taken (hisparse_request_acquire) */
} hisparse_status_t;

/* How missed records travel from the host pool to the GPU cache (Section 3.4 Phase 4). */
typedef enum {
  /* GPU threads load the missed records straight from mapped pinned host memory with 16-byte
   * vector loads and store them into their slots: the GPU-assisted IO the paper adopts. */
  HISPARSE_FETCH_ZERO_COPY = 0,
  /* The host reads the miss plan back (a stream synchronisation) and issues one batched DMA
   * copy (hipMemcpyBatchAsync) of the missed records. Not capturable in a HIP graph: calls
   * that fetch return HISPARSE_ERR_UNSUPPORTED while `stream` is capturing. */
  HISPARSE_FETCH_SDMA = 1,
  /* Timing mode (the no-IO oracle of Section 4.6): tables and slot outputs are exact, but no
   * record is copied, so the cache holds stale data and attention outputs are not valid. */
  HISPARSE_FETCH_NONE = 2,
  /* Staging DMA (the staging alternative to GPU-assisted IO, Section 3.4 Phase 4): the host reads
   * the miss plan back (a stream synchronisation), host threads gather the missed records from
   * the pool into a pinned staging buffer, one copy-engine transfer moves them to the device
   * and a kernel scatters them into their slots. Not capturable, like HISPARSE_FETCH_SDMA; the
   * cache also holds top_k * R bytes of pinned and of device staging memory per unit, which
   * its staged fetches share: each one first waits on the host until the previous one, on
   * whatever stream, has scattered out of them. */
  HISPARSE_FETCH_STAGED = 3
} hisparse_fetch_t;

/* Kind of pinned host memory backing the pool. */
typedef enum {
  HISPARSE_HOST_COHERENT = 0,      /* fine-grained, mapped (hipHostMallocCoherent|Mapped) */
  HISPARSE_HOST_NONCOHERENT = 1,   /* coarse-grained, mapped (hipHostMallocNonCoherent|Mapped) */
  HISPARSE_HOST_UNCACHED = 2       /* fine-grained uncached (hipHostMallocUncached|Mapped) */
} hisparse_host_memory_t;

/* Cache descriptor (the paper's configuration: top_k, device buffer size B, transfer block
 * size; Appendix A "Configuration", Section 3.2 "Sizing the cache"). */
typedef struct {
  int32_t num_requests;          /* >= 1 */
  int32_t num_layers;            /* >= 1 */
  int32_t units_per_request;     /* 1 (token-level) or kv heads (block/page selection) */
  int32_t capacity;              /* B: slots per unit; top_k <= B <= 16384 */
  int64_t num_records;           /* L: records per unit, 1 .. 2^31-1 */
  int32_t top_k;                 /* k: 1 .. 4096. The resolve kernel takes 16 * round_up(k, 4)
                                    + B / 4 + 8192 bytes of LDS (at most 76 KiB); create returns
                                    UNSUPPORTED on a device whose workgroups get less */
  int32_t record_bytes;          /* R: multiple of 16, 16 .. 1 MiB */
  int32_t share_group;           /* G >= 1: layers with layer % G == 0 are anchors that resolve;
                                    layer l with l % G != 0 shares the selection of anchor
                                    l - l % G (Section 3.5) */
  int32_t fetch;                 /* hisparse_fetch_t */
  int32_t host_memory;           /* hisparse_host_memory_t */
  int32_t transfer_block_bytes;  /* bytes each fetch thread keeps in flight: 16, 32, 64, 128
                                    or 256 (the paper's swap-in transfer block size); 0 = 16 */
  int32_t fetch_workgroups;      /* one-wave (64-thread) workgroups of one fetch launch,
                                    0 .. 4096, shared by its units and target layers (at least
                                    one per unit and layer); 0 = 192 for records under 4 KiB,
                                    256 for larger ones (measured best). A few hundred KB of host
                                    reads in flight saturate the link, so a thin grid moves
                                    misses as fast as a wide one while keeping few slow host
                                    reads outstanding per CU, which leaves kernels of other
                                    streams on the same CUs (attention, resolve) nearly
                                    undisturbed */
} hisparse_cache_desc_t;

/* Sparse decode attention descriptor. The token layout inside a record is
 * [tokens_per_record][token_elems] bf16 with token_elems = record_bytes / 2 / tokens_per_record;
 * the key is the token's first d_qk elements and the value its d_v elements from v_offset.
 * Supported shapes: (d_qk, d_v, v_offset) = (576, 512, 0), latent MLA where the value is the
 * first 512 dims of the 576-dim latent record; and (128, 128, 128), GQA with K then V.
 * top_k * tokens_per_record (tokens per unit) is at most 2^24, and at most 2^20 for latent MLA
 * (HISPARSE_ERR_UNSUPPORTED above that). */
typedef struct {
  int32_t q_heads;               /* query heads attending to one unit: 1 .. 256 */
  int32_t d_qk;
  int32_t d_v;
  int32_t v_offset;
  int32_t tokens_per_record;     /* 1 (token records), 16 (pages), 64 (blocks), ... */
  int32_t num_splits;            /* partitions of the token sequence reduced in a fixed order;
                                    0 = chosen from the shape alone */
  float scale;                   /* softmax scale applied to q.k */
  int32_t flags;                 /* 0 or HISPARSE_ATTN_DEFER_MERGE | HISPARSE_ATTN_BESIDE_FETCH |
                                    HISPARSE_ATTN_CARRIES_REPLAY */
} hisparse_attn_desc_t;

/* hisparse_attn_desc_t.flags: the attention call runs only its per-split workgroups (and any
 * replay it carries) and leaves the splits' partial results in d_workspace without writing
 * d_out; hisparse_attention_merge then writes d_out from them. For callers that schedule,
 * overlap or time the two kernels apart. */
#define HISPARSE_ATTN_DEFER_MERGE 1
/* hisparse_attn_desc_t.flags, a scheduling hint: the call runs beside
 * another stream's host-link fetch (e.g. two micro-batches taking turns on the link), whose slow
 * host reads occupy the memory pipelines of the CUs they run on. Unless num_splits asks for a number
 * of splits, the plan then takes fewer, longer ones: latent attention aims at half a workgroup per CU
 * instead of one; grouped-query calls of more than five rounds of a workgroup's waves (128 tokens per
 * round up to 16 heads, 64 up to 32, 32 above) take at least six rounds per split. The fetch's waves
 * find CUs without an attention workgroup, and the split partial results shrink; on a GPU of its own
 * the call is slower that way. Set it on the call and on its hisparse_attention_merge (or
 * _merge_prefetch) alike. Results differ only within rounding (other split boundaries); each plan
 * is deterministic. */
#define HISPARSE_ATTN_BESIDE_FETCH 2
/* hisparse_attn_desc_t.flags, a scheduling hint: the call carries an exact-prefetch replay
 * (hisparse_sparse_decode_prefetch, _part) whose host-link transfer takes longer than the attention
 * itself, so the launch lasts as long as the replay and the merge that follows it sits on the decode
 * chain (Section 3.5). In latent attention with fewer than 16 workgroup columns (one per unit and 64
 * heads, or 32 if there are no more), more than 256 tokens per unit and at least 2048 over all units,
 * the plan then takes splits of at least two rounds of 64 tokens: half the attention workgroups, which
 * stay hidden behind the replay and leave it more CUs, and half the split partials for the merge to
 * read. From 5 columns on the plan does so by itself, so there the hint changes nothing more.
 * Latent calls of up to 32 heads aim at half a workgroup per CU.
 * Grouped-query calls of up to 16 heads that would leave the replay fewer than a quarter of the CUs
 * take splits of at least four rounds of 128 tokens. Set it on the carrying call and on its
 * hisparse_attention_merge (or _merge_prefetch). Results differ only within rounding (other split
 * boundaries); each plan is deterministic. */
#define HISPARSE_ATTN_CARRIES_REPLAY 4

/* Human-readable name of a status code (static storage). */
const char* hisparse_status_string(hisparse_status_t status);

/* [pure host] Check a cache descriptor without touching any device. */
hisparse_status_t hisparse_validate_desc(const hisparse_cache_desc_t* desc);

/* [pure host] Check an attention descriptor against a cache descriptor's record layout. */
hisparse_status_t hisparse_validate_attn(int32_t record_bytes, int32_t top_k,
                                         const hisparse_attn_desc_t* attn);

/* [sync] Create a cache on HIP device `device`. Allocates, and owns until destroy:
 *   - per layer, a pinned mapped host pool [units][L][R] (the authoritative full KV,
 *     Section 3.2 "host KV pool"), uninitialised -- the caller stages prefill KV into it
 *     (hisparse_host_pool) before resolving;
 *   - per layer, the GPU cache [units][B][R] in HBM;
 *   - per anchor layer, the page table [units][L] int32 (-1 = host-only), slot map [units][B]
 *     int32 (-1 = empty), LRU timestamps [units][B] uint32, recency index [units][B], step clock
 *     [units] and miss plan [units][k] -- all initialised to the cold state.
 * On failure nothing stays allocated and *out is NULL. */
hisparse_status_t hisparse_cache_create(const hisparse_cache_desc_t* desc, int32_t device,
                                        hisparse_cache_t* out);

/* [sync] Release everything the handle owns. NULL is accepted. */
hisparse_status_t hisparse_cache_destroy(hisparse_cache_t cache);

/* Host address and size of layer `layer`'s pinned host pool, laid out [units][L][R]: record r
 * of unit u starts at host + (u * L + r) * R. The caller may write it whenever no GPU work
 * that reads it is in flight. */
hisparse_status_t hisparse_host_pool(hisparse_cache_t cache, int32_t layer, void** host,
                                     size_t* bytes);

/* Device address and size of layer `layer`'s GPU cache, laid out [units][B][R]. */
hisparse_status_t hisparse_layer_cache(hisparse_cache_t cache, int32_t layer, void** device,
                                       size_t* bytes);

/* [async] Return every anchor layer's units to the cold state (all slots empty, clocks 0). */
hisparse_status_t hisparse_reset(hisparse_cache_t cache, void* stream);

/* ---- Request lifecycle (Section 3.3 (1) prefill and staging, (2) admission) ----
 * A cache reserves every unit's slot caches and tables for all its layers when it is created
 * (num_layers * B * R bytes of slots per unit, the per-request reservation Section 3.3 (2)
 * sizes by B rather than by context length), so admitting a request allocates nothing: it takes
 * one of num_requests request slots, whose units are
 * [request * units_per_request, (request + 1) * units_per_request). */

/* Take a free request slot, lowest index first (host bookkeeping; no GPU work, and the kernels
 * do not consult it). All slots are free after creation. Returns HISPARSE_ERR_FULL, leaving
 * *request = -1, when every slot is taken. */
hisparse_status_t hisparse_request_acquire(hisparse_cache_t cache, int32_t* request);

/* [async] Give a request slot back: its units go back to the cold state in every anchor layer
 * (hisparse_reset_units on `stream`) and the slot is free for the next acquire at once, so
 * work for the next request on those units must be ordered after this call by `stream`.
 * Returns INVALID_ARG for a slot that is out of range or not taken. */
hisparse_status_t hisparse_request_release(hisparse_cache_t cache, int32_t request,
                                           void* stream);

/* [async] Cold state for units [first_unit, first_unit + num_units) of every anchor layer, as
 * after creation: page-table rows cleared, slots empty, stamps and clocks 0, recency index in
 * slot order, miss plans empty. Other units, the GPU caches' bytes and the host pools are
 * untouched. 1 <= num_units, first_unit + num_units <= units. */
hisparse_status_t hisparse_reset_units(hisparse_cache_t cache, int32_t first_unit,
                                       int32_t num_units, void* stream);

/* [async] Prefill staging (Section 3.3 (1)): copy records [first_record, first_record +
 * num_records) of units [first_unit, first_unit + num_units) of layers [first_layer,
 * first_layer + num_layers) from device memory into the host pools with the copy engines
 * (device-to-host hipMemcpyAsync, one per layer when num_records = L or num_units = 1, else one
 * per unit and layer).
 *   d_src  device; layer first_layer + j at d_src + j * src_layer_stride, laid out
 *          [num_units][num_records][R] (not modified).
 *   src_layer_stride  bytes, >= num_units * num_records * R; ignored when num_layers = 1.
 * The records may be resolved once this work has completed (the staging acknowledgement: an
 * event the caller records on `stream` after the call). The staged range must not be read by
 * fetches in flight. Capturable in a HIP graph. */
hisparse_status_t hisparse_stage(hisparse_cache_t cache, int32_t first_layer, int32_t num_layers,
                                 int32_t first_unit, int32_t num_units, int64_t first_record,
                                 int64_t num_records, const void* d_src,
                                 int64_t src_layer_stride, void* stream);

/* [async] Resolve one step of an anchor layer (Section 3.4 phases 1-5).
 *   d_sel    int32 [units][k]: selected positions per unit, in the indexer's order.
 *   d_slots  int32 [units][k]: out; d_slots[u][i] is the slot of unit u now holding record
 *            d_sel[u][i] (Section 3.3 (3): aligned with the selection's order); -1 for padding.
 *   d_counts int32 [units][2]: out, {hits, misses} per unit; may be NULL.
 * Replacement is LRU among the slots the step does not reference, with this step's hits
 * promoted above its newly fetched misses (Section 3.2 "Replacement policy"). Ties are
 * canonical: misses of step t are stamped 2t-1 and hits 2t (t = the unit's valid steps so
 * far + 1); victims are taken in ascending (timestamp, slot) order, empty slots first, and
 * the i-th miss in ascending position order takes the i-th victim. Misses are fetched from
 * this layer's host pool (unless fetch = HISPARSE_FETCH_NONE), and the miss plan is kept for
 * hisparse_prefetch_layer. Returns INVALID_ARG for a shared (non-anchor) layer. */
hisparse_status_t hisparse_resolve(hisparse_cache_t cache, int32_t layer, const int32_t* d_sel,
                                   int32_t* d_slots, int32_t* d_counts, void* stream);

/* [async] The two halves of hisparse_resolve, for callers that schedule or time them apart
 * (the paper's breakdown of a resolve into metadata phases and IO, Section 4.4):
 * hisparse_resolve_tables runs phases 1-3 and 5 -- every output of hisparse_resolve and the
 * miss plan, but no record is copied; hisparse_fetch then runs phase 4, copying the records of
 * the anchor layer's latest miss plan from its host pool into its GPU cache (a no-op under
 * HISPARSE_FETCH_NONE). hisparse_resolve == hisparse_resolve_tables + hisparse_fetch. */
hisparse_status_t hisparse_resolve_tables(hisparse_cache_t cache, int32_t layer,
                                          const int32_t* d_sel, int32_t* d_slots,
                                          int32_t* d_counts, void* stream);
hisparse_status_t hisparse_fetch(hisparse_cache_t cache, int32_t layer, void* stream);

/* [async] Phase 4 for entries [m * part_begin / 256, m * part_end / 256) of each unit's plan
 * of m entries only, 0 <= part_begin <= part_end <= 256: calls over adjacent ranges together
 * equal hisparse_fetch. A caller that hands the host link from one stream to another can let
 * the next stream's transfer start after the first part (an event recorded between the calls)
 * while the rest of this one still runs. */
hisparse_status_t hisparse_fetch_part(hisparse_cache_t cache, int32_t layer, int32_t part_begin,
                                      int32_t part_end, void* stream);

/* [async] hisparse_fetch (Section 3.4 Phase 4) taking turns on the host link with fetches
 * issued on other streams, ordered on the device instead of by stream events. The paper
 * overlaps the fetch with other work so that IO stays off the critical path (Section 3.5);
 * with several independent batches of units, each with its own stream, one batch's fetch
 * overlaps another's attention best when the fetches use the link one after another.
 *   d_turns int32 [2 * n_turns] (n_turns >= 1), device memory owned by the caller, zeroed with
 *     hisparse_link_turns_reset before the first launch of a sequence of turns; turn i is
 *     the pair d_turns[2i], d_turns[2i + 1]. Each turn is signalled by one launch and waited
 *     for by at most one.
 *   wait_turn: -1, or the turn whose signal this launch waits for before its first host
 *     read. The launch's waves are resident while they wait, polling d_turns.
 *   signal_turn: -1, or the turn this launch signals once signal_share / 256 (1..256) of its
 *     workgroups have finished their copies (256: all of them, the link free).
 * The copies and results equal hisparse_fetch's whatever the order of the launches: a turn
 * orders only the use of the link, never data. A wait ends by itself after about 4 ms once
 * the signalling launch has started, or after about 50 us if it has not (not yet issued, or
 * queued behind this launch), so a turn that cannot be signalled in time (reset missing, its
 * launch on a stream that waits for this one, launches serialised by a tool) costs time, not
 * correctness. For a sequence issued on streams that may run concurrently.
 * HISPARSE_ERR_UNSUPPORTED unless the cache fetches zero-copy (the host-issued paths and
 * HISPARSE_FETCH_NONE launch no kernel); INVALID_ARG for a shared layer, a null d_turns,
 * n_turns < 1, indices outside [-1, n_turns), wait_turn == signal_turn, or a share outside
 * 1..256. */
hisparse_status_t hisparse_fetch_turn(hisparse_cache_t cache, int32_t layer, int32_t* d_turns,
                                      int32_t n_turns, int32_t wait_turn, int32_t signal_turn,
                                      int32_t signal_share, void* stream);

/* [async] Zero n_turns (1..2^24) link turns, d_turns[0 .. 2 * n_turns), with a fill kernel on
 * `stream` (capturable; no memset node), launched on the calling thread's current HIP device,
 * which must hold d_turns and `stream`. See hisparse_fetch_turn. */
hisparse_status_t hisparse_link_turns_reset(int32_t* d_turns, int32_t n_turns, void* stream);

/* [async] Phase 4 for units [unit_begin, unit_begin + unit_count) of an anchor layer only
 * (Section 3.4; units are independent caches). Calls over disjoint ranges together equal
 * hisparse_fetch, so a caller can pipeline a layer's fetch with the attention of the units
 * already fetched. HISPARSE_ERR_INVALID_ARG for a range outside [0, units). */
hisparse_status_t hisparse_fetch_units(hisparse_cache_t cache, int32_t layer,
                                       int32_t unit_begin, int32_t unit_count, void* stream);

/* [async] Phase 4 of an anchor layer and the exact-prefetch replay of the same miss plan into
 * its next num_layers - 1 shared layers (Section 3.5), in one launch: equal to hisparse_fetch
 * followed by hisparse_prefetch_layer for each of those layers, for a caller with nothing to
 * overlap the replays with. HISPARSE_ERR_INVALID_ARG unless 1 <= num_layers <= share_group and
 * the layers exist. */
hisparse_status_t hisparse_fetch_group(hisparse_cache_t cache, int32_t anchor_layer,
                                       int32_t num_layers, void* stream);

/* [async] Exact prefetch (Section 3.5): replay the miss plan recorded by the latest resolve of
 * `anchor_layer` into the cache of `shared_layer` (anchor < shared < anchor + share_group),
 * copying each planned record from shared_layer's own host pool into the same slot. After the
 * replay, shared_layer's cache holds its records for the anchor's selection in the anchor's
 * slots, so its attention reads through the anchor's d_slots. The caller orders it after that
 * resolve (e.g. an event) and before the shared layer's attention, and must not start the
 * anchor's next resolve before the replay has completed. */
hisparse_status_t hisparse_prefetch_layer(hisparse_cache_t cache, int32_t anchor_layer,
                                          int32_t shared_layer, void* stream);

/* [async] hisparse_prefetch_layer for the num_layers consecutive shared layers first_shared ..
 * first_shared + num_layers - 1 of `anchor_layer`'s group, in one launch (Section 3.5): the
 * side-stream form of the replay, started as soon as the anchor's resolve has recorded its
 * plan, so that it shares the host link with the anchor's own fetch and runs under the anchor
 * layer's attention. Same ordering rules as hisparse_prefetch_layer. HISPARSE_ERR_INVALID_ARG
 * unless anchor < first_shared and first_shared + num_layers <= min(anchor + share_group,
 * num_layers), num_layers >= 1. */
hisparse_status_t hisparse_prefetch_layers(hisparse_cache_t cache, int32_t anchor_layer,
                                           int32_t first_shared, int32_t num_layers,
                                           void* stream);

/* [async] Speculative cross-layer prefetch for models whose layers do not share selections
 * (Section 3.5, the speculative alternative to exact prefetch): anchor layer `layer` takes a
 * hint, typically the previous layer's selection of the same step, as one access event of its
 * canonical LRU, exactly as hisparse_resolve would take it as a selection: the layer's clock
 * advances, hinted records already resident are refreshed, the others are fetched into its
 * least-recent slots. Its own resolve later in the step then finds them resident. No slot
 * vector is written.
 *   d_hint   int32 [units][k], positions in [0, L) or -1 for padding (invalid entries latch
 *            HISPARSE_ERR_BAD_SELECTION as in hisparse_resolve).
 *   d_counts int32 [units][2]: out, {already resident, fetched} per unit; may be NULL.
 * A wrong hint costs transfers and evictions, never correctness: the layer's resolve still
 * makes every selected record resident. The hint replaces the layer's miss plan, so replays
 * into shared layers (hisparse_prefetch_layer) must follow the layer's own resolve. */
hisparse_status_t hisparse_speculate(hisparse_cache_t cache, int32_t layer,
                                     const int32_t* d_hint, int32_t* d_counts, void* stream);

/* [async] Write-through of generated records (Section 3.3 (4)): each unit's newly generated
 * record enters the GPU caches of layers [first_layer, first_layer + num_layers) and is written
 * through to those layers' host pools, in one launch. The range covers whole share groups:
 * first_layer is an anchor and the range ends at a group boundary or at the last layer.
 *   d_pos     int32 [units]: the new record's position per unit (< 0: nothing for that unit;
 *             >= num_records: HISPARSE_ERR_BAD_SELECTION latched, state unchanged).
 *   d_records bf16 records [num_layers][units][R].
 *   d_slots   int32 [groups in the range][units], out: the slot the position now occupies in
 *             each group (-1: none).
 * Each group's anchor admits the position as a one-entry resolve event: the unit's clock
 * advances by one; a resident position is refreshed in place, otherwise the least-recent slot
 * by (timestamp, slot) takes it with the event's miss stamp, exactly as the canonical LRU does
 * for a selection {pos}. Each layer's record is then stored into that slot of the layer's cache
 * and into position pos of the layer's host pool, by the GPU over the mapped pool, so any later
 * fetch of pos on a stream ordered after this call reads it. Order the call after every
 * attention that reads the slots of the groups' current step (an admission may evict one of
 * them) and before those anchors' next resolve; the resolves' miss plans are left intact.
 * HISPARSE_FETCH_NONE updates the tables only. */
hisparse_status_t hisparse_append(hisparse_cache_t cache, int32_t first_layer,
                                  int32_t num_layers, const int32_t* d_pos,
                                  const void* d_records, int32_t* d_slots, void* stream);

/* Bytes of device workspace for hisparse_sparse_decode(_pool) over `units` units of top_k records
 * each; 0 if the descriptor is invalid. A workspace of this size serves every call of at most
 * `units` units with the same top_k, record_bytes and attn: a server that sizes one for its largest
 * batch needs no other. A scheduling hint (HISPARSE_ATTN_BESIDE_FETCH, _CARRIES_REPLAY) can lower the
 * size and another num_splits can raise it, so a caller that makes calls with several descriptors
 * takes the largest of their sizes. */
size_t hisparse_decode_workspace_bytes(int32_t units, int32_t top_k, int32_t record_bytes,
                                       const hisparse_attn_desc_t* attn);

/* [async] Sparse decode attention of one layer over its GPU cache (the consumer of Section 3.4
 * Phase 5's slot vector).
 *   d_q     bf16 [units][q_heads][d_qk] query.
 *   d_slots int32 [units][k]: slots from hisparse_resolve (the anchor's, for a shared layer);
 *           -1 entries are skipped.
 *   d_out   float32 [units][q_heads][d_v]: out_h = sum_j softmax_j(scale * q_h . key_j) value_j
 *           over the tokens of the selected records. A unit with no valid record gets zeros.
 *   d_workspace / workspace_bytes: caller-owned scratch of at least
 *           hisparse_decode_workspace_bytes(units, k, R, attn) bytes.
 * The reduction order depends only on the position of a record in the slot vector, never on
 * the slot value, so the result is bit-identical to hisparse_sparse_decode_pool over any other
 * placement of the same records. */
hisparse_status_t hisparse_sparse_decode(hisparse_cache_t cache, int32_t layer, const void* d_q,
                                         const int32_t* d_slots, float* d_out,
                                         const hisparse_attn_desc_t* attn, void* d_workspace,
                                         size_t workspace_bytes, void* stream);

/* [async] The merge of an attention call made with HISPARSE_ATTN_DEFER_MERGE: combines the
 * per-split partial results in d_workspace into d_out (float32 [units][q_heads][d_v]), in
 * the fixed split order, so deferred call + merge == the same call without the flag, bit for
 * bit. units, top_k, record_bytes and attn (HISPARSE_ATTN_DEFER_MERGE aside) must be those of
 * the deferred call,
 * whose `units` is the cache's units times the layer count for hisparse_sparse_decode_layers;
 * the workspace must not be reused in between. */
hisparse_status_t hisparse_attention_merge(int32_t units, int32_t top_k, int32_t record_bytes,
                                           const hisparse_attn_desc_t* attn, float* d_out,
                                           const void* d_workspace, size_t workspace_bytes,
                                           void* stream);

/* Bytes of device scratch each GPU holds for hisparse_sparse_decode_noalloc (64 MiB). */
#define HISPARSE_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)

/* [async] hisparse_sparse_decode without a workspace, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the split partial results go to a scratch array of HISPARSE_NOALLOC_SCRATCH_BYTES that the
 * library holds on each GPU it runs on until the process ends, and the call allocates nothing.
 * Same arguments, output and bits as hisparse_sparse_decode with a workspace.
 *   - HISPARSE_ERR_UNSUPPORTED if the call needs more scratch than that (never while
 *     hisparse_decode_workspace_bytes(units, k, R, attn) <= HISPARSE_NOALLOC_SCRATCH_BYTES);
 *   - HISPARSE_ERR_INVALID_ARG with HISPARSE_ATTN_DEFER_MERGE (the partials have no owner).
 * Every call on one GPU shares that GPU's scratch, from any handle: calls that may overlap on
 * one GPU (other streams, other host threads) race and must be ordered by the caller. */
hisparse_status_t hisparse_sparse_decode_noalloc(hisparse_cache_t cache, int32_t layer,
                                                 const void* d_q, const int32_t* d_slots,
                                                 float* d_out, const hisparse_attn_desc_t* attn,
                                                 void* stream);

/* [async] hisparse_sparse_decode of `layer` and, in the same launch, the exact-prefetch replay
 * of `anchor_layer`'s latest plan into shared layers [first_shared, first_shared + num_shared)
 * (Section 3.5): equal to hisparse_prefetch_layers followed by hisparse_sparse_decode, but the
 * replay runs in extra workgroups beside the attention, so the next layers' misses cross the
 * host link while this layer attends, on one stream. Ordering rules of
 * hisparse_prefetch_layer apply to the replay. With HISPARSE_FETCH_SDMA the replay is issued
 * on its own first (host-synchronising); with HISPARSE_FETCH_NONE nothing is copied.
 * HISPARSE_ERR_INVALID_ARG for a replay range hisparse_prefetch_layers would refuse, for
 * num_shared > 8, or if `layer` is one of the replay's targets. */
hisparse_status_t hisparse_sparse_decode_prefetch(hisparse_cache_t cache, int32_t layer,
                                                  const void* d_q, const int32_t* d_slots,
                                                  float* d_out, const hisparse_attn_desc_t* attn,
                                                  void* d_workspace, size_t workspace_bytes,
                                                  int32_t anchor_layer, int32_t first_shared,
                                                  int32_t num_shared, void* stream);

/* [async] hisparse_sparse_decode_prefetch carrying only part of the replay: entries
 * [m * part_begin / 256, m * part_end / 256) of each unit's plan of m entries, 0 <= part_begin
 * <= part_end <= 256 (0, 256: all of it, i.e. hisparse_sparse_decode_prefetch). Calls with
 * adjacent ranges, e.g. one carried by hisparse_attention_merge_prefetch and the rest by this
 * call, copy every planned record exactly once. Same ordering rules and errors. */
hisparse_status_t hisparse_sparse_decode_prefetch_part(
    hisparse_cache_t cache, int32_t layer, const void* d_q, const int32_t* d_slots,
    float* d_out, const hisparse_attn_desc_t* attn, void* d_workspace, size_t workspace_bytes,
    int32_t anchor_layer, int32_t first_shared, int32_t num_shared, int32_t part_begin,
    int32_t part_end, void* stream);

/* [async] hisparse_attention_merge of a deferred attention call made on `cache` (its units, top
 * k and record size; attn as in that call) whose launch also carries part of an exact-prefetch
 * replay (Section 3.5): entries [m * part_begin / 256, m * part_end / 256) of each unit's plan of
 * `anchor_layer`, into shared layers [first_shared, first_shared + num_shared), in extra
 * workgroups beside the merge. For a decode loop whose every attention call carries the replay
 * into a later shared layer, the merges would otherwise leave the host link idle; starting the
 * next-but-one layer's replay in them keeps it busy, and the attention call that follows carries
 * the rest (hisparse_sparse_decode_prefetch_part). Ordering rules of hisparse_prefetch_layer
 * apply to the replay. HISPARSE_ERR_INVALID_ARG for a replay range
 * hisparse_sparse_decode_prefetch_part would refuse. */
hisparse_status_t hisparse_attention_merge_prefetch(hisparse_cache_t cache,
                                                    const hisparse_attn_desc_t* attn,
                                                    float* d_out, const void* d_workspace,
                                                    size_t workspace_bytes, int32_t anchor_layer,
                                                    int32_t first_shared, int32_t num_shared,
                                                    int32_t part_begin, int32_t part_end,
                                                    void* stream);

/* [async] Sparse decode attention of layers [first_layer, first_layer + num_layers) of one
 * share group in a single launch (Section 3.5: the shared layers read their records through
 * the anchor's slots; batching them is this library's scheduling choice, the result per layer
 * is the same attention as hisparse_sparse_decode up to the split boundaries).
 *   d_q     bf16 [num_layers][units][q_heads][d_qk].
 *   d_slots int32 [units][k]: the anchor's slot vector, read by every layer.
 *   d_out   float32 [num_layers][units][q_heads][d_v].
 *   d_workspace / workspace_bytes: at least
 *           hisparse_decode_workspace_bytes(num_layers * units, k, R, attn) bytes.
 * HISPARSE_ERR_INVALID_ARG if the layers span two share groups. */
hisparse_status_t hisparse_sparse_decode_layers(hisparse_cache_t cache, int32_t first_layer,
                                                int32_t num_layers, const void* d_q,
                                                const int32_t* d_slots, float* d_out,
                                                const hisparse_attn_desc_t* attn,
                                                void* d_workspace, size_t workspace_bytes,
                                                void* stream);

/* [async] The same attention over an explicit device pool [units][records_per_unit][R], with
 * d_idx int32 [units][k] record indices into each unit's part of the pool (-1 = skip). Used for
 * a fully resident KV (indices = positions), or any other placement. One unit's part of the
 * pool, records_per_unit * R bytes, must stay below 2 GiB (HISPARSE_ERR_UNSUPPORTED otherwise;
 * the same holds for B * R of a cache). */
hisparse_status_t hisparse_sparse_decode_pool(const void* d_pool, int64_t records_per_unit,
                                              int32_t record_bytes, int32_t units, int32_t top_k,
                                              const void* d_q, const int32_t* d_idx, float* d_out,
                                              const hisparse_attn_desc_t* attn,
                                              void* d_workspace, size_t workspace_bytes,
                                              void* stream);

/* ---- Token records: writing, reading and attending to pools of K and V rows ----------------
 *
 * The calls below work on any device memory laid out as records, with no cache handle: a layer's
 * GPU cache (hisparse_layer_cache), the records handed to hisparse_append or hisparse_stage, or a
 * pool of pages of the caller's own. A record holds tokens_per_record tokens of one kv head;
 * hisparse_kv_desc_t says how a token lies in it and where the records are. */

/* What a token is made of: rows K and V. */
typedef enum {
  HISPARSE_KV_GROUPED = 0,  /* K 128 dims, V 128 dims: the (128, 128, 128) shape of
                               hisparse_attn_desc_t */
  HISPARSE_KV_LATENT = 1    /* K 512 latent dims, V 64 rotary dims: key = both (576), value = the
                               latent dims; the (576, 512, 0) shape */
} hisparse_kv_layout_t;

/* How its dims are stored. */
typedef enum {
  /* bf16 [tokens_per_record][K | V], the record layout of the sparse decode attention; token t
   * starts at t * (record_bytes / tokens_per_record). */
  HISPARSE_KV_BF16 = 0,
  /* 8 bits, n = tokens_per_record:
   *   grouped  e4m3 [n][K 128 | V 128], then float32 [n][2], the scales of K and of V;
   *   latent   e4m3 [n][512], then bf16 [n][64] (the rotary dims keep 16 bits), then float32
   *            [n], the scale of the latent dims.
   * A stored value stands for e4m3 * scale. The scale is a power of two per token and part, the
   * least one with (largest finite magnitude of the part) <= 448 * scale, at least 2^-117, and 1
   * for a part without a finite nonzero value. Values round to nearest even, infinities become
   * +-448 * scale, NaN stays NaN. Being powers of two, the scales round nothing: reading back gives
   * exactly the rounded values, and writing those again gives the same values. The exception is a part
   * whose largest finite magnitude is above 448 * 2^119, so that its scale is 2^120: from 248 * 2^120
   * on a value rounds to 2^128, which bf16 cannot hold, and with it infinities beside it are read back
   * (and attended to) as infinities. */
  HISPARSE_KV_FP8 = 1
} hisparse_kv_type_t;

/* Where the records are: record r of kv head h of request q is the record_bytes bytes at
 *   pool + q * request_stride + h * head_stride + r * record_stride.
 * Of a layer's GPU cache with B slots: num_records B, record_stride R, head_stride B * R,
 * request_stride units_per_request * B * R. Of one pool of pages shared by all requests, pages of
 * all heads [page][head]: record_stride heads * R, head_stride R, request_stride 0. */
typedef struct {
  int32_t layout;             /* hisparse_kv_layout_t */
  int32_t type;               /* hisparse_kv_type_t */
  int32_t tokens_per_record;  /* 1, 2, 4, ... 4096 */
  int32_t record_bytes;       /* multiple of 16, at least hisparse_kv_record_bytes, at most 8 MiB;
                                 for bf16 each token's share of it a multiple of 16 as well */
  int64_t num_records;        /* 1 .. 2^31 - 1: indices outside [0, num_records) are padding */
  int64_t record_stride;      /* bytes, multiples of 16, >= 0; record_stride at least record_bytes
                                 and below 2^31 */
  int64_t head_stride;
  int64_t request_stride;
} hisparse_kv_desc_t;

/* [pure host] The least record_bytes of a layout, type and tokens_per_record; 0 if there is no
 * such record. */
int32_t hisparse_kv_record_bytes(int32_t layout, int32_t type, int32_t tokens_per_record);

/* [pure host] Check a record descriptor. */
hisparse_status_t hisparse_validate_kv(const hisparse_kv_desc_t* kv);

/* [async] Write the rows of num_tokens tokens into their token slots, quantising them if the
 * records are 8-bit.
 *   d_k, d_v  bf16, row of token t and head h at t * {k,v}_token_stride + h * dims elements, dims
 *             128 and 128 (grouped) or 512 and 64 (latent): [tokens][heads][dims] arrays, or
 *             slices of a wider projection. Any alignment.
 *   d_slots   int64 [num_tokens]: token t goes to token (slot % tokens_per_record) of record
 *             (slot / tokens_per_record) of each head. A slot outside the pool (negative, or its
 *             record >= num_records) is padding: nothing is written. Slots must differ from one
 *             another; if two tokens name the same one, what it holds afterwards is unspecified
 *             (other slots are not affected). NULL: token t goes to slot t.
 * request_stride is not used: with request_stride = m * record_stride, request q's record r is
 * record q * m + r (num_records is then the bound over all requests).
 * Nothing but the slots' own rows and scales is written. num_tokens 0 does nothing.
 * HISPARSE_ERR_INVALID_ARG for a bad descriptor, null pointers, d_pool not a multiple of 16, heads
 * < 1, num_tokens < 0, negative strides, or head_stride < record_bytes with several heads;
 * HISPARSE_ERR_UNSUPPORTED if num_tokens * heads is more than 2^28 - 16 (grouped) or 2^26 - 4
 * (latent): one launch. */
hisparse_status_t hisparse_write_tokens(const hisparse_kv_desc_t* kv, int32_t heads,
                                        int32_t num_tokens, const void* d_k,
                                        int64_t k_token_stride, const void* d_v,
                                        int64_t v_token_stride, const int64_t* d_slots,
                                        void* d_pool, void* stream);

/* [async] The reverse: the rows that num_tokens token slots hold, in bf16 (8-bit values exactly), to
 * d_k and d_v laid out as above. A slot outside the pool gives rows of zeros. Slots may repeat.
 * Errors as above; a token stride below heads * dims is HISPARSE_ERR_INVALID_ARG too where num_tokens
 * > 1 (the rows would overlap). */
hisparse_status_t hisparse_read_tokens(const hisparse_kv_desc_t* kv, int32_t heads,
                                       int32_t num_tokens, const void* d_pool,
                                       const int64_t* d_slots, void* d_k, int64_t k_token_stride,
                                       void* d_v, int64_t v_token_stride, void* stream);

/* hisparse_chunk_desc_t.flags: new token i of n sees the cached tokens up to its own, number
 * len - n + i of its request's len. Without it every new token sees all of them (selected
 * records, which all precede the new tokens). */
#define HISPARSE_CHUNK_CAUSAL 1

/* Attention of a chunk of new tokens of each request over its records. */
typedef struct {
  int32_t num_requests;        /* >= 1 */
  int32_t kv_heads;            /* kv heads (units) of a request, >= 1; at most 2^20 of all requests */
  int32_t q_heads;             /* query heads on each kv head: 1 .. 256 */
  int32_t total_tokens;        /* rows of d_q and d_out: new tokens of all requests, or more */
  int32_t max_chunk;           /* the most new tokens of a request, >= 1; a longer chunk is held to
                                  its first max_chunk */
  int32_t max_records;         /* entries of a record table row: the longest request's records;
                                  max_records * tokens_per_record at most 2^30 */
  int64_t q_token_stride;      /* elements from one new token's heads to the next one's, >= 0 */
  int64_t out_token_stride;    /* >= kv_heads * q_heads * d_v */
  int64_t table_request_stride;  /* entries from one request's table to the next one's, >= 0 */
  int64_t table_head_stride;     /* and from one kv head's row to the next one's; 0: the heads
                                    share one row (a block table) */
  int32_t window;              /* 0, or the newest tokens a new token sees, its own included
                                  (needs HISPARSE_CHUNK_CAUSAL) */
  int32_t num_splits;          /* parts the cached tokens of a request are split into, merged in a fixed
                                  order: 1 .. 64 (fewer where it has fewer blocks of 64), and its
                                  results then do not depend on the rest of the batch; 0: chosen from
                                  the descriptors and the lengths of all requests of the call, so that
                                  a request's roundings may change with its neighbours */
  float scale;                 /* softmax scale applied to q.k, > 0, at most 1e6 */
  int32_t flags;               /* 0 or HISPARSE_CHUNK_CAUSAL */
} hisparse_chunk_desc_t;

/* [pure host] Check a chunk attention's descriptors. */
hisparse_status_t hisparse_validate_chunk(const hisparse_kv_desc_t* kv,
                                          const hisparse_chunk_desc_t* chunk);

/* [pure host] Bytes of device scratch for the call (0: none, d_workspace may be NULL); 0 too for
 * invalid descriptors. A workspace of this size serves every call of at most as many requests, total
 * tokens, new tokens per request and records with the same kv, heads, window and num_splits: a server
 * that sizes one for its largest batch needs no other. */
size_t hisparse_chunk_workspace_bytes(const hisparse_kv_desc_t* kv,
                                      const hisparse_chunk_desc_t* chunk);

/* [async] out = softmax(scale * q.k) v over the cached tokens that each new token sees, for every
 * query head; one call serves decoding requests (chunks of 1), drafted tokens to verify and
 * chunks of prompts side by side. The new tokens' own rows are in the cache already
 * (hisparse_write_tokens).
 *   d_table        int32, row of request q and kv head h at q * table_request_stride + h *
 *                  table_head_stride: the records that hold the request's cached tokens, in
 *                  order: cached token j is token (j % tokens_per_record) of record
 *                  table[j / tokens_per_record]. The tokens of an entry outside [0, num_records)
 *                  (padding) are not seen.
 *   d_chunk_start  int32 [num_requests + 1], ascending: request q's new tokens are rows start[q] ..
 *                  start[q + 1] - 1 of d_q and d_out. Rows outside every chunk (a batch padded to
 *                  a fixed size) are neither read nor written. Values are held to [0,
 *                  total_tokens]; where they do not ascend, what the rows of d_out and d_lse hold
 *                  afterwards is unspecified. NULL: every request has max_chunk new tokens, request q's from
 *                  row q * max_chunk; total_tokens >= num_requests * max_chunk.
 *   d_kv_len       int32 [num_requests]: cached tokens of each request, its new ones included; held
 *                  to [0, max_records * tokens_per_record]. NULL: that many everywhere. A request
 *                  with fewer cached than new tokens has new tokens that see nothing.
 *   d_q            bf16, token i's heads at i * q_token_stride, [kv_heads * q_heads][d_qk]: query
 *                  head e on kv head e / q_heads; d_qk 128 (grouped) or 576 (latent). Any
 *                  alignment.
 *   d_out          bf16 likewise with out_token_stride and d_v 128 or 512.
 *   d_lse          float32 [total_tokens][kv_heads * q_heads] or NULL: the natural logarithm of the
 *                  softmax's sum, to join results over parts of a cache. May be NULL.
 *   d_workspace    at least hisparse_chunk_workspace_bytes bytes, a multiple of 16; calls that may
 *                  overlap (other streams, graphs replayed side by side) need one each.
 * A new token that sees no cached token gives zeros and an lse of -inf. Scores, their maximum and
 * sums are kept in fp32; softmax weights are rounded to bf16 for the product with V. Where scores are
 * finite in fp32, results are too as long as the number of cached tokens times the largest |v| is below
 * 2^111. Tokens that are not seen (padding, later tokens, tokens before the window, page ends) have no
 * influence, whatever they hold, infinities and NaN included. One that is seen weighs by its score: at
 * -inf nothing (a new token that sees no other score gives what one that sees nothing gives), at +inf
 * or NaN every dim of the result and its lse are NaN. An infinity or NaN in a value that is seen makes
 * its dim of the result not finite; in a latent, key and value at once, NaN, and where its score is
 * not -inf all of the result and the lse (at -inf other dims and the lse are right or NaN too). Results
 * do not depend on where records lie.
 * HISPARSE_ERR_INVALID_ARG for bad descriptors, null or misaligned pointers, or a workspace too
 * small; HISPARSE_ERR_UNSUPPORTED for total_tokens * kv_heads * q_heads of 2^31 or more, or where
 * one launch would need 2^32 threads (512 for each 256 or fewer rows, kv head and split). More than
 * 1024 requests with starts or lengths are several launches, divided each for itself. */
hisparse_status_t hisparse_chunk_attention(const hisparse_kv_desc_t* kv,
                                           const hisparse_chunk_desc_t* chunk, const void* d_pool,
                                           const int32_t* d_table, const int32_t* d_chunk_start,
                                           const int32_t* d_kv_len, const void* d_q, void* d_out,
                                           float* d_lse, void* d_workspace,
                                           size_t workspace_bytes, void* stream);

/* ---- Before the attention: a batch's tables, rotary positions, index rows, selections -------
 *
 * One layer's step over records, in order: hisparse_plan_tokens (once for all layers) says where the
 * new tokens go, hisparse_rotate_tokens turns their rows, hisparse_write_tokens writes them,
 * hisparse_summarize_records keeps the index rows of the records they went to, and
 * hisparse_select_records chooses each new token's records, which hisparse_resolve or
 * hisparse_chunk_attention takes. No call needs a cache handle. */

/* The requests of a batch and their record tables, as in hisparse_chunk_desc_t. */
typedef struct {
  int32_t num_requests;          /* >= 1 */
  int32_t kv_heads;              /* >= 1; at most 2^20 of all requests */
  int32_t total_tokens;          /* rows of new tokens of all requests, or more; >= 0 */
  int32_t max_chunk;             /* the most new tokens of a request, >= 1; a longer chunk is held to
                                    its first max_chunk */
  int32_t max_records;           /* entries of a record table row: the longest request's records;
                                    max_records * tokens_per_record at most 2^30 */
  int32_t tokens_per_record;     /* 1, 2, 4, ... 4096 */
  int64_t table_request_stride;  /* entries from one request's table to the next one's, >= 0 */
  int64_t table_head_stride;     /* and from one kv head's row to the next one's; 0: the heads share
                                    one row (a block table) */
} hisparse_batch_desc_t;

/* [pure host] Check a batch descriptor. */
hisparse_status_t hisparse_validate_batch(const hisparse_batch_desc_t* batch);

/* [async] Block tables, slot map and positions of a batch of new tokens, from its lengths.
 *   d_new_len        int32 [num_requests]: new tokens of each request, 0 for none; held to [0,
 *                    max_chunk], to what its table row has room for, and all of them together, request
 *                    by request, to total_tokens rows.
 *   d_kv_len         int32 [num_requests]: tokens cached before, held to [0, max_records *
 *                    tokens_per_record]. NULL: none.
 *   d_free, num_free int32 [num_free]: records that no request has. The records that the new tokens
 *                    begin are taken from it in order, request by request. NULL (num_free 0): the
 *                    tables hold them already, and d_table is not written.
 *   d_free_used      int32 [1]: entries of d_free used before, held to [0, num_free]. NULL: none.
 *   d_table          int32, row of request q at q * table_request_stride (table_head_stride 0; rows
 *                    apart by at least max_records with several requests and a free list): read where a
 *                    request's cached tokens end inside a record; the entries of records that begin
 *                    are written, no other one is. -1 is written where d_free has none left: tokens in
 *                    such a record have no slot and are not seen by later calls.
 *   d_chunk_start    int32 [num_requests + 1], out: request q's new tokens are rows start[q] ..
 *                    start[q + 1] - 1.
 *   d_kv_len_out     int32 [num_requests], out: cached tokens, the new ones included. May be d_kv_len.
 *   d_free_used_out  int32 [1] or NULL, out: d_free_used and the records that begin. Above num_free: so
 *                    many were missing. May be d_free_used.
 *   d_positions      int32 [total_tokens] or NULL, out: each new token's position in its request; 0
 *                    in rows behind the last.
 *   d_slots          int64 [total_tokens] or NULL, out: its token slot, as hisparse_write_tokens takes
 *                    it, or -1 (no record, or a row behind the last), which that call skips.
 * The outputs and d_table, d_free, d_new_len must not overlap, but for the two pairs named.
 * HISPARSE_ERR_INVALID_ARG for a bad descriptor, null (d_new_len, d_table, d_chunk_start,
 * d_kv_len_out) or misaligned pointers, num_free < 0, num_free > 0 without d_free or d_free without
 * it, or table strides other than said; HISPARSE_ERR_UNSUPPORTED for num_free + total_tokens of 2^31 or
 * more. */
hisparse_status_t hisparse_plan_tokens(const hisparse_batch_desc_t* batch,
                                       const int32_t* d_new_len, const int32_t* d_kv_len,
                                       const int32_t* d_free, int32_t num_free,
                                       const int32_t* d_free_used, int32_t* d_table,
                                       int32_t* d_chunk_start, int32_t* d_kv_len_out,
                                       int32_t* d_free_used_out, int32_t* d_positions,
                                       int64_t* d_slots, void* stream);

/* Which dims make a pair, of the rotated dims 0 .. dims - 1. */
typedef enum {
  HISPARSE_ROTARY_HALF = 0,        /* i and i + dims / 2 */
  HISPARSE_ROTARY_INTERLEAVED = 1  /* 2 i and 2 i + 1 */
} hisparse_rotary_layout_t;

/* The frequency of pair i, in radians a position; f = theta^(-2 i / dims). */
typedef enum {
  HISPARSE_ROTARY_PLAIN = 0,   /* f */
  HISPARSE_ROTARY_LINEAR = 1,  /* f / factor: positions of a longer context squeezed into the trained one */
  /* f * (s + (1 - s) / factor), s = (r - low_turns) / (high_turns - low_turns) held to [0, 1], r = the
   * turns that the pair makes over the trained context, original_tokens * f / (2 pi): fast pairs as they
   * are, slow ones squeezed, a ramp between (over the turns; one over the pair's index is another). */
  HISPARSE_ROTARY_BY_PARTS = 2
} hisparse_rotary_scaling_t;

/* hisparse_rotary_desc_t.flags: turn by the negative angle: the gradient of the rows from the gradient
 * of the turned ones, or (magnitude 1) back to rows without a position. */
#define HISPARSE_ROTARY_BACK 1

typedef struct {
  int32_t dims;      /* rotated dims of a head: even, 2 .. 256 */
  int32_t layout;    /* hisparse_rotary_layout_t */
  int32_t scaling;   /* hisparse_rotary_scaling_t */
  int32_t flags;     /* 0 or HISPARSE_ROTARY_BACK */
  double theta;      /* > 0 */
  double factor;     /* > 0; not used by PLAIN */
  double original_tokens, low_turns, high_turns;  /* BY_PARTS: > 0, and low_turns < high_turns */
  double magnitude;  /* factor of the rotated dims, finite; 1: lengths are kept */
} hisparse_rotary_desc_t;

/* One array of rows to turn, bf16: row t of head h at d_in + t * in_token_stride + h * in_head_stride
 * elements, `dims` elements of which first .. first + rotary.dims - 1 are turned and the others copied.
 * Written to d_out likewise; token t's rows to row d_out_rows[t] of d_out if that is given, and nowhere
 * if that row is outside [0, num_out_rows) (a slot map of a pool of rows). Any alignment.
 * d_out may be d_in with the same strides and no d_out_rows: then only the rotated dims are written.
 * Otherwise no array written may overlap one that is read or written in the same call; out rows of a
 * token and head must not overlap, nor d_out_rows repeat a row. */
typedef struct {
  const void* d_in;
  void* d_out;
  const int64_t* d_out_rows;  /* int64 [num_tokens] or NULL */
  int64_t num_out_rows;       /* >= 0; not used without d_out_rows */
  int64_t in_token_stride, in_head_stride, out_token_stride, out_head_stride;  /* >= 0 */
  int32_t heads;              /* >= 1 */
  int32_t dims;               /* >= first + rotary.dims, at most 65536 */
  int32_t first;              /* >= 0 */
} hisparse_rotary_rows_t;

/* Arrays of rows that one call takes. */
#define HISPARSE_ROTARY_MAX_ROWS 4

/* [pure host] Check a rotary descriptor. */
hisparse_status_t hisparse_validate_rotary(const hisparse_rotary_desc_t* rotary);

/* [pure host] The dims / 2 frequencies of a descriptor, in radians a position. */
hisparse_status_t hisparse_rotary_frequencies(const hisparse_rotary_desc_t* rotary,
                                              double* frequencies);

/* [async] Rotary positions: in each of num_rows arrays (1 .. HISPARSE_ROTARY_MAX_ROWS: queries, keys, those of an
 * index) every pair (a, b) of token t becomes
 *   (a cos x - b sin x, b cos x + a sin x) * magnitude,  x = d_positions[t] * frequency of the pair,
 * angles in 64 bits, the rest in fp32, rounded to bf16 once.
 *   d_positions  int32 [num_tokens]; any value, of either sign.
 * The rows structs are read before the call returns. num_tokens 0 does nothing.
 * HISPARSE_ERR_INVALID_ARG for a bad descriptor, null or misaligned pointers, num_tokens < 0, bad heads,
 * dims, first or strides (with several heads an out_head_stride below dims, with several tokens an
 * out_token_stride below dims), or d_out equal to d_in with other strides or d_out_rows;
 * HISPARSE_ERR_UNSUPPORTED if num_tokens * heads * dims of all arrays is 2^38 or more. */
hisparse_status_t hisparse_rotate_tokens(const hisparse_rotary_desc_t* rotary, int32_t num_tokens,
                                         const int32_t* d_positions,
                                         const hisparse_rotary_rows_t* rows, int32_t num_rows,
                                         void* stream);

/* What a selection scores its candidates by, all bf16, 128 dims. */
typedef enum {
  /* a key of its own for each token: candidates are tokens; an index record holds
   * [tokens_per_record][128] */
  HISPARSE_INDEX_KEYS = 0,
  /* the least and the largest value of each dim over a record's keys: candidates are records; [2][128],
   * the least ones first */
  HISPARSE_INDEX_BOUNDS = 1,
  /* the mean of a record's keys: [128] */
  HISPARSE_INDEX_MEANS = 2
} hisparse_index_kind_t;

/* Where the index records are: that of record r of kv head h of request q at
 *   d_index + q * request_stride + h * head_stride + r * record_stride bytes.
 * r is the entry of the record table, so that an index beside a pool of pages has a record per page; or,
 * without a table, the record's place in its request (request_stride then tells the requests apart). */
typedef struct {
  int32_t kind;               /* hisparse_index_kind_t */
  int32_t tokens_per_record;  /* 1, 2, 4, ... 4096 */
  int64_t num_records;        /* 1 .. 2^31 - 1: entries outside [0, num_records) are padding */
  int64_t record_stride;      /* bytes, multiples of 16, >= 0; record_stride at least a record's bytes and
                                 below 2^31 */
  int64_t head_stride;
  int64_t request_stride;
} hisparse_index_desc_t;

/* [pure host] Check an index descriptor. */
hisparse_status_t hisparse_validate_index(const hisparse_index_desc_t* index);

/* [async] The index rows (BOUNDS or MEANS) of every record that holds new tokens of the batch, from the keys
 * of all its tokens: call it after hisparse_write_tokens, with the same lengths.
 *   kv             grouped records (HISPARSE_KV_GROUPED), bf16 or 8-bit; the keys are taken as read back.
 *   d_table        int32 as in hisparse_chunk_attention, or NULL: record j of a request is its record j.
 *                  Of an entry that is padding in the pool or in the index nothing is read or written.
 *   d_chunk_start  int32 [num_requests + 1] and
 *   d_kv_len       int32 [num_requests] as there, either may be NULL: new tokens (max_chunk each) and
 *                  cached tokens (max_records * tokens_per_record) of each request. A last record that
 *                  is not full is summarised over the tokens it holds.
 *   d_index        out: one or two rows of 128 per record and kv head.
 * Bounds are exact; a NaN in a dim makes its bounds NaN. Means are summed in fp32 in a fixed order and rounded
 * to bf16 once. Index records of other records keep what they hold. If two requests share a record that
 * both write to, each dim of its rows is that of one of them.
 * HISPARSE_ERR_INVALID_ARG for bad or differing descriptors (tokens_per_record alike in all three),
 * index kind KEYS, null or misaligned pointers (pool and index 16 bytes), a head_stride that lets kv heads'
 * index records overlap, or d_chunk_start NULL and total_tokens < num_requests * max_chunk;
 * HISPARSE_ERR_UNSUPPORTED for latent records, or where a launch would need 2^32 threads (64 for each
 * record and kv head). */
hisparse_status_t hisparse_summarize_records(const hisparse_kv_desc_t* kv,
                                             const hisparse_index_desc_t* index,
                                             const hisparse_batch_desc_t* batch,
                                             const void* d_pool, const int32_t* d_table,
                                             const int32_t* d_chunk_start, const int32_t* d_kv_len,
                                             void* d_index, void* stream);

typedef struct {
  int32_t q_heads;        /* queries on each kv head: KEYS 1 .. 128, else 1 .. 256 */
  int32_t top_k;          /* 1 .. 4096 */
  int32_t first_records;  /* >= 0: of the candidates a new token sees, so many first and */
  int32_t last_records;   /* >= 0: so many newest are always chosen; at most top_k together */
  int64_t q_token_stride;  /* elements from one new token's queries to the next one's, >= 0 */
} hisparse_select_desc_t;

/* [pure host] Check a selection's descriptors. */
hisparse_status_t hisparse_validate_select(const hisparse_index_desc_t* index,
                                           const hisparse_batch_desc_t* batch,
                                           const hisparse_select_desc_t* select);

/* [pure host] Bytes of device scratch for the call; 0 for invalid descriptors. A workspace of this size serves
 * every call of at most as many tokens and records with the same index kind and select and as many or
 * fewer kv heads. (The scores of all new tokens, held to 1 GiB or to one new token's: a call goes over its
 * tokens in as many steps as its workspace takes, and smaller workspaces, down to one new token's, are
 * accepted too. Results do not depend on it.) */
size_t hisparse_select_workspace_bytes(const hisparse_index_desc_t* index,
                                       const hisparse_batch_desc_t* batch,
                                       const hisparse_select_desc_t* select);

/* [async] The best candidates of each new token and kv head. New token i of n of a request with len cached
 * tokens, at position p = len - n + i, sees candidates 0 .. p (KEYS), or 0 .. p / tokens_per_record
 * (records, the one that holds it the last); padding entries are not seen. Candidate j scores, over the
 * kv head's queries q_e,
 *   KEYS    sum_e w_e max(0, q_e . key_j)
 *   BOUNDS  sum_e sum_d max(q_ed least_jd, q_ed largest_jd), taken as the sum over d of largest_jd times
 *           the sum of the positive q_ed, and least_jd times that of the negative ones
 *   MEANS   (sum_e q_e) . mean_j
 * and chosen are the first and last ones asked for and the best others, min(top_k, what it sees) in all.
 * The choice is that of scores in 64 bits, the lower position first among equals, NaN above everything:
 * fast scores only tell apart what their error bound does, and what that leaves open is scored again.
 * It does not depend on the rest of the batch, and index rows that are not seen have no influence,
 * whatever they hold.
 *   d_table, d_chunk_start, d_kv_len  as in hisparse_summarize_records. Rows outside every chunk (a batch
 *                padded to a fixed size) are neither read nor written.
 *   d_q          bf16, token i's queries at i * q_token_stride, [kv_heads * q_heads][128]. Any alignment.
 *   d_weights    float32 [total_tokens][kv_heads * q_heads], KEYS only, or NULL: 1.
 *   d_sel        int32 [total_tokens][kv_heads][top_k], out: the chosen candidates' positions in the
 *                request, ascending, and -1 behind them; with last_records > 0 the newest, p's own, stands
 *                at place min(top_k, p's candidates) - 1 even where padding leaves others empty. With one
 *                new token a request this is the selection hisparse_resolve takes.
 *   d_records    int32 likewise or NULL: the entry of the record table (KEYS: that times tokens_per_record
 *                and the token's place in it) instead of the position: with top_k as max_records, a
 *                request per row, chunks of 1, this and d_sel_len are d_table and d_kv_len of
 *                hisparse_chunk_attention over the selected records.
 *   d_sel_len    int32 [total_tokens] or NULL, out: tokens up to the row's own in those tables (0 for a token
 *                that sees nothing). Needs last_records > 0. Rows outside every chunk keep theirs: a caller
 *                that attends to all rows of a padded batch clears them first.
 *   d_workspace  a multiple of 16; calls that may overlap need one each.
 * HISPARSE_ERR_INVALID_ARG for bad descriptors (tokens_per_record of index and batch alike), null or
 * misaligned pointers (d_index and d_workspace 16 bytes), d_weights with another kind than KEYS, d_sel_len
 * without last_records, too small a workspace, or d_chunk_start NULL and total_tokens < num_requests * max_chunk;
 * HISPARSE_ERR_UNSUPPORTED for KEYS with d_records and num_records * tokens_per_record of 2^31 or more,
 * total_tokens * kv_heads of 2^31 or more, or kv_heads times candidates of 2^30 or more. */
hisparse_status_t hisparse_select_records(const hisparse_index_desc_t* index,
                                          const hisparse_batch_desc_t* batch,
                                          const hisparse_select_desc_t* select, const void* d_index,
                                          const int32_t* d_table, const int32_t* d_chunk_start,
                                          const int32_t* d_kv_len, const void* d_q,
                                          const float* d_weights, int32_t* d_sel,
                                          int32_t* d_records, int32_t* d_sel_len,
                                          void* d_workspace, size_t workspace_bytes, void* stream);

/* [sync] Copy an anchor layer's resolve state into host buffers (any may be NULL):
 * slot_pos int32 [units][B], slot_ts uint32 [units][B], page_table int32 [units][L],
 * order int32 [units][B] (slots by ascending (timestamp, slot)), clock uint32 [units]. */
hisparse_status_t hisparse_read_state(hisparse_cache_t cache, int32_t layer, int32_t* slot_pos,
                                      uint32_t* slot_ts, int32_t* page_table, int32_t* order,
                                      uint32_t* clock);

/* [sync] Copy an anchor layer's latest miss plan into host buffers (either may be NULL):
 * plan int32 [units][k][2] = (position, slot) for the first count[u] entries, in ascending
 * position order; count int32 [units]. */
hisparse_status_t hisparse_read_plan(hisparse_cache_t cache, int32_t layer, int32_t* plan,
                                     int32_t* count);

/* [sync] Return HISPARSE_ERR_BAD_SELECTION if a device-side selection error was latched since
 * the last check (info, if not NULL, receives {layer, unit, number of failing unit-steps}),
 * clearing the latch; otherwise HISPARSE_OK. */
hisparse_status_t hisparse_check_errors(hisparse_cache_t cache, int32_t* info);

/* Stamps per unit of the resolve kernel's phase timing (see hisparse_debug_resolve_phases). */
#define HISPARSE_RESOLVE_PHASE_SLOTS 16
/* The first units whose resolve workgroups record phase stamps. */
#define HISPARSE_RESOLVE_PHASE_UNITS 64

/* [sync] Diagnostic, Section 4.4's breakdown of the resolve into its phases: in a library built
 * with HISPARSE_PHASE_STAMPS (`python -m paper_2608_07009_amd.build --phase-stamps`, which
 * writes lib/libhisparse_phase_stamps.so), the resolve kernel stores the device's constant-rate
 * wall clock at its phase boundaries, for units below HISPARSE_RESOLVE_PHASE_UNITS, overwriting
 * the previous launch's stamps. This call waits for the current device and copies the stamps of
 * the first min(max_units, HISPARSE_RESOLVE_PHASE_UNITS) units into host_stamps (uint64
 * [units][HISPARSE_RESOLVE_PHASE_SLOTS], caller-owned): slot 0 kernel start, 1 selection staged
 * and probed (phase 1), 2 misses bucketed, 3 bucket starts scanned, 4 misses in position order
 * (phase 2), 5 victims chosen (phase 3a), 6 recency index and hit stamps written (phase 3b),
 * 7 tables, plan and slots updated (phase 5), 8 kernel end; slots 9.. are unused. A unit whose
 * selection was invalid stops after slot 4. ticks_per_s (if not NULL) receives the clock's rate.
 * Launches on several streams at once overwrite each other's stamps. In a normal build it
 * returns HISPARSE_ERR_UNSUPPORTED and touches nothing. */
hisparse_status_t hisparse_debug_resolve_phases(uint64_t* host_stamps, int32_t max_units,
                                                int64_t* ticks_per_s);

#ifdef __cplusplus
}
#endif

#endif /* HISPARSE_H */
