/*
 * gms.h -- C ABI of the restore / digest / verify data path of a GPU Memory
 * Service (GMS), written for NVIDIA B200 (sm_100a).
 *
 * Background (paper: "Fast Recovery for LLM Serving via Decoupled Device
 * Memory Lifetime in Dynamo").  Section 3.2 moves model state into device
 * allocations owned by a per-GPU service so that it outlives an engine:
 * a writer populates the allocations and commits them, later engines attach
 * read-only.  Section 4 (GMS paragraph) adds that the writer notes where each
 * tensor lies before it commits and that, when the service comes up cold, a
 * fresh writer fills the model state in again while the process is restored.
 * Section 3.1 models the cost of that as S / B_eff, and Section 5.2 observes
 * that the checkpoint tool in use moves device memory piece by piece, far
 * below what the link could carry.
 * Section 2.2 allows reuse of surviving allocations only if their contents are
 * intact.  The paper leaves the bulk data path and the integrity check
 * unspecified; this library is that path:
 *
 *   gms_manifest_build   the recorded tensor layout, turned into a work list
 *   gms_restore          scatter a packed snapshot image into the allocations,
 *                        digesting every 4 KiB block in the same pass
 *   gms_digest           digest surviving allocations in place (no writes)
 *   gms_verify           compare digests with the ones recorded at commit and
 *                        name the blocks that differ
 *   gms_kv_restore       scatter a subset of paged KV blocks (Section 6,
 *                        "Preserving KV state") through a block-index list
 *
 * The digest (fixed by this library, not by the paper; all arithmetic on
 * uint64_t, wrapping):
 *   mix(z):  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9;
 *            z = (z ^ (z >> 27)) * 0x94D049BB133111EB;  return z ^ (z >> 31);
 *   block digest  D   = XOR_{i<512} mix(w_i ^ i*G), G = 0x9E3779B97F4A7C15,
 *            w_i the little-endian u64 words of the block, a block shorter
 *            than 4096 bytes being extended with zero bytes;
 *   tensor digest T   = XOR_{b<nb} mix(D_b ^ b*G), blocks cut relative to the
 *            tensor's first byte, nb = ceil(nbytes / 4096); nbytes = 0: T = 0.
 * Results are exact integers; every output of this library is bit-reproducible.
 *
 * Conventions.
 *  - Every function returns int: GMS_OK (0) or a negative GMS_ERR_* value.
 *    Nothing throws, aborts or traps.  Host-detectable errors are returned
 *    before any device work is enqueued.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *    stream).  Device work is asynchronous with respect to the host; outputs
 *    are valid once the stream has been synchronised.
 *  - Pointers are marked (device), (host) or (device-accessible).  The caller
 *    owns every buffer it passes and keeps it alive until the stream work has
 *    completed.  The library allocates only the manifest's own small tables
 *    (by default 32 bytes per 16 KiB of payload -- 31 MB for a 16 GB manifest --
 *    plus 8 bytes per 4 KiB block once digests have been recorded, and a second
 *    copy of the 32-byte records, sorted by source offset, once gms_restore_fd
 *    or gms_restore_staged has been used on the manifest).
 *  - Calls that use the same manifest must not overlap on the GPU (they share
 *    the manifest's work counter and status word); enqueue them on one stream
 *    or order them with events.
 */
#ifndef GMS_H
#define GMS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GMS_BLOCK_BYTES 4096u

/* status codes */
#define GMS_OK 0
#define GMS_ERR_NULL (-1)     /* a required pointer is NULL                                   */
#define GMS_ERR_ALIGN (-2)    /* src_offset or dst not 16-byte aligned; bad block_bytes       */
#define GMS_ERR_RANGE (-3)    /* src_offset + nbytes exceeds the image, or overflows          */
#define GMS_ERR_OVERLAP (-4)  /* two destination ranges intersect                             */
#define GMS_ERR_DUP_ID (-5)   /* two entries carry the same tensor_id                         */
#define GMS_ERR_NOMEM (-6)    /* host or device allocation of the manifest's tables failed    */
#define GMS_ERR_CUDA (-7)     /* a CUDA runtime call failed; text via gms_last_cuda_error()   */
#define GMS_ERR_KIND (-8)     /* image_kind is not one of GMS_SRC_*                           */
#define GMS_ERR_TIMEOUT (-9)  /* a bounded device-side wait gave up (see device status word)  */
#define GMS_ERR_STATE (-10)   /* manifest has no device tables / no recorded digests          */
#define GMS_ERR_ARG (-11)     /* an argument is out of its documented range                   */
#define GMS_ERR_TOO_LARGE (-12) /* more digest blocks than gms_verify_flat_noalloc has room for */
#define GMS_ERR_IO (-13)      /* a file read failed or the file is shorter than the image     */

/* where the packed snapshot image lives */
#define GMS_SRC_DEVICE 0u      /* device memory (a staging buffer in HBM)                     */
#define GMS_SRC_HOST_MAPPED 1u /* pinned host memory mapped into the device address space     */

/* gms_manifest_build flags */
#define GMS_BUILD_HOST_ONLY 1u /* validate and build the work list on the host only (no CUDA
                                  call is made; device entry points return GMS_ERR_STATE)     */
#define GMS_BUILD_SELFTEST_STALL 2u /* self-test of the bounded waits, for test suites only: in every
                                  gms_restore / gms_capture / gms_digest of this manifest the barrier of
                                  the first block of chunk 0 is told to expect 16 bytes that are never
                                  sent, so the warp that claims it gives up after its wait limit (2 s),
                                  sets GMS_DEV_TIMEOUT, waits at most one more limit (2 s in all, not
                                  per copy) for the copies it still has in flight, and returns: the call
                                  ends by itself about 4 s after it began; the other warps finish their
                                  work.  Nothing faults; outputs of that call are incomplete by design. */

/* bits of the device status word */
#define GMS_DEV_TIMEOUT 1ull   /* a warp gave up waiting for one of its own bulk copies (2 s), then
                                  spent up to 2 s more draining the rest: worst case 4 s per call  */
#define GMS_DEV_HOLE 2ull      /* gms_kv_evict kept a token whose rows could not be copied: its source or
                                  destination id lies outside the pool; gms_kv_delta, that a state's does  */
#define GMS_DEV_FULL 4ull      /* gms_kv_plan had no free block, table entry, row or room in the ring for something */

typedef struct gms_manifest gms_manifest; /* opaque */

/* One recorded tensor layout (Section 4: what the writing client notes for each tensor before it commits). */
typedef struct {
    uint64_t tensor_id;  /* caller's identifier, unique within a manifest                     */
    uint64_t src_offset; /* byte offset of the tensor in the packed image, 16-byte aligned    */
    void *dst;           /* (device) destination, 16-byte aligned                             */
    uint64_t nbytes;     /* length in bytes, any value >= 0                                   */
} gms_entry;

typedef struct {
    uint64_t tensor_id; /* as given in the entry                                              */
    uint64_t block;     /* 4 KiB block index relative to the tensor's first byte              */
} gms_mismatch;

/*
 * gms_manifest_build -- Section 4, GMS paragraph (layout record made before
 * commit); Section 3.2 (the allocations it describes).
 * Validates `entries` (host, n of them) against an image of `image_bytes`
 * bytes and builds the work list that gms_restore / gms_digest walk: every
 * tensor is cut into chunks of 4 blocks (16 KiB; fewer for manifests too small
 * to give every warp two chunks, never more than 32) so that thousands of small
 * and a few huge tensors are served by one persistent launch.
 * Block digests are laid out in entry order: tensor t owns slots
 * [first_block(t), first_block(t) + ceil(nbytes_t/4096)).
 * The host's part is proportional to the number of tensors (validation, per-tensor
 * positions); the chunk records themselves are written by a kernel on the device,
 * on a stream of the library's own, and the call returns when they are complete
 * (it does not wait for work the caller has queued on other streams).
 * Errors: NULL, ALIGN, RANGE, OVERLAP (destinations; overlapping sources are
 * legal), DUP_ID, NOMEM, CUDA.  nbytes == 0 is legal (no blocks, T = 0).
 * Bytes of a destination beyond nbytes are never written.
 * On success *out owns host and (unless GMS_BUILD_HOST_ONLY) device tables on
 * the current device; release it with gms_manifest_destroy.
 */
int gms_manifest_build(const gms_entry *entries, size_t n, uint64_t image_bytes, uint32_t flags, gms_manifest **out);
int gms_manifest_destroy(gms_manifest *m);

/* Sizes of the outputs: number of entries, of digest blocks, and of payload bytes. */
int gms_manifest_info(const gms_manifest *m, uint64_t *n_tensors, uint64_t *n_blocks, uint64_t *payload_bytes);
/* First digest-block slot of entry `entry_index`. */
int gms_manifest_block_base(const gms_manifest *m, size_t entry_index, uint64_t *first_block);
/* Work-list introspection (host): number of chunks, and chunk `i` as
 * (entry index, byte offset inside the tensor, bytes).  Chunks partition every tensor. */
int gms_manifest_chunk_count(const gms_manifest *m, uint64_t *n_chunks);
int gms_manifest_chunk(const gms_manifest *m, uint64_t i, uint64_t *entry_index, uint64_t *tensor_byte_offset,
                       uint64_t *nbytes);

/*
 * gms_manifest_set_expected -- Section 3.2: commit makes the model state
 * immutable; the digests recorded at that moment are what later reuse is
 * checked against.  Copies n_blocks block digests (device) into the manifest
 * (device-to-device, on `stream`).
 */
int gms_manifest_set_expected(gms_manifest *m, const uint64_t *d_block_digests, void *stream);

/*
 * gms_restore -- Section 4 (cold-service repopulation), Section 3.3
 * (reconstruction after a device-invalidating failure), cost model S/B_eff of
 * Section 3.1.  For every entry: dst[0, nbytes) <- image[src_offset, +nbytes),
 * and, in the same pass over the bytes, D for each block and T for each tensor.
 *   image            (device-accessible) start of the packed image:
 *                    device memory for GMS_SRC_DEVICE, the device-side
 *                    address of pinned mapped host memory for
 *                    GMS_SRC_HOST_MAPPED; 16-byte aligned
 *   d_block_digests  (device) n_blocks u64, may be NULL
 *   d_tensor_digests (device) n u64, may be NULL
 * One persistent kernel (plus a one-block prologue that clears accumulators);
 * no per-tensor launches.  Errors: NULL, ALIGN, KIND, STATE, CUDA.
 */
int gms_restore(const gms_manifest *m, const void *image, uint32_t image_kind, uint64_t *d_block_digests,
                uint64_t *d_tensor_digests, void *stream);

/*
 * gms_capture -- the inverse of gms_restore: Section 3.1, step 3 (device state is staged into a
 * host-side image before it is serialised) and Section 3.2 (what is recorded at commit is what
 * later reuse is checked against).  For every entry: image[src_offset, +nbytes) <- dst[0, nbytes),
 * with D for each block and T for each tensor computed in the same pass -- the digests to hand to
 * gms_manifest_set_expected.  `image` (device-accessible, written) is device memory or the device
 * view of pinned mapped host memory, as `image_kind` says; bytes of the image that no entry covers
 * are left alone.  Image ranges of different entries must not overlap (GMS_ERR_OVERLAP; restore
 * allows shared sources, capture cannot).  Same kernel as gms_restore with the roles of source and
 * destination exchanged.  Errors: NULL, ALIGN, KIND, OVERLAP, STATE, CUDA.
 */
int gms_capture(const gms_manifest *m, void *image, uint32_t image_kind, uint64_t *d_block_digests,
                uint64_t *d_tensor_digests, void *stream);

/*
 * gms_digest -- Section 3.2 (a replacement engine attaches surviving
 * allocations read-only) and Section 2.2 (reuse only if contents are intact).
 * Same outputs as gms_restore, computed over the destinations where they lie;
 * the destinations are only read.
 */
int gms_digest(const gms_manifest *m, uint64_t *d_block_digests, uint64_t *d_tensor_digests, void *stream);

/*
 * gms_verify -- the trust decision of Section 2.2.  Compares
 * d_block_digests[n_blocks] (device) with the digests recorded by
 * gms_manifest_set_expected and writes the differing (tensor_id, block) pairs
 * to d_out (device, `cap` slots) in ascending (entry position, block) order.
 * *d_count (device, u64) receives the total number of differing blocks, which
 * may exceed cap; only min(count, cap) slots of d_out are written.
 * Errors: NULL, STATE (nothing recorded), CUDA.
 */
int gms_verify(const gms_manifest *m, const uint64_t *d_block_digests, gms_mismatch *d_out, uint32_t cap,
               uint64_t *d_count, void *stream);

/*
 * gms_digest_verify / gms_restore_verify -- gms_digest (resp. gms_restore) followed by gms_verify, with the
 * comparison folded into the pass that computes the digests (Section 2.2 and Section 3.2: the intact-state check
 * sits on the critical path of a reattach, so it should cost no pass of its own).  Outputs are exactly those of
 * the two separate calls: block and tensor digests, the ordered mismatch list and the total count.  While a
 * block's digest is still in a register the streaming kernel compares it with the recorded one and counts the
 * difference against the block's 2048-slot segment; what remains of gms_verify is its ordered emit, one small
 * kernel.  d_block_digests is required here (the emit pass reads it back for the segments that differ).
 * Errors: those of gms_digest / gms_restore, and STATE when nothing has been recorded.
 */
int gms_digest_verify(const gms_manifest *m, uint64_t *d_block_digests, uint64_t *d_tensor_digests, gms_mismatch *d_out,
                      uint32_t cap, uint64_t *d_count, void *stream);
int gms_restore_verify(const gms_manifest *m, const void *image, uint32_t image_kind, uint64_t *d_block_digests,
                       uint64_t *d_tensor_digests, gms_mismatch *d_out, uint32_t cap, uint64_t *d_count, void *stream);

/*
 * gms_verify_tensors -- the per-tensor summary of the same trust decision (Section 2.2): which
 * tensors may be reused as they are.  d_tensor_counts (device, n u32, entry order) receives for
 * every entry the number of its blocks whose digest differs from the recorded one (0 = intact).
 * Errors: NULL, STATE (nothing recorded), CUDA.
 */
int gms_verify_tensors(const gms_manifest *m, const uint64_t *d_block_digests, uint32_t *d_tensor_counts, void *stream);

/*
 * gms_verify_flat_noalloc -- the paper has no counterpart; this is a convenience of this library.
 *
 * Who it is for.  Some callers of a memory service cannot allocate device memory at the moment
 * they need the trust decision: a checker that attaches to a GPU whose memory has already been
 * handed out in full (service slabs plus an engine's KV pool leave no room, so cudaMalloc would
 * fail), or a watchdog that must not enter the allocator because an allocation can stall behind,
 * or disturb, the engine that is serving on the same device.  gms_verify needs a manifest, and
 * building one allocates.  This entry point compares two digest arrays the caller already holds
 * and allocates nothing: no cudaMalloc, no cudaFree, no allocating library call.  Its working
 * table (the per-segment counts of the ordered compaction) lives in a fixed array of about
 * 8 KiB inside the library image, present on every GPU that loads the library until the process
 * exits.
 *
 * What it computes.  Exactly what gms_verify reports for a manifest with the single entry
 * (tensor_id, nbytes = n_blocks * 4096): the pairs (tensor_id, b) with
 * d_computed[b] != d_expected[b], ascending in b, into d_out (device, `cap` slots), and the total
 * number of differing blocks into *d_count (device), which may exceed cap.
 *   d_computed, d_expected  (device) n_blocks u64 each
 *   n_blocks                at most GMS_NOALLOC_MAX_BLOCKS (16 GiB of payload); more is refused
 *                           with GMS_ERR_TOO_LARGE before anything is enqueued
 * Rules.  The first call on a device looks up the device address of the fixed array (a one-time
 * set-up with that device current); make that first call before starting any stream capture.
 * That first call is also when the CUDA runtime loads this library's code and the array onto the
 * device, which itself takes device memory: a caller that expects the GPU to fill up should make
 * one warm-up call with n_blocks <= 16384 and one with n_blocks > 16384 (the two sizes run
 * different kernels) while memory is still available; only calls after that are allocation-free.
 * The cached address does not survive a cudaDeviceReset of that device.
 * All calls on a device share the one array, which keeps the previous call's contents (each call
 * rewrites what it uses before use): two calls that overlap on the GPU race, so keep them on one
 * stream or order them with events.  Errors: NULL, TOO_LARGE, ARG, CUDA.
 */
#define GMS_NOALLOC_MAX_BLOCKS 4194304ull
int gms_verify_flat_noalloc(const uint64_t *d_computed, const uint64_t *d_expected, uint64_t n_blocks, uint64_t tensor_id,
                            gms_mismatch *d_out, uint32_t cap, uint64_t *d_count, void *stream);

/* Device status word of the manifest's last call (synchronises `stream`). 0 = clean; if GMS_DEV_TIMEOUT is
 * set the word is still stored and the call returns GMS_ERR_TIMEOUT (that call's outputs are incomplete). */
int gms_last_device_status(const gms_manifest *m, void *stream, uint64_t *word);

/* A paged KV pool: n_planes planes (layer x {K,V}) of n_blocks blocks. */
#define GMS_KV_IMAGE_BY_ID 1u
typedef struct {
    void *base;            /* (device) 16-byte aligned                                        */
    uint64_t plane_stride; /* bytes between planes, multiple of 16                            */
    uint64_t block_stride; /* bytes between blocks of a plane, multiple of 16, >= block_bytes */
    uint32_t n_planes;
    uint32_t n_blocks;
    uint32_t block_bytes;  /* multiple of 4096, at most 131072                                */
    uint32_t flags;        /* 0, or GMS_KV_IMAGE_BY_ID: the image is pool-shaped -- its slot for
                              list position j is slot d_block_ids[j] (a subset copy between two
                              pools of the same shape) instead of slot j (a packed image)        */
} gms_kv_pool;

/*
 * gms_kv_restore -- Section 6, "Preserving KV state": committed KV blocks
 * kept in host memory or storage are put back after recovery.  For j < n_sel
 * and every plane p:
 *   pool[p][d_block_ids[j]] <- image + p*img_plane_stride + j*img_slot_stride
 * (block_bytes bytes each), with digests
 *   d_block_digests[(j*n_planes + p)*k + c]  for 4 KiB block c of that copy,
 *                                            k = block_bytes/4096;
 *   d_kv_digests[j] = XOR_q mix(D_q ^ q*G), q = p*k + c  (the tensor digest of
 *                                            the slot's planes concatenated).
 * An id outside [0, n_blocks) is skipped: nothing is written to the pool, its
 * digests are 0, and d_status[0] counts it.  With more than one plane,
 * plane_stride must be at least (n_blocks-1)*block_stride + block_bytes
 * (planes that share bytes are refused with GMS_ERR_ARG).  That the image
 * extent covers every slot addressed, and that image and pool do not overlap,
 * is the caller's duty: the library cannot see the size of either buffer.  d_status[1] receives the device
 * status word; d_status[2..3] are scratch for the kernel's work counter.  Ids
 * must be distinct (the caller's duty; duplicates race).
 *   image        (device-accessible) as for gms_restore; strides multiples of 16
 *   d_block_ids  (device) int32[n_sel]
 *   d_block_digests (device) n_sel*n_planes*k u64, may be NULL
 *   d_kv_digests (device) n_sel u64, may be NULL
 *   d_status     (device) 4 u64
 * Errors: NULL, ALIGN, KIND, ARG, CUDA.
 */
int gms_kv_restore(const gms_kv_pool *pool, const void *image, uint64_t img_plane_stride, uint64_t img_slot_stride,
                   uint32_t image_kind, const int32_t *d_block_ids, uint32_t n_sel, uint64_t *d_block_digests,
                   uint64_t *d_kv_digests, uint64_t *d_status, void *stream);

/*
 * gms_kv_capture -- the gather direction of the same extension (Section 6: committed KV blocks are
 * kept in host memory or storage).  pool[p][d_block_ids[j]] is copied into slot j of the packed
 * image for every plane p; arguments, digest layout, skipping of out-of-range ids (the slot is left
 * alone) and status words are those of gms_kv_restore, with `image` written instead of read.
 */
int gms_kv_capture(const gms_kv_pool *pool, void *image, uint64_t img_plane_stride, uint64_t img_slot_stride,
                   uint32_t image_kind, const int32_t *d_block_ids, uint32_t n_sel, uint64_t *d_block_digests,
                   uint64_t *d_kv_digests, uint64_t *d_status, void *stream);

/*
 * gms_kv_digest -- the same extension read together with Section 2.2: KV blocks that outlived an
 * engine may be reused only if they are intact.  pool[p][d_block_ids[j]] is digested where it lies,
 * for every plane p; nothing is written to the pool and there is no image.  Digest layout, skipping
 * of out-of-range ids (digests 0, counted in d_status[0]) and status words are those of
 * gms_kv_restore, so the output compares directly with what gms_kv_restore / gms_kv_capture of the
 * same id list reported (gms_kv_verify names the differing blocks, planes and 4 KiB sub-blocks).
 * pool->flags is ignored apart from the range check.  Errors: NULL, ALIGN, ARG, RANGE, CUDA.
 */
int gms_kv_digest(const gms_kv_pool *pool, const int32_t *d_block_ids, uint32_t n_sel, uint64_t *d_block_digests,
                  uint64_t *d_kv_digests, uint64_t *d_status, void *stream);

/*
 * gms_kv_verify -- the trust decision for preserved KV state (Section 6, "Preserving KV state", read with
 * Section 2.2: state that outlived an engine is reused only if it is intact), in the terms a block manager acts
 * on.  d_computed and d_expected (device, n_sel*n_planes*k u64 each, the layout every gms_kv_* call writes:
 * slot (j*n_planes + p)*k + c) are compared -- typically what gms_kv_digest finds now against what
 * gms_kv_restore / gms_kv_capture reported when the blocks were put back or saved -- and every differing slot is
 * written to d_out (device, `cap` records) as
 *   (block_id = d_block_ids[j], plane = p, sub_block = c, list_pos = j)
 * in ascending (j, p, c) order.  *d_count (device, u64) receives the total, which may exceed cap; only
 * min(count, cap) records are written.  A list position whose id lies outside [0, pool->n_blocks) was skipped by
 * the calls that produced the digests and is never reported, whatever its slots hold.  Only n_planes, n_blocks,
 * block_bytes and flags of `pool` are read.
 *   d_scratch  (device) GMS_KV_VERIFY_SCRATCH_WORDS(n_sel*n_planes*k) u32 of working memory owned by the caller
 *              (the KV calls have no manifest to keep it in); contents before and after are meaningless, and
 *              two calls that overlap on the GPU must not share it
 * Errors: NULL, ALIGN, ARG, RANGE, CUDA.
 */
typedef struct {
    uint32_t block_id;  /* pool block, as given in the id list                        */
    uint32_t plane;     /* layer x {K,V} plane                                        */
    uint32_t sub_block; /* 4 KiB block inside the KV block                            */
    uint32_t list_pos;  /* position of the block in the id list                       */
} gms_kv_mismatch;
#define GMS_KV_VERIFY_SCRATCH_WORDS(n_slots) (((uint64_t)(n_slots) + 2047u) / 2048u + 1u)
int gms_kv_verify(const gms_kv_pool *pool, const int32_t *d_block_ids, uint32_t n_sel, const uint64_t *d_computed,
                  const uint64_t *d_expected, gms_kv_mismatch *d_out, uint32_t cap, uint64_t *d_count, uint32_t *d_scratch,
                  void *stream);

/*
 * gms_kv_attention / gms_kv_attention_shared / gms_kv_evict -- what an engine does next with the paged KV state that
 * the calls above put back (Section 6, "Preserving KV state"): attention that reads the pool where it lies, and the
 * choice of the tokens that stay in it.  All asynchronous on `stream`; no allocation, no host synchronisation; can be
 * captured into a CUDA graph.  Integer arrays on the device (lengths, tables) are read by the kernels only.
 *
 * gms_kv_layout: how one layer's tokens lie inside the pool's blocks.  Element (token, kv head, d) of block b is at
 *   base + plane*plane_stride + b*block_stride + token*token_stride + head*head_stride + d*2 bytes,
 * tokens outside heads or heads outside tokens, whichever the strides say.
 */
#define GMS_DTYPE_BF16 0u
#define GMS_DTYPE_F16 1u
typedef struct {
    uint32_t k_plane, v_plane;            /* planes of the layer's keys and values                       */
    uint32_t n_kv_heads;                  /* >= 1                                                        */
    uint32_t head_dim;                    /* 64 or 128                                                   */
    uint32_t block_tokens;                /* tokens in a block: a power of two, 16 .. 1024               */
    uint32_t dtype;                       /* GMS_DTYPE_* of pool, queries and outputs                    */
    uint32_t token_stride, head_stride;   /* bytes, multiples of 16; rows must not overlap and must end
                                             inside block_bytes                                          */
} gms_kv_layout;

/*
 * One batch of queries over cached tokens.  Sequence s has kv_lens[s] tokens in the pool, token t in slot
 * t % block_tokens of block block_table[s*table_stride + t / block_tokens]; its queries are the rows
 * cu_q[s] .. cu_q[s+1]-1 of `q`, and they belong to the LAST of those tokens (the tokens' own keys and values are
 * already in the pool).  A query at position p sees token t if t <= p and, when window > 0, t > p - window or
 * t < sinks; an id outside [0, pool->n_blocks) is a hole whose tokens nobody sees.  With c = h / (n_heads/n_kv_heads):
 *   x_t = scale * q[i,h] . K[t,c];  lse[i,h] = log sum_t exp(x_t);  out[i,h] = sum_t exp(x_t - lse) V[t,c]
 * over the t that it sees; if there are none, out is 0 and lse is -infinity.  What a query does not see cannot reach
 * its output, whatever bits it holds (NaN, infinities); a value that it sees and that is not finite makes its output non-
 * finite in that column (infinite or NaN).  Products are taken in the pool's type with 32-bit sums; the softmax weights are
 * rounded to the pool's type before the product with V (fp16: so that they count down to 2^-32 of the largest), not in lse.
 * The host sizes the launch by max_q and max_kv.  Of a sequence with more queries the first max_q are processed, of one
 * with more tokens only the first max_kv are seen (and have weights); what is left out changes no position: query i of
 * q_len stands at kv_lens[s] - q_len + i all the same.  Rows of q that are not processed or that no sequence owns leave
 * out and lse as they are.  Neither may overlap anything that is read.
 */
typedef struct {
    const void *q;                 /* (device) [total_q][n_heads][head_dim], 16-byte aligned             */
    void *out;                     /* (device) the same shape                                            */
    float *lse;                    /* (device) [total_q][n_heads], may be NULL                           */
    const int32_t *cu_q;           /* (device) n_seq + 1 ascending offsets; NULL: one query a sequence   */
    const int32_t *kv_lens;        /* (device) n_seq                                                     */
    const int32_t *block_table;    /* (device) n_seq rows of table_stride ids                            */
    void *workspace;               /* (device) gms_kv_attention*_workspace bytes, 256-byte aligned; contents
                                      before and after are meaningless; calls that overlap on the GPU must not
                                      share it                                                           */
    uint64_t *status;              /* (device) may be NULL; GMS_DEV_TIMEOUT is or-ed in if a bounded wait
                                      inside a kernel ran out (outputs are then incomplete)              */
    uint64_t workspace_bytes;
    uint64_t q_token_stride, q_head_stride;     /* bytes, multiples of 16                                */
    uint64_t out_token_stride, out_head_stride; /* bytes, multiples of 16                                */
    uint64_t table_stride;         /* entries; table_stride * block_tokens >= max_kv                     */
    uint32_t n_seq, n_heads;       /* n_heads: a multiple of n_kv_heads                                  */
    uint32_t total_q, max_q;       /* rows of q; longest query run of a sequence                         */
    uint32_t max_kv;               /* longest kv_lens (at most 2^30)                                     */
    uint32_t window, sinks;        /* window 0: every token up to the query's own is seen                */
    float scale;
} gms_kv_attn;

/*
 * Accumulated attention weights, the quantity that gms_kv_evict goes by.  For t < kv_lens[s]
 *   out[s][c][t] = decay * in[s][c][t] + sum over the call's queries i of s and the heads h of c of exp(x_t - lse[i,h])
 * (0 for tokens a query does not see); other entries of `out` are left alone.  `in` may equal `out`.  Sums are taken in
 * a fixed order: equal calls give equal bits.
 */
typedef struct {
    const float *in;                    /* (device) NULL: zeros                                          */
    float *out;                         /* (device)                                                      */
    uint64_t seq_stride, head_stride;   /* elements, of both                                             */
    float decay;
    uint32_t reserved;                  /* 0                                                             */
} gms_kv_weight;

/*
 * gms_kv_attention_workspace: bytes for this call and for every later one with no larger n_seq, total_q, max_q and max_kv
 * and the same pool layout, n_heads, window, sinks and outputs (lse given where it was not, and no weights where there were,
 * take less).
 * With weights and few queries a KV head the logits are kept: 4 bytes for each query, head and cached token that the
 * sequence's queries see (of max_kv, or of window + sinks and up to 62 more).
 * Errors: NULL, ALIGN, ARG, RANGE (index limits; table_stride; workspace_bytes too small), CUDA.
 */
int gms_kv_attention_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                               const gms_kv_weight *weight, uint64_t *nbytes);
int gms_kv_attention(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                     const gms_kv_weight *weight /* may be NULL */, void *stream);

/*
 * gms_kv_attention_shared -- the same for a batch in which whole groups of sequences begin with the same tokens (a
 * system prompt, a document).  Sequences group_start[g] .. group_start[g+1]-1 share the prefix of prefix_lens[g] tokens
 * that lies in the blocks prefix_table[g*prefix_stride + ...]; block_table and kv_lens describe what each sequence has
 * after it.  Every query sees the whole prefix, then its own sequence's tokens up to its own.  The prefix is read once
 * for all rows of the group, not once a sequence.  attn->window and attn->sinks must be 0.
 * group_start[0] = 0 and group_start[n_groups] = n_seq: a sequence outside every group gets the tokens of its own
 * alone.  Rows of a group beyond its first max_group_q are not processed, tokens of a prefix beyond max_prefix not seen.
 * The workspace's size holds for smaller n_groups, max_prefix and max_group_q too.  Errors: as gms_kv_attention.
 */
typedef struct {
    const int32_t *group_start;   /* (device) n_groups + 1, ascending                                    */
    const int32_t *prefix_lens;   /* (device) n_groups                                                   */
    const int32_t *prefix_table;  /* (device) n_groups rows of prefix_stride ids                         */
    uint64_t prefix_stride;       /* entries; prefix_stride * block_tokens >= max_prefix                 */
    uint32_t n_groups;
    uint32_t max_prefix;          /* longest prefix_lens (at most 2^30)                                  */
    uint32_t max_group_q;         /* most query rows in a group                                          */
    uint32_t reserved;            /* 0                                                                   */
} gms_kv_prefix;
int gms_kv_attention_shared_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                                      const gms_kv_prefix *prefix, uint64_t *nbytes);
int gms_kv_attention_shared(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                            const gms_kv_prefix *prefix, void *stream);

/*
 * gms_kv_evict -- shrinks the cache of n_seq sequences to at most `budget` tokens a sequence, for n_layers layers at
 * once (layer l: planes k_plane + l*layer_planes and v_plane + l*layer_planes).  Of n = lens[s] tokens, n' = min(n, budget)
 * stay; each layer and KV head chooses its own: the first `sinks`, the last `recent`, and of those between the
 * n' - sinks - recent with the largest weights (equal weights: the earlier token; NaN counts below every number).
 * When n <= budget all stay.  The kept tokens keep their order:
 *   kept[l][s][c][j]         position of the j-th kept token, j < n' (-1 for n' <= j < budget)
 *   weights_out[l][s][c][j]  its weight (entries from n' on are left alone)
 *   lens_out[s] = n'; lens_out may be lens (then the lengths are updated in place), but may not overlap it otherwise
 *   K and V of token kept[j] are copied to token j of the blocks dst_table[s*dst_stride + ...]
 * Destination blocks must be distinct and must not be source blocks (the old ones are free once the call has run).  The
 * tables must not have holes where tokens can be kept: the choice goes by weights and positions alone, and a row whose source
 * or destination id lies outside the pool is not copied, so that its place among the n' tokens holds whatever bits were there
 * before, for gms_kv_attention to see.  GMS_DEV_HOLE in `status` tells of it.  Keys carry their positions (rotary embeddings)
 * with them; afterwards the sequence is n' tokens long for gms_kv_attention.  Lens above max_len count as max_len.
 * Errors: NULL, ALIGN, ARG (sinks + recent > budget; planes outside the pool; weights_out or lens_out where
 * they may not be), RANGE, CUDA.
 */
typedef struct {
    const float *weights;               /* (device) w_*_stride elements between layers, sequences, heads */
    float *weights_out;                 /* (device) may be NULL; o_*_stride; must not overlap `weights`   */
    const int32_t *lens;                /* (device) n_seq                                                */
    int32_t *lens_out;                  /* (device) n_seq, may be NULL, may be lens                      */
    const int32_t *src_table, *dst_table;
    int32_t *kept;                      /* (device) [n_layers][n_seq][n_kv_heads][budget]                */
    uint64_t w_layer_stride, w_seq_stride, w_head_stride;
    uint64_t o_layer_stride, o_seq_stride, o_head_stride;
    uint64_t src_stride, dst_stride;    /* entries; * block_tokens >= max_len and >= min(max_len, budget) */
    uint32_t n_layers, layer_planes, n_seq, max_len;
    uint32_t budget, sinks, recent;
    uint32_t reserved;                  /* 0                                                             */
    uint64_t *status;                   /* (device) may be NULL; GMS_DEV_HOLE is or-ed in                */
} gms_kv_evict_args;
int gms_kv_evict(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_evict_args *args, void *stream);

/*
 * gms_kv_plan / gms_kv_append / gms_kv_delta -- the rest of an engine's step on the state that the calls above put back:
 * which blocks and slots the step's tokens go to, putting their keys and values there, and layers whose state is recurrent.
 * All asynchronous on `stream`; no allocation, no host synchronisation; can be captured into a CUDA graph and replayed on the
 * step after (counters and lengths are on the device and may be updated in place).
 *
 * gms_kv_plan -- block tables and slot maps from request lengths.  With B = block_tokens, for every sequence s
 *   base = max(lens - drop_lens, 0);  lens_out = base + rows;  had = ceil(lens / B);  need = ceil(lens_out / B)
 * where rows = new_lens[s], cut off where the sum over the sequences so far would pass total_rows.  drop_lens takes tokens
 * off a sequence's end first (speculated tokens that were rejected; all of them: the request has left, and its row is free for
 * another).  Free blocks are kept in a ring: free_state[0] is the position of the next one in free_ids[free_cap],
 * free_state[1] how many there are.
 *   need > had: entries had .. need-1 of the row get the next blocks of the ring, sequences in ascending order
 *   need < had: the blocks in entries need .. had-1 go to the ring's end, sequences and entries in ascending order; ids outside
 *               [0, n_blocks) (holes) do not; the entries keep what they hold.  Blocks that come back in a call are free
 *               from the next call on
 *   cu_q[0] = 0, cu_q[s+1] = cu_q[s] + rows: offsets of the sequences' rows
 *   for row cu_q[s] + i:  positions = base + i;  slots = id * B + positions % B with id = the row's entry positions / B
 *   rows from cu_q[n_seq] on (a batch padded to a fixed size): slots = -1, positions = 0
 * A token that has no block (the ring is empty: its entry gets -1; a position beyond table_blocks * B; a hole in the table) has
 * slot -1; lens_out counts it all the same, for gms_kv_attention a token in a hole.  GMS_DEV_FULL in `status` tells of an empty
 * ring, of a full table row, of rows cut off at total_rows and of blocks that a ring without room for them lost.  Lengths below 0
 * count as 0, above 2^30 as 2^30.  Everything is exact and the same in every run.
 * Neither table rows nor the ring may hold a block twice; free_cap >= n_blocks is always enough.  Outputs may not overlap inputs,
 * but lens_out may be lens and free_state_out may be free_state.
 * Errors: NULL, ALIGN, ARG, RANGE, CUDA.
 */
typedef struct {
    const int32_t *lens;           /* (device) n_seq: tokens that are cached                             */
    const int32_t *new_lens;       /* (device) n_seq: tokens to come                                     */
    const int32_t *drop_lens;      /* (device) n_seq: tokens taken off the end first; NULL: none         */
    int32_t *lens_out;             /* (device) n_seq, may be lens                                        */
    int32_t *block_table;          /* (device) n_seq rows, table_stride entries apart                    */
    int32_t *free_ids;             /* (device) free_cap                                                  */
    const int32_t *free_state;     /* (device) 2: position of the next free block, number of free blocks */
    int32_t *free_state_out;       /* (device) 2, may be free_state                                      */
    int32_t *cu_q;                 /* (device) n_seq + 1                                                 */
    int64_t *slots;                /* (device) total_rows                                                */
    int32_t *positions;            /* (device) total_rows, may be NULL                                   */
    uint64_t *status;              /* (device) may be NULL; GMS_DEV_FULL is or-ed in                     */
    uint64_t table_stride;         /* entries                                                            */
    uint32_t n_seq, total_rows;    /* total_rows < 2^31                                                  */
    uint32_t table_blocks;         /* entries of a row that may be used, at most table_stride and 2^20   */
    uint32_t free_cap;             /* < 2^31                                                             */
    uint32_t n_blocks;             /* of the pool, 1 .. 2^31 - 1                                         */
    uint32_t block_tokens;         /* a power of two, 16 .. 1024                                         */
} gms_kv_plan_args;
int gms_kv_plan(const gms_kv_plan_args *args, void *stream);

/*
 * gms_kv_append -- what stands between a layer's projections and gms_kv_attention, in one pass: queries and keys normed head by
 * head, both rotated to their positions, queries to q_out, keys and values into the pool's blocks.  For a row x of q or k
 * (head_dim elements, products and sums in 32 bits, one rounding at the end):
 *   norm (q_weight / k_weight given):  x[d] <- x[d] / sqrt(mean x^2 + eps) * (weight[d] + weight_offset)
 *   rotation: pair j < rotary_dim / 2 is elements (j, j + rotary_dim / 2) (GMS_PAIR_HALVES) or (2j, 2j + 1)
 *     (GMS_PAIR_NEIGHBOURS); with angle = positions[axes[j]][i] * inv_freq[j] (in 64 bits), c = rope_scale * cos, s = rope_scale * sin:
 *     (a, b) <- (a c - b s, b c + a s);  elements from rotary_dim on stay.
 * Several axes (time, height, width of a picture's patches): positions has n_axes rows, and axes[j] says which of them pair j
 * turns with (entries >= n_axes count as the last one; NULL: all with row 0).  Values are copied.
 * Row i's keys and values go to slot slots[i] = block * block_tokens + token; a slot outside the pool (-1: padding, a token
 * without a block) is skipped, the row's queries are written all the same.  Rows from *n_rows on are left alone altogether.
 * Slots must be distinct (the caller's duty; duplicates race).  q_out may be q (same strides), else outputs may not overlap inputs.
 * q may be NULL (n_heads 0: keys and values only), and so may k and v (both: queries only).
 * Errors: NULL, ALIGN, ARG, RANGE, CUDA.
 */
#define GMS_DTYPE_F32 2u
#define GMS_PAIR_HALVES 0u
#define GMS_PAIR_NEIGHBOURS 1u
typedef struct {
    const void *q, *k, *v;         /* (device) [rows][heads][head_dim], the layout's dtype, 16-byte aligned */
    void *q_out;                   /* (device) [rows][n_heads][head_dim]                                 */
    const int64_t *slots;          /* (device) rows                                                      */
    const int32_t *positions;      /* (device) n_axes rows of positions_stride; NULL if rotary_dim is 0  */
    const int32_t *n_rows;         /* (device) may be NULL: rows that are there (cu_q + n_seq of a plan)  */
    const float *inv_freq;         /* (device) rotary_dim / 2                                            */
    const uint8_t *axes;           /* (device) rotary_dim / 2, may be NULL                               */
    const void *q_weight, *k_weight; /* (device) head_dim of weight_dtype, each may be NULL (no norm); 16-byte aligned */
    uint64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
        out_token_stride, out_head_stride; /* bytes, multiples of 16                                     */
    uint64_t positions_stride;     /* entries, >= rows                                                   */
    uint32_t rows, n_heads;        /* rows < 2^31                                                        */
    uint32_t rotary_dim;           /* multiple of 8, at most head_dim; 0: no rotation                    */
    uint32_t n_axes, pairs;        /* 1 .. 8; GMS_PAIR_*                                                 */
    uint32_t weight_dtype;         /* GMS_DTYPE_*                                                        */
    float weight_offset, eps, rope_scale;
    uint32_t reserved;             /* 0                                                                  */
} gms_kv_append_args;
int gms_kv_append(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_append_args *args, void *stream);

/*
 * gms_kv_delta -- the gated delta rule, the recurrent layers' counterpart of attention.  A head's state is a head_dim x head_dim
 * matrix S of 32-bit numbers, [key][value], that lives in the pool, so that capture, restore, digest and verify keep it like any
 * other block: head h of a sequence is in block table[h / per], at byte (h % per) * 4 * head_dim^2 of its plane, where
 * per = block_bytes / (4 * head_dim^2) heads fit into a block.  For each of a sequence's rows in turn, with c = h / (n_heads / n_key_heads):
 *   S <- exp(g[i,h]) S;   d = beta[i,h] (v[i,h] - S^T k[i,c]);   S <- S + k[i,c] d^T;   out[i,h] = scale S^T q[i,c]
 * (unit_qk: q and k are first divided by sqrt(sum x^2 + unit_eps)).  S begins as the state in src_table, or as zeros where
 * past_lens[s] is 0, and the state after the last row goes to dst_table (a sequence without rows: as it began).  g NULL counts as
 * zeros, beta NULL as ones.  g is a logarithm, at most 0 in earnest; -infinity clears the state.
 * Sequences of more than 20 rows are done in chunks of 64 on tensor cores: products of the 16-bit inputs with S, d and decays, which
 * enter as sums of two 16-bit terms (2^-16 relative); for `out` the state before the chunk enters as one (its error is 1.1 to 1.3 times
 * that of its last rounding).  States and sums are kept in 32 bits.  What a row does not depend on cannot reach it, whatever bits it
 * holds.  Chunks in which something is not finite or near the end of the range (differences from 2^64 on; fp16: states from 2^25 on,
 * differences from 2^41 on, keys whose lengths are 2^18 apart) are done row by row: right, and slower.  (fp16: what is left of a state
 * below 2^-80 has fewer bits.)
 * src_table and dst_table may be the same (states are updated in place), and rows of src_table may be equal (several sequences go on
 * from one state).  Destination blocks must be distinct, and none may be a source block of another sequence or stand at another place of
 * its own sequence's source row (heads are done in no order: a state that is still to be read would be overwritten).  An id outside
 * [0, n_blocks) reads as zeros and is not written; GMS_DEV_HOLE in `status` tells of it.  Rows that no sequence owns, and rows of a sequence
 * beyond its first max_q, are not processed and leave `out` as it is.
 * gms_kv_delta_workspace: bytes for this call and every later one with no larger n_seq, total_q and max_q and the same heads.
 * Errors: NULL, ALIGN, ARG, RANGE, CUDA.
 */
typedef struct {
    uint32_t plane;                /* of the pool                                                        */
    uint32_t n_heads;              /* value heads, >= 1                                                  */
    uint32_t head_dim;             /* 64 or 128                                                          */
    uint32_t reserved;             /* 0                                                                  */
} gms_kv_state;
typedef struct {
    const void *q, *k, *v;         /* (device) [total_q][n_key_heads or n_heads][head_dim], 16-byte aligned */
    void *out;                     /* (device) [total_q][n_heads][head_dim]                              */
    const float *g, *beta;         /* (device) [total_q][n_heads], rows *_stride elements apart          */
    const int32_t *cu_q;           /* (device) n_seq + 1 ascending offsets; NULL: one row a sequence     */
    const int32_t *past_lens;      /* (device) n_seq; NULL: every state is read                          */
    const int32_t *src_table, *dst_table; /* (device) n_seq rows of ids, *_stride entries apart          */
    void *workspace;               /* (device) 256-byte aligned; calls that overlap must not share it    */
    uint64_t *status;              /* (device) may be NULL                                               */
    uint64_t workspace_bytes;
    uint64_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
        out_token_stride, out_head_stride; /* bytes, multiples of 16                                     */
    uint64_t g_stride, beta_stride, src_stride, dst_stride;
    uint32_t n_seq, n_key_heads;   /* n_heads is a multiple of n_key_heads                               */
    uint32_t total_q, max_q;       /* rows; longest run of a sequence                                    */
    uint32_t dtype;                /* GMS_DTYPE_BF16 or GMS_DTYPE_F16, of q, k, v and out                */
    uint32_t unit_qk;              /* 0 or 1                                                             */
    float unit_eps, scale;
} gms_kv_delta_args;
int gms_kv_delta_workspace(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, uint64_t *nbytes);
int gms_kv_delta(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, void *stream);

/*
 * Pinned, device-mapped host memory for a GMS_SRC_HOST_MAPPED image (the
 * host-resident snapshot of Section 3.1 step 3 / Section 6).  *device_view is
 * the address to pass as `image`.
 */
int gms_host_image_alloc(uint64_t nbytes, void **host_ptr, void **device_view);
int gms_host_image_free(void *host_ptr);

/*
 * gms_pipe_* / gms_restore_fd -- Section 4, GMS paragraph: with a cold service, a fresh writer
 * fills the model state in from storage while the process is being restored; Section 3.1 prices it
 * at S / B_eff.  The image is read from a file descriptor, never resident as a whole: a ring of
 * `n_buffers` pinned buffers of `buffer_bytes` each (>= 1 MiB, multiple of 4096) is filled by
 * `n_readers` threads with pread(), with a read-ahead hint for the window after (and, after
 * gms_pipe_direct_io(p, 1), bypassing the page cache with O_DIRECT where the file system allows it:
 * right for a cold snapshot on fast storage, wrong for a file the page cache already holds, so it is
 * off unless asked for), and each filled buffer is moved by the
 * copy engine into one of two device buffers of the same size (allocated by gms_pipe_create) and
 * scattered + digested from there by the restore kernel while the next one is read.  If the device
 * buffers cannot be allocated the pipe still works: the kernel then reads the pinned buffers across
 * the host link itself, which reaches about 93 % of what the copy engine does.
 * The first gms_restore_fd (or gms_restore_staged) on a manifest writes a copy of its work list sorted by
 * source offset (on the device, like the other lists) and plans the windows; that call allocates device
 * memory and synchronises, so it must not be made while a stream capture is in progress.  Later calls
 * with the same buffer size reuse the plan.
 * gms_restore_fd is synchronous: on return the stream has been synchronised and the outputs hold
 * exactly what gms_restore would have produced from the same bytes (image byte k = file byte
 * file_offset + k).  One restore at a time per pipe.  Errors: NULL, ARG (bad sizes; a chunk larger
 * than a buffer), NOMEM, STATE, IO (read error or file shorter than the image), CUDA.
 */
typedef struct gms_pipe gms_pipe; /* opaque */
typedef struct {
    uint64_t windows;          /* buffers' worth of image consumed                          */
    uint64_t bytes_read;       /* bytes read from the file                                  */
    double wait_read_seconds;  /* host time spent waiting for readers (storage-bound share) */
    double wait_gpu_seconds;   /* host time spent waiting for a buffer to be released       */
    double total_seconds;      /* wall time of the call                                     */
    uint32_t direct_io;        /* 1: the file system accepted O_DIRECT reads                */
    uint32_t copy_engine;      /* 1: windows went pinned buffer -> copy engine -> device    */
    uint32_t mapped_io;        /* 1: gms_capture_fd stored through a mapping of the file    */
    uint32_t reserved;
} gms_pipe_stats;
int gms_pipe_create(uint32_t n_buffers, uint64_t buffer_bytes, uint32_t n_readers, gms_pipe **out);
int gms_pipe_direct_io(gms_pipe *p, int enable);
int gms_pipe_mapped_writes(gms_pipe *p, int enable);
int gms_pipe_destroy(gms_pipe *p);
int gms_restore_fd(const gms_manifest *m, gms_pipe *p, int fd, uint64_t file_offset, uint64_t *d_block_digests,
                   uint64_t *d_tensor_digests, void *stream, gms_pipe_stats *stats);

/*
 * gms_capture_fd -- the way back through the same pipe: Section 3.1, steps 3 and 4 (device state is staged
 * into host memory and serialised to durable storage).  gms_capture, window by window: the kernel gathers
 * each window of the image straight into one of the pipe's pinned buffers (kernel-issued stores cross the
 * link at the copy engine's rate in this direction, so the device buffers are not used) and the pipe's
 * threads write it out with pwrite() while the next window is gathered.  File byte file_offset + k = image
 * byte k for every byte a tensor covers; bytes of the file between tensors' ranges are not written, and the
 * file is neither truncated nor synced (the caller's fsync decides when it is durable).  Digests as from
 * gms_capture.  `fd` must be open for writing; gms_pipe_direct_io does not apply.  Synchronous like
 * gms_restore_fd; in `stats`, bytes_read counts the bytes written and wait_read_seconds the time spent
 * waiting for the writers.  Errors: NULL, ARG, OVERLAP (tensors share image bytes), NOMEM, STATE, IO
 * (write error), CUDA.
 * gms_pipe_mapped_writes(p, 1): the writers store through a shared mapping of the file instead of calling
 * pwrite().  The kernel lets only one buffered write at a time into a file, so pwrite from many threads
 * runs at one core's copy rate; stores into a mapping run on all of them.  Meant for snapshots kept in
 * the page cache or on tmpfs.  Used only when `fd` is a regular file, open for reading and writing, that
 * already spans file_offset + the image (it is never extended), else pwrite is used as before
 * (stats.mapped_io says which).  The caller must have the file's blocks in that range allocated
 * (written before, or posix_fallocate): a store into a hole of a full file system raises SIGBUS, where
 * pwrite would have returned an error.  Off unless asked for.
 */
int gms_capture_fd(const gms_manifest *m, gms_pipe *p, int fd, uint64_t file_offset, uint64_t *d_block_digests,
                   uint64_t *d_tensor_digests, void *stream, gms_pipe_stats *stats);

/*
 * gms_stage_* / gms_restore_staged -- host-sourced restore with the copy engine on the link
 * (Section 5.2: the existing tool stays far below the PCIe rate; Section 3.1: S / B_eff).  Kernel-issued
 * reads of mapped host memory (gms_restore with GMS_SRC_HOST_MAPPED) top out below what the DMA
 * engine reaches on the same link.  Here the pinned host image is moved window by window with
 * cudaMemcpyAsync on an internal stream into a ring of `n_buffers` device buffers of `buffer_bytes`
 * each (>= 1 MiB, multiple of 4096), and every landed window is scattered and digested by the
 * restore kernel on the caller's stream while the next one is in flight; all ordering is done with
 * stream events, no kernel waits for a flag.  Asynchronous like gms_restore (after the first call on a
 * manifest, which uploads the sorted work list as described above): outputs are valid once
 * `stream` has been synchronised; the host image must stay untouched until then.  Results are
 * exactly those of gms_restore from the same bytes.  `host_image` (host) must be pinned memory.
 * Errors: NULL, ARG, KIND (not pinned host memory), NOMEM, STATE, CUDA.
 */
typedef struct gms_stage gms_stage; /* opaque */
int gms_stage_create(uint32_t n_buffers, uint64_t buffer_bytes, gms_stage **out);
int gms_stage_destroy(gms_stage *st);
int gms_restore_staged(const gms_manifest *m, gms_stage *st, const void *host_image, uint64_t *d_block_digests,
                       uint64_t *d_tensor_digests, void *stream);

/*
 * gms_service_* -- the substrate under the destinations: Section 4, GMS paragraph (physical
 * allocations made with cuMemCreate, a first-fit suballocator over 2 GiB slabs with dedicated
 * slabs for larger allocations, permissions set per slab) and Section 3.2 (ownership protocol:
 * EMPTY -> RW, one writer populates -> COMMITTED, immutable -> RO while n >= 1 readers hold it;
 * a writer that gives up before commit discards everything; write access returns after the last
 * reader has left; read-only is enforced with cuMemSetAccess).  Current device.  The state machine
 * lives in the process that created the service; other processes take part through the export / import
 * calls further down.
 *   create      slab_bytes = 0 means 2 GiB; GMS_SERVICE_DRY_RUN keeps the books without any CUDA
 *               call (addresses are made up and must not be dereferenced)
 *   acquire_rw  EMPTY -> RW, or COMMITTED -> RW (contents and addresses kept, slabs writable again);
 *               GMS_ERR_STATE while a writer or readers hold the service
 *   alloc       RW only; 256-byte aligned device address, first fit over the slabs, a dedicated slab
 *               if nbytes exceeds the slab size; individual allocations are never freed, only all
 *               at once (abort / destroy)
 *   commit      RW -> COMMITTED: the device is synchronised, then every slab becomes read-only
 *   abort       RW -> EMPTY: every slab is unmapped and released
 *   acquire_ro / release_ro   COMMITTED <-> RO with a reader count
 * After commit the addresses may be read by anything (gms_digest, gms_capture, an engine's
 * kernels); writing to them faults the writing context, so gms_restore / gms_kv_restore must only
 * target them in state RW (gms_service_access tells which it is).  Errors: NULL, ARG, STATE, NOMEM,
 * RANGE (access: not an address of this service), CUDA.
 */
#define GMS_STATE_EMPTY 0u
#define GMS_STATE_RW 1u
#define GMS_STATE_COMMITTED 2u
#define GMS_STATE_RO 3u
#define GMS_SERVICE_DRY_RUN 1u
#define GMS_SERVICE_SHAREABLE 2u /* slabs can be handed to other processes (gms_service_export_fd) */
typedef struct gms_service gms_service; /* opaque */
typedef struct {
    uint32_t state, readers;
    uint64_t n_slabs, n_dedicated; /* slabs in all, and those holding one oversized allocation */
    uint64_t slab_bytes;           /* regular slab size after rounding to the mapping granularity */
    uint64_t bytes_reserved;       /* sum of slab sizes                                           */
    uint64_t bytes_allocated;      /* sum of (256-byte rounded) allocation sizes                  */
    uint32_t attached;             /* 0 between gms_service_detach and gms_service_reattach        */
    uint32_t backed;               /* 0 between gms_service_release_pages and gms_service_back_pages */
} gms_service_stats;
int gms_service_create(uint64_t slab_bytes, uint32_t flags, gms_service **out);
int gms_service_destroy(gms_service *s);
int gms_service_acquire_rw(gms_service *s);
int gms_service_alloc(gms_service *s, uint64_t nbytes, void **dptr);
int gms_service_commit(gms_service *s);
int gms_service_abort(gms_service *s);
int gms_service_acquire_ro(gms_service *s);
int gms_service_release_ro(gms_service *s);
int gms_service_info(gms_service *s, gms_service_stats *out);
int gms_service_access(gms_service *s, const void *dptr, uint32_t *writable);

/*
 * Addresses that outlive their mappings.  A snapshot of an engine holds the virtual addresses of its
 * tensors (in CUDA graphs and tensor metadata) but none of the memory behind them, so both calls
 * below keep every virtual range reserved: the destination pointers of a manifest built before
 * stay valid afterwards.
 *   detach / reattach           Section 3.3: before capture the engine unmaps each service range but
 *       keeps its address reservation while the service keeps the physical memory; after restore the
 *       surviving memory is mapped read-only at the same addresses.  COMMITTED (no readers) only.
 *       Between the two calls nothing may touch the addresses (gms_service_access returns
 *       GMS_ERR_STATE) and acquire_rw / acquire_ro are refused.  Contents are preserved.
 *   release_pages / back_pages  Section 3.1 (pages released before capture, fresh pages mapped at the
 *       same addresses after restore) and Section 3.3 (after a device-invalidating failure the state
 *       is rebuilt in fresh allocations): RW only.  The physical memory of every slab is given back
 *       to the driver; back_pages maps fresh memory, writable, whose contents are undefined until the
 *       writer restores them (gms_restore, gms_kv_restore).  In between, alloc / commit are refused.
 * Both pairs synchronise the device first.  Errors: NULL, STATE, NOMEM (back_pages; the service then
 * stays without pages), CUDA.
 */
int gms_service_detach(gms_service *s);
int gms_service_reattach(gms_service *s);
int gms_service_release_pages(gms_service *s);
int gms_service_back_pages(gms_service *s);

/*
 * Across processes -- Section 4, GMS paragraph (the service process creates the physical allocations and
 * keeps their handles; clients receive them as file descriptors over Unix sockets, import them, map them and
 * set their own access) and Section 3.2 (the memory therefore outlives the engine process that filled or used
 * it, and the replacement engine attaches it read-only).  The library provides the two ends; the socket and
 * whatever is said on it (who holds the service in which state) belong to the processes that use them.
 *   gms_service_slab       size and address of slab `index` (0 .. n_slabs-1 of gms_service_info) in the service's
 *                          own address space, so that allocation addresses can be written as (slab, offset)
 *   gms_service_export_fd  a new file descriptor for slab `index` (service created with GMS_SERVICE_SHAREABLE;
 *                          GMS_ERR_STATE otherwise, in a dry run, or without pages); the caller sends it with
 *                          SCM_RIGHTS and closes its copy.  The memory lives as long as any process holds a
 *                          handle or a mapping of it.
 *   gms_import_create      the client's side, on the same GPU (the current device): imports the n descriptors
 *                          (which stay open; the caller closes them), reserves address space for each -- at
 *                          slabs[i].address where that is free -- maps it and sets this process's access:
 *                          read-only, or writable with GMS_IMPORT_WRITABLE (the writer that populates, RW in the
 *                          protocol).  GMS_IMPORT_SAME_ADDRESS: fail with GMS_ERR_RANGE unless every slab lands
 *                          at the service's address (an engine restored from a snapshot has those addresses in its
 *                          graphs and metadata, and kept the ranges free; a fresh process will often find them
 *                          taken); without it any address will do and gms_import_address tells which.  Permissions are per process: a reader's mapping stays read-only whatever the
 *                          others hold.
 *   gms_import_destroy     synchronises the device, unmaps, frees the address ranges and drops the handles; the
 *                          contents stay with the service.
 * Errors: NULL, ARG, RANGE, STATE, NOMEM, CUDA.
 */
#define GMS_IMPORT_WRITABLE 1u
#define GMS_IMPORT_SAME_ADDRESS 2u
typedef struct {
    uint64_t address, bytes;
    uint32_t dedicated, reserved;
} gms_slab_info;
typedef struct gms_import gms_import; /* opaque */
int gms_service_slab(gms_service *s, uint64_t index, gms_slab_info *out);
int gms_service_export_fd(gms_service *s, uint64_t index, int *fd);
int gms_import_create(const int *fds, const gms_slab_info *slabs, size_t n, uint32_t flags, gms_import **out);
int gms_import_address(const gms_import *imp, size_t index, void **dptr);
int gms_import_destroy(gms_import *imp);

/*
 * Tuning and test hooks.  The library reads the environment variables below once per process (the chunk lengths
 * once per gms_manifest_build), and ONLY if GMS_TUNING_HOOKS=1 is set as well; without that switch none of them has
 * any effect, so a stray variable in a serving process cannot change launch shapes or chunking.  Every setting
 * gives bit-identical results (the test suite runs the parity checks under several of them); the defaults are what
 * the published timings were taken with.
 *   GMS_GEOM_RESTORE / GMS_GEOM_DIGEST / GMS_GEOM_KV   "warps,slots,CTAs-per-SM" of the restore/capture kernel, the
 *       digest-only kernels and the KV copy kernels (defaults 9,4,1 / 16,3,1 / 8,6,1; warps 1..16, slots 3|4|6|8)
 *   GMS_CLAIM_RESTORE / GMS_CLAIM_DIGEST               "counters,chunks-per-claim" of the work-list claims
 *       (defaults 1,1 / 2,1; counters 1..32, chunks 1..64)
 *   GMS_CHUNK_BLOCKS / GMS_CHUNK_BLOCKS_DIGEST         4 KiB blocks per chunk of the copy list and of the digest
 *       list (defaults 4 / 8, fewer for small manifests; 1..32)
 *   GMS_L2_KEEP                                        0 / 1: never / always give the digest-only kernels their L2
 *       hints (payload loads evict-first, digest stores evict-last); by default they are used for payloads from
 *       256 MiB on whose digests take at most 16 MiB
 *   GMS_CHECK_TABLES                                   1: gms_manifest_build reads the work lists it wrote on the
 *       device back and compares them with a host construction of the same lists (GMS_ERR_STATE if they differ)
 */

/* Launch geometry of the streaming kernels on the current device (for reporting). */
int gms_launch_geometry(uint32_t *grid_ctas, uint32_t *warps_per_cta, uint32_t *smem_bytes);
/* Number of kernels this library has launched in this process so far (for reporting). */
uint64_t gms_kernel_launches(void);
/*
 * Makes `device` current for the calling thread's later gms_* calls.  The library links its own
 * copy of the CUDA runtime; a process that drives several GPUs (one service per GPU, Section 4)
 * selects the device here as well as in whatever else it uses.
 */
int gms_set_device(int device);

const char *gms_strerror(int status);
const char *gms_last_cuda_error(void); /* text of the last failed CUDA call on this thread */
uint32_t gms_version(void);

#ifdef __cplusplus
}
#endif
#endif /* GMS_H */
