/*
 * datastates.h -- C ABI of the MI355X snapshot hot path (libdatastates_hip.so).
 *
 * One GPU's part of the lazy, non-blocking checkpoint snapshot of
 * DataStates-LLM (arXiv 2601.16956): the fragmented, mixed-precision, possibly
 * strided model/optimizer shards of one rank are coalesced into one contiguous
 * image laid out like the checkpoint file (Sec. V-A1 "coalescing", Sec. V-A5
 * rule (1): offsets fixed in advance), the image is streamed to a pre-pinned,
 * reused host ring (Sec. V-A1; the circular host cache of Sec. V-B/V-C) in chunks that
 * need not be whole tensors (Sec. V-A4), while training continues; the
 * mutating update phase is gated on the capture (Sec. V-A2).  Restore is the
 * inverse scatter.
 *
 * Conventions
 *   - Plain C.  No HIP or torch types: a stream is passed as `void*` holding a
 *     hipStream_t (NULL = the null stream).  "dev" pointers are device
 *     addresses valid on the device that was current when the plan / engine
 *     was created; "host" pointers are ordinary host addresses.
 *   - Every function returns an int: DS_OK (0), a positive status
 *     (DS_NOT_READY, DS_EOF) or a negative error.  Nothing throws or aborts.
 *     Out-parameters are written only on DS_OK (or the documented status).
 *   - A plan is immutable once created and may be used from several threads.
 *     Requests on one engine (create / destroy, ds_snapshot_async,
 *     ds_restore_*) are serialised by the caller; the calls on an event may
 *     come from other threads than the request -- the gate from the training
 *     thread, ds_snapshot_next_chunk from ONE consumer thread, and
 *     ds_snapshot_release_chunk from any number of threads (a flush does
 *     exactly that).
 *   - The image.  For shard i:  bytes_i = itemsize(dtype_i) * prod(shape_i)
 *     (empty product = 1).  Image byte  file_offset_i + r*itemsize + b  is byte
 *     b of the element of rank r in the row-major (last index fastest)
 *     enumeration of the VIEW, which lives at
 *     base_i + itemsize * sum_j k_j * strides_i[j].  Bytes as they are: no
 *     dtype conversion, no byte swap (Sec. IV-D, Sec. V-A3: tensors are
 *     byte-addressable buffers that need no serialisation).  Every image byte
 *     that belongs to no shard is 0x00.  The image length is the end of the
 *     last shard rounded up to the alignment.
 */
#ifndef DATASTATES_H
#define DATASTATES_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DS_MAX_DIMS 6

/* element types; only the size matters to the byte mover: 4, 2, 2, 8, 1 */
typedef enum ds_dtype { DS_F32 = 0, DS_BF16 = 1, DS_F16 = 2, DS_I64 = 3, DS_U8 = 4 } ds_dtype;

/* status and error codes */
#define DS_OK 0
#define DS_NOT_READY 1 /* ds_event_query: snapshot still in flight               */
#define DS_EOF 2       /* ds_snapshot_next_chunk: every chunk has been handed out */
#define DS_EINVAL (-1)   /* null pointer, bad dtype/ndim/shape/stride/alignment value, misaligned base */
#define DS_EALIGN (-2)   /* a file_offset is not a multiple of the alignment      */
#define DS_EOVERLAP (-3) /* two shards intersect in the image, or a view addresses an element twice */
#define DS_EGAP (-4)     /* DS_PLAN_STRICT: a hole that is not alignment padding  */
#define DS_ERANGE (-5)   /* image range outside [0,total], reversed, or not a multiple of 16 */
#define DS_ENOMEM (-6)   /* host or device allocation failed                      */
#define DS_EHIP (-7)     /* a HIP call failed; see ds_last_hip_error()            */
#define DS_EBUSY (-8)    /* object still has work in flight / chunk not released  */
#define DS_ESTATE (-9)   /* call not valid in this state (e.g. release of a chunk never handed out) */
#define DS_EIO (-10)     /* a file operation failed; see ds_last_errno()           */
#define DS_EFORMAT (-11) /* not a checkpoint file of this format, or a damaged one   */
#define DS_EFAULT (-12)  /* DS_PLAN_CHECK_MEMORY: a shard is not inside one device allocation */
#define DS_ETOOBIG (-13) /* ds_pack_noalloc: the plan's tables do not fit the static table memory */

/*
 * One shard: a view into device memory plus its place in the file.
 * (Sec. IV-C: a rank owns many separate shards, cut where the parallel
 * execution plan and the optimizer sharding put the cuts, not where a
 * checkpoint layout would.)
 */
typedef struct ds_shard_desc {
  const void *base;               /* DEVICE address of element (0,...,0); multiple of the itemsize */
  uint32_t dtype;                 /* ds_dtype                                                     */
  uint32_t ndim;                  /* 0..DS_MAX_DIMS; 0 = exactly one element                      */
  int64_t shape[DS_MAX_DIMS];     /* extents >= 0 (a zero extent = empty shard, 0 bytes)          */
  int64_t strides[DS_MAX_DIMS];   /* in ELEMENTS, > 0 for every extent > 1; the view must not
                                     address any element twice (DS_EOVERLAP).  Checked exactly:
                                     by the nesting of the strides where they nest (any slice,
                                     transpose or permutation of a dense parent does), else by
                                     writing out the addresses, which is done for views of up
                                     to 2^20 elements; a larger view with strides that do not
                                     nest is refused                                              */
  uint64_t tensor_id;             /* logical tensor this shard is a slice of; kept in the plan's
                                     manifest, never touches the bytes                            */
  uint64_t file_offset;           /* byte offset of the shard in the image; multiple of `align`   */
} ds_shard_desc;

typedef struct ds_plan ds_plan;
typedef struct ds_engine ds_engine;
typedef struct ds_event ds_event;
typedef struct ds_flush ds_flush;
typedef struct ds_ckpt ds_ckpt;               /* a checkpoint file being written */
typedef struct ds_ckpt_reader ds_ckpt_reader; /* a checkpoint file opened for recovery */

/* ---- layout and plan (Sec. V-A3 composite provider, duty (a): sizes and
 *      offsets in the stream; Sec. V-A5 rule (1)) ---------------------------- */

/* Size of one element in bytes, 0 for an unknown dtype. */
int ds_itemsize(uint32_t dtype);

/*
 * Canonical layout: writes file_offset of desc[0..n) in table order, each at
 * the next multiple of `align` after the end of the one before; *total = image
 * length (a multiple of `align`).  Host-only, touches no device.
 * `align` must be a power of two >= 16.  Errors: DS_EINVAL.
 */
int ds_layout_assign(ds_shard_desc *desc, size_t n, uint64_t align, uint64_t *total);

#define DS_PLAN_STRICT 1u    /* reject holes larger than alignment padding (DS_EGAP)           */
#define DS_PLAN_HOST_ONLY 2u /* validate and build tables on the host only; such a plan can be
                                inspected but not passed to ds_pack/ds_unpack/ds_snapshot_async */
#define DS_PLAN_CHECK_MEMORY 4u /* ask the runtime, for every non-empty shard, which allocation its
                                base address lies in, and require every address of the view to be
                                inside it (DS_EFAULT otherwise): a wrong descriptor is then an error
                                here, not a memory fault in a kernel later.  Costs one runtime call
                                per shard; not with DS_PLAN_HOST_ONLY */

/*
 * Validates the table (any order of offsets; shards must be disjoint in the
 * image), normalises every view (merges dimensions that are contiguous with
 * each other, splits off the innermost contiguous run), cuts the image into
 * work-group chunks and uploads the tables to the current device.  The
 * descriptors are copied: the caller may free `desc` afterwards.  The tensors
 * themselves stay owned by the caller and must stay allocated while the plan
 * is used.  The plan is reused by every snapshot of the same shard set (Sec.
 * V-A1: what is set up once serves all later checkpoint requests).
 * Errors: DS_EINVAL, DS_EALIGN, DS_EOVERLAP, DS_EGAP, DS_EFAULT, DS_ENOMEM, DS_EHIP.
 */
int ds_plan_create(const ds_shard_desc *desc, size_t n, uint64_t align, uint32_t flags, ds_plan **out);

/*
 * One plan for a rank that writes its checkpoint as several files (Sec. VI-D:
 * 20 files for a 7B rank; Sec. V-A3: one composite provider per rank lays out
 * everything it owns).  file_of[i] < n_files names the file of shard i and
 * desc[i].file_offset counts from the start of THAT file.  The plan's one image
 * is the files' tensor regions one behind the other in file order: region f
 * spans the shards of file f from offset 0 up to the end of the last one,
 * rounded up to `align`, and starts at the sum of the regions before it (see
 * ds_plan_file).  One gather launch and one snapshot then cover all files, and
 * the file tier cuts the image at the region boundaries (ds_flush_start_files,
 * ds_ckpt_flush_snapshot_parts).  A file that no shard names has an empty
 * region.  file_of == NULL with n_files == 1 is ds_plan_create.  Everything else
 * (checks, flags, errors, ownership) as ds_plan_create; DS_PLAN_STRICT also
 * requires every file's first shard at offset 0.  n_files <= DS_MAX_FILES.
 */
#define DS_MAX_FILES 65536u
int ds_plan_create_files(const ds_shard_desc *desc, const uint32_t *file_of, size_t n, uint32_t n_files,
                         uint64_t align, uint32_t flags, ds_plan **out);

/* ds_layout_assign file by file: the canonical offset of every shard inside its own
 * file; region_bytes[n_files] (may be NULL) gets the files' tensor-region lengths,
 * *total their sum = the length of the image of ds_plan_create_files.
 * Errors: DS_EINVAL. */
int ds_layout_assign_files(ds_shard_desc *desc, const uint32_t *file_of, size_t n, uint32_t n_files,
                           uint64_t align, uint64_t *region_bytes, uint64_t *total);

/* Frees host and device tables.  The caller makes sure no kernel that uses
 * the plan is still running (synchronise the streams it was used on). */
int ds_plan_destroy(ds_plan *plan);

typedef struct ds_plan_stats {
  uint64_t total_bytes;   /* image length T                                       */
  uint64_t payload_bytes; /* sum of bytes_i; T - payload = padding                */
  uint64_t n_shards;      /* descriptors given                                    */
  uint64_t n_tiles;       /* non-empty shards (+1 if the image starts with a hole)*/
  uint64_t n_chunks;      /* work-group chunks over the whole image               */
  uint64_t chunk_bytes;   /* image bytes per work-group chunk                     */
  uint64_t n_strided;     /* shards that are not one contiguous run               */
  uint64_t align;
  uint64_t n_general_chunks; /* chunks the lean path does not take (the general path does, or the block route
                                of views with runs shorter than 16 bytes) */
  uint64_t n_files;       /* 1 for a plan of ds_plan_create                       */
} ds_plan_stats;

int ds_plan_info(const ds_plan *plan, ds_plan_stats *out);

/* Manifest entry i (table order as given): what a file header would record
 * (Sec. V-A5 rule (3)).  Any out pointer may be NULL. */
int ds_plan_shard(const ds_plan *plan, size_t i, uint64_t *tensor_id, uint32_t *dtype,
                  uint64_t *file_offset, uint64_t *nbytes);

/* File f of the plan: where its tensor region starts in the image and how long
 * it is.  Either out pointer may be NULL.  Errors: DS_EINVAL (f >= n_files). */
int ds_plan_file(const ds_plan *plan, uint32_t f, uint64_t *image_begin, uint64_t *region_bytes);

/* Manifest entry i: the file it belongs to and its offset in the IMAGE
 * (= the file_offset of ds_plan_shard + the file's image_begin). */
int ds_plan_shard_file(const ds_plan *plan, size_t i, uint32_t *file, uint64_t *image_offset);

/* Shape of manifest entry i: *ndim and the first *ndim extents of shape[DS_MAX_DIMS]
 * (the rest are set to 0).  Either out pointer may be NULL. */
int ds_plan_shard_shape(const ds_plan *plan, size_t i, uint32_t *ndim, int64_t *shape);

/* ---- the kernels (gather = Sec. V-A1 coalescing done on the device; scatter
 *      = recovery, Sec. V-A5 rule (3)) -------------------------------------- */

/*
 * Gather: writes image bytes [img_lo, img_hi) to dst_dev[0 .. img_hi-img_lo),
 * i.e. dst_dev points at where image byte img_lo goes (a staging slot, or the
 * start of a full-size buffer with img_lo = 0).  Padding bytes are written as
 * zero, so the destination need not be cleared.  img_lo <= img_hi <= total,
 * both multiples of 16; dst_dev 16-byte aligned.  Asynchronous: enqueued on
 * `stream`; the tensors must not change until it has run.  The device the
 * plan was created on must be the calling thread's current device (DS_ESTATE).
 * Errors: DS_EINVAL, DS_ERANGE, DS_ESTATE, DS_EHIP.
 */
int ds_pack(const ds_plan *plan, void *dst_dev, uint64_t img_lo, uint64_t img_hi, void *stream);

/*
 * Scatter, the exact inverse: every addressed element of every shard whose
 * image bytes lie in [img_lo, img_hi) is overwritten with src_dev[offset -
 * img_lo ...]; elements are written whole only if all their bytes are in the
 * range (ranges are multiples of 16 and itemsizes divide 16, so an element is
 * never cut).  No other byte of the tensors' memory is written.
 */
int ds_unpack(const ds_plan *plan, const void *src_dev, uint64_t img_lo, uint64_t img_hi, void *stream);

/*
 * ds_pack for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same result
 * as ds_pack, byte for byte; the difference is where the kernel finds the
 * plan's tables.  ds_pack reads them from the device allocation ds_plan_create
 * made; this call copies them (on `stream`, ahead of the kernel) into a static
 * device array of DS_PACK_NOALLOC_TABLE_BYTES that the library holds on every
 * GPU it runs on until the process ends (plans of up to 64 contiguous shards at
 * multiples of 16 bytes hand it to the kernel in its arguments instead, and use
 * no array), and calls neither hipMalloc nor
 * hipFree nor anything else that allocates.  `plan` may therefore be a
 * DS_PLAN_HOST_ONLY plan, whose creation touches no device either.
 * Limit: the tables (168 bytes per non-empty shard, 36 bytes per work-group
 * chunk of the image, i.e. about 2.3 KiB per MiB of image) must fit the array:
 * an image of about 1.7 GB with few shards does, DS_ETOOBIG otherwise
 * (returned before anything is enqueued).  Views with runs shorter than
 * 16 bytes are moved in blocks if the tables of those (176 bytes per such view,
 * 8 per block, up to 36 per other chunk) fit behind the rest, unit by unit if not.
 * All calls on one GPU share the one array and it keeps the last call's tables:
 * calls on the same stream are ordered by it, calls that may overlap on one GPU
 * (different streams, or different threads) race and are the caller's to
 * serialise.  Arguments and
 * the other errors as for ds_pack; the current device is the one that runs it.
 */
#define DS_PACK_NOALLOC_TABLE_BYTES (4u << 20)
int ds_pack_noalloc(const ds_plan *plan, void *dst_dev, uint64_t img_lo, uint64_t img_hi, void *stream);

/* ---- the snapshot engine (Sec. V-A1 pre-pinned reused pool, Sec. V-A2 lazy
 *      capture, Sec. V-A4 chunked streaming, Sec. V-C dedicated streams) ----- */

#define DS_ENGINE_AUTO_RELEASE 1u /* no consumer: a ring slot is reusable as soon as its copy is done */
#define DS_ENGINE_TRACE 2u        /* time every device-to-host copy of a snapshot (two events per chunk), for
                                     ds_event_trace */

typedef struct ds_engine_opts {
  uint64_t host_ring_bytes;  /* pinned host ring capacity, allocated and pinned once; the paper's
                                single tunable (Sec. V-B).  0 = 2 GiB                              */
  uint64_t d2h_chunk_bytes;  /* size of one ring slot = one device-to-host copy; multiple of 4096.
                                0 = 128 MiB (on one copy stream the gap between two copies costs
                                4 % of the link at 32 MiB, 1 % at 128 MiB)                          */
  uint64_t stage_slot_bytes; /* image bytes per gather launch (the last launch of an image may be
                                shorter); multiple of d2h_chunk_bytes.  0 = 1 GiB                   */
  uint32_t stage_slots;      /* device staging is one ring of stage_slots * stage_slot_bytes bytes
                                (>= 1; 0 = 2): a launch takes the next piece of it, of its own length,
                                so queued snapshots of small images share it.  With staging as large
                                as everything requested at a time, every gate opens after the gathers
                                alone, whatever the link, the host ring or the storage are doing    */
  uint32_t pack_grid_limit;  /* max work-groups resident per gather launch; 0 = one per chunk       */
  uint32_t flags;            /* DS_ENGINE_*                                                         */
  uint32_t copy_streams;     /* copy streams the chunks alternate over: 1 or 2.  0 = 1.  With 2 the gap
                                between two copies on one stream is hidden by the other stream's copy
                                (+2 % at 32 MiB chunks) -- when the two copies share the link evenly;
                                measured, they do in the first engine of a process and share it 2:1 in
                                later ones (-17 %), so one stream with large chunks is the default     */
  uint64_t first_launch_bytes; /* image bytes of the first gather launch of a snapshot; multiple of
                                d2h_chunk_bytes, <= stage_slot_bytes.  A short first launch lets the
                                first copy start earlier; the gather of the rest then runs beside that
                                copy.  0 = stage_slot_bytes (no short first launch)                  */
} ds_engine_opts;

/* Allocates the pinned ring, the device staging, a gather stream and the copy streams
 * (all at the default priority) and a host thread that issues the work.
 * Uses the current device.  The pinned ring and the device staging of a
 * destroyed engine are kept (one allocation each per process, the largest seen)
 * and handed to the next engine that fits into them: pinning is slow, a fresh
 * allocation is slow on first touch, and the first pinned allocation of a
 * process was measured to be the one the link writes fastest; the engine's
 * streams are reused likewise.  ds_config_set("drop_pinned_cache", 1) frees the
 * memory.
 * Errors: DS_EINVAL, DS_ENOMEM, DS_EHIP. */
int ds_engine_create(const ds_engine_opts *opts, ds_engine **out);

/* Waits for all snapshots in flight, then frees everything.  Events created
 * from the engine must have been destroyed.  Errors: DS_EBUSY, DS_EHIP. */
int ds_engine_destroy(ds_engine *engine);

/*
 * Checkpoint request (Sec. V-A2): records the point of consistency on
 * `compute_stream` and returns at once; gather launches and device-to-host
 * copies are issued by the engine's thread on its own streams and overlap
 * with whatever the caller enqueues next.  Between this call and the gate
 * (ds_event_wait_on_stream / ds_event_wait_captured) the caller must not
 * enqueue work that writes the tensors.  Snapshots on one engine run in the
 * order requested.  *out is owned by the caller (ds_event_destroy).
 * DS_EBUSY while a restore event of the engine is alive.
 */
int ds_snapshot_async(ds_engine *engine, const ds_plan *plan, void *compute_stream, ds_event **out);

/*
 * The lazy gate (Sec. V-A2: the update phase is delayed only if the copies
 * have not finished): makes `stream` wait until every source byte has been
 * read into staging.  Returns when the wait has been enqueued; blocks the
 * host only while the engine has not yet issued the last gather (e.g. the
 * host ring is full and the consumer is behind: the paper's back-pressure).
 * Hence, when staging is smaller than the images requested and not yet
 * copied out, the thread that calls the gate must not be the one that
 * consumes the chunks: it would wait for room that only it can make.
 */
int ds_event_wait_on_stream(ds_event *ev, void *stream);

/* Host-side form of the gate: returns when every source byte has been read. */
int ds_event_wait_captured(ds_event *ev);

/* DS_OK when the whole image has reached the host ring, else DS_NOT_READY. */
int ds_event_query(ds_event *ev);

/* Blocks the host until the whole image has reached the host ring (with a
 * consumer: until the last chunk's copy is done, which needs ring slots). */
int ds_event_wait(ds_event *ev);

/*
 * Consumer side (Sec. V-A3: the stream is exposed chunk by chunk, each an
 * address and a length): blocks until the next chunk of the image is resident in the ring,
 * then returns its host address, its offset in the image (which is the offset in
 * the file for a plan of one file; ds_plan_file maps it for a plan of several)
 * and its length.  Chunks come in image order.  DS_EOF after the last.  The memory stays valid
 * until ds_snapshot_release_chunk.  Not used with DS_ENGINE_AUTO_RELEASE.
 */
int ds_snapshot_next_chunk(ds_event *ev, const void **host_ptr, uint64_t *file_off, uint64_t *len);

/* Gives the ring slot back (Sec. V-A2: eviction after flush lets the next
 * request proceed).  Errors: DS_ESTATE if host_ptr is not a chunk handed out. */
int ds_snapshot_release_chunk(ds_event *ev, const void *host_ptr);

typedef struct ds_snapshot_stats {
  uint64_t image_bytes;
  uint64_t payload_bytes;
  uint32_t n_pack_launches;
  uint32_t n_copies;
  double pack_ms;       /* sum of gather kernel durations (HIP events on the gather stream)   */
  double copy_ms;       /* sum of device-to-host copy durations (HIP events on the copy stream) */
  double capture_ms;    /* request -> last source byte read                                   */
  double total_ms;      /* request -> last byte in the host ring                              */
  double submit_host_ms;/* host time spent inside ds_snapshot_async                           */
} ds_snapshot_stats;

/* Valid after ds_event_wait returned DS_OK. */
int ds_event_stats(ds_event *ev, ds_snapshot_stats *out);

/* One step of a snapshot on the device's clock, in milliseconds since the request
 * (what Sec. VI-D's timeline of tensors across the tiers shows, for this pipeline). */
typedef struct ds_trace_rec {
  uint32_t kind;      /* 0 = gather launch, 1 = device-to-host copy of one chunk */
  uint32_t index;     /* launch number / chunk number                           */
  uint64_t file_off;  /* image range the step covers                            */
  uint64_t len;
  double begin_ms;
  double end_ms;
} ds_trace_rec;

/*
 * Writes the records of a finished snapshot to out[0 .. cap): the gather
 * launches, then -- on an engine with DS_ENGINE_TRACE -- the copies in chunk
 * order.  *n = number of records there are (call with cap = 0 to ask).
 * Errors: DS_EBUSY (not finished), DS_ESTATE (a restore event), DS_EHIP.
 */
int ds_event_trace(ds_event *ev, ds_trace_rec *out, size_t cap, size_t *n);

/* Waits for the snapshot, releases chunks still held, frees the event. */
int ds_event_destroy(ds_event *ev);

/* ---- restore from a host image (recovery, Sec. V-A5 rule (3); the mirror image
 *      of the snapshot pipeline: pinned ring -> device staging -> scatter) ------ */

/*
 * Starts a restore of the whole image of `plan` through the engine's ring and
 * staging.  The engine must be idle: no snapshot or restore event of it may be
 * alive (DS_EBUSY).  Scatters are ordered after everything enqueued so far on
 * `compute_stream`.  The caller then repeats, in file order:
 *   ds_restore_next_slot  -> a ring slot to fill with image bytes
 *                            [file_off, file_off+len) (e.g. read from the file)
 *   ds_restore_submit     -> the slot is copied to the device; every eight chunks
 *                            (or stage_slot_bytes, if that is less) are scattered
 *                            into the tensors while the next ones are copied
 * and finally ds_event_wait (host) or ds_event_wait_on_stream (a stream that is
 * to use the restored tensors), then ds_event_destroy.
 */
int ds_restore_begin(ds_engine *engine, const ds_plan *plan, void *compute_stream, ds_event **out);

/*
 * Next ring slot, in file order.  Blocks the host only while the copy that last
 * used the slot is still in flight.  Several slots may be held at once (to read
 * ahead); DS_EBUSY if all of them are with the caller; DS_EOF after the last.
 */
int ds_restore_next_slot(ds_event *ev, void **host_ptr, uint64_t *file_off, uint64_t *len);

/* The slot has been filled.  Slots are submitted in the order they were handed
 * out (DS_ESTATE otherwise).  Returns as soon as the work is enqueued. */
int ds_restore_submit(ds_event *ev, const void *host_ptr);

/* ---- host <-> file tier (Sec. V-A4: a chunk goes on to the next tier as soon
 *      as it is resident; Sec. V-C: persistence on background threads) -------- */

#define DS_FILE_DIRECT 1u /* O_DIRECT for every transfer whose offset and length are multiples of 4 KiB
                             (ring slots are): straight from / into the ring where the kernel can pin the
                             ring's pages, else through an aligned buffer of ordinary memory (one extra
                             memory-speed copy, no page cache); anything else, and everything on a file
                             system without direct I/O, goes through a buffered descriptor */
#define DS_FILE_URING 4u  /* writes of a flush go through the kernel's io_uring interface: one thread keeps up
                             to `threads` writes in flight (Sec. V-C); where the process may not have an
                             io_uring (ds_config_get("io_uring_available") = 0) the pwrite threads are used */
#define DS_FILE_SYNC 2u   /* fsync before ds_flush_wait returns                                        */

/*
 * Starts the consumer of a snapshot taken on an engine WITHOUT
 * DS_ENGINE_AUTO_RELEASE: one thread takes the chunks as they land in the ring,
 * `threads` writer threads (0 = 4, at most 64) write each at its file offset
 * into `path` (created / truncated) and give the ring slot back.  Returns at
 * once.  The caller must not call ds_snapshot_next_chunk on `ev` itself.
 * Errors: DS_EINVAL, DS_ENOMEM, DS_EIO.
 */
int ds_flush_start(ds_event *ev, const char *path, uint32_t threads, uint32_t flags, ds_flush **out);

/*
 * The same for a snapshot of a plan of several files (ds_plan_create_files):
 * paths[f] gets the bytes of region f at file offsets 0.., so that file f is
 * exactly what ds_flush_start would write for a plan of file f's shards alone.
 * One set of `threads` writers serves all files; a ring chunk that spans a
 * region boundary is written in pieces and its slot is given back when the
 * last piece is out.  n_files must be the plan's.  Errors: as ds_flush_start.
 */
int ds_flush_start_files(ds_event *ev, const char *const *paths, uint32_t n_files, uint32_t threads,
                         uint32_t flags, ds_flush **out);

/* Waits until the whole image is in the file, closes it and frees the flush.
 * Either out pointer may be NULL.  Errors: DS_EIO (ds_last_errno()), or the
 * error that ended the snapshot. */
int ds_flush_wait(ds_flush *flush, uint64_t *bytes_written, double *seconds);

/*
 * Restore from a file written by a flush: reads the image with `threads`
 * reader threads into ring slots and feeds the restore pipeline
 * (ds_restore_begin / next_slot / submit) in file order.  Returns when the last
 * chunk has been submitted; *out is then waited for and destroyed like any
 * restore event.  The engine must be idle.  Errors: as ds_restore_begin, DS_EIO.
 */
int ds_restore_from_file(ds_engine *engine, const ds_plan *plan, const char *path, uint32_t threads,
                         uint32_t flags, void *compute_stream, ds_event **out);

/* The same out of the n_files files of a plan of several files, paths[f]
 * holding region f from its offset 0: ONE restore event, one scatter pipeline
 * for the whole rank.  n_files must be the plan's.  Errors: as above. */
int ds_restore_from_files(ds_engine *engine, const ds_plan *plan, const char *const *paths, uint32_t n_files,
                          uint32_t threads, uint32_t flags, void *compute_stream, ds_event **out);

/* errno of the file operation that last produced DS_EIO on this thread. */
int ds_last_errno(void);

/* ---- the checkpoint file (Sec. V-A5: tensors at offsets fixed in advance,
 *      serialized objects appended behind them as a concurrent log, a metadata
 *      header at the END of the file that describes both) ---------------------
 *
 * Layout, all integers little-endian:
 *   [0, T)            the tensor region: the image of the plan, byte for byte
 *   [T, E)            the object log.  A chunk of len bytes claims the next
 *                     round_up(len, 8) bytes; bytes never written read as 0
 *   [E, E+80n+32m)    the trailer: n tensor entries, then m chunk entries
 *       tensor entry (80 B): u64 tensor_id, u32 dtype, u32 ndim, u64 shape[6]
 *                     (unused extents 0), u64 file_offset, u64 nbytes; plan order
 *       chunk entry (32 B): u64 object_id, u64 seq, u64 file_offset, u64 len;
 *                     sorted by (object_id, seq); an object is the concatenation
 *                     of its chunks seq = 0, 1, ...
 *   last 64 B         the footer: char magic[8] = "DSCKPT01", u32 version = 1,
 *                     u32 flags = 0, u64 align, u64 T, u64 E, u64 n, u64 m,
 *                     u32 crc of the trailer, u32 crc of the 60 footer bytes before
 *                     it (CRC-32 of IEEE 802.3, as in zlib)
 * The paper fixes the three rules, not the bytes: the encoding is this library's.
 * A rank that writes several files per checkpoint uses either one plan and one
 * ds_ckpt per file, or ONE plan of several files (ds_plan_create_files) with one
 * ds_ckpt per file made by ds_ckpt_create_part: file f then holds region f of
 * the image as its tensor region, the plan's entries of file f (offsets inside
 * the file) as its tensor entries and an object log of its own -- byte for byte
 * the file that a plan of file f's shards alone would give.
 */

/*
 * Creates / truncates `path` for a checkpoint of `plan` (which may be a
 * DS_PLAN_HOST_ONLY plan when the tensor region comes from host memory).
 * flags: DS_FILE_DIRECT / DS_FILE_SYNC / DS_FILE_URING as for a flush.  The plan must outlive
 * the ds_ckpt.  Errors: DS_EINVAL, DS_ENOMEM, DS_EIO.
 */
int ds_ckpt_create(const char *path, const ds_plan *plan, uint32_t flags, ds_ckpt **out);

/* The writer of file `file` of a plan of several files (for a plan of one file,
 * ds_ckpt_create_part(path, plan, 0, ...) is ds_ckpt_create, which refuses a plan
 * of several).  Errors: as ds_ckpt_create. */
int ds_ckpt_create_part(const char *path, const ds_plan *plan, uint32_t file, uint32_t flags, ds_ckpt **out);

/* Fills the tensor regions of ALL files of a plan of several files from one
 * snapshot of that plan: parts[f] must be the writer of file f, n_parts the
 * plan's number of files; one flush with `threads` writers serves them all.
 * Flags are those of parts[0].  Each part is then finished on its own with
 * ds_ckpt_finish, in any order; the first of these calls waits for the flush,
 * and every part must be finished.  Errors: DS_EINVAL, DS_ESTATE, DS_ENOMEM. */
int ds_ckpt_flush_snapshot_parts(ds_ckpt *const *parts, uint32_t n_parts, ds_event *snapshot, uint32_t threads);

/* Fills the tensor region from a snapshot of the same plan: ds_flush_start on
 * this file (`threads` writers).  Once per ds_ckpt; returns at once.
 * Errors: DS_EINVAL, DS_ESTATE (a second call), DS_ENOMEM. */
int ds_ckpt_flush_snapshot(ds_ckpt *ckpt, ds_event *snapshot, uint32_t threads);

/* Writes len bytes of HOST memory at file_off of the tensor region
 * (file_off + len <= T).  Thread-safe.  Errors: DS_EINVAL, DS_ERANGE, DS_EIO. */
int ds_ckpt_write_region(ds_ckpt *ckpt, uint64_t file_off, const void *host, uint64_t len);

/*
 * Appends one chunk of a serialized object to the log.  Thread-safe and
 * concurrent with the flush of the tensors: the position is claimed with one
 * atomic add, then written.  Chunks of one object_id are numbered in call
 * order.  len may be 0 (data may then be NULL).  Errors: DS_EINVAL, DS_EIO.
 */
int ds_ckpt_append(ds_ckpt *ckpt, uint64_t object_id, const void *data, uint64_t len);

/*
 * An object state provider (Sec. V-A3): an iterator that presents the next chunk
 * of an object's serialized stream -- how many bytes, from where.  Returns 1 with
 * *data / *len set (the bytes stay valid until the next call), 0 at the end of
 * the stream, or a negative value to stop with that value as the error.
 */
typedef int (*ds_chunk_provider)(void *ctx, const void **data, uint64_t *len);

/* Drains `next` into the log: one ds_ckpt_append per chunk, in the order
 * presented, so the serializer never has to hold the whole object.  Several
 * threads may drain providers of different objects into one ds_ckpt at once.
 * *n_chunks (may be NULL) = chunks appended.  Errors: DS_EINVAL, DS_EIO, or the
 * provider's own negative value. */
int ds_ckpt_append_from(ds_ckpt *ckpt, uint64_t object_id, ds_chunk_provider next, void *ctx, uint64_t *n_chunks);

/*
 * Waits for the flush (if one was started), writes trailer and footer, syncs
 * under DS_FILE_SYNC, closes the file and frees the ds_ckpt (also on error).
 * No ds_ckpt_append may be running.  Out pointers may be NULL: the file's
 * length, seconds since ds_ckpt_create.  Errors: DS_EIO, or the error that
 * ended the snapshot / the first failed append.
 */
int ds_ckpt_finish(ds_ckpt *ckpt, uint64_t *file_bytes, double *seconds);

typedef struct ds_ckpt_layout {
  uint64_t align;
  uint64_t tensor_bytes;   /* T                              */
  uint64_t log_end;        /* E: where the trailer starts    */
  uint64_t n_tensors;
  uint64_t n_chunks;       /* log chunks                     */
  uint64_t n_objects;      /* distinct object ids            */
  uint64_t file_bytes;
} ds_ckpt_layout;

typedef struct ds_ckpt_tensor {
  uint64_t tensor_id;
  uint32_t dtype;
  uint32_t ndim;
  int64_t shape[DS_MAX_DIMS];
  uint64_t file_offset;
  uint64_t nbytes;
} ds_ckpt_tensor;

/*
 * Opens a checkpoint file and checks it: footer magic, version and checksum,
 * trailer bounds and checksum, every tensor inside [0, T) at a multiple of the
 * alignment, every chunk inside [T, E), chunk order and numbering.
 * Errors: DS_EIO (cannot open / read), DS_EFORMAT, DS_ENOMEM.
 */
int ds_ckpt_open(const char *path, ds_ckpt_reader **out);
int ds_ckpt_close(ds_ckpt_reader *reader);
int ds_ckpt_layout_info(const ds_ckpt_reader *reader, ds_ckpt_layout *out);
/* Tensor entry i (0 <= i < n_tensors). */
int ds_ckpt_tensor_info(const ds_ckpt_reader *reader, size_t i, ds_ckpt_tensor *out);
/* The k-th object in ascending id order (0 <= k < n_objects): its id and length. */
int ds_ckpt_object_at(const ds_ckpt_reader *reader, size_t k, uint64_t *object_id, uint64_t *nbytes);
/* Reads object `object_id` whole into buf (capacity cap); *len = its length.
 * Errors: DS_EINVAL (no such object), DS_ERANGE (cap too small; *len is set), DS_EIO. */
int ds_ckpt_object_read(const ds_ckpt_reader *reader, uint64_t object_id, void *buf, uint64_t cap, uint64_t *len);
/* DS_OK if the file's tensor entries, alignment and T are exactly the plan's
 * manifest (ids, dtypes, shapes, offsets, sizes, order); DS_EFORMAT if not. */
int ds_ckpt_matches_plan(const ds_ckpt_reader *reader, const ds_plan *plan);
/* ds_ckpt_matches_plan, then ds_restore_from_file on the tensor region. */
int ds_ckpt_restore(const ds_ckpt_reader *reader, ds_engine *engine, const ds_plan *plan, uint32_t threads,
                    uint32_t flags, void *compute_stream, ds_event **out);
/* The same for file `file` of a plan of several files: T is that file's region,
 * the entries are the plan's entries of that file.  ds_ckpt_matches_plan is part 0
 * of a plan of one file (DS_EINVAL for a plan of several). */
int ds_ckpt_matches_plan_part(const ds_ckpt_reader *reader, const ds_plan *plan, uint32_t file);
/* Every reader checked against its part (readers[f] = file f, n_parts = the
 * plan's number of files), then ONE restore of the whole rank out of all files
 * (ds_restore_from_files on the tensor regions).  Errors: DS_EINVAL, DS_EFORMAT,
 * and those of ds_restore_from_file. */
int ds_ckpt_restore_parts(const ds_ckpt_reader *const *readers, uint32_t n_parts, ds_engine *engine,
                          const ds_plan *plan, uint32_t threads, uint32_t flags, void *compute_stream,
                          ds_event **out);

/* ---- the training step between two snapshots -------------------------------
 *
 * Operators of the forward and backward pass that runs while a snapshot drains:
 * checkpoints of activations in 8 bits, which leave HBM to the staging that
 * opens the gate early, and the layer norms, products and activations that
 * write and read them; what joins blocks to the residual stream, the loss's log
 * probabilities, and the update.  All but the update (ds_adamw_step) only read
 * the state, so they may run before the gate of the snapshot in flight
 * (ds_event_wait_on_stream).
 *
 *   - All are asynchronous on `stream`, allocate nothing, keep nothing between
 *     calls and may be captured into a graph.  A workspace is device memory of
 *     the caller, 16-byte aligned, of the size that the function's _workspace
 *     partner names for the same arguments (ds_matmul_workspace: the same
 *     matrices; types, strides and alignment count, not the extents alone, so
 *     that a slice may need what its whole does not); it may be used by the
 *     next call on the same stream at once, and its contents mean nothing
 *     afterwards.
 *   - Results do not depend on timing: the same call on the same inputs gives
 *     the same bytes.
 *   - Sums, statistics and products are accumulated in 32 bits; a result is
 *     rounded once, when it is stored (to nearest, ties to even).
 *   - Memory that a call writes must not overlap what it reads or writes
 *     otherwise, save where a parameter says so; this is not checked.
 *   - Nothing is written, and DS_OK returned, where the output has no elements.
 */

#define DS_MX8 16u /* ds_matrix only: a checkpoint in 8 bits (below); not a type of shards */
#define DS_UF8 17u /* ds_matrix only, where a function names it: values that are not negative in 8 bits (below) */

/*
 * A matrix in device memory.  Element (i, j) is at base + itemsize *
 * (i * row_stride + j * col_stride).  Extents >= 0; the strides of extents > 1
 * are positive, one of the two is 1 and the other at least the extent of that
 * one's axis (the strides of extents of 0 and 1 are free).  Where a function
 * asks for ROWS, col_stride is the one that is 1.  dtype: DS_F32, DS_BF16,
 * DS_F16, or DS_MX8.
 *
 * DS_MX8, always ROWS: 32 neighbouring columns of a row (from column 0 on; the
 * last group may be short) share a power of two.  scale[i * scale_stride + j / 32]
 * is the byte E + 127, E = floor(log2(largest magnitude of the group)), at
 * least -126; base holds int8 codes, each the value divided by 2^(E - 6),
 * rounded to the nearest whole number (ties to even) and limited to +-127.  The
 * byte is 0 for a group of zeros, and 255 where any value of it is infinite or
 * NaN: such a group reads as NaN.  A value is off by at most half a step of
 * 2^(E - 6), by less than one where it was limited, and is representable in the
 * type it came from, so that it is read back without another rounding.  Codes
 * and scales are bytes and can be captured as shards (DS_U8).  (The values are
 * those of MXINT8 of the Open Compute Project's microscaling formats: 8-bit
 * whole numbers of 2^-6 under an E8M0 byte for 32 of them, 255 for NaN.  Where
 * that leaves a choice: the code -128 is read but never written, a group of
 * zeros has byte 0 and any other 1 at least, and a group without values has
 * codes 0.)
 *
 * DS_UF8, for values from 0 on that differ by many powers of two (second
 * moments): laid out as DS_MX8 is, with unsigned codes.  Code c under byte s is the
 * 32-bit float whose bits are (c + 8 s) << 20 -- five bits of exponent and three
 * of fraction above 2^(s - 127) -- and 0 for c = 0.  s = max(0, F - 30), F the
 * exponent field (value 2^(F - 127)) of the group's largest value; a value is
 * rounded to the nearest code (ties to even), to 1 at least if it is not 0, and
 * to the largest finite float at most.  The byte is 255, the codes 0 and the
 * values NaN where any of the group is negative, infinite or NaN.
 */
typedef struct ds_matrix {
  void *base;
  uint32_t dtype;
  uint32_t reserved; /* 0 */
  int64_t rows, cols;
  int64_t row_stride, col_stride; /* elements */
  uint8_t *scale;                 /* DS_MX8 and DS_UF8, else NULL */
  int64_t scale_stride;           /* DS_MX8 and DS_UF8: bytes from row to row, >= ceil(cols / 32); else 0 */
} ds_matrix;

/* x (DS_F32, DS_BF16, DS_F16; ROWS) into the checkpoint `saved` (DS_MX8 or DS_UF8) of
 * the same extents, and back: x is each value of `saved`, rounded where its type
 * does not hold it.  Errors: DS_EINVAL, DS_ERANGE, DS_EHIP. */
int ds_mx8_save(const ds_matrix *x, const ds_matrix *saved, void *stream);
int ds_mx8_load(const ds_matrix *saved, const ds_matrix *x, void *stream);

/*
 * Layer norm over the rows of x (DS_F32, DS_BF16, DS_F16; ROWS), eps >= 0:
 *   mean = sum_j x_j / cols, rstd = 1 / sqrt(sum_j (x_j - mean)^2 / cols + eps),
 *   y_j = (x_j - mean) * rstd * gamma_j + beta_j.
 * y: the type and extents of x, ROWS; it may be x itself.  gamma, beta: cols
 * elements of param_dtype (DS_F32, DS_BF16, DS_F16) in device memory, each may
 * be NULL (1 and 0).  mean, rstd: one float per row, each may be NULL.  saved:
 * NULL, or a DS_MX8 matrix of x's extents that x is left in, in the same pass
 * (x is read before y is written).  A row with a NaN or an infinity gives NaN
 * in y and rstd, and affects no other row.
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_layernorm_forward(const ds_matrix *x, const void *gamma, const void *beta, uint32_t param_dtype, float eps,
                         const ds_matrix *y, float *mean, float *rstd, const ds_matrix *saved, void *stream);

/*
 * Its gradient.  With h = (x - mean) * rstd and g = dy * gamma:
 *   dx = rstd * (g - sum_j g_j / cols - h * sum_j g_j h_j / cols) + residual,
 *   dgamma_j = sum over rows of dy * h,  dbeta_j = sum over rows of dy.
 * dy, dx: DS_F32, DS_BF16 or DS_F16, the same for both; ROWS.  x: that type, or the DS_MX8
 * checkpoint that the forward pass left, whose values then stand for x
 * everywhere above (mean and rstd are the forward pass's).  residual: NULL, or
 * the gradient that reaches x past the norm, of dy's type; dx may be residual
 * or dy itself.  dgamma, dbeta: cols floats, overwritten (with zeros where there
 * are no rows), each may be NULL.  Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_layernorm_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes);
int ds_layernorm_backward(const ds_matrix *dy, const ds_matrix *x, const float *mean, const float *rstd,
                          const void *gamma, uint32_t param_dtype, const ds_matrix *residual, const ds_matrix *dx,
                          float *dgamma, float *dbeta, void *workspace, uint64_t workspace_bytes, void *stream);

/* activations */
#define DS_ACT_NONE 0u
#define DS_ACT_GELU 1u      /* z * (1 + erf(z / sqrt(2))) / 2                                     */
#define DS_ACT_GELU_TANH 2u /* z * (1 + tanh(sqrt(2 / pi) * (z + 0.044715 z^3))) / 2              */
#define DS_ACT_SILU 3u      /* z / (1 + exp(-z))                                                  */
/* Results of 32 bits are off by some 2^-21 of themselves at most, far into the
 * tails (GELU_TANH: by the rounding of its argument in 32 bits, 2^-21 of
 * themselves for each unit of it); a slope by as much of its terms.  In results
 * of 16 bits exponentials are off by up to 2^-24 of themselves for each unit of
 * their argument, and factors below 2^-126 count as 0, before the one rounding. */

typedef struct ds_matmul_epilogue {
  const void *bias;          /* NULL, or b.cols elements of bias_dtype in device memory          */
  uint32_t bias_dtype;       /* DS_F32, DS_BF16 or DS_F16                                        */
  uint32_t act;              /* DS_ACT_*                                                         */
  const ds_matrix *residual; /* NULL, or a matrix of c's type and extents, ROWS; may be c itself */
  const ds_matrix *saved;    /* NULL, or a DS_MX8 matrix of c's extents: z is left in it         */
} ds_matmul_epilogue;

/*
 * z = a b + bias,  c = act(z) + residual;  a [m, k], b [k, n], c [m, n].
 * a and b: DS_BF16 or DS_F16, the same for both, each in either order (a weight
 * [out, in] is b with row_stride 1).  Either may be DS_MX8 instead: its values
 * are then rounded to the other's type (to DS_BF16 if both are DS_MX8), which is
 * exact for a checkpoint of that type.  c: DS_F32, DS_BF16 or DS_F16, ROWS.  epilogue: NULL = all of it absent.
 * With k = 0 the product is zero.  Errors: DS_EINVAL, DS_ERANGE (an extent
 * beyond 2^31 - 1, more than 2^22 tiles of c, of 64 x 64 elements at least,
 * which both functions refuse, or a workspace too small), DS_EHIP.
 */
int ds_matmul_workspace(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, uint64_t *bytes);
int ds_matmul(const ds_matrix *a, const ds_matrix *b, const ds_matrix *c, const ds_matmul_epilogue *epilogue,
              void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * The gradient of c = act(z) with z = product + bias:
 *   dz = dy * act'(z),  dbias_j = sum over rows of dz (before dz is rounded).
 * dy, dz: DS_F32, DS_BF16 or DS_F16, the same for both, ROWS.  z: that type, or a
 * DS_MX8 checkpoint.  dz may be dy itself, or z.  dbias: NULL, or cols floats, overwritten (with
 * zeros where there are no rows).  Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_activation_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes);
int ds_activation_backward(const ds_matrix *dy, const ds_matrix *z, uint32_t act, const ds_matrix *dz, float *dbias,
                           void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * A block's output u joined to the residual stream x, with what models put around
 * that: a norm behind the block, its gate, the scale of the residual, and the
 * norm in front of the next block.  Norms are by the root of the mean square.
 *   v   = u * rstd_after * after_gamma      (DS_JOIN_AFTER; else v = u),
 *         rstd_after  = 1 / sqrt(sum_j u_j^2 / cols + eps)
 *   out = keep * x + scale * gate * v
 *   y   = out * rstd_before * before_gamma  (DS_JOIN_BEFORE),
 *         rstd_before = 1 / sqrt(sum_j out_j^2 / cols + eps)
 * where out counts as it is stored, rounded to its type: the gradient has
 * nothing else to start from.  (Squares and their sums are 32-bit floats: beyond
 * their range rstd is 0.)
 */
#define DS_JOIN_AFTER 1u
#define DS_JOIN_BEFORE 2u
typedef struct ds_join {
  const void *after_gamma;  /* cols elements of param_dtype in device memory, or NULL (1); so are the next two */
  const void *gate;
  const void *before_gamma;
  uint32_t param_dtype;     /* DS_F32, DS_BF16 or DS_F16 */
  uint32_t norms;           /* DS_JOIN_*                 */
  float keep, scale;
  float eps;                /* >= 0 */
  uint32_t reserved;        /* 0 */
} ds_join;

/*
 * u, x, out, y: DS_F32, DS_BF16 or DS_F16, the same for all, ROWS, the same
 * extents.  u: NULL in front of the first block; then out = x, which `out` = NULL
 * says too, and neither `keep` nor what belongs to u counts.  y: NULL without
 * DS_JOIN_BEFORE.  rstd_after, rstd_before: one float per row, each may be NULL.
 * out may be x, and y may be u.  A row with a NaN or an infinity affects no
 * other row.  A gamma or gate that its norm or u would use is NULL where there
 * is no such norm or u.  Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_join_forward(const ds_join *join, const ds_matrix *u, const ds_matrix *x, const ds_matrix *out, const ds_matrix *y,
                    float *rstd_after, float *rstd_before, void *stream);

/*
 * Its gradient.  dout: what reaches out past the next norm, or NULL (0); dy: what
 * reaches y, NULL without DS_JOIN_BEFORE.  With h = out * rstd_before, g = dy *
 * before_gamma, k = u * rstd_after (u without that norm):
 *   d  = dout + rstd_before * (g - h * sum_j g_j h_j / cols),  dx = keep * d,
 *   dv = scale * gate * d, and with w = dv * after_gamma
 *   du = rstd_after * (w - k * sum_j w_j k_j / cols)           (dv without the norm),
 *   dbefore_j = sum over rows of dy * h,
 *   dgate_j = sum of scale * d * k * after_gamma, dafter_j = sum of scale * gate * d * k.
 * u, out: as the forward pass had and left them; rstd_*: what it left, NULL without
 * their norm.  All matrices are of one type and extent, ROWS.  Without u (NULL)
 * du, dgate and dafter are NULL and dx = d.  dx, du and the sums (cols floats,
 * overwritten, with zeros where there are no rows) may each be NULL.  dx may be
 * dout, du may be dy or u.  Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_join_backward_workspace(int64_t rows, int64_t cols, uint64_t *bytes);
int ds_join_backward(const ds_join *join, const ds_matrix *dout, const ds_matrix *dy, const ds_matrix *u, const ds_matrix *out,
                     const float *rstd_after, const float *rstd_before, const ds_matrix *du, const ds_matrix *dx,
                     float *dafter, float *dgate, float *dbefore, void *workspace, uint64_t workspace_bytes, void *stream);

/*
 * Log probabilities of given tokens.  With z = scale * x over a row of the logits
 * x (DS_F32, DS_BF16, DS_F16; ROWS), scale from 2^-64 to below 2^127 (1 / temperature):
 *   largest = max_j x_j,  logsum = log(sum_j exp(z_j - scale * largest)),
 *   logp_j = z_j - scale * largest - logsum,  logprob = logp[token],
 *   entropy = -sum_j exp(logp_j) logp_j.
 * (The two numbers hold the digits that their sum would lose, and rows that are
 * cut over several GPUs are joined by them.)
 *   - tokens: one per row in device memory; one below 0 or from cols on is none,
 *     and its logprob is 0.  May be NULL if logprob is.
 *   - logprob, largest, logsum, entropy: one float per row, each may be NULL.
 *   - The likeliest: the `top` (0 to DS_TOP_MOST) columns with the largest logits in
 *     that order, of equal ones the lowest column first: top_tokens[i * top + r]
 *     and top_logprobs[i * top + r], each may be NULL.  Columns of -infinity are left
 *     out; where fewer than `top` are left, the rest has token -1 and -infinity.
 *   - -infinity masks a column.  A row that is masked whole has logprob, largest and
 *     logsum -infinity and entropy 0.  A row with a NaN or +infinity has NaN in all
 *     its floats (logprob 0 for a token that is none) and tokens -1.
 * workspace: NULL where ds_logprobs_workspace says 0.
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
#define DS_TOP_MOST 32u
int ds_logprobs_workspace(const ds_matrix *logits, uint32_t top, uint64_t *bytes);
int ds_logprobs(const ds_matrix *logits, float scale, const int64_t *tokens, float *logprob, float *largest, float *logsum,
                float *entropy, uint32_t top, int64_t *top_tokens, float *top_logprobs, void *workspace,
                uint64_t workspace_bytes, void *stream);

/*
 * Its gradient, with p_j = exp(logp_j):
 *   dlogits_j = scale * (dlogprob * ([j = token] - p_j) - dentropy * p_j * (logp_j + entropy)).
 * largest, logsum: the forward pass's.  dlogprob: one float per row, or NULL (0);
 * tokens may then be NULL.  dentropy: likewise, and entropy (the forward pass's)
 * is needed where it is given.  dlogits: type and extents of logits, ROWS; it may
 * be logits itself.  Rows whose token is none (or dlogprob 0) and whose dentropy is 0, and rows
 * that are masked whole, have zeros whatever is in them; masked columns have p = 0.
 * (So it is that of whole rows: a part of a cut row which does not have the token would have zeros.)
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_logprobs_backward(const ds_matrix *logits, float scale, const int64_t *tokens, const float *largest,
                         const float *logsum, const float *entropy, const float *dlogprob, const float *dentropy,
                         const ds_matrix *dlogits, void *stream);

/*
 * The update, which the gate of the snapshot in flight stands in front of: AdamW
 * over all tensors of a table at once.  With t the number of this step (from 1
 * on), q = sqrt(squares) * |grad_scale|, and
 *   c = grad_scale * (q > most_norm > 0 ? most_norm / q : 1):
 *   g = c * grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   r = settings' rate * tensor's rate,
 *   param -= r * decay * param + r / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * and copy = param, rounded to copy's type (from 32 bits, as param is to its own).
 *
 * Moments are both DS_F32, or m DS_MX8 and v DS_UF8.  The latter are rounded at
 * random, without a bias (but for what the codes' limits cut: an m above 127 steps, a v below code 1), where
 * DS_MX8 and DS_UF8 otherwise say to nearest (which would lose every change that is smaller than half a step): with the 16 low bits a
 * and the 16 high bits b of the element's random number, the code of m is
 * floor(m / step + (a + 1/2) / 2^16), the sum rounded to 32 bits and the code limited
 * to +-127, and that of v is ((bits(v) + 16 b + 8) >> 20) - 8 s.  The random number of
 * element (i, j) of tensor k is mix(i * cols + j + mix(k + mix(t + mix(lo(seed) ^
 * mix(hi(seed)))))), lo and hi the halves of 32 bits of the seed, sums modulo 2^32 and
 *   mix(x): x ^= x >> 16; x *= 0x9E3779B9; x ^= x >> 15; x *= 0xBB67AE85; x ^= x >> 16.
 * What the step computes from m and v is not rounded before.
 */
typedef struct ds_adamw ds_adamw;
typedef struct ds_adamw_tensor {
  ds_matrix param; /* DS_F32, DS_BF16 or DS_F16; all matrices: ROWS, the same extents                */
  ds_matrix grad;  /* DS_F32, DS_BF16 or DS_F16                                                      */
  ds_matrix m, v;  /* both DS_F32, or DS_MX8 and DS_UF8                                              */
  ds_matrix copy;  /* DS_F32, DS_BF16 or DS_F16; all of it 0: none (its dtype is then not looked at) */
  float decay;     /* weight decay, >= 0                                                             */
  float rate;      /* factor of the settings' rate, >= 0                                             */
} ds_adamw_tensor;

typedef struct ds_adamw_settings {
  double rate, beta1, beta2, eps; /* rate >= 0; 0 <= beta < 1; eps 0 or 2^-126 at least, all within 32 bits */
  double grad_scale;              /* 1 / the scale of the loss; finite                                   */
  double most_norm;               /* norm of all gradients that is not clipped; 0: no clipping           */
  uint64_t seed;                  /* of the rounding of moments in 8 bits                                */
  const int64_t *step;            /* device memory: t (below 1 counts as 1)                              */
  const float *rate_now;          /* device memory: taken for `rate`; or NULL                            */
  const double *squares;          /* device memory: sum of all gradients' squares, before grad_scale; NULL: not known.
                                     Where it is infinite or NaN nothing is changed at all.  Needed for clipping */
} ds_adamw_settings;

/*
 * Checks the tensors and puts their table on the current device, once for all
 * steps; `tensors` may be freed afterwards.  Tensors without elements are
 * allowed; all together have at most 2^37.  Memory that the step writes must not be written for two tensors or
 * twice for one, nor hold a gradient: tables where two matrices that are written begin
 * at one address, or contiguous ones overlap, are refused (DS_EOVERLAP); interleaved views
 * are not checked.  (Two tensors may have one gradient.)
 * The table may be used from several threads; steps on the same tensors are ordered by
 * the caller.  Errors: DS_EINVAL, DS_ERANGE, DS_EOVERLAP, DS_ENOMEM, DS_EHIP.
 */
int ds_adamw_create(const ds_adamw_tensor *tensors, size_t n, ds_adamw **out);
/* As ds_plan_destroy: nothing that uses the table may still run. */
int ds_adamw_destroy(ds_adamw *table);

/* *squares (device memory) = the sum of the squares of all gradients, in 64 bits.  (Ranks that share
 * a model add theirs before the step.)  Errors, here and below: DS_EINVAL, DS_ERANGE, DS_EHIP, and
 * DS_ESTATE where the table's device is not the current one. */
int ds_adamw_squares_workspace(const ds_adamw *table, uint64_t *bytes);
int ds_adamw_squares(const ds_adamw *table, double *squares, void *workspace, uint64_t workspace_bytes, void *stream);
/* The settings are read before the call returns; what they point to, when the step runs. */
int ds_adamw_step(const ds_adamw *table, const ds_adamw_settings *settings, void *stream);

/* ---- misc ---------------------------------------------------------------- */

const char *ds_strerror(int code);

/* hipError_t of the HIP call that last produced DS_EHIP on this thread. */
int ds_last_hip_error(void);

/*
 * Measurement aid, not part of the method: a plain contiguous device-to-device
 * copy of nbytes (multiple of 16; both pointers 16-byte aligned, device
 * memory, not overlapping) with the same launch shape and memory instructions
 * as the gather kernel.  It gives the HBM rate a pure copy reaches on this
 * GPU, against which the gather is reported, and a kernel of known traffic to
 * scale hardware byte counters with.  Asynchronous on `stream`.
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_copy_probe(void *dst_dev, const void *src_dev, uint64_t nbytes, void *stream);

/*
 * For differential snapshots (the data reduction the paper's conclusions name as
 * future work; an experiment here, the engine does not use it): compares two
 * images of nbytes (multiple of 16; both pointers device memory, 16-byte
 * aligned) block by block and sets changed_dev[k] (device memory, one uint32 per
 * block, ceil(nbytes / block_bytes) of them) to 1 if block k differs anywhere,
 * else to 0.  block_bytes: a power of two >= 16 KiB.  Asynchronous on `stream`.
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_image_diff(const void *image_a_dev, const void *image_b_dev, uint64_t nbytes, uint64_t block_bytes,
                  uint32_t *changed_dev, void *stream);

/*
 * For compressed snapshots (the other data reduction the paper's conclusions name
 * as future work; an experiment here, the engine does not use it): block elision.
 * The image (nbytes, a multiple of 16; device memory, 16-byte aligned) is cut into
 * blocks of block_bytes (a power of two >= 16 KiB; the last block may be short).
 * A block all of whose 16-byte units equal its first one (zero padding,
 * zero-initialised optimizer moments, fills whose period divides 16) is CONSTANT
 * and is replaced by that unit.  Outputs, all device memory of the caller:
 *   keep_dev[k]      1 if block k is stored whole, 0 if it is constant (n_blocks x u32)
 *   pos_dev[k]       kept blocks before block k; pos_dev[n_blocks] = their number
 *                    (n_blocks + 1 x u32)
 *   patterns_dev     the first 16 bytes of every block (n_blocks x 16 bytes)
 *   packed_dev       the kept blocks one behind the other, block k in the slot of
 *                    block_bytes at pos_dev[k] * block_bytes (capacity: n_blocks slots;
 *                    of a short last block only its own bytes are written)
 * What has to leave the device is pos_dev[n_blocks] slots of packed_dev, the
 * patterns and the flags.  Asynchronous on `stream`.  The paper gives no scheme:
 * this one is the library's, defined by oracle/image_compress.py for the tests.
 * Errors: DS_EINVAL, DS_ERANGE, DS_EHIP.
 */
int ds_image_compress(const void *image_dev, uint64_t nbytes, uint64_t block_bytes, uint32_t *keep_dev,
                      uint32_t *pos_dev, void *patterns_dev, void *packed_dev, void *stream);

/*
 * Tunables for experiments, read when a plan is created / a kernel launched:
 *   "chunk_bytes"   image bytes per work-group chunk: 8, 16 (default) or 32 KiB
 *   "variant"       0 = default (non-temporal accesses; the lean gather writes the image with
 *                   write-through streaming buffer stores), 1 = plain loads and stores,
 *                   2 = non-temporal global loads and stores everywhere, 3 = default accesses but
 *                   work-group i takes chunk i (no XCD-contiguous order), 4 = default, but plans made
 *                   under it do not mark chunks for the gather's aligned-load route (tensors at
 *                   addresses that are not multiples of 16 are then read with unaligned loads),
 *                   5 = every launch is of work-groups of 16 KiB at four wavefronts per SIMD that know all
 *                   kinds of chunks (by default work-groups take 4 KiB at eight, and plans of small
 *                   contiguous shards and views with runs shorter than 16 bytes have kernels of their own)
 *   "grid_limit"    work-groups per launch of ds_pack / ds_unpack (each then walks several chunks);
 *                   0 = one per chunk or part of one (default).  Engines have their own pack_grid_limit
 *   "drop_pinned_cache"   (set only) a non-zero value frees the pinned ring and the device staging the
 *                   library keeps from the last destroyed engine for the next one (see ds_engine_create)
 *   "io_uring_available"  (get only) 1 if this process can set up an io_uring, else 0
 * Returns DS_EINVAL for an unknown key or a value out of range.
 */
int ds_config_set(const char *key, uint64_t value);
int ds_config_get(const char *key, uint64_t *value);

#ifdef __cplusplus
}
#endif
#endif /* DATASTATES_H */
