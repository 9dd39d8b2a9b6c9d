/*
 * xred.h -- C ABI of libxred: one rank's reduce step of ReduceScatter /
 * AllReduce on an AMD Instinct MI355X (gfx950).
 *
 * In a ring or one-shot ReduceScatter/AllReduce every rank, at every step,
 * reduces the chunk it received with its own chunk and forwards or keeps the
 * result (the FTAR ring pipeline and its fused ReduceCopy, Section 5 "HSDP:
 * Fault tolerant AllReduce"; collective semantics as in NCCL, Section 2.2).
 * This library performs that reduce step on one GPU, with the P peer buffers
 * already resident in local HBM.
 *
 * Definition computed by every entry point, for each element index i
 * independently:
 *
 *     out[i] = down( up(src[0][i]) (+) up(src[1][i]) (+) ... (+) up(src[P-1][i]) )
 *
 *   - a LEFT fold in source order 0..P-1 (the order is fixed, so float
 *     results are deterministic and bit-reproducible);
 *   - up(): bf16, fp16, fp8 e4m3 / e5m2 -> binary32 (exact), fp32 -> binary32,
 *     fp64 -> binary64, int8 -> uint32 (sign-extended), uint8 -> uint32
 *     (zero-extended), int32/uint32 -> uint32, int64/uint64 -> uint64; the
 *     accumulator is binary32 for float types (binary64 for fp64) and uint32
 *     / uint64 for integer types;
 *   - (+): XRED_SUM  binary32 (fp64: binary64) add, round to nearest even,
 *                    subnormals kept, or addition modulo 2^32 / 2^64;
 *          XRED_PROD binary32 (fp64: binary64) multiply, or the low 32 / 64
 *                    bits of the product;
 *          XRED_MAX / XRED_MIN  float: total order -inf < ... < -0 < +0 < ...
 *                    < +inf; a NaN among the reduced values gives the quiet
 *                    NaN 0x7FC00000 (fp64: 0x7FF8000000000000; also for P = 1
 *                    and the INIT step); int8/int32/int64 signed,
 *                    uint8/uint32/uint64 unsigned;
 *          XRED_AVG  (float types only) the XRED_SUM fold, then one division
 *                    by P in the accumulator's format, rounded to nearest even;
 *   - the accumulator starts from up(src[0][i]) (never from zero), so a column
 *     of -0.0 sums to -0.0;
 *   - down(): binary32 -> bf16 / fp16 / e5m2 round to nearest even with
 *     subnormals and overflow to +-inf; binary32 -> e4m3 (OCP "FN": no
 *     infinity, largest finite 448) round to nearest even, saturating at
 *     +-448 on overflow and for infinities; the low byte for int8 / uint8 (so
 *     their sums and products wrap modulo 2^8); identity otherwise.  NaN stays
 *     NaN; NaN payloads of SUM/PROD/AVG results are unspecified.
 *
 * Conventions shared by every call:
 *   - All functions are thread-safe and never abort; they print nothing
 *     unless XRED_TRACE is set (below).
 *   - Buffers are device pointers owned by the caller; so is the stream
 *     (a hipStream_t passed as void*, NULL = the default stream).
 *   - Every call is stream-ordered and returns once the work is enqueued.
 *     Host arrays passed in (the srcs pointer array, host-side items) are
 *     consumed before the call returns and may be reused at once.
 *   - Every argument is validated before anything is enqueued: on
 *     XRED_INVALID_ARGUMENT, XRED_UNSUPPORTED, XRED_ALIAS and
 *     XRED_OUT_OF_MEMORY nothing was enqueued.  XRED_HIP_ERROR reports a
 *     runtime failure while enqueueing; the work enqueued before it (earlier
 *     launches of a multi-launch call, a descriptor copy) stays enqueued.
 *     xred_last_error() describes the problem.  count == 0 succeeds with no
 *     launch.
 *   - Device faults (e.g. a pointer to freed memory) surface at the caller's
 *     next synchronisation of the stream, as for any HIP kernel.
 *   - Element pointers must be aligned to the element size; 16-byte aligned
 *     buffers take the fast vector path.  xred_allreduce_local,
 *     xred_reduce_scatter_local and every item of xred_batched_reduce also
 *     take it when all pointers of the call (of the item) sit at the same
 *     offset within 16 bytes (views at one element offset): the elements
 *     before the next 16-byte boundary are folded one by one.
 *     The same calls and items read in vectors too when only the sources
 *     share an offset and dst sits at another (a reduce-scatter shard of odd
 *     length), and when their sources sit at different offsets (calls and
 *     items shorter than a vector or two take a slower scalar path with the
 *     same results).
 *     xred_ring_reduce refuses chunks at different offsets (see there);
 *     xred_reduce_copy_step and xred_acc_cast read and write in vectors at any
 *     element alignment (outputs of 8- and 16-bit types a little slower where
 *     they are not 4-byte aligned); xred_allreduce_sim takes the vector path only when
 *     every buffer it touches is 16-byte aligned, else a scalar one.
 *   - Device words the library binds to a stream (the ring's relay word, the
 *     batch queue's counters) are looked up by the stream's handle.  Let a
 *     stream's work finish before destroying it if a stream created later
 *     may be handed the same handle while that work would still be running:
 *     the two would share the words.
 *
 * Environment (read once, when first needed; results never depend on them):
 *   XRED_MAX_WORKGROUPS      initial CU budget (see xred_set_max_workgroups)
 *   XRED_FUSED_WAVES_PER_CU  overrides the fused kernel's resident-wave cap
 *   XRED_RR_WG_PER_CU        workgroups per CU of the round-robin batched kernel
 *   XRED_BATCH_WG_PER_CU     workgroups per CU of host-planned range batches
 *   XRED_TRACE               anything but "0": one line on stderr per entry
 *                            point call (its arguments), per kernel launch
 *                            (kernel, grid, block, LDS bytes, stream, status)
 *                            and per failed call (status and message)
 * XRED_FUSED_WAVES_PER_CU, XRED_RR_WG_PER_CU and XRED_BATCH_WG_PER_CU are
 * tuning overrides for measurement; leave them unset.
 */
#ifndef XRED_H
#define XRED_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define XRED_API __attribute__((visibility("default")))

typedef enum {
    XRED_FLOAT32 = 0,
    XRED_BFLOAT16 = 1,
    XRED_FLOAT16 = 2,   /* IEEE binary16 */
    XRED_INT32 = 3,
    XRED_UINT32 = 4,
    XRED_INT64 = 5,
    XRED_UINT64 = 6,
    XRED_FP8_E4M3 = 7,  /* OCP 8-bit E4M3 ("FN"), saturating */
    XRED_FP8_E5M2 = 8,  /* OCP 8-bit E5M2 */
    XRED_FLOAT64 = 9,   /* IEEE binary64, accumulated in binary64 */
    XRED_INT8 = 10,
    XRED_UINT8 = 11
} xred_dtype;

/* XRED_AVG: float types only, and only where the whole reduction happens in
 * one call (fused, reduce-scatter and batched); elsewhere XRED_UNSUPPORTED. */
typedef enum { XRED_SUM = 0, XRED_PROD = 1, XRED_MAX = 2, XRED_MIN = 3, XRED_AVG = 4 } xred_op;

typedef enum {
    XRED_SUCCESS = 0,
    XRED_INVALID_ARGUMENT = 1,
    XRED_UNSUPPORTED = 2,
    XRED_ALIAS = 3,
    XRED_HIP_ERROR = 4,
    XRED_OUT_OF_MEMORY = 5
} xred_status;

enum { XRED_MAX_SRC = 64 };
enum { XRED_STEP_INIT = 1u, XRED_STEP_FINAL = 2u }; /* xred_reduce_copy_step flags */
enum { XRED_ITEMS_ON_DEVICE = 1u };                 /* xred_batched_reduce flag    */

/* One reduction of a batch: dst[i] = fold over srcs[0..nsrc) of element i,
 * for i < count.  32 bytes, naturally aligned. */
typedef struct {
    const void *const *srcs; /* nsrc source pointers (host or device array, see flags) */
    void *dst;               /* count output elements                                  */
    uint64_t count;          /* elements per source and in dst                         */
    uint32_t nsrc;           /* 1..XRED_MAX_SRC                                        */
    uint32_t reserved;       /* must be 0                                              */
} xred_item;

/*
 * AllReduce's local reduce (the per-rank reduction of FTAR's ring, Section 5;
 * AllReduce semantics, Section 2.2): dst[i] = fold_{p=0..nsrc-1} srcs[p][i],
 * i < count.
 *   srcs     host array of nsrc device pointers, each to count elements of dtype
 *   nsrc     1..XRED_MAX_SRC
 *   dst      device pointer to count elements of dtype.  dst may equal any
 *            srcs[p] exactly (in place); any other overlap is XRED_ALIAS.
 * Errors: XRED_INVALID_ARGUMENT (nsrc out of range, NULL or misaligned
 * pointer with count > 0, count*size overflow), XRED_UNSUPPORTED (dtype/op),
 * XRED_ALIAS, XRED_HIP_ERROR (launch failure).
 */
XRED_API xred_status xred_allreduce_local(const void *const *srcs, int nsrc, void *dst,
                                          size_t count, xred_dtype dtype, xred_op op,
                                          void *hip_stream);

/*
 * ReduceScatter's local reduce for rank `rank` (ReduceScatter semantics,
 * Section 2.2; the ReduceScatter phase of FTAR's ring, Section 5):
 * srcs[p] is rank p's full send buffer of nsrc*recvcount elements and
 *     dst[i] = fold_{p} srcs[p][rank*recvcount + i],  i < recvcount.
 *   rank     0 <= rank < nsrc
 *   dst      recvcount elements; may equal srcs[p] + rank*recvcount exactly
 *            (in place); any other overlap with a read slice is XRED_ALIAS.
 * Errors: as xred_allreduce_local, plus rank out of range.
 */
XRED_API xred_status xred_reduce_scatter_local(const void *const *srcs, int nsrc, int rank,
                                               void *dst, size_t recvcount, xred_dtype dtype,
                                               xred_op op, void *hip_stream);

/*
 * One step of a ring's ReduceCopy (the RedCopy / Reduce kernel operations of
 * the FTAR pipeline, Section 5): fold one incoming chunk into a local
 * accumulator chunk.
 *   flags 0                  acc[i] = acc[i] (+) up(in[i])
 *   XRED_STEP_INIT           acc[i] = up(in[i])              (acc not read)
 *   XRED_STEP_FINAL          dst[i] = down(acc[i] (+) up(in[i]))   (acc not written)
 *   INIT | FINAL             dst[i] = down(up(in[i]))              (acc unused)
 *   in       count elements of dtype
 *   acc      count accumulator elements of xred_acc_elem_size(dtype) bytes
 *            (binary32 for float dtypes, binary64 for fp64, uint32 for 8- and
 *            32-bit and uint64 for 64-bit integer dtypes), aligned to that
 *            size; may be NULL only for
 *            INIT|FINAL
 *   op       not XRED_AVG (a step does not know P; use XRED_SUM and divide)
 *   dst      count elements of dtype, used only with FINAL (may be NULL otherwise)
 * Buffers must not overlap, except dst == in exactly.
 * Errors: XRED_INVALID_ARGUMENT (unknown flag bits, NULL/misaligned pointer,
 * overflow), XRED_UNSUPPORTED, XRED_ALIAS, XRED_HIP_ERROR.
 */
XRED_API xred_status xred_reduce_copy_step(const void *in, void *acc, void *dst, size_t count,
                                           xred_dtype dtype, xred_op op, unsigned flags,
                                           void *hip_stream);

/*
 * Closing cast of a step-wise sequence: dst[i] = down(acc[i]), i < count --
 * the rounding to the I/O type that ends the ring's ReduceScatter phase once
 * the last incoming chunk has been folded into the accumulator (the Reduce of
 * the FTAR pipeline, Section 5, when the last step is not run as FINAL).
 *   acc      count accumulator elements (see xred_reduce_copy_step)
 *   dst      count elements of dtype; must not overlap acc
 * Errors: XRED_INVALID_ARGUMENT (NULL or misaligned pointer, overflow),
 * XRED_UNSUPPORTED (unknown dtype), XRED_ALIAS, XRED_HIP_ERROR.
 */
XRED_API xred_status xred_acc_cast(const void *acc, void *dst, size_t count, xred_dtype dtype,
                                   void *hip_stream);

/*
 * Many independent reductions in one launch, for latency-bound small messages
 * (the per-message software overhead T_c of the LogP model in Section 6.2 is
 * paid once per batch instead of once per message).  Each item computes the
 * xred_allreduce_local definition over its own sources.
 *   items    nitems descriptors.
 *   flags 0: `items` and every items[k].srcs are HOST memory, consumed before
 *            return (metadata by value).  Every item is validated as in
 *            xred_allreduce_local; the library stages the descriptors, with
 *            a list of every tile's item, into device memory it owns (pinned
 *            staging slots reused once the launch that read them has
 *            completed) and runs one workgroup per tile.  A batch of at most
 *            two tiles per CU and 64 KiB of staged data is read by the kernel
 *            straight from the pinned slot (no copy); batches of 256 KiB
 *            of staged data or more are copied on a stream the library owns
 *            (one per device, default priority), which the caller's stream
 *            then waits for through an event, so the copy overlaps earlier
 *            work on the caller's stream.  When a slot is free again is
 *            tracked on a second stream the library owns, never by an event
 *            left on the caller's stream, so the caller may destroy its
 *            stream as soon as the call returns.  Not capturable: on a
 *            stream under graph capture the call returns XRED_UNSUPPORTED
 *            (a replay would copy whatever a later call left in the slot).
 *   XRED_ITEMS_ON_DEVICE: `items` and every items[k].srcs are DEVICE memory,
 *            read when the kernels run, so an earlier kernel on the stream may
 *            still write them (metadata by reference, after the GPU-resident
 *            collectives of Section 6.1).  No host work per item: the kernel
 *            plans the batch from the descriptors.  Batches of 65..16384
 *            items launched eagerly take tiles in order from a counter pair
 *            in device memory the library binds to the calling stream (64
 *            streams per device, allocated once, until xred_release; the
 *            first such call on a device allocates them and waits for its
 *            stream, so it must not fall into another thread's global-mode
 *            capture); batches of up to 64 items, and all under graph
 *            capture, past 64 streams or past 16384 items, run on a kernel
 *            that keeps no state and allocates nothing, so the call can be
 *            captured in a HIP graph (same results).  Items that cannot be
 *            run safely (nsrc outside 1..64, a NULL pointer, reserved != 0)
 *            are skipped and their dst is left untouched; pointers are
 *            otherwise trusted.
 *   Items of one batch must not write memory another item reads or writes.
 * Errors: XRED_INVALID_ARGUMENT (nitems < 0, bad item in host mode, unknown
 * flags), XRED_UNSUPPORTED (also host mode under capture), XRED_ALIAS (host
 * mode, within an item),
 * XRED_OUT_OF_MEMORY (host mode: staging allocation), XRED_HIP_ERROR.
 */
XRED_API xred_status xred_batched_reduce(const xred_item *items, int nitems, xred_dtype dtype,
                                         xred_op op, unsigned flags, void *hip_stream);

/*
 * For callers that cannot allocate device memory -- code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation: the
 * device-descriptor form of xred_batched_reduce (flags XRED_ITEMS_ON_DEVICE:
 * items and every items[k].srcs are device memory, read when the kernel runs;
 * items that cannot be run safely are skipped; same results) with the tile
 * counters of its kernel in a fixed 256-byte array of device memory that the
 * library holds on each GPU it runs on until the process ends.  The call
 * allocates nothing (no hipMalloc, hipFree or allocating library routine).
 * The counters are zero when the library is loaded and every launch leaves
 * them zero, so the call can be captured in a graph and replayed; calls that
 * overlap on one GPU (other streams, other threads, replays running
 * concurrently) share the array and race: serialise them.  The first call on
 * a device looks up the array's device address.
 *   nitems   0..16384 (XRED_UNSUPPORTED beyond: the kernel plans the whole
 *            batch in on-chip memory)
 * Errors: XRED_INVALID_ARGUMENT (nitems < 0, NULL or misaligned items),
 * XRED_UNSUPPORTED (dtype/op, too many items), XRED_HIP_ERROR.
 */
XRED_API xred_status xred_batched_reduce_noalloc(const xred_item *items, int nitems,
                                                 xred_dtype dtype, xred_op op, void *hip_stream);

/*
 * All steps of a ring's ReduceCopy in one persistent launch: the FTAR
 * pipeline's in-kernel reduce (Section 5) gated by producer/consumer flags
 * in host-pinned or device memory (the host-kernel coordinated mode of
 * Section 4).  Computes dst[i] = down(fold_{s=0..nchunks-1} up(chunks[s][i])),
 * the same definition and fold order as xred_allreduce_local over the
 * chunks, with the accumulator kept on chip (LDS) between steps, so only
 * the chunks are read and only dst is written.
 *   chunks     host array of nchunks (1..XRED_MAX_SRC) device pointers to count
 *              elements each, all at one offset within 16 bytes (else
 *              XRED_UNSUPPORTED); the elements before their next 16-byte
 *              boundary are folded one by one with the tail.  dst may sit at
 *              any element offset (at another one than the chunks, results
 *              are realigned across lanes before the 16-byte stores).
 *   count      at most xred_ring_max_count(dtype) (else XRED_UNSUPPORTED)
 *   ready      NULL: every chunk is ready at launch.  Otherwise nchunks
 *              uint32 words the GPU can read coherently (hipHostMalloc'd or
 *              device memory); chunk s is read only once
 *              (int32_t)(ready[s] - epoch) >= 0 has been observed, and then
 *              with system-coherent loads, so data written before the flag
 *              is seen.  One wave of the launch polls the flags and relays
 *              their progress to the other workgroups through a word in
 *              device memory the library binds to the calling stream (up to
 *              64 streams per device, until xred_release); under graph
 *              capture, on hipStreamPerThread or past 64 streams, every
 *              workgroup polls the flags itself, which costs more with host
 *              flags.
 *   timeout_us bound on each wait (0: one second; capped at 60 s).  A
 *              workgroup whose wait makes no progress for that long writes 1
 *              to *status (if status is not NULL) and stops; dst is then
 *              unspecified.  The caller zeroes *status before the call if it
 *              wants to check it.
 * Errors: as xred_allreduce_local; XRED_UNSUPPORTED for chunks at different
 * offsets within 16 bytes or counts beyond the capacity.
 */
XRED_API xred_status xred_ring_reduce(const void *const *chunks, int nchunks, void *dst,
                                      size_t count, xred_dtype dtype, xred_op op,
                                      const uint32_t *ready, uint32_t epoch, uint64_t timeout_us,
                                      uint32_t *status, void *hip_stream);

/* Largest count xred_ring_reduce accepts for dtype on the current device. */
XRED_API size_t xred_ring_max_count(xred_dtype dtype);

/* Schedules of xred_allreduce_sim. */
typedef enum {
    XRED_SCHEDULE_RING = 0,  /* ring: 2(G-1) steps, one launch each */
    XRED_SCHEDULE_RHD = 1,   /* recursive halving-doubling, G a power of two: 2 log2(G)
                                steps, one launch each */
    XRED_SCHEDULE_RING_ONE_LAUNCH = 2, /* the ring, every step in one launch */
    XRED_SCHEDULE_RHD_ONE_LAUNCH = 3   /* halving-doubling, every step in one launch */
} xred_schedule;

/*
 * A whole AllReduce over nranks = G simulated ranks whose buffers all live on
 * this GPU, step by step: the ring of the FTAR pipeline (Section 5:
 * sendCopy, RedCopy, Reduce, RecvCopy, Recv) or the recursive
 * halving-doubling schedule (Section 2.2).  Each step is one launch holding
 * every rank's work of that step.
 *
 * Every hop is the two-source reduce down(up(received) (+) up(own)), so a
 * partial is rounded to the I/O dtype each time it travels.  In the ring,
 * chunk c is folded in arrival order c+1, c+2, ..., c+G-1, c (mod G); in
 * halving-doubling, at distance d = G/2, ..., 1 every rank combines its
 * partner's partial with its own.  Messages are zero-copy: the partial a
 * rank forwards is stored once, in that rank's own recvbuf at the chunk's
 * place, and the next rank reads it there; a reduced chunk is forwarded from
 * where it was written.  No staging buffer and no extra store per hop.
 *
 *   sendbufs, recvbufs  host arrays of G device pointers to count elements
 *              each, consumed before return.  recvbufs[r] may equal
 *              sendbufs[r] (in place); a recvbuf must not overlap any other
 *              buffer.  Sends may overlap each other.
 *   G          1..XRED_MAX_SRC; a power of two for XRED_SCHEDULE_RHD.  With
 *              one rank recvbufs[0] becomes a bitwise copy of sendbufs[0].
 *   chunks     xred_sim_chunk(count, G) elements each, i.e. ceil(count / G)
 *              rounded up to a multiple of 64; trailing chunks are short or
 *              empty.  (RHD blocks are the same chunks.)
 * The ONE_LAUNCH schedules run every step in a single launch and give the
 * same bits.  Each thread folds one element vector of one chunk in the
 * schedule's order, handing every message to the next hop in registers,
 * rounded to the I/O dtype exactly as when it is sent, and stores only the
 * final bits into every recvbufs[r]: the messages the per-step schedule
 * stores and then overwrites in its AllGather phase are never written (the
 * intermediate stores ReduceCopy avoids, Section 5).  The call reads G N and
 * writes G N elements instead of 5 (G-1) N, in one launch instead of
 * 2 (G-1) or 2 log2(G).
 * When the stream reaches the end of the call every recvbufs[r] holds the
 * same bits.  Buffers that are all 16-byte aligned take the vector path,
 * others (element-aligned) a scalar path with the same results.
 * Errors: XRED_INVALID_ARGUMENT (G out of range, unknown schedule, RHD with G
 * not a power of two, NULL or misaligned pointer, size overflow),
 * XRED_UNSUPPORTED, XRED_ALIAS, XRED_HIP_ERROR.
 */
XRED_API xred_status xred_allreduce_sim(const void *const *sendbufs, void *const *recvbufs,
                                        int nranks, size_t count, xred_dtype dtype, xred_op op,
                                        xred_schedule schedule, void *hip_stream);

/* Chunk length of xred_allreduce_sim's schedules (0 when nranks < 1). */
XRED_API size_t xred_sim_chunk(size_t count, int nranks);

/*
 * ------------------------------------------------ around a reduced activation --
 * The calls below take what a reduction over ranks produced on to the next
 * one: the partial sums of a tensor-parallel layer are folded, joined with the
 * residual stream and normalised in one pass (xred_fold_norm); a mixture of
 * experts then picks each token's experts (xred_route), orders the rows by
 * expert -- counts and offsets are the metadata of the AllToAllv that carries
 * them, resident on the GPU as in Section 6.1 -- (xred_dispatch_plan,
 * xred_dispatch) and reduces the experts' rows back to tokens (xred_combine).
 * The *_grad calls are their backward passes.
 *
 * Shared conventions, besides those at the top of this file:
 *   - dtype is XRED_FLOAT32, XRED_BFLOAT16 or XRED_FLOAT16 unless stated;
 *     all arithmetic, sums and statistics are binary32, and each output is
 *     rounded once, as down() above rounds.
 *   - Matrices are row-major with a distance between rows (xred_rows); rows
 *     need only be aligned to their element.
 *   - Nothing is allocated and nothing is kept between calls, so every call
 *     can be captured in a HIP graph; calls that need scratch memory take it
 *     from the caller (workspace, at least the size the *_workspace function
 *     gives, 16-byte aligned; its contents need not be kept or cleared).
 *   - Results do not depend on the CU budget or on the order in which
 *     workgroups run (no floating-point atomics).
 *   - An output may not overlap any other buffer of the call unless stated.
 *   - Errors: XRED_INVALID_ARGUMENT, XRED_UNSUPPORTED (types and sizes),
 *     XRED_ALIAS, XRED_HIP_ERROR; zero rows or tokens succeed with no launch
 *     where nothing is to be written.
 */

/* Row r of a matrix starts r * stride elements after data; stride is at least
 * the row's length.  data NULL: the matrix is absent. */
typedef struct {
    void *data;
    uint64_t stride;
} xred_rows;

enum { XRED_MAX_HIDDEN = 32768 };  /* elements of a row xred_fold_norm keeps on chip */
enum { XRED_MAX_EXPERTS = 1024, XRED_MAX_TOPK = 32, XRED_MAX_EXPERT_GROUPS = 64 };

/*
 * Fold of P partial sums, residual addition and root-mean-square norm:
 *     h      = (up(src[0]) + up(src[1]) + ... + up(src[P-1])) + up(residual)
 *     rstd   = 1 / sqrt(mean(h^2) + eps)                  (one value a row)
 *     y      = h * (rstd * up(weight))
 *     sum    = down(h),  out = down(y)
 *     out8   = e4m3(y / scale),  scale = max(amax, 2^-100) / 448, amax the
 *              largest |y| of the group (a NaN in a group gives NaN)
 * h is not rounded before it is normalised.  rstd, scale and y / scale are good to a
 * few units in the last place of binary32 (hardware reciprocals and square root), so
 * a y / scale that close to the middle of two e4m3 values may become either.
 *   srcs      host array of nsrc (1..XRED_MAX_SRC) device pointers, rows x
 *             hidden each, all with row distance src_stride; read before return
 *   residual  optional; weight: hidden elements of weight_dtype (dtype or
 *             XRED_FLOAT32), NULL: ones
 *   sum, out, out8, rstd   outputs, each optional, at least one of out and
 *             out8 present.  sum and out may each be one of the inputs (the
 *             same pointer and stride), out only where sum is another.
 *   scale     rows x ceil(hidden / group) binary32, present with out8
 *   group     elements of a row that share a scale: 32, 64, 128, 256 or 512
 *             (the last group may be short), or 0 for the whole row
 *   hidden    1..XRED_MAX_HIDDEN (else XRED_UNSUPPORTED)
 */
typedef struct {
    const void *const *srcs;
    uint64_t src_stride;
    uint32_t nsrc;
    uint32_t group;
    uint64_t rows, hidden;
    xred_rows residual, sum, out, out8, scale;
    const void *weight;
    float *rstd;
    xred_dtype dtype, weight_dtype;
    float eps;
} xred_fold_norm_args;
XRED_API xred_status xred_fold_norm(const xred_fold_norm_args *args, void *hip_stream);

/*
 * The gradient of xred_fold_norm's out:
 *     g       = up(dout) * up(weight),  n = up(sum) * rstd
 *     dx      = down(rstd * (g - n * mean(g * n)) + up(dsum))
 *     dweight = sum over rows of up(dout) * n             (binary32)
 * dx is the gradient of the residual and of every source alike.
 *   sum, rstd  what xred_fold_norm wrote;  dsum: optional, the gradient that
 *              reaches `sum` itself along the residual stream
 *   dx         may be dout or dsum (the same pointer and stride)
 *   dweight    hidden binary32 values, optional; set (to zero where there are
 *              no rows), not added to.  It needs the workspace.
 */
typedef struct {
    uint64_t rows, hidden;
    xred_rows dout, sum, dsum, dx;
    const void *weight;
    const float *rstd;
    float *dweight;
    void *workspace;
    uint64_t workspace_bytes;
    xred_dtype dtype, weight_dtype;
} xred_fold_norm_grad_args;
XRED_API xred_status xred_fold_norm_grad(const xred_fold_norm_grad_args *args, void *hip_stream);

/* Bytes of workspace xred_fold_norm_grad needs for dweight. */
XRED_API size_t xred_fold_norm_grad_workspace(uint64_t rows, uint64_t hidden);

/* How xred_route scores an expert. */
typedef enum { XRED_SCORE_SOFTMAX = 0, XRED_SCORE_SIGMOID = 1 } xred_score;
enum { XRED_ROUTE_RENORM = 1u };   /* xred_route flags */

/*
 * Routing of tokens to experts: each token's topk best experts by key, in
 * descending order, ties to the lowest index.
 *     softmax   score = softmax(x) over the experts, key = x + bias (the log of
 *               the score up to a constant of the row)
 *     sigmoid   score = 1 / (1 + exp(-x)),           key = score + bias
 * An expert whose logit or whose key is -inf is never chosen; a slot for which
 * none is left gets id -1 and weight 0 (all of them in a row of -inf, a
 * padding row).  A NaN key ranks above every number, so that it shows.
 * With groups > 1 the experts form that many groups of consecutive ones, and
 * only the group_topk best groups (ties to the lowest) are chosen from; a
 * group's rank is its best key (group_score 1) or the sum of its best two (2).
 *     weight    = scale * score; with XRED_ROUTE_RENORM the chosen scores are
 *                 divided by their sum first (softmax: the softmax over the
 *                 chosen logits; scores that sum to 0 stay 0)
 * bias (a balance correction) steers the choice only, not the weights.
 * With softmax it is added to the logits, and groups are ranked by logits too:
 * a router that adds its bias to the probabilities p, or ranks groups by sums of
 * them, chooses other experts.  That router is the sigmoid form on
 * log(p / (1 - p)), whose score is p up to rounding (a p of 0 is then masked).
 *   logits   tokens x experts of dtype; bias: experts binary32, or NULL
 *   ids      tokens x topk int32;  weights: tokens x topk binary32
 *   experts  1..XRED_MAX_EXPERTS, topk 1..min(experts, XRED_MAX_TOPK), groups
 *            a divisor of experts up to XRED_MAX_EXPERT_GROUPS, group_topk
 *            1..groups
 * Keys are computed in binary32 (x, then exp, + 1, 1 / and + bias, each
 * rounded), so equal inputs are chosen alike on every call.
 */
typedef struct {
    uint64_t tokens;
    uint32_t experts, topk;
    uint32_t groups, group_topk, group_score;
    uint32_t flags;
    xred_rows logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    xred_dtype dtype;
    xred_score score;
    float scale;
} xred_route_args;
XRED_API xred_status xred_route(const xred_route_args *args, void *hip_stream);

/*
 * The gradient of xred_route's weights with respect to the logits (the choice
 * itself and the bias have none): every element of dlogits is written, zero
 * where the weights do not depend on it.
 *   ids       as xred_route gave them; ids outside [0, experts) are passed over,
 *             the others of a token differ
 *   dweights  tokens x topk binary32
 *   dlogits   tokens x experts of dtype
 * score, flags and scale as in the forward call.
 */
typedef struct {
    uint64_t tokens;
    uint32_t experts, topk;
    uint32_t flags;
    xred_rows logits, dlogits;
    const int32_t *ids;
    const float *dweights;
    xred_dtype dtype;
    xred_score score;
    float scale;
} xred_route_grad_args;
XRED_API xred_status xred_route_grad(const xred_route_grad_args *args, void *hip_stream);

/*
 * Order of the routed rows by expert.  Slot j of token t (index t * topk + j)
 * with expert ids[t][j] in [0, experts) becomes row
 *     pos[t][j] = offsets[id] + the number of earlier slots of that expert
 * of the dispatched rows; any other id drops the slot, and its pos is -1.
 *   ids      tokens x topk int32;  pos: the same shape, output
 *   counts   experts int32, output: rows of each expert
 *   offsets  experts + 1 int32, output: each expert's first row, then the
 *            number of rows in all
 *   slots    optional output, tokens * topk int32: the slot of every row, for
 *            rows 0..offsets[experts] - 1 (later entries are left untouched)
 *   experts  1..XRED_MAX_EXPERTS, topk 1..XRED_MAX_TOPK (else
 *            XRED_UNSUPPORTED), tokens * topk below 2^31
 * No tokens: counts and offsets are set to 0.
 */
typedef struct {
    uint64_t tokens;
    uint32_t experts, topk;
    const int32_t *ids;
    int32_t *counts, *offsets, *pos, *slots;
    void *workspace;
    uint64_t workspace_bytes;
} xred_dispatch_plan_args;
XRED_API xred_status xred_dispatch_plan(const xred_dispatch_plan_args *args, void *hip_stream);

/* Bytes of workspace xred_dispatch_plan needs for tokens * topk = slots; 0 where
 * it needs none (small batches). */
XRED_API size_t xred_dispatch_plan_workspace(uint64_t slots, uint32_t experts);

/*
 * Rows to their places: out[pos[t][j]] = x[t] for every slot whose pos is in
 * [0, out_rows); other slots are passed over, and rows no slot names are left
 * untouched.  Bits are copied (any dtype).
 *   x          tokens x hidden;  out: out_rows x hidden, both of dtype
 *   scale, out_scale   optional, together: tokens x scale_columns and out_rows x
 *              scale_columns binary32 values that travel with the rows (the
 *              scales of 8-bit rows)
 *   pos        tokens x topk int32; the places of one call differ
 */
typedef struct {
    uint64_t tokens, hidden, out_rows, scale_columns;
    uint32_t topk;
    xred_dtype dtype;
    xred_rows x, out, scale, out_scale;
    const int32_t *pos;
} xred_dispatch_args;
XRED_API xred_status xred_dispatch(const xred_dispatch_args *args, void *hip_stream);

/*
 * The experts' rows back to their tokens, a weighted fold in slot order:
 *     out[t] = down(((up(base[t]) + w[t][0] * up(y[pos[t][0]])) + ...))
 * over the slots whose pos is in [0, y_rows); without base the fold starts from
 * the first product, and a token without a slot gives base, or 0.  Without
 * weights w is 1 (with them left out it is also the gradient of xred_dispatch).
 *   y        y_rows x hidden;  base (optional), out: tokens x hidden, of dtype;
 *            out may be base (the same pointer and stride)
 *   weights  tokens x topk binary32, or NULL;  pos: tokens x topk int32
 */
typedef struct {
    uint64_t tokens, hidden, y_rows;
    uint32_t topk;
    xred_dtype dtype;
    xred_rows y, base, out;
    const int32_t *pos;
    const float *weights;
} xred_combine_args;
XRED_API xred_status xred_combine(const xred_combine_args *args, void *hip_stream);

/*
 * The gradient of xred_combine (base's is dout itself):
 *     dy[pos[t][j]]  = down(w[t][j] * up(dout[t]))
 *     dweights[t][j] = sum over the row of up(dout[t]) * up(y[pos[t][j]])
 * for the slots whose pos is in [0, y_rows), whose places differ; the others'
 * dweights are 0, and rows of dy no slot names are left untouched.
 *   dweights  tokens x topk binary32, optional (y is then not read)
 *   dy        may be y (the same pointer and stride)
 */
typedef struct {
    uint64_t tokens, hidden, y_rows;
    uint32_t topk;
    xred_dtype dtype;
    xred_rows dout, y, dy;
    const int32_t *pos;
    const float *weights;
    float *dweights;
} xred_combine_grad_args;
XRED_API xred_status xred_combine_grad(const xred_combine_grad_args *args, void *hip_stream);

/*
 * CU budget: at most max_workgroups workgroups per launch of the fused,
 * reduce-scatter, step-wise, cast and batched kernels and of those of the calls
 * around a reduced activation (0 = no limit, the
 * default), so a reduction can run beside compute kernels on the rest of the
 * chip -- the paper's FTAR kernel uses two thread blocks and stays hidden
 * behind the network (Section 5).  Results do not depend on it.  Process-wide;
 * returns the previous value.  xred_ring_reduce applies it too, but never goes
 * below the workgroups its on-chip accumulators need (one per 4 tiles).
 * The budget bounds the workgroups a launch may have in flight; it does not
 * make a reduce run beside a kernel that fills the chip: on MI355X a bf16
 * matrix product's workgroups take whole CUs, and a reduce on another stream
 * waits for free CUs and then runs alone (measured: the two streams take the
 * sum of their times, capped or not).  xred_stream_create_partition gives the
 * reduce CUs of its own.
 */
XRED_API unsigned xred_set_max_workgroups(unsigned max_workgroups);

/*
 * Co-scheduling by a CU partition (the paper keeps its collective kernels to
 * a few thread blocks so compute keeps the rest of the GPU, Section 5).
 * Creates, on the current device, a HIP stream whose kernels run only on
 * `ncu` compute units, ncu / X of them on each of the device's X XCDs, and,
 * if `rest` is not NULL, a second stream whose kernels run only on all the
 * other CUs.  Kernels on the two streams then run at the same time, each on
 * its own CUs: a reduce launched on *stream beside a matrix product on *rest
 * (measured on MI355X: P=8 x 8 MiB bf16 reduces on 16 CUs at ~1 TB/s,
 * concurrently with the product).  A kernel sized for the whole chip runs
 * slower on a partition than the CU count alone suggests (torch's bf16
 * matrix products lost 27-37 % on any partial CU set), so the partition pays
 * off only where the compute side tolerates it.
 *   ncu     a positive multiple of X below the CU count (256 CUs, X = 8 on
 *           MI355X: 8, 16, ..., 248)
 *   stream  receives the new stream (a hipStream_t); NULL on failure
 *   rest    NULL, or receives the second stream; NULL on failure
 * Each stream is a hardware queue of its own; the runtime has few per process
 * and refuses more with XRED_HIP_ERROR (nothing is created then).  The
 * streams are ordinary HIP streams to every libxred entry point and to other
 * libraries; destroy them with xred_stream_destroy or hipStreamDestroy.
 * Errors: XRED_INVALID_ARGUMENT (stream NULL, ncu out of range),
 * XRED_UNSUPPORTED (CU count not a multiple of the XCD count),
 * XRED_HIP_ERROR.
 */
XRED_API xred_status xred_stream_create_partition(int ncu, void **stream, void **rest);

/* Waits for the work enqueued on `stream` (not NULL), then destroys it.
 * Errors: XRED_INVALID_ARGUMENT, XRED_HIP_ERROR. */
XRED_API xred_status xred_stream_destroy(void *stream);

/* Bytes per accumulator element for dtype: 4 (binary32 or uint32), 8
 * (binary64 for fp64, uint64 for int64/uint64), 0 if unknown. */
XRED_API size_t xred_acc_elem_size(xred_dtype dtype);

/* Static, human-readable name of a status code. */
XRED_API const char *xred_status_string(xred_status s);

/* Detail of the last failed call on the calling thread ("" if none). */
XRED_API const char *xred_last_error(void);

/* Library version: major*10000 + minor*100 + patch. */
XRED_API int xred_version(void);

/* Frees the library's host-mode batch staging buffers, and the ring's relay
 * words and the batch queue's counters, on every device after synchronising
 * the device work that uses them, and unbinds those from their streams.
 * Optional; later calls re-create what they need. */
XRED_API void xred_release(void);

#ifdef __cplusplus
}
#endif

#endif /* XRED_H */
