/*
 * mqgrad.h -- C ABI of libmqgrad: the per-iteration gradient codec of MQGrad
 * (arXiv 1804.08066) for one NVIDIA B200 (sm_100a).
 *
 * The paper's data path per training iteration (Algorithm 1, Section 3.2):
 *   worker:  g~ <- Quantize(g, K)                         (WorkerIterate)
 *   server:  g_p <- De-quantize(g~_p) for p = 1..P,
 *            g <- sum_p g_p / P,  w <- w - eta * g        (ReceiveQGThenSendQG, steps 6-7 of Fig. 3)
 * The paper leaves the codec itself to an external page; this library fixes it as:
 * a symmetric K-bit affine grid on [-s, +s] per bucket (s = max |x| of the bucket),
 * unbiased stochastic rounding with 16 random bits per element from Philox4x32-10,
 * and LSB-first packing of the K-bit codes into little-endian 32-bit words.
 *
 * Conventions that hold for every call
 *   - Every data pointer is caller-owned DEVICE memory unless stated otherwise; the
 *     library never allocates, frees or keeps device memory.  Arrays of pointers
 *     (codes[W], scales[W]) and segment tables are HOST arrays, read during the call.
 *   - Calls enqueue work on `cuda_stream` (a cudaStream_t passed as void*, NULL = the
 *     default stream) and return without waiting for it.
 *   - Return value: MQG_OK, or a negative mqg_status; nothing is thrown and nothing
 *     aborts.  Arguments are checked on the host before any launch; on an error
 *     nothing has been enqueued.  mqg_last_error() gives the calling thread's message.
 *   - n == 0 is a valid no-op.  Inputs must be finite; results for NaN/Inf are unspecified.
 *   - Output buffers must not overlap inputs, except `params`, updated in place.
 *   - grad, params, acc and codes must be 16-byte aligned; scales 4-byte aligned.
 *   - 1 <= bits <= 8.  L = 2^bits - 1.
 *   - bucket >= 1, and bucket % 32 == 0 unless bucket >= n (one bucket), so that every
 *     bucket's codes start on a word boundary for every bit width.
 */
#ifndef MQGRAD_H_
#define MQGRAD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int mqg_status;
enum {
    MQG_OK = 0,
    MQG_ERR_INVALID = -1,          /* null pointer, bad bucket, bad segment table, overlapping sizes */
    MQG_ERR_BITS = -2,             /* bits outside 1..8 */
    MQG_ERR_ALIGN = -3,            /* a buffer is not aligned as required */
    MQG_ERR_TOO_MANY_WORKERS = -4, /* W outside 1..MQG_MAX_WORKERS */
    MQG_ERR_CUDA = -5,             /* a CUDA runtime call failed; see mqg_last_error() */
    MQG_ERR_TIMEOUT = -6           /* a kernel's bounded wait ran out (mqg_check_timeouts) */
};

typedef enum { MQG_F32 = 0, MQG_BF16 = 1 } mqg_dtype;

#define MQG_MAX_WORKERS 32

/* Number of 32-bit words of one worker's packed stream: ceil(n * bits / 32).  Host-only helper. */
size_t mqg_code_words(uint64_t n, int bits);

/* Number of buckets (= scales) for n elements: ceil(n / bucket).  Host-only helper. */
size_t mqg_num_buckets(uint64_t n, uint64_t bucket);

/* Bytes one worker sends for n elements: 4 * code_words + 4 * num_buckets (reported, never timed). */
size_t mqg_wire_bytes(uint64_t n, int bits, uint64_t bucket);

/*
 * Quantize(g, K) of Algorithm 1 (WorkerIterate), fused with packing.
 *   grad        [in]  n elements of `dtype` (fp32, or bf16 widened exactly to fp32 in the kernel)
 *   codes       [out] mqg_code_words(n, bits) words; code i at bits [i*bits, i*bits+bits) of the
 *                     stream, bit j of the stream = bit (j % 32) of word j / 32; pad bits are zero
 *   scales      [out] mqg_num_buckets(n, bucket) floats; s_k = max |x| of bucket k, flushed to 0
 *                     below 2^-96 (then every code of the bucket is 0)
 *   seed, worker, step, elem_offset
 *                     key the random draws: element i draws from Philox4x32-10 with key = seed and
 *                     counter = ((elem_offset + i) / 8, worker, step), 16 bits per element, so the
 *                     codes are a pure function of the arguments (reproducible, order-free).
 *                     elem_offset is the element's position in the flat model; multiples of 8
 *                     take the fast path.
 * Per element: t = fma(x, L / (2 s), L / 2) in fp32, code = floor(t) + [u < t - floor(t)],
 * u = (h + 1/2) / 65536.
 */
mqg_status mqg_quantize(const void* grad, uint64_t n, int bits, uint64_t bucket, uint64_t seed,
                        uint32_t* codes, float* scales,
                        mqg_dtype dtype, uint32_t worker, uint32_t step, uint64_t elem_offset,
                        void* cuda_stream);

/*
 * Quantize(g_p, K) of Algorithm 1 for W workers whose gradients live on this device (P workers
 * simulated on one GPU, or several replicas per device), in one launch where the shape allows:
 * exactly mqg_quantize(grads[w], ..., codes[w], scales[w], worker = first_worker + w, ...) for
 * w = 0..W-1, bit for bit, without paying the per-launch fixed cost W times.
 *   grads, codes, scales  HOST arrays of W device pointers (read during the call only); each
 *                         buffer as in mqg_quantize; the outputs are what mqg_server_step and
 *                         mqg_dequant_accumulate take as codes[] / scales[]
 * Two kernels take all workers in one launch.  The first wants at least 2048 elements, elem_offset a multiple of 8 and
 * buckets of at most 16384 elements (the L2-norm variant 8192), those above 4096 a multiple of 1024.  The second takes buckets of up to 49152
 * elements (or one such gradient) with any elem_offset, a CTA to a bucket: used where the first does not apply for
 * buckets above 4096 elements, and below 65536 elements for up to 512 buckets.  Other shapes run as W launches (or more)
 * inside the call.
 * Errors: as mqg_quantize, per worker; MQG_ERR_TOO_MANY_WORKERS for W outside 1..MQG_MAX_WORKERS.
 */
mqg_status mqg_quantize_workers(const void* const* grads, int W, uint64_t n, int bits, uint64_t bucket,
                                uint64_t seed, uint32_t* const* codes, float* const* scales,
                                mqg_dtype dtype, uint32_t first_worker, uint32_t step,
                                uint64_t elem_offset, void* cuda_stream);

/*
 * De-quantize + sum of Algorithm 1 (ReceiveQGThenSendQG, before the division by P):
 *   acc[i] = ((x^_0[i] + x^_1[i]) + ... ) in worker order 0..W-1, fp32,
 *   x^_w[i] = (2 q - L) * (s / L) with one rounding for s / L and one for the product;
 *   a zero-scale bucket decodes to +0.
 *   codes, scales  [in]  HOST arrays of W device pointers, laid out as mqg_quantize writes them
 *   acc            [out] n floats; overwritten, or (add_into_acc != 0) the sum continues from the
 *                        value already there: acc = ((acc + x^_0) + x^_1) + ...
 */
mqg_status mqg_dequant_accumulate(const uint32_t* const* codes, const float* const* scales, int W,
                                  int bits, uint64_t n, float* acc,
                                  uint64_t bucket, int add_into_acc, void* cuda_stream);

/*
 * w <- w - eta * g of Algorithm 1 (WorkerIterate's update), one fused multiply-add per element:
 * params[i] = fma(-lr, acc[i], params[i]).  Pass lr = eta / P to apply the mean of P workers.
 */
mqg_status mqg_apply(float* params, const float* acc, float lr, uint64_t n, void* cuda_stream);

/*
 * The server's whole step in one pass over memory (steps 6-7 of Fig. 3, Section 3.2): unpack,
 * de-quantize and sum W workers' buffers and update the shared parameters, with exactly the
 * roundings of mqg_dequant_accumulate followed by mqg_apply.
 *   params   [in/out] n floats, updated in place
 *   acc_out  [out]    optional (may be NULL): the summed gradient, n floats
 */
mqg_status mqg_server_step(const uint32_t* const* codes, const float* const* scales, int W, int bits,
                           uint64_t n, uint64_t bucket, float* params, float lr, float* acc_out,
                           void* cuda_stream);

/*
 * The server's downlink (ReceiveQGThenSendQG of Algorithm 1, lines 3-5; steps 6-8 of Fig. 3): the
 * global gradient g = (sum_p g_p) * mean_scale, with the sum as in mqg_dequant_accumulate and one
 * rounding for the product (pass mean_scale = 1 / P for the paper's mean), is quantized again with
 * the same bit width and bucket, exactly as mqg_quantize(g, ...) with elem_offset 0 would, without
 * storing g.  Workers then apply it with mqg_server_step(W = 1, lr = eta).
 *   codes_out, scales_out [out] laid out as mqg_quantize writes them
 *   worker, step               key the random draws of this encode (use an id no worker uses)
 * Buckets (or a single bucket n) above 8192 elements are rejected with MQG_ERR_INVALID.
 */
mqg_status mqg_server_requantize(const uint32_t* const* codes, const float* const* scales, int W,
                                 int bits, uint64_t n, uint64_t bucket, float mean_scale,
                                 uint64_t seed, uint32_t* codes_out, float* scales_out,
                                 uint32_t worker, uint32_t step, void* cuda_stream);

/*
 * Codec variant: the (min, max) range scheme the footnote of Section 3.2 refers to, with nearest
 * rounding and no random draws.  Per bucket lo = min x, hi = max x (a zero of either sign stored
 * as +0), r = fl(hi - lo), L = 2^bits - 1:
 *     code = min(L, floor(fma(fl(x - lo), fl(L / r), 1/2)))      x^ = fma(code, fl(r / L), lo)
 * a bucket with r < 2^-96 is constant: every code is 0 and every x^ is lo.
 *   ranges  [out] 2 * mqg_num_buckets(n, bucket) floats, 8-byte aligned: ranges[2b] = lo,
 *                 ranges[2b + 1] = hi of bucket b
 *   codes   [out] as mqg_quantize
 * Buckets of at most 49152 elements take one pass over the gradient; larger ones two.
 * Errors as mqg_quantize; MQG_ERR_ALIGN for a ranges pointer that is not 8-byte aligned.
 */
mqg_status mqg_quantize_minmax(const void* grad, uint64_t n, int bits, uint64_t bucket, uint32_t* codes,
                               float* ranges, mqg_dtype dtype, void* cuda_stream);
/*
 * The (min, max) variant for W workers' gradients of the same shape in ONE launch (the variant's
 * counterpart of mqg_quantize_workers; the scheme the footnote of Section 3.2 points to): worker w's
 * outputs are bit-identical to mqg_quantize_minmax on its gradient.
 *   grads / codes / ranges   HOST arrays of W DEVICE pointers, each as in mqg_quantize_minmax; caller-owned
 * Shapes the batched kernel does not take run as W calls with the same results.
 * Errors as mqg_quantize_minmax, plus MQG_ERR_TOO_MANY_WORKERS for W outside 1..MQG_MAX_WORKERS.
 */
mqg_status mqg_quantize_workers_minmax(const void* const* grads, int W, uint64_t n, int bits, uint64_t bucket,
                                       uint32_t* const* codes, float* const* ranges, mqg_dtype dtype,
                                       void* cuda_stream);


/*
 * Server side of the variant: mqg_dequant_accumulate and mqg_server_step with x^ as above and the
 * same ordered sum and fused update.  `ranges` is a HOST array of W device pointers, each laid out
 * as mqg_quantize_minmax writes it.
 */
mqg_status mqg_dequant_accumulate_minmax(const uint32_t* const* codes, const float* const* ranges, int W,
                                         int bits, uint64_t n, float* acc, uint64_t bucket,
                                         int add_into_acc, void* cuda_stream);
mqg_status mqg_server_step_minmax(const uint32_t* const* codes, const float* const* ranges, int W, int bits,
                                  uint64_t n, uint64_t bucket, float* params, float lr, float* acc_out,
                                  void* cuda_stream);

/*
 * Codec variant: one bit per element with error feedback, the 1-bit scheme that the related-work
 * section (Section 2) cites: the sign of every value is sent and the quantization error is carried
 * into the next mini-batch.  With e the worker's residual (n floats kept by the caller from one
 * iteration to the next, zero before the first):
 *     v = fl(g + e);   code = 1 if v >= 0 (a zero of either sign included) else 0
 *     per bucket: neg = mean of v over the elements with code 0, pos = mean over those with code 1
 *                 (0 for an empty class), written as ranges[2b] = neg, ranges[2b + 1] = pos
 *     x^ = what mqg_server_step_minmax / mqg_dequant_accumulate_minmax with bits = 1 reconstruct from
 *          (code, neg, pos): neg for code 0, fl(fl(pos - neg) + neg) for code 1; a bucket with
 *          fl(pos - neg) < 2^-96 is constant (codes cleared, x^ = neg)
 *     e <- fl(v - x^)
 * The class sums are taken in a fixed order (inside a row of 32 elements from the bucket's start a
 * left-to-right chain over the class's members; the rows' sums by a balanced tree of adjacent
 * pairs, leaf count padded with zeros to a power of two), so the result is reproducible bit for bit.
 *   residual [in/out] n floats, 16-byte aligned, updated in place
 *   codes    [out]    mqg_code_words(n, 1) words;  ranges [out] 2 * mqg_num_buckets(n, bucket) floats,
 *                     8-byte aligned.  The server side is the (min, max) variant's with bits = 1.
 * Buckets (or a single bucket n) above 8192 elements are rejected with MQG_ERR_INVALID.
 */
mqg_status mqg_quantize_1bit_ef(const void* grad, float* residual, uint64_t n, uint64_t bucket,
                                uint32_t* codes, float* ranges, mqg_dtype dtype, void* cuda_stream);

/*
 * Codec variant: the bucket's scale is its Euclidean norm, as in the norm-scaled quantizers the
 * related-work section (Section 2) cites, instead of its largest magnitude.  Everything else is
 * mqg_quantize: same encode against [-s, +s], same draws, same packing, and the outputs are
 * consumed by the ordinary server calls (mqg_server_step, mqg_dequant_accumulate,
 * mqg_server_requantize).  Because a float sum depends on its order, the order is fixed:
 *   - the bucket is cut into rows of 32 consecutive elements from its first element; a row's sum
 *     of squares is the chain a <- fma(x_j, x_j, a), left to right, from a = 0;
 *   - the row sums are combined by a balanced binary tree of adjacent pairs (leaf count padded
 *     with zeros to a power of two); S is the root;
 *   - scales[k] = 0 if S < 2^-96 (every code of the bucket is then 0), else sqrt(S) rounded once.
 * The result is therefore reproducible bit for bit, on any device and launch shape.  Inputs whose
 * sum of squares overflows fp32 give unspecified results.
 * Buckets (or a single bucket n) above 8192 elements are rejected with MQG_ERR_INVALID: use the
 * segment form below for those.  Other arguments and errors as mqg_quantize.
 */
mqg_status mqg_quantize_l2(const void* grad, uint64_t n, int bits, uint64_t bucket, uint64_t seed,
                           uint32_t* codes, float* scales, mqg_dtype dtype, uint32_t worker,
                           uint32_t step, uint64_t elem_offset, void* cuda_stream);

/*
 * The L2-norm variant for W workers' gradients of the same shape in ONE launch (the variant's
 * counterpart of mqg_quantize_workers; related-work codec of Section 2, granularity as Section 4.1):
 * worker w's outputs are bit-identical to mqg_quantize_l2 with worker id first_worker + w.
 *   grads / codes / scales   HOST arrays of W DEVICE pointers, each as in mqg_quantize_l2; caller-owned
 * Shapes the batched kernel does not take run as W launches with the same results.
 * Errors as mqg_quantize_l2, plus MQG_ERR_TOO_MANY_WORKERS for W outside 1..MQG_MAX_WORKERS.
 */
mqg_status mqg_quantize_workers_l2(const void* const* grads, int W, uint64_t n, int bits, uint64_t bucket,
                                   uint64_t seed, uint32_t* const* codes, float* const* scales,
                                   mqg_dtype dtype, uint32_t first_worker, uint32_t step,
                                   uint64_t elem_offset, void* cuda_stream);

/*
 * The same variant with one norm per segment (per-layer scale), segment tables as in
 * mqg_quantize_segments below; the outputs go to mqg_server_step_segments.  The rows and the
 * tree of a segment start at the segment's first element.
 *   workspace        [scratch] DEVICE memory for the partial sums: at least
 *                    mqg_l2_workspace_floats(nseg, seg_off) floats (one per 8192 elements of every
 *                    segment, rounded up per segment), 4-byte aligned.  Contents on entry do not
 *                    matter and are undefined on return; calls that may run concurrently on the
 *                    device need separate workspaces.
 *   workspace_floats its size in floats; MQG_ERR_INVALID when too small.
 * The gradient is read twice (sum pass, encode pass).
 */
size_t mqg_l2_workspace_floats(int nseg, const uint64_t* seg_off);
mqg_status mqg_quantize_segments_l2(const void* grad, int nseg, const uint64_t* seg_off,
                                    const uint64_t* code_off, int bits, uint64_t seed,
                                    uint32_t* codes, float* scales, mqg_dtype dtype, uint32_t worker,
                                    uint32_t step, uint64_t elem_offset, float* workspace,
                                    size_t workspace_floats, void* cuda_stream);

/*
 * mqg_quantize_segments_l2 without the workspace argument, for callers that cannot supply device
 * memory of their own: processes whose device memory has all been handed to one pool at start-up
 * (a later allocation fails), latency-critical paths that must not run into the device-wide
 * synchronisation of an allocation, and plug-ins or callbacks whose host only lets them launch
 * work on the buffers they are given.  (The paper has no counterpart: this is a property of the
 * library's interface, not of the method.)  The partial sums go to an array inside the library
 * image instead; arguments, results and errors are otherwise exactly those of
 * mqg_quantize_segments_l2.
 *   - Limit: mqg_l2_workspace_floats(nseg, seg_off) <= MQG_L2_STATIC_WORKSPACE_FLOATS (65,536 partial
 *     sums, one per started 8192 elements of every segment: about 5 * 10^8 elements); beyond it the
 *     call returns MQG_ERR_INVALID, enqueues nothing, and mqg_last_error() names both numbers.
 *   - Cost: the array (256 KiB) occupies device memory on every GPU that loads the library, from
 *     load until the process exits, also if this function is never called.
 *   - The call allocates and frees nothing, on the host or the device.  The first call on each
 *     device looks up the array's device address (once; later calls reuse it); make that first
 *     call before any stream capture begins.
 *   - All calls on a device share the one array, and it keeps what the last call left in it.
 *     Nothing in it needs to be zero on entry (every element read is written earlier in the same
 *     call), but two calls whose kernels can overlap on the device - different streams, or
 *     different host threads on different streams - race on it and corrupt each other's scales:
 *     order them on one stream or with events.
 */
#define MQG_L2_STATIC_WORKSPACE_FLOATS 65536
mqg_status mqg_quantize_segments_l2_static(const void* grad, int nseg, const uint64_t* seg_off,
                                           const uint64_t* code_off, int bits, uint64_t seed,
                                           uint32_t* codes, float* scales, mqg_dtype dtype,
                                           uint32_t worker, uint32_t step, uint64_t elem_offset,
                                           void* cuda_stream);

/*
 * Per-layer scale (Section 4.1 quantizes the two large fully connected layers, each as a whole): the flat
 * gradient is cut into nseg segments; segment j = elements [seg_off[j], seg_off[j+1]) is ONE bucket
 * with scale scales[j], and its bit stream starts on a word boundary at word code_off[j].
 *   seg_off   [in] HOST array of nseg+1 non-decreasing element offsets (seg_off[0] may be > 0)
 *   code_off  [in] HOST array of nseg+1 word offsets; code_off[j+1] - code_off[j] >=
 *                  mqg_code_words(seg_off[j+1] - seg_off[j], bits)
 *   grad      [in] the whole flat gradient (element 0 of the array is flat index 0)
 *   codes     [out] code_off[nseg] words;  scales [out] nseg floats
 * Element i of segment j draws with position elem_offset + seg_off[j] + i.  Empty segments get
 * scale 0.
 * Performance note: a segment of at most 16384 elements is read once, and so are all of a call none of whose segments has
 * more than 65536 (bf16: and at most 16 M elements in all); longer ones are read twice.  They are encoded by the bulk-copy
 * kernels when elem_offset is a multiple of 8 and seg_off[0] one of 64 (or grad + seg_off[j] is 16-byte aligned and
 * elem_offset + seg_off[j] a multiple of 8).  mqg_server_step_segments' bulk-copy kernel applies those of 2^15 elements and
 * more, wherever they start from 2^19 (more than four workers: 2^20) elements in all on.  The results do not depend on
 * which kernel ran.
 */
mqg_status mqg_quantize_segments(const void* grad, int nseg, const uint64_t* seg_off,
                                 const uint64_t* code_off, int bits, uint64_t seed,
                                 uint32_t* codes, float* scales, mqg_dtype dtype, uint32_t worker,
                                 uint32_t step, uint64_t elem_offset, void* cuda_stream);

/*
 * mqg_quantize_segments for W workers' gradients that share one segment table, in three launches for up to 64 segments
 * and 64 (worker, long segment) pairs (short segments whole, max pass and encode pass of the longer ones) - the per-layer
 * counterpart of mqg_quantize_workers, for a host that plays several workers on one device (all
 * workers run Quantize(g, K) with the same K in an iteration; Algorithm 1, WorkerIterate line 3).
 *   grads/codes/scales [in] HOST arrays of W device pointers; worker w draws with worker id
 *                      first_worker + w; codes[w] takes code_off[nseg] words, scales[w] nseg floats
 * Worker w's outputs are bit-identical to mqg_quantize_segments(grads[w], ..., first_worker + w, ...).
 * Errors as mqg_quantize_segments, per worker; MQG_ERR_TOO_MANY_WORKERS for W outside
 * 1..MQG_MAX_WORKERS.
 */
mqg_status mqg_quantize_segments_workers(const void* const* grads, int W, int nseg, const uint64_t* seg_off,
                                         const uint64_t* code_off, int bits, uint64_t seed,
                                         uint32_t* const* codes, float* const* scales, mqg_dtype dtype,
                                         uint32_t first_worker, uint32_t step, uint64_t elem_offset,
                                         void* cuda_stream);

/* mqg_server_step for buffers written by mqg_quantize_segments (same segment tables). */
mqg_status mqg_server_step_segments(const uint32_t* const* codes, const float* const* scales, int W,
                                    int bits, int nseg, const uint64_t* seg_off,
                                    const uint64_t* code_off, float* params, float lr,
                                    float* acc_out, void* cuda_stream);

/*
 * ---- Around the codec: the global gradient norm, clipping, and the table of a model over tokens ----
 *
 * What a trainer needs right before and after the calls above: a worker clips its gradient before Quantize (Algorithm 1,
 * WorkerIterate), the server clips the sum before it applies it, and a model over tokens pulls rows of the shared
 * parameters and pushes their gradient.  The paper leaves both to the system it runs in.
 *
 * A list of gradient tensors is three HOST arrays of `count` entries, read during the call only: device pointers, element
 * counts, types.  A tensor needs its type's own alignment only (4 or 2 bytes); 16 bytes are faster.  An empty tensor's
 * pointer is not looked at, and count may be 0.  What is written (tensors, results, workspaces) must not overlap anything
 * else; of two buffers of a call, or a buffer and a tensor of its list, that do, the call is refused (MQG_ERR_INVALID).  That
 * the tensors of a list that is scaled in place do not overlap each other is the caller's to see to.
 *
 *     N = sqrt(sum over all elements of all tensors of x^2)
 *     c = 1 where N <= max_norm, else max_norm / N
 *
 * N is right for every finite gradient (at most 33 squares, a thread's share of a 16 KB tile, are summed in fp32, 64 bits from
 * there on; no square overflows or vanishes) and rounded to fp32 once (infinity above its range), after c was formed; the order of the sums is fixed by
 * the tensors' sizes, types and addresses modulo 16, so N and c are reproducible bit for bit on one device model.  A
 * NaN among the elements makes N and c NaN; an infinity makes N infinite and c zero (where max_norm is infinite too: c
 * = 1).  max_norm may be 0 or infinite, not negative or NaN (MQG_ERR_INVALID).
 *   result     [out] 2 floats: N, c.  They stay on the device: no call here waits for them.
 *   workspace  [scratch] DEVICE memory of at least mqg_norm_workspace_floats(count) floats, 8-byte aligned.  Contents on
 *              entry do not matter and are undefined on return; calls that may run concurrently (graphs captured apart
 *              among them) need separate workspaces.
 * Errors: MQG_ERR_INVALID (null pointers, unknown types, workspace too small, memory shared as above), MQG_ERR_ALIGN.
 */
size_t mqg_norm_workspace_floats(int count);

/* Measures N and c; the tensors stay as they are. */
mqg_status mqg_grad_norm(const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, float max_norm,
                         float* result, float* workspace, size_t workspace_floats, void* cuda_stream);

/*
 * Measures N and c, and scales every tensor in place: x <- c * x, one rounding to fp32 for the product and, for a bf16 tensor,
 * one to bf16.  Where c is 1 nothing is written.
 */
mqg_status mqg_clip_grad_norm(void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, float max_norm,
                              float* result, float* workspace, size_t workspace_floats, void* cuda_stream);

/*
 * Measures N and c, and writes c * x of all tensors one after another into `flat` (sum of sizes elements of flat_dtype, each
 * rounded as above): the flat gradient that mqg_quantize takes.  The tensors stay as they are; with max_norm infinite it is
 * their concatenation.
 *   flat  [out] needs its type's own alignment (4 or 2 bytes)
 */
mqg_status mqg_clip_flatten(const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count,
                            float max_norm, void* flat, mqg_dtype flat_dtype, float* result, float* workspace,
                            size_t workspace_floats, void* cuda_stream);

/*
 * x <- *factor * x for every tensor of a list, in place, rounded as above; where *factor is 1 nothing is written.
 * For a factor that comes from elsewhere (the norm of gradients that are spread over several devices), and for clipping a
 * gradient that is encoded already: scaling its `scales` (of mqg_quantize and the L2-norm variant) or `ranges` scales what
 * it decodes to.
 *   factor  [in] one float in DEVICE memory, e.g. result + 1 of the calls above
 */
mqg_status mqg_scale_grads(void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, const float* factor,
                           void* cuda_stream);

/*
 * mqg_apply of the clipped sum: params[i] = fma(-lr, fl(*factor * acc[i]), params[i]), exactly mqg_scale_grads on acc
 * followed by mqg_apply, in one pass that leaves acc as it is.  params and acc as in mqg_apply (16-byte aligned); acc may be
 * params itself.
 */
mqg_status mqg_apply_clipped(float* params, const float* acc, float lr, const float* factor, uint64_t n, void* cuda_stream);

typedef enum { MQG_I32 = 0, MQG_I64 = 1 } mqg_index;

/*
 * Rows of a table for a batch of token ids: out[t] = scale * table[ids[t]], one rounding to fp32 for the product and, for a
 * bf16 `out`, one to bf16.  An id outside 0..rows-1 marks an empty place (of a padded batch): its row of `out` is zero.
 *   table  [in] rows x dim elements, row after row; a slice of the flat parameters, for instance
 *   ids    [in] `tokens` integers;  out [out] tokens x dim elements
 * All buffers need their types' own alignment only; rows whose bytes are a multiple of 16 on 16-byte boundaries are fastest.
 * Errors: MQG_ERR_INVALID (null pointers, unknown types; rows or tokens above 2^31 - 1, dim above 2^22; an output or workspace
 * that shares memory with another buffer), MQG_ERR_ALIGN.
 */
mqg_status mqg_embedding(const void* table, mqg_dtype table_dtype, uint64_t rows, uint64_t dim, const void* ids,
                         mqg_index ids_type, uint64_t tokens, float scale, void* out, mqg_dtype out_dtype,
                         void* cuda_stream);

/*
 * The gradient of that table from the gradient of `out`:
 *     grad[v] = scale * sum over t with ids[t] = v of dout[t]            (0 for a row without tokens), or with add_into_grad
 *     grad[v] = grad[v] + scale * that sum                               (rows without tokens are not touched)
 * The tokens are sorted by id and a row's summed in ascending order of t in fp32: one after the other, a row of many tokens
 * from sums of at most 32 each, in their order.  The scale and the addition are one rounding each, and a bf16 `grad` is
 * rounded once at the end.  The order of every sum is fixed by the ids and the arguments' sizes, types and addresses
 * modulo 16: the result is reproducible bit for bit.  What stands in `dout` at empty places is not used, NaN included.
 *   grad       [out] rows x dim elements; with add_into_grad [in/out]
 *   workspace  [scratch] DEVICE memory of at least mqg_embedding_workspace_floats(tokens, rows, dim) floats, 16-byte
 *              aligned; otherwise as for the norm above
 * Other arguments and errors as mqg_embedding.
 */
size_t mqg_embedding_workspace_floats(uint64_t tokens, uint64_t rows, uint64_t dim);
mqg_status mqg_embedding_grad(const void* dout, mqg_dtype dout_dtype, const void* ids, mqg_index ids_type, uint64_t tokens,
                              uint64_t rows, uint64_t dim, float scale, void* grad, mqg_dtype grad_dtype, int add_into_grad,
                              float* workspace, size_t workspace_floats, void* cuda_stream);

/*
 * ---- Beside the codec: AdamW over many tensors, and the layer norm of a model over tokens ----
 *
 * AdamW for the server's shared parameters (or a worker's own), in the place of mqg_apply: decay is decoupled, averages are
 * corrected for their start.  For element x of tensor j, t = step:
 *     k  = grad_scale * *factor                      g  = k * grad
 *     m <- b1 m + (1 - b1) g                         v <- b2 v + ((1 - b2) g) g
 *     p <- p - (lr decay_j p + lr / (1 - b1^t) * (m / (sqrt(v) / sqrt(1 - b2^t) + eps)))
 * in fp32.  For m and v every product and sum is rounded by itself, so that they are the same bits for whoever follows the formulas; for
 * p the root and the quotient are within two units in the last place.  1 - b is formed in 64 bits.  A bf16 parameter is rounded to
 * nearest: changes below 2^-9 of it are lost, so shared parameters are better held in fp32.
 *
 * The lists are HOST arrays of `count` entries, read during the call only: pointers, element counts, types.  A tensor needs its
 * type's own alignment only; multiples of 4 elements from a 16-byte boundary on are faster.  An empty tensor's pointers are not
 * looked at, and count may be 0.  params, m, v and scales must not share memory with each other or anything else, within a list or
 * among them (MQG_ERR_INVALID); tensors of `grads` may.
 *   params      [in/out] fp32 or bf16;  grads [in] fp32 or bf16, each of its own type
 *   m, v        [in/out] the two averages; zeros before the first step
 *   decays      [in] HOST array of `count` floats, or NULL for zeros
 *   lr >= 0; 0 <= b < 1 (in fp32); eps >= 2^-50; decays >= 0; grad_scale finite (1 / P for the mean of P workers); step >= 1
 *   factor      [in] NULL, or one float in DEVICE memory: result + 1 of mqg_grad_norm, for instance.  Where it is NaN, infinite or
 *               0 (a gradient with a NaN or an infinity in it), the call changes nothing.  Without it a NaN or an infinity reaches
 *               its element's parameter and averages, and with averages in 8 bits those of its block.
 *   schedule    [in] NULL, or 4 floats in DEVICE memory that take the place of lr and step: lr, 1 - b1^t, 1 - b2^t, t (a whole
 *               number below 2^24).  For calls that are captured into a graph: the other scalars are those of the capture.
 * Errors: MQG_ERR_INVALID (the above; null pointers, unknown types, 2^42 elements or more), MQG_ERR_ALIGN.
 */
mqg_status mqg_adamw(void* const* params, const mqg_dtype* param_dtypes, const void* const* grads, const mqg_dtype* grad_dtypes,
                     float* const* m, float* const* v, const uint64_t* sizes, const float* decays, int count, double lr,
                     double beta1, double beta2, double eps, uint32_t step, float grad_scale, const float* factor,
                     const float* schedule, void* cuda_stream);

/*
 * The same with m and v in 8 bits each: every block of 256 elements of a tensor, from its first on, has a scale for each.
 *   m       [in/out] a byte an element, a float of 1 + 4 + 3 bits (e4m3, largest 448): its value is e4m3 * scales[2 b]
 *   v       [in/out] a byte an element, a float of 1 + 5 + 2 bits (e5m2, largest 57344), never negative: e5m2 * scales[2 b + 1]
 *           (codes that are infinities or NaN in these formats are that)
 *   scales  [in/out] HOST array of pointers to mqg_adamw8_scale_floats(size) floats per tensor (two to a block), 4-byte aligned
 * All three are zeros before the first step.  The parameter's step is computed from m and v before they are rounded.  Then
 * scales[2 b] = max|m| / 448, scales[2 b + 1] = max v / 57344 of the block, and m * (448 / max|m|), v * (57344 / max v) are rounded to
 * one of their two neighbours at random, up where the share above the lower neighbour plus (h + 1/2) / 2^16 reaches 1: without
 * bias, while rounding to nearest would not move an average whose steps are small beside the distance of two codes.  Only a v of
 * 2^-128 or more that would get code 0 gets code 1 instead.  Where that maximum is below 2^-110, the scale is 0 and the codes are
 * zeros (m's of the sign of m); where it is infinite or a NaN, the scale is that, and the block's values are infinite or NaN.
 *   seed    keys the draws: h has 16 bits of the Philox4x32-10 block with key = seed and counter = (q, 0xFFFFFFFF, step).  q = 32 B +
 *           l, B = blocks before this one in the whole list of the call, draws for the block's elements 4 l .. 4 l + 3 (words 0
 *           and 1, low half first) and 128 + 4 l .. 128 + 4 l + 3 (words 2 and 3); v takes h with its two bytes swapped.  The
 *           result is a pure function of the arguments.
 * Other arguments and errors as mqg_adamw.
 */
size_t mqg_adamw8_scale_floats(uint64_t n);
mqg_status mqg_adamw8(void* const* params, const mqg_dtype* param_dtypes, const void* const* grads, const mqg_dtype* grad_dtypes,
                      uint8_t* const* m, uint8_t* const* v, float* const* scales, const uint64_t* sizes, const float* decays,
                      int count, double lr, double beta1, double beta2, double eps, uint32_t step, uint64_t seed,
                      float grad_scale, const float* factor, const float* schedule, void* cuda_stream);

/*
 * Layer norm over rows of `dim` elements, each by itself:
 *     mu = mean(x)    r = 1 / sqrt(mean((x - mu)^2) + eps)    y = (x - mu) * r * weight + bias
 * in fp32 (the squares are those of the differences, no difference of large sums; the order of the sums is fixed by rows, dim, the
 * types and the addresses modulo 16), rounded once to a bf16 `y`.
 *   x             [in] rows x dim elements, row after row;  y [out] the same, of y_dtype
 *   weight, bias  [in] dim elements of weight_dtype each; NULL = ones, zeros
 *   stats         [out] NULL, or 2 floats to a row: mu, r, as the gradient takes them
 *   eps           above 0.  The rows' sums, their deviations and their squares' sum must be in fp32's range.
 * All buffers need their types' own alignment only; rows whose bytes are a multiple of 16 on 16-byte boundaries are fastest.  What
 * is written must not share memory with anything else (MQG_ERR_INVALID).  A row without elements, or no rows: nothing is done.
 * Errors: MQG_ERR_INVALID (null pointers, unknown types, eps; rows above 2^31 - 1, dim above 2^22), MQG_ERR_ALIGN.
 */
mqg_status mqg_layer_norm(const void* x, mqg_dtype x_dtype, uint64_t rows, uint64_t dim, const void* weight, const void* bias,
                          mqg_dtype weight_dtype, float eps, void* y, mqg_dtype y_dtype, float* stats, void* cuda_stream);

/*
 * Its gradient.  With h = (x - mu) * r and a = weight * dy:
 *     dx = r * (a - mean(a) - h * mean(a h))    dweight = sum over rows of dy * h    dbias = sum over rows of dy
 * Sums over rows are formed in fp32 over the rows that a thread takes, in 64 bits over the threads of a part of the rows, rounded to
 * fp32, and in 64 bits over the parts, in an order that rows, dim and the arguments' types and addresses modulo 16 fix: the result
 * is reproducible bit for bit on one device model.
 *   dy             [in] rows x dim elements;  x, weight, stats [in] as mqg_layer_norm took and wrote them
 *   dx             [out] rows x dim elements of x_dtype, or NULL
 *   dweight, dbias [out] dim elements of dweight_dtype each, or NULL; with add_into_grads the sum over rows is added to what is
 *                  there (in 64 bits, one rounding), without it `rows` = 0 gives zeros
 *   workspace      [scratch] DEVICE memory of at least mqg_layer_norm_workspace_floats(rows, dim) floats, 16-byte aligned; may be
 *                  NULL where dweight and dbias are.  Contents on entry do not matter and are undefined on return; calls that may
 *                  run concurrently (graphs captured apart among them) need separate workspaces.
 * Other arguments and errors as mqg_layer_norm.
 */
size_t mqg_layer_norm_workspace_floats(uint64_t rows, uint64_t dim);
mqg_status mqg_layer_norm_grad(const void* dy, mqg_dtype dy_dtype, const void* x, mqg_dtype x_dtype, uint64_t rows, uint64_t dim,
                               const void* weight, mqg_dtype weight_dtype, const float* stats, void* dx, void* dweight,
                               void* dbias, mqg_dtype dweight_dtype, int add_into_grads, float* workspace,
                               size_t workspace_floats, void* cuda_stream);

/*
 * Kernels stage data through shared memory with asynchronous bulk copies and wait for them on
 * barriers with a bounded number of polls; a wait that runs out makes the kernel record it in a
 * per-device counter, abandon its work and return (its outputs are then incomplete) instead of
 * hanging.  This call synchronises with the current device and stores the number of such events
 * since the library was loaded in *count (0 in a healthy run).  Returns MQG_OK or MQG_ERR_CUDA.
 */
mqg_status mqg_device_timeouts(unsigned int* count);

/*
 * The same counter as a status, for bracketing a step: synchronises with the current device, stores
 * the number of waits that ran out since the library was loaded or since the last call with
 * reset != 0 in *count (count may be NULL), clears the counter if reset != 0, and returns
 * MQG_ERR_TIMEOUT when that number is not zero (the outputs of the calls enqueued on this device
 * since the last clear are then incomplete and the step has to be repeated), else MQG_OK;
 * MQG_ERR_CUDA if the device cannot be read.  The calls themselves are asynchronous and cannot
 * report it: a kernel that gives up has long been enqueued with MQG_OK.  The paper has no
 * counterpart (its transport is a blocking push / pull; Algorithm 1).
 */
mqg_status mqg_check_timeouts(unsigned int* count, int reset);

/*
 * TEST HOOK, process-wide, not for production use: the kernels launched after this call poll a
 * barrier at most poll_limit times (0 restores the default), and with arm_only != 0 they arm their
 * barriers for the bytes of a staging copy but do not issue the copy, so that the wait runs out
 * with nothing in flight, the kernel counts it, drains and returns without writing its outputs.
 * mqg_test_wait_override(0, 0) restores normal operation.  Always returns MQG_OK.
 */
mqg_status mqg_test_wait_override(uint32_t poll_limit, int arm_only);

/*
 * TEST HOOK, process-wide, not for production use: mqg_embedding_grad sorts tokens as on a device that holds no cluster of more
 * than most_ctas CTAs (a power of two up to 16; 1: no cluster at all; 0 restores the default).  The result is the same bit for
 * bit.
 */
mqg_status mqg_test_sort_cluster(uint32_t most_ctas);

/* Message of the last error returned to the calling thread ("" if none).  Never NULL. */
const char* mqg_last_error(void);

/* Library version, major * 10000 + minor * 100 + patch. */
int mqg_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MQGRAD_H_ */
