/*
 * neuzip.h -- C ABI of the MI355X (gfx950) NeuZip codec library.
 *
 * What the library does (NeuZip, arXiv 2410.20650): a bf16 weight tensor is
 * split into its exponent bytes and a packed sign|mantissa stream (Alg. 1
 * "split"; App. D), the low-entropy exponents are entropy-coded with an
 * asymmetric numeral system (Sec. 2.2 "Compression algorithm"), and the
 * tensor is rebuilt bit-exactly into caller-provided temporary space right
 * before a layer uses it (Sec. 2.2 Eq. (3); Alg. 1 "decompression"/"merge").
 * The lossy inference variant keeps only the k leading mantissa bits
 * (Sec. 2.3), k in {3, 1, 0}.
 *
 * Conventions for every entry point
 *   - d_* arguments are DEVICE pointers owned by the caller, h_* arguments are
 *     HOST pointers owned by the caller.  Nothing is retained after the call's
 *     stream work has completed.
 *   - hip_stream is a hipStream_t passed as void* (NULL = the default stream).
 *     All kernels and copies of a call are enqueued on it.
 *   - Tensors are flat, contiguous arrays of n_elems 16-bit words (32-bit
 *     words for NEUZIP_F32); the shape of the matrix is irrelevant to the
 *     codec.  d_src / d_dst must be aligned to 16 bytes.  n_elems must be
 *     below 2^32.
 *   - A compress, recompress or update call waits for the lengths of the streams, which depend on the
 *     data, and returns while its last kernels, which complete the blobs, may still run on hip_stream.
 *     The caller's buffers are done with by then: sources have been read, new weights written.
 *     The calls of this library that read such a blob are ordered behind them, on the same stream by
 *     its own order, on another one by an event that the library makes that stream wait for (the host
 *     does not wait).  A stream under capture is not made to wait: a blob that was filled on another
 *     stream has to be complete before a capture that reads it begins.  The other direction is the
 *     caller's: a blob is not compressed into, or freed, while calls on other streams still read it.
 *   - Errors are reported through the return code only (no exceptions, no
 *     aborts, nothing is printed).  On error no output argument is modified
 *     unless stated otherwise.
 *   - If a call that compresses into an existing blob fails after its kernels
 *     have started (out of memory while growing the stream, a HIP error), that
 *     blob holds no tensor any more: decompress, linear, update, recompress and
 *     export return NEUZIP_EINVAL for it until a compress call has succeeded.
 *   - A blob belongs to the device that was current when it was created; every
 *     call that launches work on it must be made with that device current
 *     (NEUZIP_EINVAL otherwise).  neuzip_free may be called from any device.
 *   - Calls that touch different blobs may run concurrently from different
 *     host threads; compress calls are serialised inside the library because
 *     they share one per-device workspace.
 */
#ifndef NEUZIP_H
#define NEUZIP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Opaque handle of one compressed tensor.  The library owns the device memory
 * behind it until neuzip_free. */
typedef struct neuzip_blob neuzip_blob;

/* Element types.  The paper works on BFloat16 only (Sec. 2.1, footnote); the other two go beyond it.
 * NEUZIP_F32: the upper half of an IEEE binary32 word is a bf16 word (sign, the same 8 exponent
 * bits, 7 mantissa bits) and is compressed exactly as one; the lower half, 16 mantissa bits without
 * structure, is kept as a raw plane after the sign|mantissa stream.
 * NEUZIP_F16: IEEE binary16 (sign, 5 exponent bits, 10 mantissa bits); the upper byte of a word
 * (sign, exponent, two mantissa bits) is the entropy-coded symbol in place of the bf16 exponent
 * byte, the lower byte is stored in place of the sign|mantissa byte.
 * Both are lossless only: mantissa_bits must be 7 and there is no block-wise normalisation
 * (EUNSUPPORTED / EINVAL otherwise).  Header word 56 of the container holds the element type.
 * neuzip_compress, _batch, _guarded, neuzip_recompress, the three decompress calls, export and
 * import take such tensors; neuzip_linear and neuzip_update do not (EUNSUPPORTED). */
enum { NEUZIP_BF16 = 0, NEUZIP_F32 = 1, NEUZIP_F16 = 2 };

enum {
    NEUZIP_OK = 0,
    NEUZIP_EINVAL = -1,       /* bad argument (null pointer, misaligned, wrong n/dtype/mantissa_bits) */
    NEUZIP_ENOMEM = -2,       /* device or host allocation failed, or h_buf too small */
    NEUZIP_EHIP = -3,         /* a HIP runtime call failed; see neuzip_last_hip_error() */
    NEUZIP_ECORRUPT = -4,     /* a container or a decoded stream is not well formed */
    NEUZIP_EUNSUPPORTED = -5  /* a size, or a combination of element type and option, that is not supported */
};

/* Format constants of the stream (mirrored in every container header). */
enum {
    NEUZIP_PROB_BITS = 12,        /* frequencies sum to 2^12 */
    NEUZIP_CHUNK = 4096,          /* exponent symbols per independently decodable chunk */
    NEUZIP_STATES_PER_CHUNK = 16, /* rANS states per chunk, each with a private word run */
    NEUZIP_RUN = 8                /* consecutive symbols one state codes per turn */
};

/*
 * neuzip_compress -- Alg. 1 initialisation loop and the re-compression after a
 * weight update ("split", "compression", "store"); Sec. 2.3 for k < 7.
 *
 *   d_src          n_elems bf16 words on the device (read only).
 *   dtype          NEUZIP_BF16, or NEUZIP_F32 / NEUZIP_F16 (n_elems words of that type; see the element types).
 *   mantissa_bits  7 = lossless; 3, 1 or 0 = keep that many leading mantissa
 *                  bits, truncating toward zero.
 *   blob           in/out.  *blob == NULL: a new blob is created.  Otherwise
 *                  *blob must be a blob of this library with the same n_elems
 *                  and mantissa_bits; its device memory is reused (and grown
 *                  if the new stream is longer), its old content is lost, and it
 *                  keeps the guard band it was made with (neuzip_compress_guarded).
 *
 * Builds the exponent histogram, the 12-bit frequency table, encodes every
 * 4096-symbol chunk with 16 rANS states, and stores exponent stream and
 * sign|mantissa stream in device memory sized for this tensor (the word
 * section with 1/64 of headroom, 0.3 % of the container, so that a blob which
 * is compressed into again after an update seldom has to be re-allocated).
 * The host waits once, for the stream's length; the blob is complete in the order of hip_stream (see
 * the conventions).
 * n_elems == 0 yields a valid empty blob.
 */
int neuzip_compress(const void *d_src, uint64_t n_elems, int dtype, int mantissa_bits,
                    void *hip_stream, neuzip_blob **blob);

/*
 * neuzip_compress_blockwise -- the lossy variant with block-wise normalisation (Sec. 2.3, last
 * paragraph; block sizes as in the block-size study of Sec. 3).
 *
 *   block_size     0 (same as neuzip_compress) or 32, 64, 128, 256, 512 consecutive weights.
 *   mantissa_bits  3, 1 or 0 when block_size != 0 (7 -> EINVAL: normalisation is lossy).
 *
 * Reading of the paper taken here: the coefficient of a block is the 7-bit mantissa of its
 * largest-magnitude weight (first one on ties), stored in one byte per block; with
 * c = 1 + coef/128 every weight is stored as bf16(w / c) before truncation and is returned as
 * bf16(stored * c), both rounded to nearest even in IEEE binary32.  The largest weight of each
 * block is reproduced exactly.  Everything else is as for neuzip_compress; neuzip_decompress
 * and the other entry points recognise such blobs by themselves.
 */
int neuzip_compress_blockwise(const void *d_src, uint64_t n_elems, int dtype, int mantissa_bits,
                              uint32_t block_size, void *hip_stream, neuzip_blob **blob);

/*
 * neuzip_compress_batch -- the same compression (Alg. 1 backward loop: "split", "compression",
 * "store" for every weight of a layer after its update) for several tensors at once: each
 * kernel of the pipeline runs once per group of up to 8 tensors and the host waits once per
 * group, so small tensors overlap with the others.
 *
 *   d_srcs, n_elems  host arrays of count entries: device pointer (16-byte aligned) and element
 *                    count of each tensor.
 *   mantissa_bits, block_size   shared by all tensors; meaning as above.
 *   blobs            host array of count handles, in/out with the rules of neuzip_compress
 *                    (NULL entries are created; other entries must match and be distinct).
 * A group whose encoder slots would exceed the workspace limit (neuzip_set_workspace_limit) is
 * taken in parts, with one wait per part; the results are the same.
 * On error, blobs created for the failing group are released and its entries of blobs are
 * not changed; groups completed before keep their results.
 */
int neuzip_compress_batch(const void *const *d_srcs, const uint64_t *n_elems, uint32_t count, int dtype,
                          int mantissa_bits, uint32_t block_size, void *hip_stream, neuzip_blob **blobs);

/*
 * neuzip_compress_guarded / neuzip_recompress -- Alg. 1 backward loop: every weight is compressed
 * again right after its update ("compression", "store"), i.e. once per tensor per training step.
 * The exponent statistics hardly move from one step to the next, so the table of the step before
 * can code the updated tensor, and the pass that counts exponents (one of the two reads of the
 * tensor) can be left out.  Not described in the paper; the reading taken here:
 *
 *   neuzip_compress_guarded   as neuzip_compress_batch without normalisation, but the table gives
 *       f = 1 to every exponent up to `guard` (0..255) below the smallest and above the largest
 *       one that occurs, and to exponent 0 (an update w - lr * g cancels exactly to +-0 now and
 *       then), so that values an update newly produces still have a code.  guard = 0 is the
 *       plain table.  The guard is kept in the blob and in header word 52 of the container.  For
 *       NEUZIP_F16 the band is taken on the coded symbol, the word's upper byte (sign, exponent, two
 *       mantissa bits): byte values up to `guard` below the smallest and above the largest one that
 *       occurs, and byte 0.
 *   neuzip_recompress         blobs[i] (which must hold a compressed tensor) receives d_srcs[i],
 *       a tensor of neuzip_elems(blobs[i]) words, coded with the table the blob already holds:
 *       one pass over the source that splits, packs and encodes.  If a tensor holds an exponent
 *       its table has no room for, that tensor is compressed afresh (statistics, new table with
 *       the blob's guard) and rebuilt[i] is set to 1, else 0 (rebuilt may be NULL).  Block-wise
 *       normalised blobs always take the second route.  After a table has been reused
 *       neuzip_histogram reports EINVAL for the blob (no counts were taken).
 *   Both work on host arrays of count entries like neuzip_compress_batch, and the host waits
 *   once per group of up to 8 tensors.  A caller that wants a fresh table every N steps
 *   calls neuzip_compress_guarded then.
 */
int neuzip_compress_guarded(const void *const *d_srcs, const uint64_t *n_elems, uint32_t count, int dtype,
                            int mantissa_bits, uint32_t guard, void *hip_stream, neuzip_blob **blobs);
int neuzip_recompress(const void *const *d_srcs, uint32_t count, void *hip_stream, neuzip_blob *const *blobs,
                      uint32_t *rebuilt);

/*
 * neuzip_update -- the backward loop of Alg. 1 for the weights of a layer: each weight is
 * decompressed into temporary space, the optimiser step is applied, and the weight is compressed
 * again ("decompression", "merge", the update, "split", "compression", "store"); Sec. 2.2 applies
 * vanilla SGD layer by layer during the backward pass, so that neither the full set of gradients
 * nor an uncompressed model ever exists:
 *     W_hat <- decompress(c);   W_hat <- W_hat - lr * grad;   c <- compress(W_hat)
 *
 *   blobs       host array of count blobs holding lossless bf16 weights (mantissa_bits 7, no
 *               normalisation; anything else -> EUNSUPPORTED), distinct; they receive the new weights.
 *   d_grads     host array of count device pointers: the gradient of each weight, bf16 words,
 *               neuzip_elems(blobs[i]) of them, 16-byte aligned (read only).
 *   d_weights   host array of count device pointers, 16-byte aligned: temporary space of
 *               neuzip_elems(blobs[i]) bf16 words each, overlapping neither one another nor the
 *               gradients; on return it holds the new weights uncompressed (the caller may use
 *               or discard them; but see weights_ready = 2).
 *   lr          learning rate.
 *   weights_ready  NEUZIP_UPDATE_FROM_BLOB (0): the library decompresses blobs[i] itself.
 *               NEUZIP_UPDATE_WEIGHTS_READY (1): d_weights[i] already holds exactly
 *               decompress(blobs[i]) -- the backward pass has just decompressed the weight for the
 *               input gradient -- and that pass is skipped.  NEUZIP_UPDATE_WEIGHTS_READY_DISCARD (2):
 *               the same, and the caller has no use for the new weights uncompressed: they are
 *               not written back (a third less memory traffic), and d_weights[i] afterwards holds
 *               the old weight, or the new one for a tensor whose table was rebuilt.
 *               NEUZIP_UPDATE_FROM_BLOB_DISCARD (3): as 0, but d_weights is mere scratch space
 *               whose content afterwards is as for 2 (the library decompresses into it and then
 *               proceeds as for 2, which moves fewer bytes than 0).
 *   rebuilt     as for neuzip_recompress; may be NULL.
 * Reading taken for the arithmetic, which the paper leaves open: per element, in IEEE binary32,
 * the product lr * g and then the difference w - (lr * g) are each rounded to nearest (no fused
 * multiply-add), and the result is rounded to the nearest bf16, ties to even; a NaN result is
 * stored as 0x7FC0.  With weights_ready = 0 the decoder applies the step on its way out (the old
 * weight is never written) and the new weight is then coded as by neuzip_recompress; otherwise the
 * one-pass encoder of neuzip_recompress reads weight and gradient, forms the new weight, writes it
 * back to d_weights and codes it.  Either way the table the blob holds is used, with the fallback
 * to fresh statistics.  The host waits once per group of up to 8 weights.
 */
enum {
    NEUZIP_UPDATE_FROM_BLOB = 0,
    NEUZIP_UPDATE_WEIGHTS_READY = 1,
    NEUZIP_UPDATE_WEIGHTS_READY_DISCARD = 2,
    NEUZIP_UPDATE_FROM_BLOB_DISCARD = 3
};
int neuzip_update(neuzip_blob *const *blobs, const void *const *d_grads, void *const *d_weights, uint32_t count,
                  float lr, int weights_ready, void *hip_stream, uint32_t *rebuilt);

/*
 * neuzip_decompress -- Sec. 2.2 Eq. (3), Alg. 1 "decompression" + "merge":
 * decodes the exponents and reassembles bf16 words into the caller's
 * temporary space in one fused kernel.
 *
 *   d_dst    room for n_elems words of the blob's element type on the device, 16-byte aligned.
 *   n_elems, dtype must equal what the blob was made from (else EINVAL).
 *
 * Never allocates, never synchronises.  For mantissa_bits < 7 the dropped
 * mantissa bits come back as zeros.  A malformed stream is detected on the
 * device and reported by the next neuzip_check on this blob.
 */
int neuzip_decompress(const neuzip_blob *blob, void *d_dst, uint64_t n_elems, int dtype,
                      void *hip_stream);

/*
 * neuzip_decompress_sequence -- the per-layer schedule of Sec. 2.2 / Alg. 1
 * forward loop: every blob, in the given order, is decompressed into the same
 * temporary space on hip_stream, so that the whole model is never held
 * uncompressed.
 *
 *   blobs          host array of count blob handles.
 *   d_scratch      device buffer of scratch_elems bf16 words (2 * scratch_elems bytes), 16-byte
 *                  aligned; must hold the largest tensor, a binary32 blob counting two words
 *                  per element (else EINVAL, nothing is run).
 *   h_offsets      NULL, or a host array of count entries that receives where each tensor goes:
 *                  its first 16-bit word's index in the space.
 * Neighbouring blobs of one kind (element type, mantissa_bits, normalisation) that fit the space
 * together -- the projections of a layer, say -- are placed one behind the other, each at a
 * 256-byte boundary, and share one launch (at most 8 per launch), so that tensors too small to
 * fill the GPU on their own overlap; the next group starts at the front of the space again and
 * overwrites it.  When the call's work has run, the tensors of the last group are what the space
 * holds.  A caller that consumes the weights between the groups issues one call per layer.
 * Never allocates, never synchronises.
 */
int neuzip_decompress_sequence(const neuzip_blob *const *blobs, uint32_t count, void *d_scratch,
                               uint64_t scratch_elems, uint64_t *h_offsets, void *hip_stream);

/*
 * neuzip_decompress_batch -- Sec. 2.2 Eq. (3) / Alg. 1 "decompression" + "merge" for the
 * weights that a layer uses together (e.g. q, k, v, o, gate, up, down): blob i is
 * decompressed to d_dsts[i], all in as few launches as possible, so that tensors too small
 * to fill the GPU on their own overlap with the others.
 *
 *   blobs, d_dsts  host arrays of count entries; d_dsts[i] is a device buffer of
 *                  neuzip_elems(blobs[i]) words of the blob's element type, 16-byte aligned, not overlapping any
 *                  other destination.
 * Tensors are grouped by mantissa_bits (one launch per group of up to 8).  Never allocates,
 * never synchronises.  On EINVAL nothing has been launched.
 */
int neuzip_decompress_batch(const neuzip_blob *const *blobs, void *const *d_dsts, uint32_t count,
                            void *hip_stream);

/*
 * neuzip_linear -- the compressed forward pass of a linear layer, Sec. 2.2:
 *     W_hat <- decompress(c_l);   x_l <- W_hat x_{l-1} + b_l
 * as one fused kernel: the decoded weights go from the decoder's registers straight into the
 * matrix cores and W_hat is never written to memory.
 *
 *   weight        blob of a row-major out_features x in_features bf16 matrix (any mantissa_bits,
 *                 with or without block-wise normalisation; other element types ->
 *                 EUNSUPPORTED).  in_features must be a multiple of 128 and out_features *
 *                 in_features must equal neuzip_elems(weight).
 *   d_x           tokens x in_features bf16 activations, row-major, 16-byte aligned.
 *   tokens        at least 1.  The kernel holds the partial sums of up to 64 tokens; a larger
 *                 batch goes through in tiles of 64, each of which decodes the weight again (for
 *                 more than a few tiles, decompressing once and a dense GEMM is the faster way).
 *   d_bias        out_features floats on the device, or NULL.
 *   d_y           tokens x out_features floats, row-major; overwritten.
 * Products are exact, sums are accumulated in float32 by the matrix cores and, across the pieces
 * of a row, by float atomics, so the last bits can differ from run to run.  Never allocates,
 * never synchronises; a malformed stream is reported by neuzip_check as for neuzip_decompress.
 */
int neuzip_linear(const neuzip_blob *weight, uint64_t out_features, uint64_t in_features, const void *d_x,
                  uint32_t tokens, const float *d_bias, float *d_y, void *hip_stream);

/*
 * neuzip_linear_batch -- the same compressed forward pass (Sec. 2.2) for several weights that are
 * applied to the same activations, such as the q, k and v projections of an attention block or the
 * gate and up projections of an MLP: y_i <- W_hat_i x + b_i for i < count in one launch, so that
 * weights too small to fill the GPU on their own overlap with the others.
 *
 *   weights, out_features, d_y   host arrays of count entries (count at most 4, else EINVAL); weight i is
 *                 out_features[i] x in_features, d_y[i] receives tokens x out_features[i] floats.
 *                 All weights have the same mantissa_bits and are either all block-wise normalised
 *                 or none is (else EINVAL).
 *   d_bias        NULL (no biases), or a host array of count device pointers, each NULL or
 *                 out_features[i] floats.
 *   in_features, d_x, tokens     as for neuzip_linear; the activations are shared.
 * Otherwise as neuzip_linear (which is this call with count = 1).  On EINVAL nothing has been launched.
 */
int neuzip_linear_batch(const neuzip_blob *const *weights, const uint64_t *out_features, uint32_t count,
                        uint64_t in_features, const void *d_x, uint32_t tokens, const float *const *d_bias,
                        float *const *d_y, void *hip_stream);

/*
 * neuzip_linear_batch_scratch -- the same with scratch memory of the caller's, which serves for two things.
 * From 17 tokens on, most calls first lay the activations out there in the order in which the kernel reads them,
 * which makes a call on 64 tokens a third faster.  From 8 tokens on, calls whose rows end inside chunks in many
 * places store the sums of pieces of rows there (a piece lies inside one chunk or half of one) and add them up in a
 * launch of their own.
 *
 *   d_scratch      device buffer of scratch_bytes bytes, 16-byte aligned (else EINVAL), in use until the call's
 *                  work has run; or NULL.  With less than neuzip_linear_scratch_bytes() bytes the call is
 *                  neuzip_linear_batch.
 */
int neuzip_linear_batch_scratch(const neuzip_blob *const *weights, const uint64_t *out_features, uint32_t count,
                                uint64_t in_features, const void *d_x, uint32_t tokens, const float *const *d_bias,
                                float *const *d_y, void *d_scratch, uint64_t scratch_bytes, void *hip_stream);

/* The scratch memory that the call above makes use of, in bytes; 0 where it needs none.  At most the activations', their
 * last 64 tokens or fewer rounded up to a multiple of 4, and for every weight that of out_features * (in_features /
 * 2048 + 1) + 1 sums of min(tokens, 64) tokens, rounded up like that, of 4 bytes each: in_features / 2048 + 1 results
 * (14.6 for rows of 27776). */
uint64_t neuzip_linear_scratch_bytes(const uint64_t *out_features, uint32_t count, uint64_t in_features, uint32_t tokens);

/*
 * neuzip_embedding -- the rows of a compressed embedding table that a call's tokens name, scaled, straight from the blob: the
 * chunks they lie in are decoded, and nothing else.  (Sec. 2.2's compressed forward pass for the layer that is a lookup.)
 *     out[i] <- bf16(scale * W_hat[token[i]])
 *
 *   table      blob of a row-major rows x features bf16 matrix (any mantissa_bits, with or without block-wise normalisation;
 *              other element types -> EUNSUPPORTED).  features must be a multiple of 8, rows * features = neuzip_elems(table).
 *   d_tokens   count row numbers, 64-bit integers.  A number outside 0 .. rows - 1 names no row (padding): its output is zeros.
 *   scale      the product is formed in binary32 and rounded once, to nearest even; with scale = 1 every word leaves as it is.
 *   d_out      count x features bf16 words, row-major, 16-byte aligned; overwritten.
 * count = 0 is a call that does nothing.  Never allocates, never synchronises; a malformed stream is reported by neuzip_check
 * where a row ends with its chunk.  2^27 pieces of rows and more (a piece lies in one chunk, or half of one) -> EUNSUPPORTED.
 */
int neuzip_embedding(const neuzip_blob *table, uint64_t rows, uint64_t features, const int64_t *d_tokens, uint64_t count, float scale,
                     void *d_out, void *hip_stream);

/*
 * neuzip_embedding_grad -- the gradient of such a table: every row of it, as neuzip_update takes it.
 *     grad[r] <- bf16(scale * sum of grad_out[i] over the i with token[i] = r)
 *
 *   d_tokens, count, scale   as the lookup had them; a token that names no row takes no part.
 *   d_grad_out  count x features bf16 words, 16-byte aligned.
 *   rows, features   as above, rows * features below 2^32.
 *   d_grad      rows x features bf16 words, 16-byte aligned; overwritten, rows without tokens by zeros.
 *   d_scratch   device buffer of scratch_bytes bytes, at least neuzip_embedding_grad_scratch_bytes(), 16-byte aligned, in use until
 *               the call's work has run (NULL where that is 0).
 * The sums are held in binary32 and formed in an order that depends on the tokens alone, so that a call's result is the same every
 * time; scaled and rounded once.  Never allocates, never synchronises.  More than 268431360 tokens (65535 runs of 4096) or rows of more
 * than 134215680 features -> EUNSUPPORTED.
 */
int neuzip_embedding_grad(const int64_t *d_tokens, uint64_t count, const void *d_grad_out, uint64_t rows, uint64_t features, float scale,
                          void *d_grad, void *d_scratch, uint64_t scratch_bytes, void *hip_stream);
uint64_t neuzip_embedding_grad_scratch_bytes(uint64_t count, uint64_t rows, uint64_t features);

/* The activation of a gated feed-forward block: g / (1 + exp(-g)), or 0.5 g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))). */
enum { NEUZIP_SILU = 0, NEUZIP_GELU_TANH = 1 };

/*
 * neuzip_gated_linear -- the first half of a gated feed-forward block straight from its two compressed weights, for a decoding
 * batch:   h <- bf16(act(W_hat_gate x) * (W_hat_up x))
 *
 *   gate, up    blobs of out_features x in_features matrices, with the rules of neuzip_linear_batch.
 *   d_x, tokens, in_features   as for neuzip_linear.
 *   d_h         tokens x out_features bf16 words, row-major; overwritten.
 *   d_scratch   device buffer of scratch_bytes bytes, at least neuzip_gated_linear_scratch_bytes(), 16-byte aligned, in use until
 *               the call's work has run.
 * The two sums, the activation and the product are binary32; h is rounded once.  The sums are neuzip_linear's, whose last bits can
 * differ from run to run.  Never allocates, never synchronises.
 */
int neuzip_gated_linear(const neuzip_blob *gate, const neuzip_blob *up, uint64_t out_features, uint64_t in_features, const void *d_x,
                        uint32_t tokens, int activation, void *d_h, void *d_scratch, uint64_t scratch_bytes, void *hip_stream);
uint64_t neuzip_gated_linear_scratch_bytes(uint64_t out_features, uint64_t in_features, uint32_t tokens);

/*
 * neuzip_gated_forward / neuzip_gated_backward -- the same on weights that have been decompressed into temporary space (Alg. 1:
 * a training batch, or a prompt), with its backward pass.
 *     g <- x W_gate^T,  u <- x W_up^T,  h <- bf16(act(g) * u)
 *     dg <- dh * u * act'(g),  du <- dh * act(g);   dx <- dg W_gate + du W_up,  dW_gate <- dg^T x,  dW_up <- du^T x
 *
 *   d_x               tokens x in_features bf16 words, row-major, like all matrices here.
 *   d_gate_weight, d_up_weight   out_features x in_features bf16 words.
 *   in_features, out_features    multiples of 8, at most 2^22; tokens below 2^31, also 0; tokens x features from about 2^35 on -> EUNSUPPORTED.
 *   d_h               tokens x out_features bf16 words; overwritten.
 *   d_gate, d_up      NULL, or room for g and u (floats, as many as d_h has words), which the backward pass takes; both or neither.
 *   d_grad_h          tokens x out_features bf16 words.
 *   d_grad_x          tokens x in_features bf16 words, or NULL: not wanted.
 *   d_grad_gate_weight, d_grad_up_weight   out_features x in_features bf16 words each, as neuzip_update takes them; or both NULL: not
 *                     wanted.  (No tokens: zeros.)
 *   d_scratch         device buffer of scratch_bytes bytes, at least neuzip_gated_backward_scratch_bytes(), in use until the call's
 *                     work has run.
 * All pointers are aligned to 16 bytes.  Products are exact, sums binary32; h and the three gradients are rounded once, to nearest
 * even, and so are dg and du, which the matrix cores take as bf16.  Results do not change from run to run; the order that dx is summed
 * in is another where it is asked for alone.  Never allocates, never synchronises.
 */
int neuzip_gated_forward(const void *d_x, const void *d_gate_weight, const void *d_up_weight, uint64_t tokens, uint64_t out_features,
                         uint64_t in_features, int activation, void *d_h, float *d_gate, float *d_up, void *hip_stream);
int neuzip_gated_backward(const void *d_x, const void *d_gate_weight, const void *d_up_weight, const float *d_gate, const float *d_up,
                          const void *d_grad_h, uint64_t tokens, uint64_t out_features, uint64_t in_features, int activation,
                          void *d_grad_x, void *d_grad_gate_weight, void *d_grad_up_weight, void *d_scratch, uint64_t scratch_bytes,
                          void *hip_stream);
uint64_t neuzip_gated_backward_scratch_bytes(uint64_t tokens, uint64_t out_features, uint64_t in_features);

/*
 * neuzip_linear_adapters -- neuzip_linear with the low-rank adapter of each token's request beside it (fine-tuned variants of one
 * compressed model, served together):
 *     y[t] <- W_hat x[t] + b + scale[a] * B[a] (A[a] x[t]),   a = id[t]
 *
 *   weight, out_features, in_features, d_x, tokens, d_bias, d_y   as for neuzip_linear; tokens at most 65535 (else EUNSUPPORTED).
 *   d_a, d_b    adapters x rank x in_features and adapters x out_features x rank bf16 words, 16-byte aligned.  rank: a multiple of 8,
 *               at most 512 (a smaller one is filled up with zeros).
 *   d_scales    `adapters` floats, or NULL: 1.
 *   d_ids       the adapter of each token, 32-bit integers; outside 0 .. adapters - 1: the token has none.
 *   d_scratch   device buffer of scratch_bytes bytes, at least neuzip_linear_adapters_scratch_bytes(), 16-byte aligned, in use until
 *               the call's work has run.
 * The low products A x and all sums are binary32; W_hat x is neuzip_linear's, whose last bits can differ from run to run.  As there, more
 * than 64 tokens decode the weight once for every 64.  Never allocates, never synchronises.
 */
int neuzip_linear_adapters(const neuzip_blob *weight, uint64_t out_features, uint64_t in_features, const void *d_x, uint32_t tokens,
                           const float *d_bias, const void *d_a, const void *d_b, uint32_t rank, uint32_t adapters,
                           const float *d_scales, const int32_t *d_ids, float *d_y, void *d_scratch, uint64_t scratch_bytes,
                           void *hip_stream);
uint64_t neuzip_linear_adapters_scratch_bytes(uint64_t out_features, uint64_t in_features, uint32_t tokens, uint32_t rank);

/*
 * neuzip_norm -- what stands between two layers of a model: the layer's result is added to the stream, and the next layer takes the
 * stream's rows divided by their root mean square.
 *     total <- T(x + residual),   y <- bf16(total / sqrt(mean(total^2) + eps) * weight)
 *
 *   d_x         tokens x width values of x_type (NEUZIP_BF16, or NEUZIP_F32: what neuzip_linear leaves), row-major.
 *   d_residual, d_total   the stream before and after, tokens x width values of total_type (T); d_total may be d_residual.  Both NULL:
 *               there is no stream yet, total is x itself (and total_type is x_type).
 *   d_weight    width floats.
 *   width       a multiple of 8, at most 16384 (else EINVAL).  eps at least 0.
 *   d_y         tokens x width bf16 words, what the linear layers take; overwritten.
 * The sum x + residual is rounded once, to T, and the norm is that of the rounded values, which the backward pass is given; squares,
 * sums and products are binary32, y is rounded once.  All pointers aligned to 16 bytes.  tokens = 0 does nothing; 2^24 tokens and more ->
 * EUNSUPPORTED.  Results do not change from run to run.  Never allocates, never synchronises.
 */
int neuzip_norm(const void *d_x, int x_type, const void *d_residual, void *d_total, int total_type, const float *d_weight, uint64_t tokens,
                uint64_t width, float eps, void *d_y, void *hip_stream);

/*
 * neuzip_norm_backward -- its gradients.  With n = 1 / sqrt(mean(total^2) + eps) of a token and g = grad_y * weight:
 *     grad_x <- bf16(grad_total + n * (g - total * n^2 * mean(g * total))),   grad_weight <- sum over the tokens of grad_y * total * n
 *
 *   d_total, total_type   the stream as neuzip_norm left it (its x, where there was no stream).
 *   d_grad_y    tokens x width bf16 words.
 *   d_grad_total   tokens x width bf16 words, the gradient that comes back along the stream; NULL: none does.
 *   d_grad_x    tokens x width bf16 words, the gradient of x and of residual, which is one; may be d_grad_y or d_grad_total; NULL: not wanted.
 *   d_grad_weight   width floats; overwritten (no tokens: zeros); NULL: not wanted.
 *   d_scratch   device buffer of scratch_bytes bytes, at least neuzip_norm_backward_scratch_bytes(), 16-byte aligned, in use until the
 *               call's work has run; only where d_grad_weight is wanted (else NULL will do).
 * Otherwise as neuzip_norm.  The sums over the tokens are formed in an order that depends on tokens and width alone.
 */
int neuzip_norm_backward(const void *d_total, int total_type, const float *d_weight, const void *d_grad_y, const void *d_grad_total,
                         uint64_t tokens, uint64_t width, float eps, void *d_grad_x, float *d_grad_weight, void *d_scratch,
                         uint64_t scratch_bytes, void *hip_stream);
uint64_t neuzip_norm_backward_scratch_bytes(uint64_t tokens, uint64_t width);

/*
 * The cache of the keys and values that attention looks back at, in 8 bits: pages of page_tokens tokens, a scale for each page and head.
 * Element types and order are what the attention kernels read without rearranging: keys token by token, values feature by feature.
 *
 *   d_k         pages x heads x page_tokens x head_dim bytes in e4m3 (4 bits of exponent, 3 of mantissa, largest 448, no infinity).
 *   d_v         pages x heads x head_dim x page_tokens bytes, likewise.
 *   d_k_scales, d_v_scales   pages x heads floats, powers of two: a byte stands for its value times its page's and head's scale.
 *               From 2^-100, the least that neuzip_cache_append sets, to 2^119, so that 448 times it is a bf16 number, which the attention takes bytes as.
 *               (neuzip_cache_append sets 2^120 for a page and head with numbers beyond 1.75 * 2^127, of which bytes of 256 and more are infinite then.)
 *   heads, head_dim, page_tokens   head_dim 64 or 128, page_tokens 16, 32, 64 or 128 (else EINVAL).
 * d_k and d_v are aligned to 16 bytes.  A new cache needs no filling: what no token was put to is not read for its value.
 */
typedef struct {
    void *d_k, *d_v;
    float *d_k_scales, *d_v_scales;
    uint32_t pages, heads, head_dim, page_tokens;
} neuzip_cache;

/*
 * The sequences of a call, ragged: sequence s has the rows d_starts[s] .. d_starts[s + 1] - 1 of the call's tensors, its newest tokens, and with
 * them d_lengths[s] tokens in all; token p of it is in page d_table[s * table_width + p / page_tokens] of the cache, at p % page_tokens.
 *
 *   d_starts    count + 1 32-bit integers, not negative, ascending, up to the tensors' rows.  Rows from d_starts[count] on belong to nobody (a padded batch): they are not
 *               read, and what they are in an output stays as it is.
 *   d_lengths   count 32-bit integers.  A sequence with fewer tokens than rows, or with more than table_width * page_tokens, is left out: nothing
 *               of it is appended, its rows of an attention's output are zeros.
 *   d_table     count x table_width 32-bit integers.  A number outside 0 .. pages - 1 names no page: nothing is put there, and its tokens
 *               are not seen.  (With a window, pages that no token sees any more may be given back.)
 * All three are read on the device when the call's work runs, so that a captured graph follows them.  Several sequences may share pages that
 * are only read.
 */
typedef struct {
    const int32_t *d_starts, *d_lengths, *d_table;
    uint32_t count, table_width;
} neuzip_sequences;

/*
 * neuzip_cache_append -- the newest tokens' keys and values, as the projections left them, into the cache; the queries made ready on the way.
 *     k' <- rotate(k, p),  e <- the least integer from -100 on with |k'| <= 448 * 2^e for the new tokens of the page and head,
 *     byte <- e4m3(k' * 2^-e),  scale <- 2^e           and so with v, which is not rotated;  q_out <- bf16(rotate(q, p))
 *     rotate(x, p)[i] = x[i] cos - x[i + D/2] sin,  rotate(x, p)[i + D/2] = x[i + D/2] cos + x[i] sin   for i < D/2, D = head_dim
 *
 * A page whose first tokens were there before keeps its scale if it is the larger one; if not, their bytes are rounded to the new one.
 * (By powers of two: only values that become subnormal change.)  Roundings are to nearest even; the angles' products and sums binary32,
 * each rounded.  Infinities become +-448 times the scale, NaN stays NaN; neither counts for a scale.
 *
 *   type        of k, v and q: NEUZIP_F32 or NEUZIP_BF16.
 *   d_k, d_v    rows x heads x head_dim; from one row to the next k_row, v_row elements (at least heads * head_dim; parts of a projection's
 *               result), multiples of 16 bytes.
 *   d_q, q_row, q_heads, d_q_out   likewise, q_heads heads; d_q_out rows x q_heads x head_dim bf16 words without gaps.  Both NULL: no queries.
 *   d_rotary    rotary_rows x head_dim floats: of position p the head_dim / 2 cosines, then the sines; rotary_rows at least table_width * page_tokens
 *               (else EINVAL).  NULL (and 0): nothing is rotated.
 *   rows        of the tensors.
 * A page that is appended to belongs to one sequence, once in its table, and to no other call at that time.  A left-out sequence's rows of q_out
 * are zeros.  All pointers to values are aligned to 16 bytes.
 * heads from 2^16 on, and calls of (rows / page_tokens + 2 * count) * 2 * heads (and rows, with queries) from 2^24 on -> EUNSUPPORTED.
 * Never allocates, never synchronises; results do not change from run to run.
 */
int neuzip_cache_append(const neuzip_cache *cache, const neuzip_sequences *sequences, int type, const void *d_k, uint64_t k_row,
                        const void *d_v, uint64_t v_row, const void *d_q, uint64_t q_row, uint32_t q_heads, void *d_q_out,
                        const float *d_rotary, uint64_t rotary_rows, uint32_t rows, void *hip_stream);

/*
 * neuzip_cache_attention -- attention of the newest tokens over their sequences' cache, causal: the token at position p sees the keys
 * at positions j <= p, with a window those at j > p - window.
 *     out <- bf16(sum_j softmax_j(scale * q . k_j) v_j);   a token that sees no key: zeros
 *
 *   d_q, q_row  rows x q_heads x head_dim bf16 words, q_row elements from one row to the next (a multiple of 8).  q_heads is a multiple of the cache's heads;
 *               query head h reads the cache's head h / (q_heads / heads).
 *   scale       above 0 and, times log2(e), within binary32: below 2.35e38 (else EINVAL).
 *   window      0: none.
 *   longest     no sequence has more tokens; 0: table_width * page_tokens.  (It decides how the work is split, so it may be too high, not too low:
 *               results are the same but for the order of sums.)
 *   d_out       rows x q_heads x head_dim bf16 words.
 *   d_scratch   device buffer of scratch_bytes bytes, at least neuzip_cache_attention_scratch_bytes(), 16-byte aligned, in use until the call's
 *               work has run (NULL where that is 0).
 * Keys and values are taken as the cache holds them; scores, maxima, sums and the output's sums are binary32, the weights of the softmax are
 * rounded to bf16 for the matrix cores (each by at most 2^-8 of itself; their sum is that of the unrounded ones), out is rounded once.  A key that a
 * token does not see has no influence, whatever it holds.
 * All sequences of a call are cut into tiles of one height, and their keys into as many parts, by rows, count, window and longest: a prompt beside many single tokens, or
 * one text far longer than the others, is right in one call and faster in calls of their own.
 * rows * q_heads up to 2^27 - 1, and fewer than 2^23 workgroups, of which single tokens take one for each sequence, head and 16 query heads of it (else
 * EUNSUPPORTED).  Never allocates, never synchronises; results do not change from run to run.
 */
int neuzip_cache_attention(const neuzip_cache *cache, const neuzip_sequences *sequences, const void *d_q, uint64_t q_row, uint32_t q_heads,
                           uint32_t rows, float scale, uint32_t window, uint64_t longest, void *d_out, void *d_scratch,
                           uint64_t scratch_bytes, void *hip_stream);
uint64_t neuzip_cache_attention_scratch_bytes(const neuzip_cache *cache, const neuzip_sequences *sequences, uint32_t q_heads, uint32_t rows,
                                              uint32_t window, uint64_t longest);

/*
 * neuzip_logits -- what is done to the output projection's result before a token is taken from it, row by row.  With c = how often a token
 * occurs in the row's history, for each of them in this order:
 *     where c > 0:  x <- x > 0 ? x / repetition : x * repetition,  x <- x - frequency * c,  x <- x - presence;
 *     where it has one:  x <- x + its bias;   not allowed by the row's mask:  x <- -infinity
 *
 *   d_logits, d_out   rows x vocab floats, row-major; d_out may be d_logits.
 *   history     d_tokens[d_starts[r]] .. d_tokens[d_starts[r + 1] - 1] is row r's, 64-bit integers (a number outside 0 .. vocab - 1 counts for
 *               nothing).  d_starts: rows + 1 32-bit integers, ascending.  history_tokens = 0: no history.
 *   d_repetition, d_frequency, d_presence   a float for each row; NULL: 1, 0, 0.
 *   biases      d_bias_tokens, d_bias_starts as the history's, d_bias_values a float for each entry; of entries for one token in one row the last
 *               counts.  bias_entries = 0: none.
 *   d_masks     masks x ceil(vocab / 32) 32-bit words: token v is allowed if bit v % 32 of word v / 32 is set.  d_mask_ids: the mask of each row,
 *               32-bit integers; outside 0 .. masks - 1: everything is allowed.  Both NULL: no masks.  (A mask that allows nothing leaves a row of -infinity.)
 *   history_tokens, bias_entries   how many tokens and entries there are: starts beyond them are taken as them.
 * Each operation is rounded to binary32 by itself.  vocab below 2^31, rows up to 65535 (else EUNSUPPORTED); pointers aligned to their elements.
 * Never allocates, never synchronises; results do not change from run to run.
 */
int neuzip_logits(const float *d_logits, uint32_t rows, uint64_t vocab, const int64_t *d_history, uint64_t history_tokens,
                  const int32_t *d_history_starts, const float *d_repetition, const float *d_frequency, const float *d_presence,
                  const int64_t *d_bias_tokens, const float *d_bias_values, uint64_t bias_entries, const int32_t *d_bias_starts,
                  const int32_t *d_masks, uint32_t masks, const int32_t *d_mask_ids, float *d_out, void *hip_stream);

/* Releases the blob and its device memory.  NULL is a no-op. */
void neuzip_free(neuzip_blob *blob);

/* Size in bytes of the blob's container (header, table, offsets, states, run
 * lengths, words, sign|mantissa stream, padding): what neuzip_export writes.
 * This is the figure bits/weight is computed from (Sec. 2.1: compression
 * ratio).  0 for NULL. */
uint64_t neuzip_compressed_bytes(const neuzip_blob *blob);

/* Bytes of device memory the blob actually holds (container sections plus
 * alignment padding and what the decoder derives: the cumulative table, for tensors of 1024 chunks (2^22
 * elements) and more the 16 KB slot table, and for tensors of at most 2^24 elements an entry point half way
 * into each state, 5 bytes per 256 elements). */
uint64_t neuzip_device_bytes(const neuzip_blob *blob);

/* Element count, mantissa bits, normalisation block size (0 = none), guard band of the table
 * (0 = none) and element type the blob was made with (-1 for something that is not a blob). */
uint64_t neuzip_elems(const neuzip_blob *blob);
uint32_t neuzip_block_size(const neuzip_blob *blob);
uint32_t neuzip_guard(const neuzip_blob *blob);
int neuzip_mantissa_bits(const neuzip_blob *blob);
int neuzip_dtype(const neuzip_blob *blob);

/*
 * neuzip_export / neuzip_import -- the container as one flat host byte buffer
 * (App. D storage layout: compressed exponents next to the signed mantissas).
 * Export synchronises hip_stream.  With h_buf == NULL only *written is set.
 * Import validates every section on the host before anything is uploaded
 * (ECORRUPT otherwise) and creates a new blob.
 */
int neuzip_export(const neuzip_blob *blob, void *h_buf, uint64_t cap, uint64_t *written,
                  void *hip_stream);
int neuzip_import(const void *h_buf, uint64_t len, void *hip_stream, neuzip_blob **blob);

/* Exponent statistics of the tensor the blob was compressed from (Sec. 2.2):
 * h_counts receives the 256-bin histogram (EINVAL for imported blobs, which
 * carry no counts), h_freq the quantised frequencies that sum to 4096. */
int neuzip_histogram(const neuzip_blob *blob, uint32_t h_counts[256]);
int neuzip_frequencies(const neuzip_blob *blob, uint16_t h_freq[256]);

/*
 * neuzip_stream_probe -- measurement aid for the throughput experiment of Sec. 3 (the throughput
 * figure compares against plain data movement): one kernel that only moves bytes the way the fused
 * decoder does, in the decoder's launch shape -- workgroups of 512 lanes that own 32 chunks of 8 KB
 * of output and hold the decoder's LDS, a 128-bit copy of their share of the input into LDS at the
 * start, then per lane and turn a field load of 8, 4, 2 or 1 bytes and a 16-byte store 256 bytes
 * apart, four turns at a time, non-temporal stores from 128 MB of output up -- reading (nearly all
 * of) in_bytes from d_in and writing out_bytes to d_out.  Its rate is the ceiling for a decoder with
 * that access pattern and byte mix on the machine at hand.
 *   d_in, d_out   device buffers, 16-byte aligned; in_bytes and out_bytes multiples of 16; out_bytes
 *                 at least 8208; in_bytes between 1/16 of out_bytes (plus one workgroup's worth) and
 *                 about 1.2 times out_bytes; d_out is overwritten with a pattern.  EINVAL otherwise.
 * Never allocates, never synchronises.
 */
int neuzip_stream_probe(const void *d_in, uint64_t in_bytes, void *d_out, uint64_t out_bytes, void *hip_stream);

/* Synchronises hip_stream and returns ECORRUPT if any decompression of this
 * blob so far found a state that did not return to its initial value or a
 * word run that was not consumed exactly; clears the flag. */
int neuzip_check(const neuzip_blob *blob, void *hip_stream);

/*
 * neuzip_compress_noalloc -- neuzip_compress for callers that cannot allocate device or pinned
 * memory at the time of the call: code that runs where hipMalloc is forbidden (a region under
 * stream capture, a tight serving or training loop, a harness that intercepts allocation).
 *
 *   d_src, n_elems, dtype, mantissa_bits, hip_stream   as for neuzip_compress.
 *   blob    an existing blob of this library made from a tensor of the same n_elems, dtype and
 *           mantissa_bits without block-wise normalisation (else EINVAL / EUNSUPPORTED).  It
 *           receives the new tensor; its old content is lost; its guard band is kept.
 *
 * The result is the same as neuzip_compress into that blob: same table, same stream, same container.
 * What differs: the pipeline's workspace (histogram bins, encoder constants, run slots, word
 * counts, the record of the stream length) is a fixed array of about 6.6 MB inside the library's
 * device code, present once on every GPU the library runs on until the process ends, and the
 * stream length comes back by a copy from it.  The call makes no hipMalloc, hipHostMalloc or
 * hipFree.  Limits and error behaviour:
 *   - n_elems <= NEUZIP_NOALLOC_MAX_ELEMS, else EUNSUPPORTED (nothing is run).
 *   - the blob's word section is not grown: if the new stream needs more room than the blob
 *     holds, the call returns ENOMEM and the blob holds no tensor until a compress call succeeds
 *     (its fixed sections have been overwritten by then).  A blob last filled by a tensor of the
 *     same or a higher exponent entropy has room.
 *   - all calls on one GPU share that GPU's array: calls that overlap in time on one GPU (from
 *     several host threads or streams) race and must be serialised by the caller.  The array
 *     keeps the last call's contents; the call clears what has to start at zero.
 * Synchronises hip_stream once: the blob is complete when the call returns.
 */
#define NEUZIP_NOALLOC_MAX_ELEMS (1ull << 22)
int neuzip_compress_noalloc(const void *d_src, uint64_t n_elems, int dtype, int mantissa_bits,
                            void *hip_stream, neuzip_blob *blob);

/* Device bytes of the workspace that compress calls share and keep between calls: the encoder's
 * run slots -- 16 x 200 words per 4096-element chunk, 1.56 bytes per element of the largest batch
 * compressed so far, but never more than the workspace limit below -- plus word counts and histogram
 * bins.  It is not part of any blob; Sec. 2.2's peak-memory accounting has to count it while weights
 * are being compressed (training), and neuzip_release_workspace returns it (inference, once the
 * model is compressed).  0 if none is held. */
uint64_t neuzip_workspace_bytes(void);

/* Limit on the encoder's run slots, in bytes (default 384 MiB, i.e. 251 M elements; 0 restores the
 * default; at least one group of 16 chunks, 102400 bytes, is always allowed).  A batch that would need
 * more is compressed tensor by tensor, and a single tensor that would need more goes through the
 * encoder in tiles of whole chunks, with one wait for the host per tile; the containers are the
 * same.  A workspace already larger than the new limit is freed.  Applies to all compress, recompress
 * and update calls except neuzip_compress_noalloc.  Not to be called while such a call runs. */
int neuzip_set_workspace_limit(uint64_t slot_bytes);

/* Frees the per-device workspace compress keeps between calls. */
int neuzip_release_workspace(void);

const char *neuzip_strerror(int code);
/* hipError_t of the last failing HIP call on this host thread (0 if none). */
int neuzip_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif
