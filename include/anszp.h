/*
 * anszp.h -- C ABI of libanszp: inference-time tabled-ANS (tANS) decoding of
 * entropy-coded, zero-point-quantized, mixed-precision network weights on
 * AMD MI355X (gfx950), fused with dequantisation to compute-ready weights.
 *
 * Method (citations are to the paper "Efficient Neural Compression with
 * Inference-time Decoding"):
 *   Sec. II-A    the decoder is a look-up table with one entry per state holding
 *                (symbol, nb_bits, newX); a step emits the symbol, reads nb_bits
 *                bits from the compressed stream and moves to state newX + bits;
 *                transitions that read no bits allow rates below 1 bit/weight.
 *   Sec. III-A   one table per layer.
 *   Sec. III-B   several streams are decoded at once with one shared table and a
 *                vector of states (here: one GPU lane per stream).
 *   Sec. II-B    weights come from a uniform quantizer with a zero-point, so
 *                w = scale * (q - zero_point).
 *
 * General conventions
 *   - Pointers marked [device] are device addresses of the current HIP device;
 *     pointers marked [host] are ordinary host addresses.  The caller owns every
 *     buffer.  The library allocates no device memory and keeps nothing between calls but
 *     three small per-device caches (the device's number of compute units, which kernels have
 *     been given leave to use the whole of a CU's on-chip memory, and the address of the
 *     fixed plan area that anszp_decode_static_plan uses); they are tables of atomics, so
 *     calls from several host threads are safe.  anszp_build_tables allocates and frees
 *     pinned host memory for its upload and waits for the copy.
 *   - `hip_stream` is a hipStream_t (NULL = default stream).  Device work is
 *     enqueued on it and the call returns without waiting, unless stated.
 *   - Return value: 0 on success, a negative ANSZP_E_* code when the host can
 *     see the problem (nothing has been enqueued then).  Problems only the GPU
 *     can see (corrupt stream, descriptor out of range) are OR-ed into the
 *     caller's status words; no device access ever leaves the caller's buffers
 *     because every index is checked or clamped first.
 *   - No exceptions, aborts or prints cross this boundary.
 *
 * Compressed container (all little-endian)
 *   A layer is a flat row-major array of n symbols q_i in [0, 256).  It is cut
 *   into consecutive chunks of `chunk_size` symbols (the last may be short).
 *   Inside a chunk, element j belongs to stream (j mod N) and is that stream's
 *   symbol number (j div N); N = n_streams <= 64.  Each stream is a private run
 *   of 32-bit words: the bits the decoder reads, in the order it reads them,
 *   filling each word from bit 0 upwards, zero-padded to a whole word.  The
 *   nb_bits of one step are read most significant first (bits = 2*bits + next).  A chunk's
 *   payload is its N streams' words back to back in stream order and starts at
 *   a word offset that is a multiple of 4.  Each stream has one 32-bit header:
 *   bits 0..15 the decoder's initial state X (0 <= X < 2^table_log), bits
 *   16..31 the stream's length in words.  The encoder starts every stream in
 *   state X = 0 and runs over its symbols last to first, so a correct decode
 *   ends in state 0 having read exactly the stream's words.
 */
#ifndef ANSZP_H
#define ANSZP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ANSZP_ALPHABET        256   /* symbols are bytes; frequency rows have 256 entries     */
#define ANSZP_MAX_TABLE_LOG   12    /* tables have L = 2^table_log states, 1 <= table_log <= 12 */
#define ANSZP_MAX_STREAMS     64    /* streams per chunk = lanes of one wavefront              */
#define ANSZP_TABLE_WORDS_PER_STATE 8 /* a table of L states occupies 8 L 32-bit words           */

/* error codes returned by the functions */
#define ANSZP_OK              0
#define ANSZP_E_NULL         (-1)   /* a required pointer is NULL                              */
#define ANSZP_E_RANGE        (-2)   /* an argument is outside its documented range             */
#define ANSZP_E_FREQ         (-3)   /* a frequency row does not sum to 2^table_log             */
#define ANSZP_E_SYMBOL       (-4)   /* data contains a symbol whose frequency is zero          */
#define ANSZP_E_SPACE        (-5)   /* an output buffer is too small / a stream exceeds 65535 words */
#define ANSZP_E_HIP          (-6)   /* the HIP runtime reported an error                       */
#define ANSZP_E_NOMEM        (-7)   /* host allocation failed                                  */

/* bits OR-ed into status[0] by the decode kernels */
#define ANSZP_ST_BAD_DESC     1u    /* chunk descriptor points outside a buffer; chunk skipped */
#define ANSZP_ST_BAD_STATE    2u    /* a stream did not end in state 0                          */
#define ANSZP_ST_BAD_LENGTH   4u    /* a stream read more or fewer words than its header says   */
#define ANSZP_ST_INTERNAL     8u    /* a hand-over between wavefronts did not complete; chunk abandoned */
#define ANSZP_ST_BAD_FREQ     16u   /* anszp_build_tables_device, anszp_pack_layer_device: a frequency row does not sum to 2^table_log */
#define ANSZP_ST_BAD_SYMBOL   32u   /* anszp_pack_layer_device: the data contain a symbol whose frequency is zero */
#define ANSZP_ST_NO_SPACE     64u   /* anszp_pack_layer_device: payload buffer too small, or a stream longer than 65535 words */

/* output element types */
#define ANSZP_OUT_U8          0     /* decoded symbols, no dequantisation                       */
#define ANSZP_OUT_F32         1     /* IEEE binary32                                            */
#define ANSZP_OUT_BF16        2     /* bfloat16, round-to-nearest-even of the binary32 value    */

/* One chunk (32 bytes).  Arrays of these live in device memory for anszp_decode.  A descriptor
   names everything its chunk touches, so the array may be in any order.  Layer after layer, as the
   packers leave it, is the order to prefer: the chunks of a layer that stand together share its table.
   (A launch of few chunks that differ much in size, without a plan, ends sooner when the chunks with
   the most payload words come first; a plan and the kernel for many short chunks see to that themselves.) */
typedef struct {
    uint32_t layer_id;        /* selects the table and the anszp_layer_t                       */
    uint32_t n_symbols;       /* symbols in this chunk; stream k holds ceil((n_symbols-k)/N)   */
    uint64_t out_offset;      /* element index of the chunk's first symbol in `out`            */
    uint64_t payload_offset;  /* first word of the chunk in `payload`; multiple of 4           */
    uint32_t payload_words;   /* sum of the chunk's stream lengths                             */
    uint32_t stream_offset;   /* index of stream 0's header in `stream_hdr`                    */
} anszp_chunk_t;

/* One layer's quantizer (32 bytes), Sec. II-B. */
typedef struct {
    float    scale;           /* used when channel_len == 0                                    */
    uint32_t zero_point;      /* z: symbol that decodes to +0.0                                */
    uint32_t bitwidth;        /* informational: symbols are < 2^bitwidth, 1..8                 */
    uint32_t channel_len;     /* 0: one scale per layer; else elements per output channel and
                                 the scale of layer element e is scales[scales_offset + e / channel_len] */
    uint64_t scales_offset;   /* index of the layer's first channel scale in `scales`          */
    uint64_t out_base;        /* element index of the layer's first element in `out`           */
} anszp_layer_t;

/* Arguments of anszp_decode (the struct itself is read on the host). */
typedef struct {
    const uint32_t*      tables;        /* [device] n_tables * 8 * 2^table_log words from anszp_build_tables, 16-byte aligned */
    uint32_t             n_tables;
    uint32_t             table_log;     /* R, 1..12                                             */
    uint32_t             n_streams;     /* N, 1..64                                             */
    uint32_t             out_dtype;     /* ANSZP_OUT_*                                          */
    const anszp_chunk_t* chunks;        /* [device]                                             */
    uint64_t             n_chunks;      /* may be 0 (nothing is enqueued)                       */
    const uint32_t*      stream_hdr;    /* [device] one header per stream                       */
    uint64_t             n_stream_hdr;
    const uint32_t*      payload;       /* [device] 16-byte aligned                             */
    uint64_t             payload_words;
    const anszp_layer_t* layers;        /* [device] n_tables entries                            */
    const float*         scales;        /* [device] per-channel scales, may be NULL if unused   */
    uint64_t             n_scales;
    void*                out;           /* [device] out_elems elements of out_dtype, 16-byte aligned */
    uint64_t             out_elems;
    uint32_t*            status;        /* [device] 2 words: [0] OR of ANSZP_ST_*, [1] number of
                                           failing chunks.  Never cleared by the library: zero it
                                           once, read it after synchronising the stream.        */
} anszp_decode_args_t;

/* Library version (major * 100 + minor). */
int anszp_version(void);

/* Text for an ANSZP_E_* code; never NULL; static storage. */
const char* anszp_strerror(int code);

/* [host only] Turn symbol counts into table frequencies (the paper does not say how):
 * freqs[s] >= 1 exactly when counts[s] > 0 and sum(freqs) == 2^table_log.
 * counts, freqs: [host] 256 entries.  Errors: E_NULL, E_RANGE, E_FREQ (no symbols, or more
 * distinct symbols than states). */
int anszp_normalize_freqs(const uint64_t* counts, int table_log, uint32_t* freqs);

/* [host only] Sec. II-A / III-A: build n_tables decode tables from normalised frequencies.
 * freqs: [host] n_tables rows of 256.  tables: [host] n_tables * ANSZP_TABLE_WORDS_PER_STATE * 2^table_log
 * 32-bit words.  Table t occupies words [t*8L, (t+1)*8L), L = 2^table_log:
 *   words [0, L)     tables of at most 256 states: the byte table of Sec. II-A, 3 L bytes, state X at
 *                    bytes 3X (symbol), 3X+1 (nb_bits), 3X+2 (newX), the rest zero; larger tables: zero
 *   word [2L + X]    the paper's triple for state X:
 *                    bits 0..15 newX      bits 16..23 nb_bits   bits 24..31 symbol
 *   words [4L + 2(2X + b)], [4L + 2(2X + b) + 1]
 *                    the same automaton with up to 8 steps merged and one bit of look-ahead: in state
 *                    X with next stream bit b (peeked, not consumed) the next c-1 symbols are the
 *                    dominant symbol (f > L/2: its zero-bit transitions and at most one of its 1-bit
 *                    transitions, which consumes b), then `symbol` is emitted; T stream bits are
 *                    consumed in all, and with v = the next T+1 stream bits, first bit on top, the
 *                    next entry is number base + v.  A run never passes through state 0 (the step that
 *                    arrives there ends the entry), so a stream ends where an entry ends.
 *                    first word:  bits 0..4 31-T (T <= 12)   bits 9..11 c-1   bits 16..23 symbol
 *                                 bits 24..27 T   bits 28..30 c-1   bit 31 set for X = 0   other bits zero
 *                    second word: 8 * base (two's complement)
 *   words [L, 2L), [3L, 4L)  zero
 * Errors: E_NULL, E_RANGE, E_FREQ. */
int anszp_build_tables_host(const uint32_t* freqs, int n_tables, int table_log, uint32_t* tables);

/* Same, writing the tables to device memory.  tables_dev: [device], 16-byte aligned.  The
 * host-to-device copy is enqueued on hip_stream and waited for before returning.
 * Errors: as above, E_HIP, E_NOMEM. */
int anszp_build_tables(const uint32_t* freqs_host, int n_tables, int table_log,
                       uint32_t* tables_dev, void* hip_stream);

/* Sec. II-A / III-A on the device: the same tables, word for word, from normalised frequencies that
 * are already in device memory (one workgroup per table; nothing passes through the host).
 * freqs_dev: [device] n_tables rows of 256.  tables_dev: [device] n_tables * 8 * 2^table_log words,
 * 16-byte aligned.  status_dev: [device] 2 words as in anszp_decode_args_t, or NULL: a row that
 * does not sum to 2^table_log leaves its table all zero and sets ANSZP_ST_BAD_FREQ (the host cannot
 * see the rows, so this is not a return code).  Asynchronous on hip_stream; both buffers stay owned
 * by the caller.  Errors: E_NULL, E_RANGE, E_HIP. */
int anszp_build_tables_device(const uint32_t* freqs_dev, int n_tables, int table_log,
                              uint32_t* tables_dev, uint32_t* status_dev, void* hip_stream);

/* [host only] Worst-case sizes for anszp_pack_layer: number of chunks and payload words. */
int anszp_pack_bound(uint64_t n_symbols, int table_log, int n_streams, uint32_t chunk_size,
                     uint64_t* n_chunks, uint64_t* payload_words);

/* [host only] Offline compressor (Sec. II-A encoder; container described at the top).
 * Encodes one layer's symbols with the table given by freqs and appends to caller arrays:
 * chunks_out[0..n_chunks), stream_hdr_out[0..n_chunks*N), payload_out[0..*payload_words_used).
 * layer_id / out_offset / payload_word_offset / stream_offset are the positions the layer's
 * first chunk will have in the full container (payload_word_offset must be a multiple of 4).
 * Errors: E_NULL, E_RANGE, E_FREQ, E_SYMBOL, E_SPACE, E_NOMEM. */
int anszp_pack_layer(const uint8_t* symbols, uint64_t n_symbols, const uint32_t* freqs,
                     int table_log, int n_streams, uint32_t chunk_size,
                     uint32_t layer_id, uint64_t out_offset, uint64_t payload_word_offset,
                     uint32_t stream_offset,
                     anszp_chunk_t* chunks_out, uint32_t* stream_hdr_out,
                     uint32_t* payload_out, uint64_t payload_cap_words, uint64_t* payload_words_used);

/* Sec. II-A decoder + Sec. III-B parallel streams + Sec. II-B dequantisation, fused: decode
 * every chunk (one wavefront per chunk, one lane per stream) and write out[out_offset + j] for
 * each of its symbols j, as raw symbols, fp32 or bf16 weights.  One kernel launch on hip_stream.
 * Errors: E_NULL, E_RANGE (table_log, n_streams, out_dtype, n_tables == 0, n_chunks >= 2^31,
 * payload or out not 16-byte aligned). */
int anszp_decode(const anszp_decode_args_t* args, void* hip_stream);

/* The same call with the kernel chosen by hand; results are identical for every variant.
 *   0  automatic (what anszp_decode does): 2 or 4; for few short chunks, a kernel with a workgroup per chunk that does one
 *      thing after the other; for more short chunks than the chip decodes at once, a kernel with a wavefront per chunk and
 *      the table shared by a workgroup; for long enough chunks of a single stream, a kernel that
 *      decodes a stream from many places at once, started in guessed states and joined where they meet
 *   1  step-wise kernel: one look-up per symbol, exactly the loop of Sec. II-A / III-B; also the
 *      path any chunk takes whose compressed words exceed the on-chip window
 *   2  look-ahead kernel: look-ups use the look-ahead entries of the table (entry 2X + b above),
 *      compressed words and decoded symbols are staged in LDS, and the work of a chunk is split
 *      over several wavefronts of its workgroup
 *   3  step-wise kernel with sixteen chunks per workgroup sharing the tables in LDS
 *   4  streaming kernel: one look-up per symbol from compact entries in LDS, each stream's words
 *      fetched 64 bytes at a time through a ring in LDS by wavefronts that only load (what the
 *      automatic choice takes when the chunks are too large for the on-chip window)
 *   5  byte-table kernel: the decoder as Sec. II-A sizes it, for tables of at most 256 states
 *      (table_log <= 8): the 3 l-byte table (one byte each for symbol, nb_bits and newX; 192 bytes for
 *      64 states) in LDS, three byte reads and a log2(l)-bit addition per symbol
 * Errors: as anszp_decode, E_RANGE for an unknown variant or variant 5 with table_log > 8. */
int anszp_decode_variant(const anszp_decode_args_t* args, int variant, void* hip_stream);

/* For tests of the library's failure handling only.  Every wait of one wavefront for another inside the decode
 * kernels is bounded by a number of polls, after which the chunk is abandoned with ANSZP_ST_INTERNAL and its
 * workgroup drains.  polls >= 1: later launches give up after polls - 1 polls (1: at the first wait that is not
 * satisfied at once, which every launch of the look-ahead and streaming kernels has); 0: back to the default
 * (2^22).  The GPU packer's workgroups wait for the sizes of lower-numbered chunks within the same bound (default 2^16
 * polls); a chunk whose workgroup gives up is written by the launch behind it, with the same words and no status bit.
 * Process-wide, not synchronised with launches in flight. */
void anszp_test_set_spin_limit(uint32_t polls);

/* Sec. III-A: the weights of a network are decoded again at every inference, from arrays that do not
 * change.  What every launch of anszp_decode first works out on the device (which chunks of a layer
 * share a workgroup and its on-chip copy of the layer's table, in which order the chip's dies take
 * them) can therefore be prepared once: anszp_plan_decode writes it to plan_dev, anszp_decode_planned
 * decodes with it and gives the same output and status words as anszp_decode.
 *   anszp_plan_bytes    bytes of device memory a plan for n_chunks chunks takes (a record of 128 bytes per
 *                       workgroup of the launch, and as much again to sort them in: the workgroups take the
 *                       units with the longest chains first); 0 for n_chunks >= 2^31.
 *   anszp_plan_decode   args as for anszp_decode (every array already in place; out and status are not
 *                       touched); plan_dev [device, caller's, 16-byte aligned] at least
 *                       anszp_plan_bytes(args->n_chunks) bytes, written on hip_stream.  A launch that
 *                       the automatic choice does not give to the look-ahead kernel needs no plan:
 *                       nothing is written then, and anszp_decode_planned does not read plan_dev.
 *   anszp_decode_planned  the plan must have been written for these very arrays (same pointers'
 *                       contents, same scalar arguments) on this device.  A plan that was made for
 *                       another number of chunks or another kernel is refused on the device
 *                       (ANSZP_ST_BAD_DESC, nothing decoded); one whose descriptors no longer match the
 *                       arrays decodes what it describes, checked against the caller's buffers like any
 *                       descriptor: never out of bounds.
 * Errors: as anszp_decode; E_NULL for a missing plan, E_RANGE for one that is too small or misaligned. */
uint64_t anszp_plan_bytes(uint64_t n_chunks);
int anszp_plan_decode(const anszp_decode_args_t* args, void* plan_dev, uint64_t plan_bytes, void* hip_stream);
int anszp_decode_planned(const anszp_decode_args_t* args, const void* plan_dev, uint64_t plan_bytes, void* hip_stream);

/* For callers that cannot allocate device memory (code under stream capture, serving loops, harnesses
 * that forbid it): anszp_decode_planned with the plan kept in device memory of the library's own, a
 * fixed array of 1 MiB per device that holds a plan for at most 4096 chunks and stays until the
 * process ends.  Calls no allocating routine.  replan != 0: the plan is written first (as by
 * anszp_plan_decode) and the decode follows on the same stream; replan == 0: the array must still hold
 * the plan an earlier call on this device wrote for these arrays.  Every call on a device shares that
 * device's array: calls that overlap on one device (other streams, other host threads) race unless all
 * of them pass replan == 0 for the same arrays.
 * Errors: as anszp_decode; E_RANGE for more than 4096 chunks; E_HIP if the array's address cannot be found. */
int anszp_decode_static_plan(const anszp_decode_args_t* args, int replan, void* hip_stream);

/* Sec. II-B alone: out[i] = scale * (symbols[i] - zero_point) for i < n, the scale chosen as in
 * anszp_layer_t with the layer starting at element 0.  symbols_dev, scales_dev, out_dev: [device];
 * layer: [host].  out_dtype is ANSZP_OUT_F32 or ANSZP_OUT_BF16.  Errors: E_NULL, E_RANGE. */
int anszp_dequant_zp(const uint8_t* symbols_dev, uint64_t n, const anszp_layer_t* layer,
                     const float* scales_dev, uint64_t n_scales, void* out_dev, int out_dtype,
                     void* hip_stream);

/* The packer on the GPU (Sec. II-A, the encoding direction: a stream's symbols are walked backwards,
 * the state dropping low bits until the symbol's sub-range holds it): anszp_pack_layer for symbols and
 * frequencies that live in device memory, writing the same descriptors, stream headers and payload
 * words, word for word.  symbols_dev [device] n_symbols bytes; freqs_dev [device] 256 frequencies
 * summing to 2^table_log; chunks_dev [device] ceil(n_symbols / chunk_size) descriptors, stream_hdr_dev
 * [device] n_streams headers per chunk, payload_dev [device] payload_cap_words words where this layer's
 * words begin (its chunks' payload_offset fields count from payload_word_offset, a multiple of 4);
 * payload_words_used_dev [device] one 64-bit count; status_dev [device] 2 words as for anszp_decode.
 * Asynchronous on hip_stream; three kernel launches, nothing allocated.  Errors: E_NULL, E_RANGE, E_HIP on
 * the host; in status: ANSZP_ST_BAD_FREQ (nothing is written), ANSZP_ST_BAD_SYMBOL (the layer's output is
 * unspecified), ANSZP_ST_NO_SPACE (chunks that do not fit are not written; *payload_words_used_dev still
 * holds what the layer needs). */
int anszp_pack_layer_device(const uint8_t* symbols_dev, uint64_t n_symbols, const uint32_t* freqs_dev,
                            int table_log, int n_streams, uint32_t chunk_size, uint32_t layer_id,
                            uint64_t out_offset, uint64_t payload_word_offset, uint32_t stream_offset,
                            anszp_chunk_t* chunks_dev, uint32_t* stream_hdr_dev, uint32_t* payload_dev,
                            uint64_t payload_cap_words, uint64_t* payload_words_used_dev,
                            uint32_t* status_dev, void* hip_stream);

/* The same for a whole set of layers in three launches (a wavefront per chunk at a time, chunks of all layers side by
 * side).  symbols_dev [device]: the layers' symbols, layer after layer; jobs_dev [device] n_layers
 * entries in layer order; freqs_dev [device] n_layers rows of 256 frequencies summing to 2^table_log each;
 * n_chunks: the sum over the layers of ceil(n_symbols / chunk_size) (anszp_pack_bound gives each term).
 * Layer l becomes layer_id l; its chunks follow those of layer l-1 in chunks_dev and stream_hdr_dev
 * (stream_offset = chunk index * n_streams), its elements start at out_offset = first_symbol, the payload
 * starts at word 0 of payload_dev.  Writes what one anszp_pack_layer call per layer would write (and what the
 * oracle's encoder writes), word for word.  Status bits as anszp_pack_layer_device, and ANSZP_ST_BAD_DESC
 * when the jobs do not account for n_chunks chunks (those chunks get empty descriptors).
 * Errors: E_NULL, E_RANGE (table_log, n_streams, n_chunks >= 2^31 or n_chunks * n_streams >= 2^32), E_HIP. */
typedef struct {
    uint64_t first_symbol;    /* index of the layer's first symbol in symbols_dev = out_offset of its first chunk */
    uint64_t n_symbols;
    uint32_t chunk_size;      /* >= 1 */
    uint32_t first_chunk;     /* number of chunks of all layers before this one */
    uint32_t reserved[2];     /* 0 */
} anszp_pack_job_t;
int anszp_pack_layers_device(const uint8_t* symbols_dev, const anszp_pack_job_t* jobs_dev, uint32_t n_layers,
                             uint64_t n_chunks, const uint32_t* freqs_dev, int table_log, int n_streams,
                             anszp_chunk_t* chunks_dev, uint32_t* stream_hdr_dev, uint32_t* payload_dev,
                             uint64_t payload_cap_words, uint64_t* payload_words_used_dev,
                             uint32_t* status_dev, void* hip_stream);

/* What anszp_pack_layers_device or, with `single`, anszp_pack_layer_device writes, for callers that bring
 * scratch memory and have their layers' sizes on the host: the encoding tables are worked out once per layer instead of once
 * per workgroup, the jobs travel with the launches, and with `clear` the call itself clears the results, so that they may come
 * from memory with any contents.  The struct and its host arrays are read before the call returns. */
typedef struct {
    const uint8_t*  symbols;               /* [device] the layers' symbols, one layer behind the other      */
    const uint32_t* freqs;                 /* [device] n_layers rows of 256 frequencies                     */
    const uint64_t* layer_symbols;         /* [host] n_layers counts                                        */
    const uint32_t* chunk_sizes;           /* [host] n_layers sizes, each >= 1                              */
    uint32_t        n_layers, table_log, n_streams;
    uint32_t        single;                /* not 0: n_layers is 1, with the offsets and the treatment of bad frequencies of anszp_pack_layer_device */
    uint32_t        layer_id, stream_offset;             /* with `single` only (else 0)                     */
    uint32_t        clear;                 /* descriptors, headers and status to 0, payload to 0xFFFFFFFF, over the sizes below */
    uint64_t        out_offset, payload_word_offset;     /* with `single` only (else 0)                     */
    anszp_chunk_t*  chunks;                /* [device] with `clear` 16-byte aligned, as stream_hdr and payload */
    uint32_t*       stream_hdr;            /* [device]                                                      */
    uint32_t*       payload;               /* [device]                                                      */
    uint64_t        payload_cap_words;
    uint64_t        clear_chunks, clear_stream_hdr, clear_payload_words;   /* descriptors, headers, words there are */
    uint64_t*       payload_words_used;    /* [device]                                                      */
    uint32_t*       status;                /* [device] 2 words                                              */
    void*           scratch;               /* [device] 16-byte aligned, anszp_pack_scratch_bytes; in use until the launches are done */
    uint64_t        scratch_bytes;
} anszp_pack_set_t;
/* [host only] 32 + 16 + 2048 + 2 * max(2^table_log, 8) bytes a layer and 272 (0 for a table_log out of range). */
uint64_t anszp_pack_scratch_bytes(uint32_t n_layers, int table_log);
int anszp_pack_set_device(const anszp_pack_set_t* set, void* hip_stream);

/* activation layouts of anszp_conv_fused */
#define ANSZP_ACT_NHWC        0     /* [batch][h][w][channels]                                    */
#define ANSZP_ACT_C8          1     /* [batch][channels / 8][h][w][8]: blocks of 8 channels, so that
                                       the 16 pixels a matrix instruction's operand rows come from
                                       are 256 contiguous bytes; channels a multiple of 8          */

/* Arguments of anszp_conv_fused (the struct itself is read on the host).  The container fields
 * mean what they mean in anszp_decode_args_t; `chunks` points at the FIRST chunk of the layer to
 * convolve with, `n_chunks` counts the chunks from there on. */
typedef struct {
    const uint32_t*      tables;         /* [device] as for anszp_decode                          */
    uint32_t             n_tables;
    uint32_t             table_log;
    uint32_t             n_streams;
    uint32_t             layer_id;       /* the layer's table and anszp_layer_t                   */
    const anszp_chunk_t* chunks;         /* [device] the layer's chunks, in order of output channel */
    uint64_t             n_chunks;       /* at least cout / rows_per_chunk                        */
    const uint32_t*      stream_hdr;     /* [device]                                              */
    uint64_t             n_stream_hdr;
    const uint32_t*      payload;        /* [device]                                              */
    uint64_t             payload_words;
    const anszp_layer_t* layers;         /* [device] n_tables entries; channel_len is 0 or kh*kw*cin
                                            (one scale per output channel)                        */
    const float*         scales;         /* [device] may be NULL if unused                        */
    uint64_t             n_scales;
    uint32_t             rows_per_chunk; /* output channels per chunk: 1, 2, 4, 8 or 16; every chunk
                                            holds rows_per_chunk * kh*kw*cin symbols              */
    uint32_t             batch, in_h, in_w, cin, cout, kh, kw, stride, pad;
    const uint16_t*      x;              /* [device] bf16 activations in x_layout, batch * in_h * in_w * cin
                                            elements (fewer than 2^32), 16-byte aligned            */
    void*                y;              /* [device] batch * out_h * out_w * cout elements (fewer than 2^32)
                                            of y_dtype in y_layout, out = (in + 2 pad - k) / stride + 1,
                                            16-byte aligned; every element is written              */
    uint32_t             y_dtype;        /* ANSZP_OUT_F32, or ANSZP_OUT_BF16 (the fp32 result rounded
                                            to nearest even)                                      */
    uint32_t             x_layout;       /* ANSZP_ACT_*; ANSZP_ACT_C8 needs cin to be a multiple of 8 */
    uint32_t             y_layout;       /* ANSZP_ACT_*                                            */
    uint32_t*            status;         /* [device] 2 words, as for anszp_decode                 */
} anszp_conv_args_t;

/* Fused decode + convolution (the data are decoded on their way from memory to the compute
 * units, Sec. II; weights w = scale * (q - z), Sec. II-B): y = conv2d(x, w) with zero padding,
 * where the layer's symbols q, in the order [cout][kh][kw][cin], are decoded (Sec. II-A, one
 * stream per lane as in Sec. III-B) into on-chip memory and multiplied there with the activations
 * by bf16 matrix instructions with fp32 accumulation; the decoded weights are never written to
 * device memory.  q - z is exact in bf16; the scale multiplies the fp32 sums.
 * Limits: cout a multiple of 16; kh*kw*cin <= 4608; batch*out_h*out_w < 2^31.  Asynchronous on
 * hip_stream; the buffers stay the caller's.  Errors: E_NULL, E_RANGE (a limit above, misaligned
 * x or y, too few chunks), E_HIP; a chunk whose descriptor does not fit the layer, a stream that
 * ends in the wrong state or length: ANSZP_ST_* bits in status, as for anszp_decode (the outputs
 * of the affected output channels are then unspecified but finite sums of finite values).
 * The kernel reads the look-ahead entries of the layer's table (anszp_build_tables*).  The first call
 * on a device gives the kernels leave to use all of a CU's on-chip memory (a function attribute) and
 * must not be part of a stream capture: one call for all layers with channels in 32s and kernels of
 * 1 x 1 (no padding) or three wide, whatever their batch; for others one per kind of layer.  Later
 * calls may be captured into a graph and replayed. */
int anszp_conv_fused(const anszp_conv_args_t* args, void* hip_stream);

/* ---- operators that run decoded layers as a model: norm, product, quantised cache, attention ----
 * All four return before the GPU is done, allocate nothing, keep nothing and may be captured into a graph.  Element
 * types are ANSZP_OUT_F32, ANSZP_OUT_BF16 and, where said, ANSZP_I8; strides count elements, the innermost dimension is
 * contiguous, and rows may begin at any element. */
#define ANSZP_I8              3     /* signed bytes, a value is a scale times them                      */

/* Root-mean-square norm with the residual's addition: h = x + residual, y = h * (mean(h^2) + eps)^(-1/2) * weight; out is y
 * rounded to its type, or with ANSZP_I8 round(y / s) with s = max|y| / 127 of the row in out_scales (0 for a row of zeros; a row
 * that holds an infinity or a NaN, or whose y does, has NaN for a scale and zeros).  Sums in 32 bits, from h before it is rounded: |h| below 2^63 / sqrt(cols). */
typedef struct {
    const void* x;                /* [device] rows x cols of dtype                                   */
    const void* residual;         /* [device] the same, or NULL for none                             */
    void*       total;            /* [device] h rounded to dtype, or NULL; may be x or residual (same stride) */
    const void* weight;           /* [device] cols of weight_dtype                                   */
    void*       out;              /* [device] rows x cols of out_dtype; apart from the inputs        */
    float*      out_scales;       /* [device] rows; with ANSZP_I8 only                               */
    uint64_t    rows;             /* < 2^31, may be 0                                                */
    uint64_t    x_stride, residual_stride, total_stride, out_stride;
    uint32_t    cols;             /* 1 .. 2^31 - 1                                                   */
    uint32_t    dtype;            /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    uint32_t    weight_dtype;     /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    uint32_t    out_dtype;        /* ANSZP_OUT_F32, ANSZP_OUT_BF16 or ANSZP_I8                       */
    uint32_t    normalise;        /* 0: y = h (weight and eps are not read)                          */
    float       eps;
} anszp_norm_args_t;
/* Errors: E_NULL, E_RANGE (also for an output that meets an operand it may not), E_HIP. */
int anszp_rms_norm(const anszp_norm_args_t* args, void* hip_stream);

/* activations of anszp_linear */
#define ANSZP_FN_NONE        0
#define ANSZP_FN_RELU        1
#define ANSZP_FN_GELU        2     /* v / 2 * (1 + erf(v / sqrt 2)), erf to 1.5e-7                     */
#define ANSZP_FN_SILU        3     /* v / (1 + exp(-v))                                                */

/* Matrix product with its epilogue: out = act(scale * x_scales[r] * channel_scales[c] * sum_k x[r, k] w[c, k] + bias[c]) * mul[r, c]
 * + residual[r, c].  x in bf16 with weights in bf16, or x in 8 bits (as anszp_rms_norm leaves it) with weights as symbols (as
 * anszp_decode leaves them with ANSZP_OUT_U8), where w = symbol - zero_point (Sec. II-B), whatever the symbols' bitwidth.
 * Sums of bf16 products in fp32, of 8-bit ones exact. */
typedef struct {
    const void*  x;               /* [device] rows x k                                               */
    const void*  weight;          /* [device] cols x k: bf16, or with x in ANSZP_I8 symbols          */
    const float* x_scales;        /* [device] rows, or NULL                                          */
    const float* channel_scales;  /* [device] cols, or NULL                                          */
    const float* bias;            /* [device] cols, or NULL                                          */
    const void*  mul;             /* [device] rows x cols of out_dtype, or NULL                      */
    const void*  residual;        /* [device] rows x cols of out_dtype, or NULL                      */
    void*        out;             /* [device] rows x cols of out_dtype; may be mul or residual (same stride), apart from x and weight */
    uint64_t     rows, cols;      /* each < 2^31, may be 0; fewer than 2^24 tiles of 64 x 64 together */
    uint64_t     x_stride, weight_stride, mul_stride, residual_stride, out_stride;
    uint32_t     k;               /* 1 .. 2^30 (x in 8 bits: 65536, so that sums fit 32 bits)        */
    uint32_t     x_dtype;         /* ANSZP_OUT_BF16 or ANSZP_I8                                      */
    uint32_t     out_dtype;       /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    uint32_t     zero_point;      /* 0 .. 255; with x in ANSZP_I8 only                               */
    uint32_t     activation;      /* ANSZP_FN_*                                                      */
    float        scale;
    void*        workspace;       /* [device] anszp_linear_workspace_bytes, 16-byte aligned, in use until the call is done; or NULL: */
    uint64_t     workspace_bytes; /* products that would share k out over more of the chip take longer then                */
} anszp_linear_args_t;
/* [host only] Bytes of workspace with which a call is fastest (0: none); reads sizes only, no pointers. */
uint64_t anszp_linear_workspace_bytes(const anszp_linear_args_t* args);
/* Errors: E_NULL, E_RANGE (also for a workspace that is too small, and for an output that meets an operand it may not), E_HIP. */
int anszp_linear(const anszp_linear_args_t* args, void* hip_stream);

/* A paged cache of keys and values in 8 or 4 bits.  A slot is a token's place: page * page_size + token in page.  A vector (one
 * head's key or value of one token) has symbols and a pair (scale, zero-point), value = scale * (symbol - zero_point): in 4 bits
 * element 2i is the low and element 2i + 1 the high half of byte i.  The arrays are [page][head][token in page][...]. */
typedef struct {
    uint8_t* k;                   /* [device] n_pages x heads x page_size x head_dim * bits / 8 bytes, 16-byte aligned */
    float*   k_params;            /* [device] n_pages x heads x page_size x 2, 16-byte aligned; zero-points are whole, 0 .. 2^bits - 1 */
    uint8_t* v;
    float*   v_params;
    uint64_t n_pages;             /* < 2^31, and n_pages * heads * page_size < 2^32                  */
    uint32_t page_size;           /* a power of two from 16 to 65536                                 */
    uint32_t heads;               /* of keys and values, 1 .. 65535                                  */
    uint32_t head_dim;            /* 64, 128 or 256                                                  */
    uint32_t bits;                /* 8 or 4                                                          */
} anszp_cache_t;
/* [host only] What every call with a cache checks first: E_NULL, E_RANGE. */
int anszp_cache_check(const anszp_cache_t* cache);

/* Keys and values quantised into their slots, a scale and a zero-point for each vector (Sec. II-B): lo = min(0, min x), hi = max(0, max x),
 * scale = (hi - lo) * (1 / (2^bits - 1)), zero_point = round(-lo / scale), symbol = clamp(round(x / scale) + zero_point), every operation
 * rounded to binary32.  A vector that holds an infinity or a NaN, or whose range no binary32 holds, has NaN for a scale.
 * k, v: [device] n_tokens x heads x head_dim of dtype (F32 or BF16); slots: [device] n_tokens, all different; a negative one: the token is
 * not written.  status: [device] 2 words as for anszp_decode, or NULL: a slot beyond the cache is not written (ANSZP_ST_BAD_DESC,
 * counted).  Errors: E_NULL, E_RANGE, E_HIP. */
int anszp_cache_write(const anszp_cache_t* cache, const void* k, const void* v, uint32_t dtype, uint64_t k_token_stride, uint64_t k_head_stride,
                      uint64_t v_token_stride, uint64_t v_head_stride, const int64_t* slots, uint64_t n_tokens, uint32_t* status, void* hip_stream);
/* What the slots hold, as values: k, v [device] n_tokens x heads x head_dim, contiguous, of dtype (F32 or BF16), 16-byte aligned; zeros for
 * a negative slot and one beyond the cache (ANSZP_ST_BAD_DESC).  Errors: E_NULL, E_RANGE, E_HIP. */
int anszp_cache_read(const anszp_cache_t* cache, void* k, void* v, uint32_t dtype, const int64_t* slots, uint64_t n_tokens, uint32_t* status, void* hip_stream);

/* Attention of new tokens over the cache.  Sequence s has the queries starts[s] .. starts[s + 1] - 1, its last tokens: with n of them
 * and lengths[s] tokens in all (the new ones written already), number i is at position lengths[s] - n + i and sees the positions up to its own.
 *   out = sum_t softmax_t(scale * q . k_t) v_t        a query that sees nothing (a position below 0): zeros
 * Query head h reads the cache's head h / group.  Position t of sequence s is in page pages[s * table_width + t / page_size].
 * Sums and statistics in fp32; queries go into the matrix instructions in fp16 scaled by a power of two per row, keys and values
 * exactly, weights in fp16 with a scale that keeps 11 bits of each (with F32 output too) down to 2^-23 of the largest that the query sees.
 * Sums are held at up to 2^15 times a value for each token: values below 2^113 / length in size. */
typedef struct {
    anszp_cache_t  cache;
    const void*    q;             /* [device] n_tokens x (heads * group) x head_dim, bf16            */
    void*          out;           /* [device] the same shape, of out_dtype, contiguous in head_dim, rows apart */
    const int32_t* pages;         /* [device] n_seqs x table_width                                   */
    const int32_t* lengths;       /* [device] n_seqs, 0 .. table_width * page_size                   */
    const int32_t* starts;        /* [device] n_seqs + 1, from 0 to n_tokens, never falling; what is out of range is
                                     clamped, as lengths are; queries of no sequence are left unwritten */
    uint32_t*      status;        /* [device] 2 words, or NULL: ANSZP_ST_BAD_DESC for a page beyond the cache that a query would
                                     have seen; its positions are not seen, [1] grows; and for a length out of range of a
                                     sequence with new tokens, which moves their positions, [1] grows by 1 */
    void*          workspace;     /* [device] anszp_attend_workspace_bytes, 16-byte aligned, in use until the call is done */
    uint64_t       workspace_bytes;
    uint64_t       n_tokens, n_seqs;                      /* each < 2^24, may be 0; more than a launch has threads for is E_RANGE, which n_tokens * group + 16 *
                                     n_seqs < 2^28 and (n_tokens * group + 128 * n_seqs) * heads < 2^30 never are */
    uint64_t       q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    uint32_t       table_width;   /* >= 1; table_width * page_size <= 2^30                           */
    uint32_t       group;         /* query heads per head of the cache, 1 .. 256                     */
    uint32_t       out_dtype;     /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    float          scale;
} anszp_attend_args_t;
/* [host only] Bytes of workspace a call takes (0: none); reads sizes only, no pointers. */
uint64_t anszp_attend_workspace_bytes(const anszp_attend_args_t* args);
/* Errors: E_NULL, E_RANGE (also for a workspace that is too small), E_HIP. */
int anszp_attend(const anszp_attend_args_t* args, void* hip_stream);

/* ---- a serving step around them: tokens placed in the cache, looked up, adapted to their requests, drawn ----
 * The conventions are those of the operators above. */

/* New tokens placed in a paged cache.  Sequence s holds lengths[s] tokens in the pages of its row of the table, and gets new_tokens[s].
 * Free pages are a stack, free_pages[0 .. n_free - 1]; P is the page's size.
 *   old = 0 where ends[s], whose ceil(lengths[s] / P) pages go on the stack, sequence by sequence in their order, else lengths[s];
 *   need = ceil((old + new) / P) - ceil(old / P) pages are taken from the stack's end, in the sequences' order, and written to the table.
 * A sequence gets nothing (its length stays, its slots are -1) where the stack has not as many pages as it and those before it need, or
 * new_tokens[s] is negative or more than its row of the table or n_tokens has room for; lengths out of range are treated alike (those of a
 * sequence that ends are clamped).  Apart from lengths_out, n_free_out, the table's entries behind the pages that a sequence goes on with (of one
 * that ends: from its first on) and the stack's behind n_free nothing is changed.  So a call with outputs of their own may be made again, and gives the same, unless
 * a sequence both ends and gets tokens: its row then begins with other pages than those that it has to give back. */
typedef struct {
    int32_t*       pages;         /* [device] n_seqs x table_width                                   */
    const int32_t* lengths;       /* [device] n_seqs, 0 .. table_width * page_size                   */
    int32_t*       lengths_out;   /* [device] n_seqs: old + new; may be lengths                      */
    const int32_t* new_tokens;    /* [device] n_seqs                                                 */
    const int32_t* ends;          /* [device] n_seqs, 0: goes on; or NULL: all do                    */
    int32_t*       free_pages;    /* [device] free_room                                              */
    const int32_t* n_free;        /* [device] one number, 0 .. free_room                             */
    int32_t*       n_free_out;    /* [device] one number; may be n_free                              */
    int64_t*       slots;         /* [device] n_tokens: the new tokens' slots, one sequence behind the other; -1 behind the last */
    int32_t*       owners;        /* [device] n_tokens: the sequence each is of, -1 behind the last; or NULL */
    int32_t*       starts;        /* [device] n_seqs + 1: as anszp_attend takes them                 */
    uint32_t*      status;        /* [device] 2 words, or NULL: ANSZP_ST_BAD_DESC for a sequence that gets nothing though it asks, numbers out of
                                     range, a page below 0, pages that overflow the stack; [1] grows */
    void*          workspace;     /* [device] anszp_place_workspace_bytes, 16-byte aligned, in use until the call is done; NULL if none */
    uint64_t       workspace_bytes;
    uint64_t       n_seqs, n_tokens, free_room;           /* < 2^24, < 2^31, < 2^31; may be 0        */
    uint32_t       table_width;   /* >= 1; table_width * page_size <= 2^30                           */
    uint32_t       page_size;     /* a power of two from 16 to 65536                                 */
    int32_t*       last;          /* [device] n_seqs: which of all new tokens is the sequence's last one, -1 if it has none or gets nothing; or NULL */
} anszp_place_args_t;
/* [host only] Bytes of workspace a call takes (0: none); reads sizes, and whether there are `ends`. */
uint64_t anszp_place_workspace_bytes(const anszp_place_args_t* args);
/* Errors: E_NULL, E_RANGE (also for a workspace that is too small, and for an output that meets another operand), E_HIP. */
int anszp_place(const anszp_place_args_t* args, void* hip_stream);

/* Tokens looked up: out[t] = scale * row_scales[id] * (weight[id] - zero_point), id = tokens[t], with weights as symbols (Sec. II-B), or
 * scale * weight[id] with weights in bf16.  Zeros for a token below 0, and for one beyond the vocabulary (ANSZP_ST_BAD_DESC, counted). */
typedef struct {
    const int64_t* tokens;        /* [device] n_tokens                                               */
    const void*    weight;        /* [device] vocabulary x cols: symbols, or bf16                    */
    const float*   row_scales;    /* [device] vocabulary, or NULL; with symbols only                 */
    void*          out;           /* [device] n_tokens x cols of out_dtype, apart from the inputs    */
    uint32_t*      status;        /* [device] 2 words, or NULL                                       */
    uint64_t       n_tokens, vocabulary;                  /* each < 2^31, may be 0                   */
    uint64_t       weight_stride, out_stride;
    uint32_t       cols;          /* 1 .. 2^31 - 1                                                   */
    uint32_t       weight_dtype;  /* ANSZP_OUT_U8 (symbols) or ANSZP_OUT_BF16                        */
    uint32_t       zero_point;    /* 0 .. 255; with symbols only                                     */
    uint32_t       out_dtype;     /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    float          scale;
} anszp_embed_args_t;
/* Errors: E_NULL, E_RANGE, E_HIP. */
int anszp_embed(const anszp_embed_args_t* args, void* hip_stream);

/* Low-rank adapters beside a product: with i = ids[r] the adapter of row r,
 *   out = act(base + scales[i] * x_scales[r] * (x[r] a[i]^T) b[i]^T) * mul + residual
 * and without the middle term for a row that has none.  base is what anszp_linear gives without its epilogue.  Sums in fp32, and what lies between the
 * two products, too, with all its 24 bits.  A row's result depends on its own adapter alone; where that or x holds an infinity or a NaN, it has
 * infinities or NaN. */
typedef struct {
    const void*    x;             /* [device] rows x k of x_dtype                                    */
    const void*    a;             /* [device] adapters x rank x k, bf16                              */
    const void*    b;             /* [device] adapters x cols x rank, bf16                           */
    const int32_t* ids;           /* [device] rows; below 0: no adapter                              */
    const float*   x_scales;      /* [device] rows, or NULL                                          */
    const float*   scales;        /* [device] adapters, or NULL                                      */
    const void*    base;          /* [device] rows x cols of base_dtype                              */
    const void*    mul;           /* [device] rows x cols of out_dtype, or NULL                      */
    const void*    residual;      /* [device] rows x cols of out_dtype, or NULL                      */
    void*          out;           /* [device] rows x cols of out_dtype; may be base (of the same type), mul or residual (same stride), apart from the rest */
    uint32_t*      status;        /* [device] 2 words, or NULL: ANSZP_ST_BAD_DESC for an id beyond the adapters, whose row has none then, counted */
    void*          workspace;     /* [device] anszp_adapt_workspace_bytes, 16-byte aligned, in use until the call is done */
    uint64_t       workspace_bytes;
    uint64_t       rows, cols;    /* < 2^28, < 2^31, may be 0; fewer than 2^24 tiles of 64 x 32 together, rows * (rank up to a multiple of 32) < 2^33; with x or a
                                   * of fewer than 16 bytes rows * rank <= 2^32 - 256, with such a b rows * cols */
    uint64_t       x_stride, a_stride, a_row_stride, b_stride, b_row_stride, base_stride, mul_stride, residual_stride, out_stride;
    uint32_t       adapters;      /* < 2^24, may be 0                                                */
    uint32_t       k;             /* 1 .. 2^30                                                       */
    uint32_t       rank;          /* 1 .. 128                                                        */
    uint32_t       x_dtype;       /* ANSZP_OUT_BF16 or ANSZP_I8                                      */
    uint32_t       base_dtype;    /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    uint32_t       out_dtype;     /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    uint32_t       activation;    /* ANSZP_FN_*                                                      */
} anszp_adapt_args_t;
/* [host only] Bytes of workspace a call takes (0: none); reads sizes only, no pointers. */
uint64_t anszp_adapt_workspace_bytes(const anszp_adapt_args_t* args);
/* Errors: E_NULL, E_RANGE (also for a workspace that is too small, and for an output that meets an operand it may not), E_HIP. */
int anszp_adapt(const anszp_adapt_args_t* args, void* hip_stream);

/* The next token of each row from its logits l.  In the order of falling l (equal ones: the lower token first), with w = exp((l - max l) /
 * temperature), a row keeps the shortest of these beginnings: its first top_k tokens (0 and below: all); of those the shortest that has at least top_p of
 * their weight, one token at least (1 and above: all); those with w >= min_p (0: all; 1 and above: those equal to the first).  It draws the
 * first token at which the sum of the kept weights, in the same order, passes uniform * (all of it); uniforms are in [0, 1), others
 * count as the nearest.  A temperature of 0 draws the first token.  Each setting is one number for all rows, or one for each.  A row that holds a NaN, or
 * nothing above -infinity, or has a temperature below 0 or NaN, has token -1 and a chance of 0; +infinities share a row alone.
 * Weights are good to 5e-12 of each and 2^-44 of the largest (2^-62 times the vocabulary where that is more), their sums exact; a token below
 * 2^-44 of the first weighs nothing.  No result depends on the order of additions. */
typedef struct {
    const void*    logits;        /* [device] rows x vocabulary of dtype                             */
    const float*   uniforms;      /* [device] rows                                                   */
    const float*   temperatures;  /* [device] rows, or NULL: `temperature` for all; likewise the next three */
    const int32_t* top_ks;
    const float*   top_ps;
    const float*   min_ps;
    int64_t*       tokens;        /* [device] rows                                                   */
    float*         chances;       /* [device] rows: what part of the kept weight the token has, or NULL */
    uint64_t       rows;          /* < 2^31, may be 0                                                */
    uint64_t       logits_stride;
    uint32_t       vocabulary;    /* 1 .. 2^24                                                       */
    uint32_t       dtype;         /* ANSZP_OUT_F32 or ANSZP_OUT_BF16                                 */
    float          temperature;   /* >= 0                                                            */
    int32_t        top_k;         /* >= 0                                                            */
    float          top_p, min_p;  /* >= 0                                                            */
} anszp_sample_args_t;
/* Errors: E_NULL, E_RANGE, E_HIP. */
int anszp_sample(const anszp_sample_args_t* args, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ANSZP_H */
