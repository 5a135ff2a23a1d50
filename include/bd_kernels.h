/*
 * bd_kernels.h - kernel-level entry points of the block-denoising library.
 *
 * These expose block-causal attention on caller-provided tensors (the attention kernel that forwards of more than
 * 32 rows and the prompt pass run), attention on a paged cache in 8 bits with what fills it, per-kernel-class timing of a context, the in-kernel phase trace and the time of
 * the weight stream alone, so that tests can check one operation against the oracle and the benchmark can price
 * one kernel against its roofline.  The entry points themselves are not on the decode path.  Return codes as in
 * bd.h.
 */
#ifndef BD_KERNELS_H_
#define BD_KERNELS_H_

#include <stdint.h>

#include "bd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Block-causal grouped-query attention (Sec. 3.3 mask rules; Alg. 1 draft / verify masks) on explicit
 * operands: dev_q fp32 [M, n_q, D] (already rotated), dev_k / dev_v fp32 [n_prefix + M, n_kv, D] (prefix
 * keys first, then the block's own); all rounded to bf16 inside.  dev_out fp32 [M, n_q*D].
 * mode BD_MODE_BIDIR / BD_MODE_CAUSAL.  M <= 64, D in {64, 128}.  Allocates its working buffers per call
 * and synchronises the stream.  iters > 1 repeats the kernels and *avg_ms (host, may be NULL) receives the
 * mean time of one run. */
int bd_k_attention(void* hip_stream, const float* dev_q, const float* dev_k, const float* dev_v, int n_prefix, int M,
                   int n_q, int n_kv, int D, int mode, float* dev_out, int iters, float* avg_ms);

/* The same operation for callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): same arguments, layouts and result as bd_k_attention with
 * iters = 1, but every working buffer (packed K/V, bf16 Q, packed bf16 result) lives in one static device
 * array of BD_K_ATTENTION_STATIC_BYTES bytes that each GPU the library runs on holds until the process
 * ends.  The call allocates and frees nothing, records no memset node, only enqueues on hip_stream and
 * does not synchronise.  A shape whose working buffers exceed the array returns BD_E_CAPACITY (the text
 * from bd_last_error() names both sizes); bad arguments return BD_E_ARG as for bd_k_attention.  All calls
 * on one GPU share the array: calls that overlap in time on one GPU race, even on different streams. */
#define BD_K_ATTENTION_STATIC_BYTES (32u << 20)
int bd_k_attention_static(void* hip_stream, const float* dev_q, const float* dev_k, const float* dev_v, int n_prefix,
                          int M, int n_q, int n_kv, int D, int mode, float* dev_out);

/* Per-kernel-class timing of a context's forwards: enable brackets every launch with HIP events on
 * the context's stream (and drops earlier samples); read sums the elapsed time of one class. */
int bd_k_profile(bd_ctx* ctx, int enable);
int bd_k_profile_read(bd_ctx* ctx, int kclass, double* total_ms, int* launches);
int bd_k_class_count(void);
const char* bd_k_class_name(int kclass);
/* Algorithmic HBM bytes one launch of that class moves at the current cache length (weights of the
 * GEMM, or the layer's cached K/V for the attention); 0 for classes that stream nothing. */
int64_t bd_k_class_bytes(const bd_ctx* ctx, int kclass);

/* Measurement: time of reading the decoder layers' weight stream of one forward with no consumer, hand-over or barrier
 * (each wavefront its own contiguous share, as the streaming kernel's producers read it): mean of `repeats` launches
 * in milliseconds to *host_ms, the bytes read per launch to *host_bytes.  Synchronises the stream. */
int bd_k_stream_floor(bd_ctx* ctx, int repeats, double* host_ms, int64_t* host_bytes);

/* Test hook: raises the context's device-side error flag, as a forward kernel does when one of its bounded waits
 * gives up.  Every later forward kernel then returns at once (no kernel waits for anything), bd_status and the calls
 * that read a result back (bd_speculative_step, bd_quad_step) return BD_E_HIP, and the context stays unusable. */
int bd_k_raise_device_error(bd_ctx* ctx);

/* Phase trace of the forward kernel: with enable != 0 every workgroup stores a 100 MHz timestamp at each
 * phase boundary of the next forwards (start; then per layer: QKV done, barrier, attention done, barrier,
 * O done, barrier, gate/up done, barrier, down done, barrier; then LM head done, barrier).  read copies
 * the last forward's [n_wg][per_wg] table to host memory (capacity in entries).
 * While the trace is on, calls that would run a forward of 17 to 32 rows through the streaming kernel are refused
 * (BD_E_STATE): traced forwards of that size of experimental builds ran out of a bounded wait, cause not known. */
int bd_k_trace(bd_ctx* ctx, int enable);
int bd_k_trace_read(bd_ctx* ctx, unsigned long long* host_out, int capacity, int* n_wg, int* per_wg);

/* ---- attention on a key/value cache in 8 bits -----------------------------------------------------------------------
 *
 * What one decoder layer's attention needs where the cache has to be small: rotary positions (bd_k_rope), new keys and values
 * into the cache (bd_k_kv8_write), attention of the new rows on it (bd_k_kv8_attention), and the cache's values back
 * (bd_k_kv8_read).  Several sequences at once, each with its own length and page list.  All pointers are device memory of the
 * current device, owned by the caller, unless they are called host; nothing is allocated, kept, copied to the host or
 * synchronised: a call enqueues its kernels on hip_stream and can be captured into a graph (lengths, row counts and
 * page lists are read when the kernels run, so a replay follows what they hold then).
 *
 * The cache.  A pool of pages of 32 positions (BD_KV8_PAGE); a page holds, for each kv head, e4m3 codes (OCP e4m3fn) of 32 keys and
 * of 32 values, each with one scale 2^e.  Block i of a sequence (positions 32 i .. 32 i + 31) lives in page pages[i] of its list.
 *   dev_codes   uint8 [n_pages][n_kv][64 D], 16-byte aligned.  Of a page's head first the keys: byte ((t D/64 + c) 4 + g) 256 + 16 i + b
 *               is token 8 (i / 4) + 4 t + i % 4, dimension 64 c + 16 g + b; then, from byte 32 D, the values: byte
 *               (c 4 + g) 256 + 16 i + 8 u + x is token 8 g + x, dimension 32 c + 8 (i / 4) + 4 u + i % 4.
 *   dev_scales  uint32 [n_pages][n_kv]: e + 127 of the keys in bits 0..7, of the values in bits 8..15, bit 16 set where the codes of the
 *               values hold a NaN.
 *   dev_pages   int32 [n_seq][max_blocks].  A page that a call writes may be on one list only, and there once; others may be shared.
 *   dev_len     int32 [n_seq], positions that the sequence holds before the rows of the call.  No call changes it.
 *   dev_status  NULL, or one int32 to which kernels OR BD_KV8_BAD_ROWS (a length or row count that is negative, more rows than M, or positions
 *               past max_blocks pages: the sequence is left out, its outputs stay as they were) and BD_KV8_BAD_PAGE (a page index outside the
 *               pool: nothing is read or written there; to the attention its keys are invisible).
 * D 64 or 128; n_kv 1 .. 4096, n_pages n_kv 1 .. 2^31, n_seq 1 .. 65535, max_blocks 1 .. 2^25, M 1 .. 2^22 and M n_kv
 * at most 2^28, else BD_E_ARG.  Outputs may not overlap what a call reads, unless it says so.
 *
 * Rows.  A tensor of rows is [n_seq][M][heads][D] with heads and dimensions contiguous and the strides between sequences and
 * between rows given in elements (so a slice of a fused projection's output can be passed).  Rows are read and written 16 bytes at a
 * time: pointers have to be 16-byte aligned and strides multiples of 16 bytes, not negative and, where rows are written, not less than a row, else
 * BD_E_ARG (the stride of a dimension of one is not looked at).  dev_rows (int32 [n_seq], NULL = M everywhere): rows of the sequence in this
 * call, 0 .. M; the others are padding, never read (nor are their outputs written).  Row r of sequence s is position dev_len[s] + r. */
#define BD_KV8_PAGE 32
enum { BD_KV8_BAD_ROWS = 1, BD_KV8_BAD_PAGE = 2 };
typedef struct {
  uint8_t* dev_codes;
  uint32_t* dev_scales;
  const int32_t* dev_pages;
  const int32_t* dev_len;
  int32_t* dev_status;
  int32_t n_pages, n_kv, D, n_seq, max_blocks;
} bd_kv8;

/* New rows of keys and values (already rotated; dtype BD_BF16 or BD_F32) into the cache at positions dev_len[s] ...  The scale of a block, for its keys
 * and its values and each head: the smallest e in [-117, 119] with max|x| <= 448 2^e over the block's new finite rows; where the block holds
 * positions from before, not less than it was, and these are encoded again (code 2^(e_old - e)).  A code is the nearest
 * e4m3 number to x 2^-e, ties to even; infinities and what exceeds 448 saturate, a NaN stays one.  Positions of a touched
 * block behind the sequence's last row become 0, whatever they held. */
int bd_k_kv8_write(void* hip_stream, const bd_kv8* cache, const void* dev_k, int64_t k_seq_stride, int64_t k_row_stride, const void* dev_v,
                   int64_t v_seq_stride, int64_t v_row_stride, int dtype, int M, const int32_t* dev_rows);

/* The cache's values: positions dev_from[s] .. dev_from[s] + rows - 1 of each sequence (dev_from NULL: from 0) to rows 0 .. of dev_k_out and dev_v_out
 * (dtype BD_BF16 or BD_F32: code times scale is exact in both).  cache->dev_len is not looked at. */
int bd_k_kv8_read(void* hip_stream, const bd_kv8* cache, const int32_t* dev_from, int M, const int32_t* dev_rows, int dtype, void* dev_k_out,
                  int64_t k_seq_stride, int64_t k_row_stride, void* dev_v_out, int64_t v_seq_stride, int64_t v_row_stride);

/* Grouped-query attention of the rows of dev_q (bf16, n_q heads, n_q a multiple of n_kv) on the cache, which holds the rows' own keys and values already
 * (bd_k_kv8_write before): out = softmax(scale q k) v over the keys a row sees, to dev_out (bf16).  Row r at position p = dev_len[s] + r sees key j
 * where j < dev_len[s] + rows, and j <= p with BD_MODE_CAUSAL (any j with BD_MODE_BIDIR), and, with window > 0, where
 * p - j < window or j < sinks: the last `window` positions and the first `sinks` ones (window 0: no window, sinks is then not looked at).
 * A row that sees no key (all of its pages lie outside the pool) becomes NaN.  scale > 0 and at most 2^127, or 0 for 1/sqrt(D); n_q 1 .. 65536 and
 * n_seq n_kv ceil(M n_q / n_kv / 16) at most 2^22.  Products in bf16 (codes and queries exactly, the weights of the softmax rounded to it), sums and softmax in
 * fp32: scores, and values times 256 times the keys a row sees, have to stay below 2^127.
 * The launch goes by max_blocks, since the lengths are on the device: lists far longer than their sequences are answered right, but a call of a few
 * microseconds takes 2 to 7 more (35 pages and 1024 for 32 rows behind 1024 keys: 7.6 and 9.9).
 * dev_workspace: bd_k_kv8_attention_workspace bytes (may be 0: NULL then), 16-byte aligned, free for others when the call has run;
 * calls that may overlap in time need one each; too few bytes are BD_E_CAPACITY (bd_last_error says how many it takes).  The results do not depend on what it holds, and are the same on every run. */
int bd_k_kv8_attention(void* hip_stream, const bd_kv8* cache, const void* dev_q, int64_t q_seq_stride, int64_t q_row_stride, int n_q, int M,
                       const int32_t* dev_rows, int mode, int window, int sinks, float scale, void* dev_out, int64_t out_seq_stride,
                       int64_t out_row_stride, void* dev_workspace, int64_t workspace_bytes);
/* Bytes of workspace of such a call (host only, no device needed), or BD_E_ARG. */
int64_t bd_k_kv8_attention_workspace(const bd_kv8* cache, int n_q, int M, int window, int sinks);

/* Rotary positions.  A plan says what is turned: pairs of the first rotary_dim dimensions of a head (even, 2 .. D) by angle position * inv_freq[i], pair i being
 * dimensions (i, i + rotary_dim/2) with BD_ROPE_HALF or (2 i, 2 i + 1) with BD_ROPE_INTERLEAVED; the turned pair is multiplied by `amplitude`.
 * bd_k_rope_plan fills one (host only).  inv_freq[i] = theta^(-2 i/rotary_dim), and for contexts `factor` times as long as the
 * model was trained on (`trained` positions):
 *   BD_ROPE_PLAIN   as it is (factor and trained are not looked at);
 *   BD_ROPE_LINEAR  inv_freq / factor;
 *   BD_ROPE_BASE    theta factor^(rotary_dim/(rotary_dim - 2)) in place of theta (rotary_dim > 2): the fastest pair stays, the slowest is stretched by factor;
 *   BD_ROPE_PARTS   inv_freq (w + (1 - w)/factor), w = clamp((n - 1)/31, 0, 1), n = trained inv_freq/(2 pi) the turns within
 *                   the trained length; amplitude 1 + 0.1 ln(factor) (1 in the other kinds).
 * theta > 1, factor >= 1, trained >= 1, all finite, else BD_E_ARG.  Any other rule: fill the structure by hand. */
enum { BD_ROPE_HALF = 0, BD_ROPE_INTERLEAVED = 1 };
enum { BD_ROPE_PLAIN = 0, BD_ROPE_LINEAR = 1, BD_ROPE_BASE = 2, BD_ROPE_PARTS = 3 };
typedef struct {
  int32_t D, rotary_dim, layout;   /* D 64 or 128 */
  float amplitude;
  double inv_freq[64];             /* radians per position */
} bd_rope;
int bd_k_rope_plan(bd_rope* host_out, int D, int rotary_dim, int layout, double theta, int scaling, double factor, int trained);

/* Turns rows [n_seq][M][n_heads][D] (BD_BF16 or BD_F32; strides and alignment as above) from dev_x to dev_out, which may be dev_x itself with the same strides
 * (else the two may not overlap); dimensions from rotary_dim on are copied.  Row r of sequence s is at position dev_pos[s] + r (int32 [n_seq];
 * with M = 1 every row brings its own), dev_rows as above (a count outside 0 .. M is taken as the nearer end); n_heads 1 .. 65536, n_seq 1 .. 65535,
 * M 1 .. 2^22.  Angles in fp64, sines and products in fp32. */
int bd_k_rope(void* hip_stream, const bd_rope* plan, const void* dev_x, int64_t x_seq_stride, int64_t x_row_stride, void* dev_out,
              int64_t out_seq_stride, int64_t out_row_stride, int dtype, int n_heads, int n_seq, int M, const int32_t* dev_pos,
              const int32_t* dev_rows);

#ifdef __cplusplus
}
#endif
#endif /* BD_KERNELS_H_ */
