// The key/value cache in 8 bits (include/bd_kernels.h): layout of a page, arithmetic of its scales, rules on rows and on what a
// row sees, and the plan of the attention's launch, shared by host and device.
#pragma once
#include "../../include/bd_kernels.h"
#include "common.h"

namespace bd {

constexpr int kv8_e_min = -117, kv8_e_max = 119;   // 2^-9 2^-117 is the smallest normal fp32 number, 448 2^119 fits

// Byte of token t (0..31), dimension d in a page's head: keys, and values (from byte 32 D on).  Sixteen bytes of lane l = 16 g + i
// are two A-operands of the 16x16x32 product: for the keys of tile t8, row i, two k-steps; for the values rows i of two
// d-tiles over tokens 8 g ..  The keys' rows are dealt out as in the bf16 cache (kp_index): the two tiles of scores line up with the operand of the second
// product.  The values' rows put the eight results of a lane's tile pair on neighbouring dimensions: one 16-byte store.
__host__ __device__ inline int kv8_k_byte(int tok, int d, int D) {
  const int t8 = (tok >> 2) & 1, i = (tok >> 3) * 4 + (tok & 3);
  return ((t8 * (D >> 6) + (d >> 6)) * 4 + ((d >> 4) & 3)) * 256 + i * 16 + (d & 15);
}
__host__ __device__ inline int kv8_v_byte(int tok, int d) {
  return ((d >> 5) * 4 + (tok >> 3)) * 256 + (((d >> 3) & 3) * 4 + (d & 3)) * 16 + ((d >> 2) & 1) * 8 + (tok & 7);
}

// Smallest e >= kv8_e_min with amax <= 448 2^e; bits: those of a finite amax >= 0.  (448 = 1.75 2^8)
__host__ __device__ inline int kv8_exponent_of(uint32_t bits) {
  const int x = (int)(bits >> 23) - 127;
  const int e = (bits & 0x7FFFFFu) <= 0x600000u ? x - 8 : x - 7;
  return e < kv8_e_min ? kv8_e_min : e;
}
// The same as the cache has it, at most kv8_e_max.
__host__ __device__ inline int kv8_exponent(uint32_t bits) {
  const int e = kv8_exponent_of(bits);
  return e > kv8_e_max ? kv8_e_max : e;
}
// The exponent that a scale word's byte stands for; bytes that no write leaves count as the nearest that one can.
__host__ __device__ inline int kv8_byte_exponent(uint32_t byte) {
  const int e = (int)(byte & 255u) - 127;
  return e < kv8_e_min ? kv8_e_min : e > kv8_e_max ? kv8_e_max : e;
}
constexpr uint32_t kv8_v_nan = 1u << 16;

// Rows of a sequence: `rows` of at most M at positions from `first` on, within max_blocks pages.  False: left out, and reported.
__host__ __device__ inline bool kv8_rows_ok(int first, int rows, int M, int max_blocks) {
  return first >= 0 && rows >= 0 && rows <= M && (int64_t)first + rows <= (int64_t)max_blocks * BD_KV8_PAGE;
}

// Division of 0 <= x < 2^31 by the same d >= 1 every time: x/d = (floor(x mul / 2^32) + x) / 2^shift with 2^shift >= d > 2^(shift - 1) and
// mul = floor(2^32 (2^shift - d) / d) + 1 (mul + 2^32 exceeds 2^(32 + shift)/d by at most 1, too little to reach the next quotient).
struct Kv8Div { uint32_t mul, shift; };
inline Kv8Div kv8_div(int d) {
  Kv8Div v{0, 0};
  while (((int64_t)1 << v.shift) < d) ++v.shift;
  v.mul = (uint32_t)(((((uint64_t)1 << v.shift) - (uint64_t)d) << 32) / (uint64_t)d + 1);
  return v;
}
__host__ __device__ inline int kv8_quotient(int x, Kv8Div d) {
  return (int)(((uint32_t)(((uint64_t)(uint32_t)x * d.mul) >> 32) + (uint32_t)x) >> d.shift);
}

// What rows r0 .. r1 (positions n + r0 .. n + r1) of a sequence with `rows` rows can see: the blocks of the first `sinks`
// positions, then those from the window's start to the last visible key: block number idx of `count` is idx for
// idx < sink_blocks, and first_block + idx - sink_blocks from there.  [clear_lo, clear_hi): blocks from the window all of whose keys every
// row sees; clear_sinks: so many of the sink blocks too.
struct Kv8Span { int sink_blocks, first_block, count, clear_lo, clear_hi, clear_sinks; };
__host__ __device__ inline Kv8Span kv8_span(int n, int rows, int r0, int r1, int mode, int window, int sinks) {
  Kv8Span s;
  const int end = mode == BD_MODE_CAUSAL ? n + r1 + 1 : n + rows;                 // keys from here on are invisible to all
  const int all = mode == BD_MODE_CAUSAL ? n + r0 + 1 : n + rows;                 // keys up to here are not too late for any
  const int lo = window > 0 && n + r0 >= window ? n + r0 - window + 1 : 0;        // window of the first row, of the last
  const int hi = window > 0 && n + r1 >= window ? n + r1 - window + 1 : 0;
  const int snk = window > 0 ? (sinks < lo ? sinks : lo) : 0;
  s.first_block = lo / 32;
  s.sink_blocks = (snk + 31) / 32;
  if (s.sink_blocks > s.first_block) s.sink_blocks = s.first_block;
  s.count = s.sink_blocks + (end + 31) / 32 - s.first_block;
  s.clear_lo = window > 0 && hi <= sinks ? s.first_block : (hi + 31) / 32;
  s.clear_hi = all / 32;
  const int early = sinks < all ? sinks : all;
  s.clear_sinks = early / 32;
  return s;
}
__host__ __device__ inline bool kv8_sees(int p, int key, int end, int mode, int window, int sinks) {
  return key < end && (mode != BD_MODE_CAUSAL || key <= p) && (window <= 0 || p - key < window || key < sinks);
}

// Launch plan of the attention.  An item is a tile of 16 columns (column = row * G + head of the group) of a (sequence, kv head).
enum class Kv8Form { walk, wide, stream };   // one tile, eight wavefronts; two tiles, four; one tile, four, past the caches
struct Kv8Plan {
  Kv8Form form;
  int tiles;        // of a (sequence, kv head)
  int JT;           // tiles of a workgroup
  int groups;       // workgroups for a unit: (sequence, kv head, chunk)
  int chunks;       // workgroups that share out the blocks of a group, at most
  int runs, run_len;     // parts of a unit's groups that go to an XCD each, and their length
  int64_t part_floats;   // workspace: unnormalised partial results, [sequence][kv head][tile][chunk]
};
constexpr int kv8_chunk_blocks = 16, kv8_least_blocks = 64, kv8_cus = 256;
constexpr int64_t kv8_once_bytes = (int64_t)96 << 20;
inline int64_t kv8_items(int n_seq, int M, int n_q, int n_kv) { return (int64_t)n_seq * n_kv * (((int64_t)M * (n_q / n_kv) + 15) / 16); }
// Chunks for so many blocks, if there is room for them.
__host__ __device__ inline int64_t kv8_parts(int64_t blocks) { return blocks < kv8_least_blocks ? 1 : (blocks + kv8_chunk_blocks / 2) / kv8_chunk_blocks; }
inline Kv8Plan kv8_plan(int n_seq, int M, int n_q, int n_kv, int D, int max_blocks, int window, int sinks) {
  Kv8Plan p{};
  p.tiles = (int)(((int64_t)M * (n_q / n_kv) + 15) / 16);
  const int64_t items = kv8_items(n_seq, M, n_q, n_kv);
  int64_t blocks = max_blocks;
  if (window > 0) {
    const int64_t w = ((int64_t)window + M + 62) / 32 + 1 + ((int64_t)sinks + 31) / 32;
    if (w < blocks) blocks = w;
  }
  // (Times in us of passes one after another in a captured graph, with the joining kernel where there is one, at the clock that lasting work runs at.
  // Cold: other inputs from pass to pass, 500 MB in all; warm: the same ones, which the last-level cache keeps.)
  // One tile and page lists with room for more than the last-level cache keeps from one step to the next: every block has one reader, so its loads
  // pass the caches by; four wavefronts, three workgroups a CU.  Stream / walk, cold and warm: 64 sequences up to 8192 30.8 / 37.4 and 29.2 / 27.9, 8 up to
  // 32768 21.0 / 23.2 and 19.2 / 19.7, 32 up to 8192 20.9 / 23.6 and 19.0 / 20.4, 256 up to 4096 50.5 / 57.8 cold; below the limit, 16 up to 8192,
  // 14.1 / 15.0 and 13.0 / 12.2.  The lengths are on the device only, so it is the lists' room that counts, whatever the sequences hold.
  // More items than CUs: two tiles share each block that a wavefront loads and widens; four wavefronts, two workgroups a CU.
  // Else one tile and eight wavefronts, for the shortest walk.  Wide / walk: 256 items behind 2048 keys 16.3 / 11.2, 384 16.9 / 18.9, 512 17.5
  // / 20.0, 1024 rows (1024 items) behind 7168 keys 68.6 / 95.2.
  const bool once = p.tiles == 1 && (int64_t)n_seq * n_kv * blocks * 64 * D >= kv8_once_bytes;
  p.form = once ? Kv8Form::stream : items > kv8_cus && p.tiles > 1 ? Kv8Form::wide : Kv8Form::walk;
  p.JT = p.form == Kv8Form::wide ? 2 : 1;
  p.groups = ceil_div(p.tiles, p.JT);
  // Fewer items than CUs (stream: than two workgroups for each): the blocks of an item in chunks, as far as there are CUs for them.
  // 1 / 2 / 4 / 8 / 16 chunks: one row behind 8192 keys 25.9 / 18.2 / 12.6 / 10.1 / 9.2, behind 2048 9.8 / 10.0 / 8.7, behind 1500 8.5 / 9.4, behind
  // 1024 7.2 / 8.6, 32 rows behind 1024 7.6 / 9.0; 256 items behind 2048 keys 11.2 / 18.2; 64 sequences up to 8192 in stream 48.9 / 33.9 / 31.1 / 35.4 cold.  One
  // row behind 262144 keys, 64 / 128 / 256 chunks: 33.0 / 30.2 / 35.5; behind 65536, 64 / 128: 13.9 / 16.4.
  // Here too the lists' room counts: sequences far shorter than their lists use one chunk, but pay for the others' workgroups and the joining kernel.  Lists of
  // 35 / 128 / 1024 pages: 32 rows behind 1024 keys 7.6 / 10.1 / 9.9, 8 sequences up to 1024 7.3 / 9.7 (256 pages) / 14.2 (stream).
  int64_t c = kv8_parts(blocks);
  const int64_t room = (once ? 2 : 1) * kv8_cus / items;
  if (c > room) c = room;
  if (c > (once ? 128 : 64)) c = once ? 128 : 64;
  p.chunks = c < 1 ? 1 : (int)c;                        // (no room for a second workgroup: 1)
  p.part_floats = p.chunks > 1 ? items * p.chunks * (16 * D + 32) : 0;
  const int64_t units = (int64_t)n_seq * n_kv * p.chunks;
  p.runs = units >= 8 ? 1 : (int)((8 + units - 1) / units);
  if (p.runs > p.groups) p.runs = p.groups;
  p.run_len = ceil_div(p.groups, p.runs);
  return p;
}
// Chunks that a group of `count` blocks really uses.
__host__ __device__ inline int kv8_chunks_used(int count, int chunks) {
  const int c = (int)kv8_parts(count);
  return c < chunks ? c : chunks;
}

}  // namespace bd
