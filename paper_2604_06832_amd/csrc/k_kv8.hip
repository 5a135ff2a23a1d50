// Attention on a key/value cache in 8 bits, and what fills and reads it (include/bd_kernels.h: bd_rope, bd_kv8).
#include <cmath>

#include "kv8.h"
#include "launch.h"
#include "stream_fwd.h"

namespace bd {
namespace {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef short s16x2 __attribute__((ext_vector_type(2)));

struct Kv8Rows {          // a call's rows: their positions and how many of each sequence are real
  const int* first; const int* rows; int M;
};

// First position and number of rows of sequence s; false (and reported) where they make no sense.
__device__ inline bool kv8_take(const bd_kv8& c, const Kv8Rows& r, int s, int& first, int& rows) {
  first = 0;
  rows = r.M;
  if (r.first != nullptr || r.rows != nullptr) {       // two scalar loads and one wait, whichever is given
    typedef const __attribute__((address_space(4))) int* Ints;
    int x = ((Ints)(r.first != nullptr ? r.first : r.rows))[s], y = ((Ints)(r.rows != nullptr ? r.rows : r.first))[s];
    asm volatile("" : "+s"(x), "+s"(y));
    if (r.first != nullptr) first = x;
    if (r.rows != nullptr) rows = y;
  }
  if (kv8_rows_ok(first, rows, r.M, c.max_blocks)) return true;
  if (c.dev_status != nullptr && threadIdx.x == 0) atomicOr(c.dev_status, BD_KV8_BAD_ROWS);
  return false;
}
// The page, or -1 (and reported) where it lies outside the pool.
__device__ inline int kv8_in_pool(const bd_kv8& c, int page) {
  if ((unsigned)page < (unsigned)c.n_pages) return page;
  if (c.dev_status != nullptr) atomicOr(c.dev_status, BD_KV8_BAD_PAGE);
  return -1;
}
// Page of block kb of sequence s.
__device__ inline int kv8_page(const bd_kv8& c, int s, int kb) { return kv8_in_pool(c, c.dev_pages[(size_t)s * c.max_blocks + kb]); }

__device__ inline float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four e4m3 codes of y (already scaled), to nearest, ties to even.
__device__ inline uint32_t encode4(const float* y) {
  float z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = fabsf(y[i]) > 448.f ? copysignf(448.f, y[i]) : y[i];   // (a NaN stays: the comparison is false)
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], w, true);
}
__device__ inline void decode4(uint32_t w, float* y) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  y[0] = a[0]; y[1] = a[1]; y[2] = b[0]; y[3] = b[1];
}

// High bit of each byte that holds a NaN.
__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

template <typename T, int N> struct alignas(N * sizeof(T)) Pack { T x[N]; };
template <typename T> __device__ inline float to_f32(T x);
template <> __device__ inline float to_f32<float>(float x) { return x; }
template <> __device__ inline float to_f32<u16>(u16 x) { return bf16_bits_to_f32(x); }
template <typename T> __device__ inline T from_f32(float x);
template <> __device__ inline float from_f32<float>(float x) { return x; }
template <> __device__ inline u16 from_f32<u16>(float x) {
  union { __bf16 h; u16 u; } v;                       // (the conversion keeps NaN and infinity)
  v.h = (__bf16)x;
  return v.u;
}

// ---- write and read -------------------------------------------------------------------------------------------------------
// One wavefront per (block, head, keys or values), two blocks with heads of 64.  A lane has a patch of eight tokens (8 g ..) by eight dimensions:
// rows move 16 bytes a lane and a token (256 or 128 contiguous bytes a row), and of the page the lane owns whole 16-byte pieces, the keys' after
// an exchange with its neighbour, the values' after transposing bytes in registers.  Nothing crosses the wavefront: the
// block's maximum is a reduction over its lanes.  Reading is bound by the rows' bytes: 16 contexts of up to 8000 rows (2 heads of
// 128, bf16) 33.7 us, 168 MB at 5.0 TB/s (a large copy 5.15).  Eight prompts of up to 4096: read 8.7 us, 40 MB at 4.6 TB/s; written 11.5 us, 40 MB at 3.5 TB/s (a
// copy of the same bytes 7.7): every wavefront is resident at once and loads, then reduces, then stores, so the first loads' 4 us are added whole.  One block
// 3 us read, 4 us written, its launch.  Stores that pass the caches by (both together 23.5 us for 21.1 then) and the keys' codes 16 bytes a lane bring nothing.
struct Kv8CopyArgs {
  bd_kv8 c;
  Kv8Rows r;
  void* x[2];                                          // keys, values
  int64_t seq_stride[2], row_stride[2];
  Kv8Div by_heads;                                     // divisions by 2 n_kv
};

template <int D>
struct Kv8Patch {
  int lane, h, kv, g, d;                               // head, keys or values, tokens 8 g .., dimensions d ..
  int kb, lo, hi, first;                               // block; tokens [lo, hi) of the block are the call's, row r is token r - first
  bool on;                                             // there is something to do, and a page for it
  size_t ph;                                           // page and head
  uint8_t* codes;
  __device__ inline int k_byte(int t) const { return kv8_k_byte(t, d, D); }
  __device__ inline int v_byte() const { return 32 * D + kv8_v_byte(8 * g, d); }       // 64 bytes: piece r holds dimensions d + r and d + 4 + r
};
// Where the patch lies; false (for the whole wavefront): nothing to do.
template <int D>
__device__ inline bool kv8_patch(const Kv8CopyArgs& a, Kv8Patch<D>& p, int& s) {
  constexpr int per = D / 8, U = 128 / D;              // lanes of a row, blocks of a wavefront
  p.lane = threadIdx.x & 63;
  const int u = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int pair = kv8_quotient(u, a.by_heads), hk = u - pair * 2 * a.c.n_kv;
  p.h = hk >> 1;
  p.kv = hk & 1;
  p.g = (p.lane / per) & 3;
  p.d = (p.lane % per) * 8;
  s = blockIdx.z;
  int n, rows;
  if (!kv8_take(a.c, a.r, s, n, rows)) return false;
  const int kb = n / 32 + pair * U + p.lane / (4 * per);
  p.first = n - kb * 32;
  p.lo = max(p.first, 0);
  p.hi = (int)min((int64_t)n + rows - (int64_t)kb * 32, (int64_t)32);
  p.on = p.hi > p.lo;
  p.kb = kb;
  return __builtin_amdgcn_ballot_w64(p.on) != 0ull;
}
// Its page.
template <int D>
__device__ inline void kv8_patch_page(const Kv8CopyArgs& a, Kv8Patch<D>& p, int s) {
  const int page = p.on ? kv8_page(a.c, s, p.kb) : -1;
  p.on = page >= 0;
  p.ph = (size_t)max(page, 0) * a.c.n_kv + p.h;
  p.codes = a.c.dev_codes + p.ph * (64 * D);
}

// 4 x 4 bytes: byte j of word i and byte i of word j change places.
__device__ inline void transpose4(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  const uint32_t t0 = __builtin_amdgcn_perm(b, a, 0x05010400u), t1 = __builtin_amdgcn_perm(b, a, 0x07030602u);      // a0 b0 a1 b1, a2 b2 a3 b3
  const uint32_t t2 = __builtin_amdgcn_perm(d, c, 0x05010400u), t3 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  a = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
  b = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
  c = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
  d = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
}
// The values' patch, w[token][dimensions d .. d + 3 or d + 4 .. d + 7], to and from the page's order.
__device__ inline void transpose_patch(uint32_t (&w)[8][2]) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    transpose4(w[0][u], w[1][u], w[2][u], w[3][u]);
    transpose4(w[4][u], w[5][u], w[6][u], w[7][u]);
  }
}
__device__ inline void load_values(const uint8_t* from, uint32_t (&w)[8][2]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint4 v = reinterpret_cast<const uint4*>(from)[r];
    w[r][0] = v.x; w[4 + r][0] = v.y; w[r][1] = v.z; w[4 + r][1] = v.w;
  }
  transpose_patch(w);
}

// Largest of x over the 64 lanes, or over each half of them.
template <bool HALVES>
__device__ inline uint32_t lanes_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, true));       // rotations inside rows of 16 lanes
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xF, 0xF, true));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xF, 0xF, true));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xF, 0xF, true));
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)r[0], (uint32_t)r[1]);
  if constexpr (HALVES) return x;
  const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)h[0], (uint32_t)h[1]);
}
// Eight elements of a row as they are loaded: their largest magnitude (bits of fp32; infinities and NaN count), and their codes at scale 2^e.
struct Row8bf16 {
  uint4 x;
  __device__ inline void load(const u16* p) { x = *reinterpret_cast<const uint4*>(p); }
  __device__ inline uint32_t largest() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    union { uint32_t u; u16x2 h; } a{x.x & 0x7FFF7FFFu}, b{x.y & 0x7FFF7FFFu}, c{x.z & 0x7FFF7FFFu}, d{x.w & 0x7FFF7FFFu};
    a.h = __builtin_elementwise_max(__builtin_elementwise_max(a.h, b.h), __builtin_elementwise_max(c.h, d.h));
    return max(a.u << 16, a.u & 0xFFFF0000u);
  }
  __device__ inline float at(int i) const {
    const uint32_t w = i < 2 ? x.x : i < 4 ? x.y : i < 6 ? x.z : x.w;
    return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
  }
  __device__ inline uint2 codes(float scale) const { return make_uint2(pair(x.x, x.y, scale), pair(x.z, x.w, scale)); }
  __device__ static inline uint32_t pair(uint32_t lo, uint32_t hi, float scale) {
    union { uint32_t u; bf16x2 v; } a{lo}, b{hi};
    union { s16x2 s; uint32_t u; } r{s16x2{0, 0}};
    r.s = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r.s, a.v, scale, false);
    r.s = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r.s, b.v, scale, true);
    return r.u;
  }
};
struct Row8f32 {
  float4 x, y;
  __device__ inline void load(const float* p) {
    x = reinterpret_cast<const float4*>(p)[0];
    y = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ inline float at(int i) const { return i < 4 ? (i < 2 ? (i ? x.y : x.x) : (i == 2 ? x.z : x.w)) : (i < 6 ? (i == 4 ? y.x : y.y) : (i == 6 ? y.z : y.w)); }
  __device__ inline uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(at(i)) & 0x7FFFFFFFu);
    return m;
  }
  __device__ inline uint2 codes(float scale) const { return make_uint2(four(x, scale), four(y, scale)); }
  __device__ static inline uint32_t four(const float4& v, float scale) {
    union { s16x2 s; uint32_t u; } r{s16x2{0, 0}};
    r.s = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r.s, v.x, v.y, scale, false);
    r.s = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r.s, v.z, v.w, scale, true);
    return r.u;
  }
};
template <typename T> struct Row8;
template <> struct Row8<u16> : Row8bf16 {};
template <> struct Row8<float> : Row8f32 {};

template <int D, typename T>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8CopyArgs a) {
  Kv8Patch<D> p;
  int s;
  if (!kv8_patch<D>(a, p, s)) return;
  const int64_t row_stride = a.row_stride[p.kv];
  const T* x = reinterpret_cast<const T*>(a.x[p.kv]) + s * a.seq_stride[p.kv] + p.h * D + p.d;
  // all loads before the first wait: the rows, then the page's word and the codes that stay
  Row8<T> row[8] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int t = 8 * p.g + i;
    if (p.on && t >= p.lo && t < p.hi) row[i].load(x + (t - p.first) * row_stride);
  }
  kv8_patch_page<D>(a, p, s);
  int e_old = kv8_e_min;
  const bool keeps = p.on && 8 * p.g < p.lo;           // positions from before among the patch's
  uint32_t old[8][2] = {};
  if (p.on && p.lo > 0) {
    e_old = kv8_byte_exponent(a.c.dev_scales[p.ph] >> (8 * p.kv));
    if (keeps && p.kv == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint2 v = *reinterpret_cast<const uint2*>(p.codes + p.k_byte(8 * p.g + i));
        old[i][0] = v.x; old[i][1] = v.y;
      }
    } else if (keeps) {
      load_values(p.codes + p.v_byte(), old);
    }
  }
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, row[i].largest());
  amax = lanes_max<D == 64>(amax);
  uint32_t w[8][2];
  int e;
  if (__builtin_amdgcn_ballot_w64(amax >= 0x7F800000u || kv8_exponent_of(amax) > kv8_e_max) == 0ull) {
    e = max(kv8_exponent(amax), e_old);
    const float scale = two_to(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint2 c = row[i].codes(scale);
      w[i][0] = c.x; w[i][1] = c.y;
    }
  } else {                                             // infinities, NaN, or more than the largest scale holds: the finite ones decide, an element at a time
    amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const uint32_t u = __float_as_uint(row[i].at(q)) & 0x7FFFFFFFu;
        amax = max(amax, u < 0x7F800000u ? u : 0u);
      }
    amax = lanes_max<D == 64>(amax);
    e = max(kv8_exponent(amax), e_old);
    const float down = two_to(-e);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float z[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) z[q] = row[i].at(4 * u + q) * down;
        w[i][u] = encode4(z);
      }
  }
  if (keeps) {
    const float again = two_to(max(e_old - e, -126));                       // (a smaller one would give 0 all the same)
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (8 * p.g + i < p.lo) {
          if (e != e_old) {
            float z[4];
            decode4(old[i][u], z);
#pragma unroll
            for (int q = 0; q < 4; ++q) z[q] *= again;
            w[i][u] = encode4(z);
          } else {
            w[i][u] = old[i][u];
          }
        }
  }
  uint8_t* word = reinterpret_cast<uint8_t*>(a.c.dev_scales + p.ph);        // keys and values have bytes of their own
  if (p.kv == 0) {
    const bool odd = p.lane & 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t got[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) got[u] = __builtin_amdgcn_mov_dpp(odd ? w[2 * k][u] : w[2 * k + 1][u], 0xB1, 0xF, 0xF, true);      // from lane ^ 1
      const uint4 v = odd ? make_uint4(got[0], got[1], w[2 * k + 1][0], w[2 * k + 1][1]) : make_uint4(w[2 * k][0], w[2 * k][1], got[0], got[1]);
      if (p.on) *reinterpret_cast<uint4*>(p.codes + kv8_k_byte(8 * p.g + 2 * k + odd, p.d & ~15, D)) = v;
    }
    if (p.on && (p.lane & (D / 2 - 1)) == 0) word[0] = (uint8_t)(e + 127);
  } else {
    uint32_t nan = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) nan |= nan_bytes(w[i][0]) | nan_bytes(w[i][1]);
    const unsigned long long nans = __builtin_amdgcn_ballot_w64(nan != 0u) >> (p.lane & (64 - D / 2));
    constexpr unsigned long long half = D == 128 ? ~0ull : 0xFFFFFFFFull;   // the lanes of one block
    transpose_patch(w);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (p.on) reinterpret_cast<uint4*>(p.codes + p.v_byte())[r] = make_uint4(w[r][0], w[4 + r][0], w[r][1], w[4 + r][1]);
    if (p.on && (p.lane & (D / 2 - 1)) == 0) {
      word[1] = (uint8_t)(e + 127);
      word[2] = (nans & half) != 0ull;
      word[3] = 0;
    }
  }
}

template <int D, typename T>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8CopyArgs a) {
  Kv8Patch<D> p;
  int s;
  if (!kv8_patch<D>(a, p, s)) return;
  kv8_patch_page<D>(a, p, s);
  if (!p.on || 8 * p.g >= p.hi || 8 * p.g + 8 <= p.lo) return;
  const int64_t row_stride = a.row_stride[p.kv];
  T* x = reinterpret_cast<T*>(a.x[p.kv]) + s * a.seq_stride[p.kv] + p.h * D + p.d;
  uint32_t w[8][2];
  if (p.kv == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint2 v = *reinterpret_cast<const uint2*>(p.codes + p.k_byte(8 * p.g + i));
      w[i][0] = v.x; w[i][1] = v.y;
    }
  } else {
    load_values(p.codes + p.v_byte(), w);
  }
  const float up = two_to(kv8_byte_exponent(a.c.dev_scales[p.ph] >> (8 * p.kv)));
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int t = 8 * p.g + i;
    float y[8];
    decode4(w[i][0], y);
    decode4(w[i][1], y + 4);
    if (t < p.lo || t >= p.hi) continue;
#pragma unroll
    for (int q = 0; q < 8 / N; ++q) {
      Pack<T, N> v;
#pragma unroll
      for (int e = 0; e < N; ++e) v.x[e] = from_f32<T>(y[q * N + e] * up);
      *reinterpret_cast<Pack<T, N>*>(x + (t - p.first) * row_stride + q * N) = v;
    }
  }
}

// ---- attention ----------------------------------------------------------------------------------------------------------
struct Kv8AttnArgs {
  bd_kv8 c;
  Kv8Rows r;
  const u16* q; u16* out;
  int64_t q_seq, q_row, o_seq, o_row;
  float* part;
  int n_q, mode, window, sinks;
  float c_log2;                 // scale * log2(e)
  int tiles, groups, chunks, runs, run_len, G;
  Kv8Div by_len, by_runs, by_chunks, by_kv, by_G;      // divisions by run_len, runs, chunks, n_kv, G
};
constexpr int kv8_nowhere = 1 << 25;      // number of a block that is none: past every sequence's end
constexpr float kv8_lowest = -3.0e38f;   // start of a running maximum: below every finite score, and finite itself

// A block's codes, as the lanes load them.
template <int D>
struct Kv8Block {
  uint4 k[2][D / 64], v[D / 32];
};
// ONCE: they pass the caches by.
template <bool ONCE>
__device__ inline uint4 kv8_load(const uint4* p) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  if constexpr (!ONCE) return *p;
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <int D, bool ONCE>
__device__ inline void kv8_load_k(Kv8Block<D>& b, const uint4* p) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) b.k[t][j] = kv8_load<ONCE>(p + (t * (D / 64) + j) * 64);
}
template <int D, bool ONCE>
__device__ inline void kv8_load_v(Kv8Block<D>& b, const uint4* p) {
#pragma unroll
  for (int j = 0; j < D / 32; ++j) b.v[j] = kv8_load<ONCE>(p + (D / 32 + j) * 64);
}
// Eight codes times 2^e as a bf16 operand (exact: four bits, and an exponent that bf16 has).
__device__ inline bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  union { bf16x8 v; bf16x2 h[4]; } o;
  o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return o.v;
}
__device__ inline uint32_t without_nan(uint32_t w) { return w & ~((nan_bytes(w) >> 7) * 255u); }

// What a wavefront knows of the rows it works for.
template <int JT>
struct Kv8Cols {
  int p[JT];                    // position of its column's row in each tile
  int end;                      // keys from here on are invisible
};
template <int JT>
__device__ inline bool kv8_visible(const Kv8Cols<JT>& w, const Kv8AttnArgs& a, int jt, int key) {
  return kv8_sees(w.p[jt], key, w.end, a.mode, a.window, a.sinks);
}

// What a wavefront knows of a block: its number, whether every row sees all of it, whether its values hold a NaN; the scales; the lane's codes.
constexpr uint32_t kv8_clear = 1u << 31, kv8_has_nan = 1u << 30, kv8_number = (1u << 26) - 1;
struct Kv8Of {
  uint32_t info;
  float ks, vs;
  const uint4* codes;
};

// One block of 32 keys against JT tiles of 16 columns.  S^T = K Q^T, so that a lane has eight scores of one column, and O^T = V^T P^T.
// The running maximum follows the scores only when one exceeds it by more than 2^8: weights up to 256 lose nothing, and most
// blocks need no maximum across lanes.  The sum of the weights is a product too, with a row of ones: what divides the result are the
// same rounded weights that make it.  Once a block's keys are in operands the next block's are loaded over them, then likewise the values: each
// load has the other half of a step to arrive.
template <int D, int JT, bool ONCE>
__device__ inline void kv8_step(Kv8Block<D>& b, const Kv8Of& of, const Kv8Of& next, const bf16x8 (&qf)[JT][D / 32], f32x4 (&O)[JT][D / 16],
                                float (&mrun)[JT], f32x4 (&L)[JT], const Kv8Cols<JT>& cols, const Kv8AttnArgs& a, int g) {
  constexpr int DT = D / 16;
  const float c = a.c_log2;
  f32x4 s[JT][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) s[jt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const bf16x8 k0 = widen8(b.k[t][j].x, b.k[t][j].y, of.ks), k1 = widen8(b.k[t][j].z, b.k[t][j].w, of.ks);
#pragma unroll
      for (int jt = 0; jt < JT; ++jt) s[jt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[jt][2 * j], s[jt][t], 0, 0, 0);
#pragma unroll
      for (int jt = 0; jt < JT; ++jt) s[jt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[jt][2 * j + 1], s[jt][t], 0, 0, 0);
    }
  }
  __builtin_amdgcn_sched_barrier(0);                    // (the loads stay behind the last use of what they overwrite)
  kv8_load_k<D, ONCE>(b, next.codes);
  if ((of.info & kv8_clear) == 0u) {
    const int key = (int)(of.info & kv8_number) * 32 + 8 * g;
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[jt][e >> 2][e & 3] = kv8_visible<JT>(cols, a, jt, key + e) ? s[jt][e >> 2][e & 3] : -INFINITY;
    if ((of.info & kv8_has_nan) != 0u) {
      // 0 times a NaN would reach rows that do not see it: kv8_nan_rows puts it where it belongs
#pragma unroll
      for (int j = 0; j < D / 32; ++j) b.v[j] = make_uint4(without_nan(b.v[j].x), without_nan(b.v[j].y), without_nan(b.v[j].z), without_nan(b.v[j].w));
    }
  }
  float m[JT];
  bool move = false;
#pragma unroll
  for (int jt = 0; jt < JT; ++jt) {
    m[jt] = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) m[jt] = fmaxf(m[jt], s[jt][e >> 2][e & 3]);
    move |= m[jt] * c > mrun[jt] + 8.f;
  }
  if (__builtin_amdgcn_ballot_w64(move) != 0ull) {
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
      const float mnew = fmaxf(mrun[jt], rows_max(m[jt]) * c);
      const float alpha = __builtin_amdgcn_exp2f(mrun[jt] - mnew);
      mrun[jt] = mnew;
      L[jt] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[jt][dt] *= alpha;
    }
  }
  bf16x8 p8[JT];
#pragma unroll
  for (int jt = 0; jt < JT; ++jt)
#pragma unroll
    for (int e = 0; e < 8; ++e)         // (rounded for the product: by at most 2^-8 of a weight, independently from key to key; an invisible key's is 0)
      p8[jt][e] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[jt][e >> 2][e & 3], c, -mrun[jt]));
  bf16x8 one;
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = (__bf16)1.f;
#pragma unroll
  for (int jt = 0; jt < JT; ++jt) L[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, p8[jt], L[jt], 0, 0, 0);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const bf16x8 v0 = widen8(b.v[j].x, b.v[j].y, of.vs), v1 = widen8(b.v[j].z, b.v[j].w, of.vs);
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) O[jt][2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p8[jt], O[jt][2 * j], 0, 0, 0);
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) O[jt][2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p8[jt], O[jt][2 * j + 1], 0, 0, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
  kv8_load_v<D, ONCE>(b, next.codes);
  asm volatile("" ::: "memory");                        // (or they are shared with the walk for NaN and live in registers until then)
}

// A block with NaN among its values that not every row sees all of: results become NaN where a row sees one of its dimension.
template <int D, int JT>
__device__ inline void kv8_nan_rows(const uint4* codes, f32x4 (&O)[JT][D / 16], int kb, const Kv8Cols<JT>& cols, const Kv8AttnArgs& a, int g) {
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const uint4 v = codes[(D / 32 + j) * 64];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t n0 = nan_bytes(u ? v.z : v.x), n1 = nan_bytes(u ? v.w : v.y);
      bf16x8 bad;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad[e] = ((e < 4 ? n0 : n1) >> (8 * (e & 3) + 7) & 1u) != 0u ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
      for (int jt = 0; jt < JT; ++jt) {
        bf16x8 seen;
#pragma unroll
        for (int e = 0; e < 8; ++e) seen[e] = kv8_visible<JT>(cols, a, jt, kb * 32 + 8 * g + e) ? (__bf16)1.f : (__bf16)0.f;
        const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) O[jt][2 * j + u][r] = count[r] > 0.f ? NAN : O[jt][2 * j + u][r];
      }
    }
  }
}

// Eight neighbouring dimensions of a column's result: [32 c + 8 g, + 8).
__device__ inline void kv8_store(u16* o, const f32x4& a, const f32x4& b, float inv) {
  union { bf16x8 v; uint4 u; } w;
#pragma unroll
  for (int r = 0; r < 4; ++r) { w.v[r] = (__bf16)(a[r] * inv); w.v[4 + r] = (__bf16)(b[r] * inv); }
  *reinterpret_cast<uint4*>(o) = w.u;
}

// Softmax over a stream of blocks: O = sum 2^(s - m) v, L = sum 2^(s - m), both rescaled when m moves; O/L at the end.  Bound by the cache's
// bytes where few rows read much (64 sequences up to 8192, 137 MB: 26.4 us without the joining kernel, 5.2 TB/s; 24.8 where the last-level cache keeps them), and by the issue of
// vector instructions beside the products where many rows do (1024 rows behind 7168 keys, 64 GFLOP: 67 us, 0.96 PFLOP/s, and 77 to 80 in the first
// launches after a pause, before the clock has risen; a large library product reaches 1.2): a block
// costs a wavefront 34 products for two tiles, 64 conversions of pairs of codes and 16 exponentials.  A block of 32 rows behind 1024 keys 7.1 us, most of it
// the launch and dependent loads (arguments, page and length, codes).
// A workgroup of NW wavefronts takes JT tiles of a (sequence, kv head) and one of the chunks of their blocks: block number idx belongs to
// chunk idx % chunks and in it to wavefront (idx / chunks) % NW.  The wavefronts merge through LDS; a group in one chunk stores its result, of several each
// leaves an unnormalised partial, which kv8_merge_kernel sums in the order of the chunks.  The groups of a (sequence, kv head, chunk), which
// read the same blocks, go to one XCD (numbers that differ by multiples of 8), where its L2 serves all but the first, or are dealt to several
// where there are fewer than 8 such units (all of a unit on one XCD took four times as long for those 1024 rows); the last groups, which see most, start first.
template <int D, int JT, int NW, bool ONCE>
__global__ __launch_bounds__(NW * 64, JT == 1 ? 3 : 2) void kv8_attn_kernel(Kv8AttnArgs a) {
  constexpr int DT = D / 16;
  __shared__ f32x4 sO[NW * JT * DT * 64];                               // [NW][JT][DT][64]
  __shared__ float sm[NW * JT * 16], sl[NW * JT * 16];                  // [NW][JT][16]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  // (all arguments with one wait)
  asm volatile("" ::"s"(a.c.dev_codes), "s"(a.c.dev_scales), "s"(a.c.dev_pages), "s"(a.c.max_blocks), "s"(a.r.first), "s"(a.q), "s"(a.q_row), "s"(a.window),
               "s"(a.c_log2), "s"(a.tiles), "s"(a.by_runs.mul), "s"(a.by_G.mul));
  const int eighth = blockIdx.x >> 3, turn = kv8_quotient(eighth, a.by_len), run = turn * 8 + (blockIdx.x & 7), unit = kv8_quotient(run, a.by_runs);
  const int grp = a.groups - 1 - ((eighth - turn * a.run_len) * a.runs + run - unit * a.runs);
  if (grp < 0 || unit >= a.c.n_seq * a.c.n_kv * a.chunks) return;
  const int sh = kv8_quotient(unit, a.by_chunks), chunk = unit - sh * a.chunks, s = kv8_quotient(sh, a.by_kv), h = sh - s * a.c.n_kv;
  // without a window and chunks the wavefront's first blocks are known before the length is: their pages are asked for at the same time
  const bool from_0 = a.window == 0 && a.chunks == 1;
  int early = a.c.dev_pages[(size_t)s * a.c.max_blocks + min(wave + lane * NW, a.c.max_blocks - 1)];
  int n, rows;
  if (!kv8_take(a.c, a.r, s, n, rows)) return;
  const int G = a.G, ncols = rows * G, c0 = grp * JT * 16;
  if (c0 >= ncols) return;
  const int r0 = kv8_quotient(c0, a.by_G), r1 = kv8_quotient(min(c0 + JT * 16, ncols) - 1, a.by_G);
  const Kv8Span sp = kv8_span(n, rows, r0, r1, a.mode, a.window, a.sinks);
  const int used = JT == 1 ? kv8_chunks_used(sp.count, a.chunks) : 1;     // (several tiles are taken where there is no room for chunks)
  if (chunk >= used) return;
  const int step = NW * used, first = wave * used + chunk;
  const int left = (sp.count - first + step - 1);
  const int cnt = __builtin_amdgcn_readfirstlane(sp.count <= first ? 0 : used == 1 ? left / NW : left / step);
  // what there is to know of the wavefront's next 64 blocks, one a lane; a block whose page lies outside the pool, and one past the last, is
  // invisible to all, with the codes of page 0 for its own
  uint32_t my_info, my_head, my_word;
  float my_ks, my_vs;
  auto ask = [&](int base) {                            // (page 0's own scales are asked for where there is no block, and not used)
    my_info = (uint32_t)kv8_nowhere | kv8_has_nan;
    my_head = (uint32_t)h;
    if (base + lane < cnt) {
      const int idx = first + (base + lane) * step;
      const bool sink = idx < sp.sink_blocks;
      const int kb = sink ? idx : sp.first_block + idx - sp.sink_blocks;
      const int page = kv8_in_pool(a.c, base == 0 && from_0 ? early : a.c.dev_pages[(size_t)s * a.c.max_blocks + kb]);
      if (page >= 0) {
        my_head = (uint32_t)page * (uint32_t)a.c.n_kv + (uint32_t)h;
        const bool clear = sink ? kb < sp.clear_sinks : kb >= sp.clear_lo && kb < sp.clear_hi;
        my_info = (uint32_t)kb | (clear ? kv8_clear : 0u);
      }
    }
    my_word = a.c.dev_scales[my_head];
  };
  auto know = [&]() {
    const bool there = (my_info & kv8_number) != (uint32_t)kv8_nowhere;
    if (there && (my_word & kv8_v_nan) != 0u) my_info |= kv8_has_nan;
    my_ks = two_to(there ? kv8_byte_exponent(my_word) : 0);
    my_vs = two_to(there ? kv8_byte_exponent(my_word >> 8) : 0);
    // waited for here: behind a branch that may have left loads open, every later wait would be one for all of them
    asm volatile("" : "+v"(my_info), "+v"(my_head), "+v"(my_ks), "+v"(my_vs));
  };
  auto look_up = [&](int base) {
    ask(base);
    know();
  };
  ask(0);
  bf16x8 qf[JT][D / 32];
  f32x4 O[JT][DT], L[JT];
  float mrun[JT];
  Kv8Cols<JT> cols;
  cols.end = n + rows;
#pragma unroll
  for (int jt = 0; jt < JT; ++jt) {
    const int cc = min(c0 + jt * 16 + col, ncols - 1);                   // (columns past the last one repeat it and store nothing)
    const int r = kv8_quotient(cc, a.by_G);
    cols.p[jt] = n + r;
    const u16* qp = a.q + s * a.q_seq + r * a.q_row + (h * G + cc - r * G) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      qf[jt][2 * j] = *reinterpret_cast<const bf16x8*>(qp + 64 * j);
      qf[jt][2 * j + 1] = *reinterpret_cast<const bf16x8*>(qp + 64 * j + 8);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[jt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    L[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
    mrun[jt] = kv8_lowest;
  }
  auto codes_of = [&](int i) {
    const uint32_t head = (uint32_t)__builtin_amdgcn_readlane((int)my_head, i & 63);
    return reinterpret_cast<const uint4*>(a.c.dev_codes + (size_t)head * (64 * D)) + lane;
  };
  auto block_of = [&](int i) {
    if ((i & 63) == 0 && i > 0) look_up(i);
    return Kv8Of{(uint32_t)__builtin_amdgcn_readlane((int)my_info, i & 63), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_ks), i & 63)),
                 __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_vs), i & 63)),
                 codes_of(i)};
  };
  bool nan = false;
  if (cnt > 0) {
    Kv8Block<D> b;
    kv8_load_k<D, ONCE>(b, codes_of(0));                // (before the scales are there)
    __builtin_amdgcn_sched_barrier(0);                  // (in the order in which the loop will ask for them: its first wait has to hold for this entry to it too)
    kv8_load_v<D, ONCE>(b, codes_of(0));
    __builtin_amdgcn_sched_barrier(0);
    know();
    Kv8Of of = block_of(0);
    for (int i = 0; i < cnt; ++i) {
      const Kv8Of next = block_of(i + 1);
      kv8_step<D, JT, ONCE>(b, of, next, qf, O, mrun, L, cols, a, g);
      nan |= (of.info & (kv8_clear | kv8_has_nan)) == kv8_has_nan && (of.info & kv8_number) != (uint32_t)kv8_nowhere;
      of = next;
    }
  }
  if (nan) {
    look_up(0);
    for (int i = 0; i < cnt; ++i) {
      const Kv8Of of = block_of(i);
      const int kb = (int)(of.info & kv8_number);
      if ((of.info & (kv8_clear | kv8_has_nan)) == kv8_has_nan && kb != kv8_nowhere) kv8_nan_rows<D, JT>(of.codes, O, kb, cols, a, g);
    }
  }
#pragma unroll
  for (int jt = 0; jt < JT; ++jt) {
    if (g == 0) {
      sm[(wave * JT + jt) * 16 + col] = mrun[jt];
      sl[(wave * JT + jt) * 16 + col] = L[jt][0];
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) sO[((wave * JT + jt) * DT + dt) * 64 + lane] = O[jt][dt];
  }
  __syncthreads();
  // the wavefronts share out the pairs of d-tiles
  for (int item = wave; item < JT * (DT / 2); item += NW) {
    const int jt = item / (DT / 2), j = item % (DT / 2), cc = c0 + jt * 16 + col, r = kv8_quotient(cc, a.by_G);
    float m = kv8_lowest, f[NW], l = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, sm[(w * JT + jt) * 16 + col]);
    f32x4 o0 = f32x4{0.f, 0.f, 0.f, 0.f}, o1 = o0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      f[w] = __builtin_amdgcn_exp2f(sm[(w * JT + jt) * 16 + col] - m);
      l += sl[(w * JT + jt) * 16 + col] * f[w];
      o0 += sO[((w * JT + jt) * DT + 2 * j) * 64 + lane] * f[w];
      o1 += sO[((w * JT + jt) * DT + 2 * j + 1) * 64 + lane] * f[w];
    }
    if (used == 1) {
      if (cc < ncols) kv8_store(a.out + s * a.o_seq + r * a.o_row + (h * G + cc - r * G) * D + 32 * j + 8 * g, o0, o1, 1.f / l);
    } else if constexpr (JT == 1) {
      float* pp = a.part + ((((int64_t)s * a.c.n_kv + h) * a.tiles + grp) * a.chunks + chunk) * (16 * D + 32);
      *reinterpret_cast<f32x4*>(pp + (2 * j * 64 + lane) * 4) = o0;
      *reinterpret_cast<f32x4*>(pp + ((2 * j + 1) * 64 + lane) * 4) = o1;
      if (j == 0 && g == 0) {
        pp[16 * D + col] = m;
        pp[16 * D + 16 + col] = l;
      }
    }
  }
}

// The chunks of a tile summed in their order: one wavefront per (sequence, kv head, tile, pair of d-tiles).  All it does is to wait for memory, so
// the first eight partials are asked for before it is known how many there are (those that no group left are not looked at): 3.5 to 4.5 us, 2.1 to 2.4 where
// there is nothing to join.  With more than eight, four wavefronts take eight at a time in turn: 8 rows behind 32768 keys, 32 chunks, 12.3 instead of 14.6 us.
template <int D, int W>
__global__ __launch_bounds__(64 * W) void kv8_merge_kernel(Kv8AttnArgs a) {
  constexpr int P = 8, size = 16 * D + 32;
  const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const int j = blockIdx.x % (D / 32), item = blockIdx.x / (D / 32), sh = item / a.tiles, tile = item - sh * a.tiles;
  const int s = kv8_quotient(sh, a.by_kv), h = sh - s * a.c.n_kv;
  const float* base = a.part + (int64_t)item * a.chunks * size;
  float pm[P], pl[P];
  f32x4 p0[P], p1[P];
  auto ask = [&](int from) {
#pragma unroll
    for (int c = 0; c < P; ++c) {
      const float* pp = base + min(from + c, a.chunks - 1) * size;
      pm[c] = pp[16 * D + col];
      pl[c] = pp[16 * D + 16 + col];
      p0[c] = *reinterpret_cast<const f32x4*>(pp + (2 * j * 64 + lane) * 4);
      p1[c] = *reinterpret_cast<const f32x4*>(pp + ((2 * j + 1) * 64 + lane) * 4);
    }
  };
  ask(wave * P);
  int n, rows;
  if (!kv8_take(a.c, a.r, s, n, rows)) return;
  const int G = a.G, ncols = rows * G, c0 = tile * 16, cc = c0 + col;
  if (c0 >= ncols) return;
  const Kv8Span sp = kv8_span(n, rows, kv8_quotient(c0, a.by_G), kv8_quotient(min(c0 + 16, ncols) - 1, a.by_G), a.mode, a.window, a.sinks);
  const int used = kv8_chunks_used(sp.count, a.chunks);
  if (used == 1) return;
  float m = kv8_lowest, l = 0.f;
  f32x4 o0 = f32x4{0.f, 0.f, 0.f, 0.f}, o1 = o0;
  for (int from = wave * P;;) {
    float top = m;
#pragma unroll
    for (int c = 0; c < P; ++c) top = from + c < used ? fmaxf(top, pm[c]) : top;
    const float again = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= again;
    o0 *= again;
    o1 *= again;
#pragma unroll
    for (int c = 0; c < P; ++c)
      if (from + c < used) {
        const float f = __builtin_amdgcn_exp2f(pm[c] - m);
        l += pl[c] * f;
        o0 += p0[c] * f;
        o1 += p1[c] * f;
      }
    from += W * P;
    if (from >= used) break;
    ask(from);
  }
  if constexpr (W > 1) {
    __shared__ f32x4 so[W][2][64];
    __shared__ float2 sml[W][16];
    so[wave][0][lane] = o0;
    so[wave][1][lane] = o1;
    if (g == 0) sml[wave][col] = make_float2(m, l);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, sml[w][col].x);
    l = 0.f;
    o0 = o1 = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(sml[w][col].x - m);
      l += sml[w][col].y * f;
      o0 += so[w][0][lane] * f;
      o1 += so[w][1][lane] * f;
    }
  }
  const int r = kv8_quotient(cc, a.by_G);
  if (cc < ncols) kv8_store(a.out + s * a.o_seq + r * a.o_row + (h * G + cc - r * G) * D + 32 * j + 8 * g, o0, o1, 1.f / l);
}

// ---- rotary positions -----------------------------------------------------------------------------------------------------
struct RopeArgs {
  bd_rope plan;
  const void* x; void* y;
  int64_t x_seq, x_row, y_seq, y_row;
  const int* pos; const int* rows;
  int heads, M;
  Kv8Div by_items;                                     // divisions by the items of a row
};

// A workgroup takes `per` rows: sines and cosines of their angles once for all heads (fp64 up to the reduced angle: at position 2^20 an
// angle in fp32 is off by up to 2^-5), then the heads.  Bound by the rows' bytes, 16384 rows of 18 heads of 128 in fp32 63 us, 302 MB
// at 4.8 TB/s, in bf16 29 us, 151 MB at 5.2 TB/s: 16 a lane and access, VEC, where the two halves of a rotary part fall on 16 bytes (with neighbouring pairs
// always), else an element at a time (a part of 66 of each head: 65 us in fp32, 44 in bf16).
constexpr int kRopeRows = 4;
__host__ __device__ inline int rope_item_log(int D, int N) { return (D == 128 ? 6 : 5) - (N == 8 ? 3 : N == 4 ? 2 : 0); }
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int per) {
  __shared__ float2 s_cs[kRopeRows][64];               // (cosine, sine)
  const int s = blockIdx.y, r0 = blockIdx.x * per, tid = threadIdx.x;
  const int n = min(max(min(a.rows != nullptr ? a.rows[s] : a.M, a.M), 0) - r0, per);
  if (n <= 0) return;
  const int R2 = a.plan.rotary_dim >> 1, D = a.plan.D;
  if (tid < 64 * n && (tid & 63) < R2) {
    const double turns = ((double)a.pos[s] + (r0 + (tid >> 6))) * a.plan.inv_freq[tid & 63] * 0.15915494309189533577;   // 1/(2 pi)
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    s_cs[tid >> 6][tid & 63] = make_float2(cs * a.plan.amplitude, sn * a.plan.amplitude);
  }
  __syncthreads();
  const T* x = reinterpret_cast<const T*>(a.x) + s * a.x_seq + r0 * a.x_row;
  T* y = reinterpret_cast<T*>(a.y) + s * a.y_seq + r0 * a.y_row;
  const bool half = a.plan.layout == BD_ROPE_HALF, in_place = a.x == a.y;
  constexpr int N = VEC ? 16 / sizeof(T) : 1;
  typedef Pack<T, N> V;
  // an item: two vectors of a head whose elements make pairs (half), or that lie side by side (neighbouring pairs and the rest of the head)
  const int item_log = rope_item_log(D, N), items = a.heads << item_log;
  for (int i = tid; i < n * items; i += 256) {
    const int r = kv8_quotient(i, a.by_items), k = i - r * items, h = k >> item_log, j = k & ((1 << item_log) - 1);
    const bool turn = j * N < R2;
    if (in_place && !turn) continue;
    const int d0 = h * D + (half && turn ? j * N : 2 * j * N), d1 = half && turn ? d0 + R2 : d0 + N;
    const V u = *reinterpret_cast<const V*>(x + r * a.x_row + d0), v = *reinterpret_cast<const V*>(x + r * a.x_row + d1);
    V p = u, q = v;
    if (turn) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        // half: pair (u[e], v[e]); neighbours: pairs lie along u, then v
        const float2 cs = s_cs[r][min(j * N + e, 63)];
        if (half || N == 1) {
          const float b0 = to_f32(u.x[e]), b1 = to_f32(v.x[e]);
          p.x[e] = from_f32<T>(b0 * cs.x - b1 * cs.y);
          q.x[e] = from_f32<T>(b1 * cs.x + b0 * cs.y);
        } else if (j * N + e < R2) {
          const int at = (2 * e) % N;
          const float b0 = to_f32(2 * e < N ? u.x[at] : v.x[at]), b1 = to_f32(2 * e < N ? u.x[at + (N > 1)] : v.x[at + (N > 1)]);
          (2 * e < N ? p : q).x[at] = from_f32<T>(b0 * cs.x - b1 * cs.y);
          (2 * e < N ? p : q).x[at + (N > 1)] = from_f32<T>(b1 * cs.x + b0 * cs.y);
        }
      }
    }
    *reinterpret_cast<V*>(y + r * a.y_row + d0) = p;
    *reinterpret_cast<V*>(y + r * a.y_row + d1) = q;
  }
}

// ---- host side --------------------------------------------------------------------------------------------------------------
constexpr int kMaxRows = 1 << 22;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_cache(const bd_kv8* c, int M, bool shape_only = false) {
  if (c == nullptr) return BD_E_ARG;
  if ((c->D != 64 && c->D != 128) || c->n_pages < 1 || c->n_kv < 1 || c->n_kv > 4096 || c->n_seq < 1 || c->n_seq > 65535 || c->max_blocks < 1 ||
      c->max_blocks > (1 << 25) || (int64_t)c->n_pages * c->n_kv > ((int64_t)1 << 31) || M < 1 || M > kMaxRows ||
      (int64_t)M * c->n_kv > (1 << 28))
    return BD_E_ARG;
  if (shape_only) return BD_OK;
  if (c->dev_codes == nullptr || !aligned16(c->dev_codes) || c->dev_scales == nullptr || c->dev_pages == nullptr) return BD_E_ARG;
  return BD_OK;
}
// Rows tensor: not null, 16-byte aligned, strides of whole 16 bytes, at least `least` elements (a row, where rows are written).
int check_rows(const void* p, int dtype, int64_t seq_stride, int64_t row_stride, int n_seq, int M, int64_t least = 0) {
  if (dtype != BD_BF16 && dtype != BD_F32) return BD_E_DTYPE;
  const int64_t unit = dtype == BD_F32 ? 4 : 8;
  if (p == nullptr || !aligned16(p)) return BD_E_ARG;
  if (n_seq > 1 && (seq_stride < least || seq_stride % unit != 0)) return BD_E_ARG;
  if (M > 1 && (row_stride < least || row_stride % unit != 0)) return BD_E_ARG;
  return BD_OK;
}

// Blocks of 32 positions that M rows can touch.
int blocks_of(int M, int max_blocks) {
  const int b = (M + 62) / 32;
  return b < max_blocks ? b : max_blocks;
}

// A launch in one call to the runtime, with its own status: 0.6 us less on the host than the triple brackets and a look at the last error.
template <typename... P>
int launch(hipStream_t s, void (*kernel)(P...), dim3 grid, int threads, P... args) {
  void* list[] = {&args...};
  HIP_TRY(hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), list, 0, s));
  return BD_OK;
}

template <typename K>
int launch_copy(hipStream_t s, K kernel, const Kv8CopyArgs& a) {
  const int wavefronts = ceil_div(blocks_of(a.r.M, a.c.max_blocks), 128 / a.c.D) * 2 * a.c.n_kv;
  return launch(s, kernel, dim3(ceil_div(wavefronts, 4), 1, a.c.n_seq), 256, a);
}

template <int D, int JT, int NW, bool ONCE>
int launch_attn(hipStream_t s, const Kv8AttnArgs& a, const Kv8Plan& p) {
  const int64_t units = (int64_t)a.c.n_seq * a.c.n_kv * p.chunks, groups = (units * p.runs + 7) / 8 * 8 * p.run_len;
  BD_TRY(launch(s, kv8_attn_kernel<D, JT, NW, ONCE>, dim3((unsigned)groups), NW * 64, a));
  if (JT == 1 && p.chunks > 1) {
    const dim3 grid((unsigned)((int64_t)a.c.n_seq * a.c.n_kv * p.tiles * (D / 32)));
    BD_TRY(p.chunks > 8 ? launch(s, kv8_merge_kernel<D, 4>, grid, 256, a) : launch(s, kv8_merge_kernel<D, 1>, grid, 64, a));
  }
  return BD_OK;
}
template <int D>
int launch_attn_form(hipStream_t s, const Kv8AttnArgs& a, const Kv8Plan& p) {
  switch (p.form) {
    case Kv8Form::wide: return launch_attn<D, 2, 4, false>(s, a, p);
    case Kv8Form::stream: return launch_attn<D, 1, 4, true>(s, a, p);
    default: return launch_attn<D, 1, 8, false>(s, a, p);
  }
}

int check_attn(const bd_kv8* c, int n_q, int M, int window, int sinks, bool shape_only, Kv8Plan* p) {
  BD_TRY(check_cache(c, M, shape_only));
  if (n_q < 1 || n_q > (1 << 16) || n_q % c->n_kv != 0 || window < 0 || sinks < 0) return BD_E_ARG;
  if (kv8_items(c->n_seq, M, n_q, c->n_kv) > ((int64_t)1 << 22)) return BD_E_ARG;      // (a launch has less than 2^32 threads)
  *p = kv8_plan(c->n_seq, M, n_q, c->n_kv, c->D, c->max_blocks, window, sinks);
  return BD_OK;
}

}  // namespace
}  // namespace bd

using namespace bd;

extern "C" int bd_k_kv8_write(void* hip_stream, const bd_kv8* cache, const void* dev_k, int64_t k_seq_stride, int64_t k_row_stride, const void* dev_v,
                              int64_t v_seq_stride, int64_t v_row_stride, int dtype, int M, const int32_t* dev_rows) {
  BD_TRY(check_cache(cache, M));
  BD_TRY(check_rows(dev_k, dtype, k_seq_stride, k_row_stride, cache->n_seq, M));
  BD_TRY(check_rows(dev_v, dtype, v_seq_stride, v_row_stride, cache->n_seq, M));
  if (cache->dev_len == nullptr) return BD_E_ARG;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Kv8CopyArgs a{*cache, {cache->dev_len, dev_rows, M}, {const_cast<void*>(dev_k), const_cast<void*>(dev_v)}, {k_seq_stride, v_seq_stride}, {k_row_stride, v_row_stride}, kv8_div(2 * cache->n_kv)};
  if (cache->D == 128) return dtype == BD_F32 ? launch_copy(s, kv8_write_kernel<128, float>, a) : launch_copy(s, kv8_write_kernel<128, u16>, a);
  return dtype == BD_F32 ? launch_copy(s, kv8_write_kernel<64, float>, a) : launch_copy(s, kv8_write_kernel<64, u16>, a);
}

extern "C" int bd_k_kv8_read(void* hip_stream, const bd_kv8* cache, const int32_t* dev_from, int M, const int32_t* dev_rows, int dtype,
                             void* dev_k_out, int64_t k_seq_stride, int64_t k_row_stride, void* dev_v_out, int64_t v_seq_stride,
                             int64_t v_row_stride) {
  BD_TRY(check_cache(cache, M));
  const int64_t least = (int64_t)cache->n_kv * cache->D;
  BD_TRY(check_rows(dev_k_out, dtype, k_seq_stride, k_row_stride, cache->n_seq, M, least));
  BD_TRY(check_rows(dev_v_out, dtype, v_seq_stride, v_row_stride, cache->n_seq, M, least));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Kv8CopyArgs a{*cache, {dev_from, dev_rows, M}, {dev_k_out, dev_v_out}, {k_seq_stride, v_seq_stride}, {k_row_stride, v_row_stride}, kv8_div(2 * cache->n_kv)};
  if (cache->D == 128) return dtype == BD_F32 ? launch_copy(s, kv8_read_kernel<128, float>, a) : launch_copy(s, kv8_read_kernel<128, u16>, a);
  return dtype == BD_F32 ? launch_copy(s, kv8_read_kernel<64, float>, a) : launch_copy(s, kv8_read_kernel<64, u16>, a);
}

extern "C" int64_t bd_k_kv8_attention_workspace(const bd_kv8* cache, int n_q, int M, int window, int sinks) {
  Kv8Plan p;
  BD_TRY(check_attn(cache, n_q, M, window, sinks, true, &p));
  return p.part_floats * 4;
}

extern "C" int bd_k_kv8_attention(void* hip_stream, const bd_kv8* cache, const void* dev_q, int64_t q_seq_stride, int64_t q_row_stride, int n_q,
                                  int M, const int32_t* dev_rows, int mode, int window, int sinks, float scale, void* dev_out,
                                  int64_t out_seq_stride, int64_t out_row_stride, void* dev_workspace, int64_t workspace_bytes) {
  Kv8Plan p;
  BD_TRY(check_attn(cache, n_q, M, window, sinks, false, &p));
  BD_TRY(check_rows(dev_q, BD_BF16, q_seq_stride, q_row_stride, cache->n_seq, M));
  BD_TRY(check_rows(dev_out, BD_BF16, out_seq_stride, out_row_stride, cache->n_seq, M, (int64_t)n_q * cache->D));
  if (cache->dev_len == nullptr || (mode != BD_MODE_BIDIR && mode != BD_MODE_CAUSAL) || !(scale >= 0.f && scale <= 0x1p127f)) return BD_E_ARG;     // (times log2 e finite)
  if (p.part_floats > 0 && (dev_workspace == nullptr || !aligned16(dev_workspace))) return BD_E_ARG;
  if (workspace_bytes < p.part_floats * 4) {
    set_last_error("bd_k_kv8_attention: this shape needs %lld bytes of workspace, got %lld", (long long)p.part_floats * 4, (long long)workspace_bytes);
    return BD_E_CAPACITY;
  }
  Kv8AttnArgs a{};
  a.c = *cache;
  a.r = {cache->dev_len, dev_rows, M};
  a.q = static_cast<const u16*>(dev_q); a.out = static_cast<u16*>(dev_out);
  a.q_seq = q_seq_stride; a.q_row = q_row_stride; a.o_seq = out_seq_stride; a.o_row = out_row_stride;
  a.part = static_cast<float*>(dev_workspace);
  a.n_q = n_q; a.mode = mode; a.window = window; a.sinks = sinks;
  a.c_log2 = (scale > 0.f ? scale : 1.f / std::sqrt((float)cache->D)) * 1.4426950408889634f;
  a.tiles = p.tiles; a.groups = p.groups; a.chunks = p.chunks; a.runs = p.runs; a.run_len = p.run_len; a.G = n_q / cache->n_kv;
  a.by_len = kv8_div(p.run_len); a.by_runs = kv8_div(p.runs); a.by_chunks = kv8_div(p.chunks); a.by_kv = kv8_div(cache->n_kv); a.by_G = kv8_div(a.G);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (cache->D == 128) return launch_attn_form<128>(s, a, p);
  return launch_attn_form<64>(s, a, p);
}

extern "C" int bd_k_rope_plan(bd_rope* out, int D, int rotary_dim, int layout, double theta, int scaling, double factor, int trained) {
  if (out == nullptr || (D != 64 && D != 128) || rotary_dim < 2 || rotary_dim > D || rotary_dim % 2 != 0) return BD_E_ARG;
  if (layout != BD_ROPE_HALF && layout != BD_ROPE_INTERLEAVED) return BD_E_ARG;
  if (scaling < BD_ROPE_PLAIN || scaling > BD_ROPE_PARTS || !(theta > 1.0) || !std::isfinite(theta)) return BD_E_ARG;
  if (scaling != BD_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor) || trained < 1)) return BD_E_ARG;
  if (scaling == BD_ROPE_BASE) {
    if (rotary_dim <= 2) return BD_E_ARG;
    theta *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    if (!std::isfinite(theta)) return BD_E_ARG;
  }
  bd_rope p{};
  p.D = D; p.rotary_dim = rotary_dim; p.layout = layout;
  p.amplitude = scaling == BD_ROPE_PARTS ? (float)(1.0 + 0.1 * std::log(factor)) : 1.f;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / rotary_dim);
    if (scaling == BD_ROPE_LINEAR) f /= factor;
    if (scaling == BD_ROPE_PARTS) {
      double w = (trained * f / 6.283185307179586477 - 1.0) / 31.0;
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      f = f * w + f / factor * (1.0 - w);
    }
    p.inv_freq[i] = f;
  }
  *out = p;
  return BD_OK;
}

extern "C" int bd_k_rope(void* hip_stream, const bd_rope* plan, const void* dev_x, int64_t x_seq_stride, int64_t x_row_stride, void* dev_out,
                         int64_t out_seq_stride, int64_t out_row_stride, int dtype, int n_heads, int n_seq, int M, const int32_t* dev_pos,
                         const int32_t* dev_rows) {
  if (plan == nullptr || (plan->D != 64 && plan->D != 128) || plan->rotary_dim < 2 || plan->rotary_dim > plan->D || plan->rotary_dim % 2 != 0 ||
      (plan->layout != BD_ROPE_HALF && plan->layout != BD_ROPE_INTERLEAVED))
    return BD_E_ARG;
  if (n_heads < 1 || n_heads > (1 << 16) || n_seq < 1 || n_seq > 65535 || M < 1 || M > kMaxRows || dev_pos == nullptr) return BD_E_ARG;
  BD_TRY(check_rows(dev_x, dtype, x_seq_stride, x_row_stride, n_seq, M));
  BD_TRY(check_rows(dev_out, dtype, out_seq_stride, out_row_stride, n_seq, M, (int64_t)n_heads * plan->D));
  if (dev_x == dev_out && ((n_seq > 1 && x_seq_stride != out_seq_stride) || (M > 1 && x_row_stride != out_row_stride))) return BD_E_ARG;
  RopeArgs a{};
  a.plan = *plan;
  a.x = dev_x; a.y = dev_out; a.x_seq = x_seq_stride; a.x_row = x_row_stride; a.y_seq = out_seq_stride; a.y_row = out_row_stride;
  a.pos = dev_pos; a.rows = dev_rows; a.heads = n_heads; a.M = M;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int N = dtype == BD_F32 ? 4 : 8;
  const bool vec = plan->layout == BD_ROPE_INTERLEAVED || plan->rotary_dim % (2 * N) == 0;
  // Few rows: a workgroup each, for more lanes at work.  One / four rows a workgroup (18 heads of 128; us in a captured graph): 1024 rows 5.0 / 6.4 in bf16, 6.6 / 7.5
  // in fp32, 2048 6.6 / 7.5 and 9.0 / 8.8, 4096 9.7 / 9.1 and 19.7 / 18.7, 8192 15.0 / 14.4 and 31.4 / 32.8, 16384 32.2 / 31.9 and 55.9 / 60.5 (so fp32 gains
  // from four around 4096 rows only).
  const int per = (int64_t)M * n_seq >= 4096 ? kRopeRows : 1;
  a.by_items = kv8_div(n_heads << rope_item_log(plan->D, vec ? N : 1));
  const dim3 grid(ceil_div(M, per), n_seq);
  if (dtype == BD_F32) return launch(s, vec ? rope_kernel<float, true> : rope_kernel<float, false>, grid, 256, a, per);
  return launch(s, vec ? rope_kernel<u16, true> : rope_kernel<u16, false>, grid, 256, a, per);
}
