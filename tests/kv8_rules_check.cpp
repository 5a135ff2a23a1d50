// Checks of what csrc/kv8.h says (layout of a page, scales, rows, spans of visible blocks, launch plan), and of the refusals of the entry points in
// csrc/k_kv8.hip, for tests/test_kv8_cpu.py: host code only, built with AddressSanitizer and UndefinedBehaviorSanitizer.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <vector>

#include "../paper_2604_06832_amd/csrc/kv8.h"

using namespace bd;

static int failures = 0;
#define CHECK(cond)                                                                                 \
  do {                                                                                              \
    if (!(cond) && ++failures < 20) std::printf("FAILED line %d: %s\n", __LINE__, #cond);           \
  } while (0)

static void layout() {
  for (int D : {64, 128}) {
    std::vector<int> seen(64 * D, 0);
    for (int t = 0; t < 32; ++t)
      for (int d = 0; d < D; ++d) {
        const int k = kv8_k_byte(t, d, D), v = 32 * D + kv8_v_byte(t, d);
        CHECK(k >= 0 && k < 32 * D && v >= 32 * D && v < 64 * D);
        ++seen[k];
        ++seen[v];
        if (d % 8 == 0) CHECK(kv8_k_byte(t, d + 7, D) == k + 7 && k % 8 == 0);      // what a thread stores at once
        if (t % 8 == 0) CHECK(32 * D + kv8_v_byte(t + 7, d) == v + 7 && v % 8 == 0);
      }
    for (int n : seen) CHECK(n == 1);
  }
}

static void exponents() {
  auto bits = [](float f) { uint32_t u; std::memcpy(&u, &f, 4); return u; };
  for (int x = -149; x <= 127; ++x)
    for (float m : {1.f, 1.25f, 1.75f, std::nextafterf(1.75f, 2.f), std::nextafterf(2.f, 1.f)}) {
      const float a = std::ldexp(m, x);
      if (!(a > 0.f) || !std::isfinite(a)) continue;
      int e = kv8_e_min;
      while (e < kv8_e_max && (double)a > 448.0 * std::ldexp(1.0, e)) ++e;
      CHECK(kv8_exponent(bits(a)) == e);
    }
  CHECK(kv8_exponent(0) == kv8_e_min);
  for (int b = 0; b < 256; ++b) CHECK(kv8_byte_exponent(b) >= kv8_e_min && kv8_byte_exponent(b) <= kv8_e_max);
  CHECK(kv8_byte_exponent(0x300u | (127 + 5)) == 5);
}

static void quotients() {
  const int big = std::numeric_limits<int>::max();
  std::vector<int> ds;
  for (int d = 1; d <= 4100; ++d) ds.push_back(d);
  for (int b = 13; b < 31; ++b)
    for (int o : {-1, 0, 1}) ds.push_back((1 << b) + o);
  for (int d : {big - 1, big, 1000003, 65536 * 64}) ds.push_back(d);
  for (int d : ds) {
    const Kv8Div v = kv8_div(d);
    auto at = [&](int64_t x) { if (x >= 0 && x <= big) CHECK(kv8_quotient((int)x, v) == (int)x / d); };
    for (int64_t k : {0, 1, 2, 3, 7, 100, 4095, 65537, big / d - 1, big / d})
      for (int o : {-1, 0, 1}) at(k * d + o);               // (an int64: past the range it is left out)
    for (int x : {0, 1, big - 1, big}) at(x);
  }
}

static void rows() {
  const int big = std::numeric_limits<int>::max();
  CHECK(kv8_rows_ok(0, 0, 1, 1) && kv8_rows_ok(0, 32, 32, 1) && kv8_rows_ok(32, 0, 4, 1) && kv8_rows_ok(31, 1, 4, 1));
  CHECK(!kv8_rows_ok(0, 33, 64, 1) && !kv8_rows_ok(-1, 1, 4, 1) && !kv8_rows_ok(0, -1, 4, 1) && !kv8_rows_ok(0, 5, 4, 1));
  CHECK(!kv8_rows_ok(31, 2, 4, 1) && !kv8_rows_ok(big, big, big, 1 << 25) && !kv8_rows_ok(big, 1, 4, 1 << 25));
  CHECK(!kv8_rows_ok(std::numeric_limits<int>::min(), 1, 4, 4));
}

// Every key that a row sees lies in a block of the span, no block twice, none past the sequence's pages, and blocks called clear are seen whole.
static void span() {
  std::srand(1);
  for (int it = 0; it < 60000; ++it) {
    const int n = std::rand() % 300, rows = 1 + std::rand() % 70;
    const int r0 = std::rand() % rows, r1 = r0 + std::rand() % (rows - r0);
    const int mode = std::rand() % 2, window = std::rand() % 3 ? 1 + std::rand() % 200 : 0, sinks = std::rand() % 4 ? std::rand() % 150 : 0;
    const Kv8Span s = kv8_span(n, rows, r0, r1, mode, window, sinks);
    const int end = n + rows, last = (end + 31) / 32;
    CHECK(s.count >= 1 && s.sink_blocks >= 0 && s.sink_blocks <= s.first_block);
    std::vector<int> in(last + 1, 0);
    for (int i = 0; i < s.count; ++i) {
      const int kb = i < s.sink_blocks ? i : s.first_block + i - s.sink_blocks;
      CHECK(kb >= 0 && kb < last);
      if (kb < 0 || kb >= last) break;
      ++in[kb];
      CHECK(in[kb] == 1);
      const bool clear = i < s.sink_blocks ? kb < s.clear_sinks : kb >= s.clear_lo && kb < s.clear_hi;
      for (int r = r0; clear && r <= r1; ++r)
        for (int j = kb * 32; j < kb * 32 + 32; ++j) CHECK(kv8_sees(n + r, j, end, mode, window, sinks));
    }
    for (int r = r0; r <= r1; ++r) {
      CHECK(kv8_sees(n + r, n + r, end, mode, window, sinks));            // no row is empty
      for (int j = 0; j < end; ++j)
        if (kv8_sees(n + r, j, end, mode, window, sinks)) CHECK(in[j / 32] == 1);
    }
  }
}

static void plan() {
  std::srand(2);
  for (int it = 0; it < 20000; ++it) {
    const int n_kv = 1 + std::rand() % 8, G = 1 + std::rand() % 16, n_seq = 1 + std::rand() % 200, M = 1 + std::rand() % 2000;
    const int blocks = 1 + std::rand() % 3000, window = std::rand() % 2 ? 1 + std::rand() % 5000 : 0, D = std::rand() % 2 ? 64 : 128;
    const Kv8Plan p = kv8_plan(n_seq, M, n_kv * G, n_kv, D, blocks, window, 4);
    CHECK(p.tiles * 16 >= M * G && (p.tiles - 1) * 16 < M * G && p.JT >= 1 && p.groups * p.JT >= p.tiles && (p.groups - 1) * p.JT < p.tiles);
    CHECK(p.chunks >= 1 && p.chunks <= (p.form == Kv8Form::stream ? 128 : 64));
    CHECK(p.JT == 1 || p.chunks == 1);                       // (the joining kernel knows single tiles only)
    CHECK(p.runs >= 1 && p.runs * p.run_len >= p.groups && (p.runs == 1 || (int64_t)n_seq * n_kv * p.chunks < 8));
    // what the kernel makes of its number: every (unit, group) once
    const int64_t units = (int64_t)n_seq * n_kv * p.chunks, grid = (units * p.runs + 7) / 8 * 8 * p.run_len;
    if (grid < 20000 && it < 2000) {
      std::vector<int> seen(units * p.groups, 0);
      for (int64_t b = 0; b < grid; ++b) {
        const int64_t run = (b / (8 * p.run_len)) * 8 + (b & 7), unit = run / p.runs, grp = p.groups - 1 - ((b >> 3) % p.run_len * p.runs + run % p.runs);
        if (grp >= 0 && unit < units) ++seen[unit * p.groups + grp];
      }
      for (int n : seen) CHECK(n == 1);
    }
    CHECK(p.chunks > 1 ? p.part_floats == (int64_t)n_seq * n_kv * p.tiles * p.chunks * (16 * D + 32) : p.part_floats == 0);
    for (int c : {0, 1, 7, 8, 9, 100, 3000}) CHECK(kv8_chunks_used(c, p.chunks) >= 1 && kv8_chunks_used(c, p.chunks) <= p.chunks);
  }
}

alignas(16) static unsigned char mem[256];
static int32_t ints[4] = {0, 0, 0, 0};

static void refusals() {
  // (device pointers in earnest; a refused call looks at none of them)
  bd_kv8 c{mem, reinterpret_cast<uint32_t*>(mem), ints, ints, nullptr, 4, 2, 64, 2, 8};
  auto with = [&](auto f) { bd_kv8 x = c; f(x); return x; };
  auto write = [&](const bd_kv8* x, const void* k = mem, int64_t s0 = 512, int64_t s1 = 128, int dt = BD_BF16, int M = 4) {
    return bd_k_kv8_write(nullptr, x, k, s0, s1, mem, 512, 128, dt, M, nullptr);
  };
  auto read = [&](const bd_kv8* x, void* k = mem, int64_t s0 = 512, int64_t s1 = 128, int dt = BD_BF16, int M = 4) {
    return bd_k_kv8_read(nullptr, x, ints, M, nullptr, dt, k, s0, s1, mem, 512, 128);
  };
  int mode = BD_MODE_CAUSAL, window = 0, sinks = 0, n_q = 4, M = 4;
  float scale = 0.f;
  int64_t q_row = 256, o_row = 256;
  void* ws = mem;
  int64_t wsn = 1 << 30;
  const void* q = mem;
  auto attn = [&](const bd_kv8* x) { return bd_k_kv8_attention(nullptr, x, q, 1024, q_row, n_q, M, nullptr, mode, window, sinks, scale, mem, 1024, o_row, ws, wsn); };
  const bd_kv8 bad[] = {with([](bd_kv8& x) { x.D = 96; }), with([](bd_kv8& x) { x.D = 0; }), with([](bd_kv8& x) { x.n_pages = 0; }), with([](bd_kv8& x) { x.n_kv = 0; }),
                        with([](bd_kv8& x) { x.n_kv = 5000; }), with([](bd_kv8& x) { x.n_seq = 0; }), with([](bd_kv8& x) { x.n_seq = 65536; }),
                        with([](bd_kv8& x) { x.max_blocks = 0; }), with([](bd_kv8& x) { x.max_blocks = (1 << 25) + 1; })};
  for (const bd_kv8& x : bad) {
    CHECK(write(&x) == BD_E_ARG && read(&x) == BD_E_ARG && attn(&x) == BD_E_ARG);
    CHECK(bd_k_kv8_attention_workspace(&x, 4, 4, 0, 0) == BD_E_ARG);
  }
  const bd_kv8 null[] = {with([](bd_kv8& x) { x.dev_codes = nullptr; }), with([](bd_kv8& x) { ++x.dev_codes; }), with([](bd_kv8& x) { x.dev_scales = nullptr; }),
                         with([](bd_kv8& x) { x.dev_pages = nullptr; })};
  for (const bd_kv8& x : null) CHECK(write(&x) == BD_E_ARG && read(&x) == BD_E_ARG && attn(&x) == BD_E_ARG);
  const bd_kv8 no_len = with([](bd_kv8& x) { x.dev_len = nullptr; });
  CHECK(write(&no_len) == BD_E_ARG && attn(&no_len) == BD_E_ARG);
  CHECK(write(nullptr) == BD_E_ARG && read(nullptr) == BD_E_ARG && attn(nullptr) == BD_E_ARG && bd_k_kv8_attention_workspace(nullptr, 4, 4, 0, 0) == BD_E_ARG);
  for (int m : {0, -1, (1 << 22) + 1}) CHECK(write(&c, mem, 512, 128, BD_BF16, m) == BD_E_ARG && read(&c, mem, 512, 128, BD_BF16, m) == BD_E_ARG);
  CHECK(write(&c, mem, 512, 128, BD_FP8_E4M3) == BD_E_DTYPE && read(&c, mem, 512, 128, 7) == BD_E_DTYPE);
  CHECK(write(&c, nullptr) == BD_E_ARG && write(&c, mem + 2) == BD_E_ARG && read(&c, mem + 8) == BD_E_ARG);
  CHECK(write(&c, mem, 516, 128) == BD_E_ARG && write(&c, mem, 512, 132) == BD_E_ARG && write(&c, mem, -512, 128) == BD_E_ARG && write(&c, mem, 512, -128) == BD_E_ARG);
  CHECK(read(&c, mem, 512, 120) == BD_E_ARG && read(&c, mem, 120, 128) == BD_E_ARG && read(&c, mem, 512, 0) == BD_E_ARG);
  for (int v : {-1, 2}) { mode = v; CHECK(attn(&c) == BD_E_ARG); }
  mode = BD_MODE_BIDIR;
  window = -1; CHECK(attn(&c) == BD_E_ARG); window = 0;
  sinks = -1; CHECK(attn(&c) == BD_E_ARG); sinks = 0;
  for (int v : {0, -4, 5, 1 << 17}) { n_q = v; CHECK(attn(&c) == BD_E_ARG); } n_q = 4;
  for (int v : {0, (1 << 22) + 1}) { M = v; CHECK(attn(&c) == BD_E_ARG); } M = 4;
  for (float v : {-1.f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity()}) { scale = v; CHECK(attn(&c) == BD_E_ARG); } scale = 0.f;
  for (float v : {std::ldexp(1.f, 127) * 1.001f, 3e38f, std::numeric_limits<float>::max()}) { scale = v; CHECK(attn(&c) == BD_E_ARG); } scale = 0.f;      // (times log2 e infinite)
  M = 1 << 22; n_q = 8; CHECK(attn(&c) == BD_E_ARG); M = 4; n_q = 4;       // more tiles than a launch has room for
  {
    bd_kv8 many = c;
    many.n_kv = 4096;
    CHECK(write(&many, mem, 1 << 20, 1 << 20, BD_BF16, (1 << 16) + 1) == BD_E_ARG);
    many.n_pages = 1 << 20;
    CHECK(write(&many, mem, 1 << 20, 1 << 20) == BD_E_ARG);
  }
  q_row = 252; CHECK(attn(&c) == BD_E_ARG); q_row = 256;
  o_row = 248; CHECK(attn(&c) == BD_E_ARG); o_row = 256;
  q = nullptr; CHECK(attn(&c) == BD_E_ARG); q = mem;
  bd_kv8 longer = c;
  longer.max_blocks = 4096;
  const int64_t need = bd_k_kv8_attention_workspace(&longer, 4, 4, 0, 0);
  CHECK(need > 0);
  wsn = need - 1; CHECK(attn(&longer) == BD_E_CAPACITY && std::strstr(bd_last_error(), "workspace") != nullptr);
  wsn = need; ws = nullptr; CHECK(attn(&longer) == BD_E_ARG);
  ws = mem + 4; CHECK(attn(&longer) == BD_E_ARG);

  bd_rope p;
  CHECK(bd_k_rope_plan(nullptr, 128, 128, 0, 1e6, 0, 1.0, 1) == BD_E_ARG);
  struct { int D, R, layout; double theta; int scaling; double factor; int trained; } plans[] = {
      {96, 64, 0, 1e6, 0, 1, 1}, {64, 66, 0, 1e6, 0, 1, 1}, {64, 0, 0, 1e6, 0, 1, 1}, {64, 33, 0, 1e6, 0, 1, 1}, {64, 64, 2, 1e6, 0, 1, 1}, {64, 64, -1, 1e6, 0, 1, 1},
      {64, 64, 0, 1.0, 0, 1, 1}, {64, 64, 0, NAN, 0, 1, 1}, {64, 64, 0, INFINITY, 0, 1, 1}, {64, 64, 0, 1e6, 4, 2, 1}, {64, 64, 0, 1e6, -1, 2, 1}, {64, 64, 0, 1e6, 1, 0.5, 1},
      {64, 64, 0, 1e6, 3, 2, 0}, {64, 64, 0, 1e6, 1, NAN, 1}, {64, 2, 0, 1e6, 2, 2, 1}, {64, 4, 0, 1e300, 2, 1e300, 1}};
  for (auto& x : plans) CHECK(bd_k_rope_plan(&p, x.D, x.R, x.layout, x.theta, x.scaling, x.factor, x.trained) == BD_E_ARG);
  CHECK(bd_k_rope_plan(&p, 128, 64, BD_ROPE_INTERLEAVED, 1e4, BD_ROPE_PLAIN, 0.0, 0) == BD_OK && p.inv_freq[0] == 1.0 && p.amplitude == 1.f && p.rotary_dim == 64);
  auto rope = [&](const bd_rope* pl, const void* x = mem, int64_t xs = 128, int dt = BD_F32, int heads = 1, int n = 1, int m = 2, const int32_t* pos = ints) {
    return bd_k_rope(nullptr, pl, x, 256, xs, mem, 256, 128, dt, heads, n, m, pos, nullptr);
  };
  CHECK(rope(nullptr) == BD_E_ARG && rope(&p, nullptr) == BD_E_ARG && rope(&p, mem + 4) == BD_E_ARG && rope(&p, mem, 130) == BD_E_ARG && rope(&p, mem, 128, 9) == BD_E_DTYPE);
  CHECK(rope(&p, mem, 128, BD_F32, 0) == BD_E_ARG && rope(&p, mem, 128, BD_F32, 2) == BD_E_ARG && rope(&p, mem, 128, BD_F32, 1, 0) == BD_E_ARG &&
        rope(&p, mem, 128, BD_F32, 1, 1, 0) == BD_E_ARG && rope(&p, mem, 128, BD_F32, 1, 1, 2, nullptr) == BD_E_ARG);
  CHECK(rope(&p, mem, 192) == BD_E_ARG);                     // in place with another stride
  for (auto f : {+[](bd_rope& x) { x.D = 32; }, +[](bd_rope& x) { x.rotary_dim = 130; }, +[](bd_rope& x) { x.rotary_dim = 7; }, +[](bd_rope& x) { x.layout = 5; }}) {
    bd_rope x = p;
    f(x);
    CHECK(rope(&x) == BD_E_ARG);
  }
}

int main() {
  layout();
  exponents();
  quotients();
  rows();
  span();
  plan();
  refusals();
  std::printf(failures == 0 ? "ALL OK\n" : "%d failures\n", failures);
  return failures != 0;
}
