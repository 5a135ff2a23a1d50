"""The 8-bit key/value cache (write, read, attention) and the rotary positions on the GPU, through the binding, against plain implementations in 64
bits that follow the definitions in include/bd_kernels.h: values and scales exactly, attention and rotation within bounds derived from
the roundings they are allowed."""
import math

import numpy as np
import pytest
import torch

from paper_2604_06832_amd import binding

pytestmark = pytest.mark.gpu

BIDIR, CAUSAL = binding.BD_MODE_BIDIR, binding.BD_MODE_CAUSAL
E_MIN, E_MAX = -117, 119
F32, BF16 = torch.float32, torch.bfloat16


# ---- plain implementations ------------------------------------------------------------------------------------------------

def nearest_e4m3(x):
    """Nearest e4m3 value (four significant bits, subnormals in steps of 2^-9, at most 448), ties to even; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 1.0))
    step = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    y = np.minimum(np.rint(a / step) * step, 448.0)
    y = np.where(np.isinf(x), 448.0, y) * np.sign(np.where(np.isnan(x), 1.0, x))
    return np.where(np.isnan(x), np.nan, y)


def exponent(amax):
    for e in range(E_MIN, E_MAX):
        if amax <= 448.0 * 2.0 ** e:
            return e
    return E_MAX


class PlainCache:
    """One sequence: values (code times scale) and exponents, block by block."""

    def __init__(self, blocks, n_kv, D):
        self.v = np.zeros((2, blocks * 32, n_kv, D))
        self.e = np.full((2, blocks, n_kv), E_MIN)

    def write(self, n, k, v):
        for x, new in enumerate((k, v)):
            rows = len(new)
            for b in range(n // 32, -(-(n + rows) // 32) if rows else 0):
                lo, hi = max(n, 32 * b), min(n + rows, 32 * b + 32)
                for h in range(new.shape[1]):
                    part = new[lo - n:hi - n, h].astype(np.float64)
                    fin = np.abs(part[np.isfinite(part)])
                    e = exponent(fin.max() if fin.size else 0.0)
                    if lo > 32 * b:
                        e = max(e, self.e[x, b, h])
                        self.v[x, 32 * b:lo, h] = nearest_e4m3(self.v[x, 32 * b:lo, h] * 2.0 ** -e) * 2.0 ** e
                    self.v[x, lo:hi, h] = nearest_e4m3(part * 2.0 ** -float(e)) * 2.0 ** e
                    self.v[x, hi:32 * b + 32, h] = 0.0
                    self.e[x, b, h] = e


def sees(p, key, end, mode, window, sinks):
    s = key < end
    if mode == CAUSAL:
        s = s & (key <= p)
    if window:
        s = s & ((p - key < window) | (key < sinks))
    return s


def plain_attention(q, k, v, n, mode, window, sinks, scale):
    """q [rows, n_q, D], k and v [n + rows, n_kv, D] in 64 bits: result, and the bound on what the kernel may be off by.

    The kernel rounds the weights w of the softmax to bf16, each by at most 2^-8 of itself, and divides by the sum of the rounded ones: the result o moves
    by sum w_j d_j (v_j - o) / sum w_j with |d_j| <= 2^-8, at most 2^-8 (a + |o|) with a = sum w_j |v_j| / sum w_j.  Its result is rounded by 2^-8 |o| more.  A score
    is a sum of D products in fp32, off by at most D 2^-23 sum|q k|, which moves a weight by that times the scale, relatively; twice that, for
    numerator and denominator, and 2^-20 for the exponentials and sums."""
    rows, n_q, D = q.shape
    G = n_q // k.shape[1]
    at, key = n + np.arange(rows)[:, None], np.arange(n + rows)[None]
    vis = sees(at, key, n + rows, mode, window, sinks)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(n_q):
        kh, vh = k[:, h // G], v[:, h // G]
        s = np.where(vis, scale * (q[:, h] @ kh.T), -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        moved = 2 * scale * D * 2.0 ** -23 * np.where(vis, np.abs(q[:, h]) @ np.abs(kh).T, 0).max(1, keepdims=True) + 2.0 ** -20
        a = w @ np.abs(vh)
        out[:, h] = w @ vh
        tol[:, h] = 2.0 ** -8 * (2 * np.abs(out[:, h]) + a) * (1 + 2.0 ** -8) + moved * (a + np.abs(out[:, h]))
    return out, tol


def plain_rope(x, first, plan):
    y = x.astype(np.float64).copy()
    R = plan.rotary_dim
    for i in range(R // 2):
        a, b = (i, i + R // 2) if plan.layout == binding.BD_ROPE_HALF else (2 * i, 2 * i + 1)
        t = (first + np.arange(len(x)))[:, None] * plan.inv_freq[i]
        c, s = np.cos(t) * plan.amplitude, np.sin(t) * plan.amplitude
        u, w = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        y[..., a], y[..., b] = u * c - w * s, w * c + u * s
    return y


def cuda_ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def random_heads(rng, rows, heads, D, kind="n"):
    x = rng.standard_normal((rows, heads, D))
    if kind == "k":
        x = (x + rng.standard_normal((heads, D))) * np.where(rng.random((heads, D)) < 4 / D, 5.0, 0.8)
    return x


class Rig:
    """A cache of n_seq sequences with pages dealt out in random order, and its plain counterpart."""

    def __init__(self, rng, n_seq, blocks, n_kv, D, spare=2):
        self.n_seq, self.blocks, self.n_kv, self.D = n_seq, blocks, n_kv, D
        n_pages = n_seq * blocks + spare
        self.table = rng.permutation(n_pages)[:n_seq * blocks].reshape(n_seq, blocks)
        self.codes = torch.randint(0, 256, (n_pages, n_kv, 64 * D), dtype=torch.uint8, device="cuda")        # (unwritten pages hold anything, NaN too)
        self.scales = torch.randint(0, 1 << 30, (n_pages, n_kv), dtype=torch.int32, device="cuda")
        self.lens, self.status = cuda_ints([0] * n_seq), cuda_ints([0])
        self.pages = cuda_ints(self.table.tolist())
        self.cache = binding.Kv8Cache(self.codes, self.scales, self.pages, self.lens, self.status)
        self.plain = [PlainCache(blocks, n_kv, D) for _ in range(n_seq)]

    def write(self, lens, k, v, rows=None, plain=True):
        """k, v: per sequence [rows, n_kv, D]; padded here with what must not be read."""
        M = max(1, max(len(x) for x in k))
        dtype = self.dtype
        pad = torch.full((2, self.n_seq, M, self.n_kv, self.D), float("nan"), dtype=dtype, device="cuda")
        for s in range(self.n_seq):
            pad[0, s, :len(k[s])] = torch.from_numpy(k[s]).to(dtype)
            pad[1, s, :len(v[s])] = torch.from_numpy(v[s]).to(dtype)
        self.lens.copy_(cuda_ints(lens))
        self.cache.bd_k_kv8_write(pad[0], pad[1], rows=cuda_ints([len(x) for x in k]))
        for s in range(self.n_seq):
            self.plain[s].write(lens[s], pad[0, s, :len(k[s])].float().cpu().numpy(), pad[1, s, :len(v[s])].float().cpu().numpy())

    dtype = F32

    def read(self, start, rows, dtype=F32):
        M = max(1, max(rows))
        k = torch.full((self.n_seq, M, self.n_kv, self.D), 7.25, dtype=dtype, device="cuda")
        v = k.clone()
        self.cache.bd_k_kv8_read(cuda_ints(start), k, v, rows=cuda_ints(rows))
        return k, v

    def check(self, upto):
        """Positions [0, upto[s]) and the exponents of their blocks are the plain ones, exactly."""
        for dtype in (F32, BF16):
            k, v = self.read([0] * self.n_seq, upto, dtype)
            for s in range(self.n_seq):
                for x, got in enumerate((k, v)):
                    np.testing.assert_array_equal(got[s, :upto[s]].double().cpu().numpy(), self.plain[s].v[x, :upto[s]])
                    assert (got[s, upto[s]:] == 7.25).all()                                   # rows past the count stay as they were
        word = self.scales.cpu().numpy().astype(np.int64)[self.table]
        for s in range(self.n_seq):
            n = -(-upto[s] // 32)
            np.testing.assert_array_equal(word[s, :n] & 255, self.plain[s].e[0, :n] + 127)
            np.testing.assert_array_equal(word[s, :n] >> 8 & 255, self.plain[s].e[1, :n] + 127)
        assert int(self.status) == 0


# ---- write and read ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_kv,D", [(1, 64), (2, 128), (3, 64), (8, 128)])
def test_rows_come_back_as_the_nearest_codes(dtype, n_kv, D):
    rng = np.random.default_rng(n_kv * D)
    rig = Rig(rng, 4, 7, n_kv, D)
    rig.dtype = dtype
    new = lambda rows, scale: [random_heads(rng, r, n_kv, D, "k") * scale for r in rows]      # noqa: E731
    # prompts of all kinds of lengths, then appends that start inside a block and grow or do not grow its scale
    rig.write([0, 0, 0, 0], new([1, 32, 70, 0], 1.0), new([1, 32, 70, 0], 1.0))
    rig.check([1, 32, 70, 0])
    rig.write([1, 32, 70, 0], new([1, 5, 64, 33], 40.0), new([1, 5, 64, 33], 0.01))
    rig.check([2, 37, 134, 33])
    rig.write([2, 37, 134, 33], new([150, 0, 3, 31], 0.3), new([150, 0, 3, 31], 300.0))
    rig.check([152, 37, 137, 64])
    # cut back inside a block and written again: the positions behind are gone, the block's scale stays where earlier rows hold it
    rig.write([40, 33, 130, 64], new([2, 1, 1, 0], 1e-3), new([2, 1, 1, 0], 1e-3))
    rig.check([64, 64, 160, 64])                                                              # (cleared up to the end of the touched block)


@pytest.mark.parametrize("D", [64, 128])
def test_values_at_the_ends_of_the_range(D):
    rng = np.random.default_rng(5)
    rig = Rig(rng, 1, 12, 1, D)
    rows = np.zeros((32 * 9, 1, D))
    rows[0, 0, :4] = [np.inf, -np.inf, 1.0, 3.0]                       # infinities saturate and do not move the scale
    rows[32, 0, :3] = [np.nan, 2.0, -5.0]                              # a NaN stays one
    rows[64, 0, :3] = [3.4e38, -1e30, 1.0]                             # past 448 2^119
    rows[96, 0, :5] = [2.0 ** -149, 2.0 ** -126, 1.5 * 2.0 ** -127, 2.0 ** -128, -2.0 ** -126]
    rows[128, 0, :8] = [448.0, 432.0, 440.0, 17.0, 18.0, 19.0, 2.0 ** -9, 2.0 ** -10]      # ties, to even
    rows[160:192, 0] = np.exp2(rng.uniform(-25, 5, (32, D))) * rng.choice([-1, 1], (32, D))  # down through the subnormal codes
    rows[192, 0, 0] = 449.0                                            # one step over
    rows[224:256, 0] = rng.integers(-64, 65, (32, D)) / 16.0
    rows[256, 0, :3] = [np.inf, np.nan, -np.inf]                       # nothing finite but zeros
    half = rng.permutation(rows.reshape(9, -1), axis=1).reshape(rows.shape)
    rig.write([0], [rows], [half])
    rig.check([rows.shape[0]])
    # more rows behind a block that holds such values
    rig.write([288], [rows[:20]], [half[32:52]])
    rig.write([308], [rows[224:230] * 1e5], [half[224:230] * 1e-30])
    rig.check([314])


def test_strided_rows_and_shared_pages():
    """Keys and values as slices of a projection's output, M the outer dimension; a prefix page on two lists."""
    rng = np.random.default_rng(11)
    n_kv, D, M = 2, 128, 40
    rig = Rig(rng, 2, 4, n_kv, D)
    first = random_heads(rng, 32, n_kv, D)
    rig.write([0, 0], [first, first[:0]], [first, first[:0]])
    rig.table[1, 0] = rig.table[0, 0]                                  # sequence 1 goes on from the same first block
    rig.pages.copy_(cuda_ints(rig.table.tolist()))
    rig.plain[1].v[:, :32], rig.plain[1].e[:, :1] = rig.plain[0].v[:, :32], rig.plain[0].e[:, :1]
    qkv = torch.randn((M, 2, 3 * n_kv + 2, D), device="cuda").to(BF16).transpose(0, 1)          # [n_seq, M, heads, D], rows outside
    k, v = qkv[:, :, 1:1 + n_kv], qkv[:, :, 3 + n_kv:3 + 2 * n_kv]
    rig.lens.copy_(cuda_ints([32, 32]))
    rig.cache.bd_k_kv8_write(k, v)
    for s in range(2):
        rig.plain[s].write(32, k[s].float().cpu().numpy(), v[s].float().cpu().numpy())
    rig.check([72, 72])
    out = torch.zeros((72, 2, 2 * n_kv + 1, D), device="cuda", dtype=BF16).transpose(0, 1)
    rig.cache.bd_k_kv8_read(None, out[:, :, :n_kv], out[:, :, n_kv:2 * n_kv])
    for s in range(2):
        np.testing.assert_array_equal(out[s, :, :n_kv].double().cpu().numpy(), rig.plain[s].v[0, :72])
        np.testing.assert_array_equal(out[s, :, n_kv:2 * n_kv].double().cpu().numpy(), rig.plain[s].v[1, :72])
    assert (out[:, :, 2 * n_kv:] == 0).all()


@pytest.mark.parametrize("M", [3, 75])
def test_read_from_the_middle(M):
    rng = np.random.default_rng(M)
    rig = Rig(rng, 3, 6, 2, 64)
    x = [random_heads(rng, 190, 2, 64) for _ in range(3)]
    rig.write([0, 0, 0], x, x[::-1])
    start, rows = [0, 31, 190 - M], [M, M - 1, M]
    k, v = rig.read(start, rows, BF16)
    for s in range(3):
        np.testing.assert_array_equal(k[s, :rows[s]].double().cpu().numpy(), rig.plain[s].v[0, start[s]:start[s] + rows[s]])
        np.testing.assert_array_equal(v[s, :rows[s]].double().cpu().numpy(), rig.plain[s].v[1, start[s]:start[s] + rows[s]])
    assert (k[1, rows[1]:] == 7.25).all()


def test_a_new_cache_holds_zeros_until_it_is_written():
    pages = cuda_ints([[2, 0], [1, 3]])
    cache = binding.Kv8Cache.empty(4, 2, 64, pages, cuda_ints([0, 0]))
    k, v = torch.full((2, 2, 40, 2, 64), 7.25, device="cuda")
    cache.bd_k_kv8_read(None, k, v)
    assert (k == 0).all() and (v == 0).all()
    x = torch.randint(-8, 9, (2, 40, 2, 64), device="cuda").float()    # (integers to 8 are e4m3 numbers)
    cache.bd_k_kv8_write(x, -x)
    cache.bd_k_kv8_read(None, k, v)
    assert torch.equal(k, x) and torch.equal(v, -x)


def test_pages_past_32_bits_of_bytes():
    n_pages, n_kv, D = 300000, 2, 128                                  # 4.9 GB of codes
    codes = torch.zeros((n_pages, n_kv, 64 * D), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, n_kv), dtype=torch.int32, device="cuda")
    cache = binding.Kv8Cache(codes, scales, cuda_ints([[n_pages - 1, 5, n_pages - 2]]), cuda_ints([0]))
    rng = np.random.default_rng(3)
    x = torch.from_numpy(random_heads(rng, 80, n_kv, D)).to(BF16).cuda()[None]
    cache.bd_k_kv8_write(x, -x)
    plain = PlainCache(3, n_kv, D)
    plain.write(0, x[0].float().cpu().numpy(), -x[0].float().cpu().numpy())
    k, v = torch.empty((1, 80, n_kv, D), device="cuda"), torch.empty((1, 80, n_kv, D), device="cuda")
    cache.bd_k_kv8_read(None, k, v)
    np.testing.assert_array_equal(k[0].double().cpu().numpy(), plain.v[0, :80])
    np.testing.assert_array_equal(v[0].double().cpu().numpy(), plain.v[1, :80])
    q = torch.randn((1, 1, 4, D), device="cuda").to(BF16)
    cache.lens.fill_(79)
    out = cache.bd_k_kv8_attention(q, torch.empty_like(q), CAUSAL)
    want, tol = plain_attention(q[0].double().cpu().numpy(), plain.v[0, :80], plain.v[1, :80], 79, CAUSAL, 0, 0, D ** -0.5)
    assert (np.abs(out[0].double().cpu().numpy() - want) <= tol).all()


# ---- attention --------------------------------------------------------------------------------------------------------------

def in_form(rig, form, n_q, M):
    """The cache as a call that takes another form of the kernel has it, and how many times over: more (sequence, kv head, tile) items than CUs
    (all sequences again and again, on the same pages), or page lists long enough for a cache that is not kept (nothing in their rest)."""
    n, n_kv, D = rig.n_seq, rig.n_kv, rig.D
    tiles = -(-M * (n_q // n_kv) // 16)
    if form == "wide" and tiles > 1:
        times = 256 // (n * n_kv * tiles) + 1
        return binding.Kv8Cache(rig.codes, rig.scales, rig.pages.repeat(times, 1), rig.lens.repeat(times), rig.status), times
    if form == "stream" and tiles == 1:
        pages = torch.full((n, (96 << 20) // (n * n_kv * 64 * D) + 1), -1, dtype=torch.int32, device="cuda")
        pages[:, :rig.blocks] = rig.pages
        return binding.Kv8Cache(rig.codes, rig.scales, pages, rig.lens, rig.status), 1
    return None, 0


def attend(rig, q, lens, rows, mode, window=0, sinks=0, scale=0.0, workspace=None):
    """The rows of q (per sequence [rows, n_q, D]) through the cache, which holds everything already, in the forms that they can take: compared, and
    returned as the plain call gives them."""
    n_q, D = q[0].shape[1:]
    M = max(1, max(rows))
    pad = torch.full((rig.n_seq, M, n_q, D), float("nan"), dtype=BF16, device="cuda")
    for s in range(rig.n_seq):
        pad[s, :rows[s]] = torch.from_numpy(q[s]).to(BF16)
    out = torch.full_like(pad, 3.5)
    rig.lens.copy_(cuda_ints(lens))
    rig.cache.bd_k_kv8_attention(pad, out, mode, window, sinks, scale, rows=cuda_ints(rows), workspace=workspace)
    outs = [out]
    for form in ("wide", "stream"):
        cache, times = in_form(rig, form, n_q, M)
        if times:
            again = torch.full((times * rig.n_seq, M, n_q, D), 3.5, dtype=BF16, device="cuda")
            cache.bd_k_kv8_attention(pad.repeat(times, 1, 1, 1), again, mode, window, sinks, scale, rows=cuda_ints(rows * times))
            again = again.view(times, *pad.shape)
            assert torch.equal(again, again[:1].expand_as(again))
            outs.append(again[0])
    worst = 0.0
    for s in range(rig.n_seq):
        for o in outs:
            assert (o[s, rows[s]:] == 3.5).all()
        if rows[s] == 0:
            continue
        end = lens[s] + rows[s]
        want, tol = plain_attention(pad[s, :rows[s]].double().cpu().numpy(), rig.plain[s].v[0, :end], rig.plain[s].v[1, :end], lens[s], mode, window, sinks,
                                    scale or D ** -0.5)
        for o in outs:
            got = o[s, :rows[s]].double().cpu().numpy()
            assert np.isfinite(got).all()
            worst = max(worst, float((np.abs(got - want) / np.maximum(tol, 1e-30)).max()))
            assert (np.abs(got - want) <= tol).all(), f"sequence {s}: {np.abs(got - want).max()} off, {worst} of the bound"
    assert int(rig.status) == 0
    print(f"attention: {worst:.2f} of the bound, {len(outs)} forms", flush=True)
    return out


def filled(rng, ends, n_kv, D, spare_blocks=2):
    rig = Rig(rng, len(ends), -(-max(ends) // 32) + spare_blocks, n_kv, D)
    rig.dtype = BF16
    rig.write([0] * len(ends), [random_heads(rng, e, n_kv, D, "k") for e in ends], [random_heads(rng, e, n_kv, D) for e in ends])
    return rig


@pytest.mark.parametrize("mode", [BIDIR, CAUSAL])
@pytest.mark.parametrize("n_q,n_kv,D,lens,rows", [
    (4, 2, 64, [0], [1]), (4, 2, 64, [0], [5]), (16, 2, 128, [1], [1]), (16, 2, 128, [31], [1]), (16, 2, 128, [32], [1]), (16, 2, 128, [1024], [32]),
    (16, 2, 128, [1000], [64]), (6, 2, 128, [77], [3]), (5, 1, 64, [300], [7]), (8, 8, 64, [513], [16]), (28, 4, 128, [95], [33]), (1, 1, 128, [64], [1]),
    (16, 2, 128, [700, 0, 33, 5, 1999], [3, 1, 0, 4, 2]), (32, 8, 128, [255, 256, 257], [1, 1, 1]), (48, 1, 64, [10, 200], [2, 9]), (16, 2, 128, [200], [300]),
    (4, 2, 64, [0], [700])])
def test_attention_matches_the_softmax_in_64_bits(n_q, n_kv, D, lens, rows, mode):
    rng = np.random.default_rng(sum(lens) + sum(rows) + D)
    rig = filled(rng, [a + b for a, b in zip(lens, rows)], n_kv, D)
    attend(rig, [random_heads(rng, r, n_q, D) * 1.5 for r in rows], lens, rows, mode)


@pytest.mark.parametrize("mode", [BIDIR, CAUSAL])
@pytest.mark.parametrize("n,rows,window,sinks", [
    (500, 32, 1, 0), (500, 32, 64, 4), (500, 7, 100, 33), (500, 1, 31, 0), (500, 1, 33, 32), (90, 40, 20, 1), (500, 32, 400, 100), (500, 32, 10000, 5),
    (0, 20, 3, 2), (300, 200, 50, 70), (3000, 16, 128, 4), (33, 1, 2, 31)])
def test_attention_with_a_window_and_first_tokens(n, rows, window, sinks, mode):
    rng = np.random.default_rng(n + rows + window)
    rig = filled(rng, [n + rows], 2, 64)
    attend(rig, [random_heads(rng, rows, 6, 64) * 1.5], [n], [rows], mode, window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (5000, 8)])
def test_attention_on_a_long_cache(window, sinks):
    rng = np.random.default_rng(8)
    rig = filled(rng, [40003, 9001], 1, 128)
    attend(rig, [random_heads(rng, 3, 8, 128), random_heads(rng, 1, 8, 128)], [40000, 9000], [3, 1], CAUSAL, window, sinks)


@pytest.mark.parametrize("lens", [[300], [2600], [70001], [40000, 10, 3000]])
def test_single_tokens_in_one_to_a_hundred_and_more_chunks(lens):
    rng = np.random.default_rng(lens[0])
    rig = filled(rng, [n + 1 for n in lens], 1, 64)
    attend(rig, [random_heads(rng, 1, 8, 64) * 1.5 for _ in lens], lens, [1] * len(lens), CAUSAL)


@pytest.mark.parametrize("n_seq,M,n_q,n,blocks", [(64, 8, 8, 17000, 540), (14, 40, 8, 8500, 270), (512, 1, 8, 8500, 400)])
def test_more_blocks_than_a_wavefront_looks_up_at_once(n_seq, M, n_q, n, blocks):
    """Many sequences on the same pages, so long that every wavefront walks more than 64 blocks: one tile and eight wavefronts, two tiles and four, and one tile
    of a cache that is not kept."""
    rng = np.random.default_rng(n_seq)
    D, n_kv = 64, 2 if n_seq == 64 else 1
    rig = filled(rng, [n + M], n_kv, D)
    pages = torch.full((n_seq, blocks), -1, dtype=torch.int32, device="cuda")
    pages[:, :rig.blocks] = rig.pages
    cache = binding.Kv8Cache(rig.codes, rig.scales, pages, cuda_ints([n] * n_seq), rig.status)
    assert cache.bd_k_kv8_attention_workspace(n_q, M) == 0             # one chunk each
    q = torch.from_numpy(random_heads(rng, M, n_q, D) * 1.5).to(BF16).cuda()[None].repeat(n_seq, 1, 1, 1)
    out = cache.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL)
    want, tol = plain_attention(q[0].double().cpu().numpy(), rig.plain[0].v[0, :n + M], rig.plain[0].v[1, :n + M], n, CAUSAL, 0, 0, D ** -0.5)
    assert (np.abs(out[0].double().cpu().numpy() - want) <= tol).all()
    assert torch.equal(out, out[:1].expand_as(out)) and int(rig.status) == 0


def test_the_last_positions_that_a_page_list_can_hold():
    """Rows up to position 2^30 give the bits that they give at the start of a cache (a window's keys are all that either sees)."""
    rng = np.random.default_rng(24)
    codes, scales = torch.zeros((16, 2, 64 * 128), dtype=torch.uint8, device="cuda"), torch.zeros((16, 2), dtype=torch.int32, device="cuda")
    status, outs, values = cuda_ints([0]), [], []
    k, v, q = (torch.from_numpy(random_heads(rng, r, h, 128)).to(BF16).cuda()[None] for r, h in ((104, 2), (104, 2), (8, 16)))
    for blocks, first in ((1 << 25, 2 ** 30 - 104), (8, 24)):
        pages = torch.full((1, blocks), -1, dtype=torch.int32, device="cuda")
        pages[0, first // 32:first // 32 + 4] = cuda_ints([3, 11, 0, 7])
        lens = cuda_ints([first])
        cache = binding.Kv8Cache(codes, scales, pages, lens, status)
        cache.bd_k_kv8_write(k, v)
        values.append(torch.zeros((2, 1, 104, 2, 128), device="cuda"))
        cache.bd_k_kv8_read(lens, *values[-1])
        lens += 96
        outs.append(cache.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL, window=64))
        codes.zero_()
    assert torch.equal(values[0], values[1]) and torch.equal(outs[0], outs[1])
    assert bool(values[0].any()) and bool(outs[0].any()) and int(status) == 0


def test_scores_far_apart_and_the_scale_argument():
    """Weights that are all but one, and maxima that move late: the largest scores at the end of the cache."""
    rng = np.random.default_rng(9)
    rig = Rig(rng, 1, 20, 1, 64)
    n = 600
    k, v = random_heads(rng, n, 1, 64), random_heads(rng, n, 1, 64)
    k *= np.linspace(0.1, 30, n)[:, None, None]
    rig.write([0], [k], [v])
    q = [random_heads(rng, 4, 2, 64) * 3]
    attend(rig, q, [n - 4], [4], BIDIR)
    attend(rig, q, [n - 4], [4], CAUSAL, 0, 0, 0.011)
    attend(rig, q, [n - 4], [4], CAUSAL, 100, 3, 1.7)


@pytest.mark.parametrize("rows,form", [(8, "plain"), (8, "wide"), (4, "plain"), (4, "stream")])
def test_what_a_row_does_not_see_does_not_reach_it(rows, form):
    """NaN among keys and values: rows that see one are NaN (all of a row by a key, its dimension by a value), the others as if there were none."""
    rng = np.random.default_rng(12)
    n, D, n_q = 70, 64, 4
    rig = filled(rng, [n + rows + 10], 1, D)
    cache, times = (rig.cache, 1) if form == "plain" else in_form(rig, form, n_q, rows)

    def run(q, start, *args, **kw):
        rig.lens.fill_(start)
        cache.lens.fill_(start)
        q = q.repeat(times, 1, 1, 1)
        out = cache.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL, *args, **kw)
        assert torch.equal(out.nan_to_num(777.0), out[:1].expand_as(out).nan_to_num(777.0))
        return out[0]

    q = torch.from_numpy(random_heads(rng, rows, n_q, D)).to(BF16).cuda()[None]
    j, i = rows - 3, rows - 2                                          # the rows with the bad value and the bad key
    nan_v, nan_k = random_heads(rng, rows + 10, 1, D), random_heads(rng, rows + 10, 1, D)
    good_k, good_v = nan_k.copy(), nan_v.copy()
    nan_v[j, 0, 9] = np.nan
    nan_k[i, 0, 0] = np.nan
    nan_v[rows + 2:], nan_k[rows + 2:] = np.nan, np.nan               # and all behind the last row
    good_k[i, 0, 0], good_v[j, 0, 9], good_k[rows + 2:], good_v[rows + 2:] = 0.0, 0.0, 0.0, 0.0
    rig.write([n], [good_k], [good_v])
    clean = run(q, n)
    rig.write([n], [nan_k], [nan_v])
    out = run(q, n)
    assert torch.equal(out[:j], clean[:j])
    assert torch.isnan(out[j, :, 9]).all() and torch.isnan(out[i:]).all()
    keep = [d for d in range(D) if d != 9]
    assert torch.equal(out[j][:, keep], clean[j][:, keep])
    # a window that leaves them out again, and a query that is NaN itself: only its own row
    rig.write([n + rows], [random_heads(rng, rows, 1, D)], [random_heads(rng, rows, 1, D)])
    q = torch.from_numpy(random_heads(rng, rows, n_q, D)).to(BF16).cuda()[None]
    q[0, 2, 1, 0] = float("nan")
    out = run(q, n + rows, window=2, sinks=10)
    bad = torch.isnan(out).any(-1)
    assert bad[2, 1] and int(bad.sum()) == 1 and torch.isnan(out[2, 1]).all()


def test_bad_rows_and_pages_are_reported_and_touch_nothing():
    rng = np.random.default_rng(13)
    rig = filled(rng, [100, 100, 100], 2, 64, spare_blocks=0)          # 4 blocks: 128 positions
    before, words = rig.codes.clone(), rig.scales.clone()
    k = torch.randn((3, 8, 2, 64), device="cuda")
    q, out = torch.randn((3, 8, 4, 64), device="cuda").to(BF16), torch.full((3, 8, 4, 64), 2.5, dtype=BF16, device="cuda")
    for lens, rows in (([-1, 200, 121], [8, 1, 8]), ([2 ** 31 - 1, 100, 100], [8, -1, 9])):
        rig.lens.copy_(cuda_ints(lens))
        r = cuda_ints(rows)
        rig.cache.bd_k_kv8_write(k, k, rows=r)
        got = k.clone()
        rig.cache.bd_k_kv8_read(rig.lens, got, got.clone(), rows=r)
        rig.cache.bd_k_kv8_attention(q, out, CAUSAL, rows=r)
        assert int(rig.status) == binding.BD_KV8_BAD_ROWS
        assert torch.equal(got, k) and (out == 2.5).all() and torch.equal(rig.codes, before) and torch.equal(rig.scales, words)
        rig.status.zero_()
    # pages outside the pool: their block is left out, all else goes on
    rig.pages[0, 1], rig.pages[1, 3] = -1, rig.codes.shape[0]
    rig.lens.copy_(cuda_ints([56, 92, 92]))
    rig.cache.bd_k_kv8_write(k, k)                                     # rows 56 .. 63: block 1; 92 .. 99: blocks 2 and 3
    assert int(rig.status) == binding.BD_KV8_BAD_PAGE
    for s, n in ((1, 92), (2, 92)):
        x = k[s].cpu().numpy()
        rig.plain[s].write(n, x, x)
    kk, vv = torch.full((3, 128, 2, 64), 4.5, device="cuda"), torch.full((3, 128, 2, 64), 4.5, device="cuda")
    rig.cache.bd_k_kv8_read(None, kk, vv)
    np.testing.assert_array_equal(kk[2, :100].double().cpu().numpy(), rig.plain[2].v[0, :100])
    np.testing.assert_array_equal(kk[1, :96].double().cpu().numpy(), rig.plain[1].v[0, :96])
    assert (kk[1, 96:] == 4.5).all() and (kk[0, 32:64] == 4.5).all() and not (kk[0, :32] == 4.5).all()
    rig.status.zero_()
    rig.cache.bd_k_kv8_attention(q, out, BIDIR)
    assert int(rig.status) == binding.BD_KV8_BAD_PAGE
    # sequence 0 as if positions 32 .. 63 were not there: its rows are at 56 .. 63, the cache's 0 .. 31 are what they see
    want, tol = plain_attention(np.concatenate([np.zeros((24, 4, 64)), q[0].double().cpu().numpy()]), rig.plain[0].v[0, :32], rig.plain[0].v[1, :32], 0, BIDIR, 0, 0, 0.125)
    assert (np.abs(out[0].double().cpu().numpy() - want[24:]) <= tol[24:]).all()
    end = plain_attention(q[2].double().cpu().numpy(), rig.plain[2].v[0, :100], rig.plain[2].v[1, :100], 92, BIDIR, 0, 0, 0.125)
    assert (np.abs(out[2].double().cpu().numpy() - end[0]) <= end[1]).all()


def test_no_page_in_the_pool_gives_nan_and_a_report():
    rig = filled(np.random.default_rng(14), [40], 1, 64)
    rig.pages.fill_(-5)
    q = torch.randn((1, 1, 2, 64), device="cuda").to(BF16)
    rig.lens.fill_(39)
    out = rig.cache.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL)
    assert int(rig.status) == binding.BD_KV8_BAD_PAGE and torch.isnan(out).all()


def test_results_are_the_same_on_every_run_and_whatever_the_workspace_holds():
    rng = np.random.default_rng(15)
    lens, rows = [3000, 2500], [4, 3]
    rig = filled(rng, [3004, 2503], 2, 128)
    size = rig.cache.bd_k_kv8_attention_workspace(16, 4)
    assert size > 0
    q = [random_heads(rng, r, 16, 128) for r in rows]
    outs = [attend(rig, q, lens, rows, CAUSAL, workspace=torch.full((size,), fill, dtype=torch.uint8, device="cuda")) for fill in (0, 255, 127)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.equal(outs[0], attend(rig, q, lens, rows, CAUSAL))
    with pytest.raises(binding.BdError) as e:
        rig.cache.bd_k_kv8_attention(torch.zeros((2, 4, 16, 128), dtype=BF16, device="cuda"), torch.zeros((2, 4, 16, 128), dtype=BF16, device="cuda"), CAUSAL,
                                     workspace=torch.zeros(size - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.BD_E_CAPACITY


def test_attention_on_views_and_on_another_stream():
    """Queries as a slice of a projection's output, results into a slice of a larger tensor, on a stream of their own."""
    rng = np.random.default_rng(16)
    n, M, n_q, n_kv, D = 333, 6, 8, 2, 64
    rig = filled(rng, [n + M, n + M], n_kv, D)
    qkv = torch.randn((M, 2, n_q + 2 * n_kv, D), device="cuda").to(BF16).transpose(0, 1)
    big = torch.zeros((2, M, 2 * n_q, D), dtype=BF16, device="cuda")
    rig.lens.fill_(n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rig.cache.bd_k_kv8_attention(qkv[:, :, :n_q], big[:, :, n_q:], BIDIR)
    side.synchronize()
    for s in range(2):
        want, tol = plain_attention(qkv[s, :, :n_q].double().cpu().numpy(), rig.plain[s].v[0, :n + M], rig.plain[s].v[1, :n + M], n, BIDIR, 0, 0, D ** -0.5)
        assert (np.abs(big[s, :, n_q:].double().cpu().numpy() - want) <= tol).all()
    assert (big[:, :, :n_q] == 0).all()


# ---- rotary positions ---------------------------------------------------------------------------------------------------------

def rope_tolerance(want, x, dtype, amplitude):
    """Sine and cosine to a few 2^-24 (taken as 2^-22 with the amplitude's and the products' roundings), then the result's own."""
    pair = np.abs(x).max(-1, keepdims=True) * 2 * amplitude
    return pair * 2.0 ** -21 + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [binding.BD_ROPE_HALF, binding.BD_ROPE_INTERLEAVED])
@pytest.mark.parametrize("D,R,heads,M,pos", [
    (64, 64, 6, 5, [0, 3]), (128, 128, 18, 33, [1000, 7]), (128, 64, 3, 2, [999999, 0]), (64, 2, 1, 9, [5, 6]), (128, 34, 2, 70, [12345, 2]), (64, 50, 40, 1, [2 ** 31 - 2, 1]),
    (128, 32, 8, 3, [40, 0])])
def test_rope_against_the_rotation_in_64_bits(D, R, heads, M, pos, layout, dtype):
    x = torch.randn((2, M, heads, D), device="cuda").to(dtype)
    plan = binding.bd_k_rope_plan(D, R, layout, 1e6)
    got = binding.bd_k_rope(plan, x, cuda_ints(pos))
    for s in range(2):
        src = x[s].double().cpu().numpy()
        want = plain_rope(src, pos[s], plan)
        tol = rope_tolerance(want, src, dtype, 1.0)
        tol[..., R:] = 0.0                                             # the rest of the head is copied
        # (2^31 turns in fp64 are off by up to 2^31 2^-53 radians: nothing)
        assert (np.abs(got[s].double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("scaling", [binding.BD_ROPE_LINEAR, binding.BD_ROPE_BASE, binding.BD_ROPE_PARTS])
def test_rope_for_long_contexts_in_place_and_padded(scaling):
    plan = binding.bd_k_rope_plan(128, 96, binding.BD_ROPE_HALF, 1e4, scaling, 16.0, 4096)
    qkv = torch.randn((3, 9, 8, 128), device="cuda")
    src = qkv.double().cpu().numpy()
    x = qkv[:, :, 1:6]                                                 # some heads of a larger tensor, in place
    pos, rows = [60000, 0, 17], [9, 0, 4]
    binding.bd_k_rope(plan, x, cuda_ints(pos), out=x, rows=cuda_ints(rows))
    want = src.copy()
    tol = np.zeros(src.shape)
    for s in range(3):
        want[s, :rows[s], 1:6] = plain_rope(src[s, :rows[s], 1:6], pos[s], plan)
        tol[s, :rows[s], 1:6, :96] = rope_tolerance(want[s, :rows[s], 1:6], src[s, :rows[s], 1:6], F32, plan.amplitude)[..., :96]
    assert (np.abs(qkv.double().cpu().numpy() - want) <= tol).all()


def test_rope_with_a_position_for_each_row():
    """M = 1: every row brings its own position (the groups of a quadratic step)."""
    plan = binding.bd_k_rope_plan(64)
    pos = [100 + i + j for i in range(4) for j in range(5)]
    x = torch.randn((20, 1, 4, 64), device="cuda").to(BF16)
    got = binding.bd_k_rope(plan, x, cuda_ints(pos))
    for i, p in enumerate(pos):
        src = x[i].double().cpu().numpy()
        want = plain_rope(src, p, plan)
        assert (np.abs(got[i].double().cpu().numpy() - want) <= rope_tolerance(want, src, BF16, 1.0)).all()


def test_rope_takes_counts_outside_the_rows_as_the_nearer_end():
    plan = binding.bd_k_rope_plan(64)
    x = torch.randn((4, 1100, 2, 64), device="cuda").to(BF16)          # (4400 rows: several of a sequence to a workgroup)
    pos = cuda_ints([0, 5, 9, 1])
    out = torch.full_like(x, 7.25)
    binding.bd_k_rope(plan, x, pos, out=out, rows=cuda_ints([-2 ** 31, -1, 2 ** 31 - 1, 1101]))
    whole = binding.bd_k_rope(plan, x, pos)
    assert (out[:2] == 7.25).all() and torch.equal(out[2:], whole[2:])


# ---- together -------------------------------------------------------------------------------------------------------------------

def layer(cache, plan, qkv, turned, out, n_q, n_kv, mode, rows=None, workspace=None):
    """One layer's attention part: the heads of Q and K turned, K and V into the cache, attention."""
    binding.bd_k_rope(plan, qkv[:, :, :n_q + n_kv], cache.lens, out=turned, rows=rows)
    cache.bd_k_kv8_write(turned[:, :, n_q:], qkv[:, :, n_q + n_kv:], rows=rows)
    cache.bd_k_kv8_attention(turned[:, :, :n_q], out, mode, rows=rows, workspace=workspace)


def test_a_context_built_block_by_block_and_a_captured_step():
    """Prompt, blocks and single tokens of three sequences through rope, write and attention, against the plain ones; the step is captured once and
    replayed as the lengths move on, with eager work in between."""
    rng = np.random.default_rng(21)
    n_seq, n_q, n_kv, D, M = 3, 8, 2, 64, 12
    rig = Rig(rng, n_seq, 12, n_kv, D)
    plan = binding.bd_k_rope_plan(D)
    qkv = torch.zeros((n_seq, M, n_q + 2 * n_kv, D), dtype=BF16, device="cuda")
    turned = torch.zeros((n_seq, M, n_q + n_kv, D), dtype=BF16, device="cuda")
    out = torch.zeros((n_seq, M, n_q, D), dtype=BF16, device="cuda")
    rows = cuda_ints([0] * n_seq)
    lens = [0] * n_seq
    size = rig.cache.bd_k_kv8_attention_workspace(n_q, M)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    def step(count, run):
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        rows.copy_(cuda_ints(count))
        rig.lens.copy_(cuda_ints(lens))
        run()
        torch.cuda.synchronize()
        t = turned.double().cpu().numpy()
        for s in range(n_seq):
            r, n = count[s], lens[s]
            if r == 0:
                continue
            src = qkv[s, :r, :n_q + n_kv].double().cpu().numpy()
            want = plain_rope(src, n, plan)
            assert (np.abs(t[s, :r] - want) <= rope_tolerance(want, src, BF16, 1.0)).all()
            rig.plain[s].write(n, t[s, :r, n_q:].astype(np.float32), qkv[s, :r, n_q + n_kv:].float().cpu().numpy())
            want, tol = plain_attention(t[s, :r, :n_q], rig.plain[s].v[0, :n + r], rig.plain[s].v[1, :n + r], n, CAUSAL, 0, 0, D ** -0.5)
            assert (np.abs(out[s, :r].double().cpu().numpy() - want) <= tol).all()
            lens[s] += r

    eager = lambda: layer(rig.cache, plan, qkv, turned, out, n_q, n_kv, CAUSAL, rows, ws)         # noqa: E731
    step([12, 7, 1], eager)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.current_stream())
        eager()                                                        # (writes the same rows again)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eager()
    for count in ([12, 12, 12], [1, 1, 1], [0, 5, 12], [12, 12, 3]):
        step(count, graph.replay)
        lens[0] -= 1 if lens[0] > 20 else 0                            # a rejected draft: the last position is written again
        step([2, 1, 1], eager)
    for count in ([11, 12, 12], [1, 0, 1]):
        step(count, graph.replay)
    rig.check(lens)


def test_two_graphs_with_a_workspace_each_do_not_disturb_one_another():
    rng = np.random.default_rng(22)
    rig = filled(rng, [3000], 2, 64)
    rig.lens.fill_(2990)
    qs = [torch.randn((1, 10, 8, 64), device="cuda").to(BF16) for _ in range(2)]
    outs = [torch.zeros_like(q) for q in qs]
    size = rig.cache.bd_k_kv8_attention_workspace(8, 10)
    graphs = []
    for q, out in zip(qs, outs):
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        rig.cache.bd_k_kv8_attention(q, out, CAUSAL, workspace=ws)
        want = out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            rig.cache.bd_k_kv8_attention(q, out, CAUSAL, workspace=ws)
        graphs.append((g, out, want, ws, torch.cuda.Stream()))
    for _ in range(5):
        for g, out, _, _, stream in graphs:
            out.zero_()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for _, out, want, _, _ in graphs:
            assert torch.equal(out, want)


def test_binding_refuses_what_does_not_fit():
    rig = filled(np.random.default_rng(23), [40, 40], 2, 64)
    c = rig.cache
    k = torch.zeros((2, 4, 2, 64), dtype=BF16, device="cuda")
    q = torch.zeros((2, 4, 4, 64), dtype=BF16, device="cuda")
    for call in (lambda: c.bd_k_kv8_write(k, k.float()), lambda: c.bd_k_kv8_write(k[:1], k[:1]), lambda: c.bd_k_kv8_write(k, k[:, :3]),
                 lambda: c.bd_k_kv8_write(k.half(), k.half()), lambda: c.bd_k_kv8_write(k.transpose(2, 3).contiguous().transpose(2, 3), k),
                 lambda: c.bd_k_kv8_write(k, k, rows=torch.zeros(2, device="cuda")), lambda: c.bd_k_kv8_write(k, k, rows=cuda_ints([1])),
                 lambda: c.bd_k_kv8_write(k.cpu(), k.cpu()), lambda: c.bd_k_kv8_read(None, k, k[:, :2]), lambda: c.bd_k_kv8_attention(q.float(), q.float(), CAUSAL),
                 lambda: c.bd_k_kv8_attention(q, q[:, :2], CAUSAL), lambda: c.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL, window=2 ** 32 + 8), lambda: binding.bd_k_rope(binding.bd_k_rope_plan(64), q, cuda_ints([0])),
                 lambda: binding.bd_k_rope(binding.bd_k_rope_plan(128), q, cuda_ints([0, 0])),
                 lambda: binding.Kv8Cache(rig.codes, rig.scales[:1], rig.pages, rig.lens), lambda: binding.Kv8Cache(rig.codes, rig.scales, rig.pages, rig.lens[:1])):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros(2 * 4 * 4 * 64 + 8, dtype=BF16, device="cuda")[4:-4].view(2, 4, 4, 64)     # 8 bytes off
    for call, code in ((lambda: c.bd_k_kv8_attention(odd, q, CAUSAL), binding.BD_E_ARG), (lambda: c.bd_k_kv8_attention(q, torch.zeros_like(q), 5), binding.BD_E_ARG),
                       (lambda: c.bd_k_kv8_attention(q[:, :, :3], torch.zeros_like(q[:, :, :3]), CAUSAL), binding.BD_E_ARG),
                       (lambda: c.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL, window=-1), binding.BD_E_ARG),
                       (lambda: binding.bd_k_rope(binding.bd_k_rope_plan(64), odd, cuda_ints([0, 0])), binding.BD_E_ARG),
                       (lambda: binding.Kv8Cache(torch.zeros((2, 1, 96 * 64), dtype=torch.uint8, device="cuda"), cuda_ints([[0], [0]]), rig.pages, rig.lens)
                        .bd_k_kv8_attention_workspace(4, 4), binding.BD_E_ARG)):
        with pytest.raises(binding.BdError) as e:
            call()
        assert e.value.code == code


def test_lengths_move_on_in_place_and_are_not_replaced():
    rig = filled(np.random.default_rng(25), [40, 40], 1, 64)
    c, x = rig.cache, torch.ones((2, 1, 1, 64), device="cuda")
    for name in ("codes", "scales", "pages", "lens", "status"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name).clone())
    rig.lens.fill_(20)
    c.lens += 20                                                       # (the same tensor: the calls see it)
    c.bd_k_kv8_write(x, x)
    assert rig.lens.tolist() == [40, 40]
    k, v = rig.read([40, 40], [1, 1])
    assert (k == 1).all() and (v == 1).all()


def test_calls_refuse_numbers_past_32_bits():
    rig = filled(np.random.default_rng(26), [40], 1, 64)
    c, big = rig.cache, 1 << 32
    x = torch.zeros((1, 1, 1, 64), dtype=BF16, device="cuda")
    many = x.expand(1, big + 1, 1, 64)
    for call in (lambda: c.bd_k_kv8_attention(x, torch.zeros_like(x), big), lambda: c.bd_k_kv8_attention(x, torch.zeros_like(x), CAUSAL, window=5 - big),
                 lambda: c.bd_k_kv8_attention(x, torch.zeros_like(x), CAUSAL, window=5, sinks=4 - big), lambda: c.bd_k_kv8_attention(many, many, CAUSAL),
                 lambda: c.bd_k_kv8_write(many, many), lambda: binding.bd_k_rope(binding.bd_k_rope_plan(64), many, cuda_ints([0]), out=many)):
        with pytest.raises(ValueError):
            call()


def test_a_short_workspace_says_so():
    rig = filled(np.random.default_rng(27), [3000], 1, 64)
    rig.lens.fill_(2999)
    q = torch.zeros((1, 1, 4, 64), dtype=BF16, device="cuda")
    size = rig.cache.bd_k_kv8_attention_workspace(4, 1)
    with pytest.raises(binding.BdError, match=f"{size} bytes of workspace, got {size - 16}") as e:
        rig.cache.bd_k_kv8_attention(q, torch.zeros_like(q), CAUSAL, workspace=torch.zeros(size - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.BD_E_CAPACITY and "capacity exceeded" not in str(e.value)


def test_the_largest_scale():
    """Scores of 0 stay 0 (the scale times log2 e is finite): every visible value counts the same."""
    rig = filled(np.random.default_rng(28), [100], 1, 64)
    attend(rig, [np.zeros((4, 2, 64))], [96], [4], CAUSAL, scale=2.0 ** 127)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [binding.BD_ROPE_HALF, binding.BD_ROPE_INTERLEAVED])
@pytest.mark.parametrize("D,R", [(64, 64), (64, 34), (128, 128), (128, 80), (128, 42)])
def test_rope_of_many_rows_against_the_rotation_in_64_bits(D, R, layout, dtype):
    """Several rows to a workgroup, its last one with three, one, two rows and all four; rotary parts whose halves fall on 16 bytes, and others."""
    M, rows, pos = 1027, [1027, 1025, 1026, 1024], [0, 70001, 2 ** 30, 5]
    x = torch.randn((4, M, 3, D), device="cuda").to(dtype)
    plan = binding.bd_k_rope_plan(D, R, layout, 1e6, binding.BD_ROPE_PARTS, 4.0, 8192)
    out = torch.full_like(x, 7.25)
    binding.bd_k_rope(plan, x, cuda_ints(pos), out=out, rows=cuda_ints(rows))
    for s in range(4):
        n = rows[s]
        src = x[s, :n].double().cpu().numpy()
        want = plain_rope(src, pos[s], plan)
        tol = rope_tolerance(want, src, dtype, plan.amplitude)
        tol[..., R:] = 0.0
        assert (np.abs(out[s, :n].double().cpu().numpy() - want) <= tol).all(), f"sequence {s}"
        assert (out[s, n:] == 7.25).all()
    y = x.clone()
    binding.bd_k_rope(plan, y, cuda_ints(pos), out=y, rows=cuda_ints(rows))        # in place: the same
    for s in range(4):
        assert torch.equal(y[s, :rows[s]], out[s, :rows[s]]) and torch.equal(y[s, rows[s]:], x[s, rows[s]:])
