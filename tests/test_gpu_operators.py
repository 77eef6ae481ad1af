"""The operators in the 8-bit container against plain implementations in 64 bits.

Rounding to E4M3 and the pages of the cache are compared exactly: scales are powers of two, so there is one rounding, to a
grid that the oracle writes down.

The matrix product: E4M3 products and scales are exact, so only sums and the last rounding are not.  The tensor cores add 32
products to the accumulator at a time, aligned to the largest of them; what is cut off each time is below a few units of 2^-24
of the largest, and the largest is at most S = sum |x w|.  Bound: (C / 32 + 1) 2^-22 S, and half a step of the result's type.

The attention: with p the exact weights (sum 1), a weight is rounded to 11 bits (2^-11 relative), and a score's absolute
error d (in powers of two) changes it by a factor 2^d: d is D 2^-23 A for A = sum |q k| in those units, accumulated like
above, and twice 2^-22 for the exponential and the products around it.  Numerator and denominator both have the second kind.  Bound: (2^-11 + 4 ln 2
(D 2^-23 A + 2^-21)) sum p |v|, and half a step of the result's type."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2609_34185_b200 as ep

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
gpu = pytest.mark.gpu


# ---- oracles in 64 bits ----------------------------------------------------------------------------------------------

GRID = sorted({(1 + f / 8) * 2.0 ** e for e in range(-6, 9) for f in range(8)} - {480.0} | {f / 8 * 2.0 ** -6 for f in range(8)})
GRID = torch.tensor(GRID, dtype=torch.float64)


def on_grid(x):
    """The nearest E4M3 value, ties to the one with an even last bit; NaN for what is not finite."""
    a = x.abs().nan_to_num(0.0, 0.0, 0.0).clamp(max=448.0).contiguous()
    hi = torch.searchsorted(GRID, a).clamp(max=len(GRID) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = GRID[hi] - a, a - GRID[lo]
    index = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.where(x.isfinite(), torch.copysign(GRID[index], x), math.nan)


def fitting(amax, zero, least):
    """The smallest power of two s, at least 2^least, with amax <= 448 s."""
    if amax == 0:
        return zero
    s = 2.0 ** least
    while amax > 448 * s:
        s *= 2
    return s


def quantized(x, rows):
    x = x.double().cpu()
    T, C = x.shape
    q = torch.empty_like(x)
    s = torch.empty(-(-T // rows), -(-C // 128), dtype=torch.float64)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            block = x[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128]
            fine = block[block.isfinite()]
            s[i, j] = fitting(float(fine.abs().max()) if fine.numel() else 0.0, 1.0, -126)
            q[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128] = on_grid(block / s[i, j])
    return q, s


def same(got, want):
    got, want = got.float().double().cpu(), want.cpu()
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def cuda(seed):
    return torch.Generator("cuda").manual_seed(seed)


# ---- rounding ----------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,C,rows", [(1, 1, 1), (1, 5120, 1), (3, 127, 1), (7, 129, 1), (2, 2056, 1), (130, 1000, 1), (1, 128, 128), (128, 128, 128),
                                      (129, 200, 128), (300, 1032, 128), (127, 77, 128)])
def test_quantize(T, C, rows, dtype):
    g = cuda(T * 7919 + C)
    x = (torch.randn(T, C, generator=g, device="cuda") * torch.exp(6 * torch.randn(T, 1, generator=g, device="cuda"))).clamp(-60000, 60000).to(dtype)
    q, s = ep.quantize_blocks(x, rows)
    want, scales = quantized(x, rows)
    assert q.dtype == E4M3 and s.dtype == E8M0
    assert same(s, scales) and same(q, want)


@gpu
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_edges(rows):
    # one block per case: powers and fractions around 448 2^k, halfway values, the smallest and largest numbers, zeros, what is not finite
    inf, nan = math.inf, math.nan
    cases = [[448.0], [448.0001], [449.0], [896.0], [897.0], [0.0], [-0.0], [inf], [nan], [-inf, 1.0], [nan, -3.0], [1e-40], [1.2e-38], [3.4e38], [2.0 ** -126, 2.0 ** -130],
             [448.0, 0.001953125, 0.0009765625, 0.00146484375, 17.0, 19.0, 21.0, -17.0, -19.0], [3.4e38, 1.0, inf, nan, -inf], [1.75, 1.76, -1.0625, 1.1875]]
    x = torch.zeros(len(cases) * rows, 128)
    for i, c in enumerate(cases):
        x[i * rows + rows // 2, 3:3 + len(c)] = torch.tensor(c)
    q, s = ep.quantize_blocks(x.cuda(), rows)
    want, scales = quantized(x, rows)
    assert same(s, scales) and same(q, want)


@gpu
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_views_and_outputs(rows, dtype):
    # rows of any distance and alignment, results into parts of larger buffers whose other bytes stay
    base = torch.randn(140, 700, generator=cuda(5), device="cuda").to(dtype)
    for c0, C in ((0, 700), (8, 512), (1, 333), (3, 690)):
        x = base[:, c0:c0 + C]
        shape = (-(-140 // rows), -(-C // 128))
        qb = torch.full((140, C + 9), 3, dtype=torch.uint8, device="cuda").view(E4M3)
        sb = torch.full((shape[0], shape[1] + 2), 3, dtype=torch.uint8, device="cuda").view(E8M0)
        ep.quantize_blocks(x, rows, out=(qb[:, 5:5 + C], sb[:, 1:1 + shape[1]]))
        want, scales = quantized(x, rows)
        assert same(qb[:, 5:5 + C], want) and same(sb[:, 1:1 + shape[1]], scales)
        rest = qb.view(torch.uint8).clone()
        rest[:, 5:5 + C] = 3
        assert bool((rest == 3).all())
        rest = sb.view(torch.uint8).clone()
        rest[:, 1:1 + shape[1]] = 3
        assert bool((rest == 3).all())


# ---- product -----------------------------------------------------------------------------------------------------------

def operands(T, R, C, seed, pitch=0):
    g = cuda(seed)
    x = torch.randn(T, C, generator=g, device="cuda") * torch.exp(2 * torch.randn(T, 1, generator=g, device="cuda"))
    x *= torch.exp2(torch.randint(-6, 7, (1, -(-C // 128)), generator=g, device="cuda").float()).repeat_interleave(128, 1)[:, :C]
    w = torch.randn(R, C, generator=g, device="cuda")
    w *= torch.exp2(torch.randint(-6, 7, (-(-R // 128), -(-C // 128)), generator=g, device="cuda").float()).repeat_interleave(128, 0)[:R].repeat_interleave(128, 1)[:, :C]
    (xq, xs), (wq, ws) = ep.quantize_blocks(x), ep.quantize_blocks(w, 128)
    if pitch:
        xb, wb = (torch.full((n, C + pitch), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3) for n in (T, R))      # NaN between the rows
        xb[:, :C], wb[:, :C] = xq, wq
        xq, wq = xb[:, :C], wb[:, :C]
    return xq, xs, wq, ws


def product(xq, xs, wq, ws, a=None):
    """The product and the sum of magnitudes, in 64 bits."""
    C, R = xq.shape[1], wq.shape[0]
    x = xq.float().double() * (xs.float().double().repeat_interleave(128, 1)[:, :C] if xs is not None else 1)
    w = wq.float().double()
    if ws is not None:
        w = w * ws.float().double().repeat_interleave(128, 0)[:R].repeat_interleave(128, 1)[:, :C]
    if a is not None:
        w = w * a.double()[:, None]
    return x @ w.t(), x.abs() @ w.abs().t()


def check_product(y, want, S, C):
    bound = (C / 32 + 1) * 2.0 ** -22 * S + HALF_STEP[y.dtype] * want.abs() * (1 + 2.0 ** -10) + 1e-30
    if y.dtype == torch.float16:
        bound = bound + 2.0 ** -25
    err = (y.double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


@gpu
@pytest.mark.parametrize("T,R,C", [(1, 1, 16), (1, 128, 128), (1, 512, 5120), (5, 200, 144), (16, 129, 1040), (17, 300, 2048), (33, 1000, 640), (64, 64, 8192), (65, 257, 400),
                                   (127, 128, 1024), (128, 384, 256), (129, 520, 3840), (300, 1000, 528), (700, 2100, 784)])
@pytest.mark.parametrize("out", [ep.BF16, ep.FP16, ep.FP32])
def test_matmul(T, R, C, out):
    xq, xs, wq, ws = operands(T, R, C, T + 3 * R + 7 * C)
    a = torch.rand(R, generator=cuda(R), device="cuda") * 2.0 ** -14 + 2.0 ** -16
    y = ep.fp8_matmul(xq, xs, wq, ws, a, out)
    want, S = product(xq, xs, wq, ws, a)
    check_product(y, want, S, C)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("T,R,C", [(3, 10240, 784), (100, 300, 1040), (128, 2000, 256), (1500, 600, 2064), (2000, 5000, 272), (4100, 2600, 128), (193, 8200, 1936), (513, 257, 16)])
def test_matmul_shapes_of_the_ways_it_is_shared_out(T, R, C):
    # three CTAs per tile; two tiles of 64 tokens; pairs of CTAs with several tiles each, one block of columns, odd numbers of blocks, ragged edges
    xq, xs, wq, ws = operands(T, R, C, T + R + C)
    a = torch.rand(R, generator=cuda(R), device="cuda") + 0.5
    for out in (ep.BF16, ep.FP32):
        y = ep.fp8_matmul(xq, xs, wq, ws, a, out)
        want, S = product(xq, xs, wq, ws, a)
        check_product(y, want, S, C)
    assert torch.equal(ep.fp8_matmul(xq, xs, wq, ws, a, ep.FP32), y)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("T", [2, 40, 200])
def test_matmul_without_scales_and_with_strides(T):
    R, C = 330, 912
    xq, xs, wq, ws = operands(T, R, C, 11 * T, pitch=48)
    buffer = torch.full((T, R + 7), 5.0, device="cuda", dtype=torch.bfloat16)
    y = buffer[:, 3:3 + R]
    ep.fp8_matmul(xq, xs, wq, out=y)
    want, S = product(xq, xs, wq, None)
    check_product(y, want, S, C)
    assert bool((buffer[:, :3] == 5).all()) and bool((buffer[:, 3 + R:] == 5).all())
    wide = torch.full((T, xs.shape[1] + 5), 0xFF, dtype=torch.uint8, device="cuda").view(E8M0)                       # NaN between the scales
    wide[:, 2:2 + xs.shape[1]] = xs
    ep.fp8_matmul(xq, wide[:, 2:2 + xs.shape[1]], wq, ws, out=y)
    want, S = product(xq, xs, wq, ws)
    check_product(y, want, S, C)


@gpu
@pytest.mark.parametrize("T", [1, 20, 150])
def test_matmul_nan_stays_in_its_row(T):
    R, C = 260, 1280
    xq, xs, wq, ws = operands(T, R, C, 77)
    want, S = product(xq, xs, wq, ws)
    xq, wq = xq.view(torch.uint8).clone(), wq.view(torch.uint8).clone()
    wq[131, 700] = 0xFF
    xq[T // 2, 1279] = 0x7F
    y = ep.fp8_matmul(xq.view(E4M3), xs, wq.view(E4M3), ws, out_dtype=ep.FP32)
    bad = torch.zeros(T, R, dtype=torch.bool, device="cuda")
    bad[T // 2], bad[:, 131] = True, True
    assert torch.equal(y.isnan(), bad)
    check_product(torch.where(bad, 0.0, y), torch.where(bad, 0.0, want), S, C)


@gpu
def test_matmul_large_magnitudes():
    # scales at both ends of E8M0, products that meet in the middle
    xq, _, wq, _ = operands(9, 140, 384, 5)
    xs = torch.full((9, 3), 2.0 ** 100, device="cuda").to(E8M0)
    ws = torch.full((2, 3), 2.0 ** -110, device="cuda").to(E8M0)
    y = ep.fp8_matmul(xq, xs, wq, ws, out_dtype=ep.FP32)
    want, S = product(xq, xs, wq, ws)
    check_product(y, want, S, 384)


@gpu
def test_matmul_is_the_same_every_time():
    xq, xs, wq, ws = operands(10, 700, 5120, 3)
    first = ep.fp8_matmul(xq, xs, wq, ws, out_dtype=ep.FP32)
    for _ in range(20):
        assert torch.equal(ep.fp8_matmul(xq, xs, wq, ws, out_dtype=ep.FP32), first)


# ---- cache -------------------------------------------------------------------------------------------------------------

class Plain:
    """A cache in 64 bits: what was written, the pages' scales and values."""

    def __init__(self, cache):
        self.k, self.v, self.ks, self.vs = (t.float().double().cpu() for t in cache)

    def append(self, k, v, table, lens, starts):
        page = self.k.shape[2]
        for b, ln in enumerate(lens):
            rows = list(range(starts[b], starts[b + 1]))
            rows = rows[max(0, len(rows) - ln):]
            first = ln - len(rows)
            for j in range(first // page, -(-ln // page) if rows else 0):
                p, lo, hi = table[b][j], max(first, j * page), min(ln, (j + 1) * page)
                for values, scales, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
                    for h in range(values.shape[1]):
                        new = x[rows[lo - first]:rows[hi - 1 - first] + 1, h].double().cpu()
                        fine = new[new.isfinite()]
                        s = fitting(float(fine.abs().max()) if fine.numel() else 0.0, 2.0 ** -100, -100)
                        if lo > j * page:
                            s = max(s, float(scales[p, h]))
                            values[p, h, :lo - j * page] = on_grid(values[p, h, :lo - j * page] * (float(scales[p, h]) / s))
                        values[p, h, lo - j * page:hi - j * page] = on_grid(new / s)
                        scales[p, h] = s


def ints(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def paged(lens, page, spare=2, seed=0, columns=None):
    """A table for requests of these lengths, pages in random order, and the number of pages."""
    blocks = [-(-n // page) for n in lens]
    pages = sum(blocks) + spare
    order = np.random.default_rng(seed).permutation(pages).tolist()
    columns = columns or max(max(blocks), 1)
    table, at = [], 0
    for n in blocks:
        table.append(order[at:at + n] + [0] * (columns - n))
        at += n
    return table, pages


def offsets(news):
    return [sum(news[:i]) for i in range(len(news) + 1)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,D,page,steps", [(1, 64, 16, [[1, 0, 3], [1, 1, 1], [16, 15, 14]]), (3, 128, 16, [[40, 1, 17], [1, 1, 1], [1, 30, 0]]),
                                            (2, 128, 64, [[64, 63, 65], [1, 1, 1], [1, 1, 1], [100, 0, 5]]), (2, 64, 256, [[300, 2, 1], [1, 1, 1], [9, 255, 0]]),
                                            (1, 128, 128, [[7, 0, 0], [0, 0, 200], [1, 1, 1]])])
def test_append(H, D, page, steps, dtype):
    B = 3
    ends = [sum(s[b] for s in steps) for b in range(B)]
    table, pages = paged(ends, page, seed=H + D + page)
    cache = ep.kv_cache(pages, H, D, page)
    for t in cache[:2]:
        t.view(torch.uint8).fill_(0x7E)                   # what nobody writes stays
    plain, lens, g = Plain(cache), [0] * B, cuda(D + page)
    for i, news in enumerate(steps):
        lens = [a + b for a, b in zip(lens, news)]
        n = sum(news)
        # later tokens larger now and then, so that scales grow; a request's channel of zeros, a NaN and an infinity
        k = torch.randn(n, H, D, generator=g, device="cuda") * 4.0 ** (i % 3) * 2.0 ** torch.randint(-8, 9, (n, 1, 1), generator=g, device="cuda")
        v = torch.randn(n, H, D, generator=g, device="cuda") * (0.0 if i == 0 else 1e-3)
        if n > 2:
            k[1, 0, 5], v[n - 1, H - 1, D - 1], v[0, 0, 0] = math.nan, math.inf, -math.inf
        k, v = k.to(dtype), v.to(dtype)
        ep.cache_append(cache, k, v, ints(table), ints(lens), ints(offsets(news)))
        plain.append(k, v, table, lens, offsets(news))
        assert same(cache.k_scales, plain.ks) and same(cache.v_scales, plain.vs)
        assert same(cache.k, plain.k) and same(cache.v, plain.v)
    assert ep.last_device_status() == 0


@gpu
def test_append_strided_rows_and_fewer_tokens_than_rows():
    # rows of one fused projection; a request whose length is less than its rows keeps the last of them; a row of nobody
    H, D, page = 2, 64, 32
    qkv = torch.randn(50, (4 + 2 * H) * D, generator=cuda(2), device="cuda").to(torch.bfloat16)
    k, v = (qkv[:, (4 + i * H) * D:(4 + (i + 1) * H) * D].unflatten(1, (H, D)) for i in range(2))
    lens, starts = [10, 0, 25], [0, 15, 20, 49]
    table, pages = paged([10, 1, 25], page)
    cache = ep.kv_cache(pages, H, D, page)
    plain = Plain(cache)
    ep.cache_append(cache, k, v, ints(table), ints(lens), ints(starts))
    plain.append(k, v, table, lens, starts)
    assert same(cache.k, plain.k) and same(cache.v, plain.v) and same(cache.k_scales, plain.ks) and same(cache.v_scales, plain.vs)


def filled(lens, H, D, page, seed, spare=2, columns=None):
    """A cache with random tokens for requests of these lengths; what lies behind a request's last token is NaN."""
    table, pages = paged(lens, page, spare, seed, columns)
    g = cuda(seed)
    cache = ep.kv_cache(pages, H, D, page)
    for values, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        x = torch.randn(pages, H, page, D, generator=g, device="cuda")
        scales.copy_(torch.exp2(torch.randint(-6, 3, (pages, H), generator=g, device="cuda").float()))
        values.copy_(x.mul_(2).clamp_(-448, 448).to(E4M3))
    cache.v_scales.mul_(3.7)                              # any positive scale serves the attention
    used = torch.zeros(pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            used[table[b][j], :min(page, n - j * page)] = True
    for t in cache[:2]:
        t.view(torch.uint8).masked_fill_(~used.cuda()[:, None, :, None], 0x7F)
    return cache, table


def attended(q, cache, table, lens, starts, scale, causal, dead=()):
    """Output, bound and log-sum-exp in 64 bits; NaN where a row sees a NaN."""
    N, Hq, D = q.shape
    H, page = cache[0].shape[1], cache[0].shape[2]
    G = Hq // H
    o = torch.zeros(N, Hq, D, dtype=torch.float64)
    bound, lse = torch.zeros_like(o), torch.full((N, Hq), -math.inf, dtype=torch.float64)
    k, v, ks, vs = (t.float().double().cpu() for t in cache)
    q = q.double().cpu()
    for b, ln in enumerate(lens):
        n = starts[b + 1] - starts[b]
        ids = table[b][:-(-ln // page)]
        if not n or not ln:
            continue
        alive = torch.tensor([ids[j // page] not in dead for j in range(ln)])
        ids = [0 if i in dead else i for i in ids]
        for h in range(H):
            K = (k[ids, h] * ks[ids, h, None, None]).reshape(-1, D)[:ln]
            V = (v[ids, h] * vs[ids, h, None, None]).reshape(-1, D)[:ln]
            for i in range(n):
                sees = ((torch.arange(ln) <= ln - n + i) if causal else torch.ones(ln, dtype=torch.bool)) & alive
                if not sees.any():
                    continue
                Q = q[starts[b] + i, h * G:(h + 1) * G]
                x = Q @ K[sees].t() * scale
                A = (Q.abs() @ K[sees].abs().t() * abs(scale) * math.log2(math.e)).nan_to_num(0.0).amax(1, keepdim=True)
                p = torch.softmax(x, 1)
                at = slice(h * G, (h + 1) * G)
                o[starts[b] + i, at] = p @ V[sees]
                lse[starts[b] + i, at] = torch.logsumexp(x, 1)
                bound[starts[b] + i, at] = (2.0 ** -11 + 4 * math.log(2) * (D * 2.0 ** -23 * A + 2.0 ** -21)) * (p @ V[sees].abs())
    return o, bound, lse


def check_attention(got, want, bound):
    got64 = got.double().cpu()
    bound = bound + HALF_STEP[got.dtype] * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -24
    assert torch.equal(got64.isnan(), want.isnan())
    err = (got64 - want).abs().nan_to_num(0.0)
    assert bool((err <= bound.nan_to_num(0.0) + want.isnan()).all()), float((err / bound).nan_to_num(0.0).max())


ATTENTION = [  # heads per group, heads, dim, page, tokens, rows
    (1, 1, 64, 16, [1], [1]), (1, 1, 128, 16, [0], [1]), (5, 2, 128, 64, [131, 1, 64, 0, 700], [1, 1, 1, 1, 1]), (8, 1, 128, 16, [257, 255, 33], [1, 1, 1]),
    (16, 1, 64, 32, [300], [1]), (3, 2, 64, 256, [513, 90], [2, 1]), (4, 1, 128, 128, [1000, 4, 2], [4, 4, 4]), (8, 2, 128, 64, [77, 400], [4, 3]),
    (5, 1, 128, 64, [200], [200]), (2, 2, 64, 16, [100, 333, 40], [37, 1, 40]), (4, 2, 128, 32, [500, 90, 10], [100, 0, 10]), (32, 1, 128, 64, [600], [2]),
    (1, 8, 128, 64, [2100], [1]), (7, 1, 64, 64, [129, 65], [65, 64]),
]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("G,H,D,page,lens,news", ATTENTION)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(G, H, D, page, lens, news, causal, dtype):
    cache, table = filled(lens, H, D, page, seed=G + D + page + len(lens))
    starts = offsets(news)
    q = torch.randn(starts[-1], G * H, D, generator=cuda(D), device="cuda").mul_(1.5).to(dtype)
    lse = torch.full((starts[-1], G * H), 7.0, device="cuda")
    out = torch.full_like(q, 9.0)
    ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts), scale=0.2, causal=causal, out=out, lse=lse)
    want, bound, want_lse = attended(q, cache, table, lens, starts, 0.2, causal)
    check_attention(out, want, bound)
    seen = want_lse > -math.inf
    assert torch.equal(lse.cpu() > -math.inf, seen)
    assert bool(((lse.double().cpu() - want_lse)[seen].abs() <= 1e-3).all())
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("G,H,lens", [(5, 8, [9000, 17, 4000, 1]), (1, 1, [30000]), (16, 2, [5000, 5001, 4999])])
def test_attention_split_over_many_ctas(G, H, lens):
    # segments that many CTAs share, and several segments in one CTA; the same bits every time
    cache, table = filled(lens, H, 128, 64, seed=41)
    starts = list(range(len(lens) + 1))
    q = torch.randn(len(lens), G * H, 128, generator=cuda(8), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts))
    want, bound, _ = attended(q, cache, table, lens, starts, 128 ** -0.5, True)
    check_attention(out, want, bound)
    for _ in range(5):
        assert torch.equal(ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts)), out)


@gpu
def test_attention_scores_far_apart():
    # rows of very different size, scores of hundreds, a first token that takes everything and one that comes last
    lens, starts = [600, 90], [0, 3, 5]
    cache, table = filled(lens, 2, 128, 64, seed=12)
    cache.k.view(torch.uint8)[table[0][0], :, 0] = 0x70       # 128 everywhere
    cache.k.view(torch.uint8)[table[1][1], :, 25] = 0x70
    q = torch.randn(5, 6, 128, generator=cuda(4), device="cuda") * torch.tensor([1e-20, 1.0, 30.0, 1e-3, 8.0], device="cuda")[:, None, None]
    for dtype in (torch.bfloat16, torch.float16):
        x = q.abs().to(dtype)
        out = ep.cache_attention(x, cache, ints(table), ints(lens), ints(starts))
        want, bound, _ = attended(x, cache, table, lens, starts, 128 ** -0.5, True)
        check_attention(out, want, bound)


@gpu
@pytest.mark.parametrize("news,G", [([9, 3], 1), ([70, 40], 4)])
def test_attention_nan_counts_for_the_rows_that_see_it(news, G):
    lens, starts = [100, 60], offsets(news)
    cache, table = filled(lens, 1, 64, 16, seed=3)
    cache.k.view(torch.uint8)[table[0][6], 0, 1, 7] = 0x7F     # token 97 of the first request
    cache.v.view(torch.uint8)[table[1][3], 0, 10, 33] = 0xFF   # token 58 of the second, one column
    q = torch.randn(starts[-1], G, 64, generator=cuda(6), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts))
    want, bound, _ = attended(q, cache, table, lens, starts, 0.125, True)
    assert want[starts[1] - 3:starts[1]].isnan().all() and not want[:starts[1] - 3].isnan().any()
    assert want[-2:, :, 33].isnan().all() and want.isnan().sum() == 3 * G * 64 + 2 * G
    check_attention(out, want, bound)


@gpu
def test_attention_strides_and_rows_of_nobody():
    G, H, D, lens, starts = 4, 2, 64, [50, 70], [2, 3, 5]
    cache, table = filled(lens, H, D, 32, seed=9, columns=5)
    qkv = torch.randn(7, (G * H + 2 * H) * D, generator=cuda(1), device="cuda").to(torch.float16)
    q = qkv[:, :G * H * D].unflatten(1, (G * H, D))
    buffer = torch.full((7, G * H, D + 8), 3.0, dtype=torch.float16, device="cuda")
    out = buffer[:, :, :D]
    wide = torch.full((2, 9), 10 ** 6, dtype=torch.int32, device="cuda")
    wide[:, 2:7] = ints(table)
    ep.cache_attention(q, cache, wide[:, 2:7], ints(lens), ints(starts), out=out)
    want, bound, _ = attended(q, cache, table, lens, starts, 0.125, True)
    check_attention(out[2:5], want[2:5], bound[2:5])
    assert bool((buffer[:, :, D:] == 3).all()) and bool((out[:2] == 3).all()) and bool((out[5:] == 3).all())


# ---- several at once, captures, other streams ----------------------------------------------------------------------------

@gpu
def test_a_layer_from_its_stream_to_its_output():
    """A layer as it is served: weights decoded into the container, activations rounded, projections, cache, attention,
    output projection; over two steps, the second of single tokens, each also from a captured graph."""
    H, G, D, page = 2, 4, 128, 64
    C, Hq = 512, H * G
    rng = np.random.default_rng(8)
    blobs, scales = [], []
    for R, cols in (((Hq + 2 * H) * D, C), (C, Hq * D)):
        W = rng.standard_normal((R, cols)).astype(np.float32) * 0.05
        a = np.abs(W).max(1) / 448
        blobs.append(ep.upload(ep.encode((W / a[:, None]).astype(np.float32), 5.0)))
        scales.append(torch.from_numpy(a).cuda())
    weights = [ep.decode(b, ep.FP8_E4M3) for b in blobs]
    table, pages = paged([141, 40], page)
    cache = ep.kv_cache(pages, H, D, page)
    plain = Plain(cache)
    lens = [0, 0]
    for news in ([140, 39], [1, 1]):
        lens = [a + b for a, b in zip(lens, news)]
        starts, n = offsets(news), sum(news)
        x = torch.randn(n, C, generator=cuda(n), device="cuda").to(torch.bfloat16)
        t, sl, st = ints(table), ints(lens), ints(starts)

        def layer():
            xq, xs = ep.quantize_blocks(x)
            qkv = ep.fp8_matmul(xq, xs, weights[0], row_scale=scales[0])
            heads = qkv.unflatten(1, (Hq + 2 * H, D))
            ep.cache_append(cache, heads[:, Hq:Hq + H], heads[:, Hq + H:], t, sl, st)
            o = ep.cache_attention(heads[:, :Hq], cache, t, sl, st)
            oq, os = ep.quantize_blocks(o.flatten(1))
            return xq, xs, qkv, o, oq, os, ep.fp8_matmul(oq, os, weights[1], row_scale=scales[1])

        xq, xs, qkv, o, oq, os, y = layer()
        assert same(xq, quantized(x, 1)[0])
        check_product(qkv, *product(xq, xs, weights[0], None, scales[0]), C)
        heads = qkv.unflatten(1, (Hq + 2 * H, D))
        plain.append(heads[:, Hq:Hq + H], heads[:, Hq + H:], table, lens, starts)
        assert same(cache.k, plain.k) and same(cache.v, plain.v)
        want, bound, _ = attended(heads[:, :Hq], cache, table, lens, starts, D ** -0.5, True)
        check_attention(o, want, bound)
        assert same(oq, quantized(o.flatten(1), 1)[0])
        check_product(y, *product(oq, os, weights[1], None, scales[1]), Hq * D)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            again = layer()
        graph.replay()                                    # (the same tokens at the same places: the cache stays as it is)
        torch.cuda.synchronize()
        for a, b in zip(again, (xq, xs, qkv, o, oq, os, y)):
            assert torch.equal(a.float(), b.float())
    assert ep.last_device_status() == 0


@gpu
def test_captured_attention_serves_other_lengths():
    lens = [700, 30, 256]
    cache, table = filled(lens, 2, 128, 64, seed=21)
    q = torch.randn(3, 8, 128, generator=cuda(2), device="cuda").to(torch.bfloat16)
    t, sl, st = ints(table), ints(lens), ints([0, 1, 2, 3])
    ep.cache_attention(q, cache, t, sl, st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ep.cache_attention(q, cache, t, sl, st)
    for now in ([700, 30, 256], [1, 5, 100], [650, 0, 3]):
        sl.copy_(ints(now))
        graph.replay()
        want, bound, _ = attended(q, cache, table, now, [0, 1, 2, 3], 128 ** -0.5, True)
        check_attention(out, want, bound)


@gpu
def test_calls_on_two_streams():
    xq, xs, wq, ws = operands(40, 2000, 4096, 6)
    lens = [3000, 100]
    cache, table = filled(lens, 4, 128, 64, seed=5)
    q = torch.randn(2, 8, 128, generator=cuda(3), device="cuda").to(torch.bfloat16)
    t, sl, st = ints(table), ints(lens), ints([0, 1, 2])
    y, o = ep.fp8_matmul(xq, xs, wq, ws), ep.cache_attention(q, cache, t, sl, st)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(20):
        s = streams[i % 2]
        got.append((ep.fp8_matmul(xq, xs, wq, ws, stream=s), ep.cache_attention(q, cache, t, sl, st, stream=s)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, y) and torch.equal(b, o) for a, b in got)


@gpu
def test_pages_outside_the_cache_are_passed_over():
    lens, starts = [100, 40], [0, 1, 2]
    cache, table = filled(lens, 1, 64, 32, seed=15)
    bad = [row[:] for row in table]
    bad[0][1], bad[1][1] = len(cache.k) + 5, -3
    q = torch.randn(2, 4, 64, generator=cuda(1), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(bad), ints(lens), ints(starts))
    with pytest.raises(ep.EntroPackError) as e:
        ep.binding._check(ep.last_device_status(), "status")
    assert e.value.status == -9
    want, bound, _ = attended(q, cache, bad, lens, starts, 0.125, True, dead=(len(cache.k) + 5, -3))
    check_attention(out, want, bound)
    before = [t.clone() for t in cache]
    k = torch.randn(2, 1, 64, generator=cuda(7), device="cuda").to(torch.bfloat16)
    bad[0][3], bad[1][1] = 10 ** 9, -2 ** 31
    ep.cache_append(cache, k, k, ints(bad), ints(lens), ints(starts))
    assert ep.last_device_status() == -9 and ep.last_device_status() == 0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, cache))


@gpu
def test_lengths_and_starts_outside_are_cut():
    cache, table = filled([64, 64], 1, 64, 32, seed=2, spare=0)
    q = torch.randn(3, 2, 64, generator=cuda(5), device="cuda").to(torch.bfloat16)
    out = torch.full_like(q, 4.0)
    ep.cache_attention(q, cache, ints(table), ints([2 ** 31 - 1, -7]), ints([-5, 2, 10 ** 6]), out=out)
    want, bound, _ = attended(q, cache, table, [64, 0], [0, 2, 3], 0.125, True)
    check_attention(out, want, bound)
    ep.cache_append(cache, q[:, :1], q[:, :1], ints(table), ints([2 ** 31 - 1, -7]), ints([-5, 2, 10 ** 6]))
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("new", [1, 100])
def test_a_cache_beyond_32_bits_of_bytes(new):
    # 4.5 GB of keys and of values, the requests' pages at its end; against the same pages in a small cache
    H, D, page, pages = 8, 128, 128, 36000
    big, small = ep.kv_cache(pages, H, D, page), ep.kv_cache(8, H, D, page)
    lens, starts = [300, 500], [0, new, 2 * new]
    near, far = [[0, 1, 2, 0], [3, 4, 5, 6]], [[pages - 1, pages - 2, pages - 3, 0], [pages - 4, pages - 5, pages - 6, pages - 7]]
    g = cuda(50)
    k, v = (torch.randn(800, H, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(2 * new, 4 * H, D, generator=g, device="cuda").to(torch.bfloat16)
    out = []
    for cache, table in ((small, near), (big, far)):
        ep.cache_append(cache, k, v, ints(table), ints(lens), ints([0, 300, 800]))
        out.append(ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts)))
    assert torch.equal(out[0], out[1]) and ep.last_device_status() == 0
    for a, b in zip(small, big):
        assert torch.equal(a.view(torch.uint8)[[0, 1, 2, 3, 4, 5, 6]], b.view(torch.uint8)[[pages - 1 - i for i in range(7)]])


@gpu
def test_requests_that_share_full_pages():
    # a common prefix of two pages, each request's own tokens behind it
    H, D, page = 2, 64, 32
    cache, table = filled([64, 90, 70], H, D, page, seed=77)
    shared = [table[0][:2] + table[1][2:3], table[0][:2] + table[2][2:3]]
    k = torch.randn(2, H, D, generator=cuda(4), device="cuda").to(torch.bfloat16)
    plain = Plain(cache)
    lens = [91, 71]
    ep.cache_append(cache, k, k, ints(shared), ints(lens), ints([0, 1, 2]))
    plain.append(k, k, shared, lens, [0, 1, 2])
    assert same(cache.k, plain.k) and same(cache.v_scales, plain.vs)
    q = torch.randn(2, 4 * H, D, generator=cuda(6), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(shared), ints(lens), ints([0, 1, 2]))
    want, bound, _ = attended(q, cache, shared, lens, [0, 1, 2], 0.125, True)
    check_attention(out, want, bound)


@gpu
@pytest.mark.parametrize("news", [[1, 1], [70, 90]])
def test_attention_scales_at_their_limits(news):
    # value scales far apart, a page of zeros as append leaves it, keys of scale 0, a scale of 0 or below
    G, H, lens, starts = 4, 1, [300, 130], offsets(news)
    cache, table = filled(lens, H, 128, 32, seed=19)
    cache.v_scales[table[0][1]], cache.v_scales[table[0][3]], cache.v_scales[table[1][0]] = 2.0 ** 40, 2.0 ** -60, 2.0 ** -30
    cache.v_scales[table[0][4]] = 2.0 ** -100
    cache.v.view(torch.uint8)[table[0][4]] = 0
    cache.k_scales[table[0][2]] = 0.0
    q = torch.randn(starts[-1], G, 128, generator=cuda(3), device="cuda").to(torch.bfloat16)
    for scale in (0.1, 0.0, -0.3):
        out = ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts), scale=scale)
        want, bound, _ = attended(q, cache, table, lens, starts, scale, True)
        check_attention(out, want, bound + 1e-7 * bound.amax(2, keepdim=True))
    tiny = ep.KVCache(cache.k, cache.v, cache.k_scales, torch.full_like(cache.v_scales, 2.0 ** -100))
    out = ep.cache_attention(q.half(), tiny, ints(table), ints(lens), ints(starts))
    assert bool((out == 0).all())                         # (below binary16's range)


@gpu
@pytest.mark.parametrize("news", [[1, 1, 1], [70, 90, 3]])
@pytest.mark.parametrize("zeros,large", [(1, 2.0 ** 20), (1, 2.0 ** 60), (3, 2.0 ** 100), (35, 2.0 ** 60), (1, 2.0 ** -70)])
def test_attention_first_pages_of_zeros(news, zeros, large):
    # pages of zeros as append leaves them, then values that their scale of 2^-100 is no measure for; a long request whose work CTAs share; one of zeros alone
    G, H, page, lens, starts = 4, 2, 16, [16 * zeros + 150, 9000, 130], offsets(news)
    cache, table = filled(lens, H, 128, page, seed=29)
    for b, n in enumerate((zeros, zeros, len(table[2]))):
        for i in table[b][:n]:
            cache.v_scales[i] = 2.0 ** -100
            cache.v.view(torch.uint8)[i] = 0
        for j, i in enumerate(table[b][n:-(-lens[b] // page)]):
            cache.v_scales[i] = min(large * 2.0 ** ((0, 7, -30, 40)[j % 4]), 2.0 ** 110)
    q = torch.randn(starts[-1], G * H, 128, generator=cuda(3), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts))
    want, bound, _ = attended(q, cache, table, lens, starts, 128 ** -0.5, True)
    up = max(1.0, 1 / large)                              # (the bound's last term is an absolute one)
    check_attention(out * up, want * up, (bound + 1e-7 * bound.amax(2, keepdim=True)) * up)
    assert bool((out[starts[2]:] == 0).all()) and ep.last_device_status() == 0


@gpu
def test_one_token_with_strides_that_mean_nothing():
    # a row of something turned round, and of buffers with odd rows
    H, G, D, C = 2, 4, 64, 256
    turned = lambda n, seed: torch.randn(n * D, generator=cuda(seed), device="cuda").to(torch.bfloat16).as_strided((1, n, D), (1, D, 1))  # noqa: E731
    k, v, q = turned(H, 1), turned(H, 2), turned(H * G, 3)
    assert k.stride(0) == 1
    caches = [filled([70], H, D, 32, seed=6) for _ in range(2)]
    got = []
    for (cache, table), copy in zip(caches, (lambda t: t, lambda t: t.flatten().clone().view(t.shape))):
        t, sl, st = ints(table), ints([70]), ints([0, 1])
        ep.cache_append(cache, copy(k), copy(v), t, sl, st)
        out = torch.empty(H * G * D, dtype=torch.bfloat16, device="cuda").as_strided((1, H * G, D), (1, D, 1))
        got.append((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scales, ep.cache_attention(copy(q), cache, t, sl, st, out=out)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    one = torch.randn(3, D, generator=cuda(4), device="cuda").to(torch.bfloat16)                      # one head: its stride means nothing either
    cache, table = filled([70], 1, D, 32, seed=7)
    odd = torch.zeros(3, 1, D + 8, dtype=torch.bfloat16, device="cuda").as_strided((3, 1, D), (D + 8, 3, 1))
    odd.copy_(one[:, None])
    a = ep.cache_attention(odd, cache, ints(table), ints([70]), ints([0, 3]))
    assert torch.equal(a, ep.cache_attention(one[:, None], cache, ints(table), ints([70]), ints([0, 3])))
    xb, wq = torch.randn(4, C + 24, generator=cuda(5), device="cuda"), ep.quantize_blocks(torch.randn(50, C, generator=cuda(6), device="cuda"), 128)
    xq = torch.zeros(4, C + 24, dtype=torch.uint8, device="cuda").view(E4M3)[:1, :C]
    xs = torch.zeros(2, 1, dtype=torch.uint8, device="cuda").view(E8M0).t()
    ep.quantize_blocks(xb[:1, :C], out=(xq, xs))
    y = torch.zeros(50, 1, device="cuda").t()
    ep.fp8_matmul(xq, xs, *wq, out=y)
    check_product(y, *product(xq, xs, *wq), C)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("B,H,G,D,page,steps,new", [(150, 8, 1, 64, 16, 40, 1), (16, 8, 4, 128, 32, 30, 7)])
def test_steps_one_behind_another_need_no_wait(B, H, G, D, page, steps, new):
    # each call may come up while the one before still runs: pages and scales that one step writes are read by the next on other SMs
    table, pages = paged([steps * new] * B, page, seed=B)
    t, st, g = ints(table), ints([i * new for i in range(B + 1)]), cuda(B)
    lens = [ints([(i + 1) * new] * B) for i in range(steps)]
    x = [(torch.randn(B * new, H, D, generator=g, device="cuda") * 2.0 ** (i / 6)).to(torch.bfloat16) for i in range(steps)]       # (so that scales grow)
    q = torch.randn(B * new, G * H, D, generator=g, device="cuda").to(torch.bfloat16)
    got = []
    for wait in (True, False):
        cache, outs = ep.kv_cache(pages, H, D, page), []
        for i in range(steps):
            ep.cache_append(cache, x[i], x[i], t, lens[i], st)
            if wait:
                torch.cuda.synchronize()
            outs.append(ep.cache_attention(q, cache, t, lens[i], st))
            if wait:
                torch.cuda.synchronize()
        got.append(outs + [cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scales, cache.v_scales])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got)) and ep.last_device_status() == 0


@gpu
def test_two_graphs_at_once_with_their_own_workspaces():
    lens = [2000, 700]
    cache, table = filled(lens, 4, 128, 64, seed=5)
    t, sl = ints(table), ints(lens)
    graphs, outs, want, keep = [], [], [], []
    for n in (1, 60):
        st = ints([0, n, 2 * n])
        q = torch.randn(2 * n, 16, 128, generator=cuda(n), device="cuda").to(torch.bfloat16)
        ws = torch.empty(ep.cache_attention_workspace_bytes(2 * n, 2, 16, 4, 128), dtype=torch.uint8, device="cuda")
        want.append(ep.cache_attention(q, cache, t, sl, st))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(ep.cache_attention(q, cache, t, sl, st, workspace=ws))
        graphs.append(graph)
        keep.append((q, st, ws))
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@gpu
def test_nothing_to_do():
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    q, s = ep.quantize_blocks(x)
    assert q.shape == (0, 256) and s.shape == (0, 2)
    w, ws = ep.quantize_blocks(torch.ones(40, 256, device="cuda"), 128)
    assert ep.fp8_matmul(q, s, w, ws).shape == (0, 40)
    cache = ep.kv_cache(2, 1, 64, 16)
    e = torch.empty(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    ep.cache_append(cache, e, e, ints([[0]]), ints([5]), ints([0, 0]))
    assert ep.cache_attention(e, cache, ints([[0]]), ints([5]), ints([0, 0])).shape == (0, 1, 64)
    torch.cuda.synchronize()


@gpu
def test_refusals():
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=torch.float32, device="cuda").to(dtype)  # noqa: E731
    x = z(4, 256)
    for call in (lambda: ep.quantize_blocks(x.double()), lambda: ep.quantize_blocks(x[0]), lambda: ep.quantize_blocks(x.t()), lambda: ep.quantize_blocks(x, 64),
                 lambda: ep.quantize_blocks(x, out=(z(4, 255, dtype=E4M3), z(4, 2, dtype=E8M0))), lambda: ep.quantize_blocks(x.cpu())):
        with pytest.raises(ValueError):
            call()
    q, s = ep.quantize_blocks(x)
    w = z(30, 256, dtype=E4M3)
    for call in (lambda: ep.fp8_matmul(x, s, w), lambda: ep.fp8_matmul(q, s, w[:, :128]), lambda: ep.fp8_matmul(q, s[:3], w), lambda: ep.fp8_matmul(q, s, w, s),
                 lambda: ep.fp8_matmul(q, s, w, row_scale=z(30)), lambda: ep.fp8_matmul(q, s, w, out=z(4, 31)), lambda: ep.fp8_matmul(q, s, w, out_dtype=ep.INT8),
                 lambda: ep.fp8_matmul(q, s.cpu(), w)):
        with pytest.raises(ValueError):
            call()
    for a, sc, b in ((z(4, 40, dtype=E4M3), z(4, 1, dtype=E8M0), z(30, 40, dtype=E4M3)), (z(4, 257, dtype=E4M3)[:, 1:], s, w), (q, s, z(30, 264, dtype=E4M3)[:, :256])):
        with pytest.raises(ep.EntroPackError) as e:      # what the copy engine cannot read
            ep.fp8_matmul(a, sc, b)
        assert e.value.status == -3
    cache = ep.kv_cache(4, 2, 64, 16)
    k, t, n, st = z(3, 2, 64), ints([[0, 1], [2, 3]]), ints([5, 6]), ints([0, 1, 3])
    for call in (lambda: ep.cache_append(cache, k.float(), k.float(), t, n, st), lambda: ep.cache_append(cache, k, k[:2], t, n, st), lambda: ep.cache_append(cache, k, k, t.long(), n, st),
                 lambda: ep.cache_append(cache, k, k, t, n[:1], st), lambda: ep.cache_append(cache, k, k, t, n, st[:2]), lambda: ep.cache_attention(z(3, 3, 64), cache, t, n, st),
                 lambda: ep.cache_attention(z(3, 4, 32), cache, t, n, st), lambda: ep.cache_attention(z(3, 4, 64), cache, t.cpu(), n, st),
                 lambda: ep.cache_attention(z(3, 4, 64), cache, t, n, st, lse=z(3, 4)), lambda: ep.cache_attention(z(3, 4, 64), cache[:2] + (cache[2][:3],) + cache[3:], t, n, st)):
        with pytest.raises(ValueError):
            call()
    big = ints([list(range(4)) * 10])
    with pytest.raises(ep.EntroPackError) as e:
        ep.cache_attention(z(1, 2, 64), cache, big, n[:1], st[:2], workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -7
    for odd in (ep.kv_cache(2, 1, 32, 16), ep.kv_cache(2, 1, 64, 24), ep.kv_cache(2, 1, 64, 8)):
        with pytest.raises(ep.EntroPackError) as e:
            ep.cache_append(odd, *(z(1, 1, odd.k.shape[3]),) * 2, t[:1], n[:1], st[:2])
        assert e.value.status == -3
    with pytest.raises(ep.EntroPackError) as e:
        ep.cache_append(cache, *(z(3, 2, 66)[:, :, 1:65],) * 2, t, n, st)
    assert e.value.status == -3


def test_entry_points_refuse_without_a_gpu():
    """The C entry points check their arguments before they touch a device: statuses, not crashes."""
    L, B = ep.load(), ep.binding
    p = 1 << 20                                           # an address that is never read

    def checked(layout, call, names, **fine):
        def f(**other):
            values = {**fine, **other}
            return call(layout.pack(*(values[n] for n in names.split())), None)
        return f

    quantize = checked(B.QUANTIZE_JOB, L.ep_quantize_blocks, "x q s ldx ldq lds T C rows dtype", x=p, q=p, s=p, ldx=4, ldq=4, lds=1, T=4, C=4, rows=1, dtype=ep.BF16)
    for other in ({"x": 0}, {"q": 0}, {"s": 0}, {"dtype": ep.INT8}, {"ldx": 3}, {"ldq": 3}, {"lds": 0}, {"rows": 2}, {"x": p + 1}, {"C": 0}):
        assert quantize(**other) == -1, other
    assert quantize(T=0, x=0) == 0 and L.ep_quantize_blocks(None, None) == -1
    matmul = checked(B.MATMUL_JOB, L.ep_fp8_matmul, "x xs w ws a y ldx ldxs ldw ldws ldy T R C dtype", x=p, xs=p, w=p, ws=0, a=0, y=p, ldx=256, ldxs=2, ldw=256, ldws=0, ldy=64,
                     T=4, R=64, C=256, dtype=ep.BF16)
    for other in ({"x": 0}, {"xs": 0}, {"w": 0}, {"y": 0}, {"ldx": 255}, {"dtype": ep.INT8}, {"ldy": 63}, {"ldxs": 1}, {"ws": p, "ldws": 1}, {"y": p + 1}, {"a": p + 2}):
        assert matmul(**other) == -1, other
    for other in ({"C": 248}, {"ldx": 264}, {"ldw": 264}, {"w": p + 8}, {"x": p + 8}):
        assert matmul(**other) == -3, other
    assert matmul(T=0) == 0 and L.ep_fp8_matmul(None, None) == -1
    shared = dict(k=p, v=p, ks=p, vs=p, pages=4, heads=2, page=16, dim=64, table=p, lens=p, starts=p, ldt=2, columns=2, B=1, N=1)
    head = "k v ks vs pages heads page dim table lens starts ldt columns B N "
    append = checked(B.APPEND_JOB, L.ep_cache_append, head + "xk xv ldk ldkh ldv ldvh dtype", xk=p, xv=p, ldk=128, ldkh=64, ldv=128, ldvh=64, dtype=ep.BF16, **shared)
    attend = checked(B.ATTENTION_JOB, L.ep_cache_attention, head + "q o lse ws bytes ldq ldqh ldo ldoh scale Hq dtype causal", q=p, o=p, lse=0, ws=0, bytes=0, ldq=256, ldqh=64,
                     ldo=256, ldoh=64, scale=1.0, Hq=4, dtype=ep.BF16, causal=1, **shared)
    for call in (append, attend):
        for other, status in (({"k": 0}, -1), ({"vs": 0}, -1), ({"table": 0}, -1), ({"columns": 3}, -1), ({"columns": 0}, -1), ({"dtype": ep.FP32}, -1), ({"pages": 0}, -1), ({"k": p + 8}, -1),
                              ({"lens": p + 2}, -1), ({"page": 24}, -3), ({"page": 512}, -3), ({"page": 8}, -3), ({"dim": 96}, -3), ({"pages": 1 << 28}, -3), ({"heads": 1 << 20}, -3)):
            assert call(**other) == status, other
        assert call(B=0) == 0 and call(N=0, k=0) == 0
    assert append(ldk=129) == -3 and append(ldvh=4) == -3 and append(xk=p + 8) == -3 and append(xv=0) == -1 and L.ep_cache_append(None, None) == -1
    assert attend(Hq=3) == -1 and attend(Hq=0) == -1 and attend(ldq=255) == -3 and attend(o=p + 8) == -3 and attend(B=5000, ldt=2) == -3 and L.ep_cache_attention(None, None) == -1
    assert "page" in ep.strerror(-9)


PROMPTS = [  # heads per group, heads, dim, page, tokens, rows: enough rows for the kernel of prompts
    (8, 4, 128, 64, [300], [300]), (5, 8, 128, 64, [1000], [260]), (4, 8, 64, 16, [129, 700, 300], [129, 200, 1]), (1, 16, 128, 16, [700, 0, 640], [650, 3, 0]),
    (8, 8, 128, 256, [140, 128], [140, 128]), (16, 16, 64, 32, [257], [70]), (3, 16, 128, 128, [90, 555], [200, 300]), (2, 32, 64, 64, [385], [384]),
]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("G,H,D,page,lens,news", PROMPTS)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_prompts(G, H, D, page, lens, news, causal, dtype):
    # (a few heads are looked at: the oracle is slow)
    cache, table = filled(lens, H, D, page, seed=G + D + page + len(lens))
    starts = offsets(news)
    q = torch.randn(starts[-1], G * H, D, generator=cuda(D), device="cuda").mul_(1.5).to(dtype)
    lse = torch.full((starts[-1], G * H), 7.0, device="cuda")
    out = torch.full_like(q, 9.0)
    ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts), scale=-0.2 if H == 4 else 0.2, causal=causal, out=out, lse=lse)
    for h in {0, H // 2, H - 1}:
        part = [t[:, h:h + 1].contiguous() for t in cache]
        at = slice(h * G, (h + 1) * G)
        want, bound, want_lse = attended(q[:, at], part, table, lens, starts, -0.2 if H == 4 else 0.2, causal)
        check_attention(out[:, at], want, bound)
        seen = want_lse > -math.inf
        assert torch.equal(lse[:, at].cpu() > -math.inf, seen)
        assert bool(((lse[:, at].double().cpu() - want_lse)[seen].abs() <= 1e-3).all())
    assert ep.last_device_status() == 0


@gpu
def test_attention_of_prompts_with_nan_and_pages_outside():
    G, H, lens, news = 8, 8, [300, 200, 420], [160, 140, 130]
    starts = offsets(news)
    cache, table = filled(lens, H, 128, 32, seed=31)
    for t in (cache.k, cache.v):
        t.view(torch.uint8)[table[0][8], :, 5, 9] = 0x7F       # token 261 of the first request: seen by its last 39 rows
    cache.v.view(torch.uint8)[table[0][9], :, 3, 100] = 0xFF   # token 291, another column
    cache.v.view(torch.uint8)[table[2][1], :, 0, 77] = 0x7F    # token 32 of the third: every row sees it
    bad = [row[:] for row in table]
    bad[1][2], bad[1][6] = 10 ** 8, -1
    q = torch.randn(starts[-1], G * H, 128, generator=cuda(9), device="cuda").to(torch.bfloat16)
    out = ep.cache_attention(q, cache, ints(bad), ints(lens), ints(starts))
    assert ep.last_device_status() == -9
    for h in (0, 5):
        at = slice(h * G, (h + 1) * G)
        want, bound, _ = attended(q[:, at], [t[:, h:h + 1].contiguous() for t in cache], bad, lens, starts, 128 ** -0.5, True, dead=(10 ** 8, -1))
        assert want[121:160].isnan().all() and not want[:121].isnan().any() and want[-130:, :, 77].isnan().all() and want[-130:].isnan().sum() == 130 * G
        check_attention(out[:, at], want, bound)


@gpu
def test_attention_of_prompts_scores_far_apart():
    lens, news, G, H = [700], [260], 8, 8
    cache, table = filled(lens, H, 128, 64, seed=13)
    cache.k.view(torch.uint8)[table[0][5], :, 60] = 0x70       # 128 everywhere, in a late tile: the reference moves
    cache.k.view(torch.uint8)[table[0][0], :, 3] = 0xF0        # -128 everywhere
    size = torch.exp2(torch.linspace(-60, 6, 260, device="cuda"))[:, None, None]
    for dtype in (torch.bfloat16, torch.float16):
        q = (torch.randn(260, G * H, 128, generator=cuda(4), device="cuda").abs() * size).to(dtype)
        out = ep.cache_attention(q, cache, ints(table), ints(lens), ints([0, 260]))
        for h in (0, 7):
            at = slice(h * G, (h + 1) * G)
            want, bound, _ = attended(q[:, at], [t[:, h:h + 1].contiguous() for t in cache], table, lens, [0, 260], 128 ** -0.5, True)
            check_attention(out[:, at], want, bound)


@gpu
def test_attention_of_prompts_many_units_and_captured():
    # more units than SMs, several per CTA; the same bits again, from a graph and with other lengths
    lens, news, G, H = [900, 300, 450, 130], [400, 300, 350, 64], 4, 32
    cache, table = filled(lens, H, 64, 64, seed=17)
    starts = offsets(news)
    q = torch.randn(starts[-1], G * H, 64, generator=cuda(2), device="cuda").to(torch.bfloat16)
    t, sl, st = ints(table), ints(lens), ints(starts)
    first = ep.cache_attention(q, cache, t, sl, st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ep.cache_attention(q, cache, t, sl, st)
    for now, rows in ((lens, starts), ([500, 300, 0, 64], starts), ([900, 20, 450, 130], [0, 1, 21, 400, 401])):
        sl.copy_(ints(now)), st.copy_(ints(rows))
        for _ in range(3):
            graph.replay()
        for h in (0, 31):
            at = slice(h * G, (h + 1) * G)
            want, bound, _ = attended(q[:, at], [c[:, h:h + 1].contiguous() for c in cache], table, now, rows, 0.125, True)
            check_attention(out[:rows[-1], at], want[:rows[-1]], bound[:rows[-1]])
        if now is lens:
            assert torch.equal(out, first)


@gpu
@pytest.mark.parametrize("N,G", [(4096, 8), (4096, 32)])
def test_rows_that_several_requests_claim_are_refused(N, G):
    # starts that go up and down between 0 and N: 2048 requests each claim all rows, more than 2^32 pieces of work
    B, H, page, columns = 4096, 8, 256, 64
    cache = ep.kv_cache(1, H, 64, page)
    table, lens = torch.zeros(B, columns, dtype=torch.int32, device="cuda"), torch.full((B,), columns * page, dtype=torch.int32, device="cuda")
    starts = ints([0, N] * (B // 2) + [0])
    q = torch.zeros(N, H * G, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 4.0)
    ep.cache_attention(q, cache, table, lens, starts, out=out)
    assert ep.last_device_status() == -9 and ep.last_device_status() == 0
    assert bool((out == 4.0).all())


def many_requests(B, kind):
    """Rows and tokens of B requests, some without rows or tokens."""
    r = np.random.default_rng(B)
    lens = r.integers(0, 200, B)
    lens[r.random(B) < 0.1] = 0
    if kind == "few":                                     # three rows each, or none
        news = np.where(r.random(B) < 0.05, 0, 3)
    elif kind in ("first", "middle", "last"):             # a prompt among single tokens
        news, at = np.ones(B, int), {"first": 0, "middle": B // 2, "last": B - 1}[kind]
        news[at], lens[at] = B + 100, B + 150
    elif kind == "alone":                                 # most requests have no rows
        news = np.zeros(B, int)
        news[0], lens[0], news[1], lens[1], news[B - 1], lens[B - 1] = 3 * B + 200, 3 * B + 210, 1, 1, 2, 90
    else:
        news = np.full(B, int(kind))
        lens[B // 3::97] = 700                            # (of two to four units: cut between CTAs now and then)
    return news.tolist(), lens.tolist()


@gpu
@pytest.mark.parametrize("B,kind,G,D,page", [
    # prompts' kernel: 512 requests are one to a thread, more are several
    (512, "few", 8, 64, 64), (513, "few", 8, 64, 64), (513, "few", 8, 128, 256), (600, "few", 8, 128, 16), (1025, "few", 8, 64, 32), (4096, "few", 8, 64, 64), (600, "alone", 5, 64, 64),
    (600, "first", 8, 64, 32), (600, "middle", 8, 128, 64), (600, "last", 8, 64, 64), (1025, "middle", 8, 64, 64), (700, "1", 20, 64, 64), (600, "4", 5, 128, 64),
    # single tokens: twelve warps with up to eight rows a request, eight with up to sixteen
    (385, "1", 5, 64, 64), (1000, "1", 8, 128, 256), (4096, "1", 5, 64, 32), (257, "2", 7, 64, 64), (1025, "2", 7, 128, 16), (4096, "2", 7, 64, 64)])
def test_attention_of_many_requests(B, kind, G, D, page):
    news, lens = many_requests(B, kind)
    starts = [2 + s for s in offsets(news)]
    N = starts[-1] + 3                                    # rows of nobody before and after
    cache, table = filled(lens, 1, D, page, seed=B + D)
    q = torch.randn(N, G, D, generator=cuda(B), device="cuda").mul_(1.5).to(torch.bfloat16)
    out, lse = torch.full_like(q, 9.0), torch.full((N, G), 7.0, device="cuda")
    ep.cache_attention(q, cache, ints(table), ints(lens), ints(starts), scale=0.2, out=out, lse=lse)
    want, bound, want_lse = attended(q, cache, table, lens, starts, 0.2, True)
    mine = slice(starts[0], starts[-1])
    check_attention(out[mine], want[mine], bound[mine])
    seen = want_lse[mine] > -math.inf
    assert torch.equal(lse[mine].cpu() > -math.inf, seen)
    assert bool(((lse[mine].double().cpu() - want_lse[mine])[seen].abs() <= 1e-3).all())
    for t, value in ((out, 9.0), (lse, 7.0)):
        assert bool((t[:2] == value).all()) and bool((t[-3:] == value).all())
    assert ep.last_device_status() == 0


FIRST_CALLS = """
import torch, {name} as ep
x = torch.randn(3, 256, device="cuda").to(torch.bfloat16)
w = torch.randn(384, 256, device="cuda")
cache = ep.kv_cache(8, 1, 64, 64)
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
table, lens, starts = ints([[0, 1, 2, 3, 4, 5]]), ints([3]), ints([0, 3])

def layer(rows):
    xq, xs = ep.quantize_blocks(x)
    wq, ws = ep.quantize_blocks(w, 128)
    y = ep.fp8_matmul(xq, xs, wq, ws).unflatten(1, (6, 64))
    ep.cache_append(cache, y[:, :1], y[:, 1:2], table, lens, starts)
    return ep.cache_attention(y[:rows, 2:], cache, table, lens, ints_of[rows])

ints_of = {{1: ints([0, 1]), 3: starts}}
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a, b = layer(1), layer(3)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(a, layer(1)) and torch.equal(b, layer(3)) and bool(a.isfinite().all()) and float(b.float().abs().sum()) > 0
assert ep.last_device_status() == 0
print("captured")
"""


@gpu
def test_first_calls_of_a_process_can_be_captured():
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(name=ep.__name__)], capture_output=True, text=True, timeout=300,
                          cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0 and done.stdout.split() == ["captured"], done.stderr[-2000:]
