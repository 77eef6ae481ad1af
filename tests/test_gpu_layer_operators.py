"""The INT8 product with its rounding, the norms around a block and rotary positions against plain implementations in 64 bits.

Rounding to INT8 is defined operation by operation in 32 bits, so it is compared exactly with the same operations of numpy; a norm that
rounds to a container gives exactly what the rounding operator gives for its 32-bit result.

The product: the sum is exact (integers below 2^31); it is rounded to 32 bits, multiplied by two scales and the bias is added, four roundings of
2^-24 each of |v| + |bias| for v = a s sum, and half a step of the result's type (of fp16 at least half of its smallest step, 2^-25).

The norms: a row's sum passes through at most 64 additions in a thread, two times five between lanes and a few roundings around it, so a sum of squares is off by less
than 80 2^-24 of itself and the factor 1 / sqrt by half of that and 4 more; a mean by 80 2^-24 of the mean magnitude.  Two norms after one another, with
gate, residual, weight and bias, stay below K = 256 units of 2^-24 of the magnitudes that went into a value: those of its own terms, and (through
mean and factor) the row's mean and largest ratio of the terms' magnitude to the result's, which the oracle carries along.  Half a step of the type besides.

Rotary: the angle's fraction of a turn is rounded to 24 bits of half a turn, pi 2^-25 radians, after 32 of 64 bits were cut off (2 pi 2^-32); its
frequency to 2^-52 of itself twice over.  Cosine and sine are good to 2 units of 2^-24 (CUDA's bound for sincospi is 2), the factor and the two products and
their sum add 4 of |u| + |v|.  The oracle's angles are in 80 bits."""
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
SMALLEST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
CODE = {torch.bfloat16: ep.BF16, torch.float16: ep.FP16, torch.float32: ep.FP32}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
U = 2.0 ** -24
gpu = pytest.mark.gpu


def cuda(seed):
    return torch.Generator("cuda").manual_seed(seed)


# ---- rounding to INT8 --------------------------------------------------------------------------------------------------

def rounded_rows(x):
    """q and s by numpy's operations in 32 bits."""
    x = x.float().cpu().numpy()
    q, s = np.zeros(x.shape, np.int8), np.ones(x.shape[0], np.float32)
    for t, row in enumerate(x):
        if not np.isfinite(row).all():
            s[t] = np.nan
        elif (row != 0).any():
            m = max(np.abs(row).max(), np.float32(2.0 ** -119))
            s[t] = m / np.float32(127)
            q[t] = np.rint(row * (np.float32(127) / m)).astype(np.int8)
    return q, s


def assert_rows(got, want):
    assert np.array_equal(got[1].cpu().numpy(), want[1], equal_nan=True)
    assert np.array_equal(got[0].cpu().numpy(), want[0])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C", [(1, 1), (1, 5120), (3, 127), (7, 256), (9, 264), (130, 1000), (2, 4097), (3, 8200), (2, 16400), (5, 17408), (2, 32768), (2, 32769), (3, 70001),
                                 (1, 200000)])
def test_quantize_rows(T, C, dtype):
    g = cuda(T * 7919 + C)
    x = (torch.randn(T, C, generator=g, device="cuda") * torch.exp(6 * torch.randn(T, 1, generator=g, device="cuda"))).clamp(-60000, 60000).to(dtype)
    q, s = ep.quantize_rows(x)
    assert q.dtype == torch.int8 and s.dtype == torch.float32
    assert_rows((q, s), rounded_rows(x))


@gpu
@pytest.mark.parametrize("C", [9, 64, 40000])
def test_quantize_rows_edges(C):
    inf, nan = math.inf, math.nan
    cases = [[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5], [0.0], [-0.0], [inf, 1.0], [1.0, -inf], [nan, 5.0], [1e-40, -3e-41], [1.4e-45], [2.0 ** -119, 2.0 ** -120],
             [3.4028234e38, -1e38], [1.0, -1.0], [1e-3, 0.9999999]]
    x = torch.zeros(len(cases), C)
    for i, c in enumerate(cases):
        x[i, C - len(c):] = torch.tensor(c)
    got = ep.quantize_rows(x.cuda())
    assert_rows(got, rounded_rows(x))
    assert got[0].min() >= -127


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C", [(1201, 5), (1300, 9), (1184, 60), (1211, 128), (1250, 250), (1201, 264), (1190, 700), (1203, 1500), (1187, 2056), (1185, 4096), (1184, 4104)])
def test_quantize_rows_of_many_rows(T, C, dtype):
    x = (torch.randn(T, C, generator=cuda(T + C), device="cuda") * torch.exp(3 * torch.randn(T, 1, generator=cuda(C), device="cuda"))).clamp(-60000, 60000).to(dtype)
    x[7], x[T - 1, C - 1] = 0.0, math.inf
    assert_rows(ep.quantize_rows(x), rounded_rows(x))


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("C", [8, 300, 33000])
def test_quantize_rows_what_is_not_finite_in_16_bits(C, dtype):
    x = torch.randn(6, C, generator=cuda(8), device="cuda").to(dtype)
    x[1, C - 1], x[2, 0], x[3, C // 2], x[4] = math.inf, -math.inf, math.nan, 0.0
    assert_rows(ep.quantize_rows(x), rounded_rows(x))


@gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_quantize_rows_views_and_outputs(dtype):
    # rows of any distance and alignment, results into parts of larger buffers whose other bytes stay
    base = torch.randn(70, 700, generator=cuda(5), device="cuda").to(dtype)
    for c0, C in ((0, 700), (8, 512), (1, 333), (3, 690)):
        x = base[:, c0:c0 + C]
        qb, sb = torch.full((70, C + 9), 3, dtype=torch.int8, device="cuda"), torch.full((72,), 3.0, device="cuda")
        ep.quantize_rows(x, out=(qb[:, 5:5 + C], sb[1:71]))
        assert_rows((qb[:, 5:5 + C], sb[1:71]), rounded_rows(x))
        assert (qb[:, :5] == 3).all() and (qb[:, 5 + C:] == 3).all() and sb[0] == 3 and sb[71] == 3


# ---- product -------------------------------------------------------------------------------------------------------------

def check_product(y, x, s, w, a, bias):
    v = x.double() @ w.double().t() * s.double()[:, None]
    if a is not None:
        v *= a.double()
    want, size = v, v.abs()
    if bias is not None:
        want, size = v + bias.double(), size + bias.double().abs()
    bound = 4 * U * size + HALF_STEP[y.dtype] * want.abs() * (1 + 2 ** -10) + SMALLEST[y.dtype]
    top = 65504.0 if y.dtype == torch.float16 else math.inf
    over = want.abs() > top * (1 - 2.0 ** -11)
    assert ((y.double() - want).abs() <= bound)[~over].all()
    assert (y.double().abs() >= top * (1 - 2.0 ** -11))[over].all()


def operands(T, R, C, seed, full=False):
    g = cuda(seed)
    lo, hi = (-128, 128) if full else (-127, 128)
    x = torch.randint(lo, hi, (T, C), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(lo, hi, (R, C), generator=g, device="cuda", dtype=torch.int8)
    s = torch.rand(T, generator=g, device="cuda") * 0.01
    a = torch.rand(R, generator=g, device="cuda") * 0.01
    bias = torch.randn(R, generator=g, device="cuda") * 20
    return x, s, w, a, bias


@gpu
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("T,R,C", [(1, 1, 16), (1, 10240, 3840), (2, 7, 48), (5, 130, 128), (16, 1185, 1040), (17, 129, 256), (31, 20000, 144), (33, 3000, 1744), (48, 5120, 4352),
                                   (64, 64, 8192), (65, 1000, 272), (100, 2049, 528), (128, 128, 128), (129, 257, 400), (200, 4096, 96), (257, 255, 1024), (300, 1, 64), (777, 3000, 1744),
                                   (1025, 511, 16), (2000, 2000, 2000)])
def test_product(T, R, C, out):
    x, s, w, a, bias = operands(T, R, C, T * 31 + R + C)
    check_product(ep.int8_matmul(x, s, w, row_scale=a, bias=bias, out_dtype=CODE[out]), x, s, w, a, bias)
    check_product(ep.int8_matmul(x, s, w, out_dtype=CODE[out]), x, s, w, None, None)


@gpu
@pytest.mark.parametrize("T,R,C", [(1, 64, 8208), (7, 1000, 4112), (20, 1000, 8192), (33, 2049, 8208), (48, 300, 16400), (64, 1024, 8192), (64, 5120, 17424), (1, 17408, 5120), (3, 19001, 528),
                                   (64, 30000, 128), (150, 10240, 2000), (192, 8000, 2064), (400, 4096, 512), (513, 4100, 1040), (900, 2100, 3088)])
def test_product_shapes_of_the_ways_it_is_shared_out(T, R, C):
    # strips alone and in clusters of two and eight, one round and several; pairs of 128, 192 and 256 tokens; with columns left over from whole blocks and without
    x, s, w, a, bias = operands(T, R, C, T + R + C)
    check_product(ep.int8_matmul(x, s, w, a, bias, out_dtype=ep.FP32), x, s, w, a, bias)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("T", [1, 40, 130, 600])
def test_product_of_the_largest_sums(T):
    # -128 x -128 over the most columns there may be: 2^31 - 2^18, which 32 bits just hold
    C, R = 131056, 70
    x, s, w, a, _ = operands(T, R, C, 3, True)
    x[0], w[0], w[1] = -128, -128, 127
    s[0] = 1.0
    y = ep.int8_matmul(x, s, w, out_dtype=ep.FP32)
    assert y[0, 0] == 128 * 128 * C and y[0, 1].double() == -128 * 127 * C
    check_product(y, x, s, w, None, None)


@gpu
@pytest.mark.parametrize("T", [1, 20, 64, 127, 500])
def test_product_views_and_outputs(T):
    # rows of any distance (16 bytes), results into a part of a larger buffer whose other values stay; scales that are not finite
    x, s, w, a, bias = operands(T, 333, 640, 9)
    x, w = x[:, 16:16 + 528], w[:, 32:32 + 528]
    s[T // 2] = math.nan
    a[5], a[7] = math.inf, 0.0
    buffer = torch.full((T + 2, 400), 7.0, dtype=torch.bfloat16, device="cuda")
    y = ep.int8_matmul(x, s, w, row_scale=a, bias=bias, out=buffer[1:T + 1, 3:336])
    assert y[T // 2].isnan().all()
    fine = torch.arange(T, device="cuda") != T // 2
    assert y[fine][:, 5].isinf().all() and (y[fine][:, 7] == bias[7].to(torch.bfloat16)).all()
    keep = [i for i in range(333) if i not in (5, 7)]
    check_product(y[fine][:, keep], x[fine], s[fine], w[keep], a[keep], bias[keep])
    assert (buffer[0] == 7).all() and (buffer[T + 1] == 7).all() and (buffer[:, :3] == 7).all() and (buffer[:, 336:] == 7).all()


@gpu
def test_product_of_a_decoded_weight():
    # a stream decoded to INT8, its rows' scales kept apart, by rounded activations
    rng = np.random.default_rng(4)
    W = (rng.standard_normal((264, 512)) * 0.02).astype(np.float32)
    a = (np.abs(W).max(1) / 127).astype(np.float32)
    d = ep.upload(ep.encode(W / a[:, None], 6.0))
    w = ep.decode(d, ep.INT8)
    x = torch.randn(21, 512, generator=cuda(1), device="cuda", dtype=torch.bfloat16)
    q, s = ep.quantize_rows(x)
    y = ep.int8_matmul(q, s, w, row_scale=torch.from_numpy(a).cuda(), out_dtype=ep.FP32)
    check_product(y, q, s, w, torch.from_numpy(a).cuda(), None)
    want = x.double() @ torch.from_numpy(W).double().cuda().t()
    assert (y.double() - want).norm() < 0.05 * want.norm()


@gpu
def test_product_the_same_every_time():
    x, s, w, a, bias = operands(700, 1000, 1040, 12)
    first = ep.int8_matmul(x, s, w, a, bias, out_dtype=ep.FP32)
    for T in (1, 16, 40, 128, 200, 700):                  # a token's row does not depend on what is multiplied beside it
        assert torch.equal(ep.int8_matmul(x[:T], s[:T], w, a, bias, out_dtype=ep.FP32), first[:T])


# ---- norms -----------------------------------------------------------------------------------------------------------------

def rows_of(v, T):
    v = v.double()
    return v[None].expand(T, -1) if v.dim() == 1 else v.repeat_interleave(T // v.shape[0], 0)


def unit(v, size, center, eps):
    """The norm of v, and the magnitudes that went into it: `size` those of v's own terms."""
    if center:
        mean = v.mean(1, keepdim=True)
        v, size = v - mean, size + size.mean(1, keepdim=True)
    f = 1 / (v.square().mean(1, keepdim=True) + eps).sqrt()
    # errors of size d in v move the factor by up to mean(|v| d) / mean(v^2) of itself
    spread = (v.abs() * size).mean(1, keepdim=True) / (v.square().mean(1, keepdim=True) + eps)
    return v * f, (size + v.abs() * (1 + spread)) * f


def normed(x, weight=None, bias=None, residual=None, residual_scale=1.0, gate=None, post_weight=None, weight_offset=0.0, eps=1e-6, center=False):
    """z and r in 64 bits, each with the magnitudes of its errors."""
    T = x.shape[0]
    r = x.double()
    size = r.abs()
    if post_weight is not None:
        r, size = unit(r, size, center, eps)
        p = weight_offset + rows_of(post_weight, T)
        r, size = r * p, size * p.abs()
    if gate is not None:
        r, size = r * rows_of(gate, T), size * rows_of(gate, T).abs()
    if residual is not None:
        r, size = r + residual_scale * residual.double(), size + (residual_scale * residual.double()).abs()
    z, zsize = unit(r, size, center, eps)
    if weight is not None:
        w = weight_offset + rows_of(weight, T)
        z, zsize = z * w, zsize * w.abs()
    if bias is not None:
        z, zsize = z + rows_of(bias, T), zsize + rows_of(bias, T).abs()
    return (z, zsize), (r, size)


def near(got, want):
    value, size = want
    bound = 256 * U * size + HALF_STEP[got.dtype] * (value.abs() + 256 * U * size) + SMALLEST[got.dtype]
    return bool(((got.double() - value).abs() <= bound).all())


def norm_inputs(T, C, dtype, wide, groups, seed, vectors=None):
    g, vectors = cuda(seed), vectors or dtype
    x = (torch.randn(T, C, generator=g, device="cuda") * 2 + 0.3).to(dtype)
    h = (torch.randn(T, C, generator=g, device="cuda") * 4 - 0.5).to(wide)
    v = lambda n, at, spread: (at + spread * torch.randn((C,) if n == 1 else (n, C), generator=g, device="cuda")).to(vectors)  # noqa: E731
    return x, dict(residual=h, weight=v(groups, 1.0, 0.3), bias=v(groups, 0.0, 0.5), gate=v(groups, 0.2, 0.7), post_weight=v(1, 0.5, 0.2))


SIZES = [(1, 1), (1, 5120), (3, 7), (4, 64), (6, 255), (5, 256), (130, 260), (9, 1000), (2, 1024), (12, 2056), (3, 4100), (2, 8192), (2, 8200), (3, 16384), (2, 17408), (2, 32768), (1, 32767)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C", SIZES)
def test_norm_alone(T, C, dtype):
    x, v = norm_inputs(T, C, dtype, dtype, 1, T + C)
    assert near(ep.norm(x), normed(x)[0])
    assert near(ep.norm(x, v["weight"], eps=1e-5), normed(x, v["weight"], eps=1e-5)[0])
    if C > 1:
        assert near(ep.norm(x, v["weight"], v["bias"], center=True, eps=1e-5), normed(x, v["weight"], v["bias"], center=True, eps=1e-5)[0])


@gpu
@pytest.mark.parametrize("dtype,wide,vectors", [(torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32, torch.float32), (torch.float16, torch.float16, torch.float32),
                                                (torch.float32, torch.float32, torch.bfloat16), (torch.float32, torch.float16, torch.float16), (torch.float16, torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("T,C", SIZES[1:])
@pytest.mark.parametrize("center", [False, True])
def test_norm_of_a_block(T, C, dtype, wide, vectors, center):
    x, v = norm_inputs(T, C, dtype, wide, T, T * 3 + C, vectors)
    for left in ((), ("post_weight",), ("gate", "bias"), ("post_weight", "gate", "bias", "weight")):
        given = {k: t for k, t in v.items() if k not in left}
        z, r = ep.norm(x, residual_scale=0.7, weight_offset=1.0, center=center, **given)
        want, r_want = normed(x, residual_scale=0.7, weight_offset=1.0, center=center, **given)
        assert z.dtype == dtype and r.dtype == wide
        assert near(z, want) and near(r, r_want)


@gpu
@pytest.mark.parametrize("T,groups", [(12, 1), (12, 3), (12, 12), (1000, 2), (1000, 5)])
def test_norm_groups(T, groups):
    x, v = norm_inputs(T, 384, torch.bfloat16, torch.float32, groups, 8)
    z, r = ep.norm(x, weight_offset=1.0, center=True, **v)
    want, r_want = normed(x, weight_offset=1.0, center=True, **v)
    assert near(z, want) and near(r, r_want)


@gpu
@pytest.mark.parametrize("T,groups,more", [(6000, 2, 2), (6000, 3, 6), (6000, 12, 4), (6000, 4, 6), (5000, 50, 1), (4000, 1, 1000), (2000, 2000, 2), (1500, 1, 3), (296 * 5, 296, 148)])
@pytest.mark.parametrize("C", [72, 1000, 3848])
def test_norm_groups_of_many_rows(T, C, groups, more):
    x, v = norm_inputs(T, C, torch.float16, torch.float32, groups, T + C)
    v["gate"] = norm_inputs(T, C, torch.float16, torch.float32, more, C)[1]["gate"]
    for left in ((), ("weight",), ("gate", "bias")):
        given = {k: t for k, t in v.items() if k not in left}
        z, r = ep.norm(x, weight_offset=1.0, center=True, **given)
        want, r_want = normed(x, weight_offset=1.0, center=True, **given)
        assert near(z, want) and near(r, r_want)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T,C", [(1201, 8), (1203, 64), (5000, 256), (3001, 264), (1205, 520), (1500, 1000), (2501, 2048), (1301, 5120), (1200, 8200), (1190, 17408), (1184, 32768), (1900, 136), (2000, 12000), (1200, 1028), (1300, 16384), (1190, 12808), (1500, 14336)])
@pytest.mark.parametrize("center", [False, True])
def test_norm_of_many_rows(T, C, dtype, wide, center):
    x, v = norm_inputs(T, C, dtype, wide, 1, T * 3 + C)
    for left in ((), ("post_weight", "gate"), ("residual", "bias")):
        given = {k: t for k, t in v.items() if k not in left}
        z, r = ep.norm(x, residual_scale=0.7, center=center, residual_out=None if "residual" in given else torch.empty_like(x), **given)
        want, r_want = normed(x, residual_scale=0.7, center=center, **given)
        assert near(z, want) and near(r, r_want)
        if C < 10000:
            z, _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.FP32, **given)
            (q, s), _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.FP8_E4M3, **given)
            (q8, s8), _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.INT8, **given)
            same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731
            assert all(map(same, (q, s, q8, s8), ep.quantize_blocks(z) + ep.quantize_rows(z)))
    if "residual" in v:                                    # in place: the residual, and z over x
        h, x2 = v["residual"].clone(), x.clone()
        z, r = ep.norm(x, **v)
        z2, r2 = ep.norm(x2, **{**v, "residual": h}, out=x2, residual_out=h)
        assert z2 is x2 and r2 is h and torch.equal(z, z2) and torch.equal(r, r2)
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T,C", [(120001, 8), (70000, 24), (30011, 64), (30000, 72), (20001, 128), (9000, 136), (10007, 256)])
def test_norm_of_many_short_rows(T, C, dtype, wide):
    x, v = norm_inputs(T, C, dtype, wide, 1, T + C)
    x[5], x[T - 3, 3] = 0.0, math.inf
    for center in (False, True):
        for left in ((), ("post_weight", "gate", "bias")):
            given = {k: t for k, t in v.items() if k not in left}
            z, r = ep.norm(x, residual_scale=0.7, center=center, **given)
            want, r_want = normed(x, residual_scale=0.7, center=center, **given)
            fine = torch.arange(T, device="cuda") != T - 3
            assert near(z[fine], tuple(t[fine] for t in want)) and near(r[fine], tuple(t[fine] for t in r_want))
            z, _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.FP32, **given)
            (q, s), _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.FP8_E4M3, **given)
            (q8, s8), _ = ep.norm(x, residual_scale=0.7, center=center, residual_out=r, out_dtype=ep.INT8, **given)
            same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731
            assert all(map(same, (q, s, q8, s8), ep.quantize_blocks(z) + ep.quantize_rows(z)))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C", SIZES + [(70, 640)])
def test_norm_into_the_containers(T, C, dtype):
    # what the rounding operators make of the 32-bit result
    x, v = norm_inputs(T, C, dtype, dtype, 1, T + 2 * C)
    z, r = ep.norm(x, out_dtype=ep.FP32, **v)
    for code, f in ((ep.FP8_E4M3, ep.quantize_blocks), (ep.INT8, ep.quantize_rows)):
        (q, s), again = ep.norm(x, out_dtype=code, **v)
        q2, s2 = f(z)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s.view(torch.uint8), s2.view(torch.uint8)) and torch.equal(r, again)


@gpu
def test_norm_edges():
    # rows of zeros, of what is not finite, huge and tiny ones, a row whose values are all the same
    inf, nan = math.inf, math.nan
    x = torch.randn(8, 300, generator=cuda(3), device="cuda")
    x[0] = 0.0
    x[1, 5], x[2, 299], x[3, 0] = inf, nan, -inf
    x[4] *= 1e15
    x[5] *= 1e-18
    x[6] = 3.0
    z = ep.norm(x)
    assert (z[0] == 0).all() and near(z[4:], normed(x[4:])[0])
    assert z[1][5].isnan() and (z[1].nan_to_num(0.0) == 0).all() and z[2].isnan().all() and z[3][0].isnan()
    centred = ep.norm(x, center=True)
    assert (centred[0] == 0).all() and centred[1:4].isnan().all() and near(centred[4:], normed(x[4:], center=True)[0])
    (q, s), (q8, s8) = ep.norm(x, out_dtype=ep.FP8_E4M3), ep.norm(x, out_dtype=ep.INT8)
    assert (s.float()[0] == 1).all() and (q.float()[0] == 0).all() and q.float()[2].isnan().all() and torch.equal(q.float()[1].isnan(), z[1].isnan())
    assert s8[0] == 1 and (q8[:4] == 0).all() and s8[1:4].isnan().all() and s8[4:].isfinite().all()


@gpu
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, torch.float32), (torch.float32, torch.float16)])
def test_norm_views_and_outputs(dtype, wide):
    # rows of any distance and alignment; the residual in place; results into parts of larger buffers whose other values stay
    T, C = 33, 200
    for c0 in (0, 8, 1, 3):
        x, v = norm_inputs(T, C + 20, dtype, wide, 3, 20 + c0)
        cut = lambda t: t[..., c0:c0 + C]  # noqa: E731
        x, v = cut(x), {k: cut(t) for k, t in v.items()}
        want, r_want = normed(x, **v)
        kept = v["residual"].clone()
        for code, extra in ((None, 9), (ep.FP8_E4M3, 9), (ep.INT8, 9)):
            h = torch.full((T + 2, C + 20), 5.0, dtype=wide, device="cuda")
            h[1:-1, c0:c0 + C] = kept
            here = h[1:-1, c0:c0 + C]
            if code is None:
                zb = torch.full((T, C + extra), 3.0, dtype=dtype, device="cuda")
                out = zb[:, c0:c0 + C]
            else:
                zb = torch.full((T, C + extra), 3, dtype=torch.uint8, device="cuda").view(E4M3 if code == ep.FP8_E4M3 else torch.int8)
                sb = torch.full((T, 4), 3, dtype=torch.uint8, device="cuda").view(E8M0) if code == ep.FP8_E4M3 else torch.full((T,), 3.0, device="cuda")
                out = (zb[:, c0:c0 + C], sb[:, 1:3] if code == ep.FP8_E4M3 else sb)
            got, r = ep.norm(x, **{**v, "residual": here}, out=out, residual_out=here)
            assert near(r, r_want) and r.data_ptr() == here.data_ptr()
            h[1:-1, c0:c0 + C] = 5.0
            assert (h == 5).all()
            left = zb.view(torch.uint8).view(T, -1).clone() if code is not None else zb.clone()
            three = 3 if code is not None else 3.0
            left[:, c0:c0 + C] = three
            assert (left == three).all()
            if code is None:
                assert near(got, want)
            elif code == ep.FP8_E4M3:
                z32 = ep.norm(x, **v, out_dtype=ep.FP32)[0]
                q, s = ep.quantize_blocks(z32)
                assert torch.equal(got[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got[1].view(torch.uint8), s.view(torch.uint8))
                assert (sb.view(torch.uint8)[:, 0] == 3).all() and (sb.view(torch.uint8)[:, 3] == 3).all()


@gpu
def test_norm_without_writing_the_residual():
    x, v = norm_inputs(10, 256, torch.bfloat16, torch.bfloat16, 1, 2)
    z, r = ep.norm(x, **v)
    assert torch.equal(ep.norm(x, residual_out=False, **v), z)
    v.pop("residual")                                      # no residual, but its place wanted: r = gate * b
    r = torch.empty(10, 256, device="cuda")
    z, again = ep.norm(x, residual_out=r, **v)
    want, r_want = normed(x, **v)
    assert again is r and near(z, want) and near(r, r_want)


# ---- rotary positions ------------------------------------------------------------------------------------------------------

def turned(x, at, f, next, factor):
    """The rotation in 64 bits with angles in 80, and the magnitudes of its pairs and the angles' error in radians."""
    pairs = len(f)
    two_pi = 8 * np.arctan(np.longdouble(1))
    turns = at.cpu().numpy().astype(np.longdouble)[:, None] * (f.cpu().numpy().astype(np.longdouble) / two_pi)
    a = ((turns - np.rint(turns)) * two_pi).astype(np.float64)
    cos, sin = (torch.from_numpy(t)[:, None].to(x.device) * factor for t in (np.cos(a), np.sin(a)))
    o, size, error = x.double(), x.double().abs() * 0, torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    u, v = (o[..., 0:2 * pairs:2], o[..., 1:2 * pairs:2]) if next else (o[..., :pairs], o[..., pairs:2 * pairs])
    first, second, both = u * cos - v * sin, v * cos + u * sin, (u.abs() + v.abs()) * abs(factor)
    off = math.pi * 2 ** -25 + 2 * math.pi * 2 ** -32 + torch.from_numpy(np.abs(turns).astype(np.float64)).to(x.device)[:, None] * two_pi.astype(np.float64) * 2.0 ** -51
    o = o.clone()
    for at_, value in ((slice(0, 2 * pairs, 2) if next else slice(0, pairs), first), (slice(1, 2 * pairs, 2) if next else slice(pairs, 2 * pairs), second)):
        o[..., at_], size[..., at_], error[..., at_] = value, both, off.expand(value.shape)
    return o, size, error


def check_turn(got, x, at, f, next, factor):
    want, size, off = turned(x, at, f, next, factor)
    bound = size * (off + 6 * U) + HALF_STEP[got.dtype] * want.abs() * (1 + 2 ** -10) + SMALLEST[got.dtype] * (size > 0)
    assert ((got.double() - want).abs() <= bound).all()
    assert torch.equal(got[..., 2 * len(f):], x[..., 2 * len(f):])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("next", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 2, 2), (1, 48, 128, 128), (3, 5, 64, 64), (17, 40, 128, 64), (200, 1, 128, 128), (333, 3, 80, 32), (5, 2, 96, 36), (7, 3, 37, 10), (2, 9, 256, 256),
                                       (1025, 8, 64, 16), (4, 300, 128, 128), (2, 2, 1024, 1024), (3, 1, 1023, 1022), (6, 4, 72, 72)])
def test_rotary(T, H, D, rot, next, dtype):
    g = cuda(T + H + D + rot)
    x = torch.randn(T, H, D, generator=g, device="cuda").to(dtype)
    f = ep.rotary_frequencies(rot)
    at = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)
    check_turn(ep.rotary(x, at, f, interleaved=next), x, at, f, next, 1.0)
    here = x.clone()
    assert ep.rotary(here, at.long(), f, interleaved=next, factor=1.25, out=here) is here
    check_turn(here, x, at, f, next, 1.25)


@gpu
@pytest.mark.parametrize("next", [False, True])
def test_rotary_far_and_negative_positions(next):
    at = torch.tensor([0, 1, -1, 200000, -200000, 1 << 24, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31), 1 << 40, -(1 << 33) - 7], device="cuda")
    x = torch.randn(len(at), 2, 64, generator=cuda(1), device="cuda")
    for f in (ep.rotary_frequencies(64, 1e6, 8.0, 8192.0), torch.tensor([0.0, math.pi, 2 * math.pi, -1.0, 100.0, 1e-12], dtype=torch.float64, device="cuda")):
        check_turn(ep.rotary(x, at, f, interleaved=next), x, at, f, next, 1.0)
    near = at.abs() < 2 ** 31
    f = ep.rotary_frequencies(64)
    assert torch.equal(ep.rotary(x[near], at[near].int(), f), ep.rotary(x[near], at[near], f))


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("next", [False, True])
def test_rotary_views_and_outputs(next, dtype):
    # heads inside the rows of a product, of any distance and alignment; everything beside them stays
    T, f = 19, ep.rotary_frequencies(64)
    at = torch.arange(100, 100 + T, device="cuda")
    for c0, stride in ((0, 96), (8, 96), (4, 100), (1, 97)):
        rows = torch.randn(T, 7 * stride, generator=cuda(c0), device="cuda").to(dtype)
        before = rows.clone()
        heads = lambda t: t.view(T, 7, stride)[:, 1:6, c0:c0 + 80]  # noqa: E731
        ep.rotary(heads(rows), at, f, interleaved=next, out=heads(rows))
        check_turn(heads(rows), heads(before), at, f, next, 1.0)
        heads(rows)[:] = heads(before)
        assert torch.equal(rows, before)
        other = torch.full((T, 5, 90), 2.0, dtype=dtype, device="cuda")
        ep.rotary(heads(rows), at, f, interleaved=next, out=other[..., 3:83])
        check_turn(other[..., 3:83], heads(before), at, f, next, 1.0)
        assert (other[..., :3] == 2).all() and (other[..., 83:] == 2).all()


@gpu
def test_scores_depend_on_distances_alone():
    f = ep.rotary_frequencies(128, 1e6)
    q, k = torch.randn(2, 1, 1, 128, generator=cuda(6), device="cuda").expand(2, 50, 1, 128).contiguous()
    at = torch.arange(50, device="cuda") * 9973
    scores = [(ep.rotary(q, at + d, f).double() * ep.rotary(k, at, f).double()).sum((1, 2)) for d in (0, 5, 1000)]
    bound = (q[0].abs().double().reshape(2, 64).sum(0) * k[0].abs().double().reshape(2, 64).sum(0)).sum() * 2 * 2 * 2 * (math.pi * 2 ** -25 + 7 * U + 1e-8)
    for s in scores:
        assert (s - s[0]).abs().max() <= bound


# ---- together, and as calls --------------------------------------------------------------------------------------------------

def layer(d, x, h, at, cache, table, lens, starts, a, w8, f, heads, kv, dim, stream=None):
    """From one block's output to the next one's, everything by the library."""
    (xq, xs), h = ep.norm(x, residual=h, out_dtype=ep.INT8, stream=stream)
    qkv = ep.int8_matmul(xq, xs, d["qkv"], row_scale=a["qkv"], bias=a["bias"], stream=stream).view(x.shape[0], heads + 2 * kv, dim)
    turning = qkv[:, :heads + kv]
    ep.rotary(turning, at, f, out=turning, stream=stream)
    ep.cache_append(cache, qkv[:, heads:heads + kv], qkv[:, heads + kv:], table, lens, starts, stream=stream)
    o = ep.cache_attention(qkv[:, :heads], cache, table, lens, starts, stream=stream)
    oq, os = ep.quantize_rows(o.view(x.shape[0], -1), stream=stream)
    y = ep.int8_matmul(oq, os, d["o"], row_scale=a["o"], stream=stream)
    (yq, ys), h = ep.norm(y, w8, residual=h, out_dtype=ep.FP8_E4M3, stream=stream)
    return ep.fp8_matmul(yq, ys, d["last"], stream=stream), h


def model(seed, heads=8, kv=2, dim=64, C=512):
    g = cuda(seed)
    w = lambda r, c: torch.randn(r, c, generator=g, device="cuda") * c ** -0.5  # noqa: E731
    plain = {"qkv": w((heads + 2 * kv) * dim, C), "o": w(C, heads * dim), "last": w(C, C)}
    q = {k: ep.quantize_rows(t) for k, t in plain.items() if k != "last"}
    d = {k: t[0] for k, t in q.items()}
    a = {k: t[1] for k, t in q.items()}
    d["last"] = plain["last"].clamp(-448, 448).to(E4M3)
    plain["last"] = d["last"].float()
    a["bias"] = torch.randn((heads + 2 * kv) * dim, generator=g, device="cuda") * 0.1
    return d, a, plain


def plain_layer(plain, a, x, h, f, heads, kv, dim, w8):
    """One request's tokens 0 .. T in 64 bits."""
    T = x.shape[0]
    r = x.double() + h.double()
    n = lambda t: t / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    qkv = (n(r) @ plain["qkv"].double().t() + a["bias"].double()).view(T, heads + 2 * kv, dim)
    at = torch.arange(T, device="cuda")
    qkv[:, :heads + kv] = turned(qkv[:, :heads + kv], at, f, False, 1.0)[0]
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    k, v = (t.repeat_interleave(heads // kv, 1) for t in (k, v))
    p = torch.einsum("ihd,jhd->hij", q, k) * dim ** -0.5
    p = torch.softmax(p.masked_fill(at[None] > at[:, None], -math.inf), -1)
    r = torch.einsum("hij,jhd->ihd", p, v).reshape(T, -1) @ plain["o"].double().t() + r
    return (n(r) * w8.double()) @ plain["last"].double().t(), r


@gpu
def test_a_layer_through_the_operators():
    # A prompt, then single tokens on top of it, against the whole in 64 bits.  What stands between is the containers' rounding, at random: E4M3
    # at most 2^-4, on average 2.6 % (keys, values, the last activations), INT8 a row's maximum / 127 / sqrt(12), 0.8 % (activations, weights).
    # y has the last activations' 2.6 % and, through r, a part of the others': below 8 %; r is x + h, exact, and an attention of a fraction of their size.
    heads, kv, dim, C, T = 8, 2, 64, 512, 40
    d, a, plain = model(11)
    f, w8 = ep.rotary_frequencies(dim), 1 + 0.1 * torch.randn(C, generator=cuda(1), device="cuda")
    x, h = (torch.randn(T, C, generator=cuda(s), device="cuda", dtype=torch.bfloat16) for s in (2, 3))
    want, r_want = plain_layer(plain, a, x, h, f, heads, kv, dim, w8)
    cache = ep.kv_cache(4, kv, dim, 16)
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = [layer(d, x[:35], h[:35], torch.arange(35, device="cuda"), cache, table, i32(35), i32(0, 35), a, w8, f, heads, kv, dim)]
    for t in range(35, T):
        got.append(layer(d, x[t:t + 1], h[t:t + 1], i32(t), cache, table, i32(t + 1), i32(0, 1), a, w8, f, heads, kv, dim))
    y, r = (torch.cat(t).double() for t in zip(*got))
    assert (y - want).norm() < 0.08 * want.norm() and (r - r_want).norm() < 0.03 * r_want.norm()
    assert ep.last_device_status() == 0


def each_operator(seed=1, T=40):
    """Calls of every operator, their inputs, and outputs to fill."""
    x, v = norm_inputs(T, 512, torch.bfloat16, torch.bfloat16, 1, seed)
    qx, s, w, a, bias = operands(T, 300, 512, seed)
    heads, f, at = torch.randn(T, 4, 64, generator=cuda(seed), device="cuda"), ep.rotary_frequencies(64), torch.arange(T, device="cuda")
    outs = [(torch.empty(T, 512, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")), torch.empty(T, 300, dtype=torch.float16, device="cuda"),
            torch.empty_like(x), torch.empty_like(x), torch.empty_like(heads)]
    calls = lambda stream=None: (ep.quantize_rows(x, out=outs[0], stream=stream), ep.int8_matmul(qx, s, w, a, bias, out=outs[1], stream=stream),  # noqa: E731
                                 ep.norm(x, out=outs[2], residual_out=outs[3], stream=stream, **v), ep.rotary(heads, at, f, out=outs[4], stream=stream))
    flat = lambda: [outs[0][0], outs[0][1]] + outs[1:]  # noqa: E731
    return calls, flat, (x, qx, heads)


@gpu
@pytest.mark.parametrize("T", [1, 40, 300])
def test_captured_and_replayed(T):
    calls, flat, inputs = each_operator(5, T)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        calls()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for t in inputs:                                       # new values in the same places
        t.copy_(t.flip(0))
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in flat()]
    for t in flat():
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(flat(), want))


@gpu
def test_on_a_given_stream():
    calls, flat, _ = each_operator(7)
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in flat()]
    for t in flat():
        t.zero_()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(1000000)
    calls(stream)
    stream.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(flat(), want))


@gpu
@pytest.mark.parametrize("T", [3, 40, 1500])
def test_two_graphs_at_once(T):
    # the same operators on other data, on two streams side by side, many times
    made = []
    for seed in (11, 12):
        calls, flat, _ = each_operator(seed, T)
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in flat()]
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(5):
                calls()
        for t in flat():
            t.zero_()
        made.append((graph, stream, flat, want, calls))    # (calls holds the inputs)
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream, *_ in made:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, flat, want, _ in made:
        assert all(torch.equal(g, w) for g, w in zip(flat(), want))
    assert ep.last_device_status() == 0


@gpu
def test_steps_one_behind_another_need_no_wait():
    # each operator reads what the one before it wrote, and each may come up while that one still runs: the same bits as with waits
    x0 = torch.randn(50, 1024, generator=cuda(2), device="cuda", dtype=torch.bfloat16)
    w, a = ep.quantize_rows(torch.randn(1024, 1024, generator=cuda(3), device="cuda") * 0.03)
    f, at = ep.rotary_frequencies(64), torch.arange(50, device="cuda")

    def steps(wait):
        x, h = x0, x0
        for _ in range(20):
            (q, s), h = ep.norm(x, residual=h, out_dtype=ep.INT8)
            wait()
            x = ep.int8_matmul(q, s, w, row_scale=a)
            wait()
            heads = x.view(50, 16, 64)
            ep.rotary(heads, at, f, out=heads)
            wait()
            q, s = ep.quantize_rows(x)
            wait()
            x = ep.int8_matmul(q, s, w, row_scale=a)
            wait()
        torch.cuda.synchronize()
        return x, h

    want = steps(torch.cuda.synchronize)
    for _ in range(3):
        assert all(torch.equal(g, w) for g, w in zip(steps(lambda: None), want))


FIRST_CALLS = """
import torch, {name} as ep
torch.zeros(1, device="cuda")
x = torch.randn(1300, 512, device="cuda", dtype=torch.bfloat16)
w = torch.randint(-127, 128, (300, 512), device="cuda", dtype=torch.int8)
at, f = torch.arange(1300, device="cuda"), ep.rotary_frequencies(64)
q, s = torch.empty(1300, 512, device="cuda", dtype=torch.int8), torch.empty(1300, device="cuda")
outs = [torch.empty(1300, 512, device="cuda", dtype=torch.bfloat16), torch.empty(1300, 300, device="cuda"), torch.empty(5, 300, device="cuda"), torch.empty(1300, 8, 64, device="cuda", dtype=torch.bfloat16)]
torch.cuda.synchronize()
def calls():
    ep.norm(x, out=outs[0])
    ep.quantize_rows(x, out=(q, s))
    ep.int8_matmul(q, s, w, out=outs[1])
    ep.int8_matmul(q[:5], s[:5], w, out=outs[2])
    ep.rotary(x.view(1300, 8, 64), at, f, out=outs[3])
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in outs]
calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, outs)) and outs[1].abs().sum() > 0
print("captured")
"""


@gpu
def test_first_calls_of_a_process_can_be_captured():
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(name=ep.__name__)], capture_output=True, text=True, timeout=300,
                          cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0 and done.stdout.split() == ["captured"], done.stderr[-2000:]


@gpu
def test_no_rows():
    e = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    q, s = ep.quantize_rows(e(0, 64))
    assert q.shape == (0, 64) and s.shape == (0,)
    assert ep.int8_matmul(q, s, e(48, 64, dtype=torch.int8)).shape == (0, 48)
    z, r = ep.norm(e(0, 64), e(64), residual=e(0, 64))
    assert z.shape == r.shape == (0, 64)
    assert ep.rotary(e(0, 4, 64), e(0, dtype=torch.int32), ep.rotary_frequencies(64)).shape == (0, 4, 64)


@gpu
def test_norm_of_no_rows_to_eight_bits():
    x, w = torch.empty(0, 300, dtype=torch.bfloat16, device="cuda"), torch.ones(300, device="cuda")
    q, s = ep.norm(x, w, out_dtype=ep.INT8)
    assert q.shape == (0, 300) and q.dtype == torch.int8 and s.shape == (0,)
    (q, s), r = ep.norm(x, w, residual=x, out_dtype=ep.FP8_E4M3)
    assert q.shape == r.shape == (0, 300) and s.shape == (0, 3)


@gpu
def test_more_than_32_bits_of_values():
    # rows and outputs beyond 2^31 values and 2^32 bytes: the last row is as the first
    T, C = 70000, 32768
    x = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    x[0] = torch.randn(C, generator=cuda(1), device="cuda")
    x[-1] = x[0]
    x[-2] = 0
    q, s = ep.quantize_rows(x)
    assert torch.equal(q[0], q[-1]) and s[0] == s[-1] and (q[-2] == 0).all()
    z = ep.norm(x, out=x)                                  # (each row is read before it is written)
    assert torch.equal(z[0], z[-1])
    del q
    a, w = (torch.randint(-127, 128, (n, 64), generator=cuda(n), device="cuda", dtype=torch.int8) for n in (T, C))
    a[-1], s[0] = a[0], 0.01
    s[-1] = s[0]
    y = ep.int8_matmul(a, s, w)
    assert torch.equal(y[0], y[-1]) and torch.equal(y[0], ((w.double() @ a[0].double()).float() * s[0]).to(torch.bfloat16))
    del y
    heads = z.view(T, 256, 128)
    at = torch.zeros(T, dtype=torch.int32, device="cuda")
    at[0] = at[-1] = 77
    out = ep.rotary(heads, at, ep.rotary_frequencies(128), out=heads)
    assert torch.equal(out[0], out[-1]) and (out[-2] == 0).all()


@gpu
def test_refusals():
    f = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
    i8, f32 = torch.int8, torch.float32
    x, w, s = f(4, 64, dtype=i8), f(32, 64, dtype=i8), f(4, dtype=f32)
    wrong = [
        lambda: ep.quantize_rows(f(4)), lambda: ep.quantize_rows(f(4, 8, dtype=torch.int8)), lambda: ep.quantize_rows(torch.zeros(4, 8)),
        lambda: ep.quantize_rows(f(8, 4).t()), lambda: ep.quantize_rows(f(4, 8), out=(f(4, 8, dtype=i8), f(3, dtype=f32))),
        lambda: ep.quantize_rows(f(4, 8), out=(f(4, 8), f(4, dtype=f32))), lambda: ep.quantize_rows(f(4, 8), out=(f(4, 8, dtype=i8), None)),
        lambda: ep.int8_matmul(x, s, f(32, 48, dtype=i8)), lambda: ep.int8_matmul(x, None, w), lambda: ep.int8_matmul(x, s[:3], w), lambda: ep.int8_matmul(x, s, w, row_scale=s),
        lambda: ep.int8_matmul(x, s, w, bias=f(32)), lambda: ep.int8_matmul(x, s, w, out=f(4, 31)), lambda: ep.int8_matmul(x, s, w, out_dtype=ep.INT8),
        lambda: ep.int8_matmul(x.view(torch.uint8), s, w), lambda: ep.int8_matmul(x, s, w.cpu()),
        lambda: ep.norm(f(4)), lambda: ep.norm(f(4, 8), f(7)), lambda: ep.norm(f(4, 8), f(3, 8)), lambda: ep.norm(f(4, 8), f(0, 8)), lambda: ep.norm(f(4, 8), out_dtype=ep.UINT8),
        lambda: ep.norm(f(4, 8), residual=f(4, 7)), lambda: ep.norm(f(4, 8), residual=f(4, 8), residual_out=f(4, 8, dtype=f32)), lambda: ep.norm(f(4, 8), out=(f(4, 8, dtype=i8), None)),
        lambda: ep.norm(f(4, 8), out=f(4, 8, dtype=i8)), lambda: ep.norm(f(4, 8), f(8, dtype=i8)), lambda: ep.norm(f(4, 8), f(8, 4).t()), lambda: ep.norm(f(4, 8), torch.zeros(8)),
        lambda: ep.norm(f(4, 8), out=(f(4, 8), f(4, dtype=f32))),
        lambda: ep.rotary(f(4, 64), f(4, dtype=torch.int32), ep.rotary_frequencies(64)), lambda: ep.rotary(f(4, 2, 64), f(3, dtype=torch.int32), ep.rotary_frequencies(64)),
        lambda: ep.rotary(f(4, 2, 64), f(4, dtype=f32), ep.rotary_frequencies(64)), lambda: ep.rotary(f(4, 2, 64), f(4, dtype=torch.int32), ep.rotary_frequencies(64).float()),
        lambda: ep.rotary(f(4, 2, 64), f(4, dtype=torch.int32), ep.rotary_frequencies(66)), lambda: ep.rotary(f(4, 64, 2).transpose(1, 2), f(4, dtype=torch.int32), ep.rotary_frequencies(64)),
        lambda: ep.rotary(f(4, 2, 64), f(4, dtype=torch.int32), ep.rotary_frequencies(64)[:0]), lambda: ep.rotary(f(4, 2, 64), f(4, dtype=torch.int32), ep.rotary_frequencies(64, device="cpu")),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    unsupported = [lambda: ep.int8_matmul(f(4, 24, dtype=i8), s, f(32, 24, dtype=i8)), lambda: ep.int8_matmul(f(4, 80, dtype=i8)[:, 3:67], s, w),
                   lambda: ep.int8_matmul(f(4, 131072, dtype=i8), s, f(2, 131072, dtype=i8)), lambda: ep.norm(f(2, 32769))]
    for call in unsupported:
        with pytest.raises(ep.EntroPackError) as e:
            call()
        assert e.value.status == -3


@gpu
@pytest.mark.parametrize("next", [False, True])
def test_rotary_of_heads_before_rows(next):
    # each head's rows side by side, the tightest that lie apart; one row or one head may have any distance; what overlaps is refused
    T, H, D, f = 21, 3, 64, ep.rotary_frequencies(64)
    x, at = torch.randn(T, H, D, generator=cuda(4), device="cuda"), torch.arange(T, device="cuda") * 7
    out = torch.zeros(H, T, D, device="cuda").transpose(0, 1)
    assert ep.rotary(x, at, f, interleaved=next, out=out) is out
    check_turn(out, x, at, f, next, 1.0)
    here = x.transpose(0, 1).contiguous().transpose(0, 1)
    check_turn(ep.rotary(here, at, f, interleaved=next, out=here), x, at, f, next, 1.0)
    room = torch.zeros(T * H * D, device="cuda")
    for shape, stride in (((1, H, D), (1, D, 1)), ((T, 1, D), (D, 3, 1))):
        rows, heads = shape[:2]
        out = room.as_strided(shape, stride)
        check_turn(ep.rotary(x[:rows, :heads], at[:rows], f, interleaved=next, out=out), x[:rows, :heads], at[:rows], f, next, 1.0)
    for stride in ((D, D, 1), (2 * D + 32, D, 1), (D, T * D - 1, 1)):
        with pytest.raises(ep.EntroPackError) as e:
            ep.rotary(x, at, f, out=room.as_strided((T, H, D), stride))
        assert e.value.status == -1


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,C", [(1, 5120), (16, 5120), (9, 1001), (2, 17408), (40000, 128), (1300, 1000), (1200, 12808)])
def test_norm_in_the_places_of_what_it_reads(T, C, dtype):
    # z over x or over the residual, r over the other one or over x alone: the same bits as with places of their own; another type is refused
    x, v = norm_inputs(T, C, dtype, dtype, 1, T + C)
    want, r_want = ep.norm(x, **v)
    for z_over, r_over in (("h", None), ("h", "x"), ("x", "h"), ("x", None), (None, "x"), (None, "h")):
        here = {"x": x.clone(), "h": v["residual"].clone(), None: None}
        got = ep.norm(here["x"], **{**v, "residual": here["h"]}, out=here[z_over], residual_out=here[r_over])
        assert torch.equal(got[0], want) and torch.equal(got[1], r_want)
        assert all(over is None or g is here[over] for g, over in zip(got, (z_over, r_over)))
    other = torch.float16
    for call in (lambda: ep.norm(x, **v, out=v["residual"].view(torch.int16 if dtype != torch.float32 else torch.int32).view(other)[:, :C]),
                 lambda: ep.norm(x, out=x, residual_out=x), lambda: ep.norm(x, residual_out=x.view(other)[:, :C])):
        with pytest.raises(ep.EntroPackError) as e:
            call()
        assert e.value.status == -1
    assert ep.last_device_status() == 0


def angles(at, f):
    """position * frequency as fractions of a turn, exactly, nearest to 0, in doubles: 1 / 2 pi to 80 digits, whole numbers."""
    from fractions import Fraction
    inverse = Fraction(15915494309189533576888376337251436203445964574045644874766734405889679763422653509, 10 ** 83)
    one = lambda p, w: (p * Fraction(w) * inverse + Fraction(1, 2)) % 1 - Fraction(1, 2)  # noqa: E731
    return torch.tensor([[float(one(p, w)) for w in f.tolist()] for p in at.tolist()], dtype=torch.float64, device="cuda") * (2 * math.pi)


FAR = [1, -5, 200000, (1 << 31) - 1, 1 << 40, (1 << 45) + 1, 1 << 50, -(1 << 56) - 12345, (1 << 60) + 3, (1 << 63) - 1, -(1 << 63)]


@gpu
@pytest.mark.parametrize("next", [False, True])
def test_rotary_as_far_as_64_bits_reach(next):
    # Pairs (1, 0) show the cosine and sine themselves: 2 units for CUDA's sincospi; pi 2^-25 for the angle in a float, 2 pi 2^-32 for what is cut off before that; and what the
    # position makes of its step's rounding, to 2^-64 of a turn (half a turn: to one less) and 2^-52 of itself.
    at = torch.tensor(FAR, device="cuda")
    for f in (ep.rotary_frequencies(64, 1e6, 8.0, 8192.0), torch.tensor([1.0, 0.5, 3.6e-6, 1e-9, 1e-12, 2.5, -1.0, math.pi], dtype=torch.float64, device="cuda")):
        n = len(f)
        x = torch.zeros(len(at), 1, 2 * n, device="cuda")
        (x[..., 0::2] if next else x[..., :n]).fill_(1)
        y = ep.rotary(x, at, f, interleaved=next).double()[:, 0]
        cos, sin = (y[:, 0::2], y[:, 1::2]) if next else (y[:, :n], y[:, n:])
        a = angles(at, f)
        bound = 2 * U + math.pi * 2.0 ** -25 + 2 * math.pi * 2.0 ** -32 + at.double().abs()[:, None] * (f.abs() * 2.0 ** -52 + 2.0 ** -61)
        assert ((cos - a.cos()).abs() <= bound).all() and ((sin - a.sin()).abs() <= bound).all()


@gpu
@pytest.mark.parametrize("next", [False, True])
def test_rotary_in_32_bits_keeps_the_bits_of_an_angle(next):
    # Near half a turn the sine is small and shows the angle: 4 units of it for sincospi, which takes from half of it to one and a half, 1 for the sum with the rest; the rest d
    # (below pi 2^-24) is good to 3 units of itself and to one of 2^-56 of a turn that is cut off.  And the position's share, as above.
    f = torch.tensor([math.pi + d for d in (1e-3, -1e-3, 3.1e-4, 7e-5, -2.2e-5, 1e-5)] + [2 * math.pi + 1e-4, 1e-4], dtype=torch.float64, device="cuda")
    at = torch.tensor([1, -1, 3, -17, 251, -249, 901], device="cuda")
    n = len(f)
    x = torch.zeros(len(at), 1, 2 * n, device="cuda")
    (x[..., 0::2] if next else x[..., :n]).fill_(1)
    y = ep.rotary(x, at, f, interleaved=next).double()[:, 0]
    cos, sin = (y[:, 0::2], y[:, 1::2]) if next else (y[:, :n], y[:, n:])
    a = angles(at, f)
    share = at.double().abs()[:, None] * (f.abs() * 2.0 ** -52 + 2.0 ** -61) + 2 * math.pi * 2.0 ** -56 + 3 * U * math.pi * 2.0 ** -24
    assert ((sin - a.sin()).abs() <= 8 * U * a.sin().abs() + share).all()
    assert ((cos - a.cos()).abs() <= 2.6 * U + share).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,C", [(4, 64), (16, 512), (7, 1001), (40000, 128), (1300, 1000), (1190, 12808)])
def test_norm_keeps_the_sign_of_a_zero(T, C, dtype):
    # without an offset nothing is added to a vector: a weight or gate of -0 turns the sign of what it multiplies, whichever kernel takes the rows
    x = (torch.rand(T, C, generator=cuda(C), device="cuda") + 0.5).to(dtype)
    w = torch.full((C,), -0.0, dtype=dtype, device="cuda")
    p, one = torch.where(torch.arange(C, device="cuda") % 3 == 0, w, torch.ones_like(w)), torch.ones_like(w)
    z = ep.norm(x, w)
    assert (z == 0).all() and z.signbit().all()
    r = torch.empty_like(x)
    z = ep.norm(x, one, one * -0.0, gate=p, post_weight=one, residual_out=r)[0]
    assert torch.equal(r.signbit(), r == 0) and torch.equal(z.signbit(), z == 0) and torch.equal(z == 0, (p == 0).expand(T, C))


@gpu
def test_on_a_given_stream_while_the_current_one_is_busy():
    # What the given stream holds when it has ended, looked at from itself, while a wait of a second or two still stands before everything on the current stream.  (Once
    # before that, since the first launch of a kernel waits for the device.)
    calls, flat, (x, qx, heads) = each_operator(9)
    ones, at, f = torch.ones(len(qx), device="cuda"), torch.arange(len(heads), device="cuda"), ep.rotary_frequencies(64)
    fresh = lambda stream=None: [*ep.quantize_rows(x, stream=stream), ep.norm(x, stream=stream), *ep.norm(x, residual=x, out_dtype=ep.FP8_E4M3, stream=stream)[0],  # noqa: E731
                                 ep.int8_matmul(qx, ones, qx, stream=stream), ep.rotary(heads, at, f, stream=stream)]
    same = lambda a, b: len(a) == len(b) and all([torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b)])  # noqa: E731
    calls()
    want, stream = [t.clone() for t in flat()] + fresh(), torch.cuda.Stream()
    for busy in (False, True):
        for t in flat():
            t.zero_()
        torch.cuda.synchronize()
        if busy:
            torch.cuda._sleep(4_000_000_000)
        calls(stream)
        new = fresh(stream)
        with torch.cuda.stream(stream):
            got = [t.clone() for t in flat() + new]
            assert same(got, want)
        stream.synchronize()
        assert torch.cuda.current_stream().query() != busy
        torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T,C,groups", [(40000, 128, 1), (30011, 64, 1), (9000, 256, 1), (1300, 1000, 1), (2501, 2048, 1), (1190, 12808, 1), (2400, 12800, 2), (2400, 12800, 4), (1200, 16384, 3)])
def test_norm_of_many_rows_with_an_offset(T, C, groups, dtype, wide):
    # weights stored without their 1, vectors of 16 bits where they have to wait as they lie in memory, alone and for each group; a row of zeros and one that is not finite
    x, v = norm_inputs(T, C, dtype, wide, groups, T + C)
    zero, bad = T // 3, T // 2
    x[zero] = v["residual"][zero] = 0
    x[bad, C - 1] = math.inf
    fine = torch.arange(T, device="cuda") != bad
    for center in (False, True):
        for left in ((), ("gate",), ("post_weight", "bias")):
            given = {k: t for k, t in v.items() if k not in left}
            z, r = ep.norm(x, weight_offset=1.0, residual_scale=0.7, center=center, **given)
            want, r_want = normed(x, weight_offset=1.0, residual_scale=0.7, center=center, **given)
            assert near(z[fine], tuple(t[fine] for t in want)) and near(r[fine], tuple(t[fine] for t in r_want))
            assert z[bad].isnan().any() and (r[zero] == 0).all()
            assert torch.equal(z[zero], rows_of(v["bias"], T)[zero].to(dtype) if "bias" in given else torch.zeros_like(z[zero]))
    assert ep.last_device_status() == 0


@gpu
@pytest.mark.parametrize("dtype,wide", [(torch.bfloat16, torch.float32), (torch.float32, torch.float16)])
@pytest.mark.parametrize("c0", [0, 8, 1, 3])
def test_norm_to_int8_in_views(c0, dtype, wide):
    # values and scales of rows of any distance and alignment are those of the 32-bit result
    T, C = 33, 200
    x, v = norm_inputs(T, C + 20, dtype, wide, 3, 20 + c0)
    x, v = x[..., c0:c0 + C], {k: t[..., c0:c0 + C] for k, t in v.items()}
    values, scales = torch.full((T, C + 29), 3, dtype=torch.int8, device="cuda"), torch.full((T + 2,), 3.0, device="cuda")
    out = (values[:, c0:c0 + C], scales[1:T + 1])
    got, r = ep.norm(x, **v, out=out)
    z, r32 = ep.norm(x, **v, out_dtype=ep.FP32)
    q, s = ep.quantize_rows(z)
    assert got is out and torch.equal(got[0], q) and torch.equal(got[1], s) and torch.equal(r, r32)
    assert (values[:, :c0] == 3).all() and (values[:, c0 + C:] == 3).all() and scales[0] == scales[T + 1] == 3


@gpu
@pytest.mark.parametrize("dtype", [E4M3, torch.int8])
def test_norm_refuses_values_without_their_scales(dtype):
    x, q = torch.zeros(4, 256, device="cuda"), torch.zeros(4, 256, dtype=torch.uint8, device="cuda").view(dtype)
    with pytest.raises(ValueError):
        ep.norm(x, out=(q, None))
    with pytest.raises(ValueError):
        ep.norm(x, out=(q,))
