"""What the INT8 product, the norms and rotary positions refuse and compute without a GPU."""
import math
import struct

import numpy as np
import pytest
import torch

import paper_2609_34185_b200 as ep

P = 1 << 20                                               # an address that is never read
BAD, UNSUPPORTED = -1, -3
B = ep.binding


def vector(d=0, ld=0, groups=0, dtype=ep.BF16):
    return d, ld, groups, dtype


def rows_job(x=P, q=P, s=P, ldx=64, ldq=64, T=4, C=64, dtype=ep.BF16):
    return ep.load().ep_quantize_rows(B.QUANTIZE_ROWS_JOB.pack(x, q, s, ldx, ldq, T, C, dtype), None)


def matmul_job(x=P, xs=P, w=P, a=0, bias=0, y=P, ldx=64, ldw=64, ldy=32, T=4, R=32, C=64, dtype=ep.BF16):
    return ep.load().ep_int8_matmul(B.INT8_MATMUL_JOB.pack(x, xs, w, a, bias, y, ldx, ldw, ldy, T, R, C, dtype), None)


def norm_job(x=P, h=0, r=0, z=P, s=0, ldx=64, ldh=64, ldr=64, ldz=64, lds=1, w=vector(), d=vector(), g=vector(), p=vector(), T=4, C=64, dtype=ep.BF16, hdtype=ep.BF16, zdtype=ep.BF16):
    return ep.load().ep_norm(B.NORM_JOB.pack(x, h, r, z, s, ldx, ldh, ldr, ldz, lds, *w, *d, *g, *p, 1.0, 0.0, 1e-6, T, C, dtype, hdtype, zdtype, 0), None)


def rotary_job(x=P, o=2 * P, at=P, f=P, ldx=64, ldxh=64, ldo=64, ldoh=64, T=4, H=1, D=64, pairs=32, dtype=ep.BF16, bits=32):
    return ep.load().ep_rotary(B.ROTARY_JOB.pack(x, o, at, f, ldx, ldxh, ldo, ldoh, T, H, D, pairs, 1.0, dtype, bits, 0), None)


@pytest.mark.parametrize("job,wrong", [
    (rows_job, [dict(x=0), dict(q=0), dict(s=0), dict(C=0), dict(ldx=63), dict(ldq=63), dict(dtype=ep.INT8), dict(x=P + 1), dict(s=P + 2), dict(ldx=1 << 40)]),
    (matmul_job, [dict(x=0), dict(xs=0), dict(w=0), dict(y=0), dict(R=0), dict(C=0), dict(dtype=ep.INT8), dict(ldx=48), dict(ldw=48), dict(ldy=31), dict(y=P + 1), dict(xs=P + 2),
                  dict(a=P + 2), dict(bias=P + 1)]),
    (norm_job, [dict(x=0), dict(z=0), dict(C=0), dict(ldx=63), dict(ldz=63), dict(dtype=ep.INT8), dict(zdtype=ep.UINT8), dict(zdtype=ep.INT8), dict(zdtype=ep.FP8_E4M3),
                dict(zdtype=ep.FP8_E4M3, s=P, lds=0), dict(zdtype=ep.INT8, s=P + 1), dict(h=P, ldh=63), dict(r=P, ldr=10), dict(h=P, hdtype=ep.INT8), dict(h=P, r=P, ldh=64, ldr=72),
                dict(w=vector(P, 64, 3)), dict(w=vector(P, 64, 0)), dict(d=vector(P, 60, 2)), dict(g=vector(P, 64, 1, ep.INT8)), dict(p=vector(P + 1, 64, 1))]),
    (rotary_job, [dict(x=0), dict(o=0), dict(at=0), dict(f=0), dict(H=0), dict(H=65536), dict(pairs=0), dict(pairs=33), dict(D=1025), dict(dtype=ep.INT8), dict(bits=16), dict(at=P + 2),
                  dict(at=P + 4, bits=64), dict(f=P + 4), dict(ldx=-1), dict(x=P, o=P, ldo=72), dict(x=P + 1), dict(ldo=32), dict(H=2, ldoh=0), dict(H=2, ldo=128, ldoh=63)]),
])
def test_bad_arguments(job, wrong):
    assert job(T=0) == 0
    for w in wrong:
        assert job(**w) == BAD, w


@pytest.mark.parametrize("wrong", [dict(zdtype=ep.FP32), dict(zdtype=ep.FP16), dict(ldz=72), dict(zdtype=ep.INT8, s=3 * P), dict(zdtype=ep.FP8_E4M3, s=3 * P), dict(z=2 * P, r=2 * P)])
def test_norm_over_what_it_reads(wrong):
    """z in x's place has x's type and ld, and z and r have places of their own."""
    assert norm_job(T=0, **wrong) == 0 and norm_job(**wrong) == BAD


def test_unsupported():
    for w in (dict(C=56), dict(ldx=72), dict(ldw=72), dict(x=P + 8), dict(w=P + 8), dict(C=1 << 17, ldx=1 << 17, ldw=1 << 17)):
        assert matmul_job(**w) == UNSUPPORTED, w
    assert norm_job(C=32769, ldx=32769, ldz=32769) == UNSUPPORTED


def test_null_jobs():
    L = ep.load()
    assert [f(None, None) for f in (L.ep_quantize_rows, L.ep_int8_matmul, L.ep_norm, L.ep_rotary)] == [BAD] * 4


def test_jobs_are_laid_out_as_in_c():
    # sizes that the compiler gives the structs (eight-byte alignment, as on every 64-bit Linux)
    assert [j.size for j in (B.QUANTIZE_ROWS_JOB, B.INT8_MATMUL_JOB, B.NORM_JOB, B.ROTARY_JOB)] == [56, 88, 216, 96]
    assert struct.calcsize("@PqIi") == 24


def test_frequencies():
    got = ep.rotary_frequencies(128, 1e6, device="cpu").numpy()
    want = [1e6 ** (-2 * i / 128) for i in range(64)]
    assert got.dtype == np.float64 and np.allclose(got, want, rtol=1e-14)
    assert np.allclose(ep.rotary_frequencies(128, 1e6, 4.0, device="cpu").numpy(), np.array(want) / 4, rtol=1e-14)
    some = ep.rotary_frequencies(128, 1e6, 4.0, 8192.0, 32.0, 1.0, device="cpu").numpy()
    turns = 8192 * np.array(want) / (2 * math.pi)
    k = np.clip((turns - 1) / 31, 0, 1)
    assert np.allclose(some, np.array(want) * (k + (1 - k) / 4), rtol=1e-13)
    assert (some[turns > 32] == np.array(got)[turns > 32]).all() and np.allclose(some[turns < 1], got[turns < 1] / 4, rtol=1e-14)


def test_frequencies_refused():
    for dim in (0, 1, 7):
        with pytest.raises(ValueError):
            ep.rotary_frequencies(dim, device="cpu")
    for kw in (dict(base=0.0), dict(base=-1.0), dict(base=math.nan), dict(stretch=0.5), dict(stretch=math.inf), dict(original=-1.0), dict(original=10.0, fast=1.0, slow=1.0),
               dict(original=math.nan)):
        with pytest.raises(ep.EntroPackError):
            ep.rotary_frequencies(64, device="cpu", **kw)


def test_tensors_of_the_host_are_refused():
    z = torch.zeros
    for call in (lambda: ep.quantize_rows(z(4, 8)), lambda: ep.int8_matmul(z(4, 16, dtype=torch.int8), z(4), z(8, 16, dtype=torch.int8)), lambda: ep.norm(z(4, 8)),
                 lambda: ep.rotary(z(4, 2, 8), z(4, dtype=torch.int32), ep.rotary_frequencies(8, device="cpu"))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("wrong", [dict(ldo=64, ldoh=64), dict(ldo=96, ldoh=64), dict(ldo=64, ldoh=64, T=2, H=2), dict(ldo=64, ldoh=255), dict(ldo=191, ldoh=64, H=3),
                                   dict(o=P, ldx=64, ldxh=64, ldo=64, ldoh=64), dict(ldo=(1 << 40) - 1, ldoh=(1 << 40) - 1, T=1 << 30)])
def test_rotary_of_outputs_that_overlap(wrong):
    """A row's heads reach into the next row, or a head's rows into the next head: two places for one value."""
    assert rotary_job(**{"T": 5, "H": 2, **wrong}) == BAD


@pytest.mark.parametrize("wrong", [dict(h=2 * P, z=2 * P, hdtype=ep.FP32), dict(h=2 * P, z=2 * P, zdtype=ep.FP16), dict(h=2 * P, z=2 * P, ldz=72), dict(h=2 * P, z=2 * P, zdtype=ep.INT8, s=3 * P),
                                   dict(h=2 * P, z=2 * P, r=3 * P, zdtype=ep.FP8_E4M3, s=4 * P), dict(r=P, z=2 * P, hdtype=ep.FP32), dict(r=P, z=2 * P, dtype=ep.FP32, ldx=64),
                                   dict(r=P, z=2 * P, ldr=72), dict(h=3 * P, r=P, z=2 * P, ldh=72, ldr=72), dict(x=P, h=P, z=2 * P, r=P, hdtype=ep.FP16)])
def test_norm_over_a_residual_or_with_r_over_x(wrong):
    """z in the residual's place and r in x's place have the type and ld of what was there."""
    assert norm_job(T=0, **wrong) == 0 and norm_job(**wrong) == BAD


def test_results_in_the_place_of_operands():
    """Other rows, or other tiles, still have to be read there."""
    for w in (dict(q=P), dict(q=P, dtype=ep.FP32), dict(q=P, ldq=128)):
        assert rows_job(T=0, **w) == 0 and rows_job(x=P, **w) == BAD, w
    for w in (dict(x=P, w=2 * P), dict(x=2 * P, w=P), dict(x=P, w=2 * P, dtype=ep.FP32)):
        assert matmul_job(T=0, y=P, **w) == 0 and matmul_job(y=P, **w) == BAD, w


def test_frequencies_that_are_none():
    """What is not a finite number is refused, wherever it comes from: header and kernels ask for finite frequencies."""
    for kw in (dict(original=10.0, fast=math.inf, slow=-math.inf), dict(original=10.0, fast=1.0, slow=-math.inf), dict(original=1e308, base=5e-324), dict(base=5e-324)):
        with pytest.raises(ep.EntroPackError) as e:
            ep.rotary_frequencies(256, device="cpu", **kw)
        assert e.value.status == BAD
    assert np.isfinite(ep.rotary_frequencies(256, device="cpu", original=10.0, stretch=2.0, fast=math.inf).numpy()).all()
