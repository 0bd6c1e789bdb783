"""Rows whose squares leave the range of fp32, next to ordinary rows of the same warp: norm, tangent, 8-bit rows and backward against the
fp64 oracle, with the bounds of the ordinary ones (64 roundings, 128 for the scale's gradient).

The factor that brings a row back is a power of two, exact in itself; 1 / r beyond 2^126 is a denormal number, off by up to 2^-22 of itself, which is
four roundings more for each of the two such factors that enter a result: the 64 have room for them (sums of at most 40 elements a thread and 10
steps between threads, and some ten operations, take 60 of them in the worst case of one sign; signs are drawn here).
"""
import numpy as np
import pytest
import torch

from oracle import row_ops_numpy as orn
from paper_2511_19797_b200 import binding
from tests.test_row_ops_gpu import DTYPES, _check_8_bits, _close, _dev, _draw, _np

pytestmark = pytest.mark.gpu

# the sizes of a call's rows; rows of normals times 4e37 stay below 2^128, those of "largest" hold the type's largest values
LARGE, TINY = [1.0, 4e37, 1e30, 1.0, 2e19, 1e17, 3.0, 1e36], [1e-30, 1.0, 1e-37, 1e-25, 1e-10, 1e-20, 1.0, 1e-16]
WIDTHS = [8, 64, 333, 1152, 1151, 2560, 4096, 16384]


def _rows(seed, D, dtype, sizes):
    t = _draw(seed, len(sizes), D).double().clamp_(-6, 6) * torch.tensor(sizes, dtype=torch.float64)[:, None]
    assert t.abs().max() < 3.38e38
    return t.to(dtype)


def _largest(seed, D, dtype):
    return torch.sign(_draw(seed, 3, D)).to(dtype) * torch.finfo(dtype).max


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("sizes", [LARGE, TINY])
def test_norm_and_tangent(D, dtype, sizes):
    h, g = _rows(D, D, dtype, sizes), 1 + _draw(D + 9, D, std=0.3)
    # tangents of the size of the rows; and ordinary ones where the quotient of the two is a number of the type
    ordinary = [1.0 if s > 1e-30 else s for s in sizes]
    for eps in (0.0, 1e-6, 1e-36):
        for th in (_rows(D + 1, D, dtype, [min(s, 1e37) for s in sizes]), _rows(D + 2, D, dtype, ordinary)):
            y, _, ty, _ = binding.tvm_attn_rmsnorm_jvp_fwd(*_dev(h, None, th, None, g), eps=eps)
            want = orn.rmsnorm_jvp_fwd(*map(_np, (h, None, th, None, g)), eps)
            _close(y, want["y"], what="y")
            _close(ty, want["ty"], what="ty")
            assert torch.equal(y, binding.tvm_attn_rmsnorm_jvp_fwd(*_dev(h, None, None, None, g), eps=eps)[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_rows_of_the_largest_and_the_smallest_values(D, dtype):
    g = 1 + _draw(D + 9, D, std=0.3)
    small = _draw(D, 4, D).to(dtype) * 1e-39      # denormal numbers: exact inputs, whatever they were rounded from
    for h in (_largest(D, D, dtype), small, torch.cat([_largest(D, D, dtype), small])):
        for eps in (0.0, 1e-6):
            want = orn.rmsnorm_jvp_fwd(*map(_np, (h, None, None, None, g)), eps)["y"]
            _close(binding.tvm_attn_rmsnorm_jvp_fwd(*_dev(h, None, None, None, g), eps=eps)[0], want)
            q, s, _ = binding.tvm_attn_rmsnorm_s8(*_dev(h, None, g), eps=eps)
            _check_8_bits(q, s, want[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("sizes", [LARGE, TINY])
def test_8_bits(D, dtype, sizes):
    x, g = _rows(D, D, dtype, sizes), 1 + _draw(D + 9, D, std=0.3)
    for eps in (0.0, 1e-6, 1e-36):
        for scale in (g, None, 100 * g):          # (the scaled sum itself leaves the range)
            q, s, _ = binding.tvm_attn_rmsnorm_s8(*_dev(x, None, scale), eps=eps)
            _check_8_bits(q, s, orn.rmsnorm_jvp_fwd(*map(_np, (x, None, None, None, scale)), eps)["y"][0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("sizes", [LARGE, TINY])
def test_backward(D, dtype, sizes):
    h, g = _rows(D, D, dtype, sizes), 1 + _draw(D + 9, D, std=0.3)
    # cotangents of the size of the rows give dx and dtx of order one; 2^-20 of it where their sum over the rows would leave the range
    like = [s * 2.0 ** -20 if s > 1e19 else s for s in sizes]
    dy, dty = _rows(D + 1, D, dtype, like), _rows(D + 2, D, dtype, like)
    near, ordinary = _rows(D + 3, D, dtype, sizes), _rows(D + 4, D, dtype, [1.0 if s > 1e-15 else s for s in sizes])
    dh, dth = (_rows(D + 5 + k, D, dtype, [1.0] * len(sizes)) for k in range(2))
    for eps in (0.0, 1e-6):
        for ins in ((h, dy, None, None, None, None), (h, dy, near, dty, None, None), (h, dy, ordinary, dty, dh, dth), (h, torch.zeros_like(dy), near, dty, None, dth)):
            for scale in (g, None):
                got = binding.tvm_attn_rmsnorm_jvp_bwd(*_dev(*ins, scale), eps=eps)
                want = orn.rmsnorm_jvp_bwd(*map(_np, (*ins, scale)), eps)
                for name, v in zip(("dx", "dtx", "dg"), got):
                    if v is not None:
                        _close(v, want[name], 128 if name == "dg" else 64, what=(name, eps))
