"""The rounding of rows to 8 bits: q = 127 v / max|v| to the nearest whole number, ties to even.

Of two bf16 values the quotient 127 v / max|v| is a tie or at least its own 2^-16th part away from one: with 8-bit significands a and b,
127 a / b - (k + 1/2) = (254 a - (2 k + 1) b) / (2 b), whose numerator is a whole number.  127 v / max|v| in 64 bits, which is off by 2^-53 of
itself and exact at a tie, therefore rounds as the quotient does, and the kernels' values have to be equal to that.  Of other fp32 values the
kernels round the quotient to fp32 in between, by 2^-18 at most (127 < 2^7).
"""
import numpy as np
import pytest
import torch

from paper_2511_19797_b200 import binding

pytestmark = pytest.mark.gpu


def _steps(v):
    v = v.double().numpy()
    return 127.0 * v / np.abs(v).max(axis=-1, keepdims=True)


def _all_quotients(exponent):
    """(128, 1152): row m has 128 + m as its largest element, and all quotients of bf16 elements of a 254th of that and more (times 2^exponent)."""
    a = torch.arange(128, 256, dtype=torch.float64)
    rows = (a[None, :] * 2.0 ** -torch.arange(9, dtype=torch.float64)[:, None]).reshape(1, -1).repeat(128, 1)
    rows = torch.minimum(rows, a[:, None])
    rows[:, ::3] *= -1
    x = (rows * 2.0 ** exponent).bfloat16()
    assert torch.equal(x.double(), rows * 2.0 ** exponent)
    return x


@pytest.mark.parametrize("exponent", [0, -7, 119, -118])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_quotient_of_bf16_values(dtype, exponent):
    x = _all_quotients(exponent)
    want = np.rint(_steps(x))
    ties = _steps(x) % 1.0 == 0.5
    assert ties.any(axis=1).all() and ties[254 - 128].sum() >= 127      # half of the largest element is one; of 254 all odd numbers are
    top = x.float().abs().amax(-1).numpy()
    # rows on 16 bytes, rows off them, rows of a few elements on the lanes of a warp
    off = torch.zeros(128, 1155, dtype=dtype, device="cuda")[:, 1:1153]
    off.copy_(x)
    for v in (x.to(dtype).cuda(), off):
        q, s = binding.tvm_attn_quantize_s8(v)
        assert np.array_equal(q.cpu().numpy(), want)
        assert np.array_equal(s.cpu().numpy(), top / np.float32(127))
    parts = x.reshape(128, 16, 72).clone()
    parts[..., 0] = x.abs().amax(-1)[:, None]
    q, _ = binding.tvm_attn_quantize_s8(parts.to(dtype).cuda())
    assert np.array_equal(q.cpu().numpy(), np.rint(_steps(parts)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_quotient_behind_the_norm(dtype):
    """The norm divides out: with a scale of a power of two, or none, the 8-bit values are those of h itself."""
    x = _all_quotients(-7).to(dtype)
    want = np.rint(_steps(x))
    for g in (None, torch.full((1152,), 0.25, device="cuda")):
        for res in (None, x.cuda()):
            q, _, _ = binding.tvm_attn_rmsnorm_s8(x.cuda(), res, g)
            assert np.array_equal(q.cpu().numpy(), want)


@pytest.mark.parametrize("D", [72, 768, 1152, 4096])
def test_ties_of_ordinary_rows(D):
    x = torch.randn(2000, D, generator=torch.Generator().manual_seed(D)).bfloat16()
    want = np.rint(_steps(x))
    assert (_steps(x) % 1.0 == 0.5).any()
    assert np.array_equal(binding.tvm_attn_quantize_s8(x.cuda())[0].cpu().numpy(), want)
    assert np.array_equal(binding.tvm_attn_rmsnorm_s8(x.cuda())[0].cpu().numpy(), want)


@pytest.mark.parametrize("D", [100, 1151, 2048])
def test_fp32_rows(D):
    x = torch.randn(3000, D, generator=torch.Generator().manual_seed(D + 1))
    q, s = binding.tvm_attn_quantize_s8(x.cuda())
    assert (np.abs(q.cpu().double().numpy() - _steps(x)) <= 0.5 + 2.0 ** -18 + 2.0 ** -30).all()
    assert np.array_equal(s.cpu().numpy(), x.abs().amax(-1).numpy() / np.float32(127))


@pytest.mark.parametrize("dtype,step", [(torch.bfloat16, 2.0 ** -133), (torch.float32, 2.0 ** -149), (torch.float32, 2.0 ** 121)])
@pytest.mark.parametrize("D", [127, 256])
def test_rows_of_the_smallest_and_the_largest_numbers(dtype, step, D):
    """Whole multiples of the type's smallest number (denormal), up to 127 of it, and of one next to its largest."""
    top = torch.arange(1, 128, dtype=torch.float64)[:, None]
    x = (torch.minimum(torch.arange(D, dtype=torch.float64)[None, :] % 127 + 1, top) * step).to(dtype)
    q, s = binding.tvm_attn_quantize_s8(x.cuda())
    assert np.array_equal(q.cpu().numpy(), np.rint(_steps(x)))
    # a scale below 2^-126 has fewer bits: within one of them
    assert (np.abs(s.cpu().double().numpy() - top[:, 0].numpy() * step / 127) <= np.maximum(top[:, 0].numpy() * step / 127 * 2.0 ** -24, 2.0 ** -149)).all()
    q8, _, _ = binding.tvm_attn_rmsnorm_s8(x.cuda(), eps=0.0)
    assert np.array_equal(q8.cpu().numpy(), np.rint(_steps(x)))
