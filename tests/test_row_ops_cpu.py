"""Refusals of the operators on rows, checked before any GPU work: at the C entry points, with pointers that are never followed,
and in the Python binding."""
import ctypes

import pytest
import torch

from paper_2511_19797_b200 import binding, build

OK, INVALID, UNSUPPORTED, SMALL = 0, -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _rows(k=0, row=0, batch=0, ptr=None):
    return ctypes.byref(binding.Rows(ptr if ptr is not None else 4096 + 256 * k, row, batch))


def _params(B=2, T=4, D=64, dtype=binding.BF16, eps=1e-6):
    return ctypes.byref(binding.RowsParams(B, T, D, dtype, eps))


def _fwd(lib, p=None, x=0, res=None, tx=None, tres=None, g=None, y=1, h=None, ty=None, th=None):
    a = [t if t is None or not isinstance(t, int) else _rows(t) for t in (x, res, tx, tres)]
    b = [t if t is None or not isinstance(t, int) else _rows(t) for t in (y, h, ty, th)]
    return lib.tvm_attn_rmsnorm_jvp_fwd(p or _params(), *a, g, *b, None)


@pytest.mark.parametrize("p", [dict(B=-1), dict(T=-1), dict(D=0), dict(dtype=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_bad_parameters(lib, p):
    assert _fwd(lib, _params(**p)) == INVALID
    assert lib.tvm_attn_rmsnorm_jvp_workspace_bytes(_params(**p)) == 0
    assert lib.tvm_attn_quantize_s8(_params(**p), _rows(0), _rows(1), 4096, None) == INVALID
    assert lib.tvm_attn_rmsnorm_s8(_params(**p), _rows(0), None, None, _rows(1), 4096, None, None) == INVALID
    assert lib.tvm_attn_rmsnorm_jvp_bwd(_params(**p), _rows(0), _rows(1), None, None, None, None, None, _rows(2), None, None, None, 0, None) == INVALID


def test_sizes_beyond_the_limits(lib):
    for p in (dict(D=16385), dict(B=1 << 16, T=1 << 15)):
        assert _fwd(lib, _params(**p)) == UNSUPPORTED
    assert _fwd(lib, None, x=None) == INVALID and lib.tvm_attn_rmsnorm_jvp_fwd(None, *[None] * 10) == INVALID


def test_outputs_and_inputs_that_do_not_belong_together(lib):
    for bad in (dict(y=None), dict(res=2), dict(h=2), dict(tx=2), dict(ty=2), dict(tres=2, th=3), dict(tx=2, ty=3, tres=4), dict(tx=2, ty=3, th=4)):
        assert _fwd(lib, **bad) == INVALID, bad
    def back(h=0, dy=1, dh=None, th=None, dty=None, dth=None, g=None, dx=2, dtx=None, dg=None, ws=None, size=0):
        a = [None if t is None else _rows(t) for t in (h, dy, dh, th, dty, dth)]
        return lib.tvm_attn_rmsnorm_jvp_bwd(_params(), *a, g, *[None if t is None else _rows(t) for t in (dx, dtx)], dg, ws, size, None)
    for bad in (dict(h=None), dict(dy=None), dict(dx=None), dict(th=3), dict(dty=3), dict(th=3, dty=4), dict(dtx=3), dict(dth=3), dict(g=4096), dict(dg=4096),
                dict(g=4096, dg=8192), dict(g=4096, dg=8192, ws=8200, size=1 << 30), dict(g=4096, dg=8194, ws=8192, size=1 << 30)):
        assert back(**bad) == INVALID, bad
    need = lib.tvm_attn_rmsnorm_jvp_workspace_bytes(_params())
    assert need >= 64 * 4 and back(g=4096, dg=8192, ws=16384, size=need - 1) == SMALL
    assert lib.tvm_attn_rmsnorm_s8(_params(), _rows(0), _rows(2), None, _rows(1), 4096, None, None) == INVALID      # a sum, and nowhere to put it
    assert lib.tvm_attn_rmsnorm_s8(_params(), _rows(0), None, None, _rows(1), None, None, None) == INVALID          # no scales
    assert lib.tvm_attn_quantize_s8(_params(), _rows(0), _rows(1), 4098, None) == INVALID                           # misaligned scales


@pytest.mark.parametrize("row,batch,ptr", [(63, 1000, 4096), (64, 63, 4096), (-64, 1000, 4096), (0, 64, 4096), (64, 0, 4096), (64, 256, 4097), (1 << 41, 1 << 42, 4096)])
def test_strides_and_pointers_of_rows(lib, row, batch, ptr):
    bad = _rows(row=row, batch=batch, ptr=ptr)
    assert lib.tvm_attn_rmsnorm_jvp_fwd(_params(), bad, None, None, None, None, _rows(1), None, None, None, None) == INVALID
    assert lib.tvm_attn_rmsnorm_jvp_fwd(_params(), _rows(1), None, None, None, None, bad, None, None, None, None) == INVALID
    assert lib.tvm_attn_quantize_s8(_params(), bad, _rows(1), 4096, None) == INVALID


def test_outputs_on_top_of_one_another_or_of_inputs_that_lie_differently(lib):
    def fwd(x, y, res=None, h=None):
        return lib.tvm_attn_rmsnorm_jvp_fwd(_params(), x, res, None, None, None, y, h, None, None, None)

    assert fwd(_rows(0), _rows(2), _rows(1), _rows(2)) == INVALID                    # y and h in one place
    assert fwd(_rows(0), _rows(0, row=128, batch=1024)) == INVALID                   # y over x, at other strides
    assert fwd(_rows(0), _rows(1, row=128, batch=1024), _rows(1), _rows(2)) == INVALID
    back = lambda dx, dtx: lib.tvm_attn_rmsnorm_jvp_bwd(_params(), _rows(0), _rows(1), None, _rows(2), _rows(3), None, None, dx, dtx, None, None, 0, None)  # noqa: E731
    assert back(_rows(4), _rows(4)) == INVALID and back(_rows(0, row=64, batch=512), _rows(4)) == INVALID
    assert lib.tvm_attn_quantize_s8(_params(), _rows(0), _rows(0), 4096, None) == INVALID
    assert lib.tvm_attn_rmsnorm_s8(_params(), _rows(0), _rows(1), None, _rows(1), 4096, _rows(2), None) == INVALID


def test_calls_without_rows_need_nothing(lib):
    for p in (dict(B=0), dict(T=0)):
        assert lib.tvm_attn_rmsnorm_jvp_fwd(_params(**p), *[None] * 10) == OK
        assert lib.tvm_attn_rmsnorm_s8(_params(**p), *[None] * 7) == OK and lib.tvm_attn_quantize_s8(_params(**p), *[None] * 4) == OK
        assert lib.tvm_attn_rmsnorm_jvp_bwd(_params(**p), *[None] * 11, 0, None) == OK
    assert lib.tvm_attn_linear_s8(ctypes.byref(binding.LinearParams(0, 8, 16, 0, 0, 0, 0)), *[None] * 7) == OK


def test_products(lib):
    good = dict(M=4, N=8, K=32, dtype=0, ldq=0, ldw=0, ldy=0)
    ptrs = [4096, 8192, 12288, 16384, None, 20480]

    def call(ptrs=ptrs, **p):
        return lib.tvm_attn_linear_s8(ctypes.byref(binding.LinearParams(**{**good, **p})), *ptrs, None)

    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(dtype=2), dict(ldq=16), dict(ldq=40), dict(ldw=31), dict(ldw=33), dict(K=33), dict(ldy=7), dict(ldq=-32)):
        assert call(**bad) == INVALID, bad
    assert call(K=65552) == UNSUPPORTED and call(ldq=1 << 40) == UNSUPPORTED
    for k, p in ((0, None), (0, 4104), (1, None), (1, 8194), (2, None), (2, 12296), (3, None), (3, 16386), (4, 4098), (5, None), (5, 20481)):
        assert call([p if i == k else v for i, v in enumerate(ptrs)]) == INVALID, (k, p)
    assert lib.tvm_attn_linear_s8(None, *ptrs, None) == INVALID


def test_binding_refuses_what_does_not_fit():
    x, f = torch.zeros(2, 3, 32, dtype=torch.bfloat16), torch.zeros(32)
    q, s = torch.zeros(2, 3, 32, dtype=torch.int8), torch.zeros(2, 3)
    w, ws = torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8)
    calls = [lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x), lambda: binding.tvm_attn_rmsnorm_jvp_bwd(x, x), lambda: binding.tvm_attn_rmsnorm_s8(x),
             lambda: binding.tvm_attn_quantize_s8(x), lambda: binding.tvm_attn_linear_s8(q, s, w, ws)]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="tangent"):
        binding.tvm_attn_rmsnorm_jvp_fwd(x, x, None, x)
    with pytest.raises(ValueError, match="together"):
        binding.tvm_attn_rmsnorm_jvp_bwd(x, x, x)
    with pytest.raises(ValueError, match="cotangent"):
        binding.tvm_attn_rmsnorm_jvp_bwd(x, x, dth=x)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        binding.tvm_attn_linear_s8(q, s, w, ws, dtype=torch.float16)
    with pytest.raises(ValueError, match="int8"):
        binding.tvm_attn_linear_s8(x, s, w, ws)
    with pytest.raises(ValueError, match="int8"):
        binding.tvm_attn_linear_s8(q[..., :16], s, w, ws)
    with pytest.raises(ValueError, match="torch.Tensor"):
        binding.tvm_attn_quantize_s8([1.0])
    assert binding.tvm_attn_rmsnorm_jvp_workspace_bytes(1152) % (1152 * 4) == 0 and binding.tvm_attn_rmsnorm_jvp_workspace_bytes(16385) == 0
