"""GPU parity of the operators on rows of the model width against the fp64 oracle on the same seeded inputs.

Bounds, for each element: half a step of the output's type relative to the value (bf16 2^-8, fp32 2^-24), and for the fp32 arithmetic
in between ROUNDINGS times 2^-24 of the sum of the magnitudes of the terms that the formula adds up (the oracle's `size`).  A row's
sums go over at most 40 elements a thread and 10 steps between threads, and enter a result as a factor, together with some ten more
operations: 64 roundings bound that.  The scale's gradient adds up to 15 rows a thread in the cases here, 20 rows within a block and 24 steps of the
reduction on top of its terms' own roundings: 128.
"""
import numpy as np
import pytest
import torch

from oracle import row_ops_numpy as orn
from paper_2511_19797_b200 import binding

pytestmark = pytest.mark.gpu

EPS = 1e-6
ULP = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: ULP}
DTYPES = [torch.bfloat16, torch.float32]


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _draw(seed, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=_gen(seed)) * std).to(dtype)


def _np(t):
    return None if t is None else t.detach().cpu().double().numpy()


def _close(got, want, roundings=64, what=""):
    value, size = want
    if value is None:
        assert got is None, what
        return
    err, bound = np.abs(_np(got) - value), HALF[got.dtype] * np.abs(value) + roundings * ULP * size + 1e-37
    assert got.shape == value.shape and not (err > bound).any() and np.isfinite(err).all(), (what, float((err / bound).max()))


def _dev(*ts):
    return [None if t is None else t.cuda() for t in ts]


def _fwd_case(shape, dtype, res, tan, tres, scale, seed, place=lambda t: t):
    x, r, t, tr = (_draw(seed + k, *shape, dtype=dtype, std=0.5 + 0.5 * k) for k in range(4))
    g = 1 + _draw(seed + 9, shape[-1], std=0.3) if scale else None
    r, t, tr = r if res else None, t if tan else None, tr if tres else None
    got = binding.tvm_attn_rmsnorm_jvp_fwd(*(None if v is None else place(v.cuda()) for v in (x, r, t, tr)), None if g is None else g.cuda(), eps=EPS)
    want = orn.rmsnorm_jvp_fwd(*map(_np, (x, r, t, tr, g)), EPS)
    for name, v in zip(("y", "h", "ty", "th"), got):
        _close(v, want[name], what=name)


# every split of a row over lanes and blocks, widths that are no multiple of a chunk, one row and many, widths of one element
WIDTHS = [1, 2, 5, 8, 16, 24, 40, 72, 100, 127, 128, 256, 333, 512, 768, 1000, 1024, 1151, 1152, 1280, 1288, 2048, 2303, 4096, 5000, 8192, 16384]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_norm_at_every_split_of_a_row(D, dtype):
    for rows in ((1,), (37,)) if D > 4096 else ((1,), (3, 67)):
        _fwd_case(rows + (D,), dtype, True, True, True, True, seed=D)
    _fwd_case((19, D), dtype, True, False, False, False, seed=D + 1)


@pytest.mark.parametrize("res,tan,tres", [(False, False, False), (True, False, False), (False, True, False), (True, True, False), (False, True, True), (True, True, True)])
@pytest.mark.parametrize("scale", [True, False])
def test_norm_with_every_set_of_inputs(res, tan, tres, scale):
    for dtype in DTYPES:
        _fwd_case((2, 45, 1152), dtype, res, tan, tres, scale, seed=5)
        _fwd_case((33, 77), dtype, res, tan, tres, scale, seed=6)


def test_norm_of_many_rows():
    _fwd_case((40001, 64), torch.bfloat16, True, True, True, True, seed=1)      # more rows than one sweep of the grid covers
    _fwd_case((9501, 2056), torch.bfloat16, True, False, False, True, seed=2)   # rows with a block each


def _bwd_case(shape, dtype, tan, dh, dth, scale, seed, place=lambda t: t, roundings=128):
    h, dy, t, dty, vh, vth = (_draw(seed + k, *shape, dtype=dtype) for k in range(6))
    g = 1 + _draw(seed + 9, shape[-1], std=0.3) if scale else None
    t, dty = (t, dty) if tan else (None, None)
    vh, vth = vh if dh else None, vth if dth else None
    got = binding.tvm_attn_rmsnorm_jvp_bwd(*(None if v is None else place(v.cuda()) for v in (h, dy, t, dty, vh, vth)), None if g is None else g.cuda(), eps=EPS)
    want = orn.rmsnorm_jvp_bwd(*map(_np, (h, dy, t, dty, vh, vth, g)), EPS)
    if not scale:
        want["dg"] = (None, None)
    for name, v in zip(("dx", "dtx", "dg"), got):
        _close(v, want[name], roundings if name == "dg" else 64, what=name)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_backward_at_every_split_of_a_row(D, dtype):
    for rows in ((1,), (37,)) if D > 4096 else ((1,), (3, 67)):
        _bwd_case(rows + (D,), dtype, True, True, True, True, seed=D)
    _bwd_case((19, D), dtype, False, False, False, True, seed=D + 1)


@pytest.mark.parametrize("tan,dh,dth", [(False, False, False), (False, True, False), (True, False, False), (True, True, False), (True, False, True), (True, True, True)])
@pytest.mark.parametrize("scale", [True, False])
def test_backward_with_every_set_of_inputs(tan, dh, dth, scale):
    for dtype in DTYPES:
        _bwd_case((2, 45, 1152), dtype, tan, dh, dth, scale, seed=5)
        _bwd_case((33, 77), dtype, tan, dh, dth, scale, seed=6)


def test_backward_of_many_rows():
    _bwd_case((5 * 1024, 1152), torch.bfloat16, True, True, True, True, seed=1)
    _bwd_case((2000, 2056), torch.bfloat16, True, False, False, True, seed=2)


def test_backward_against_differences():
    """The gradient of a scalar of all four outputs, by central differences of the fp32 forward along random directions."""
    shape, step = (6, 200), 2.0 ** -9
    x, res, tx, tres, dy, dty, dh, dth = (_draw(70 + k, *shape).cuda() for k in range(8))
    g = (1 + _draw(79, 200, std=0.3)).cuda()

    def loss(x, g, tx):
        y, h, ty, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, g, eps=1e-3)
        return sum((a.double() * b.double()).sum() for a, b in ((y, dy), (ty, dty), (h, dh), (th, dth)))

    _, h, _, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, g, eps=1e-3)
    grads = binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, dh, dth, g, eps=1e-3)
    for k, (at, d) in enumerate(zip((x, tx, g), grads)):
        way = torch.sign(_draw(90 + k, *at.shape)).cuda() * step
        ends = [(x + s * way if k == 0 else x, g + s * way if k == 2 else g, tx + s * way if k == 1 else tx) for s in (1, -1)]
        diff, want = float(loss(*ends[0]) - loss(*ends[1])) / 2, float((d.double() * way.double()).sum())
        # third-order term: elements move by 2^-9 of rows with unit rms; fp32 evaluations of 1200 terms of order 1 each
        assert abs(diff - want) <= 1200 * step ** 3 * 16 + 64 * ULP * 1200 * 8, (k, diff, want)


def _placements():
    def padded(t):      # rows with a gap, which starts on 16 bytes or not
        buf = torch.full(t.shape[:-1] + (t.shape[-1] + 24,), 7.0, dtype=t.dtype, device=t.device)
        buf[..., 8:-16] = t
        return buf[..., 8:-16]

    def odd(t):
        buf = torch.full(t.shape[:-1] + (t.shape[-1] + 3,), 7.0, dtype=t.dtype, device=t.device)
        buf[..., 1:-2] = t
        return buf[..., 1:-2]

    def cut(t):         # rows 1.. of longer batches: two strides
        buf = torch.full((t.shape[0], t.shape[1] + 2, t.shape[2]), 7.0, dtype=t.dtype, device=t.device)
        buf[:, 1:-1] = t
        return buf[:, 1:-1]

    def swapped(t):     # (T, B, D) in memory
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    return {"padded": padded, "odd": odd, "cut": cut, "swapped": swapped}


@pytest.mark.parametrize("how", ["padded", "odd", "cut", "swapped"])
@pytest.mark.parametrize("D", [72, 1152, 2560])
def test_rows_in_place(how, D):
    place = _placements()[how]
    _fwd_case((3, 21, D), torch.bfloat16, True, True, True, True, seed=3, place=place)
    _bwd_case((3, 21, D), torch.bfloat16, True, True, True, True, seed=4, place=place)
    x, res = (_draw(5 + k, 3, 21, D, dtype=torch.bfloat16).cuda() for k in range(2))
    q, s, h = binding.tvm_attn_rmsnorm_s8(place(x), place(res), eps=EPS)
    want = orn.rmsnorm_jvp_fwd(_np(x), _np(res), None, None, None, EPS)
    _check_8_bits(q, s, want["y"][0])
    _close(h, want["h"])


def test_outputs_given_strided_and_in_place():
    shape, place = (3, 21, 1152), _placements()
    x, res, tx, tres = (_draw(20 + k, *shape, dtype=torch.bfloat16).cuda() for k in range(4))
    want = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres)
    outs = [place["cut"](torch.zeros_like(x)) for _ in range(4)]
    got = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, out=outs)
    for a, b, o in zip(got, want, outs):
        assert a is o and torch.equal(a, b)
        rest = o._base.clone()
        rest[:, 1:-1] = 7.0
        assert (rest == 7.0).all()        # what lies around the rows is left as it was
    # the sums over the residual stream, the norms over what came in
    a, r, t, tr = x.clone(), res.clone(), tx.clone(), tres.clone()
    for v, w in zip(binding.tvm_attn_rmsnorm_jvp_fwd(a, r, t, tr, out=(a, r, t, tr)), want):
        assert torch.equal(v, w)
    h, dy, th, dty, dh, dth = (_draw(30 + k, *shape, dtype=torch.bfloat16).cuda() for k in range(6))
    want = binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, dh, dth)
    got = binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, dh, dth, out=(dh, dth, None))
    assert got[0] is dh and got[1] is dth and torch.equal(dh, want[0]) and torch.equal(dth, want[1])


def test_gradients_of_the_scale_are_bit_reproducible():
    h, dy, th, dty = (_draw(40 + k, 3000, 1152, dtype=torch.bfloat16).cuda() for k in range(4))
    g = torch.ones(1152, device="cuda")
    runs = [binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, g=g)[2] for _ in range(3)]
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 1152, 1151, 4096])
def test_norm_of_rows_whose_squares_leave_the_range(D, dtype):
    """1e-30 to 1e30, next to ordinary rows of the same warp; without eps the tiny ones are normalised like all others."""
    x = _draw(1, 12, D).double() * torch.tensor([1.0, 1e30, 1e-30, 1e20, 1.0, 1e-25, 3.0, 1e25, 1e-10, 1e10, 1.0, 1e-20])[:, None]
    x = x.to(dtype)
    for eps in (0.0, 1e-6):
        (y, _, _, _), want = binding.tvm_attn_rmsnorm_jvp_fwd(x.cuda(), eps=eps), orn.rmsnorm_jvp_fwd(_np(x), None, None, None, None, eps)["y"]
        _close(y, want)
        q, s, _ = binding.tvm_attn_rmsnorm_s8(x.cuda(), eps=eps)
        _check_8_bits(q, s, want[0])
        dx, _, _ = binding.tvm_attn_rmsnorm_jvp_bwd(x[:, :].cuda(), torch.zeros_like(x).cuda(), eps=eps)
        assert not dx.any()


def test_empty_calls():
    g = torch.ones(64, device="cuda")
    for shape in ((0, 64), (3, 0, 64), (0, 5, 64)):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        y, h, ty, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, x, x, x, g)
        assert y.shape == h.shape == ty.shape == th.shape == x.shape
        dx, dtx, dg = binding.tvm_attn_rmsnorm_jvp_bwd(x, x, x, x, x, x, g)
        assert dx.shape == dtx.shape == x.shape and dg.shape == (64,) and not dg.any()
        q, s = binding.tvm_attn_quantize_s8(x)
        assert q.shape == x.shape and s.shape == x.shape[:-1]
        w = torch.ones(8, 64, dtype=torch.int8, device="cuda")
        assert binding.tvm_attn_linear_s8(q, s, w, torch.ones(8, device="cuda")).shape == x.shape[:-1] + (8,)


# ---------------------------------------------------------------- 8-bit rows
def _check_8_bits(q, s, v):
    """v: what the rows stand for, in 64 bits.  The scale is fp32 arithmetic on a row's maximum; a value is within half a step of
    what it stands for, but for the roundings of its quotient, which is at most 127."""
    want_s, steps = orn.rows_to_8_bits(v)
    assert (np.abs(_np(s) - want_s) <= 64 * ULP * want_s + 1e-44).all()
    assert (np.abs(_np(q) - steps) <= 0.5 + 64 * ULP * 127).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_rows_in_8_bits(D, dtype):
    x, res = (_draw(D + k, 2, 9, D, dtype=dtype) for k in range(2))
    g = 1 + _draw(D + 9, D, std=0.3)
    q, s = binding.tvm_attn_quantize_s8(x.cuda())
    _check_8_bits(q, s, _np(x))
    assert q.stride(-2) % 16 == 0 and q.data_ptr() % 16 == 0
    for r, scale in ((res, g), (None, g), (res, None)):
        q, s, h = binding.tvm_attn_rmsnorm_s8(x.cuda(), *_dev(r, scale), eps=EPS)
        want = orn.rmsnorm_jvp_fwd(_np(x), _np(r), None, None, _np(scale), EPS)
        _check_8_bits(q, s, want["y"][0])
        _close(h, want["h"])


def test_rows_in_8_bits_with_nothing_in_them_and_with_what_no_scale_holds():
    x = _draw(3, 6, 300)
    x[1] = 0.0
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    x[4] *= 1e-38
    x[5, 0] = float("-inf")
    for cols in (300, 296):
        v = x[:, :cols].contiguous().cuda()
        bad = [row for row in (2, 3, 5) if not torch.isfinite(v[row]).all()]     # (the NaN stands behind the 296th element)
        for q, s in (binding.tvm_attn_quantize_s8(v), binding.tvm_attn_rmsnorm_s8(v, eps=1e-30)[:2]):
            assert s[1] == 0 and not q[1].any()
            for row in bad:
                assert not torch.isfinite(s[row]) and not q[row].any()
            assert torch.isfinite(s[[0, 1, 4]]).all() and q[0].abs().max() == 127 and q[4].abs().max() == 127
        w = torch.ones(16, cols, dtype=torch.int8, device="cuda")
        wq, _ = binding.tvm_attn_quantize_s8(w.float())
        y = binding.tvm_attn_linear_s8(q, s, wq, torch.ones(16, device="cuda"))
        assert torch.isfinite(y[[0, 1, 4]]).all() and not torch.isfinite(y[bad]).any()


def test_8_bit_outputs_given():
    x = _draw(4, 5, 100, dtype=torch.bfloat16).cuda()
    q, s = binding.tvm_attn_quantize_s8(x)
    buf, scales = torch.full((5, 103), 9, dtype=torch.int8, device="cuda"), torch.empty(5, device="cuda")
    got = binding.tvm_attn_quantize_s8(x, out=(buf[:, 1:101], scales))
    assert torch.equal(got[0], q) and torch.equal(scales, s) and (buf[:, 0] == 9).all() and (buf[:, 101:] == 9).all()


# ---------------------------------------------------------------- products
def _rows8(seed, rows, K, lo=-128):
    q = torch.randint(lo, 128, (rows, K), generator=_gen(seed), dtype=torch.int64).to(torch.int8)
    pitch = (K + 15) // 16 * 16
    buf = torch.full((rows, pitch), 77, dtype=torch.int8, device="cuda")     # what lies behind a row does not count
    buf[:, :K] = q.cuda()
    return q, buf[:, :K]


def _linear_case(M, N, K, dtype, bias, seed=0, out=None):
    q, dq = _rows8(seed + 1, M, K)
    w, dw = _rows8(seed + 2, N, K)
    s, ws = _draw(seed + 3, M).abs() * 1e-2, _draw(seed + 4, N).abs() * 1e-2
    b = _draw(seed + 5, N) if bias else None
    got = binding.tvm_attn_linear_s8(dq, s.cuda(), dw, ws.cuda(), None if b is None else b.cuda(), dtype=dtype, out=out)
    # four roundings: of the sum to fp32, of its products with the two scales, of the sum with the bias
    _close(got, orn.linear_s8(q.numpy(), _np(s), w.numpy(), _np(ws), _np(b)), roundings=4)
    binding.tvm_attn_check_status()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 1, 16), (1, 17, 100), (2, 16, 64), (3, 31, 33), (7, 250, 1152), (8, 768, 768), (9, 40, 15), (16, 100, 300), (17, 129, 4096),
                                   (32, 64, 640), (33, 1152, 128), (63, 70, 47), (64, 512, 2048), (1, 4608, 1152), (5, 33, 8200)])
def test_products_of_few_rows(M, N, K, dtype):
    _linear_case(M, N, K, dtype, bias=True, seed=M + N + K)
    _linear_case(M, N, K, dtype, bias=False, seed=M + N)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(65, 1, 1), (65, 8, 16), (128, 64, 128), (129, 65, 127), (200, 128, 129), (256, 256, 1152), (257, 257, 300), (300, 1000, 333), (512, 96, 64), (77, 192, 4096),
                                   (1000, 333, 768), (2048, 3456, 1152), (4099, 640, 257), (640, 4097, 160)])
def test_products_of_many_rows(M, N, K, dtype):
    _linear_case(M, N, K, dtype, bias=True, seed=M + N + K)
    _linear_case(M, N, K, dtype, bias=False, seed=M + N)


@pytest.mark.parametrize("M", [3, 200])
def test_products_of_extreme_values_are_exact(M):
    """Sums up to 65536 x 2^14 = 2^30, where fp32 sums would not be whole numbers."""
    K, N = 65536, 48
    q, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    q[1, ::2], w[1, :] = 127, 127
    y = binding.tvm_attn_linear_s8(q.cuda(), torch.ones(M, device="cuda"), w.cuda(), torch.ones(N, device="cuda"), dtype=torch.float32)
    assert torch.equal(y.cpu().double(), (q.double() @ w.double().t()).float().double())


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("dtype", DTYPES)
def test_products_into_given_rows(M, dtype):
    for N, pad, at in ((64, 8, 0), (100, 28, 4), (33, 2, 1)):     # rows that begin on 16 bytes, and rows that do not
        buf = torch.full((M + 2, N + pad), 7.0, dtype=dtype, device="cuda")
        out = buf[1 : M + 1, at : at + N]
        _linear_case(M, N, 200, dtype, True, out=out)
        out.fill_(7.0)
        assert (buf == 7.0).all()                                  # nothing was written around them


def _linear_on_gpu(q, s, w, ws, bias):
    """The definition in 64 bits (whole numbers below 2^53 are exact in a 64-bit product of matrices), and the size of its terms."""
    y = (q.double() @ w.double().t()) * s.double()[:, None] * ws.double()
    b = torch.zeros_like(ws) if bias is None else bias
    return (y + b.double()).cpu().numpy(), (y.abs() + b.double().abs()).cpu().numpy()


# every number of CTAs that share k, tiles of 16 to 256 tokens, every width of a tile of channels, several tiles a pair
@pytest.mark.parametrize("M,N,K", [(3, 14336, 4096), (16, 2000, 1024), (17, 9000, 896), (31, 130, 385), (40, 1152, 4608), (63, 7000, 520), (65, 768, 2304), (100, 640, 8192), (128, 128, 128),
                                   (130, 333, 5000), (200, 1280, 6144), (255, 96, 4100), (256, 4608, 1152), (300, 4224, 768), (1000, 8200, 136), (5000, 3456, 1152), (9472, 2056, 300), (20000, 200, 64)])
def test_products_of_every_kind(M, N, K):
    for dtype in DTYPES:
        (_, q), (_, w) = _rows8(M, M, K), _rows8(N, N, K)
        s, ws, b = (_draw(K + 3, M).abs() * 1e-2).cuda(), (_draw(K + 4, N).abs() * 1e-2).cuda(), _draw(K + 5, N).cuda()
        _close(binding.tvm_attn_linear_s8(q, s, w, ws, b, dtype=dtype), _linear_on_gpu(q, s, w, ws, b), roundings=4)
    binding.tvm_attn_check_status()


def test_products_of_drawn_sizes():
    rng = np.random.default_rng(11)
    for i in range(60):
        M, N, K = (int(round(np.exp(rng.uniform(np.log(lo), np.log(hi))))) for lo, hi in ((1, 3000), (1, 5000), (1, 6000)))
        dtype, bias = DTYPES[i % 2], bool(rng.integers(2))
        (_, q), (_, w) = _rows8(i, M, K), _rows8(i + 100, N, K)
        s, ws, b = (_draw(i, M).abs() * 1e-2).cuda(), (_draw(i + 1, N).abs() * 1e-2).cuda(), _draw(i + 2, N).cuda() if bias else None
        got, (value, size) = binding.tvm_attn_linear_s8(q, s, w, ws, b, dtype=dtype), _linear_on_gpu(q, s, w, ws, b)
        _close(got, (value, size), roundings=4, what=(M, N, K, dtype, bias))


@pytest.mark.parametrize("M", [2, 70, 300])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N", [1, 7, 61, 101, 250])
def test_products_into_rows_on_16_bytes_with_a_ragged_end(M, dtype, N):
    """Rows of any length whose starts lie on 16 bytes: what lies behind them is left as it was."""
    buf = torch.full((M + 2, 512), 7.0, dtype=dtype, device="cuda")
    out = buf[1 : M + 1, 8 : 8 + N]
    _linear_case(M, N, 200, dtype, True, out=out)
    out.fill_(7.0)
    assert (buf == 7.0).all()


@pytest.mark.parametrize("M", [2, 33, 300])
def test_product_outputs_far_apart(M):
    N, K = 40, 64
    gap = ((1 << 32) // (M - 1) + 64) // 16 * 16       # the last row lies beyond 2^32 elements
    buf = torch.empty(gap * (M - 1) + 64, dtype=torch.bfloat16, device="cuda")
    _linear_case(M, N, K, torch.bfloat16, True, out=buf.as_strided((M, N), (gap, 1), 0))


def test_products_do_nothing_after_a_time_out_until_it_is_reported():
    (_, q), (_, w) = _rows8(1, 300, 64), _rows8(2, 40, 64)
    s, ws = torch.ones(300, device="cuda"), torch.ones(40, device="cuda")
    want = binding.tvm_attn_linear_s8(q, s, w, ws)
    for M in (300, 20):
        y = torch.full((M, 40), 7.0, dtype=torch.bfloat16, device="cuda")
        binding.tvm_attn_selftest_timeout(1_000_000)
        binding.tvm_attn_linear_s8(q[:M], s[:M], w, ws, out=y)
        with pytest.raises(binding.TvmAttnError, match="DEVICE_TIMEOUT"):
            binding.tvm_attn_check_status()
        assert (y == 7.0).all()
        assert torch.equal(binding.tvm_attn_linear_s8(q[:M], s[:M], w, ws), want[:M])


def test_product_shapes_and_strides():
    q, s = binding.tvm_attn_quantize_s8(_draw(1, 2, 3, 5, 48).cuda())
    w, ws = binding.tvm_attn_quantize_s8(_draw(2, 40, 48).cuda())
    y = binding.tvm_attn_linear_s8(q, s, w, ws)
    assert y.shape == (2, 3, 5, 40) and torch.equal(y.reshape(30, 40), binding.tvm_attn_linear_s8(q.reshape(30, 48), s.reshape(30), w, ws))
    one = binding.tvm_attn_linear_s8(q[0, 0, 0], s[0, 0, 0], w, ws)
    assert one.shape == (40,) and torch.equal(one, y[0, 0, 0])
    part = binding.tvm_attn_linear_s8(q.reshape(30, 48)[::3], s.reshape(30)[::3].contiguous(), w[::2], ws[::2].contiguous())
    assert torch.equal(part, y.reshape(30, 40)[::3, ::2])


def test_refusals():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(64, device="cuda")
    for bad in (lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, x.float()), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, x[:2]), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x.half()),
                lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, g=f.bfloat16()), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, g=f[:32]), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, g=f.cpu()),
                lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x.t()), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x[:1].expand(4, 64)),
                lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, out=(x, x, None, None)), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, out=(None, None, None, None)),
                lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, out=(x,)), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x[:, :0]),
                lambda: binding.tvm_attn_rmsnorm_jvp_bwd(x, x, g=f, out=(x, None, None)), lambda: binding.tvm_attn_rmsnorm_jvp_bwd(x, x, out=(x, None, f)),
                lambda: binding.tvm_attn_quantize_s8(x, out=(x, f[:4])), lambda: binding.tvm_attn_quantize_s8(x, out=(x.to(torch.int8), f[:3])),
                lambda: binding.tvm_attn_rmsnorm_jvp_fwd(torch.zeros(3, 5, 3, 128, dtype=torch.bfloat16, device="cuda")[:, ::2, ::2, :64])):
        with pytest.raises(ValueError):
            bad()
    q, s, w, ws = x.to(torch.int8), f[:4], torch.zeros(8, 64, dtype=torch.int8, device="cuda"), f[:8]
    for bad in (lambda: binding.tvm_attn_linear_s8(q, f[:3], w, ws), lambda: binding.tvm_attn_linear_s8(q, s, w, f[:7]), lambda: binding.tvm_attn_linear_s8(q, s, w, ws, f[:7]),
                lambda: binding.tvm_attn_linear_s8(q, s, w[:, :32], ws), lambda: binding.tvm_attn_linear_s8(q, s, w.cpu(), ws), lambda: binding.tvm_attn_linear_s8(q, s.double(), w, ws),
                lambda: binding.tvm_attn_linear_s8(q, s, w, ws, out=x[:, :8].float()), lambda: binding.tvm_attn_linear_s8(q, s, w, ws, out=x[:, :7])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: binding.tvm_attn_rmsnorm_jvp_fwd(x, eps=-1.0), lambda: binding.tvm_attn_rmsnorm_jvp_fwd(torch.zeros(1, 16385, device="cuda")),
                lambda: binding.tvm_attn_rmsnorm_jvp_bwd(x, x, g=f, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
                lambda: binding.tvm_attn_linear_s8(q[:, 1:33], s, w[:, 1:33], ws), lambda: binding.tvm_attn_linear_s8(q[:, :33].contiguous(), s, w[:, :33].contiguous(), ws)):
        with pytest.raises(binding.TvmAttnError):
            bad()


# ---------------------------------------------------------------- together
def _block(x, res, tx, tres, w, g, heads):
    """Norm in front of an attention layer of bf16 weights, with tangents: y, h, then attention of the fused projection."""
    B, T, D = x.shape
    y, h, ty, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, g)
    qkv, tqkv = ((v @ w.t()).reshape(B, T, 3, heads, D // heads).permute(2, 0, 3, 1, 4) for v in (y, ty))
    return h, th, binding.tvm_attn_jvp_fwd(*qkv, *tqkv)[:2]


def test_norm_feeds_the_attention_with_its_tangent():
    """The tangent that comes out of norm, projection and attention is the directional derivative of the primal."""
    B, T, D, heads = 2, 40, 64, 2
    x, res, tx, tres = (_draw(50 + k, B, T, D).cuda() for k in range(4))
    w, g, step = _draw(55, 3 * D, D, std=D ** -0.5).cuda(), (1 + _draw(56, D, std=0.2)).cuda(), 2.0 ** -7
    _, _, (_, tO) = _block(x, res, tx, tres, w, g, heads)
    ends = [_block(x + s * step * tx, res + s * step * tres, tx, tres, w, g, heads)[2][0].double() for s in (1, -1)]
    diff = (ends[0] - ends[1]) / (2 * step)
    # second order: step^2 times third derivatives of order ten; fp32 results divided by the step
    assert float((diff - tO.double()).abs().max()) <= 40 * step ** 2 + 256 * ULP / step


def test_sampler_block_in_8_bits():
    """Residual, norm, 8 bits, fused QKV projection, attention, 8 bits, output projection: against the same chain in 64 bits of the
    same 8-bit values where the attention's inputs are equal, and against an unquantised chain for the size of the whole."""
    B, T, heads, d = 2, 130, 4, 72
    D = heads * d
    x, res = (_draw(60 + k, B, T, D, dtype=torch.bfloat16).cuda() for k in range(2))
    W, Wo = _draw(62, 3 * D, D, std=D ** -0.5).cuda(), _draw(63, D, D, std=D ** -0.5).cuda()
    (wq, ws), (oq, os_) = binding.tvm_attn_quantize_s8(W), binding.tvm_attn_quantize_s8(Wo)
    q, s, h = binding.tvm_attn_rmsnorm_s8(x, res)
    qkv = binding.tvm_attn_linear_s8(q, s, wq, ws)
    exact = (q.double() * s.double()[..., None]) @ (wq.double() * ws.double()[:, None]).t()
    assert float(((qkv.double() - exact).abs() / (exact.abs() * 2.0 ** -8 + 2.0 ** -20)).max()) <= 1.0
    Q, K, V = qkv.reshape(B, T, 3, heads, d).permute(2, 0, 3, 1, 4)         # slices of the projection, read in place
    zero = torch.zeros_like(qkv).reshape(B, T, 3, heads, d).permute(2, 0, 3, 1, 4)
    O = binding.tvm_attn_jvp_fwd(Q, K, V, *zero, out=None)[0]
    o8, so = binding.tvm_attn_quantize_s8(O.permute(0, 2, 1, 3).reshape(B, T, D))
    y = binding.tvm_attn_linear_s8(o8, so, oq, os_)
    hd = x.double() + res.double()
    u = hd / (hd.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    Qd, Kd, Vd = (u @ W.double().t()).reshape(B, T, 3, heads, d).permute(2, 0, 3, 1, 4)
    Od = torch.softmax(Qd @ Kd.transpose(-1, -2) * d ** -0.5, -1) @ Vd
    yd = Od.permute(0, 2, 1, 3).reshape(B, T, D) @ Wo.double().t()
    # steps of 1/127 of a row's largest element (some 3 to 4 times its rms), uniform errors of 1/sqrt(12) steps: 1 % a quantised operand
    assert float((y.double() - yd).norm() / yd.norm()) <= 0.05
    assert torch.equal(h, (x.float() + res.float()).bfloat16())
    binding.tvm_attn_check_status()


# ---------------------------------------------------------------- streams, graphs
def _everything(x, res, w, ws, g):
    y, h, ty, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, res, x, g)
    dx, dtx, dg = binding.tvm_attn_rmsnorm_jvp_bwd(h, y, th, ty, y, ty, g)
    q, s, _ = binding.tvm_attn_rmsnorm_s8(x, res, g)
    a, sa = binding.tvm_attn_quantize_s8(y)
    return y, h, ty, th, dx, dtx, dg, s, binding.tvm_attn_linear_s8(q, s, w, ws), binding.tvm_attn_linear_s8(a[:7], sa[:7], w, ws, dtype=torch.float32)


def _graph_inputs():
    x, res = (_draw(80 + k, 700, 1152, dtype=torch.bfloat16).cuda() for k in range(2))
    w, ws = binding.tvm_attn_quantize_s8(_draw(82, 500, 1152).cuda())
    return x, res, w, ws, (1 + _draw(83, 1152, std=0.2)).cuda()


def test_captured_calls_replay_bit_for_bit():
    args = _graph_inputs()
    want = _everything(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _everything(*args)
    for shift in (0, 1):
        if shift:
            args[0].copy_(args[0].roll(1, 0))
            want = _everything(*args)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_calls_in_a_row_wait_for_one_another():
    """Kernels are set up while the one in front of them ends: the same buffers written and read by call after call."""
    w, ws = binding.tvm_attn_quantize_s8(_draw(90, 640, 1152).cuda())
    for rows in (1, 2, 5, 100, 3000):
        xs = [_draw(91 + k, rows, 1152, dtype=torch.bfloat16).cuda() for k in range(4)]
        want = []
        for x in xs:
            q, s, h = binding.tvm_attn_rmsnorm_s8(x, xs[0])
            torch.cuda.synchronize()
            want.append((h, binding.tvm_attn_linear_s8(q, s, w, ws)))
            torch.cuda.synchronize()
        q, s, h = binding.tvm_attn_rmsnorm_s8(xs[0], xs[0])
        y = torch.empty(rows, 640, dtype=torch.bfloat16, device="cuda")
        got = []
        for i in range(24):
            binding.tvm_attn_rmsnorm_s8(xs[i % 4], xs[0], out=(q, s, h))
            binding.tvm_attn_linear_s8(q, s, w, ws, out=y)
            got.append((h.clone(), y.clone()))
        for i, (a, b) in enumerate(got):
            assert torch.equal(a, want[i % 4][0]) and torch.equal(b, want[i % 4][1]), (rows, i)


def test_calls_on_other_streams():
    args = _graph_inputs()
    want = _everything(*args)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for st in streams:      # at the same time
            with torch.cuda.stream(st):
                got.append(_everything(*args))
        torch.cuda.synchronize()
        for g in got:
            for a, b in zip(g, want):
                assert torch.equal(a, b)
    y, h, _, _ = binding.tvm_attn_rmsnorm_jvp_fwd(args[0], args[1], g=args[4], stream=streams[0])
    q, s = binding.tvm_attn_quantize_s8(y, stream=streams[0])
    z = binding.tvm_attn_linear_s8(q, s, args[2], args[3], stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, binding.tvm_attn_linear_s8(*binding.tvm_attn_quantize_s8(want[0]), args[2], args[3]))


@pytest.mark.parametrize("M", [1, 5000])
def test_offsets_beyond_32_bits(M):
    """Rows so far apart that element offsets pass 2^32 (the rows of one call span 4 GB and more)."""
    K, N = 64, 32
    gap = (1 << 33) // (M if M > 1 else 1)
    gap -= gap % 16
    buf = torch.empty((1 << 33) + 4096, dtype=torch.int8, device="cuda")
    q = buf.as_strided((M, K), (gap, 1), 0) if M > 1 else buf.as_strided((2, K), (1 << 32, 1), 0)
    v = _rows8(1, q.shape[0], K)[1]
    q.copy_(v)
    s = torch.ones(q.shape[0], device="cuda")
    w, dw = _rows8(2, N, K)
    assert torch.equal(binding.tvm_attn_linear_s8(q, s, dw, torch.ones(N, device="cuda")), binding.tvm_attn_linear_s8(v, s, dw, torch.ones(N, device="cuda")))
    far = buf.view(torch.bfloat16).as_strided((q.shape[0], K), (gap // 2 if M > 1 else 1 << 31, 1), 0)
    x = _draw(3, q.shape[0], K, dtype=torch.bfloat16).cuda()
    far.copy_(x)
    assert torch.equal(binding.tvm_attn_rmsnorm_jvp_fwd(far)[0], binding.tvm_attn_rmsnorm_jvp_fwd(x)[0])


def test_backward_of_rows_beyond_32_bits():
    """Two rows 4 GB apart, in all tensors or in some of them."""
    D = 1152
    buf = torch.empty((1 << 31) + 16 * D, dtype=torch.bfloat16, device="cuda")
    near = [_draw(100 + k, 2, D, dtype=torch.bfloat16).cuda() for k in range(6)]
    g = (1 + _draw(110, D, std=0.2)).cuda()
    want = binding.tvm_attn_rmsnorm_jvp_bwd(*near, g)
    far = [buf.as_strided((2, D), (1 << 31, 1), k * D) for k in range(8)]
    for f, n in zip(far, near):
        f.copy_(n)
    for some in ((0, 1, 2, 3, 4, 5), (1,), (0, 3)):
        got = binding.tvm_attn_rmsnorm_jvp_bwd(*(far[k] if k in some else near[k] for k in range(6)), g)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    dg = torch.empty_like(g)
    got = binding.tvm_attn_rmsnorm_jvp_bwd(*far[:6], g, out=(far[6], far[7], dg))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_calls_from_several_threads_next_to_the_attention():
    """Host threads with a stream each: norms and products of every kind, and attention, whose kernels take the same tensor memory."""
    import threading
    args = _graph_inputs()
    Q, K, V, tQ, tK, tV = (_draw(120 + k, 2, 4, 600, 64, dtype=torch.bfloat16).cuda() for k in range(6))

    def attention():
        saved = binding.tvm_attn_jvp_fwd(Q, K, V, tQ, tK, tV)
        return tuple(saved) + tuple(binding.tvm_attn_jvp_bwd(Q, K, V, tQ, tK, tV, *saved, Q, tQ))

    def products():
        q, s = binding.tvm_attn_quantize_s8(args[0])
        return tuple(binding.tvm_attn_linear_s8(q[:m], s[:m], args[2], args[3]) for m in (1, 2, 16, 60, 130, 250, 700))

    jobs = [attention, products, lambda: _everything(*args), products]
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = jobs[i]()
                torch.cuda.current_stream().synchronize()
                wrong.extend((i, k) for k, (a, b) in enumerate(zip(got, want[i])) if not torch.equal(a, b))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong[:5]
    binding.tvm_attn_check_status()


def test_a_first_call_under_capture():
    """A kernel's first launch may come inside a capture: shapes that no test before has used choose their kernels there."""
    (_, q), (_, w) = _rows8(1, 500, 272), _rows8(2, 330, 272)
    s, ws, x = torch.ones(500, device="cuda"), torch.ones(330, device="cuda"), _draw(3, 90, 2600, dtype=torch.bfloat16).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [binding.tvm_attn_linear_s8(q[:m], s[:m], w, ws, dtype=torch.float32) for m in (1, 30, 500)] + [binding.tvm_attn_rmsnorm_jvp_bwd(x, x, x, x)[0]]
    graph.replay()
    torch.cuda.synchronize()
    want = [binding.tvm_attn_linear_s8(q[:m], s[:m], w, ws, dtype=torch.float32) for m in (1, 30, 500)] + [binding.tvm_attn_rmsnorm_jvp_bwd(x, x, x, x)[0]]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [72, 333, 1152, 2560, 8192, 16384])
def test_in_place_at_every_split_of_a_row(D, dtype):
    """Outputs over each of the inputs in turn, several rows a block."""
    rows, g = 1500 if D < 3000 else 300, (1 + _draw(9, D, std=0.2)).cuda()
    src = [_draw(130 + k, rows, D, dtype=dtype).cuda() for k in range(6)]
    want = binding.tvm_attn_rmsnorm_jvp_bwd(*src, g)
    for a, b in ((0, 2), (1, 3), (2, 0), (4, 5), (5, 4), (3, 1)):
        t = [v.clone() for v in src]
        got = binding.tvm_attn_rmsnorm_jvp_bwd(*t, g, out=(t[a], t[b], torch.empty_like(g)))
        assert all(torch.equal(x, y) for x, y in zip(got, want)), (a, b)
    want = binding.tvm_attn_rmsnorm_jvp_fwd(*src[:4], g)
    for order in ((0, 1, 2, 3), (3, 2, 1, 0), (1, 0, 3, 2), (2, 3, 0, 1)):
        t = [v.clone() for v in src[:4]]
        got = binding.tvm_attn_rmsnorm_jvp_fwd(*t, g, out=[t[k] for k in order])
        assert all(torch.equal(x, y) for x, y in zip(got, want)), order
    q, s, h = binding.tvm_attn_rmsnorm_s8(*src[:2], g)
    t = [v.clone() for v in src[:2]]
    got = binding.tvm_attn_rmsnorm_s8(*t, g, out=(torch.empty_like(q), torch.empty_like(s), t[0]))
    assert torch.equal(got[0], q) and torch.equal(got[1], s) and torch.equal(t[0], h)
