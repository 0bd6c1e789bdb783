"""Dependent launches without anything between them: a kernel is set up while the one in front of it ends, so every buffer that two calls share is written
behind a reader, read behind a writer and written behind a writer here, by each kind of kernel, in a stream and in a replayed graph."""
import pytest
import torch

from paper_2511_19797_b200 import binding
from tests.test_row_ops_gpu import _draw

pytestmark = pytest.mark.gpu


def _alone(call):
    """The call with nothing in flight in front of it, on a copy of its result's memory."""
    torch.cuda.synchronize()
    r = [t.clone() for t in call() if t is not None]
    torch.cuda.synchronize()
    return r


def _both(enqueue):
    """Runs `enqueue` in the current stream, then twice as a graph; the results of each."""
    got = enqueue()
    torch.cuda.synchronize()
    yield got
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = enqueue()
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        yield got


# products of one and two tokens, of few on clusters, of many on pairs of CTAs; rows on warps and with a block each
@pytest.mark.parametrize("rows,D,N", [(1, 1152, 640), (2, 96, 640), (5, 1152, 640), (100, 1152, 1000), (250, 4096, 520), (3000, 1152, 640), (3000, 200, 333)])
def test_8_bit_rows_and_products_over_the_same_buffers(rows, D, N):
    w, ws = binding.tvm_attn_quantize_s8(_draw(1, N, D).cuda())
    xs = [_draw(2 + k, rows, D, dtype=torch.bfloat16).cuda() for k in range(4)]
    q, s = binding.tvm_attn_quantize_s8(xs[0])
    h, last = torch.empty_like(xs[0]), torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    ys = [torch.empty(rows, N, dtype=torch.bfloat16, device="cuda") for _ in range(16)]

    def step(i, y):
        binding.tvm_attn_rmsnorm_s8(xs[i % 4], xs[(i + 1) % 4], out=(q, s, h))
        return h, binding.tvm_attn_linear_s8(q, s, w, ws, out=y)

    want = [_alone(lambda: step(i, last))[1] for i in range(4)]

    def enqueue():
        for i in range(len(ys)):
            step(i, last)                                       # a product over the one before
            binding.tvm_attn_linear_s8(q, s, w, ws, out=ys[i])  # the next norm writes q, s and h that this one reads
        return ys + [last]

    for got in _both(enqueue):
        for i, y in enumerate(got):
            assert torch.equal(y, want[min(i, len(ys) - 1) % 4]), i


@pytest.mark.parametrize("rows,D,dtype", [(1, 1152, torch.bfloat16), (40, 72, torch.bfloat16), (900, 1152, torch.bfloat16), (300, 8192, torch.float32), (500, 333, torch.float32)])
def test_norms_and_backwards_over_the_same_buffers(rows, D, dtype):
    """Backward behind backward with one workspace, each on what the forward in front of it has just written."""
    sets = [[_draw(10 * j + k, rows, D, dtype=dtype).cuda() for k in range(6)] for j in range(3)]
    g = (1 + _draw(99, D, std=0.2)).cuda()
    ws = torch.empty(binding.tvm_attn_rmsnorm_jvp_workspace_bytes(D, binding.BF16 if dtype is torch.bfloat16 else binding.FP32), dtype=torch.uint8, device="cuda")
    y, h, ty, th, dx, dtx = (torch.empty_like(sets[0][0]) for _ in range(6))
    keep = [[torch.empty_like(dx), torch.empty_like(dx), torch.empty_like(g)] for _ in range(9)]

    def step(j, dg):
        x, res, tx, tres, dy, dty = sets[j]
        binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, g, out=(y, h, ty, th))
        return binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, y, ty, g, out=(dx, dtx, dg), workspace=ws)

    want = [_alone(lambda: step(j, keep[0][2])) for j in range(3)]

    def enqueue():
        for i, (a, b, dg) in enumerate(keep):
            step(i % 3, dg)
            x, res, tx, tres, dy, dty = sets[i % 3]
            binding.tvm_attn_rmsnorm_jvp_bwd(h, dy, th, dty, y, ty, g, out=(a, b, dg), workspace=ws)     # the partial sums again, before anyone else
        return [t for k in keep for t in k]

    for got in _both(enqueue):
        for i, t in enumerate(got):
            assert torch.equal(t, want[i // 3 % 3][i % 3]), i


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [72, 512, 1152, 2048, 8192])
def test_the_same_bits_with_and_without_tangents(D, dtype):
    x, res, tx, tres = (_draw(k, 300, D, dtype=dtype).cuda() for k in range(4))
    for g in (None, (1 + _draw(9, D, std=0.2)).cuda()):
        y, h, ty, th = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, tx, tres, g)
        y1, h1, _, _ = binding.tvm_attn_rmsnorm_jvp_fwd(x, res, g=g)
        assert torch.equal(y, y1) and torch.equal(h, h1)
        assert torch.equal(th, (tx.float() + tres.float()).to(dtype))


@pytest.mark.parametrize("captured", [False, True])
def test_branches_that_part_and_meet(captured):
    """A norm on one stream, products of its rows on two others, a norm of their sum behind both: a dependent launch waits for what its stream waits for."""
    x = _draw(1, 2000, 1152, dtype=torch.bfloat16).cuda()
    w, ws = binding.tvm_attn_quantize_s8(_draw(2, 1152, 1152, std=0.03).cuda())
    q, s, h = binding.tvm_attn_rmsnorm_s8(x, x)
    a, b, y, hh = (torch.empty_like(x) for _ in range(4))
    sides = [torch.cuda.Stream() for _ in range(2)]

    def enqueue():
        main = torch.cuda.current_stream()
        for _ in range(5):
            binding.tvm_attn_rmsnorm_s8(x, x, out=(q, s, h))
            for st, out, rows in zip(sides, (a, b), (2000, 60)):
                st.wait_stream(main)
                with torch.cuda.stream(st):
                    binding.tvm_attn_linear_s8(q[:rows], s[:rows], w, ws, out=out[:rows])
            for st in sides:
                main.wait_stream(st)
            binding.tvm_attn_rmsnorm_jvp_fwd(a, b, out=(y, hh, None, None))
            for t in (a, b, q):
                t.fill_(3)                  # nothing of the round before is left to be right by chance

    b.fill_(3)
    torch.cuda.synchronize()
    binding.tvm_attn_rmsnorm_s8(x, x, out=(q, s, h))
    a0 = binding.tvm_attn_linear_s8(q, s, w, ws)
    b0 = torch.full_like(b, 3)
    b0[:60] = binding.tvm_attn_linear_s8(q[:60], s[:60], w, ws)
    want = binding.tvm_attn_rmsnorm_jvp_fwd(a0, b0)[:2]
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            enqueue()
        for _ in range(3):
            graph.replay()
    else:
        enqueue()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(hh, want[1])
