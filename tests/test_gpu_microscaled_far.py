"""Calls at their limits of place and order: offsets beyond 32 bits, rows behind the last token, and a process whose first calls are captured."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, enec
from test_gpu_microscaled_exact import grid_weights, rounded, whole_numbers
from test_gpu_microscaled_moe import inputs

pytestmark = pytest.mark.gpu


def far_rows(rows, cols, ld, dtype):
    """A tensor of rows x cols whose rows lie ld values apart, and its memory; nothing but the rows is touched."""
    wide = torch.empty(rows * ld, dtype=dtype, device="cuda")
    return wide.as_strided((rows, cols), (ld, 1))


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, ld_x, ld_y", [(16, 1 << 28, (1 << 28) + 1), (40, 1 << 26, 1 << 27), (300, (1 << 23) + 1, 1 << 24), (300, 1 << 24, (1 << 23) + 3)])
def test_rows_of_activations_and_results_beyond_32_bits(dt, tokens, ld_x, ld_y):
    E = enec()
    rows, cols = 200, 700
    g = torch.Generator().manual_seed(tokens)
    x, w = (whole_numbers((tokens, cols), g) / 32).to(DTYPES[dt]), grid_weights(rows, cols, g)
    stream = torch.from_numpy(ref.stream(w[None])).cuda()
    xs, y = far_rows(tokens, cols, ld_x, DTYPES[dt]), far_rows(tokens + 1, rows + 1, ld_y, DTYPES[dt])
    assert tokens * ld_x * 2 > 1 << 32 and tokens * ld_y * 2 > 1 << 32
    xs.copy_(x)
    y.fill_(5)
    status = status_tensor()
    want = rounded(x.double().numpy() @ w.T, dt)
    assert E.enec_matmul_microscaled(xs, dt, tokens, ld_x, stream, stream.numel(), rows, cols, y, ld_y, status) == 0
    assert torch.equal(y[:tokens, :rows].cpu(), want) and (y[:tokens, rows] == 5).all() and (y[tokens] == 5).all()
    # the same x as a stream: whole numbers up to 8 are not all in E2M1, so the product is that of the stream's values
    small = torch.empty(E.enec_microscaled_size(1, tokens, cols), dtype=torch.uint8, device="cuda")
    assert E.enec_quantize_microscaled(xs, dt, 1, tokens, cols, ld_x, small, small.numel(), status) == 0
    values = ref.values(x.double().numpy())
    assert np.array_equal(small.cpu().numpy(), ref.stream(x.double().numpy()[None]))
    y.fill_(5)
    assert E.enec_matmul_microscaled_both(small, small.numel(), tokens, stream, stream.numel(), rows, cols, dt, y, ld_y, status) == 0
    assert torch.equal(y[:tokens, :rows].cpu(), rounded(values @ w.T, dt)) and (y[:tokens, rows] == 5).all() and (y[tokens] == 5).all()
    back = far_rows(tokens + 1, cols + 1, ld_x, DTYPES[dt])
    back.fill_(5)
    assert E.enec_dequantize_microscaled(small, small.numel(), dt, 1, tokens, cols, back, ld_x, status) == 0
    assert torch.equal(back[:tokens, :cols].cpu(), rounded(values, dt)) and (back[:tokens, cols] == 5).all() and (back[tokens] == 5).all()
    assert int(status.item()) == 0


@pytest.mark.parametrize("tokens", [3, 40])
def test_rows_of_a_layer_beyond_32_bits(tokens):
    E = enec()
    hidden, inter, experts, top, ld_x, ld_y = 300, 128, 4, 2, (1 << 32) // tokens // 16 * 8, (1 << 32) // tokens + 1
    x, router, weights = inputs(tokens, hidden, inter, experts, 0, 5)
    streams = [E.quantize_tensor(w.cuda()) for w in weights]
    args = [a for s in streams for a in (s, s.numel())]
    space = torch.empty(E.enec_moe_microscaled_workspace(tokens, hidden, inter, experts, top), dtype=torch.uint8, device="cuda")
    far_x, far_y, near_y = far_rows(tokens, hidden, ld_x, x.dtype), far_rows(tokens + 1, hidden + 1, ld_y, x.dtype), torch.empty(tokens, hidden, dtype=x.dtype, device="cuda")
    far_x.copy_(x)
    far_y.fill_(5)
    router = router.cuda()
    for xs, ld, y, ldy in ((x.cuda(), hidden, near_y, hidden), (far_x, ld_x, far_y, ld_y)):
        assert E.enec_moe_microscaled(xs, 0, tokens, hidden, ld, router, experts, top, True, *args, inter, y, ldy, space, space.numel()) == 0
    assert torch.equal(far_y[:tokens, :hidden], near_y) and (far_y[:tokens, hidden] == 5).all() and (far_y[tokens] == 5).all()


@pytest.mark.parametrize("tokens", [4, 64, 300])
def test_streams_beyond_32_bits(tokens):
    """A stream of 4.6 GB: its last rows against the same rows as a stream of their own, in sums that are exact."""
    E = enec()
    rows, cols, tail = 131072, 65536, 300
    w = torch.randint(-3, 4, (rows, cols), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    w[:, ::32] = 4
    stream = E.quantize_tensor(w)
    assert stream.numel() > 1 << 32
    last = E.quantize_tensor(w[-tail:])
    back = E.dequantize_tensor(stream, torch.bfloat16, (rows, cols))
    assert torch.equal(back[-tail:], w[-tail:]) and torch.equal(back[:tail], w[:tail])
    del back, w
    x = torch.randint(-2, 3, (tokens, cols), device="cuda").to(torch.bfloat16)   # sums below 65536 x 4 x 2
    y, z = torch.empty(tokens, rows, dtype=torch.bfloat16, device="cuda"), torch.empty(tokens, tail, dtype=torch.bfloat16, device="cuda")
    xs = E.quantize_tensor(x)
    for big, small in ((lambda: E.enec_matmul_microscaled(x, 0, tokens, cols, stream, stream.numel(), rows, cols, y, rows),
                        lambda: E.enec_matmul_microscaled(x, 0, tokens, cols, last, last.numel(), tail, cols, z, tail)),
                       (lambda: E.enec_matmul_microscaled_both(xs, xs.numel(), tokens, stream, stream.numel(), rows, cols, 0, y, rows),
                        lambda: E.enec_matmul_microscaled_both(xs, xs.numel(), tokens, last, last.numel(), tail, cols, 0, z, tail))):
        assert big() == 0 and small() == 0
        assert torch.equal(y[:, -tail:], z) and z.abs().max() > 0


FIRST_CALLS = '''
import torch
import paper_2604_03298_b200 as E
g = torch.Generator().manual_seed(1)
x = torch.randn(300, 512, generator=g).cuda().to(torch.DTYPE)
w = torch.randn(700, 512, generator=g).cuda().to(torch.DTYPE)
experts = [torch.randn(4, r, c, generator=g).cuda().to(torch.DTYPE) for r, c in ((256, 512), (256, 512), (512, 256))]
router = torch.randn(4, 512, generator=g).cuda().to(torch.DTYPE)
def empty(*shape): return torch.zeros(E.enec_microscaled_size(*shape), dtype=torch.uint8, device="cuda")
ws, xs, es = empty(1, 700, 512), empty(1, 300, 512), [empty(*e.shape) for e in experts]
back = torch.zeros_like(w)
ys = [torch.zeros(n, 700, dtype=x.dtype, device="cuda") for n in (3, 40, 300, 300)]
layer = torch.zeros(5, 512, dtype=x.dtype, device="cuda")
space = torch.zeros(E.enec_moe_microscaled_workspace(5, 512, 256, 4, 2), dtype=torch.uint8, device="cuda")
outputs = [ws, xs, back, layer, *es, *ys]
def run():
    ok = E.enec_quantize_microscaled(w, DT, 1, 700, 512, 512, ws, ws.numel())
    ok |= E.enec_quantize_microscaled(x, DT, 1, 300, 512, 512, xs, xs.numel())
    ok |= E.enec_dequantize_microscaled(ws, ws.numel(), DT, 1, 700, 512, back, 512)
    for y in ys[:3]: ok |= E.enec_matmul_microscaled(x, DT, y.shape[0], 512, ws, ws.numel(), 700, 512, y, 700)
    ok |= E.enec_matmul_microscaled_both(xs, xs.numel(), 300, ws, ws.numel(), 700, 512, DT, ys[3], 700)
    for e, s in zip(experts, es): ok |= E.enec_quantize_microscaled(e, DT, *e.shape, e.shape[2], s, s.numel())
    ok |= E.enec_moe_microscaled(x, DT, 5, 512, 512, router, 4, 2, True, es[0], es[0].numel(), es[1], es[1].numel(), es[2], es[2].numel(), 256, layer, 512,
                                 space, space.numel())
    assert ok == 0, ok
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
assert all((o == 0).all() for o in outputs)
graph.replay()
torch.cuda.synchronize()
replayed = [o.clone() for o in outputs]
for o in outputs: o.zero_()
run()
torch.cuda.synchronize()
assert all(torch.equal(a, b) and (a != 0).any() for a, b in zip(replayed, outputs))
'''


@pytest.mark.parametrize("dt, name", [(0, "bfloat16"), (1, "float16")])
def test_a_process_whose_first_calls_are_captured(dt, name):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = FIRST_CALLS.replace("torch.DTYPE", "torch." + name).replace("DT,", f"{dt},").replace(", DT)", f", {dt})")
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-2000:]
