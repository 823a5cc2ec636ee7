"""The product of two microscaled streams against the exact product of their values."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, HALF_STEP, drawn, enec

pytestmark = pytest.mark.gpu


def check(tokens, rows, cols, dt, gap=0, seed=0, spread=0):
    E = enec()
    g = torch.Generator().manual_seed(seed + 5 * tokens + 3 * rows + cols)
    x, w = torch.randn(tokens, cols, generator=g), torch.randn(rows, cols, generator=g)
    if spread:
        x = x * torch.exp2(torch.randint(-spread, spread, (tokens, 1), generator=g).float())
        w = w * torch.exp2(torch.randint(-spread, spread, (rows, 1), generator=g).float())
    xs, ws = (torch.from_numpy(ref.stream(v.double().numpy()[None])).cuda() for v in (x, w))
    xv, wv = ref.values(x.double().numpy()), ref.values(w.double().numpy())
    y = torch.full((tokens, rows + gap), 5.0, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert E.enec_matmul_microscaled_both(xs, xs.numel(), tokens, ws, ws.numel(), rows, cols, dt, y, rows + gap, status) == 0
    got = y.cpu().double().numpy()
    assert int(status.item()) == 0
    exact = xv @ wv.T
    # products are exact; the sums are fp32's, at most one rounding of 2^-24 of the magnitudes' sum for each term; y's own rounding
    bound = HALF_STEP[dt] * np.abs(exact) + (cols + 16) * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T) + torch.finfo(DTYPES[dt]).smallest_normal * HALF_STEP[dt]
    off = np.abs(got[:, :rows] - exact)
    assert (off <= bound).all(), (off / bound).max()
    assert (got[:, rows:] == 5).all()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("cols", [1, 64, 256, 300, 1000, 2055])
def test_one_tile(dt, cols):
    check(128, 128, cols, dt)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 15, 64, 65, 129, 192, 200, 400])
@pytest.mark.parametrize("rows", [1, 127, 200, 515])
def test_ragged(dt, tokens, rows):
    check(tokens, rows, 700, dt, gap=(rows % 3))


@pytest.mark.parametrize("tokens, rows, cols", [(2000, 4096, 512), (1500, 5000, 300), (577, 9000, 64), (192, 20000, 256)])
def test_large_tiles(tokens, rows, cols):
    check(tokens, rows, cols, 0)


@pytest.mark.parametrize("tokens, rows", [(70, 130), (600, 8200)])
def test_scales_of_all_sizes(tokens, rows):
    check(tokens, rows, 320, 0, spread=30)


@pytest.mark.parametrize("tokens", [3, 500])
def test_nan_blocks_wrong_headers_and_no_columns(tokens):
    E = enec()
    x, w = drawn((tokens, 320), 2, 1), drawn((300, 320), 2, 2)
    x[1, 40], w[7, 300] = float("nan"), float("inf")
    xs, ws = E.quantize_tensor(x.cuda()), E.quantize_tensor(w.cuda())
    y = torch.zeros(tokens, 300, dtype=torch.bfloat16, device="cuda")
    status = status_tensor()
    assert E.enec_matmul_microscaled_both(xs, xs.numel(), tokens, ws, ws.numel(), 300, 320, 0, y, 300, status) == 0
    bad = torch.isnan(y).cpu()
    want = torch.zeros_like(bad)
    want[1, :] = True
    want[:, 7] = True
    assert torch.equal(bad, want) and int(status.item()) == 0
    for which in (0, 1):
        streams = [xs.clone(), ws.clone()]
        streams[which][13] ^= 1
        y.fill_(5)
        status.zero_()
        assert E.enec_matmul_microscaled_both(streams[0], xs.numel(), tokens, streams[1], ws.numel(), 300, 320, 0, y, 300, status) == 0
        assert int(status.item()) == -4 and (y == 5).all()
    none_x, none_w = (torch.from_numpy(ref.stream(np.zeros((1, n, 0)))).cuda() for n in (tokens, 300))
    assert E.enec_matmul_microscaled_both(none_x, none_x.numel(), tokens, none_w, none_w.numel(), 300, 0, 0, y, 300) == 0
    assert (y == 0).all()


def test_quantised_activations_through_the_product_captured_and_on_two_streams():
    """The run of a prompt's product: quantise, multiply, on one stream each; bit-identical eager, concurrent and replayed."""
    E = enec()
    x, w = drawn((333, 1000), 0, 1).cuda(), E.quantize_tensor(drawn((700, 1000), 2, 2).cuda())
    size = E.enec_microscaled_size(1, 333, 1000)

    def call(y, xs):
        assert E.enec_quantize_microscaled(x, 0, 1, 333, 1000, 1000, xs, size) == 0
        assert E.enec_matmul_microscaled_both(xs, size, 333, w, w.numel(), 700, 1000, 0, y, 700) == 0
    ys = [torch.zeros(333, 700, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    xss = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    call(ys[0], xss[0])
    torch.cuda.synchronize()
    for i in (1, 2):
        s = torch.cuda.Stream(priority=-1)
        with torch.cuda.stream(s):
            call(ys[i], xss[i])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ys[3], xss[3])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(ys[0], y) for y in ys[1:])
