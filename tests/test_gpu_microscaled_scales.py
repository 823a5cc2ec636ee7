"""Products whose neighbouring blocks differ by powers of two: nothing of W is lost beside a larger block of the same row."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor
from test_gpu_microscaled import DTYPES, HALF_STEP, block_tops, enec, strided

pytestmark = pytest.mark.gpu


def product(x, w, dt, gap_x=0):
    """y of x and the stream of w on the GPU, as float64, with W's values."""
    E = enec()
    (tokens, cols), rows = x.shape, w.shape[0]
    stream = torch.from_numpy(ref.stream(w[None])).cuda()
    y = torch.full((tokens, rows + 1), 5.0, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert E.enec_matmul_microscaled(strided(x, gap_x, float("nan")), dt, tokens, cols + gap_x, stream, stream.numel(), rows, cols, y, rows + 1,
                                     status) == 0
    got = y.cpu().double().numpy()
    assert int(status.item()) == 0 and (got[:, rows:] == 5).all()
    return got[:, :rows], ref.values(w)


def bound_of(x, w, dt):
    """Of 17 tokens and more operands are not rounded: y's own rounding, half of its smallest step, and fp32 sums of n terms, n roundings of
    2^-24 of the magnitudes' sum. Up to 16 tokens x counts to 2^-22 of its block's largest, and digits' magnitudes add up to three times
    a value's (see product_bound)."""
    few = x.shape[0] <= 16
    off = 2.0 ** -22 * block_tops(x) if few else np.zeros_like(x)
    exact = x @ w.T
    tiny = torch.finfo(DTYPES[dt]).smallest_normal * HALF_STEP[dt]
    sums = (3 if few else 1) * (x.shape[1] + 16) * 2.0 ** -24 * ((np.abs(x) + off) @ np.abs(w).T)
    return exact, HALF_STEP[dt] * np.abs(exact) + (1 + HALF_STEP[dt]) * (sums + off @ np.abs(w).T) + tiny


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 16, 17, 300])
@pytest.mark.parametrize("cols", [64, 4096])
def test_a_small_block_beside_a_large_one(dt, tokens, cols):
    """Columns 0 to 31 hold 4096, 32 to 63 1.5 x 2^-17, the others nothing; x is zero at the first and 60000 at the second:
    32 x 1.5 x 2^-17 x 60000, a whole number of steps of 2^-11 below 2^5, so that all sums are exact."""
    w = np.zeros((130, cols))
    w[:, :32], w[:, 32:64] = 4096.0, 1.5 * 2.0 ** -17
    x = torch.zeros(tokens, cols)
    x[:, 32:64] = 60000.0
    x = x.to(DTYPES[dt])
    got, values = product(x, w, dt)
    exact = x.double().numpy() @ values.T
    assert (exact > 21).all()
    assert np.array_equal(got, torch.from_numpy(exact).to(DTYPES[dt]).double().numpy())


# blocks `spread` powers of two apart in a row, x zero against the large ones, or (spread 0) everywhere something else; the sizes share
# out columns to clusters, to one CTA, to 256 rows a CTA, and take rows of x from odd addresses
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols, gap", [(3, 150, 700, 0), (16, 70, 2055, 1), (17, 150, 700, 0), (17, 70, 4100, 1), (300, 150, 330, 0), (40, 200, 999, 1),
                                                     (520, 5000, 290, 0), (520, 5000, 290, 3)])
@pytest.mark.parametrize("spread", [10, 20, 24, 36, 37, 40, 60, 100])
def test_blocks_of_a_row_far_apart(dt, tokens, rows, cols, gap, spread):
    g = torch.Generator().manual_seed(spread + cols)
    blocks = -(-cols // 32)
    large = torch.rand(rows, blocks, generator=g) < 0.3
    large[:, 0] = False
    quiet = torch.rand(blocks, generator=g) < 0.5                        # blocks of columns where x is zero, the only ones with large weights
    quiet[0] = False
    power = torch.where(large & quiet, float(spread - 12), -12.0)
    power[:, -1] = torch.where(torch.rand(rows, generator=g) < 0.5, -15.0, power[:, -1])
    power[: rows // 3] = -12.0                                           # rows without any
    w = torch.randn(rows, blocks, 32, generator=g).clamp(-3.9, 3.9)
    w[:, :, 0] = 4.0                                                     # a block's largest: its scale is its power of two
    w = (w * torch.exp2(power)[..., None]).reshape(rows, -1)[:, :cols].double().numpy()
    x = torch.randn(tokens, blocks, 32, generator=g) * torch.where(quiet, 0.0, 1.0)[:, None]
    x = x.reshape(tokens, -1)[:, :cols].to(DTYPES[dt])
    got, values = product(x, w, dt, gap)
    exact, bound = bound_of(x.double().numpy(), values, dt)
    off = np.abs(got - exact)
    assert (off <= bound).all(), (off / bound).max()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [16, 17, 140])
def test_rows_of_zeros_and_tiny_blocks(dt, tokens):
    """Blocks of zeros (scale byte 0) and blocks far below anything that counts lie beside ordinary ones without changing them; a row of such
    blocks alone is zero in fp16 and keeps its values in bf16."""
    g = torch.Generator().manual_seed(tokens)
    w = torch.randn(96, 512, generator=g).double()
    w[::3, 64:200] = 0
    w[1::3, 300:420] *= 2.0 ** -110
    w[90:] *= 2.0 ** -90
    w[95] = 0
    x = torch.randn(tokens, 512, generator=g).to(DTYPES[dt])
    got, values = product(x, w.numpy(), dt)
    exact, bound = bound_of(x.double().numpy(), values, dt)
    off = np.abs(got - exact)
    assert (off <= bound).all(), (off / bound).max()
    assert (got[:, 95] == 0).all() and (dt == 0 or (got[:, 90:] == 0).all())


@pytest.mark.parametrize("tokens", [16, 17, 300])
def test_all_scales_of_bf16(tokens):
    """A row for every scale byte from 0 to 252. Values of x are at 2^-60 and at 2^60, so that the smallest and the largest scales' results are
    normal numbers; others are compared where they are not beyond the type's range."""
    g = torch.Generator().manual_seed(tokens)
    power = torch.arange(253).double() - 127
    w = torch.randn(253, 96, generator=g).clamp(-3.9, 3.9).double()
    w[:, ::32] = 4.0
    w = w * torch.exp2(power)[:, None]
    x = torch.randn(tokens, 96, generator=g)
    x[::2] *= 2.0 ** -60
    x[1::2] *= 2.0 ** 60
    x = x.to(torch.bfloat16)
    got, values = product(x, w.numpy(), 0)
    exact, bound = bound_of(x.double().numpy(), values, 0)
    size = np.abs(x.double().numpy()) @ np.abs(values).T
    inside = (size < 2.0 ** 126) & (size > 2.0 ** -100)
    assert inside[::2, 240:].all() and (tokens == 1 or inside[1::2, :10].all())
    off = np.abs(got - exact)
    assert (off <= bound)[inside].all(), (off / bound)[inside].max()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [17, 140, 300])
def test_infinities_times_weights_of_17_tokens_and_more(dt, tokens):
    """Sums of a token with one infinity are infinite as the weights' signs say, and NaN where the weight is zero."""
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn(tokens, 320, generator=g).to(DTYPES[dt])
    x[1, 100], x[16, 7] = float("inf"), float("-inf")
    w = torch.randn(70, 320, generator=g).double().numpy()
    got, values = product(x, w, dt)
    for token, col, sign in ((1, 100, 1), (16, 7, -1)):
        want = np.where(values[:, col] == 0, np.nan, sign * np.sign(values[:, col]) * np.inf)
        assert np.isnan(want).any() and np.array_equal(got[token], want, equal_nan=True)
    keep = [t for t in range(tokens) if t not in (1, 16)]
    exact, bound = bound_of(x[keep].double().numpy(), values, dt)
    assert (np.abs(got[keep] - exact) <= bound).all()
