"""Microscaled 4-bit streams on the GPU: bytes, values and products against plain numpy in 64 bits (microscaled_reference)."""
import numpy as np
import pytest
import torch

import microscaled_reference as ref
from gpu_util import status_tensor

pytestmark = pytest.mark.gpu

DTYPES = {0: torch.bfloat16, 1: torch.float16, 2: torch.float32}
HALF_STEP = {dt: torch.finfo(t).eps / 2 for dt, t in DTYPES.items()}   # of a rounding, relative to the value


def enec():
    import paper_2604_03298_b200
    return paper_2604_03298_b200


def drawn(shape, dt, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if kind == "wide":       # exponents all over the type's range, zeros, the largest and the smallest values
        limit = {0: 120, 1: 13, 2: 120}[dt]
        x = x * torch.exp2(torch.randint(-limit, limit, (*shape[:-1], 1), generator=g).float())
        x = torch.where(torch.rand(shape, generator=g) < 0.1, torch.zeros(()), x)
    if kind == "grid":       # borders and ties
        x = torch.randint(-32, 33, shape, generator=g).float() / 4
    return x.to(DTYPES[dt])


def strided(x, gap, fill):
    """x on the GPU in rows `gap` values further apart, the gaps filled with `fill`."""
    wide = torch.full((*x.shape[:-1], x.shape[-1] + gap), fill, dtype=x.dtype)
    wide[..., :x.shape[-1]] = x
    return wide.cuda()


SHAPES = [(1, 1, 1), (1, 1, 32), (1, 3, 33), (1, 128, 256), (1, 129, 257), (2, 37, 100), (3, 127, 511), (1, 300, 2047), (2, 5, 8)]


@pytest.mark.parametrize("dt", [0, 1, 2])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind, gap", [("normal", 0), ("wide", 1), ("grid", 3), ("normal", 8)])
def test_stream_is_the_definitions_byte_for_byte(dt, shape, kind, gap):
    E = enec()
    x = drawn(shape, dt, 100 * dt + 7 * shape[1] + shape[2], kind)
    size = E.enec_microscaled_size(*shape)
    buf = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    status = status_tensor()
    assert E.enec_quantize_microscaled(strided(x, gap, float("nan")), dt, *shape, shape[2] + gap, buf, size, status) == 0
    got = buf.cpu().numpy()
    assert int(status.item()) == 0
    assert np.array_equal(got[:size], ref.stream(x.double().numpy()))
    assert (got[size:] == 0xA5).all()


@pytest.mark.parametrize("dt", [0, 1, 2])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gap", [0, 1, 3, 8])
def test_values_of_a_stream(dt, shape, gap):
    """Exact in bf16 and fp32; in fp16 the nearest value, which torch's conversion of the exact one gives. Gaps stay as they were."""
    E = enec()
    x = drawn(shape, 2, 11 + shape[2], "normal") * 0.3
    stream = torch.from_numpy(ref.stream(x.double().numpy())).cuda()
    out = torch.full((*shape[:-1], shape[2] + gap), 7.0, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert E.enec_dequantize_microscaled(stream, stream.numel(), dt, *shape, out, shape[2] + gap, status) == 0
    got = out.cpu()
    assert int(status.item()) == 0
    assert torch.equal(got[..., :shape[2]], torch.from_numpy(ref.values(x.double().numpy())).to(DTYPES[dt]))
    assert (got[..., shape[2]:] == 7).all()


@pytest.mark.parametrize("dt", [0, 1, 2])
def test_extreme_blocks(dt):
    """Infinities and NaN make their block NaN and no other; zeros keep their sign; the smallest and largest finite values."""
    E = enec()
    info = torch.finfo(DTYPES[dt])
    x = torch.ones(10, 96)
    x[0, 5], x[1, 40], x[2, 95] = float("inf"), float("-inf"), float("nan")
    x[3] = 0.0
    x[4] = -0.0
    x[5], x[6] = info.max, -info.max
    x[7] = info.tiny
    x[8] = info.smallest_normal * info.eps          # the smallest subnormal number
    x[9, ::2] = info.max
    x = x.to(DTYPES[dt])
    stream = E.quantize_tensor(x.cuda())
    assert np.array_equal(stream.cpu().numpy(), ref.stream(x.double().numpy()[None]))
    back = E.dequantize_tensor(stream, DTYPES[dt], x.shape).cpu()
    want = torch.from_numpy(ref.values(x.double().numpy())).to(DTYPES[dt])
    assert torch.equal(torch.isnan(back), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(back), torch.nan_to_num(want))
    assert torch.isnan(back[0, :32]).all() and not torch.isnan(back[0, 32:]).any()


def test_empty_shapes_and_wrong_headers():
    E = enec()
    status = status_tensor()
    for shape in ((0, 4, 4), (2, 0, 7), (2, 3, 0)):
        size = E.enec_microscaled_size(*shape)
        buf = torch.zeros(size, dtype=torch.uint8, device="cuda")
        assert E.enec_quantize_microscaled(None, 0, *shape, max(shape[2], 1), buf, size, status) == 0
        assert np.array_equal(buf.cpu().numpy(), ref.stream(np.zeros(shape)))
        assert E.enec_dequantize_microscaled(buf, size, 0, *shape, None, max(shape[2], 1), status) == 0
        assert int(status.item()) == 0
    x = drawn((5, 300), 0, 3).cuda()
    stream = E.quantize_tensor(x)
    for at, shape in ((0, (5, 300)), (4, (5, 300)), (8, (5, 300)), (24, (5, 300)), (None, (4, 300)), (None, (5, 299))):
        bad = stream.clone()
        if at is not None:
            bad[at] += 1
        out = torch.full(shape, 3.0, dtype=torch.bfloat16, device="cuda")
        y = torch.full((2, shape[0]), 3.0, dtype=torch.bfloat16, device="cuda")
        status.zero_()
        assert E.enec_dequantize_microscaled(bad, bad.numel(), 0, 1, *shape, out, shape[1], status) == 0
        assert int(status.item()) == -4 and (out == 3).all()
        status.zero_()
        assert E.enec_matmul_microscaled(x, 0, 2, 300, bad, bad.numel(), *shape, y, shape[0], status) == 0
        assert int(status.item()) == -4 and (y == 3).all()
        with pytest.raises(E.EnecError):
            E.dequantize_tensor(bad, torch.bfloat16, shape)


def block_tops(x):
    """For every value the largest magnitude of the 32 neighbours that it stands among."""
    blocks = ref.blocks_of(x)
    tops = np.repeat(np.abs(blocks).max(-1), 32, axis=-1)
    return tops[..., :np.shape(x)[-1]]


def product_bound(x, w, dt):
    """The product and how far it may be off: its own rounding; values of x to 2^-22 of the largest of their block; and fp32 sums, n terms
    with at most n roundings of 2^-24 relative to the sum of magnitudes. Up to 16 tokens a value is a sum of digits from -4 to 3 times
    powers of 8, whose magnitudes add up to at most 3 times its own (4 = 8 - 4 is the worst) and what its block's rounding adds."""
    tops = 2.0 ** -22 * block_tops(x)
    exact = x @ w.T
    return exact, (HALF_STEP[dt] * np.abs(exact) + 3 * (x.shape[1] + 16) * 2.0 ** -24 * ((np.abs(x) + tops) @ np.abs(w).T)
                   + (1 + HALF_STEP[dt]) * (tops @ np.abs(w).T))


def check_product(tokens, rows, cols, dt, gap_x=0, gap_y=0, scale=1.0, seed=0, call="enec_matmul_microscaled"):
    E = enec()
    g = torch.Generator().manual_seed(seed + tokens * 7 + rows * 3 + cols)
    x = (torch.randn(tokens, cols, generator=g) * scale).to(DTYPES[dt])
    w = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-6, 3, (rows, 1), generator=g).float())
    stream = torch.from_numpy(ref.stream(w.double().numpy()[None])).cuda()
    values = ref.values(w.double().numpy())
    y = torch.full((tokens, rows + gap_y), 5.0, dtype=DTYPES[dt], device="cuda")
    status = status_tensor()
    assert E.enec_matmul_microscaled(strided(x, gap_x, float("nan")), dt, tokens, cols + gap_x, stream, stream.numel(), rows, cols, y, rows + gap_y,
                                     status) == 0
    got = y.cpu().double().numpy()
    assert int(status.item()) == 0
    exact, bound = product_bound(x.double().numpy(), values, dt)
    tiny = torch.finfo(DTYPES[dt]).smallest_normal * torch.finfo(DTYPES[dt]).eps
    off = np.abs(got[:, :rows] - exact)
    assert (off <= bound + tiny / 2).all(), (off / (bound + tiny)).max()
    assert (got[:, rows:] == 5).all()


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 16, 17, 32, 33, 100])
@pytest.mark.parametrize("rows, cols", [(1, 1), (16, 128), (129, 300), (100, 1408), (515, 2055)])
def test_product(dt, tokens, rows, cols):
    check_product(tokens, rows, cols, dt)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [1, 5, 40, 130])
@pytest.mark.parametrize("gap_x, gap_y", [(1, 0), (8, 3), (0, 1), (3, 8)])
def test_product_with_rows_apart(dt, tokens, gap_x, gap_y):
    check_product(tokens, 200, 333, dt, gap_x, gap_y)
    check_product(tokens, 256, 512, dt, gap_x, gap_y)


@pytest.mark.parametrize("tokens", [1, 8, 32, 200])
@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e5, 1e30])
def test_product_of_small_and_large_activations(tokens, scale):
    check_product(tokens, 130, 700, 0, scale=scale)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols, gap", [(2000, 4096, 320, 0), (1500, 5000, 257, 1), (2047, 3969, 64, 8), (257, 16500, 100, 0)])
def test_product_of_many_tiles(dt, tokens, rows, cols, gap):
    check_product(tokens, rows, cols, dt, gap)


# steps of 64 columns are shared out among warps that issue and warps that bring weights back: fewer steps than warps, odd
# numbers of them, more than the stages hold
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [17, 80, 144, 256])
@pytest.mark.parametrize("cols", [8, 64, 72, 128, 192, 256, 320, 448, 832, 2112])
def test_product_of_few_steps(dt, tokens, cols):
    check_product(tokens, 150, cols, dt)
    check_product(tokens, 150, cols, dt, 3)


# the columns of a tile shared out: to 6 CTAs, to 4 since 16 times 8 would not run at once, to 7, 5 and 3; the last ones with less than the others
@pytest.mark.parametrize("tokens, rows, cols", [(17, 1024, 4100), (100, 2048, 4096), (70, 300, 3400), (33, 640, 2300), (256, 5100, 1500)])
def test_product_of_shared_columns(tokens, rows, cols):
    check_product(tokens, rows, cols, 0)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens, rows, cols", [(8, 48, 14336), (32, 40, 14336), (3, 20, 60000), (1, 4096, 4096), (65, 20, 20000)])
def test_product_of_long_rows(dt, tokens, rows, cols):
    check_product(tokens, rows, cols, dt)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("tokens", [2, 140])
def test_infinities_and_nan_stay_in_their_token_and_their_row(dt, tokens):
    """An infinity or a NaN among a token's values: none of that token's results is finite, others are as without it. A weight block
    of NaN: its row for every token, others not."""
    E = enec()
    x = drawn((tokens, 320), dt, 5)
    w = drawn((70, 320), 2, 6)
    clean = E.quantize_tensor(w.cuda())
    y = torch.empty(tokens, 70, dtype=DTYPES[dt], device="cuda")
    base = torch.empty_like(y)
    assert E.enec_matmul_microscaled(x.cuda(), dt, tokens, 320, clean, clean.numel(), 70, 320, base, 70) == 0
    for value in (float("inf"), float("-inf"), float("nan")):
        bad = x.clone()
        bad[1, 100] = value
        assert E.enec_matmul_microscaled(bad.cuda(), dt, tokens, 320, clean, clean.numel(), 70, 320, y, 70) == 0
        assert not torch.isfinite(y[1]).any()
        assert torch.equal(y[0], base[0]) and torch.equal(y[2:], base[2:])
    w[3, 7] = float("nan")
    dirty = E.quantize_tensor(w.cuda())
    assert E.enec_matmul_microscaled(x.cuda(), dt, tokens, 320, dirty, dirty.numel(), 70, 320, y, 70) == 0
    assert torch.isnan(y[:, 3]).all()
    keep = [i for i in range(70) if i != 3]
    assert torch.equal(y[:, keep], base[:, keep])


@pytest.mark.parametrize("tokens", [1, 16, 200])
def test_product_of_no_columns_is_zero(tokens):
    E = enec()
    stream = torch.from_numpy(ref.stream(np.zeros((1, 9, 0)))).cuda()
    y = torch.full((tokens, 12), 5.0, dtype=torch.float16, device="cuda")
    assert E.enec_matmul_microscaled(None, 1, tokens, 0, stream, stream.numel(), 9, 0, y, 12) == 0
    assert (y[:, :9] == 0).all() and (y[:, 9:] == 5).all()


@pytest.mark.parametrize("tokens", [1, 8, 50, 300])
def test_repeated_captured_and_concurrent_calls_agree_bit_for_bit(tokens):
    E = enec()
    x, w = drawn((tokens, 1000), 0, 1).cuda(), drawn((300, 1000), 2, 2)
    stream = E.quantize_tensor(w.cuda())
    ys = [torch.zeros(tokens, 300, dtype=torch.bfloat16, device="cuda") for _ in range(4)]

    def call(y):
        assert E.enec_matmul_microscaled(x, 0, tokens, 1000, stream, stream.numel(), 300, 1000, y, 300) == 0
    call(ys[0])
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(priority=-1) for _ in range(2)]
    for s, y in zip(side, ys[1:3]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call(y)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(ys[3])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(ys[0], y) for y in ys[1:])


def test_quantize_tensor_takes_views():
    """Rows apart, transposed, unaligned and broadcast views: the stream is that of the dense copy."""
    E = enec()
    wide = torch.randn(70, 400, device="cuda").to(torch.float16)
    for view in (wide[:, :300], wide[3:, 8:], wide[:, 1:], wide.t(), wide[:1].expand(5, 400), wide[::2]):
        got = E.quantize_tensor(view)
        assert torch.equal(got, E.quantize_tensor(view.contiguous().clone()))
        assert np.array_equal(got.cpu().numpy(), ref.stream(view.cpu().double().numpy()[None]))
    with pytest.raises(ValueError):
        E.quantize_tensor(wide[0])


def test_layer_of_products_one_after_another():
    """As they are used together: a decoder layer's gate, up and down products of a few tokens on streams made from one checkpoint tensor,
    the same layer for a prompt, and the same with 4-bit activations; the three agree where they compute the same."""
    E = enec()
    hidden, ffn = 512, 1100
    g = torch.Generator().manual_seed(3)
    ws = [E.quantize_tensor((torch.randn(r, c, generator=g) * c ** -0.5).to(torch.bfloat16).cuda()) for r, c in ((ffn, hidden), (ffn, hidden), (hidden, ffn))]
    x = torch.randn(300, hidden, generator=g).to(torch.bfloat16).cuda()

    def product(x, w, rows):
        y = torch.empty(x.shape[0], rows, dtype=x.dtype, device="cuda")
        assert E.enec_matmul_microscaled(x, 0, x.shape[0], x.shape[1], w, w.numel(), rows, x.shape[1], y, rows) == 0
        return y

    def layer(x):
        a, u = product(x, ws[0], ffn), product(x, ws[1], ffn)
        return product((torch.nn.functional.silu(a.float()) * u.float()).to(x.dtype), ws[2], hidden)
    many, few = layer(x), torch.cat([layer(x[i:i + 10].contiguous()) for i in range(0, 300, 10)])
    # Both forms round their results once. Where an exact sum lies beside a border between two bf16 values they may fall on either side, one
    # step (at most 2^-7 of the value) apart: a and u, through |silu'| <= 1.1, then their rounded product, then y. 1.05 covers the steps'
    # own products and the fp32 sums, which are 2^-11 of the steps.
    v = [torch.from_numpy(ref.values(E.dequantize_tensor(w, torch.float32, s).cpu().numpy())) for w, s in zip(ws, ((ffn, hidden), (ffn, hidden), (hidden, ffn)))]
    a, u = x.cpu().double() @ v[0].T, x.cpu().double() @ v[1].T
    h = torch.nn.functional.silu(a)
    step = 2.0 ** -7
    off = 1.05 * step * (1.1 * a.abs() * u.abs() + 2 * h.abs() * u.abs())
    many, few = many.cpu().double(), few.cpu().double()
    assert ((many - few).abs() <= 1.05 * (off @ v[2].abs().T + step * many.abs())).all()
