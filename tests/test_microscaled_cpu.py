"""The microscaled calls' boundary without a GPU: stream sizes, and every refusal that the host makes before it touches the device."""
import ctypes as C

import numpy as np
import pytest

import microscaled_reference as ref

OK, INVALID, DTYPE, SMALL, LARGE = 0, -1, -2, -3, -8


@pytest.fixture(scope="module")
def lib():
    from paper_2604_03298_b200 import build
    build.build()
    import paper_2604_03298_b200 as enec
    return enec.lib()


P = 1 << 20   # an address that is 16-byte aligned and never read: every call below is refused before it is used


@pytest.mark.parametrize("shape", [(0, 0, 0), (1, 0, 5), (1, 5, 0), (1, 1, 1), (1, 128, 256), (1, 129, 257), (3, 1411, 2047), (7, 127, 255)])
def test_size_is_header_and_records(lib, shape):
    assert lib.enec_microscaled_size(*shape) == ref.stream_bytes(*shape)


def test_size_of_shapes_that_are_too_large(lib):
    assert lib.enec_microscaled_size(1 << 31, 1, 1) == 0
    assert lib.enec_microscaled_size(1, 1 << 31, 1) == 0
    assert lib.enec_microscaled_size(1, 1, 1 << 31) == 0
    assert lib.enec_microscaled_size((1 << 29) + 1, 1, 1) == 0
    assert lib.enec_microscaled_size(1 << 29, 1, 1) == 128 + (1 << 29) * 17408
    assert lib.enec_microscaled_size(1 << 30, 1 << 30, 1 << 30) == 0


def test_reference_quantises_by_the_definition():
    """Borders between codes, ties to the even one, saturation, the scale of powers of two and their neighbours, empty and bad blocks."""
    x = np.zeros((1, 32))
    x[0, :16] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -6, -5, -3.5, -2.5, -1.75, -1.25, -0.75, -0.25]
    assert ref.values(x)[0, :16].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -6, -4, -4, -2, -2, -1, -1, 0]
    x[0, 0] = 7.9
    assert ref.values(x)[0, 0] == 6
    x[0, 0] = 8.0                                            # floor(log2) = 3: the scale becomes 2
    assert ref.values(x)[0, :4].tolist() == [8, 4, 4, 2]     # 5 / 2 = 2.5 -> 2, 3.5 / 2 = 1.75 -> 2, 2.5 / 2 = 1.25 -> 1
    byte, code = ref.encode(np.zeros((1, 5)))
    assert byte.tolist() == [[0]] and not code.any()
    for bad in (np.inf, -np.inf, np.nan):
        x[0, 3] = bad
        byte, code = ref.encode(x)
        assert byte.tolist() == [[255]] and not code.any()


def quantize(lib, d_in=P, dt=0, batch=1, rows=8, cols=64, ld=64, d_out=P, cap=1 << 20):
    return lib.enec_quantize_microscaled(d_in, dt, batch, rows, cols, ld, d_out, cap, None, None)


def dequantize(lib, d_in=P, size=1 << 20, dt=0, batch=1, rows=8, cols=64, d_out=P, ld=64):
    return lib.enec_dequantize_microscaled(d_in, size, dt, batch, rows, cols, d_out, ld, None, None)


def matmul(lib, d_x=P, dt=0, tokens=4, ld_x=64, d_w=P, size=1 << 20, rows=8, cols=64, d_y=P, ld_y=8):
    return lib.enec_matmul_microscaled(d_x, dt, tokens, ld_x, d_w, size, rows, cols, d_y, ld_y, None, None)


@pytest.mark.parametrize("changed, want", [
    (dict(dt=3), DTYPE), (dict(dt=-1), DTYPE), (dict(d_in=None), INVALID), (dict(d_out=None), INVALID), (dict(d_in=P + 2), INVALID),
    (dict(d_out=P + 8), INVALID), (dict(ld=63), INVALID), (dict(ld=1 << 36), INVALID), (dict(cap=128 + 17407), SMALL),
    (dict(rows=129, cap=128 + 17408), SMALL), (dict(rows=1 << 31), LARGE), (dict(batch=1 << 30), LARGE)])
def test_quantize_refuses(lib, changed, want):
    assert quantize(lib, **changed) == want


@pytest.mark.parametrize("changed, want", [
    (dict(dt=3), DTYPE), (dict(d_in=None), INVALID), (dict(d_out=None), INVALID), (dict(d_in=P + 4), INVALID), (dict(d_out=P + 2), INVALID),
    (dict(ld=63), INVALID), (dict(size=128 + 17407), SMALL), (dict(cols=1 << 31), LARGE), (dict(batch=1 << 30), LARGE)])
def test_dequantize_refuses(lib, changed, want):
    assert dequantize(lib, **changed) == want


@pytest.mark.parametrize("changed, want", [
    (dict(dt=2), DTYPE), (dict(dt=7), DTYPE), (dict(d_x=None), INVALID), (dict(d_w=None), INVALID), (dict(d_y=None), INVALID),
    (dict(d_x=P + 2), INVALID), (dict(d_w=P + 8), INVALID), (dict(d_y=P + 2), INVALID), (dict(ld_x=63), INVALID), (dict(ld_y=7), INVALID),
    (dict(size=17408), SMALL), (dict(rows=1 << 31, ld_y=1 << 31), LARGE), (dict(tokens=1 << 31), LARGE),
    (dict(tokens=0), OK), (dict(rows=0), OK)])
def test_matmul_refuses_or_has_nothing_to_do(lib, changed, want):
    assert matmul(lib, **changed) == want


def both(lib, d_x=P, x_size=1 << 20, tokens=4, d_w=P, w_size=1 << 20, rows=8, cols=64, dt=0, d_y=P, ld_y=8):
    return lib.enec_matmul_microscaled_both(d_x, x_size, tokens, d_w, w_size, rows, cols, dt, d_y, ld_y, None, None)


@pytest.mark.parametrize("changed, want", [
    (dict(dt=2), DTYPE), (dict(dt=5), DTYPE), (dict(d_x=None), INVALID), (dict(d_w=None), INVALID), (dict(d_y=None), INVALID),
    (dict(d_x=P + 2), INVALID), (dict(d_w=P + 8), INVALID), (dict(d_y=P + 2), INVALID), (dict(ld_y=7), INVALID), (dict(ld_y=1 << 36), INVALID),
    (dict(x_size=17408), SMALL), (dict(w_size=17408), SMALL), (dict(tokens=129, x_size=128 + 17408), SMALL), (dict(rows=1 << 31, ld_y=1 << 31), LARGE),
    (dict(tokens=1 << 31), LARGE), (dict(tokens=0), OK), (dict(rows=0), OK)])
def test_both_refuses_or_has_nothing_to_do(lib, changed, want):
    assert both(lib, **changed) == want


def moe(lib, d_x=P, dt=0, tokens=4, hidden=64, ld_x=64, d_router=P, experts=8, top=2, renormalize=1, d_gate=P, gate=1 << 20, d_up=P, up=1 << 20,
        d_down=P, down=1 << 20, inter=32, d_y=P, ld_y=64, d_workspace=P, workspace=1 << 20):
    return lib.enec_moe_microscaled(d_x, dt, tokens, hidden, ld_x, d_router, experts, top, renormalize, d_gate, gate, d_up, up, d_down, down, inter,
                                    d_y, ld_y, d_workspace, workspace, None, None)


@pytest.mark.parametrize("changed, want", [
    (dict(dt=2), DTYPE), (dict(tokens=65), LARGE), (dict(experts=513), LARGE), (dict(top=17), LARGE), (dict(tokens=64, experts=385), LARGE),
    (dict(hidden=1 << 24, ld_x=1 << 24, ld_y=1 << 24), LARGE), (dict(inter=1 << 24), LARGE),
    (dict(top=0), INVALID), (dict(top=9), INVALID), (dict(experts=0), INVALID), (dict(hidden=0), INVALID), (dict(inter=0), INVALID),
    (dict(ld_x=63), INVALID), (dict(ld_y=63), INVALID), (dict(gate=128 + 8 * 17408 - 1), SMALL), (dict(up=0), SMALL), (dict(down=17408), SMALL),
    (dict(workspace=64), SMALL), (dict(tokens=0), OK)]
    + [({name: bad}, INVALID) for name in ("d_x", "d_router", "d_gate", "d_up", "d_down", "d_y", "d_workspace") for bad in (None, P + 8)])
def test_moe_refuses_or_has_nothing_to_do(lib, changed, want):
    assert moe(lib, **changed) == want


def test_moe_workspace_holds_the_pairs_values(lib):
    f = lib.enec_moe_microscaled_workspace
    assert f(65, 64, 32, 8, 2) == 0 and f(4, 64, 32, 513, 2) == 0
    for tokens, hidden, inter, experts, top in ((1, 1, 1, 1, 1), (4, 64, 32, 8, 2), (64, 2048, 1408, 64, 6)):
        pairs = tokens * top
        assert f(tokens, hidden, inter, experts, top) >= pairs * (hidden + inter) * 4 + pairs * 8


def test_import_and_host_functions_without_a_torch_for_cuda():
    """A torch built without CUDA has no raw streams: the package is importable there, and what only the host computes works."""
    import os
    import subprocess
    import sys
    code = ("import torch\n"
            "del torch._C._cuda_getCurrentRawStream\n"
            "import paper_2604_03298_b200 as E\n"
            "assert E.enec_microscaled_size(1, 128, 256) == 128 + 17408 and E.enec_max_compressed_size(0, 1 << 20) > 0\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
