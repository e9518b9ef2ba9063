"""Host-side checks that need no GPU of the operators that complete a layer: sizes, refusals before any device work, workspaces."""
import ctypes

import pytest
import torch

import paper_2107_06876_amd as lcn
from paper_2107_06876_amd import encoder
from paper_2107_06876_amd.binding import BF16, ERR_ALLOC, ERR_INVALID_ARG, F32, OK

FAKE = 256 * 1024   # never read: the calls below are refused before any device work


@pytest.fixture(scope="module")
def lib():
    return encoder._library()


def _bytes(f, *sizes):
    out = ctypes.c_size_t(0)
    return f(*sizes, ctypes.byref(out)), out.value


# ---- layer norm ------------------------------------------------------------------


@pytest.mark.parametrize("rows,dim,dtype", [(-1, 4, F32), (4, 0, F32), (4, 4, 7), (4, (1 << 20) + 1, F32), ((1 << 30) + 1, 4, BF16),
                                            (1 << 30, (1 << 12) + 1, BF16)])
def test_norm_sizes_out_of_range(lib, rows, dim, dtype):
    assert _bytes(lib.lcn_layer_norm_workspace_bytes, rows, dim, dtype)[0] == ERR_INVALID_ARG
    assert lib.lcn_layer_norm(FAKE, FAKE, FAKE, rows, dim, dtype, 1e-5, FAKE, FAKE, FAKE, None) == ERR_INVALID_ARG
    assert lib.lcn_layer_norm_backward(FAKE, FAKE, FAKE, FAKE, FAKE, None, rows, dim, dtype, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                       None) == ERR_INVALID_ARG


def test_norm_arguments(lib):
    for at in (0, 7):
        args = [FAKE, FAKE, FAKE, 20, 60, F32, 1e-5, FAKE, FAKE, FAKE, None]
        args[at] = None
        assert lib.lcn_layer_norm(*args) == ERR_INVALID_ARG
    for eps in (-1e-9, float("nan"), float("inf")):
        assert lib.lcn_layer_norm(FAKE, FAKE, FAKE, 20, 60, F32, eps, FAKE, FAKE, FAKE, None) == ERR_INVALID_ARG
    good = [FAKE, FAKE, FAKE, FAKE, FAKE, None, 20, 60, F32, FAKE, FAKE, FAKE, FAKE, 1 << 40, None]
    for at in (0, 2, 3, 4):
        args = list(good)
        args[at] = None
        assert lib.lcn_layer_norm_backward(*args) == ERR_INVALID_ARG
    st, n = _bytes(lib.lcn_layer_norm_workspace_bytes, 20, 60, F32)
    assert st == OK and n > 0
    for space, size in ((FAKE, n - 1), (None, n), (FAKE + 128, n)):
        args = list(good)
        args[12], args[13] = space, size
        assert lib.lcn_layer_norm_backward(*args) == ERR_ALLOC
    assert _bytes(lib.lcn_layer_norm_workspace_bytes, 0, 60, F32) == (OK, 0)
    assert lib.lcn_layer_norm(None, None, None, 0, 60, F32, 1e-5, None, None, None, None) == OK
    assert lib.lcn_layer_norm_backward(None, None, None, None, None, None, 20, 60, F32, None, None, None, None, 0, None) == OK


def test_norm_of_tensors_that_are_not_on_a_device():
    with pytest.raises(ValueError):
        lcn.lcn_layer_norm(torch.ones(4, 6))
    with pytest.raises(ValueError):
        lcn.lcn_layer_norm_backward(torch.ones(4, 6), None, torch.ones(4), torch.ones(4), torch.ones(4, 6))


# ---- gated layer -----------------------------------------------------------------


@pytest.mark.parametrize("rows,d_in,d_out,dtype", [
    (-1, 4, 4, F32), (4, 0, 4, F32), (4, 4, 0, F32), (4, 4, 4, 7), (4, (1 << 20) + 1, 4, F32), (4, 4, (1 << 19) + 1, F32),
    ((1 << 30) + 1, 4, 4, BF16), (1 << 30, 8, (1 << 11) + 1, BF16), (1 << 30, (1 << 12) + 1, 8, BF16)])
def test_gated_sizes_out_of_range(lib, rows, d_in, d_out, dtype):
    for backward in (0, 1):
        assert _bytes(lib.lcn_gated_linear_workspace_bytes, rows, d_in, d_out, dtype, backward)[0] == ERR_INVALID_ARG
    assert lib.lcn_gated_linear(FAKE, FAKE, None, rows, d_in, d_out, dtype, 0, FAKE, None, FAKE, 1 << 62, None) == ERR_INVALID_ARG
    assert lib.lcn_gated_linear_backward(FAKE, FAKE, FAKE, FAKE, rows, d_in, d_out, dtype, 0, FAKE, FAKE, None, FAKE, 1 << 62,
                                         None) == ERR_INVALID_ARG


def test_gated_arguments(lib):
    good = [FAKE, FAKE, None, 20, 600, 600, F32, 4, FAKE, None, FAKE, 1 << 40, None]
    for at in (0, 1, 8):
        bad = list(good)
        bad[at] = None
        assert lib.lcn_gated_linear(*bad) == ERR_INVALID_ARG
    for act in (-1, 5):
        bad = list(good)
        bad[7] = act
        assert lib.lcn_gated_linear(*bad) == ERR_INVALID_ARG
    good = [FAKE, FAKE, FAKE, FAKE, 20, 60, 60, F32, 4, FAKE, FAKE, None, FAKE, 1 << 40, None]
    for at in range(4):
        bad = list(good)
        bad[at] = None
        assert lib.lcn_gated_linear_backward(*bad) == ERR_INVALID_ARG
    bad = list(good)
    bad[8] = 5
    assert lib.lcn_gated_linear_backward(*bad) == ERR_INVALID_ARG
    assert lib.lcn_gated_linear_backward(None, None, None, None, 20, 60, 60, F32, 4, None, None, None, None, 0, None) == OK


def test_gated_kept(lib):
    """Rows of both sums in whole pieces of eight: floats, or 16 bits a value; aligned."""
    f = lib.lcn_gated_linear_kept_bytes
    assert _bytes(f, 10, 24, F32) == (OK, 10 * 2 * 24 * 4) and _bytes(f, 10, 20, BF16) == (OK, 10 * 2 * 24 * 2)
    assert _bytes(f, 0, 20, BF16) == (OK, 0)
    for rows, d_out, dtype in ((-1, 4, F32), (4, 0, F32), (4, 4, 3), (4, (1 << 19) + 1, F32), (1 << 30, (1 << 11) + 1, BF16)):
        assert _bytes(f, rows, d_out, dtype)[0] == ERR_INVALID_ARG
    args = [FAKE, FAKE, None, 20, 600, 600, F32, 4, FAKE, FAKE + 8, FAKE, 1 << 40, None]
    assert lib.lcn_gated_linear(*args) == ERR_INVALID_ARG
    args = [FAKE, FAKE, FAKE + 8, FAKE, 20, 60, 60, F32, 4, FAKE, FAKE, None, FAKE, 1 << 40, None]
    assert lib.lcn_gated_linear_backward(*args) == ERR_INVALID_ARG


def test_gated_workspaces(lib):
    for dtype in (F32, BF16):
        for rows, a, b in ((1, 16, 16), (20, 300, 600), (5000, 300, 20000), (70000, 1024, 4096)):
            st, n = _bytes(lib.lcn_gated_linear_workspace_bytes, rows, a, b, dtype, 0)
            assert st == OK and (n == 0) == (rows <= 8 or (rows == 20 and dtype == F32))   # those that read W as it lies
            if n:
                assert lib.lcn_gated_linear(FAKE, FAKE, None, rows, a, b, dtype, 4, FAKE, None, FAKE, n - 1, None) == ERR_ALLOC
                assert lib.lcn_gated_linear(FAKE, FAKE, None, rows, a, b, dtype, 4, FAKE, None, FAKE + 64, n, None) == ERR_ALLOC
            st, n = _bytes(lib.lcn_gated_linear_workspace_bytes, rows, a, b, dtype, 1)
            assert st == OK and n > 0
            assert lib.lcn_gated_linear_backward(FAKE, FAKE, FAKE, FAKE, rows, a, b, dtype, 4, FAKE, FAKE, None, FAKE, n - 1,
                                                 None) == ERR_ALLOC
    assert _bytes(lib.lcn_gated_linear_workspace_bytes, 0, 4, 4, F32, 1) == (OK, 0)


def test_gated_tensors_that_are_not_on_a_device():
    with pytest.raises(ValueError):
        lcn.lcn_gated_linear(torch.ones(4, 6), torch.ones(4, 6))


# ---- orthogonalisation -----------------------------------------------------------


def _triples(*c):
    return (ctypes.c_float * len(c))(*c)


UPDATE = _triples(*(3.4445, -4.7750, 2.0315) * 5)


@pytest.mark.parametrize("count,rows,cols,dtype", [
    (-1, 4, 4, F32), (1, 0, 4, F32), (1, 4, 0, F32), (1, 4, 4, 7), ((1 << 20) + 1, 4, 4, F32), (1, (1 << 20) + 1, 4, F32),
    (1, 4, (1 << 20) + 1, F32), (1, 32769, 32769, BF16), (1 << 20, 1 << 10, (1 << 10) + 1, BF16),
    (1 << 20, 1, 1 << 17, BF16)])
def test_orthogonal_sizes_out_of_range(lib, count, rows, cols, dtype):
    assert _bytes(lib.lcn_orthogonalise_workspace_bytes, count, rows, cols, dtype)[0] == ERR_INVALID_ARG
    assert lib.lcn_orthogonalise(FAKE, count, rows, cols, dtype, 5, UPDATE, 1e-7, 1.0, FAKE, FAKE, 1 << 62, None) == ERR_INVALID_ARG


def test_orthogonal_arguments(lib):
    good = [FAKE, 1, 200, 600, F32, 5, UPDATE, 1e-7, 1.0, FAKE, FAKE, 0, None]
    for at, value in ((0, None), (6, None), (9, None), (5, 0), (5, 65), (7, -1.0), (7, float("nan")), (7, float("inf")),
                      (8, float("inf")), (8, float("nan"))):
        bad = list(good)
        bad[at] = value
        assert lib.lcn_orthogonalise(*bad) == ERR_INVALID_ARG
    for c in (_triples(4.1, 0.0, 0.0), _triples(float("nan"), 0.0, 0.0), _triples(1.0, float("inf"), 0.0), _triples(70.0, -1000.0, 1000.0),
              _triples(0.0, 0.0, 4.5), _triples(3.0, -8.0, 12.0)):
        bad = list(good)
        bad[5], bad[6] = 1, c
        assert lib.lcn_orthogonalise(*bad) == ERR_INVALID_ARG
    # values that a first step lets grow are seen by the next: 2 s four times over leaves 16
    bad = list(good)
    bad[5], bad[6] = 4, _triples(*(2.0, 0.0, 0.0) * 4)
    assert lib.lcn_orthogonalise(*bad) == ERR_INVALID_ARG
    for c in (_triples(4.0, 0.0, 0.0), _triples(3.4445, -4.7750, 2.0315), _triples(1.5, -0.5, 0.0), _triples(0.0, 0.0, 0.0)):
        ok = list(good)
        ok[5], ok[6] = 1, c
        assert lib.lcn_orthogonalise(*ok) == ERR_ALLOC


def test_orthogonal_workspaces(lib):
    for dtype in (F32, BF16):
        for count, rows, cols in ((1, 20, 60), (8, 96, 32), (1, 300, 300), (4, 8192, 1024)):
            st, n = _bytes(lib.lcn_orthogonalise_workspace_bytes, count, rows, cols, dtype)
            assert st == OK
            if n:
                for space, size in ((FAKE, n - 1), (None, n), (FAKE + 64, n)):
                    assert lib.lcn_orthogonalise(FAKE, count, rows, cols, dtype, 5, UPDATE, 1e-7, 1.0, FAKE, space, size,
                                                 None) == ERR_ALLOC
    assert _bytes(lib.lcn_orthogonalise_workspace_bytes, 0, 4, 4, F32) == (OK, 0)
    assert lib.lcn_orthogonalise(None, 0, 4, 4, F32, 5, UPDATE, 1e-7, 1.0, None, None, 0, None) == OK


def test_orthogonal_tensors_that_are_not_on_a_device():
    with pytest.raises(ValueError):
        lcn.lcn_orthogonalise(torch.ones(4, 6))
