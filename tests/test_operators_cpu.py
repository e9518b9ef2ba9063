"""Host-side checks of the encoder operators that need no GPU: sizes, refusals before any device work, workspaces."""
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


def test_exported():
    for name in ("lcn_linear", "lcn_linear_backward", "lcn_cross_entropy", "lcn_cross_entropy_backward", "lcn_attention",
                 "lcn_attention_backward", "ACT_NONE", "ACT_TANH", "ACT_RELU", "ACT_GELU", "ACT_SILU"):
        assert hasattr(lcn, name)


@pytest.mark.parametrize("sizes", [(-1, 4, 4, F32), (4, 0, 4, F32), (4, 4, 0, F32), (4, 4, 4, 7), (4, (1 << 20) + 1, 4, F32),
                                   ((1 << 30) + 1, 4, 4, BF16)])
def test_sizes_out_of_range(lib, sizes):
    rows, d_in, d_out, dtype = sizes
    assert _bytes(lib.lcn_linear_workspace_bytes, rows, d_in, d_out, dtype, 0)[0] == ERR_INVALID_ARG
    assert lib.lcn_linear(FAKE, FAKE, None, None, rows, d_in, d_out, dtype, 0, FAKE, None, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    assert lib.lcn_linear_backward(FAKE, FAKE, FAKE, FAKE, rows, d_in, d_out, dtype, 0, FAKE, FAKE, None, FAKE, 1 << 30,
                                   None) == ERR_INVALID_ARG
    vocab, dim = d_out, d_in
    assert _bytes(lib.lcn_cross_entropy_workspace_bytes, rows, vocab, dim, dtype, 1)[0] == ERR_INVALID_ARG
    assert lib.lcn_cross_entropy(FAKE, FAKE, None, FAKE, rows, vocab, dim, dtype, 1.0, FAKE, FAKE, FAKE, 1 << 30,
                                 None) == ERR_INVALID_ARG
    assert lib.lcn_cross_entropy_backward(FAKE, FAKE, None, FAKE, FAKE, FAKE, rows, vocab, dim, dtype, 1.0, FAKE, FAKE, None,
                                          FAKE, 1 << 30, None) == ERR_INVALID_ARG


def test_null_pointers_and_activations(lib):
    good = [FAKE, FAKE, None, None, 20, 600, 600, F32, 0, FAKE, None, FAKE, 1 << 30, None]
    for at in (0, 1, 9):
        bad = list(good)
        bad[at] = None
        assert lib.lcn_linear(*bad) == ERR_INVALID_ARG
    for act in (-1, 5):
        bad = list(good)
        bad[8] = act
        assert lib.lcn_linear(*bad) == ERR_INVALID_ARG
    # an activation's gradient needs z, dw needs x, dx needs W
    assert lib.lcn_linear_backward(FAKE, FAKE, None, FAKE, 20, 60, 60, F32, 1, FAKE, FAKE, None, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    assert lib.lcn_linear_backward(None, FAKE, FAKE, FAKE, 20, 60, 60, F32, 1, FAKE, FAKE, None, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    assert lib.lcn_linear_backward(FAKE, None, FAKE, FAKE, 20, 60, 60, F32, 1, FAKE, FAKE, None, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    for at in (0, 1, 3, 9, 10):
        bad = [FAKE, FAKE, None, FAKE, 20, 60, 60, F32, 1.0, FAKE, FAKE, FAKE, 1 << 30, None]
        bad[at if at < 9 else at] = None
        assert lib.lcn_cross_entropy(*bad) == ERR_INVALID_ARG
    assert lib.lcn_cross_entropy(FAKE, FAKE, None, FAKE, 20, 60, 60, F32, float("nan"), FAKE, FAKE, FAKE, 1 << 30, None) == ERR_INVALID_ARG


def test_workspaces(lib):
    for dtype in (F32, BF16):
        for backward in (0, 1):
            for rows, a, b in ((1, 16, 16), (20, 300, 600), (5000, 300, 20000), (70000, 1024, 4096)):
                st, n = _bytes(lib.lcn_linear_workspace_bytes, rows, a, b, dtype, backward)
                assert st == OK
                if n:   # one byte less is refused
                    args = ([FAKE, FAKE, None, None, rows, a, b, dtype, 0, FAKE, None, FAKE, n - 1, None] if not backward else
                            [FAKE, FAKE, FAKE, FAKE, rows, a, b, dtype, 0, FAKE, FAKE, None, FAKE, n - 1, None])
                    f = lib.lcn_linear_backward if backward else lib.lcn_linear
                    assert f(*args) == ERR_ALLOC
                st, n = _bytes(lib.lcn_cross_entropy_workspace_bytes, rows, b, a, dtype, backward)
                assert st == OK and n > 0
                assert lib.lcn_cross_entropy(FAKE, FAKE, None, FAKE, rows, b, a, dtype, 1.0, FAKE, FAKE, FAKE, 8, None) == ERR_ALLOC
    # G of a piece, not of the whole vocabulary: 200 000 words by 100 000 rows would be 40 GB
    st, n = _bytes(lib.lcn_cross_entropy_workspace_bytes, 100000, 200000, 300, BF16, 1)
    assert st == OK and n < 4 << 30
    assert _bytes(lib.lcn_linear_workspace_bytes, 0, 4, 4, F32, 1) == (OK, 0)


def _desc(**kw):
    d = encoder.AttentionDesc(2, 4, 2, 32, BF16, 1, 0.1, 0.0, 100, 300, 0, FAKE, FAKE, None, None, 0, 0, 0, 0, 0, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


@pytest.mark.parametrize("bad", [
    dict(num_sets=-1), dict(heads=0), dict(kv_heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=129), dict(dtype=2),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(total_q=-1),
    dict(total_k=(1 << 30) + 1), dict(max_q=-1), dict(q_off=None), dict(k_off=None), dict(q_token=-1), dict(v_head=(1 << 22) + 1)])
def test_attention_descriptions(lib, bad):
    out = ctypes.c_size_t(0)
    assert lib.lcn_attention_workspace_bytes(_desc(**bad), 0, ctypes.byref(out)) == ERR_INVALID_ARG
    assert lib.lcn_attention(_desc(**bad), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    assert lib.lcn_attention_backward(_desc(**bad), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30,
                                      None) == ERR_INVALID_ARG


def test_attention_pointers_and_workspaces(lib):
    assert lib.lcn_attention(None, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None) == ERR_INVALID_ARG
    for at in range(1, 6):
        args = [_desc(), FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None]
        args[at] = None
        assert lib.lcn_attention(*args) == ERR_INVALID_ARG
    # dk and dv come together
    assert lib.lcn_attention_backward(_desc(), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 30, None) == ERR_INVALID_ARG
    out = ctypes.c_size_t(0)
    assert lib.lcn_attention_workspace_bytes(_desc(), 1, ctypes.byref(out)) == OK and out.value >= 4 * 100 * 4
    assert lib.lcn_attention_backward(_desc(), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, out.value - 1,
                                      None) == ERR_ALLOC
    single = dict(total_q=2, max_q=1, total_k=60000)
    assert lib.lcn_attention_workspace_bytes(_desc(**single), 0, ctypes.byref(out)) == OK and out.value > 0
    assert lib.lcn_attention(_desc(**single), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, out.value - 1, None) == ERR_ALLOC


def test_tensors_that_are_not_on_a_device():
    x, w = torch.ones(4, 6), torch.ones(3, 6)
    with pytest.raises(ValueError):
        lcn.lcn_linear(x, w)
    with pytest.raises(ValueError):
        lcn.lcn_cross_entropy(x, w, torch.zeros(4, dtype=torch.int64))
    q, o = torch.ones(4, 2, 8), torch.tensor([0, 4])
    with pytest.raises(ValueError):
        lcn.lcn_attention(q, q, q, o, o)


@pytest.mark.parametrize("rows,a,b", [(1 << 30, 8, (1 << 12) + 1), (1 << 30, (1 << 12) + 1, 8), (1 << 23, 16, 1 << 20)])
def test_results_with_more_tiles_than_are_numbered(lib, rows, a, b):
    for f in (lib.lcn_linear_workspace_bytes, lambda rows, a, b, *more: lib.lcn_cross_entropy_workspace_bytes(rows, b, a, *more)):
        for backward in (0, 1):
            assert _bytes(f, rows, a, b, BF16, backward)[0] == ERR_INVALID_ARG
            assert _bytes(f, rows // 2, a, b // 2 + 1 if b > a else b, BF16, backward)[0] == OK
    assert lib.lcn_linear(FAKE, FAKE, None, None, rows, a, b, BF16, 0, FAKE, None, FAKE, 1 << 62, None) == ERR_INVALID_ARG
    assert lib.lcn_cross_entropy(FAKE, FAKE, None, FAKE, rows, b, a, BF16, 1.0, FAKE, FAKE, FAKE, 1 << 62, None) == ERR_INVALID_ARG


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (4, 1), (8, 1)])
def test_a_largest_number_of_queries_beyond_all_queries(lib, heads, kv_heads):
    """max_q says no more than total_q does; times the heads of a group it must not wrap around."""
    def space(max_q):
        out = ctypes.c_size_t(0)
        assert lib.lcn_attention_workspace_bytes(_desc(heads=heads, kv_heads=kv_heads, total_q=3, total_k=600, max_q=max_q), 0,
                                                 ctypes.byref(out)) == OK
        return out.value
    want = space(3)
    assert want > 0
    for max_q in (4, 1 << 20, 1 << 59, 1 << 61, 1 << 62, (1 << 63) - 1):
        assert space(max_q) == want


def test_backward_workspaces_of_a_cross_entropy(lib):
    for dtype in (F32, BF16):
        for rows, dim, vocab in ((1, 16, 16), (20, 300, 600), (5000, 300, 20000), (70000, 1024, 4096)):
            st, n = _bytes(lib.lcn_cross_entropy_workspace_bytes, rows, vocab, dim, dtype, 1)
            assert st == OK and n > 0
            assert lib.lcn_cross_entropy_backward(FAKE, FAKE, None, FAKE, FAKE, FAKE, rows, vocab, dim, dtype, 1.0, FAKE, FAKE, FAKE,
                                                  FAKE, n - 1, None) == ERR_ALLOC


@pytest.mark.parametrize("clear", [-1, 2])
def test_a_description_clears_or_not(lib, clear):
    out = ctypes.c_size_t(0)
    assert lib.lcn_attention_workspace_bytes(_desc(clear=clear), 0, ctypes.byref(out)) == ERR_INVALID_ARG
    for good in (0, 1):
        assert lib.lcn_attention_workspace_bytes(_desc(clear=good), 0, ctypes.byref(out)) == OK
