"""Argument checks of the text model's entry points (no kernel is launched: every call is refused or empty)."""
import ctypes as C

import pytest

from paper_2011_06295_amd import binding as B

LIB = B.raw_library()
A, X, Y, W = 1 << 20, 1 << 24, 1 << 28, 1 << 32        # addresses that are never read


def _embed(table=A, tokens=X, out=Y, vocab=10, dim=4, n=2, t=3, dtype=B.SC_F32, flags=0):
    return LIB.sparse_conv_embed(table, tokens, out, vocab, dim, n, t, dtype, 1.0, flags, None)


@pytest.mark.parametrize("change", [
    {"table": None}, {"tokens": None}, {"out": None}, {"vocab": 0}, {"dim": 0}, {"n": -1}, {"t": -1}, {"dtype": B.SC_I8}, {"dtype": 7}, {"flags": 4},
    {"flags": 8}, {"table": A + 2}, {"out": Y + 1}, {"tokens": X + 2}, {"tokens": X + 4, "flags": 2}, {"out": A + 156}, {"out": X + 20},
    {"dtype": B.SC_BF16, "out": Y + 1}])
def test_lookup_refuses(change):
    assert _embed(**change) == B.SC_EINVAL


def test_lookup_limits_and_empty_calls():
    assert _embed(vocab=1 << 31) == B.SC_EUNSUPPORTED
    assert _embed(n=1 << 16, t=1 << 15) == B.SC_EUNSUPPORTED
    assert _embed(n=0) == B.SC_OK and _embed(t=0, table=None) == B.SC_OK


def _grad(grad=A, tokens=X, out=Y, vocab=10, dim=4, n=2, t=3, g=B.SC_F32, w=B.SC_F32, padding=-1, flags=0, work=W, nbytes=1 << 30):
    return LIB.sparse_conv_embed_backward(grad, tokens, out, vocab, dim, n, t, g, w, 1.0, padding, flags, work, nbytes, None)


@pytest.mark.parametrize("change", [
    {"grad": None}, {"tokens": None}, {"out": None}, {"vocab": 0}, {"dim": -1}, {"n": -1}, {"g": B.SC_I8}, {"g": B.SC_F16, "w": B.SC_BF16}, {"g": B.SC_F32, "w": B.SC_F16},
    {"padding": -2}, {"padding": 10}, {"flags": 8}, {"out": A + 92}, {"out": X + 8}, {"out": Y + 2}, {"grad": A + 1, "g": B.SC_F16}])
def test_gradient_refuses(change):
    assert _grad(**change) == B.SC_EINVAL


def test_gradient_workspace_is_reported_and_checked():
    n = C.c_longlong(-1)
    assert LIB.sparse_conv_embed_backward_workspace(10, 4, 2, 3, B.SC_F32, 0, None) == B.SC_EINVAL
    assert LIB.sparse_conv_embed_backward_workspace(0, 4, 2, 3, B.SC_F32, 0, C.byref(n)) == B.SC_EINVAL and n.value == -1
    for flags in (0, 1, 2, 3):
        for vocab, dim, s, t in [(10, 4, 0, 3), (10, 4, 2, 3), (1000, 300, 128, 64), (100000, 1024, 8, 4096), ((1 << 31) - 1, 8, 1, 100000)]:
            assert LIB.sparse_conv_embed_backward_workspace(vocab, dim, s, t, B.SC_F16, flags, C.byref(n)) == B.SC_OK and n.value >= 0
            if n.value:
                big = dict(vocab=vocab, dim=dim, n=s, t=t, g=B.SC_F16, flags=flags, grad=1 << 44, tokens=1 << 45, out=1 << 46)
                assert _grad(**big, work=None) == B.SC_EINVAL
                assert _grad(**big, nbytes=n.value - 1) == B.SC_EINVAL
                assert _grad(**big, work=W + 4, nbytes=n.value) == B.SC_EINVAL
                assert _grad(**big, work=1 << 46, nbytes=n.value) == B.SC_EINVAL
    assert _grad(n=0, flags=B.SC_EMBED_ACCUMULATE) == B.SC_OK


@pytest.mark.parametrize("change", [
    {"x": None}, {"q": None}, {"scale": None}, {"rows": -1}, {"K": 0}, {"ldx": 99}, {"dtype": B.SC_I8}, {"dtype": -1}, {"q": X + 8}, {"scale": Y + 2}, {"x": A + 2}, {"q": A}])
def test_quantize_refuses(change):
    a = dict(dict(x=A, q=X, scale=Y, rows=3, K=100, ldx=100, dtype=B.SC_F32), **change)
    assert LIB.sparse_conv_int8_quantize(a["x"], a["q"], a["scale"], a["rows"], a["K"], a["ldx"], a["dtype"], None) == B.SC_EINVAL


def _linear(x=A, xs=None, w=X, ws=Y, bias=None, out=W, M=3, N=5, K=100, ldx=100, ldo=5, i=B.SC_F32, o=B.SC_F32, flags=0, work=1 << 36, nbytes=1 << 34):
    return LIB.sparse_conv_int8_linear(x, xs, w, ws, bias, out, M, N, K, ldx, ldo, i, o, flags, work, nbytes, None)


@pytest.mark.parametrize("change", [
    {"x": None}, {"w": None}, {"ws": None}, {"out": None}, {"M": -1}, {"N": 0}, {"K": 0}, {"ldx": 99}, {"ldo": 4}, {"i": 9}, {"o": B.SC_I8}, {"flags": 2}, {"flags": 4},
    {"w": X + 8}, {"ws": Y + 1}, {"out": W + 2}, {"x": A + 2}, {"bias": Y + 65}, {"i": B.SC_I8, "xs": None, "ldx": 128}, {"i": B.SC_I8, "xs": Y + 64, "ldx": 100},
    {"i": B.SC_I8, "xs": Y + 64, "ldx": 128, "x": A + 4}, {"out": A + 40}, {"out": X + 16}, {"out": Y}, {"bias": W}])
def test_layer_refuses(change):
    assert _linear(**change) == B.SC_EINVAL


def test_layer_limits_workspace_and_empty_calls():
    assert _linear(K=131072, ldx=131072) == B.SC_EUNSUPPORTED
    assert _linear(M=1 << 24) == B.SC_EUNSUPPORTED and _linear(N=1 << 24, ldo=1 << 24) == B.SC_EUNSUPPORTED
    assert _linear(M=0, x=None) == B.SC_OK
    n = C.c_longlong(-1)
    assert LIB.sparse_conv_int8_linear_workspace(3, 5, 100, B.SC_F32, B.SC_F32, None) == B.SC_EINVAL
    assert LIB.sparse_conv_int8_linear_workspace(3, 5, 131072, B.SC_F32, B.SC_F32, C.byref(n)) == B.SC_EUNSUPPORTED and n.value == -1
    for M in (1, 4, 5, 16, 100, 1000):
        assert LIB.sparse_conv_int8_linear_workspace(M, 70, 1000, B.SC_F16, B.SC_F16, C.byref(n)) == B.SC_OK and n.value >= 0
        if n.value:
            assert _linear(M=M, N=70, K=1000, ldx=1000, ldo=70, i=B.SC_F16, o=B.SC_F16, work=None) == B.SC_EINVAL
            assert _linear(M=M, N=70, K=1000, ldx=1000, ldo=70, i=B.SC_F16, o=B.SC_F16, nbytes=n.value - 1) == B.SC_EINVAL
            assert _linear(M=M, N=70, K=1000, ldx=1000, ldo=70, i=B.SC_F16, o=B.SC_F16, work=W, nbytes=n.value) == B.SC_EINVAL


def test_pitch_of_rows():
    assert [B.int8_pitch(k) for k in (1, 127, 128, 129, 1000)] == [128, 128, 128, 256, 1024]


def test_convolution_layers_refuse_the_operators_types():
    import numpy as np
    w, m, h = np.ones((2, 3, 3, 3), np.float32), np.ones((2, 3, 3, 3), np.uint8), C.c_void_p()
    for dtype in (B.SC_BF16, B.SC_I8):
        assert LIB.sparse_conv_create(C.byref(h), w.ctypes.data, m.ctypes.data, 2, 3, 3, 3, dtype, 0) == B.SC_EINVAL


def test_every_product_kernel_has_a_layer_in_the_tests():
    from test_gpu_text import LARGE_LAYERS, LAYERS
    choice = LIB["_ZN2sc11int8_kernelEiii"]        # sc::int8_kernel(M, N, K)
    choice.argtypes = [C.c_int] * 3
    reached = {}
    for M, K, N in LAYERS + LARGE_LAYERS:
        reached.setdefault(choice(M, N, K), []).append((M, K, N))
    assert set(reached) == set(range(11)), reached
    assert any(m * n > 256 for m, n in [(-(-M // 256), -(-N // 256)) for M, _, N in reached[7]])      # a workgroup takes several tiles


def test_every_kernel_that_quantises_has_a_layer_in_the_tests():
    from test_gpu_text import LAYERS
    choice = LIB["_ZN2sc15int8_own_kernelEiiii"]        # sc::int8_own_kernel(M, N, K, in_dtype)
    choice.argtypes = [C.c_int] * 4
    n = C.c_longlong()
    for dtype in (B.SC_F32, B.SC_F16, B.SC_BF16):
        reached = {}
        for M, K, N in LAYERS:
            kernel = choice(M, N, K, dtype)
            reached.setdefault(kernel, []).append(M)
            assert LIB.sparse_conv_int8_linear_workspace(M, N, K, dtype, dtype, C.byref(n)) == B.SC_OK and (n.value > 0) == (kernel < 0)
        assert set(reached) == {-1, 0, 1, 2}, reached
        assert all(min(reached[k]) <= 16 < max(reached[k]) for k in (0, 1, 2)), reached


def test_tensor_calls_refuse_before_they_touch_anything():
    """The compiled side of text.py, given what is no CUDA tensor, no tensor, too few arguments."""
    import torch
    from paper_2011_06295_amd import text
    calls = text._calls
    table, tokens = torch.zeros(4, 3), torch.zeros(2, dtype=torch.int64)
    for args in [(table, tokens, None, False, 1.0, 0), (3, tokens, None, False, 1.0, 0), (table, None, None, False, 1.0, 0), (table, tokens, None, False, 1, 0), (table,), ()]:
        with pytest.raises(ValueError):
            calls.embed(*args)
    for args in [(table, table, tokens, None, False, False, 1.0, -1, 0), (table, None, tokens, None, False, False, 1.0, -1, 0), (table,)]:
        with pytest.raises(ValueError):
            calls.embed_backward(*args)
    weight, scale = torch.zeros((2, 128), dtype=torch.int8), torch.zeros(2)
    for args in [(torch.zeros(2, 5), None, weight, scale, None, 4, False, None, None, 0), (torch.zeros((1, 4), dtype=torch.int32), None, weight, scale, None, 4, False, None, None, 0),
                 (torch.zeros(2, 4), None, weight, scale, None, 4, False, torch.zeros(2, 3), None, 0), (torch.zeros(2, 4), None, weight, scale, None, 4, False, None, "f32", 0),
                 (torch.zeros(2, 4), scale, weight, scale, None, 4, False, None, None, 0), (5, None, weight, scale, None, 4, False, None, None, 0), ()]:
        with pytest.raises(ValueError):
            calls.linear(*args)
    with pytest.raises(ValueError):
        text.Embedding(table)
    with pytest.raises(ValueError):
        text.Int8Linear(table)
    with pytest.raises(TypeError):
        calls.bind(1, 2)
