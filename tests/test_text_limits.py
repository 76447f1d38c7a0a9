"""Sizes at the ends of what the text model's entry points take (no kernel is launched: every call is refused)."""
import ctypes as C

import pytest

from paper_2011_06295_amd import binding as B

LIB = B.raw_library()
A, X, Y, W = 1 << 42, 1 << 43, 1 << 44, 1 << 46        # addresses that are never read


@pytest.mark.parametrize("n, t, dim, dtype, flags", [
    (1 << 25, 2, 1, B.SC_F32, B.SC_EMBED_CHANNELS_FIRST), (1 << 23, 65, 1, B.SC_F16, B.SC_EMBED_CHANNELS_FIRST), (1 << 21, 2, 513, B.SC_F32, B.SC_EMBED_CHANNELS_FIRST),
    (1, (1 << 31) - 1, 64, B.SC_F16, 0), (1 << 15, (1 << 16) - 1, 36, B.SC_F32, 0)])
def test_lookup_of_more_than_a_launch_holds_is_refused(n, t, dim, dtype, flags):
    assert LIB.sparse_conv_embed(A, X, Y, 1000, dim, n, t, dtype, 1.0, flags, None) == B.SC_EUNSUPPORTED


@pytest.mark.parametrize("n, t, dim, flags", [
    (1 << 25, 2, 1, B.SC_EMBED_CHANNELS_FIRST), (1 << 30, 1, 1, 0), (1 << 27, 4, 16, 0), (1 << 25, 8, 513, 0), (1 << 25, 8, 513, B.SC_EMBED_ACCUMULATE)])
def test_gradient_of_more_than_a_launch_holds_is_refused(n, t, dim, flags):
    assert LIB.sparse_conv_embed_backward(A, X, Y, 1000, dim, n, t, B.SC_F32, B.SC_F32, 1.0, -1, flags, W, 1 << 46, None) == B.SC_EUNSUPPORTED


@pytest.mark.parametrize("tokens", [1 << 17, (1 << 20) + 3, 1 << 24, (1 << 29) - 64])
@pytest.mark.parametrize("vocab", [9, 1000, 131072, (1 << 31) - 1])
def test_scratch_memory_of_the_sort_grows_with_the_tokens(tokens, vocab):
    """Keys and places twice, a window of sums for 32 tokens, and counts of a bounded number of workgroups (of 1024 digits at most), for
    every workgroup reads them all."""
    n = C.c_longlong(-1)
    assert LIB.sparse_conv_embed_backward_workspace(vocab, 1, 1, tokens, B.SC_F32, 0, C.byref(n)) == B.SC_OK
    assert 16 * tokens <= n.value <= 16 * tokens + tokens // 8 + 512 * 1024 * 4 + 8 * 256


def test_sizes_whose_bytes_pass_64_bits_are_refused():
    big = (1 << 31) - 1
    assert LIB.sparse_conv_embed(A, X, Y, big, big, 1, 1, B.SC_F32, 1.0, 0, None) == B.SC_EUNSUPPORTED
    assert LIB.sparse_conv_embed(A, X, Y, 1, big, 1, big, B.SC_F32, 1.0, 0, None) == B.SC_EUNSUPPORTED
    n = C.c_longlong(-1)
    for vocab, dim, words in ((big, big, 1), (1, big, big)):
        assert LIB.sparse_conv_embed_backward(A, X, Y, vocab, dim, 1, words, B.SC_F32, B.SC_F32, 1.0, -1, 0, W, 1 << 46, None) == B.SC_EUNSUPPORTED
        assert LIB.sparse_conv_embed_backward_workspace(vocab, dim, 1, words, B.SC_F32, 0, C.byref(n)) == B.SC_EUNSUPPORTED and n.value == -1
    for apart in (1 << 62, 1 << 61, (1 << 45) - 1):
        assert LIB.sparse_conv_int8_quantize(A, X, Y, 3, 100, apart, B.SC_F32, None) == B.SC_EUNSUPPORTED
        for ldx, ldo in ((apart, 5), (100, apart)):
            assert LIB.sparse_conv_int8_linear(A, None, X, Y, None, 1 << 45, 3, 5, 100, ldx, ldo, B.SC_F32, B.SC_F32, 0, W, 1 << 40, None) == B.SC_EUNSUPPORTED


def test_layer_s_scratch_memory_overlaps_no_scales_and_no_bias():
    n = C.c_longlong()
    M, N, K = 1000, 70, 1000
    assert LIB.sparse_conv_int8_linear_workspace(M, N, K, B.SC_F16, B.SC_F16, C.byref(n)) == B.SC_OK and n.value > 4096

    def call(scale=Y, bias=None):
        return LIB.sparse_conv_int8_linear(A, None, X, scale, bias, 1 << 45, M, N, K, K, N, B.SC_F16, B.SC_F16, 0, W, n.value, None)

    for inside in (W, W + 4096, W + n.value - 4, W - 4 * N + 4):
        assert call(scale=inside) == B.SC_EINVAL
        assert call(bias=inside) == B.SC_EINVAL
