"""Every kernel of the layer and its gradients, in every form that sizes drawn at large take, is one that a GPU test compares with 64 bits; refusals.  Needs no GPU."""
import ctypes as C
import math
import random

import pytest

from paper_2011_06295_amd import binding as B
from test_gpu_train import ACTIVATIONS, GRADIENTS, LARGE_GRADIENTS, LARGE_LAYERS, LAYERS
from test_gpu_train_forms import FORM_GRADIENTS, FORM_LAYERS

LIB = B.raw_library()
ACT = {None: B.SC_ACT_NONE, "relu": B.SC_ACT_RELU, "gelu": B.SC_ACT_GELU, "silu": B.SC_ACT_SILU}


def _function(name, numbers):
    f = LIB[f"_ZN2sc{len(name)}{name}E" + "i" * numbers]          # sc::name(int, ...)
    f.argtypes = [C.c_int] * numbers
    return f


LAYER, LAYER_FORM = _function("linear_kernel", 4), _function("linear_form", 4)
GRADIENT, GRADIENT_FORM = _function("linear_grad_kernel", 5), _function("linear_grad_form", 5)


def _layer(dtype, M, K, N):
    return LAYER(dtype, M, N, K), LAYER_FORM(dtype, M, N, K)


def _gradients(dtype, M, K, N, act):
    """One launch: its kernel and form; laid out: the two products' kernels, and whether their sums are split."""
    kernel, form = GRADIENT(dtype, M, N, K, ACT[act]), GRADIENT_FORM(dtype, M, N, K, ACT[act])
    return {("both", kernel, form)} if kernel < 1000 else {("x", kernel // 1000, form & 8), ("w", kernel % 1000, form & 16)}


def _drawn(count):
    rng = random.Random(1)

    def size():
        return int(round(math.exp(rng.uniform(0.0, math.log(16384.0)))))
    for _ in range(count):
        sizes = [size(), size(), size()]
        if rng.random() < 0.6:
            sizes[1:] = [-(-v // 64) * 64 for v in sizes[1:]]
        if math.prod(sizes) <= 2 ** 39:
            yield sizes


@pytest.mark.parametrize("dtype", [B.SC_F32, B.SC_F16, B.SC_BF16])
def test_drawn_sizes_take_no_form_that_is_not_tested(dtype):
    layers = {_layer(dtype, *sizes) for sizes in LAYERS + LARGE_LAYERS + FORM_LAYERS}
    gradients = set()
    for i, sizes in enumerate(GRADIENTS):          # the activations that test_gpu_train.py gives them
        gradients |= _gradients(dtype, *sizes, ACTIVATIONS[i % 4]) | _gradients(dtype, *sizes, ACTIVATIONS[(i + 2) % 4])
    for i, sizes in enumerate(LARGE_GRADIENTS):
        gradients |= _gradients(dtype, *sizes, ACTIVATIONS[(i + 2) % 4])
    for case in FORM_GRADIENTS:
        gradients |= _gradients(dtype, *case)
    for sizes in _drawn(8000):
        assert _layer(dtype, *sizes) in layers, sizes
        for act in ACTIVATIONS:
            assert _gradients(dtype, *sizes, act) <= gradients, (sizes, act)
    # (both tiles, with and without the slope in them, short rows, every way to split the sums)
    forms = {form for kind, _, form in gradients if kind == "both"}
    assert {f & 5 for f in forms} == {0, 1, 4, 5} and {f & 7 for f in forms} >= {2, 3, 6, 7} and {f & 24 for f in forms} == {0, 8, 16, 24}


def test_first_moments_of_8_bits_need_a_beta_that_moves_them():
    tensors = (B.AdamwTensor * 1)()

    def step(beta1, state, count=0):
        return LIB.sparse_conv_adamw(tensors, count, B.SC_F32, B.SC_F32, state, 1e-3, beta1, 0.999, 1e-8, 0.0, 1.0, 1, None, None)
    for beta1 in (0.0, 0.5, 0.9):
        assert step(beta1, B.SC_E4M3) == step(beta1, B.SC_F32) == B.SC_OK
    for beta1 in (0.900001, 0.95, 0.99):
        assert step(beta1, B.SC_E4M3) == step(beta1, B.SC_E4M3, 1) == B.SC_EUNSUPPORTED and step(beta1, B.SC_F32) == B.SC_OK
