"""Forms of the layer's and its gradients' kernels that ordinary sizes take (tiles of either size, the slope worked out as d is loaded, rows of less than
16 bytes, sums split over workgroups), against 64 bits.

Bounds are those of test_gpu_train.py, which says where they come from.  test_train_forms_host.py checks that the sizes of both files reach
every kernel in every form that sizes drawn at large take."""
import pytest

from test_gpu_train import _check_gradient, _check_layer

pytestmark = pytest.mark.gpu

FORM_LAYERS = [  # M, K, N
    (12, 1, 1), (44, 2, 15032), (365, 3605, 357), (174, 10752, 256), (370, 5824, 1088), (5, 15912, 3), (1255, 2816, 1728), (5, 64, 15360), (974, 15168, 1856),
    (2289, 1216, 768)]
FORM_GRADIENTS = [  # M, K, N, activation
    (773, 1, 1, "gelu"), (1, 1, 2396, None), (1, 1, 2396, "relu"), (2405, 1, 1, None), (2405, 1, 1, "relu"), (1, 4, 3393, "relu"), (1, 8, 2896, None), (33, 11218, 1, "relu"),
    (3, 10906, 35, "relu"), (35, 14008, 1, None), (248, 173, 2389, "relu"), (2799, 290, 107, "gelu"), (97, 308, 2936, "gelu"), (4752, 169, 162, None), (71, 320, 4416, None),
    (3801, 320, 128, "relu"), (2551, 98, 628, "relu"), (8426, 269, 1, "gelu"), (13685, 198, 3, "gelu"), (4507, 664, 2, None), (178, 645, 3376, "gelu"), (2318, 704, 384, "relu"),
    (621, 9486, 1, "gelu"), (2004, 1, 2992, "relu"), (3342, 8, 2730, "relu"), (2725, 174, 2378, None), (4025, 1, 1, "relu"), (9, 48, 14667, "relu"), (65, 245, 4100, "relu"),
    (9385, 162, 34, "gelu"), (5309, 384, 4480, "relu"), (407, 2, 9177, "relu"), (910, 3617, 4211, "relu"), (2497, 4, 9970, None), (4081, 64, 5952, None), (3196, 5824, 256, None),
    (2513, 2, 1749, None), (230, 16384, 64, "relu"), (1897, 4, 2786, None), (11003, 525, 1, "gelu"), (2, 15936, 384, "gelu"), (207, 4032, 64, "silu"), (117, 6605, 6, "silu")]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_forms_of_the_layer(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(51)
    for i, (M, K, N) in enumerate(FORM_LAYERS):
        print(f"form of the layer {dtype} {M}x{K} -> {N}", flush=True)
        _check_layer(gen, M, K, N, dtype, (None, "relu", "gelu", "silu")[i % 4], i % 3 == 1, i % 5 != 2, i % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_forms_of_the_gradients(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(52)
    for i, (M, K, N, act) in enumerate(FORM_GRADIENTS):
        print(f"form of the gradients {dtype} {M}x{K} -> {N} {act}", flush=True)
        _check_gradient(gen, M, K, N, dtype, act, i % 2 == 1)
