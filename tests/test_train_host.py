"""Argument checks of the layer's, the loss's and the AdamW step's entry points (no kernel is launched: every call is refused or empty)."""
import ctypes as C

import pytest

from paper_2011_06295_amd import binding as B

LIB = B.raw_library()
X, W, BIAS, R, OUT, Z, WORK = (1 << n for n in (40, 41, 42, 43, 44, 45, 46))        # addresses that are never read
F32, F16, BF16 = B.SC_F32, B.SC_F16, B.SC_BF16


def _linear(x=X, w=W, bias=BIAS, residual=None, out=OUT, z=None, M=3, N=5, K=64, ldx=64, ldw=64, ldr=5, ldo=5, dtype=F32, act=0, work=WORK, nbytes=1 << 30):
    return LIB.sparse_conv_linear(x, w, bias, residual, out, z, M, N, K, ldx, ldw, ldr, ldo, dtype, act, work, nbytes, None)


@pytest.mark.parametrize("change", [
    {"x": None}, {"w": None}, {"out": None}, {"M": -1}, {"N": 0}, {"K": 0}, {"ldx": 63}, {"ldw": 63}, {"ldo": 4}, {"residual": R, "ldr": 4}, {"dtype": B.SC_I8}, {"dtype": 9},
    {"dtype": -1}, {"act": 4}, {"act": -1}, {"x": X + 2}, {"w": W + 1}, {"bias": BIAS + 2}, {"out": OUT + 2}, {"z": Z + 1}, {"residual": R + 3}, {"dtype": F16, "out": OUT + 1},
    {"out": X}, {"out": X + 3 * 64 * 4 - 4}, {"out": W + 4}, {"out": BIAS}, {"out": BIAS + 16}, {"z": OUT}, {"z": OUT + 4}, {"z": X}, {"z": W}, {"z": BIAS}, {"residual": R, "z": R},
    {"residual": OUT + 4}, {"residual": OUT, "ldr": 6, "ldo": 5}])
def test_layer_refuses(change):
    assert _linear(**change) == B.SC_EINVAL


def test_layer_limits_workspace_and_empty_calls():
    for name in ("M", "N", "K"):
        big = {name: (1 << 20) + 1, "ldx": 1 << 21, "ldw": 1 << 21, "ldo": 1 << 21}
        assert _linear(**big) == B.SC_EUNSUPPORTED
    for name in ("ldx", "ldw", "ldo"):
        assert _linear(**{name: 1 << 31}) == B.SC_EUNSUPPORTED
    assert _linear(M=1 << 20, N=1 << 16, ldo=1 << 16) == B.SC_EUNSUPPORTED and _linear(N=1 << 20, K=1 << 16, ldx=1 << 16, ldw=1 << 16, ldo=1 << 20) == B.SC_EUNSUPPORTED
    assert _linear(M=0, x=None) == B.SC_OK
    n = C.c_longlong(-1)

    def need(x=X, w=W, M=3, N=5, K=64, ldx=64, ldw=64, dtype=F32):
        assert LIB.sparse_conv_linear_workspace(x, w, M, N, K, ldx, ldw, dtype, C.byref(n)) == B.SC_OK
        return n.value
    assert LIB.sparse_conv_linear_workspace(X, W, 3, 5, 64, 64, 64, F32, None) == B.SC_EINVAL
    assert LIB.sparse_conv_linear_workspace(X, W, 3, 5, 64, 63, 64, F32, C.byref(n)) == B.SC_EINVAL and n.value == -1
    assert need() == 0 and need(M=0) == 0 and need(M=1, ldx=77) == 0 and need(x=X + 4) == 0          # few rows are read as they lie
    big = dict(M=4000, N=1501, K=1024, ldx=1024, ldw=1024, dtype=F16)
    whole = need(**big)
    for change, rows in (({"x": X + 2}, 4000), ({"w": W + 2}, 1501), ({"ldx": 1025}, 4000), ({"ldw": 1030}, 1501), ({"K": 1023}, 5501)):
        assert need(**dict(big, **change)) >= whole + rows * 2048
    for change in ({"x": X + 2}, {"ldw": 1030}, {"K": 1023}):
        case = dict(big, **change)
        size = need(**case)
        case.update(ldr=1501, ldo=1501)
        assert _linear(**case, work=None) == B.SC_EINVAL and _linear(**case, nbytes=size - 1) == B.SC_EINVAL and _linear(**case, work=WORK + 8) == B.SC_EINVAL
        for inside in (X, W, BIAS, OUT):
            assert _linear(**case, work=inside, nbytes=size) == B.SC_EINVAL
        assert _linear(**case, z=Z, work=Z) == B.SC_EINVAL and _linear(**case, residual=R, work=R) == B.SC_EINVAL


def _backward(grad=R, z=Z, x=X, w=W, gx=OUT, gw=1 << 47, gb=1 << 48, M=3, N=5, K=64, ldg=5, ldx=64, ldw=64, dtype=F32, act=2, flags=0, work=WORK, nbytes=1 << 30):
    return LIB.sparse_conv_linear_backward(grad, z, x, w, gx, gw, gb, M, N, K, ldg, ldx, ldw, dtype, act, flags, work, nbytes, None)


@pytest.mark.parametrize("change", [
    {"grad": None}, {"z": None}, {"x": None}, {"w": None}, {"M": -1}, {"N": 0}, {"K": 0}, {"ldg": 4}, {"ldx": 63}, {"ldw": 1}, {"dtype": B.SC_I8}, {"act": 5}, {"flags": 2}, {"flags": 3},
    {"grad": R + 2}, {"z": Z + 2}, {"x": X + 1}, {"w": W + 2}, {"gx": OUT + 2}, {"gw": (1 << 47) + 2}, {"gb": (1 << 48) + 2}, {"gx": R}, {"gx": X}, {"gx": W + 64}, {"gx": Z},
    {"gw": W}, {"gw": OUT + 4}, {"gb": OUT}, {"gb": 1 << 47}, {"gb": R}])
def test_gradient_refuses(change):
    assert _backward(**change) == B.SC_EINVAL


@pytest.mark.parametrize("change", [{"work": None}, {"nbytes": 16}, {"work": WORK + 4}, {"work": R}, {"work": X}, {"work": W}, {"work": Z}, {"work": OUT}, {"work": 1 << 47}, {"work": 1 << 48}])
def test_gradient_refuses_scratch_memory(change):
    n = C.c_longlong(-1)
    assert LIB.sparse_conv_linear_backward_workspace(R, X, W, OUT, 1 << 47, 1 << 48, 4000, 1500, 1024, 1500, 1024, 1024, F16, 2, C.byref(n)) == B.SC_OK and n.value > 4000 * 1500 * 2
    assert _backward(**dict(dict(M=4000, N=1500, K=1024, ldg=1500, ldx=1024, ldw=1024, dtype=F16, nbytes=n.value), **change)) == B.SC_EINVAL


def test_gradient_limits_and_empty_calls():
    assert _backward(M=(1 << 20) + 1) == B.SC_EUNSUPPORTED and _backward(N=1 << 21, ldg=1 << 21) == B.SC_EUNSUPPORTED and _backward(ldg=1 << 31) == B.SC_EUNSUPPORTED
    assert _backward(M=0, flags=B.SC_LINEAR_ACCUMULATE, grad=None, x=None, w=None, z=None, work=None) == B.SC_OK
    assert _backward(gx=None, gw=None, gb=None, grad=None, x=None, w=None, act=0, z=None, work=None, nbytes=0) == B.SC_OK
    n = C.c_longlong(-1)
    sizes = []
    for wanted in range(8):
        p = [1 << 47 if wanted >> i & 1 else None for i in range(3)]
        assert LIB.sparse_conv_linear_backward_workspace(R, X, W, *p, 300, 50, 70, 50, 70, 70, F16, 2, C.byref(n)) == B.SC_OK
        sizes.append(n.value)
    assert sizes[0] == 0 and max(sizes) == sizes[7] >= 0
    assert LIB.sparse_conv_linear_backward_workspace(R, X, W, OUT, OUT, OUT, 300, 50, 70, 49, 70, 70, F16, 2, C.byref(n)) == B.SC_EINVAL


def _loss(logits=X, labels=W, weights=None, loss=OUT, grad=Z, rows=3, classes=10, ldl=10, ldg=10, dtype=F32, flags=0):
    return LIB.sparse_conv_cross_entropy(logits, labels, weights, loss, grad, rows, classes, ldl, ldg, dtype, 1.0, flags, None)


@pytest.mark.parametrize("change", [
    {"logits": None}, {"labels": None}, {"loss": None}, {"rows": -1}, {"classes": 0}, {"ldl": 9}, {"ldg": 9}, {"dtype": B.SC_I8}, {"flags": 2}, {"logits": X + 2}, {"labels": W + 2},
    {"labels": W + 4, "flags": 1}, {"weights": R + 1}, {"loss": OUT + 2}, {"grad": Z + 2}, {"loss": X}, {"loss": W + 8}, {"loss": Z + 116}, {"weights": OUT}, {"grad": X + 4},
    {"grad": X, "ldg": 11}, {"grad": W}, {"weights": R, "grad": R}])
def test_loss_refuses(change):
    assert _loss(**change) == B.SC_EINVAL


def test_loss_limits_and_empty_calls():
    assert _loss(rows=0, logits=None) == B.SC_OK
    big = 0x7fffffff - (1 << 20) + 1
    assert _loss(classes=big, ldl=big, ldg=big) == B.SC_EUNSUPPORTED and _loss(rows=big) == B.SC_EUNSUPPORTED
    assert _loss(ldl=1 << 45) == B.SC_EUNSUPPORTED and _loss(ldg=1 << 45) == B.SC_EUNSUPPORTED
    assert _loss(logits=1 << 50, rows=(1 << 26) + 1, classes=2000, ldl=2000, grad=None) == B.SC_EUNSUPPORTED       # more workgroups than a launch counts


def _tensor(**change):
    a = dict(dict(param=X, grad=W, m=R, v=OUT, m_scale=Z, v_scale=WORK, master=None, count=300), **change)
    return B.AdamwTensor(**a)


def _adamw(tensors, p=F32, g=F32, s=F32, rate=1e-3, b1=0.9, b2=0.999, eps=1e-8, decay=0.0, scale=1.0, step=1, counted=None, count=None):
    array = (B.AdamwTensor * max(1, len(tensors)))(*tensors)
    return LIB.sparse_conv_adamw(array, len(tensors) if count is None else count, p, g, s, rate, b1, b2, eps, decay, scale, step, counted, None)


@pytest.mark.parametrize("change", [
    {"param": None}, {"grad": None}, {"m": None}, {"v": None}, {"param": X + 2}, {"grad": W + 1}, {"m": R + 2}, {"v": OUT + 1}, {"count": -1}, {"grad": X}, {"m": X + 1196}, {"v": R},
    {"master": X}, {"master": Z + 2}])
def test_step_refuses_tensors(change):
    assert _adamw([_tensor(**change)]) == B.SC_EINVAL
    assert _adamw([_tensor(param=1 << 50, grad=1 << 51, m=1 << 52, v=1 << 53, master=change.get("master") and 1 << 54), _tensor(**change)]) == B.SC_EINVAL


@pytest.mark.parametrize("change", [{"m_scale": None}, {"v_scale": None}, {"m_scale": Z + 2}, {"v_scale": Z + 4}, {"m_scale": R}, {"v_scale": R + 296}])
def test_step_refuses_scales_of_8_bit_states(change):
    assert _adamw([_tensor(**change)], s=B.SC_E4M3) == B.SC_EINVAL


@pytest.mark.parametrize("change", [
    {"p": B.SC_I8}, {"g": 7}, {"s": F16}, {"s": B.SC_I8}, {"p": F16, "g": BF16}, {"p": BF16, "g": F16}, {"rate": -1.0}, {"rate": float("nan")}, {"rate": float("inf")}, {"b1": 1.0}, {"b1": -0.1},
    {"b2": 1.0}, {"b2": float("nan")}, {"eps": -1e-9}, {"decay": -0.1}, {"scale": float("inf")}, {"step": 0}, {"step": -3}, {"counted": Z + 8}, {"count": -1}])
def test_step_refuses(change):
    assert _adamw([_tensor()], **change) == B.SC_EINVAL


def test_step_limits_and_empty_calls():
    assert _adamw([]) == B.SC_OK
    assert _adamw([_tensor(count=0, param=None, grad=None, m=None, v=None)] * 3) == B.SC_OK
    assert _adamw([_tensor(), _tensor(master=1 << 50)]) == B.SC_EINVAL           # all with, or all without
    assert _adamw([_tensor(count=(1 << 34) + 1)]) == B.SC_EUNSUPPORTED
    for args in ((None, Z, 0.9, 0.9), (X, None, 0.9, 0.9), (X + 4, Z, 0.9, 0.9), (X, Z + 8, 0.9, 0.9), (X, X, 0.9, 0.9), (X, Z, 1.0, 0.9), (X, Z, 0.9, -1.0)):
        assert LIB.sparse_conv_adamw_count(*args, None) == B.SC_EINVAL


def test_tensor_calls_refuse_before_they_touch_anything():
    """The compiled side of text.py, given what is no CUDA tensor, no tensor, too few arguments."""
    import torch
    from paper_2011_06295_amd import text
    calls = text._calls
    w, x = torch.zeros(4, 8), torch.zeros(2, 8)
    for args in [(x, w, None, None, None, False, 0, 0), (None, w, None, None, None, False, 0, 0), (x, 3, None, None, None, False, 0, 0), (x, w), ()]:
        with pytest.raises(ValueError):
            calls.layer(*args)
    for args in [(x, x, w, None, True, True, True, False, 0, 0), (x, x, None, None, True, True, True, False, 0, 0), (x,), ()]:
        with pytest.raises(ValueError):
            calls.layer_backward(*args)
    for args in [(x, torch.zeros(2, dtype=torch.int64), None, True, 1.0, 0), (x, None, None, True, 1.0, 0), (None, None, None, True, 1.0, 0), (x, x, None, True, 1, 0), ()]:
        with pytest.raises(ValueError):
            calls.cross_entropy(*args)
    rule = (1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0)
    for args in [([x], [x], x, x, None, None, None, None, rule, 1, 0), ([x], [], x, x, None, None, None, None, rule, 1, 0), ([x], [x], None, x, None, None, None, None, rule, 1, 0), ()]:
        with pytest.raises(ValueError):
            calls.adamw(*args)
    with pytest.raises(ValueError):
        text.Linear(w)
    with pytest.raises(ValueError):
        text.cross_entropy(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        text.AdamW([w])
