"""The layer with bias, activation and residual, its gradients, the classifier's loss and AdamW steps against plain statements in 64 bits.

Bounds: u is half a unit in the last place of the output type, `tiny` half its smallest step, e = 2^-24.  A sum of K products in fp32, in any
order and with each addition off by a whole unit: 2 (K + 2) e times the sum of sizes.  Activations have slopes of at most 1.13, and as they are computed
(erf within four units; exp within |z| + 2 units, which the factors around it outweigh) are off by 8 e (1 + |z|) at most, their slopes by 8 e.
Loss: at most 160 + classes / 1024 additions lie between an exponential and the sum; an exponential at z - lse is off by |z - lse| + 4 units."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
E = 2.0 ** -24
ACTIVATIONS = [None, "relu", "gelu", "silu"]


def _types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _act(z, act):
    import torch
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z * torch.sigmoid(z) if act == "silu" else z


def _slope(z, act):
    import torch
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _within(got, ref, bound, what):
    import torch
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((err - bound)[bad].max())} at {torch.nonzero(bad)[0].tolist()}"


def _mm(a, b):
    """a [M][K] times b [N][K], transposed, in 64 bits (on the GPU, in pieces of rows)."""
    return a.double() @ b.double().t().contiguous()


# ---------------------------------------------------------------- layer

LAYERS = [  # M, K, N: every kernel (test_train_host.py), one token and row, odd sizes, ends inside tiles
    (1, 1, 1), (1, 64, 10), (1, 4096, 640), (2, 7, 3), (3, 200, 6), (5, 1001, 70), (16, 64, 16), (17, 96, 33), (24, 2048, 520), (33, 128, 257),
    (40, 4096, 96), (64, 512, 64), (65, 72, 130), (100, 136, 1000), (128, 200, 256), (203, 1001, 1111), (250, 2048, 300), (256, 64, 512), (515, 328, 700),
    (1000, 40, 24), (64, 16384, 64), (300, 8192, 40), (700, 1500, 1100), (20, 520, 4100), (20, 264, 4100), (48, 136, 2100), (40, 64, 2100), (520, 264, 777), (48, 1032, 4100),
    (40, 8192, 300), (20, 512, 8200), (900, 8192, 96), (8200, 264, 96), (4100, 512, 777), (264, 8192, 777), (20, 2048, 4160), (880, 136, 520),
    (360, 8192, 40), (880, 8192, 100)]
LARGE_LAYERS = [(2048, 1024, 2048), (4200, 512, 4100), (2300, 264, 4097), (2300, 1001, 777), (8200, 520, 8264), (3000, 4096, 3000), (8192, 2048, 2048)]


def _layer_case(gen, M, K, N, dtype, residual):
    import torch
    t = _types()[dtype]
    x = torch.randn((M, K), generator=gen, device="cuda").to(t)
    w = (torch.randn((N, K), generator=gen, device="cuda") * (1.5 / math.sqrt(K))).to(t)
    bias = torch.randn(N, generator=gen, device="cuda") * 0.5
    r = torch.randn((M, N), generator=gen, device="cuda").to(t) if residual else None
    return x, w, bias, r


def _check_layer(gen, M, K, N, dtype, act, residual, with_bias, keep):
    from paper_2011_06295_amd import text
    x, w, bias, r = _layer_case(gen, M, K, N, dtype, residual)
    bias = bias if with_bias else None
    layer = text.Linear(w, bias, activation=act)
    got = layer.forward(x, residual=r, keep=keep)
    y, kept = got if keep else (got, None)
    z, size = _mm(x, w), _mm(x.abs(), w.abs())
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    off = 2 * (K + 2) * E * size
    ref = _act(z, act)
    bound = 1.13 * off + (8 * E * (1 + z.abs()) if act in ("gelu", "silu") else 0.0)
    if residual:
        ref = ref + r.double()
        bound = bound + E * ref.abs()
    what = (M, K, N, dtype, act, residual, with_bias)
    _within(y, ref, bound + U[dtype] * (ref.abs() + bound) + TINY[dtype], what)
    if keep:
        _within(kept, z, off + U[dtype] * (z.abs() + off) + TINY[dtype], what + ("z",))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_layer(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i, (M, K, N) in enumerate(LAYERS):
        print(f"layer {dtype} {M}x{K} -> {N}", flush=True)
        _check_layer(gen, M, K, N, dtype, ACTIVATIONS[i % 4], i % 3 == 1, i % 5 != 2, i % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_layer(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    for i, (M, K, N) in enumerate(LARGE_LAYERS):
        print(f"large layer {dtype} {M}x{K} -> {N}", flush=True)
        _check_layer(gen, M, K, N, dtype, ACTIVATIONS[(i + 2) % 4], i % 2 == 0, True, i != 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_layer_on_rows_that_lie_apart_and_at_odd_addresses(dtype):
    """Strided x, weight, residual and output, starting one element past a multiple of 16 bytes; what lies between the rows stays."""
    import torch
    from paper_2011_06295_amd import text
    t = _types()[dtype]
    gen = torch.Generator(device="cuda").manual_seed(3)
    for M, K, N in ((1, 24, 16), (5, 64, 40), (37, 129, 66), (150, 256, 200)):
        for shift, gap in ((0, 0), (1, 3), (8, 8), (0, 1)):
            def rows(R, C, scale=1.0):
                store = (torch.randn(R * (C + gap) + shift + 8, generator=gen, device="cuda") * scale).to(t)
                return store, store[shift:shift + R * (C + gap)].view(R, C + gap)[:, :C]
            _, x = rows(M, K)
            _, w = rows(N, K, 1.0 / math.sqrt(K))
            _, r = rows(M, N)
            store, out = rows(M, N)
            before = store.clone()
            y = text.Linear(w, None, activation="relu").forward(x, residual=r, out=out)
            assert y.data_ptr() == out.data_ptr()
            z = _mm(x, w)
            off = 2 * (K + 2) * E * _mm(x.abs(), w.abs())
            ref = z.clamp(min=0.0) + r.double()
            _within(out, ref, off + E * ref.abs() + U[dtype] * (ref.abs() + off) + TINY[dtype], (M, K, N, shift, gap))
            mask = torch.ones_like(store, dtype=torch.bool)
            mask[shift:shift + M * (N + gap)].view(M, N + gap)[:, :N] = False
            assert torch.equal(store[mask], before[mask])
            again = r.clone()          # the residual in place
            assert torch.equal(text.Linear(w, None, activation="relu").forward(x, residual=again, out=again), out)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_is_no_number_stays_in_its_row_and_column(dtype):
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(4)
    for M, K, N in ((3, 100, 20), (70, 72, 40), (300, 512, 260), (5, 2048, 300)):
        x, w, bias, _ = _layer_case(gen, M, K, N, dtype, False)
        layer = text.Linear(w, bias)
        clean = layer.forward(x)
        x[M // 2, K - 1], x[0, 0] = math.nan, math.inf
        w[N - 1, 0] = -math.inf
        y = layer.forward(x)
        assert bool(torch.isnan(y[M // 2]).all()) and not bool(torch.isfinite(y[0]).any()) and not bool(torch.isfinite(y[:, N - 1]).any())
        rest = torch.ones_like(y, dtype=torch.bool)
        rest[M // 2], rest[0], rest[:, N - 1] = False, False, False
        assert torch.equal(y[rest], clean[rest])


# ---------------------------------------------------------------- gradients of the layer

GRADIENTS = [(1, 1, 1), (1, 64, 10), (2, 7, 3), (3, 200, 6), (16, 64, 16), (37, 129, 66), (128, 200, 256), (128, 256, 6), (203, 1001, 111), (515, 328, 700),
             (1021, 300, 77), (4099, 40, 24), (20000, 16, 8), (64, 2048, 300)]
LARGE_GRADIENTS = [(2048, 1024, 2048), (2300, 1100, 1030), (8200, 520, 8264), (3000, 3000, 3000), (8192, 1024, 1024), (256, 4096, 4096), (700, 2048, 4096),
                   (4100, 1032, 4104), (64, 4096, 4096), (1021, 1001, 777), (256, 1001, 777), (4100, 4096, 96), (20, 2048, 8200), (2100, 2048, 777), (4100, 2048, 520),
                   (264, 4096, 2100), (40, 2048, 8200), (4100, 4096, 777), (128, 4096, 8200)]


def _check_gradient(gen, M, K, N, dtype, act, accumulate):
    import torch
    from paper_2011_06295_amd import text
    x, w, bias, g = _layer_case(gen, M, K, N, dtype, True)
    z = torch.randn((M, N), generator=gen, device="cuda").to(_types()[dtype]) * 2
    layer = text.Linear(w, bias, activation=act)
    what = (M, K, N, dtype, act, accumulate)
    if accumulate:
        gw0, gb0 = torch.randn_like(w), torch.randn_like(bias)
        gx, gw, gb = layer.backward(g, x, z if act else None, grad_weight=gw0.clone(), grad_bias=gb0.clone(), accumulate=True)
    else:
        gx, gw, gb = layer.backward(g, x, z if act else None)
    assert gx.dtype == x.dtype and gw.dtype == w.dtype and gb.dtype == torch.float32
    d = g.double() * _slope(z.double(), act) if act else g.double()
    off = (9 * E * g.double().abs() if act in ("gelu", "silu") else 0.0) * torch.ones_like(d)      # of d before it is rounded
    rounded = off + (U[dtype] * (d.abs() + off) + TINY[dtype] if act else 0.0)
    for name, got, ref, size, wrong, count in (
            ("x", gx, d @ w.double(), d.abs() @ w.double().abs(), rounded @ w.double().abs(), N),
            ("weight", gw, d.t().contiguous() @ x.double(), d.t().abs().contiguous() @ x.double().abs(), rounded.t().contiguous() @ x.double().abs(), M)):
        bound = wrong + 2 * (count + 2) * E * (size + wrong)
        if accumulate and name == "weight":
            ref = ref + gw0.double()
            bound = bound + E * (ref.abs() + bound)
        _within(got, ref, bound + U[dtype] * (ref.abs() + bound) + TINY[dtype], what + (name,))
    ref, bound = d.sum(0), off.sum(0) + 2 * (M + 2) * E * (d.abs() + off).sum(0)
    if accumulate:
        ref, bound = ref + gb0.double(), bound + E * gb0.double().abs()
    _within(gb, ref, bound + E * ref.abs() + TINY["f32"], what + ("bias",))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradient(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    for i, (M, K, N) in enumerate(GRADIENTS):
        print(f"gradient {dtype} {M}x{K} -> {N}", flush=True)
        _check_gradient(gen, M, K, N, dtype, ACTIVATIONS[i % 4], i % 3 == 2)
        _check_gradient(gen, M, K, N, dtype, ACTIVATIONS[(i + 2) % 4], False)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_gradient(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(6)
    for i, (M, K, N) in enumerate(LARGE_GRADIENTS):
        print(f"large gradient {dtype} {M}x{K} -> {N}", flush=True)
        _check_gradient(gen, M, K, N, dtype, ACTIVATIONS[(i + 2) % 4], i == 1)


def test_gradient_against_differences():
    """fp32: the sum of out * g for a step of h either way in one place; central differences are off by h^2 / 6 times the third derivative (below 2 for a
    place's z, which moves by |x| or |w| < 4 times h) and by the rounding of the two sums over 2 h."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(7)
    M, K, N, h = 9, 21, 14, 2.0 ** -6
    for act in ACTIVATIONS:
        x, w, bias, g = _layer_case(gen, M, K, N, "f32", True)
        if act == "relu":          # away from the kink
            bias = bias + 40.0 * torch.sign(bias)
        layer = text.Linear(w, bias, activation=act)
        y, z = layer.forward(x, keep=True)
        gx, gw, gb = layer.backward(g, x, z)
        size = float((g.abs() * (y.abs() + _mm(x.abs(), w.abs()))).sum())
        for tensor, grad, place in ((x, gx, (3, 5)), (w, gw, (7, 20)), (bias, gb, (2,))):
            sums = []
            for sign in (1, -1):
                kept = float(tensor[place])
                tensor[place] = kept + sign * h
                sums.append(float((layer.forward(x).double() * g.double()).sum()))
                tensor[place] = kept
            bound = h * h / 6 * 2 * 64 * float(g.abs().sum()) + 2 * 2 * (K + 10) * E * size / (2 * h)
            assert abs((sums[0] - sums[1]) / (2 * h) - float(grad[place])) <= bound, (act, place)


def test_gradient_leaves_out_what_is_not_wanted():
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, w, bias, g = _layer_case(gen, 70, 50, 30, "f32", True)
    layer = text.Linear(w, bias, activation="gelu")
    z = torch.randn_like(g)
    all_three = layer.backward(g, x, z)
    for wanted in range(8):
        flags = [bool(wanted >> i & 1) for i in range(3)]
        got = layer.backward(g, x if flags[1] else None, z, *flags)
        for flag, a, b in zip(flags, got, all_three):
            assert (a is None) if not flag else torch.equal(a, b)
    assert text.Linear(w).backward(g, x)[2] is None
    out = [torch.full_like(t, 7.0) for t in all_three]
    got = layer.backward(g, x, z, *out)
    assert all(a is b for a, b in zip(got, out)) or all(a.data_ptr() == b.data_ptr() for a, b in zip(got, out))
    assert all(torch.equal(a, b) for a, b in zip(out, all_three))


def test_layers_of_no_rows_and_many_dimensions():
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(9)
    w, bias = torch.randn((6, 40), generator=gen, device="cuda"), torch.randn(6, generator=gen, device="cuda")
    layer = text.Linear(w, bias, activation="silu")
    x = torch.randn((2, 3, 40), generator=gen, device="cuda")
    assert torch.equal(layer.forward(x).reshape(6, 6), layer.forward(x.reshape(6, 40)))
    assert layer.forward(x[0, 0]).shape == (6,)
    y, z = layer.forward(torch.empty((0, 40), device="cuda"), keep=True)
    assert y.shape == z.shape == (0, 6)
    gx, gw, gb = layer.backward(y, torch.empty((0, 40), device="cuda"), z)
    assert gx.shape == (0, 40) and gw.shape == (6, 40) and int(torch.count_nonzero(gw)) == 0 and int(torch.count_nonzero(gb)) == 0
    kept = torch.ones_like(w)
    assert torch.equal(layer.backward(y, torch.empty((0, 40), device="cuda"), z, False, kept, False, accumulate=True)[1], torch.ones_like(w))


# ---------------------------------------------------------------- loss

LOSSES = [(1, 1), (1, 2), (128, 6), (3, 16), (7, 17), (65, 33), (5, 64), (9, 127), (33, 129), (4, 512), (6, 513), (3, 1000), (5, 1025), (4, 2049), (3, 4096), (2, 8200), (3, 16385),
          (2, 32768), (3, 40001), (2, 65537), (2, 131072), (1, 131073), (1, 300001), (5000, 10)]


def _check_loss(logits, labels, weights, scale, dtype, what, in_place=False):
    import torch
    from paper_2011_06295_amd import text
    classes = logits.shape[1]
    z = logits.double()
    given = logits.clone() if in_place else logits
    loss, grad = text.cross_entropy(given, labels, weights, grad=given if in_place else True, scale=scale)
    s = (torch.ones(len(z), device="cuda") if weights is None else weights).double() * float(np.float32(scale))
    counts = (labels >= 0) & (labels < classes) & (s != 0)
    z = torch.where(counts[:, None], z, torch.zeros_like(z))
    at = labels.long().clamp(0, classes - 1)[:, None]
    lse = torch.logsumexp(z, 1)
    label = z.gather(1, at)[:, 0]
    ref = torch.where(counts, s * (lse - label), torch.zeros_like(s))
    of_sum = 2 * (168 + classes / 1024) * E
    top = z.amax(1)
    off = s.abs() * (of_sum + 2 * E * (top.abs() + label.abs() + lse.abs() + (lse - top).abs())) + 4 * E * ref.abs()
    _within(loss, ref, off + TINY["f32"], what)
    p = torch.exp(z - lse[:, None])
    far = torch.where(torch.isinf(z), torch.zeros_like(z), (z - lse[:, None]).abs() + 2 * lse.abs()[:, None])
    ref = p.clone().scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float64)) * s[:, None]
    ref = torch.where(counts[:, None], ref, torch.zeros_like(ref))
    off = s.abs()[:, None] * p * (of_sum + 4 * E * (far + 4)) + 4 * E * (ref.abs() + s.abs()[:, None] * (p > 0.5))
    assert grad.dtype == logits.dtype
    _within(grad, ref, off + U[dtype] * (ref.abs() + off) + TINY[dtype], what)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_loss(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(11)
    for i, (rows, classes) in enumerate(LOSSES):
        print(f"loss {dtype} {rows}x{classes}", flush=True)
        logits = (3.0 * torch.randn((rows, classes), generator=gen, device="cuda")).to(_types()[dtype])
        labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
        weights = torch.rand(rows, generator=gen, device="cuda") if i % 2 else None
        if i % 3 == 1:
            labels = labels.int()
        if rows > 2 and i % 4 == 0:        # rows that do not count, forbidden classes
            labels[0], labels[1] = -1, classes
            logits[:, ::3] = -math.inf
            logits[:, -1] = 0.5
            labels[2:] = classes - 1
            if weights is None:
                weights = torch.ones(rows, device="cuda")
            weights[2] = 0.0
            logits[2] = math.nan           # (not read)
        _check_loss(logits, labels, weights, (1.0, 0.37)[i % 2], dtype, (rows, classes, dtype), in_place=i % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_loss_of_logits_far_from_zero(dtype):
    """Differences of logits are exact in fp32 here, so an offset of them all costs nothing."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(12)
    for rows, classes, offset in ((40, 6, 30000.0), (7, 129, -30000.0), (5, 1025, 20000.0), (3, 4096, 50000.0), (2, 40001, -50000.0), (2, 131072, 30000.0)):
        step = {"f32": 2.0 ** -6, "f16": 32.0, "bf16": 256.0}[dtype]
        logits = (offset + step * torch.randint(-300 if dtype == "f32" else -2, 300 if dtype == "f32" else 3, (rows, classes), generator=gen, device="cuda")).to(_types()[dtype])
        labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
        loss, grad = text.cross_entropy(logits, labels)
        z = logits.double()
        top = z.amax(1, keepdim=True)
        lse, far = torch.logsumexp(z - top, 1, keepdim=True), top - z
        of_sum = 2 * (168 + classes / 1024) * E
        label = far.gather(1, labels[:, None])
        ref = (lse + label)[:, 0]
        _within(loss, ref, of_sum + 4 * E * (ref.abs() + lse[:, 0]) + TINY["f32"], (rows, classes))
        p = torch.exp(-far - lse)
        ref = p.scatter_add(1, labels[:, None], torch.full_like(label, -1.0))
        off = p * (of_sum + 4 * E * (far + lse + 4)) + 4 * E * (ref.abs() + (p > 0.5))
        _within(grad, ref, off + U[dtype] * (ref.abs() + off) + TINY[dtype], (rows, classes))


def test_loss_of_rows_that_lie_apart():
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(12)
    for classes in (5, 100, 3001, 140_000):
        for dtype in _types().values():
            store = torch.randn((4, classes + 3), generator=gen, device="cuda").to(dtype)
            room = torch.full((4, classes + 5), 9.0, dtype=dtype, device="cuda")
            labels = torch.randint(0, classes, (4,), generator=gen, device="cuda")
            loss, grad = text.cross_entropy(store[:, 1:classes + 1], labels, grad=room[:, 2:classes + 2])
            want = text.cross_entropy(store[:, 1:classes + 1].contiguous(), labels)
            assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])
            assert bool((room[:, :2] == 9.0).all()) and bool((room[:, classes + 2:] == 9.0).all())
            assert text.cross_entropy(store[:, 1:classes + 1], labels, grad=False)[1] is None
            assert torch.equal(text.cross_entropy(store[:, 1:classes + 1], labels, grad=False)[0], loss)


def test_rows_without_a_loss():
    """Nothing but forbidden classes, plus infinity, a NaN: NaN in that row alone.  A forbidden label: infinite, with a finite gradient."""
    import torch
    from paper_2011_06295_amd import text
    for classes in (6, 70, 900, 5000, 70_000, 200_000):
        for dtype in _types().values():
            logits = torch.zeros((6, classes), dtype=dtype, device="cuda")
            logits[1] = -math.inf
            logits[2, classes // 2] = math.inf
            logits[3, classes - 1] = math.nan
            logits[4, 1] = -math.inf
            labels = torch.ones(6, dtype=torch.int64, device="cuda")
            loss, grad = text.cross_entropy(logits, labels)
            assert torch.isnan(loss).tolist() == [False, True, True, True, False, False] and float(loss[4]) == math.inf
            assert torch.isnan(grad).any(1).tolist() == [False, True, True, True, False, False]
            assert float(grad[4, 1]) == -1.0 and bool((grad[5] == grad[0]).all())
            far = torch.full((2, classes), -6e4 if dtype == torch.float16 else -3e38, dtype=dtype, device="cuda")      # the lowest values, masks in some programs
            far[0, 1] = 2.0
            loss, grad = text.cross_entropy(far, labels[:2])
            assert abs(float(loss[0])) <= 4 * E and bool(torch.isfinite(loss).all()) and bool(torch.isfinite(grad).all())
            assert abs(float(loss[1]) - math.log(classes)) <= 2 * (168 + classes / 1024) * E + 4 * E * math.log(classes)


# ---------------------------------------------------------------- AdamW

SHAPES = [(7,), (300, 41), (256,), (1,), (255,), (257,), (3, 5, 7), (2048,), (2049,), (100_003,), (0,), (64, 64)]


def _start(gen, dtype, grad_dtype, bits, master, shapes=SHAPES, odd=True, **more):
    import torch
    from paper_2011_06295_amd import text

    def make(t, scale):
        out = []
        for i, shape in enumerate(shapes):
            n = math.prod(shape)
            store = (torch.randn(n + 3, generator=gen, device="cuda") * scale).to(t)
            out.append(store[i % 3 if odd else 0:][:n].view(shape))         # parameters and gradients at odd addresses
        return out
    params = make(_types()[dtype], 0.1)
    optimizer = text.AdamW(params, rate=3e-3, betas=(0.9, 0.98), eps=1e-7, decay=0.02, bits=bits, master=master, **more)
    return params, optimizer, lambda: make(_types()[grad_dtype], 0.02)


def _values(optimizer, name):
    import torch
    t = getattr(optimizer, name)
    if optimizer.bits == 32:
        return t.double()
    return (t.double().view(-1, 256) * getattr(optimizer, name + "_scale").double()[:, None]).view(-1)


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_adamw(types, bits, master):
    """Several steps, each from the state that the one before left.  m and v: four and five roundings; the step: ten and m's; 8 bits: half a step of
    a number of four digits for m (to the nearest), a whole one for v."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(21)
    params, opt, gradients = _start(gen, *types, bits, master)
    total, dtype = opt.m.numel(), types[0]
    inside = torch.zeros(total, dtype=torch.bool, device="cuda")
    for begin, p in zip(opt.begins, params):
        inside[begin:begin + p.numel()] = True

    def flat(tensors):
        out = torch.zeros(total, dtype=torch.float64, device="cuda")
        for begin, t in zip(opt.begins, tensors):
            out[begin:begin + t.numel()] = t.double().reshape(-1)
        return out
    for step in range(1, 5):
        grads = gradients()
        scale = 0.5 if step == 2 else 1.0
        m0, v0, p0, g = _values(opt, "m"), _values(opt, "v"), opt.master.double() if master else flat(params), flat(grads) * scale
        opt.step(grads, scale)
        assert opt.steps == step
        m, v = 0.9 * m0 + 0.1 * g, 0.98 * v0 + 0.02 * g * g
        m_off, v_off = 4 * E * (0.9 * m0.abs() + 0.1 * g.abs()), 5 * E * v
        root = torch.sqrt(v / (1 - 0.98 ** step)) + 1e-7
        update = 3e-3 * (m / (1 - 0.9 ** step)) / root
        p = p0 * (1 - 3e-3 * 0.02) - update
        off = 12 * E * update.abs() + 3e-3 / (1 - 0.9 ** step) * m_off / root + 3 * E * p0.abs() + E * p.abs() + 1e-37
        what = (types, bits, master, step)
        if master:
            _within(opt.master, p, off, what + ("master",))
            assert torch.equal(flat(params), opt.master.to(_types()[dtype]).double())
        else:
            _within(flat(params), p, off + U[dtype] * (p.abs() + off) + TINY[dtype], what)
        if bits == 32:
            _within(opt.m, m, m_off + 1e-37, what + ("m",))
            _within(opt.v, v, v_off + 1e-37, what + ("v",))
        else:
            for name, exact, wrong in (("m", m, m_off), ("v", v, v_off)):
                largest = exact.abs().view(-1, 256).amax(1)
                s = getattr(opt, name + "_scale").double()
                _within(s, largest / 448, wrong.view(-1, 256).amax(1) / 448 + 4 * E * s, what + (name, "scales"))      # (m's terms may cancel)
                room = s.repeat_interleave(256)
                unit = torch.maximum(room * 2.0 ** -9, exact.abs() * 2.0 ** -3)             # no less than the step between numbers
                _within(_values(opt, name), exact, wrong + 10 * E * exact.abs() + unit * (0.5 if name == "m" else 1.0) * (1 + 2.0 ** -20), what + (name,))
            assert bool((opt.v.float()[(v > 0)] > 0).all())
        for t in (opt.m, opt.v) + ((opt.master,) if master else ()):
            assert int(torch.count_nonzero(t.float()[~inside])) == 0       # behind a tensor's end


def test_states_in_8_bits_keep_what_small_changes_add_up_to():
    """v of a steady gradient after 2000 steps, each of which changes it by less than half a step between numbers: near 1 - b2^t of its square.  (To the
    nearest number it would stay where rounding first held it.)  What one element holds wanders; 8192 of them agree to a few hundredths."""
    import torch
    from paper_2011_06295_amd import text
    p = torch.zeros(8192, device="cuda")
    opt = text.AdamW([p], rate=0.0, betas=(0.9, 0.999), bits=8)
    size = torch.linspace(0.3, 1.0, 8192, device="cuda")
    for _ in range(2000):
        opt.step([size])
    ratio = (_values(opt, "v") / (size.double() ** 2 * (1 - 0.999 ** 2000))).view(32, 256)
    assert float((ratio.mean() - 1).abs()) < 0.02 and float((ratio.mean(1) - 1).abs().max()) < 0.06
    assert float((_values(opt, "m") / size.double() - 1).abs().max()) < 2.0 ** -4 * 10 * 1.01      # (to the nearest number: a tenth of the gradient moves it)


def test_adamw_steps_in_a_row_are_the_same_bits_and_some_gradients_may_be_missing():
    import torch
    for bits in (8, 32):
        results = []
        for _ in range(2):
            gen = torch.Generator(device="cuda").manual_seed(22)
            params, opt, gradients = _start(gen, "bf16", "bf16", bits, True)
            for _ in range(3):
                grads = gradients()
                grads[3] = None
                before = params[3].clone()
                opt.step(grads)
                assert torch.equal(params[3], before)
            results.append([p.clone() for p in params] + [opt.m.float(), opt.v.float(), opt.master])
        assert all(torch.equal(a, b) for a, b in zip(*results))


def test_adamw_of_many_tensors():
    """More tensors than one launch takes, with empty ones between."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(23)
    shapes = [((i * 37) % 600 + (i % 7 == 0) * 3000,) if i % 11 else (0,) for i in range(173)]
    params, opt, gradients = _start(gen, "f32", "f32", 32, False, shapes)
    start, grads = [p.double() for p in params], gradients()
    opt.step(grads)
    for p, p0, g in zip(params, start, grads):
        g = g.double()
        ref = p0 * (1 - 3e-3 * 0.02) - 3e-3 * g / (g.abs() + 1e-7)
        _within(p, ref, 4 * E * p0.abs() + 16 * E * 3e-3 + E * ref.abs(), p.shape)


def test_adamw_in_a_graph_counts_its_steps():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(24)
    for bits in (32, 8):
        state = gen.get_state()
        params, opt, gradients = _start(gen, "f32", "f32", bits, False, counted=True)
        gen.set_state(state)
        others, plain, _ = _start(gen, "f32", "f32", bits, False)
        grads = gradients()
        opt.step(grads)           # (outside, then recorded)
        plain.step(grads)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            opt.step(grads)
        for _ in range(4):
            for g, new in zip(grads, gradients()):
                g.copy_(new)
            graph.replay()
            torch.cuda.synchronize()
            plain.step(grads)
            torch.cuda.synchronize()
            for a, b in zip(params, others):
                assert float((a - b).abs().max() if a.numel() else 0.0) <= 8 * E * 1.0       # (the corrections may round differently by a unit)
            if bits == 32:
                assert torch.equal(opt.m, plain.m) and torch.equal(opt.v, plain.v)
        assert int(opt.steps) == plain.steps == 5


def test_adamw_refused_steps_do_not_count_and_plain_ones_are_not_recorded():
    import torch
    from paper_2011_06295_amd import text
    for bits in (32, 8):
        for counted in (True, False):
            p = torch.ones(600, device="cuda", dtype=torch.bfloat16)
            opt = text.AdamW([p], bits=bits, counted=counted, master=True)
            g = torch.ones(600, device="cuda", dtype=torch.bfloat16)
            opt.step([g])
            before = [t.clone() for t in (p, opt.m.view(torch.uint8), opt.master)]
            for bad in ([g.half()], [p], [opt.master[:600]], [g[:599]], [g, g], [g.cpu()], [g.double()]):
                with pytest.raises((ValueError, RuntimeError)):
                    opt.step(bad)
            with pytest.raises((ValueError, RuntimeError)):
                opt.step([g], scale=math.inf)
            opt.rate = -1.0
            with pytest.raises((ValueError, RuntimeError)):
                opt.step([g])
            opt.rate = 1e-3
            assert int(opt.steps) == 1 and all(torch.equal(a, b) for a, b in zip(before, (p, opt.m.view(torch.uint8), opt.master)))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q = p + 1
        with pytest.raises(RuntimeError, match="counted"):
            opt.step([g])
    assert opt.steps == 1


# ---------------------------------------------------------------- the model that runs them together

def _small_model(seed, **more):
    import torch
    from paper_2011_06295_amd import text_model
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    vocab, dim, classes, width = 400, 40, 5, 30
    filters = [((rng.standard_normal((12, dim, 1, s)) * 0.3).astype(np.float32), (rng.random((12, dim, 1, s)) < 0.3).astype(np.uint8),
                (rng.standard_normal(12) * 0.1).astype(np.float32)) for s in (2, 3)]
    table = torch.randn((vocab, dim), generator=gen, device="cuda")
    table[0] = 0.0
    hidden, classifier = torch.randn((width, 24), generator=gen, device="cuda") * 0.3, torch.randn((classes, width), generator=gen, device="cuda") * 0.3
    model = text_model.ClassifierModel(table, filters, hidden, classifier, **more)
    model.hidden.bias.copy_(torch.randn(width, generator=gen, device="cuda") * 0.1)
    tokens, labels = text_model.sentences(9, 21, vocab, classes, seed=seed)
    return model, filters, tokens, labels


@pytest.mark.parametrize("activation", ["relu", "gelu", "silu"])
def test_model_s_gradients_against_64_bits(activation):
    """fp32 features, bounded by 1e-5 of their largest (the convolutions' own tolerance), go through two layers, the loss and back: 4e-5 of each
    gradient's largest."""
    import torch
    model, filters, tokens, labels = _small_model(41, activation=activation)
    losses, grads = model.gradients(tokens, labels)
    leaves = [t.double().cpu().requires_grad_(True) for t in (model.words.table, model.hidden.weight, model.hidden.bias, model.classifier.weight, model.classifier.bias)]
    table, w1, b1, w2, b2 = leaves
    x = table[tokens.cpu()].permute(0, 2, 1)[:, :, None]
    features = torch.cat([torch.relu(torch.nn.functional.conv2d(x, torch.from_numpy(w * m).double(), torch.from_numpy(b).double())).squeeze(2).amax(2) for w, m, b in filters], 1)
    logits = _act(features @ w1.t() + b1, activation) @ w2.t() + b2
    each = torch.nn.functional.cross_entropy(logits, labels.cpu(), reduction="none") / len(tokens)
    each.sum().backward()
    assert float((losses.double().cpu() - each.detach()).abs().max()) <= 4e-5 * float(each.detach().max())
    leaves[0].grad[0] = 0.0          # the padding word
    for got, leaf in zip(grads, leaves):
        assert float((got.double().cpu() - leaf.grad).abs().max()) <= 4e-5 * float(leaf.grad.abs().max()), got.shape
    model.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_model_s_step_moves_its_parameters_by_the_optimizer_s_rule(bits):
    """The first step: the sign of each gradient times the rate, but where the gradient is as small as eps; decay."""
    import torch
    model, _, tokens, labels = _small_model(42, bits=bits, rate=1e-2, decay=0.1)
    parameters = model.optimizer.params
    before = [p.double() for p in parameters]
    _, grads = model.gradients(tokens, labels)
    first = float(model.train_step(tokens, labels))
    for p, p0, g in zip(parameters, before, grads):
        g = g.double()
        ref = p0 * (1 - 1e-2 * 0.1) - 1e-2 * g / (g.abs() + 1e-8)
        _within(p, ref, 4 * E * p0.abs() + 16 * E * 1e-2 + E * ref.abs(), p.shape)
    assert float(model.words.table[0].abs().max()) == 0.0
    assert math.isfinite(first) and math.isfinite(float(model.train_step(tokens, labels)))
    model.close()


# ---------------------------------------------------------------- streams, graphs, refusals

def test_layer_and_loss_on_another_stream_and_in_a_graph():
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(31)
    for dtype, (M, K, N) in (("f32", (40, 129, 66)), ("bf16", (300, 512, 260)), ("f16", (64, 16384, 64))):
        x, w, bias, _ = _layer_case(gen, M, K, N, dtype, False)
        layer = text.Linear(w, bias, activation="gelu")
        labels = torch.randint(0, N, (M,), generator=gen, device="cuda")

        def step():
            y, z = layer.forward(x, keep=True)
            loss, grad = text.cross_entropy(y, labels, scale=1.0 / M)
            return (y, z, loss, grad) + layer.backward(grad, x, z)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
            step()
        torch.cuda.synchronize()
        for a, b in zip(other, step()):
            assert torch.equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            recorded = step()
        for seed in range(4):
            x.copy_(torch.randn((M, K), generator=gen, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            want = step()
            torch.cuda.synchronize()
            for a, b in zip(recorded, want):
                assert torch.equal(a, b), seed


def test_wrappers_refuse_what_they_cannot_run():
    import torch
    from paper_2011_06295_amd import text
    w, bias = torch.ones((6, 8), device="cuda"), torch.zeros(6, device="cuda")
    for bad in (dict(weight=w.cpu()), dict(weight=w.t()), dict(weight=w.double()), dict(weight=w[0]), dict(weight=w, bias=bias[:5]), dict(weight=w, bias=bias.half()),
                dict(weight=w, bias=bias.cpu()), dict(weight=w, activation="tanh")):
        with pytest.raises(ValueError):
            text.Linear(**bad)
    layer = text.Linear(w, bias, activation="gelu")
    x, g = torch.ones((4, 8), device="cuda"), torch.ones((4, 6), device="cuda")
    for args in ((x[:, :7],), (x.half(),), (x.cpu(),), (torch.ones((8, 4), device="cuda").t(),), (x, g[:3]), (x, g.half()), (x, None, False, g[:, :5]), (x, None, False, g.half())):
        with pytest.raises(ValueError):
            layer.forward(*args)
    with pytest.raises(RuntimeError):
        layer.forward(x, out=x[:, :6])         # overlaps what is read
    for args in ((g, x), (g[:, :5], x, g), (g, x[:3], g), (g, None, g), (g, x, g[:3]), (g, x, g, True, True, torch.zeros(5, device="cuda")), (g, x, g, 3)):
        with pytest.raises(ValueError):
            layer.backward(*args)
    with pytest.raises(ValueError):
        layer.backward(g, x, g, accumulate=True)
    labels = torch.zeros(4, dtype=torch.int64, device="cuda")
    for args in ((g.cpu(), labels), (g.double(), labels), (g, labels[:3]), (g, labels.float()), (g, labels, labels), (g, labels, None, g[:3]), (g, labels, None, 5), (g[:, :0], labels)):
        with pytest.raises(ValueError):
            text.cross_entropy(*args)
    p = torch.ones(10, device="cuda")
    for args in (([],), ([p.cpu()],), ([p, p.half()],), ([p, p],), ([p, p[5:]],), ([p.double()],), ([w.t()],)):
        with pytest.raises(ValueError):
            text.AdamW(*args)
    for more in (dict(bits=16), dict(rate=-1.0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(decay=-1.0)):
        with pytest.raises(ValueError):
            text.AdamW([p], **more)
    opt = text.AdamW([p])
    for grads in ([], [p.half()[:5]], [p.cpu()], [torch.ones(20, device="cuda")[::2]], [p, p], [3]):
        with pytest.raises(ValueError):
            opt.step(grads)
    assert opt.steps == 0
