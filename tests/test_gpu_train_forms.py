"""Forms of the layer's and its gradients' kernels that ordinary sizes take (tiles of either size, the slope worked out as d is loaded, rows of less than
16 bytes, sums split over workgroups), and gradients of arrays that lie apart and at odd addresses, against 64 bits.

Bounds are those of test_gpu_train.py, which says where they come from.  test_train_forms_host.py checks that the sizes of both files reach
every kernel in every form that sizes drawn at large take."""
import math

import pytest

from test_gpu_train import E, TINY, U, _act, _check_gradient, _check_layer, _layer_case, _mm, _slope, _types, _values, _within

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


def _apart(gen, R, C, shift, gap, t, scale=1.0):
    """(memory, [R][C] of it): rows C + gap elements apart from element `shift` on, NaN in all that is not theirs."""
    import torch
    store = torch.full((R * (C + gap) + shift + 8,), math.nan, dtype=t, device="cuda")
    rows = store[shift:shift + R * (C + gap)].view(R, C + gap)[:, :C]
    rows.copy_(torch.randn((R, C), generator=gen, device="cuda") * scale)
    return store, rows


# M, K, N: one launch in tiles of either size, with the slope worked out in it or before; laid out.
APART = [(5, 64, 40), (37, 129, 66), (150, 256, 200), (300, 304, 300), (1021, 300, 77), (1000, 640, 776), (2100, 1032, 1040),
         (3000, 2056, 2056), (4100, 4104, 4096)]
WAYS = [  # shift and gap of grad, x, weight; 8 elements are 16 bytes or 32
    ((0, 0), (0, 0), (0, 0)), ((8, 8), (8, 8), (8, 8)), ((1, 3), (0, 0), (0, 0)), ((0, 0), (1, 0), (0, 8)), ((0, 8), (0, 1), (0, 0)), ((0, 0), (0, 0), (2, 0)), ((0, 1), (3, 5), (1, 2))]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_of_rows_that_lie_apart_and_at_odd_addresses(dtype):
    """Strided grad, x and weight, NaN between their rows; z, which has no gaps, and the gradients that are written at odd addresses."""
    import torch
    from paper_2011_06295_amd import text
    t = _types()[dtype]
    gen = torch.Generator(device="cuda").manual_seed(53)
    for i, (M, K, N) in enumerate(APART):
        for j, way in enumerate(WAYS):
            act = (None, "relu", "gelu", "silu")[(i + j) % 4]
            print(f"apart {dtype} {M}x{K} -> {N} {way} {act}", flush=True)
            g, x, w = (_apart(gen, R, C, shift, gap, t, scale)[1] for (R, C, scale), (shift, gap) in zip(((M, N, 1.0), (M, K, 1.0), (N, K, 1.5 / math.sqrt(K))), way))
            z = _apart(gen, 1, M * N, 1 + j % 3, 0, t, 2.0)[1].view(M, N)
            stores, outs = zip(*(_apart(gen, 1, n, shift, 0, kind) for n, shift, kind in ((M * K, 1 + j % 2, t), (N * K, 3, t), (N, 1, torch.float32))))
            before = [s.clone() for s in stores]
            outs = [o.view(shape) for o, shape in zip(outs, ((M, K), (N, K), (N,)))]
            gw0, gb0, accumulate = outs[1].double(), outs[2].double(), j % 2 == 1
            layer = text.Linear(w, torch.zeros(N, device="cuda"), activation=act)
            layer.backward(g, x, z if act else None, *outs, accumulate=accumulate)
            d = g.double() * _slope(z.double(), act)
            off = (9 * E * g.double().abs() if act in ("gelu", "silu") else 0.0) * torch.ones_like(d)
            rounded = off + (U[dtype] * (d.abs() + off) + TINY[dtype] if act else 0.0)
            what = (M, K, N, dtype, act, way)
            for name, got, ref, size, wrong, count in (
                    ("x", outs[0], d @ w.double(), d.abs() @ w.double().abs(), rounded @ w.double().abs(), N),
                    ("weight", outs[1], d.t().contiguous() @ x.double(), d.t().abs().contiguous() @ x.double().abs(), rounded.t().contiguous() @ x.double().abs(), M)):
                bound = wrong + 2 * (count + 2) * E * (size + wrong)
                if accumulate and name == "weight":
                    ref = ref + gw0
                    bound = bound + E * (ref.abs() + bound)
                _within(got, ref, bound + U[dtype] * (ref.abs() + bound) + TINY[dtype], what + (name,))
            ref, bound = d.sum(0), off.sum(0) + 2 * (M + 2) * E * (d.abs() + off).sum(0)
            if accumulate:
                ref, bound = ref + gb0, bound + E * gb0.abs()
            _within(outs[2], ref, bound + E * ref.abs() + TINY["f32"], what + ("bias",))
            for store, was, out in zip(stores, before, outs):          # nothing else is written
                first = out.storage_offset()
                assert bool(torch.isnan(store[:first]).all()) and bool(torch.isnan(store[first + out.numel():]).all()) and store.shape == was.shape


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_large_layers_of_rows_that_lie_apart(dtype):
    """Layers that are laid out: neither, one or both of x and the weight copied because of their address or distance alone; NaN between the rows."""
    import torch
    from paper_2011_06295_amd import binding as B
    from paper_2011_06295_amd import text
    t = _types()[dtype]
    gen = torch.Generator(device="cuda").manual_seed(54)
    for M, K, N in ((16, 2048, 4160), (900, 1024, 1304), (4100, 2048, 2056)):
        copied = set()
        for j, (_, of_x, of_w) in enumerate(WAYS):
            act = (None, "relu", "gelu", "silu")[j % 4]
            print(f"large apart {dtype} {M}x{K} -> {N} {of_x} {of_w} {act}", flush=True)
            x, w = _apart(gen, M, K, *of_x, t)[1], _apart(gen, N, K, *of_w, t, 1.5 / math.sqrt(K))[1]
            r = _apart(gen, M, N, 1, j, t)[1]
            store, out = _apart(gen, M, N, 3, 2, t)
            layer = text.Linear(w, None, activation=act)
            layer.forward(x, residual=r, out=out)
            z, off = _mm(x, w), 2 * (K + 2) * E * _mm(x.abs(), w.abs())
            ref = _act(z, act) + r.double()
            bound = 1.13 * off + (8 * E * (1 + z.abs()) if act in ("gelu", "silu") else 0.0) + E * ref.abs()
            _within(out, ref, bound + U[dtype] * (ref.abs() + bound) + TINY[dtype], (M, K, N, dtype, of_x, of_w, act))
            mask = torch.ones_like(store, dtype=torch.bool)
            mask[3:3 + M * (N + 2)].view(M, N + 2)[:, :N] = False
            assert bool(torch.isnan(store[mask]).all())
            copied.add(B.sparse_conv_linear_workspace(x.data_ptr(), w.data_ptr(), M, N, K, x.stride(0), w.stride(0), {"f32": B.SC_F32, "f16": B.SC_F16, "bf16": B.SC_BF16}[dtype]))
        assert M < 4100 or len(copied) == 4, copied


# M, K, N: one launch in tiles of either size; d formed before it; laid out
GRADIENT_WAYS = [(9, 40, 24), (300, 300, 300), (305, 2203, 253), (1021, 1001, 777), (4100, 2056, 4104)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_relu_stops_gradients_that_are_no_number(dtype):
    """Where z is not above 0 the gradient behind a ReLU is 0, also of an infinity or a NaN: all gradients are those of a grad with zeros there."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(55)
    for M, K, N in GRADIENT_WAYS:
        print(f"relu {dtype} {M}x{K} -> {N}", flush=True)
        x, w, bias, g = _layer_case(gen, M, K, N, dtype, True)
        z = torch.randn((M, N), generator=gen, device="cuda").to(_types()[dtype])
        z[0, 0], z[1, 1], z[2, 2], z[3, 3] = 0.0, -1.0, -math.inf, 1.0
        clean = torch.where(z > 0, g, torch.zeros_like(g))
        g = torch.where(z > 0, g, torch.full_like(g, math.inf))
        g[1, 1], g[2, 2] = -math.inf, math.nan
        layer = text.Linear(w, bias, activation="relu")
        for got, want in zip(layer.backward(g, x, z), layer.backward(clean, x, z)):
            assert bool(torch.isfinite(want).all()) and torch.equal(got, want)
        g[3, 3] = math.inf          # one that it passes on
        gx, gw, gb = layer.backward(g, x, z)
        assert not bool(torch.isfinite(gx[3]).any()) and not bool(torch.isfinite(gw[3]).any()) and float(gb[3]) == math.inf
        assert bool(torch.isfinite(gx[4:]).all()) and bool(torch.isfinite(gw[4:]).all()) and bool(torch.isfinite(gb[4:]).all())


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_slopes_of_what_went_past_16_bits(act):
    """z outside binary16's range is kept as an infinity; the layer's output is 0 or as large, and the slope 0 or 1."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(56)
    for M, K, N in GRADIENT_WAYS:
        print(f"past 16 bits {M}x{K} -> {N} {act}", flush=True)
        x, w, bias, g = _layer_case(gen, M, K, N, "f16", True)
        x[0], x[2], w[1] = 0.0, 0.0, 0.0
        x[0, 0], x[2, 0], w[1, 0] = -3000.0, 3000.0, 40.0          # z of 120000 either way in column 1
        w[2:, 0] = 0.0
        w[0, 0] = 0.0
        layer = text.Linear(w, bias, activation=act)
        y, z = layer.forward(x, keep=True)
        assert float(z[0, 1]) == -math.inf and float(z[2, 1]) == math.inf and float(y[0, 1]) == 0.0 and float(y[2, 1]) == math.inf
        flat = z.clone()
        flat[0, 1], flat[2, 1] = -60000.0, 60000.0          # slopes of 0 and 1 as well
        got = layer.backward(g, x, z)
        for a, b in zip(got, layer.backward(g, x, flat)):
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
        z[4, 3] = math.nan
        gx, gw, gb = layer.backward(g, x, z)
        assert bool(torch.isnan(gx[4]).all()) and bool(torch.isnan(gw[3]).all()) and math.isnan(float(gb[3])) and torch.equal(gx[:4], got[0][:4]) and torch.equal(gx[5:], got[0][5:])


# ---------------------------------------------------------------- AdamW

@pytest.mark.parametrize("master", [False, True])
def test_weight_decay_below_the_weights_own_rounding(master):
    """What a step of a small rate takes off fp32 weights, on average over 2^22 of them.  A weight in 0.5 .. 1 moves in steps of 2^-24; updates of all sizes
    up to the rate make each rounding as good as random, off by 2^-24 / sqrt(12) (and by a second one of that size at most), and their mean by
    2^-24 / sqrt(6) / 2^11 = 1.2e-11.  Six times that is less than a hundredth of the decay, 1e-8 and more."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(61)
    for rate in (2e-6, 5e-6, 1e-5):
        n, decay, eps = 1 << 22, 0.01, 1e-2
        start = torch.rand(n, generator=gen, device="cuda") * 0.5 + 0.5
        grad = 1e-2 * torch.randn(n, generator=gen, device="cuda")
        p = start.to(torch.bfloat16) if master else start.clone()
        opt = text.AdamW([p], rate=rate, eps=eps, decay=decay, master=master)
        if master:
            opt.master.copy_(start)
        opt.step([grad])
        moved = (opt.master if master else p).double() - start.double()
        update = rate * grad.double() / (grad.double().abs() + eps)          # the first step: m over the root of v is the gradient over its size
        took, ref = float((-moved - update).mean()), rate * decay * float(start.double().mean())
        assert ref > 1.4e-8 and abs(took - ref) <= 8e-11 + 16 * E * rate, (rate, took, ref)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_infinite_weights_stay(dtype):
    """Places that a program has masked by infinities, with gradients of zero and others, with and without decay."""
    import torch
    from paper_2011_06295_amd import text
    for bits in (8, 32):
        for master in (False, True):
            for decay in (0.0, 0.01):
                p = torch.ones(600, dtype=_types()[dtype], device="cuda")
                p[3], p[4], p[300], p[301] = -math.inf, math.inf, -math.inf, math.inf
                g = torch.ones_like(p)
                g[:5] = 0.0
                kept = p.clone()
                opt = text.AdamW([p], rate=1e-2, decay=decay, bits=bits, master=master)
                for _ in range(3):
                    opt.step([g])
                infinite = torch.isinf(kept)
                assert torch.equal(p[infinite], kept[infinite]) and bool(torch.isfinite(p[~infinite]).all()) and float(p[100]) < 1.0
                g[301] = math.nan
                opt.step([g])
                assert math.isnan(float(p[301])) and float(p[3]) == -math.inf


def test_first_moments_of_8_bits_follow_the_gradient():
    """m under steady gradients, after they turn, after they fall to a third and after they end, beside an element that keeps the block's scale.
    m rests where (1 - b) |g - m| is half a step between numbers or less: a 16th of m where it has to grow, an 18th where it has to shrink (1.125 to 1); where the
    steps are 2^-9 of the scale, (1 - b) times it within 2^-10.  The scale itself is off by an ulp or so a step."""
    import torch
    from paper_2011_06295_amd import text
    for beta in (0.0, 0.5, 0.8, 0.9):
        n = 8 * 256
        size = torch.linspace(0.1, 0.9, n, device="cuda")
        top = torch.arange(n, device="cuda") % 256 == 0
        size[top] = 1.0
        opt = text.AdamW([torch.zeros(n, device="cuda")], rate=0.0, betas=(beta, 0.999), bits=8)
        slack, below, above = 1.001, 1 / (1 + 1 / 16 / (1 - beta)), 1 / (1 - 1 / 18 / (1 - beta))
        for factor in (1.0, -1.0, 0.3, -0.3, 0.0):
            g = torch.where(top, size, factor * size)
            for _ in range(300):
                opt.step([g])
            m = _values(opt, "m")[~top]
            if factor == 0.0:
                assert float(m.abs().max()) <= 2.0 ** -10 / (1 - beta) * float(opt.m_scale.max()) * slack
            else:
                ratio = m / g.double()[~top]
                assert below / slack <= float(ratio.min()) and float(ratio.max()) <= above * slack, (beta, factor)
    for beta in (0.95, 0.99):
        with pytest.raises(ValueError, match="beta1"):
            text.AdamW([torch.zeros(8, device="cuda")], betas=(beta, 0.999), bits=8)
        text.AdamW([torch.zeros(8, device="cuda")], betas=(beta, 0.999))
        opt = text.AdamW([torch.zeros(8, device="cuda")], bits=8, counted=True)
        opt.betas = (beta, 0.999)
        with pytest.raises(RuntimeError):
            opt.step([torch.ones(8, device="cuda")])
        assert int(opt.steps) == 0


def test_second_moments_of_8_bits_keep_their_average_down_to_the_smallest_number():
    """One step from zero, v of each size beside an element that sets the block's scale to 1 / 448 of its own.  On average what it should be, within six deviations of
    65280 roundings, half a step each at most; below the smallest number, 2^-9 of the scale, that number."""
    import torch
    from paper_2011_06295_amd import text
    n = 256 * 256
    top = torch.arange(n, device="cuda") % 256 == 0
    for times in (1e-3, 0.1, 0.9, 1.1, 1.5, 2.7, 7.3, 1000.0):          # v over the smallest number
        g = torch.full((n,), math.sqrt(times / 229376.0), device="cuda")
        g[top] = 1.0
        opt = text.AdamW([torch.zeros(n, device="cuda")], rate=0.0, betas=(0.9, 0.5), bits=8)
        opt.step([g])
        v, scale = _values(opt, "v")[~top], float(opt.v_scale[0])
        smallest = scale * 2.0 ** -9
        assert abs(float(_values(opt, "v")[top].min()) - 0.5) <= 4 * E
        if times < 1.0:
            assert bool((v == smallest).all())
        else:
            step = smallest * max(1.0, 2.0 ** (math.floor(math.log2(times)) - 3))
            assert abs(float(v.mean()) - 0.5 * times / 229376.0) <= 6 * 0.5 * step / math.sqrt(65280.0) + 1e-6 * float(v.mean()), times
