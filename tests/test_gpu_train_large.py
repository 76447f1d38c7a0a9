"""Arrays of more than 2^31 elements through the layer, its gradients, the loss and AdamW: what lies past the 32-bit offsets against 64 bits.  Bounds as in
test_gpu_train.py."""
import math

import pytest

from test_gpu_train import E, TINY, U, _act, _mm, _slope, _within

pytestmark = pytest.mark.gpu


def _bf16(gen, *shape):
    import torch
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("K,N", [(16, 4096), (512, 4104)])
def test_layer_and_gradients(K, N):
    """2^31 outputs and more; the last rows, and those around the 2^31st element, of the layer, of z and of grad_x; the sums over all rows."""
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(71)
    M = 2 ** 31 // N + 5000
    x, w, bias = _bf16(gen, M, K), (torch.randn((N, K), generator=gen, device="cuda") / math.sqrt(K)).to(torch.bfloat16), torch.randn(N, generator=gen, device="cuda")
    layer = text.Linear(w, bias, activation="silu")
    y, z = layer.forward(x, keep=True)
    middle = 2 ** 31 // N
    rows = torch.cat([torch.arange(64, device="cuda"), torch.arange(middle - 64, middle + 64, device="cuda"), torch.arange(M - 200, M, device="cuda")])
    exact, off = _mm(x[rows], w) + bias.double(), 2 * (K + 2) * E * (_mm(x[rows].abs(), w.abs()) + bias.double().abs())
    _within(z[rows], exact, off + U["bf16"] * (exact.abs() + off) + TINY["bf16"], (K, N, "z"))
    ref, bound = _act(exact, "silu"), 1.13 * off + 8 * E * (1 + exact.abs())
    _within(y[rows], ref, bound + U["bf16"] * (ref.abs() + bound) + TINY["bf16"], (K, N))
    del y
    g = _bf16(gen, M, N)
    gx, gw, gb = layer.backward(g, x, z)
    sums = [torch.zeros((N, K), dtype=torch.float64, device="cuda") for _ in range(3)] + [torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(3)]

    def behind(part):
        d = g[part].double() * _slope(z[part].double(), "silu")
        off = 9 * E * g[part].double().abs()
        return d, off, off + U["bf16"] * (d.abs() + off) + TINY["bf16"]
    d, off, rounded = behind(rows)
    size, wrong = d.abs() @ w.double().abs(), rounded @ w.double().abs()
    ref, bound = d @ w.double(), wrong + 2 * (N + 2) * E * (size + wrong)
    _within(gx[rows], ref, bound + U["bf16"] * (ref.abs() + bound) + TINY["bf16"], (K, N, "x"))
    for part in torch.arange(M, device="cuda").split(40000):
        d, off, rounded = behind(part)
        xd = x[part].double()
        for total, term in zip(sums, (d.t().contiguous() @ xd, d.abs().t().contiguous() @ xd.abs(), rounded.t().contiguous() @ xd.abs(), d.sum(0), d.abs().sum(0), off.sum(0))):
            total += term
    bound = sums[2] + 2 * (M + 2) * E * (sums[1] + sums[2])
    _within(gw, sums[0], bound + U["bf16"] * (sums[0].abs() + bound) + TINY["bf16"], (K, N, "weight"))
    bound = sums[5] + 2 * (M + 2) * E * (sums[4] + sums[5])
    _within(gb, sums[3], bound + E * sums[3].abs(), (K, N, "bias"))
    # (the bounds of sums over so many rows are wide: a gradient of the last row alone shows that it is among them)
    only = torch.zeros_like(g)
    only[M - 1] = g[M - 1]
    _, gw, gb = layer.backward(only, x, z, grad_x=False)
    d, off, rounded = (t.t().contiguous() for t in behind(torch.tensor([M - 1], device="cuda")))
    last = x[M - 1:].double()
    ref, bound = d @ last, rounded @ last.abs() + 6 * E * ((d.abs() + rounded) @ last.abs())
    _within(gw, ref, bound + U["bf16"] * (ref.abs() + bound) + TINY["bf16"], (K, N, "weight of one row"))
    _within(gb, d[:, 0], off[:, 0] + 6 * E * d[:, 0].abs(), (K, N, "bias of one row"))


@pytest.mark.parametrize("rows,classes", [(32800, 65536), (32800, 65600), (54_000_000, 40)])
def test_loss(rows, classes):
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(72)
    logits = _bf16(gen, rows, classes)
    labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
    middle = 2 ** 31 // classes
    at = torch.cat([torch.arange(middle - 8, middle + 8, device="cuda"), torch.arange(rows - 32, rows, device="cuda")])
    z, label = logits[at].double(), labels[at][:, None]
    loss, grad = text.cross_entropy(logits, labels, grad=logits)
    assert grad.data_ptr() == logits.data_ptr()
    lse = torch.logsumexp(z, 1, keepdim=True)
    of_sum = 2 * (168 + classes / 1024) * E
    ref = (lse - z.gather(1, label))[:, 0]
    _within(loss[at], ref, of_sum + 2 * E * (z.amax(1).abs() + z.gather(1, label)[:, 0].abs() + 2 * lse[:, 0].abs()) + 4 * E * ref.abs(), (rows, classes))
    p = torch.exp(z - lse)
    ref = p.scatter_add(1, label, torch.full_like(lse, -1.0))
    off = p * (of_sum + 4 * E * ((z - lse).abs() + 2 * lse.abs() + 4)) + 4 * E * (ref.abs() + (p > 0.5))
    _within(grad[at], ref, off + U["bf16"] * (ref.abs() + off) + TINY["bf16"], (rows, classes))


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits):
    import torch
    from paper_2011_06295_amd import text
    gen = torch.Generator(device="cuda").manual_seed(73)
    n = 2 ** 31 + 70_001
    p, g = torch.empty(n, dtype=torch.bfloat16, device="cuda"), torch.empty(n, dtype=torch.bfloat16, device="cuda")
    for t in (p, g):
        for part in t.split(2 ** 28):
            part.normal_(generator=gen)
    at = torch.cat([torch.arange(1000, device="cuda"), torch.arange(2 ** 31 - 1000, n, device="cuda")])
    before, grad = p[at].double(), g[at].double()
    opt = text.AdamW([p], rate=1e-2, betas=(0.9, 0.98), eps=1e-6, decay=0.1, bits=bits)
    opt.step([g])
    ref = before * (1 - 1e-2 * 0.1) - 1e-2 * grad / (grad.abs() + 1e-6)
    off = 16 * E * 1e-2 + 4 * E * before.abs()
    _within(p[at], ref, off + U["bf16"] * (ref.abs() + off), bits)
    if bits == 32:
        _within(opt.m[at], 0.1 * grad, 4 * E * grad.abs(), "m")
        _within(opt.v[at], 0.02 * grad * grad, 5 * E * grad * grad, "v")
    else:
        blocks = at // 256
        for name, exact, half in (("m", 0.1 * grad, 0.5), ("v", 0.02 * grad * grad, 1.0)):
            scale = getattr(opt, name + "_scale")[blocks].double()
            got = getattr(opt, name)[at].double() * scale
            unit = torch.maximum(scale * 2.0 ** -9, exact.abs() * 2.0 ** -3)
            _within(got, exact, 16 * E * exact.abs() + unit * half * (1 + 2.0 ** -20), name)
