"""The operators that train what follows the convolutions of a text model, as its program calls them: a fully connected
layer with bias, activation and residual, its gradients, the loss of a classifier with the gradient of its logits, and an
AdamW step over many tensors at once.

A case is one call (`kind` "linear", "gradient", "loss" or "adamw").  Sizes are those of this repository's own text model
(128 sentences, 200 features, 6 classes, a table of 20000 x 300) and general ones of language models, from one token to
tens of thousands.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 256          # elements that share a scale where states take 8 bits
RATE, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
TAKEN = 100          # steps that came before the one measured

# tensors of an AdamW step: shapes
SETS = {
    # the text model: word vectors, a hidden layer, the classifier
    "text": [(20000, 300), (256, 200), (256,), (6, 256), (6,)],
    # a deep stack of narrow layers: matrices, biases and norms, some of odd sizes
    "deep": [(512, 512), (512,), (512, 1024), (1024,), (1024, 512), (512,), (511, 129), (7,)] * 24,
    # the layers of a wide model
    "wide": [(4096, 4096), (4096,), (10240, 4096), (4096, 10240)] * 2 + [(32768, 4096)],
}


def linear(name, dtype, m, k, n, act=None, residual=False, keep=False):
    """act: None, "relu", "gelu" or "silu".  keep: what goes into the activation is an output too, for the gradients."""
    case = dict(kind="linear", dtype=dtype, m=m, k=k, n=n, act=act or "", residual=residual, keep=keep)
    return dict(case, name=name) if name else case


def gradient(name, dtype, m, k, n, act=None):
    """Gradients of the input, the weights and the bias."""
    case = dict(kind="gradient", dtype=dtype, m=m, k=k, n=n, act=act or "")
    return dict(case, name=name) if name else case


def loss(name, dtype, m, n, masked=False):
    """m rows of n classes.  masked: some rows do not count, and some classes are forbidden (minus infinity)."""
    case = dict(kind="loss", dtype=dtype, m=m, n=n, masked=masked)
    return dict(case, name=name) if name else case


def adamw(name, dtype, tensors, bits=32, master=False):
    """tensors: a set above, or shapes as text ("5x300,7").  bits: of the states.  master: 32-bit weights are kept beside."""
    case = dict(kind="adamw", dtype=dtype, tensors=tensors, bits=bits, master=master)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token while a model answers: the weights are read once
        linear("linear_one_bf16", "bf16", 1, 4096, 4096, act="silu", residual=True),
        # the tokens of some answers at a time
        linear("linear_few_f16", "f16", 24, 4096, 8192, act="gelu"),
        # odd sizes throughout, in fp32
        linear("linear_ragged_f32", "f32", 203, 1001, 1111, act="relu", residual=True),
        # a long prompt or a training batch on a wide layer, with what its gradients need
        linear("linear_large_bf16", "bf16", 8192, 4096, 8192, act="gelu", keep=True),
        # the text model's classifier in training
        gradient("gradient_text_f32", "f32", 128, 200, 256, act="relu"),
        # odd sizes throughout, in binary16
        gradient("gradient_odd_f16", "f16", 1021, 1001, 777, act="silu"),
        # a training batch on a wide layer: the largest products
        gradient("gradient_large_bf16", "bf16", 8192, 4096, 8192, act="gelu"),
        # the text model's loss
        loss("loss_text_f32", "f32", 128, 6),
        # a training batch of a language model: a large table of words, padded sentences
        loss("loss_words_bf16", "bf16", 4096, 65536, masked=True),
        # the text model's parameters
        adamw("adamw_text_f32", "f32", "text"),
        # many small tensors in binary16 with 32-bit weights beside them
        adamw("adamw_deep_f16", "f16", "deep", bits=32, master=True),
        # a wide model whose states take 8 bits
        adamw("adamw_wide_bf16", "bf16", "wide", bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, at most as much work as the largest listed one of its kind."""
    most = {}
    for case in listed():
        cost, kind = work(case), case["kind"]
        most[kind] = [max(a, b) for a, b in zip(most.get(kind, [0, 0]), (cost["bytes"], cost["flops"]))]
    while True:
        kind = rng.choice(("linear", "linear", "gradient", "loss", "adamw"))
        dtype = rng.choice(("f32", "f16", "bf16"))
        if kind in ("linear", "gradient"):
            m = rng.choice((1, _log_int(rng, 1, 64), _log_int(rng, 1, 8192))) if kind == "linear" else _log_int(rng, 8, 8192)
            k, n = _log_int(rng, 64, 8192), _log_int(rng, 6, 8192)
            if rng.random() < 0.6:       # most layers are whole numbers of 64
                k, n = -(-k // 64) * 64, -(-n // 64) * 64
            act = rng.choice((None, "relu", "gelu", "silu"))
            if kind == "linear":
                case = linear("", dtype, m, k, n, act, rng.random() < 0.4, rng.random() < 0.3)
            else:
                case = gradient("", dtype, m, k, n, act)
        elif kind == "loss":
            n = _log_int(rng, 2, 131072)
            case = loss("", dtype, _log_int(rng, 1, 16384), n, n >= 16 and rng.random() < 0.5)
        else:
            shapes = []
            for _ in range(_log_int(rng, 1, 150)):
                rows, cols = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
                shapes.append(str(cols) if rng.random() < 0.4 else "%dx%d" % (rows, cols))
            bits = rng.choice((8, 32))
            case = adamw("", dtype, ",".join(shapes), bits, dtype != "f32" and rng.random() < 0.4)
        cost = work(case)
        if cost["bytes"] <= most[kind][0] and cost["flops"] <= most[kind][1]:
            return case


def _shapes(case):
    given = SETS.get(case["tensors"])
    return given or [tuple(int(v) for v in shape.split("x")) for shape in case["tensors"].split(",")]


def work(case):
    """linear: input, weights, bias, residual, outputs.  gradient: the gradient that comes in, what went into the activation,
    input, weights, the three gradients.  loss: logits, labels, weights of rows, losses, gradient.  adamw: gradients are read,
    parameters and states read and written."""
    kind, b = case["kind"], BYTES[case["dtype"]]
    if kind == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": (m * k + n * k + m * n * (1 + case["residual"] + case["keep"])) * b + 4 * n, "flops": 2 * m * n * k}
    if kind == "gradient":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": (m * n * (2 if case["act"] else 1) + 2 * m * k + 2 * n * k) * b + 4 * n, "flops": 4 * m * n * k}
    if kind == "loss":
        m, n = case["m"], case["n"]
        return {"bytes": 2 * m * n * b + m * 16, "flops": 5 * m * n}
    count = sum(math.prod(shape) for shape in _shapes(case))
    state = 4 if case["bits"] == 32 else 1
    each = b + 4 * state + (8 + b if case["master"] else 2 * b)
    scales = 16 * count // BLOCK if case["bits"] == 8 else 0
    return {"bytes": each * count + scales, "flops": 14 * count}


# ---------------------------------------------------------------- what a program has in hand

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _rand(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda", dtype=torch.float32)


def _begins(case):
    """First element of each tensor, and of what would follow: each begins at a whole number of blocks."""
    begins = [0]
    for shape in _shapes(case):
        begins.append(begins[-1] + -(-math.prod(shape) // BLOCK) * BLOCK)
    return begins


def _filled(case, flat):
    """`flat` with zeros behind each tensor's last element."""
    begins = _begins(case)
    for begin, end, shape in zip(begins, begins[1:], _shapes(case)):
        flat[begin + math.prod(shape):end] = 0.0
    return flat


def _views(case, flat):
    return [flat[begin:begin + math.prod(shape)].view(shape) for begin, shape in zip(_begins(case), _shapes(case))]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, kind = TYPES[case["dtype"]], case["kind"]
    state = {"case": case}
    if kind in ("linear", "gradient"):
        m, k, n = case["m"], case["k"], case["n"]
        state["x"] = _randn(gen, m, k).to(dtype)
        state["w"] = (_randn(gen, n, k) / math.sqrt(k)).to(dtype)
        state["bias"] = 0.1 * _randn(gen, n)
        if kind == "gradient":
            state["grad"] = _randn(gen, m, n).to(dtype)
            state["z"] = _randn(gen, m, n).to(dtype)
        elif case["residual"]:
            state["residual"] = _randn(gen, m, n).to(dtype)
        if own:
            from paper_2011_06295_amd import text
            state["layer"] = text.Linear(state["w"], state["bias"], activation=case["act"] or None)
        return state
    if kind == "loss":
        m, n = case["m"], case["n"]
        logits = 2.0 * _randn(gen, m, n)
        state["labels"] = torch.randint(0, n, (m,), generator=gen, device="cuda")
        state["weights"] = torch.full((m,), 1.0 / m, device="cuda")
        if case["masked"]:
            forbidden = _rand(gen, n) < 0.1
            forbidden[0] = False
            logits[:, forbidden] = -math.inf
            state["labels"] = torch.where(forbidden[state["labels"]], 0, state["labels"])
            state["weights"] *= _rand(gen, m) < 0.8
        state["logits"] = logits.to(dtype)
        return state
    # in the middle of training
    total = _begins(case)[-1]
    size = torch.exp(2.0 * _randn(gen, total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1) * 1e-3      # gradients differ from place to place
    state["grad"] = _filled(case, _randn(gen, total) * size).to(dtype)
    weights = _filled(case, 0.05 * _randn(gen, total))
    m = _filled(case, 0.3 * _randn(gen, total) * size)
    v = _filled(case, (0.05 + 0.1 * _rand(gen, total)) * size * size)
    state["p"] = weights.to(dtype)
    state["master"] = weights if case["master"] else None
    state["m"], state["m_scale"], state["v"], state["v_scale"] = m, None, v, None
    if case["bits"] == 8:
        state["m"], state["m_scale"] = (t.clone() for t in _codes(m))
        state["v"], state["v_scale"] = (t.clone() for t in _codes(v, torch.full_like(v, 0.5)))
        if not own:      # places within the tensors, which the rounding of v goes by
            begins = torch.tensor(_begins(case), device="cuda")
            at = torch.arange(total, device="cuda")
            state["place"] = at - begins[torch.searchsorted(begins, at, right=True) - 1]
    state["step"] = TAKEN
    if own:
        from paper_2011_06295_amd import text
        optimizer = text.AdamW(_views(case, state["p"]), rate=RATE, betas=(BETA1, BETA2), eps=EPS, decay=DECAY, bits=case["bits"],
                               master=case["master"])
        optimizer.steps = TAKEN
        for name in ("m", "v", "m_scale", "v_scale", "master"):
            if state[name] is not None:
                getattr(optimizer, name).copy_(state[name])
        state["optimizer"], state["grads"] = optimizer, _views(case, state["grad"])
    return state


# ---------------------------------------------------------------- 8-bit states

def _codes(x, noise=None):
    """(numbers of 8 bits, e4m3, and fp32 scales) of x, a scale for each block: the largest size over 448.  To the nearest number; with
    noise (0 <= noise < 1) up where what is left of a whole step and the noise pass one, and to the smallest number at least."""
    x = x.reshape(-1, BLOCK)
    largest = x.abs().amax(1, keepdim=True)
    counts = largest >= 2.0 ** -100
    y = x * torch.where(counts, 448.0 / torch.where(counts, largest, 1.0), 0.0)
    if noise is not None:
        exponent = torch.frexp(y).exponent - 4                       # a number of 8 bits has 4 digits, and 2^-9 is the smallest
        step = torch.ldexp(torch.ones_like(y), exponent.clamp(min=-9))
        whole = torch.floor(y / step + noise.reshape(-1, BLOCK)) * step
        y = torch.where(y > 0.0, whole.clamp(min=2.0 ** -9), 0.0)
    y = y.clamp(-448.0, 448.0)
    return y.to(torch.float8_e4m3fn).reshape(-1), torch.where(counts, largest / 448.0, 0.0).reshape(-1)


def _noise(place, step):
    """Numbers in [0, 1) that depend on an element's place in its tensor and on the step alone: a 32-bit integer hash."""
    low = 0xffffffff
    h = (place * 0x9e3779b9 + step * 0xbb67ae85) & low
    h = ((h ^ (h >> 16)) * 0x6a09e667) & low
    h = ((h ^ (h >> 15)) * 0xbb67ae85) & low
    return ((h ^ (h >> 16)) >> 8).float() * 2.0 ** -24


# ---------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    kind, dtype = case["kind"], TYPES[case["dtype"]]
    if own:
        if kind == "linear":
            return state["layer"].forward(state["x"], residual=state.get("residual"), keep=case["keep"])
        if kind == "gradient":
            return state["layer"].backward(state["grad"], state["x"], state["z"] if case["act"] else None)
        if kind == "loss":
            from paper_2011_06295_amd import text
            return text.cross_entropy(state["logits"], state["labels"], state["weights"])
        optimizer = state["optimizer"]
        optimizer.step(state["grads"])
        kept = [optimizer.m, optimizer.v] + ([optimizer.m_scale, optimizer.v_scale] if case["bits"] == 8 else [])
        return [state["p"]] + kept + ([optimizer.master] if case["master"] else [])
    if kind == "linear":
        z = state["x"].float() @ state["w"].float().t() + state["bias"]
        y = _act(z, case["act"])
        if case["residual"]:
            y = y + state["residual"].float()
        return (y.to(dtype), z.to(dtype)) if case["keep"] else y.to(dtype)
    if kind == "gradient":
        g = state["grad"].float()
        if case["act"]:
            g = g * _slope(state["z"].float(), case["act"])
        return (g @ state["w"].float()).to(dtype), (g.t() @ state["x"].float()).to(dtype), g.sum(0)
    if kind == "loss":
        z, labels, weights = state["logits"].float(), state["labels"][:, None], state["weights"][:, None]
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        losses = (torch.log(total) + top - z.gather(1, labels)) * weights
        p = e / total
        p.scatter_add_(1, labels, torch.full_like(weights, -1.0))
        return losses[:, 0], (p * weights).to(dtype)
    return _step(state)


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0.0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _step(state):
    case, g = state["case"], state["grad"].float()
    state["step"] += 1
    small = case["bits"] == 8
    m, v = state["m"], state["v"]
    if small:
        m = (m.float().reshape(-1, BLOCK) * state["m_scale"][:, None]).reshape(-1)
        v = (v.float().reshape(-1, BLOCK) * state["v_scale"][:, None]).reshape(-1)
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * (g * g)
    p = state["master"] if case["master"] else state["p"].float()
    unbiased = torch.sqrt(v / (1.0 - BETA2 ** state["step"])) + EPS
    p = p * (1.0 - RATE * DECAY) - (RATE / (1.0 - BETA1 ** state["step"])) * m / unbiased
    if small:
        m, m_scale = _codes(m)
        v, v_scale = _codes(v, _noise(state["place"], state["step"]))
        state["m_scale"].copy_(m_scale)
        state["v_scale"].copy_(v_scale)
    state["m"].copy_(m)
    state["v"].copy_(v)
    state["p"].copy_(p)
    kept = [state["p"], state["m"], state["v"]] + ([state["m_scale"], state["v_scale"]] if small else [])
    if case["master"]:
        state["master"].copy_(p)
        kept.append(state["master"])
    return kept


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """The definitions in 64 bits.  For states of 8 bits: the values over their scales, before they are rounded."""
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind in ("linear", "gradient"):
        x, w = state["x"].double(), state["w"].double()
        if kind == "linear":
            z = torch.addmm(state["bias"].double(), x, w.t().contiguous())
            y = {"": lambda: z, "relu": lambda: z * (z > 0), "gelu": lambda: z * (1.0 - 0.5 * torch.erfc(z / math.sqrt(2.0))),
                 "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
            if case["residual"]:
                y = y + state["residual"].double()
            return (y, z) if case["keep"] else y
        grad, z = state["grad"].double(), state["z"].double()
        if case["act"] == "relu":
            grad = torch.where(z > 0, grad, torch.zeros_like(grad))
        elif case["act"] == "gelu":
            grad = grad * (1.0 - 0.5 * torch.erfc(z / math.sqrt(2.0)) + z * torch.exp(-z.square() / 2.0) / math.sqrt(2.0 * math.pi))
        elif case["act"] == "silu":
            s = torch.sigmoid(z)
            grad = grad * (s + z * s * torch.sigmoid(-z))
        return torch.mm(grad, w), torch.mm(grad.t().contiguous(), x), torch.mv(grad.t().contiguous(), torch.ones(case["m"], device="cuda", dtype=torch.float64))
    if kind == "loss":
        rows = torch.arange(case["m"], device="cuda")
        losses, grad = [], []
        for part in rows.split(1024):      # some rows at a time
            z, label, weight = state["logits"][part].double(), state["labels"][part], state["weights"][part].double()
            total = torch.logsumexp(z, 1)
            losses.append((total - z[torch.arange(len(part), device="cuda"), label]) * weight)
            p = torch.exp(z - total[:, None])
            p[torch.arange(len(part), device="cuda"), label] -= 1.0
            grad.append(p.mul_(weight[:, None]))
        return torch.cat(losses), torch.cat(grad)
    g, step, small = state["grad"].double(), state["step"] + 1, case["bits"] == 8
    m, v = state["m"].double(), state["v"].double()
    if small:
        m = m * state["m_scale"].double().repeat_interleave(BLOCK)
        v = v * state["v_scale"].double().repeat_interleave(BLOCK)
    m = m + (g - m) * (1.0 - BETA1)
    v = v + (g * g - v) * (1.0 - BETA2)
    p = (state["master"] if case["master"] else state["p"]).double()
    p = p - RATE * DECAY * p - RATE * (m / (1.0 - BETA1 ** step)) / (torch.sqrt(v / (1.0 - BETA2 ** step)) + EPS)
    kept = [p, m, v]
    if small:
        scales = [t.reshape(-1, BLOCK).abs().amax(1) / 448.0 for t in (m, v)]
        kept[1:] = [torch.where(s > 0, t.reshape(-1, BLOCK).t() / s, 0.0).t().reshape(-1) for t, s in zip((m, v), scales)] + scales
    return kept + ([p] if case["master"] else [])
