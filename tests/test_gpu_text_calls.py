"""Calls of the text model's operators: sizes past one launch, and what a program that uses them beside PyTorch relies on."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _memory_goes_back():
    yield
    import torch
    torch.cuda.empty_cache()


def test_gradient_of_a_table_of_more_than_64_gb():
    """More zeros than one launch can write (2^32 threads of 16 bytes): few tokens, and none."""
    import torch
    from paper_2011_06295_amd import text
    vocab, dim = 4_300_003, 4096
    table = torch.full((vocab, dim), 7.0, device="cuda")
    layer = text.Embedding(table)
    rows = torch.tensor([0, 1, vocab // 2, vocab - 2, vocab - 1, 1], device="cuda")
    grad = torch.ones((6, dim), device="cuda")
    layer.backward(grad, rows, out=table)
    want = torch.tensor([1.0, 2.0, 1.0, 1.0, 1.0], device="cuda")[:, None].expand(5, dim)
    assert torch.equal(table[rows[:5]], want)
    table[rows[:5]] = 0.0
    assert sum(int(torch.count_nonzero(part)) for part in table.split(200_000)) == 0
    table.fill_(7.0)
    layer.backward(grad[:0], rows[:0], out=table)
    assert sum(int(torch.count_nonzero(part)) for part in table.split(200_000)) == 0


@pytest.mark.parametrize("case", [(1, 1_200_003, 131_071, 2, "f32"), (1, 2_500_001, 700, 1, "bf16"), (1300, 1000, 3_000_017, 3, "f16"), (1, 600_000, 5, 4, "f32")])
@pytest.mark.parametrize("first", [False, True])
def test_gradient_of_more_tokens_than_workgroups_sort_at_once(case, first):
    """Bound: a sum of m fp32 terms in any order, (m + 1) 2^-24 times the sum of their sizes."""
    import torch
    from paper_2011_06295_amd import text
    n, t, vocab, dim, dtype = case
    gen = torch.Generator(device="cuda").manual_seed(t)
    u = torch.rand((n, t), generator=gen, device="cuda", dtype=torch.float64)
    tokens = (u ** 3 * (vocab + 2)).long() - 1              # some rows have many tokens; both ends outside the table
    grad = torch.randn((n, t, dim), generator=gen, device="cuda").to({"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype])
    layer = text.Embedding(torch.empty((vocab, dim), device="cuda"))
    given = grad.transpose(1, 2)[:, :, None].contiguous() if first else grad
    out = layer.backward(given, tokens, channels_first=first)
    assert torch.equal(layer.backward(given, tokens, channels_first=first, out=torch.full_like(out, 7.0)), out)
    tok, g = tokens.reshape(-1).cpu(), grad.reshape(-1, dim).double().cpu()
    keep = (tok >= 0) & (tok < vocab)
    ref, size, count = (torch.zeros((vocab, dim), dtype=torch.float64) for _ in range(3))
    for total, terms in ((ref, g), (size, g.abs()), (count, torch.ones_like(g))):
        total.index_add_(0, tok[keep], terms[keep])
    bound = (count + 1) * 2.0 ** -24 * size
    assert bool(((out.double().cpu() - ref).abs() <= bound + 2.0 ** -24 * (ref.abs() + bound) + 2.0 ** -149).all())


@pytest.mark.parametrize("dim", [2 ** 31 - 1, 2 ** 31 - 300, 2 ** 31 - 514])
def test_vectors_of_nearly_2_to_the_31(dim):
    """The longest rows: their last pieces and column blocks end next to what an int holds."""
    import torch
    from paper_2011_06295_amd import text
    dtype = torch.float16
    table = torch.full((1, dim), 3.0, dtype=dtype, device="cuda")
    places = torch.tensor([0, 1, 4095, dim // 2, dim - 514, dim - 9, dim - 2, dim - 1], device="cuda")
    table[0, places] = torch.arange(1, 9, device="cuda", dtype=dtype)
    layer = text.Embedding(table, scale=2.0)
    tokens = torch.zeros(1, dtype=torch.int64, device="cuda")

    def is_twice_the_table(y):
        return all(torch.equal(a, b * 2.0) for a, b in zip(y.split(1 << 28), table[0].split(1 << 28)))

    y = layer.forward(tokens)
    assert is_twice_the_table(y[0])
    g = layer.backward(table, tokens, out=y)
    assert is_twice_the_table(g[0])


def test_out_of_memory_is_pytorch_s_own_exception():
    """Outputs and scratch memory of more bytes than the card has: the allocator refuses them before anything is enqueued."""
    import torch
    from paper_2011_06295_amd import text
    tokens = torch.zeros(1 << 20, dtype=torch.int32, device="cuda")
    wide = text.Embedding(torch.zeros((2, 1 << 20), dtype=torch.float16, device="cuda"))
    with pytest.raises(torch.OutOfMemoryError):
        wide.forward(tokens)
    layer = text.Int8Linear.from_quantized(torch.zeros((1 << 20, 1), dtype=torch.int8, device="cuda"), torch.ones(1 << 20, device="cuda"))
    with pytest.raises(torch.OutOfMemoryError):
        layer.forward(torch.zeros((1 << 20, 1), device="cuda"))
    assert wide.forward(tokens[:1]).shape == (1, 1 << 20)       # the next call runs


def test_writes_into_a_given_tensor_raise_its_version():
    import torch
    from paper_2011_06295_amd import text
    emb = text.Embedding(torch.ones((10, 4), device="cuda"))
    tokens = torch.zeros(3, dtype=torch.int64, device="cuda")
    out = torch.zeros((3, 4), device="cuda")
    layer = text.Int8Linear(torch.ones((5, 4), device="cuda"))
    y = torch.zeros((3, 5), device="cuda")
    for tensor, call in ((out, lambda: emb.forward(tokens, out=out)), (emb.table, lambda: emb.backward(out, tokens, out=emb.table, accumulate=True)),
                         (y, lambda: layer.forward(out, out=y))):
        before = tensor._version
        call()
        assert tensor._version > before
    # what autograd has saved and a call overwrites: noticed by backward
    x = torch.ones((3, 4), device="cuda", requires_grad=True)
    kept = torch.ones((3, 4), device="cuda")
    product = (x * kept).sum()
    emb.forward(tokens, out=kept)
    with pytest.raises(RuntimeError):
        product.backward()
    with torch.inference_mode():
        held = torch.zeros((3, 4), device="cuda")
        emb.forward(tokens, out=held)
    assert torch.equal(emb.forward(tokens, out=held), emb.forward(tokens))      # an inference tensor has no version


def test_model_s_gradient_is_of_the_tokens_that_forward_saw():
    import torch
    from paper_2011_06295_amd import text_model
    model = text_model.TextModel.synthetic(vocab=500)
    tokens, _ = text_model.sentences(8, 64, 500)
    other, _ = text_model.sentences(8, 64, 500, seed=3)
    g = torch.ones((8, 6), device="cuda")
    model.forward(tokens)
    want = model.table_gradient(g)
    batch = tokens.clone()                  # a buffer that the program fills anew for each batch
    model.forward(batch)
    batch.copy_(other)
    assert torch.equal(model.table_gradient(g), want)
    model.close()


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("count", [1, 60, 5000, 9000])
def test_64_bit_tokens_whose_low_32_bits_name_a_row(first, count):
    """They lie outside the table: zeros, and no gradient, on every path (one look at a token's low bits among them)."""
    import torch
    from paper_2011_06295_amd import text
    vocab, dim = 600, 24
    gen = torch.Generator(device="cuda").manual_seed(count)
    table = torch.randn((vocab, dim), generator=gen, device="cuda")
    inside = torch.randint(0, vocab, (2, count), generator=gen, device="cuda")
    far = torch.tensor([1 << 32, -(1 << 32), 1 << 40, -(1 << 63), (1 << 63) - (1 << 32), -(1 << 31) * 2 * 3], device="cuda")
    tokens = inside + far[torch.randint(0, len(far), inside.shape, generator=gen, device="cuda")]
    assert bool(((tokens & 0xffffffff) == inside).all())
    layer = text.Embedding(table)
    assert int(torch.count_nonzero(layer.forward(tokens, channels_first=first))) == 0
    kept = torch.rand(inside.shape, generator=gen, device="cuda") < 0.5
    kept[0, 0] = True
    tokens = torch.where(kept, inside, tokens)
    y = layer.forward(tokens, channels_first=first)
    want = table[inside] * kept[..., None]
    assert torch.equal(y, want.transpose(1, 2)[:, :, None] if first else want)
    g = torch.ones_like(y)
    named = torch.zeros(vocab, device="cuda").index_add_(0, inside[kept], torch.ones(int(kept.sum()), device="cuda"))
    out = layer.backward(g, tokens, channels_first=first)
    assert torch.equal(out, named[:, None].expand(vocab, dim))         # whole numbers: exact in fp32


@pytest.mark.parametrize("relu", [False, True])
def test_layer_s_outputs_past_the_largest_binary16(relu):
    """They are infinities of the right sign (zero below, with ReLU), whichever kernel multiplies."""
    import torch
    from paper_2011_06295_amd import text
    for M, K, N in ((1, 256, 64), (3, 4096, 70), (40, 1000, 300), (300, 1000, 260), (2048, 512, 2048)):
        sign = torch.where(torch.arange(N, device="cuda") % 2 == 0, 1.0, -1.0)
        layer = text.Int8Linear.from_quantized(torch.full((N, K), 100, dtype=torch.int8, device="cuda"), sign * 1e3, relu=relu)
        y = layer.forward(torch.ones((M, K), device="cuda"), dtype=torch.float16)
        want = sign * float("inf")
        assert torch.equal(y, (want.clamp(min=0.0) if relu else want).to(torch.float16).expand(M, N)), (M, K, N)
