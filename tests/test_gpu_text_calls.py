"""Calls of the text model's operators: sizes past one launch, and what a program that uses them beside PyTorch relies on."""
import pytest

pytestmark = pytest.mark.gpu


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
