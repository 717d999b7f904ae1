"""The MLP block of examples/mlp_block.py on batches smaller than it was made for."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def one_step(block, X, dY):
    Y = block.forward(X).clone()
    block.search(11)
    dX = block.backward(dY).clone()
    torch.cuda.synchronize()
    assert int(block.fc1.b["status_word"].item()) == 0 and int(block.fc2.b["status_word"].item()) == 0
    return [Y, dX] + [t.clone() for layer in (block.fc1, block.fc2) for t in (layer.db, layer.b["dW"])]


@pytest.mark.parametrize("most,T,width,hidden", [(300, 97, 128, 352), (300, 1, 64, 96), (64, 63, 160, 64), (5696, 5632, 1536, 256)])
def test_a_smaller_batch_gives_what_a_block_of_its_size_gives(most, T, width, hidden):
    """Bit for bit, after a step on the full batch has left its values in every buffer.  5632 of 5696 tokens: the smaller batch
    is cut into more pieces."""
    import mlp_block
    g = torch.Generator(device="cuda").manual_seed(9)
    rows = torch.randn(2, most, width, generator=g, device="cuda").to(torch.bfloat16)
    X, dY = rows[0, :T].contiguous(), rows[1, :T].contiguous()
    large, exact = mlp_block.SparseMLP(most, width, hidden, seed=3), mlp_block.SparseMLP(T, width, hidden, seed=3)
    one_step(large, rows[0].contiguous(), rows[1].contiguous())
    got, want = one_step(large, X, dY), one_step(exact, X, dY)
    for a, b in zip(got, want):
        assert a.shape == b.shape and torch.equal(a, b)


def test_more_tokens_than_the_block_was_made_for_are_refused():
    import mlp_block
    block = mlp_block.SparseMLP(8, 64, 96)
    with pytest.raises(ValueError, match="at most 8"):
        block.forward(torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda"))
