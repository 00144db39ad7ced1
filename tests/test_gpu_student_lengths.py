"""A student tagger (paper_2308_03291_amd/tagger.py) and a teacher whose tags past the lengths are not masked."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_positions_past_the_lengths_do_not_count():
    """A teacher's emissions there are anything: loss and gradients are those of a teacher that names no tag there."""
    from paper_2308_03291_amd import tagger
    V, T, N = 30, 6, 25
    s = tagger.Student(V, T, 12, 16, 4, seed=5)
    ids, tags, lengths = tagger.language(7, N, V, T, seed=6)
    assert int(lengths.min()) < N
    emit = 3 * torch.randn(7, N, T, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    masked, bare = tagger.top_emissions(emit, 3, lengths), tagger.top_emissions(emit, 3)
    assert bool((masked[0] < 0).any()) and not bool((bare[0] < 0).any())
    want, want_grads = s.loss_and_gradients(ids, tags, lengths, teacher=masked, share=0.4)
    loss, grads = s.loss_and_gradients(ids, tags, lengths, teacher=bare, share=0.4)
    assert torch.equal(loss, want)
    for k in want_grads:
        assert torch.equal(grads[k], want_grads[k]), k
