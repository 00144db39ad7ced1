"""Calls of the layers of include/lccrf_layers.h at the edges of what their header allows: repeated entries over the logits themselves."""
import pytest
import torch

import layers_reference as ref
from test_gpu_layers import DEV, TYPES, U, _dirty_memory, check, crf, generator, normal  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- distillation ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V,K", [(5003, 100), (9001, 128), (20011, 200), (40009, 256)])
def test_distill_over_the_logits_with_entries_that_only_repeat(crf, t, V, K):
    """From the 65th entry on every class has been named before: the loss reads their logits, nothing else does, and other waves overwrite them."""
    g = generator(V + K)
    logits, dloss = normal(g, 40, V, dtype=t, scale=3.0), normal(g, 40)
    first = torch.stack([torch.randperm(V, generator=g, device=DEV)[:64] for _ in range(40)])
    ids = first[:, torch.arange(K, device=DEV) % 64].to(torch.int32).contiguous()
    teacher = normal(g, 40, K)
    want = ref.distill(logits, ids, teacher, 2.0, dloss)
    apart_loss, over_loss = torch.empty(40, device=DEV), torch.empty(40, device=DEV)
    apart = crf.lccrf_distill_grad(dloss, logits, ids, teacher, temperature=2.0, loss=apart_loss)
    check(apart, want["dlogits"], "dlogits")
    check(apart_loss, want["loss"], "loss")
    for _ in range(3):
        over = logits.clone()
        assert torch.equal(crf.lccrf_distill_grad(dloss, over, ids, teacher, temperature=2.0, loss=over_loss, out=over), apart)
        assert torch.equal(over_loss, apart_loss)
