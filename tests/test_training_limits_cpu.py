"""Token embedding, AdamW over many tensors and gradient norm without a GPU: calls at the edge of what they take, which
are answered rightly or refused. Where a call would reach the device, a stand-in takes the library's place."""
import pytest


@pytest.mark.parametrize("grad_enabled", [True, False])
def test_a_forward_mode_derivative_is_refused_and_not_dropped(monkeypatch, grad_enabled):
    # a dual weight does not require grad, yet its tangent would be lost on the way past autograd
    import torch
    from torch.autograd import forward_ad
    from paper_2605_21442_amd import training as TR
    monkeypatch.setattr(TR, "embedding_forward", lambda ids, w, *a, **k: (w.detach()[ids], None))
    ids, w = torch.tensor([1, 2]), torch.randn(4, 8)
    with forward_ad.dual_level(), torch.set_grad_enabled(grad_enabled):
        with pytest.raises(NotImplementedError, match="forward mode"):
            TR.token_embedding(ids, forward_ad.make_dual(w, torch.ones_like(w)))
        assert torch.equal(TR.token_embedding(ids, w), w[ids])          # (without a tangent nothing is refused)
