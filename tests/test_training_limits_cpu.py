"""Token embedding, AdamW over many tensors and gradient norm without a GPU: calls at the edge of what they take, which
are answered rightly or refused. Where a call would reach the device, a stand-in takes the library's place."""
import numpy as np
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


TABLE = np.dtype([("n", "i8"), ("data", "u8"), ("pad", "i4"), ("dtype", "i4")])


def test_tensors_that_stand_where_they_did_but_lie_otherwise_are_noticed():
    # a step walks a parameter's memory from its address on: as many elements as there were, in their order
    import torch
    from paper_2605_21442_amd.training import _native
    p = torch.zeros(6, 6)
    t = np.zeros(1, dtype=TABLE)
    stands = lambda x: _native().stand_at([x], t, TABLE.itemsize, 8, 0, 20)
    assert _native().describe([p], None, -1, t, TABLE.itemsize, 8, 0, 20) and stands(p)
    mine = p.data
    for other in (mine.t(), mine[:3], mine.view(torch.int32), mine.view(torch.bfloat16)[:3], torch._neg_view(mine)):
        p.data = other
        assert p.data_ptr() == mine.data_ptr() and not stands(p)
    p.data = mine.view(36)                             # the same memory, as other rows
    assert stands(p)
    x = torch.zeros(4, 8)
    part = x[1:3]
    assert _native().describe([part], None, -1, t, TABLE.itemsize, 8, 0, 20) and stands(part)
    x.untyped_storage().resize_(0)
    assert not stands(part)
    for bad in (None, 3, torch.eye(6).to_sparse(), torch.zeros(6, 6, device="meta")):
        assert not stands(bad)
    for offsets in ((8, -1, 20), (8, 0, -1), (8, 17, 20), (8, 0, 21), (20, 0, 20)):
        assert not _native().stand_at([p], t, TABLE.itemsize, *offsets), offsets


def test_a_subclass_with_memory_of_its_own_stands_too():
    import torch
    from paper_2605_21442_amd.training import _native

    class Logged(torch.Tensor):
        @classmethod
        def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
            with torch._C._DisableTorchDispatch():
                return func(*args, **(kwargs or {}))

    p = torch.zeros(6, 6)
    t = np.zeros(1, dtype=TABLE)
    assert _native().describe([p], None, -1, t, TABLE.itemsize, 8, 0, 20)
    assert _native().stand_at([p.as_subclass(Logged)], t, TABLE.itemsize, 8, 0, 20)
