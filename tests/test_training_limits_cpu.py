"""Token embedding, AdamW over many tensors and gradient norm without a GPU: calls at the edge of what they take, which
are answered rightly or refused. Where a call would reach the device, a stand-in takes the library's place."""
import ctypes
import types

import numpy as np
import pytest


class OnGpu:
    """Host tensors that AdamWTensors takes for parameters, and the calls that it makes of the library: for each its table of
    tensors, its constants, and its bits."""

    def __init__(self, monkeypatch):
        import torch
        from paper_2605_21442_amd import training as TR
        native = TR._native()
        here = types.SimpleNamespace(stand_at=native.stand_at, changed=native.changed,
                                     describe=lambda tensors, shapes, device, *a: native.describe(tensors, shapes, -1, *a))

        class Param(torch.Tensor):
            is_cuda = property(lambda self: True)

        def call(table, count, groups, n_groups, bits, scale, seed, stream):
            rows = (ctypes.c_char * (count * TR._TENSOR.itemsize)).from_address(table)
            opts = [TR.B.LceAdamW.from_address(groups + k * ctypes.sizeof(TR.B.LceAdamW)) for k in range(n_groups)]
            self.calls.append((np.frombuffer(bytes(rows), dtype=TR._TENSOR),
                               [{f: getattr(o, f) for f, _ in o._fields_} for o in opts], bits))

        self.calls, self.param = [], lambda *shape: torch.zeros(*shape).as_subclass(Param)
        monkeypatch.setattr(TR, "_native", lambda: here)
        monkeypatch.setattr(TR, "_dense", lambda grads, dev: ([g.contiguous() for g in grads], [TR._DTYPES[g.dtype] for g in grads]))
        monkeypatch.setattr(TR, "_stream", lambda dev: 0)
        monkeypatch.setattr(TR, "_on", lambda dev: TR._HERE)
        monkeypatch.setattr(TR.B, "lce_adamw_tensors_step",
                            lambda t, n, g, *a: call(t, n, ctypes.addressof(g) if isinstance(g, ctypes.Array) else g, *a))


@pytest.fixture
def on_gpu(monkeypatch):
    return OnGpu(monkeypatch)


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


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_follows_the_state_where_it_was_moved(on_gpu, bits):
    import torch
    from paper_2605_21442_amd import AdamWTensors
    ps = [on_gpu.param(40), on_gpu.param(3, 5)]
    ps[1] = ps[1].bfloat16()
    opt = AdamWTensors(ps, state_bits=bits, master_weights=True)
    names = ["exp_avg", "exp_avg_sq", "master"] if bits == 32 else ["exp_avg", "exp_avg_root", "units", "master"]
    gs = [torch.ones(40), torch.ones(3, 5)]

    def addresses_are_the_states():
        t = on_gpu.calls[-1][0]
        size = bits // 8
        for k, off in enumerate(opt.offsets):
            assert t["exp_avg"][k] == opt.exp_avg.data_ptr() + off * size
            assert t["exp_avg_sq"][k] == getattr(opt, names[1]).data_ptr() + off * size
            assert t["units"][k] == (opt.units.data_ptr() + off // 16 if bits == 8 else 0)
        assert t["master"].tolist() == [0, opt.master.data_ptr() + 4 * opt.offsets[1]]     # (of the bf16 tensor)

    opt.step(gs)
    addresses_are_the_states()
    for name in names:
        before = getattr(opt, name).data_ptr()
        setattr(opt, name, getattr(opt, name).clone())
        opt.step(gs)
        assert getattr(opt, name).data_ptr() != before
        addresses_are_the_states()
        getattr(opt, name).data = getattr(opt, name).clone()
        opt.step(gs)
        addresses_are_the_states()
    done = len(on_gpu.calls)
    for name in names:
        own = getattr(opt, name)
        freed = own.clone()
        freed.untyped_storage().resize_(0)
        for bad in (None, own[:-1], own.view(-1)[1:], own.to(torch.float64), own.to("meta"), freed, "no tensor"):
            setattr(opt, name, bad)
            with pytest.raises(ValueError, match=name):
                opt.step(gs)
            if bits == 8:
                with pytest.raises(ValueError, match=name):
                    opt.moments()
        setattr(opt, name, own)
    assert len(on_gpu.calls) == done
    opt.step(gs)
    addresses_are_the_states()


def test_only_the_tensors_of_the_call_count_as_changed(on_gpu):
    # a graph that saved a parameter without a gradient in this step can still be run backward
    import torch
    from paper_2605_21442_amd import AdamWTensors
    a, b = on_gpu.param(4), torch.nn.Parameter(on_gpu.param(4))
    opt = AdamWTensors([a, b])
    x = torch.ones(4, requires_grad=True)
    loss = (b * x).sum()
    versions = [a._version, b._version]
    opt.step([torch.ones(4), None])
    assert [a._version, b._version] == [versions[0] + 1, versions[1]]
    loss.backward()
    opt.step([None, None])
    assert [a._version, b._version] == [versions[0] + 1, versions[1]]
    loss = (b * x).sum()
    opt.step([torch.ones(4), torch.ones(4)])
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_bias_correction_goes_by_the_steps_that_a_tensor_took_part_in(on_gpu):
    import copy
    import torch
    from paper_2605_21442_amd import AdamWTensors
    make = lambda: AdamWTensors([dict(params=[on_gpu.param(4), on_gpu.param(5)]), dict(params=[on_gpu.param(6)], lr=0.5),
                                 dict(params=[on_gpu.param(3)], lr=0.25)])
    opt = make()
    gs = [torch.ones(4), torch.ones(5), torch.ones(6), torch.ones(3)]

    def taken(*have):
        """{tensor size: (rate, step)} of one step with these gradients."""
        opt.step([g if k in have else None for k, g in enumerate(gs)])
        t, opts, _ = on_gpu.calls[-1]
        return {int(r["n"]): (opts[r["group"]]["lr"], opts[r["group"]]["step"]) for r in t}

    a, b, c = (float(np.float32(x)) for x in (1e-3, 0.5, 0.25))
    assert taken(0, 1, 2, 3) == {4: (a, 1), 5: (a, 1), 6: (b, 1), 3: (c, 1)}
    assert taken(0, 2) == {4: (a, 2), 6: (b, 2)}
    assert taken(0) == {4: (a, 3)}
    assert taken() == {} and opt.step_count == 4
    assert taken(0, 1, 2, 3) == {4: (a, 4), 5: (a, 2), 6: (b, 3), 3: (c, 2)}
    assert opt.missed.tolist() == [1, 3, 2, 3]
    state = copy.deepcopy(opt.state_dict())
    assert taken(1, 3) == {5: (a, 3), 3: (c, 3)}
    opt = make()
    opt.load_state_dict(state)
    assert taken(1, 2) == {5: (a, 3), 6: (b, 4)}
    del state["missed"]                                # a checkpoint that does not say: every tensor took part
    opt = make()
    opt.load_state_dict(state)
    assert taken(0, 1, 2, 3) == {4: (a, 6), 5: (a, 6), 6: (b, 6), 3: (c, 6)}
    with pytest.raises(ValueError, match="number of tensors"):
        opt.load_state_dict(dict(state, missed=[0, 0]))
    before = opt.missed.copy(), opt.step_count
    with pytest.raises(ValueError):
        opt.step([gs[0], None, gs[1], None])           # refused: no count moves
    assert (opt.missed == before[0]).all() and opt.step_count == before[1]


def test_a_bare_tensor_is_not_taken_apart(on_gpu):
    # list() of a matrix gives views of its rows, which have no gradients of their own
    from paper_2605_21442_amd import AdamWTensors
    w, b = on_gpu.param(6, 4), on_gpu.param(3)
    with pytest.raises(TypeError, match="rows"):
        AdamWTensors(w)
    opt = AdamWTensors([dict(params=w, lr=0.5), dict(params=[b])])
    assert len(opt.params) == 2 and opt.params[0] is w and opt.params[1] is b and opt.groups[0]["lr"] == 0.5


def test_a_checkpoint_of_other_tensors_is_refused(on_gpu):
    # sizes of the same padded total, in another order or other groups: each tensor would get another one's moments
    import copy
    import torch
    from paper_2605_21442_amd import AdamWTensors
    make = lambda *shapes, cut=1, **kw: AdamWTensors([dict(params=[on_gpu.param(*s) for s in part]) for part in (shapes[:cut], shapes[cut:])],
                                                     **kw)
    for kw in (dict(), dict(state_bits=8), dict(master_weights=True)):
        a = make((3, 5), (40,), (2, 7), **kw)
        a.exp_avg.fill_(3)
        state = copy.deepcopy(a.state_dict())
        for other in (make((40,), (3, 5), (2, 7), **kw), make((2, 7), (40,), (3, 5), **kw), make((5, 3), (40,), (2, 7), **kw),
                      make((3, 5), (41,), (2, 7), **kw), make((3, 5), (40,), (2, 7), cut=2, **kw)):
            assert other.exp_avg.shape == a.exp_avg.shape
            with pytest.raises(ValueError, match="other"):
                other.load_state_dict(state)
            assert not other.exp_avg.any() and other.step_count == 0
        same = make((3, 5), (40,), (2, 7), **kw)
        same.load_state_dict(state)
        assert torch.equal(same.exp_avg, a.exp_avg)
        same = make((40,), (3, 5), (2, 7), **kw)
        same.load_state_dict({k: v for k, v in state.items() if k not in ("shapes", "group_of")})     # one that does not say


def test_a_checkpoint_without_its_step_changes_nothing(on_gpu):
    from paper_2605_21442_amd import AdamWTensors
    a, b = AdamWTensors([on_gpu.param(4)]), AdamWTensors([on_gpu.param(4)])
    a.exp_avg.fill_(1)
    state = a.state_dict()
    del state["step"]
    with pytest.raises(KeyError):
        b.load_state_dict(state)
    assert not b.exp_avg.any()


def test_a_gradient_without_memory_is_not_taken_for_zeros(on_gpu):
    import torch
    from paper_2605_21442_amd import AdamWTensors, training as TR

    class Wrapper(torch.Tensor):
        @staticmethod
        def __new__(cls, t):
            return torch.Tensor._make_wrapper_subclass(cls, t.shape, dtype=t.dtype, device="cuda:0")

        @classmethod
        def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
            raise AssertionError(func)

    freed, cut = torch.ones(3), torch.ones(8)
    freed.untyped_storage().resize_(0)
    for bad in (Wrapper(torch.ones(3)), freed):
        with pytest.raises(TypeError, match="memory"):
            AdamWTensors([on_gpu.param(4), on_gpu.param(3)]).step([torch.ones(4), bad])
        with pytest.raises(TypeError, match="memory"):
            TR.grad_norm([torch.ones(4), bad])
        assert not on_gpu.calls
    AdamWTensors([on_gpu.param(4), on_gpu.param(0), on_gpu.param(2)]).step([torch.ones(4), torch.ones(0), None])
    assert len(on_gpu.calls) == 1
    t = np.zeros(1, dtype=TABLE)
    fills = lambda x: TR._native().describe([x], None, -1, t, TABLE.itemsize, 8, 0, 20)
    assert fills(cut) and fills(cut[5:]) and fills(torch.zeros(0))
    assert freed.numel() == 3 and not fills(freed)
    tail = cut[5:]
    cut.untyped_storage().resize_(24)                  # six of its elements
    assert not fills(cut) and not fills(tail) and fills(cut[:6])
    with pytest.raises(TypeError, match="memory"):
        AdamWTensors([on_gpu.param(8)]).step([cut])


def test_the_losss_names_do_not_need_the_other_operators():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import sys, paper_2605_21442_amd as p\n"
            "sys.modules['paper_2605_21442_amd.training'] = None\n"          # importing it fails
            "assert p.linear_cross_entropy and p.AdamWState and p.LinearKD\n"
            "try: p.grad_norm\n"
            "except ImportError: pass\n"
            "else: raise AssertionError('imported')\n"
            "del sys.modules['paper_2605_21442_amd.training']\n"
            "assert all(getattr(p, n) for n in p.__all__)\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stderr


def test_an_extension_of_another_interpreter_or_torch_is_not_used(monkeypatch):
    # it reads torch's own structures: one built for others would read something else
    import sysconfig
    import torch
    from paper_2605_21442_amd import build, training as TR
    assert build.TENSORS_OUT.endswith("_tensors" + sysconfig.get_config_var("EXT_SUFFIX"))
    assert TR._native().__file__ == build.TENSORS_OUT
    monkeypatch.setattr(TR, "_ext", None)
    monkeypatch.setattr(torch, "__version__", "1.2.3+rocm")
    with pytest.raises(RuntimeError, match="built for torch"):
        TR._native()


def test_a_gradient_whose_sort_would_hold_the_gpu_is_refused():
    # (nothing is launched: the sizes are refused, or the workspace is missing)
    from paper_2605_21442_amd import binding as B
    at = 0x100000
    for n, v, ok in [((1 << 30) - 1, (1 << 30) - 1, False), (1 << 24, (1 << 29) + 1, False), (1 << 24, 1 << 29, True),
                     ((1 << 23) - 1, (1 << 30) - 1, True), ((1 << 30) - 1, 1 << 18, True), (1 << 20, (1 << 30) - 1, True)]:
        p = B.embedding(n, 8, v)
        for call in (lambda: B.lce_embedding_workspace_size(p), lambda: B.lce_embedding_backward(p, at, 2 * at, 3 * at, 0, 0, 0)):
            try:
                call()
                code = 0
            except B.LceError as e:
                code = e.code
            assert code == (B.LCE_ERR_SHAPE if not ok else code) and (not ok or code in (0, B.LCE_ERR_NULL)), (n, v, code)
