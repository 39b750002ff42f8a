"""Token embedding, AdamW over many tensors and gradient norm without a GPU: sizes and refusals of the C
entry points (nothing is launched on the made-up addresses), and the oracle's own pins."""
import ctypes
import os

import numpy as np
import pytest

from oracle import training_oracle as T
from paper_2605_21442_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="liblce.so not built")

A, C, D, E, F, G, H = (0x100000 * k for k in range(1, 8))


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), B.LCE_ERR_SHAPE), (dict(n=1 << 30), B.LCE_ERR_SHAPE), (dict(d=0), B.LCE_ERR_SHAPE),
    (dict(d=1 << 20), B.LCE_ERR_SHAPE), (dict(v=0), B.LCE_ERR_SHAPE), (dict(v=1 << 30), B.LCE_ERR_SHAPE),
    (dict(d=60), B.LCE_ERR_UNSUPPORTED), (dict(id_bytes=2), B.LCE_ERR_UNSUPPORTED), (dict(dtype=2), B.LCE_ERR_UNSUPPORTED),
    (dict(dtype=B.LCE_DTYPE_F32, dw_dtype=B.LCE_DTYPE_BF16), B.LCE_ERR_UNSUPPORTED), (dict(ld_w=32), B.LCE_ERR_SHAPE),
    (dict(ld_x=32), B.LCE_ERR_SHAPE), (dict(ld_w=68), B.LCE_ERR_ALIGN), (dict(ld_x=68), B.LCE_ERR_ALIGN),
    (dict(scale=float("nan")), B.LCE_ERR_ARG), (dict(scale=float("inf")), B.LCE_ERR_ARG),
    (dict(flags=B.LCE_FLAG_REUSE_FORWARD), B.LCE_ERR_ARG), (dict(flags=8), B.LCE_ERR_ARG),
    (dict(v_total=99), B.LCE_ERR_SHAPE), (dict(v_total=200, v_begin=101), B.LCE_ERR_SHAPE), (dict(v_begin=1), B.LCE_ERR_SHAPE),
    (dict(v=1 << 29, d=512), B.LCE_ERR_SHAPE), (dict(v=1 << 18, d=1 << 18, dw_dtype=B.LCE_DTYPE_F32), B.LCE_ERR_SHAPE),
    (dict(v_total=200, v_begin=-1), B.LCE_ERR_SHAPE), (dict(v_begin=(1 << 63) - 1), B.LCE_ERR_SHAPE),
])
def test_bad_embeddings_are_rejected(kw, code):
    with pytest.raises(B.LceError) as e:
        B.lce_embedding_workspace_size(B.embedding(**{**dict(n=8, d=64, v=100), **kw}))
    assert e.value.code == code


def test_embedding_reserved_field_must_be_zero():
    p = B.embedding(8, 64, 100)
    p.reserved = 1
    with pytest.raises(B.LceError) as e:
        B.lce_embedding_workspace_size(p)
    assert e.value.code == B.LCE_ERR_ARG


def test_embedding_argument_checks_run_before_any_launch():
    p = B.embedding(8, 64, 100, v_total=200, v_begin=100)
    ws = B.lce_embedding_workspace_size(p)
    fwd = dict(W=A, ids=C, out=D, dev_status=0, stream=0)
    for change, code in [(dict(W=0), B.LCE_ERR_NULL), (dict(ids=0), B.LCE_ERR_NULL), (dict(out=0), B.LCE_ERR_NULL),
                         (dict(W=A + 8), B.LCE_ERR_ALIGN), (dict(ids=C + 4), B.LCE_ERR_ALIGN), (dict(out=D + 2), B.LCE_ERR_ALIGN)]:
        with pytest.raises(B.LceError) as e:
            B.lce_embedding_forward(p, **{**fwd, **change})
        assert e.value.code == code, change
    bwd = dict(ids=A, dOut=C, dW=D, workspace=E, workspace_bytes=ws, stream=0)
    for change, code in [(dict(ids=0), B.LCE_ERR_NULL), (dict(dOut=0), B.LCE_ERR_NULL), (dict(dW=0), B.LCE_ERR_NULL),
                         (dict(workspace=0), B.LCE_ERR_NULL), (dict(ids=A + 4), B.LCE_ERR_ALIGN), (dict(dOut=C + 4), B.LCE_ERR_ALIGN),
                         (dict(dW=D + 8), B.LCE_ERR_ALIGN), (dict(workspace=E + 16), B.LCE_ERR_ALIGN),
                         (dict(workspace_bytes=ws - 1), B.LCE_ERR_WORKSPACE)]:
        with pytest.raises(B.LceError) as e:
            B.lce_embedding_backward(p, **{**bwd, **change})
        assert e.value.code == code, change


def test_embedding_workspace_is_linear_in_tokens_and_ids():
    # 8 bytes per token, 4 per id (rounded up to whole buckets) and fp32 sums of at most 8192 rows
    for n, d, v in [(0, 8, 1), (1, 8, 5), (16384, 4096, 128256), (32768, 3584, 152064), (1 << 20, 8192, 1 << 18), (5000, 64, 1 << 21)]:
        size = B.lce_embedding_workspace_size(B.embedding(n, d, v))
        assert 8 * n + 4 * v <= size <= 8 * n + 8 * v + 4096 + 4 * d * min(8192, 2 * n + 2), (n, d, v)


def _tensor(**kw):
    f = dict(param=A, grad=C, exp_avg=D, exp_avg_sq=E, units=None, master=None, n=100, place=0, group=0,
             param_dtype=0, grad_dtype=0, reserved=0)
    return B.LceAdamWTensor(**{**f, **kw})


OPT = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1)


def _adamw(tensors, groups=(OPT,), bits=32, scale=0, count=None):
    t = (B.LceAdamWTensor * max(1, len(tensors)))(*tensors)
    g = (B.LceAdamW * max(1, len(groups)))(*(B.adamw(**o) for o in groups))
    B.lce_adamw_tensors_step(ctypes.addressof(t), len(tensors) if count is None else count, ctypes.addressof(g), len(groups),
                             bits, scale, 0, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), B.LCE_ERR_SHAPE), (dict(n=1 << 35), B.LCE_ERR_SHAPE), (dict(param=0), B.LCE_ERR_NULL),
    (dict(exp_avg=0), B.LCE_ERR_NULL), (dict(exp_avg_sq=0), B.LCE_ERR_NULL), (dict(param=A + 1), B.LCE_ERR_ALIGN),
    (dict(param=A + 2, param_dtype=1), B.LCE_ERR_ALIGN), (dict(grad=C + 1), B.LCE_ERR_ALIGN),
    (dict(grad=C + 2, grad_dtype=1), B.LCE_ERR_ALIGN), (dict(exp_avg=D + 8), B.LCE_ERR_ALIGN),
    (dict(exp_avg_sq=E + 4), B.LCE_ERR_ALIGN), (dict(master=F + 2), B.LCE_ERR_ALIGN), (dict(param_dtype=2), B.LCE_ERR_UNSUPPORTED),
    (dict(grad_dtype=-1), B.LCE_ERR_UNSUPPORTED), (dict(group=1), B.LCE_ERR_ARG), (dict(group=-1), B.LCE_ERR_ARG),
    (dict(place=16), B.LCE_ERR_ARG), (dict(place=-32), B.LCE_ERR_ARG), (dict(reserved=1), B.LCE_ERR_ARG),
    (dict(master=F, param_dtype=1), B.LCE_ERR_ARG), (dict(units=F), B.LCE_ERR_ARG),
])
def test_bad_tensors_are_rejected_before_any_launch(kw, code):
    # behind a good one: nothing may have been launched when the bad one is found
    with pytest.raises(B.LceError) as e:
        _adamw([_tensor(), _tensor(**kw)])
    assert e.value.code == code


def test_adamw_tensors_argument_checks():
    for bits, code in [(16, B.LCE_ERR_UNSUPPORTED), (0, B.LCE_ERR_UNSUPPORTED), (8, B.LCE_ERR_NULL)]:   # 8: no units
        with pytest.raises(B.LceError) as e:
            _adamw([_tensor()], bits=bits)
        assert e.value.code == code, bits
    with pytest.raises(B.LceError) as e:
        _adamw([_tensor(units=F + 1)], bits=8)
    assert e.value.code == B.LCE_ERR_ALIGN
    for kw, code in [(dict(groups=()), B.LCE_ERR_ARG), (dict(count=-1), B.LCE_ERR_SHAPE), (dict(scale=A + 2), B.LCE_ERR_ALIGN),
                     (dict(groups=(OPT, dict(OPT, step=0))), B.LCE_ERR_ARG), (dict(groups=(dict(OPT, beta2=1.0),)), B.LCE_ERR_ARG)]:
        with pytest.raises(B.LceError) as e:
            _adamw([_tensor()], **kw)
        assert e.value.code == code, kw
    for args in [(0, 1, A, 1), (A, 1, 0, 1)]:
        with pytest.raises(B.LceError) as e:
            B.lce_adamw_tensors_step(*args, 32, 0, 0, 0)
        assert e.value.code == B.LCE_ERR_NULL
    _adamw([])                                     # nothing to do, nothing launched
    _adamw([_tensor(n=0, param=0, exp_avg=0)])


def test_moments_argument_checks():
    ok = dict(n=100, exp_avg=A, exp_avg_sq=C, units=D, first=E, root=F, stream=0)
    for change, code in [(dict(n=-1), B.LCE_ERR_SHAPE), (dict(units=0), B.LCE_ERR_NULL), (dict(first=0), B.LCE_ERR_NULL),
                         (dict(exp_avg=A + 8), B.LCE_ERR_ALIGN), (dict(root=F + 2), B.LCE_ERR_ALIGN)]:
        with pytest.raises(B.LceError) as e:
            B.lce_adamw_moments(**{**ok, **change})
        assert e.value.code == code, change
    B.lce_adamw_moments(**{**ok, "n": 0})


def _norm(grads, max_norm=1.0, norm=A, factor=C, workspace=D, nbytes=None):
    t = (B.LceGrad * max(1, len(grads)))(*(B.LceGrad(*g) for g in grads))
    size = B.lce_grad_norm_workspace_size(ctypes.addressof(t), len(grads))
    B.lce_grad_norm(ctypes.addressof(t), len(grads), max_norm, norm, factor, workspace, size if nbytes is None else nbytes, 0)


def test_grad_norm_argument_checks():
    for grads, code in [([(A, -1, 0, 0)], B.LCE_ERR_SHAPE), ([(A, 1 << 35, 0, 0)], B.LCE_ERR_SHAPE), ([(0, 4, 0, 0)], B.LCE_ERR_NULL),
                        ([(A + 1, 4, 0, 0)], B.LCE_ERR_ALIGN), ([(A + 2, 4, 1, 0)], B.LCE_ERR_ALIGN),
                        ([(A, 4, 3, 0)], B.LCE_ERR_UNSUPPORTED), ([(A, 4, 0, 1)], B.LCE_ERR_ARG)]:
        with pytest.raises(B.LceError) as e:
            _norm(grads)
        assert e.value.code == code, grads
    for kw, code in [(dict(max_norm=0.0), B.LCE_ERR_ARG), (dict(max_norm=float("nan")), B.LCE_ERR_ARG), (dict(norm=0), B.LCE_ERR_NULL),
                     (dict(workspace=0), B.LCE_ERR_NULL), (dict(workspace=D + 8), B.LCE_ERR_ALIGN), (dict(norm=A + 2), B.LCE_ERR_ALIGN),
                     (dict(nbytes=0), B.LCE_ERR_WORKSPACE)]:
        with pytest.raises(B.LceError) as e:
            _norm([(A, 100, 0, 0)], **kw)
        assert e.value.code == code, kw


def test_front_end_refuses_what_it_cannot_run():
    import torch
    from paper_2605_21442_amd import AdamWTensors, grad_norm, token_embedding
    from paper_2605_21442_amd import training as TR
    cpu = torch.zeros(4, 8, dtype=torch.bfloat16)
    ids = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        token_embedding(ids, cpu)                       # not on a GPU
    with pytest.raises(TypeError):
        token_embedding(ids, cpu.half())
    with pytest.raises(ValueError):
        token_embedding(ids, cpu[0])
    with pytest.raises(ValueError):
        TR.embedding_backward(ids, cpu, 4)
    with pytest.raises(ValueError):
        grad_norm([cpu])
    with pytest.raises(TypeError):
        grad_norm([cpu.double()])
    with pytest.raises(ValueError):
        grad_norm([None])
    for bad in [dict(params=[cpu]), dict(params=[]), dict(params=[cpu], state_bits=4),
                dict(params=[{"params": [cpu], "momentum": 1}])]:
        with pytest.raises(ValueError):
            AdamWTensors(**bad)
    with pytest.raises(TypeError):
        AdamWTensors([cpu.half()])


# ---- the oracle -----------------------------------------------------------------------------------

def test_codes_of_the_8_bit_moments():
    # every code stands for a value of its own, in order, and holds itself exactly; the largest block value is held
    # within a code of the topmost binades
    for k, top in [(3, 127), (4, 255)]:
        c = np.arange(top + 1)
        x = T.value(c, np.full(top + 1, 127), k)
        assert np.all(np.diff(x) > 0) and x[1] == 1.0
        at, _ = T.place_between(x, np.full(top + 1, 127), k)
        assert np.array_equal(at, c)
        rng = np.random.default_rng(1)
        a = np.concatenate([rng.uniform(1, 2, 1000), [1, 2 - 2.0 ** -k, np.nextafter(2 - 2.0 ** -k, 0)]]) * 2.0 ** 5
        for v in a:
            s = T.units(np.array([v]), k)
            at, _ = T.place_between(np.array([v]), s, k)
            # below the last code, so that rounding up stays within the codes (the sum of whole codes and the
            # part has 53 bits: a part 2^-51 below 1 shows as 1)
            assert (14 << k) <= at[0] <= top


def test_rounding_hash_is_even():
    # 16-bit uniforms over neighbouring elements, steps and both halves of a pair: means and correlations within
    # five standard deviations of independent draws
    n = 4096
    draws = np.stack([T.pair_uniform(0, n, s) for s in (0, 1, 2, 3, 0x9E3779B9, 12345)])
    sd = 1 / np.sqrt(12 * n)
    assert np.all(np.abs(draws.mean(1) - 0.5 * (1 - 2.0 ** -16)) < 5 * sd)
    for x, y in [(draws[0], draws[1]), (draws[0], draws[4]), (draws[2], draws[3]), (draws[0][:-1], draws[0][1:]),
                 (draws[1][:-2], draws[1][2:]), (draws[5][0::2], draws[5][1::2])]:
        assert abs(np.corrcoef(x, y)[0, 1]) < 5 / np.sqrt(x.size)
    hist = np.histogram(draws, 64, (0, 1))[0]
    assert np.all(np.abs(hist - draws.size / 64) < 5 * np.sqrt(draws.size / 64))


# ---- the extension that reads lists of tensors, on host tensors (device -1) -------------------------

def _native():
    from paper_2605_21442_amd.training import _native
    return _native()


TABLE = np.dtype([("n", "i8"), ("data", "u8"), ("pad", "i4"), ("dtype", "i4")])


def test_describe_fills_a_table():
    import torch
    x = torch.zeros(100, dtype=torch.bfloat16)
    ts = [x, x[3:7], torch.zeros(2, 3), torch.nn.Parameter(torch.zeros(5)), torch.zeros(0)]
    t = np.full(len(ts), 0, dtype=TABLE)
    t["pad"] = 77
    assert _native().describe(ts, None, -1, t, TABLE.itemsize, 8, 0, 20)
    assert t["data"].tolist() == [a.data_ptr() for a in ts] and t["n"].tolist() == [100, 4, 6, 5, 0]
    assert t["dtype"].tolist() == [0, 0, 1, 1, 1] and (t["pad"] == 77).all()
    t["n"] = -5
    assert _native().describe(ts, [a.shape for a in ts], -1, t, TABLE.itemsize, 8, -1, 20)
    assert (t["n"] == -5).all()                        # not asked for
    assert _native().stand_at(ts, t, TABLE.itemsize, 8) and not _native().stand_at(ts[1:], t, TABLE.itemsize, 8)
    assert _native().describe([], None, -1, t, TABLE.itemsize, 8, 0, 20)


def test_describe_leaves_to_the_caller_what_is_not_plain_memory():
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        fake = torch.empty(4)
    good = torch.zeros(4, 4)
    t = np.zeros(2, dtype=TABLE)
    bad = [None, 3, good.T, good[:, 1:], good.half(), good.to(torch.int32), good.to_sparse(), good.to("meta"), fake]
    for x in bad:
        assert not _native().describe([good, x], None, -1, t, TABLE.itemsize, 8, 0, 20), type(x)
    assert not _native().describe([good], None, 0, t, TABLE.itemsize, 8, 0, 20)          # not on that device
    for shape in [(16,), (4, 4, 1), (4, 5), (4, "x"), (4, None), [4, 4], None, ()]:
        assert not _native().describe([good], [shape], -1, t, TABLE.itemsize, 8, 0, 20), shape


def test_describe_refuses_a_table_that_does_not_fit():
    import torch
    g = torch.zeros(4)
    t = np.zeros(2, dtype=TABLE)
    d = _native().describe
    for args in [([g] * 3, None, -1, t, TABLE.itemsize, 8, 0, 20), ([g], None, -1, t, TABLE.itemsize, 20, 0, 20),
                 ([g], None, -1, t, TABLE.itemsize, -1, 0, 20), ([g], None, -1, t, TABLE.itemsize, 8, 0, 21),
                 ([g], None, -1, t, TABLE.itemsize, 8, 20, 20), ([g], None, -1, t, 0, 8, 0, 20), ([g], [g, g], -1, t, TABLE.itemsize, 8, 0, 20)]:
        with pytest.raises(ValueError):
            d(*args)
    with pytest.raises(TypeError):
        d((g,), None, -1, t, TABLE.itemsize, 8, 0, 20)
    frozen = np.zeros(2, dtype=TABLE)
    frozen.flags.writeable = False
    with pytest.raises(TypeError):                     # the interpreter asks for a writable buffer
        d([g], None, -1, frozen, TABLE.itemsize, 8, 0, 20)
    with pytest.raises(TypeError):
        _native().changed((g,))


def test_changed_counts_as_an_in_place_change():
    import torch
    p = torch.zeros(3, requires_grad=True)
    with torch.inference_mode():
        q = torch.zeros(3)
    before = p._version
    _native().changed([p, q, None])
    assert p._version == before + 1


def test_missing_extension_fails_loudly(monkeypatch):
    import sys
    from paper_2605_21442_amd import training
    monkeypatch.setattr(training, "_ext", None)
    monkeypatch.setitem(sys.modules, "paper_2605_21442_amd._tensors", None)
    monkeypatch.delattr("paper_2605_21442_amd._tensors", raising=False)
    with pytest.raises(RuntimeError, match="not built"):
        training._native()
