"""Token embedding and its gradient against the float64 oracle.

Tolerances count roundings: a stored value is off by at most half a step of its type (2^-8 of it for bf16, 2^-24 for
fp32); the scaled lookup has one fp32 rounding before that. A gradient of k tokens has k - 1 additions, one product
and at most one further addition in fp32, each off by 2^-24 of a partial result, none larger than the sum of magnitudes."""
import numpy as np
import pytest

from oracle import training_oracle as T

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _draw(shape, dtype, seed, std=1.0):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return (std * torch.randn(shape, device="cuda:0", generator=g)).to(_dt(dtype))


def _id_list(n, v, seed, kind):
    rng = np.random.default_rng(seed)
    if kind == "one":                     # every token the same id
        return np.full(n, v // 2, dtype=np.int64)
    if kind == "zipf":
        p = 1.0 / np.arange(1, v + 1)
        return rng.choice(v, size=n, p=p / p.sum())
    if kind == "each":                    # every id once, shuffled
        return rng.permutation(v)[:n] if n <= v else np.arange(n) % v
    return rng.integers(0, v, n)


def _np(x):
    return x.double().cpu().numpy()


def _check_grad(dw, ids, dout, v, dtype, scale=1.0, padding=None, v_begin=0, old=None):
    ref, k, mag = T.embedding_grad(ids, _np(dout), v, scale, padding, v_begin)
    got = _np(dw)
    touched = k > 0
    old64 = np.zeros_like(ref) if old is None else _np(old)
    tol = (k[:, None] + 3) * 2.0 ** -24 * 1.01 * (mag + np.abs(old64))
    ref = ref + old64
    tol = tol + (np.abs(ref) + tol) * HALF[dtype]
    bad = np.abs(got - ref) > tol
    assert not bad[touched].any(), np.argwhere(bad & touched[:, None])[:5]
    assert np.array_equal(got[~touched], old64[~touched])      # exactly: zeros, or left as they were


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("n,d,v,scale", [(1, 8, 1, 1.0), (1, 2048, 300, 0.5), (7, 72, 13, 1.0), (513, 264, 1000, 11.3125),
                                         (2049, 520, 4099, 1.0)])
def test_lookup(n, d, v, scale, bits, dtype):
    import torch
    from paper_2605_21442_amd.training import embedding_forward
    print(f"case lookup n={n} d={d} v={v} {dtype} int{bits}", flush=True)
    w = _draw((v, d), dtype, 1)
    ids = _id_list(n, v, 2, "zipf")
    out, status = embedding_forward(torch.from_numpy(ids).to("cuda:0", torch.int32 if bits == 32 else torch.int64), w, scale)
    ref = T.embedding(_np(w), ids, scale)
    assert int(status.item()) == 0 and out.shape == (n, d) and out.dtype == w.dtype
    if scale == 1.0:
        assert np.array_equal(_np(out), ref)
    else:
        assert np.all(np.abs(_np(out) - ref) <= np.abs(ref) * (HALF[dtype] + 2.0 ** -23))


def test_lookup_of_ids_outside_and_of_padding():
    import torch
    from paper_2605_21442_amd.training import embedding_forward
    v, d = 50, 16
    w = _draw((v, d), "bf16", 3)
    t = lambda *x: torch.tensor(x, device="cuda:0")
    big = 1 << 40
    for ids, pad, status in [((0, 49, 3), None, 0), ((0, 50), None, 2), ((-1, 2), None, 2), ((-100, 2), -100, 0), ((big, 2), None, 2),
                             ((big, 2), big, 0), ((7, 7), 7, 0), ((-(1 << 63), 1), None, 0)]:
        out, s = embedding_forward(t(*ids), w, 1.0, pad)
        # the id that stands for "no padding" is taken as padding: a row of zeros without a complaint
        assert int(s.item()) == status, ids
        assert np.array_equal(_np(out), T.embedding(_np(w), np.array(ids)))
    out, s = embedding_forward(torch.empty(0, dtype=torch.int64, device="cuda:0"), w)
    assert out.shape == (0, d) and int(s.item()) == 0


def test_shards_sum_to_the_whole():
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    n, d, v = 300, 40, 101
    w, x = _draw((v, d), "bf16", 4), _draw((n, d), "bf16", 5)
    ids = torch.from_numpy(_id_list(n, v, 6, "zipf")).to("cuda:0")
    ids[5] = v                     # in no shard
    whole, s = embedding_forward(ids, w)
    assert int(s.item()) == 2
    parts, cuts = torch.zeros_like(whole), [0, 1, 40, 101]
    dw = embedding_backward(ids, x, v, 2.0)
    for a, b in zip(cuts, cuts[1:]):
        out, s = embedding_forward(ids, w[a:b], v_begin=a, v_total=v)
        assert int(s.item()) == 2
        parts += out
        assert torch.equal(embedding_backward(ids, x, b - a, 2.0, v_begin=a, v_total=v), dw[a:b])
    assert torch.equal(parts, whole)


@pytest.mark.parametrize("kind", ["one", "zipf", "each", "flat"])
@pytest.mark.parametrize("n,d,v", [(1, 8, 1), (1, 8, 7), (63, 64, 5), (65, 520, 300), (1025, 72, 4099), (4097, 264, 777)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient(n, d, v, kind, dtype):
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    print(f"case grad n={n} d={d} v={v} {kind} {dtype}", flush=True)
    ids, x = _id_list(n, v, 7, kind), _draw((n, d), dtype, 8)
    t = torch.from_numpy(ids).to("cuda:0", torch.int32)
    dw = embedding_backward(t, x, v, 1.5, padding_idx=0)
    _check_grad(dw, ids, x, v, dtype, 1.5, 0)
    again = embedding_backward(t.long(), x, v, 1.5, padding_idx=0)
    assert torch.equal(again, dw)                      # the same bits, whatever the ids' type
    old = _draw((v, d), dtype, 9)
    acc = old.clone()
    assert embedding_backward(t, x, v, 1.5, accumulate_into=acc) is acc
    _check_grad(acc, ids, x, v, dtype, 1.5, None, old=old)
    if dtype == "bf16":
        wide = embedding_backward(t, x, v, 1.5, dw_dtype=torch.float32)
        _check_grad(wide, ids, x, v, "f32", 1.5)
        old = _draw((v, d), "f32", 10)
        acc = old.clone()
        embedding_backward(t, x, v, 1.5, accumulate_into=acc)
        _check_grad(acc, ids, x, v, "f32", 1.5, None, old=old)


@pytest.mark.parametrize("n,d,v", [(16384, 2048, 128256), (9001, 4096, 152064), (70001, 64, 131072), (300000, 8, 3)])
def test_gradient_of_long_batches(n, d, v):
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    print(f"case long grad n={n} d={d} v={v}", flush=True)
    ids = torch.from_numpy(_id_list(n, v, 11, "zipf")).to("cuda:0")
    x = _draw((n, d), "bf16", 12)
    dw = embedding_backward(ids, x, v)
    ref = torch.zeros(v, d, dtype=torch.float64, device="cuda:0").index_add_(0, ids, x.double())
    mag = torch.zeros(v, d, dtype=torch.float64, device="cuda:0").index_add_(0, ids, x.double().abs())
    k = torch.bincount(ids, minlength=v)[:, None]
    tol = (k + 3) * 2.0 ** -24 * 1.01 * mag
    assert bool((torch.abs(dw.double() - ref) <= tol + (ref.abs() + tol) * 2.0 ** -8).all())


@pytest.mark.parametrize("kind", ["one", "zipf"])
@pytest.mark.parametrize("n,d,v", [(1024, 2048, 3000), (1024, 2056, 3000), (1025, 512, 3000), (512, 4096, 700), (513, 4096, 700),
                                   (4, 1 << 16, 9), (900, 8, 1 << 19)])
def test_gradient_where_its_forms_meet(n, d, v, kind):
    # with and without the sort, one after the other of either size
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    print(f"case forms n={n} d={d} v={v} {kind}", flush=True)
    ids, x = _id_list(n, v, 62, kind), _draw((n, d), "bf16", 63)
    ids[::7] = v + 5
    t = torch.from_numpy(ids).to("cuda:0")
    dw = embedding_backward(t, x, v, 0.25, padding_idx=1)
    ref = torch.zeros(v + 6, d, dtype=torch.float64, device="cuda:0").index_add_(0, t, x.double() * 0.25)[:v]
    mag = torch.zeros(v + 6, d, dtype=torch.float64, device="cuda:0").index_add_(0, t, x.double().abs() * 0.25)[:v]
    k = torch.bincount(t, minlength=v)[:v, None]
    ref[1] = mag[1] = 0
    tol = (k + 3) * 2.0 ** -24 * 1.01 * mag
    assert bool((torch.abs(dw.double() - ref) <= tol + (ref.abs() + tol) * 2.0 ** -8).all())
    old = _draw((v, d), "f32", 64)
    acc = embedding_backward(t.int(), x, v, 0.25, padding_idx=1, accumulate_into=old.clone())
    tol = tol + (k + 3) * 2.0 ** -24 * old.double().abs()
    assert bool((torch.abs(acc.double() - ref - old.double()) <= tol + (ref + old.double()).abs() * 2.0 ** -24).all())
    untouched = (k[:, 0] == 0)
    untouched[1] = True
    assert torch.equal(acc[untouched], old[untouched]) and not dw[untouched].any()


def test_gradient_of_no_tokens():
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    none = torch.empty(0, dtype=torch.int64, device="cuda:0")
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda:0")
    assert not embedding_backward(none, x, 100).any()
    acc = _draw((100, 64), "bf16", 13)
    assert torch.equal(embedding_backward(none, x, 100, accumulate_into=acc.clone()), acc)
    # and of tokens that all fall outside, or are padding
    ids = torch.tensor([100, -5, 7, 1 << 40], device="cuda:0")
    x = _draw((4, 64), "bf16", 14)
    assert not embedding_backward(ids, x, 100, padding_idx=7).any()


def test_gradient_with_infinite_and_nan_rows():
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    ids = torch.tensor([3, 4, 3, 5, 6], device="cuda:0")
    x = torch.ones(5, 8, dtype=torch.bfloat16, device="cuda:0")
    x[0, 0], x[3, 1], x[4] = float("inf"), float("nan"), float("nan")
    dw = embedding_backward(ids, x, 10, padding_idx=6)
    assert dw[3, 0] == float("inf") and dw[3, 1] == 2 and dw[5, 1].isnan() and dw[5, 0] == 1 and (dw[4] == 1).all()
    assert (dw[6] == 0).all() and torch.isfinite(dw[7:]).all()     # padded rows are not read into anything


def test_strides_alignment_and_copies():
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    n, d, v = 70, 48, 33
    ids = torch.from_numpy(_id_list(n, v, 15, "flat")).to("cuda:0")
    w, x = _draw((v, d), "bf16", 16), _draw((n, d), "bf16", 17)
    ref, dref = embedding_forward(ids, w)[0], embedding_backward(ids, x, v)
    wide = torch.zeros(v, d + 16, dtype=torch.bfloat16, device="cuda:0")
    wide[:, 8:8 + d] = w                                            # row stride 64, start at 16 bytes
    assert torch.equal(embedding_forward(ids, wide[:, 8:8 + d])[0], ref)
    odd = torch.zeros(n * d + 3, dtype=torch.bfloat16, device="cuda:0")
    odd[3:] = x.reshape(-1)
    assert torch.equal(embedding_backward(ids, odd[3:].view(n, d), v), dref)        # misaligned: copied
    xw = torch.zeros(n, d + 8, dtype=torch.bfloat16, device="cuda:0")
    xw[:, :d] = x
    assert torch.equal(embedding_backward(ids, xw[:, :d], v), dref)                # row stride
    assert torch.equal(embedding_backward(ids, x.T.contiguous().T, v), dref)       # columns apart
    one = x[:1].expand(n, d)
    assert torch.equal(embedding_backward(ids, one, v), embedding_backward(ids, one.contiguous(), v))
    two = torch.stack((ids, ids + 1), 1)[:, 0]                                      # strided ids
    assert torch.equal(embedding_backward(two, x, v), dref)
    back = torch.zeros(n + 1, dtype=torch.int64, device="cuda:0")
    back[1:] = ids
    assert torch.equal(embedding_forward(back[1:], w)[0], ref)                      # ids aligned to 8 bytes only
    with pytest.raises(ValueError):
        embedding_backward(ids, x, v, accumulate_into=torch.zeros(v, d + 8, dtype=torch.bfloat16, device="cuda:0"))
    with pytest.raises(ValueError):
        embedding_backward(ids, x, v, accumulate_into=torch.zeros(d, v, dtype=torch.bfloat16, device="cuda:0").T)
    with pytest.raises(ValueError):
        embedding_backward(ids[:-1], x, v)
    with pytest.raises(TypeError):
        embedding_backward(ids, x, v, dw_dtype=torch.float16)
    with pytest.raises(ValueError):
        embedding_forward(ids.cpu(), w)


def test_autograd_gives_the_formula_and_the_differences():
    import torch
    from paper_2605_21442_amd import token_embedding
    v, d = 20, 16
    w = _draw((v, d), "f32", 18).requires_grad_()
    ids = torch.tensor([[1, 2, 2, 19], [0, 2, 5, 1]], device="cuda:0")
    up = _draw((2, 4, d), "f32", 19)
    out = token_embedding(ids, w, scale=3.0, padding_idx=5)
    assert out.shape == (2, 4, d)
    (out * up).sum().backward()
    ref = torch.zeros(v, d, dtype=torch.float64, device="cuda:0")
    ref.index_add_(0, ids.reshape(-1), 3.0 * up.reshape(-1, d).double())
    ref[5] = 0
    assert torch.allclose(w.grad.double(), ref, rtol=2.0 ** -22, atol=1e-6)
    # the loss is linear in w: a central difference in float64 of the sum over w + h e is exact up to rounding
    for r, c in [(2, 3), (19, 0), (0, 15)]:
        with torch.no_grad():
            f = []
            for h in (0.5, -0.5):
                w2 = w.detach().clone()
                w2[r, c] += h
                f.append(float((token_embedding(ids, w2, 3.0, 5).double() * up.double()).sum()))
        # w + h and the scaled row round once each: 2^-24 of |w| + 1/2, times 3 |up|, twice
        assert abs((f[0] - f[1]) - float(ref[r, c])) <= 4 * 2.0 ** -23 * 3 * float((w.detach().abs().max() + 1) * up.abs().sum())
    assert token_embedding(ids, w.detach()).grad_fn is None
    with torch.no_grad():
        assert token_embedding(ids, w).grad_fn is None
    (g,) = torch.autograd.grad(token_embedding(ids, w).square().sum(), w, create_graph=True)
    with pytest.raises(RuntimeError):                   # no second derivative, and none taken for zero
        g.sum().backward()


def test_tied_weights_join_the_heads_gradient():
    # one training step of a tied pair: lookup, loss, head gradient, embedding gradient added to it
    import torch
    from paper_2605_21442_amd import linear_cross_entropy, token_embedding
    from paper_2605_21442_amd.training import embedding_backward
    from paper_2605_21442_amd import autograd as AG
    n, d, v = 200, 64, 500
    w = _draw((v, d), "bf16", 20, 0.2)
    ids = torch.from_numpy(_id_list(n + 1, v, 21, "zipf")).to("cuda:0")
    h = token_embedding(ids[:-1], w, scale=8.0)
    loss, lse, nv, _, ws = AG.forward(h, w, ids[1:], keep_workspace=True)
    dh, dw = AG.backward(h, w, ids[1:], lse, nv, torch.ones(1, device="cuda:0"), workspace=ws)
    head = dw.clone()
    embedding_backward(ids[:-1], dh, v, 8.0, accumulate_into=dw)
    _check_grad(dw, ids[:-1].cpu().numpy(), dh, v, "bf16", 8.0, old=head)
    # autograd on the same leaf: both gradients, rounded to bf16 each and added once
    leaf = w.clone().requires_grad_()
    linear_cross_entropy(token_embedding(ids[:-1], leaf, scale=8.0), leaf, ids[1:]).backward()
    own = embedding_backward(ids[:-1], dh, v, 8.0)
    ref = head.double() + own.double()
    assert bool((torch.abs(leaf.grad.double() - ref) <= ref.abs() * 2.0 ** -8).all())


def test_other_streams_and_two_calls_at_once():
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    n, d, v = 5000, 256, 3000
    ids = [torch.from_numpy(_id_list(n, v, 30 + k, "zipf")).to("cuda:0") for k in range(2)]
    w, x = _draw((v, d), "bf16", 32), _draw((n, d), "bf16", 33)
    ref = [(embedding_forward(i, w)[0], embedding_backward(i, x, v)) for i in ids]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, i in zip(streams, ids):
            with torch.cuda.stream(s):
                got.append((embedding_forward(i, w)[0], embedding_backward(i, x, v)))
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_captured_lookup_and_gradient_replay_like_eager():
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    n, d, v = 3000, 128, 2000
    ids = torch.from_numpy(_id_list(n, v, 40, "zipf")).to("cuda:0")
    w, x = _draw((v, d), "bf16", 41), _draw((n, d), "bf16", 42)
    acc0 = _draw((v, d), "bf16", 43)
    acc = acc0.clone()
    embedding_backward(ids, x, v, accumulate_into=acc.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, status = embedding_forward(ids, w)
        dw = embedding_backward(ids, x, v)
        embedding_backward(ids, x, v, accumulate_into=acc)
    for rep in range(3):
        ids.copy_(torch.from_numpy(_id_list(n, v, 44 + rep, "zipf")).to("cuda:0"))
        x.copy_(_draw((n, d), "bf16", 50 + rep))
        acc.copy_(acc0)
        dw.fill_(float("nan"))
        out.fill_(float("nan"))
        _ = (x.float() @ x.float().T).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, embedding_forward(ids, w)[0]) and int(status.item()) == 0
        assert torch.equal(dw, embedding_backward(ids, x, v))
        assert torch.equal(acc, embedding_backward(ids, x, v, accumulate_into=acc0.clone()))


def test_rows_past_32_bit_byte_offsets():
    # W and dW of 2.2 * 2^31 bytes: rows whose byte offset needs more than 32 bits, first and last of them
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    v, d = 300000, 8192
    w = torch.zeros(v, d, dtype=torch.bfloat16, device="cuda:0")
    ids = torch.tensor([0, 131071, 131072, 262143, 262144, 299999, 299999], device="cuda:0")
    w[ids[:-1]] = _draw((6, d), "bf16", 60)
    out, _ = embedding_forward(ids, w)
    assert torch.equal(out, w[ids])
    x = _draw((7, d), "bf16", 61)
    dw = embedding_backward(ids, x, v, accumulate_into=w)
    ref = out.double()
    ref[5] = ref[6] = out[5].double() + x[6].double()
    got = dw[ids].double()
    ref = ref + x.double()
    ref[6] = ref[5]
    assert bool((torch.abs(got - ref) <= 1e-6 + ref.abs() * (2.0 ** -8 + 2.0 ** -20)).all())


def test_outputs_and_gradients_past_32_bit_offsets():
    # out and dOut of 2^32 + elements; whole numbers whose sums fp32 holds exactly
    import torch
    from paper_2605_21442_amd.training import embedding_backward, embedding_forward
    n, d, v = 530000, 8192, 1000
    print(f"case n={n} d={d} v={v}", flush=True)
    w = torch.arange(v, device="cuda:0").remainder(127).to(torch.bfloat16)[:, None].expand(v, d).contiguous()
    ids = torch.arange(n, device="cuda:0").remainder(v)
    out, _ = embedding_forward(ids, w)
    for a in (0, 262143, 524287, 524288, n - 1):
        assert torch.equal(out[a], w[a % v])
    assert torch.equal(out[:, 0], w[ids, 0]) and torch.equal(out[:, d - 1], w[ids, 0])
    x = out
    x.copy_(torch.arange(n, device="cuda:0").remainder(7).to(torch.bfloat16)[:, None].expand(n, d))
    dw = embedding_backward(ids, x, v, dw_dtype=torch.float32)
    ref = torch.zeros(v, dtype=torch.float64, device="cuda:0").index_add_(0, ids, torch.arange(n, device="cuda:0").remainder(7).double())
    assert bool((dw.double() == ref[:, None]).all())


def test_adding_to_a_gradient_is_noticed_by_autograd():
    import torch
    from paper_2605_21442_amd.training import embedding_backward
    a = torch.zeros(4, 8, device="cuda:0")
    version = a._version
    embedding_backward(torch.tensor([1, 2], device="cuda:0"), torch.ones(2, 8, device="cuda:0"), 4, accumulate_into=a)
    assert a._version > version
