"""torch front end of the library's other training operators: tensors in, tensors out, work in liblce.so.

* ``token_embedding(ids, weight)``: the input end of the vocabulary matrix whose output end is
  ``linear_cross_entropy``'s; its gradient adds each id's tokens in a fixed order, into a fresh
  [V, D] tensor or into the head's gradient (tied weights).
* ``grad_norm(grads, max_norm)``: the norm of all gradients and the factor that clips them, on the device.
* ``AdamWTensors(params)``: an AdamW step over all tensors of a model, moments in 32 or 8 bits,
  with the arithmetic of ``AdamWState``.
"""
from __future__ import annotations

import contextlib
import math

import numpy as np
import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import binding as B
from .autograd import _rows_usable

_DTYPES = {torch.bfloat16: B.LCE_DTYPE_BF16, torch.float32: B.LCE_DTYPE_F32}


_ext = None


def _native():
    """The extension that reads lists of tensors (csrc/tensors.cpp); like liblce.so it is needed, not replaced."""
    global _ext
    if _ext is None:
        how = "; run `python -c 'import __graft_entry__ as g; g.build()'` from the repository root"
        try:
            from . import _tensors
        except ImportError as e:
            raise RuntimeError("the extension _tensors is not built for this Python and torch" + how) from e
        if not torch.__version__.startswith(_tensors.torch_version):
            raise RuntimeError(f"the extension _tensors was built for torch {_tensors.torch_version}, not {torch.__version__}" + how)
        _ext = _tensors
    return _ext


def _stream(dev: torch.device) -> int:
    return _native().current_stream(dev.index)


_HERE = contextlib.nullcontext()


def _on(dev: torch.device):
    """The tensors' device as the current one while a call is enqueued: its default stream has no device of its own."""
    return _HERE if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


# ---- token embedding ----------------------------------------------------------------------------

def _rows(x: torch.Tensor, name: str) -> tuple[torch.Tensor, int]:
    if x.dtype not in _DTYPES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {x.dtype}")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if _native().negative(x):        # its memory holds the values with the other sign, also after contiguous()
        x = x.resolve_neg()
    x2 = x.reshape(-1, x.shape[-1]) if x.dim() != 2 else x
    if not _rows_usable(tuple(x2.shape), x2.stride(), x2.data_ptr()):
        x2 = x2.contiguous()
        if x2.data_ptr() % 16:       # already dense, but its start is not aligned
            x2 = x2.clone()
    return x2, (x2.stride(0) if x2.shape[0] > 1 else x2.shape[1])


def _ids(ids: torch.Tensor, dev: torch.device) -> torch.Tensor:
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"ids must be int32 or int64, got {ids.dtype}")
    if ids.device != dev:
        raise ValueError(f"ids are on {ids.device}, the other operand on {dev}")
    return ids if ids.dim() == 1 and ids.is_contiguous() else ids.reshape(-1).contiguous()


def embedding_forward(ids: torch.Tensor, weight: torch.Tensor, scale: float = 1.0, padding_idx: int | None = None,
                      v_begin: int = 0, v_total: int = 0, want_status: bool = True):
    """(out, status int32 [1] or None) from lce_embedding_forward: ``scale * weight[ids]``, shaped like ids with the
    hidden size behind; rows of ids that the weight does not hold are 0. ``v_begin`` and ``v_total`` say
    which ids a vocabulary shard holds, as for ``forward_shard``."""
    if weight.dim() != 2:
        raise ValueError(f"weight must be [V, D], got {tuple(weight.shape)}")
    w, ldw = _rows(weight, "weight")
    t = _ids(ids, w.device)
    v, d = w.shape
    dev, kind = w.device, _DTYPES[w.dtype]
    # (B.embedding's structure, in place: a call of few tokens takes as long as the host does)
    p = B.LceEmbedding(t.numel(), d, v, ldw, 0, v_begin, v_total, B.LCE_NO_PADDING if padding_idx is None else padding_idx,
                       scale, t.element_size(), kind, kind, 0, 0)
    out = torch.empty((*ids.shape, d), dtype=w.dtype, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev) if want_status else None
    with _on(dev):
        B.lce_embedding_forward(p, w.data_ptr(), t.data_ptr(), out.data_ptr(), status.data_ptr() if want_status else 0,
                                _stream(dev))
    return out, status


def embedding_backward(ids: torch.Tensor, grad_out: torch.Tensor, v: int, scale: float = 1.0,
                       padding_idx: int | None = None, v_begin: int = 0, v_total: int = 0,
                       accumulate_into: torch.Tensor | None = None, dw_dtype: torch.dtype | None = None):
    """dW [v, D] from lce_embedding_backward: per id the scaled sum of its tokens' rows of ``grad_out``. With
    ``accumulate_into`` (a dense [v, D] tensor of grad_out's dtype or float32, such as the head's dW) the sums
    are added to it in place and it is returned; otherwise dW is new, of grad_out's dtype or ``dw_dtype``."""
    x, ldx = _rows(grad_out, "grad_out")
    t = _ids(ids, x.device)
    n, d = x.shape
    if t.numel() != n:
        raise ValueError(f"ids has {t.numel()} entries for {n} rows of grad_out")
    if accumulate_into is not None:
        dw = accumulate_into
        if (tuple(dw.shape) != (v, d) or not dw.is_contiguous() or dw.is_neg() or dw.device != x.device
                or dw.dtype not in (x.dtype, torch.float32)):
            raise ValueError(f"accumulate_into must be a contiguous [{v}, {d}] tensor of grad_out's dtype or float32 on its device")
    else:
        dw_dtype = x.dtype if dw_dtype is None else dw_dtype
        if dw_dtype not in (x.dtype, torch.float32):
            raise TypeError(f"dw_dtype must be {x.dtype} or float32, got {dw_dtype}")
        dw = torch.empty((v, d), dtype=dw_dtype, device=x.device)
    dev = x.device
    p = B.LceEmbedding(n, d, v, 0, ldx, v_begin, v_total, B.LCE_NO_PADDING if padding_idx is None else padding_idx, scale,
                       t.element_size(), _DTYPES[x.dtype], _DTYPES[dw.dtype],
                       B.LCE_FLAG_ACCUMULATE_DW if accumulate_into is not None else 0, 0)
    nbytes = B.lce_embedding_workspace_size(p)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    with _on(dev):
        B.lce_embedding_backward(p, t.data_ptr(), x.data_ptr(), dw.data_ptr(), ws.data_ptr(), nbytes, _stream(dev))
    if accumulate_into is not None and not dw.is_inference():
        increment_version(dw)
    return dw


class TokenEmbedding(torch.autograd.Function):
    """Scaled lookup of rows by id; the backward returns the weight's gradient, dense. (To capture a training step into a
    graph beside eager ones of the same weights, capture ``embedding_forward`` and ``embedding_backward``: torch's own
    accumulation of a leaf's gradient may not move between a live eager graph and a capture.)"""

    @staticmethod
    def forward(ctx, ids, weight, scale=1.0, padding_idx=None):
        out, _ = embedding_forward(ids, weight, scale, padding_idx, want_status=False)
        ctx.save_for_backward(ids)
        ctx.opts = (weight.shape[0], scale, padding_idx)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        (ids,) = ctx.saved_tensors
        v, scale, padding_idx = ctx.opts
        dw = embedding_backward(ids, grad, v, scale, padding_idx) if ctx.needs_input_grad[1] else None
        return None, dw, None, None


def token_embedding(ids: torch.Tensor, weight: torch.Tensor, scale: float = 1.0,
                    padding_idx: int | None = None) -> torch.Tensor:
    """``scale * weight[ids]``: the token embedding, with a gradient for the weight [V, D] (bf16 or fp32). Tokens
    of ``padding_idx`` give no gradient; one that is no id of the vocabulary, such as -1 or -100, stands for tokens whose
    rows are zeros (it does not count from the end). An id outside the vocabulary gives a row of zeros and no gradient
    (``embedding_forward`` also reports it). Forward-mode derivatives are refused."""
    if not (weight.requires_grad and torch.is_grad_enabled()) and not _native().dual(weight):
        return embedding_forward(ids, weight, scale, padding_idx, want_status=False)[0]
    return TokenEmbedding.apply(ids, weight, scale, padding_idx)


# ---- gradient norm ------------------------------------------------------------------------------

_GRAD = np.dtype([("data", "u8"), ("n", "i8"), ("dtype", "i4"), ("reserved", "i4")])


def _dense(grads: list, dev_index: int | None) -> tuple[list, list]:
    """(the given tensors, contiguous; their lce_dtype_t), for lists that the extension does not take as they are: what is
    not contiguous is copied, other types and several devices are refused."""
    kinds = {g.dtype for g in grads}
    if not kinds <= _DTYPES.keys():
        raise TypeError(f"gradients must be bfloat16 or float32, got {kinds - _DTYPES.keys()}")
    where = {g.get_device() for g in grads}
    if -1 in where or len(where) > 1 or (dev_index is not None and where and where != {dev_index}):
        raise ValueError("gradients must be GPU tensors on one device")
    return [g.resolve_neg().contiguous() for g in grads], [_DTYPES[g.dtype] for g in grads]


def _list_dense(grads: list, dtypes: list, t: np.ndarray, data: str, dtype: str) -> None:
    """The tensors of ``_dense`` into a table that holds their sizes. The library takes a gradient without an address for
    zeros: one without memory of its own is refused."""
    t[data] = [g.data_ptr() for g in grads]
    t[dtype] = dtypes
    if ((t[data] == 0) & (t["n"] > 0)).any() or not _native().stand_at(grads, t, t.dtype.itemsize,
                                                                       *(t.dtype.fields[k][1] for k in (data, "n", dtype))):
        raise TypeError("gradients must have memory of their own (a wrapper, or a tensor whose storage was resized, has not)")


def grad_norm(grads, max_norm: float = math.inf) -> tuple[torch.Tensor, torch.Tensor]:
    """(norm, factor), fp32 scalars on the device, from lce_grad_norm: the norm of all tensors of ``grads``
    together (None entries are left out) and ``min(1, max_norm / (norm + 1e-6))``, for ``AdamWTensors.step``'s
    ``grad_scale``. The factor is NaN where the norm is not finite. Nothing waits for the device."""
    grads = list(grads)
    t = np.zeros(len(grads), dtype=_GRAD)
    first = grads[0].get_device() if grads and grads[0] is not None else -1
    if first < 0 or not _native().describe(grads, None, first, t, _GRAD.itemsize, 0, 8, 16):
        grads, dtypes = _dense([g for g in grads if g is not None], None)
        if not grads:
            raise ValueError("no gradients")
        t = np.zeros(len(grads), dtype=_GRAD)
        t["n"] = [g.numel() for g in grads]
        _list_dense(grads, dtypes, t, "data", "dtype")
    dev = grads[0].device
    addr = t.ctypes.data
    nbytes = B.lce_grad_norm_workspace_size(addr, len(grads))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    out = torch.empty(2, dtype=torch.float32, device=dev)
    with _on(dev):
        B.lce_grad_norm(addr, len(grads), max_norm, out.data_ptr(), out.data_ptr() + 4, ws.data_ptr(), nbytes, _stream(dev))
    norm, factor = out.unbind()
    return norm, factor


# ---- AdamW over many tensors --------------------------------------------------------------------

_TENSOR = np.dtype([(k, "u8") for k in ("param", "grad", "exp_avg", "exp_avg_sq", "units", "master")]
                   + [("n", "i8"), ("place", "i8")] + [(k, "i4") for k in ("group", "param_dtype", "grad_dtype", "reserved")])
_BLOCK = 32      # elements of a block of the 8-bit moments


class AdamWTensors:
    """AdamW over many tensors at once (lce_adamw_tensors_step). ``params`` are contiguous bf16 or fp32 GPU tensors
    that do not overlap, or groups of them: dicts with "params" (tensors, or one) and any of lr, betas, eps and weight_decay, which
    ``groups`` holds and a schedule may change between steps. ``master_weights`` keeps fp32 copies of the bf16 tensors.

    The state is flat: tensor i stands at ``offsets[i]`` of ``exp_avg``, ``exp_avg_sq`` and ``master``, in whole blocks
    of 32 elements. ``state_bits=8`` holds each moment in a byte per element and a unit byte per block
    (``exp_avg``, ``exp_avg_root``, ``units`` [blocks, 2]; the form is described at lce_adamw_tensors_step);
    its rounding draws on ``seed`` and the step count. These tensors may be replaced or moved between steps by others of
    their type and size on the same device."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 master_weights: bool = False, state_bits: int = 32, seed: int = 0):
        if state_bits not in (32, 8):
            raise ValueError(f"state_bits must be 32 or 8, got {state_bits}")
        if isinstance(params, torch.Tensor):
            raise TypeError("params must be a list of tensors or of groups, not a tensor (its rows would be taken for parameters)")
        params = list(params)
        groups = params if params and isinstance(params[0], dict) else [{"params": params}]
        self.params, self.groups, at = [], [], []
        for k, g in enumerate(groups):
            unknown = set(g) - {"params", "lr", "betas", "eps", "weight_decay"}
            if unknown:
                raise ValueError(f"unknown group options {sorted(unknown)}")
            opts = dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay)
            opts.update({o: x for o, x in g.items() if o != "params"})
            self.groups.append(opts)
            members = [g["params"]] if isinstance(g["params"], torch.Tensor) else list(g["params"])
            self.params += members
            at += [k] * len(members)
        if not self.params:
            raise ValueError("no parameters")
        dev = self.params[0].device
        for p in self.params:
            if p.dtype not in _DTYPES:
                raise TypeError(f"parameters must be bfloat16 or float32, got {p.dtype}")
            if not p.is_cuda or p.device != dev or not p.is_contiguous() or p.is_neg():
                raise ValueError("parameters must be contiguous GPU tensors on one device, since they are updated in place")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("parameters overlap (is one given twice?)")
        self.device, self.state_bits, self.seed, self.step_count = dev, state_bits, int(seed), 0
        self.missed = np.zeros(len(self.params), dtype=np.int64)       # steps that each tensor had no gradient in
        self.offsets, total = [], 0
        for p in self.params:
            self.offsets.append(total)
            total += -(-p.numel() // _BLOCK) * _BLOCK
        kind = torch.float32 if state_bits == 32 else torch.uint8
        self.exp_avg = torch.zeros(total, dtype=kind, device=dev)
        second = torch.zeros_like(self.exp_avg)
        self.units = None
        if state_bits == 32:
            self.exp_avg_sq = second
        else:
            self.exp_avg_root = second
            self.units = torch.zeros((total // _BLOCK, 2), dtype=torch.uint8, device=dev)
        self.master = None
        if master_weights:
            self.master = torch.zeros(total, dtype=torch.float32, device=dev)
            with torch.no_grad():
                for p, m in zip(self.params, self.master.split([-(-p.numel() // _BLOCK) * _BLOCK for p in self.params])):
                    m[:p.numel()].view(p.shape).copy_(p)
        self._shapes = [p.shape for p in self.params]
        t = np.zeros(len(self.params), dtype=_TENSOR)
        t["param"] = [p.data_ptr() for p in self.params]
        t["n"] = [p.numel() for p in self.params]
        t["place"], t["group"] = self.offsets, at
        t["param_dtype"] = [_DTYPES[p.dtype] for p in self.params]
        self._table = t
        self._names = ["exp_avg"] + (["exp_avg_sq"] if state_bits == 32 else ["exp_avg_root", "units"])
        self._names += ["master"] if master_weights else []
        self._forms = [(getattr(self, k).shape, getattr(self, k).dtype) for k in self._names]
        self._address_state()

    def _address_state(self) -> None:
        """The addresses of the state's tensors, into the table of the call."""
        state = [getattr(self, k) for k in self._names]
        for k, x, (shape, dtype) in zip(self._names, state, self._forms):
            if not (isinstance(x, torch.Tensor) and x.shape == shape and x.dtype == dtype and x.device == self.device
                    and x.is_contiguous() and not x.is_neg()
                    and (x.storage_offset() + x.numel()) * x.element_size() <= x.untyped_storage().nbytes()):
                raise ValueError(f"{k} must be a contiguous {dtype} tensor of {tuple(shape)} on {self.device}, since it is updated "
                                 "in place")
        t, off, at = self._table, self._table["place"].astype(np.uint64), {k: x.data_ptr() for k, x in zip(self._names, state)}
        t["exp_avg"] = at["exp_avg"] + off * state[0].element_size()
        t["exp_avg_sq"] = at[self._names[1]] + off * state[1].element_size()
        if "units" in at:
            t["units"] = at["units"] + off // 16
        if "master" in at:
            t["master"] = np.where(t["param_dtype"] == B.LCE_DTYPE_BF16, at["master"] + 4 * off, 0)
        self._state_table = np.zeros(len(state), dtype=_GRAD)
        self._state_table["data"] = list(at.values())
        self._state_table["n"] = [x.numel() for x in state]
        self._state_table["dtype"] = [2 if x.dtype == torch.uint8 else _DTYPES[x.dtype] for x in state]

    def _check_state(self) -> None:
        """Follows the state's tensors where they were replaced or moved (a checkpoint, offloading) since the last call."""
        if not _native().stand_at([getattr(self, k) for k in self._names], self._state_table, _GRAD.itemsize, 0, 8, 16):
            self._address_state()

    def _seed_of(self, step: int) -> int:
        return (self.seed * 0x9E3779B9 + step * 0x6A09E667) & 0xFFFFFFFF

    def step(self, grads=None, grad_scale: torch.Tensor | None = None, seed: int | None = None) -> None:
        """One update. ``grads``: a gradient (bf16 or fp32, shaped like its tensor) or None per parameter, by default
        the parameters' ``.grad``; a tensor without one is left as it is, moments included, and its bias correction goes by
        the steps that it took part in (``step_count - missed``). ``grad_scale``: an fp32 GPU scalar that multiplies every
        gradient first (``grad_norm``'s factor); where it is not finite, nothing changes but ``step_count``: the host does
        not know, and the bias correction of later steps counts that one. ``seed``: 32 bits for the rounding of 8-bit
        moments, by default from the state's seed and the step. A step captured into a graph keeps the count, the rates
        and the seed that it was captured with in every replay."""
        params = self.params
        native = _native()
        if len(params) != len(self._table) or not native.stand_at(params, self._table, _TENSOR.itemsize,
                                                                  *(_TENSOR.fields[k][1] for k in ("param", "n", "param_dtype"))):
            raise ValueError("a parameter's storage, type or layout has changed since the state was made")
        self._check_state()
        grads = [p.grad for p in params] if grads is None else list(grads)
        if len(grads) != len(params):
            raise ValueError(f"{len(grads)} gradients for {len(params)} parameters")
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                       or grad_scale.device != self.device or grad_scale.is_neg()):
            raise ValueError("grad_scale must be a one-element float32 tensor on the parameters' device")
        t, out = self._table.copy(), []
        if not native.describe(grads, self._shapes, self.device.index, t, _TENSOR.itemsize, _TENSOR.fields["grad"][1], -1,
                               _TENSOR.fields["grad_dtype"][1]):
            have, out = [k for k, g in enumerate(grads) if g is not None], [k for k, g in enumerate(grads) if g is None]
            grads, t, params = [grads[k] for k in have], t[have], [params[k] for k in have]     # (the call is of these alone)
            if any(g.shape != self._shapes[k] for g, k in zip(grads, have)):
                raise ValueError("gradients must be shaped like their parameters")
            grads, dtypes = _dense(grads, self.device.index)
            _list_dense(grads, dtypes, t, "grad", "grad_dtype")
        step = self.step_count + 1
        # the constants' rows: the groups, or each group at each of its tensors' step counts
        rows = [(k, 0) for k in range(len(self.groups))]
        late = np.delete(self.missed, out) if out else self.missed
        if late.any():
            pairs, row = np.unique(np.stack((t["group"], late)), axis=1, return_inverse=True)
            rows, t["group"] = pairs.T.tolist(), row.reshape(-1)
        opts = (B.LceAdamW * len(rows))(*(
            B.adamw(g["lr"], g["betas"][0], g["betas"][1], g["eps"], g["weight_decay"], step - late)
            for g, late in ((self.groups[k], late) for k, late in rows)))
        with _on(self.device):
            B.lce_adamw_tensors_step(t.ctypes.data, len(t), opts, len(opts), self.state_bits,
                                     grad_scale.data_ptr() if grad_scale is not None else 0,
                                     self._seed_of(step) if seed is None else seed, _stream(self.device))
        native.changed(params)                 # a graph that saved one of them before refuses its backward now
        self.step_count = step
        self.missed[out] += 1

    def moments(self) -> tuple[torch.Tensor, torch.Tensor]:
        """(first moment, root of the second), flat and exactly what the 8-bit state stands for, as bf16
        (lce_adamw_moments)."""
        if self.state_bits != 8:
            raise ValueError("32-bit moments are exp_avg and exp_avg_sq themselves")
        self._check_state()
        first = torch.empty(self.exp_avg.shape, dtype=torch.bfloat16, device=self.device)
        root = torch.empty_like(first)
        with _on(self.device):
            B.lce_adamw_moments(first.numel(), self.exp_avg.data_ptr(), self.exp_avg_root.data_ptr(), self.units.data_ptr(),
                                first.data_ptr(), root.data_ptr(), _stream(self.device))
        return first, root

    def state_dict(self) -> dict:
        """State for checkpointing (tensors are shared, not copied)."""
        sd = {"step": self.step_count, "missed": self.missed.tolist(), "seed": self.seed,
              "state_bits": self.state_bits, "groups": [dict(g) for g in self.groups], "exp_avg": self.exp_avg, "master": self.master,
              "shapes": [tuple(s) for s in self._shapes], "group_of": self._table["group"].tolist()}
        return sd | ({"exp_avg_sq": self.exp_avg_sq} if self.state_bits == 32
                     else {"exp_avg_root": self.exp_avg_root, "units": self.units})

    def load_state_dict(self, sd: dict) -> None:
        """Restore a state_dict: moments (and master copies) are copied into this state's tensors. The tensors must be those
        of the checkpoint in its order: other shapes or another split into groups are refused."""
        names = ["exp_avg", "exp_avg_sq"] if self.state_bits == 32 else ["exp_avg", "exp_avg_root", "units"]
        if any(n not in sd for n in names) or sd.get("state_bits", self.state_bits) != self.state_bits:
            raise ValueError(f"the checkpoint does not hold {self.state_bits}-bit moments")
        if (sd.get("master") is None) != (self.master is None):
            raise ValueError("master-weight setting differs from the checkpoint")
        if len(sd.get("groups", self.groups)) != len(self.groups):
            raise ValueError("the checkpoint has another number of groups")
        own = self._shapes, self._table["group"].tolist()
        if [tuple(s) for s in sd.get("shapes", own[0])] != own[0] or list(sd.get("group_of", own[1])) != own[1]:
            raise ValueError("the checkpoint is of tensors of other shapes, or in another order or other groups")
        step, missed = int(sd["step"]), np.array(sd.get("missed", [0] * len(self.params)), dtype=np.int64)
        if missed.shape != self.missed.shape:
            raise ValueError("the checkpoint has another number of tensors")
        names += ["master"] if self.master is not None else []
        for n in names:
            own = getattr(self, n)
            if sd[n].shape != own.shape or sd[n].dtype != own.dtype:
                raise ValueError(f"{n} is {tuple(sd[n].shape)} {sd[n].dtype} in the checkpoint, {tuple(own.shape)} {own.dtype} here")
        for n in names:
            getattr(self, n).copy_(sd[n])
        self.step_count, self.missed = step, missed
        self.seed = int(sd.get("seed", self.seed))
        for g, x in zip(self.groups, sd.get("groups", [])):
            g.update(x)
