"""Buffer management around one plan: PyTorch supplies device memory and the stream, the C ABI
does all the arithmetic."""
from __future__ import annotations

import threading

import numpy as np
import torch

from . import binding
from .binding import (ASI_ADAMW_BLOCK, ASI_BF16, ASI_F32, ASI_NORM_LAYER, ASI_NORM_RMS, ASI_OK, AdamwDesc, AdamwTensor, Batch, Branch,
                      BranchDesc, Dropout, EmbeddingDesc, HeadDesc, LogprobDesc, Plan)


def _stream_handle(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


class LayerRunner:
    """Device buffers of one layer (two factor buffers that alternate as previous/new, core, dW,
    workspaces) and the calls that fill them."""

    def __init__(self, kind, dims, ranks, cout, k=1, stride=1, pad=0, groups=1, bf16=False,
                 device="cuda:0", generic_only=False, flags=0):
        if not torch.cuda.is_available():
            raise RuntimeError("the ASI path needs a CUDA device; there is no CPU fallback")
        self.plan = Plan(kind, dims, ranks, cout, k, stride, pad, groups, bf16,
                         generic_only=generic_only, flags=flags)
        self.dims, self.ranks, self.bf16 = tuple(dims), tuple(ranks), bf16
        self.device = torch.device(device)
        info = self.plan.info
        f32 = dict(dtype=torch.float32, device=self.device)
        self.U = [torch.zeros(info.u_elems, **f32), torch.zeros(info.u_elems, **f32)]
        self.cur = 0                       # index of the buffer holding the latest factors
        self.core = torch.zeros(info.core_elems, **f32)
        self.dW = torch.zeros(info.dw_elems, **f32)
        self.ws_c = torch.zeros(info.compress_ws_bytes, dtype=torch.uint8, device=self.device)
        self.ws_w = torch.zeros(info.wgrad_ws_bytes, dtype=torch.uint8, device=self.device)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32

    # -- host <-> device helpers ---------------------------------------------------------
    def to_device(self, x: np.ndarray) -> torch.Tensor:
        t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(self.device)
        return t.to(self.in_dtype).contiguous()

    def set_factors(self, U_list):
        flat = np.concatenate([np.ascontiguousarray(u, dtype=np.float32).ravel() for u in U_list])
        self.U[self.cur].copy_(torch.from_numpy(flat))

    def factors(self, which=None):
        buf = self.U[self.cur if which is None else which].cpu().numpy()
        out, off = [], 0
        for d, r in zip(self.dims, self.ranks):
            out.append(buf[off:off + d * r].reshape(d, r).copy())
            off += d * r
        return out

    @property
    def dW_shape(self):
        """[Cout, C / groups, kh, kw] or [Dout, Din], row-major in dW."""
        d = self.plan.desc
        if self.plan.kind == "conv":
            return d.cout, d.dims[1] // d.groups, d.kh, d.kw
        return d.cout, d.dims[d.ndim - 1]

    def core_np(self):
        return self.core.cpu().numpy().reshape(self.ranks).copy()

    def dW_np(self, shape):
        return self.dW.cpu().numpy().reshape(shape).copy()

    # -- the path ------------------------------------------------------------------------
    def compress(self, act: torch.Tensor, stream=None):
        prev, new = self.U[self.cur], self.U[1 - self.cur]
        self.plan.compress(act.data_ptr(), prev.data_ptr(), new.data_ptr(), self.core.data_ptr(),
                           self.ws_c.data_ptr(), self.ws_c.numel(), _stream_handle(stream))
        self.cur = 1 - self.cur

    def init_factors(self, act: torch.Tensor, omega: torch.Tensor, stream=None):
        new = self.U[1 - self.cur]
        self.plan.init_factors(act.data_ptr(), omega.data_ptr(), new.data_ptr(), self.core.data_ptr(),
                               self.ws_c.data_ptr(), self.ws_c.numel(), _stream_handle(stream))
        self.cur = 1 - self.cur

    def init_factors_seeded(self, act: torch.Tensor, seed: int, stream=None):
        """Cold start with the library's counter-based Gaussian test matrices (allocates its scratch once)."""
        need = self.plan.init_seeded_ws_bytes()
        if getattr(self, "ws_seed", None) is None or self.ws_seed.numel() < need:
            with torch.cuda.stream(stream):    # (memory that this stream is done with)
                self.ws_seed = torch.empty(need, dtype=torch.uint8, device=self.core.device)
        new = self.U[1 - self.cur]
        self.plan.init_factors_seeded(act.data_ptr(), seed, new.data_ptr(), self.core.data_ptr(),
                                      self.ws_seed.data_ptr(), self.ws_seed.numel(), _stream_handle(stream))
        self.cur = 1 - self.cur

    def wgrad(self, dY: torch.Tensor, stream=None):
        self.plan.wgrad(self.core.data_ptr(), self.U[self.cur].data_ptr(), dY.data_ptr(),
                        self.dW.data_ptr(), self.ws_w.data_ptr(), self.ws_w.numel(),
                        _stream_handle(stream))

    def device_status(self, stream=None):
        return self.plan.poll_status(self.ws_c.data_ptr(), _stream_handle(stream))

    def ok(self):
        return self.device_status() == ASI_OK


class StepRunner:
    """The layers of one training step behind the batched entry points: one asi_compress_batched call
    for the forward pass, one asi_wgrad_batched call for the backward pass."""

    def __init__(self, runners):
        self.runners = list(runners)
        self.batch = Batch([r.plan for r in self.runners])

    def compress(self, acts, stream=None):
        rs = self.runners
        self.batch.compress([a.data_ptr() for a in acts], [r.U[r.cur].data_ptr() for r in rs],
                            [r.U[1 - r.cur].data_ptr() for r in rs], [r.core.data_ptr() for r in rs],
                            [r.ws_c.data_ptr() for r in rs], [r.ws_c.numel() for r in rs], _stream_handle(stream))
        for r in rs:
            r.cur = 1 - r.cur

    def wgrad(self, dys, stream=None):
        rs = self.runners
        self.batch.wgrad([r.core.data_ptr() for r in rs], [r.U[r.cur].data_ptr() for r in rs],
                         [d.data_ptr() for d in dys], [r.dW.data_ptr() for r in rs],
                         [r.ws_w.data_ptr() for r in rs], [r.ws_w.numel() for r in rs], _stream_handle(stream))

    def optimizer(self, weights, **kw):
        """AdamW over the layers' weights (one for each, fp32 or bf16, of dW's sizes, or with neighbouring ones
        joined or one of them split) and the dW buffers of the layers."""
        weights = list(weights)

        def parts(shape):                  # what lies together, from whole rows down to neighbours
            return {int(np.prod(shape[i:], dtype=np.int64)) for i in range(len(shape))}

        for r, w in zip(self.runners, weights):
            have, need = parts(w.shape) | {1}, parts(r.dW_shape) | {1}
            if not (have <= need or need <= have):
                raise ValueError(f"weight: {r.dW_shape} is needed, as dW is laid out, got {tuple(w.shape)}")
        return AdamWRunner(weights, [r.dW for r in self.runners], **kw)


# ---- the rest of a language model's training step ---------------------------------------------------

_DTYPES = {torch.float32: ASI_F32, torch.bfloat16: ASI_BF16}


# handle of a device's current stream, without a stream object for each call where torch offers that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Descriptor(threading.local):
    """A descriptor for each thread: the library reads it while other threads may prepare calls of theirs."""

    def __init__(self, first):
        self.desc = type(first).from_buffer_copy(first)


class _Runner:
    """Calls on a stream, and buffers of the runner's own (`_own`) that any stream of its device may use: one that was not
    current when they were made waits for what was queued there (what filled them, and what used their memory before), and
    the allocator learns of it, so that the memory of a runner that is dropped is not given away beneath it."""

    def _made(self, device):
        """To be called where the buffers have been made, on the device's current stream."""
        with torch.cuda.device(device):
            self._captured = torch.cuda.is_current_stream_capturing()
            self._ready = torch.cuda.current_stream().record_event()
        self._streams = {_raw_stream(device.index)}

    @property
    def desc(self):
        return self._descriptor.desc

    def _own(self):
        return ()

    def _lend(self, stream):
        for x in self._own():
            x.record_stream(stream)
        with torch.cuda.stream(stream):
            # (a capture cannot wait for what is not part of it; the graph's user has it behind them)
            if torch.cuda.is_current_stream_capturing() == self._captured:
                stream.wait_event(self._ready)
                self._streams.add(stream.cuda_stream)

    def _call(self, stream, function, *args):
        """function(*args, handle) with the runner's device current, on `stream` or that device's current stream."""
        device = self.device
        if stream is not None and stream.device != device:
            raise ValueError(f"a stream of {device} is needed, got one of {stream.device}")
        if torch.cuda.current_device() != device.index:
            with torch.cuda.device(device):
                return self._call(stream, function, *args)
        handle = _raw_stream(device.index) if stream is None else stream.cuda_stream
        if handle not in self._streams:
            self._lend(torch.cuda.current_stream(device) if stream is None else stream)
        function(*args, handle)


def _cuda_device(device):
    d = torch.device(device)
    if d.type != "cuda":
        raise ValueError("the ASI path needs a CUDA device; there is no CPU fallback")
    if not torch.cuda.is_available():
        raise RuntimeError("the ASI path needs a CUDA device; there is no CPU fallback")
    return torch.device("cuda", torch.cuda.current_device() if d.index is None else d.index)


def _take(name, x, shape, dtype, device):
    """The address of a contiguous tensor of that shape and type on that device."""
    if x.dtype != dtype or x.shape != shape or x.device != device or not x.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} on {device} is needed, got {x.dtype} "
                         f"{tuple(x.shape)} on {x.device}")
    return x.data_ptr()


_address = torch.Tensor.data_ptr


def _result(name):
    """A result buffer as an attribute; another one may take its place."""
    def put(self, x):
        self._bind({**self._results, name: x})

    return property(lambda self: self._results[name], put)


class _RowResults(_Runner):
    """Result buffers of a value (or `top_k` values) a row, which another contiguous buffer may replace."""

    logp, entropy, lse, top_logp, top_ids = map(_result, ("logp", "entropy", "lse", "top_logp", "top_ids"))

    def _new(self):
        return {name: torch.zeros(self.rows, *more, dtype=dtype, device=self.device) if 0 not in more else None
                for name, more, dtype in self._layout()}

    def _layout(self):
        """Name, sizes behind the rows and type of each result, in the order of the library's arguments."""
        return [(name, (), torch.float32) for name in ("logp", "entropy", "lse")] + [
            ("top_logp", (self.top_k,), torch.float32), ("top_ids", (self.top_k,), torch.int64)]

    def _bind(self, results):
        """Takes buffers for the results, checked, and notes where they lie and for how many rows."""
        at, rows = {}, {}
        for name, more, dtype in self._layout():
            x = results[name]
            if 0 in more:
                if x is not None:
                    raise ValueError(f"{name}: there are no top entries")
                at[name] = 0
                continue
            if (not isinstance(x, torch.Tensor) or x.dim() != 1 + len(more) or tuple(x.shape[1:]) != more or x.dtype != dtype
                    or x.device != self.device or not x.is_contiguous() or (x.numel() and not x.data_ptr())):
                raise ValueError(f"{name}: contiguous {dtype} rows of {more} on {self.device} are needed, got "
                                 + (f"{x.dtype} {tuple(x.shape)} on {x.device}" if isinstance(x, torch.Tensor) else f"{x!r}"))
            at[name], rows[name] = x.data_ptr(), x.shape[0]
        self._results = dict(results)
        self._buffers = tuple(x for x in self._results.values() if x is not None)
        self._at = tuple(map(_address, self._buffers))
        self._most, self._most_stats = min(rows.values()), min(rows["entropy"], rows["lse"])
        self._stats, self._top = (at["logp"], at["entropy"], at["lse"]), (at["top_logp"], at["top_ids"])

    def _outputs(self, n, stats=False):
        """The results have room for n rows where they lie now (their memory may have been exchanged since the last call)."""
        if tuple(map(_address, self._buffers)) != self._at:
            self._bind(self._results)
        if n > (self._most_stats if stats else self._most):
            raise ValueError(f"results of {n} rows or more are needed, there are {[len(x) for x in self._buffers]}")

    def _own(self):
        return self._buffers


class LogprobRunner(_RowResults):
    """Log probabilities of given tokens over logits of up to `rows` rows: device buffers of the results (logp, entropy,
    lse; top_logp and top_ids where top_k > 0) and the calls that fill them.  A shorter batch fills the first rows and leaves
    the others as they were.  backward() reads lse and entropy of the last forward() or loss(), or those that it is given.
    Another contiguous buffer may be assigned to each result.  Calls that may run at the same time share these results: they
    need a runner each."""

    def __init__(self, rows, vocab, bf16=False, scale=1.0, ignore_index=-100, top_k=0, device="cuda:0"):
        self.device = _cuda_device(device)
        self.rows, self.vocab, self.top_k = int(rows), int(vocab), int(top_k)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32
        self._descriptor = _Descriptor(LogprobDesc(_DTYPES[self.in_dtype], self.top_k, 0, self.vocab, 0, 0, int(ignore_index),
                                                   float(scale)))
        self._bind(self._new())
        self._made(self.device)

    def _rows_of(self, name, x):
        """Rows and row stride of logits or their gradient."""
        if x.dim() == 2 and x.dtype == self.in_dtype and x.device == self.device:
            (n, v), (ld, one) = x.shape, x.stride()
            if n <= self.rows and v == self.vocab and (one == 1 or v == 1) and (ld >= v or n <= 1):
                return n, max(ld, v)
        raise ValueError(f"{name}: {self.in_dtype} rows [<= {self.rows}, {self.vocab}] on {self.device} are needed, each "
                         f"contiguous, got {x.dtype} {tuple(x.shape)}, strides {x.stride()}, on {x.device}")

    def _inputs(self, logits, targets, dlogits=None):
        d = self._descriptor.desc
        n, ld = self._rows_of("logits", logits)
        d.rows, d.ld, d.ld_grad = n, ld, ld
        if dlogits is not None:
            m, d.ld_grad = self._rows_of("dlogits", dlogits)
            if m != n:
                raise ValueError(f"dlogits: {n} rows are needed, got {m}")
        return d, n, _take("targets", targets, (n,), torch.int64, self.device)

    def _weights(self, n, dlogp, dentropy):
        return (_take("dlogp", dlogp, (n,), torch.float32, self.device),
                _take("dentropy", dentropy, (n,), torch.float32, self.device) if dentropy is not None else 0)

    def forward(self, logits, targets, stream=None):
        desc, n, y = self._inputs(logits, targets)
        self._outputs(n)
        self._call(stream, binding.token_logprobs, desc, logits.data_ptr(), y, *self._stats, *self._top)

    def backward(self, logits, targets, dlogp, dentropy, dlogits, stream=None, lse=None, entropy=None):
        """The gradient of sum(dlogp * logp + dentropy * entropy) into dlogits, from the lse and entropy that forward() left, or
        from those given (a value a row of logits: what forward() left for an earlier batch); dentropy may be None, and dlogits
        may be logits itself."""
        desc, n, y = self._inputs(logits, targets, dlogits)
        if lse is None and entropy is None:
            self._outputs(n, stats=True)
            _, h, z = self._stats
        elif lse is None or (entropy is None and dentropy is not None):
            raise ValueError("lse and entropy (where dentropy is there) come together, from the same forward()")
        else:
            z = _take("lse", lse, (n,), torch.float32, self.device)
            h = _take("entropy", entropy, (n,), torch.float32, self.device) if entropy is not None else 0
        self._call(stream, binding.token_logprobs_grad, desc, logits.data_ptr(), y, z, h,
                   *self._weights(n, dlogp, dentropy), dlogits.data_ptr())

    def loss(self, logits, targets, dlogp, dentropy, dlogits, stream=None):
        """forward() without the top entries, and backward(), in one pass over the logits."""
        desc, n, y = self._inputs(logits, targets, dlogits)
        self._outputs(n)
        self._call(stream, binding.token_loss, desc, logits.data_ptr(), y, *self._weights(n, dlogp, dentropy),
                   *self._stats, dlogits.data_ptr())


class EmbeddingRunner(_Runner):
    """Embedding lookup of up to `tokens` tokens and its weight gradient, with the workspace of the latter: calls of wgrad() (and
    graphs captured from them) that may run at the same time need a runner each; threads may share one for forward()."""

    def __init__(self, vocab, dim, tokens, bf16=False, bf16_table=False, scale=1.0, padding_idx=None, device="cuda:0"):
        self.device = _cuda_device(device)
        self.vocab, self.dim, self.tokens = int(vocab), int(dim), int(tokens)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32
        self.table_dtype = torch.bfloat16 if bf16_table else torch.float32
        self._descriptor = _Descriptor(EmbeddingDesc(_DTYPES[self.table_dtype], _DTYPES[self.in_dtype], self.vocab, self.dim,
                                                     self.tokens, -1 if padding_idx is None else int(padding_idx), float(scale)))
        # as large as the longest batch needs
        self.ws = torch.empty(binding.embedding_wgrad_ws_bytes(self.desc), dtype=torch.uint8, device=self.device)
        self._made(self.device)

    def _own(self):
        return (self.ws,)

    def _ids(self, ids):
        n = ids.numel()
        if ids.dtype != torch.int64 or ids.device != self.device or not ids.is_contiguous() or n > self.tokens:
            raise ValueError(f"ids: a contiguous int64 tensor of up to {self.tokens} tokens on {self.device} is needed, got "
                             f"{ids.dtype} {tuple(ids.shape)} on {ids.device}")
        desc = self._descriptor.desc
        desc.tokens = n
        return desc, (*ids.shape, self.dim)

    def forward(self, table, ids, out, stream=None):
        desc, shape = self._ids(ids)
        w = _take("table", table, (self.vocab, self.dim), self.table_dtype, self.device)
        o = _take("out", out, shape, self.in_dtype, self.device)
        self._call(stream, binding.embedding_forward, desc, w, ids.data_ptr(), o)

    def wgrad(self, ids, dOut, dW, accumulate=False, stream=None):
        """dW (fp32 [vocab, dim]) overwritten with, or increased by, the gradient."""
        desc, shape = self._ids(ids)
        d = _take("dOut", dOut, shape, self.in_dtype, self.device)
        w = _take("dW", dW, (self.vocab, self.dim), torch.float32, self.device)
        self._call(stream, binding.embedding_wgrad, desc, ids.data_ptr(), d, w, accumulate, self.ws.data_ptr(),
                   self.ws.numel())


class AdamWRunner(_Runner):
    """AdamW over a list of weights and their gradient buffers (the dW of layer runners, for example): holds the states and
    steps all tensors in one call.  States may be given (to resume); the 8-bit ones are float8_e4m3fn with one
    float8_e8m0fnu (or uint8) scale for each ASI_ADAMW_BLOCK elements of a tensor.  `copies` (bf16) receive the new weights.

    A weight, gradient or copy whose memory is exchanged (`w.data = ...`) is found by the next step().  The states stay where
    they were when the runner was made: values are loaded with copy_(), other memory with rebind().  All of it is kept alive
    until then."""

    def __init__(self, weights, grads, bits8=False, copies=None, exp_avg=None, exp_avg_sq=None, exp_avg_scale=None,
                 exp_avg_sq_scale=None):
        weights, grads = tuple(weights), tuple(grads)
        if not weights or len(grads) != len(weights):
            raise ValueError("one gradient for each of one or more weights is needed")
        self.device = _cuda_device(weights[0].device)
        self.bits8, self.t = bool(bits8), 0
        wd, gd = weights[0].dtype, grads[0].dtype
        if wd not in _DTYPES or gd not in _DTYPES:
            raise ValueError("weights and gradients are fp32 or bf16")
        sd = torch.float8_e4m3fn if self.bits8 else torch.float32
        new = []

        def states(given, dtype, per, fill):
            if given is not None:
                return tuple(given)
            made = [torch.empty(-(-w.numel() // per), dtype=dtype, device=self.device) for w in weights]
            for x in made:
                x.view(torch.uint8).fill_(fill)
            new.extend(made)
            return tuple(made)

        none = (None,) * len(weights)
        self._tensors = dict(weights=weights, grads=grads, exp_avg=states(exp_avg, sd, 1, 0), exp_avg_sq=states(exp_avg_sq, sd, 1, 0))
        for name, given in (("exp_avg_scale", exp_avg_scale), ("exp_avg_sq_scale", exp_avg_sq_scale)):
            self._tensors[name] = states(given, torch.float8_e8m0fnu, ASI_ADAMW_BLOCK, 127) if self.bits8 else none
        self._tensors["copies"] = tuple(copies) if copies is not None else none
        if any(len(x) != len(weights) for x in self._tensors.values()):
            raise ValueError("one state (scale, copy) for each weight is needed")
        self._types = wd, gd, sd
        self._descriptor = _Descriptor(AdamwDesc(weight_dtype=_DTYPES[wd], grad_dtype=_DTYPES[gd],
                                                 state_bits=8 if self.bits8 else 32))
        self._watched = (*weights, *grads, *(c for c in self._tensors["copies"] if c is not None))
        self._states = new
        self.rebind()
        self._made(self.device)

    weights, grads, copies, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale = (
        property(lambda self, name=name: self._tensors[name])
        for name in ("weights", "grads", "copies", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"))

    def rebind(self):
        """Takes all tensors as they lie now, checked like those that the runner was made with."""
        wd, gd, sd = self._types
        table, kept = (AdamwTensor * len(self.weights))(), []

        def at(name, x, n, *dtypes):
            address = x.data_ptr()
            if (x.dtype not in dtypes or x.numel() != n or x.device != self.device or not x.is_contiguous()
                    or (n and not address)):
                raise ValueError(f"{name}: {n} contiguous values of {dtypes[0]} on {self.device} are needed, got {x.dtype} "
                                 f"{tuple(x.shape)} on {x.device}")
            kept.append(x.untyped_storage())       # (not x, which may let go of it)
            return address

        for e, w, g, m, v, ms, vs, c in zip(table, self.weights, self.grads, self.exp_avg, self.exp_avg_sq, self.exp_avg_scale,
                                            self.exp_avg_sq_scale, self.copies):
            n = w.numel()
            e.weight, e.grad = at("weight", w, n, wd), at("grad", g, n, gd)
            e.exp_avg, e.exp_avg_sq = at("exp_avg", m, n, sd), at("exp_avg_sq", v, n, sd)
            if self.bits8:
                scale = -(-n // ASI_ADAMW_BLOCK), torch.float8_e8m0fnu, torch.uint8
                e.exp_avg_scale, e.exp_avg_sq_scale = at("exp_avg_scale", ms, *scale), at("exp_avg_sq_scale", vs, *scale)
            e.copy = at("copy", c, n, torch.bfloat16) if c is not None else None
            e.n = n
        self._table, self._kept = table, kept
        self._at = tuple(map(_address, self._watched))

    def _own(self):
        return self._states                # (those that were given are their owner's)

    def step(self, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=None, grad_scale=None, stream=None):
        """One step.  `step` counts from 1 (default: one more than at the call before, which then was not counted on the device).
        lr (fp32) and step (int64) may be one-element device tensors, so that a captured graph reads new values; grad_scale
        (fp32) is one if given."""
        d = self._descriptor.desc
        d.beta1, d.beta2, d.eps, d.weight_decay = beta1, beta2, eps, weight_decay
        d.lr_dev = d.step_dev = d.grad_scale = None
        if isinstance(lr, torch.Tensor):
            d.lr, d.lr_dev = 0.0, _take("lr", lr.reshape(1), (1,), torch.float32, self.device)
        else:
            d.lr = lr
        if isinstance(step, torch.Tensor):
            d.step, d.step_dev = 1, _take("step", step.reshape(1), (1,), torch.int64, self.device)
        elif step is None and self.t is None:
            raise ValueError("the step before was counted on the device: which one this is has to be given")
        else:
            d.step = self.t + 1 if step is None else int(step)
        if grad_scale is not None:
            d.grad_scale = _take("grad_scale", grad_scale.reshape(1), (1,), torch.float32, self.device)
        if tuple(map(_address, self._watched)) != self._at:
            self.rebind()
        self._call(stream, binding.adamw_step, d, self._table, len(self._table))
        self.t = None if isinstance(step, torch.Tensor) else d.step


# ---- a block's other operators, and the output layer with its loss ------------------------------------

def _drop(p, seed, stream_id):
    return Dropout(float(p), int(seed), int(stream_id), 0, None)


class _Masked(_Descriptor):
    """... and the part of it that draws the mask."""

    def __init__(self, first):
        super().__init__(first)
        self.drop, self.on_device = getattr(self.desc, "drop", self.desc), False


class _Steps(_Runner):
    """A mask for each step: `step` may be a number, or a one-element int64 device tensor that a captured graph reads."""

    def _at_step(self, local, step):
        drop = local.drop
        if isinstance(step, torch.Tensor):
            drop.step, drop.step_dev = 0, _take("step", step.reshape(1), (1,), torch.int64, self.device)
            local.on_device = True
        else:
            drop.step = int(step)
            if local.on_device:
                drop.step_dev, local.on_device = None, False


class DropoutRunner(_Steps):
    """Dropout whose mask follows from (seed, stream_id, step) and an element's place: nothing is kept between forward() and
    backward(), which have to be given the same step.  No buffers of its own: calls may run at the same time."""

    def __init__(self, p, seed, stream_id=0, bf16=False, device="cuda:0"):
        self.device = _cuda_device(device)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32
        self._descriptor = _Masked(_drop(p, seed, stream_id))
        self._made(self.device)

    def forward(self, x, out, step=0, residual=None, stream=None):
        """out = x with elements dropped and the others scaled, plus residual if given.  out may be x or residual."""
        local, dtype, device, shape = self._descriptor, self.in_dtype, self.device, x.shape
        self._at_step(local, step)
        a, o = _take("x", x, shape, dtype, device), _take("out", out, shape, dtype, device)
        r = _take("residual", residual, shape, dtype, device) if residual is not None else 0
        self._call(stream, binding.dropout, local.desc, _DTYPES[dtype], x.numel(), a, r, o)

    def backward(self, dout, dx, step=0, stream=None):
        """dx = the gradient of x (that of residual is dout itself).  dx may be dout."""
        self.forward(dout, dx, step, stream=stream)


class ResidualNormRunner(_Steps):
    """The end of a block for up to `rows` rows: norm after its branch, gate, dropout, residual sum and the next block's norm, and their
    gradient.  Holds the rows' statistics (`stats`, that backward() reads as the last forward() left them; another
    contiguous fp32 [>= rows, 4] buffer may be assigned) and the backward workspace: calls (and graphs captured from them) that may run
    at the same time need a runner each.  Biases are for norm="layer" alone."""

    def __init__(self, rows, dim, bf16=False, bf16_residual=False, norm="rms", norm_after=False, rows_per_gate=0, eps=1e-5, res_scale=1.0,
                 branch_scale=1.0, dropout=0.0, seed=0, stream_id=0, device="cuda:0"):
        self.device = _cuda_device(device)
        self.rows, self.dim, self.rows_per_gate = int(rows), int(dim), int(rows_per_gate)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32
        self.res_dtype = torch.bfloat16 if bf16_residual else torch.float32
        self.norm_after = bool(norm_after)
        kinds = dict(rms=ASI_NORM_RMS, layer=ASI_NORM_LAYER)
        if norm not in kinds:
            raise ValueError(f"norm: one of {sorted(kinds)} is needed, got {norm!r}")
        self._descriptor = _Masked(BranchDesc(_DTYPES[self.in_dtype], _DTYPES[self.res_dtype], kinds[norm], self.norm_after, self.rows,
                                              self.dim, self.rows_per_gate, eps, res_scale, branch_scale, _drop(dropout, seed, stream_id)))
        self._row = torch.Size((self.dim,))
        self.stats = torch.zeros(self.rows, 4, dtype=torch.float32, device=self.device)
        self.ws = torch.empty(binding.branch_backward_ws_bytes(self.desc), dtype=torch.uint8, device=self.device)
        self._made(self.device)

    def _own(self):
        return (self._stats, self.ws)

    @property
    def stats(self):
        return self._stats

    @stats.setter
    def stats(self, x):
        _take("stats", x, (len(x), 4), torch.float32, self.device)
        self._stats, self._stats_at, self._most = x, x.data_ptr(), min(self.rows, len(x))

    def _begin(self, y, step):
        """The thread's descriptor for y's rows, how many these are, their sizes, and the statistics' address."""
        local, shape = self._descriptor, y.shape
        if self._stats.data_ptr() != self._stats_at:       # (its memory was exchanged)
            self.stats = self._stats
        n = y.numel() // self.dim
        if not shape or shape[-1] != self.dim or n > self._most:
            raise ValueError(f"y: up to {self._most} rows of {self.dim} are needed (as many as the runner and its stats have), got {tuple(shape)}")
        local.desc.rows = n
        self._at_step(local, step)
        return local.desc, n, shape, self._stats_at

    def _shared(self, n, gate, after, next):
        """Addresses of the gate and of the norms' weights and biases."""
        per, row, f32, device = self.rows_per_gate, self._row, torch.float32, self.device
        if (gate is None) is bool(per):
            raise ValueError("gate: the runner was made " + ("with" if per else "without") + " one")
        (aw, ab), (nw, nb) = after, next
        return (_take("gate", gate, (-(-n // per), self.dim), f32, device) if per else 0,
                0 if aw is None else _take("after's weight", aw, row, f32, device), 0 if ab is None else _take("after's bias", ab, row, f32, device),
                0 if nw is None else _take("next's weight", nw, row, f32, device), 0 if nb is None else _take("next's bias", nb, row, f32, device))

    def forward(self, y, h, h_out, x=None, gate=None, after=(None, None), next=(None, None), step=0, stream=None):
        """h_out = res_scale h + branch_scale drop(gate norm(y)), x = norm(h_out); `after` and `next` are (weight, bias) of the two
        norms.  h may be None (0), h_out may be h; without x no norm follows."""
        d, n, shape, stats = self._begin(y, step)
        it, rt, device = self.in_dtype, self.res_dtype, self.device
        buffers = binding.Branch.pack(
            _take("y", y, shape, it, device), 0 if h is None else _take("h", h, shape, rt, device), *self._shared(n, gate, after, next),
            _take("h_out", h_out, shape, rt, device), 0 if x is None else _take("x", x, shape, it, device), stats, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        self._call(stream, binding.branch_forward, d, buffers)

    def backward(self, y, h_out, dx, dh_out, dy, dh=None, gate=None, after=(None, None), next=(None, None), dgate=None, dafter=(None, None),
                 dnext=(None, None), accumulate=False, step=0, stream=None):
        """Gradients from those of x (dx) and h_out (dh_out; either may be None): dy and dh overwritten, dgate, dafter and dnext (where
        given) overwritten or, with accumulate, increased.  dy may be dx, dh may be dh_out."""
        d, n, shape, stats = self._begin(y, step)
        it, rt, f32, device, row = self.in_dtype, self.res_dtype, torch.float32, self.device, self._row
        per, (daw, dab), (dnw, dnb) = self.rows_per_gate, dafter, dnext
        if dgate is not None and not per:
            raise ValueError("dgate: the runner was made without a gate")
        buffers = binding.Branch.pack(
            _take("y", y, shape, it, device), 0, *self._shared(n, gate, after, next), 0 if h_out is None else _take("h_out", h_out, shape, rt, device), 0,
            stats, 0 if dx is None else _take("dx", dx, shape, it, device), 0 if dh_out is None else _take("dh_out", dh_out, shape, rt, device),
            _take("dy", dy, shape, it, device), 0 if dh is None else _take("dh", dh, shape, rt, device),
            0 if dgate is None else _take("dgate", dgate, (-(-n // per), self.dim), f32, device),
            0 if daw is None else _take("dafter's weight", daw, row, f32, device), 0 if dab is None else _take("dafter's bias", dab, row, f32, device),
            0 if dnw is None else _take("dnext's weight", dnw, row, f32, device), 0 if dnb is None else _take("dnext's bias", dnb, row, f32, device))
        self._call(stream, binding.branch_backward, d, buffers, accumulate, self.ws.data_ptr(), self.ws.numel())


class HeadRunner(_RowResults):
    """Output layer and loss for up to `rows` hidden states, without logits: log probabilities of given tokens (logp, entropy and lse, as of
    LogprobRunner) and the gradients of hidden states and weight.  Holds these results and the workspace (for `grad` that of the
    gradients, `vocab_chunk` columns of the logits' gradient at a time, 0: the library's choice): calls (and graphs captured
    from them) that may run at the same time need a runner each."""

    top_k = 0

    def __init__(self, rows, vocab, dim, bf16=False, bf16_dw=False, scale=1.0, ignore_index=-100, vocab_chunk=0, grad=True, flags=0,
                 device="cuda:0"):
        self.device = _cuda_device(device)
        self.rows, self.vocab, self.dim, self.grad = int(rows), int(vocab), int(dim), bool(grad)
        self.in_dtype = torch.bfloat16 if bf16 else torch.float32
        self.dw_dtype = torch.bfloat16 if bf16_dw else torch.float32
        self._descriptor = _Descriptor(HeadDesc(_DTYPES[self.in_dtype], _DTYPES[self.dw_dtype], self.rows, self.vocab, self.dim,
                                                int(vocab_chunk), int(ignore_index), float(scale), int(flags)))
        self.ws = torch.empty(binding.head_ws_bytes(self.desc, self.grad), dtype=torch.uint8, device=self.device)
        self.ws[:256].zero_()              # (the status word, before the first call)
        self._bind(self._new())
        self._made(self.device)

    def _own(self):
        return (self.ws, *self._buffers)

    def _inputs(self, x, weight, targets):
        d, n = self._descriptor.desc, targets.numel()
        if n > self.rows:
            raise ValueError(f"targets: up to {self.rows} are needed, got {n}")
        d.rows = n
        return d, n, (_take("x", x, (*targets.shape, self.dim), self.in_dtype, self.device),
                      _take("weight", weight, (self.vocab, self.dim), self.in_dtype, self.device),
                      _take("targets", targets, targets.shape, torch.int64, self.device))

    def _gradients(self, n, x, dlogp, dentropy, dx, dw, stream):
        """Addresses of weights and gradients, and the weights, to be held until the call is queued."""
        if not self.grad:
            raise ValueError("the runner was made without gradients")
        weights = [w if w is None or w.is_contiguous() else self._copy(w, stream) for w in (dlogp, dentropy)]
        return (tuple(0 if w is None else _take(name, w.view(-1), (n,), torch.float32, self.device) for name, w in zip(("dlogp", "dentropy"), weights)),
                (_take("dx", dx, x.shape, self.in_dtype, self.device) if dx is not None else 0,
                 _take("dw", dw, (self.vocab, self.dim), self.dw_dtype, self.device) if dw is not None else 0), weights)

    @staticmethod
    def _copy(x, stream):
        with torch.cuda.stream(stream):        # (the call's own, in whose order it is read and its memory used again)
            return x.contiguous()

    def forward(self, x, weight, targets, stream=None):
        desc, n, inputs = self._inputs(x, weight, targets)
        self._outputs(n)
        self._call(stream, binding.head_logprobs, desc, *inputs, *self._stats, self.ws.data_ptr(), self.ws.numel())

    def backward(self, x, weight, targets, dlogp, dentropy, dx, dw, accumulate=False, stream=None, lse=None, entropy=None):
        """The gradient of sum(dlogp * logp + dentropy * entropy) into dx and dw (either may be None; dw is increased with accumulate),
        from the lse and entropy that forward() left, or from those given."""
        desc, n, inputs = self._inputs(x, weight, targets)
        weights, grads, _held = self._gradients(n, x, dlogp, dentropy, dx, dw, stream)
        if lse is None and entropy is None:
            self._outputs(n, stats=True)
            _, h, z = self._stats
        elif lse is None or (entropy is None and dentropy is not None):
            raise ValueError("lse and entropy (where dentropy is there) come together, from the same forward()")
        else:
            z = _take("lse", lse, (n,), torch.float32, self.device)
            h = _take("entropy", entropy, (n,), torch.float32, self.device) if entropy is not None else 0
        self._call(stream, binding.head_grad, desc, *inputs, z, h, *weights, *grads, accumulate, self.ws.data_ptr(), self.ws.numel())

    def loss(self, x, weight, targets, dlogp, dentropy, dx, dw, accumulate=False, stream=None):
        """forward() and backward() in one, for weights that do not depend on the result."""
        desc, n, inputs = self._inputs(x, weight, targets)
        weights, grads, _held = self._gradients(n, x, dlogp, dentropy, dx, dw, stream)
        self._outputs(n)
        self._call(stream, binding.head_loss, desc, *inputs, *weights, *self._stats, *grads, accumulate, self.ws.data_ptr(),
                   self.ws.numel())

    def device_status(self, stream=None):
        """ASI_OK, or ASI_ERR_TIMEOUT where a bounded wait of the last call expired.  Synchronises."""
        handle = _raw_stream(self.device.index) if stream is None else stream.cuda_stream
        return binding.head_status(self.ws.data_ptr(), handle)
