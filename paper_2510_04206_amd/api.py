"""Convenience layer over the C ABI: allocates outputs/workspace with torch, then calls it."""
from __future__ import annotations

from typing import Optional

import torch

from . import _binding as B

_CODES = {torch.bfloat16: B.AGRL_BF16, torch.float32: B.AGRL_F32}


def _need(t: torch.Tensor, name: str, shape, dtypes) -> None:
    """The binding sees only addresses: what a tensor must be is checked here."""
    if t.shape != shape:
        raise ValueError(f"agrl: {name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype not in dtypes:
        raise TypeError(f"agrl: {name} has dtype {t.dtype}, expected one of {dtypes}")


def _row_stride(t: torch.Tensor) -> int:
    """Elements between rows (a single row has no neighbour: its own length)."""
    return t.stride(-2) if t.shape[-2] > 1 else max(t.shape[-1], 1)


def _capturing(stream) -> bool:
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Owned:
    """Buffers of a handle, its device and the order of its calls.  They share the workspace and the
    outputs, so a call on another stream than the last one's first waits for all that stream was
    given, and the allocator is told of the use.  Calls under capture wait for nothing outside it:
    whoever captures has synchronised before, and orders the replays and the handle's other calls.
    The work goes to the handle's device, whichever is current."""

    def __init__(self, device):
        self._last = torch.cuda.current_stream(torch.device(device))
        self._index = self._last.device_index
        self.device = torch.device("cuda", self._index)
        self._raw = self._last.cuda_stream
        self._told = {self._raw}
        self._buffers = ()

    def _keep(self, *buffers):
        self._buffers = tuple(b for b in buffers if b is not None)

    def _need(self, t, name, shape, dtypes):
        if t.shape != shape or t.dtype not in dtypes:
            _need(t, name, shape, dtypes)
        if t.device != self.device:          # (looked at here first: a call costs a small norm 0.1 us)
            self._same_device(t, name)

    def _same_device(self, t, name):
        if t.device != self.device:
            raise ValueError(f"agrl: {name} is on {t.device}, the handle on {self.device}")

    def _there(self, call, *args):
        with torch.cuda.device(self._index):
            return call(*args)

    def _order(self, stream):
        """Puts a call on `stream` (None: the current one) behind the handle's last one.  Returns the
        stream, or None if the handle's device is not the current one."""
        if torch.cuda.current_device() != self._index:
            return None
        if stream is None:
            raw = torch._C._cuda_getCurrentRawStream(self._index)
        else:
            raw = stream.cuda_stream
            if stream.device_index != self._index:
                raise ValueError(f"agrl: the stream is {stream.device}'s, the handle on {self.device}")
        if raw == self._raw:
            return self._last
        use = stream if stream is not None else torch.cuda.current_stream(self.device)
        if _capturing(use):
            return use
        if _capturing(self._last):
            raise RuntimeError("agrl: the stream of this handle's last call is being captured")
        use.wait_stream(self._last)
        if raw not in self._told:
            for b in self._buffers:
                b.record_stream(use)
            self._told.add(raw)
        self._last, self._raw = use, raw
        return use


def task_adv_norm(traj_id: torch.Tensor, action_mask: torch.Tensor, traj_task: torch.Tensor,
                  traj_group: Optional[torch.Tensor], reward: torch.Tensor, n_task: int,
                  n_group: int = 0, opt=None, with_tokens: bool = True, stream=None,
                  member_ranges: bool = True) -> dict:
    """agrl_task_adv_norm on device tensors; returns the outputs as a dict.

    member_ranges: pass a scratch array as agrl_options.adv_ranges (unless the
    options already name one), so that each group's and task's wave scans only
    its members' index span; the results are bit-identical without it."""
    dev = traj_id.device
    T_g, n_traj = traj_id.numel(), traj_task.numel()
    if member_ranges:
        o = B.agrl_options(**opt) if isinstance(opt, dict) else (opt or B.agrl_options())
        if not o.adv_ranges:
            n_seg = (n_group if traj_group is not None else 0) + n_task
            scratch = torch.empty(max(2 * n_seg, 1), dtype=torch.int32, device=dev)
            o.adv_ranges = scratch.data_ptr()
        opt = o
    out = dict(act_count=torch.empty(n_traj, dtype=torch.int32, device=dev),
               task_count=torch.empty(n_task, dtype=torch.int64, device=dev),
               task_mean=torch.empty(n_task, dtype=torch.float32, device=dev),
               task_std=torch.empty(n_task, dtype=torch.float32, device=dev),
               adv_traj=torch.empty(n_traj, dtype=torch.float32, device=dev),
               adv_tok=torch.empty(T_g, dtype=torch.float32, device=dev) if with_tokens else None)
    if member_ranges and "scratch" in locals():
        out["member_ranges"] = scratch     # kept alive with the outputs
    B.agrl_task_adv_norm(T_g, n_traj, n_task, n_group, traj_id, action_mask, traj_task,
                         traj_group, reward, opt, out["act_count"], out["task_count"],
                         out["task_mean"], out["task_std"], out["adv_traj"], out["adv_tok"],
                         stream)
    return out


def sequence_mean_weights(traj_id: torch.Tensor, action_mask: torch.Tensor, n_traj: int,
                          stream=None):
    """agrl_sequence_mean_weights: (seq_count [n_traj] int32, token_weight [T] fp32), the
    per-token weights of the sequence-level aggregation (pass token_weight's pointer as
    agrl_options.token_weight)."""
    dev = traj_id.device
    seq_count = torch.empty(n_traj, dtype=torch.int32, device=dev)
    token_weight = torch.empty(traj_id.numel(), dtype=torch.float32, device=dev)
    B.agrl_sequence_mean_weights(traj_id.numel(), n_traj, traj_id, action_mask, seq_count,
                                 token_weight, stream)
    return seq_count, token_weight


class PolicyLoss:
    """Forward/backward of the fused policy loss for one micro-batch shape.

    Holds the workspace (sized for T tokens with at most max_act action
    tokens) and the output buffers, so repeated steps allocate nothing.
    """

    def __init__(self, T: int, d: int, V: int, dtype: torch.dtype, max_act: int = 0,
                 eps_low: float = 0.2, eps_high: float = 0.2, n_norm: int = 0, opt=None,
                 device="cuda"):
        self.T, self.d, self.V, self.max_act = int(T), int(d), int(V), int(max_act)
        self.code = B.AGRL_BF16 if dtype == torch.bfloat16 else B.AGRL_F32
        self.eps_low, self.eps_high, self.n_norm = float(eps_low), float(eps_high), int(n_norm)
        self.opt = B.agrl_options(**opt) if isinstance(opt, dict) else opt
        self.ws_bytes = B.agrl_policy_loss_workspace_size(self.T, self.max_act, self.d, self.V,
                                                          self.code, self.opt)
        # vocabulary columns per backward chunk (the last chunk holds the rest)
        self.vocab_chunk = B.agrl_policy_loss_vocab_chunk(self.T, self.max_act, self.d, self.V,
                                                          self.code, self.opt)
        dev = torch.device(device)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)
        self.logp = torch.empty(self.T, dtype=torch.float32, device=dev)
        self.lse = torch.empty(self.T, dtype=torch.float32, device=dev)
        self.n_clip = torch.empty(2, dtype=torch.int64, device=dev)
        self.dH = torch.empty((self.T, self.d), dtype=torch.float32, device=dev)
        self.dW = torch.empty((self.V, self.d), dtype=torch.float32, device=dev)

    def forward(self, H, W, token_id, action_mask, adv_tok, old_logp, stream=None):
        B.agrl_policy_loss_fwd(self.T, self.max_act, self.d, self.V, self.code, H, W, token_id,
                               action_mask, adv_tok, old_logp, self.eps_low, self.eps_high,
                               self.n_norm, self.opt, self.workspace, self.ws_bytes, self.loss,
                               self.logp, self.lse, self.n_clip, stream)
        return self.loss, self.logp, self.lse, self.n_clip

    def backward(self, H, W, token_id, action_mask, adv_tok, old_logp, grad_loss: float = 1.0,
                 stream=None):
        B.agrl_policy_loss_bwd(self.T, self.max_act, self.d, self.V, self.code, H, W, token_id,
                               action_mask, adv_tok, old_logp, self.eps_low, self.eps_high,
                               self.n_norm, self.opt, self.lse, self.logp, float(grad_loss),
                               self.workspace, self.ws_bytes, self.dH, self.dW, stream)
        return self.dH, self.dW


class TokenLogprob:
    """Forward-only token log-probabilities for one packed-batch shape.

    Holds its workspace and outputs; ``__call__`` returns (logp, lse), fp32 [T],
    zero on observation tokens.
    """

    def __init__(self, T: int, d: int, V: int, dtype: torch.dtype, max_act: int = 0, opt=None,
                 device="cuda"):
        self.T, self.d, self.V, self.max_act = int(T), int(d), int(V), int(max_act)
        self.code = B.AGRL_BF16 if dtype == torch.bfloat16 else B.AGRL_F32
        self.opt = B.agrl_options(**opt) if isinstance(opt, dict) else opt
        self.ws_bytes = B.agrl_token_logprob_workspace_size(self.T, self.max_act, self.d, self.V,
                                                            self.code, self.opt)
        dev = torch.device(device)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)
        self.logp = torch.empty(self.T, dtype=torch.float32, device=dev)
        self.lse = torch.empty(self.T, dtype=torch.float32, device=dev)

    def __call__(self, H, W, token_id, action_mask, stream=None):
        B.agrl_token_logprob(self.T, self.max_act, self.d, self.V, self.code, H, W, token_id,
                             action_mask, self.opt, self.workspace, self.ws_bytes, self.logp,
                             self.lse, stream)
        return self.logp, self.lse


class TokenNorm(_Owned):
    """Layer or RMS norm of T token rows of d, forward and backward (agrl_token_norm_*).

    Holds its outputs and the workspace, so repeated steps allocate nothing.  ``forward``
    returns (y, mean, rstd), mean None for kind "rms"; ``backward`` reads the mean and rstd of
    the last forward and returns (dx, dweight, dbias), dbias None for kind "rms" unless
    ``bias_grad``.  Rows of x and dy may lie further apart than their length.  grads=False
    leaves the backward's buffers out.
    """

    def __init__(self, T: int, d: int, dtype: torch.dtype, kind: str = "layer", eps: float = 1e-5,
                 grads: bool = True, bias_grad: Optional[bool] = None, device="cuda"):
        super().__init__(device)
        if kind not in ("layer", "rms"):
            raise ValueError("agrl: kind is 'layer' or 'rms'")
        if dtype not in _CODES:
            raise TypeError(f"unsupported dtype {dtype}")
        self.T, self.d, self.dtype, self.eps = int(T), int(d), dtype, float(eps)
        self.kind = B.AGRL_NORM_LAYER if kind == "layer" else B.AGRL_NORM_RMS
        new = lambda *n, dt=torch.float32: torch.empty(n, dtype=dt, device=self.device)  # noqa: E731
        self.y = new(self.T, self.d, dt=dtype)
        self.mean = new(self.T) if kind == "layer" else None
        self.rstd = new(self.T)
        self.dx = self.dweight = self.dbias = self.workspace = None
        self.ws_bytes = 0
        if grads:
            self.ws_bytes = B.agrl_token_norm_bwd_workspace_size(self.T, self.d)
            self.workspace = new(max(self.ws_bytes, 4), dt=torch.uint8)
            self.dx = new(self.T, self.d, dt=dtype)
            self.dweight = new(self.d)
            if bias_grad or (bias_grad is None and kind == "layer"):
                self.dbias = new(self.d)
        self._keep(self.y, self.mean, self.rstd, self.workspace, self.dx, self.dweight, self.dbias)

    def _check(self, x, weight, action_mask):
        self._need(x, "x", (self.T, self.d), (self.dtype,))
        if weight is not None:
            self._need(weight, "weight", (self.d,), _CODES)
        if action_mask is not None:
            self._need(action_mask, "action_mask", (self.T,), (torch.uint8,))

    def forward(self, x, weight=None, bias=None, action_mask=None, stream=None):
        self._check(x, weight, action_mask)
        par = weight if weight is not None else bias
        if bias is not None:
            self._need(bias, "bias", (self.d,), (par.dtype,))
        on = self._order(stream)
        if on is None:
            return self._there(self.forward, x, weight, bias, action_mask, stream)
        B.agrl_token_norm_fwd(self.T, self.d, self.kind, _CODES[self.dtype],
                              B.AGRL_F32 if par is None else _CODES[par.dtype], x, _row_stride(x),
                              weight, bias, action_mask, self.eps, self.y, self.d, self.mean,
                              self.rstd, on)
        return self.y, self.mean, self.rstd

    def backward(self, x, weight, dy, action_mask=None, accumulate: bool = False, stream=None):
        if self.dx is None:
            raise ValueError("agrl: this TokenNorm was made with grads=False")
        self._check(x, weight, action_mask)
        self._need(dy, "dy", (self.T, self.d), _CODES)
        on = self._order(stream)
        if on is None:
            return self._there(self.backward, x, weight, dy, action_mask, accumulate, stream)
        B.agrl_token_norm_bwd(self.T, self.d, self.kind, _CODES[self.dtype],
                              B.AGRL_F32 if weight is None else _CODES[weight.dtype],
                              _CODES[dy.dtype], x, _row_stride(x), weight, action_mask, dy,
                              _row_stride(dy), self.mean, self.rstd, int(accumulate),
                              self.workspace, self.ws_bytes, self.dx, self.d, self.dweight,
                              self.dbias, on)
        return self.dx, self.dweight, self.dbias


class _Stack(_Owned):
    """What Orthogonalize and MuonStep share: a stack of matrices' shape, options and workspace."""

    def __init__(self, m, n, code_of, batch, steps, coeffs, eps, device):
        super().__init__(device)
        if code_of not in _CODES:
            raise TypeError(f"unsupported dtype {code_of}")
        if steps < 1:
            raise ValueError("agrl: steps is at least 1")
        self.m, self.n = int(m), int(n)
        self.batch = None if batch is None else int(batch)
        self.shape = (self.m, self.n) if batch is None else (self.batch, self.m, self.n)
        self.count = 1 if batch is None else self.batch
        self.dtype, self.code = code_of, _CODES[code_of]
        a, b, c = (0.0, 0.0, 0.0) if coeffs is None else coeffs
        self.ns = B.agrl_ns_options(steps=int(steps), a=a, b=b, c=c, eps=eps)
        self.ws_bytes = B.agrl_orthogonalize_workspace_size(self.count, self.m, self.n, self.code)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.device)
        self._keep(self.workspace)

    @staticmethod
    def _strides(t):
        return _row_stride(t), (t.stride(0) if t.dim() == 3 else 0)


class Orthogonalize(_Stack):
    """Newton-Schulz orthogonalisation of [m, n] matrices (agrl_orthogonalize), a stack of them
    with ``batch``.  Holds the workspace and the output.  ``__call__`` takes fp32 or bf16 and
    returns the output.  The result's type sets the products' precision: fp32 as fp32 products;
    bf16, of more than 128 rows and columns, operands of 11 bits, which leave up to 2e-3 of the
    result's norm, a few times more where entries repeat (include/agrl.h).  coeffs of three zeros and
    eps=0 select the defaults."""

    def __init__(self, m: int, n: int, out_dtype: torch.dtype = torch.bfloat16,
                 batch: Optional[int] = None, steps: int = 5, coeffs=None, eps: float = 1e-7,
                 device="cuda"):
        super().__init__(m, n, out_dtype, batch, steps, coeffs, eps, device)
        self.out = torch.empty(self.shape, dtype=out_dtype, device=self.device)
        self._keep(self.workspace, self.out)

    def __call__(self, g, stream=None):
        self._need(g, "g", self.shape, _CODES)
        on = self._order(stream)
        if on is None:
            return self._there(self, g, stream)
        B.agrl_orthogonalize(self.count, self.m, self.n, _CODES[g.dtype], g, *self._strides(g),
                             self.code, self.ns, self.workspace, self.ws_bytes, self.out, self.n,
                             self.m * self.n, on)
        return self.out


class MuonStep(_Stack):
    """One step of the orthogonalised-momentum optimiser for [m, n] weights, or a stack of them
    (agrl_muon_step).  Holds the workspace; the caller holds the weight and the fp32 momentum,
    which ``__call__`` updates in place.  The weight's type sets the products' precision, as the
    result's does for Orthogonalize.  scale=0 selects sqrt(max(1, m / n))."""

    def __init__(self, m: int, n: int, param_dtype: torch.dtype = torch.float32,
                 batch: Optional[int] = None, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, scale: float = 0.0, steps: int = 5, coeffs=None,
                 eps: float = 1e-7, device="cuda"):
        super().__init__(m, n, param_dtype, batch, steps, coeffs, eps, device)
        self.mu, self.nesterov = float(momentum), int(bool(nesterov))
        self.weight_decay, self.scale = float(weight_decay), float(scale)

    def __call__(self, param, grad, momentum, lr: float, stream=None):
        self._need(param, "param", self.shape, (self.dtype,))
        self._need(grad, "grad", self.shape, _CODES)
        self._need(momentum, "momentum", self.shape, (torch.float32,))
        on = self._order(stream)
        if on is None:
            return self._there(self, param, grad, momentum, lr, stream)
        B.agrl_muon_step(self.count, self.m, self.n, _CODES[grad.dtype], grad, *self._strides(grad),
                         self.code, param, *self._strides(param), momentum, float(lr), self.mu,
                         self.nesterov, self.weight_decay, self.scale, self.ns, self.workspace,
                         self.ws_bytes, on)
        return param


class TokenEmbedding(_Owned):
    """Embedding of T packed token ids, rows of a [V, d] weight (agrl_token_embed_*).

    ``forward`` returns y [T, d] = scale weight[token_id], in ``dtype`` whatever the weight's type (w_dtype,
    by default the same).  ``backward`` adds up dy's rows by id, in a fixed order, into ``dweight`` [V, d]
    fp32: its own, or the one given (a tied head's: ``dweight=loss.dW`` and accumulate=True).  Tokens whose
    live_mask is 0 are not read: y is +0 there, dy goes nowhere.  grads=False leaves the backward out.
    """

    def __init__(self, T: int, V: int, d: int, dtype: torch.dtype, w_dtype: Optional[torch.dtype] = None,
                 scale: float = 1.0, grads: bool = True, dweight: Optional[torch.Tensor] = None,
                 device="cuda"):
        super().__init__(device)
        self.w_dtype = dtype if w_dtype is None else w_dtype
        for t in (dtype, self.w_dtype):
            if t not in _CODES:
                raise TypeError(f"unsupported dtype {t}")
        self.T, self.V, self.d, self.dtype, self.scale = int(T), int(V), int(d), dtype, float(scale)
        self.y = torch.empty((self.T, self.d), dtype=dtype, device=self.device)
        self.dweight = self.workspace = None
        self.ws_bytes = 0
        if grads:
            self.ws_bytes = B.agrl_token_embed_bwd_workspace_size(self.T, self.d, self.V)
            self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.device)
            if dweight is not None:
                self._need(dweight, "dweight", (self.V, self.d), (torch.float32,))
            self.dweight = dweight if dweight is not None else torch.empty(
                (self.V, self.d), dtype=torch.float32, device=self.device)
        self._keep(self.y, self.workspace, self.dweight)

    def _check(self, token_id, live_mask):
        self._need(token_id, "token_id", (self.T,), (torch.int32,))
        if live_mask is not None:
            self._need(live_mask, "live_mask", (self.T,), (torch.uint8,))

    def forward(self, weight, token_id, live_mask=None, stream=None):
        self._need(weight, "weight", (self.V, self.d), (self.w_dtype,))
        self._check(token_id, live_mask)
        on = self._order(stream)
        if on is None:
            return self._there(self.forward, weight, token_id, live_mask, stream)
        B.agrl_token_embed_fwd(self.T, self.d, self.V, _CODES[self.w_dtype], _CODES[self.dtype], weight,
                               token_id, live_mask, self.scale, self.y, self.d, on)
        return self.y

    def backward(self, token_id, dy, live_mask=None, accumulate: bool = False, stream=None):
        if self.dweight is None:
            raise ValueError("agrl: this TokenEmbedding was made with grads=False")
        self._check(token_id, live_mask)
        self._need(dy, "dy", (self.T, self.d), _CODES)
        on = self._order(stream)
        if on is None:
            return self._there(self.backward, token_id, dy, live_mask, accumulate, stream)
        B.agrl_token_embed_bwd(self.T, self.d, self.V, _CODES[dy.dtype], token_id, live_mask, dy,
                               _row_stride(dy), self.scale, int(accumulate), self.workspace,
                               self.ws_bytes, self.dweight, on)
        return self.dweight


class TokenRotation(_Owned):
    """Rotation of [T, n_head, d] heads by their tokens' positions (agrl_rotate_heads): the first ``rot``
    elements (all by default) in pairs, half a rotated part apart or neighbours (``interleaved``).

    ``__call__`` returns the handle's output, or ``out`` (x itself rotates in place; a view of a fused
    projection's heads does).  position [T] int32; None: the row's number.  inverse=True turns
    back: the gradient of the rotation.
    """

    def __init__(self, T: int, n_head: int, d: int, dtype: torch.dtype, rot: Optional[int] = None,
                 base: float = 10000.0, interleaved: bool = False, output: bool = True, device="cuda"):
        super().__init__(device)
        if dtype not in _CODES:
            raise TypeError(f"unsupported dtype {dtype}")
        self.T, self.n_head, self.d, self.dtype = int(T), int(n_head), int(d), dtype
        self.shape = (self.T, self.n_head, self.d)
        self.rot, self.base = self.d if rot is None else int(rot), float(base)
        self.interleaved = int(bool(interleaved))
        self.out = torch.empty(self.shape, dtype=dtype, device=self.device) if output else None
        self._keep(self.out)

    def __call__(self, x, position=None, inverse: bool = False, out=None, stream=None):
        self._need(x, "x", self.shape, (self.dtype,))
        if position is not None:
            self._need(position, "position", (self.T,), (torch.int32,))
        if out is None:
            if self.out is None:
                raise ValueError("agrl: this TokenRotation was made with output=False: name out")
            out = self.out
        else:
            self._need(out, "out", self.shape, (self.dtype,))
        on = self._order(stream)
        if on is None:
            return self._there(self, x, position, inverse, out, stream)
        B.agrl_rotate_heads(self.T, self.n_head, self.d, self.rot, _CODES[self.dtype], x, position,
                            self.base, self.interleaved, int(bool(inverse)), out, on)
        return out


class PackedAttention(_Owned):
    """Causal attention within each sequence of a packed stream of T tokens, n_head query heads over n_kv
    key heads (agrl_attention_*).

    ``forward(q, k, v, seq_start)`` returns (o [T, n_head, d], lse [n_head, T] fp32); ``backward(q, k, v,
    seq_start, do)`` reads the o and lse of the last forward, or those given (copies that a program keeps of an earlier
    one, so that layers can share a handle), and returns (dq, dk, dv), three views of
    ``dqkv`` [T, n_head + 2 n_kv, d], the gradient of a fused projection's output.  seq_start
    [n_seq + 1] int32: sequence i is the tokens seq_start[i] .. seq_start[i + 1] - 1; the values of tokens outside
    do not matter, and they get +0.  q, k and v may be views with any strides of rows and heads.
    scale=None: 1 / sqrt(d).  grads=False leaves the backward out.
    """

    def __init__(self, T: int, n_head: int, n_kv: int, d: int, dtype: torch.dtype,
                 scale: Optional[float] = None, grads: bool = True, device="cuda"):
        super().__init__(device)
        if dtype not in _CODES:
            raise TypeError(f"unsupported dtype {dtype}")
        self.T, self.n_head, self.n_kv, self.d, self.dtype = int(T), int(n_head), int(n_kv), int(d), dtype
        self.scale = self.d ** -0.5 if scale is None else float(scale)
        new = lambda *n, dt=torch.float32: torch.empty(n, dtype=dt, device=self.device)  # noqa: E731
        self.o = new(self.T, self.n_head, self.d, dt=dtype)
        self.lse = new(self.n_head, self.T)
        self.dqkv = self.dq = self.dk = self.dv = self.workspace = None
        self.ws_bytes = 0
        if grads:
            self.ws_bytes = B.agrl_attention_bwd_workspace_size(self.T, self.n_head, self.n_kv, self.d,
                                                                _CODES[dtype])
            self.workspace = new(max(self.ws_bytes, 1), dt=torch.uint8)
            self.dqkv = new(self.T, self.n_head + 2 * self.n_kv, self.d, dt=dtype)
            self.dq, self.dk, self.dv = self.dqkv.split((self.n_head, self.n_kv, self.n_kv), 1)
        self._keep(self.o, self.lse, self.workspace, self.dqkv)

    def _check(self, q, k, v, seq_start):
        self._need(q, "q", (self.T, self.n_head, self.d), (self.dtype,))
        self._need(k, "k", (self.T, self.n_kv, self.d), (self.dtype,))
        self._need(v, "v", (self.T, self.n_kv, self.d), (self.dtype,))
        self._need(seq_start, "seq_start", (max(seq_start.numel(), 1),), (torch.int32,))

    def forward(self, q, k, v, seq_start, stream=None):
        self._check(q, k, v, seq_start)
        on = self._order(stream)
        if on is None:
            return self._there(self.forward, q, k, v, seq_start, stream)
        B.agrl_attention_fwd(self.T, seq_start.numel() - 1, self.n_head, self.n_kv, self.d,
                             _CODES[self.dtype], q, k, v, seq_start, self.scale, self.o, self.lse, on)
        return self.o, self.lse

    def backward(self, q, k, v, seq_start, do, stream=None, o=None, lse=None):
        if self.dqkv is None:
            raise ValueError("agrl: this PackedAttention was made with grads=False")
        if (o is None) != (lse is None):
            raise ValueError("agrl: o and lse of one forward belong together")
        self._check(q, k, v, seq_start)
        self._need(do, "do", (self.T, self.n_head, self.d), (self.dtype,))
        if o is not None:
            self._need(o, "o", (self.T, self.n_head, self.d), (self.dtype,))
            self._need(lse, "lse", (self.n_head, self.T), (torch.float32,))
        on = self._order(stream)
        if on is None:
            return self._there(self.backward, q, k, v, seq_start, do, stream, o, lse)
        if o is None:
            o, lse = self.o, self.lse
        B.agrl_attention_bwd(self.T, seq_start.numel() - 1, self.n_head, self.n_kv, self.d,
                             _CODES[self.dtype], q, k, v, seq_start, self.scale, o, lse, do,
                             self.workspace, self.ws_bytes, self.dq, self.dk, self.dv, on)
        return self.dq, self.dk, self.dv
