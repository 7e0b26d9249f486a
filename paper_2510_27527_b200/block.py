"""What stands around the NVFP4 linears of a block, as torch modules: `NVFP4LayerNorm` (layer norm over the last dimension), `swiglu`, `NVFP4MLP`
(layer norm, gate and up projections, SwiGLU, down projection) and, for answering token by token, `NVFP4FrozenLinear` / `NVFP4FrozenMLP`, whose
weights are quantized once. For backward the norm and SwiGLU keep their inputs in 8 bits (1.03 bytes an element instead of 2): gradients are then
those at the rounded inputs. With checkpoint=False they keep the inputs themselves. The linears keep their FP4 operands. Argument marshalling only:
every step runs in the library's kernels.
"""
from __future__ import annotations

import dataclasses

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .module import NVFP4Linear, _needs_function, _wants_grad


def _rows(x: torch.Tensor, features: int, where: str) -> torch.Tensor:
    """x as a matrix of rows on 16-byte boundaries, a copy where it is not."""
    if x.dim() == 0 or x.shape[-1] != features:
        raise RuntimeError(f"{where}: input of shape {tuple(x.shape)} for {features} features")
    m = x if x.dim() == 2 else x.reshape(-1, features)
    size = m.element_size()
    if (m.stride(1) == 1 or features == 1) and (m.shape[0] <= 1 or m.stride(0) * size % 16 == 0 and m.stride(0) >= features) and m.data_ptr() % 16 == 0:
        return m
    out = torch.empty((m.shape[0], (features * size + 15) // 16 * 16 // size), dtype=m.dtype, device=m.device)[:, :features]
    return out.copy_(m)


def _bf16(x: torch.Tensor) -> torch.Tensor:
    return x if x.dtype == torch.bfloat16 else x.to(torch.bfloat16)


def _save(ctx, checkpoint: bool) -> int:
    """What a call keeps. (Nothing where it goes through its function for a trace alone.)"""
    return (B.SAVE_CKPT8 if checkpoint else B.SAVE_INPUT) if True in ctx.needs_input_grad else B.SAVE_NOTHING


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, eps, checkpoint):
        y, s = B.nvfp4_layernorm_fwd(x, gamma, beta, eps, _save(ctx, checkpoint))
        if s is not None:
            ctx.save_for_backward(gamma, s.stats, x if s.x8 is None else s.x8.buf)
            ctx.saved = (int(s.T), int(s.D), s.x_dtype, s.has_beta, checkpoint)  # (under jit.trace sizes are tensors)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        gamma, stats, x = ctx.saved_tensors
        T, D, x_dtype, has_beta, checkpoint = ctx.saved
        kept = dict(x8=B.Ckpt8(x, T, D)) if checkpoint else dict(X=_rows(x, D, "NVFP4LayerNorm"))  # (a hook may have given it other strides)
        dx, dgamma, dbeta = B.nvfp4_layernorm_bwd(_rows(_bf16(dy), D, "NVFP4LayerNorm"), B.LayerNormSaved(T, D, x_dtype, stats, gamma, has_beta, **kept))
        return dx, dgamma, dbeta, None, None


class _SwigluFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, u, checkpoint):
        h, s = B.nvfp4_swiglu_fwd(g, u, _save(ctx, checkpoint))
        if s is not None:
            ctx.save_for_backward(*((g, u) if s.g8 is None else (s.g8.buf, s.u8.buf)))
            ctx.saved = (int(s.T), int(s.D), checkpoint)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        (a, b), (T, D, checkpoint) = ctx.saved_tensors, ctx.saved
        s = B.SwigluSaved(T, D, g8=B.Ckpt8(a, T, D), u8=B.Ckpt8(b, T, D)) if checkpoint else B.SwigluSaved(T, D, _rows(a, D, "swiglu"), _rows(b, D, "swiglu"))
        return *B.nvfp4_swiglu_bwd(_rows(_bf16(dh), D, "swiglu"), s), None


def _gemv(x, codes, scales, global_scales, outlier_cols, keep_cols, outlier_weight, bias, form):
    N, K, gs_mode, dev_status = form
    W = B.Operand(codes, scales, global_scales, N, K, gs_mode, B.SF_TILED128x4)
    return B.nvfp4_gemv(x, W, B.DT_BF16, bias, None if outlier_cols is None else (outlier_cols, keep_cols), outlier_weight, None, dev_status)


class _FrozenFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, *args):
        return _gemv(*args)

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("NVFP4FrozenLinear has no gradient")


def _layer_norm_call(x, gamma, beta, eps, checkpoint):
    if _needs_function(x, gamma, beta):
        return _LayerNormFn.apply(x, gamma, beta, eps, checkpoint)
    return B.nvfp4_layernorm_fwd(x, gamma, beta, eps, B.SAVE_NOTHING)[0]


def _swiglu_call(g, u, checkpoint):
    if _needs_function(g, u):
        return _SwigluFn.apply(g, u, checkpoint)
    return B.nvfp4_swiglu_fwd(g, u, B.SAVE_NOTHING)[0]


# (a compiler would not see what the library writes)
_layer_norm, _swiglu = torch.compiler.disable(_layer_norm_call), torch.compiler.disable(_swiglu_call)


def swiglu(g: torch.Tensor, u: torch.Tensor, checkpoint: bool = True) -> torch.Tensor:
    """silu(g) * u of two BF16 tensors of the same shape, with gradients. `checkpoint`: they are those at g and u rounded to 8 bits."""
    if g.shape != u.shape or g.dtype != torch.bfloat16 or u.dtype != torch.bfloat16:
        raise RuntimeError(f"swiglu: {g.dtype} {tuple(g.shape)} and {u.dtype} {tuple(u.shape)}, not two BF16 tensors of one shape")
    D = g.shape[-1] if g.dim() else 0
    h = _swiglu(_rows(g, D, "swiglu"), _rows(u, D, "swiglu"), checkpoint)
    return h if g.dim() == 2 else h.reshape(g.shape)


class NVFP4LayerNorm(torch.nn.Module):
    """Layer norm over the last dimension with nn.LayerNorm's parameters, BF16 or FP32 in, BF16 out; the parameters' sums and the statistics are FP32.
    `checkpoint`: gradients are those at the input rounded to 8 bits."""

    def __init__(self, features: int, eps: float = 1e-5, bias: bool = True, checkpoint: bool = True, dtype: torch.dtype = torch.bfloat16, device="cuda"):
        super().__init__()
        self.features, self.eps, self.checkpoint = features, eps, checkpoint
        self.weight = torch.nn.Parameter(torch.ones(features, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(features, dtype=dtype, device=device)) if bias else None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.dtype not in (torch.bfloat16, torch.float32):
            raise RuntimeError(f"NVFP4LayerNorm: input of type {x.dtype}, not BF16 or FP32")
        y = _layer_norm(_rows(x, self.features, "NVFP4LayerNorm"), self.weight, self.bias, self.eps, self.checkpoint)
        return y if x.dim() == 2 else y.reshape(x.shape)


class _Frozen(torch.nn.Module):
    """A module whose buffers keep the types they were frozen in: a model's change of type is not for them, one of device is."""

    def _apply(self, fn, recurse=True):
        before = {n: b for n, b in self._buffers.items() if b is not None}
        super()._apply(fn, recurse)
        for n, b in before.items():
            if self._buffers[n].dtype != b.dtype:
                self._buffers[n] = b.to(self._buffers[n].device)
        return self


class NVFP4FrozenLinear(_Frozen):
    """y = x W-hat^T (+ bias) with the weights as NVFP4Linear's forward quantizes them (OutControl's outlier channels in high precision) and x in
    BF16: for answering, a few tokens at a time (every 32 are a pass over the weights; a prompt goes faster through the layer itself, with x in FP4).
    No gradients. A wait that runs out is reported in the layer's cfg.dev_status, as in training."""

    dev_status = None
    _names = ("codes", "scales", "global_scales", "outlier_cols", "keep_cols", "outlier_weight", "bias")

    def __init__(self, layer: NVFP4Linear):
        super().__init__()
        self.in_features, self.out_features = layer.in_features, layer.out_features
        if not layer.weight.is_cuda or layer.weight.dtype != torch.bfloat16:
            raise RuntimeError(f"NVFP4FrozenLinear: weights of {layer.weight.dtype} on {layer.weight.device}, not BF16 on a CUDA device")
        cfg = dataclasses.replace(layer.cfg, y_dtype=B.DT_BF16)
        self.gs_mode, self.n_out, self.dev_status = cfg.gs_mode, cfg.n_out, cfg.dev_status
        with torch.no_grad(), torch.cuda.device(layer.weight.device):  # the call that quantizes the weights in training, on one token
            _, saved = B.nvfp4_linear_fwd(torch.ones((1, self.in_features), dtype=torch.bfloat16, device=layer.weight.device), layer.weight.detach(), cfg)
            index = saved.index if self.n_out else (None, None)
            for name, t in (("codes", saved.qw.codes), ("scales", saved.qw.sf), ("global_scales", saved.qw.gscale), ("outlier_cols", index[0]), ("keep_cols", index[1]),
                            ("outlier_weight", saved.W_out), ("bias", None if layer.bias is None else layer.bias.detach())):
                self.register_buffer(name, None if t is None else t.clone())

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if _wants_grad(x):
            raise RuntimeError("NVFP4FrozenLinear has no gradient: use it under torch.no_grad()")
        rows = _rows(_bf16(x), self.in_features, "NVFP4FrozenLinear")
        h = self._buffers  # (a module's own look-up is slower: 2 us for the seven)
        if len(h) != len(self._names):  # (one is parametrized)
            h = {n: getattr(self, n) for n in self._names}
        args = (rows, h["codes"], h["scales"], h["global_scales"], h["outlier_cols"], h["keep_cols"], h["outlier_weight"], h["bias"],
                (self.out_features, self.in_features - self.n_out, self.gs_mode, self.dev_status))
        y = _FrozenFn.apply(*args) if _needs_function(rows, args[3], args[6], args[7]) else _gemv(*args)
        return y if x.dim() == 2 else y.reshape(*x.shape[:-1], self.out_features)


class NVFP4MLP(torch.nn.Module):
    """down(silu(gate(n)) * up(n)), n = norm(x): the MLP of a block with layer norm in front and NVFP4 linears (the caller adds the residual). Blocks with
    another norm take the parts: `swiglu` between three `NVFP4Linear`. `cfg` configures the gate and up projections, `down_cfg` the down projection
    (default: cfg without its outlier channels, which are channels of x)."""

    def __init__(self, hidden: int, ffn: int, cfg: B.LayerConfig | None = None, down_cfg: B.LayerConfig | None = None, checkpoint: bool = True, eps: float = 1e-5,
                 norm_bias: bool = True, norm_dtype: torch.dtype = torch.bfloat16, device="cuda"):
        super().__init__()
        self.checkpoint = checkpoint
        if down_cfg is None and cfg is not None:
            down_cfg = dataclasses.replace(cfg, outliers=None) if cfg.n_out else cfg
        self.norm = NVFP4LayerNorm(hidden, eps, norm_bias, checkpoint, norm_dtype, device)
        self.gate = NVFP4Linear(hidden, ffn, cfg=cfg, device=device)
        self.up = NVFP4Linear(hidden, ffn, cfg=cfg, device=device)
        self.down = NVFP4Linear(ffn, hidden, cfg=down_cfg, device=device)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        n = self.norm(x)
        return self.down(swiglu(self.gate(n), self.up(n), self.checkpoint))

    def frozen(self) -> "NVFP4FrozenMLP":
        """The same MLP for answering, its weights quantized now."""
        return NVFP4FrozenMLP(self)


class NVFP4FrozenMLP(_Frozen):
    """NVFP4MLP for a few tokens at a time: its weights quantized once, activations in BF16. No gradients."""

    def __init__(self, mlp: NVFP4MLP):
        super().__init__()
        self.features, self.eps = mlp.norm.features, mlp.norm.eps
        self.register_buffer("norm_weight", mlp.norm.weight.detach().clone())
        self.register_buffer("norm_bias", None if mlp.norm.bias is None else mlp.norm.bias.detach().clone())
        self.gate, self.up, self.down = (NVFP4FrozenLinear(layer) for layer in (mlp.gate, mlp.up, mlp.down))

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if _wants_grad(x):
            raise RuntimeError("NVFP4FrozenMLP has no gradient: use it under torch.no_grad()")
        n = _layer_norm_call(_rows(x, self.features, "NVFP4FrozenMLP"), self.norm_weight, self.norm_bias, self.eps, False)
        y = self.down(_swiglu_call(self.gate(n), self.up(n), False))
        return y if x.dim() == 2 else y.reshape(x.shape)
