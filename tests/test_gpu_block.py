"""The modules around the linears, and a block's MLP as a whole: trained with checkpoints in 8 bits, frozen, answered from."""
import copy

import numpy as np
import pytest
import torch

from oracle import block_ops as O
from oracle import nvfp4_oracle as orc
from paper_2510_27527_b200 import synth
from tests.block_util import BF16, device_rows, host, inputs

pytestmark = pytest.mark.gpu


def mlp(hidden=200, ffn=520, checkpoint=True, seed=3, **kw):
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4MLP

    torch.manual_seed(seed)
    m = NVFP4MLP(hidden, ffn, b.LayerConfig(seed=5, **kw), checkpoint=checkpoint)
    for i, layer in enumerate((m.gate, m.up, m.down)):
        layer.layer_id = i
    with torch.no_grad():
        m.norm.weight.add_(torch.randn(hidden, device="cuda") * 0.1)
        m.norm.bias.add_(torch.randn(hidden, device="cuda") * 0.1)
    return m


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("shape", [(7, 200), (2, 33, 200), (200,), (0, 200)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_norm_module(shape, dtype, checkpoint):
    """Forward and gradients are the binding's, in the input's shape and types."""
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4LayerNorm

    ln = NVFP4LayerNorm(200, checkpoint=checkpoint, dtype=torch.float32)
    with torch.no_grad():
        ln.weight.add_(torch.randn(200, device="cuda"))
    x = torch.randn(shape, device="cuda").to(dtype).requires_grad_()
    y = ln(x)
    dy = torch.randn_like(y)
    y.backward(dy)
    rows = x.detach().reshape(-1, 200)
    want, saved = b.nvfp4_layernorm_fwd(rows, ln.weight.detach(), ln.bias.detach(), 1e-5, 2 if checkpoint else 1)
    dx, dg, db = b.nvfp4_layernorm_bwd(dy.reshape(-1, 200), saved)
    assert y.dtype == torch.bfloat16 and y.shape == x.shape and torch.equal(y.reshape(-1, 200), want)
    assert x.grad.dtype == dtype and torch.equal(x.grad.reshape(-1, 200), dx) and torch.equal(ln.weight.grad, dg) and torch.equal(ln.bias.grad, db)
    with torch.no_grad():
        assert torch.equal(ln(x), y)


def test_rows_that_are_not_aligned_are_copied():
    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    base = torch.randn(9, 300, device="cuda").bfloat16()
    ln = NVFP4LayerNorm(33)
    odd = base[:, 5:38]  # rows off their boundaries
    strided = base.T[:33, :9].T  # columns at a stride
    for x in (odd, strided, odd.contiguous(), base[::2, :33], base[:1, 1:34].expand(4, 33)):
        y = ln(x)
        want = O.layernorm(host(x), np.ones(33), np.zeros(33), 1e-5)[0]
        assert np.all(np.abs(host(y) - want) <= BF16 * np.abs(want) + 2.0 ** -17 * (1 + np.abs(want)))
        assert torch.equal(swiglu(x, x), swiglu(x.clone(), x.clone()))


@pytest.mark.parametrize("checkpoint", [False, True])
def test_mlp_is_the_chain_of_its_calls(checkpoint):
    """Forward and every gradient, bit for bit, against the library's calls one after another; the keys of the stochastic rounding are the layers'."""
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.module import call_seed

    m = mlp(checkpoint=checkpoint)
    x = torch.from_numpy(inputs(96, 200, 1)).cuda().bfloat16().requires_grad_()
    dy = b.upload_bf16(synth.gradients(96, 200, 2, 1e-3))
    y = m(x)
    y.backward(dy)
    save = 2 if checkpoint else 1
    n, s_norm = b.nvfp4_layernorm_fwd(x.detach(), m.norm.weight.detach(), m.norm.bias.detach(), 1e-5, save)
    cfg = lambda i: b.LayerConfig(seed=call_seed(5, i, 0), dw_dtype=b.DT_BF16)  # noqa: E731
    c = [cfg(i) for i in range(3)]
    g, s_gate = b.nvfp4_linear_fwd(n, m.gate.weight.detach(), c[0])
    u, s_up = b.nvfp4_linear_fwd(n, m.up.weight.detach(), c[1])
    h, s_act = b.nvfp4_swiglu_fwd(g, u, save)
    want, s_down = b.nvfp4_linear_fwd(h, m.down.weight.detach(), c[2])
    assert torch.equal(y, want)
    dh, dw_down = b.nvfp4_linear_bwd(dy, s_down, c[2])
    dg, du = b.nvfp4_swiglu_bwd(dh, s_act)
    dn_u, dw_up = b.nvfp4_linear_bwd(du, s_up, c[1])
    dn_g, dw_gate = b.nvfp4_linear_bwd(dg, s_gate, c[0])
    dx, dgamma, dbeta = b.nvfp4_layernorm_bwd(dn_u + dn_g, s_norm)
    for got, ref in ((m.down.weight.grad, dw_down), (m.up.weight.grad, dw_up), (m.gate.weight.grad, dw_gate), (x.grad, dx), (m.norm.weight.grad, dgamma),
                     (m.norm.bias.grad, dbeta)):
        assert torch.equal(got, ref)


def test_checkpoints_hold_less():
    """What forward leaves for backward, in bytes: 8-bit checkpoints against the inputs themselves."""
    T, hidden, ffn = 4096, 256, 1024
    held = []
    for checkpoint in (False, True):
        m = mlp(hidden, ffn, checkpoint)
        x = torch.randn(T, hidden, device="cuda").bfloat16().requires_grad_()
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        y = m(x)
        held.append(torch.cuda.memory_allocated() - before)
        y.sum().backward()
        del m, x, y
    # without: g and u, 4 bytes an element (x is the caller's own); with: g, u and x at 33 / 32 bytes. The rest is the same.
    saved = held[0] - held[1]
    want = T * ffn * (4 - 2 * 33 / 32) - T * hidden * 33 / 32
    assert abs(saved - want) < 2 ** 20, (held, want)


@pytest.mark.parametrize("gs,n_out,extra", [(0, 0, {}), (1, 0, {}), (2, 12, {}), (0, 7, dict(outlier_fp8=True)), (0, 0, dict(w_block16=True))])
@pytest.mark.parametrize("tokens", [1, 5])
def test_frozen_linear(tokens, gs, n_out, extra):
    """The frozen layer multiplies by exactly the weights that the layer's forward uses."""
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.module import NVFP4Linear

    D, C = 272, 150
    outl = synth.outlier_channels(D, n_out, 5) if n_out else None
    layer = NVFP4Linear(D, C, bias=True, cfg=b.LayerConfig(gs_mode=gs, outliers=outl, **extra))
    with torch.no_grad():
        layer.bias.add_(torch.randn(C, device="cuda"))
    frozen = layer.frozen()
    _, saved = b.nvfp4_linear_fwd(torch.randn(3, D, device="cuda").bfloat16(), layer.weight.detach(), layer.cfg)
    W = saved.qw
    assert torch.equal(frozen.codes, W.codes) and torch.equal(frozen.scales, W.sf) and torch.equal(frozen.global_scales, W.gscale)
    keep = np.arange(D) if outl is None else np.setdiff1d(np.arange(D), outl)
    dense = np.zeros((C, D))
    nb = W.Kp // 16
    codes = W.codes.cpu().numpy().reshape(C, W.Kp // 2)
    nib = np.stack([codes & 15, codes >> 4], 2).reshape(C, W.Kp)
    values = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    e4m3 = torch.from_numpy(W.sf_linear()).view(torch.float8_e4m3fn).double().numpy()
    gscale = host(W.gscale)
    wide = {0: lambda: np.full((C, nb), gscale[0]), 1: lambda: np.repeat(gscale[:, None], nb, 1), 2: lambda: np.repeat(gscale.reshape(C, -1), 8, 1)}[gs]()
    dense[:, keep] = (values.reshape(C, nb, 16) * (e4m3 * wide)[..., None]).reshape(C, W.Kp)[:, : len(keep)]
    if n_out:
        dense[:, outl] = host(saved.W_out)[:, :n_out]
    x = inputs(tokens, D, 3)
    with torch.no_grad():
        y = frozen(device_rows(x, torch.bfloat16))
    want = x.astype(np.float64) @ dense.T + host(layer.bias)
    absdot = np.abs(x).astype(np.float64) @ np.abs(dense).T + np.abs(host(layer.bias))
    assert np.all(np.abs(host(y) - want) <= 2.0 ** -15 * absdot + BF16 * np.abs(want))


@pytest.mark.parametrize("tokens", [1, 2, 9])
def test_answering_with_a_trained_mlp(tokens):
    """A few steps of training, then frozen: its answer is the chain of the calls, in every shape, captured and not, saved and loaded."""
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4FrozenMLP

    m = mlp(outliers=None)
    opt = torch.optim.SGD(m.parameters(), lr=1e-2)
    for i in range(3):
        x = torch.randn(64, 200, device="cuda").bfloat16()
        opt.zero_grad()
        (m(x) - x).square().mean().backward()
        assert all(torch.isfinite(p.grad).all() for p in m.parameters())
        opt.step()
    frozen = m.frozen()
    x = torch.randn(tokens, 200, device="cuda").bfloat16()
    with torch.no_grad():
        y = frozen(x)
        n = b.nvfp4_layernorm_fwd(x, m.norm.weight.detach(), m.norm.bias.detach(), 1e-5, 0)[0]
        h = b.nvfp4_swiglu_fwd(frozen.gate(n), frozen.up(n), 0)[0]
        assert torch.equal(y, frozen.down(h))
        assert torch.equal(frozen(x.reshape(1, tokens, 200)), y.reshape(1, tokens, 200))
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            out = frozen(x)
        first, kept = y.clone(), x.clone()
        x.copy_(torch.randn_like(x))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, frozen(x)) and not torch.equal(out, first)
        other = NVFP4FrozenMLP(mlp(seed=9))
        other.load_state_dict(frozen.state_dict())
        assert torch.equal(other(kept), first)
    with pytest.raises(RuntimeError, match="no gradient"):
        frozen(x.clone().requires_grad_())
    other = copy.deepcopy(frozen)
    other.gate.half(), other.up.double(), other.down.float()  # the operands keep their types
    with torch.no_grad():
        assert torch.equal(other(kept), first)


def test_mlp_with_outlier_channels():
    """The gate and up projections' outlier channels are channels of the normed input; frozen, they are multiplied in BF16."""
    m = mlp(outliers=np.array([0, 17, 199]), rht=True)
    x = torch.from_numpy(inputs(64, 200, 1)).cuda().bfloat16().requires_grad_()
    y = m(x)
    y.backward(torch.ones_like(y))
    assert all(torch.isfinite(p.grad).all() for p in (x, *m.parameters()))
    frozen = m.frozen()
    assert frozen.gate.n_out == 3 and frozen.down.n_out == 0
    only = torch.zeros(4, 200, device="cuda").bfloat16()  # the other channels' codes are multiplied by zero
    only[:, [0, 17, 199]] = torch.randn(4, 3, device="cuda").bfloat16()
    with torch.no_grad():
        got = host(frozen.gate(only))
    w = host(m.gate.weight)
    want, absdot = host(only) @ w.T, np.abs(host(only)) @ np.abs(w).T
    assert np.all(np.abs(got - want) <= 2.0 ** -15 * absdot + BF16 * np.abs(want))


def test_training_step_captured():
    """Forward and backward of the MLP in a CUDA graph give what eager calls with the same keys give."""
    m = mlp()
    x, dy = torch.randn(80, 200, device="cuda").bfloat16().requires_grad_(), torch.randn(80, 200, device="cuda").bfloat16()
    params = list(m.parameters())

    def step():
        for layer in (m.gate, m.up, m.down):
            layer._calls = 0
        y = m(x)
        return (y, *torch.autograd.grad(y, [x, *params], dy))

    want = [t.detach().clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p.detach(), q) for p, q in zip(got, want))


def test_double_backward_is_refused_and_changed_inputs_are_noticed():
    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    x = torch.randn(8, 64, device="cuda").bfloat16().requires_grad_()
    ln = NVFP4LayerNorm(64)
    (gx,) = torch.autograd.grad(ln(x).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        gx.float().sum().backward()
    a = (x * 1).detach().requires_grad_()
    leaf = a * 1
    h = swiglu(leaf, leaf, checkpoint=False)
    with torch.no_grad():
        leaf.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        h.sum().backward()


def test_compiled():
    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    ln = NVFP4LayerNorm(64)
    f = torch.compile(lambda x: swiglu(ln(x), ln(x) + 1), backend="eager")
    x = torch.randn(8, 64, device="cuda").bfloat16().requires_grad_()
    y = f(x)
    y.sum().backward()
    got = x.grad.clone()
    x.grad = None
    want = swiglu(ln(x), ln(x) + 1)
    want.sum().backward()
    assert torch.equal(y, want) and torch.equal(got, x.grad)
