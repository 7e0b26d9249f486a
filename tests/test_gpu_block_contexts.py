"""The modules around the linears where autograd is not the only one who looks on: traces, forward-mode tangents, function transformations.
The rules are NVFP4Linear's: a trace gets the autograd function, which refuses the others."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def mk(*shape):
    return torch.randn(*shape, device="cuda").to(torch.bfloat16)


def norm(weight_grad):
    from paper_2510_27527_b200.block import NVFP4LayerNorm

    return NVFP4LayerNorm(64).requires_grad_(weight_grad)


class Gated(torch.nn.Module):
    def __init__(self, weight_grad):
        super().__init__()
        self.u = torch.nn.Parameter(mk(6, 64), requires_grad=weight_grad)  # (a tracer takes no other tensors that want gradients)

    def forward(self, x):
        from paper_2510_27527_b200.block import swiglu

        return swiglu(x, self.u)


def frozen(kind):
    from paper_2510_27527_b200 import binding as b
    from paper_2510_27527_b200.block import NVFP4MLP
    from paper_2510_27527_b200.module import NVFP4Linear

    if kind == "mlp":
        return NVFP4MLP(64, 128).frozen()
    return NVFP4Linear(64, 40, bias=True, cfg=b.LayerConfig(outliers=np.array([1, 60]) if kind == "outliers" else None)).frozen()


CALLS = [lambda: norm(False), lambda: norm(True), lambda: Gated(False), lambda: Gated(True), lambda: frozen("linear"), lambda: frozen("outliers"), lambda: frozen("mlp")]
calls = pytest.mark.parametrize("made", CALLS, ids=["norm", "norm with gradients", "swiglu", "swiglu with gradients", "frozen linear", "with outliers", "frozen mlp"])


@pytest.mark.filterwarnings("ignore::torch.jit.TracerWarning", "ignore::DeprecationWarning")
@pytest.mark.parametrize("grad", [False, True])
@calls
def test_a_trace_computes_what_the_call_computes(made, grad):
    f, x = made(), mk(6, 64)
    with torch.set_grad_enabled(grad):
        traced = torch.jit.trace(f, x, check_trace=False)
        for other in (2 * x, mk(6, 64)):
            assert torch.equal(traced(other), f(other))
        odd = mk(6, 70)[:, 3:67]  # rows off their boundaries
        assert torch.equal(torch.jit.trace(f, odd, check_trace=False)(odd), f(odd))


@pytest.mark.filterwarnings("ignore::torch.jit.TracerWarning", "ignore::DeprecationWarning")
@pytest.mark.parametrize("traced_with_grad", [False, True])
def test_gradients_through_a_trace(traced_with_grad):
    from paper_2510_27527_b200.block import swiglu

    class Both(torch.nn.Sequential):
        def forward(self, t):
            return swiglu(self[0](t), t)

    ln, x, dy = norm(True), mk(6, 64), mk(6, 64)
    f = Both(ln)
    with torch.set_grad_enabled(traced_with_grad):
        traced = torch.jit.trace(f, x, check_trace=False)
    got, want = ([*torch.autograd.grad(g(xi), (xi, ln.weight, ln.bias), dy)] for g, xi in ((traced, x.clone().requires_grad_()), (f, x.clone().requires_grad_())))
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("grad", [False, True])
@calls
def test_tangents_are_refused(made, grad):
    import torch.autograd.forward_ad as fa

    f, x = made(), mk(6, 64)
    with torch.set_grad_enabled(grad), fa.dual_level():
        with pytest.raises(NotImplementedError, match="jvp"):
            f(fa.make_dual(x, torch.ones_like(x)))


@pytest.mark.parametrize("name,made", [("weight", lambda: norm(False)), ("bias", lambda: norm(False)), ("bias", lambda: frozen("linear")), ("outlier_weight", lambda: frozen("outliers")),
                                       ("norm_weight", lambda: frozen("mlp"))])
def test_tangents_of_parameters_are_refused(name, made):
    import torch.autograd.forward_ad as fa

    f, x = made(), mk(6, 64)
    p = getattr(f, name).detach()
    with torch.no_grad(), fa.dual_level(), pytest.raises(NotImplementedError, match="jvp"):
        torch.func.functional_call(f, {name: fa.make_dual(p, torch.ones_like(p))}, (x,))


@pytest.mark.parametrize("grad", [False, True])
@calls
def test_transforms_are_refused(made, grad):
    f, x = made(), mk(6, 64)
    with torch.set_grad_enabled(grad):
        for call in (lambda: torch.func.vmap(f)(x[None]), lambda: torch.func.jvp(f, (x,), (x,))):
            with pytest.raises(RuntimeError):
                call()


def test_a_frozen_layers_parameters_have_no_gradient():
    f, x = frozen("linear"), mk(6, 64)
    bias = f.bias.clone().requires_grad_()
    y = torch.func.functional_call(f, {"bias": bias}, (x,))
    with pytest.raises(RuntimeError, match="no gradient"):
        y.sum().backward()


@pytest.mark.parametrize("norm_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("change", ["half", "double", "float", "bfloat16"])
def test_a_frozen_models_change_of_type_changes_no_answer(change, norm_dtype):
    from paper_2510_27527_b200.block import NVFP4MLP

    mlp, x = NVFP4MLP(64, 128, norm_dtype=norm_dtype), mk(3, 64)
    with torch.no_grad():
        mlp.norm.weight.add_(torch.randn(64, device="cuda") * 0.1)
        f = mlp.frozen()
        want = f(x)
        assert torch.equal(getattr(f, change)()(x), want) and f.norm_weight.dtype == norm_dtype
        assert torch.equal(torch.nn.Sequential(f).to(torch.float16)(x), want)


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("width", [64, 33])  # (rows of 33 are padded, their copies are not)
def test_inputs_kept_elsewhere(width, checkpoint):
    """torch.autograd.graph.save_on_cpu brings back contiguous copies."""
    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    ln, x, dy = NVFP4LayerNorm(width, checkpoint=checkpoint), mk(6, width).requires_grad_(), mk(6, width)

    def step():
        y = swiglu(ln(x), x * 1, checkpoint)
        return y, lambda: torch.autograd.grad(y, (x, ln.weight, ln.bias), dy)

    want = step()[1]()
    with torch.autograd.graph.save_on_cpu():
        y, grads = step()
    assert all(torch.equal(p, q) for p, q in zip(grads(), want))


@pytest.mark.parametrize("backend", ["eager", "inductor"])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_compiled_autograd(checkpoint, backend):
    from torch._dynamo import compiled_autograd

    from paper_2510_27527_b200.block import NVFP4LayerNorm, swiglu

    torch._dynamo.reset()
    ln, dy, got = NVFP4LayerNorm(64, checkpoint=checkpoint), mk(6, 64), []
    x = mk(6, 64).requires_grad_()
    for compiled in (False, True, True):
        x.grad = ln.weight.grad = ln.bias.grad = None
        y = swiglu(ln(x), x, checkpoint)
        if compiled:
            with compiled_autograd._enable(torch.compile(backend=backend)):
                y.backward(dy)
        else:
            y.backward(dy)
        got.append((y.detach(), x.grad, ln.weight.grad, ln.bias.grad))
    assert all(torch.equal(p, q) for g in got[1:] for p, q in zip(got[0], g))
    torch._dynamo.reset()


def test_frozen_layers_with_a_parametrized_bias():
    import torch.nn.utils.parametrize as parametrize

    class Twice(torch.nn.Module):
        def forward(self, v):
            return 2 * v

    f, g, x = frozen("linear"), frozen("linear"), mk(3, 64)
    with torch.no_grad():
        g.load_state_dict(f.state_dict())
        f.bias.copy_(mk(40))
        g.bias.copy_(2 * f.bias)
        parametrize.register_parametrization(f, "bias", Twice())
        assert torch.equal(f(x), g(x))


@pytest.mark.parametrize("backend", ["eager", "inductor"])
@pytest.mark.parametrize("kind", ["linear", "outliers", "mlp"])
def test_compiled_frozen_modules(kind, backend):
    torch._dynamo.reset()
    f = frozen(kind)
    with torch.no_grad():
        g = torch.compile(f, backend=backend)
        for x in (mk(3, 64), mk(3, 64), mk(7, 64)):
            assert torch.equal(g(x), f(x))
    torch._dynamo.reset()
