"""The layer operators under torch.autograd: what is written, recorded and refused, and in which shapes."""
import pytest
import torch

from paper_1902_01064_b200 import hop, nn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def randn(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


# ------------------------------------------------------------------------------------------------ gradients into destinations
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_first_layers_weight_gradient_is_written(accumulate):
    """x is data and w a working copy: neither requires a gradient, only the destination asks for one."""
    off = nn.group_offsets([20, 0, 28], DEV)
    x, w, dy = randn(1, 48, 64), randn(2, 3, 40, 64), randn(3, 48, 40)
    G = torch.full((3, 40, 64), 7.0, device=DEV)
    want = nn.grouped_linear_dw(dy, x, off)
    y = nn.GroupedLinear.apply(x, w, off, G, accumulate)
    assert torch.equal(y, nn.grouped_linear(x, w, off))
    y.backward(dy)
    assert torch.equal(G, want + 7.0 if accumulate else want)
    assert x.grad is None and w.grad is None


def test_a_first_norms_vector_gradients_are_written():
    off = nn.group_offsets([20, 28], DEV)
    x, v = randn(1, 48, 64), 1 + 0.1 * randn(2, 2, 64, dtype=torch.float32)
    G = torch.full((2, 64), 7.0, device=DEV)
    r, h = nn.ResidualNorm.apply(x, None, None, None, None, None, v, None, off, dict(out=dict(dw_pre=G)))
    dh = randn(3, 48, 64)
    h.backward(dh)
    assert torch.equal(G, nn.residual_norm_backward(None, dh, x, w_pre=v, offsets=off).dw_pre)


def test_nothing_is_recorded_where_nothing_asks_for_a_gradient():
    off = nn.group_offsets([20, 28], DEV)
    x, w, G = randn(1, 48, 64), randn(2, 2, 40, 64), torch.zeros(2, 40, 64, device=DEV)
    assert not nn.GroupedLinear.apply(x, w, off).requires_grad
    with torch.no_grad():
        assert not nn.GroupedLinear.apply(x, w, off, G).requires_grad


class NoGradient(torch.autograd.Function):
    @staticmethod
    def forward(ctx, v):
        return v * 1

    @staticmethod
    def backward(ctx, g):
        return None


def test_destinations_of_a_result_without_gradient_become_zero():
    x, v, G = randn(1, 10, 64).requires_grad_(), 1 + 0.1 * randn(2, 1, 64, dtype=torch.float32), torch.full((1, 64), 7.0, device=DEV)
    r, h = nn.ResidualNorm.apply(x, None, None, None, None, None, v, None, None, dict(out=dict(dw_pre=G)))
    (NoGradient.apply(h).float().sum() + NoGradient.apply(r).float().sum()).backward()
    assert bool((G == 0).all()) and (x.grad is None or bool((x.grad == 0).all()))


# ------------------------------------------------------------------------------------------------ second derivatives
def calls():
    x, w, v = randn(1, 12, 32).requires_grad_(), randn(2, 1, 24, 32).requires_grad_(), (1 + randn(3, 1, 32, dtype=torch.float32)).requires_grad_()
    b = randn(4, 12, 32).requires_grad_()
    options = dict(p=0.2, seed=5)
    return [("product", lambda: nn.GroupedLinear.apply(torch.tanh(x), w), [x, w]),
            ("norm", lambda: sum(nn.ResidualNorm.apply(torch.tanh(x), b, v, None, None, None, v, None, None, options)), [x, b, v]),
            ("norm without b", lambda: nn.ResidualNorm.apply(torch.tanh(x), None, None, None, None, None, v, None, None, None)[1], [x, v]),
            ("dropout", lambda: nn.Dropout.apply(torch.tanh(x), 0.3, 7), [x])]


@pytest.mark.parametrize("which", range(4))
def test_a_second_derivative_raises(which):
    name, call, leaves = calls()[which]
    for loss in (lambda y: y.float().square().sum(), lambda y: y.float().sum()):     # (the sum's own gradient requires none)
        if name == "dropout" and loss(torch.ones(1)) == 1 and loss(torch.full((1,), 2.0)) == 2:
            continue        # linear all the way: its gradient depends on nothing
        grads = torch.autograd.grad(loss(call()), leaves, create_graph=True)
        with pytest.raises(RuntimeError, match="once|second"):
            torch.autograd.grad(sum(g.float().square().sum() for g in grads), leaves, allow_unused=True)


@pytest.mark.parametrize("which", range(4))
def test_create_graph_alone_gives_the_same_gradients(which):
    _, call, leaves = calls()[which]
    first = torch.autograd.grad(call().float().square().sum(), leaves)
    again = torch.autograd.grad(call().float().square().sum(), leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
