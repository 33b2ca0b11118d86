"""The layer operators under torch.autograd and on callers' destinations: what is written, recorded and refused, in which shapes."""
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


# ------------------------------------------------------------------------------------------------ more than two dimensions
@pytest.mark.parametrize("shape", [(6, 10, 40), (2, 3, 5, 33), (40,), (0, 4, 40), (60, 40)])
@pytest.mark.parametrize("with_b,token", [(True, False), (True, True), (False, False)])
def test_block_end_keeps_the_shape_of_its_rows(shape, with_b, token):
    D = shape[-1]
    flat = lambda t: None if t is None else t.reshape(-1 if t.numel() else 0, D)  # noqa: E731
    x, b, t = randn(1, *shape), randn(2, *shape) if with_b else None, randn(3, *shape) if token else None
    w_post, w_pre = (1 + 0.1 * randn(4 + i, 1, D, dtype=torch.float32) for i in range(2))
    kw = dict(w_pre=w_pre, **(dict(w_post=w_post, p=0.2, seed=3) if with_b else {}))
    r, h = nn.residual_norm(x, b, token_gate=t, **kw)
    r2, h2 = nn.residual_norm(flat(x), flat(b), token_gate=flat(t), **kw)
    assert r.shape == h.shape == x.shape and torch.equal(flat(r), r2) and torch.equal(flat(h), h2)
    dr, dh = randn(6, *shape), randn(7, *shape)
    g = nn.residual_norm_backward(dr, dh, r, b, token_gate=t, **kw)
    g2 = nn.residual_norm_backward(flat(dr), flat(dh), r2, flat(b), token_gate=flat(t), **kw)
    for name in nn.NormGrads._fields:
        a, c = getattr(g, name), getattr(g2, name)
        assert (a is None) == (c is None)
        if a is not None and name in ("dx", "db", "dtoken_gate"):
            assert a.shape == x.shape and torch.equal(flat(a), c), name
        elif a is not None:
            assert torch.equal(a, c), name
    # under autograd
    leaf = [None if v is None else v.clone().requires_grad_() for v in (x, b, t)]
    opts = dict(p=0.2, seed=3) if with_b else {}
    r3, h3 = nn.ResidualNorm.apply(leaf[0], leaf[1], w_post if with_b else None, None, None, leaf[2], w_pre, None, None, opts)
    assert r3.shape == h3.shape == x.shape and torch.equal(h3, h)
    torch.autograd.backward([r3, h3], [dr, dh])
    for v, name in zip(leaf, ("dx", "db", "dtoken_gate")):
        assert v is None or torch.equal(v.grad, getattr(g, name)), name


# ------------------------------------------------------------------------------------------------ gradients of any strides
BEHIND = [("transposed", lambda y: y.transpose(0, 1), (10, 6)), ("summed", lambda y: y.float().sum(1), (6,)), ("mean of the columns", lambda y: y.float().mean(-1), (6, 10)),
          ("last first", lambda y: y.permute(2, 0, 1), None)]


@pytest.mark.parametrize("name,behind,lead", BEHIND, ids=[b[0] for b in BEHIND])
def test_wrappers_take_gradients_of_any_strides(name, behind, lead):
    x = randn(1, 6, 10, 40).requires_grad_()
    w, v, b = randn(2, 1, 24, 40), 1 + 0.1 * randn(3, 1, 40, dtype=torch.float32), randn(4, 6, 10, 40).requires_grad_()
    forms = [(lambda: nn.GroupedLinear.apply(x, w), [x]), (lambda: nn.Dropout.apply(x, 0.3, 5), [x]),
             (lambda: nn.ResidualNorm.apply(x, b, v, None, None, None, v, None, None, None)[1], [x, b])]
    for call, leaves in forms:
        y = call()
        z = behind(y)
        g = randn(8, *z.shape, dtype=z.dtype)
        got = torch.autograd.grad(z, leaves, g)
        plain = y.detach().clone().requires_grad_()
        dy = torch.autograd.grad(behind(plain), plain, g)[0].contiguous()
        want = torch.autograd.grad(call(), leaves, dy)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), name


# ------------------------------------------------------------------------------------------------ what out= writes
def writers():
    off = nn.group_offsets([4, 6], DEV)
    x, w, dy = randn(1, 10, 16), randn(2, 2, 16, 16), randn(3, 10, 16)
    v = randn(4, 2, 16, dtype=torch.float32)
    return [(lambda o: nn.dropout(x, 0.5, 1, out=o), (10, 16), torch.bfloat16), (lambda o: nn.dropout_backward(o, 0.5, 1, out=o), (10, 16), torch.bfloat16),
            (lambda o: nn.grouped_linear(x, w, off, out=o), (10, 16), torch.bfloat16), (lambda o: nn.grouped_linear_dx(dy, w, off, out=o), (10, 16), torch.bfloat16),
            (lambda o: nn.grouped_linear_dw(dy, x, off, out=o), (2, 16, 16), torch.float32),
            (lambda o: nn.residual_norm_backward(None, dy, x, w_pre=v, offsets=off, out=dict(dw_pre=o)), (2, 16), torch.float32)]


@pytest.mark.parametrize("which", range(6))
def test_a_saved_tensor_that_is_written_raises_in_backward(which):
    write, shape, dtype = writers()[which]
    a = torch.ones(shape, dtype=dtype, device=DEV, requires_grad=True)
    saved = randn(9, *shape, dtype=dtype)
    loss = (a * saved).sum()
    write(saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("which", range(6))
def test_a_destination_that_requires_a_gradient_is_refused(which):
    write, shape, dtype = writers()[which]
    leaf = torch.ones(shape, dtype=dtype, device=DEV, requires_grad=True)
    for out in (leaf, leaf * 2):
        with pytest.raises(hop.HopError) as e:
            write(out)
        assert e.value.code == hop.E_ARG
    with torch.no_grad():
        write(leaf)                     # as torch: allowed where nothing is recorded


def test_destinations_that_share_memory_with_an_operand_are_refused():
    x, w, big = randn(1, 300, 256), randn(2, 1, 256, 256), randn(3, 301, 256)
    wide = randn(4, 300, 512)
    g, v = randn(5, 2, 64, 64), randn(6, 1, 256, dtype=torch.float32)
    bad = [lambda: nn.grouped_linear(x, w, out=x), lambda: nn.grouped_linear(x, w, out=w[0][:1].expand(300, 256)),
           lambda: nn.grouped_linear(big[1:], w, out=big[:-1]), lambda: nn.grouped_linear_dx(wide[:, :256], w, out=wide[:, :256]),
           lambda: nn.grouped_linear(x[:256], w, out=w[0]), lambda: nn.grouped_linear_dw(g[0], g[1], out=g[:1], out_dtype=None),
           lambda: nn.dropout(big[1:], 0.5, 1, out=big[:-1]), lambda: nn.dropout(wide.view(-1, 256)[:300], 0.5, 1, out=wide[:, :256]),
           lambda: nn.residual_norm_backward(None, x, x, w_pre=v, out=dict(dw_pre=v)),
           lambda: nn.residual_norm_backward(x, x, x, randn(7, 300, 256), w_pre=v, w_post=v.clone(), out=dict(dw_pre=(d := torch.empty_like(v)), dw_post=d))]
    for i, call in enumerate(bad):
        with pytest.raises(hop.HopError) as e:
            call()
        assert e.value.code == hop.E_ARG, i


def test_views_side_by_side_in_one_buffer_are_not():
    wide, w = randn(1, 300, 512), randn(2, 1, 256, 256)
    want = nn.grouped_linear(wide[:, :256].clone(), w)
    nn.grouped_linear(wide[:, :256], w, out=wide[:, 256:])
    assert torch.equal(wide[:, 256:], want)
    halves = randn(3, 600, 256)
    want = nn.dropout(halves[:300].clone(), 0.5, 1)
    nn.dropout(halves[:300], 0.5, 1, out=halves[300:])
    assert torch.equal(halves[300:], want)
    nn.dropout(halves[:300], 0.5, 1, out=halves[:300])
    assert torch.equal(halves[:300], want)


def test_arguments_that_have_no_truth_value_are_refused():
    x, many = torch.ones(4, 16, dtype=torch.bfloat16, device=DEV), torch.ones(2, device=DEV)
    out = torch.zeros(1, 16, 16, device=DEV)
    for call in (lambda: nn.residual_norm(x, x, post=many), lambda: nn.residual_norm(x, pre=many), lambda: nn.grouped_linear_dw(x, x, out=out, accumulate=many)):
        with pytest.raises(hop.HopError) as e:
            call()
        assert e.value.code == hop.E_ARG
    assert bool((out == 0).all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("counts", [[5, 0, 40], [0, 0]], ids=str)
def test_vector_gradients_of_a_group_without_rows_are_zero_whatever_its_vectors_hold(kind, counts):
    """An idle worker's replica may hold anything: its part of G is a sum over nothing."""
    E, T, D = len(counts), sum(counts), 72
    names = ("w_post", "gate", "w_pre") + (("c_post", "c_pre") if kind == "layer" else ())
    v = {n: 1 + 0.1 * randn(i, E, D, dtype=torch.float32) for i, n in enumerate(names)}
    for t in v.values():
        for g, c in enumerate(counts):
            if not c:
                t[g, ::2], t[g, 1::2] = float("nan"), float("inf")
    rows = [randn(9 + i, T, D) for i in range(4)]
    g = nn.residual_norm_backward(*rows, offsets=nn.group_offsets(counts, DEV), kind=kind, p=0.1, seed=3, **v)
    for n in names:
        d = getattr(g, "d" + n)
        assert bool((d[[i for i, c in enumerate(counts) if not c]] == 0).all()), n
        assert bool(d.isfinite().all()), n


@pytest.mark.parametrize("shape", [(0, 40), (0, 4, 40), (3, 0, 40)])
def test_levels_without_rows_pass_backward(shape):
    """All workers idle: the gradients that autograd expands from a sum over nothing have stride 0 along the columns too."""
    lead = shape[:-1]
    x, w = randn(1, *shape).requires_grad_(), randn(2, 1, 24, 40).requires_grad_()
    y = nn.GroupedLinear.apply(x, w)
    assert y.shape == (*lead, 24)
    y.sum().backward()
    assert x.grad.shape == x.shape and bool((w.grad == 0).all())
    v = torch.ones(40, device=DEV, requires_grad=True)
    r, h = nn.ResidualNorm.apply(x, x, v, None, None, None, v, None)
    (r.float().sum() + h.float().sum()).backward()
    assert r.shape == h.shape == x.shape and bool((v.grad == 0).all())
    z = nn.Dropout.apply(x, 0.3, 1)
    z.sum().backward()
    assert z.shape == x.shape
