"""A second derivative of an operator's autograd function raises; it does not come out
without its share.  The helper on the CPU, the functions on the GPU."""
import pytest

torch = pytest.importorskip("torch")


def test_gradients_that_are_differentiated_again_raise():
    from paper_2606_00601_amd._bind import _differentiable_once

    class Cube(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            ctx.save_for_backward(x)
            return x ** 3

        @staticmethod
        def backward(ctx, dy):
            (x,) = ctx.saved_tensors
            g = (3 * x.detach() ** 2 * dy.detach())
            return _differentiable_once("cube", (g, None, g), (x, None, dy))[0]

    x = torch.tensor([1.0, 2.0], requires_grad=True)
    (g,) = torch.autograd.grad(Cube.apply(x).sum(), x)
    assert torch.equal(g, 3 * x.detach() ** 2) and not g.requires_grad
    (g,) = torch.autograd.grad(Cube.apply(x).sum(), x, create_graph=True)
    assert torch.equal(g.detach(), 3 * x.detach() ** 2)
    # beside a term that has a second derivative: the share would be missing in silence
    with pytest.raises(RuntimeError, match="cube cannot be differentiated twice"):
        (g.square().sum() + x.square().sum()).backward()


def _cases(sw):
    r = lambda *s: torch.randn(*s, device="cuda").requires_grad_(True)  # noqa: E731
    g = (-torch.rand(1, 40, 2, device="cuda")).requires_grad_(True)
    yield "linear_attn_fn", sw.linear_attn_fn, (r(1, 40, 2, 16), r(1, 40, 2, 16), r(1, 40, 2, 16), g)
    yield "residual_norm_fn", lambda x, w, res: sw.residual_norm_fn(x, w, res)[0], (r(9, 32), r(32), r(9, 32))
    yield "gated_norm_fn", sw.gated_norm_fn, (r(9, 32), r(9, 32), r(32))
    A = (-torch.rand(8, 16, device="cuda")).requires_grad_(True)
    yield "selective_scan_fn", sw.selective_scan_fn, (r(2, 8, 30), r(2, 8, 30), A, r(2, 30, 16), r(2, 30, 16))


@pytest.mark.gpu
def test_every_function_refuses_a_second_derivative():
    import paper_2606_00601_amd as sw
    for name, fn, args in _cases(sw):
        print("case", name, flush=True)
        plain = torch.autograd.grad(fn(*args).sum(), args)
        graph = torch.autograd.grad(fn(*args).sum(), args, create_graph=True)
        assert all(torch.equal(a, b.detach()) for a, b in zip(plain, graph))
        assert not any(a.requires_grad for a in plain)
        with pytest.raises(RuntimeError, match=f"{name} cannot be differentiated twice"):
            (graph[0].square().sum() + args[0].square().sum()).backward()
