"""What autograd makes of the layers' functions with the kernels under them: second
derivatives by way of other tensors, checkpoints, weights changed under way, forward
derivatives, traces."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from torch.utils.checkpoint import checkpoint  # noqa: E402

from paper_2608_05033_amd import experts, gcn  # noqa: E402


def numbers(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda().requires_grad_()


def transform8(X, W):
    return gcn._PackedTransform.apply(X, W, "e4m3", "e4m3")[0]


def norm_transform(X, W):
    gamma, beta = torch.linspace(0.5, 1.5, X.shape[1]).cuda(), torch.linspace(-1, 1, X.shape[1]).cuda()
    return gcn._NormTransform.apply(X, gamma, beta, W, 4, 1e-5, "silu", "e4m3", "e4m3")[0]


@pytest.fixture(params=["transform4", "transform8", "norm"])
def layer(request):
    return {"transform4": gcn.transform4, "transform8": transform8, "norm": norm_transform}[request.param]


@pytest.mark.parametrize("of", ["X", "W"])
def test_second_derivatives_are_never_left_out(layer, of):
    """X and W come from tensors that other parts of the sum depend on too."""
    a, b = numbers(50, 40, seed=1), numbers(40, 24, seed=2)
    X, W = torch.sin(a), torch.cos(b)
    Z = layer(X, W)
    v = W if of == "X" else X
    g, = torch.autograd.grad(Z.sum(), v, create_graph=True)
    assert torch.equal(g, torch.autograd.grad(layer(X, W).sum(), v)[0])
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(Z.sum() + g.square().sum(), a if of == "X" else b)


@pytest.mark.parametrize("create", [False, True])
def test_a_layer_within_a_checkpoint(layer, create):
    X, W = numbers(50, 40, seed=1), numbers(40, 24, seed=2)
    want = torch.autograd.grad(layer(X, W).sum(), (X, W))
    got = torch.autograd.grad(checkpoint(layer, X, W, use_reentrant=False).sum(), (X, W), create_graph=create)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_changed_between_the_passes():
    """The backward pass of transform4 takes the weights that the forward pass packed."""
    X, W = numbers(50, 40, seed=1), numbers(40, 24, seed=2)
    want = torch.autograd.grad(gcn.transform4(X, W).sum(), (X, W))
    Z = gcn.transform4(X, W)
    with torch.no_grad():
        W.mul_(3)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(Z.sum(), (X, W)), want))


def test_forward_derivatives_are_refused():
    import torch.autograd.forward_ad as forward

    r = experts.route(torch.tensor([[0, 1], [1, 2], [2, -1]], device="cuda"), 3)
    x, y, w = (torch.ones(*size, device="cuda") for size in ((3, 8), (6, 8), (3, 2)))
    want = experts.dispatch(x, r), experts.combine(y, r, w)
    with forward.dual_level():
        dual = {v: forward.make_dual(v, torch.ones_like(v)) for v in (x, y, w)}
        for f in (lambda: experts.dispatch(dual[x], r), lambda: experts.combine(dual[y], r),
                  lambda: experts.combine(dual[y], r, w), lambda: experts.combine(y, r, dual[w]),
                  lambda: gcn.transform4(dual[x], torch.ones(8, 4, device="cuda"))):
            with pytest.raises(NotImplementedError, match="forward mode"):
                f()
        assert torch.equal(experts.dispatch(x, r), want[0]) and torch.equal(experts.combine(y, r, w), want[1])


def test_traced_calls_are_recorded():
    r = experts.route(torch.tensor([[0, 1], [1, 2], [2, -1]], device="cuda"), 3)

    def step(x, w):
        return experts.combine(experts.dispatch(x, r), r, w), experts.combine(experts.dispatch(x, r), r)

    x, w = numbers(3, 8, seed=1).detach(), numbers(3, 2, seed=2).detach()
    traced = torch.jit.trace(step, (torch.ones_like(x), torch.ones_like(w)), check_trace=False)
    assert all(torch.equal(a, b) for a, b in zip(traced(x, w), step(x, w)))


def test_transform4_without_gradients(monkeypatch):
    """Nothing is packed for a backward pass; the result has the same bits."""
    X, W = numbers(500, 40, seed=1), numbers(40, 24, seed=2)
    want = gcn.transform4(X, W).detach()
    monkeypatch.setattr(gcn.dense, "pack4_both", None)
    with torch.no_grad():
        assert torch.equal(gcn.transform4(X, W), want)
    assert torch.equal(gcn.transform4(X.detach(), W.detach()), want)


def test_kept_tables_go_through_autograds_hooks():
    """Packed copies moved to the host between the passes give the same gradients; ones
    that stay there, or come back as something else, are refused."""
    X, W = numbers(50, 40, seed=1), numbers(40, 24, seed=2)
    want = torch.autograd.grad(gcn.transform4(X, W).sum(), (X, W))
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (t.device, t.cpu()), lambda kept: kept[1].to(kept[0])):
        Z = gcn.transform4(X, W)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(Z.sum(), (X, W)), want))
    for back in (lambda t: t, lambda t: t.cuda()[:-16], lambda t: t.cuda().float()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), back):
            Z = gcn.transform4(X, W)
        with pytest.raises(ValueError, match="store"):
            torch.autograd.grad(Z.sum(), (X, W))
