"""What autograd makes of the layers' functions, on the CPU: the operators on the GPU
have plain stand-ins here that round nothing, so that every gradient that is given has
a plain form beside it."""
import pytest

torch = pytest.importorskip("torch")

from torch.utils.checkpoint import checkpoint  # noqa: E402

from paper_2608_05033_amd import experts, gcn  # noqa: E402


class Table:
    """A packed table whose codes are the numbers themselves."""

    def __init__(self, codes, scales, cols, format="e4m3"):
        self.codes, self.scales, self.rows, self.cols, self.format = codes, scales, codes.shape[0], cols, format
        self.store = codes

    @classmethod
    def of(cls, store, rows, cols):
        assert store.shape == (rows, cols)
        return cls(store, None, cols)


class Dense:
    """dense.py without the GPU; `calls` counts what was asked for."""

    Packed = Packed4 = Table

    def __init__(self):
        self.calls = []

    def _pack(self, x, transpose, fmt="e4m3"):
        v = (x.t() if transpose else x).detach().clone()
        return Table(v, torch.zeros(0), v.shape[1], fmt)

    def pack4(self, x, transpose=False):
        self.calls.append("pack4_transposed" if transpose else "pack4")
        return self._pack(x, transpose)

    def pack4_both(self, x):
        self.calls.append("pack4_both")
        return self._pack(x, False), self._pack(x, True)

    def product4(self, x, w, bias=None, dtype=torch.float32):
        self.calls.append("product4")
        return (x.codes @ w.codes.t()).to(dtype)

    def pack(self, x, format="e4m3", transpose=False):
        return self._pack(x, transpose, format)

    def product(self, x, w, bias=None, dtype=torch.float32):
        return (x.codes @ w.codes.t()).to(dtype)

    def weight_gradient(self, x, g):
        return x.codes.t() @ g

    def group_norm(self, A, groups, gamma, beta, eps, activation, keep, pack_y, dense_y):
        """No norm at all: A gamma + beta."""
        out = Dense()
        out.x, out.y_packed = self._pack(A, False), self._pack(A * gamma + beta, False)
        out.mean, out.rstd = torch.zeros(1), torch.ones(1)
        return out

    def group_norm_backward(self, dH, A, mean, rstd, groups, gamma, beta, eps, activation):
        return dH * gamma, (dH * A.codes).sum(0), dH.sum(0)


@pytest.fixture
def dense(monkeypatch):
    d = Dense()
    monkeypatch.setattr(gcn, "dense", d)
    return d


def numbers(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).requires_grad_()


def transform8(X, W):
    return first(gcn._PackedTransform.apply(X, W, "e4m3", "e4m3"))


def norm_transform(X, W):
    gamma, beta = torch.linspace(0.5, 1.5, X.shape[1]), torch.linspace(-1, 1, X.shape[1])
    return first(gcn._NormTransform.apply(X, gamma, beta, W, 1, 1e-5, "none", "e4m3", "e4m3"))


def first(out):
    return out[0] if isinstance(out, tuple) else out


def plain_norm(X, W):
    return (X * torch.linspace(0.5, 1.5, X.shape[1]) + torch.linspace(-1, 1, X.shape[1])) @ W


LAYERS = {"transform4": (gcn.transform4, torch.matmul), "transform8": (transform8, torch.matmul),
          "norm": (norm_transform, plain_norm)}


@pytest.fixture(params=LAYERS)
def layer(request, dense):
    return LAYERS[request.param]


def test_first_derivatives(layer):
    call, plain = layer
    X, W, dZ = numbers(5, 4, seed=1), numbers(4, 3, seed=2), numbers(5, 3, seed=3).detach()
    for create in (False, True):
        got = torch.autograd.grad(call(X, W), (X, W), dZ, create_graph=create)
        for a, b in zip(got, torch.autograd.grad(plain(X, W), (X, W), dZ)):
            assert torch.allclose(a, b, rtol=0, atol=1e-5)


@pytest.mark.parametrize("create", [False, True])
def test_a_layer_within_a_checkpoint(layer, create):
    """The kept tensors are asked for once, as a checkpoint that computes them anew
    wants it."""
    call, plain = layer
    X, W = numbers(5, 4, seed=1), numbers(4, 3, seed=2)
    Z = checkpoint(call, X, W, use_reentrant=False)
    got = torch.autograd.grad(Z.sum(), (X, W), create_graph=create)
    for a, b in zip(got, torch.autograd.grad(plain(X, W).sum(), (X, W))):
        assert torch.allclose(a, b, rtol=0, atol=1e-5)


# ------------------------------------------------------ rows to experts and back ---
class Order:
    """A route of every row to two experts, its numbers on the CPU."""

    rows, k = 3, 2

    def __init__(self):
        self.place = torch.tensor([[0, 3], [4, 1], [2, -1]], dtype=torch.int32)
        self.source = torch.tensor([0, 1, 2, 0, 1, -1], dtype=torch.int32)

    def kept(self):
        return self.place, self.source


def sorted_rows(x, r):
    there = (r.source >= 0)[:, None]
    return torch.where(there, x[r.source.clamp(min=0).long()], torch.zeros(()))


def summed(y, r, weights=None):
    w = torch.ones(r.rows, r.k) if weights is None else weights
    return (torch.where(r.place >= 0, w, torch.zeros(()))[:, :, None] * y[r.place.clamp(min=0).long()]).sum(1)


def summed_backward(dout, y, r, weights=None, need_dy=True, need_dweights=True):
    at, there = r.place.clamp(min=0).long(), r.place >= 0
    dy = torch.zeros(r.rows * r.k, dout.shape[1])
    dy[at[there]] = (weights[:, :, None] * dout[:, None])[there]
    dweights = torch.where(there, (dout[:, None] * y[at]).sum(2), torch.zeros(())) if need_dweights else None
    return dy if need_dy else None, dweights


@pytest.fixture
def order(monkeypatch):
    """The stand-ins work on memory, as the library's calls do: torch sees an empty
    result of theirs and not how it is filled."""
    def raw(call):
        def on_memory(first, *args):
            values = [torch.from_numpy(v.detach().numpy()) if isinstance(v, torch.Tensor) else v
                      for v in (first, *args)]
            result = call(*values)
            out = first.detach().new_empty(result.shape)
            out.numpy()[:] = result.numpy()
            return out
        return on_memory

    def raw_backward(*args):
        return summed_backward(*(v.detach() if isinstance(v, torch.Tensor) else v for v in args))

    monkeypatch.setattr(experts, "_dispatch", raw(sorted_rows))
    monkeypatch.setattr(experts, "_combine", raw(summed))
    monkeypatch.setattr(experts, "combine_backward", raw_backward)
    return Order()


@pytest.mark.parametrize("create", [False, True])
@pytest.mark.parametrize("around", [lambda f, *v: f(*v), lambda f, *v: checkpoint(f, *v, use_reentrant=False)],
                         ids=["alone", "checkpoint"])
def test_rows_to_experts_and_back(order, around, create):
    x, w = numbers(3, 4, seed=1), numbers(3, 2, seed=2)

    def step(x, w):
        return experts.combine(experts.dispatch(x, order), order, w)

    got = torch.autograd.grad(around(step, x, w).sum(), (x, w), create_graph=create)
    for a, b in zip(got, torch.autograd.grad(summed(sorted_rows(x, order), order, w).sum(), (x, w))):
        assert torch.allclose(a, b, rtol=0, atol=1e-5)


# ----------------------------------------------------------- second derivatives ---
@pytest.mark.parametrize("unused", [False, True])
@pytest.mark.parametrize("of", ["X", "W"])
def test_second_derivatives_are_never_left_out(layer, of, unused):
    """The weights' gradient depends on X and that of X on the weights.  X and W come
    from tensors that other parts of the sum depend on too: without an error a gradient
    that lacks this part would come back."""
    call, _ = layer
    a, b = numbers(5, 4, seed=1), numbers(4, 3, seed=2)
    X, W = torch.sin(a), torch.cos(b)
    Z = call(X, W)
    g, = torch.autograd.grad(Z.sum(), W if of == "X" else X, create_graph=True)
    assert g.requires_grad
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(Z.sum() + g.square().sum(), a if of == "X" else b, allow_unused=unused)


def test_second_derivatives_by_the_output_gradient(layer):
    call, _ = layer
    X, W, dZ = numbers(5, 4, seed=1), numbers(4, 3, seed=2), numbers(5, 3, seed=3)
    for v in (X, W):
        g, = torch.autograd.grad(call(X, W), v, dZ, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(g.sum() + dZ.sum(), dZ)


@pytest.mark.parametrize("of", ["y", "weights"])
def test_second_derivatives_of_weighted_sums(order, of):
    a, b = numbers(6, 4, seed=1), numbers(3, 2, seed=2)
    y, w = torch.sin(a), torch.cos(b)
    out = experts.combine(y, order, w)
    g, = torch.autograd.grad(out.sum(), w if of == "y" else y, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(out.sum() + g.square().sum(), a if of == "y" else b)


def test_nothing_is_kept_for_second_derivatives(layer):
    """What a gradient hangs on is of no size."""
    call, _ = layer
    X, W = numbers(5, 4, seed=1), numbers(4, 3, seed=2)
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t), t)[1], lambda t: t):
        Z = call(X, W)
    assert not any(t.untyped_storage().data_ptr() in (X.untyped_storage().data_ptr(), Z.untyped_storage().data_ptr())
                   for t in seen)
    torch.autograd.grad(Z.sum(), (X, W))


# ------------------------------------------------------------------ forward mode ---
def test_forward_derivatives_are_refused(order, layer):
    """A tangent is never left out: torch names the function that has no rule for it."""
    import torch.autograd.forward_ad as forward

    x, y, w = torch.ones(3, 4), torch.ones(6, 4), torch.ones(3, 2)
    with forward.dual_level():
        dual = {v: forward.make_dual(v, torch.ones_like(v)) for v in (x, y, w)}
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                for f in (lambda: experts.dispatch(dual[x], order), lambda: experts.combine(dual[y], order),
                          lambda: experts.combine(dual[y], order, w), lambda: experts.combine(y, order, dual[w]),
                          lambda: experts.combine(dual[y], order, dual[w]),
                          lambda: layer[0](dual[x], torch.ones(4, 3))):
                    with pytest.raises(NotImplementedError, match="forward mode"):
                        f()
        # tensors without a tangent are as they were
        assert torch.equal(experts.dispatch(x, order), sorted_rows(x, order))
        assert torch.equal(experts.combine(y, order, w), summed(y, order, w))


def test_traced_calls_are_recorded(order):
    """A trace holds the call, and not the memory that its result had when it was traced."""
    def step(x, w):
        return experts.combine(experts.dispatch(x, order), order, w)

    traced = torch.jit.trace(step, (torch.ones(3, 4), torch.ones(3, 2)), check_trace=False)
    x, w = numbers(3, 4, seed=1).detach(), numbers(3, 2, seed=2).detach()
    assert torch.equal(traced(x, w), step(x, w))
    plain = torch.jit.trace(lambda x: experts.combine(experts.dispatch(x, order), order), torch.ones(3, 4),
                            check_trace=False)
    assert torch.equal(plain(x), experts.combine(experts.dispatch(x, order), order))


# ------------------------------------------------------- only what is asked for ---
@pytest.mark.parametrize("need_X,need_W,grad,forward,backward", [
    (True, True, True, ["pack4_both", "pack4_both", "product4"], ["pack4_both", "product4", "product4"]),
    (True, False, True, ["pack4", "pack4_both", "product4"], ["pack4", "product4"]),
    (False, True, True, ["pack4_both", "pack4_transposed", "product4"], ["pack4_transposed", "product4"]),
    (False, False, True, ["pack4", "pack4_transposed", "product4"], None),
    (True, True, False, ["pack4", "pack4_transposed", "product4"], None)])
def test_transform4_packs_what_is_needed(dense, need_X, need_W, grad, forward, backward):
    """X both ways only where the weights have a gradient, and nothing for a backward
    pass that gradients switched off will not run."""
    X, W = numbers(5, 4, seed=1).requires_grad_(need_X), numbers(4, 3, seed=2).requires_grad_(need_W)
    with torch.set_grad_enabled(grad):
        Z = gcn.transform4(X, W)
    assert dense.calls == forward
    assert torch.equal(Z.detach(), (X @ W).detach()) and Z.requires_grad == (backward is not None)
    if backward is not None:
        dense.calls = []
        Z.sum().backward()
        assert dense.calls == backward
