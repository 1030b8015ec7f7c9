"""What autograd makes of the GCN with 8-bit node tables: the features' gradient,
second derivatives, tables changed under way, parameters that stand still."""
import pytest

import gen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

import scipy.sparse  # noqa: E402

from paper_2608_05033_amd import dense, gcn  # noqa: E402

IN, HIDDEN, CLASSES, GROUPS = 48, 32, 8, 4


@pytest.fixture(scope="module")
def case():
    A = gen.rmat(10, 12000, nmax=1000, seed=3)
    X = torch.from_numpy(gen.dense_normal(A.m, IN, seed=1)).cuda()
    R = torch.from_numpy(gen.dense_normal(A.m, CLASSES, seed=2)).cuda()
    model = gcn.GCN2Packed(A, IN, HIDDEN, CLASSES, device="cuda", seed=5, groups=GROUPS, activation="silu")
    yield A, X, R, model
    model.agg.destroy()


def grads(model, X, R):
    """Gradients of sum(logits R): the parameters', by name, and the features'."""
    for p in model.parameters():
        p.grad = None
    (model(X) * R).sum().backward()
    out = {name: None if p.grad is None else p.grad.clone() for name, p in model.named_parameters()}
    out["X"] = X.grad if isinstance(X, torch.Tensor) else None
    return out


# ------------------------------------------------------ features' gradient ---
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_features_have_a_gradient(case, dtype):
    """Against the 64-bit network without roundings: a value rounded to 4 significant
    bits moves by 2.6 % rms at most, and this gradient goes through six such tables
    (X, A1, H1, two output gradients, two weights), so it stays within 0.15 in
    2-norm, as the parameters' do."""
    A, X, R, model = case
    X = X.to(dtype, copy=True).requires_grad_()
    got = grads(model, X, R)["X"]
    assert got.dtype == dtype and got.shape == X.shape

    dense_A = torch.from_numpy(scipy.sparse.csr_matrix((A.values, A.colidx, A.rowptr), shape=(A.m, A.k)).toarray()).double()
    x = X.detach().double().cpu().requires_grad_()
    p = {k: v.detach().double().cpu() for k, v in model.named_parameters()}
    v = (dense_A @ (x @ p["W1"])).view(A.m, GROUPS, -1)
    mean = v.mean((0, 2), keepdim=True)
    xh = (v - mean) / torch.sqrt(((v - mean) ** 2).mean((0, 2), keepdim=True) + model.eps)
    z = xh.reshape(A.m, HIDDEN) * p["gamma"] + p["beta"]
    ((dense_A @ ((z * torch.sigmoid(z)) @ p["W2"])) * R.double().cpu()).sum().backward()
    assert (got.double().cpu() - x.grad).norm() <= 0.15 * x.grad.norm()


def test_parameters_gradients_do_not_depend_on_the_features(case):
    """The same bits with features that require a gradient, that do not, and packed."""
    _, X, R, model = case
    first = grads(model, X.clone().requires_grad_(), R)
    for other in (X, dense.pack(X, model.format)):
        again = grads(model, other, R)
        assert again["X"] is None
        for name, _ in model.named_parameters():
            assert torch.equal(again[name], first[name]), name


# ----------------------------------------------------- second derivatives ---
@pytest.mark.parametrize("loss", [lambda y, R: (y * R).sum(), lambda y, R: y.square().sum()], ids=["linear", "square"])
@pytest.mark.parametrize("of", ["W1", "gamma", "W2", "X"])
def test_second_derivatives_are_refused(case, of, loss):
    """The kernels' gradients have no derivatives of their own: asking for them
    beside others that are there is an error, not a sum without those terms."""
    _, X, R, model = case
    X = X.clone().requires_grad_()
    v = X if of == "X" else getattr(model, of)
    g, = torch.autograd.grad(loss(model(X), R), v, create_graph=True)
    plain, = torch.autograd.grad(loss(model(X), R), v)
    assert torch.equal(g, plain)
    with pytest.raises(RuntimeError, match="second derivatives"):
        (g.square().sum() + v.square().sum()).backward()


# ------------------------------------------------- tables changed under way ---
@pytest.mark.parametrize("part", ["codes", "scales"])
def test_a_packed_table_written_between_the_passes_is_noticed(case, part):
    """The backward pass reads the features once more; written in between, they are
    not what the forward pass read, and autograd says so as for any tensor."""
    _, X, R, model = case
    X8 = dense.pack(X, model.format)
    loss = (model(X8) * R).sum()
    getattr(X8, part).zero_()
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()


def test_kept_tables_go_through_autograds_hooks(case):
    """Kept tables moved to the host between the passes, as torch's own hook does it,
    give the same gradients."""
    _, X, R, model = case
    want = grads(model, X.clone().requires_grad_(), R)
    seen = []

    def away(t):
        seen.append(t.dtype)
        return t.device, t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(away, lambda kept: kept[1].to(kept[0])):
        got = grads(model, X.clone().requires_grad_(), R)
    assert seen.count(torch.uint8) == 6
    for name, g in want.items():
        assert torch.equal(got[name], g), name


# --------------------------------------------- parameters that stand still ---
@pytest.mark.parametrize("still,calls", [(["W1"], {"weight_gradient": 1, "group_norm_backward": 1}),
                                         (["W2"], {"weight_gradient": 1, "group_norm_backward": 1}),
                                         (["W1", "gamma", "beta"], {"weight_gradient": 1, "group_norm_backward": 0}),
                                         (["W1", "W2", "beta"], {"weight_gradient": 0, "group_norm_backward": 1})])
def test_gradients_that_nobody_needs_are_not_computed(case, still, calls, monkeypatch):
    """The others keep their bits."""
    _, X, R, model = case
    want = grads(model, X, R)
    counted = dict.fromkeys(calls, 0)

    def counting(name, call):
        def counted_call(*args, **kw):
            counted[name] += 1
            return call(*args, **kw)
        return counted_call

    for name in calls:
        monkeypatch.setattr(dense, name, counting(name, getattr(dense, name)))
    try:
        for name in still:
            getattr(model, name).requires_grad_(False)
        got = grads(model, X, R)
    finally:
        for p in model.parameters():
            p.requires_grad_(True)
    assert counted == calls
    for name, _ in model.named_parameters():
        assert got[name] is None if name in still else torch.equal(got[name], want[name]), name
