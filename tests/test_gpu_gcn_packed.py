"""The GCN with a group norm and 8-bit node tables: one step against the fp64
network without rounding, its own gradients against differences along the
gradient, and a short training run."""
import numpy as np
import pytest

import gen
import dense_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

import scipy.sparse  # noqa: E402

from paper_2608_05033_amd import dense, gcn  # noqa: E402


def graph(seed):
    return gen.rmat(11, 25000, nmax=2000, seed=seed)


def exact_step(A, X, labels, model):
    """fp64 loss and gradients of the network without 8-bit roundings."""
    Ah = scipy.sparse.csr_matrix((A.values.astype(np.float64), A.colidx, A.rowptr), shape=(A.m, A.k))
    get = lambda p: p.detach().cpu().numpy().astype(np.float64)  # noqa: E731
    W1, W2, gamma, beta, X = get(model.W1), get(model.W2), get(model.gamma), get(model.beta), X.astype(np.float64)
    off = np.array([0, A.m])
    P1 = Ah @ (X @ W1)
    H1, mean, rstd, _, _ = ref.norm(P1, model.groups, gamma, beta, model.eps, model.activation, off)
    P2 = Ah @ (H1 @ W2)
    z = P2 - P2.max(axis=1, keepdims=True)
    prob = np.exp(z) / np.exp(z).sum(axis=1, keepdims=True)
    loss = -np.mean(np.log(prob[np.arange(A.m), labels]))
    prob[np.arange(A.m), labels] -= 1.0
    dZ2 = Ah.T @ (prob / A.m)
    dP1, dgamma, dbeta = ref.norm_backward(dZ2 @ W2.T, P1, mean, rstd, model.groups, gamma, beta, model.activation,
                                           off)[:3]
    return loss, {"W1": X.T @ (Ah.T @ dP1), "W2": H1.T @ dZ2, "gamma": dgamma, "beta": dbeta}


@pytest.mark.parametrize("activation", ["relu", "silu"])
def test_step_against_the_network_without_roundings(activation):
    """Rounding to 4 significant bits moves a value by 2.6 % rms at most; a
    gradient goes through four such tables (X, A1, H1, dZ) and two weights, so
    it stays within 0.15 of the exact one in 2-norm, and the loss closer."""
    A = graph(7)
    X = gen.dense_normal(A.m, 48, seed=1)
    labels = (np.arange(A.m) * 7919 % 8).astype(np.int64)
    model = gcn.GCN2Packed(A, 48, 32, 8, device="cuda", seed=5, groups=4, activation=activation)
    try:
        out = model(torch.from_numpy(X).cuda())
        loss = torch.nn.functional.cross_entropy(out, torch.from_numpy(labels).cuda())
        loss.backward()
        want, grads = exact_step(A, X, labels, model)
        assert abs(loss.item() - want) <= 0.02 * want
        for name, g in grads.items():
            got = getattr(model, name).grad.cpu().numpy()
            assert np.linalg.norm(got - g) <= 0.15 * np.linalg.norm(g), name
    finally:
        model.agg.destroy()


@pytest.mark.parametrize("packed_once", [False, True])
def test_training_reduces_loss(packed_once):
    """Labels a fixed random GCN can produce; 40 Adam epochs cut the loss as they
    do for the network in fp32."""
    A = graph(11)
    X = torch.from_numpy(gen.dense_normal(A.m, 32, seed=2)).cuda()
    teacher = gcn.GCN2(A, 32, 16, 4, device="cuda", seed=99)
    student = gcn.GCN2Packed(A, 32, 16, 4, device="cuda", seed=1, groups=4)
    try:
        with torch.no_grad():
            labels = teacher(X).argmax(dim=1)
        opt = torch.optim.Adam(student.parameters(), lr=0.02)
        data = dense.pack(X, student.format) if packed_once else X
        losses = [gcn.train_epoch(student, data, labels, opt).item() for _ in range(40)]
        print(f"packed gcn training loss {losses[0]:.4f} -> {losses[-1]:.4f}", flush=True)
        assert all(np.isfinite(losses)) and losses[-1] < 0.7 * losses[0]
    finally:
        teacher.agg.destroy()
        student.agg.destroy()
