"""Every kernel of the 4-bit products by name (nibble_cases.py), each asked for before
it runs: results of every type with and without a bias, sums that are exact, NaN that
stays in its row and column, and for rows sorted by expert biases of their own, rows
without an expert and both orders of X."""
import numpy as np
import pytest

import nibble_cases as cases
import nibble_reference as ref
from test_gpu_nibble import HALF_ULP, TYPES, of, random_table, to64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2608_05033_amd as sd  # noqa: E402
from paper_2608_05033_amd import dense, experts  # noqa: E402


def takes(case, dtype, rows, cols, n, count=0):
    """The call takes the kernel that the case is named for."""
    assert sd.sd_nibble_product_form(rows, cols, n, count, dense.TYPES[TYPES[dtype]]) == cases.chosen(case, dtype)


def close(y, want, size, cols, dtype):
    """A block's products are summed exactly; each addition of a block's sum, of at most
    64 parts of the sum and of the bias is off by at most 2^-23 of the magnitudes summed.
    Then one rounding to the type."""
    bound = (-(-cols // 32) + 66) * 2.0 ** -23 * size
    if dtype != "f32":
        bound = bound + HALF_ULP[dtype] * np.abs(want) + 2.0 ** -25
    err = np.abs(to64(y) - want)
    assert np.all(err <= bound + 1e-37), float((err - bound).max())
    if dtype == "f32":
        assert np.linalg.norm(err) <= 2e-7 * np.linalg.norm(size)


def smaller(table, by):
    """The same codes at scales 2^by lower."""
    return dense.Packed4(table.codes, (table.scales.to(torch.int32) - by).to(torch.uint8), table.cols)


@pytest.mark.parametrize("name", cases.PRODUCTS)
def test_products(name):
    case = cases.PRODUCTS[name]
    rows, cols, n = case[0]
    X, W = random_table(rows, cols, 1, 2), smaller(random_table(n, cols, 2, 2), 7)
    x, w = of(X), of(W)
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    b = np.random.default_rng(3).standard_normal(n).astype(np.float32)
    B, b = torch.from_numpy(b).cuda(), b.astype(np.float64)
    for dtype in TYPES:
        print(f"case {name} {rows}x{cols}x{n} {dtype}", flush=True)
        takes(case, dtype, rows, cols, n)
        close(dense.product4(X, W, dtype=TYPES[dtype]), want, size, cols, dtype)
        close(dense.product4(X, W, B, TYPES[dtype]), want + b, size + np.abs(b), cols, dtype)


@pytest.mark.parametrize("name", cases.PRODUCTS)
def test_exact_sums_and_nan(name):
    """Whole quarters below 2^22 at every step, to fp32; to 16 bits the same, rounded
    once.  A NaN in the last block of one row of each side stays in that row and column,
    and scales behind the last block take no part."""
    case = cases.PRODUCTS[name]
    rows, cols, n = case[0]
    X, W = random_table(rows, cols, 4, 0), random_table(n, cols, 5, 0)
    want = torch.from_numpy(of(X) @ of(W).T).float()
    last = (cols - 1) // 32
    for p, row in ((X, rows // 2), (W, n - 1)):
        p.scales[last // 4, row, last % 4] = 255
        p.scales[last // 4, :, last % 4 + 1:] = 255
    want[rows // 2], want[:, n - 1] = float("nan"), float("nan")
    for dtype, t in TYPES.items():
        print(f"case {name} {rows}x{cols}x{n} {dtype}", flush=True)
        takes(case, dtype, rows, cols, n)
        got = dense.product4(X, W, dtype=t).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got, 0), torch.nan_to_num(want.to(t), 0))


@pytest.mark.parametrize("name", cases.EXPERTS)
def test_experts(name):
    """Some experts more in demand than others, one without rows where there are
    enough, one entry in twenty without an expert."""
    case = cases.EXPERTS[name]
    rows, k, count, cols, n = case[0]
    g = np.random.default_rng(rows)
    c = np.minimum(g.integers(0, count, (rows, k)), g.integers(0, count + 1, (rows, k)))
    if count > 4:
        c[c == 1] = 2
    c[g.random((rows, k)) < 0.05] = -1
    r = experts.route(torch.from_numpy(c).cuda(), count)
    X, W = random_table(rows, cols, 6, 2), smaller(random_table(count * n, cols, 7, 2), 7)
    at = r.source.clamp(min=0).long()
    Xs = dense.Packed4(X.codes[at], X.scales[:, at].contiguous(), cols)
    x, w = of(X), of(W).reshape(count, n, cols)
    b = g.standard_normal((count, n)).astype(np.float32)
    B = torch.from_numpy(b).cuda()
    offsets, _, source = ref.route_fast(c, count)
    want, size = np.zeros((rows * k, n)), np.zeros((rows * k, n))
    biases = np.zeros((rows * k, n))
    for e in range(count):
        lo, hi = offsets[e], offsets[e + 1]
        want[lo:hi] = x[source[lo:hi]] @ w[e].T
        size[lo:hi] = np.abs(x[source[lo:hi]]) @ np.abs(w[e]).T
        biases[lo:hi] = b[e]
    have = offsets[count]
    for dtype, t in TYPES.items():
        print(f"case experts {name} {rows}x{k} of {count}, {cols} to {n} {dtype}", flush=True)
        takes(case, dtype, rows * k, cols, n, count)
        for bias, add in ((None, 0 * biases), (B, biases)):
            y = experts.product(X, W, r, bias, t)
            close(y[:have], want[:have] + add[:have], size[:have] + np.abs(add[:have]), cols, dtype)
            assert not y[have:].any()
            assert torch.equal(y, experts.product(Xs, W, r, bias, t, sorted=True))
    # a NaN in one row of X reaches that row's entries alone, one in the weights its expert's column alone
    X.scales[0, 0, 0] = 255
    W.scales[0, int(c.max()) * n, 0] = 255
    first, column = source[:have] == 0, np.zeros((have, n), bool)
    column[offsets[c.max()]:offsets[c.max() + 1], 0] = True
    for t in TYPES.values():
        nan = torch.isnan(experts.product(X, W, r, None, t)).cpu().numpy()
        assert np.array_equal(nan[:have], first[:, None] | column) and not nan[have:].any()
