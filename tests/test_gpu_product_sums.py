"""Products of 8-bit tables are summed in 32 bits whatever the result's type:
sums that cancel, codes of very different sizes side by side, and the error of
16-bit results before their one rounding."""
import numpy as np
import pytest

import dense_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_05033_amd import dense  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# rows, n: one row, few, a table long and narrow, tiles of every size (256 compute units)
SIZES = [(1, 64), (64, 200), (500, 700), (700, 1000), (1100, 1030), (2100, 1700), (3500, 3580), (13000, 60), (13000, 120)]


def packed(x, fmt="e4m3"):
    p = dense.pack(torch.from_numpy(np.ascontiguousarray(x)).float().cuda(), fmt)
    return p, ref.values(p.codes.cpu().numpy(), p.scales.cpu().numpy(), p.cols, fmt)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n", SIZES)
def test_what_is_left_of_large_terms_that_cancel(rows, n, dtype):
    """Each run of 8 neighbouring k holds 256 and -256 times 256, a zero times the
    largest code, and a small product; every partial sum has at most 24 bits, so
    the result is exact."""
    print(f"case cancelling {rows}x{n} {dtype}", flush=True)
    cols = 128
    x, w = np.zeros((rows, cols)), np.zeros((n, cols))
    x[:, 0::8], w[:, 0::8] = 256, 256
    x[:, 1::8], w[:, 1::8] = -256, 256
    x[:, 2::8], w[:, 2::8] = 0, 448
    x[:, 3::8], w[:, 3::8] = 0.5, 0.5
    x[:, 4::8], w[:, 4::8] = 448, 0
    X, x64 = packed(x)
    W, w64 = packed(w)
    assert np.array_equal(x64, x) and np.array_equal(w64, w)
    y = dense.product(X, W, dtype=TYPES[dtype])
    assert torch.equal(y, torch.full_like(y, 4.0))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("x_fmt,w_fmt", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("rows,n", [(5, 70), (130, 260), (2100, 1700)])
def test_codes_of_all_sizes(rows, n, x_fmt, w_fmt, dtype):
    """Magnitudes over the formats' whole range, subnormal codes and zeros among
    them.  Each of the cols + 1 additions is off by at most 2^-24 of the magnitudes
    summed, then the result is rounded once."""
    print(f"case all sizes {rows}x{n} {x_fmt} {w_fmt} {dtype}", flush=True)
    cols, g = 300, np.random.default_rng(rows)

    def table(r, fmt):
        span = {"e4m3": (-10, 9), "e5m2": (-17, 16)}[fmt]
        v = np.ldexp(g.choice([-1.0, 0.0, 1.0], (r, cols), p=[0.45, 0.1, 0.45]) * (1 + g.random((r, cols))),
                     g.integers(*span, (r, cols)))
        top = ref.FORMATS[fmt][2]
        v = np.clip(v, -top, top)
        v[:, ::128] = top  # the scale is 1
        return v

    # f16 holds results below 65504
    X, x64 = packed(table(rows, x_fmt) * 2.0 ** -40, x_fmt)
    W, w64 = packed(table(n, w_fmt) * 2.0 ** 20, w_fmt)
    want, size = x64 @ w64.T, np.abs(x64) @ np.abs(w64).T
    got = dense.product(X, W, dtype=TYPES[dtype]).double().cpu().numpy()
    bound = (cols + 2) * 2.0 ** -24 * size
    if dtype != "f32":
        bound = bound + HALF_ULP[dtype] * np.abs(want) * 1.001
    if dtype == "f16":
        bound = bound + 2.0 ** -25
    assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,n", SIZES)
def test_error_before_the_rounding(rows, n, dtype):
    """All rows alike and a bias of minus the result: what is left is the sum's own
    error.  In 2-norm that is 1e-6 of the result as for 32-bit results, 2^-24 of it
    for the bias's rounding among it."""
    print(f"case before rounding {rows}x{n} {dtype}", flush=True)
    cols, g = 640, np.random.default_rng(n)
    X, x64 = packed(np.repeat(g.standard_normal((1, cols)), rows, 0))
    W, w64 = packed(g.standard_normal((n, cols)))
    want = x64[0] @ w64.T
    bias = torch.from_numpy(-want).float().cuda()
    left = dense.product(X, W, bias, TYPES[dtype]).double().cpu().numpy()
    err = left - (want + bias.double().cpu().numpy())
    assert np.linalg.norm(err) <= 1e-6 * np.linalg.norm(np.broadcast_to(want, err.shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("power", [-100, -118, -126, -133, -140])
def test_numbers_at_the_end_of_bf16(power, fmt, dtype):
    """Tables of tiny numbers times large ones: a number of the table is off by at most
    half of 2^-133, the least one of bf16, and by nothing where it is a multiple."""
    g = np.random.default_rng(-power)
    X, x64 = packed(g.standard_normal((40, 200)) * 2.0 ** power, fmt)
    W, w64 = packed(g.standard_normal((30, 200)) * 2.0 ** 110)
    held = np.round(x64 / 2.0 ** -133) * 2.0 ** -133  # to nearest, ties to even
    if power >= (-110 if fmt == "e4m3" else -100):
        assert np.array_equal(held, x64)
    want, size = held @ w64.T, np.abs(held) @ np.abs(w64).T
    got = dense.product(X, W, dtype=TYPES[dtype]).double().cpu().numpy()
    assert np.all(np.abs(got - want) <= 202 * 2.0 ** -24 * size + HALF_ULP[dtype] * 1.001 * np.abs(want))


@pytest.mark.parametrize("power", [-100, -118, -126, -133])
def test_gradients_of_tiny_numbers(power):
    """G of fp32 is cut into terms of bf16: what is under 2^-133 is left out of a number."""
    g = np.random.default_rng(-power)
    X, x64 = packed(g.standard_normal((300, 20)) * 2.0 ** 100)
    G = (g.standard_normal((300, 24)) * 2.0 ** power).astype(np.float32)
    got = dense.weight_gradient(X, torch.from_numpy(G).cuda()).double().cpu().numpy()
    want, size = x64.T @ G.astype(np.float64), np.abs(x64).T @ np.abs(G.astype(np.float64))
    assert np.all(np.abs(got - want) <= (300 / 16 + 64) * 2.0 ** -24 * size + np.abs(x64).sum(0)[:, None] * 2.0 ** -133)
