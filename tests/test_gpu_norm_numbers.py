"""Group norm where numbers are out of the ordinary: eps 0, empty segments,
little spread around a large mean, magnitudes far from 1.  Segments are given so
that both ways of running, teams and chunks, meet each case."""
import numpy as np
import pytest

import dense_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_05033_amd import dense  # noqa: E402


def to64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def gpu(x, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


# --------------------------------------------------- eps 0, empty segments ---
@pytest.mark.parametrize("keep", [None, "e4m3"])
@pytest.mark.parametrize("channels,groups", [(16, 2), (96, 6), (132, 3)])
@pytest.mark.parametrize("cuts", [[0, 0, 11, 11, 30, 40], [0, 7, 7, 7, 19], [0, 0, 5, 9, 9], [0, 0, 6000, 6000, 9000]])
def test_gradients_beside_empty_segments_without_eps(cuts, channels, groups, keep):
    """An empty segment's rstd is infinite with eps 0; it has no rows, so nothing of
    it is in any gradient.  Bounds as for segments that have rows."""
    print(f"case empty segments {cuts} channels {channels} keep {keep}", flush=True)
    off, g = np.array(cuts), np.random.default_rng(channels + len(cuts))
    rows = int(off[-1])
    x = g.standard_normal((rows, channels)).astype(np.float32).astype(np.float64)
    dy = g.standard_normal((rows, channels)).astype(np.float32).astype(np.float64)
    w = (1 + 0.2 * g.standard_normal(channels)).astype(np.float32)
    how = {"offsets": gpu(off, torch.int32), "eps": 0.0, "activation": "silu"}
    out = dense.group_norm(gpu(x), groups, gpu(w), keep=keep, **how)
    seen = x if keep is None else ref.values(out.x.codes.cpu().numpy(), out.x.scales.cpu().numpy(), channels, keep)
    got = dense.group_norm_backward(gpu(dy), out.x, out.mean, out.rstd, groups, gpu(w), **how)
    mean, rstd = to64(out.mean), to64(out.rstd)
    empty = np.diff(off) == 0
    assert np.isposinf(rstd[empty]).all() and (mean[empty] == 0).all() and np.isfinite(rstd[~empty]).all()
    dx, dw, db, size, size_w, size_b, _ = ref.norm_backward(dy, seen, mean, rstd, groups, w.astype(np.float64), None,
                                                            "silu", off)
    grown = 1 + np.abs(seen).max() * rstd[~empty].max()
    assert np.all(np.abs(to64(got[0]) - dx) <= 2.0 ** -19 * grown * size)
    assert np.all(np.abs(to64(got[1]) - dw) <= 2.0 ** -19 * grown * (size_w + size_b))
    assert np.all(np.abs(to64(got[2]) - db) <= 2.0 ** -19 * grown * size_b)


# ------------------------------------------- little spread, a large mean ---
WAYS = [  # rows, channels, groups, cuts: teams, chunks, pieces of both
    (33, 24, 2, [0, 33]), (700, 35, 7, [0, 3, 3, 500, 700]), (5000, 24, 2, [0, 5000]), (100000, 32, 4, [0, 100000]),
    (9000, 130, 10, [0, 1, 4097, 4097, 9000]), (300, 1028, 4, [0, 120, 300])]


def cut(cuts):
    return {"offsets": gpu(np.array(cuts), torch.int32)}


@pytest.mark.parametrize("dtype,value", [(torch.float32, 1234567.0), (torch.float32, -3.3333334e7), (torch.float32, 0.1),
                                         (torch.bfloat16, 999424.0), (torch.float16, 60032.0), (torch.float32, 3e-7)])
@pytest.mark.parametrize("rows,channels,groups,cuts", WAYS)
def test_constant_groups_have_no_variance(rows, channels, groups, cuts, value, dtype):
    """All numbers of a group alike: mean is the number, rstd is eps^-1/2 to a
    rounding of its operations, y is 0 and dx is rstd (dh - mean(dh))."""
    print(f"case constant {value} {rows}x{channels} {dtype}", flush=True)
    x = torch.full((rows, channels), value, device="cuda").to(dtype)
    out = dense.group_norm(x, groups, **cut(cuts))
    full = np.diff(cuts) > 0
    assert (out.y == 0).all()
    assert (out.mean[gpu(full, torch.bool)] == x[0, 0].float()).all() and (out.mean[gpu(~full, torch.bool)] == 0).all()
    assert np.allclose(to64(out.rstd), 1e-5 ** -0.5, rtol=2.0 ** -21, atol=0)
    dy = np.random.default_rng(rows).standard_normal((rows, channels)).astype(np.float32).astype(np.float64)
    dy = to64(gpu(dy, dtype))
    dx, dw, db = dense.group_norm_backward(gpu(dy, dtype), x, out.mean, out.rstd, groups, **cut(cuts))
    want, _, want_b, size, _, size_b, _ = ref.norm_backward(dy, to64(x), to64(out.mean), to64(out.rstd), groups, None, None,
                                                           "none", np.array(cuts))
    half_ulp = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    assert np.all(np.abs(to64(dx) - want) <= 2.0 ** -19 * size + half_ulp * 1.01 * np.abs(want) + 2.0 ** -25)
    assert not dw.any() and np.all(np.abs(to64(db) - want_b) <= 2.0 ** -19 * size_b)


@pytest.mark.parametrize("first", [None, 0.0, 3e7])
@pytest.mark.parametrize("mean,spread", [(1e6, 0.5), (1e7, 3.0), (-12345.0, 0.01)])
@pytest.mark.parametrize("rows,channels,groups,cuts", WAYS)
def test_little_spread_around_a_large_mean(rows, channels, groups, cuts, mean, spread, first):
    """Spreads of a few units in the last place of the numbers, at the usual eps;
    with a first number of each segment that is far from the others too.  rstd is
    right to some roundings of 2^-24, the mean to one of its own."""
    print(f"case spread {spread} around {mean}, first {first}, {rows}x{channels}", flush=True)
    g = np.random.default_rng(rows + channels)
    x = (mean + spread * g.standard_normal((rows, channels))).astype(np.float32)
    if first is not None:
        x[[c for c in cuts[:-1] if c < rows]] = first
    out = dense.group_norm(gpu(x), groups, **cut(cuts))
    _, want_mean, want_rstd, _, _ = ref.norm(x.astype(np.float64), groups, None, None, 1e-5, "none", cuts)
    assert np.allclose(to64(out.rstd), want_rstd, rtol=2e-6, atol=0)
    assert np.allclose(to64(out.mean), want_mean, rtol=2.0 ** -23, atol=0)


# --------------------------------------------------- magnitudes far from 1 ---
@pytest.mark.parametrize("power", [-100, -80, -63, 0, 66, 90, 100])
@pytest.mark.parametrize("rows,channels,groups,cuts", WAYS)
def test_magnitudes_far_from_one(rows, channels, groups, cuts, power):
    """Without eps, numbers times a power of two have the same xh, y, dweight and
    dbias, and dx over that power, whatever becomes of their squares in 32 bits.
    The bounds are those of ordinary numbers."""
    print(f"case 2^{power} {rows}x{channels}", flush=True)
    g, off, kind = np.random.default_rng(channels), np.array(cuts), "silu"
    x = np.ldexp((g.standard_normal((rows, channels)) + 0.5).astype(np.float32).astype(np.float64), power)
    w = (1 + 0.2 * g.standard_normal(channels)).astype(np.float32).astype(np.float64)
    b = (0.2 * g.standard_normal(channels)).astype(np.float32).astype(np.float64)
    dy = g.standard_normal((rows, channels)).astype(np.float32).astype(np.float64)
    how = {"offsets": gpu(off, torch.int32), "eps": 0.0, "activation": kind}
    t = gpu(x)
    assert np.array_equal(to64(t), x)
    out = dense.group_norm(t, groups, gpu(w), gpu(b), **how)
    y, mean, rstd, xh, z = ref.norm(x, groups, w, b, 0.0, kind, off)
    full = np.diff(off) > 0
    assert np.allclose(to64(out.rstd)[full], rstd[full], rtol=2e-6, atol=0)
    per, seg = channels // groups, np.repeat(np.arange(len(off) - 1), np.diff(off))
    spread = lambda v: np.repeat(v[seg], per, axis=1)  # noqa: E731
    size = (np.abs(x) + np.abs(spread(mean))) * spread(rstd) * np.abs(w) + np.abs(b) + np.abs(z)
    assert np.all(np.abs(to64(out.y) - y) <= 2.0 ** -20 * size)
    got = dense.group_norm_backward(gpu(dy), t, out.mean, out.rstd, groups, gpu(w), gpu(b), **how)
    dx, dw, db, size, size_w, size_b, _ = ref.norm_backward(dy, x, to64(out.mean), to64(out.rstd), groups, w, b, kind, off)
    grown = 1 + np.abs(x).max() * rstd[full].max()
    assert np.all(np.abs(to64(got[0]) - dx) <= 2.0 ** -19 * grown * size)
    assert np.all(np.abs(to64(got[1]) - dw) <= 2.0 ** -19 * grown * (size_w + size_b))
    assert np.all(np.abs(to64(got[2]) - db) <= 2.0 ** -19 * grown * size_b)
