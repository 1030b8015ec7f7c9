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
