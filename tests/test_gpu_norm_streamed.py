"""Group norm whose 16-bit results are 64 MB or more and go past the caches: all
of the result against 64 bits, whole vectors of channels and others, segments
long and short."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_05033_amd import dense  # noqa: E402

HALF_ULP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("channels", [128, 132, 130])
@pytest.mark.parametrize("length", [32, 1 << 17])
def test_large_results_in_16_bits(length, channels, dtype):
    """The bounds are those of 32-bit arithmetic on the numbers that form a value
    (2^-20 of them forward, 2^-19 backward), then one rounding."""
    print(f"case streamed length {length} channels {channels} {dtype}", flush=True)
    segments, groups = -(-(1 << 18) // length) + 1, 2
    rows = segments * length
    assert rows * channels * 2 >= 64 << 20
    g = torch.Generator(device="cuda").manual_seed(channels + length)
    x = (torch.randn(rows, channels, generator=g, device="cuda") + 0.5).to(dtype)
    dy = torch.randn(rows, channels, generator=g, device="cuda").mul_(0.1).to(dtype)
    w = 1 + 0.2 * torch.randn(channels, generator=g, device="cuda")
    b = 0.2 * torch.randn(channels, generator=g, device="cuda")
    out = dense.group_norm(x, groups, w, b, 1e-5, "silu", segments=segments)
    dx, _, _ = dense.group_norm_backward(dy, x, out.mean, out.rstd, groups, w, b, 1e-5, "silu", segments=segments)

    per = channels // groups
    for s0 in range(0, segments, max(1, segments // 4)):  # a part of the segments at a time
        s1 = min(segments, s0 + max(1, segments // 4))
        part = slice(s0 * length, s1 * length)
        v = x[part].double().view(s1 - s0, length, groups, per)
        ww, bb = w.double().view(1, 1, groups, per), b.double().view(1, 1, groups, per)
        mean = v.mean((1, 3), keepdim=True)
        rstd = (((v - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5) ** -0.5
        xh = (v - mean) * rstd
        z = xh * ww + bb
        p = torch.sigmoid(z)
        size = (v.abs() + mean.abs()) * rstd * ww.abs() + bb.abs() + z.abs()
        y = out.y[part].double().view_as(v)
        assert ((y - z * p).abs() <= 2.0 ** -20 * size + HALF_ULP[dtype] * 1.01 * (z * p).abs() + 2.0 ** -24).all()
        d = dy[part].double().view_as(v)
        dh = d * (p + z * p * (1 - p)) * ww
        want = rstd * (dh - dh.mean((1, 3), keepdim=True) - xh * (dh * xh).mean((1, 3), keepdim=True))
        dw = (d * ww).abs()
        size = rstd * (dw + dw.mean((1, 3), keepdim=True) + xh.abs() * (dw * xh.abs()).mean((1, 3), keepdim=True))
        grown = 1 + float(v.abs().max() * rstd.max())
        got = dx[part].double().view_as(v)
        assert ((got - want).abs() <= 2.0 ** -19 * grown * size + HALF_ULP[dtype] * 1.01 * want.abs() + 2.0 ** -24).all()
