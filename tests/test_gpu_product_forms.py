"""Every form of the product of 8-bit tables.  Which one runs follows from how
many tiles the result has against the card's compute units; the sizes here are
made from that number, so each of them takes the form it is named for."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2608_05033_amd as sd  # noqa: E402
from paper_2608_05033_amd import dense  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CUS = torch.cuda.get_device_properties(0).multi_processor_count
ENOUGH = 3 * CUS // 4  # workgroups a form needs before a larger tile is taken


# ------------------------------------------------------- tables of no columns ---
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,n", [(7, 40), (64 * ENOUGH, 1), (64 * ENOUGH + 13, 47), (64 * ENOUGH + 700, 128),
                                    (128 * ENOUGH + 5, 100), (3500, 3580), (1000, 1030)])
def test_no_columns(rows, n, dtype):
    """A sum over nothing: the bias, or zeros.  There are no codes and no scales to
    read, and their pointers may be null."""
    print(f"case no columns {rows}x0x{n} {dtype}", flush=True)
    X, W = dense.pack(torch.zeros(rows, 0, device="cuda")), dense.pack(torch.zeros(n, 0, device="cuda"))
    bias = torch.linspace(-3, 5, n, device="cuda")
    assert not dense.product(X, W, dtype=TYPES[dtype]).any()
    assert torch.equal(dense.product(X, W, bias, TYPES[dtype]), bias.to(TYPES[dtype]).expand(rows, n))


# ------------------------------------------------------------- every form ---
A = next(a for a in range(1, 100) if a * a >= ENOUGH)  # A x A tiles are enough
# rows, n, columns of the tables: one block and several, odd and even numbers of
# them, whole and ending inside a block, a few codes past 16 among them
FORMS = {
    "tiles 256 x 256": (256 * A - 85, 256 * A - 13, (40, 384, 513, 1024)),
    "tiles 128 x 128": (128 * A - 50, 128 * A - 9, (40, 384, 513, 1024)),
    "tiles 128 x 128, long": (128 * ENOUGH + 5, 100, (513, 640, 700)),
    "64 x 64": (64 * A - 21, 64 * A - 3, (40, 384, 513, 1025)),
    "32 x 64": (32 * A - 3, 64 * A - 5, (40, 384, 513, 1025)),
    "32 x 32": (32 * A - 7, 32 * A - 3, (40, 384, 513, 1025)),
    "16 x 16": (130, 261, (40, 384, 513, 2050)),
    "narrow, 64": (64 * ENOUGH + 13, 47, (16, 128, 300, 512)),
    "narrow, 128": (64 * ENOUGH + 700, 121, (17, 256, 300, 512)),
}
HALF_ULP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def operand(rows, cols, fmt, g, size=1.0):
    """A packed table whose rows lie further apart than they have to, with NaN
    codes in between, and its values in 64 bits."""
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    p = dense.pack(x * size, fmt)
    wide = torch.full((rows, p.codes.shape[1] + 48), 0x7F, dtype=torch.uint8, device="cuda")
    wide[:, :p.codes.shape[1]] = p.codes
    return dense.Packed(wide, p.scales, cols, fmt), dense.unpack(p).double()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("form", FORMS)
def test_every_form(form, formats, dtype):
    """All results against 64 bits: each of the cols + 1 additions is off by at most
    2^-24 of the magnitudes summed, then one rounding.  Nothing beside Y is written."""
    rows, n, widths = FORMS[form]
    for at, cols in enumerate(widths):
        print(f"case {form}: {rows}x{cols}x{n} {formats} {dtype}", flush=True)
        g = torch.Generator(device="cuda").manual_seed(cols)
        X, x64 = operand(rows, cols, formats[0], g)
        W, w64 = operand(n, cols, formats[1], g, cols ** -0.5)
        bias = torch.randn(n, generator=g, device="cuda") if at % 2 else None
        space = torch.full((rows + 2, n + 3), 7.0, dtype=TYPES[dtype], device="cuda")
        sd.sd_pack_product(X.c, W.c, bias, space, dense.TYPES[TYPES[dtype]], n + 3, torch.cuda.current_stream())
        assert (space[rows:] == 7).all() and (space[:, n:] == 7).all()
        y = space[:rows, :n]
        want, size = x64 @ w64.t().contiguous(), x64.abs() @ w64.abs().t().contiguous()
        if bias is not None:
            want, size = want + bias.double(), size + bias.double().abs()
        bound = (cols + 2) * 2.0 ** -24 * size + HALF_ULP[dtype] * 1.001 * want.abs() + (2.0 ** -25 if dtype == "f16" else 0)
        assert ((y.double() - want).abs() <= bound).all()
        if dtype == "f32":
            assert (y.double() - want).norm() <= 1e-6 * want.norm()
        assert torch.equal(dense.product(X, W, bias, TYPES[dtype]), y)
