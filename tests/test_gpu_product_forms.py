"""Every form of the product of 8-bit tables.  Which one runs follows from how
many tiles the result has against the card's compute units; the sizes here are
made from that number, so each of them takes the form it is named for."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

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
