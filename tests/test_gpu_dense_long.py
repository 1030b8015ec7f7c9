"""Dense operators on tables so long that their workgroups pass 2^32 threads,
more than a launch holds along one dimension."""
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.slow]

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_05033_amd import dense  # noqa: E402


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


def test_pack_of_more_than_two_to_the_29_rows():
    """One fp32 column: 32 rows a workgroup of 256 threads.  Numbers of 4 significant
    bits come back as they were."""
    rows = (1 << 29) + 5
    x = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(16).add_(1).float().view(rows, 1)
    p = dense.pack(x)
    y = dense.unpack(p)
    assert torch.equal(x, y)
    assert not p.codes[-100:, 1:].any() and (p.scales[0, -100:] < 127).all()


def test_product_with_almost_two_to_the_31_columns():
    """One row: tiles of 128 columns, 256 threads each."""
    n = (1 << 31) - 65
    codes = torch.full((n, 16), 0x38, dtype=torch.uint8, device="cuda")  # 1
    for at in (0, 1 << 30, n - 1):
        codes[at] = 0x40  # 2
    w = dense.Packed(codes, torch.full((1, n), 127, dtype=torch.uint8, device="cuda"), 16)
    x = dense.pack(torch.ones(1, 16, device="cuda"))
    y = dense.product(x, w, dtype=torch.bfloat16)
    for at in (0, 1 << 30, n - 1):
        assert y[0, at] == 32
        y[0, at] = 16
    assert (y == 16).all()


def test_weight_gradient_with_more_than_two_to_the_30_columns():
    """One row of fp32: tiles of 64 columns, 256 threads each; 24 bits of G come through."""
    n = (1 << 30) + 70
    g = torch.arange(n, dtype=torch.int32, device="cuda").remainder_((1 << 24) - 3).float().view(1, n)
    dw = dense.weight_gradient(dense.pack(torch.full((1, 1), 2.0, device="cuda")), g)
    assert torch.equal(dw, g.mul_(2))
