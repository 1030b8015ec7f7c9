"""Numbers of experts that do not fit the library's 32 bits are refused before they are
cut off to smaller ones."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_05033_amd import experts  # noqa: E402

LONG = [(4, 2, (1 << 32) + 3), (4, 2, 1 << 31), (4, 2, -(1 << 32) + 3), (0, (1 << 32) + 1, 3), (0, 1 << 31, 3)]


@pytest.mark.parametrize("rows,k,count", LONG)
def test_sizes(rows, k, count):
    with pytest.raises(ValueError, match="2\\^31"):
        experts._route_size(rows, k, count)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("rows,k,count", LONG)
def test_routes(rows, k, count):
    with pytest.raises(ValueError, match="2\\^31"):
        experts.route(torch.zeros(rows, k, dtype=torch.int32, device="cuda"), count)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_a_route_of_other_tensors():
    ints = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="2\\^31"):
        experts.Route(ints, torch.zeros(0, (1 << 32) + 1, dtype=torch.int32, device="cuda"), ints[:0])
