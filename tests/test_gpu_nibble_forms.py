"""Every form of the 4-bit products at its edges: sizes that the choice of tiles,
of buffers and of a split sum goes by, with the results' types, biases, rows of NaN
and exact sums.  Sizes are made from the card's compute units."""
import gc

import numpy as np
import pytest

import nibble_reference as ref
from test_gpu_nibble import TYPES, check_product, of, random_table, to64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU container
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_05033_amd import dense, experts  # noqa: E402

CUS = torch.cuda.get_device_properties(0).multi_processor_count
SIDE = int((0.75 * CUS) ** 0.5) + 1  # SIDE * SIDE large tiles are enough for the card
MANY = int((2 * CUS) ** 0.5) + 1  # MANY * MANY of 40 stages are, of rows sorted by expert

# rows, columns, results: forms from the largest tiles to the smallest, odd and whole numbers of stages
FORMS = {
    "large": (256 * SIDE, 2048, 256 * SIDE),
    "large_odd": (256 * SIDE - 57, 2100, 256 * SIDE - 13),
    "large_ten": (256 * SIDE - 1, 2500, 256 * SIDE - 255 + 200),
    "large_long": (256 * SIDE - 57, 256 * 12 + 70, 256 * SIDE - 13),
    "many": (256 * SIDE, 512, 256 * SIDE),
    "many_odd": (256 * SIDE - 57, 130, 256 * SIDE - 13),
    "many_three": (128 * CUS + 5, 600, 70),
    "many_narrow": (64 * CUS + 65, 33, 5),
    "middle": (128 * 8 + 1, 1000, 128 * 8 - 3),
    "middle_one_stage": (128 * 9, 32, 128 * 9),
    "middle_deep": (128 * 11 - 7, 256 * 25 + 40, 128 * 12 - 60),
    "split": (260, 256 * 40 - 5, 300),
    "split_many": (70, 256 * 90 + 33, 65),
    "split_one_row": (1, 256 * 70, 40),
    "thirty_two": (40, 2048, 32 * CUS // 2 + 5),
    "thirty_two_short": (33, 300, 32 * CUS + 1),
    "sixteen": (9, 3000, 333),
    "sixteen_short": (17, 1024, 16),
    "sixteen_long": (16, 1100, 128 * CUS - 3),
    "along": (1000, 700, 1000),
    "along_one_group": (3001, 100, 301),
    "along_thin": (9, 300, 64 * CUS + 17),
    "along_thin_rows": (64 * CUS + 5, 513, 16),
}


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_forms(form, dtype):
    rows, cols, n = FORMS[form]
    print(f"case {form} {rows}x{cols}x{n} {dtype}", flush=True)
    X, W = random_table(rows, cols, 1, 2), random_table(n, cols, 2, 2)
    W = dense.Packed4(W.codes, (W.scales.to(torch.int32) - 7).to(torch.uint8), cols)
    x, w = of(X), of(W)
    b = np.random.default_rng(3).standard_normal(n).astype(np.float32)
    check_product(dense.product4(X, W, torch.from_numpy(b).cuda(), TYPES[dtype]), x, w, b.astype(np.float64), dtype)
    if dtype == "bf16":
        check_product(dense.product4(X, W, dtype=TYPES[dtype]), x, w, None, dtype)


@pytest.mark.parametrize("form", FORMS)
def test_forms_are_exact_and_keep_nan(form):
    """Whole quarters below 2^22 at every step; a NaN in the last block of one row of
    each side stays in that row and column.  Codes of every kind lie behind the last block."""
    rows, cols, n = FORMS[form]
    X, W = random_table(rows, cols, 4, 0), random_table(n, cols, 5, 0)
    want = of(X) @ of(W).T
    last = (cols - 1) // 32
    for p, row in ((X, rows // 2), (W, n - 1)):
        p.scales[last // 4, row, last % 4] = 255
        p.scales[last // 4, :, last % 4 + 1:] = 255  # behind the last block: of no effect
    want[rows // 2], want[:, n - 1] = np.nan, np.nan
    wide = torch.full((n, W.codes.shape[1] + 32), 0x77, dtype=torch.uint8, device="cuda")
    wide[:, :W.codes.shape[1]] = W.codes
    got = to64(dense.product4(X, dense.Packed4(wide, W.scales, cols)))
    assert np.array_equal(got, want, equal_nan=True)


EXPERTS = {
    "large": (128 * SIDE, 2, 3, 2060, 256 * SIDE - 9),
    "large_one": (256 * SIDE, 1, 1, 2048, 256 * SIDE),
    "large_many": (128 * MANY - 5, 2, 2, 256 * 40 - 180, 256 * MANY - 9),
    "large_many_one": (256 * MANY, 1, 1, 256 * 40, 256 * MANY),
    "many": (128 * SIDE, 2, 3, 520, 256 * SIDE - 9),
    "many_short": (900, 2, 7, 200, 2000),
    "middle": (700, 2, 5, 257, 600),
    "middle_deep": (500, 1, 4, 256 * 24 + 1, 700),
    "few_of_each": (30, 4, 40, 700, 300),
    "few_of_each_many": (40, 4, 60, 90, 1100),
    "thirty_two": (300, 1, 2, 1100, 130),
    "sixteen": (3, 2, 9, 900, 70),
    "along": (40, 3, 60, 1030, 1111),
    "few_long": (30, 2, 11, 256 * 17 + 3, 128 * CUS // 6 + 77),
    "many_kinds": (700, 3, 200, 700, 500),
    "along_eight_of_each": (200, 2, 50, 40, 2048 + 31),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", EXPERTS)
def test_forms_of_experts(form, dtype):
    rows, k, count, cols, n = EXPERTS[form]
    print(f"case experts {form} {rows}x{k} of {count}, {cols} to {n} {dtype}", flush=True)
    g = np.random.default_rng(rows)
    c = g.integers(-1, count, (rows, k))
    r = experts.route(torch.from_numpy(c).cuda(), count)
    X, W = random_table(rows, cols, 6, 2), random_table(count * n, cols, 7, 2)
    W = dense.Packed4(W.codes, (W.scales.to(torch.int32) - 7).to(torch.uint8), cols)
    b = g.standard_normal((count, n)).astype(np.float32)
    y = experts.product(X, W, r, torch.from_numpy(b).cuda(), TYPES[dtype])
    offsets, _, source = ref.route_fast(c, count)
    x, w = of(X), of(W).reshape(count, n, cols)
    for e in range(count):
        lo, hi = offsets[e], offsets[e + 1]
        if lo < hi:
            check_product(y[lo:hi], x[source[lo:hi]], w[e], b[e].astype(np.float64), dtype)
    assert not y[offsets[count]:].any()
    at = r.source.clamp(min=0).long()
    Xs = dense.Packed4(X.codes[at], X.scales[:, at].contiguous(), cols)
    assert torch.equal(y, experts.product(Xs, W, r, torch.from_numpy(b).cuda(), TYPES[dtype], sorted=True))


def test_tables_far_apart_in_memory():
    """Rows so far apart that their distances pass 32 bits take the forms that keep
    them in 64 bits."""
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GiB")
    ld, rows = (1 << 23) + 16, 600
    store = torch.zeros(rows * ld, dtype=torch.uint8, device="cuda")
    X = random_table(rows, 300, 8, 0)
    far = store.as_strided((rows, X.codes.shape[1]), (ld, 1))
    far.copy_(X.codes)
    F = dense.Packed4(far, X.scales, 300)
    W = random_table(700, 300, 9, 0)
    want = of(X) @ of(W).T
    assert np.array_equal(to64(dense.product4(F, W)), want)
    assert np.array_equal(to64(dense.product4(W, F)), want.T)
    c = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    assert np.array_equal(to64(experts.product(F, W, experts.route(c, 1))), want)
    assert np.array_equal(to64(experts.product(W, F, experts.route(torch.zeros(700, 1, dtype=torch.int32).cuda(), 1))),
                          want.T)


@pytest.mark.parametrize("name,at", [("sd_nibble_product", 6), ("sd_route", 3)])
def test_workspaces_live_until_the_call_is_enqueued(name, at, monkeypatch):
    """Memory given back before could be another thread's by then."""
    seen = []

    class Watch:
        def __init__(self, lib):
            self.lib = lib

        def __getattr__(self, what):
            f = getattr(self.lib, what)
            if what != name:
                return f

            def call(*args):
                seen.append(any(t.data_ptr() == args[at] for t in gc.get_objects()
                                if type(t) is torch.Tensor and t.dtype == torch.uint8 and t.is_cuda))
                return f(*args)

            return call

    for module in (dense, experts):
        monkeypatch.setattr(module, "_lib", Watch(module._lib))
    X = random_table(64, 40000, 1, 2)
    dense.product4(X, X)
    experts.route(torch.zeros(30000, 2, dtype=torch.int32, device="cuda"), 3)
    assert seen == [True]


def test_streams_at_once():
    """Split sums and sorts on several streams at the same time, each with a workspace of its own."""
    X = [random_table(64, 40000, 20 + i, 2) for i in range(4)]
    W = random_table(70, 40000, 30, 2)
    c = [torch.randint(-1, 30, (30000, 2), generator=torch.Generator().manual_seed(i)).cuda() for i in range(4)]
    want = [dense.product4(x, W) for x in X], [experts.route(v, 30).place.clone() for v in c]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for s, x, v in zip(streams, X, c):
            with torch.cuda.stream(s):
                got[0].append(dense.product4(x, W))
                got[1].append(experts.route(v, 30).place)
    torch.cuda.synchronize()
    for i in range(12):
        assert torch.equal(got[0][i], want[0][i % 4]) and torch.equal(got[1][i], want[1][i % 4])
