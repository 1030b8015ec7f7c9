"""CPU tests of the C ABI of the 4-bit tables and of the rows sorted by expert:
struct layouts against the header, workspace sizes, and every refusal, none of
which needs a GPU.  The pointers are numbers that no call follows: each call here
is refused before."""
import ctypes
import os
import subprocess

import pytest

import paper_2608_05033_amd as sd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address that is never read
BIG = 1 << 40
F32 = sd.SD_TYPE_F32


def table(rows=4, cols=40, ld=None, reserved=0, codes=P, scales=2 * P):
    return sd.sd_nibble_t(rows, cols, -(-cols // 32) * 16 if ld is None else ld, reserved, codes, scales)


def route(rows=6, k=2, experts=3, offsets=P, place=2 * P, source=3 * P):
    return sd.sd_route_t(rows, k, experts, offsets, place, source)


def refused(status, call, *args):
    with pytest.raises(sd.SparseDittoError) as e:
        call(*args)
    assert e.value.status == status, (e.value, args)


def each(status, call, good, bad):
    """call refuses `good` with any of the (position, value) put in."""
    for at, value in bad:
        refused(status, call, *(good[:at] + [value] + good[at + 1:]))


def test_struct_layouts_match_header(tmp_path):
    structs = {"sd_nibble_t": sd.sd_nibble_t, "sd_route_t": sd.sd_route_t}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "sparseditto.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'printf("{name} {f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "probe"), str(src)])
    for line in subprocess.check_output([str(tmp_path / "probe")]).decode().splitlines():
        name, field, value = line.split()
        got = ctypes.sizeof(structs[name]) if field == "size" else getattr(structs[name], field).offset
        assert got == int(value), line


BAD_TABLE = [dict(rows=-1), dict(cols=-1), dict(reserved=1), dict(ld=40), dict(ld=16), dict(codes=None),
             dict(scales=None), dict(codes=P + 8), dict(scales=P + 2)]
LONG_TABLE = [dict(rows=1 << 31), dict(cols=(1 << 31) - 1, ld=1 << 31), dict(ld=1 << 41)]


@pytest.mark.parametrize("bad", BAD_TABLE + LONG_TABLE)
def test_tables_are_checked_everywhere(bad):
    status = sd.SD_ERR_OVERFLOW if bad in LONG_TABLE else sd.SD_ERR_INVALID_VALUE
    p, ok = table(**bad), table(rows=bad.get("rows", 4), cols=bad.get("cols", 40))
    refused(status, sd.sd_nibble_pack, P, F32, 40, 1, p)
    refused(status, sd.sd_nibble_pack_both, P, F32, 40, 1, p, ok)
    refused(status, sd.sd_nibble_pack_both, P, F32, 40, 1, ok, p)
    refused(status, sd.sd_nibble_unpack, p, P, F32, 40)
    refused(status, sd.sd_nibble_product, p, ok, None, P, F32, 1 << 20, P, BIG)
    refused(status, sd.sd_nibble_product, ok, p, None, P, F32, 1 << 20, P, BIG)
    refused(status, sd.sd_expert_product, p, ok, route(), 0, None, P, F32, 1 << 20)
    refused(status, sd.sd_expert_product, ok, p, route(), 0, None, P, F32, 1 << 20)


def test_packing_refusals():
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_pack, [P, F32, 40, 1, table()],
         [(0, None), (0, P + 2), (1, 0), (1, 4), (2, -1), (3, -1), (4, None)])
    each(sd.SD_ERR_OVERFLOW, sd.sd_nibble_pack, [P, F32, 40, 1, table()], [(2, 1 << 41), (3, 1 << 32)])
    good = [P, F32, 40, 1, table(), table(rows=40, cols=4)]
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_pack_both, good,
         [(0, None), (0, P + 2), (1, 0), (2, -1), (3, -1), (4, None), (4, table(cols=41)), (5, None), (5, table()),
          (5, table(rows=40, cols=4, codes=None))])
    each(sd.SD_ERR_OVERFLOW, sd.sd_nibble_pack_both, good, [(2, 1 << 32), (3, 1 << 32)])
    refused(sd.SD_ERR_OVERFLOW, sd.sd_nibble_pack_both, P, F32, 1 << 32, 2, *good[4:])
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_unpack, [table(), P, F32, 40],
         [(0, None), (1, None), (1, P + 1), (2, 0), (3, 39)])
    refused(sd.SD_ERR_OVERFLOW, sd.sd_nibble_unpack, table(), P, F32, 1 << 31)


def test_product_refusals():
    good = [table(), table(rows=5), P, P, F32, 5, P, BIG]
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_product, good,
         [(0, None), (1, None), (1, table(rows=5, cols=41)), (2, P + 2), (3, None), (3, P + 2), (4, 9), (5, 4)])
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_product_size, -1, 1, 1)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_product_size, 1, 1, -1)
    refused(sd.SD_ERR_OVERFLOW, sd.sd_nibble_product_size, 1, 1, 1 << 31)
    # few results of a long sum: what workgroups have summed goes to the workspace
    long = [table(rows=64, cols=1 << 18), table(rows=64, cols=1 << 18), None, P, F32, 64]
    need = sd.sd_nibble_product_size(64, 1 << 18, 64)
    if need:
        for work, size in ((None, need), (P, need - 1), (P + 8, need)):
            refused(sd.SD_ERR_INVALID_VALUE, sd.sd_nibble_product, *long, work, size)
    assert need <= 64 << 20


BAD_ROUTE = [dict(rows=-1), dict(k=0), dict(experts=0), dict(offsets=None), dict(place=None), dict(source=None),
             dict(offsets=P + 2), dict(place=P + 2), dict(source=P + 2)]
LONG_ROUTE = [dict(rows=1 << 31, k=1), dict(rows=1 << 30, k=2)]
WIDE_ROUTE = [dict(experts=4096)]


@pytest.mark.parametrize("bad", BAD_ROUTE + LONG_ROUTE + WIDE_ROUTE)
def test_routes_are_checked_everywhere(bad):
    status = sd.SD_ERR_OVERFLOW if bad in LONG_ROUTE else \
        sd.SD_ERR_UNSUPPORTED if bad in WIDE_ROUTE else sd.SD_ERR_INVALID_VALUE
    r = route(**bad)
    refused(status, sd.sd_route, P, 4, r, P, BIG)
    refused(status, sd.sd_dispatch, r, P, F32, 8, 8, P, 8)
    refused(status, sd.sd_combine, r, P, F32, 8, 8, P, P, 8)
    refused(status, sd.sd_combine_backward, r, P, F32, 8, 8, P, 8, P, P, 8, P)
    refused(status, sd.sd_expert_product, table(rows=6), table(rows=12), r, 0, None, P, F32, 4)
    if not set(bad) & {"offsets", "place", "source"}:
        refused(status, sd.sd_route_size, r.rows, r.k, r.experts)


def test_route_refusals_and_workspace():
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_route, [P, 4, route(), None, 0],
         [(0, None), (0, P + 2), (1, 2), (1, 0), (2, None)])
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_route, P + 4, 8, route(), None, 0)
    assert sd.sd_route_size(0, 2, 8) == 0 and sd.sd_route_size(37, 2, 16) == 0
    need = sd.sd_route_size(100000, 2, 8)
    assert need > 0
    for work, size in ((None, need), (P, need - 1), (P + 8, need)):
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_route, P, 4, route(rows=100000, experts=8), work, size)
    assert sd.sd_route_size((1 << 31) - 1, 1, 4095) <= 65 << 20


def test_exchange_refusals():
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_dispatch, [route(), P, F32, 8, 8, P, 8],
         [(0, None), (1, None), (1, P + 2), (2, 0), (3, -1), (4, 7), (5, None), (5, P + 1), (6, 7)])
    each(sd.SD_ERR_OVERFLOW, sd.sd_dispatch, [route(), P, F32, 8, 8, P, 8], [(3, 1 << 31), (4, 1 << 31), (6, 1 << 31)])
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_combine, [route(), P, F32, 8, 8, P, P, 8],
         [(0, None), (1, None), (2, 7), (3, -1), (4, 7), (5, P + 2), (6, None), (7, 7)])
    each(sd.SD_ERR_OVERFLOW, sd.sd_combine, [route(), P, F32, 8, 8, P, P, 8], [(3, 1 << 31), (4, 1 << 31)])
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_combine_backward, [route(), P, F32, 8, 8, P, 8, P, P, 8, P],
         [(0, None), (1, None), (2, 0), (3, -1), (4, 7), (5, None), (6, 7), (7, P + 2), (8, P + 2), (9, 7), (10, P + 2)])


def test_expert_product_refusals():
    good = [table(rows=6), table(rows=15), route(), 0, P, P, F32, 5]
    each(sd.SD_ERR_INVALID_VALUE, sd.sd_expert_product, good,
         [(0, table(rows=12)), (0, table(rows=6, cols=41)), (1, table(rows=16)), (2, None), (3, 1), (3, 2), (4, P + 2),
          (5, None), (6, 0), (7, 4)])


def test_tensor_functions_refuse_what_they_cannot_take():
    """The Python layer names the argument before anything reaches the library."""
    torch = pytest.importorskip("torch")
    from paper_2608_05033_amd import dense, experts, gcn

    host, ints = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: dense.pack4(host), lambda: dense.pack4(host[0]), lambda: dense.pack4_both(host),
                 lambda: dense.pack4(host.double()),
                 lambda: dense.Packed4(host, host, 8), lambda: dense.Packed4(ints.byte(), ints.byte(), 4),
                 lambda: experts.route(ints, 3), lambda: experts.route(host, 3), lambda: experts.route(ints[0], 3),
                 lambda: experts.Route(ints[0], ints, ints.view(-1)), lambda: gcn.transform4(host, host)):
        with pytest.raises(ValueError):
            call()
