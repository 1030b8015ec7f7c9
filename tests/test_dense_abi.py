"""CPU tests of the dense operators' C ABI: struct layouts against the header,
workspace sizes, and every refusal, none of which needs a GPU.  The pointers
are numbers that no call follows: each call here is refused before."""
import ctypes
import os
import subprocess

import pytest

import paper_2608_05033_amd as sd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address that is never read


def packed(rows=4, cols=40, ld=None, format=sd.SD_PACK_E4M3, reserved=0, codes=P, scales=2 * P):
    return sd.sd_packed_t(rows, cols, -(-cols // 16) * 16 if ld is None else ld, format, reserved, codes, scales)


def norm(rows=8, segments=2, offsets=None, longest=0, channels=12, groups=3, type=sd.SD_TYPE_F32,
         activation=sd.SD_ACT_NONE, eps=1e-5, reserved=0, weight=None, bias=None):
    return sd.sd_norm_t(rows, segments, offsets, longest, channels, groups, type, activation, eps, reserved, weight, bias)


def refused(status, call, *args):
    with pytest.raises(sd.SparseDittoError) as e:
        call(*args)
    assert e.value.status == status, (e.value, args)


def test_struct_layouts_match_header(tmp_path):
    structs = {"sd_packed_t": sd.sd_packed_t, "sd_norm_t": sd.sd_norm_t}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "sparseditto.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'printf("{name} {f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    lines += [f'printf("{n} value %d\\n", (int){n});' for n in
              ("SD_TYPE_F32", "SD_TYPE_F16", "SD_TYPE_BF16", "SD_PACK_E4M3", "SD_PACK_E5M2", "SD_ACT_NONE",
               "SD_ACT_RELU", "SD_ACT_SILU", "SD_ACT_GELU")]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "probe"), str(src)])
    for line in subprocess.check_output([str(tmp_path / "probe")]).decode().splitlines():
        name, field, value = line.split()
        if field == "value":
            assert getattr(sd, name) == int(value)
        elif field == "size":
            assert ctypes.sizeof(structs[name]) == int(value)
        else:
            assert getattr(structs[name], field).offset == int(value), line


BAD_PACKED = [dict(rows=-1), dict(cols=-1), dict(format=0), dict(format=3), dict(reserved=1), dict(ld=41), dict(ld=32),
              dict(codes=None), dict(scales=None), dict(codes=P + 8)]
LONG_PACKED = [dict(rows=1 << 31), dict(cols=(1 << 31) - 1, ld=1 << 31), dict(ld=1 << 41)]


@pytest.mark.parametrize("bad", BAD_PACKED + LONG_PACKED)
def test_packed_tables_are_checked_everywhere(bad):
    status = sd.SD_ERR_OVERFLOW if bad in LONG_PACKED else sd.SD_ERR_INVALID_VALUE
    p, ok = packed(**bad), packed(rows=bad.get("rows", 4), cols=bad.get("cols", 40), ld=bad.get("ld"))
    refused(status, sd.sd_pack, P, sd.SD_TYPE_F32, 40, 1, p)
    refused(status, sd.sd_unpack, p, P, sd.SD_TYPE_F32, 40)
    refused(status, sd.sd_pack_product, p, ok, None, P, sd.SD_TYPE_F32, 1 << 20)
    refused(status, sd.sd_pack_product, ok, p, None, P, sd.SD_TYPE_F32, 1 << 20)
    refused(status, sd.sd_pack_gradient, p, P, sd.SD_TYPE_F32, 8, 8, P, P, 1 << 40)


def test_pack_refusals():
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, None, sd.SD_TYPE_F32, 40, 1, packed())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, P, sd.SD_TYPE_F32, 40, 1, None)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, P, 4, 40, 1, packed())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, P, sd.SD_TYPE_F32, -1, 1, packed())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, P, sd.SD_TYPE_F32, 40, -1, packed())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack, P + 1, sd.SD_TYPE_BF16, 40, 1, packed())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_unpack, packed(), None, sd.SD_TYPE_F32, 40)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_unpack, packed(), P, 0, 40)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_unpack, packed(), P, sd.SD_TYPE_F32, 39)


def test_product_refusals():
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_product, packed(cols=40), packed(cols=41), None, P, sd.SD_TYPE_F32, 4)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_product, packed(), packed(), None, None, sd.SD_TYPE_F32, 4)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_product, packed(), packed(), None, P, 9, 4)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_product, packed(), packed(), None, P, sd.SD_TYPE_F32, 3)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_product, packed(), packed(), P + 2, P, sd.SD_TYPE_F32, 4)


def test_gradient_refusals_and_workspace():
    need = sd.sd_pack_gradient_size(100000, 40, 8)
    assert need > 0 and sd.sd_pack_gradient_size(0, 40, 8) == 0
    big = packed(rows=100000)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 8, 8, P, P, need - 1)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 8, 8, P, None, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 8, 8, P, P + 4, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 8, 8, None, P, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 8, 7, P, P, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, None, sd.SD_TYPE_F32, 8, 8, P, P, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, -1, 8, P, P, need)
    refused(sd.SD_ERR_OVERFLOW, sd.sd_pack_gradient, big, P, sd.SD_TYPE_F32, 1 << 31, 1 << 31, P, P, need)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_pack_gradient_size, -1, 1, 1)
    refused(sd.SD_ERR_OVERFLOW, sd.sd_pack_gradient_size, 1 << 31, 1, 1)


BAD_NORM = [dict(rows=-1), dict(channels=0), dict(groups=0), dict(groups=5), dict(segments=-1), dict(segments=3),
            dict(segments=0), dict(segments=0, offsets=P), dict(type=0), dict(activation=4), dict(activation=-1),
            dict(eps=-1.0), dict(eps=float("nan")), dict(reserved=1), dict(longest=-1)]
LONG_NORM = [dict(rows=1 << 31, segments=1), dict(segments=1 << 31, offsets=P), dict(channels=1 << 25, groups=1)]


@pytest.mark.parametrize("bad", BAD_NORM + LONG_NORM)
def test_norm_shapes_are_checked_everywhere(bad):
    status = sd.SD_ERR_OVERFLOW if bad in LONG_NORM else sd.SD_ERR_INVALID_VALUE
    d = norm(**bad)
    refused(status, sd.sd_group_norm_size, d)
    refused(status, sd.sd_group_norm, d, P, 1 << 26, P, 1 << 26, None, None, P, P, P, 1 << 40)
    refused(status, sd.sd_group_norm_backward, d, P, 1 << 26, P, 1 << 26, None, P, P, P, 1 << 26, P, P, P, 1 << 40)


def test_norm_refusals():
    d = norm()
    forward, backward = sd.sd_group_norm_size(d)
    good = [d, P, 12, P, 12, None, None, P, P, P, forward]
    for at, value in ((1, None), (1, P + 2), (2, 11), (3, None), (4, 11), (7, None), (8, None),
                      (5, packed(8, 16)), (6, packed(7, 12)), (5, packed(8, 12, format=7))):
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(good[:at] + [value] + good[at + 1:]))
    if forward:
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(good[:10] + [forward - 1]))
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(good[:9] + [None, forward]))
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(good[:9] + [P + 8, forward]))
    good = [d, P, 12, P, 12, None, P, P, P, 12, P, P, P, backward]
    for at, value in ((1, None), (2, 11), (3, None), (4, 11), (5, packed(8, 12)), (6, None), (7, None), (8, None),
                      (9, 11)):
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_backward, *(good[:at] + [value] + good[at + 1:]))
    if backward:
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_backward, *(good[:13] + [backward - 1]))
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_backward, *(good[:12] + [None, backward]))


def test_workspaces_stay_small():
    """The long table's workspace is some thousand rows; many short segments do
    not ask for one per segment and channel."""
    forward, backward = sd.sd_group_norm_size(norm(rows=2400000, segments=1, channels=128, groups=8))
    assert forward <= 16 << 20 and backward <= 16 << 20
    assert sd.sd_pack_gradient_size(2400000, 128, 128) <= 64 << 20


def test_tensor_functions_refuse_what_they_cannot_take():
    """The Python layer names the argument before anything reaches the library."""
    torch = pytest.importorskip("torch")
    from paper_2608_05033_amd import dense

    host = torch.zeros(4, 8)
    for call in (lambda: dense.pack(host), lambda: dense.group_norm(host, 2), lambda: dense.pack(host[0]),
                 lambda: dense.pack(host.double()), lambda: dense.Packed(host, host, 8),
                 lambda: dense.group_norm_backward(host, host, host, host, 2)):
        with pytest.raises(ValueError):
            call()
