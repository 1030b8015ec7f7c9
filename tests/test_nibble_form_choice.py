"""Which kernel a 4-bit product takes, asked for on the CPU (256 compute units): the
cases that the GPU tests run by name take the kernels that they are named for, and all
of them are among these."""
import ctypes

import pytest

import nibble_cases as cases
import paper_2608_05033_amd as sd

TYPES = {"f32": sd.SD_TYPE_F32, "f16": sd.SD_TYPE_F16, "bf16": sd.SD_TYPE_BF16}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", cases.PRODUCTS)
def test_products(name, dtype):
    case = cases.PRODUCTS[name]
    rows, cols, n = case[0]
    form, parts = cases.chosen(case, dtype)
    assert sd.sd_nibble_product_form(rows, cols, n, 0, TYPES[dtype]) == (form, parts)
    assert sd.sd_nibble_product_size(rows, cols, n) == (4 * parts * rows * n if parts > 1 else 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", cases.EXPERTS)
def test_experts(name, dtype):
    case = cases.EXPERTS[name]
    rows, k, experts, cols, n = case[0]
    assert sd.sd_nibble_product_form(rows * k, cols, n, experts, TYPES[dtype]) == cases.chosen(case, dtype)


@pytest.mark.parametrize("table", [cases.PRODUCTS, cases.EXPERTS])
@pytest.mark.parametrize("dtype", TYPES)
def test_every_kernel_is_among_them(table, dtype):
    assert {cases.chosen(case, dtype)[0] for case in table.values()} == set(sd.NIBBLE_FORMS)


def test_parts_of_both_ways_to_join():
    """The join takes one thread for four columns below 16 parts, eight from there on;
    the results' last columns fill no four."""
    joined = [(case[0][2], case[1][1]) for case in cases.PRODUCTS.values() if case[1][1] > 1]
    assert any(n % 4 and parts < 16 for n, parts in joined) and any(n % 4 and parts >= 16 for n, parts in joined)


def test_one_form_more_than_rows_are_near():
    """Columns so many that rows lie further apart than the tiles count."""
    assert sd.sd_nibble_product_form(4000, (1 << 24) + 1, 4000, 0, sd.SD_TYPE_F32)[0] == "rows_32"
    assert sd.sd_nibble_product_form(1 << 20, 1 << 14, 4000, 4, sd.SD_TYPE_F32)[0] == "rows_32"


def test_refusals():
    good = [4, 40, 5, 0, sd.SD_TYPE_F32]
    for status, at, value in ((sd.SD_ERR_INVALID_VALUE, 0, 0), (sd.SD_ERR_INVALID_VALUE, 0, -1),
                              (sd.SD_ERR_INVALID_VALUE, 1, -1), (sd.SD_ERR_INVALID_VALUE, 2, 0),
                              (sd.SD_ERR_INVALID_VALUE, 3, -1), (sd.SD_ERR_INVALID_VALUE, 4, 9),
                              (sd.SD_ERR_OVERFLOW, 0, 1 << 31), (sd.SD_ERR_OVERFLOW, 1, (1 << 31) - 1),
                              (sd.SD_ERR_OVERFLOW, 2, 1 << 31), (sd.SD_ERR_UNSUPPORTED, 3, 4096)):
        with pytest.raises(sd.SparseDittoError) as e:
            sd.sd_nibble_product_form(*good[:at], value, *good[at + 1:])
        assert e.value.status == status, (at, value)
    form = ctypes.c_int32()
    assert sd._lib.sd_nibble_product_form(*good, None, form) == sd.SD_ERR_INVALID_VALUE
    assert sd._lib.sd_nibble_product_form(*good, form, None) == sd.SD_ERR_INVALID_VALUE
