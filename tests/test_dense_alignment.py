"""CPU tests of what the group norm's C ABI refuses besides sizes: vectors that are
not aligned to their type.  The pointers are numbers that no call follows."""
import pytest

import paper_2608_05033_amd as sd
from test_dense_abi import P, norm, packed, refused


def calls(d):
    forward, backward = sd.sd_group_norm_size(norm(offsets=P))
    return ([d, P, 12, P, 12, None, None, P, P, P, max(forward, 1 << 20)],
            [d, P, 12, P, 12, None, P, P, P, 12, P, P, P, max(backward, 1 << 20)])


@pytest.mark.parametrize("field", ["offsets", "weight", "bias"])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_a_norms_own_vectors_are_aligned(field, off):
    d = norm(**{field: P + off})
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_size, d)
    forward, backward = calls(d)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *forward)
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_backward, *backward)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_statistics_and_gradients_are_aligned(off):
    forward, backward = calls(norm())
    for at in (7, 8):  # mean, rstd
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(forward[:at] + [P + off] + forward[at + 1:]))
    for at in (6, 7, 10, 11):  # mean, rstd, dweight, dbias
        refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm_backward, *(backward[:at] + [P + off] + backward[at + 1:]))


def test_packed_codes_are_aligned_in_copies_too():
    forward, _ = calls(norm())
    refused(sd.SD_ERR_INVALID_VALUE, sd.sd_group_norm, *(forward[:5] + [packed(8, 12, codes=P + 4)] + forward[6:]))
