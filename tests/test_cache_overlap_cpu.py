"""State-cache calls whose arrays lie over one another are refused (no GPU: every
call fails validation, or ends before a launch)."""
import ctypes

import pytest

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import _Model, _StateCache

EINVAL = -1
STATES, CODES, SCALES, SLOTS = 0x7f0000001000, 0x7f1000000000, 0x7f2000000000, 0x7f3000000000
CODE_BYTES, SCALE_BYTES = 3 * 100 * 16, 3 * 2 * 16 * 4      # three slots of 100 cells


def call(lib, write, slots=SLOTS, codes=CODES, scales=SCALES, n=4):
    cache = _StateCache(0, 64, 3, 100, codes, scales)
    fn = lib.octree_nca_state_cache_write if write else lib.octree_nca_state_cache_read
    return fn(ctypes.byref(_Model(2, 16, 64, 3, 0)), ctypes.byref(cache), STATES, 0, 100, n, slots,
              0, None)


@pytest.mark.parametrize("slots", [CODES, CODES + 8, CODES + CODE_BYTES - 8, CODES - 24, SCALES,
                                   SCALES + SCALE_BYTES - 8, SCALES - 8])
def test_a_write_s_slot_list_lies_outside_the_cache(library_path, slots):
    assert call(octnca.lib(), True, slots) == EINVAL


@pytest.mark.parametrize("write", [True, False])
def test_codes_and_scales_lie_apart(library_path, write):
    for scales in (CODES, CODES + CODE_BYTES - 16, CODES - SCALE_BYTES + 16):
        assert call(octnca.lib(), write, scales=scales) == EINVAL
