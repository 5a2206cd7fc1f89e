"""The number of states of a state-cache call is bounded (no GPU: the calls fail
validation)."""
import ctypes

import pytest

import paper_2508_06993_amd as octnca
from paper_2508_06993_amd import _Model, _StateCache

ESHAPE = -3


@pytest.mark.parametrize("write", [True, False])
@pytest.mark.parametrize("slots", [None, 0x7d0000000000])
def test_states_of_a_call(library_path, write, slots):
    """The kernels step from state to state in 32 bits: the last step from the
    largest numbers of states would leave them."""
    cache = _StateCache(0, 64, 1 << 32, 1, 0x7e0000000000, 0x7f0000000000)
    lib = octnca.lib()
    fn = lib.octree_nca_state_cache_write if write else lib.octree_nca_state_cache_read
    for n in (2 ** 31 - 1, 2 ** 31 - 2 ** 16, 2 ** 31 - 2 ** 17):
        assert fn(ctypes.byref(_Model(2, 12, 48, 3, 1)), ctypes.byref(cache), 0x7c0000000000, 0, 1,
                  n, slots, 0, None) == ESHAPE
