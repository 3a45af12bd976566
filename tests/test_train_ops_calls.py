"""Calls of the training operators that the library takes or refuses before a device is touched."""
import ctypes

import pytest

from paper_2512_15773_b200 import binding, build

P = 1 << 16                                 # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_an_empty_batch_with_copies_is_a_call_with_nothing_to_do(lib):
    """Tensors without values have no address: neither x nor the copies."""
    n, none = binding.NormT(1, 0, 16, 64, 8, 1, 1e-5), binding.SavedT(None, None)
    for sx, sy in ((none, None), (None, none), (none, none)):
        assert lib.tsdp_group_norm(0, n, None, 0, 64, P, P, None, None, 0, 64, None, None, sx, sy, None) == 0
    one = binding.NormT(1, 1, 16, 64, 8, 1, 1e-5)
    assert lib.tsdp_group_norm(0, one, P, 0, 64, P, P, None, P, 0, 64, None, None, none, None, None) == 1
