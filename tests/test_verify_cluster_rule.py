"""How many CTAs a sequence of a verification gets, from how many clusters of each size find room."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ctas():
    from paper_2601_03700_gb300 import build
    build.build()
    import paper_2601_03700_gb300 as adept
    f = adept.load_library().adept_debug_verify_ctas
    f.restype = ctypes.c_int
    return lambda n_seq, *at_once: f(n_seq, (ctypes.c_int * 5)(*at_once))


def test_sizes_that_do_not_fit_at_all(ctas):
    """No cluster of 16 (or of several sizes) finds room: the next smaller that does, down to CTAs by themselves."""
    assert ctas(1, 152, 76, 36, 16, 0) == 8
    assert ctas(1, 152, 76, 0, 0, 0) == 2
    assert ctas(1, 152, 0, 0, 0, 0) == 1
    assert ctas(1, 0, 0, 0, 0, 0) == 1


def test_all_sequences_at_once_or_nearly(ctas):
    room = (152, 76, 36, 16, 7)
    assert [ctas(n, *room) for n in (1, 7, 8, 16, 18, 19, 36, 40, 41, 76, 85, 86, 1000)] == [16, 16, 8, 8, 8, 4, 4, 4, 2, 2, 2, 1, 1]
    assert ctas(1, 152, 76, 36, 16, 1) == 16
