"""Calls that need no device to be refused: no handle."""
import pytest

from paper_2507_23387_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_calls_without_a_handle_are_refused(lib):
    bad = binding.INVALID_ARG
    assert lib.sgemm_cube_embedding(None, 1, 1, 1, 0, None, None, 1, 1.0, None, 1, None) == bad
    assert lib.sgemm_cube_embedding_backward(None, 1, 1, 1, 0, None, None, 1, 1.0, 0, None, 1, None) == bad
    assert lib.sgemm_cube_cross_entropy(None, 1, 1, 1, None, None, 0, None, None, None, None, None) == bad
    assert lib.sgemm_cube_cross_entropy_backward(None, 1, 1, 1, None, None, 0, None, None, None, None, None, None, 1, None, 1, None,
                                                 None) == bad
    assert lib.sgemm_cube_orthogonalize(None, 1, 1, 0, None, 1, 1, None, 1e-7, 1.0, None, 1, 1.0, None, 1, None) == bad
