"""A packed operand is looked at like a tensor before its pointers are handed on: its device, and whether anything has
been packed into it.  No device is needed: -1 is the CPU's number."""
import pytest

from paper_2507_23387_b200 import binding


def test_another_device_is_refused():
    p = binding.PackedMatrix(3, 5, device="cpu")
    p.packed = True
    assert binding._operand(p, -1) is p.operand
    with pytest.raises(AssertionError):
        binding._operand(p, 0)


def test_an_unpacked_one_is_refused():
    p = binding.PackedMatrix(3, 5, device="cpu")
    with pytest.raises(AssertionError):
        binding._operand(p, -1)
