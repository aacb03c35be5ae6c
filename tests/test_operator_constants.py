"""CPU checks of the language-model operators' boundary: the binding's constants are the header's, and the entry
points refuse a missing handle before they look at a device."""
import ctypes
import os
import re

import pytest

from paper_2507_23387_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OPERATORS = ["sgemm_cube_pack", "sgemm_cube_linear", "sgemm_cube_linear_backward", "sgemm_cube_layer_norm",
             "sgemm_cube_layer_norm_backward", "sgemm_cube_token_logprobs", "sgemm_cube_token_logprobs_backward"]


def _enum_values():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sgemm_cube.h")).read(), flags=re.S)
    return {n: int(v) for n, v in re.findall(r"\bSGEMM_CUBE_(\w+)\s*=\s*(-?\d+)", text)}


@pytest.mark.parametrize("name", ["WEIGHT_KN", "WEIGHT_NK", "ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_GELU_TANH", "ACT_SILU",
                                  "F32", "F16", "BF16"])
def test_constants_are_the_headers(name):
    assert getattr(binding, name) == _enum_values()[name]


@pytest.mark.parametrize("name", OPERATORS)
def test_missing_handle_is_refused(name):
    build.build()
    f = getattr(binding.load(), name)
    args = [0.0 if t in (ctypes.c_float, ctypes.c_double) else 0 if t in (ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t) else None
            for t in f.argtypes]
    assert f(*args) == binding.INVALID_ARG
