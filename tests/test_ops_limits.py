"""CPU: what the C entry points of the sequence operators refuse at the ends of their ranges (nothing here reaches a GPU)."""
import ctypes

import pytest

import ops_structures as st
from paper_1804_10223_amd import binding, ops
from test_ops_oracle import AT, _own, _scan_arguments, _seq


@pytest.mark.parametrize("name", ["u", "dt", "z", "B", "C", "y"])
def test_two_steps_of_a_scan_are_at_most_2_25_elements_apart(name):
    lib, far = ops._library(), _seq(step=(1 << 25) + 1, sample=8)
    s = _scan_arguments(steps=2, **({} if name == "y" else {name: far}))
    y = far if name == "y" else _seq()
    assert lib.sprnn_scan_forward(0, ctypes.byref(s), None, y, None, None, None, 0, None) == binding.SPRNN_ERR_INVALID
    g = st.ScanGradientBuffers(u=_own(y))
    assert lib.sprnn_scan_backward(0, ctypes.byref(s), _seq(), None, AT, ctypes.byref(g), AT, 1 << 40, None) == binding.SPRNN_ERR_INVALID
