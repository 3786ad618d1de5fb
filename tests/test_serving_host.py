"""Arguments of the failure-detection knob of the calls without a context (no GPU)."""
import pytest

from paper_2406_13035_b200 import binding as B
from paper_2406_13035_b200 import build


def test_fault_injection_refuses():
    build.build_library()
    lib = B.load_library()
    for bad in [(-1, -1, 0), (0, -2, 0), (0, -1, -1)]:
        assert lib.d2o_set_static_fault_injection(*bad) == 1, bad
    with pytest.raises(B.D2OError):
        B.d2o_set_static_fault_injection(wait_limit_us=-5)
    B.d2o_set_static_fault_injection(2000, 0, 3)
    B.d2o_set_static_fault_injection()
