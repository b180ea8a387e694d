import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


def _ensure_built():
    """Build the CPU-side libraries only when nothing is built yet."""
    import oracle.build
    import workloads.build
    if not os.path.exists(os.path.join(ROOT, "oracle", "liboracle.so")):
        oracle.build.build()
    if not (os.path.exists(os.path.join(ROOT, "workloads", "libtaot_gen_host.so"))
            and os.path.exists(os.path.join(ROOT, "workloads", "libtaot_gen_dev.so"))):
        workloads.build.build()


_ensure_built()


@pytest.fixture(scope="session")
def gpu():
    """Skip unless a GPU is visible; tests using this are also marked `gpu`."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    return torch.device("cuda:0")


# Tests whose expected values are wrong: their oracle ranks groups by the sum of two logits where no bias is given, the
# definition by the sum of two scores (10 + 0 > 4 + 4, but sigmoid(10) + sigmoid(0) < 2 sigmoid(4)).  They run as they
# are and have to fail; tests/test_gpu_route_groups.py has the same calls with the definition's values.
_WRONG_VALUES = {"test_gpu_route.py": ("test_groups_by_two[64-4-6]", "test_groups_by_two[256-8-8]",
                                       "test_groups_by_two[1000-8-8]", "test_groups_by_two[4096-16-8]",
                                       "test_more_experts_than_registers[9000-8]")}


def pytest_collection_modifyitems(items):
    for item in items:
        if item.name in _WRONG_VALUES.get(item.path.name, ()):
            item.add_marker(pytest.mark.xfail(reason="its oracle adds logits for a group's two best scores",
                                              raises=AssertionError, strict=True))
