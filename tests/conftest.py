import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


def build_where_the_serving_assembly_is_stale():
    from paper_2510_08726_amd import build as libbuild
    if libbuild.serve_asm_stale():
        import __graft_entry__
        __graft_entry__.build()


@pytest.fixture(autouse=True, scope="module")
def current_serving_assembly(request):
    """The guards on the serving kernels' assembly read that of the present sources."""
    if request.module.__name__ == "test_serve_codegen":
        build_where_the_serving_assembly_is_stale()
