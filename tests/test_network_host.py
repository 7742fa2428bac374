"""The host side of the calls around a feature network's step and its serving
against a HIP runtime of the test's own (tests/host), on the CPU."""
import os

from paper_1706_05544_amd import build as b
from test_layers_host import run_driver


def test_calls_leave_the_threads_device_as_it_was(tmp_path):
    run_driver(tmp_path, "network_device_driver",
               [os.path.join(b.CSRC, "network.cpp")])


def test_no_exception_leaves_a_call_that_finds_no_memory(tmp_path):
    # (the executable's operator new stands in for the library's)
    from paper_1706_05544_amd import native as nv
    nv.load()
    run_driver(tmp_path, "network_memory_driver",
               [nv.LIB_PATH, "-rdynamic",
                "-Wl,-rpath," + os.path.dirname(nv.LIB_PATH)])
