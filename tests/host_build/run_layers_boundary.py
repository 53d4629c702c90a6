"""Runs the CPU boundary tests of the operators between two drops against a given build of the library's host side: like
run_boundary_tests.py beside it, which runs the ones of the sparsification path."""
import ctypes
import os
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sanitized = os.path.abspath(sys.argv[1])
_real = ctypes.CDLL


class _Redirect(_real):
    def __init__(self, name, *args, **kwargs):
        if name is not None and os.path.basename(str(name)) == "libuniprefill.so":
            name = sanitized
        super().__init__(name, *args, **kwargs)


ctypes.CDLL = _Redirect
sys.exit(pytest.main([os.path.join(os.path.dirname(HERE), "test_host_layers.py"), "-q", "-x", "-p", "no:cacheprovider"]))
