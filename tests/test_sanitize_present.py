"""Where the drivers' sources are, the module that builds them has to import: its
absence (as in a copy of the tree without them) skips tests, a fault in it must not."""
import importlib
import os

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(not os.path.isfile(os.path.join(HERE, "test_sanitize.py")),
                    reason="a tree without the sanitizer drivers")
def test_module_of_the_sanitizer_drivers_imports():
    base = importlib.import_module("tests.test_sanitize")
    for name in ("CSRC", "HERE", "ROOT", "SAN", "_run", "_env", "_check_clean", "pytestmark"):
        assert hasattr(base, name), name
