"""The package names its modules."""
import importlib
import os
import pkgutil

import paper_2606_12688_amd as pkg


def test_every_public_module_is_listed():
    found = {m.name for m in pkgutil.iter_modules([os.path.dirname(pkg.__file__)]) if not m.name.startswith("_")}
    found -= {"libmstar_attn"}  # the built library, no Python module
    assert set(pkg.__all__) == found
    for name in pkg.__all__:
        assert importlib.import_module(f"{pkg.__name__}.{name}").__doc__
