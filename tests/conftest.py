import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(scope="session")
def oracle_mod():
    import oracle
    oracle.build(force=False)
    return oracle


_stubs = []


@pytest.fixture(autouse=True)
def stubs_outlive_their_addresses(request, monkeypatch):
    """A native module calls a test's stand-ins for the library (its class Stubs) by address, for as long as the module is there.
    So they live on whether or not the test keeps them: else the next cyclic collection frees the code behind the addresses."""
    stubs = getattr(getattr(request, "module", None), "Stubs", None)
    if stubs is None:
        return
    make = stubs.__init__

    def init(self, *args):
        _stubs.append(self)
        make(self, *args)
    monkeypatch.setattr(stubs, "__init__", init)
