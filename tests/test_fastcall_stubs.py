"""Stand-ins for the library's entry points live as long as the native module that was given their addresses."""
import gc
import weakref

import pytest

from tests import test_fastcall_host, test_fastcall_pages
from tests.test_fastcall_host import ENTRIES, module  # noqa: F401  (fixture)
from tests.test_fastcall_pages import MORE, NAMES, Stubs, every_call


def test_stubs_that_the_test_does_not_keep(module):  # noqa: F811
    made = weakref.ref(Stubs(module, ENTRIES + MORE))
    gc.collect()
    assert made() is not None
    for name, f in every_call(module).items():
        assert f() is not NotImplemented, name
    assert set(made().calls) == {"window", "remap", "compact", "copy_pages"} and len(NAMES) == 4


@pytest.mark.parametrize("of", [test_fastcall_host, test_fastcall_pages])
def test_files_whose_stubs_are_kept(of):
    assert isinstance(of.Stubs, type)                   # (the fixture of conftest.py finds them by this name)
