"""The binding's native module belongs to one interpreter: its file says so, and another's does not count as built."""
import importlib
import os
import sysconfig

import pytest

from paper_2609_34060_b200 import build as kbuild


@pytest.fixture
def other(monkeypatch):
    """build() as another interpreter would see it (the compiler's headers stay this one's: the file is not imported)."""
    suffix = ".cpython-300-elsewhere.so"
    made, stamp = os.path.join(kbuild.HERE, "_marshal" + suffix), os.path.join(kbuild.OBJ, "stamp" + suffix)
    kbuild.build()
    monkeypatch.setattr(kbuild, "EXT_SUFFIX", suffix, raising=False)
    monkeypatch.setattr(kbuild, "MARSHAL", made)
    yield made, stamp
    for f in (made, stamp):
        if os.path.exists(f):
            os.remove(f)


def test_the_file_carries_the_interpreters_tag():
    kbuild.build()
    m = importlib.import_module("paper_2609_34060_b200._marshal")
    assert m.__file__ == kbuild.MARSHAL and kbuild.MARSHAL.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert not os.path.exists(os.path.join(kbuild.HERE, "_marshal.so"))


def test_another_interpreter_builds_its_own(other):
    made, stamp = other
    lib = os.stat(kbuild.LIB).st_mtime_ns
    kbuild.build()
    assert os.path.exists(made) and os.stat(kbuild.LIB).st_mtime_ns == lib      # the library itself is anybody's
    first = os.stat(made).st_mtime_ns
    kbuild.build()
    assert os.stat(made).st_mtime_ns == first
    with open(stamp, "w") as f:
        f.write("of other sources")
    kbuild.build()
    assert os.stat(made).st_mtime_ns != first
