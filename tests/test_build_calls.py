"""The compiled Python calls' place in the build: one interpreter's are not another's."""
import os
import sysconfig

import pytest

from paper_2511_04063_b200 import build


@pytest.fixture(autouse=True)
def built():
    build.build()


def test_the_module_carries_the_interpreters_tag():
    suffix = sysconfig.get_config_var("EXT_SUFFIX")
    assert suffix != ".so" and os.path.basename(build.CALLS) == "_calls" + suffix and os.path.exists(build.CALLS)
    assert not os.path.exists(os.path.join(build.HERE, "_calls.so"))     # (any interpreter would load that one)
    from paper_2511_04063_b200 import _calls
    assert _calls.__file__ == build.CALLS
