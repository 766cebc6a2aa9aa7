"""Tests that bind the compiled Python calls to stand-ins leave nothing behind for the ones after them."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_operators_are_bound_again_after_the_calls_tests(tmp_path):
    before, after = tmp_path / "test_before.py", tmp_path / "test_after.py"
    before.write_text("import sys; sys.path.insert(0, %r)\n"
                      "def test_the_operators_were_called():\n"
                      "    from paper_2511_04063_b200 import _calls, binding\n"
                      "    binding._calls = _calls\n" % ROOT)
    after.write_text("def test_the_next_call_binds_the_library():\n"
                     "    from paper_2511_04063_b200 import binding\n"
                     "    assert binding._calls is None\n")
    for name in ("test_mx_abi.py", "test_mx_calls.py"):
        ran = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-p", "no:randomly", str(before),
                              os.path.join(ROOT, "tests", name), str(after)], cwd=ROOT, capture_output=True, text=True, timeout=600)
        assert ran.returncode == 0, ran.stdout[-2000:]
