"""Host tests make their addresses up; where a device is visible no call of theirs may get past the checks with one."""
import os
import subprocess
import sys

from conftest import PASS_MADE_UP_ADDRESSES, ROOT

# A run that takes a device for visible, and counts the calls that got as far as a launch: without a device they fail there.
PLUGIN = """
import pytest
import torch

from paper_2609_37899_amd import soma

torch.cuda.device_count = lambda: 1
lib = soma.load()
launched = []


class Counting:
    def __getattr__(self, name):
        f = getattr(lib, name)

        def call(*args):
            rc = f(*args)
            if rc == soma.SOMA_EDEVICE:
                launched.append(name)
            return rc
        return call


def pytest_sessionstart(session):
    soma._lib = Counting()


def pytest_sessionfinish(session):
    print("launched:", *launched)
"""


def test_no_call_with_made_up_addresses_is_launched(tmp_path):
    (tmp_path / "as_if_visible.py").write_text(PLUGIN)
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([str(tmp_path), ROOT]))
    out = subprocess.run([sys.executable, "-m", "pytest", "-q", "-rs", "-p", "as_if_visible", "tests/test_block_host.py",
                          "tests/test_train_host.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    assert "launched:\n" in out.stdout + "\n", out.stdout
    assert "SKIPPED" in out.stdout


def test_the_tests_are_there():
    """Names that are left alone by mistake would run."""
    for name, test in PASS_MADE_UP_ADDRESSES:
        with open(os.path.join(ROOT, "tests", name)) as f:
            assert f"def {test}(" in f.read()
