"""What the entry points launch, without a GPU: the checks of tests/launch_checks.py, each in a process of its own whose
HIP runtime is a stub that notes launches."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    from paper_2506_12541_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2506_12541_amd.build import build
        build()
    so = tmp_path_factory.mktemp("stub") / "launch_stub.so"
    subprocess.run(["gcc", "-shared", "-fPIC", os.path.join(HERE, "launch_stub.c"), "-o", str(so)], check=True)
    return str(so)


@pytest.mark.parametrize("check", ["copied_rows", "rotary_steps", "launches_fit"])
def test_launches(stub, check):
    r = subprocess.run([sys.executable, os.path.join(HERE, "launch_checks.py"), stub, check], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and r.stdout == "checked\n", r.stdout + r.stderr
