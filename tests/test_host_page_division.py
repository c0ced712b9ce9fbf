"""How a divided attention over 16-bit pages deals the sequences' tokens to workgroups, on the CPU: all tiles once, never more parts than slots,
never more partial results than the scratch has room for."""
import os
import subprocess

import pytest

from paper_2602_02958_amd import build as qbuild

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host_page_division") / "host_page_division")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, *qbuild.FLAGS, "--offload-host-only", os.path.join(HERE, "host_page_division.cpp"), "-o", exe],
                   check=True, stderr=subprocess.DEVNULL)
    text = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    return dict(line.split(" ", 1) for line in text.splitlines())


@pytest.mark.parametrize("name", ["few", "many"])
def test_host_rule(rules, name):
    assert rules[name] == "ok"
