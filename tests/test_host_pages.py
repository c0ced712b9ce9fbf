"""Where the tokens of an attention over 16-bit pages lie, walked through on the CPU: every token that is seen is met once, and no address
that a wavefront forms lies outside them."""
import os
import subprocess

import pytest

from paper_2602_02958_amd import build as qbuild

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host_pages") / "host_pages")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, *qbuild.FLAGS, "--offload-host-only", os.path.join(HERE, "host_pages.cpp"), "-o", exe],
                   check=True, stderr=subprocess.DEVNULL)
    text = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    return dict(line.split(" ", 1) for line in text.splitlines())


@pytest.mark.parametrize("name", ["quotients", "small_paged", "small_rows", "large_paged", "large_rows"])
def test_host_rule(rules, name):
    assert rules[name] == "ok"
