"""The phase steps of RoPE are 64-bit fractions that the host takes out of an 80-bit long double: a
build whose long double is another format must stop, not give other angles."""
import os
import subprocess

import pytest

from paper_2606_13126_amd import build

INCLUDE = os.path.join(build.ROOT, "include")


def compiled(*flags):
    cmd = [build.hipcc(), "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "-I", INCLUDE, *flags,
           os.path.join(build.CSRC, "pic_host.cpp")]
    return subprocess.run(cmd, capture_output=True, text=True)


@pytest.mark.parametrize("bits", [64, 128])
def test_other_long_doubles_do_not_compile(bits):
    res = compiled("-Xarch_host", f"-mlong-double-{bits}")
    assert res.returncode != 0 and "80-bit long double" in res.stderr, res.stderr


def test_the_built_one_compiles():
    res = compiled()
    assert res.returncode == 0, res.stderr
