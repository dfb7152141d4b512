"""The many-row attention of drafted trees finds 16-byte chunks by an exclusive or on LDS addresses,
within rows of 2 D bytes: its keys have to start at a multiple of one, wherever the compiler puts the
kernel's shared arrays."""
import os
import subprocess

from paper_2606_13126_amd import build

CHECK = """
#include "pic_tree.hip"
namespace pic { namespace {
template <int D> constexpr bool rows_aligned() {
    return alignof(TreeLds<D, true>) % (2 * D) == 0 && offsetof(TreeLds<D COMMA true>, stages) % (2 * D) == 0;
}
static_assert(rows_aligned<64>() && rows_aligned<128>(), "keys in LDS are not aligned to their rows");
} }
"""


def test_keys_in_lds_start_at_a_row(tmp_path):
    src = tmp_path / "check.hip"
    src.write_text("#define COMMA ,\n" + CHECK)
    res = subprocess.run([build.hipcc(), "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "-Wno-invalid-offsetof", "-I",
                          build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(src)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
