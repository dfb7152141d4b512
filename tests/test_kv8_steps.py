"""The many-row attention over 8-bit codes reads the keys' operands of a step some products ahead: never more of them
than the step has, in any instance (128 rows of 64 dims have four)."""
import os
import subprocess

from paper_2606_13126_amd import build

CHECK = """
#include "pic_kv8.hip"
namespace pic { namespace {
template <int D, int WR> constexpr bool within() {
    typedef Kv8Many<D, WR> S;
    return S::TAKEN == D / 16 * (WR == 4 ? 1 : 2) && S::AHEAD >= 1 && S::AHEAD <= S::TAKEN;
}
static_assert(within<64, 4>() && within<64, 8>() && within<128, 4>() && within<128, 8>(), "read past a step's operands");
} }
"""


def test_reads_ahead_stay_within_a_step(tmp_path):
    src = tmp_path / "check.hip"
    src.write_text(CHECK)
    res = subprocess.run([build.hipcc(), "--offload-arch=gfx950", "-std=c++17", "-fsyntax-only", "-I",
                          build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(src)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
