"""What the paged cache and its attention say of their memory and their launches, without a GPU."""
import os
import shutil
import subprocess
import sys
import textwrap

import numpy as np
import pytest

from paper_2309_15531_amd import binding as B
from test_cache_host_cpu import CALLS
from test_host_path_cpu import PREAMBLE

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    if not os.path.exists(B.LIB_PATH):
        from paper_2309_15531_amd.build import build
        build(verbose=False)
    fake = tmp_path_factory.mktemp("fake") / "libfake_hip.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "host", "fake_hip_events.cpp"), "-o", str(fake)], check=True)

    def go(body):
        res = subprocess.run([sys.executable, "-c", PREAMBLE + "from ctypes import c_float\n" + CALLS + textwrap.dedent(body), str(fake), B.LIB_PATH],
                             capture_output=True, text=True, timeout=120)
        assert res.returncode == 0, res.stdout + res.stderr
    return go


@pytest.mark.parametrize("pages,page,heads,dim", [(1 << 25, 64, 1, 64), (1 << 26, 32, 1, 64), (2 ** 31 - 1, 32, 8, 128), (1 << 15, 1 << 16, 1, 256),
                                                  (2 ** 31 - 1, 65536, 1024, 256)])
def test_a_pool_of_2_31_positions_has_no_size(pages, page, heads, dim):
    """No other call takes one, and the largest product of these numbers passes 64 bits."""
    assert B.load_library().adadim_mx4_cache_bytes(pages, page, heads, dim) == 0


def test_the_largest_pools_have_their_size():
    for pages, page, heads, dim in (((1 << 26) - 1, 32, 1024, 256), ((1 << 15) - 1, 1 << 16, 1024, 256)):
        assert B.load_library().adadim_mx4_cache_bytes(pages, page, heads, dim) == int(np.prod(B.mx4_cache_shape(pages, page, heads, dim), dtype=object))


def test_a_profile_charges_each_launch_once(run):
    """The events of a kernel frame its launch alone: of two launches of a call the second does not lie within the first one's."""
    run("""
    ctx = context()
    assert attend(ctx, 300, 100000, group=1) == OK             # (clears the counters)
    assert lib.adadim_profile(ctx, 1) == OK
    for call, kernels in ((lambda: attend(ctx, 300, 100000, group=1), ("mx4_attend_tiles", "mx4_attend_join")), (lambda: attend(ctx, 1, 100000), ("mx4_attend_few",)),
                          (lambda: reserve(ctx, 9000), ("cache_reserve_plan", "cache_reserve_rows")), (lambda: trim(ctx, 1, 70000), ("cache_trim_plan", "cache_trim_pages"))):
        fake.fake_reset()
        assert call() == OK, lib.adadim_last_error(ctx)
        order = [c.split()[0] if c == "record" else c.split()[1] for c in calls() if c == "record" or c.startswith("launch")]
        assert len(order) == 3 * len(kernels), order
        for i, k in enumerate(kernels):
            assert order[3 * i] == order[3 * i + 2] == "record" and k in order[3 * i + 1], order
    """)
