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


@pytest.mark.parametrize("dim,few,many", [(64, 18, 139), (128, 35, 274), (256, 68, 542)])
def test_partial_sums_stay_within_the_scratch_that_is_stated(run, dim, few, many):
    """Batches of all sizes, with hints that fit them and others; the bounds in units of 10^6 bytes, with the counters."""
    run(f"""
    import random
    r = random.Random({dim})
    largest = {{True: 0, False: 0}}
    contexts = {{True: context(), False: context()}}
    for i in range(6000):
        n, heads, group = r.choice((1, 1, 2, 7, 64, 300, 4096)), r.choice((1, 1, 2, 8, 32)), r.choice((1, 4, 16))
        tokens = min(n * r.choice((1, 4, 33, 300, 4000, 30000)), 1 << 20, (1 << 25) // (heads * group))
        hint, length, window = r.choice((0, 1, 17, 257, 3000)), r.choice((0, 100, 5000, 100000, 1 << 20)), r.choice((0, 0, 3000))
        new = -(-tokens // n) if hint == 0 else min(hint, tokens)
        few = new * group <= 256
        fake.fake_reset()
        assert lib.adadim_mx4_attention(contexts[few], A, 0, c_int64(tokens), c_int64(heads * group * {dim}), heads * group, A, c_int64(1 << 20), 64, heads, {dim},
                                        A, c_int64(1 << 14), n, A, A, A, 0, c_int64(heads * group * {dim}), c_float(1.0), 1, c_int64(window), c_int64(hint),
                                        c_int64(length)) == OK, lib.adadim_last_error(contexts[few])
        assert any(("mx4_attend_few" if few else "mx4_attend_tiles") in c for c in calls()), calls()
        largest[few] = max([largest[few]] + [int(c.split()[1]) for c in calls() if c.startswith("hipMalloc")])
    assert {few} * 0.9e6 < largest[True] <= {few} * 1e6 and {many} * 0.9e6 < largest[False] <= {many} * 1e6, largest
    """)
