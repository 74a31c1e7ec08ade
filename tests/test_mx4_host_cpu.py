"""The host path of the microscaled operators: memory that a kernel would read where there is none, without a GPU."""
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

from mx4_group_forms import MX4_GROUP_FORMS
from paper_2309_15531_amd import binding as B
from test_host_path_cpu import PREAMBLE
from test_mx4_plan_cpu import plans  # noqa: F401  (the fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
def matmul(ctx, rows, out, inn):
    return lib.adadim_mx4_matmul(ctx, A, None, 0, c_int64(rows), c_int64(inn), A, A, c_int64(out), c_int64(inn), A, 2, c_int64(out))
def experts(ctx, x_type, tokens, rows, out, inn, n=8, X=A, xs=A):
    return lib.adadim_mx4_matmul_experts(ctx, X, xs, x_type, c_int64(tokens), c_int64(inn), A, c_int64(rows), A, n, A, A, c_int64(out),
                                         c_int64(inn), A, 2, c_int64(out))
def names():
    return [c.split()[1] for c in calls() if c.startswith("launch")]
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    if not os.path.exists(B.LIB_PATH):
        from paper_2309_15531_amd.build import build
        build(verbose=False)
    fake = tmp_path_factory.mktemp("fake") / "libfake_hip.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(ROOT, "tests", "host", "fake_hip_memory.cpp"), "-o",
                    str(fake)], check=True)

    def go(body):
        res = subprocess.run([sys.executable, "-c", PREAMBLE + CALLS + textwrap.dedent(body), str(fake), B.LIB_PATH],
                             capture_output=True, text=True, timeout=120)
        assert res.returncode == 0, res.stdout + res.stderr
        return res.stdout
    return go


@pytest.mark.parametrize("x_type", [B.TYPE_F16, B.TYPE_BF16, B.TYPE_MX4])
@pytest.mark.parametrize("rows,out,inn,kernel", [(3, 96, 256, "mx4_rows"), (619, 4312, 136, None), (1999, 837, 160, None), (5000, 4096, 1024, None)])
def test_without_tokens_no_kernel_reads_x(run, x_type, rows, out, inn, kernel):
    """No row of X exists, so rows[] can name none: rows of zeros.  X and its scales may be NULL then; what a kernel reads in place of a
    row that does not exist has to be memory of the library's own."""
    run(f"""
    ctx = context()
    for X in (None, A):
        fake.fake_reset()
        assert experts(ctx, {x_type}, 0, {rows}, {out}, {inn}, X=X, xs=X) == OK, lib.adadim_last_error(ctx)
        order = names()
        assert len(order) == 2 and "mx4_copy_rows" in order[0], order
        assert {kernel!r} is None or {kernel!r} in order[1], order
        given = dict(c.split() for c in calls() if c.startswith("x"))
        assert int(given["x"], 16) not in (0, A.value), given
        assert {x_type} != {B.TYPE_MX4} or int(given["x_scales"], 16) not in (0, A.value), given
    """)


@pytest.mark.parametrize("small,large,clear,kernel", [
    ("matmul(ctx, 12, 96, 8192)", "matmul(ctx, 40, 1500, 8192)", "mx4_zero_tickets", "mx4_rows"),
    ("gemv(ctx, 1024, 1024)", "gemv(ctx, 28672, 8192)", "gemv_zero", "gemv_ic_tiles"),
    # (the same columns at a larger pitch: nothing but the zeros behind the last token row grows)
    ("hessian(ctx, 4096)", "hessian(ctx, 16384)", "zero_f32", "gram_tiles")])
def test_memory_of_the_size_before_a_failed_growth_is_cleared_again(run, small, large, clear, kernel):
    """Growing frees a slot before it allocates.  Where the allocation fails, a call that needs what there was before gets new memory of the
    old size: the counters and zeros in it are not those that were cleared."""
    run(f"""
    def hessian(ctx, ldx):
        return lib.adadim_hessian(ctx, A, c_int64(4096), c_int64(4096), c_int64(ldx), A, 0)
    ctx = context()
    assert {small} == OK, lib.adadim_last_error(ctx)
    assert sum({clear!r} in c for c in names()) == 1, names()
    fake.fake_reset()
    assert {small} == OK and not any({clear!r} in c for c in names()), names()
    fake.fake_reset()
    fake.fake_fail(b"hipMalloc", 1)
    assert {large} == EHIP
    assert [c.split()[0] for c in calls() if c.startswith(("have", "free"))] == ["free"], calls()
    for again in range(2):
        fake.fake_reset()
        assert {small} == OK, lib.adadim_last_error(ctx)
        order = [c for c in names() if {clear!r} in c or {kernel!r} in c]
        assert [{clear!r} in c for c in order] == ([True, False] if again == 0 else [False]), order
    """)


def test_zeros_whose_clearing_was_only_recorded_are_cleared_again(run):
    """The clearing launch fails, and the next call is recorded: what it records has not run for the calls outside the graph."""
    run("""
    def hessian(ctx):
        return lib.adadim_hessian(ctx, A, c_int64(4096), c_int64(4096), c_int64(4096), A, 0)
    ctx = context()
    fake.fake_fail(b"zero_f32", 1)
    assert hessian(ctx) == EHIP
    g = c_void_p()
    assert lib.adadim_capture_begin(ctx) == OK
    assert hessian(ctx) == OK, lib.adadim_last_error(ctx)
    assert lib.adadim_capture_end(ctx, byref(g)) == OK
    for again in range(2):
        fake.fake_reset()
        assert hessian(ctx) == OK
        assert sum("zero_f32" in c for c in names()) == (again == 0), names()
    lib.adadim_graph_destroy(g)
    """)


def test_tickets_of_the_loss_whose_clearing_failed_are_cleared_by_the_next_call(run):
    """The workgroup that finds itself last writes the loss: with other than zeros to count from there may be none."""
    run("""
    def loss(ctx):
        arr = (c_void_p * 1)(A)
        return lib.adadim_layer_error_batch(ctx, 1, arr, 2, c_int64(512), c_int64(512), A, A, None, A)
    ctx = context()
    fake.fake_fail(b"fill_zero_f32", 2)                            # (the first clears the zeros behind the operands)
    assert loss(ctx) == EHIP
    for again in range(2):
        fake.fake_reset()
        assert loss(ctx) == OK, lib.adadim_last_error(ctx)
        assert sum("fill_zero_f32" in c for c in names()) == (again == 0), names()
    """)


@pytest.mark.parametrize("small,large", [
    ("matmul(ctx, 12, 96, 8192)", "matmul(ctx, 40, 1500, 8192)"),                                # counters and sums of shares
    ("matmul(ctx, 700, 512, 333)", "matmul(ctx, 3000, 512, 333)"),                               # X copied
    ("route(ctx, 700)", "route(ctx, 7000)"),                                                     # masks and counts of the chunks
    ("gemv(ctx, 1024, 1024)", "gemv(ctx, 28672, 8192)")])
def test_scratch_that_a_graph_was_recorded_with_outlives_the_calls_that_outgrow_it(run, small, large):
    """A graph holds the addresses of the context's scratch.  A larger call makes the slot grow; the replay afterwards must find its memory."""
    run(f"""
    def route(ctx, tokens):
        return lib.adadim_expert_route(ctx, A, 2, c_int64(tokens), c_int64(16), 16, 2, 1, A, A, A, A, A)
    def memory(what):
        return [c.split()[1] for c in calls() if c.split()[0] == what]
    ctx = context()
    assert {small} == OK, lib.adadim_last_error(ctx)
    held = memory("have")
    assert len(held) == 1, held
    g = c_void_p()
    assert lib.adadim_capture_begin(ctx) == OK
    assert {small} == OK, lib.adadim_last_error(ctx)
    assert lib.adadim_capture_end(ctx, byref(g)) == OK
    fake.fake_reset()
    assert {large} == OK, lib.adadim_last_error(ctx)
    assert len(memory("have")) == 1 and memory("free") == [], calls()
    assert lib.adadim_graph_launch(ctx, g) == OK
    # the larger one was recorded by nobody: it goes when it is outgrown in turn, and all go with the context
    assert {small} == OK and {large} == OK
    assert len(memory("have")) == 1 and memory("free") == [], calls()
    held += memory("have")
    lib.adadim_graph_destroy(g)
    lib.adadim_destroy(ctx)
    assert sorted(memory("free")) == sorted(held), (calls(), held)
    """)


def test_scratch_that_no_graph_was_recorded_with_is_given_back(run):
    run("""
    ctx = context()
    assert matmul(ctx, 12, 96, 8192) == OK and matmul(ctx, 40, 1500, 8192) == OK
    assert [c.split()[0] for c in calls() if c.startswith(("have", "free"))] == ["have", "free", "have"], calls()
    g = c_void_p()
    assert lib.adadim_capture_begin(ctx) == OK                     # (a recording of something else)
    assert gemv(ctx, 32, 4) != OK
    assert lib.adadim_capture_end(ctx, byref(g)) == OK
    fake.fake_reset()
    assert matmul(ctx, 263, 3651, 6120) == OK
    assert [c.split()[0] for c in calls() if c.startswith(("have", "free"))] == ["free", "have"], calls()
    """)


def test_no_launch_of_more_work_items_than_there_can_be(run):
    """A launch takes less than 2^32 threads along an axis.  Calls that would need more are refused, those that just do not are made."""
    run("""
    def quantize(ctx, rows, cols):
        return lib.adadim_mx4_quantize(ctx, A, 1, c_int64(rows), c_int64(cols), c_int64(cols), A, A, None, 0, None)
    def dequantize(ctx, rows, cols):
        return lib.adadim_mx4_dequantize(ctx, A, A, c_int64(rows), c_int64(cols), A, 1, c_int64(cols))
    def route(ctx, tokens, experts):
        return lib.adadim_expert_route(ctx, A, 2, c_int64(tokens), c_int64(experts), experts, 1, 1, A, A, A, A, A)
    def combine(ctx, tokens, cols):
        return lib.adadim_expert_combine(ctx, A, 1, c_int64(16), c_int64(cols), c_int64(cols), A, A, c_int64(tokens), 2, A, 1, c_int64(cols))
    def product(ctx, x_type, rows, out, inn):
        return lib.adadim_mx4_matmul(ctx, A, A, x_type, c_int64(rows), c_int64(inn), A, A, c_int64(out), c_int64(inn), A, 2, c_int64(out))
    def most():
        grids = [[int(v) for v in c.split()[2:5]] for c in calls() if c.startswith("launch")]
        return max((x * threads for x, y, threads in grids), default=0)
    ctx = context()
    top = 1 << 32
    edges = [(quantize, (1 << 28, 64), (1 << 28) - 16), (quantize, (1 << 20, 1 << 17), (1 << 20) - 16), (dequantize, (1 << 28, 512), (1 << 28) - 16),
             (combine, (1 << 24, 2048), (1 << 24) - 1), (combine, (1 << 23, 2049), (1 << 23) - 1), (combine, (1 << 30, 8), None),
             (route, (1 << 28, 4), None), (lambda c, n, i: product(c, 1, n, 64, i), (1 << 28, 1), None),
             (lambda c, n, i: product(c, 3, n, i, 128), (1 << 30, 512), None), (lambda c, n, i: product(c, 1, n, i, 128), (1 << 30, 512), None)]
    for call, (n, other), less in edges:
        fake.fake_reset()
        assert call(ctx, n, other) == EINVAL and not names(), (n, other, names(), most())
        if less:
            assert call(ctx, less, other) == OK and 0 < most() < top, (less, other, most(), lib.adadim_last_error(ctx))
    """)


def test_the_forms_of_many_experts(plans):  # noqa: F811
    sizes = [(rows, out, inn, experts, mx, 0) for mx, experts, rows, out, inn in MX4_GROUP_FORMS]
    assert [p[0] for p in plans(sizes)] == list(MX4_GROUP_FORMS.values())
    for mx in (False, True):
        assert {f for k, f in MX4_GROUP_FORMS.items() if k[0] == mx} == {"ring32", "ring64", "ring64w", "mid", "big"}
