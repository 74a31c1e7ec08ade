"""Which kernel a microscaled product takes, and the library's host path around the kernels that share a contraction, without a GPU."""
import os
import random
import shutil
import subprocess

import pytest

from mx4_forms import MX4_FORMS
from test_host_path_cpu import run  # noqa: F401  (the fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["rows", "ring32", "ring64", "ring64w", "mid", "big"]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """Lines "rows out in experts mx copy" to the plans, each checked to be one that the kernels can run."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = tmp_path_factory.mktemp("plan") / "mx4_plan_check"
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(ROOT, "tests", "host", "mx4_plan_check.cpp"), "-o", str(exe)], check=True)

    def go(sizes):
        text = "\n".join(" ".join(str(int(v)) for v in s) for s in sizes)
        lines = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=120).stdout.splitlines()
        assert len(lines) == len(sizes)
        for s, l in zip(sizes, lines):
            assert l.endswith(" ok"), (s, l)
        return [(NAMES[f], sh, o, r) for f, sh, o, r in ([int(v) for v in l.split()[:4]] for l in lines)]
    return go


def test_the_forms_of_the_listed_sizes(plans):
    sizes = [(rows, out, inn, experts, mx, not mx and inn % 8 != 0) for mx, experts, rows, out, inn in MX4_FORMS]
    assert plans(sizes) == list(MX4_FORMS.values())


def test_the_listed_sizes_reach_every_form():
    for mx in (False, True):
        for experts in (False, True):
            mine = {v for k, v in MX4_FORMS.items() if k[0] == mx and bool(k[1]) == experts}
            assert {f for f, *_ in mine} == set(NAMES)
            assert {s for _, s, *_ in mine} == ({1} if experts else {1, 2, 4, 8})
            assert {(o, r) for f, _, o, r in mine if f == "rows"} >= {(o, r) for o in (1, 2) for r in ((1, 2) if experts else (1, 2, 4))}
        assert any(k[0] == mx and v[2] == 4 for k, v in MX4_FORMS.items())


def test_plans_of_any_sizes(plans):
    r = random.Random(3)
    size = lambda top: int(2.0 ** r.uniform(0, top))
    sizes = [(size(20), size(18), size(18), r.choice([0, 0, 1, 2, 7, 64, 256, 1024]), mx, not mx and r.random() < 0.2)
             for mx in (0, 1) for _ in range(30000)]
    sizes += [(n, o, i, e, mx, 0) for n in (1, 2 ** 31 - 1) for o in (1, 2 ** 31 - 1) for i in (1, 2 ** 31 - 1) for e in (0, 1, 1024) for mx in (0, 1)]
    plans(sizes)


MATMUL = """
def product(ctx, rows, out, inn):
    return lib.adadim_mx4_matmul(ctx, A, None, 0, c_int64(rows), c_int64(inn), A, A, c_int64(out), c_int64(inn), A, 2, c_int64(out))
SHARED, LARGER, PLAIN = (12, 96, 8192), (40, 1500, 8192), (5, 4096, 128)
"""


@pytest.mark.parametrize("what,nth", [("hipMalloc", 1), ("mx4_zero_tickets", 1), ("mx4_rows", 1)])
def test_counters_of_shares_are_cleared_before_their_first_use(run, what, nth):  # noqa: F811
    """An allocation or a launch fails in the first call; the next one clears the counters before a kernel counts on them, once."""
    run(MATMUL + f"""
ctx = context()
fake.fake_fail(b"{what}", {nth})
assert product(ctx, *SHARED) == EHIP
assert product(ctx, *SHARED) == OK, lib.adadim_last_error(ctx)
assert product(ctx, *SHARED) == OK
order = [c.split()[1] for c in calls() if c.startswith("launch") and "mx4" in c]
assert "mx4_zero_tickets" in order[0] and sum("mx4_zero_tickets" in c for c in order) == 1, order
assert "mx4_rows" in order[-1], order
""")


def test_counters_of_shares_after_the_slot_grew_or_was_recorded(run):  # noqa: F811
    """A slot that has grown is other memory; a clearing that was only recorded has not run for the calls outside the graph."""
    run(MATMUL + """
ctx = context()
assert product(ctx, *PLAIN) == OK and not launched("mx4_zero_tickets")
assert product(ctx, *SHARED) == OK and len(launched("mx4_zero_tickets")) == 1
fake.fake_reset()
assert product(ctx, *SHARED) == OK and not launched("mx4_zero_tickets")
assert product(ctx, *LARGER) == OK and len(launched("mx4_zero_tickets")) == 1
fake.fake_reset()
assert product(ctx, *SHARED) == OK and not launched("mx4_zero_tickets")

ctx = context()
g = c_void_p()
assert lib.adadim_capture_begin(ctx) == OK
assert product(ctx, *SHARED) != OK                             # no room to be had while recording
assert lib.adadim_capture_end(ctx, byref(g)) == OK
lib.adadim_graph_destroy(g)

ctx = context()
fake.fake_fail(b"mx4_zero_tickets", 1)
assert product(ctx, *SHARED) == EHIP                           # the slot is there, its counters are not cleared
assert lib.adadim_capture_begin(ctx) == OK
assert product(ctx, *SHARED) == OK
assert lib.adadim_capture_end(ctx, byref(g)) == OK
fake.fake_reset()
assert product(ctx, *SHARED) == OK and len(launched("mx4_zero_tickets")) == 1
fake.fake_reset()
assert product(ctx, *SHARED) == OK and not launched("mx4_zero_tickets")
lib.adadim_graph_destroy(g)
""")


def test_failures_of_the_other_calls_fail_no_later_one(run):  # noqa: F811
    """An allocation or a launch that fails is reported by its own call and by no other; the next one does all its work."""
    run(MATMUL + """
def odd(ctx):                                                  # rows that have to be copied for the tiles
    return lib.adadim_mx4_matmul(ctx, A, None, 0, c_int64(700), c_int64(333), A, A, c_int64(512), c_int64(333), A, 2, c_int64(512))
def route(ctx, tokens=700):
    return lib.adadim_expert_route(ctx, A, 2, c_int64(tokens), c_int64(16), 16, 2, 1, A, A, A, A, A)
def experts(ctx):
    return lib.adadim_mx4_matmul_experts(ctx, A, None, 1, c_int64(8), c_int64(256), A, c_int64(16), A, 64, A, A, c_int64(96), c_int64(256), A, 1, c_int64(96))
def combine(ctx):
    return lib.adadim_expert_combine(ctx, A, 1, c_int64(16), c_int64(96), c_int64(96), A, A, c_int64(8), 2, A, 1, c_int64(96))
def quantize(ctx):
    return lib.adadim_mx4_quantize(ctx, A, 1, c_int64(8), c_int64(96), c_int64(96), A, A, None, 0, None)
def dequantize(ctx):
    return lib.adadim_mx4_dequantize(ctx, A, A, c_int64(8), c_int64(96), A, 1, c_int64(96))
for call, kernels, allocates in ((odd, ["mx4_copy_rows", "mx4_ring"], True), (route, ["route_choose", "route_place"], True),
                                 (lambda c: route(c, 5), ["route_choose"], False), (lambda c: route(c, 0), ["route_none"], False),
                                 (experts, ["mx4_rows"], False), (combine, ["combine_rows"], False),
                                 (quantize, ["mx4_quantize_rows"], False), (dequantize, ["mx4_dequantize_rows"], False)):
    for what in kernels + ["hipMalloc"] * allocates:
        ctx = context()
        fake.fake_reset()
        fake.fake_fail(what.encode(), 1)
        assert call(ctx) == EHIP, what
        assert product(ctx, *PLAIN) == OK, what
        fake.fake_reset()
        assert call(ctx) == OK, lib.adadim_last_error(ctx)
        order = [c.split()[1] for c in calls() if c.startswith("launch")]
        assert len(order) == len(kernels) and all(k in o for k, o in zip(kernels, order)), order
        lib.adadim_destroy(ctx)
# workgroups of the few-row kernel: for as many groups as there are rows
ctx = context()
fake.fake_reset()
assert experts(ctx) == OK
assert launched("mx4_rows")[0].split()[3] == "16", launched("mx4_rows")
""")
