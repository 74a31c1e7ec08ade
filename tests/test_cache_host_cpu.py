"""The host path of the paged cache and its attention, without a GPU: which kernels a call launches, and its scratch."""
import pytest

from test_mx4_host_cpu import run  # noqa: F401  (the fixture)

CALLS = """
def attend(ctx, new, length, sequences=1, group=8, heads=8, dim=128, window=0):
    n = sequences * new
    return lib.adadim_mx4_attention(ctx, A, 0, c_int64(n), c_int64(heads * group * dim), heads * group, A, c_int64(1 << 20), 64, heads, dim, A,
                                    c_int64(1 << 14), sequences, A, A, A, 0, c_int64(heads * group * dim), c_float(1.0), 1, c_int64(window),
                                    c_int64(new), c_int64(length))
def reserve(ctx, tokens, n=4):
    return lib.adadim_cache_reserve(ctx, A, A, n, 64, A, c_int64(100), A, c_int64(100), A, A, A, A, A, c_int64(tokens), A, A)
def trim(ctx, n, width):
    return lib.adadim_cache_trim(ctx, A, A, n, 64, A, c_int64(width), A, c_int64(100), A, A, A)
def launched(*of):
    return [next((k for k in of if k in c), c) for c in names()]
"""
ATTEND = "launched('mx4_attend_zero', 'mx4_attend_few', 'mx4_attend_tiles', 'mx4_attend_join')"


def body(text):
    return "from ctypes import c_float\n" + CALLS + text


def test_launches_of_a_call(run):
    run(body(f"""
ctx = context()
def of(call):
    fake.fake_reset()
    assert call == OK, lib.adadim_last_error(ctx)
for new, length, group, want in ((1, 100, 8, ['few']), (32, 100, 8, ['few']), (33, 100, 8, ['tiles']), (1, 100000, 8, ['zero', 'few']), (1, 100000, 8, ['few']),
                                 (300, 100000, 1, ['zero', 'tiles', 'join']), (300, 100000, 1, ['tiles', 'join']), (1000, 100, 1, ['tiles']), (1, 5, 1024, ['tiles'])):
    fake.fake_reset()
    assert attend(ctx, new, length, group=group) == OK, lib.adadim_last_error(ctx)
    assert {ATTEND} == ['mx4_attend_' + w for w in want], (new, length, names())
# of new tokens nothing is known: the mean of 64 sequences' 64 is one each
fake.fake_reset()
assert lib.adadim_mx4_attention(ctx, A, 0, c_int64(64), c_int64(8192), 64, A, c_int64(1 << 20), 64, 8, 128, A, c_int64(16), 64, A, A, A, 0, c_int64(8192),
                                c_float(1.0), 1, c_int64(0), c_int64(0), c_int64(0)) == OK and {ATTEND} == ['mx4_attend_few'], names()
fake.fake_reset()
assert attend(ctx, 1, 1000, sequences=4096) == OK and {ATTEND} == ['mx4_attend_few']
for tokens, want in ((0, 1), (8192, 1), (8193, 2), (1 << 20, 2)):
    fake.fake_reset()
    assert reserve(ctx, tokens) == OK and len(names()) == want, (tokens, names())
for n, width, want in ((1, 65536, 1), (1, 65537, 2), (4096, 16, 1), (4096, 17, 2)):
    fake.fake_reset()
    assert trim(ctx, n, width) == OK and len(names()) == want, (n, width, names())
"""))


def test_counters_are_cleared_again_after_a_failed_growth(run):
    """Who finds itself last joins the shares: with other than zeros to count from there may be none."""
    run(body(f"""
ctx = context()
assert attend(ctx, 1, 100000) == OK
fake.fake_reset()
assert attend(ctx, 1, 100000) == OK and {ATTEND} == ['mx4_attend_few']
fake.fake_reset()
fake.fake_fail(b"hipMalloc", 1)
assert attend(ctx, 2, 100000, sequences=8) == EHIP
for again in range(2):
    fake.fake_reset()
    assert attend(ctx, 1, 100000) == OK, lib.adadim_last_error(ctx)
    assert {ATTEND} == (['mx4_attend_zero', 'mx4_attend_few'] if again == 0 else ['mx4_attend_few']), names()
fake.fake_reset()
fake.fake_fail(b"mx4_attend_few", 1)
assert attend(ctx, 1, 100000) == EHIP
assert attend(ctx, 1, 100000) == OK
"""))


def test_scratch_does_not_grow_while_a_graph_is_recorded(run):
    run(body("""
for call, small in ((lambda c: attend(c, 1, 100000), lambda c: attend(c, 1, 100)), (lambda c: reserve(c, 9000), lambda c: reserve(c, 50)),
                    (lambda c: trim(c, 1, 70000), lambda c: trim(c, 1, 20))):
    ctx, g = context(), c_void_p()
    assert small(ctx) == OK
    assert lib.adadim_capture_begin(ctx) == OK
    assert small(ctx) == OK and call(ctx) == EHIP and b"scratch" in lib.adadim_last_error(ctx)
    assert lib.adadim_capture_end(ctx, byref(g)) == OK
    lib.adadim_graph_destroy(g)
    assert call(ctx) == OK
    assert lib.adadim_capture_begin(ctx) == OK
    assert call(ctx) == OK, lib.adadim_last_error(ctx)
    assert lib.adadim_capture_end(ctx, byref(g)) == OK
    lib.adadim_graph_destroy(g)
"""))
