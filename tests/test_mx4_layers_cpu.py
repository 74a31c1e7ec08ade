"""The layers over the microscaled operators without a GPU: on which stream they allocate and compute, and in which order streams wait.

The library runs on its context's stream, torch on its current one.  Here both are written down by stand-ins that compute nothing."""
import contextlib

import pytest
import torch

from paper_2309_15531_amd import mx4


class Stream:
    def __init__(self, log, number):
        self.log, self.cuda_stream = log, number

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))


class Machine:
    """torch.cuda's streams and a context: every library call, allocation and activation with the stream that is current."""

    def __init__(self, monkeypatch, own, current):
        self.log, self.stream, self.recording = [], own, None
        self.current = [Stream(self.log, current)]

        @contextlib.contextmanager
        def stream(s):
            self.current.append(s)
            try:
                yield
            finally:
                self.current.pop()

        empty = torch.empty

        def allocate(*size, device=None, **kw):
            self.log.append(("empty", self.current[-1].cuda_stream))
            return empty(*size, **kw)

        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.current[-1])
        monkeypatch.setattr(mx4, "_raw_stream", lambda device: self.current[-1].cuda_stream, raising=False)
        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda n, *a: Stream(self.log, n))
        monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: Stream(self.log, 0))
        monkeypatch.setattr(mx4.torch, "empty", allocate)

    def __getattr__(self, name):
        if not name.startswith("adadim_"):
            raise AttributeError(name)
        return lambda *a, **k: self.log.append((name, self.current[-1].cuda_stream))

    def alloc_score(self, rows, cols, device):
        return torch.empty(rows * cols, dtype=torch.float16)

    def activation(self, h):
        self.log.append(("activation", self.current[-1].cuda_stream))
        return h[:, :64]


class Hessian:
    colscale = Hs = hmeta = None


def calls(m):
    """(name of the call, what it does) of everything that a user can do with a layer."""
    one, up, down = mx4.Mx4Weight(m, 64, 32), mx4.Mx4Weight(m, 96, 32, 4), mx4.Mx4Weight(m, 32, 64, 4)
    x, logits = torch.zeros(5, 32, dtype=torch.bfloat16), torch.zeros(5, 4)
    del m.log[:]
    return {
        "store": lambda: one.store(torch.zeros(64, 32)), "scored": lambda: up.store(torch.zeros(96, 32), 1, Hessian),
        "values": lambda: one.values(), "quantize_rows": lambda: mx4.quantize_rows(m, x),
        "linear": lambda: mx4.Mx4Linear(one)(x), "linear mx4": lambda: mx4.Mx4Linear(one, mx4_inputs=1)(x),
        "experts": lambda: mx4.Mx4Experts(up, down, 2, m.activation)(x, logits),
        "experts mx4": lambda: mx4.Mx4Experts(up, down, 2, m.activation, mx4_inputs=1)(x, logits),
        "experts into Y": lambda: mx4.Mx4Experts(up, down, 2, m.activation)(x, logits, torch.zeros(5, 32)),
    }


NAMES = ["store", "scored", "values", "quantize_rows", "linear", "linear mx4", "experts", "experts mx4", "experts into Y"]


@pytest.mark.parametrize("what", NAMES)
@pytest.mark.parametrize("own,current", [(7, 3), (0, 3), (7, 0)])
def test_with_another_current_stream_the_streams_wait_for_each_other(monkeypatch, what, own, current):
    """The context's stream waits for the caller's before the first library call, the caller's for the context's behind the last; between
    them torch's own work and the memory that does not outlast the call are the context's."""
    m = Machine(monkeypatch, own, current)
    calls(m)[what]()
    log = m.log
    first, last = log.index(("wait", own, current)), log.index(("wait", current, own))
    assert [e for e in log if e[0] == "wait"] == [log[first], log[last]] and last == len(log) - 1
    assert all(e[0] == "empty" and e[1] == current for e in log[:first]), "what the caller gets is the caller's stream's"
    assert len(log[first + 1:last]) > 0 and all(e[1] == own for e in log[first + 1:last]), log
    assert any(e[0] == "activation" for e in log) == what.startswith("experts")
    assert m.current[-1].cuda_stream == current and len(m.current) == 1


@pytest.mark.parametrize("what", NAMES)
@pytest.mark.parametrize("number", [0, 7])
def test_on_the_contexts_own_stream_nothing_waits(monkeypatch, what, number):
    m = Machine(monkeypatch, number, number)
    calls(m)[what]()
    assert not any(e[0] == "wait" for e in m.log) and {e[1] for e in m.log} == {number}


@pytest.mark.parametrize("what", ["linear", "experts"])
def test_a_call_that_raises_leaves_the_streams_in_order(monkeypatch, what):
    m = Machine(monkeypatch, 7, 3)
    call = calls(m)[what]

    def refuse(*a, **k):
        raise ValueError("no")
    m.adadim_mx4_matmul = m.adadim_expert_combine = refuse
    with pytest.raises(ValueError, match="no"):
        call()
    assert m.log[-1] == ("wait", 3, 7) and len(m.current) == 1


# ------------------------------------------------------------------------------------------ while a graph is recorded
class Library:
    """Stands in for the shared library: every call succeeds, a recording yields the next handle."""

    def __init__(self):
        self.graphs = 0

    def __getattr__(self, name):
        return lambda *a: 0

    def adadim_capture_end(self, h, out):
        self.graphs += 1
        out._obj.value = 100 + self.graphs
        return 0


class Pool:
    live = []

    def __init__(self):
        Pool.live.append(self)


def recorder(monkeypatch, own, current):
    """A context with its own bookkeeping of recordings, and the pool that torch allocates from at each call."""
    from paper_2309_15531_amd import binding as B
    m = Machine(monkeypatch, own, current)
    pools = [None]

    @contextlib.contextmanager
    def use(pool):
        assert pools[-1] is None, "pools do not nest"
        pools.append(pool)
        try:
            yield
        finally:
            pools.pop()

    class Recorder(B.Context):
        def __init__(self):
            self._lib, self._h, self.stream = Library(), None, own
            self._graphs = {}

        alloc_score = lambda self, rows, cols, device: torch.empty(rows * cols, dtype=torch.float16)

    for name in dir(B.Context):
        if name.startswith(("adadim_mx4", "adadim_expert", "adadim_layer")):
            setattr(Recorder, name, lambda self, *a, _n=name, **k: m.log.append((_n, m.current[-1].cuda_stream)))
    empty = mx4.torch.empty

    def allocate(*size, **kw):
        m.log.append(("from", pools[-1]))
        return empty(*size, **kw)
    Pool.live = []
    monkeypatch.setattr(torch.cuda, "MemPool", Pool)
    monkeypatch.setattr(torch.cuda, "use_mem_pool", use)
    monkeypatch.setattr(mx4.torch, "empty", allocate)
    c = Recorder()
    c.log, c.activation = m.log, lambda h: torch.empty(h.shape[0], 64)
    return c


@pytest.mark.parametrize("what", NAMES)
def test_what_a_recorded_call_allocates_lives_as_long_as_the_graph(monkeypatch, what):
    """A replay writes to the addresses of the recording: they belong to a pool that nothing else takes memory from."""
    c = recorder(monkeypatch, 7, 7)
    todo = calls(c)
    c.adadim_capture_begin()
    todo[what]()
    todo[what]()
    graph = c.adadim_capture_end()
    taken = [e[1] for e in c.log if e[0] == "from"]
    if taken:
        assert len(Pool.live) == 1 and all(p is Pool.live[0] for p in taken), "one pool for the whole recording, and no other memory"
        assert c._graphs[graph] == [Pool.live[0]]
    else:
        assert what == "store"
    del c.log[:]
    todo[what]()
    assert all(e[1] is None for e in c.log if e[0] == "from"), "behind the recording memory is ordinary again"
    c.adadim_graph_destroy(graph)
    assert not c._graphs


def test_recordings_keep_what_is_theirs(monkeypatch):
    c = recorder(monkeypatch, 7, 7)
    todo = calls(c)
    graphs = []
    for _ in range(2):
        c.adadim_capture_begin()
        todo["experts mx4"]()
        graphs.append(c.adadim_capture_end())
    c.adadim_capture_begin()
    graphs.append(c.adadim_capture_end())
    assert [c._graphs.get(g) for g in graphs] == [[Pool.live[0]], [Pool.live[1]], None]
    c.adadim_graph_destroy(graphs[0])
    c.adadim_graph_destroy(None)
    assert list(c._graphs) == [graphs[1]]


def test_a_recording_that_fails_keeps_nothing(monkeypatch):
    from paper_2309_15531_amd import binding as B
    c = recorder(monkeypatch, 7, 7)
    todo = calls(c)
    c.adadim_capture_begin()
    todo["linear mx4"]()
    c._lib.adadim_capture_end = lambda h, out: B.EHIP
    c.last_error = lambda: "no"
    with pytest.raises(B.AdaDimError):
        c.adadim_capture_end()
    assert c.recording is None and not c._graphs
    c._lib.adadim_capture_begin = lambda h: B.EINVAL
    with pytest.raises(B.AdaDimError):
        c.adadim_capture_begin()
    assert c.recording is None


@pytest.mark.parametrize("what", NAMES)
def test_from_another_stream_nothing_is_recorded(monkeypatch, what):
    """Torch's own work there would not be part of the recording, and waiting for it would break it."""
    c = recorder(monkeypatch, 7, 3)
    todo = calls(c)
    c.adadim_capture_begin()
    with pytest.raises(ValueError, match="stream"):
        todo[what]()
    assert not any(e[0] == "wait" or e[0].startswith("adadim_") for e in c.log)


def test_host_tensors_are_refused_by_name():
    from paper_2309_15531_amd import binding as B
    ctx = B.Context(stream=0)
    one = mx4.Mx4Weight(ctx, 64, 32, device="cpu")
    for call in (lambda: mx4.Mx4Linear(one)(torch.zeros(5, 32, dtype=torch.bfloat16)), lambda: one.store(torch.zeros(64, 32)),
                 lambda: mx4.quantize_rows(ctx, torch.zeros(5, 32)), lambda: one.values()):
        with pytest.raises(TypeError, match="device tensor"):
            call()
    ctx.close()
