"""Host-side checks of the decode entry points and of their binding that need no GPU, beside test_decode_abi.py."""
import pytest

from paper_2607_25291_amd import binding as B


def refused(status, call, *a, **kw):
    with pytest.raises(B.CosaError) as e:
        call(*a, **kw)
    assert e.value.status == status, str(e.value)


def test_outputs_of_an_empty_page_map_must_not_overlap():
    def call(cu=None, slots=None, rows=0, taken=None):
        B.cosa_page_map(0, 16, 8, None, None, None, 0, None, None, None, cu, slots, rows, taken, stream=0)
    call()
    call(rows=9)  # nothing to write to
    for kw in (dict(cu=4096, taken=4096), dict(cu=4096, slots=4088, rows=2), dict(taken=4096 + 8 * 9 - 4, slots=4096, rows=9)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
        assert "overlap" in B.cosa_last_error()


class Cuda:
    """A tensor that says it lives on a GPU."""

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def two_gpus(monkeypatch):
    """Two GPUs whose current streams are the default ones; calls return (device they were made on, stream)."""
    import torch
    state = {"current": 0, "calls": []}

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, state["current"] = state["current"], self.index

        def __exit__(self, *_):
            state["current"] = self.before

    class Lib:
        def __getattr__(self, name):
            def call(*args):
                state["calls"].append((name, state["current"], args[-1]))
                return B.COSA_OK
            return call
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(B, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(B, "_get_device", lambda: state["current"])
    monkeypatch.setattr(B, "lib", Lib)
    return state


def all_calls(t, q, **kw):
    """Every entry point that enqueues work, with t for its tensors and q for rows [4, 8, 128] of them."""
    p, kv, b = B.DecodeProblem(4, 8, 8, 32), B.CosaPagedKv(16, 16, 16, 64, 16), B.page_budget(8)
    B.cosa_page_map(4, 64, 32, t, t, t, 4, t, t, t, t, t, 4, t, **kw)
    B.cosa_kv_append(8, 128, 64, 16, t, t, t, 4, q, q, t, **kw)
    B.cosa_page_score(p, q, kv, t, t, t, **kw)
    B.cosa_page_select(p, 64, t, t, b, t, t, **kw)
    B.cosa_decode_attention(p, q, kv, t, t, 64, t, **kw)
    B.cosa_decode_attention_listed(p, q, kv, t, t, t, 8, t, 64, t, **kw)
    B.cosa_decode_sparse(p, q, kv, t, t, b, t, 64, t, **kw)


@pytest.mark.parametrize("stream", [None, 0, "default", "own"])
@pytest.mark.parametrize("device", [0, 1])
def test_default_streams_are_those_of_the_tensors_device(two_gpus, device, stream):
    """The null stream belongs to whichever device is current: work on another one's tensors is enqueued with that device
    current, which then is as it was. A stream of its own names its device itself."""
    import torch

    class Stream:
        cuda_stream = 0 if stream == "default" else 1 << 20
        device = torch.device("cuda", 1)
    t = Cuda(torch.zeros(4, dtype=torch.int32), device)
    q = Cuda(torch.zeros(4, 8, 128, dtype=torch.bfloat16), device)
    kw = {"stream": Stream() if isinstance(stream, str) else stream}
    if isinstance(stream, str) and device == 0:
        with pytest.raises(ValueError):
            all_calls(t, q, **kw)
        return
    all_calls(t, q, **kw)
    assert two_gpus["current"] == 0 and len(two_gpus["calls"]) == 7
    for name, current, handle in two_gpus["calls"]:
        if stream == "own":
            assert handle == 1 << 20, name
        else:
            assert (current, handle) == (device, 0), name


def test_a_budget_above_the_tables_width_is_no_longer_list():
    """cosa_decode_sparse: a list holds at most the table's pages, so a larger budget is neither too long nor too much
    work; the lists' memory is what it asks for."""
    def call(budget, max_pages=32, page=64, ws=None, batch=4):
        B.cosa_decode_sparse(B.DecodeProblem(batch, 8, 2, max_pages), 16, B.CosaPagedKv(16, 16, 16, page, 16), 16, 16, budget,
                             ws, 0, 1 << 30, stream=0)
    for page, pages in ((64, 1 << 25), (1 << 20, 1 << 11), (16, 2 ** 31 - 1), (1 << 20, 2 ** 31 - 1)):
        # everything is right but the workspace
        refused(B.COSA_ERR_WORKSPACE, call, B.page_budget(pages), page=page)
        refused(B.COSA_ERR_WORKSPACE, call, B.page_budget(pages), page=page, max_pages=0)
        call(B.page_budget(pages), page=page, batch=0)
    # where the table is as wide, the limits are its own
    refused(B.COSA_ERR_UNSUPPORTED, call, B.page_budget(1 << 11), page=1 << 20, max_pages=1 << 11)


def test_rows_that_are_not_the_problems(two_gpus):
    """Query, key and value tensors must hold the rows that the call reads: its heads and head_dim, at least its sequences
    or tokens, two bytes an element."""
    import torch
    z = lambda *s, dt=torch.bfloat16: Cuda(torch.zeros(*s, dtype=dt))
    t = Cuda(torch.zeros(4, dtype=torch.int32))
    good = z(4, 8, 128)
    all_calls(t, good)
    all_calls(t, z(6, 8, 128))                     # padded
    all_calls(t, Cuda(torch.zeros(4, 24, 128, dtype=torch.int16)[:, 8:16]))
    p, kv, b = B.DecodeProblem(4, 8, 8, 32), B.CosaPagedKv(16, 16, 16, 64, 16), B.page_budget(8)
    calls = [lambda q: B.cosa_kv_append(8, 128, 64, 16, t, t, t, 4, q, good, t),
             lambda q: B.cosa_kv_append(8, 128, 64, 16, t, t, t, 4, good, q, t),
             lambda q: B.cosa_page_score(p, q, kv, t, t, t),
             lambda q: B.cosa_decode_attention(p, q, kv, t, t, 64, t),
             lambda q: B.cosa_decode_attention_listed(p, q, kv, t, t, t, 8, t, 64, t),
             lambda q: B.cosa_decode_sparse(p, q, kv, t, t, b, t, 64, t)]
    n = len(two_gpus["calls"])
    for call in calls:
        for bad in (z(3, 8, 128), z(4, 24, 128), z(4, 4, 128), z(4, 8, 64), z(4, 8, 256), z(4, 1024),
                    z(4, 8, 128, dt=torch.float32), z(4, 8, 128, dt=torch.uint8)):
            with pytest.raises(ValueError):
                call(bad)
    assert len(two_gpus["calls"]) == n
    # a raw C problem says the same, and raw pointers pass
    raw = B.CosaDecodeProblem(4, 8, 8, 128, 32, 0, 0.0)
    B.cosa_page_score(raw, good, kv, t, t, t)
    B.cosa_page_score(raw, 16, kv, t, t, t)
    with pytest.raises(ValueError):
        B.cosa_page_score(raw, z(4, 24, 128), kv, t, t, t)
    B.cosa_kv_append(8, 128, 64, 16, t, t, t, 0, z(0, 8, 128), z(0, 8, 128), t)
