"""Host-side checks of the decode entry points that need no GPU: declared and exported symbols, refusals
before anything is enqueued, workspace layout, and what the binding refuses."""
import ctypes
import dataclasses
import subprocess

import pytest

from paper_2607_25291_amd import binding as B

EXPECTED = {"cosa_page_map", "cosa_kv_append", "cosa_page_score", "cosa_page_select",
            "cosa_decode_workspace_bytes", "cosa_decode_attention", "cosa_decode_attention_listed",
            "cosa_decode_sparse_workspace_layout", "cosa_decode_sparse_workspace_bytes",
            "cosa_decode_sparse"}

GOOD = B.DecodeProblem(4, 8, 2, 32)
WS = 64 << 20
BUDGET = B.page_budget(8)


def kv(page=64, n_pages=16, k=16, v=16, table=16):
    return B.CosaPagedKv(k, v, table, page, n_pages)


def change(**kw):
    return dataclasses.replace(GOOD, **kw)


CALLS = {
    "score": lambda p=GOOD, c=None, q=16, bounds=16, lens=16, out=16: B.cosa_page_score(
        p, q, c or kv(), bounds, lens, out, stream=0),
    "decode": lambda p=GOOD, c=None, q=16, lens=16, ws=256, n=WS, o=1 << 30: B.cosa_decode_attention(
        p, q, c or kv(), lens, ws, n, o, stream=0),
    "listed": lambda p=GOOD, c=None, q=16, lens=16, ws=256, n=WS, o=1 << 30, pages=16, count=16, width=8:
        B.cosa_decode_attention_listed(p, q, c or kv(), lens, pages, count, width, ws, n, o, stream=0),
    "sparse": lambda p=GOOD, c=None, q=16, bounds=16, lens=16, budget=BUDGET, ws=256, n=WS, o=1 << 30:
        B.cosa_decode_sparse(p, q, c or kv(), bounds, lens, budget, ws, n, o, stream=0),
}


def refused(status, call, *a, **kw):
    with pytest.raises(B.CosaError) as e:
        call(*a, **kw)
    assert e.value.status == status, str(e.value)
    assert B.cosa_status_string(status) in str(e.value)


def test_symbols():
    assert set(B.declared_symbols(B.DECODE_HEADER_PATH)) == EXPECTED
    out = subprocess.run(["nm", "-D", "--defined-only", B.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    assert EXPECTED <= {line.split()[-1] for line in out.splitlines() if " T " in line}
    for name in EXPECTED:
        assert hasattr(B.lib(), name) and callable(getattr(B, name))


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("problem,status", [
    (change(batch=-1), B.COSA_ERR_INVALID_ARG),
    (change(max_pages=-1), B.COSA_ERR_INVALID_ARG),
    (change(n_q_heads=9), B.COSA_ERR_INVALID_ARG),
    (change(n_kv_heads=0), B.COSA_ERR_INVALID_ARG),
    (change(head_dim=0), B.COSA_ERR_INVALID_ARG),
    (change(head_dim=64), B.COSA_ERR_UNSUPPORTED),
    (change(q_stride=8 * 128 - 8), B.COSA_ERR_INVALID_ARG),
    (change(q_stride=8 * 128 + 4), B.COSA_ERR_INVALID_ARG),
    (change(q_stride=-8), B.COSA_ERR_INVALID_ARG),
    (change(sm_scale=-1.0), B.COSA_ERR_INVALID_ARG),
    (change(sm_scale=float("inf")), B.COSA_ERR_INVALID_ARG),
    (change(max_pages=1 << 25), B.COSA_ERR_UNSUPPORTED),      # 2^31 tokens at 64 a page
    (change(batch=1 << 30), B.COSA_ERR_UNSUPPORTED),
])
def test_problem_refusals(call, problem, status):
    refused(status, CALLS[call], problem)


@pytest.mark.parametrize("call", list(CALLS))
def test_cache_refusals(call):
    for bad in (kv(page=48), kv(page=8), kv(page=1 << 21), kv(n_pages=0), kv(n_pages=2 ** 31 + 1),
                kv(table=None)):
        refused(B.COSA_ERR_INVALID_ARG, CALLS[call], c=bad)
    if call != "score":
        for bad in (kv(k=None), kv(v=None), kv(k=24), kv(v=24)):
            refused(B.COSA_ERR_INVALID_ARG, CALLS[call], c=bad)
    refused(B.COSA_ERR_INVALID_ARG, CALLS[call], q=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS[call], q=8)
    refused(B.COSA_ERR_INVALID_ARG, CALLS[call], lens=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS[call], **{"out" if call == "score" else "o": None})
    if call != "score":
        # queries of 4 sequences, 2048 bytes each: o inside them, and just behind
        for o in (16, 16 + 4 * 2048 - 16):
            refused(B.COSA_ERR_INVALID_ARG, CALLS[call], o=o)
            assert "overlap" in B.cosa_last_error()
        refused(B.COSA_ERR_WORKSPACE, CALLS[call], o=16 + 4 * 2048, ws=None)


def test_workspace_refusals():
    need = {"decode": B.cosa_decode_workspace_bytes(GOOD), "listed": B.cosa_decode_workspace_bytes(GOOD),
            "sparse": B.cosa_decode_sparse_workspace_bytes(GOOD, BUDGET)}
    for call, n in need.items():
        refused(B.COSA_ERR_WORKSPACE, CALLS[call], n=n - 1)
        refused(B.COSA_ERR_WORKSPACE, CALLS[call], ws=None)
        refused(B.COSA_ERR_INVALID_ARG, CALLS[call], ws=264)
        refused(B.COSA_ERR_INVALID_ARG, CALLS[call], o=24)


def test_list_and_budget_refusals():
    refused(B.COSA_ERR_INVALID_ARG, CALLS["listed"], pages=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS["listed"], count=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS["listed"], width=0)
    refused(B.COSA_ERR_UNSUPPORTED, CALLS["listed"], width=1 << 25)
    select = lambda p=GOOD, page=64, lens=16, score=16, b=BUDGET, pages=16, count=16: B.cosa_page_select(
        p, page, lens, score, b, pages, count, stream=0)
    for kw in (dict(fraction=0.0), dict(fraction=1.5), dict(fraction=float("nan")), dict(min_pages=0),
               dict(min_pages=9), dict(sink_pages=-1), dict(recent_pages=-1), dict(sink_pages=5, recent_pages=4)):
        bad = B.page_budget(8, **kw)
        refused(B.COSA_ERR_INVALID_ARG, select, b=bad)
        refused(B.COSA_ERR_INVALID_ARG, CALLS["sparse"], budget=bad)
    refused(B.COSA_ERR_INVALID_ARG, select, b=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS["sparse"], budget=None)
    for kw in (dict(lens=None), dict(score=None), dict(pages=None), dict(count=None), dict(page=24)):
        refused(B.COSA_ERR_INVALID_ARG, select, **kw)
    refused(B.COSA_ERR_UNSUPPORTED, select, p=change(max_pages=32769))
    refused(B.COSA_ERR_UNSUPPORTED, CALLS["sparse"], p=change(max_pages=32769))
    refused(B.COSA_ERR_UNSUPPORTED, select, p=change(n_q_heads=2 * 1025))
    refused(B.COSA_ERR_INVALID_ARG, CALLS["sparse"], bounds=None)
    refused(B.COSA_ERR_INVALID_ARG, CALLS["score"], bounds=24)


def test_page_map_refusals():
    def call(batch=4, page=16, width=8, cached=4096, new=8192, free=12288, cap=5, n_free=16384, table=20480, lens=24576,
             cu=28672, slots=32768, rows=9, taken=36864):
        B.cosa_page_map(batch, page, width, cached, new, free, cap, n_free, table, lens, cu, slots, rows, taken, stream=0)
    for kw in (dict(batch=-1), dict(page=0), dict(page=20), dict(width=-1), dict(cap=-1), dict(rows=-1),
               dict(cached=None), dict(new=None), dict(free=None), dict(n_free=None), dict(table=None),
               dict(lens=None), dict(cu=None), dict(slots=None), dict(taken=None)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
    # in place, one array for two outputs, the end of one in the other
    for kw in (dict(lens=4096), dict(lens=8192), dict(taken=16384), dict(table=12288), dict(cu=24576),
               dict(taken=32768 + 8 * 9 - 4), dict(table=24576 - 4 * 4 * 8 + 4), dict(cu=4096 - 4 * 5 + 4)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
        assert "overlap" in B.cosa_last_error()
    refused(B.COSA_ERR_UNSUPPORTED, call, batch=8193)
    refused(B.COSA_ERR_UNSUPPORTED, call, width=1 << 27)


def test_append_refusals():
    def call(heads=2, d=128, page=16, n_pages=4, kc=1 << 20, vc=2 << 20, bounds=3 << 20, n=3, k=4 << 20, v=5 << 20,
             slots=6 << 20, ks=0, vs=0):
        B.cosa_kv_append(heads, d, page, n_pages, kc, vc, bounds, n, k, v, slots, ks, vs, stream=0)
    for kw in (dict(heads=0), dict(d=0), dict(page=33), dict(n_pages=0), dict(n=-1), dict(kc=None), dict(vc=None),
               dict(k=None), dict(v=None), dict(slots=None), dict(kc=8), dict(vc=8), dict(bounds=8), dict(k=8),
               dict(v=8), dict(ks=248), dict(vs=260), dict(ks=-8)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
    # rows taken from the caches, one cache for both, the last row's end in a cache
    for kw in (dict(k=(1 << 20) + 1024), dict(v=2 << 20), dict(slots=(1 << 20) + 32768 - 8), dict(vc=1 << 20),
               dict(bounds=(1 << 20) + 32768 - 16), dict(k=(2 << 20) - 2 * (2 * 512 + 256) + 16, ks=512),
               dict(bounds=(4 << 20) - 4096 + 16)):
        refused(B.COSA_ERR_INVALID_ARG, call, **kw)
        assert "overlap" in B.cosa_last_error(), kw
    refused(B.COSA_ERR_UNSUPPORTED, call, d=64)
    refused(B.COSA_ERR_UNSUPPORTED, call, n=2 ** 31)


def test_empty_problems_launch_nothing():
    none = B.DecodeProblem(0, 8, 2, 32)
    B.cosa_page_map(0, 16, 8, None, None, None, 0, None, None, None, None, None, 0, None, stream=0)
    B.cosa_kv_append(2, 128, 16, 4, None, None, None, 0, None, None, None, stream=0)
    CALLS["score"](none, q=None, bounds=None, lens=None, out=None)
    B.cosa_page_select(none, 64, None, None, BUDGET, None, None, stream=0)
    CALLS["decode"](none, q=None, lens=None, ws=None, n=0, o=None)
    CALLS["listed"](none, q=None, lens=None, ws=None, n=0, o=None, pages=None, count=None)
    CALLS["sparse"](none, q=None, bounds=None, lens=None, ws=None, n=0, o=None)
    assert B.cosa_last_error() == ""


def test_sparse_layout():
    p = B.DecodeProblem(3, 28, 4, 77)
    lay = B.cosa_decode_sparse_workspace_layout(p, B.page_budget(9))
    al = lambda x: (x + 255) // 256 * 256
    assert lay.score == 0
    assert lay.pages == al(4 * 3 * 28 * 77)
    assert lay.count == al(lay.pages + 4 * 3 * 4 * 9)
    assert lay.partial == al(lay.count + 4 * 3 * 4)
    assert lay.total == al(lay.partial + B.cosa_decode_workspace_bytes(p))
    assert B.cosa_decode_sparse_workspace_bytes(p, B.page_budget(9)) == lay.total
    refused(B.COSA_ERR_INVALID_ARG, B.cosa_decode_workspace_bytes, B.DecodeProblem(1, 3, 2, 4))
    with pytest.raises(B.CosaError):
        B.cosa_decode_sparse_workspace_bytes(p, B.page_budget(0))


def test_structs_match_the_header():
    """The C structs' sizes as the header's fields give them (64-bit ABI)."""
    assert ctypes.sizeof(B.CosaDecodeProblem) == 40
    assert ctypes.sizeof(B.CosaPageBudget) == 20
    assert ctypes.sizeof(B.CosaDecodeSparseLayout) == 40


def test_binding_refuses_cpu_tensors_and_overlapping_rows():
    import torch
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.cosa_page_score(GOOD, q, kv(), 16, 16, 16, stream=0)

    class Cuda:  # a tensor that says it lives on a GPU
        def __init__(self, t, device=0):
            self.t, self.device_index = t, device

        def get_device(self):
            return self.device_index

        def __getattr__(self, name):
            return getattr(self.t, name)
    wide = torch.zeros(4, 24, 128, dtype=torch.bfloat16)
    assert B._rows(Cuda(wide[:, 4:12]), 0)[1] == 24 * 128
    assert B._rows(Cuda(wide[:1, 4:12]), 0)[1] == 8 * 128
    assert B._rows(Cuda(wide), 24 * 128)[1] == 24 * 128
    assert B._rows(40, 16) == (40, 16)
    for bad in (wide[:, :8, ::2], wide[:, ::2], q[:1].expand(4, 8, 128), wide[0]):
        with pytest.raises(ValueError):
            B._rows(Cuda(bad), 0)
    with pytest.raises(ValueError):
        B._rows(Cuda(wide), 8)
    # one device for all tensors, and its stream
    one, other = Cuda(wide), Cuda(wide, 1)
    assert B._place(0, one, None, 7, one)[1] == [wide.data_ptr(), None, 7, wide.data_ptr()]
    with pytest.raises(ValueError):
        B._place(0, one, other)
    with pytest.raises(ValueError):
        B._place(0, one, Cuda(wide[:, ::2]))
    with pytest.raises(ValueError):
        B._rows(one, 0, other)
