"""Host-side checks of the serving entry points that need no GPU: declared and exported symbols, refusals before
anything is enqueued, workspaces, and what the binding refuses."""
import dataclasses
import subprocess

import pytest

from paper_2607_25291_amd import binding as B
from tests.test_decode_calls import Cuda, refused, two_gpus  # noqa: F401

EXPECTED = {"cosa_chunk_workspace_bytes", "cosa_chunk_attention", "cosa_page_fork", "cosa_page_copy",
            "cosa_page_workspace_bytes", "cosa_page_release", "cosa_page_compact"}

GOOD = B.ChunkProblem(4, 8, 2, 32, 100)
WS = 1 << 30
FAR = 1 << 40  # pointers: q, o, lse and the workspace lie apart


def kv(page=64, n_pages=16, k=16, v=16, table=16):
    return B.CosaPagedKv(k, v, table, page, n_pages)


def change(**kw):
    return dataclasses.replace(GOOD, **kw)


def chunk(p=GOOD, c=None, q=16, lens=16, cu=16, ws=FAR, n=WS, o=2 * FAR, lse=3 * FAR):
    B.cosa_chunk_attention(p, q, c or kv(), lens, cu, ws, n, o, lse, stream=0)


def test_symbols():
    assert set(B.declared_symbols(B.SERVING_HEADER_PATH)) == EXPECTED
    out = subprocess.run(["nm", "-D", "--defined-only", B.LIB_PATH], capture_output=True, text=True,
                         check=True).stdout
    assert EXPECTED <= {line.split()[-1] for line in out.splitlines() if " T " in line}
    for name in EXPECTED:
        assert hasattr(B.lib(), name) and callable(getattr(B, name))


@pytest.mark.parametrize("problem,status", [
    (change(batch=-1), B.COSA_ERR_INVALID_ARG),
    (change(max_pages=-1), B.COSA_ERR_INVALID_ARG),
    (change(n_rows=-1), B.COSA_ERR_INVALID_ARG),
    (change(n_q_heads=9), B.COSA_ERR_INVALID_ARG),
    (change(n_q_heads=0), B.COSA_ERR_INVALID_ARG),
    (change(n_kv_heads=0), B.COSA_ERR_INVALID_ARG),
    (change(head_dim=0), B.COSA_ERR_INVALID_ARG),
    (change(head_dim=64), B.COSA_ERR_UNSUPPORTED),
    (change(q_stride=8 * 128 - 8), B.COSA_ERR_INVALID_ARG),
    (change(q_stride=8 * 128 + 4), B.COSA_ERR_INVALID_ARG),
    (change(q_stride=-8), B.COSA_ERR_INVALID_ARG),
    (change(sm_scale=-1.0), B.COSA_ERR_INVALID_ARG),
    (change(sm_scale=float("nan")), B.COSA_ERR_INVALID_ARG),
    (change(max_pages=1 << 25), B.COSA_ERR_UNSUPPORTED),      # 2^31 tokens at 64 a page
    (change(batch=1 << 22), B.COSA_ERR_UNSUPPORTED),
    (change(n_rows=1 << 22), B.COSA_ERR_UNSUPPORTED),
    (change(n_q_heads=2 ** 12, n_rows=2 ** 19), B.COSA_ERR_UNSUPPORTED),
    (change(batch=2 ** 22 - 1, n_rows=2 ** 22 - 1, max_pages=2 ** 24), B.COSA_ERR_UNSUPPORTED),  # offsets could ask for 2^62 slots
])
def test_chunk_problems(problem, status):
    refused(status, chunk, problem)


@pytest.mark.parametrize("kw,status", [
    (dict(c=kv(page=24)), B.COSA_ERR_INVALID_ARG),
    (dict(c=kv(page=8)), B.COSA_ERR_INVALID_ARG),
    (dict(c=kv(n_pages=0)), B.COSA_ERR_INVALID_ARG),
    (dict(c=kv(k=None)), B.COSA_ERR_INVALID_ARG),
    (dict(c=kv(v=8)), B.COSA_ERR_INVALID_ARG),
    (dict(c=kv(table=None)), B.COSA_ERR_INVALID_ARG),
    (dict(q=None), B.COSA_ERR_INVALID_ARG),
    (dict(q=24), B.COSA_ERR_INVALID_ARG),
    (dict(lens=None), B.COSA_ERR_INVALID_ARG),
    (dict(cu=None), B.COSA_ERR_INVALID_ARG),
    (dict(o=None), B.COSA_ERR_INVALID_ARG),
    (dict(o=2 * FAR + 8), B.COSA_ERR_INVALID_ARG),
    (dict(ws=None), B.COSA_ERR_WORKSPACE),
    (dict(n=B.cosa_chunk_workspace_bytes(GOOD) - 1), B.COSA_ERR_WORKSPACE),
    (dict(ws=FAR + 8), B.COSA_ERR_INVALID_ARG),
    (dict(o=16 + 2 * 8 * 128 * 99), B.COSA_ERR_INVALID_ARG),    # o in q's last row
    (dict(lse=16), B.COSA_ERR_INVALID_ARG),
    (dict(lse=2 * FAR + 64), B.COSA_ERR_INVALID_ARG),
    (dict(ws=2 * FAR - 4096), B.COSA_ERR_INVALID_ARG),
])
def test_chunk_refusals(kw, status):
    refused(status, chunk, **kw)


def test_calls_without_rows_do_nothing():
    chunk(change(n_rows=0), q=None, lens=None, cu=None, ws=None, n=0, o=None, lse=None)
    chunk(change(batch=0), q=None, lens=None, cu=None, ws=None, n=0, o=None, lse=None)
    refused(B.COSA_ERR_INVALID_ARG, chunk, change(n_rows=0, n_kv_heads=3))  # arguments are checked all the same


def test_chunk_workspace():
    few = B.cosa_chunk_workspace_bytes(change(n_rows=1))
    assert few < B.cosa_chunk_workspace_bytes(GOOD) < 70 << 20
    with pytest.raises(B.CosaError):
        B.cosa_chunk_workspace_bytes(change(head_dim=64))
    # at most 256 rows of each of 2 * 256 partial results, and 256 records
    assert B.cosa_chunk_workspace_bytes(change(n_rows=1 << 20)) == 256 * 16 + 512 * 256 * 130 * 4


def test_query_rows():
    import torch
    t = Cuda(torch.zeros(100, 8, 128, dtype=torch.bfloat16))
    for bad in (torch.zeros(99, 8, 128, dtype=torch.bfloat16), torch.zeros(100, 4, 128, dtype=torch.bfloat16),
                torch.zeros(100, 8, 128), torch.zeros(100, 8, 64, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            chunk(q=Cuda(bad), lens=t, cu=t, ws=t, o=t, lse=None)
    with pytest.raises(ValueError):
        chunk(q=Cuda(torch.zeros(100, 8, 128, dtype=torch.bfloat16), device=1), lens=t, cu=t, ws=t, o=t, lse=None)


# Pointers of distinct arrays: the i-th argument's, far from the others.
def at(i):
    return (i + 1) * FAR


def fork(n0=4, n1=6, page=64, width=32, cap=100, **kw):
    names = ["parent", "table", "lens", "free", "n_free", "new_table", "new_lens", "src", "dst", "rows", "taken"]
    a = {n: at(i) for i, n in enumerate(names)} | kw
    B.cosa_page_fork(n0, n1, page, width, a["parent"], a["table"], a["lens"], 0, a["free"], cap, a["n_free"], a["new_table"],
                     a["new_lens"], a["src"], a["dst"], a["rows"], a["taken"], stream=0)


def copy(hkv=8, d=128, page=64, n_pages=100, most=10, **kw):
    a = {n: at(i) for i, n in enumerate(["k", "v", "bounds", "src", "dst", "rows", "n"])} | kw
    B.cosa_page_copy(hkv, d, page, n_pages, a["k"], a["v"], a["bounds"], a["src"], a["dst"], a["rows"], most, a["n"], stream=0)


def release(page=64, width=32, n_pages=100, n0=4, n1=5, cap=100, out_cap=100, bytes_=WS, **kw):
    names = ["ot", "ol", "nt", "nl", "free", "n_free", "taken", "out", "n_out", "ws"]
    a = {n: at(i) for i, n in enumerate(names)} | kw
    B.cosa_page_release(page, width, n_pages, n0, a["ot"], a["ol"], n1, a["nt"], a["nl"], a["free"], cap, a["n_free"],
                        a["taken"], a["out"], out_cap, a["n_out"], a["ws"], bytes_, stream=0)


def compact(n=4, page=64, width=32, n_pages=100, most=10, cap=100, bytes_=WS, **kw):
    names = ["table", "lens", "new", "src", "dst", "n_moves", "free", "n_free", "ws"]
    a = {x: at(i) for i, x in enumerate(names)} | kw
    B.cosa_page_compact(n, page, width, n_pages, a["table"], a["lens"], most, a["new"], a["src"], a["dst"], a["n_moves"],
                        a["free"], cap, a["n_free"], a["ws"], bytes_, stream=0)


BAD, UNSUPPORTED, SPACE = B.COSA_ERR_INVALID_ARG, B.COSA_ERR_UNSUPPORTED, B.COSA_ERR_WORKSPACE


@pytest.mark.parametrize("call,kw,status", [
    (fork, dict(n0=-1), BAD), (fork, dict(n1=-1), BAD), (fork, dict(page=17), BAD), (fork, dict(width=-1), BAD),
    (fork, dict(cap=-1), BAD), (fork, dict(n0=8193), UNSUPPORTED), (fork, dict(n1=8193), UNSUPPORTED),
    (fork, dict(width=1 << 25), UNSUPPORTED), (fork, dict(parent=None), BAD), (fork, dict(table=None), BAD),
    (fork, dict(lens=None), BAD), (fork, dict(free=None), BAD), (fork, dict(n_free=None), BAD), (fork, dict(new_table=None), BAD),
    (fork, dict(new_lens=None), BAD), (fork, dict(src=None), BAD), (fork, dict(dst=None), BAD), (fork, dict(rows=None), BAD),
    (fork, dict(taken=None), BAD), (fork, dict(new_table=at(1)), BAD), (fork, dict(new_lens=at(2)), BAD),
    (fork, dict(new_table=at(1) + 4 * 4 * 32 - 4), BAD), (fork, dict(taken=at(4)), BAD), (fork, dict(src=at(8)), BAD),
    (fork, dict(dst=at(9) + 20), BAD), (fork, dict(n1=0, taken=None), BAD),
    (copy, dict(hkv=0), BAD), (copy, dict(d=64), UNSUPPORTED), (copy, dict(d=0), BAD), (copy, dict(page=8), BAD),
    (copy, dict(n_pages=0), BAD), (copy, dict(most=-1), BAD), (copy, dict(most=2 ** 28), UNSUPPORTED),
    (copy, dict(hkv=1 << 12, page=1 << 20, n_pages=1), UNSUPPORTED), (copy, dict(k=None), BAD), (copy, dict(v=None), BAD),
    (copy, dict(src=None), BAD), (copy, dict(dst=None), BAD), (copy, dict(n=None), BAD), (copy, dict(k=at(0) + 8), BAD),
    (copy, dict(bounds=at(2) + 2), BAD), (copy, dict(v=at(0) + 256), BAD), (copy, dict(src=at(0) + 256), BAD),
    (copy, dict(n=at(2)), BAD),
    (release, dict(page=0), BAD), (release, dict(width=-1), BAD), (release, dict(n_pages=0), BAD), (release, dict(n0=-1), BAD),
    (release, dict(n1=-1), BAD), (release, dict(cap=-1), BAD), (release, dict(out_cap=-1), BAD),
    (release, dict(n_pages=2 ** 28 + 1), UNSUPPORTED), (release, dict(cap=2 ** 28 + 1), UNSUPPORTED),
    (release, dict(n0=1 << 24), UNSUPPORTED), (release, dict(n1=1 << 20, width=1 << 11), UNSUPPORTED),
    (release, dict(width=1 << 25), UNSUPPORTED), (release, dict(ot=None), BAD), (release, dict(ol=None), BAD),
    (release, dict(nt=None), BAD), (release, dict(nl=None), BAD), (release, dict(free=None), BAD), (release, dict(n_free=None), BAD),
    (release, dict(out=None), BAD), (release, dict(n_out=None), BAD), (release, dict(ws=None), SPACE),
    (release, dict(bytes_=B.cosa_page_workspace_bytes(100) - 1), SPACE), (release, dict(ws=at(9) + 8), BAD),
    (release, dict(out=at(4)), BAD), (release, dict(out=at(4) + 396), BAD), (release, dict(n_out=at(6)), BAD),
    (release, dict(n_out=at(7)), BAD), (release, dict(ws=at(7)), BAD), (release, dict(ws=at(0)), BAD),
    (compact, dict(n=-1), BAD), (compact, dict(page=48), BAD), (compact, dict(width=-1), BAD), (compact, dict(n_pages=0), BAD),
    (compact, dict(n_pages=2 ** 28 + 1), UNSUPPORTED), (compact, dict(most=-1), BAD), (compact, dict(cap=-1), BAD),
    (compact, dict(n=1 << 20, width=1 << 11), UNSUPPORTED), (compact, dict(table=None), BAD), (compact, dict(lens=None), BAD),
    (compact, dict(new=None), BAD), (compact, dict(src=None), BAD), (compact, dict(dst=None), BAD),
    (compact, dict(n_moves=None), BAD), (compact, dict(free=None), BAD), (compact, dict(n_free=None), BAD),
    (compact, dict(ws=None), SPACE), (compact, dict(bytes_=100), SPACE), (compact, dict(ws=at(8) + 4), BAD),
    (compact, dict(new=at(0) + 4), BAD), (compact, dict(src=at(1)), BAD), (compact, dict(dst=at(3) + 36), BAD),
    (compact, dict(free=at(0)), BAD), (compact, dict(n_free=at(5)), BAD), (compact, dict(ws=at(2)), BAD),
])
def test_page_refusals(call, kw, status):
    refused(status, call, **kw)


def test_page_workspace():
    for n in (0, -1, 2 ** 28 + 1):
        with pytest.raises(B.CosaError):
            B.cosa_page_workspace_bytes(n)
    assert B.cosa_page_workspace_bytes(1) < B.cosa_page_workspace_bytes(10 ** 6) < 2.1 * 10 ** 6
    assert B.cosa_page_workspace_bytes(2 ** 28) < 2.01 * 2 ** 28


def test_copying_nothing():
    copy(most=0, k=None, v=None, src=None, dst=None, n=None)


def all_calls(t, q, **kw):
    """Every entry point that enqueues work, with t for its tensors and q for rows [100, 8, 128] of them."""
    B.cosa_chunk_attention(GOOD, q, kv(), t, t, t, WS, t, t, **kw)
    B.cosa_page_fork(4, 4, 64, 32, t, t, t, 0, t, 4, t, t, t, t, t, t, t, **kw)
    B.cosa_page_copy(8, 128, 64, 16, t, t, t, t, t, t, 4, t, **kw)
    B.cosa_page_release(64, 32, 16, 4, t, t, 4, t, t, t, 4, t, t, t, 4, t, t, WS, **kw)
    B.cosa_page_compact(4, 64, 32, 16, t, t, 4, t, t, t, t, t, 4, t, t, WS, **kw)


@pytest.mark.parametrize("stream", [None, 0, "own"])
def test_streams_of_another_device(two_gpus, stream):  # noqa: F811
    import torch

    class Stream:
        cuda_stream = 1 << 20
        device = torch.device("cuda", 1)
    t = Cuda(torch.zeros(4, dtype=torch.int32), 1)
    q = Cuda(torch.zeros(100, 8, 128, dtype=torch.bfloat16), 1)
    all_calls(t, q, stream=Stream() if stream == "own" else stream)
    assert two_gpus["current"] == 0 and len(two_gpus["calls"]) == len(EXPECTED) - 2
    for name, current, handle in two_gpus["calls"]:
        assert handle == 1 << 20 if stream == "own" else (current, handle) == (1, 0), name
