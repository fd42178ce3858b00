"""Host-side checks of the serving entry points that need no GPU: declared and exported symbols, refusals before
anything is enqueued, workspaces, and what the binding refuses."""
import dataclasses
import subprocess

import pytest

from paper_2607_25291_amd import binding as B
from tests.test_decode_calls import Cuda, refused, two_gpus  # noqa: F401

EXPECTED = {"cosa_chunk_workspace_bytes", "cosa_chunk_attention"}

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


def all_calls(t, q, **kw):
    """Every entry point that enqueues work, with t for its tensors and q for rows [100, 8, 128] of them."""
    B.cosa_chunk_attention(GOOD, q, kv(), t, t, t, WS, t, t, **kw)


@pytest.mark.parametrize("stream", [None, 0, "own"])
def test_streams_of_another_device(two_gpus, stream):  # noqa: F811
    import torch

    class Stream:
        cuda_stream = 1 << 20
        device = torch.device("cuda", 1)
    t = Cuda(torch.zeros(4, dtype=torch.int32), 1)
    q = Cuda(torch.zeros(100, 8, 128, dtype=torch.bfloat16), 1)
    all_calls(t, q, stream=Stream() if stream == "own" else stream)
    assert two_gpus["current"] == 0 and len(two_gpus["calls"]) == len(EXPECTED) - 1
    for name, current, handle in two_gpus["calls"]:
        assert handle == 1 << 20 if stream == "own" else (current, handle) == (1, 0), name
