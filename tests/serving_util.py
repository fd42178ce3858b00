"""Inputs and tolerances shared by the GPU tests of the serving operators."""
from __future__ import annotations

import numpy as np

from paper_2607_25291_amd import binding as B
from tests.decode_util import as_f64
from tests.gpu_util import dev, torch


def check_chunk(o, lse, ref, longest):
    """o (bf16) and lse (fp32) against the oracle's (o, lse, weight, magnitude); rows of no sequence are NaN in both.

    A logit is a fp32 sum of 128 exact products: off by at most 128 * 2^-24 of the sum of magnitudes, 2^-17 mag; exp turns
    it into a relative error of a weight, counted for the numerator and for the sum (2^-16 mag). exp2 and its argument
    add less than 2^-15 (numerator and sum). A weight enters the product with V as one bf16: half a step, 2^-8. The
    fp32 sums run over longest / 16 steps of a product, and the partial results of 256 ranges: (longest / 16 + 600) 2^-24 of
    the weight in numerator and sum. The result is rounded to bf16 once: 2^-8 of the value."""
    ro, rl, wt, mag = ref
    rest = 2.0 ** -15 + 2.0 ** -16 * mag + (longest / 16 + 600) * 2.0 ** -23
    nobody = np.isnan(rl)
    assert (np.isnan(lse) == nobody).all() if lse is not None else True
    assert (np.isnan(o) == nobody[..., None]).all()
    err = np.abs(o - ro)[~nobody]
    tol = (2.0 ** -8 * np.abs(ro) + (2.0 ** -8 + rest)[..., None] * wt + 1e-30)[~nobody]
    assert (err <= tol).all(), f"o off by {err.max()}, worst ratio {(err / tol).max()}"
    if lse is not None:
        dead = np.isneginf(rl)
        assert (np.isneginf(lse) == dead).all()
        live = ~dead & ~nobody
        e = np.abs(lse[live] - rl[live])
        t = rest[live] / 2 + 2.0 ** -23 * (4 + np.abs(rl[live]))
        assert (e <= t).all(), f"lse off by {e.max()}, worst ratio {(e / t).max()}"


def run_chunk(p, cache, q, cu, lse=True, stream=None, kv=None, lens=None):
    """(o, lse) tensors of one call with its own workspace, NaN in everything that it does not write."""
    t = torch()
    kv = kv or cache.upload()
    n = B.cosa_chunk_workspace_bytes(p)
    ws = t.full((n,), 0xFF, dtype=t.uint8, device="cuda")
    o = t.full((p.n_rows, p.n_q_heads, 128), 0x7FC0, dtype=t.int16, device="cuda")
    ls = t.full((p.n_rows, p.n_q_heads), float("nan"), device="cuda") if lse else None
    B.cosa_chunk_attention(p, q, kv, cache.lens_d if lens is None else lens, cu, ws, n, o, ls, stream=stream)
    t.cuda.synchronize()
    return o, ls


def host(o, lse):
    return as_f64(o), None if lse is None else lse.cpu().numpy().astype(np.float64)


def offsets(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
