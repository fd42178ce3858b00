"""Inputs and tolerances shared by the GPU tests of the decode-side operators."""
from __future__ import annotations

import numpy as np

from paper_2607_25291_amd import binding as B
from paper_2607_25291_amd.inputs import f32_to_bf16_bits
from tests.gpu_util import dev, torch

NAN_BITS = np.uint16(0x7FC0)


def normal(rng, *shape, scale=1.0):
    return f32_to_bf16_bits(scale * rng.standard_normal(shape, dtype=np.float32))


class Cache:
    """A paged cache for sequences of the given lengths: random pages, and NaN in every place that no
    sequence's tokens occupy (unused pages and rows behind a sequence's end). Table entries behind the last page
    are far outside the cache."""

    def __init__(self, rng, lens, n_kv_heads, page, width=None, spare=3, sinks=True):
        self.lens = np.asarray(lens, np.int32)
        self.page, self.n_kv_heads = page, n_kv_heads
        pages = [-(-int(n) // page) for n in lens]
        self.width = max(pages + [0]) if width is None else width
        self.n_pages = sum(pages) + spare
        perm = rng.permutation(self.n_pages)
        shape = (self.n_pages, n_kv_heads, page, 128)
        self.k, self.v = np.full(shape, NAN_BITS), np.full(shape, NAN_BITS)
        self.table = np.full((len(pages), self.width), 2 ** 31 - 1, np.int32)
        at = 0
        for n, (length, p) in enumerate(zip(lens, pages)):
            self.table[n, :p] = perm[at:at + p]
            at += p
            for j in range(p):
                rows = min(page, int(length) - j * page)
                x = rng.standard_normal((n_kv_heads, rows, 128), dtype=np.float32)
                if j == 0 and sinks:
                    x[:, :4] *= 4.0
                self.k[self.table[n, j], :, :rows] = f32_to_bf16_bits(x)
                self.v[self.table[n, j], :, :rows] = normal(rng, n_kv_heads, rows, 128)

    def upload(self):
        self.k_d, self.v_d, self.table_d, self.lens_d = map(dev, (self.k, self.v, self.table, self.lens))
        return B.paged_kv(self.k_d, self.v_d, self.table_d, self.page, self.n_pages)


def as_f64(t):
    """bf16 bits on the GPU (int16) -> float64 on the host."""
    return (t.cpu().numpy().view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def check_attention(o, lse, ref, longest):
    """o (bf16) and lse (fp32) against the oracle's (o, lse, weight, magnitude).

    A logit is a fp32 sum of 128 exact products: off by at most 128 * 2^-24 of the sum of magnitudes, 2^-17 mag; exp
    turns it into a relative error of a weight, counted for the numerator and for the sum (2^-16 mag). A
    weight enters the product as two bf16 terms (2^-17; 2^-16 with exp2 and the sum's own), and the fp32 sums
    run over at most longest / 128 steps of a wave, 32 products each, and the partial results of 512
    workgroups: (longest / 128 + 32 + 516) 2^-24 of the weight in numerator and sum. The result is rounded to
    bf16 once: half a step, 2^-8 of the value."""
    ro, rl, wt, mag = ref
    steps = longest / 128 + 548
    rel = 2.0 ** -15 + 2.0 ** -16 * mag + steps * 2.0 ** -23
    err = np.abs(o - ro)
    tol = 2.0 ** -8 * np.abs(ro) + rel[..., None] * wt + 1e-30
    assert np.isfinite(o).all()
    assert (err <= tol).all(), f"o off by {err.max()}, worst ratio {(err / tol).max()}"
    if lse is not None:
        dead = np.isneginf(rl)
        assert (np.isneginf(lse) == dead).all()
        live = ~dead
        e = np.abs(lse[live] - rl[live])
        t = (rel / 2 + 2.0 ** -23 * (4 + np.abs(np.where(dead, 0, rl))))[live]
        assert (e <= t).all(), f"lse off by {e.max()}, worst ratio {(e / t).max()}"


def run_decode(p, cache, q, lists=None, lse=True, stream=None, kv=None):
    """(o, lse) tensors of one call with its own workspace; lists: (pages, count) numpy."""
    t = torch()
    kv = kv or cache.upload()
    n = B.cosa_decode_workspace_bytes(p)
    ws = t.full((n,), 0xFF, dtype=t.uint8, device="cuda")  # NaN wherever it is read as scratch
    o = t.full((p.batch, p.n_q_heads, 128), 0x7FC0, dtype=t.int16, device="cuda")
    ls = t.full((p.batch, p.n_q_heads), float("nan"), device="cuda") if lse else None
    if lists is None:
        B.cosa_decode_attention(p, q, kv, cache.lens_d, ws, n, o, ls, stream=stream)
    else:
        pages, count = (x if hasattr(x, "data_ptr") else dev(np.asarray(x, np.int32)) for x in lists)
        B.cosa_decode_attention_listed(p, q, kv, cache.lens_d, pages, count, pages.shape[2], ws, n, o, ls,
                                       stream=stream)
    t.cuda.synchronize()
    return o, ls
