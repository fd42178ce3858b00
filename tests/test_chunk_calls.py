"""What attention of chunks of new tokens refuses on the host where its outputs lie in its inputs: no GPU needed."""
import pytest

from paper_2607_25291_amd import binding as B
from tests.test_decode_calls import refused

FAR = 1 << 44  # arrays that lie apart
P = B.ChunkProblem(4, 8, 2, 32, 100)
PAGE, PAGES = 64, 16
CACHE = PAGES * 2 * PAGE * 128 * 2  # bytes of K and of V
SIZES = {"q": 100 * 8 * 256, "k": CACHE, "v": CACHE, "table": 4 * 32 * 4, "lens": 4 * 4, "cu": 5 * 4}
OUT = {"o": 100 * 8 * 256, "lse": 100 * 8 * 4, "ws": B.cosa_chunk_workspace_bytes(P)}
AT = {name: (i + 1) * FAR for i, name in enumerate([*SIZES, *OUT])}


def call(p=P, n_pages=PAGES, page=PAGE, **at):
    a = {**AT, **at}
    B.cosa_chunk_attention(p, a["q"], B.CosaPagedKv(a["k"], a["v"], a["table"], page, n_pages), a["lens"], a["cu"], a["ws"],
                           OUT["ws"], a["o"], a["lse"], stream=0)


@pytest.mark.parametrize("name", OUT)
@pytest.mark.parametrize("other", [*SIZES, *OUT])
def test_outputs_within_inputs_or_each_other(name, other):
    if name == other:
        return
    size = {**SIZES, **OUT}[other]
    refused(B.COSA_ERR_INVALID_ARG, call, **{name: AT[other]})
    refused(B.COSA_ERR_INVALID_ARG, call, **{name: AT[other] + (size - 1) // 16 * 16})      # its first bytes in the last ones
    refused(B.COSA_ERR_INVALID_ARG, call, **{name: AT[other] - (OUT[name] - 1) // 16 * 16})  # its last bytes in the first ones


def test_caches_too_large_for_64_bits_of_bytes():
    """2^31 pages of 2^20 tokens of 16 heads: 2^63 bytes."""
    big = B.ChunkProblem(4, 16, 16, 32, 100)
    refused(B.COSA_ERR_INVALID_ARG, call, big, 2 ** 31, 1 << 20, o=AT["k"] + (1 << 40))


def test_queries_of_a_wide_projection_end_with_their_last_row():
    """q_stride 12 heads: the last row ends after 8 of them; what lies behind it is not q."""
    p = B.ChunkProblem(4, 8, 2, 32, 100, q_stride=12 * 128)
    end = AT["q"] + 2 * (99 * 12 + 8) * 128
    refused(B.COSA_ERR_INVALID_ARG, call, p, o=end - 16)
    refused(B.COSA_ERR_INVALID_ARG, call, p, lse=end - 16)
