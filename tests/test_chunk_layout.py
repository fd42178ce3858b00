"""Where attention of chunks of new tokens keeps its partial results, as far as its workspace shows it: no GPU needed."""
import pytest

from paper_2607_25291_amd import binding as B


@pytest.mark.parametrize("group", [*range(1, 42), 51, 85, 127, 128, 129, 255, 256, 257, 300])
def test_partial_results_lie_at_multiples_of_16_bytes(group):
    """256 records of 16 bytes, then 2 * 256 partial results of equal size, which vector loads and stores of 16 bytes read and
    write: that size has to be a multiple of 16 whatever the rows of a unit are."""
    for n_rows in [*range(1, 20), 85, 100, 255, 256, 257, 5000]:
        n = B.cosa_chunk_workspace_bytes(B.ChunkProblem(2, group, 1, 32, n_rows)) - 256 * 16
        assert n > 0 and n % 512 == 0 and n // 512 % 16 == 0, (group, n_rows, n)
