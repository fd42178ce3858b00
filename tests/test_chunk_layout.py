"""Where attention of chunks of new tokens keeps its partial results, as far as its workspace shows it, and its words in LDS: no
GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2607_25291_amd import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_25291_amd", "csrc")


@pytest.mark.parametrize("group", [*range(1, 42), 51, 85, 127, 128, 129, 255, 256, 257, 300])
def test_partial_results_lie_at_multiples_of_16_bytes(group):
    """256 records of 16 bytes, then 2 * 256 partial results of equal size, which vector loads and stores of 16 bytes read and
    write: that size has to be a multiple of 16 whatever the rows of a unit are."""
    for n_rows in [*range(1, 20), 85, 100, 255, 256, 257, 5000]:
        n = B.cosa_chunk_workspace_bytes(B.ChunkProblem(2, group, 1, 32, n_rows)) - 256 * 16
        assert n > 0 and n % 512 == 0 and n // 512 % 16 == 0, (group, n_rows, n)


def test_lds_words_that_are_read_16_bytes_at_a_time(tmp_path):
    """The kernel's LDS structure, compiled for the host: the words that it reads and writes as vectors."""
    with open(os.path.join(CSRC, "chunk_attention.hip")) as f:
        body = re.search(r"struct Lds \{.*?\n\};\n", f.read(), re.S).group(0)
    (tmp_path / "lds.cpp").write_text(
        "#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include \"chunk_split.h\"\nusing cosa::kChunkRows;\n"
        "constexpr int kTileBytes = cosa::kChunkTile * 128 * 2;\n" + body +
        'int main() { printf("%zu %zu %zu %zu\\n", offsetof(Lds, v), offsetof(Lds, k), offsetof(Lds, unit), offsetof(Lds, odd)); }\n')
    exe = str(tmp_path / "lds")
    subprocess.run(["g++", "-std=c++17", f"-I{CSRC}", "-o", exe, str(tmp_path / "lds.cpp")], check=True)
    at = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert len(at) == 4 and all(x % 16 == 0 for x in at), at
