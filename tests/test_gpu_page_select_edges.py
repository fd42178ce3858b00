"""Page selection at the ends of its range: the widest list."""
import numpy as np
import pytest

from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from tests.gpu_util import dev, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [2, 5])
@pytest.mark.parametrize("width", [40, 1100])  # 256 and 1024 threads a row
def test_the_widest_list(width, heads):
    """A list of 2^31 - 1 pages: all but the sequence's own pages are -1, and nothing behind the list changes."""
    t = torch()
    most = 2 ** 31 - 1
    print(f"[page select] a list of {most} pages, {width} pages, {heads} heads", flush=True)
    rng = np.random.default_rng(width)
    score = rng.standard_normal((1, heads, width)).astype(np.float32)
    lens = [16 * width - 3]
    pages = t.full((most + 9,), 5, dtype=t.int32, device="cuda")
    count = t.full((1,), -7, dtype=t.int32, device="cuda")
    budget = B.page_budget(most, fraction=0.5)
    B.cosa_page_select(B.DecodeProblem(1, heads, 1, width), 16, dev(np.array(lens, np.int32)), dev(score), budget, pages,
                       count)
    t.cuda.synchronize()
    k = width // 2
    want, _ = D.page_select(score, lens, 16, 1, 0.5, 1, k, 1, 1)
    assert count.item() == k and np.array_equal(pages[:k].cpu().numpy(), want[0, 0])
    for a in range(k, most, 2 ** 28):
        assert (pages[a:min(a + 2 ** 28, most)] == -1).all()
    assert (pages[most:] == 5).all()
