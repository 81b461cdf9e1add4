"""The 4-bit cache's plan where a step asks for more than there is room for, and where its lengths do not belong together."""
import pytest

import kv4_reference as ref
from test_gpu_kv4 import cache_of, check_plan, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_more", [0, 300, 1500])
def test_requests_without_rows_are_served_behind_an_overflow(n_more):
    """The second request's prompt does not fit.  Behind it one ends, one waits, one is taken back without rows, one reserves a block and one has a
    row: all but the last are served, and the blocks that were held come back."""
    n = 7 + n_more
    c = cache_of(2, 2, 32, "bf16", 16, 40 + n_more, n, 200, 2000)
    blocks = ref.Blocks(40 + n_more, n, 200, 16)
    held = [5, 0, 50, 33, 64, 16, 7] + [1] * n_more
    check_plan(c, blocks, [0] * n, [0] * n, held, sum(held))
    free = c.n_free.item()
    assert free == 40 - (1 + 0 + 4 + 3 + 4 + 1 + 1)
    start = [5, 0, 0, 33, 20, 20, 7] + [0, 1] * (n_more // 2)   # half of the others end, half wait
    end = [6, 101, 0, 33, 20, 20, 8] + [0, 1] * (n_more // 2)
    held_next = check_plan(c, blocks, held, start, end, 101)
    assert c.served[:7].tolist() == [1, 0, 1, 1, 1, 1, 0] and c.served[7:n].all()
    assert held_next == [6, 0, 0, 33, 20, 20, 7] + [0, 1] * (n_more // 2)
    assert c.n_free.item() == free + 4 + 2 - 1 + n_more // 2
    assert c.row_start[:8].tolist() == [0, 1] + [101] * 6 and c.positions[0].item() == 5 and (c.positions[1:101] == -1).all()
    # what came back is given out again, and the prompt fits once the step has room for it
    again = [0, 101, 0, 33, 20, 20, 8] + held_next[7:]
    start = [0, 0, 0, 33, 20, 20, 7] + held_next[7:]
    held_next = check_plan(c, blocks, held_next, start, again, 102)
    assert c.served[:n].all() and held_next == again
    c.close()
