"""The 4-bit cache's plan where a step asks for more than there is room for, and where its lengths do not belong together."""
import pytest
import torch

import kv4_reference as ref
from test_gpu_kv4 import Requests, cache_of, check_plan, dev, rand

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


@pytest.mark.parametrize("n_more", [0, 600])
def test_rows_that_begin_behind_what_is_held_are_refused(n_more):
    """Between what such a request held and its rows lie positions that nobody has written: in blocks of its own or in blocks that
    another request has given back."""
    n = 5 + n_more
    c = cache_of(2, 2, 32, "bf16", 16, 30 + n_more, n, 200, 2000)
    blocks = ref.Blocks(30 + n_more, n, 200, 16)
    held = [20, 0, 20, 33, 20] + [3] * n_more
    check_plan(c, blocks, [0] * n, [0] * n, held, sum(held))
    free = c.n_free.item()
    # one position on, from position 1 of an empty request, exactly at what is held, one past a block's end, blocks taken ahead
    start, end = [21, 1, 20, 50, 60] + [3] * n_more, [22, 2, 22, 51, 60] + [4] * n_more
    held_next = check_plan(c, blocks, held, start, end, 5 + n_more)
    assert c.served[:5].tolist() == [0, 0, 1, 0, 1] and c.served[5:n].all()
    assert held_next == [20, 0, 22, 33, 60] + [4] * n_more
    assert c.slots[0].item() == c.slots[1].item() == c.slots[4].item() == -1 and (c.slots[2:4] >= 0).all()
    assert c.n_free.item() == free - 2
    q = rand((5 + n_more, 2, 32), "bf16", 3)
    out, lse = c.attend(0, q, lse=True)
    assert not out[[0, 1, 4]].any() and torch.isneginf(lse[[0, 1, 4]]).all()
    c.close()


def captured(call):
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


def test_captured_calls_after_another_plan():
    """Graphs of an attention and of an append alone, replayed after plans of fewer and of more rows, of other tiles, and of their own
    shape: arrays that are too short for the plan are not touched, nor rows of a plan before, and later calls are not disturbed."""
    heads, kvh, hd, n = 160, 2, 128, 1500
    s = Requests([n, 400], [2, 1], heads, kvh, hd, "bf16", 64, seed=41)

    def step(rows):
        s.rows = rows
        s.q = rand((sum(rows), heads, hd), "bf16", 42 + sum(rows))
        s.step()
        return s.q, torch.full_like(s.q, 7.0)

    shapes = ([2, 1], [2, 2], [40, 3], [140, 10])  # 3 and 4 rows of tiles of 32 entries (80 heads a kv head), wide tiles
    graphs = []
    for rows in shapes:
        q, out = step(rows)
        graphs.append((captured(lambda: s.c.attend(0, q, out=out)), q, out))
    for planned in (3, 0, 1, 2, 3, 0):
        q, _ = step(shapes[planned])
        for i, (graph, gq, out) in enumerate(graphs):
            out.fill_(7.0)
            if i == planned:
                gq.copy_(q)
            graph.replay()
            torch.cuda.synchronize()
            if i == planned:
                s.check(out)
                assert torch.equal(out, s.c.attend(0, q))
            else:
                assert (out == 7.0).all(), (planned, i)
    # an append of five rows after a plan of two: slots 2 .. 4 are still those of the plan before
    kv = rand((5, kvh, hd), "bf16", 50)
    lengths = dev([n, 400])
    s.c.plan(lengths, dev([n - 5, 400]), lengths, 5)
    graph = captured(lambda: s.c.append(0, kv, kv))
    written = [t.clone() for t in s.c.read(0, s.c.slots[:5].clone())]
    slots = s.c.slots[:5].clone()
    s.c.plan(lengths, dev([n, 398]), lengths, 2)
    kv.mul_(2)
    graph.replay()
    k, v = s.c.read(0, slots)
    assert torch.equal(k, written[0]) and torch.equal(v, written[1])
    k, _ = s.c.read(0, s.c.slots[:2].clone())
    assert torch.equal(k.cpu().double(), ref.held(kv[:2]))
    s.c.close()
