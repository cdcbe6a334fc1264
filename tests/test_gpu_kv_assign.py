"""dmr_kv_assign against the definition, whole numbers: equal."""
import numpy as np
import pytest
import torch

import paper_2602_02711_amd as dmr

import attn_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def state(seed, requests, max_new, max_old, page, spare, extra_cols=2):
    """Lengths of a step, a table whose rows hold the old tokens' pages, and a stack with `spare` pages more than needed."""
    rng = np.random.default_rng(seed)
    new = rng.integers(0, max_new + 1, requests)
    old = rng.integers(0, max_old + 1, requests)
    width = max(1, -(-(max_old + max_new) // page) + extra_cols)
    held = -(-old // page)
    need = -(-(old + new) // page) - held
    order = rng.permutation(int(held.sum() + need.sum()) + 40).astype(np.int32)
    table = np.full((requests, width), -7, np.int32)
    at = 0
    for b in range(requests):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    return new, old, order[at:], max(0, int(need.sum()) + spare), table


def check(new, lens, stack, free, table, page, rows, in_place=False):
    want = ref.assign([int(v) for v in new], [int(v) for v in lens], stack, free, table, page, rows)
    d_table, d_lens, d_count = dev(table), dev(lens), dev([free, -1])
    out = None
    if in_place:
        out = (dev([-9] * (len(new) + 1)), d_lens, dev([-9] * rows), dev([-9] * rows), d_count)
    got = dmr.dmr_kv_assign(dev(new), d_lens, dev(stack), d_count if in_place else d_count[:1], d_table, page, rows, out=out)
    for name, g, w in zip(("query_start", "kv_lens", "positions", "slots", "left"), got, want):
        assert g.cpu().tolist() == list(w), name
    assert np.array_equal(d_table.cpu().numpy(), want[5])
    return want


@pytest.mark.parametrize("requests,max_new,max_old,page", [
    (1, 1, 0, 16), (1, 0, 0, 16), (1, 1, 40, 16), (3, 5, 100, 16), (64, 1, 9000, 16), (64, 1, 500, 256), (65, 3, 63, 64),
    (200, 160, 700, 64), (7, 2000, 5000, 32), (1023, 2, 50, 16), (1024, 1, 200, 16), (1025, 3, 100, 32), (2500, 4, 64, 16),
    (2, 20000, 300, 128)])
@pytest.mark.parametrize("in_place", [False, True])
def test_lengths_to_slots(requests, max_new, max_old, page, in_place):
    new, old, stack, free, table = state(requests * 7 + page, requests, max_new, max_old, page, 3)
    rows = int(new.sum())
    check(new, old, stack, free, table, page, rows, in_place)
    check(new, old, stack, free, table, page, rows + 5, in_place)             # a padded step
    check(new, old, stack, min(free - 3, len(stack)), table, page, rows, in_place)      # the stack to its last page


@pytest.mark.parametrize("requests,max_new,max_old,page", [(6, 40, 60, 16), (300, 9, 90, 16), (1500, 20, 40, 16), (40, 300, 50, 32)])
def test_refusals(requests, max_new, max_old, page):
    new, old, stack, free, table = state(requests + page, requests, max_new, max_old, page, 0)
    rows = int(new.sum())
    some = check(new, old, stack, free // 2, table, page, rows)               # too few pages
    assert 0 < some[4][1] < requests
    assert check(new, old, stack, 0, table, page, rows)[4][1] > 0
    assert check(new, old, stack, -3, table, page, rows)[4][1] > 0            # read as an empty stack
    check(new, old, stack, len(stack) + 50, table, page, rows)                # and one past its array as a full one
    assert check(new, old, stack, free, table, page, rows // 2)[4][1] > 0     # too few rows
    narrow = table[:, :max(1, table.shape[1] // 2)]
    check(new, old, stack, free, narrow, page, rows)                          # a narrow table
    assert check(new, old, stack, free, table[:, :1], page, rows)[4][1] > 0   # and one too narrow
    # refused lengths are read again, negative counts are none, a huge count is refused and so are all behind it
    lens = np.array(some[1])
    assert (lens < 0).any()
    check(new, lens, stack, free, table, page, rows)
    odd = new.copy()
    odd[::2] = -odd[::2]
    check(odd, lens, stack, free, table, page, rows)
    odd[requests // 2] = 2 ** 31 - 1
    assert check(odd, lens, stack, free, table, page, rows)[4][1] >= requests - requests // 2
    lens[0] = -2 ** 31
    check(new, lens, stack, free, table, page, rows)


def test_no_requests_no_rows():
    for rows in (0, 5, 5000):
        got = dmr.dmr_kv_assign(dev([]), dev([]), dev([3]), dev([1]), dev(np.zeros((0, 4))), 16, rows)
        assert got[0].tolist() == [0] and got[3].tolist() == [-1] * rows and got[4].tolist() == [1, 0]
    check([0, 0], [0, 5], [3], 1, np.array([[-1], [2]], np.int32), 16, 0)


def test_graph_of_steps_updates_its_own_state():
    requests, page, width = 70, 16, 6
    rng = np.random.default_rng(5)
    stack = rng.permutation(requests * width).astype(np.int32)
    table, lens, free = np.full((requests, width), -1, np.int32), [0] * requests, len(stack)
    d_new, d_lens, d_stack, d_count, d_table = dev([1] * requests), dev(lens), dev(stack), dev([free, 0]), dev(table)
    out = (dev([0] * (requests + 1)), d_lens, dev([0] * requests), dev([0] * requests), d_count)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        dmr.dmr_kv_assign(d_new, d_lens, d_stack, d_count, d_table, page, requests, out=out)
    for step in range(width * page + 3):                  # the last steps pass the table
        new = rng.integers(0, 2, requests)
        d_new.copy_(dev(new))
        graph.replay()
        want = ref.assign(new.tolist(), lens, stack, free, table, page, requests)
        lens, free, table = want[1], want[4][0], want[5]
        for g, w in zip(out, want):
            assert g.cpu().tolist() == list(w), step
        assert np.array_equal(d_table.cpu().numpy(), table)
