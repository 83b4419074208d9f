"""mcsd_build_page_tables against a sequential statement (whole numbers, equal)."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding

pytestmark = pytest.mark.gpu


def _state(rng, B, W, cap, free, ps, longest):
    start = rng.integers(0, longest + 1, B).astype(np.int32)
    held = np.minimum(-(-start // ps) + rng.integers(0, 3, B), W).astype(np.int32)
    held = np.where(held * ps < start, W, held).astype(np.int32)
    ids = rng.permutation(cap).astype(np.int32)
    while held.sum() + free > cap:
        held = np.minimum(held, held.max() - 1 if held.max() else 0).astype(np.int32)
        start = np.minimum(start, held * ps).astype(np.int32)
    table = np.full((B, W), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    head = int(rng.integers(0, cap))
    ring = np.full(cap, -7, dtype=np.int32)
    ring[(head + np.arange(free)) % cap] = ids[at:at + free]
    return start, held, table, ring, head


def _run(start, count, held, table, ring, head, free, ps, *, in_place, n_slots=None):
    c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    t, h, r, s = c(table), c(held), c(ring), torch.tensor([head, free, 0, 0], dtype=torch.int32, device="cuda")
    outs = {} if in_place else dict(held_out=torch.full_like(h, -9), ring_state_out=torch.full_like(s, -9))
    plan = binding.PageTables(t, h, r, s, ps, **outs)
    total = int(np.maximum(np.where(start < 0, 0, count), 0).sum())
    slots = torch.full(((total if n_slots is None else n_slots) + 5,), -5, dtype=torch.int64, device="cuda")
    plan.mcsd_build_page_tables(c(start), c(count.astype(np.int32)), slots=slots[:-5] if n_slots is None else slots[:n_slots])
    torch.cuda.synchronize()
    if not in_place:
        assert np.array_equal(h.cpu().numpy(), held) and s.tolist() == [head, free, 0, 0]
    else:
        assert s.tolist()[2:] == [0, 0]
    return plan, t, r, slots, total


def _check(plan, t, r, slots, total, want):
    table, held, ring, head, free, want_slots, cu, status = want
    assert np.array_equal(t.cpu().numpy(), table)
    assert np.array_equal(plan.held_out.cpu().numpy(), held)
    assert np.array_equal(r.cpu().numpy(), ring)
    assert plan.ring_state_out.tolist()[:2] == [head, free]
    assert np.array_equal(plan.cu_tokens.cpu().numpy(), cu)
    assert np.array_equal(plan.status.cpu().numpy(), status)
    n = min(slots.numel() - 5, total)
    assert np.array_equal(slots[:n].cpu().numpy(), want_slots[:n])
    assert (slots[n:] == -5).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,W,free,ps,longest,most", [(1, 4, 4, 16, 20, 20), (1, 1, 0, 16, 16, 1), (3, 10, 9, 16, 100, 60), (8, 40, 3, 16, 300, 45),
                                                      (8, 40, 0, 64, 300, 45), (33, 20, 200, 128, 2000, 500), (1025, 8, 900, 32, 200, 40),
                                                      (300, 64, 4000, 16, 500, 500), (4096, 3, 2000, 16, 30, 20)])
def test_against_sequential(in_place, B, W, free, ps, longest, most):
    rng = np.random.default_rng(B * 7 + free)
    for _ in range(3):
        start, held, table, ring, head = _state(rng, B, W, B * W + free + 3, free, ps, min(longest, W * ps))
        count = rng.integers(0, most + 1, B)
        if B > 2:
            start[1] = -1                            # an unused entry
            start[B // 2], count[B // 2] = 0, 0      # a request that ended: all its pages go back
            count[B - 1] = W * ps + 1                # wider than the table
        want = ref.page_tables(start, count, table, held, ring, head, free, ps)
        _check(*_run(start, count, held, table, ring, head, free, ps, in_place=in_place), want)


def test_refusal_is_in_order_and_leaves_the_sequence():
    ps, W = 16, 8
    start = np.array([0, 16, 0, 5, 0], dtype=np.int32)
    count = np.array([32, 16 * 5, 16, 3, 0])
    held = np.array([0, 1, 0, 1, 2], dtype=np.int32)
    table = np.full((5, W), -1, dtype=np.int32)
    table[1, 0], table[3, 0], table[4, :2] = 50, 51, [52, 53]
    ring = np.arange(100, 110).astype(np.int32)
    want = ref.page_tables(start, count, table, held, ring, 8, 4, ps)
    assert list(want[7]) == [0, 16, 16, 0, 0] and list(want[1]) == [2, 1, 0, 1, 0] and want[4] == 4
    _check(*_run(start, count, held, table, ring, 8, 4, ps, in_place=True), want)


def test_slots_beyond_the_buffer_are_not_written_and_uniform_counts():
    rng = np.random.default_rng(5)
    start, held, table, ring, head = _state(rng, 6, 30, 300, 60, 16, 200)
    count = np.full(6, 45)
    want = ref.page_tables(start, count, table, held, ring, head, 60, 16)
    _check(*_run(start, count, held, table, ring, head, 60, 16, in_place=False, n_slots=100), want)
    c = lambda a: torch.from_numpy(a).cuda()
    plan = binding.PageTables(c(table), c(held), c(ring), torch.tensor([head, 60, 0, 0], dtype=torch.int32, device="cuda"), 16)
    slots = torch.empty(6 * 45, dtype=torch.int64, device="cuda")
    plan.mcsd_build_page_tables(c(start), 45, slots=slots)
    assert np.array_equal(slots.cpu().numpy(), want[5]) and np.array_equal(plan.table.cpu().numpy(), want[0])


def test_a_strided_table():
    rng = np.random.default_rng(6)
    start, held, table, ring, head = _state(rng, 5, 12, 100, 30, 16, 100)
    count = rng.integers(0, 60, 5)
    want = ref.page_tables(start, count, table, held, ring, head, 30, 16)
    big = torch.full((5, 20), -3, dtype=torch.int32, device="cuda")
    big[:, :12] = torch.from_numpy(table).cuda()
    c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    plan = binding.PageTables(big[:, :12], c(held), c(ring), torch.tensor([head, 30, 0, 0], dtype=torch.int32, device="cuda"), 16)
    plan.mcsd_build_page_tables(c(start), c(count.astype(np.int32)))
    assert np.array_equal(big[:, :12].cpu().numpy(), want[0]) and (big[:, 12:] == -3).all()


def test_many_steps_captured_and_replayed_never_share_or_lose_a_page():
    """A captured call replayed with changing lengths: every page is held by one sequence or free, always."""
    B, W, n_pages, ps = 16, 20, 150, 16
    plan = binding.PageTables.empty(B, W, n_pages, ps)
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    count = torch.zeros(B, dtype=torch.int32, device="cuda")
    slots = torch.empty(4096, dtype=torch.int64, device="cuda")
    plan.mcsd_build_page_tables(start, count, slots=slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.mcsd_build_page_tables(start, count, slots=slots)
    rng = np.random.default_rng(1)
    for step in range(60):
        held = plan.held.cpu().numpy()
        table, ring, (head, free) = plan.table.cpu().numpy(), plan.ring.cpu().numpy(), plan.ring_state.tolist()[:2]
        s = np.minimum(rng.integers(0, W * ps, B), held * ps).astype(np.int32)
        n = rng.integers(0, 100, B).astype(np.int32)
        ended = rng.random(B) < 0.15
        s[ended], n[ended] = 0, 0
        start.copy_(torch.from_numpy(s)), count.copy_(torch.from_numpy(n))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.page_tables(s, n, table, held, ring, head, free, ps)
        assert np.array_equal(plan.table.cpu().numpy(), want[0]) and np.array_equal(plan.held.cpu().numpy(), want[1])
        assert plan.ring_state.tolist() == [want[3], want[4], 0, 0]
        owned = [int(p) for b in range(B) for p in want[0][b, :want[1][b]]]
        spare = [int(want[2][(want[3] + k) % n_pages]) for k in range(want[4])]
        assert sorted(owned + spare) == list(range(n_pages))
