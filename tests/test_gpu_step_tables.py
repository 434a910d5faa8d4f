"""GPU tests of a step's tables (page tables, row offsets, positions, slots, the pool)
against the oracle.  Whole numbers: everything is equal."""

import random

import numpy as np
import pytest
import torch

from oracle import paging as OP
from paper_2609_04098_amd import paging as P
from tests.gpu_common import log

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _oracle(r):
    return OP.Pool(r.page_table.cpu().tolist(), r.kv_len.tolist(), r.free_pages.tolist(), r.free_count.item(), r.page_size)


def _check(r, step, want, cu, pos, slots, marks):
    assert step.batch.cu_rows.tolist() == list(cu)
    n = int(cu[-1])
    assert np.array_equal(step.positions.cpu().numpy()[:n], pos)
    assert np.array_equal(step.slots.cpu().numpy()[:n], slots)
    assert (step.positions[n:] == marks).all() and (step.slots[n:] == marks).all()      # rows behind: as they were
    assert r.kv_len.tolist() == want.kv_len and r.free_count.item() == want.count
    assert r.page_table.tolist() == want.table and r.free_pages.tolist() == want.stack


def _run(r, new, drop, kept, rows, out=None):
    want = _oracle(r)
    zeros = [0] * len(new)
    cu, pos, slots = want.step(new, drop or zeros, kept or zeros, rows)
    step = out if out is not None else P.Step(r, rows)
    step.positions.fill_(-5)
    step.slots.fill_(-5)
    P.step_tables(r, _i32(new), rows, None if drop is None else _i32(drop), None if kept is None else _i32(kept), out=step)
    _check(r, step, want, cu, pos, slots, -5)
    return step


@pytest.mark.parametrize("n,width,pages,page,most,rows", [
    (1, 1, 1, 16, 3, 1), (1, 40, 64, 16, 300, 300), (3, 4, 8, 32, 40, 64), (63, 9, 300, 16, 30, 700),
    (64, 5, 200, 128, 9, 64), (65, 7, 500, 64, 200, 4000), (1023, 3, 2000, 16, 5, 3000), (1025, 3, 2500, 16, 5, 8192),
    (2048, 2, 3000, 16, 3, 4096), (2049, 2, 3000, 16, 3, 4096), (40, 300, 6000, 16, 4000, 9000),
    (1500, 40, 20000, 32, 300, 60000), (3000, 20, 30000, 16, 100, 100000)])
def test_steps_of_a_loop(n, width, pages, page, most, rows):
    """Steps on one state, with drafts that are rejected, requests that end and
    prompts in their place, until the pool is empty and again."""
    log("tables %s" % ((n, width, pages, page, most, rows),))
    rng = random.Random(n + width)
    r = P.alloc_requests(n, width, pages, page, "cuda")
    for i in range(6):
        new = [rng.choice([0, 1, 1, rng.randint(0, 4), rng.randint(0, most)]) for _ in range(n)]
        drop = [rng.choice([0, 0, 1, rng.randint(0, 5), 1 << 30]) for _ in range(n)] if i % 3 else None
        kept = [rng.choice([0, page, 2 * page, 5]) for _ in range(n)] if i % 2 else None
        _run(r, new, drop, kept, rows)


def test_numbers_that_make_no_sense():
    """Lengths, counts and pages out of range are cut, and no access leaves its buffer."""
    r = P.alloc_requests(5, 3, 10, 16, "cuda")
    r.kv_len.copy_(_i32([-3, 1 << 30, 48, 20, 2 ** 31 - 1]))
    r.page_table.copy_(_i32([[1, 2, 3], [-1, 99, 4], [5, 6, 7], [1 << 30, -2 ** 31, 0], [8, 9, 9]]))
    r.free_count.fill_(7)
    _run(r, [1, -4, 1, 3, 2 ** 31 - 1], [-1, 40, 2 ** 31 - 1, 0, 17], [0, 0, -8, 0, 2 ** 31 - 1], 6)
    r.free_count.fill_(-2)
    _run(r, [1, 1, 1, 1, 1], None, None, 6)
    r.free_count.fill_(1000)
    _run(r, [16, 16, 16, 16, 16], [48] * 5, None, 100)


def test_more_than_the_pool_takes_back():
    r = P.alloc_requests(4, 6, 8, 16, "cuda")
    r.kv_len.copy_(_i32([96, 96, 90, 1]))
    r.page_table.copy_(torch.arange(24, device="cuda").view(4, 6) % 8)
    r.free_count.fill_(3)
    _run(r, [1, 0, 2, 1], [96, 96, 90, 0], None, 10)
    r.kv_len.copy_(_i32([96, 96, 90, 1]))
    _run(r, [1, 0, 2, 1], [96, 96, 90, 0], None, 10000)      # (the form of many rows)


def test_nothing_to_do():
    r = P.alloc_requests(0, 4, 3, 16, "cuda")
    step = P.step_tables(r, _i32([]), 4)
    assert step.batch.cu_rows.tolist() == [0] and r.free_count.item() == 3
    r = P.alloc_requests(2, 0, 3, 16, "cuda")                 # no table
    _run(r, [1, 0], None, None, 4)
    r = P.alloc_requests(2, 3, 3, 16, "cuda")
    _run(r, [1, 1], None, None, 0)
    _run(r, [0, 0], None, None, 0)


def test_strided_table_and_a_row_of_its_own():
    wide = torch.full((5, 11), -9, dtype=torch.int32, device="cuda")
    r = P.Requests(wide[:, 2:6], torch.zeros(5, dtype=torch.int32, device="cuda"),
                   torch.arange(20, dtype=torch.int32, device="cuda"), _i32([20]), 16)
    _run(r, [60, 1, 17, 0, 33], None, None, 200)
    assert (wide[:, :2] == -9).all() and (wide[:, 6:] == -9).all()
    one = P.Requests(torch.as_strided(wide, (1, 4), (1, 1)), torch.zeros(1, dtype=torch.int32, device="cuda"),
                     torch.arange(20, dtype=torch.int32, device="cuda"), _i32([20]), 16)
    _run(one, [64], None, None, 64)


def test_another_stream_and_a_step_without_positions():
    r = P.alloc_requests(3, 4, 12, 16, "cuda")
    want = _oracle(r)
    side = torch.cuda.Stream()
    new = _i32([20, 3, 40])
    side.wait_stream(torch.cuda.current_stream())
    step = P.step_tables(r, new, 80, stream=side)
    side.synchronize()
    cu, pos, slots = want.step([20, 3, 40], [0] * 3, [0] * 3, 80)
    assert step.batch.cu_rows.tolist() == list(cu) and step.slots[:63].tolist() == list(slots)
    cu_rows, ws = _i32([0] * 4), torch.empty(P._p.step_tables_workspace(3), dtype=torch.uint8, device="cuda")
    P._p.step_tables(None, r.ref, new.data_ptr(), None, None, cu_rows.data_ptr(), None, None, 80, ws.data_ptr(), ws.numel())
    cu, _, _ = want.step([20, 3, 40], [0] * 3, [0] * 3, 80)
    assert cu_rows.tolist() == list(cu) and r.page_table.tolist() == want.table


@pytest.mark.parametrize("rows", [60, 9000])
def test_captured_steps(rows):
    """A captured step, replayed with other lengths between eager ones."""
    r = P.alloc_requests(4, 700, 3000, 16, "cuda")
    new, drop = _i32([1] * 4), _i32([0] * 4)
    step = P.Step(r, rows)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.step_tables(r, new, rows, drop, out=step)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.step_tables(r, new, rows, drop, out=step)
    rng = random.Random(rows)
    for i in range(5):
        a = [rng.randint(0, rows // 5) for _ in range(4)]
        d = [rng.choice([0, 3, 10000]) for _ in range(4)]
        new.copy_(_i32(a))
        drop.copy_(_i32(d))
        want = _oracle(r)
        cu, pos, slots = want.step(a, d, [0] * 4, rows)
        step.positions.fill_(-5)
        step.slots.fill_(-5)
        graph.replay()
        _check(r, step, want, cu, pos, slots, -5)
        if i % 2:
            _run(r, [1, 2, 0, 1], [0, 1, 0, 0], None, rows)
