"""Forks and compactions of tables that hold numbers outside the pool, or lengths outside the table: such an entry counts as no page, whoever goes on with
it, and is never looked up; the status says so."""
import pytest
import torch

from tests.test_gpu_page_moves import state
from tests.test_gpu_paged import F, ctx, i32  # noqa: F401

pytestmark = pytest.mark.gpu
GUARD = 5


def numbers(n_pages):
    return [n_pages, n_pages + 3, -7, (1 << 31) - 1, -(1 << 31)]


@pytest.mark.parametrize("n_pages", [16, 16384, 16385, 40000])       # up to 16384 pages in one launch, else in two
@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("parent", [None, [0, 1, 2, 3], [0, 1, 1, -1], [1, 1, 2, 3]])
@pytest.mark.parametrize("place", [0, 1])
def test_fork_with_an_entry_outside_the_pool(F, ctx, n_pages, which, parent, place):
    """Sequence 1 has 70 tokens, the last page partly filled; `place` 1 is that page."""
    pt, shares, o, _ = state(F, [(0, [10, 70, 64, 5])], 4, n_pages, 5)
    pt.table[1, place] = numbers(n_pages)[which]
    store = torch.full((n_pages + 2 * 4096,), GUARD, dtype=torch.int32, device="cuda")   # (words that say "shared" behind the holders, and before)
    shares = store[4096:4096 + n_pages].zero_()
    good = int(pt.table[1, 1 - place])
    first = [int(pt.table[b, 0]) for b in range(4)]
    free = pt.free_pages.tolist()[:int(pt.n_free)]
    copies, n = torch.full((4, 3), -9, dtype=torch.int32, device="cuda"), i32([-9])
    F.flux_page_fork(ctx, pt, shares, None if parent is None else i32(parent), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_PAGE
    who = parent or [0, 1, 2, 3]
    row = [-1 if place == 0 else good, -1 if place == 1 else good]
    lens = [10, 70, 64, 5]
    assert pt.kv_len.tolist() == [lens[p] if p >= 0 else 0 for p in who]
    holders = sum(p == 1 for p in who)
    table, listed = pt.table.tolist(), int(n)
    # the page that the sequences share if `place` is the other one: partly filled where it is the last, so the second of them gets a copy
    copied = holders > 1 and place == 0
    assert listed == (1 if copied else 0)
    seen = 0
    for b, p in enumerate(who):
        if p < 0:
            assert table[b] == [-1] * 4
        elif p != 1:
            assert table[b] == [first[p], -1, -1, -1]
        elif copied and seen:
            assert table[b] == [row[0], copies[0, 1].item(), -1, -1] and copies[0].tolist() == [good, table[b][1], 6]
        else:
            assert table[b] == row + [-1, -1]
        seen += p == 1
    assert copies[listed:].eq(-9).all()
    want = [0] * n_pages
    if not copied:
        want[good] = holders - 1
    assert shares.tolist() == want
    assert bool((store[:4096] == GUARD).all()) and bool((store[4096 + n_pages:] == GUARD).all())
    gone = sorted((first[b] for b in range(4) if b not in who and b != 1), reverse=True)
    free = free + gone
    assert pt.free_pages.tolist()[:int(pt.n_free)] == (free[:-1] if copied else free)


@pytest.mark.parametrize("n_pages", [16, 20000])
@pytest.mark.parametrize("length", [257, 1 << 30, -1])
@pytest.mark.parametrize("parent", [[0, 0, 2, 3], [0, -1, 2, 3], [0, 1, 2, 3], [1, 0, 2, 3]])
def test_fork_with_a_length_outside_the_table(F, ctx, n_pages, length, parent):
    """Sequence 1 has it: reported whether or not anybody goes on with what it holds."""
    pt, shares, o, _ = state(F, [(0, [10, 256, 64, 5])], 4, n_pages, 5)
    had = [int(pt.table[b, 0]) for b in range(4)]
    pt.kv_len[1] = length
    cut = min(max(length, 0), 256)
    copies, n = torch.full((4, 3), -9, dtype=torch.int32, device="cuda"), i32([-9])
    F.flux_page_fork(ctx, pt, shares, i32(parent), None, copies, n)
    assert F.flux_last_device_status(ctx) == F.FLUX_DEV_BAD_LENGTH
    lens = [10, cut, 64, 5]
    assert pt.kv_len.tolist() == [lens[p] if p >= 0 else 0 for p in parent]
    assert [int(pt.table[b, 0]) for b in (2, 3)] == had[2:]


@pytest.mark.parametrize("n_pages", [5, 300, 70000])
@pytest.mark.parametrize("which", range(5))
def test_compact_with_an_entry_outside_the_pool_where_nothing_moves(F, ctx, n_pages, which):
    pt, _, _, _ = state(F, [(0, [10, 200])], 5, n_pages, 3)
    pt.table[:, :] = i32([[0, -1, -1, -1, -1], [1, 2, 3, 4, -1]])
    pt.free_pages[:n_pages - 5] = torch.arange(5, n_pages, dtype=torch.int32, device="cuda")
    pt.n_free[0] = n_pages - 5
    moves, n = torch.full((16, 3), -9, dtype=torch.int32, device="cuda"), i32([-9])
    for bad in (False, True):
        if bad:
            pt.table[1, 2] = numbers(n_pages)[which]
        before = pt.table.clone()
        F.flux_page_compact(ctx, pt, None, moves, n)
        assert F.flux_last_device_status(ctx) == (F.FLUX_DEV_BAD_PAGE if bad else 0)
        assert n.tolist() == [0] and bool((moves == -9).all()) and torch.equal(pt.table, before)
        assert pt.free_pages.tolist()[:n_pages - 5] == list(range(n_pages - 1, 4, -1)) and int(pt.n_free) == n_pages - 5
