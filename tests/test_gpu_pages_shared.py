"""Sequences that share a page, have unequal numbers of rows in it, and grow: who keeps it, and that nobody's rows are written over."""
import numpy as np
import pytest

import paper_2407_21018_amd as thk
from oracle import step as O
from test_gpu_step import Books


def state(B, n_free, page_rows, seed, pinned):
    """Groups of sequences, a full page and a partly filled one in common, of which each has as many rows as it likes."""
    rng = np.random.default_rng(seed)
    held, table, now, rows, refs, b = [], [], [], [], [], 0
    while b < B:
        users = min(int(rng.integers(1, 6)), B - b)
        pages = [len(refs), len(refs) + 1]
        refs += [users, users + int(rng.random() < 0.2)]      # (a user outside the batch)
        for _ in range(users):
            n = page_rows + int(rng.integers(1, page_rows))
            now.append(n)
            rows.append(n if rng.random() < 0.05 else n + int(rng.choice([1, 64, page_rows])))
            held.append(2)
            table.append(pages + [-1, -1])
        b += users
    n = len(refs) + n_free + pinned
    refs += [0] * n_free + [1] * pinned
    order = rng.permutation(n)      # pages of any number
    table = [[int(order[p]) if p >= 0 else -1 for p in t] for t in table]
    shuffled = [0] * n
    for p, r in enumerate(refs):
        shuffled[order[p]] = r
    return rows, now, held, table, shuffled


def nobody_is_written_over(rows, now, held, table, room, page_rows):
    """Who may write a page has in it at least the rows of everybody else who still uses it."""
    users = {}
    for b in range(len(rows)):
        e = now[b] // page_rows
        if now[b] % page_rows and e < held[b]:
            users.setdefault(table[b][e], []).append((now[b] % page_rows, min(rows[b], room[b]) > now[b]))
    for page, all_of_it in users.items():
        writers = [n for n, writes in all_of_it if writes]
        assert len(writers) <= 1, page
        assert not writers or writers[0] >= max(n for n, _ in all_of_it), page


@pytest.mark.parametrize("n_free", [0, 1, 7, 40])
def test_the_rule_keeps_rows(n_free):
    for seed in range(30):
        rows, now, held, table, refs = state(40, n_free, 256, seed, 3)
        got = O.reserve(rows, now, held, table, refs, 256)
        nobody_is_written_over(rows, now, got[0], got[1], got[3], 256)
    # the case of two: 130 rows stay where they are, and the sequence of 100 waits
    got = O.reserve([101, 131], [100, 130], [1, 1], [[0, -1], [0, -1]], [2], 256)
    assert got[3] == [100, 256] and got[4] == [[-1, -1, 0, 0]] * 2


@pytest.mark.gpu
@pytest.mark.parametrize("B,pinned", [(2, 0), (64, 30), (64, 9000), (65, 9000), (900, 200), (900, 60000), (1025, 0), (4096, 0), (4097, 0), (6000, 50000)])
@pytest.mark.parametrize("short", [0, 0.1, 0.6, 2.0])
def test_unequal_rows_in_a_shared_page(B, pinned, short):
    """Every form of the call, with no free page, some, and enough."""
    print(f"shared B={B} pinned={pinned} free={short}", flush=True)
    rows, now, held, table, refs = state(B, int(short * B), 256, B + pinned, pinned)
    books = Books(B, 256, 4, len(refs), held, table, refs)
    books.reserve(rows, now)
    room = books.room.tolist()
    nobody_is_written_over(rows, now, books.held.tolist(), books.table.tolist(), room, 256)
    books.reserve(rows, [min(r, n + 64) if r > n else n for n, r in zip(now, room)])      # a step on, those that could have grown


def test_more_sequences_than_there_are_marks_are_refused():
    address, status = 4096, []
    pages = thk.make_pages(0, 64, 1, 4)
    for B in ((1 << 30) + 1, 2 ** 31 - 1):
        shape = thk.make_shape(1, B, 1, 1, 128, 64, 1, 1)
        assert thk.thk_workspace_bytes(shape, thk.THK_OP_PAGED_RESERVE) == 0
        with pytest.raises(thk.ThkError) as e:
            thk.thk_paged_reserve(shape, pages, *[address] * 7, (address, 1 << 60), stream=0)
        status.append(e.value.status)
    assert status == [2, 2]      # THK_ERR_SHAPE
    assert thk.thk_workspace_bytes(thk.make_shape(1, 1 << 30, 1, 1, 128, 64, 1, 1), thk.THK_OP_PAGED_RESERVE) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("B,n_pages", [(1, 3), (60, 500), (60, 9000), (900, 3000), (900, 60000), (2000, 9000), (4100, 9000)])
def test_free_pages_with_negative_counts(B, n_pages):
    """They are free as those with none are, and the count of one that nobody gets stays what it was."""
    print(f"negative counts B={B} n_pages={n_pages}", flush=True)
    rng = np.random.default_rng(n_pages)
    refs = rng.choice([0, -1, -2, -1000, 1, 3], n_pages)
    books = Books(B, 128, 3, n_pages, refs=refs)
    rows = rng.integers(0, 200, B)
    books.reserve(rows)
    books.reserve(rows + rng.integers(0, 100, B), rows)
    books.reserve([0] * B)
    after = books.refs.cpu().numpy()
    assert (after[refs > 0] == refs[refs > 0]).all() and ((after == refs) | (after == 0)).all()
