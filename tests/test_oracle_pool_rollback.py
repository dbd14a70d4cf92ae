"""The oracle's page pool when sequences go back without a release: reserved pages belong to one sequence, what others read stays."""
import numpy as np

from oracle import sparse_oracle as S


def test_reserved_pages_are_named_once_and_others_keep_theirs():
    rng, granted = np.random.default_rng(1), 0
    for _ in range(60):
        p, lens = S.Pool(5, 4, 14), [0] * 5
        for _ in range(12):
            slot = int(rng.integers(0, 5))
            if rng.random() < 0.4:
                src = int(rng.integers(0, 5))
                if src != slot and np.all(p.table[src, :-(-lens[src] // 64)] >= 0):
                    p.fork(src, slot, lens[src])
                    lens[slot] = lens[src]
                continue
            lens[slot] = [lens[slot], lens[slot] // 64 * 64, 0][int(rng.integers(0, 3))]
            new = int(rng.integers(1, 256 - lens[slot] + 1)) if lens[slot] < 256 else 0
            before, p.empty = p.table.copy(), False
            copies = p.reserve([(slot, lens[slot], new)])
            others = [s for s in range(5) if s != slot]
            assert np.array_equal(before[others], p.table[others])
            p.check()
            if p.empty or not new:
                continue
            granted += 1
            lens[slot] += new
            pages = p.table[slot, (lens[slot] - new) // 64:(lens[slot] - 1) // 64 + 1]
            assert np.all(pages >= 0) and np.all(p.refs[pages] == 1)
            assert len(copies) <= (1 if (lens[slot] - new) % 64 else 0)
    assert granted > 100


def test_an_empty_pool_locks_every_shared_page_that_would_be_written():
    p = S.Pool(2, 3, 3)
    p.reserve([(0, 0, 190)])
    p.fork(0, 1, 190)
    assert p.reserve([(1, 64, 65)]) == [] and p.empty and p.table[1].tolist() == [0, -3, -4]
    p.release(0)
    p.empty = False
    assert p.reserve([(1, 64, 65)]) == [] and not p.empty and p.table[1].tolist() == [0, 1, 2]
