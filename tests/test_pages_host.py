"""Page pool against a model of it, and what the page mover refuses (no GPU)."""
import numpy as np
import pytest

from paper_2605_06914_amd import (TAPER_EBLOCK, TAPER_EHIP, TAPER_EINVAL, TAPER_ELEN, TAPER_ENOMEM, PageMover, PagePool, TaperError, remap_pages)
from tests.latent_ref import Batch


def refused(status, f, *a, **kw):
    with pytest.raises(TaperError) as e:
        f(*a, **kw)
    assert e.value.status == status, e.value


def test_pool_gives_the_lowest_free_pages_and_counts_their_users():
    p = PagePool(10)
    a = p.alloc(4)
    assert list(a) == [0, 1, 2, 3] and p.free_pages == 6
    p.share([1, 1, 2])
    assert [p.users(i) for i in range(5)] == [1, 3, 2, 1, 0] and p.users(10) == -1 and p.users(-1) == -1
    assert p.release([1, 0, 3]) == 2 and p.free_pages == 8
    assert list(p.alloc(3)) == [0, 3, 4]
    assert p.release([1, 1]) == 1 and p.users(1) == 0
    refused(TAPER_ENOMEM, p.alloc, 7)
    assert p.free_pages == 6 and len(p.alloc(6)) == 6 and p.free_pages == 0 and len(p.alloc(0)) == 0


def test_pool_refusals_change_nothing():
    p = PagePool(8)
    p.alloc(3)
    before = [p.users(i) for i in range(8)]
    refused(TAPER_EBLOCK, p.share, [0, 5])
    refused(TAPER_EBLOCK, p.share, [0, 8])
    refused(TAPER_EBLOCK, p.share, [0, -1])
    refused(TAPER_EBLOCK, p.release, [0, 1, 0])
    refused(TAPER_EINVAL, p.alloc, -1)
    refused(TAPER_EBLOCK, p.fork, [0, 7], 20)
    refused(TAPER_EBLOCK, p.fork, [7, 0], 20)
    refused(TAPER_EINVAL, p.fork, [0], 20)
    assert [p.users(i) for i in range(8)] == before and p.free_pages == 5
    p.alloc(5)
    refused(TAPER_ENOMEM, p.fork, [0, 1], 20)
    assert p.users(0) == 1 and p.users(1) == 1
    refused(TAPER_EINVAL, PagePool, 0)


def test_fork_shares_full_pages_and_copies_the_last():
    p = PagePool(10)
    row = p.alloc(3)
    child, copy = p.fork(row, 40)
    assert list(child) == [0, 1, 3] and copy == (2, 3) and [p.users(i) for i in range(4)] == [2, 2, 1, 1]
    child, copy = p.fork(row, 48)
    assert list(child) == [0, 1, 2] and copy is None and p.users(2) == 2
    child, copy = p.fork(row, 0)
    assert len(child) == 0 and copy is None
    child, copy = p.fork(row, 1)
    assert list(child) == [4] and copy == (0, 4)


@pytest.mark.parametrize("seed", range(6))
def test_pool_and_compaction_against_a_model(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 200))
    pool, users, rows = PagePool(n), np.zeros(n, int), []
    for _ in range(300):
        what = rng.integers(0, 5)
        if what == 0 and pool.free_pages:
            k = int(rng.integers(1, pool.free_pages + 1))
            got = pool.alloc(k)
            assert list(got) == list(np.nonzero(users == 0)[0][:k])
            users[got] += 1
            rows.append(got)
        elif what == 1 and rows:
            r = rows[rng.integers(len(rows))]
            pool.share(r)
            users[r] += 1
            rows.append(r.copy())
        elif what == 2 and rows:
            r = rows.pop(rng.integers(len(rows)))
            users[r] -= 1
            assert pool.release(r) == int((users[r] == 0).sum())
        elif what == 3 and rows:
            most = int(rng.integers(0, 8)) if rng.random() < 0.5 else -1
            src, dst = pool.compact(most)
            assert most < 0 or len(src) <= most
            assert not set(src) & set(dst) and (users[src] > 0).all() and (users[dst] == 0).all() and (src > dst).all()
            users[dst], users[src] = users[src], 0
            rows = [remap_pages(r, src, dst) for r in rows]
            if most < 0:
                assert (users[:int((users > 0).sum())] > 0).all()
        assert [pool.users(i) for i in range(n)] == list(users) and pool.free_pages == int((users == 0).sum())


def test_remap_leaves_other_entries():
    t = np.array([[3, -1], [5, 7]], np.int32)
    assert remap_pages(t, [7, 3], [0, 1]).tolist() == [[1, -1], [5, 0]]
    refused(TAPER_EINVAL, remap_pages, t, [7, 7], [0, 1])
    refused(TAPER_EINVAL, remap_pages, t, [7], [0, 1])


@pytest.mark.parametrize("bad", [("kv", 8, 96), ("kv", 0, 64), ("latent", 2, 576), ("latent", 1, 512), (7, 1, 64)])
def test_mover_formats(bad):
    refused(TAPER_EINVAL, PageMover, *bad, device=-1)
    refused(TAPER_EINVAL, PageMover, "kv", 8, 128, page_size=32, device=-1)


def test_copies_that_are_refused():
    m = PageMover.kv(8, 128, device=-1)
    ok = [4096, 8192]
    refused(TAPER_EHIP, m.copy, ok, [0, 0], [1, 2], 4)  # (fine but for the device)
    refused(TAPER_EBLOCK, m.copy, ok, [0, 4], [1, 2], 4)
    refused(TAPER_EBLOCK, m.copy, ok, [0, 1], [2, -1], 4)
    refused(TAPER_EINVAL, m.copy, ok, [0, 1], [2, 2], 4)
    refused(TAPER_EINVAL, m.copy, ok, [0, 1], [1, 2], 4)
    refused(TAPER_EINVAL, m.copy, ok, [0], [0], 4)
    refused(TAPER_EINVAL, m.copy, [], [0], [1], 4)
    refused(TAPER_EINVAL, m.copy, [4096, 0], [0], [1], 4)
    refused(TAPER_EINVAL, m.copy, [4104], [0], [1], 4)
    refused(TAPER_EINVAL, m.copy, ok, [0], [1, 2], 4)
    refused(TAPER_EINVAL, m.copy, ok, [0], [1], 0)
    for _ in range(3):  # what one call named does not count for the next
        refused(TAPER_EHIP, m.copy, ok, [1], [2], 4)
        refused(TAPER_EHIP, m.copy, ok, [2], [1], 4)


def test_joins_that_are_refused():
    b = Batch([(20, [[3, 17]]), (32, [[5]])], 1, spare=6)
    m = PageMover.latent(512, device=-1)
    free = b.unreferenced

    def pack(dst, first=(0, 0), table=b.table, seg_len=b.seg_len):
        d = np.full((2, 4), -1, np.int32)
        for s, row in enumerate(dst):
            d[s, :len(row)] = row
        m.pack([4096], table, b.prefix, b.seg_start, seg_len, d, b.n_pages, first_token=list(first))

    refused(TAPER_EHIP, pack, [free[:3], free[3:6]])                       # fine but for the device
    refused(TAPER_EHIP, pack, [free[:2], free[3:4]], first=(16, 32))
    refused(TAPER_EHIP, pack, [free[:3], []], first=(0, 32), seg_len=[3, 17, 0])
    refused(TAPER_EHIP, pack, [[b.table[0, 0], *free[:1]], free[3:4]], first=(16, 32))  # a page before first_token is not read
    refused(TAPER_ELEN, pack, [free[:3], free[3:6]], first=(8, 0))
    refused(TAPER_ELEN, pack, [free[:3], free[3:6]], first=(0, 48))
    refused(TAPER_ELEN, pack, [free[:3], free[3:6]], first=(-16, 0))
    refused(TAPER_EBLOCK, pack, [free[:2], free[3:6]])
    refused(TAPER_EINVAL, pack, [free[:3], free[2:5]])
    refused(TAPER_EINVAL, pack, [free[:3], [free[3], free[4], b.table[1, 2]]])
    refused(TAPER_EINVAL, pack, [[b.table[0, 1], *free[:1]], free[3:4]], first=(16, 32))
    bad = b.table.copy()
    bad[0, 1] = b.n_pages
    refused(TAPER_EBLOCK, pack, [free[:3], free[3:6]], table=bad)
    with pytest.raises(TaperError):
        m.pack([4096], b.table, b.prefix, b.seg_start, b.seg_len, np.full((2, 2), 0, np.int32), b.n_pages)
