"""Page copies and joins on the GPU against indexing on the CPU, bit for bit."""
import gc

import numpy as np
import pytest

from tests.latent_ref import Batch, pages_of, pool_of, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_left_to_collect():
    """Objects of the test before that only the collector frees: their end waits for the device, which no stream that is being
    recorded survives."""
    gc.collect()
FORMATS = [("kv", 8, 128), ("kv", 1, 64), ("kv", 3, 128), ("latent", 1, 576), ("latent", 1, 320)]


def mover_of(fmt):
    from paper_2605_06914_amd import PageMover
    return PageMover(*fmt, device=0)


def kv_rows(pool, heads, d):
    """[pages][2][heads][16 d] as a row a slot: K [d/8][16][8], V [4][d][4]."""
    n = pool.shape[0]
    k = pool[:, 0].reshape(n, heads, d // 8, 16, 8).transpose(0, 3, 1, 2, 4).reshape(n * 16, -1)
    v = pool[:, 1].reshape(n, heads, 4, d, 4).transpose(0, 2, 4, 1, 3).reshape(n * 16, -1)
    return np.concatenate([k, v], 1)


def kv_pool(rows, heads, d):
    n = rows.shape[0] // 16
    k = rows[:, :heads * d].reshape(n, 16, heads, d // 8, 8).transpose(0, 2, 3, 1, 4).reshape(n, heads, -1)
    v = rows[:, heads * d:].reshape(n, 4, 4, heads, d).transpose(0, 3, 1, 4, 2).reshape(n, heads, -1)
    return np.ascontiguousarray(np.stack([k, v], 1))


def make_pools(fmt, n_pages, layers, seed):
    """Any bit patterns, NaN among them, as int16."""
    kind, heads, dim = fmt
    rng = np.random.default_rng(seed)
    width = 2 * heads * dim if kind == "kv" else dim
    rows = [rng.integers(-2 ** 15, 2 ** 15, (n_pages * 16, width)).astype(np.int16) for _ in range(layers)]
    return rows, [kv_pool(r, heads, dim) if kind == "kv" else pool_of(r) for r in rows]


def on_device(pools):
    import torch
    return [torch.from_numpy(p).to("cuda:0").view(torch.bfloat16) for p in pools]


def back(t):
    import torch
    return t.view(torch.int16).cpu().numpy()


SIZES = [(1, 1), (7, 3), (256, 2), (257, 2)]


@pytest.mark.parametrize("fmt,n,layers", [(f, *s) for f in FORMATS for s in SIZES] + [(("kv", 1, 64), 300, 70), (("latent", 1, 320), 3, 129)], ids=str)
def test_copy(fmt, n, layers):
    import torch
    rng = np.random.default_rng(n)
    n_pages = 2 * n + 3
    _, pools = make_pools(fmt, n_pages, layers, n)
    ids = rng.permutation(n_pages).astype(np.int32)
    src, dst = ids[:n].copy(), ids[n:2 * n]
    src[n // 2:] = src[0]  # one page many times
    dev = on_device(pools)
    mover_of(fmt).copy(dev, src, dst, n_pages)
    torch.cuda.synchronize()
    for p, t in zip(pools, dev):
        p[dst] = p[src]
        assert np.array_equal(back(t), p)


REQUESTS = [(5, [[3, 0, 20, 1]]), (0, [[16]]), (64, [[1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1]]), (33, [[]]),
            (0, [[2, 700, 13]]), (16, [[16, 16]]), (130, [[31, 7, 64, 2]])]


@pytest.mark.parametrize("fmt", FORMATS, ids=str)
@pytest.mark.parametrize("whole", [True, False])
def test_pack(fmt, whole):
    import torch
    b = Batch(REQUESTS, 1, spare=400)
    first = np.array([0 if whole else p // 16 * 16 for p, _ in REQUESTS], np.int32)
    first[3] = 32
    total = [len(b.slots(s)) for s in range(b.S)]
    n_dst = [pages_of(t - f) for t, f in zip(total, first)]
    dst = np.full((b.S, max(n_dst) + 1), -1, np.int32)
    cut = np.cumsum([0] + n_dst)
    for s in range(b.S):
        dst[s, :n_dst[s]] = b.unreferenced[cut[s]:cut[s + 1]]
    rows, pools = make_pools(fmt, b.n_pages, 2, 3)
    dev = on_device(pools)
    mover_of(fmt).pack(dev, b.table, b.prefix, b.seg_start, b.seg_len, dst, b.n_pages, first_token=first)
    torch.cuda.synchronize()
    for r, t in zip(rows, dev):
        for s in range(b.S):
            slots = b.slots(s)[first[s]:]
            i = np.arange(len(slots))
            r[dst[s, i // 16].astype(np.int64) * 16 + i % 16] = r[slots]
        got = back(t)
        assert np.array_equal(kv_rows(got, fmt[1], fmt[2]) if fmt[0] == "kv" else rows_of(got), r)


def test_recorded_copies_replay_and_joins_are_not_recorded():
    import torch
    from paper_2605_06914_amd import TAPER_EINVAL, TaperError
    fmt, n = ("kv", 1, 64), 600
    rng = np.random.default_rng(5)
    mover = mover_of(fmt)
    ids = rng.permutation(2 * n + 2).astype(np.int32)
    _, pools = make_pools(fmt, 2 * n + 2, 2, 6)
    dev = on_device(pools)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        mover.copy(dev, ids[:n], ids[n:2 * n], 2 * n + 2)
        with pytest.raises(TaperError) as e:
            mover.pack(dev, ids[None, :1], [5], [0, 0], [], ids[None, 1:2], 2 * n + 2)
        assert e.value.status == TAPER_EINVAL
    for r in range(3):
        _, pools = make_pools(fmt, 2 * n + 2, 2, 10 + r)
        for t, p in zip(dev, pools):
            t.copy_(on_device([p])[0])
        g.replay()
        torch.cuda.synchronize()
        for t, p in zip(dev, pools):
            p[ids[n:2 * n]] = p[ids[:n]]
            assert np.array_equal(back(t), p)
        mover.copy(dev, ids[n:2 * n], ids[:n], 2 * n + 2)  # (eager, through the mover's own lists)
        torch.cuda.synchronize()


def test_many_calls_in_flight_on_two_streams():
    """More calls than the mover has lists: each waits for the one whose list it takes."""
    import torch
    fmt, n = ("latent", 1, 320), 300
    mover = mover_of(fmt)
    _, a = make_pools(fmt, 2 * n, 1, 1)
    _, c = make_pools(fmt, 2 * n, 1, 2)
    dev = [on_device(a), on_device(c)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    rng = np.random.default_rng(3)
    for i in range(24):
        ids = rng.permutation(2 * n).astype(np.int32)
        mover.copy(dev[i % 2], ids[:n], ids[n:], 2 * n, stream=streams[i % 2])
        (a, c)[i % 2][0][ids[n:]] = (a, c)[i % 2][0][ids[:n]]
    torch.cuda.synchronize()
    assert np.array_equal(back(dev[0][0]), a[0]) and np.array_equal(back(dev[1][0]), c[0])
