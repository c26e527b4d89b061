"""Latent-cache attention (decode step and prompts) and append on the GPU against the definition in 64 bits."""
import gc

import numpy as np
import pytest

from tests.latent_ref import RMS, ROPE, Batch, attention, pool_of, rows_of, to_bf16, values

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_left_to_collect():
    """Objects of the test before that only the collector frees: their end waits for the device, which no stream that is being
    recorded survives."""
    gc.collect()


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).to("cuda:0")
    return t.to(torch.bfloat16) if dtype is None and t.dtype == torch.float32 else t


def context(H, R, hd, **kw):
    from paper_2605_06914_amd import LatentContext
    return LatentContext(H, R, hd, device=0, **kw)


def plan_of(ctx, b, prompt=False, **kw):
    if prompt:
        return ctx.prompt_plan_build(b.table, b.group, b.prefix, b.seg_len, b.new, b.n_pages)
    return ctx.plan_build(b.table, b.group, b.prefix, b.seg_len, b.n_pages, seg_start=b.seg_start, **kw)


def run(ctx, b, q, w, tok, prompt=False, plan=None, stream=None, **kw):
    import torch
    q_d, w_d, pages = dev(q), dev(w), dev(pool_of(tok))
    H, hd = w.shape[0], w.shape[1] // 2
    out = torch.full((q.shape[0], H, hd), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.full((q.shape[0], H), float("nan"), device="cuda:0")
    plan = plan or plan_of(ctx, b, prompt, **kw)
    (ctx.prompt_attention if prompt else ctx.decode_step_attention)(plan, q_d, w_d, pages, out, lse)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def check(got, want, what):
    (out, lse), (ref, ref_lse, tol, tol_lse) = got, want
    assert np.isfinite(out).all() and np.isfinite(lse).all(), what
    err, rms = np.abs(out - ref), float(np.sqrt(np.mean(ref ** 2)))
    print(f"[latent] {what}: max {err.max():.2e} (bound there {tol.flat[err.argmax()]:.2e}), rms {np.sqrt(np.mean(err ** 2)) / rms:.2e} of the result's", flush=True)
    assert (err <= tol).all(), f"{what}: {np.argwhere(err > tol)[:5]}"
    assert np.sqrt(np.mean(err ** 2)) <= RMS * rms, what
    assert (np.abs(lse - ref_lse) <= tol_lse).all(), what


SHAPES = [(16, 512, 128), (128, 512, 128), (20, 512, 64), (5, 256, 64), (1, 256, 128), (64, 256, 128)]
SERIAL = [(0, [[n]]) for n in (1, 15, 16, 17, 63, 64, 65, 130, 300)] + [(n, [[0]]) for n in (1, 33, 64, 129)]
BRANCHES = [(37, [[0], [1], [16], [70]]), (64, [[5]] * 3), (0, [[9]]), (200, [[3], [0]]), (1, [[1]] * 5)]


@pytest.mark.parametrize("H,R,hd", SHAPES)
@pytest.mark.parametrize("requests", [SERIAL, BRANCHES], ids=["serial", "branches"])
def test_decode_step(H, R, hd, requests):
    b = Batch(requests, 1)
    q, w, tok = values(b, H, R, hd, 2)
    ctx = context(H, R, hd)
    check(run(ctx, b, q, w, tok), attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, True), f"decode H {H} R {R} hd {hd}")


@pytest.mark.parametrize("workgroups", [1, 7, 64, 4096])
def test_decode_step_cut_in_other_ways(workgroups):
    """One long context and a wide request, cut for few and for many workgroups."""
    H, R, hd = 24, 512, 128
    b = Batch([(0, [[2500]]), (700, [[n] for n in range(0, 36, 3)]), (40, [[100, 0, 31], [2, 2]])], 3)
    q, w, tok = values(b, H, R, hd, 4)
    ctx = context(H, R, hd, scale=0.11)
    check(run(ctx, b, q, w, tok, target_workgroups=workgroups), attention(b, q, w, tok, H, R, hd, 0.11, True), f"{workgroups} workgroups")


def test_decode_step_is_the_same_every_time_and_branches_do_not_see_each_other():
    H, R, hd = 32, 512, 128
    b = Batch([(900, [[10], [200], [40]]), (0, [[333]])], 5)
    q, w, tok = values(b, H, R, hd, 6)
    ctx = context(H, R, hd)
    first = run(ctx, b, q, w, tok)
    for _ in range(5):
        again = run(ctx, b, q, w, tok)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])
    other = tok.copy()
    other[b.slots(1)[900:]] = 3.0  # a sibling's own tokens
    changed = run(ctx, b, q, w, other)
    assert np.array_equal(first[0][[0, 2, 3]], changed[0][[0, 2, 3]]) and not np.array_equal(first[0][1], changed[0][1])


def test_scores_far_apart_and_equal_ones():
    """Scores of some hundreds (one token has all the weight), and all equal."""
    H, R, hd = 16, 256, 64
    b = Batch([(70, [[40], [0]])], 7)
    q, w, tok = values(b, H, R, hd, 8)
    live = b.slots(0)
    q[0] *= 64
    q[1] = 0
    want = attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, True)
    out, lse = run(context(H, R, hd), b, q, w, tok)
    assert np.isfinite(out).all()
    mean = tok[live[:70], :R].astype(np.float64).mean(0)
    ref = np.einsum("hvr,r->hv", w[:, hd:].astype(np.float64), mean)
    assert (np.abs(out[1] - ref) <= want[2][1]).all()
    assert (np.abs(out - want[0]) <= want[2]).all()


@pytest.mark.parametrize("H,R,hd", SHAPES)
def test_prompts_of_ragged_lengths(H, R, hd):
    requests = [(0, [[n]]) for n in (1, 2, 15, 16, 17, 64, 127, 128, 129, 200)] + [(0, [[90]]), (0, [[300]])]
    b = Batch(requests, 9, new=[1, 2, 15, 16, 17, 64, 127, 128, 129, 200, 0, 7])
    q, w, tok = values(b, H, R, hd, 10)
    check(run(context(H, R, hd), b, q, w, tok, True), attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, False), f"prompts H {H} R {R} hd {hd}")


@pytest.mark.parametrize("H,R,hd", [(16, 512, 128), (5, 256, 64)])
def test_prompts_behind_cached_tokens_and_shared_prefixes(H, R, hd):
    requests = [(100, [[20], [1], [150], [0]]), (16, [[16], [5]]), (1, [[1]]), (0, [[700]]), (63, [[65]])]
    b = Batch(requests, 11, new=[20, 1, 130, 0, 3, 5, 1, 33, 64])
    q, w, tok = values(b, H, R, hd, 12)
    check(run(context(H, R, hd), b, q, w, tok, True), attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, False), f"prefixes H {H} R {R} hd {hd}")


@pytest.mark.parametrize("n,R,wide", [(1, 512, False), (37, 256, True), (5000, 512, True), (0, 512, False)])
def test_append_writes_its_slots_and_nothing_else(n, R, wide):
    import torch
    rng = np.random.default_rng(n)
    n_pages = n // 16 + 4
    before = to_bf16(rng.standard_normal((n_pages * 16, R + ROPE)))
    rows = to_bf16(rng.standard_normal((n, R + ROPE + (64 if wide else 0))))
    slots = rng.permutation(n_pages * 16)[:n].astype(np.int64)
    if n > 4:
        slots[1::4] = -1
        slots[2] = n_pages * 16  # behind the pool
    pages, rows_d = dev(pool_of(before)), dev(rows)
    ctx = context(16, R, 128)
    if wide:
        latent, rope = rows_d[:, 64:64 + R], rows_d[:, 64 + R:]
    else:
        latent, rope = rows_d[:, :R].contiguous(), rows_d[:, R:].contiguous()
    ctx.append(latent, rope, dev(slots), pages, n_pages)
    torch.cuda.synchronize()
    keep = (slots >= 0) & (slots < n_pages * 16)
    before[slots[keep]] = rows[keep][:, -(R + ROPE):]
    assert np.array_equal(rows_of(pages.float().cpu().numpy()), before)


@pytest.mark.parametrize("H,R,hd", [(16, 512, 128), (5, 256, 64)])
def test_the_normaliser_of_short_contexts_is_as_exact_as_its_type(H, R, hd):
    """lse is fp32, whatever the operands are: rounded queries (decode) and keys (prompts) must not be seen in it.  2-norm over all rows:
    first-order effects are taken out, so that what is left is U^2 of a score (1.5e-5 of 1, averaged over the row's tokens) in a decode
    step, and for prompts 2^-11 of a key (3e-4 of a score of 1, over the square root of 128 tokens and more) for rows that see many,
    against values of 1 to 6."""
    requests = [(0, [[n]]) for n in (1, 2, 3, 5, 9, 17, 33, 40)] + [(19, [[3], [30]]), (5, [[1], [180]])]
    b = Batch(requests, 21, new=[1, 2, 3, 5, 9, 17, 33, 2, 3, 30, 1, 100])
    q, w, tok = values(b, H, R, hd, 22)
    want = attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, False)
    got = run(context(H, R, hd), b, q, w, tok, True)
    check(got, want, "short prompts")
    assert np.linalg.norm(got[1] - want[1]) <= 1e-5 * np.linalg.norm(want[1])
    b.new[:] = 1
    q = q[:b.S]
    want = attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, True)
    got = run(context(H, R, hd), b, q, w, tok)
    check(got, want, "short decode")
    assert np.linalg.norm(got[1] - want[1]) <= 1e-5 * np.linalg.norm(want[1])


@pytest.mark.parametrize("factor", [2.0 ** 18, 2.0 ** -16])
def test_prompts_whose_keys_and_values_half_precision_does_not_hold(factor):
    """Some tokens' latents far larger or smaller than half precision (the queries see to it that the scores stay of order one)."""
    H, R, hd = 8, 512, 128
    b = Batch([(70, [[90], [20]]), (0, [[150]])], 31, new=[40, 20, 150])
    q, w, tok = values(b, H, R, hd, 32)
    q[..., :hd] /= np.float32(factor)
    some = np.concatenate([b.slots(0)[:40], b.slots(2)])
    tok[some, :R] *= np.float32(factor)
    want = attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, False)
    out, lse = run(context(H, R, hd), b, q, w, tok, True)
    err = np.abs(out - want[0])
    assert (err <= want[2]).all() and (np.abs(lse - want[1]) <= want[3]).all()
    for rows in (slice(0, 60), slice(60, 210)):  # (their sizes differ by the factor)
        assert np.sqrt(np.mean(err[rows] ** 2)) <= RMS * np.sqrt(np.mean(want[0][rows] ** 2))


def test_few_new_tokens_behind_a_long_context_are_cut_into_pieces():
    H, R, hd = 4, 512, 128
    b = Batch([(0, [[3000]]), (1100, [[500], [3]])], 41, new=[20, 300, 3])
    q, w, tok = values(b, H, R, hd, 42)
    check(run(context(H, R, hd), b, q, w, tok, True), attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, False), "pieces")


def setup(seed, H=16, R=512, hd=128, requests=None, new=None):
    import torch
    b = Batch(requests or [(150, [[10], [70]]), (0, [[333]])], seed, new=new)
    q, w, tok = values(b, H, R, hd, seed + 1)
    d = dict(b=b, host=(q, w, tok), q=dev(q), w=dev(w), pages=dev(pool_of(tok)),
             out=torch.zeros(q.shape[0], H, hd, dtype=torch.bfloat16, device="cuda:0"), lse=torch.zeros(q.shape[0], H, device="cuda:0"))
    return d


@pytest.mark.parametrize("prompt", [False, True])
def test_recorded_calls_replay_beside_eager_ones(prompt):
    """Two plans of one context in two graphs, replayed with new inputs, other plans and eager calls in between."""
    import torch
    ctx = context(16, 512, 128)
    new = [10, 33, 200] if prompt else None
    one, two = setup(1, new=new), setup(5, new=new)
    call = ctx.prompt_attention if prompt else ctx.decode_step_attention
    graphs = []
    side = torch.cuda.Stream()
    for d in (one, two):
        d["plan"] = plan_of(ctx, d["b"], prompt)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(d["plan"], d["q"], d["w"], d["pages"], d["out"], d["lse"])
        graphs.append(g)
    for round_ in range(4):
        for d, g in zip((one, two), graphs):
            d["q"].copy_(dev(to_bf16(np.random.default_rng(round_).standard_normal(tuple(d["q"].shape)))))
            d["out"].zero_()
            g.replay()
            torch.cuda.synchronize()
            got = d["out"].clone(), d["lse"].clone()
            extra = plan_of(ctx, d["b"], prompt)  # (a plan of its own for the eager call)
            d["out"].zero_()
            call(extra, d["q"], d["w"], d["pages"], d["out"], d["lse"])
            torch.cuda.synchronize()
            assert torch.equal(got[0], d["out"]) and torch.equal(got[1], d["lse"]) and d["out"].float().abs().sum() > 0
            extra.free()


def test_calls_on_another_stream_and_without_lse():
    import torch
    ctx, s = context(16, 512, 128), torch.cuda.Stream()
    d = setup(9)
    plan = plan_of(ctx, d["b"])
    ctx.decode_step_attention(plan, d["q"], d["w"], d["pages"], d["out"], d["lse"])
    torch.cuda.synchronize()
    first = d["out"].clone()
    with torch.cuda.stream(s):
        d["out"].zero_()
        ctx.decode_step_attention(plan, d["q"], d["w"], d["pages"], d["out"])
    s.synchronize()
    assert torch.equal(first, d["out"])
    s.wait_stream(torch.cuda.current_stream())
    ctx.decode_step_attention(plan, d["q"], d["w"], d["pages"], d["out"], stream=s)
    s.synchronize()
    assert torch.equal(first, d["out"])


def test_freed_plans_hand_their_memory_on():
    import torch
    ctx = context(16, 512, 128)
    for n in range(6):
        d = setup(30 + n, requests=[(0, [[100 + 300 * (n % 3)]]), (20 * n, [[1], [2]])])
        plan = plan_of(ctx, d["b"])
        ctx.decode_step_attention(plan, d["q"], d["w"], d["pages"], d["out"], d["lse"])
        plan.free()
        torch.cuda.synchronize()
        want = attention(d["b"], *d["host"], 16, 512, 128, 192 ** -0.5, True)
        assert (np.abs(d["out"].double().cpu().numpy() - want[0]) <= want[2]).all()


def test_tensors_that_do_not_fit_are_refused():
    import torch
    from paper_2605_06914_amd import TAPER_EINVAL, TaperError
    ctx, d = context(16, 512, 128), setup(9)
    plan = plan_of(ctx, d["b"])
    good = dict(q=d["q"], w_up=d["w"], pages=d["pages"], out=d["out"], lse=d["lse"])
    for name, bad in [("q", d["q"][:-1]), ("q", d["q"].float()), ("q", d["q"].cpu()), ("q", d["q"].transpose(0, 1)), ("w_up", d["w"][:, 1:].contiguous()),
                      ("pages", d["pages"][1:]), ("out", d["out"][:, :15].contiguous()), ("lse", d["lse"].double()), ("lse", d["lse"][:2]),
                      ("q", torch.empty(d["q"].numel() + 1, dtype=torch.bfloat16, device="cuda:0")[1:])]:
        with pytest.raises(TaperError) as e:
            ctx.decode_step_attention(plan, **dict(good, **{name: bad}))
        assert e.value.status == TAPER_EINVAL, name
    n = 8
    rows = torch.zeros(n, 576, dtype=torch.bfloat16, device="cuda:0")
    slots = torch.zeros(n, dtype=torch.int64, device="cuda:0")
    pages = d["pages"]
    for latent, rope, s in [(rows[:, :511], rows[:, 512:], slots), (rows[:7, :512], rows[:, 512:], slots), (rows[:, :512].float(), rows[:, 512:], slots),
                            (rows[:, :512], rows[:, 511:575], slots), (rows[:, :512], rows[:, 512:], slots.int()),
                            (torch.zeros(512, n, dtype=torch.bfloat16, device="cuda:0").t(), rows[:, 512:], slots)]:
        with pytest.raises(TaperError) as e:
            ctx.append(latent, rope, s, pages, d["b"].n_pages)
        assert e.value.status == TAPER_EINVAL


def test_a_request_from_its_prompt_through_branches_and_their_join():
    """As an engine uses them together: pages from a pool, a prompt in two chunks, a fork in mid-page, branches that decode for some
    steps, their join into one prefix, compaction of the pool, a step of the joined request; each attention against the definition."""
    import torch
    from paper_2605_06914_amd import PageMover, PagePool, append_slots, remap_pages
    H, R, hd, layers = 16, 512, 128, 2
    rng = np.random.default_rng(77)
    n_pages = 64
    pool, ctx, mover = PagePool(n_pages), context(H, R, hd), PageMover.latent(R, device=0)
    pool.alloc(7)
    pools = [torch.full((n_pages, 72, 16, 8), float("nan"), dtype=torch.bfloat16, device="cuda:0") for _ in range(layers)]
    w = to_bf16(rng.standard_normal((H, 2 * hd, R)) * R ** -0.5)
    w_d = dev(w)
    tokens = [dict() for _ in range(layers)]  # what each branch has seen: per layer, branch -> [values of its tokens]

    def fresh(n):
        return to_bf16(rng.standard_normal((layers, n, R + ROPE)))

    def put(rows, slots):
        for l in range(layers):
            x = dev(rows[l])
            ctx.append(x[:, :R], x[:, R:], dev(np.asarray(slots, np.int64)), pools[l], n_pages)

    def compare(q, out, seen):
        """q, out of some rows; seen: per row the tokens it sees."""
        for r in range(len(q)):
            c = seen[r].astype(np.float64)
            for h in range(0, H, 5):
                k, v = c[:, :R] @ w[h, :hd].T.astype(np.float64), c[:, :R] @ w[h, hd:].T.astype(np.float64)
                s = (k @ q[r, h, :hd] + c[:, R:] @ q[r, h, hd:]) * (hd + ROPE) ** -0.5
                p = np.exp(s - s.max())
                ref = p @ v / p.sum()
                # (the same four roundings as elsewhere, bounded by their effect on scores of one: 6 U of the values' mean size)
                assert np.abs(out[r, h] - ref).max() <= 6 * 2.0 ** -8 * np.sqrt((p ** 2 @ v ** 2) / p.sum() ** 2).max() * 4 + 2.0 ** -8 * np.abs(ref).max()

    # the prompt: 90 tokens, in chunks of 50 and 40
    row = np.zeros(0, np.int32)
    prompt = fresh(90)
    have = 0
    for n in (50, 40):
        row = np.concatenate([row, pool.alloc((have + n + 15) // 16 - len(row))])
        t = np.arange(have, have + n)
        put(prompt[:, have:have + n], row[t // 16].astype(np.int64) * 16 + t % 16)
        have += n
        plan = ctx.prompt_plan_build(row[None], [0], [0], [have], [n], n_pages)
        for l in range(layers):
            q = to_bf16(rng.standard_normal((n, H, hd + ROPE)))
            out = torch.empty(n, H, hd, dtype=torch.bfloat16, device="cuda:0")
            ctx.prompt_attention(plan, dev(q), w_d, pools[l], out)
            some = [0, n // 2, n - 1]
            compare(q[some], out.double().cpu().numpy()[some], [prompt[l, :have - n + 1 + i] for i in some])
        plan.free()
    # two children fork after 85 tokens (in the middle of a page), each private from then on; 5 steps
    rows, moves = [], []
    for _ in range(2):
        child, copy = pool.fork(row, 85)
        rows.append(child)
        moves.append(copy)
    mover.copy(pools, [m[0] for m in moves], [m[1] for m in moves], n_pages)
    pool.release(row)
    # as branches of one request: 80 shared tokens on full pages, then 5 of the copied page and what they generate
    own = [list(prompt[:, 80:85].transpose(1, 0, 2)) for _ in range(2)]
    lens = [5, 5]
    for step in range(5):
        for i in range(2):
            if lens[i] % 16 == 0:
                rows[i] = np.concatenate([rows[i], pool.alloc(1)])
        table = np.full((2, max(map(len, rows))), -1, np.int32)
        for i in range(2):
            table[i, :len(rows[i])] = rows[i]
        slots, _ = append_slots(table, [80, 80], [0, 1, 2], lens, 16, n_pages)
        x = fresh(2)
        put(x, slots)
        for i in range(2):
            own[i].append(x[:, i])
            lens[i] += 1
        plan = ctx.plan_build(table, [0, 0], [80, 80], lens, n_pages)
        for l in range(layers):
            q = to_bf16(rng.standard_normal((2, H, hd + ROPE)))
            out = torch.empty(2, H, hd, dtype=torch.bfloat16, device="cuda:0")
            ctx.decode_step_attention(plan, dev(q), w_d, pools[l], out)
            compare(q, out.double().cpu().numpy(), [np.concatenate([prompt[l, :80], np.stack([t[l] for t in own[i]])]) for i in range(2)])
        plan.free()
    # join: prefix, then both branches, one contiguous run; what was theirs is free again; the pool moves to its front
    joined = np.concatenate([rows[0][:5], pool.alloc(2)])
    src = np.concatenate([rows[0], rows[1][5:]])
    mover.pack(pools, src[None], [80], [0, 2], lens, joined[None, 5:], n_pages, first_token=[80])
    pool.share(joined[:5])
    for r in rows:
        pool.release(r)
    pool.release(np.arange(7))
    src, dst = pool.compact()
    mover.copy(pools, src, dst, n_pages)
    joined = remap_pages(joined, src, dst)
    assert sorted(joined) == list(range(7)) and pool.free_pages == n_pages - 7
    plan = ctx.plan_build(joined[None], [0], [100], [0], n_pages)
    for l in range(layers):
        q = to_bf16(rng.standard_normal((1, H, hd + ROPE)))
        out = torch.empty(1, H, hd, dtype=torch.bfloat16, device="cuda:0")
        ctx.decode_step_attention(plan, dev(q), w_d, pools[l], out)
        compare(q, out.double().cpu().numpy(), [np.concatenate([prompt[l, :80], *[np.stack([t[l] for t in own[i]]) for i in range(2)]])])


def test_a_plan_is_not_built_on_a_stream_that_is_being_recorded():
    import torch
    from paper_2605_06914_amd import TAPER_EINVAL, TaperError
    ctx, d = context(16, 512, 128), setup(9)
    plan = plan_of(ctx, d["b"])
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.decode_step_attention(plan, d["q"], d["w"], d["pages"], d["out"])
        for prompt in (False, True):
            with pytest.raises(TaperError) as e:
                plan_of(ctx, d["b"], prompt)
            assert e.value.status == TAPER_EINVAL
    g.replay()
    torch.cuda.synchronize()
    assert d["out"].float().abs().sum() > 0


def test_pages_beyond_four_gigabytes():
    """The far end of a pool of 4.6 GB: append, copy, decode step and prompt there."""
    import torch
    from paper_2605_06914_amd import PageMover
    H, R, hd, n_pages = 8, 512, 128, 250000
    pages = torch.zeros(n_pages, 72, 16, 8, dtype=torch.bfloat16, device="cuda:0")
    rng = np.random.default_rng(3)
    b = Batch([(0, [[100]]), (40, [[9], [33]])], 50, new=[7, 9, 3])
    q, w, tok = values(b, H, R, hd, 51)
    far = n_pages - 1 - rng.permutation(60)[:b.n_pages].astype(np.int64)  # where each page of the batch lies
    live = np.nonzero(np.isfinite(tok[:, 0]))[0]
    ctx, mover = context(H, R, hd), PageMover.latent(R, device=0)
    rows = dev(tok[live])
    ctx.append(rows[:, :R], rows[:, R:], dev((far[live // 16] - 100) * 16 + live % 16), pages, n_pages)
    mover.copy([pages], far - 100, far, n_pages)
    b.table = np.where(b.table >= 0, far[b.table], -1).astype(np.int32)
    b.n_pages = n_pages
    plan = ctx.prompt_plan_build(b.table, b.group, b.prefix, b.seg_len, b.new, n_pages)
    out = torch.empty(19, H, hd, dtype=torch.bfloat16, device="cuda:0")
    ctx.prompt_attention(plan, dev(q), dev(w), pages, out)
    back = np.full_like(tok, np.nan)
    back[live] = tok[live]
    near = Batch([(0, [[100]]), (40, [[9], [33]])], 50, new=[7, 9, 3])
    want = attention(near, q, w, back, H, R, hd, (hd + ROPE) ** -0.5, False)
    assert (np.abs(out.double().cpu().numpy() - want[0]) <= want[2]).all()
    plan = ctx.plan_build(b.table, b.group, b.prefix, b.seg_len, n_pages)
    ctx.decode_step_attention(plan, dev(q[:3]), dev(w), pages, out)
    near.new[:] = 1
    want = attention(near, q[:3], w, back, H, R, hd, (hd + ROPE) ** -0.5, True)
    assert (np.abs(out[:3].double().cpu().numpy() - want[0]) <= want[2]).all()


def test_heads_whose_keys_and_values_are_expanded_in_turns():
    """256 heads of 36000 tokens are 4.7 GB: more than are expanded at a time.  Some heads of both turns."""
    import torch
    H, R, hd, T, n = 256, 512, 128, 36000, 5
    b = Batch([(0, [[T]])], 60, new=[n])
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    make = lambda *shape, std=1.0: torch.empty(shape, dtype=torch.bfloat16, device="cuda:0").normal_(0.0, std, generator=gen)
    q, w, pages = make(n, H, hd + ROPE), make(H, 2 * hd, R, std=R ** -0.5), make(b.n_pages, 72, 16, 8)
    ctx = context(H, R, hd)
    plan = plan_of(ctx, b, True)
    out, lse = torch.empty(n, H, hd, dtype=torch.bfloat16, device="cuda:0"), torch.empty(n, H, device="cuda:0")
    ctx.prompt_attention(plan, q, w, pages, out, lse)
    torch.cuda.synchronize()
    plan.free()
    some = [0, 100, 231, 232, 233, 255]
    tok = rows_of(pages.float().cpu().numpy())
    want = attention(b, q.float().cpu().numpy()[:, some], w.float().cpu().numpy()[some], tok, len(some), R, hd, (hd + ROPE) ** -0.5, False)
    assert (np.abs(out.double().cpu().numpy()[:, some] - want[0]) <= want[2]).all()
    assert (np.abs(lse.double().cpu().numpy()[:, some] - want[1]) <= want[3]).all()


@pytest.mark.parametrize("prompt", [False, True])
def test_many_tokens_of_small_weight(prompt):
    """One token with a score 17 above 40000 equal ones, of which each has the weight 2^-24.5 and all together 0.0017; its own value is 0."""
    H, R, hd, T = 2, 256, 64, 40000
    b = Batch([(0, [[T]])], 61, new=[3 if prompt else 1])
    q, w, tok = values(b, H, R, hd, 62)
    live = b.slots(0)
    q[..., :hd], q[..., hd:] = 0, 1
    tok[live, :R], tok[live, R:] = tok[live[5], :R], 0
    tok[live[0], :R], tok[live[0], R:] = 0, 3
    want = attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, not prompt)
    check(run(context(H, R, hd), b, q, w, tok, prompt), want, "small weights")


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("part,factor", [("plain", 0.0), ("plain", 2.0 ** -24), ("plain", 2.0 ** -100), ("rotated", 0.0), ("rotated", 2.0 ** -100), ("both", 0.0)])
def test_queries_whose_parts_are_far_apart(prompt, part, factor):
    H, R, hd = 16, 512, 128
    b = Batch([(40, [[30], [7]]), (0, [[200]])], 71, new=[30, 5, 120] if prompt else None)
    q, w, tok = values(b, H, R, hd, 72)
    if part != "rotated":
        q[..., :hd] *= np.float32(factor)
    if part != "plain":
        q[..., hd:] *= np.float32(factor)
    check(run(context(H, R, hd), b, q, w, tok, prompt), attention(b, q, w, tok, H, R, hd, (hd + ROPE) ** -0.5, not prompt), f"{part} x {factor}")
